// Attention of queries to the keys of their scene, forward and backward (entry points: sc_attention.hip).
//
//     S = scale q k^T,   P = softmax of S over the keys that a query sees,   o = P v,   lse = log of the sum of exp(S)
//     backward: dv = P^T do,  dP = do v^T,  delta = sum(do o),  dS = P (dP - delta),  dq = scale dS k,  dk = scale dS^T q
//
// The heads of queries that share a head of keys are columns next to each other: column c of a scene and a head of keys is row c / per, head c % per.
// A wavefront holds NB blocks of 16 columns in registers as the matrix instruction's second operand and walks the other side's rows through LDS,
// two buffers deep, 16 bytes a lane straight from global memory.  S comes out transposed, rows of the walked side down a lane's registers, its column along the lanes:
// the maximum and the sum of a column are then a lane's own (of its quarter of the rows), and four registers are four consecutive rows, which is how the
// transposing LDS read hands out the second product's first operand.  So weights go from one product to the next without leaving their registers.
//
// What bounds it: the matrix cores for long scenes, next to the vector unit (an exponential, two multiplications, an addition and a share of a comparison and of a conversion for every
// score); vector instructions ahead of and behind the products for scenes of tens; memory for single rows over long caches; a few trips to memory, one after the other, for little of everything.
// us of the call, a copy on this card 5.1 TB/s, the library's largest product 1120 TFLOP/s in 16 bits and 152 in 32:
//     one row, 77 keys, 8 heads of 32, bf16                     5.1
//     8 rows, 262144 keys, 16 heads of 128 over 4, f16          111    537 MB, 4.8 TB/s with the parts' join of 8; the walk alone 5.1
//     53373 rows in 1112 scenes, 8 heads of 16, f16              29.6  55 MB; 10 million vector instructions, 16 us of every SIMD's time
//     16384 rows in 3 causal scenes, 16 heads of 128 over 4, bf16  381 to 427 by the card's clock    915 to 1026 TFLOP/s
//     backward 110545 rows in 2303 scenes, 8 heads of 16, f16   163    230 MB; 53 million vector instructions, 86 us
//     backward 16384 rows in 4 causal scenes, 16 heads of 64 over 4, bf16  806 to 817    656 to 665 TFLOP/s of the five products that it cannot do without, 918 to 931 of the seven that it does
#pragma once

#include "sc_product.h"
#include "sc_scenes.h"

namespace sc {

struct HeadRows {                      // rows of one of the operands' heads
    char* data;
    int64_t row, head;                 // bytes
};
struct Attention {
    HeadRows q, k, v, out;             // backward: out is the forward call's
    float* lse;                        // [q_rows][q_heads], may be null forward
    const int32_t *q_starts, *k_starts, *k_lens;
    int scenes;
    int64_t q_rows, k_rows;
    int D, per, k_heads;               // per: heads of queries that share one of keys
    uint32_t per_magic;                // ceil(2^(31 + s) / per), 2^s >= per > 2^(s - 1): c / per is the high word of c per_magic, s - 1 bits down, for c < 2^31
    int per_shift;                     // s - 1
    int causal;
    float scale, scale_log2;           // ... times log2 e
    int64_t units;                     // column tiles there can be at most
    int parts;                         // of the walked rows; above 1 results go to the workspace
    int part_keys;                     // keys that a part has at least
    float2* part_sums;                 // [part][q_rows][q_heads]: exponent that the weights were taken against, sum
    float* part_out;                   // [part][q_rows][q_heads][D]
    // backward
    HeadRows dout, dq, dk, dv;
    int64_t k_units;
    int k_parts, part_rows;            // of the queries that the keys' columns walk
    float *part_dk, *part_dv;          // [part][k_rows][k_heads][D]
    float *against, *delta;            // [q_heads][q_rows]: lse times log2 e, infinite for a row that sees nothing; -sum(do o)
};

__device__ __forceinline__ int row_of_column(const Attention& p, int c) { return p.per == 1 ? c : (int)(__umulhi((uint32_t)c, p.per_magic) >> p.per_shift); }
// log2 of a tile of columns
constexpr int log2_of(int tile) { return tile == 16 ? 4 : tile == 32 ? 5 : tile == 64 ? 6 : tile == 128 ? 7 : 8; }
__device__ inline Scene scene_of_queries(const Attention& p, int log2, int64_t u) {
    int64_t first = 0, first_k = 0;
    int count = 0, count_k = 0, scene;
    Scene s = find_scene(p.q_starts, p.scenes, p.q_rows, p.per, log2, u, p.units, first, count, scene);
    s.tile = __builtin_amdgcn_readfirstlane(s.tile);
    if (s.tile < 0) return s;
    first_k = first;
    count_k = count;
    if (p.k_starts != p.q_starts || p.k_lens != nullptr || p.k_rows != p.q_rows) scene_rows(p.k_starts, p.k_lens, p.k_rows, scene, first_k, count_k);
    s.q0 = uniform64(first);
    s.nq = __builtin_amdgcn_readfirstlane(count);
    s.k0 = uniform64(first_k);
    s.nk = __builtin_amdgcn_readfirstlane(count_k);
    return s;
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------
// A tile is rows of LINE chunks of 16 bytes.  Where a chunk lies in its line is turned by the line's number so that both reads meet every bank once: 16-byte reads along
// the lines go 16 lanes a cycle, a chunk of lines 0-3 and 12-15 and its neighbour of lines 4-11; transposing reads 32 lanes, two chunks of eight consecutive lines;
// 32-bit reads across 64 bytes of lines 0, 4, 8 and 12.  Not so in lines of 128 bytes of f32: those four all begin in the same half of the banks, so that 32-bit reads across them meet every bank of it
// twice (the counters have a cycle for each matrix instruction of the keys' gradients).
template <int DT, int LINE>
__device__ constexpr int tile_turn(int line) {
    constexpr int WIDE = LINE < 16 ? LINE : 16;
    const int m = (line / (16 / WIDE)) & (WIDE - 1);
    if (DT == SC_F32) return m;
    const int half = WIDE / 2;
    return (((m & (half - 1)) ^ (m >= half ? half / 2 : 0)) << 1) | (m >= half ? 1 : 0);
}

template <int DT, int DPAD>
struct HeadShape {
    static constexpr int PER = 16 / ELEM<DT>, LINE = DPAD / PER, BYTES = DPAD * ELEM<DT>;
    static constexpr int KS = LINE / 4;            // steps of 64 bytes along a row
    static constexpr int CB = DPAD / 16;           // blocks of 16 channels
    static constexpr int STEP = DT == SC_F32 ? 16 : 32;   // rows that a step of the second product takes
};

// 16 bytes a lane straight into LDS as load_to_lds, from an address that the wavefront shares and an offset of the lane's.  A vector instruction (v_readfirstlane)
// may have written that address just before, and a load that takes it from scalar registers needs five wait states behind such a write, which the compiler does not
// see to inside assembly.
__device__ inline void load_to_lds_at(const void* base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base), "s"(lds) : "m0", "memory");
}
// The chunk that a row of D channels ends inside of: the row's last 16 bytes, or what there is if it has fewer; shifted() puts them in their place, with zeros behind them.
template <int DT>
__device__ __forceinline__ uint4 end_of_row(const char* row, int D) {
    constexpr int PER = 16 / ELEM<DT>;
    if (D >= PER) return load_chunk(row != nullptr ? row + (D - PER) * ELEM<DT> : (const char*)&g_no_chunk);
    uint32_t w[4] = {0, 0, 0, 0};
    if (row != nullptr) {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (j < D) {
                if constexpr (DT == SC_F32) w[j] = reinterpret_cast<const uint32_t*>(row)[j];
                else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[j] << (16 * (j & 1));
            }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT>
__device__ __forceinline__ u32x4 shifted(uint4 v, int D) {
    constexpr int PER = 16 / ELEM<DT>;
    const int by = D >= PER ? 8 * ELEM<DT> * (PER - D % PER) : 0;       // bits: channels of the chunk before
    unsigned __int128 bits = (unsigned __int128)(((uint64_t)v.w << 32) | v.z) << 64 | (((uint64_t)v.y << 32) | v.x);
    bits >>= by & 127;
    return u32x4{(uint32_t)bits, (uint32_t)(bits >> 32), (uint32_t)(bits >> 64), (uint32_t)(bits >> 96)};
}
// The loads of one operand's tiles by NTH threads: rows first .. of a scene's head.  Zeros stand for rows that are not there and for channels beyond D: whole chunks of those
// are cleared once, by clear(), and never written again.  WHOLE: D is a multiple of a chunk's channels.
template <int DT, int DPAD, int ROWS, int NTH, bool WHOLE>
struct TileLoader {
    using H = HeadShape<DT, DPAD>;
    static constexpr int PASSES = ROWS * H::LINE / NTH, LINES = NTH / H::LINE;       // lines of a pass
    static_assert(ROWS * H::LINE % NTH == 0 && NTH % H::LINE == 0 && PASSES > 0, "whole passes of whole lines");
    const char* base;                  // of the scene's first row
    int64_t row;
    int D;
    uint4 last;
    // The turn of a line is the exclusive or of its bits' turns, so that of a pass's line follows from the first pass's.
    __device__ __forceinline__ static int chunk_of(int i) {
        const int tid = (int)threadIdx.x % NTH;
        return (tid % H::LINE) ^ tile_turn<DT, H::LINE>(tid / H::LINE) ^ tile_turn<DT, H::LINE>(i * LINES);
    }
    __device__ __forceinline__ void clear(uint32_t lds) const {
        const int tid = (int)threadIdx.x % NTH;
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (chunk_of(i) * H::PER >= D) *(__attribute__((address_space(3))) u32x4*)(lds + (i * NTH + tid) * 16) = u32x4{0, 0, 0, 0};
    }
    // Whole chunks go straight to LDS; the one that D ends inside of, a row's last, through a register of the thread that has the row's number.
    __device__ __forceinline__ void fetch(int first, int left, uint32_t lds) {
        const int tid = (int)threadIdx.x % NTH, wave = __builtin_amdgcn_readfirstlane(tid >> 6), line = tid / H::LINE, whole = D / H::PER;
        const char* const from = (const char*)uniform64((int64_t)(base + (int64_t)first * row));
        if (left >= ROWS) {
            const uint32_t offset = (uint32_t)line * (uint32_t)row;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int chunk = chunk_of(i);
                if (D == DPAD || chunk < whole)
                    load_to_lds_at((const void*)uniform64((int64_t)(from + (int64_t)(i * LINES) * row)), offset + chunk * 16, __builtin_amdgcn_readfirstlane(lds + (i * NTH + wave * 64) * 16));
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < PASSES; ++i) {
                const int at = line + i * LINES, chunk = (tid % H::LINE) ^ tile_turn<DT, H::LINE>(at);
                const char* const src = from + (int64_t)at * row + chunk * 16;
                if (WHOLE || chunk != whole)
                    load_to_lds(at < left && chunk < whole ? (const void*)src : (const void*)&g_no_chunk, __builtin_amdgcn_readfirstlane(lds + (i * NTH + wave * 64) * 16));
            }
        }
        if constexpr (!WHOLE) last = end_of_row<DT>((const char*)(tid < ROWS && tid < left ? from + (int64_t)tid * row : nullptr), D);
    }
    // ... and from there to LDS, once all loads have arrived.
    __device__ __forceinline__ void settle(uint32_t lds) const {
        if constexpr (!WHOLE) {
            const int tid = (int)threadIdx.x % NTH, whole = D / H::PER;
            if (tid < ROWS && D % H::PER != 0) *(__attribute__((address_space(3))) u32x4*)(lds + tid * H::BYTES + (whole ^ tile_turn<DT, H::LINE>(tid)) * 16) = shifted<DT>(last, D);
        }
    }
};
// What a lane reads of a tile, whose first byte lies at a multiple of 1024: the chunk's number is in bits of its own of the address, so others of a line follow by an exclusive or.
// `apart`, the way to the other operand's tile, goes into the instruction's offset: added to the address it cost an addition a read, and the compiler took 16 bytes as two reads of 8
// that met banks twice.
template <int DT>
__device__ __forceinline__ f32x4 multiply(u32x4 a, uint4 b, f32x4 c) {
    if constexpr (DT == SC_F32) return multiply<DT>(__builtin_bit_cast(uint4, a), b, c);
    else if constexpr (DT == SC_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// Rows as they lie (16 rows, 64 bytes of channels a step) ...
template <int DT, int DPAD>
struct RowReader {
    using H = HeadShape<DT, DPAD>;
    uint32_t at;
    __device__ explicit RowReader(uint32_t lds) {
        const int i = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
        at = lds + i * H::BYTES + (g ^ tile_turn<DT, H::LINE>(i)) * 16;
    }
    __device__ __forceinline__ u32x4 read(uint32_t tile, int block, int k, int apart = 0) const {
        const uint32_t p = ((at + tile) ^ (k * 64)) + (block * (16 * H::BYTES) + apart);
        return *(lds_u32x4)p;
    }
};
// ... or across them: a block of 16 channels, of the rows 4 g .. 4 g + 3 of each 16, which are the rows that the quarter g of the lanes holds of S.
template <int DT, int DPAD>
struct ChannelReader {
    using H = HeadShape<DT, DPAD>;
    static constexpr int N = DT == SC_F32 ? 4 : 1;
    uint32_t at[N];
    __device__ explicit ChannelReader(uint32_t lds) {
        const int i = threadIdx.x & 15, g = (threadIdx.x >> 4) & 3;
        if constexpr (DT == SC_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) at[j] = lds + (4 * g + j) * H::BYTES + ((i >> 2) ^ tile_turn<DT, H::LINE>(4 * g + j)) * 16 + (i & 3) * 4;
        } else {                                   // a lane hands in 4 channels of row 4 g + i / 4 and gets channel i of the four rows
            const int line = 4 * g + (i >> 2);
            at[0] = lds + line * H::BYTES + (((i >> 1) & 1) ^ tile_turn<DT, H::LINE>(line)) * 16 + (i & 1) * 8;
        }
    }
    __device__ __forceinline__ uint4 read(uint32_t tile, int step, int c, int apart = 0) const {
        if constexpr (DT == SC_F32) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(lds_uint32)(((at[j] + tile) ^ (c * 64)) + (step * (H::STEP * H::BYTES) + apart));
            return make_uint4(v[0], v[1], v[2], v[3]);
        } else {
            const uint32_t p = ((at[0] + tile) ^ (c * 32)) + (step * (H::STEP * H::BYTES) + apart);
            const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
            const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 16 * H::BYTES)));
            return make_uint4(a.x, a.y, b.x, b.y);
        }
    }
};
// Weights of a step as the second product's second operand: rounded once to the rows' type (f32: as they are), or the matrix cores would need two products, of a weight and of
// what rounding left of it.  An error of a result's own rounding comes to it: of dq in bf16 0.0025 of its norm in place of the 0.0017 that the result's type costs.
// Forward the sum is of the weights ahead of that rounding, which spares turning them back.  So where one key has nearly all the weight of a row, and came at less than 2^CALM above
// the exponent that was followed, its rounding does not cancel: the row is its value times a factor that is off 1 by half a step of the type at most (2^-8 bf16, 2^-11 f16).
template <int DT, int ST>
__device__ __forceinline__ uint4 weights_of(const f32x4 (&p)[ST], int step) {
    if constexpr (DT == SC_F32) {
        return __builtin_bit_cast(uint4, p[step]);
    } else {
        const f32x4 a = p[2 * step], b = p[2 * step + 1];
        return make_uint4(round2<DT>(a[0], a[1]), round2<DT>(a[2], a[3]), round2<DT>(b[0], b[1]), round2<DT>(b[2], b[3]));
    }
}
// A row's channels as the first product's second operand; zeros for channels beyond D and for a column that is none (null).
template <int DT, int DPAD, bool WHOLE>
__device__ __forceinline__ void load_columns(const char* row, int D, uint4 (&q)[HeadShape<DT, DPAD>::KS]) {
    using H = HeadShape<DT, DPAD>;
    const int g = (threadIdx.x >> 4) & 3;
    const int whole = D / H::PER;
#pragma unroll
    for (int k = 0; k < H::KS; ++k) {
        const int chunk = 4 * k + g;
        q[k] = load_chunk(row != nullptr && chunk < whole ? row + chunk * 16 : (const char*)&g_no_chunk);
    }
    if constexpr (!WHOLE) {
        if (D % H::PER != 0) {
            const u32x4 last = shifted<DT>(end_of_row<DT>(row, D), D);
#pragma unroll
            for (int k = 0; k < H::KS; ++k) q[k] = 4 * k + g == whole ? __builtin_bit_cast(uint4, last) : q[k];
        }
    }
}
// Four consecutive channels of a row, those from D on left alone.
template <int DT, bool WHOLE = false>
__device__ __forceinline__ void store4(char* row, int channel, int D, f32x4 v) {
    if (WHOLE ? channel < D : channel + 4 <= D) {
        if constexpr (DT == SC_F32) {
            store_chunk(row + channel * 4, __builtin_bit_cast(uint4, v));
        } else {
            typedef uint32_t half_chunk __attribute__((ext_vector_type(2), aligned(2)));
            *reinterpret_cast<half_chunk*>(row + channel * 2) = half_chunk{round2<DT>(v[0], v[1]), round2<DT>(v[2], v[3])};
        }
    } else if (!WHOLE) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (channel + j < D) store_elem<DT>(row, channel + j, v[j]);
    }
}
// Over the four quarters of the lanes, the same bits in all of them: two registers that hold a number and each other's halves, or neighbouring quarters, after a swap.
template <class F>
__device__ inline float over_quarters(float v, F&& join) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, v);
    const auto a = __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    v = join(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const uint32_t half = __builtin_bit_cast(uint32_t, v);
    const auto b = __builtin_amdgcn_permlane32_swap(half, half, false, false);
    return join(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}
__device__ inline float over_quarters_max(float v) {
    return over_quarters(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int CONTROL>
__device__ inline float from_lane(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true)); }
__device__ inline float over_lanes_max(float v) {                 // the other of two, the other two of four, mirrored in eight and in sixteen; the quarters
    v = fmaxf(v, from_lane<0xb1>(v));
    v = fmaxf(v, from_lane<0x4e>(v));
    v = fmaxf(v, from_lane<0x141>(v));
    v = fmaxf(v, from_lane<0x140>(v));
    return over_quarters_max(v);
}
__device__ inline float over_quarters_sum(float v) {
    return over_quarters(v, [](float a, float b) { return a + b; });
}
// Row r of a head whose first row is at `base`: strides of rows are below 2^32 bytes.
__device__ __forceinline__ char* row_at(char* base, int r, int64_t row) { return base + (uint64_t)(uint32_t)r * (uint32_t)row; }
// All loads have arrived.  Said to the compiler too, which otherwise waits in the loop for the columns' loads ahead of it, and with them for the next tile's.
__device__ inline void loads_done() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0)
    asm volatile("" ::: "memory");
}

constexpr float NO_SCORE = -__builtin_inff();

// ---- forward --------------------------------------------------------------------------------------------
// Weights are taken against an exponent that follows the largest score only when that is more than CALM beyond it: sums and results are then scaled anew, which is
// rare behind the first tiles.  A weight is at most 2^(CALM + LIFT); the 16-bit floats of 5 exponent bits get their weights lifted so that small ones are not
// rounded off (their least normal number is 2^-14).
constexpr float CALM = 8.f;
template <int DT>
constexpr float LIFT = DT == SC_F16 ? 6.f : 0.f;

// Of a column, the same in its four lanes but for the sum, of which each has its rows'.
struct Running {
    float top;                         // largest exponent (score times log2 e) followed so far, minus infinity: none seen
    float against;                     // what exponents are taken against
    float sum;
};

// A larger score: what sums and results are scaled by.
template <int DT>
__device__ __forceinline__ float follow(Running& run, float score) {
    const float top = fmaxf(run.top, score), against = top == NO_SCORE ? 0.f : top - LIFT<DT>;
    const float factor = run.top == NO_SCORE ? 0.f : __builtin_amdgcn_exp2f(run.against - against);
    run.top = top;
    run.against = against;
    run.sum *= factor;
    return factor;
}
// SHARED: a wavefront has 16 NB columns of its own, and all walk the same tiles.  SPLIT: the wavefronts share 16 NB columns and take every WAVES-th tile each.
// ALONE: a wavefront has columns and tiles to itself, neighbours the next head of the same scene: rows of short heads share lines of memory.
enum Share { SHARED, SPLIT, ALONE };
template <int DT, int DPAD, int SHARE>
constexpr int walked_tile() {          // rows
    constexpr int BYTES = DPAD * ELEM<DT>;
    if (SHARE == SHARED) return BYTES >= 1024 ? 16 : BYTES >= 512 ? 32 : 64;
    return DT == SC_F32 && BYTES >= 512 ? 16 : 32;
}
template <int DT, int DPAD, int SHARE>
constexpr int walked_bytes() {         // two operands, two buffers; of a wavefront if it has its own
    return 4 * walked_tile<DT, DPAD, SHARE>() * DPAD * ELEM<DT>;
}
template <int DT, int DPAD, int SHARE>
constexpr int wavefronts() {
    constexpr int BYTES = walked_bytes<DT, DPAD, SHARE>();
    if (SHARE == SHARED) return 4;
    if (SHARE == SPLIT) return BYTES > 32768 ? 2 : 4;
    return BYTES > 32768 ? 1 : BYTES > 16384 ? 2 : 4;
}
// Blocks of 16 columns that go through a tile together, each row read from LDS once for all of them; ALONE one by one, and those only that have columns.
template <int NB, int SHARE>
constexpr int blocks_together() { return SHARE == ALONE ? 1 : NB; }
// What a workgroup, or a wavefront ALONE, works on: neighbours have the heads of one unit.
struct Item {
    int64_t unit;
    int head, part;
};
template <int SHARE, int WAVES>
__device__ inline Item item_of(int k_heads, int parts) {
    uint32_t n = blockIdx.y * gridDim.x + blockIdx.x;
    if constexpr (SHARE == ALONE) {    // runs of four workgroups to an XCD
        n = ((n / (4 * NUM_XCD) * NUM_XCD + n % NUM_XCD) * 4 + n / NUM_XCD % 4) * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    }
    const uint32_t rest = n / (uint32_t)k_heads, unit = rest / (uint32_t)parts;
    return Item{unit, (int)(n - rest * (uint32_t)k_heads), (int)(rest - unit * (uint32_t)parts)};
}
// The share of `all` steps that a part has: equal ones but for one step, and no more parts than there are `least` of the walked rows for.  In 32 bits: the three divisions
// of 64 were 350 scalar instructions, 0.3 us ahead of a kernel of 10.
__device__ inline void part_of(int all, int rows, int part, int parts, int least, int& from, int& to) {
    uint32_t used = ((uint32_t)all * (uint32_t)rows + (uint32_t)(least - 1)) / (uint32_t)least;
    used = used < (uint32_t)parts ? used : (uint32_t)parts;
    if ((uint32_t)part >= used) {
        from = to = 0;
        return;
    }
    const uint32_t each = (uint32_t)all / used, more = (uint32_t)all - each * used;
    from = (int)(each * (uint32_t)part) + ((uint32_t)part < more ? part : (int)more);
    to = from + (int)each + ((uint32_t)part < more ? 1 : 0);
}

template <int DT, int DPAD, int NB, int SHARE, bool WHOLE>
__global__ void __launch_bounds__((64 * wavefronts<DT, DPAD, SHARE>()), (NB * HeadShape<DT, DPAD>::BYTES >= 1024 ? 1 : SHARE == ALONE && HeadShape<DT, DPAD>::BYTES <= 64 ? (WHOLE ? 4 : 3) : 2))
k_attention(const Attention p) {
    using H = HeadShape<DT, DPAD>;
    constexpr int WAVES = wavefronts<DT, DPAD, SHARE>(), KT = walked_tile<DT, DPAD, SHARE>(), ST = KT / 16, TILE_BYTES = KT * H::BYTES;
    constexpr int COLUMNS = 16 * NB * (SHARE == SHARED ? WAVES : 1), TOGETHER = blocks_together<NB, SHARE>();
    // A wavefront's columns all go through a tile that its last one sees a key of: behind the last key that its first one sees there are 16 NB - 1 more, and the rest of a tile.
    static_assert(16 * NB - 1 + KT - 1 <= SC_ATTENTION_REACH, "keys with a weight of zero meet their values no further");
    extern __shared__ __align__(1024) uint4 attention_lds_words[];
    const Item item = item_of<SHARE, WAVES>(p.k_heads, p.parts);
    const int head_k = item.head, part = item.part;
    const int64_t unit = p.units - 1 - item.unit;                 // the last first: behind a causal mask they take longest
    if (unit < 0) return;
    const Scene scene = scene_of_queries(p, log2_of(COLUMNS), unit);
    if (scene.tile < 0) return;

    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int columns = scene.nq * p.per, column0 = scene.tile * COLUMNS + (SHARE == SHARED ? wave * 16 * NB : 0);
    const int ahead = scene.nk - scene.nq;
    // keys that a column sees: those below its limit
    auto limit_of = [&](int column) {
        if (!p.causal) return scene.nk;
        const int n = row_of_column(p, column) + ahead + 1;
        return n < 0 ? 0 : n < scene.nk ? n : scene.nk;
    };
    // row and head of a column, -1 where there is none; found again behind the loop, which has other use for the registers
    auto place_of = [&](int c, int& row, int& head) __attribute__((always_inline)) {
        row = c < columns ? row_of_column(p, c) : -1;
        head = head_k * p.per + (c < columns ? c - row * p.per : 0);
    };
    int limit[NB];
    uint4 q[NB][H::KS];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int c = column0 + 16 * n + i;
        int row, head;
        place_of(c, row, head);
        limit[n] = row >= 0 ? limit_of(c) : 0;
        load_columns<DT, DPAD, WHOLE>(row >= 0 ? row_at(p.q.data + scene.q0 * p.q.row + head * p.q.head, row, p.q.row) : nullptr, p.D, q[n]);
    }
    const int first_limit = column0 < columns ? __builtin_amdgcn_readfirstlane(limit_of(column0)) : 0;          // of the wavefront's columns the least and the largest
    const int last_column = column0 + 16 * NB < columns ? column0 + 16 * NB - 1 : columns - 1;
    const int wave_limit = column0 < columns ? __builtin_amdgcn_readfirstlane(limit_of(last_column)) : 0;
    const int all_last = scene.tile * COLUMNS + COLUMNS < columns ? scene.tile * COLUMNS + COLUMNS - 1 : columns - 1;
    const int tiles = (__builtin_amdgcn_readfirstlane(limit_of(all_last)) + KT - 1) / KT;
    int from = 0, to = tiles;
    if (p.parts > 1) part_of(tiles, KT, part, p.parts, p.part_keys, from, to);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)attention_lds_words;
    const uint32_t mine = lds0 + (SHARE == SHARED ? 0 : wave * (4 * TILE_BYTES));
    TileLoader<DT, DPAD, KT, SHARE == SHARED ? 64 * WAVES : 64, WHOLE> keys{p.k.data + scene.k0 * p.k.row + head_k * p.k.head, p.k.row, p.D},
        values{p.v.data + scene.k0 * p.v.row + head_k * p.v.head, p.v.row, p.D};
    const RowReader<DT, DPAD> rows(mine);
    const ChannelReader<DT, DPAD> channels(mine + TILE_BYTES);
    f32x4 out[NB][H::CB];
    Running run[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        run[n] = Running{NO_SCORE, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < H::CB; ++c) out[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    constexpr int STRIDE = SHARE == SPLIT ? WAVES : 1;
    if (p.D < DPAD) {
#pragma unroll
        for (int b = 0; b < 4; ++b) keys.clear(mine + b * TILE_BYTES);
    }
    auto bring = [&](int t, uint32_t buffer) __attribute__((always_inline)) {
        keys.fetch(t * KT, scene.nk - t * KT, mine + buffer);
        values.fetch(t * KT, scene.nk - t * KT, mine + buffer + TILE_BYTES);
    };
    uint32_t buffer = 0;
    const int begin = from + (SHARE == SPLIT ? wave : 0);
    if (begin < to) bring(begin, 0);
    for (int t = begin; t < to; t += STRIDE) {
        loads_done();
        keys.settle(mine + buffer);
        values.settle(mine + buffer + TILE_BYTES);
        if constexpr (SHARE == SHARED) lds_barrier();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + STRIDE < to) bring(t + STRIDE, buffer ^ (2 * TILE_BYTES));
        const int key0 = t * KT;
        if (SHARE == ALONE || key0 < wave_limit) {
#pragma unroll
            for (int n0 = 0; n0 < NB; n0 += TOGETHER) {
                if (SHARE == ALONE && column0 + 16 * n0 >= columns) break;
                f32x4 s[TOGETHER][ST];
#pragma unroll
                for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                    for (int b = 0; b < ST; ++b) s[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < H::KS; ++k)
#pragma unroll
                    for (int b = 0; b < ST; ++b) {
                        const u32x4 a = rows.read(buffer, b, k);
#pragma unroll
                        for (int n = 0; n < TOGETHER; ++n) s[n][b] = multiply<DT>(a, q[n0 + n][k], s[n][b]);
                    }
                if (key0 + KT > first_limit) {
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                        for (int b = 0; b < ST; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][b][r] = key0 + 16 * b + 4 * g + r < limit[n0 + n] ? s[n][b][r] : NO_SCORE;
                }
                float most[TOGETHER];
                bool calm = true;
#pragma unroll
                for (int n = 0; n < TOGETHER; ++n) {
                    most[n] = s[n][0][0];
#pragma unroll
                    for (int b = 0; b < ST; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) most[n] = fmaxf(most[n], s[n][b][r]);
                    most[n] *= p.scale_log2;
                    calm = calm && most[n] <= run[n0 + n].top + CALM;
                }
                if (!__all(calm)) {
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n) {
                        const float factor = follow<DT>(run[n0 + n], over_quarters_max(most[n]));
#pragma unroll
                        for (int c = 0; c < H::CB; ++c)
#pragma unroll
                            for (int r = 0; r < 4; ++r) out[n0 + n][c][r] *= factor;
                    }
                }
#pragma unroll
                for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                    for (int b = 0; b < ST; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[n][b][r] = __builtin_amdgcn_exp2f(fmaf(s[n][b][r], p.scale_log2, -run[n0 + n].against));
                            run[n0 + n].sum += s[n][b][r];
                        }
#pragma unroll
                for (int u = 0; u < KT / H::STEP; ++u) {
                    uint4 w[TOGETHER];
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n) w[n] = weights_of<DT, ST>(s[n], u);
#pragma unroll
                    for (int c = 0; c < H::CB; ++c) {
                        const uint4 a = channels.read(buffer, u, c);
#pragma unroll
                        for (int n = 0; n < TOGETHER; ++n) out[n0 + n][c] = multiply<DT>(a, w[n], out[n0 + n][c]);
                    }
                }
            }
        }
        buffer ^= 2 * TILE_BYTES;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) run[n].sum = over_quarters_sum(run[n].sum);

    if constexpr (SHARE == SPLIT) {                                        // the wavefronts' columns come together: wavefront w adds up every WAVES-th block of channels
        static_assert(NB == 1, "a block of columns");
        static_assert((16 * DPAD * 4 + 16 * 8) <= 4 * TILE_BYTES, "fits what the wavefront's tiles took");
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        float* const shared = reinterpret_cast<float*>(attention_lds_words);
        constexpr int APART = TILE_BYTES;                         // floats from wavefront to wavefront: its own four tiles
        float* const own = shared + wave * APART;
        if (g == 0) {
            own[2 * i] = run[0].sum == 0.f ? NO_SCORE : run[0].against;       // a sum that is no number has seen keys
            own[2 * i + 1] = run[0].sum;
        }
#pragma unroll
        for (int c = 0; c < H::CB; ++c)
#pragma unroll
            for (int r = 0; r < 4; ++r) own[32 + (16 * c + 4 * g + r) * 16 + i] = out[0][c][r];
        __syncthreads();
        float top = NO_SCORE;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, shared[w * APART + 2 * i]);
        float sum = 0.f, factor[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float theirs = shared[w * APART + 2 * i];
            factor[w] = theirs == NO_SCORE ? 0.f : __builtin_amdgcn_exp2f(theirs - top);
            sum += theirs == NO_SCORE ? 0.f : factor[w] * shared[w * APART + 2 * i + 1];
        }
        run[0].against = top == NO_SCORE ? 0.f : top;
        run[0].sum = sum;
#pragma unroll
        for (int c = 0; c < H::CB; ++c) {
            if (c % WAVES != wave) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += factor[w] == 0.f ? 0.f : factor[w] * shared[w * APART + 32 + (16 * c + 4 * g + r) * 16 + i];
                out[0][c][r] = v;
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        int c = column0 + 16 * n + i, row_there, head;
        asm volatile("" : "+v"(c));
        place_of(c, row_there, head);
        if (row_there < 0) continue;
        const int64_t row = scene.q0 + row_there, entry = row * (p.k_heads * p.per) + head;
        const bool first_writer = g == 0 && (SHARE != SPLIT || wave == 0);
        if (p.parts > 1) {
            const int64_t at = (int64_t)part * p.q_rows * (p.k_heads * p.per) + entry;
            if (first_writer) p.part_sums[at] = make_float2(run[n].against, run[n].sum);
            if (from < to) {
#pragma unroll
                for (int c = 0; c < H::CB; ++c)
                    if (SHARE != SPLIT || c % WAVES == wave) store4<SC_F32, WHOLE>((char*)(p.part_out + at * p.D), 16 * c + 4 * g, p.D, out[n][c]);
            }
        } else {
            const float inverse = run[n].sum == 0.f ? 0.f : 1.f / run[n].sum;
            char* const to_row = row_at(p.out.data + scene.q0 * p.out.row + head * p.out.head, row_there, p.out.row);
#pragma unroll
            for (int c = 0; c < H::CB; ++c)
                if (SHARE != SPLIT || c % WAVES == wave) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[n][c][r] *= inverse;
                    store4<DT, WHOLE>(to_row, 16 * c + 4 * g, p.D, out[n][c]);
                }
            if (p.lse != nullptr && first_writer) p.lse[entry] = run[n].sum == 0.f ? NO_SCORE : (__log2f(run[n].sum) + run[n].against) * 0.69314718055994531f;
        }
    }
}

// ---- backward -------------------------------------------------------------------------------------------
// Two kernels, so that every gradient is summed by one wavefront in one order: queries' columns walk the keys, keys' columns walk the queries.  The weights are made
// again in both from lse: seven products where five would do, and no atomics, no sums in memory.  (Gradients of queries added up over blocks of 128 keys would be 56 parts of a scene of 7069.)
// The walked rows go through the registers 32 at a time.
template <int DT, int DPAD, int SHARE>
constexpr int SUB = walked_tile<DT, DPAD, SHARE>() < 32 ? 16 : 32;

template <int DT, int DPAD, int NB, bool WHOLE>
constexpr int grad_waves(int rows, int results) {                 // wavefronts on a SIMD that the registers leave room for
    return NB * (rows * HeadShape<DT, DPAD>::KS * 4 + results * HeadShape<DT, DPAD>::CB * 4) > (DT == SC_F32 || !WHOLE ? 120 : 180) ? 1 : 2;
}

// Gradients of scores are a weight, some 1 / keys, times what may be small itself: in f16, whose least normal number is 2^-14, most of a long scene's would be rounded off.
// A wavefront therefore holds them times a power of two, `factor`, that its first ones set (the largest comes to 2^7 to 2^8, so those down to 2^-21 of it are normal), and sets it anew, with what is summed so far,
// when some come near f16's end.  The weights
// themselves are at most 1 and are lifted by 2^14 in the keys' kernel.
template <int DT>
constexpr float WEIGHT_LIFT = DT == SC_F16 ? 14.f : 0.f;
struct GradScale {
    int log2 = 0;
    float factor = 1.f;
    bool set = false;
};
// What sums and the gradients at hand, of which `most` is the lane's largest, are to be multiplied by: 1 almost always.  Past 2^60 there is nothing to win: a result of
// f16 has no use for what is smaller, and gradients to come have to fit.
__device__ __forceinline__ float rescale(GradScale& scale, float most) {
    if (scale.set ? __all(most <= 32768.f) : !__any(most > 0.f)) return 1.f;
    most = over_lanes_max(most < __builtin_inff() ? most : 0.f);              // what is not finite stays so
    if (scale.set ? most <= 32768.f : most == 0.f) return 1.f;
    const int log2 = max(-60, min(60, scale.log2 + 8 - __builtin_amdgcn_frexp_expf(most)));
    const float by = ldexpf(1.f, log2 - scale.log2);
    scale = GradScale{log2, ldexpf(1.f, log2), true};
    return by;
}

template <int DT, int DPAD, int NB, int SHARE, bool WHOLE>
__global__ void __launch_bounds__((64 * wavefronts<DT, DPAD, SHARE>()), (grad_waves<DT, DPAD, NB, WHOLE>(2, 1)))
k_attention_dq(const Attention p) {
    using H = HeadShape<DT, DPAD>;
    constexpr int WAVES = wavefronts<DT, DPAD, SHARE>(), KT = walked_tile<DT, DPAD, SHARE>(), TILE_BYTES = KT * H::BYTES, COLUMNS = 16 * NB * (SHARE == SHARED ? WAVES : 1);
    constexpr int SUB = sc::SUB<DT, DPAD, SHARE>, SUB_BLOCKS = SUB / 16, TOGETHER = blocks_together<NB, SHARE>();
    extern __shared__ __align__(1024) uint4 attention_lds_words[];
    const Item item = item_of<SHARE, WAVES>(p.k_heads, p.parts);
    const int head_k = item.head, part = item.part;
    const int64_t unit = p.units - 1 - item.unit;
    if (unit < 0) return;
    const Scene scene = scene_of_queries(p, log2_of(COLUMNS), unit);
    if (scene.tile < 0) return;

    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int columns = scene.nq * p.per, column0 = scene.tile * COLUMNS + (SHARE == SHARED ? wave * 16 * NB : 0);
    const int ahead = scene.nk - scene.nq;
    auto limit_of = [&](int column) {
        if (!p.causal) return scene.nk;
        const int n = row_of_column(p, column) + ahead + 1;
        return n < 0 ? 0 : n < scene.nk ? n : scene.nk;
    };
    const int first_limit = column0 < columns ? __builtin_amdgcn_readfirstlane(limit_of(column0)) : 0;
    const int last_column = column0 + 16 * NB < columns ? column0 + 16 * NB - 1 : columns - 1;
    const int wave_limit = column0 < columns ? __builtin_amdgcn_readfirstlane(limit_of(last_column)) : 0;
    const int all_last = scene.tile * COLUMNS + COLUMNS < columns ? scene.tile * COLUMNS + COLUMNS - 1 : columns - 1;
    const int tiles = (__builtin_amdgcn_readfirstlane(limit_of(all_last)) + KT - 1) / KT;

    int from = 0, to = tiles;
    if (p.parts > 1) part_of(tiles, KT, part, p.parts, p.part_keys, from, to);

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)attention_lds_words + (SHARE == SHARED ? 0 : wave * (4 * TILE_BYTES));
    TileLoader<DT, DPAD, KT, SHARE == SHARED ? 64 * WAVES : 64, WHOLE> keys{p.k.data + scene.k0 * p.k.row + head_k * p.k.head, p.k.row, p.D},
        values{p.v.data + scene.k0 * p.v.row + head_k * p.v.head, p.v.row, p.D};
    const RowReader<DT, DPAD> rows(lds0);
    const ChannelReader<DT, DPAD> channels(lds0);
    auto bring = [&](int t, uint32_t buffer) __attribute__((always_inline)) {
        keys.fetch(t * KT, scene.nk - t * KT, lds0 + buffer);
        values.fetch(t * KT, scene.nk - t * KT, lds0 + buffer + TILE_BYTES);
    };
    if (p.D < DPAD) {
#pragma unroll
        for (int b = 0; b < 4; ++b) keys.clear(lds0 + b * TILE_BYTES);
    }
    uint32_t buffer = 0;
    GradScale scale;
    if (from < to) bring(from, 0);
    int row_of[NB], head_of[NB], limit[NB];
    bool there[NB];
    uint4 q[NB][H::KS], dout[NB][H::KS], out[NB][H::KS];
    float against[NB], delta[NB];
    f32x4 dq[NB][H::CB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {                                // every load ahead of the first use of one
        const int c = column0 + 16 * n + i;
        there[n] = c < columns;
        row_of[n] = there[n] ? row_of_column(p, c) : 0;
        head_of[n] = head_k * p.per + (there[n] ? c - row_of[n] * p.per : 0);
        limit[n] = there[n] ? limit_of(c) : 0;
        load_columns<DT, DPAD, WHOLE>(there[n] ? row_at(p.q.data + scene.q0 * p.q.row + head_of[n] * p.q.head, row_of[n], p.q.row) : nullptr, p.D, q[n]);
        load_columns<DT, DPAD, WHOLE>(there[n] ? row_at(p.dout.data + scene.q0 * p.dout.row + head_of[n] * p.dout.head, row_of[n], p.dout.row) : nullptr, p.D, dout[n]);
        load_columns<DT, DPAD, WHOLE>(there[n] ? row_at(p.out.data + scene.q0 * p.out.row + head_of[n] * p.out.head, row_of[n], p.out.row) : nullptr, p.D, out[n]);
        against[n] = there[n] ? p.lse[(scene.q0 + row_of[n]) * (p.k_heads * p.per) + head_of[n]] : NO_SCORE;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int64_t row = scene.q0 + row_of[n];
        against[n] = against[n] == NO_SCORE ? -NO_SCORE : against[n] * 1.4426950408889634f;
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < H::KS; ++k) {
            const uint32_t a[4] = {dout[n][k].x, dout[n][k].y, dout[n][k].z, dout[n][k].w}, b[4] = {out[n][k].x, out[n][k].y, out[n][k].z, out[n][k].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (DT == SC_F32) {
                    sum = fmaf(__builtin_bit_cast(float, a[j]), __builtin_bit_cast(float, b[j]), sum);
                } else {
                    sum = fmaf(to_float<DT>(a[j] & 0xffffu), to_float<DT>(b[j] & 0xffffu), sum);
                    sum = fmaf(to_float<DT>(a[j] >> 16), to_float<DT>(b[j] >> 16), sum);
                }
            }
        }
        delta[n] = over_quarters_sum(sum);
        if (there[n] && g == 0 && part == 0) {                    // for the keys' kernel, a head's rows together
            p.against[(int64_t)head_of[n] * p.q_rows + row] = against[n] - WEIGHT_LIFT<DT>;
            p.delta[(int64_t)head_of[n] * p.q_rows + row] = -delta[n];
        }
#pragma unroll
        for (int c = 0; c < H::CB; ++c) dq[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int t = from; t < to; ++t) {
        loads_done();
        keys.settle(lds0 + buffer);
        values.settle(lds0 + buffer + TILE_BYTES);
        if constexpr (SHARE == SHARED) lds_barrier();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + 1 < to) bring(t + 1, buffer ^ (2 * TILE_BYTES));
#pragma unroll 1
        for (int h = 0; h < KT / SUB; ++h) {
            const int key0 = t * KT + h * SUB;
            const uint32_t tile = buffer + h * (SUB * H::BYTES);
            if (key0 >= wave_limit) break;
#pragma unroll
            for (int n0 = 0; n0 < NB; n0 += TOGETHER) {
                if (SHARE == ALONE && column0 + 16 * n0 >= columns) break;
                f32x4 s[TOGETHER][SUB_BLOCKS], dp[TOGETHER][SUB_BLOCKS];
#pragma unroll
                for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b) {
                        s[n][b] = f32x4{0.f, 0.f, 0.f, 0.f};
                        dp[n][b] = f32x4{-delta[n0 + n], -delta[n0 + n], -delta[n0 + n], -delta[n0 + n]};      // taken away here it costs no instruction
                    }
#pragma unroll
                for (int k = 0; k < H::KS; ++k)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b) {
                        const u32x4 a = rows.read(tile, b, k), v = rows.read(tile, b, k, TILE_BYTES);
#pragma unroll
                        for (int n = 0; n < TOGETHER; ++n) {
                            s[n][b] = multiply<DT>(a, q[n0 + n][k], s[n][b]);
                            dp[n][b] = multiply<DT>(v, dout[n0 + n][k], dp[n][b]);
                        }
                    }
#pragma unroll
                for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            s[n][b][r] = __builtin_amdgcn_exp2f(fmaf(s[n][b][r], p.scale_log2, scale.log2 - against[n0 + n])) * dp[n][b][r];
                if (key0 + SUB > first_limit) {
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                        for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) s[n][b][r] = key0 + 16 * b + 4 * g + r < limit[n0 + n] ? s[n][b][r] : 0.f;
                }
                if constexpr (DT == SC_F16) {
                    float most = 0.f;
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                        for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) most = fmaxf(most, fabsf(s[n][b][r]));
                    const bool summed = scale.set;                // or nothing but zeros so far
                    const float by = rescale(scale, most);
                    if (by != 1.f) {
#pragma unroll
                        for (int n = 0; n < TOGETHER; ++n)
#pragma unroll
                            for (int b = 0; b < SUB_BLOCKS; ++b) s[n][b] *= by;
                        if (summed) {
#pragma unroll
                            for (int n = 0; n < NB; ++n)
#pragma unroll
                                for (int c = 0; c < H::CB; ++c) dq[n][c] *= by;
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < SUB / H::STEP; ++u) {
                    uint4 w[TOGETHER];
#pragma unroll
                    for (int n = 0; n < TOGETHER; ++n) w[n] = weights_of<DT, SUB_BLOCKS>(s[n], u);
#pragma unroll
                    for (int c = 0; c < H::CB; ++c) {
                        const uint4 a = channels.read(tile, u, c);
#pragma unroll
                        for (int n = 0; n < TOGETHER; ++n) dq[n0 + n][c] = multiply<DT>(a, w[n], dq[n0 + n][c]);
                    }
                }
            }
        }
        buffer ^= 2 * TILE_BYTES;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        if (!there[n]) continue;
        const int64_t row = scene.q0 + row_of[n];
        float* const to_part = p.parts > 1 ? p.part_out + (((int64_t)part * p.q_rows + row) * (p.k_heads * p.per) + head_of[n]) * p.D : nullptr;
        char* const to_row = row_at(p.dq.data + scene.q0 * p.dq.row + head_of[n] * p.dq.head, row_of[n], p.dq.row);
#pragma unroll
        for (int c = 0; c < H::CB; ++c) {
            if constexpr (DT == SC_F16) dq[n][c] *= 1.f / scale.factor;
            if (p.parts > 1) {
                store4<SC_F32, WHOLE>((char*)to_part, 16 * c + 4 * g, p.D, dq[n][c]);
                continue;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) dq[n][c][r] *= p.scale;
            store4<DT, WHOLE>(to_row, 16 * c + 4 * g, p.D, dq[n][c]);
        }
    }
}

// Stand for rows that are not there: a weight of zero.
__device__ float g_no_weight = __builtin_inff();

constexpr int SUMS_BYTES = 4 * 64 * sizeof(float);
template <int DT, int DPAD, int NB, int SHARE, bool WHOLE>
__global__ void __launch_bounds__((64 * wavefronts<DT, DPAD, SHARE>()), (grad_waves<DT, DPAD, NB, WHOLE>(2, 2)))
k_attention_dkv(const Attention p) {
    using H = HeadShape<DT, DPAD>;
    constexpr int WAVES = wavefronts<DT, DPAD, SHARE>(), RT = walked_tile<DT, DPAD, SHARE>(), TILE_BYTES = RT * H::BYTES, COLUMNS = 16 * NB * (SHARE == SHARED ? WAVES : 1);
    constexpr int SUB = sc::SUB<DT, DPAD, SHARE>, SUB_BLOCKS = SUB / 16, TOGETHER = blocks_together<NB, SHARE>();
    extern __shared__ __align__(1024) uint4 attention_lds_words[];
    const Item item = item_of<SHARE, WAVES>(p.k_heads, p.k_parts);
    const int head_k = item.head, part = item.part;
    const int64_t unit = item.unit;                               // behind a causal mask the first take longest
    if (unit >= p.k_units) return;
    int64_t k0 = 0, q0 = 0, first_all = 0;
    int nk = 0, nq = 0, all = 0, scene_at;
    const int at = __builtin_amdgcn_readfirstlane(find_scene(p.k_starts, p.scenes, p.k_rows, 1, log2_of(COLUMNS), unit, p.k_units, first_all, all, scene_at).tile);
    if (at < 0) return;
    k0 = q0 = first_all;
    nk = nq = all;
    if (p.k_lens != nullptr) scene_rows(p.k_starts, p.k_lens, p.k_rows, scene_at, k0, nk);
    if (p.q_starts != p.k_starts || p.q_rows != p.k_rows) scene_rows(p.q_starts, nullptr, p.q_rows, scene_at, q0, nq);
    k0 = uniform64(k0);
    q0 = uniform64(q0);
    nk = __builtin_amdgcn_readfirstlane(nk);
    nq = __builtin_amdgcn_readfirstlane(nq);
    if (at * COLUMNS >= nk) return;

    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int column0 = at * COLUMNS + (SHARE == SHARED ? wave * 16 * NB : 0), ahead = nk - nq;
    // rows that see key c: c - ahead on
    const int tiles = (nq + RT - 1) / RT;
    int first_row = p.causal ? at * COLUMNS - ahead : 0;
    first_row = first_row < 0 ? 0 : first_row;
    const int first_tile = first_row / RT < tiles ? first_row / RT : tiles;
    const int last_column = column0 + 16 * NB - 1 < nk ? column0 + 16 * NB - 1 : nk - 1;

    constexpr uint32_t SUMS = 4 * TILE_BYTES;                     // exponents and deltas of a tile's rows, 64 words each, two buffers
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)attention_lds_words + (SHARE == SHARED ? 0 : wave * (SUMS + SUMS_BYTES));
    const RowReader<DT, DPAD> rows(lds0);
    const ChannelReader<DT, DPAD> channels(lds0);
    const int each = tiles - first_tile, total = each * p.per;
    int from = 0, to = total;
    if (p.k_parts > 1) part_of(total, RT, part, p.k_parts, p.part_rows, from, to);
    TileLoader<DT, DPAD, RT, SHARE == SHARED ? 64 * WAVES : 64, WHOLE> queries{nullptr, p.q.row, p.D}, grads{nullptr, p.dout.row, p.D};
    int next_head = 0, next = 0;                                  // of the tile to bring
    if (p.k_parts > 1 && from < to) {
        next_head = (int)((uint32_t)from / (uint32_t)each);
        next = from - next_head * each;
    }
    auto bring = [&](int which) __attribute__((always_inline)) {
        const int t = first_tile + next, head = head_k * p.per + next_head, left = nq - t * RT;
        queries.base = p.q.data + q0 * p.q.row + head * p.q.head;
        grads.base = p.dout.data + q0 * p.dout.row + head * p.dout.head;
        queries.fetch(t * RT, left, lds0 + which * (2 * TILE_BYTES));
        grads.fetch(t * RT, left, lds0 + which * (2 * TILE_BYTES) + TILE_BYTES);
        const int64_t from = (int64_t)head * p.q_rows + q0 + t * RT + lane;
        // all lanes, with nothing for those beyond the tile: a branch of some lanes would be one more place where the compiler may save registers for them alone
        if (SHARE != SHARED || wave == 0)
            load_word_to_lds(lane < RT && lane < left ? (const void*)(p.against + from) : (const void*)&g_no_weight, __builtin_amdgcn_readfirstlane(lds0 + SUMS + which * 512));
        if (SHARE != SHARED || wave == WAVES - 1)
            load_word_to_lds(lane < RT && lane < left ? (const void*)(p.delta + from) : (const void*)&g_no_chunk, __builtin_amdgcn_readfirstlane(lds0 + SUMS + which * 512 + 256));
    };
    if (p.D < DPAD) {
#pragma unroll
        for (int b = 0; b < 4; ++b) queries.clear(lds0 + b * TILE_BYTES);
    }
    if (from < to) bring(0);
    uint4 k[NB][H::KS], v[NB][H::KS];
    f32x4 dk[NB][H::CB], dv[NB][H::CB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int c = column0 + 16 * n + i;
        load_columns<DT, DPAD, WHOLE>(c < nk ? row_at(p.k.data + k0 * p.k.row + head_k * p.k.head, c, p.k.row) : nullptr, p.D, k[n]);
        load_columns<DT, DPAD, WHOLE>(c < nk ? row_at(p.v.data + k0 * p.v.row + head_k * p.v.head, c, p.v.row) : nullptr, p.D, v[n]);
#pragma unroll
        for (int c = 0; c < H::CB; ++c) dk[n][c] = dv[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    int which = 0;
    GradScale scale;
    for (int n = from; n < to; ++n, which ^= 1) {
        loads_done();
        queries.settle(lds0 + which * (2 * TILE_BYTES));
        grads.settle(lds0 + which * (2 * TILE_BYTES) + TILE_BYTES);
        if constexpr (SHARE == SHARED) lds_barrier();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        const int row_tile = (first_tile + next) * RT;
        if (++next == each) {
            next = 0;
            ++next_head;
        }
        if (n + 1 < to) bring(which ^ 1);
#pragma unroll 1
        for (int h = 0; h < RT / SUB; ++h) {
            const int row0 = row_tile + h * SUB;
            const uint32_t tile = which * (2 * TILE_BYTES) + h * (SUB * H::BYTES);
            if (p.causal && row0 + SUB - 1 + ahead < column0) continue;       // none of the rows sees any of the keys
            if (row0 >= nq || column0 >= nk) break;
            const bool masked = p.causal && row0 + ahead < last_column;
#pragma unroll
            for (int m0 = 0; m0 < NB; m0 += TOGETHER) {
                if (SHARE == ALONE && column0 + 16 * m0 >= nk) break;
                f32x4 s[TOGETHER][SUB_BLOCKS], dp[TOGETHER][SUB_BLOCKS];
#pragma unroll
                for (int m = 0; m < TOGETHER; ++m)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b) s[m][b] = f32x4{0.f, 0.f, 0.f, 0.f};
                f32x4 against[SUB_BLOCKS];
#pragma unroll
                for (int b = 0; b < SUB_BLOCKS; ++b) {
                    const uint32_t sums = lds0 + SUMS + which * 512 + (h * SUB + 16 * b + 4 * g) * 4;
                    against[b] = __builtin_bit_cast(f32x4, *(lds_u32x4)sums);
                    const f32x4 delta = __builtin_bit_cast(f32x4, *(lds_u32x4)(sums + 256));
#pragma unroll
                    for (int m = 0; m < TOGETHER; ++m) dp[m][b] = delta;
                }
#pragma unroll
                for (int c = 0; c < H::KS; ++c)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b) {
                        const u32x4 a = rows.read(tile, b, c), d = rows.read(tile, b, c, TILE_BYTES);
#pragma unroll
                        for (int m = 0; m < TOGETHER; ++m) {
                            s[m][b] = multiply<DT>(a, k[m0 + m][c], s[m][b]);
                            dp[m][b] = multiply<DT>(d, v[m0 + m][c], dp[m][b]);
                        }
                    }
                const float lowered = DT == SC_F16 ? scale.factor * 0x1p-14f : 1.f;         // the weights' lift taken back
#pragma unroll
                for (int m = 0; m < TOGETHER; ++m)
#pragma unroll
                    for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            s[m][b][r] = __builtin_amdgcn_exp2f(fmaf(s[m][b][r], p.scale_log2, -against[b][r]));
                            dp[m][b][r] = s[m][b][r] * (DT == SC_F16 ? dp[m][b][r] * lowered : dp[m][b][r]);
                        }
                if (masked) {
#pragma unroll
                    for (int m = 0; m < TOGETHER; ++m)
#pragma unroll
                        for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) {
                                const bool seen = row0 + 16 * b + 4 * g + r + ahead >= column0 + 16 * (m0 + m) + i;
                                s[m][b][r] = seen ? s[m][b][r] : 0.f;
                                dp[m][b][r] = seen ? dp[m][b][r] : 0.f;
                            }
                }
                if constexpr (DT == SC_F16) {
                    float most = 0.f;                             // of columns that are keys: the weight of one that is none is exp(-lse), however large
#pragma unroll
                    for (int m = 0; m < TOGETHER; ++m) {
                        float of_column = 0.f;
#pragma unroll
                        for (int b = 0; b < SUB_BLOCKS; ++b)
#pragma unroll
                            for (int r = 0; r < 4; ++r) of_column = fmaxf(of_column, fabsf(dp[m][b][r]));
                        most = i < nk - column0 - 16 * (m0 + m) ? fmaxf(most, of_column) : most;
                    }
                    const bool summed = scale.set;                // or nothing but zeros so far
                    const float by = rescale(scale, most);
                    if (by != 1.f) {
#pragma unroll
                        for (int m = 0; m < TOGETHER; ++m)
#pragma unroll
                            for (int b = 0; b < SUB_BLOCKS; ++b) dp[m][b] *= by;
                        if (summed) {
#pragma unroll
                            for (int m = 0; m < NB; ++m)
#pragma unroll
                                for (int c = 0; c < H::CB; ++c) dk[m][c] *= by;
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < SUB / H::STEP; ++u) {
                    uint4 w[TOGETHER], z[TOGETHER];
#pragma unroll
                    for (int m = 0; m < TOGETHER; ++m) {
                        w[m] = weights_of<DT, SUB_BLOCKS>(s[m], u);
                        z[m] = weights_of<DT, SUB_BLOCKS>(dp[m], u);
                    }
#pragma unroll
                    for (int c = 0; c < H::CB; ++c) {
                        const uint4 a = channels.read(tile, u, c, TILE_BYTES), b = channels.read(tile, u, c);
#pragma unroll
                        for (int m = 0; m < TOGETHER; ++m) {
                            dv[m0 + m][c] = multiply<DT>(a, w[m], dv[m0 + m][c]);
                            dk[m0 + m][c] = multiply<DT>(b, z[m], dk[m0 + m][c]);
                        }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int c = column0 + 16 * n + i;
        if (c >= nk) continue;
        const int64_t at_part = (((int64_t)part * p.k_rows + k0 + c) * p.k_heads + head_k) * p.D;
        char* const to_k = row_at(p.dk.data + k0 * p.dk.row + head_k * p.dk.head, c, p.dk.row);
        char* const to_v = row_at(p.dv.data + k0 * p.dv.row + head_k * p.dv.head, c, p.dv.row);
#pragma unroll
        for (int b = 0; b < H::CB; ++b) {
            if constexpr (DT == SC_F16) {
                dk[n][b] *= 1.f / scale.factor;
                dv[n][b] *= 0x1p-14f;
            }
            if (p.k_parts > 1) {
                store4<SC_F32, WHOLE>((char*)(p.part_dk + at_part), 16 * b + 4 * g, p.D, dk[n][b]);
                store4<SC_F32, WHOLE>((char*)(p.part_dv + at_part), 16 * b + 4 * g, p.D, dv[n][b]);
                continue;
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) dk[n][b][r] *= p.scale;
            store4<DT, WHOLE>(to_k, 16 * b + 4 * g, p.D, dk[n][b]);
            store4<DT, WHOLE>(to_v, 16 * b + 4 * g, p.D, dv[n][b]);
        }
    }
}
// Four channels of a partial result, of which `there` are.
__device__ __forceinline__ f32x4 partial4(const float* p, int there) {
    if (there >= 4) return __builtin_bit_cast(f32x4, load_chunk(p));
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < there) v[j] = p[j];
    return v;
}
// Parts of a gradient added up, in their order: a workgroup has JOIN_ROWS rows of a scene.
constexpr int JOIN_ROWS = 4, JOIN_ROWS_LOG2 = 2;
template <int DT>
__global__ void __launch_bounds__(256)
k_attention_grad_join(const int32_t* __restrict__ starts, const int32_t* __restrict__ lens, int scenes, int64_t rows, int heads, int D, int parts,
                      const float* __restrict__ a, HeadRows to_a, float scale_a, const float* __restrict__ b, HeadRows to_b) {
    int64_t first = 0;
    int count = 0, scene;
    const int tile = __builtin_amdgcn_readfirstlane(find_scene(starts, scenes, rows, 1, JOIN_ROWS_LOG2, (int64_t)blockIdx.y * gridDim.x + blockIdx.x, scene_units(rows, scenes, JOIN_ROWS), first, count, scene).tile);
    if (tile < 0) return;
    if (lens != nullptr) scene_rows(starts, lens, rows, scene, first, count);
    const int here = count - tile * JOIN_ROWS < JOIN_ROWS ? count - tile * JOIN_ROWS : JOIN_ROWS, fours = (D + 3) / 4, row_items = heads * fours;
    const int64_t row0 = first + tile * JOIN_ROWS, apart = rows * heads * D;
    for (int i = threadIdx.x; i < here * row_items; i += 256) {
        const int r = i / row_items, head = (i - r * row_items) / fours, channel = (i - r * row_items - head * fours) * 4;
        const int64_t at = ((row0 + r) * heads + head) * D + channel;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float* const from = w == 0 ? a : b;
            if (from == nullptr) continue;
            f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
            for (int k = 0; k < parts; ++k) {
                v += partial4(from + k * apart + at, D - channel);
            }
            const HeadRows to = w == 0 ? to_a : to_b;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] *= w == 0 ? scale_a : 1.f;
            store4<DT>(to.data + (row0 + r) * to.row + head * to.head, channel, D, v);
        }
    }
}

// Parts joined: a thread has four channels of a row's head.
template <int DT>
__global__ void __launch_bounds__(256)
k_attention_join_rows(const Attention p, int64_t entries, int q_heads) {
    const int fours = (p.D + 3) / 4;
    const int64_t item = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x, entry = item / fours;
    if (entry >= entries) return;
    const int64_t row = entry / q_heads;
    if (p.q_starts != nullptr && (row < p.q_starts[0] || row >= p.q_starts[p.scenes])) return;        // a row of no scene stays as it is
    const int channel = (int)(item - entry * fours) * 4;
    float top = NO_SCORE, sum = 0.f;
#pragma unroll 8
    for (int k = 0; k < p.parts; ++k) {
        const float2 s = p.part_sums[k * entries + entry];
        top = s.y == 0.f ? top : fmaxf(top, s.x);
    }
    f32x4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < p.parts; ++k) {
        const float2 s = p.part_sums[k * entries + entry];
        const bool seen = s.y != 0.f;                            // nothing seen: its results were not written
        const float factor = seen ? __builtin_amdgcn_exp2f(s.x - top) : 0.f;
        sum = seen ? fmaf(factor, s.y, sum) : sum;
        const float* const from = p.part_out + (k * entries + entry) * p.D + channel;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = seen && channel + j < p.D ? fmaf(factor, from[j], v[j]) : v[j];
    }
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= inverse;
    store4<DT>(p.out.data + row * p.out.row + (entry - row * q_heads) * p.out.head, channel, p.D, v);
    if (p.lse != nullptr && channel == 0) p.lse[entry] = sum == 0.f ? NO_SCORE : (__log2f(sum) + top) * 0.69314718055994531f;
}
// Many parts of few rows: a workgroup has a row's head, its threads four channels and every so many of the parts.
template <int DT>
__global__ void __launch_bounds__(256)
k_attention_join(const Attention p, int64_t entries, int q_heads) {
    __shared__ float factors[ATTENTION_PARTS_MAX];
    __shared__ float2 of_wave[4];
    __shared__ f32x4 shared[256];
    const int64_t entry = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (entry >= entries) return;
    const int64_t row = entry / q_heads;
    if (p.q_starts != nullptr && (row < p.q_starts[0] || row >= p.q_starts[p.scenes])) return;        // a row of no scene stays as it is
    const int tid = threadIdx.x, wave = tid >> 6;
    const float2 mine = tid < p.parts ? p.part_sums[tid * entries + entry] : make_float2(0.f, 0.f);
    const bool seen = mine.y != 0.f;                             // nothing seen: its results were not written
    float top = seen ? mine.x : NO_SCORE;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    if ((tid & 63) == 0) of_wave[wave].x = top;
    __syncthreads();
    top = fmaxf(fmaxf(of_wave[0].x, of_wave[1].x), fmaxf(of_wave[2].x, of_wave[3].x));
    const float factor = seen ? __builtin_amdgcn_exp2f(mine.x - top) : 0.f;
    factors[tid] = factor;
    float sum = seen ? factor * mine.y : 0.f;
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) sum += __shfl_xor(sum, d);
    if ((tid & 63) == 0) of_wave[wave].y = sum;
    __syncthreads();
    sum = (of_wave[0].y + of_wave[1].y) + (of_wave[2].y + of_wave[3].y);
    int log2 = 0;
    while (4 << log2 < p.D) ++log2;
    const int channel = (tid & ((1 << log2) - 1)) * 4, first = tid >> log2, step = 256 >> log2;
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    if (channel < p.D) {
#pragma unroll 4
        for (int k = first; k < p.parts; k += step) {
            if (factors[k] == 0.f) continue;
            const f32x4 from = partial4(p.part_out + (k * entries + entry) * p.D + channel, p.D - channel);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = fmaf(factors[k], from[j], v[j]);
        }
    }
    shared[tid] = v;
    __syncthreads();
    if (first != 0 || channel >= p.D) return;
    for (int k = 1; k < step; ++k) v += shared[tid + (k << log2)];
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] *= inverse;
    store4<DT>(p.out.data + row * p.out.row + (entry - row * q_heads) * p.out.head, channel, p.D, v);
    if (p.lse != nullptr && channel == 0) p.lse[entry] = sum == 0.f ? NO_SCORE : (__log2f(sum) + top) * 0.69314718055994531f;
}

// ---- launches -------------------------------------------------------------------------------------------
// Workgroups for so many items, of which a workgroup has one or each of its wavefronts ALONE.
template <int SHARE, int WAVES>
inline int64_t blocks_for(int64_t items) {
    if (SHARE != ALONE) return items;
    constexpr int64_t RUN = 4 * NUM_XCD;
    return ((items + WAVES - 1) / WAVES + RUN - 1) / RUN * RUN;
}
inline dim3 grid_of(int64_t blocks) { return dim3((unsigned)grid_columns(blocks), (unsigned)grid_rows(blocks)); }
constexpr int64_t BLOCKS_MAX = INT32_MAX / 4 - 2 * GRID_COLUMNS;

template <int DT, int DPAD, int NB, int SHARE, bool WHOLE>
int start_attention(Attention p, hipStream_t s) {
    constexpr auto kernel = k_attention<DT, DPAD, NB, SHARE, WHOLE>;
    constexpr int WAVES = wavefronts<DT, DPAD, SHARE>();
    constexpr size_t lds = (size_t)(SHARE == SHARED ? 1 : WAVES) * walked_bytes<DT, DPAD, SHARE>();
    static_assert(lds <= 163840, "of a CU");
    p.units = scene_units(p.q_rows * p.per, p.scenes, 16 * NB * (SHARE == SHARED ? WAVES : 1));
    const int64_t blocks = blocks_for<SHARE, WAVES>(p.units * p.k_heads * p.parts);
    if (blocks > BLOCKS_MAX) return SC_EINVAL;
    static bool done[MAX_DEVICES];
    const int rc = allow_lds((const void*)kernel, lds, done);
    if (rc != SC_OK) return rc;
    SC_LAUNCH(KID_ATTENTION, kernel, grid_of(blocks), dim3(64 * WAVES), lds, s, p);
    return SC_OK;
}
template <int DT, int DPAD, bool WHOLE>
int choose_attention(const Attention& p, AttentionShape shape, hipStream_t s) {
    constexpr int NB = DPAD == 256 ? 1 : 2, WIDE = DPAD * ELEM<DT> <= 128 ? 4 : NB;      // 256 channels, f16, two blocks / one: 9310 rows of 32 + 8 heads in 38 scenes 266 / 208 us
    if (shape == ATTENTION_FEW) return start_attention<DT, DPAD, 1, SPLIT, WHOLE>(p, s);
    if (shape == ATTENTION_SHORT) return start_attention<DT, DPAD, NB, ALONE, WHOLE>(p, s);
    if (shape == ATTENTION_SHORT_64) return start_attention<DT, DPAD, WIDE, ALONE, WHOLE>(p, s);
    return start_attention<DT, DPAD, NB, SHARED, WHOLE>(p, s);
}
template <int DT, bool WHOLE>
int choose_head(const Attention& p, AttentionShape shape, hipStream_t s) {
    return p.D <= 32 ? choose_attention<DT, 32, WHOLE>(p, shape, s) : p.D <= 64 ? choose_attention<DT, 64, WHOLE>(p, shape, s)
           : p.D <= 128 ? choose_attention<DT, 128, WHOLE>(p, shape, s) : choose_attention<DT, 256, WHOLE>(p, shape, s);
}
template <int DT>
int launch_attention(const Attention& p, AttentionShape shape, hipStream_t s) {
    const int rc = p.D * ELEM<DT> % 16 == 0 ? choose_head<DT, true>(p, shape, s) : choose_head<DT, false>(p, shape, s);
    if (rc != SC_OK || p.parts == 1) return rc;
    const int q_heads = p.k_heads * p.per;
    const int64_t entries = p.q_rows * q_heads;
    if (entries > BLOCKS_MAX) return SC_EINVAL;
    const int64_t items = entries * ((p.D + 3) / 4);
    if (join_by_rows(p.parts, items)) {
        SC_LAUNCH(KID_ATTENTION_JOIN, k_attention_join_rows<DT>, grid_of((items + 255) / 256), dim3(256), 0, s, p, entries, q_heads);
        return SC_OK;
    }
    SC_LAUNCH(KID_ATTENTION_JOIN, k_attention_join<DT>, grid_of(entries), dim3(256), 0, s, p, entries, q_heads);
    return SC_OK;
}

template <int DT, int DPAD, int NB, int SHARE, bool WHOLE>
int start_attention_grad(Attention p, hipStream_t s) {
    constexpr auto of_queries = k_attention_dq<DT, DPAD, NB, SHARE, WHOLE>;
    constexpr auto of_keys = k_attention_dkv<DT, DPAD, NB, SHARE, WHOLE>;
    constexpr int WAVES = wavefronts<DT, DPAD, SHARE>(), COLUMNS = 16 * NB * (SHARE == SHARED ? WAVES : 1);
    constexpr size_t lds = (size_t)(SHARE == SHARED ? 1 : WAVES) * walked_bytes<DT, DPAD, SHARE>(), lds_keys = lds + (SHARE == SHARED ? 1 : WAVES) * SUMS_BYTES;
    static_assert(lds_keys <= 163840, "of a CU");
    p.units = scene_units(p.q_rows * p.per, p.scenes, COLUMNS);
    p.k_units = scene_units(p.k_rows, p.scenes, COLUMNS);
    const int64_t blocks = blocks_for<SHARE, WAVES>(p.units * p.k_heads * p.parts), key_blocks = blocks_for<SHARE, WAVES>(p.k_units * p.k_heads * p.k_parts);
    if (blocks > BLOCKS_MAX || key_blocks > BLOCKS_MAX) return SC_EINVAL;
    static bool done_queries[MAX_DEVICES], done_keys[MAX_DEVICES];
    int rc = allow_lds((const void*)of_queries, lds, done_queries);
    if (rc == SC_OK) rc = allow_lds((const void*)of_keys, lds_keys, done_keys);
    if (rc != SC_OK) return rc;
    if (p.q_rows > 0) SC_LAUNCH(KID_ATTENTION_DQ, of_queries, grid_of(blocks), dim3(64 * WAVES), lds, s, p);
    if (p.k_rows > 0) SC_LAUNCH(KID_ATTENTION_DKV, of_keys, grid_of(key_blocks), dim3(64 * WAVES), lds_keys, s, p);
    return SC_OK;
}
template <int DT, int DPAD, bool WHOLE>
int choose_attention_grad(const Attention& p, bool alone, hipStream_t s) {
    constexpr int NB = DPAD == 256 || (DT == SC_F32 && DPAD == 128) ? 1 : 2;
    return alone ? start_attention_grad<DT, DPAD, NB, ALONE, WHOLE>(p, s) : start_attention_grad<DT, DPAD, NB, SHARED, WHOLE>(p, s);
}
template <int DT, bool WHOLE>
int choose_head_grad(const Attention& p, bool alone, hipStream_t s) {
    return p.D <= 32 ? choose_attention_grad<DT, 32, WHOLE>(p, alone, s) : p.D <= 64 ? choose_attention_grad<DT, 64, WHOLE>(p, alone, s)
           : p.D <= 128 ? choose_attention_grad<DT, 128, WHOLE>(p, alone, s) : choose_attention_grad<DT, 256, WHOLE>(p, alone, s);
}
template <int DT>
int launch_attention_grad(const Attention& p, bool alone, hipStream_t s) {
    const int rc = p.D * ELEM<DT> % 16 == 0 ? choose_head_grad<DT, true>(p, alone, s) : choose_head_grad<DT, false>(p, alone, s);
    if (rc != SC_OK) return rc;
    const int q_heads = p.k_heads * p.per;
    if (p.parts > 1 && p.q_rows > 0)
        SC_LAUNCH(KID_ATTENTION_JOIN, k_attention_grad_join<DT>, grid_of(scene_units(p.q_rows, p.scenes, JOIN_ROWS)), dim3(256), 0, s, p.q_starts, (const int32_t*)nullptr,
                  p.scenes, p.q_rows, q_heads, p.D, p.parts, p.part_out, p.dq, p.scale, (const float*)nullptr, p.dq);
    if (p.k_parts > 1 && p.k_rows > 0)
        SC_LAUNCH(KID_ATTENTION_JOIN, k_attention_grad_join<DT>, grid_of(scene_units(p.k_rows, p.scenes, JOIN_ROWS)), dim3(256), 0, s, p.k_starts, p.k_lens, p.scenes,
                  p.k_rows, p.k_heads, p.D, p.k_parts, p.part_dk, p.dk, p.scale, p.part_dv, p.dv);
    return SC_OK;
}

}  // namespace sc
