// Products of feature rows with weights, and of feature rows with gradient rows: one tile kernel for linear layers and for
// layers whose weights differ by group of rows (sc_layers.hip).
//
//     FWD   out[p][n] = act(sum_k a[row(p)][k] w[g][k][n] + bias[g][n]) + residual[p][n]     k: C_in,  n: C_out
//     DX    out[p][n] = sum_k a[row(p)][k] w[g][n][k]                                        k: C_out, n: C_in
//     DX_ACT  the same with a[row(p)][k] act'(pre[p][k]) in place of a, rounded to its type, which is kept in kept[p][k]; sums over p before the rounding
//     DW    out[g][m][n] = sum_p a[row(p)][m] b[row'(p)][n],  bias[g][n] = sum_p b[row'(p)][n]   p: entries of group g
//
// A workgroup owns a BM x BN tile of the result and walks the summed axis in steps of 128 bytes (KW times that where KW sets of
// wavefronts share the axis).  Both operands pass through LDS, two buffers deep, 16 bytes a lane straight from global memory: the step
// that follows is in flight while one is multiplied.  A tile is stored as it lies in memory, either as rows along the summed axis (a lane's operand
// is then 16 consecutive bytes) or as rows across it (weights in the forward product, both sides of DW), which the transposing LDS
// read turns into operand order on the way to the registers, so nothing is ever re-laid out in memory.  Chunks of 16 bytes are permuted inside a
// line by the line's number so that the lanes of one LDS access meet different banks; the permutation is in the address that a lane
// loads from, because a load into LDS fills it in the order of the lanes.
// The weights' side is the matrix instruction's first operand, so that a lane ends up with four consecutive columns of one row; one exchange between
// lanes makes them eight, which go out with bias, activation and residual in the registers they were summed in.
//
// What bounds it: memory up to some hundred channels, the matrix cores from about 1000 x 1000 on, a way through LDS in between (an operand's byte is read BM or BN
// over 16 times from there), and the launch with one trip to memory for few rows.  bf16, us, a copy on this card 5.1 TB/s, the library's largest product 1135 TFLOP/s:
//     one row 1024 -> 4096                  5.1     8.4 MB of weights, launch and latency; 4.2 in a row of calls (2.0 TB/s)
//     53 k x 64 -> 256, f16, both outputs  17.4     61.5 MB, 3.5 TB/s: one step of the axis, then GELU and the stores; nothing to hide them behind but other workgroups
//     10^6 x 128 -> 128                    87.7     512 MB, 5.8 TB/s
//     32768 x 2048 -> 2048                  261     1054 TFLOP/s (with residual and cold 290)
//     16384 rows in 16 groups, 512 -> 2048 SiLU 61.2   562 TFLOP/s
//     the gradients: 16384 in 16 groups 2048 -> 512  58.9   583 TFLOP/s; weights 16384 x 512 x 2048 65.4   525 TFLOP/s; 10^6 x 128 -> 128 107   4.8 TB/s
// Steps of 128 bytes two deep leave room for two to four workgroups on a CU, which hide each other's barriers: three steps deep was slower everywhere (fewer of them).
#pragma once

#include <type_traits>

#include "sc_conv.h"

namespace sc {

enum ProductMode { PRODUCT_FWD, PRODUCT_DX, PRODUCT_DX_ACT, PRODUCT_DW };

struct Product {
    const void* a;                 // rows
    int64_t lda, a_rows;           // elements from row to row, rows there are
    const int32_t* a_list;         // row of an entry; null: the entry's own number
    const void* b;                 // weights, or (DW) the other rows
    int64_t ldb, b_rows;
    const int32_t* b_list;         // DW
    const int32_t* starts;         // first entry of every group and the end of the last; null: one group of n
    int groups;
    int64_t n, per;                // entries; DW: entries per part of a group
    int M, N, K;                   // channels: FWD K -> N, DX K -> N, DW M x N
    int64_t units;                 // row tiles there can be at most (DW: parts)
    int run;                       // consecutive tiles that one XCD takes: product_run
    const void* bias;
    int act;
    const void* residual;
    int64_t ldr;
    void* pre;                     // DX_ACT: read
    int64_t ldp;
    void* out;
    int64_t ldo;
    int out_f32;                   // FWD
    void* kept;                    // DX_ACT
    int64_t ldk;
    void* out_bias;                // DW
    float* bias_sums;              // DX_ACT: [bias_units][K], null: not wanted; DW: the same, null: the sums of b's rows instead
    int bias_log2;                 // DW: 2^bias_log2 entries in a unit
    float* partial;                // DW: [slot][(M + 1) N], null if no group can have two parts
    int64_t slots;                 // ... how many
};

// ---- elements ---------------------------------------------------------------------------------------
template <int DT>
constexpr int ELEM = DT == SC_F32 ? 4 : 2;

struct __attribute__((packed, aligned(2))) Chunk2 {      // 16 bytes at any 2-byte boundary: the hardware takes them as they are
    uint32_t v[4];
};
__device__ inline uint4 load_chunk(const void* p) {
    const Chunk2 c = *reinterpret_cast<const Chunk2*>(p);
    return make_uint4(c.v[0], c.v[1], c.v[2], c.v[3]);
}
// STREAMED: the line is not kept for others to come
template <bool STREAMED = false>
__device__ inline void store_chunk(void* p, uint4 v) {
    typedef uint32_t chunk __attribute__((ext_vector_type(4), aligned(2)));
    const chunk c{v.x, v.y, v.z, v.w};
    if constexpr (STREAMED) __builtin_nontemporal_store(c, reinterpret_cast<chunk*>(p));
    else *reinterpret_cast<chunk*>(p) = c;
}
template <int DT>
__device__ inline float to_float(uint32_t bits16) {
    if constexpr (DT == SC_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
    else return __builtin_bit_cast(float, bits16 << 16);
}
// two values rounded to nearest even, one instruction of gfx950
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <int DT>
__device__ inline uint32_t round2(float lo, float hi) {
    const f32x2 v{lo, hi};
    if constexpr (DT == SC_F16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
template <int DT>
__device__ inline float load_elem(const void* p, int64_t i) {
    if constexpr (DT == SC_F32) return reinterpret_cast<const float*>(p)[i];
    else return to_float<DT>(reinterpret_cast<const uint16_t*>(p)[i]);
}
template <int DT>
__device__ inline void store_elem(void* p, int64_t i, float v) {
    if constexpr (DT == SC_F32) reinterpret_cast<float*>(p)[i] = v;
    else reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)round2<DT>(v, 0.f);
}
// up to eight consecutive elements, those from `count` on are zeros / left alone
template <int DT>
__device__ inline void load8(const void* base, int64_t i, int count, float (&v)[8]) {
    const char* p = reinterpret_cast<const char*>(base) + i * ELEM<DT>;
    if (count >= 8) {
        if constexpr (DT == SC_F32) {
            const uint4 a = load_chunk(p), b = load_chunk(p + 16);
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, w[j]);
        } else {
            const uint4 a = load_chunk(p);
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = to_float<DT>(w[j] & 0xffffu);
                v[2 * j + 1] = to_float<DT>(w[j] >> 16);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < count ? load_elem<DT>(p, j) : 0.f;
    }
}
template <int DT, bool STREAMED = false>
__device__ inline void store8(void* base, int64_t i, int count, const float (&v)[8]) {
    char* p = reinterpret_cast<char*>(base) + i * ELEM<DT>;
    if (count >= 8) {
        if constexpr (DT == SC_F32) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __builtin_bit_cast(uint32_t, v[j]);
            store_chunk<STREAMED>(p, make_uint4(w[0], w[1], w[2], w[3]));
            store_chunk<STREAMED>(p + 16, make_uint4(w[4], w[5], w[6], w[7]));
        } else {
            store_chunk<STREAMED>(p, make_uint4(round2<DT>(v[0], v[1]), round2<DT>(v[2], v[3]), round2<DT>(v[4], v[5]), round2<DT>(v[6], v[7])));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) store_elem<DT>(p, j, v[j]);
    }
}

template <int DT>
__device__ inline void store_row(void* base, int64_t i, const float (&v)[8], bool streamed) {
    if (streamed) {
        asm volatile("; streamed");                    // or the compiler takes the two stores for one
        store8<DT, true>(base, i, 8, v);
        asm volatile("; streamed");
    } else {
        store8<DT>(base, i, 8, v);
    }
}
// eight consecutive elements on their way
template <int DT>
struct Eight {
    uint4 raw[DT == SC_F32 ? 2 : 1];
    __device__ void clear() {
        raw[0] = make_uint4(0, 0, 0, 0);
        if constexpr (DT == SC_F32) raw[1] = make_uint4(0, 0, 0, 0);
    }
    __device__ void load(const void* base, int64_t i) {
        const char* p = reinterpret_cast<const char*>(base) + i * ELEM<DT>;
        raw[0] = load_chunk(p);
        if constexpr (DT == SC_F32) raw[1] = load_chunk(p + 16);
    }
    __device__ void to_floats(float (&v)[8]) const {
        if constexpr (DT == SC_F32) {
            const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __builtin_bit_cast(float, w[j]);
        } else {
            const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = to_float<DT>(w[j] & 0xffffu);
                v[2 * j + 1] = to_float<DT>(w[j] >> 16);
            }
        }
    }
    __device__ void add_to(float (&v)[8]) const {
        float mine[8];
        to_floats(mine);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += mine[j];
    }
};

// ---- activations ------------------------------------------------------------------------------------
// Phi(v) = (1 + erf(v / sqrt 2)) / 2.  32-bit layers: the library's erf.  16-bit ones: Phi(-x) = t (a1 + t (a2 + ...)) exp(-x^2 / 2) with t = 1 / (1 + 0.2975 x) for
// x >= 0, six coefficients fitted by weighted least squares (Lawson's iteration) on [0, 13.5] so that it is off by 4e-7 at most and by 2.2e-5 of itself at most, a twentieth of
// a rounding to f16, wherever the exponential is no smaller than 32 bits hold.  A third of the instructions, and its exponential is the density that the derivative needs.
__device__ inline float gauss_tail(float v, float& density) {          // Phi(-|v|), exp(-v^2 / 2)
    const float t = __builtin_amdgcn_rcpf(fmaf(0.2975f, fminf(fabsf(v), 64.f), 1.f));
    density = __builtin_amdgcn_exp2f(v * v * -0.72134752f);
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, fmaf(t, -0.0817488205f, 0.237007448f), -0.0388572812f), 0.153909454f), 0.110420202f), 0.119268826f);
    return poly * density;
}
template <int DT>
__device__ inline float gauss_cdf(float v, float& density) {
    if constexpr (DT == SC_F32) {
        density = expf(-0.5f * v * v);
        return 0.5f * erfcf(v * -0.70710678f);
    } else {
        const float tail = gauss_tail(v, density);
        return v < 0.f ? tail : 1.f - tail;
    }
}
template <int DT>
__device__ inline float sigmoid(float v) {
    if constexpr (DT == SC_F32) return 1.f / (1.f + expf(-v));
    else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.44269504f));
}
// v times the weight of its activation.  Minus infinity counts as the lowest number: times its weight of zero it is zero, the limit.
template <int DT>
__device__ inline float activate(float v, int act) {
    if (act == SC_ACT_RELU) return v > 0.f || v != v ? v : 0.f;
    if (act == SC_ACT_NONE) return v;
    float density;
    // v Phi(v) = max(v, 0) - |v| Phi(-|v|); beyond 64 the last factor is zero (a NaN is in the density)
    if (DT != SC_F32 && act == SC_ACT_GELU) return fmaf(-fminf(fabsf(v), 64.f), gauss_tail(v, density), fmaxf(v, 0.f));
    const float w = act == SC_ACT_GELU ? gauss_cdf<DT>(v, density) : sigmoid<DT>(v);
    return fmaxf(v, -3.4e38f) * w;                      // a NaN is in w as well
}
template <int DT>
__device__ inline void activate8(float (&v)[8], int act) {       // one look at the kind for all of them
    if (act == SC_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activate<DT>(v[j], SC_ACT_GELU);
    } else if (act == SC_ACT_SILU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activate<DT>(v[j], SC_ACT_SILU);
    } else if (act == SC_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = activate<DT>(v[j], SC_ACT_RELU);
    }
}
template <int DT>
__device__ inline float slope(float v, int act) {
    if (act == SC_ACT_RELU) return v > 0.f || v != v ? 1.f : 0.f;
    if (act == SC_ACT_NONE) return 1.f;
    if (act == SC_ACT_GELU) {
        float density;
        const float w = gauss_cdf<DT>(v, density);
        return density == 0.f ? w : fmaf(v * 0.39894228f, density, w);
    }
    const float s = sigmoid<DT>(v), rest = 1.f - s;
    return s == 0.f || rest == 0.f ? s : s * fmaf(v, rest, 1.f);
}

// ---- which entries a unit of work has -------------------------------------------------------------------
struct Part {
    int g;                         // group, -1: none
    int64_t first, last;           // its entries here
    int parts;                     // of the group
    int64_t slot;                  // DW: of this part among the parts of groups that have several
};
// Unit u of the groups cut into parts of `per` entries; DW: a group without entries is one empty part, since its result is zero.
// Sixty-four groups a step, so a workgroup's search grows with the groups, and a call's with their square where they are short: 131072 rows of 64 f16, forward / rows' / weights' gradient, in 64 groups
// 8.8 / 7.3 / 17 us, 1024 20 / 18 / 40, 8192 0.30 / 0.25 / 0.54 ms, 65536 11 / 9.3 / 22 ms.
// Called by whole wavefronts; the result is in scalar registers.  Starts that do not ascend make parts of wrong entries, never of entries outside [0, n).
template <bool EMPTY_TOO>
__device__ inline Part find_part(const int32_t* __restrict__ starts, int groups, int64_t n, int64_t per, int64_t u) {
    Part p{-1, 0, 0, 1, 0};
    if (starts == nullptr) {
        const int64_t parts = (n + per - 1) / per;
        p.parts = (int)(parts > 1 ? parts : 1);
        if (u >= p.parts || (!EMPTY_TOO && n == 0)) return p;
        p.g = 0;
        p.first = u * per;
        p.last = p.first + per < n ? p.first + per : n;
        p.slot = u;
        return p;
    }
    const int lane = threadIdx.x & 63;
    int64_t base = 0, slots = 0;
    for (int g0 = 0; g0 < groups; g0 += WAVE) {
        const int g = g0 + lane;
        int64_t lo = 0, hi = 0;
        if (g < groups) {
            lo = starts[g];
            hi = starts[g + 1];
            lo = lo < 0 ? 0 : lo > n ? n : lo;
            hi = hi < lo ? lo : hi > n ? n : hi;
        }
        const uint32_t len = (uint32_t)(hi - lo), step = (uint32_t)per;
        int count = (int)(len / step + (len % step != 0));
        if (EMPTY_TOO && g < groups && count == 0) count = 1;
        int upto = count, upto_slots = count > 1 ? count : 0;
#pragma unroll
        for (int d = 1; d < WAVE; d <<= 1) {
            const int other = __shfl_up(upto, d), other_slots = __shfl_up(upto_slots, d);
            if (lane >= d) {
                upto += other;
                upto_slots += other_slots;
            }
        }
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (u < base + total) {
            const uint64_t beyond = __ballot((int64_t)upto + base > u);
            const int at = __builtin_ctzll(beyond);
            p.g = g0 + at;
            p.parts = __builtin_amdgcn_readlane(count, at);
            const int64_t nth = u - base - (__builtin_amdgcn_readlane(upto, at) - p.parts);
            const int64_t first = __builtin_amdgcn_readlane((int)lo, at), end = __builtin_amdgcn_readlane((int)hi, at);
            p.first = first + nth * per;
            p.last = p.first + per < end ? p.first + per : end;
            p.slot = slots + __builtin_amdgcn_readlane(upto_slots, at) - (p.parts > 1 ? p.parts : 0) + nth;
            return p;
        }
        base += total;
        slots += __builtin_amdgcn_readlane(upto_slots, 63);
    }
    return p;
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------
// Stands in for chunks that lie beyond an operand's rows or channels.
__device__ __align__(16) uint4 g_no_chunk;
// Stands in for entries of a list beyond its end.
__device__ int32_t g_no_row = -1;
constexpr int RING = 256;          // bytes of LDS for the rows of a step's entries; two of them for each operand
// 4 bytes per lane from global memory straight into LDS, as load_to_lds does with 16
__device__ inline void load_word_to_lds(const void* src, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(src), "s"(lds) : "m0", "memory");
}

// Where a chunk of a line lies in it: its number, turned by the line's, so that what the LDS hands out in one cycle fills its 64 banks once.
// ALONG: lines are rows of the tile, LINE chunks of the summed axis.  16-byte reads go 16 lanes a cycle, lanes 0-3, 12-15, 20-23 and 24-27 (or the others of 32): one
// chunk of lines 0-3 and 12-15 and the next chunk of lines 4-11.
template <int LINE>
__device__ constexpr int along_turn(int line) {
    if (LINE == 4) return (((line >> 2) ^ (line >> 3)) & 1) * 2 + ((line >> 3) & 1);
    return LINE == 8 ? (line >> 1) & 7 : line & 15;
}
// ACROSS: lines are places on the summed axis, LINE chunks of tile rows.  32 lanes of a 16-bit read take 32 bytes of four lines and of the four that
// are 8 further on, 64 lanes of a 32-bit one 64 bytes of lines 0, 4, 8 and 12.
template <int DT, int LINE>
__device__ constexpr int across_turn(int line) {
    if (DT == SC_F32) return LINE >= 16 ? line & 12 : LINE == 8 ? line & 4 : 0;
    return LINE >= 16 ? 2 * (line & 3) + (line & 8) : LINE == 8 ? (line & 2) + (line & 8) / 2 : (line & 8) / 4;
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) const u32x4* lds_u32x4;
typedef __attribute__((address_space(3))) const uint32_t* lds_uint32;

// LDS addresses from which a lane reads its operands of T blocks of 16 rows, in the first buffer
template <int DT, int LINE, int T, int PARTS>
struct AlongReader {
    uint32_t at[PARTS];
    // row0: the wavefront's first row; chunk0: its set's first chunk; both multiples that leave the turn alone
    __device__ AlongReader(uint32_t tile, int row0, int chunk0) {
        const int i = threadIdx.x & 15, o = (threadIdx.x >> 4) & 3;
        for (int c = 0; c < PARTS; ++c) at[c] = tile + ((row0 + i) * LINE + ((chunk0 + 4 * c + o) ^ along_turn<LINE>(i))) * 16;
    }
    // block t, chunks 4 c .. 4 c + 3, a chunk for each 16 lanes
    __device__ uint4 read(uint32_t buffer, int t, int c) const { return __builtin_bit_cast(uint4, *(lds_u32x4)(at[c] + buffer + t * (16 * LINE * 16))); }
};
template <int DT, int LINE, int T, int PARTS>
struct AcrossReader {
    uint32_t at[T];
    __device__ AcrossReader(uint32_t tile, int col0, int line0) {
        const int i = threadIdx.x & 15, o = (threadIdx.x >> 4) & 3;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if constexpr (DT == SC_F32) {
                const int line = line0 + 4 * o, col = col0 + 16 * t + i;
                at[t] = tile + (line * LINE + ((col >> 2) ^ across_turn<DT, LINE>(line))) * 16 + (col & 3) * 4;
            } else {                        // a lane hands in 4 columns of line i / 4 and gets column i of the four lines
                const int line = line0 + 8 * o + (i >> 2), col = col0 + 16 * t + 4 * (i & 3);
                at[t] = tile + (line * LINE + ((col >> 3) ^ across_turn<DT, LINE>(line))) * 16 + (col & 4) * 2;
            }
        }
    }
    __device__ uint4 read(uint32_t buffer, int t, int c) const {
        const uint32_t p = at[t] + buffer;
        if constexpr (DT == SC_F32) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(lds_uint32)(p + (16 * c + j) * (LINE * 16));
            return make_uint4(v[0], v[1], v[2], v[3]);
        } else {
            uint2 v[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                v[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + (32 * c + 4 * h) * (LINE * 16))));
            return make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
        }
    }
};
template <int DT>
__device__ inline f32x4 multiply(uint4 a, uint4 b, f32x4 c) {
    if constexpr (DT == SC_F32) {
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, x[j]), __builtin_bit_cast(float, y[j]), c, 0, 0, 0);
        return c;
    } else {
        return mfma16x16x32<DT>(a, b, c);
    }
}

// What one thread brings of an operand's tiles: PASSES chunks a step, straight into LDS and from any address that suits their elements.  `end` is where the
// summed axis ends (ALONG: channels, ACROSS: rows of the operand that count), STRIDE how much of it a step takes.  Zeros stand for what lies beyond it: other
// values there, infinities among them, would be in every sum.  Beyond a line's other end they are in sums that are not stored, so there whatever follows in
// memory is read, except behind the operand's last element, where nothing may follow.  WHOLE: lines are whole chunks.
template <int DT, bool ACROSS, int LINES, int LINE, int NTH, int STRIDE, bool WHOLE>
struct Loader {
    static constexpr int PASSES = LINES * LINE / NTH, PER = 16 / ELEM<DT>;
    static_assert(LINES * LINE % NTH == 0 && NTH % LINE == 0, "whole passes of whole lines");
    uint32_t ld, rows;                         // bytes from row to row; rows of the operand
    int64_t first, end;                        // ACROSS: the summed entries; ALONG: first is 0
    const char* base;
    const int32_t* list;                       // ACROSS
    int limit, col0;                           // ACROSS: channels there are, and the tile's first
    const char* ptr[PASSES];                   // of the step that is fetched next; ACROSS with a list: unused
    uint32_t ring;                             // ACROSS with a list: its rows of the steps ahead, in LDS

    __device__ __forceinline__ static int line_of(int i) { return (i * NTH + (int)threadIdx.x) / LINE; }
    __device__ __forceinline__ static int chunk_of(int i) {
        const int line = line_of(i), c = (int)threadIdx.x % LINE;
        return c ^ (ACROSS ? across_turn<DT, LINE>(line) : along_turn<LINE>(line));
    }
    // ALONG: lines are rows begin .. of the operand, or those that the list names from there on.  Beyond the last, and for a row that is none,
    // some other row is read: the results are not used.
    __device__ __forceinline__ void start_along(const int32_t* rows_list, int64_t begin, int64_t stop) {
        first = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            int64_t r = begin + line_of(i);
            if (r >= stop) r = stop - 1;
            if (rows_list != nullptr) r = rows_list[r];
            if (r < 0 || r >= rows) r = 0;
            ptr[i] = base + (uint64_t)(uint32_t)r * ld + chunk_of(i) * 16;
        }
    }
    // ACROSS: the channels of a pass's chunk that there are; a chunk beyond the last reads the first
    __device__ __forceinline__ int channels(int i) const { return limit - (col0 + chunk_of(i) * PER); }
    __device__ __forceinline__ const char* column(int i) const {
        const int channel = col0 + chunk_of(i) * PER;
        return base + (int64_t)(channel < limit ? channel : 0) * ELEM<DT>;
    }
    // ... whose 16 bytes, `offset` bytes from the base, may reach beyond the operand's last element
    __device__ __forceinline__ int64_t extent() const { return (int64_t)(rows - 1) * ld + (int64_t)limit * ELEM<DT>; }
    __device__ __forceinline__ int readable(int i, int64_t offset) const { return WHOLE || offset + 16 <= extent() ? PER : channels(i); }
    __device__ __forceinline__ void start_across() {
        if (list != nullptr) return;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) ptr[i] = column(i) + (uint64_t)(uint32_t)(first + line_of(i)) * ld;
    }
    // The rows of step s, by one wavefront, a step before its chunks are asked for.  They go through LDS like the chunks: in registers the compiler
    // moves them at the end of the loop, and waits for them and for all that was asked for since.
    __device__ __forceinline__ void ask_rows(int s) {
        static_assert(!ACROSS || STRIDE <= WAVE, "a step's rows are one load");
        const int lane = threadIdx.x & 63;
        const int64_t e = first + (int64_t)s * STRIDE + lane;
        load_word_to_lds(lane < STRIDE && e < end ? list + e : &g_no_row, __builtin_amdgcn_readfirstlane(ring + (s & 1) * RING));
    }
    // one chunk of which `there` elements are to be read, PER or more: all
    __device__ __forceinline__ static void bring(const char* p, int there, uint32_t lds, int i) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t pass = lds + i * NTH * 16;
        if (WHOLE || there >= PER || there <= 0) {
            load_to_lds(there > 0 ? (const void*)p : (const void*)&g_no_chunk, __builtin_amdgcn_readfirstlane(pass + wave * 1024));
        } else {
            uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (j < there) {
                    if constexpr (DT == SC_F32) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
                    else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
                }
            *(__attribute__((address_space(3))) u32x4*)(pass + threadIdx.x * 16) = u32x4{w[0], w[1], w[2], w[3]};
        }
    }
    __device__ __forceinline__ void fetch(int s, uint32_t lds) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t from = first + (int64_t)s * STRIDE;
        if (ACROSS && list != nullptr) {
            uint32_t r[PASSES];
#pragma unroll
            for (int i = 0; i < PASSES; ++i) r[i] = *(lds_uint32)(ring + (s & 1) * RING + line_of(i) * 4);
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const char* p = column(i) + (uint64_t)r[i] * ld;
                bring(p, r[i] < rows ? readable(i, p - base) : 0, lds, i);
            }
        } else if (from + STRIDE <= end &&
                   (!ACROSS || WHOLE || (from + STRIDE - 1) * ld + (int64_t)((limit + PER - 1) / PER) * 16 <= extent())) {
            const uint64_t step = ACROSS ? (uint64_t)STRIDE * ld : STRIDE * ELEM<DT>;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                load_to_lds(ptr[i], __builtin_amdgcn_readfirstlane(lds + (i * NTH + wave * 64) * 16));
                ptr[i] += step;
            }
        } else {
            const int left = end > from ? (int)(end - from < STRIDE ? end - from : STRIDE) : 0;
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                if constexpr (ACROSS) {
                    bring(ptr[i], line_of(i) < left ? readable(i, ptr[i] - base) : 0, lds, i);
                    ptr[i] += (uint64_t)STRIDE * ld;
                } else {
                    bring(ptr[i], left - chunk_of(i) * PER, lds, i);
                }
            }
        }
    }
};

// The rows of DX_ACT: gradient and value ahead of the activation come through registers a step ahead, their product goes to LDS and, by the first of the
// workgroups with these rows (`keep`), to memory for the weight gradient that follows.
template <int DT, int LINES, int LINE, int NTH, int STRIDE, bool WHOLE, bool SUMS>
struct GradLoader {
    static constexpr int PASSES = LINES * LINE / NTH, PER = 16 / ELEM<DT>;
    // SUMS: column sums before the rounding, a wavefront's lines the unit
    static constexpr int WAVE_LINES = 64 / LINE, UNIT = PASSES * WAVE_LINES;
    float* sums;                       // of this wavefront's unit, null: none
    const char* grad[PASSES];          // at the next step's chunk
    const char* pre[PASSES];
    char* kept;                        // of pass 0; the others' lines follow `kept_pass` bytes apart
    int64_t kept_pass;
    bool row_ok[PASSES], entry_ok[PASSES];
    uint4 g[PASSES], v[PASSES];
    int depth, act;
    bool keep;

    __device__ __forceinline__ static int line_of(int i) { return (int)(threadIdx.x >> 6) * UNIT + i * WAVE_LINES + (int)(threadIdx.x & 63) / LINE; }
    __device__ __forceinline__ static int chunk_of() { return (int)threadIdx.x % LINE; }
    __device__ __forceinline__ static uint32_t place_of(int i) { return (line_of(i) * LINE + (chunk_of() ^ along_turn<LINE>(line_of(i)))) * 16; }
    __device__ __forceinline__ void start(const Product& p, int g, int64_t begin, int64_t stop) {
        depth = p.K;
        act = p.act;
        if constexpr (SUMS) {
            static_assert(UNIT == 1 << bias_log2(true, LINES == 128 ? TILE_128_32 : LINES == 32 ? TILE_32_64 : TILE_16_32), "units of the rules");
            const int64_t mine = begin + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * UNIT;
            sums = keep && mine < stop ? p.bias_sums + (mine / UNIT + g) * p.K : nullptr;
        }
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int64_t e = begin + line_of(i);
            entry_ok[i] = e < stop;
            const int64_t at = entry_ok[i] ? e : begin;
            const int64_t r = p.a_list != nullptr ? p.a_list[at] : at;
            row_ok[i] = r >= 0 && r < p.a_rows;
            const int offset = chunk_of() * 16;
            grad[i] = (const char*)p.a + (row_ok[i] ? r : 0) * (p.lda * ELEM<DT>) + offset;
            pre[i] = (const char*)p.pre + at * (p.ldp * ELEM<DT>) + offset;
        }
        kept_pass = WAVE_LINES * (p.ldk * ELEM<DT>);
        kept = (char*)p.kept + (begin + line_of(0)) * (p.ldk * ELEM<DT>) + chunk_of() * 16;
    }
    __device__ __forceinline__ static uint4 some(const char* p, int there) {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (j < there) {
                if constexpr (DT == SC_F32) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
                else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void fetch(int s) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int there = depth - s * STRIDE - chunk_of() * PER;
            g[i] = v[i] = make_uint4(0, 0, 0, 0);
            if (there >= PER || (WHOLE && there > 0)) {
                if (row_ok[i]) g[i] = load_chunk(grad[i]);
                v[i] = load_chunk(pre[i]);
            } else if (!WHOLE && there > 0) {
                if (row_ok[i]) g[i] = some(grad[i], there);
                v[i] = some(pre[i], there);
            }
            grad[i] += STRIDE * ELEM<DT>;
            pre[i] += STRIDE * ELEM<DT>;
        }
    }
    // The sums of a wavefront's lines, of which lanes LINE apart have eight columns each: for 8 and 16 lanes a product with ones adds what is 16 lanes apart.
    __device__ __forceinline__ void write_sums(int s, const float (&sum)[8]) const {
        const int lane = threadIdx.x & 63, row = lane >> 4;
        const int col = s * STRIDE + chunk_of() * PER;
        float out[LINE / 8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float v;
            if constexpr (LINE == 32) {
                v = sum[j] + __shfl_xor(sum[j], 32);
                if (j / 4 == lane >> 5) out[j % 4] = v;
            } else {
                v = __builtin_amdgcn_mfma_f32_16x16x4f32(1.f, sum[j], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0)[0];
                if constexpr (LINE == 8) {                   // and the other eight of sixteen
                    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));
                    if (lane >> 3 == j) out[0] = v;
                } else if (row == j % 4) {
                    out[j / 4] = v;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int k = 0; k < LINE / 8; ++k) {
            const int c = col + (LINE == 32 ? 4 * (lane >> 5) + k : LINE == 16 ? 4 * k + row : lane >> 3);
            if (sums != nullptr && c < depth) sums[c] = out[k];
        }
    }
    __device__ __forceinline__ void finish(int s, uint32_t lds) {
        float sum[8];
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int there = depth - s * STRIDE - chunk_of() * PER;
            const uint32_t gw[4] = {g[i].x, g[i].y, g[i].z, g[i].w}, vw[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t w[4];
            float d32[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (DT == SC_F32) {
                    w[j] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, gw[j]) * slope<DT>(__builtin_bit_cast(float, vw[j]), act));
                } else {
                    const float lo = to_float<DT>(gw[j] & 0xffffu) * slope<DT>(to_float<DT>(vw[j] & 0xffffu), act);
                    const float hi = to_float<DT>(gw[j] >> 16) * slope<DT>(to_float<DT>(vw[j] >> 16), act);
                    w[j] = round2<DT>(lo, hi);
                    d32[2 * j] = lo;
                    d32[2 * j + 1] = hi;
                }
            }
            // no row, no channel: zeros, whatever the value ahead of the activation
            const bool some_of_it = row_ok[i] && there > 0;
            const uint4 d = some_of_it ? make_uint4(w[0], w[1], w[2], w[3]) : make_uint4(0, 0, 0, 0);
            if constexpr (SUMS) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float mine = some_of_it && entry_ok[i] ? d32[j] : 0.f;
                    sum[j] = i == 0 ? mine : sum[j] + mine;
                }
                if (i == PASSES - 1) write_sums(s, sum);
                __builtin_amdgcn_sched_barrier(0);         // one pass at a time: registers for four wavefronts
            }
            *(__attribute__((address_space(3))) u32x4*)(lds + place_of(i)) = u32x4{d.x, d.y, d.z, d.w};
            if (keep && entry_ok[i] && there > 0) {
                char* const to = kept + i * kept_pass;
                if (WHOLE || there >= PER) {
                    store_chunk(to, d);
                } else {
                    const uint32_t dw[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
                    for (int j = 0; j < PER; ++j)
                        if (j < there) {
                            if constexpr (DT == SC_F32) reinterpret_cast<uint32_t*>(to)[j] = dw[j];
                            else reinterpret_cast<uint16_t*>(to)[j] = (uint16_t)(dw[j / 2] >> (16 * (j & 1)));
                        }
                }
            }
        }
        kept += STRIDE * ELEM<DT>;
    }
};

// ---- the kernel -----------------------------------------------------------------------------------------
// WM x WN wavefronts share a tile, KW sets of them the summed axis, of which a set takes SB bytes a step.  WHOLE: the operands' lines are whole chunks
// of 16 bytes, at any alignment of their elements (what the others need is in registers through the whole loop: weight gradients 36 us or 29).
// RESIDUAL: there may be one; what is held of it costs the others wavefronts (128 x 128: 174 registers or 123).  DX_ACT: a bias wants the sums of the gradient's columns.
template <int DT, int MODE, int BM_, int BN_, int WM_, int WN_, int KW_, int SB_>
struct ProductShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KW = KW_, SB = SB_;
    static constexpr int NTH = 64 * WM * WN * KW, TM = BM / 16 / WM, TN = BN / 16 / WN;
    static constexpr int STEP = SB / ELEM<DT>;                        // places on the summed axis per set and step
    static constexpr bool A_ACROSS = MODE == PRODUCT_DW, B_ACROSS = MODE == PRODUCT_FWD || MODE == PRODUCT_DW;
    static constexpr int A_LINES = A_ACROSS ? STEP * KW : BM, A_LINE = A_ACROSS ? BM * ELEM<DT> / 16 : SB / 16 * KW;
    static constexpr int B_LINES = B_ACROSS ? STEP * KW : BN, B_LINE = B_ACROSS ? BN * ELEM<DT> / 16 : SB / 16 * KW;
    static constexpr int A_CHUNKS = A_LINES * A_LINE, B_CHUNKS = B_LINES * B_LINE;
    static constexpr int SHARES = MODE == PRODUCT_DW ? NTH * 4 : 0;       // of a bias' sums, a float a thread
    static constexpr int BUFFER = (A_CHUNKS + B_CHUNKS) * 16, RINGS = MODE == PRODUCT_DW ? 4 * RING : 0;
    static constexpr int SUMS = (KW - 1) * WM * WN * TM * TN * 64 * 16;  // what the sets hand over in the end
    static constexpr int PIECES = WM * WN * 16 * (TN * 16 + 4) * 4;      // results on their way out
    static constexpr int lds(int64_t steps) {
        const int buffers = RINGS + (steps > 1 ? 2 : 1) * BUFFER, end = SUMS > PIECES ? SUMS : PIECES;
        return SHARES + (buffers > end ? buffers : end);
    }
};

// entry m names no row of a
__device__ inline bool no_row(const Product& p, int64_t m) {
    const int64_t r = p.a_list != nullptr ? p.a_list[m] : m;
    return r < 0 || r >= p.a_rows;
}

template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, int SB, bool WHOLE, bool RESIDUAL>
__global__ void __launch_bounds__(64 * WM * WN * KW, 2)
k_product(const Product p) {
    using S = ProductShape<DT, MODE, BM, BN, WM, WN, KW, SB>;
    constexpr int NTH = S::NTH, TM = S::TM, TN = S::TN;
    extern __shared__ __align__(16) uint4 all_lds[];
    uint4* const product_lds = all_lds + S::SHARES / 16;

    // runs of consecutive tiles, which share rows, go to one XCD; those that do not exist after all are the last of every XCD
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x, turn = block / NUM_XCD, run = (uint32_t)p.run;
    const uint32_t unit = (turn / run * NUM_XCD + block % NUM_XCD) * run + turn % run;
    const uint32_t n_tiles = (uint32_t)(p.N + BN - 1) / BN;
    uint32_t row_unit;
    int m_tile = 0, n_tile;
    if constexpr (MODE == PRODUCT_DW) {
        const uint32_t m_tiles = p.M > BM ? (uint32_t)(p.M + BM - 1) / BM : 1u;
        row_unit = unit / (m_tiles * n_tiles);
        // bands of four tiles of m, across n: a run of them reads few columns of both sides
        const uint32_t tile = unit - row_unit * (m_tiles * n_tiles), band = tile / (4 * n_tiles), in_band = tile - band * (4 * n_tiles);
        const uint32_t high = m_tiles - 4 * band < 4 ? m_tiles - 4 * band : 4;
        n_tile = (int)(in_band / high);
        m_tile = (int)(4 * band + in_band - n_tile * high);
    } else {
        row_unit = unit / n_tiles;
        n_tile = (int)(unit - row_unit * n_tiles);
    }
    if (row_unit >= p.units) return;
    const Part part = find_part<MODE == PRODUCT_DW>(p.starts, p.groups, p.n, MODE == PRODUCT_DW ? p.per : BM, row_unit);
    const int g = __builtin_amdgcn_readfirstlane(part.g);
    if (g < 0 || (part.parts > 1 && MODE == PRODUCT_DW && part.slot >= p.slots)) return;     // the whole workgroup, before any barrier

    const int lane = threadIdx.x & 63, i = lane & 15, o = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int set = wave / (WM * WN), wm = wave % (WM * WN) / WN, wn = wave % WN;
    const int n0 = n_tile * BN, m0 = m_tile * BM;
    const uint32_t rings = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)product_lds, lds0 = rings + S::RINGS;

    constexpr int STRIDE = S::STEP * KW;
    Loader<DT, S::A_ACROSS, S::A_LINES, S::A_LINE, NTH, STRIDE, WHOLE> la;
    GradLoader<DT, MODE == PRODUCT_DX_ACT ? S::A_LINES : 0, S::A_LINE, NTH, STRIDE, WHOLE, MODE == PRODUCT_DX_ACT && RESIDUAL> lg;
    Loader<DT, S::B_ACROSS, S::B_LINES, S::B_LINE, NTH, STRIDE, WHOLE> lb;
    la.base = (const char*)p.a;
    la.ld = (uint32_t)(p.lda * ELEM<DT>);
    la.rows = (uint32_t)p.a_rows;
    lb.ld = (uint32_t)(p.ldb * ELEM<DT>);
    int64_t depth;                                      // of the summed axis
    int32_t row_of[TM];                                 // rows of a that the lane's results are of
    if constexpr (MODE == PRODUCT_DW) {
        depth = p.M == 0 && p.bias_sums != nullptr ? 0 : part.last - part.first;
        la.list = p.a_list;
        la.ring = rings;
        la.first = part.first;
        la.end = p.a_list != nullptr || p.a_rows > part.last ? part.last : p.a_rows;
        la.limit = p.M;
        la.col0 = m0;
        if (p.M == 0) {                                 // sums of b's rows only: zeros for a
            la.base = (const char*)&g_no_chunk;
            la.ld = 0;
            la.list = nullptr;
            la.end = part.last;
        }
        la.start_across();
        lb.base = (const char*)p.b;
        lb.rows = (uint32_t)p.b_rows;
        lb.list = p.b_list;
        lb.ring = rings + 2 * RING;
        lb.first = part.first;
        lb.end = p.b_list != nullptr || p.b_rows > part.last ? part.last : p.b_rows;
        lb.limit = p.N;
        lb.col0 = n0;
        lb.start_across();
    } else {
        depth = p.a_rows > 0 ? p.K : 0;
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
            const int64_t e = part.first + (wm * TM + tm) * 16 + i;
            row_of[tm] = (int32_t)e;
            if (p.a_list != nullptr && e < part.last) row_of[tm] = p.a_list[e];
        }
        if (depth > 0) {
            if constexpr (MODE == PRODUCT_DX_ACT) {
                lg.keep = n_tile == 0;
                lg.start(p, g, part.first, part.last);
            } else {
                la.list = nullptr;
                la.end = p.K;
                la.start_along(p.a_list, part.first, part.last);
            }
            lb.base = (const char*)p.b + (int64_t)g * p.K * p.N * ELEM<DT>;
            lb.list = nullptr;
            lb.first = 0;
            lb.end = p.K;
            if constexpr (MODE == PRODUCT_FWD) {
                lb.rows = p.K;
                lb.limit = p.N;
                lb.col0 = n0;
                lb.start_across();
            } else {
                lb.rows = p.N;
                lb.start_along(nullptr, n0, p.N);
            }
        }
    }
    const int steps = (int)((depth + STRIDE - 1) / STRIDE);
    auto ask_rows = [&](int s) __attribute__((always_inline)) {
        if constexpr (MODE == PRODUCT_DW) {
            static_assert(WM * WN > 1, "a wavefront for each side's list");
            if (wave == 0 && la.list != nullptr) la.ask_rows(s);
            if (wave == 1 && lb.list != nullptr) lb.ask_rows(s);
        }
    };
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const uint32_t at = lds0 + (s & 1) * S::BUFFER;
        if constexpr (MODE != PRODUCT_DX_ACT) la.fetch(s, at);
        lb.fetch(s, at + S::A_CHUNKS * 16);
        if constexpr (MODE == PRODUCT_DX_ACT) lg.fetch(s);
        ask_rows(s + 1);
    };
    // DX_ACT: what a step's registers hold goes to LDS, and the step is complete
    auto finish = [&](int s) __attribute__((always_inline)) {
        if constexpr (MODE == PRODUCT_DX_ACT) {
            __builtin_amdgcn_s_waitcnt(0x0f70);
            lg.finish(s, lds0 + (s & 1) * S::BUFFER);
        }
    };
    typename std::conditional<S::A_ACROSS, AcrossReader<DT, S::A_LINE, TM, SB / 64>, AlongReader<DT, S::A_LINE, TM, SB / 64>>::type ra(
        lds0, wm * TM * 16, set * (S::A_ACROSS ? S::STEP : SB / 16));
    typename std::conditional<S::B_ACROSS, AcrossReader<DT, S::B_LINE, TN, SB / 64>, AlongReader<DT, S::B_LINE, TN, SB / 64>>::type rb(
        lds0 + S::A_CHUNKS * 16, wn * TN * 16, set * (S::B_ACROSS ? S::STEP : SB / 16));

    f32x4 acc[TM][TN], ones_sum[TN];
#pragma unroll
    for (int tm = 0; tm < TM; ++tm)
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) ones_sum[tn] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool sums = MODE == PRODUCT_DW && p.out_bias != nullptr && p.bias_sums == nullptr && m_tile == 0 && wm == 0;
    const uint32_t one = DT == SC_F32 ? 0x3f800000u : DT == SC_F16 ? 0x3c003c00u : 0x3f803f80u;

    if constexpr (MODE == PRODUCT_DW) {
        if (la.list != nullptr || lb.list != nullptr) {
            ask_rows(0);
            __builtin_amdgcn_s_waitcnt(0x0f70);
            lds_barrier();
        }
    }
    if (steps > 0) {
        fetch(0);
        finish(0);
    }
    // A bias' sums that are there already, by all wavefronts: every so many'th unit of a column, sixteen asked for at a time.
    const bool ready_sums = MODE == PRODUCT_DW && p.out_bias != nullptr && p.bias_sums != nullptr && m_tile == 0;
    if constexpr (MODE == PRODUCT_DW) {
        if (ready_sums) {
            constexpr int SHARES = NTH / BN;
            const int col = n0 + (int)threadIdx.x % BN;
            float share = 0.f;
            if (col < p.N) {
                const float* src = p.bias_sums + ((part.first >> p.bias_log2) + g) * p.N + col;
                const int count = (int)((part.last - part.first + (1 << p.bias_log2) - 1) >> p.bias_log2);
                for (int u = (int)threadIdx.x / BN; u < count; u += 16 * SHARES) {
                    float term[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const uint32_t at = (uint32_t)(u + k * SHARES < count ? u + k * SHARES : u);
                        term[k] = src[(uint64_t)at * (uint32_t)p.N];
                    }
#pragma unroll
                    for (int k = 0; k < 16; ++k) share += u + k * SHARES < count ? term[k] : 0.f;
                }
            }
            reinterpret_cast<float*>(all_lds)[threadIdx.x] = share;
        }
    }
    for (int s = 0; s < steps; ++s) {
        if constexpr (MODE != PRODUCT_DX_ACT) __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0): the step's chunks are in LDS
        lds_barrier();                                 // ... of all wavefronts, which are done with the other buffer
        if (s + 1 < steps) fetch(s + 1);
        const uint32_t buffer = (s & 1) * S::BUFFER;
#pragma unroll
        for (int c = 0; c < SB / 64; ++c) {
            uint4 fa[TM], fb[TN];
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) fb[tn] = rb.read(buffer, tn, c);
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) fa[tm] = ra.read(buffer, tm, c);
#pragma unroll
            for (int tm = 0; tm < TM; ++tm)
#pragma unroll
                for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = multiply<DT>(fb[tn], fa[tm], acc[tm][tn]);
            if constexpr (MODE == PRODUCT_DW) {
                if (sums) {
#pragma unroll
                    for (int tn = 0; tn < TN; ++tn) ones_sum[tn] = multiply<DT>(fb[tn], make_uint4(one, one, one, one), ones_sum[tn]);
                }
            }
        }
        if (s + 1 < steps) finish(s + 1);
    }

    if constexpr (KW > 1) {                            // the sets' sums, in the order of the sets
        float4* sum = reinterpret_cast<float4*>(product_lds);
        constexpr int SHARE = WM * WN * TM * TN * 64;
        lds_barrier();
        if (set > 0) {
#pragma unroll
            for (int tm = 0; tm < TM; ++tm)
#pragma unroll
                for (int tn = 0; tn < TN; ++tn)
                    sum[(set - 1) * SHARE + ((wave % (WM * WN)) * TM * TN + tm * TN + tn) * 64 + lane] =
                        make_float4(acc[tm][tn][0], acc[tm][tn][1], acc[tm][tn][2], acc[tm][tn][3]);
        }
        lds_barrier();
        if (set > 0) return;
#pragma unroll
        for (int other = 0; other < KW - 1; ++other)
#pragma unroll
            for (int tm = 0; tm < TM; ++tm)
#pragma unroll
                for (int tn = 0; tn < TN; ++tn) {
                    const float4 v = sum[other * SHARE + ((wave % (WM * WN)) * TM * TN + tm * TN + tn) * 64 + lane];
                    acc[tm][tn][0] += v.x;
                    acc[tm][tn][1] += v.y;
                    acc[tm][tn][2] += v.z;
                    acc[tm][tn][3] += v.w;
                }
    }

    // A lane has columns 4 o .. 4 o + 3 of every block's 16 and row i.  Two blocks' odd and even rows of lanes change places, and it has eight
    // columns in a row of one block; four lanes have 32 columns of a row.
    constexpr int COLS = TN * 16;
    static_assert(TN % 2 == 0, "blocks by pairs");
    const int col_wave = n0 + wn * COLS;
    const int64_t first_row = (MODE == PRODUCT_DW ? m0 : part.first) + wm * TM * 16, end_row = MODE == PRODUCT_DW ? p.M : part.last;
    const int64_t slot_row = part.slot * (p.M + 1);    // DW, several parts: rows of sums in front of this part's
    const bool to_partial = MODE == PRODUCT_DW && part.parts > 1;
    const void* const bias_row = MODE == PRODUCT_FWD && p.bias != nullptr ? (const char*)p.bias + (int64_t)g * p.N * ELEM<DT> : nullptr;
    // Rows of results are streamed: their lines, written in two halves, otherwise leave the L2 in halves too, a third more of them than there are (10^6 rows 128 -> 128
    // 129 us and 95, which is the rate of a copy; 110545 x 256 -> 256 39.8 and 35.5).  Not where rows start inside a 64-byte half.  Partial sums are not,
    // they are read back at once.
    const int out_size = MODE == PRODUCT_FWD && p.out_f32 ? 4 : ELEM<DT>;
    const bool stream_out = (((uintptr_t)p.out | (uintptr_t)(p.ldo * out_size)) & 63) == 0, stream_pre = (((uintptr_t)p.pre | (uintptr_t)(p.ldp * out_size)) & 63) == 0;
    // Whatever is loaded is asked for ahead of the stores of the columns before: loads and stores are waited for in one order.
    constexpr int PAIRS = TN / 2;
    const int left = (p.N - col_wave) / 32, pairs = left < PAIRS ? (left > 0 ? left : 0) : PAIRS;
    const int whole_cols = 32 * pairs;
    const int col_lane = col_wave + 16 * (o & 1) + 8 * (o >> 1);
    Eight<DT> bias[MODE == PRODUCT_FWD ? PAIRS : 1], add[RESIDUAL ? 2 : 1][RESIDUAL ? TM : 1];
    const bool early = RESIDUAL && p.residual != nullptr && p.out_f32 == 0;
    if constexpr (MODE == PRODUCT_FWD) {
        if (bias_row != nullptr) {
#pragma unroll
            for (int u = 0; u < PAIRS; ++u)
                if (u < pairs) bias[u].load(bias_row, col_lane + 32 * u);
        }
    }
    auto ask = [&](int u) __attribute__((always_inline)) {
        if constexpr (RESIDUAL) {
            if (early && u < pairs) {
#pragma unroll
                for (int tm = 0; tm < TM; ++tm) {
                    const int64_t m = first_row + tm * 16 + i;
                    if (m < end_row) add[u & 1][tm].load(p.residual, m * p.ldr + col_lane + 32 * u);
                }
            }
        }
    };
    ask(0);
#pragma unroll
    for (int u = 0; u < PAIRS; ++u) {
        if (u >= pairs) break;
        if (u + 1 < PAIRS) ask(u + 1);
        const int col = col_lane + 32 * u;
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const auto pair = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, (float)acc[tm][2 * u][j]),
                                                                   __builtin_bit_cast(uint32_t, (float)acc[tm][2 * u + 1][j]), false, false);
                v[j] = __builtin_bit_cast(float, (uint32_t)pair[0]);
                v[4 + j] = __builtin_bit_cast(float, (uint32_t)pair[1]);
            }
            const int64_t m = first_row + tm * 16 + i;
            if (m >= end_row) continue;
            if constexpr (MODE == PRODUCT_DW) {
                if (to_partial) store8<SC_F32>(p.partial, (slot_row + m) * p.N + col, 8, v);
                else store8<DT>(p.out, ((int64_t)g * p.M + m) * p.N + col, 8, v);
            } else {
                if (row_of[tm] < 0 || row_of[tm] >= p.a_rows) {          // no such row: zeros
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = 0.f;
                }
                if constexpr (MODE == PRODUCT_FWD) {
                    if (bias_row != nullptr) bias[u].add_to(v);
                    if (p.pre != nullptr) {
                        if (p.out_f32) store_row<SC_F32>(p.pre, m * p.ldp + col, v, stream_pre);
                        else store_row<DT>(p.pre, m * p.ldp + col, v, stream_pre);
                    }
                    activate8<DT>(v, p.act);
                    if constexpr (RESIDUAL) {
                        if (early) {
                            add[u & 1][tm].add_to(v);
                        } else if (p.residual != nullptr) {
                            Eight<SC_F32> late;
                            late.load(p.residual, m * p.ldr + col);
                            late.add_to(v);
                        }
                    }
                    if (p.out_f32) {
                        store_row<SC_F32>(p.out, m * p.ldo + col, v, stream_out);
                        continue;
                    }
                }
                store_row<DT>(p.out, m * p.ldo + col, v, stream_out);
            }
        }
    }
    // The columns that are left: 16 rows at a time through LDS, a wavefront's own piece of it, up to eight columns a lane; one copy of the code.
    const int rest = p.N - col_wave - whole_cols < COLS - whole_cols ? p.N - col_wave - whole_cols : COLS - whole_cols;
    if constexpr (KW == 1 || WM * WN > 1) lds_barrier();     // the operands, or the sums, have been read by all
    if constexpr (MODE == PRODUCT_DW) {
        const int col = n0 + (int)threadIdx.x;
        if (ready_sums && threadIdx.x < BN && col < p.N) {       // their shares, in order
            float total = 0.f;
#pragma unroll
            for (int k = 0; k < NTH / BN; ++k) total += reinterpret_cast<const float*>(all_lds)[k * BN + threadIdx.x];
            if (to_partial) p.partial[(slot_row + p.M) * p.N + col] = total;
            else store_elem<DT>(p.out_bias, (int64_t)g * p.N + col, total);
        }
    }
    if (rest <= 0 && !sums) return;
    constexpr int PITCH = COLS + 4;
    float* const piece = reinterpret_cast<float*>(product_lds) + (wave % (WM * WN)) * (16 * PITCH);
    if (sums) {
        if (i == 0) {
#pragma unroll
            for (int tn = 0; tn < TN; ++tn)
                *reinterpret_cast<float4*>(piece + 16 * tn + 4 * o) = make_float4(ones_sum[tn][0], ones_sum[tn][1], ones_sum[tn][2], ones_sum[tn][3]);
        }
        asm volatile("" ::: "memory");                 // a wavefront's LDS accesses keep their order
        for (int c = lane; c < COLS && col_wave + c < p.N; c += 64) {
            if (to_partial) p.partial[(slot_row + p.M) * p.N + col_wave + c] = piece[c];
            else store_elem<DT>(p.out_bias, (int64_t)g * p.N + col_wave + c, piece[c]);
        }
        asm volatile("" ::: "memory");
    }
    if (rest <= 0) return;
    const int chunks = (rest + 7) / 8, turn_rows = 64 / chunks, row0 = lane / chunks, c = (lane - row0 * chunks) * 8;
    const int col = col_wave + whole_cols + c, there = rest - c < 8 ? rest - c : 8;
    float bias_late[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) bias_late[j] = 0.f;
    if (bias_row != nullptr) load8<DT>(bias_row, col, there, bias_late);
#pragma unroll 1
    for (int tm = 0; tm < TM; ++tm) {
#pragma unroll
        for (int k = 0; k < TM; ++k)
            if (tm == k) {
#pragma unroll
                for (int tn = 0; tn < TN; ++tn)
                    *reinterpret_cast<float4*>(piece + i * PITCH + 16 * tn + 4 * o) = make_float4(acc[k][tn][0], acc[k][tn][1], acc[k][tn][2], acc[k][tn][3]);
            }
        asm volatile("" ::: "memory");
#pragma unroll 1
        for (int r = row0; r < 16 && row0 < turn_rows; r += turn_rows) {
            const int64_t m = first_row + tm * 16 + r;
            if (m >= end_row) break;
            const float4 lo = *reinterpret_cast<const float4*>(piece + r * PITCH + whole_cols + c), hi = *reinterpret_cast<const float4*>(piece + r * PITCH + whole_cols + c + 4);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            if constexpr (MODE == PRODUCT_DW) {
                if (to_partial) store8<SC_F32>(p.partial, (slot_row + m) * p.N + col, there, v);
                else store8<DT>(p.out, ((int64_t)g * p.M + m) * p.N + col, there, v);
            } else {
                if (no_row(p, m)) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = 0.f;
                }
                if constexpr (MODE == PRODUCT_FWD) {
                    float add[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        v[j] += bias_late[j];
                        add[j] = 0.f;
                    }
                    if (RESIDUAL && p.residual != nullptr) {
                        if (p.out_f32) load8<SC_F32>(p.residual, m * p.ldr + col, there, add);
                        else load8<DT>(p.residual, m * p.ldr + col, there, add);
                    }
                    if (p.pre != nullptr) {
                        if (p.out_f32) store8<SC_F32>(p.pre, m * p.ldp + col, there, v);
                        else store8<DT>(p.pre, m * p.ldp + col, there, v);
                    }
                    activate8<DT>(v, p.act);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += add[j];
                    if (p.out_f32) {
                        store8<SC_F32>(p.out, m * p.ldo + col, there, v);
                        continue;
                    }
                }
                store8<DT>(p.out, m * p.ldo + col, there, v);
            }
        }
        asm volatile("" ::: "memory");
    }
}

// ---- host ----------------------------------------------------------------------------------------------
// The three products for one element type (sc_product_*.hip, one translation unit each).
int launch_product_f32(int mode, const Product& p, int cus, hipStream_t s);
int launch_product_f16(int mode, const Product& p, int cus, hipStream_t s);
int launch_product_bf16(int mode, const Product& p, int cus, hipStream_t s);

template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, int SB, bool WHOLE, bool RESIDUAL>
int start_product(Product p, hipStream_t s) {
    using S = ProductShape<DT, MODE, BM, BN, WM, WN, KW, SB>;
    constexpr auto kernel = k_product<DT, MODE, BM, BN, WM, WN, KW, SB, WHOLE, RESIDUAL>;
    const int64_t n_tiles = (p.N + BN - 1) / BN, m_tiles = MODE == PRODUCT_DW && p.M > BM ? (p.M + BM - 1) / BM : 1;
    if (MODE != PRODUCT_DW) {
        // groups: the tiles that are full, and one that is not of every group that there can be
        p.units = p.starts == nullptr ? (p.n + BM - 1) / BM : p.n / BM + (p.groups < p.n ? p.groups : p.n);
    }
    p.run = (int)product_run(p.units, n_tiles * m_tiles);
    const int64_t turns = NUM_XCD * (int64_t)p.run, blocks = (p.units * n_tiles * m_tiles + turns - 1) / turns * turns;
    if (blocks > INT32_MAX - 2 * GRID_COLUMNS) return SC_EINVAL;
    const dim3 grid((unsigned)grid_columns(blocks), (unsigned)grid_rows(blocks));
    const int64_t depth = MODE == PRODUCT_DW ? p.per : p.K;
    const size_t lds = S::lds((depth + S::STEP * KW - 1) / (S::STEP * KW));
    static bool done[MAX_DEVICES];
    const int rc = allow_lds((const void*)kernel, S::lds(2), done);
    if (rc != SC_OK) return rc;
    SC_LAUNCH(KID_PRODUCT, kernel, grid, dim3(S::NTH), lds, s, p);
    return SC_OK;
}
// TWO: large tiles have a kernel without residual apart.
template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, int SB, bool RESIDUAL>
int start_product(const Product& p, hipStream_t s) {
    constexpr int PER = 16 / ELEM<DT>;
    const bool whole = p.N % PER == 0 && (MODE == PRODUCT_DW ? p.M : p.K) % PER == 0;      // DX: its weights' lines are K long
    const bool along = (MODE == PRODUCT_DX || MODE == PRODUCT_DX_ACT) && p.K % PER == 0;
    return whole || along ? start_product<DT, MODE, BM, BN, WM, WN, KW, SB, true, RESIDUAL>(p, s)
                          : start_product<DT, MODE, BM, BN, WM, WN, KW, SB, false, RESIDUAL>(p, s);
}
template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, int SB = 128, bool TWO = false>
int run_product(const Product& p, hipStream_t s) {
    if constexpr (MODE == PRODUCT_DX_ACT && DT != SC_F32) {
        if (p.bias_sums != nullptr) return start_product<DT, MODE, BM, BN, WM, WN, KW, SB, true>(p, s);
    }
    if constexpr (MODE != PRODUCT_FWD) return start_product<DT, MODE, BM, BN, WM, WN, KW, SB, false>(p, s);
    else if (TWO && p.residual == nullptr) return start_product<DT, MODE, BM, BN, WM, WN, KW, SB, !TWO>(p, s);
    else return start_product<DT, MODE, BM, BN, WM, WN, KW, SB, true>(p, s);
}
// Which tile: row_tile, weight_tile.
template <int DT, int MODE>
int choose_product(const Product& p, int cus, hipStream_t s) {
    if constexpr (MODE == PRODUCT_DW) {
        switch (weight_tile(p.M, p.N)) {
            case WEIGHTS_64_64: return run_product<DT, MODE, 64, 64, 2, 2, 1>(p, s);
            case WEIGHTS_64_128: return run_product<DT, MODE, 64, 128, 2, 2, 1>(p, s);
            case WEIGHTS_128_64: return run_product<DT, MODE, 128, 64, 2, 2, 1>(p, s);
            default: return run_product<DT, MODE, 128, 128, 2, 2, 1>(p, s);
        }
    } else if constexpr (MODE == PRODUCT_DX_ACT) {     // the tiles that act_in_product leaves
        switch (row_tile(p.n, p.starts == nullptr ? 0 : p.groups, p.N, p.K, false, false, cus)) {
            case TILE_16_32: return run_product<DT, MODE, 16, 32, 1, 1, 4>(p, s);
            case TILE_32_64: return run_product<DT, MODE, 32, 64, 2, 2, 2>(p, s);
            default: return run_product<DT, MODE, 128, 32, 4, 1, 1>(p, s);
        }
    } else {
        constexpr bool FWD = MODE == PRODUCT_FWD, WIDE = DT != SC_F32;
        switch (row_tile(p.n, p.starts == nullptr ? 0 : p.groups, p.N, p.K, FWD, WIDE, cus)) {
            case TILE_16_32: return run_product<DT, MODE, 16, 32, 1, 1, 4>(p, s);
            case TILE_16_32_DEEP: return run_product<DT, MODE, 16, 32, 1, 1, 8>(p, s);
            case TILE_32_64: return run_product<DT, MODE, 32, 64, 2, 2, 2>(p, s);
            case TILE_64_64: return run_product<DT, MODE, 64, 64, 2, 2, 1>(p, s);
            case TILE_64_64_DEEP: return run_product<DT, MODE, 64, 64, 2, 2, 2>(p, s);
            case TILE_128_32: return run_product<DT, MODE, 128, 32, 4, 1, 1>(p, s);
            case TILE_128_64: return run_product<DT, MODE, 128, 64, 4, 1, 1, 128, true>(p, s);
            case TILE_128_128_SHORT:
                if constexpr (FWD) return run_product<DT, MODE, 128, 128, 2, 2, 1, 64, true>(p, s);
                break;
            case TILE_LARGE:
                if constexpr (WIDE && FWD) return run_product<DT, MODE, 128, 256, 2, 2, 1, 64, true>(p, s);
                else if constexpr (WIDE) return run_product<DT, MODE, 256, 256, 2, 4, 1, 128, true>(p, s);
                break;
            default: break;
        }
        return run_product<DT, MODE, 128, 128, 2, 2, 1, 128, true>(p, s);
    }
}
template <int DT>
int launch_product(int mode, const Product& p, int cus, hipStream_t s) {
    if (mode == PRODUCT_FWD) return choose_product<DT, PRODUCT_FWD>(p, cus, s);
    if (mode == PRODUCT_DX) return choose_product<DT, PRODUCT_DX>(p, cus, s);
    if (mode == PRODUCT_DX_ACT) return choose_product<DT, PRODUCT_DX_ACT>(p, cus, s);
    return choose_product<DT, PRODUCT_DW>(p, cus, s);
}

}  // namespace sc
