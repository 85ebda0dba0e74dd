// Products of feature rows with weights, and of feature rows with gradient rows: one tile kernel for linear layers and for
// layers whose weights differ by group of rows (sc_linear.hip, sc_grouped.hip).
//
//     FWD   out[p][n] = act(sum_k a[row(p)][k] w[g][k][n] + bias[g][n]) + residual[p][n]     k: C_in,  n: C_out
//     DX    out[p][n] = sum_k a[row(p)][k] w[g][n][k]                                        k: C_out, n: C_in
//     DW    out[g][m][n] = sum_p a[row(p)][m] b[row'(p)][n],  bias[g][n] = sum_p b[row'(p)][n]   p: entries of group g
//
// A workgroup owns a BM x BN tile of the result and walks the summed axis in steps of 128 bytes (KW times that where KW sets of
// wavefronts share the axis).  Both operands pass through LDS, two buffers deep, 16 bytes a lane straight from global memory: the step
// that follows is in flight while one is multiplied.  A tile is stored as it lies in memory, either as rows along the summed axis (a lane's operand
// is then 16 consecutive bytes) or as rows across it (weights in the forward product, both sides of DW), which the transposing LDS
// read turns into operand order on the way to the registers, so nothing is ever re-laid out in memory.  Chunks of 16 bytes are permuted inside a
// line by the line's number so that the lanes of one LDS access meet different banks; the permutation is in the address that a lane
// loads from, because a load into LDS fills it in the order of the lanes.
// The weights' side is the matrix instruction's first operand, so that a lane ends up with consecutive columns of one row; the
// columns are dealt to pairs of 16-column blocks such that there are eight of them: 16 bytes of 16-bit results, a row's 64 bytes by four lanes.
#pragma once

#include "sc_conv.h"

namespace sc {

enum ProductMode { PRODUCT_FWD, PRODUCT_DX, PRODUCT_DW };

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
    const void* bias;
    int act;
    const void* residual;
    int64_t ldr;
    void* pre;
    int64_t ldp;
    void* out;
    int64_t ldo;
    int out_f32;                   // FWD
    void* out_bias;                // DW
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
__device__ inline void store_chunk(void* p, uint4 v) {
    Chunk2 c;
    c.v[0] = v.x; c.v[1] = v.y; c.v[2] = v.z; c.v[3] = v.w;
    *reinterpret_cast<Chunk2*>(p) = c;
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
template <int DT>
__device__ inline void store8(void* base, int64_t i, int count, const float (&v)[8]) {
    char* p = reinterpret_cast<char*>(base) + i * ELEM<DT>;
    if (count >= 8) {
        if constexpr (DT == SC_F32) {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = __builtin_bit_cast(uint32_t, v[j]);
            store_chunk(p, make_uint4(w[0], w[1], w[2], w[3]));
            store_chunk(p + 16, make_uint4(w[4], w[5], w[6], w[7]));
        } else {
            store_chunk(p, make_uint4(round2<DT>(v[0], v[1]), round2<DT>(v[2], v[3]), round2<DT>(v[4], v[5]), round2<DT>(v[6], v[7])));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) store_elem<DT>(p, j, v[j]);
    }
}

// ---- activations ------------------------------------------------------------------------------------
// Phi(v) = (1 + erf(v / sqrt 2)) / 2.  32-bit layers: the library's erf.  16-bit ones: the rational approximation 7.1.26 of Abramowitz and
// Stegun, erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2) with t = 1 / (1 + 0.3275911 x) for x >= 0, off by 1.5e-7 at most, far below a rounding
// to 16 bits; a third of the instructions, and its exponential is the density that the derivative needs.
__device__ inline float gauss_tail(float v, float& density) {          // Phi(-|v|), exp(-v^2 / 2)
    const float x = fabsf(v) * 0.70710678f;
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, x, 1.f));
    density = __builtin_amdgcn_exp2f(v * v * -0.72134752f);
    const float poly = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return 0.5f * poly * density;
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
    const float w = act == SC_ACT_GELU ? gauss_cdf<DT>(v, density) : sigmoid<DT>(v);
    return fmaxf(v, -3.4e38f) * w;                      // a NaN is in w as well
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
    int64_t group_slot;            // of the group's first part
};
// Unit u of the groups cut into parts of `per` entries; DW: a group without entries is one empty part, since its result is zero.
// Called by whole wavefronts.  Starts that do not ascend make parts of wrong entries, never of entries outside [0, n).
template <bool EMPTY_TOO>
__device__ inline Part find_part(const int32_t* __restrict__ starts, int groups, int64_t n, int64_t per, int64_t u) {
    Part p{-1, 0, 0, 1, 0, 0};
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
        const int total = __shfl(upto, 63);
        if (u < base + total) {
            const uint64_t beyond = __ballot((int64_t)upto + base > u);
            const int at = __builtin_ctzll(beyond);
            p.g = g0 + at;
            p.parts = __shfl(count, at);
            const int64_t nth = u - base - (__shfl(upto, at) - p.parts);
            const int64_t first = __shfl((int)lo, at), end = __shfl((int)hi, at);
            p.first = first + nth * per;
            p.last = p.first + per < end ? p.first + per : end;
            p.group_slot = slots + __shfl(upto_slots, at) - (p.parts > 1 ? p.parts : 0);
            p.slot = p.group_slot + nth;
            return p;
        }
        base += total;
        slots += __shfl(upto_slots, 63);
    }
    return p;
}

// ---- tiles in LDS ---------------------------------------------------------------------------------------
// Stands in for chunks that lie beyond an operand's rows or channels.
__device__ __align__(16) uint4 g_no_chunk;

// ALONG: lines are rows of the tile, LINE chunks of the summed axis.  A lane's operand is one chunk of one line.
template <int LINE>
__device__ constexpr int along_turn(int line) { return LINE == 8 ? (line >> 1) & 7 : line & 7; }
// ACROSS: lines are places on the summed axis, LINE chunks of tile rows.  A 16-bit read takes 8 bytes from each of four lines and four
// chunks, a 32-bit one words of lines four apart.
template <int DT, int LINE>
__device__ constexpr int across_turn(int line) {
    if (DT == SC_F32) return LINE >= 16 ? ((line >> 2) & 1) | (line & 8) : LINE >= 8 ? (line >> 2) & 1 : 0;
    return LINE >= 16 ? 4 * (line & 3) : LINE == 8 ? 4 * ((line >> 1) & 1) : 0;
}

// Row or column `i` (0..15) of block t of a wavefront's share: blocks of 16 in a row, or DEALT by pairs so that a result's lane has
// eight consecutive ones.
template <bool DEALT>
__device__ constexpr int place(int t, int i) { return DEALT ? 32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3) : 16 * t + i; }

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) const char* lds_bytes;

// the operand of lane (i = lane % 16, o = lane / 16) for block t and chunks 4 s .. 4 s + 3 of the summed axis (from chunk or line `at0` on)
template <int DT, int LINE, bool DEALT>
__device__ inline uint4 operand_along(const uint4* tile, int row0, int t, int chunk0, int s, int i, int o) {
    const int line = row0 + place<DEALT>(t, i), c = chunk0 + 4 * s + o;
    return tile[line * LINE + (c ^ along_turn<LINE>(line))];
}
template <int DT, int LINE, bool DEALT>
__device__ inline uint4 operand_across(const uint4* tile, int col0, int t, int line0, int s, int i, int o) {
    if constexpr (DT == SC_F32) {
        const int col = col0 + place<DEALT>(t, i);
        uint32_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int line = line0 + 16 * s + 4 * o + j;
            v[j] = reinterpret_cast<const uint32_t*>(tile)[(line * LINE + ((col >> 2) ^ across_turn<DT, LINE>(line))) * 4 + (col & 3)];
        }
        return make_uint4(v[0], v[1], v[2], v[3]);
    } else {
        // lane i hands in 4 columns of line i / 4 and gets column i of the four lines
        const int col = col0 + place<DEALT>(t, 4 * (i & 3));
        uint2 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int line = line0 + 32 * s + 8 * o + 4 * h + (i >> 2);
            const char* p = reinterpret_cast<const char*>(tile + line * LINE + ((col >> 3) ^ across_turn<DT, LINE>(line))) + (col & 4) * 2;
            v[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(lds_bytes)p));
        }
        return make_uint4(v[0].x, v[0].y, v[1].x, v[1].y);
    }
}
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

// What the chunks that one thread brings of a tile have in common over the steps.  PASSES chunks each, `LINES` lines.
template <int DT, bool ACROSS, int LINES, int LINE, int NTH, bool WHOLE>
struct Loader {
    static constexpr int PASSES = LINES * LINE / NTH, PER = 16 / ELEM<DT>;
    static_assert(LINES * LINE % NTH == 0 && NTH % LINE == 0, "whole passes of whole lines");
    const char* base;
    int64_t ld, rows, last;        // bytes from row to row; rows of the operand; ACROSS: end of the entries
    const int32_t* list;
    int limit, col0;               // channels there are; ACROSS: first of them here
    const char* row[ACROSS ? 1 : PASSES];      // ALONG: the lines' rows, null: none
    int32_t at[ACROSS ? PASSES : 1];           // ACROSS: rows of the step that is loaded next, negative: none
    uint4 held[WHOLE ? 1 : PASSES];

    __device__ static int line_of(int i) { return (i * NTH + (int)threadIdx.x) / LINE; }
    __device__ static int chunk_of(int i) {
        const int line = line_of(i), c = (int)threadIdx.x % LINE;
        return c ^ (ACROSS ? across_turn<DT, LINE>(line) : along_turn<LINE>(line));
    }
    // ALONG: rows first .. of the operand, or of the list
    __device__ void rows_along(int64_t first, int64_t end) {
        if constexpr (!ACROSS) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int64_t e = first + line_of(i);
                int64_t r = e < end ? e : -1;
                if (r >= 0 && list != nullptr) r = list[e];
                row[i] = r >= 0 && r < rows ? base + r * ld : nullptr;
            }
        }
    }
    // ACROSS: the rows of the lines of the step that starts at entry `first`
    __device__ void rows_across(int64_t first) {
        if constexpr (ACROSS) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) {
                const int64_t e = first + line_of(i);
                at[i] = e < last ? (int32_t)e : -1;
                // not looked at before it is used, a step later: a comparison here would wait for it, and for the chunks ahead of it
                if (list != nullptr && e < last) at[i] = list[e];
            }
        }
    }
    // ALONG: `k` is the step's first channel
    __device__ void fetch(int k, uint32_t lds) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int channel = (ACROSS ? col0 : k) + chunk_of(i) * PER;
            const char* line;
            bool ok;
            if constexpr (ACROSS) {
                ok = at[i] >= 0 && at[i] < rows;
                line = base + (int64_t)(ok ? at[i] : 0) * ld;
            } else {
                ok = row[i] != nullptr;
                line = row[i];
            }
            const char* p = line + (int64_t)channel * ELEM<DT>;
            if constexpr (WHOLE) {         // channels are whole chunks
                const void* src = ok && channel < limit ? (const void*)p : (const void*)&g_no_chunk;
                load_to_lds(src, __builtin_amdgcn_readfirstlane(lds + (i * NTH + wave * 64) * 16));
            } else {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (ok && channel + PER <= limit) {
                    v = load_chunk(p);
                } else if (ok) {
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < PER; ++j)
                        if (channel + j < limit) {
                            if constexpr (DT == SC_F32) w[j] = reinterpret_cast<const uint32_t*>(p)[j];
                            else w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[j] << (16 * (j & 1));
                        }
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
                held[i] = v;
            }
        }
    }
    __device__ void put(uint4* tile) {
        if constexpr (!WHOLE) {
#pragma unroll
            for (int i = 0; i < PASSES; ++i) tile[i * NTH + threadIdx.x] = held[i];
        }
    }
};

// ---- the kernel -----------------------------------------------------------------------------------------
// WM x WN wavefronts share a tile, KW sets of them the summed axis.  WHOLE: rows and channels are whole chunks of 16 bytes, aligned;
// otherwise chunks pass through registers, by unaligned loads, element by element at the end of a row.
template <int DT, int MODE, int BM_, int BN_, int WM_, int WN_, int KW_>
struct ProductShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, KW = KW_;
    static constexpr int NTH = 64 * WM * WN * KW, TM = BM / 16 / WM, TN = BN / 16 / WN;
    static constexpr int STEP = 128 / ELEM<DT>;                       // places on the summed axis per set and step
    static constexpr bool A_ACROSS = MODE == PRODUCT_DW, B_ACROSS = MODE != PRODUCT_DX;
    static constexpr int A_LINES = A_ACROSS ? STEP * KW : BM, A_LINE = A_ACROSS ? BM * ELEM<DT> / 16 : 8 * KW;
    static constexpr int B_LINES = B_ACROSS ? STEP * KW : BN, B_LINE = B_ACROSS ? BN * ELEM<DT> / 16 : 8 * KW;
    static constexpr int A_CHUNKS = A_LINES * A_LINE, B_CHUNKS = B_LINES * B_LINE;
    static constexpr int BUFFER = (A_CHUNKS + B_CHUNKS) * 16;
    static constexpr int SUMS = (KW - 1) * WM * WN * TM * TN * 64 * 16;  // what the sets hand over in the end
    static constexpr int lds(bool several_steps) { return (several_steps ? 2 : 1) * BUFFER > SUMS ? (several_steps ? 2 : 1) * BUFFER : SUMS; }
};

template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, bool WHOLE>
__global__ void __launch_bounds__(64 * WM * WN * KW)
k_product(const Product p) {
    using S = ProductShape<DT, MODE, BM, BN, WM, WN, KW>;
    constexpr int NTH = S::NTH, TM = S::TM, TN = S::TN;
    constexpr bool DEALT = TN % 2 == 0;
    extern __shared__ __align__(16) uint4 product_lds[];

    const int64_t unit = xcd_unit(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
    const int n_tiles = (p.N + BN - 1) / BN;
    int64_t row_unit;
    int m_tile = 0, n_tile;
    if constexpr (MODE == PRODUCT_DW) {
        const int m_tiles = p.M > BM ? (p.M + BM - 1) / BM : 1;
        row_unit = unit / (m_tiles * n_tiles);
        const int tile = (int)(unit - row_unit * (m_tiles * n_tiles));
        m_tile = tile / n_tiles;
        n_tile = tile - m_tile * n_tiles;
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
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)product_lds;

    Loader<DT, S::A_ACROSS, S::A_LINES, S::A_LINE, NTH, WHOLE> la;
    Loader<DT, S::B_ACROSS, S::B_LINES, S::B_LINE, NTH, WHOLE> lb;
    la.base = (const char*)p.a;
    la.ld = p.lda * ELEM<DT>;
    la.rows = p.a_rows;
    la.list = p.a_list;
    la.last = part.last;
    la.limit = MODE == PRODUCT_DW ? p.M : p.K;
    la.col0 = m0;
    lb.ld = p.ldb * ELEM<DT>;
    lb.col0 = n0;
    int64_t depth;                                      // of the summed axis
    if constexpr (MODE == PRODUCT_DW) {
        lb.base = (const char*)p.b;
        lb.rows = p.b_rows;
        lb.list = p.b_list;
        lb.last = part.last;
        lb.limit = p.N;
        depth = part.last - part.first;
        la.rows_across(part.first);
        lb.rows_across(part.first);
    } else {
        lb.base = (const char*)p.b + (int64_t)g * p.K * p.N * ELEM<DT>;
        lb.list = nullptr;
        depth = p.K;
        la.rows_along(part.first, part.last);
        if constexpr (MODE == PRODUCT_FWD) {
            lb.rows = p.K;
            lb.last = p.K;
            lb.limit = p.N;
            lb.rows_across(0);
        } else {
            lb.rows = p.N;
            lb.limit = p.K;
            lb.rows_along(n0, p.N);
        }
    }
    constexpr int STRIDE = S::STEP * KW;
    const int steps = (int)((depth + STRIDE - 1) / STRIDE);
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const uint32_t at = lds0 + (s & 1) * S::BUFFER;
        la.fetch(s * STRIDE, at);
        lb.fetch(s * STRIDE, at + S::A_CHUNKS * 16);
        if constexpr (S::A_ACROSS) la.rows_across(part.first + (int64_t)(s + 1) * STRIDE);
        if constexpr (S::B_ACROSS) lb.rows_across((MODE == PRODUCT_DW ? part.first : 0) + (int64_t)(s + 1) * STRIDE);
    };
    auto put = [&](int s) __attribute__((always_inline)) {
        uint4* at = product_lds + (s & 1) * (S::BUFFER / 16);
        la.put(at);
        lb.put(at + S::A_CHUNKS);
    };

    f32x4 acc[TM][TN], ones_sum[TN];
#pragma unroll
    for (int tm = 0; tm < TM; ++tm)
#pragma unroll
        for (int tn = 0; tn < TN; ++tn) acc[tm][tn] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int tn = 0; tn < TN; ++tn) ones_sum[tn] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bool sums = MODE == PRODUCT_DW && p.out_bias != nullptr && m_tile == 0 && wm == 0;
    const uint32_t one = DT == SC_F32 ? 0x3f800000u : DT == SC_F16 ? 0x3c003c00u : 0x3f803f80u;

    if (steps > 0) {
        fetch(0);
        put(0);
    }
    for (int s = 0; s < steps; ++s) {
        if constexpr (WHOLE) __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0): the step's chunks are in LDS
        lds_barrier();                                 // ... of all wavefronts, which are done with the other buffer
        if (s + 1 < steps) fetch(s + 1);
        const uint4* ta = product_lds + (s & 1) * (S::BUFFER / 16);
        const uint4* tb = ta + S::A_CHUNKS;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            uint4 fa[TM], fb[TN];
#pragma unroll
            for (int tn = 0; tn < TN; ++tn) {
                if constexpr (S::B_ACROSS) fb[tn] = operand_across<DT, S::B_LINE, DEALT>(tb, wn * TN * 16, tn, set * S::STEP, c, i, o);
                else fb[tn] = operand_along<DT, S::B_LINE, DEALT>(tb, wn * TN * 16, tn, set * 8, c, i, o);
            }
#pragma unroll
            for (int tm = 0; tm < TM; ++tm) {
                if constexpr (S::A_ACROSS) fa[tm] = operand_across<DT, S::A_LINE, false>(ta, wm * TM * 16, tm, set * S::STEP, c, i, o);
                else fa[tm] = operand_along<DT, S::A_LINE, false>(ta, wm * TM * 16, tm, set * 8, c, i, o);
            }
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
        if (s + 1 < steps) put(s + 1);
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

    // A lane has columns 4 o .. 4 o + 3 of every block's 16 and row i: eight in a row from two blocks.
    constexpr int PAIRS = DEALT ? TN / 2 : TN, WIDTH = DEALT ? 8 : 4;
    const int col_lane = n0 + wn * TN * 16 + WIDTH * o;
#pragma unroll
    for (int u = 0; u < PAIRS; ++u) {
        const int col = col_lane + (DEALT ? 32 : 16) * u;
        const int there = p.N - col < WIDTH ? p.N - col : WIDTH;
        if (there <= 0) continue;
        float bias[8];
        if constexpr (MODE == PRODUCT_FWD) {
#pragma unroll
            for (int j = 0; j < 8; ++j) bias[j] = 0.f;
            if (p.bias != nullptr) load8<DT>(p.bias, (int64_t)g * p.N + col, there, bias);
        }
        if constexpr (MODE == PRODUCT_DW) {
            if (sums && i == 0) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = j < WIDTH ? ones_sum[DEALT ? 2 * u + (j >> 2) : u][j & 3] : 0.f;
                if (part.parts > 1) store8<SC_F32>(p.partial, (part.slot * (p.M + 1) + p.M) * p.N + col, there, v);
                else store8<DT>(p.out_bias, (int64_t)g * p.N + col, there, v);
            }
        }
#pragma unroll
        for (int tm = 0; tm < TM; ++tm) {
            const int r = wm * TM * 16 + tm * 16 + i;
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < WIDTH ? acc[tm][DEALT ? 2 * u + (j >> 2) : u][j & 3] : 0.f;
            if constexpr (MODE == PRODUCT_DW) {
                const int m = m0 + r;
                if (m >= p.M) continue;
                if (part.parts > 1) store8<SC_F32>(p.partial, (part.slot * (p.M + 1) + m) * p.N + col, there, v);
                else store8<DT>(p.out, ((int64_t)g * p.M + m) * p.N + col, there, v);
            } else {
                const int64_t e = part.first + r;
                if (e >= part.last) continue;
                if constexpr (MODE == PRODUCT_FWD) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] += bias[j];
                    if (p.pre != nullptr) {
                        if (p.out_f32) store8<SC_F32>(p.pre, e * p.ldp + col, there, v);
                        else store8<DT>(p.pre, e * p.ldp + col, there, v);
                    }
                    if (p.act != SC_ACT_NONE) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = activate<DT>(v[j], p.act);
                    }
                    if (p.residual != nullptr) {
                        float add[8];
                        if (p.out_f32) load8<SC_F32>(p.residual, e * p.ldr + col, there, add);
                        else load8<DT>(p.residual, e * p.ldr + col, there, add);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] += add[j];
                    }
                    if (p.out_f32) {
                        store8<SC_F32>(p.out, e * p.ldo + col, there, v);
                        continue;
                    }
                }
                store8<DT>(p.out, e * p.ldo + col, there, v);
            }
        }
    }
}

// ---- host ----------------------------------------------------------------------------------------------
// The three products for one element type (sc_product_*.hip, one translation unit each).
int launch_product_f32(int mode, const Product& p, bool whole, int cus, hipStream_t s);
int launch_product_f16(int mode, const Product& p, bool whole, int cus, hipStream_t s);
int launch_product_bf16(int mode, const Product& p, bool whole, int cus, hipStream_t s);

template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW, bool WHOLE>
int run_product(Product p, hipStream_t s) {
    using S = ProductShape<DT, MODE, BM, BN, WM, WN, KW>;
    const int64_t n_tiles = (p.N + BN - 1) / BN, m_tiles = MODE == PRODUCT_DW && p.M > BM ? (p.M + BM - 1) / BM : 1;
    if (MODE != PRODUCT_DW) {
        const int64_t tails = p.starts == nullptr ? 1 : p.groups < p.n ? p.groups : p.n;
        p.units = p.n / BM + tails;                    // a tile that is not full per group, and those that are
    }
    const int64_t blocks = (p.units * n_tiles * m_tiles + NUM_XCD - 1) / NUM_XCD * NUM_XCD;
    if (blocks > INT32_MAX) return SC_EINVAL;
    const dim3 grid((unsigned)grid_columns(blocks), (unsigned)grid_rows(blocks));
    const int64_t depth = MODE == PRODUCT_DW ? p.per : p.K;
    const size_t lds = S::lds(depth > S::STEP * KW);
    static bool done[MAX_DEVICES];
    const int rc = allow_lds((const void*)k_product<DT, MODE, BM, BN, WM, WN, KW, WHOLE>, S::lds(true), done);
    if (rc != SC_OK) return rc;
    SC_LAUNCH(KID_PRODUCT, (k_product<DT, MODE, BM, BN, WM, WN, KW, WHOLE>), grid, dim3(S::NTH), lds, s, p);
    return SC_OK;
}
template <int DT, int MODE, int BM, int BN, int WM, int WN, int KW>
int run_product(const Product& p, bool whole, hipStream_t s) {
    return whole ? run_product<DT, MODE, BM, BN, WM, WN, KW, true>(p, s) : run_product<DT, MODE, BM, BN, WM, WN, KW, false>(p, s);
}
// Which tile: product_tile.
template <int DT, int MODE>
int choose_product(const Product& p, bool whole, int cus, hipStream_t s) {
    (void)cus;
    if constexpr (MODE == PRODUCT_DW) {
        switch (weight_tile(p.M, p.N)) {
            case 64: return run_product<DT, MODE, 64, 64, 2, 2, 1>(p, whole, s);
            default: return run_product<DT, MODE, 128, 128, 2, 2, 1>(p, whole, s);
        }
    } else {
        switch (row_tile(p.n, p.starts == nullptr ? 1 : p.groups, p.N, p.K)) {
            case ROWS_FEW: return run_product<DT, MODE, 16, 64, 1, 1, 4>(p, whole, s);
            case COLUMNS_32: return run_product<DT, MODE, 128, 32, 4, 1, 1>(p, whole, s);
            case COLUMNS_64: return run_product<DT, MODE, 128, 64, 4, 1, 1>(p, whole, s);
            default: return run_product<DT, MODE, 128, 128, 2, 2, 1>(p, whole, s);
        }
    }
}
template <int DT>
int launch_product(int mode, const Product& p, bool whole, int cus, hipStream_t s) {
    if (mode == PRODUCT_FWD) return choose_product<DT, PRODUCT_FWD>(p, whole, cus, s);
    if (mode == PRODUCT_DX) return choose_product<DT, PRODUCT_DX>(p, whole, cus, s);
    return choose_product<DT, PRODUCT_DW>(p, whole, cus, s);
}

}  // namespace sc
