// Norm and rotation of queries and keys, forward and backward.
//
//     n = v / sqrt(mean(v^2) + eps) gain,    (n_a, n_b) -> (n_a cos t - n_b sin t, n_a sin t + n_b cos t),    t = pos[axis(j)] f_j
//     backward: d = the gradient turned by -t,  u = d gain,  w = v / rms,
//     dv = (u - w mean(u w)) / rms,   dgain = sum over rows and heads of d w
//
// Everything is read once and written once, so memory is the bound.  A lane holds eight pairs of a head (16 bytes of each side of
// them, or 32 bytes in a row), a group of lanes a whole head, so the mean is a few exchanges between neighbouring lanes and nothing passes through
// LDS.  A group of lanes takes several heads of one row at a time: their loads are in flight together and the row's angles are
// made once for them.  Angles are counted in turns: a coordinate times a frequency of 48 bits, of which the whole turns are
// dropped before the sine, so a coordinate of 65534 is as exact as one of 1.
// 261574 rows of 8 + 8 heads of 32, bf16: 540 MB in 108 to 116 us, 4.7 to 5.0 TB/s, the rate of a copy (heads at a time 4 / 2 / 1: 108 / 109 / 130); backward 110545
// rows of 8 + 2 heads of 64, f16: 425 MB in 94 us, 4.5 TB/s (2 / 1 at a time 97 / 116; four hold too many registers), and 5 us for the gains.
// Stores past the caches were slower (119 and 166).
#include "sc_heads.h"
#include "sc_product.h"

namespace sc {
namespace {

constexpr int PAIRS_A_LANE = 8;
constexpr int ROPE_THREADS = 256;

struct PairTurn {                      // of the table: turns per unit of the axis' coordinate = high + low
    float high, low;
    int axis, unused;
};
static_assert(sizeof(PairTurn) == 16, "one load");

struct Heads {
    char* data;
    int64_t row, head;                 // bytes
    int heads;
};
struct Rope {
    Heads in[2], out[2], grad[2];      // queries, keys; forward: in -> out, backward: in, grad -> out
    const void* gain[2];
    float* partial[2];                 // backward: [workgroup][D], null: not wanted
    int blocks[2];                     // workgroups of each; queries' first
    int64_t rows;
    const int32_t* pos;
    int64_t ld_pos;
    int axes, D;
    const PairTurn* table;
    float eps;
    int lanes_log2;                    // lanes of a head
};

struct RopeSections {
    int pairs[SC_AXES_MAX];
};
__global__ void __launch_bounds__(512)
k_rope_table(PairTurn* __restrict__ table, int half, int axes, RopeSections sections, double base) {
    const int j = threadIdx.x;
    if (j >= half) return;
    PairTurn t{0.f, 0.f, 0, 0};
    int first = 0;
    for (int a = 0; a < axes; ++a) {
        const int i = j - first, m = sections.pairs[a];
        if (i >= 0 && i < m) {
            const double turns = pow(base, -(double)i / (double)m) * 0.15915494309189533577;
            t.high = (float)turns;
            t.low = (float)(turns - (double)t.high);
            t.axis = a;
        }
        first += m;
    }
    table[j] = t;
}

// cos and sin of one pair's angle
template <int DT>
__device__ inline void turn_of(const PairTurn& t, float at, float& c, float& s) {
    const float x = fmaf(at, t.low, fmaf(at, t.high, -rintf(at * t.high)));      // the whole turns leave an exact product
    if constexpr (DT == SC_F32) {
        sincospif(2.f * x, &s, &c);
    } else {                                            // the hardware's, in turns: off by about 1e-6, a rounding to 16 bits is 2^-9 or 2^-12
        s = __builtin_amdgcn_sinf(x);
        c = __builtin_amdgcn_cosf(x);
    }
}

// A lane's eight pairs of one head: a[i], b[i].  It takes chunk c (of eight channels) of the lower half of the head's lanes' and the one as many further on as
// the head has lanes, or (halves) pairs 8 c .. 8 c + 7 with their partners, so that the lanes of a head read consecutive chunks.
// Its channels on their way: two chunks.  WHOLE: they are whole.
template <int DT, bool WHOLE>
struct Pairs {
    Eight<DT> raw[WHOLE ? 2 : 1];
    float parts[WHOLE ? 1 : 2][8];
    __device__ void clear() {
        if constexpr (WHOLE) {
            raw[0].clear();
            raw[1].clear();
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) parts[0][i] = parts[1][i] = 0.f;
        }
    }
    // channels at and at2 on, of the `count` and `count2` that there are
    __device__ void load(const char* head, int at, int count, int at2, int count2) {
        if constexpr (WHOLE) {
            raw[0].load(head, at);
            if (count2 > 0) raw[1].load(head, at2);
            else raw[1].clear();
        } else {
            load8<DT>(head, at, count, parts[0]);
            load8<DT>(head, at2, count2, parts[1]);
        }
    }
    template <bool ADJACENT>
    __device__ void take(float (&a)[8], float (&b)[8]) const {
        float v[2][8];
        if constexpr (WHOLE) {
            raw[0].to_floats(v[0]);
            raw[1].to_floats(v[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[0][i] = parts[0][i];
                v[1][i] = parts[1][i];
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = ADJACENT ? v[i >> 2][(2 * i) & 7] : v[0][i];
            b[i] = ADJACENT ? v[i >> 2][(2 * i + 1) & 7] : v[1][i];
        }
    }
};
template <int DT, bool ADJACENT, bool WHOLE>
__device__ inline void store_pairs(char* head, int at, int count, int at2, int count2, const float (&a)[8], const float (&b)[8]) {
    float v[2][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (ADJACENT) {
            v[i >> 2][(2 * i) & 7] = a[i];
            v[i >> 2][(2 * i + 1) & 7] = b[i];
        } else {
            v[0][i] = a[i];
            v[1][i] = b[i];
        }
    }
    store8<DT>(head, at, WHOLE ? 8 : count, v[0]);
    if (!WHOLE || count2 > 0) store8<DT>(head, at2, WHOLE ? 8 : count2, v[1]);
}
template <int CONTROL>
__device__ inline float from_lane(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true)); }
// The sum over 2^log2 neighbouring lanes, the same bits in all of them.
__device__ inline float sum_of_lanes(float v, int log2) {
    if (log2 > 0) v += from_lane<0xb1>(v);             // the other of two, the other two of four
    if (log2 > 1) v += from_lane<0x4e>(v);
    if (log2 > 2) v += from_lane<0x141>(v);            // mirrored in 8 and in 16 lanes: fours, and then eights, are alike by now
    if (log2 > 3) v += from_lane<0x140>(v);
    if (log2 > 4) v += __shfl_xor(v, 16);
    if (log2 > 5) v += __shfl_xor(v, 32);
    return v;
}

// How heads divide into chunks: evenly; with a last chunk that reaches back over the one before it (both lanes come to the same values and store them, one
// of them counts them in the sums); or there is not one whole chunk.
enum HeadShape { HEAD_EVEN, HEAD_OVERLAP, HEAD_SMALL };
template <int DT, bool ADJACENT, bool BACKWARD, int TOGETHER, int SHAPE>
__global__ void __launch_bounds__(ROPE_THREADS)
k_rope(const Rope p) {
    const int which = blockIdx.x < (unsigned)p.blocks[0] ? 0 : 1;
    const int64_t block = blockIdx.x - (which ? p.blocks[0] : 0), blocks = p.blocks[which];
    const Heads in = p.in[which], out = p.out[which], grad = p.grad[which];
    const void* const gain = p.gain[which];
    const int half = p.D / 2, lanes = 1 << p.lanes_log2;
    const int c0 = (int)threadIdx.x & (lanes - 1);
    // the lane's two chunks, and how much of them there is; heads whose lanes are not a power of two leave some idle
    constexpr bool WHOLE = SHAPE != HEAD_SMALL;
    const int side = ADJACENT ? p.D : half;             // channels that chunks of one kind cover
    int at = 8 * c0, at2 = ADJACENT ? 8 * (c0 + lanes) : half + 8 * c0;
    const int count = side - at, count2 = p.D - at2;
    const bool on = count > 0;
    int twice = 0, twice2 = 0;                          // channels of the chunks that the lane before has too
    if constexpr (SHAPE == HEAD_OVERLAP) {
        if (on && count < 8) twice = 8 - count;
        if (on && count2 > 0 && count2 < 8) twice2 = 8 - count2;
        at -= twice;
        at2 -= twice2;
    }
    // pair i of the lane, of a and b; whether it counts
    auto pair_at = [&](int i) __attribute__((always_inline)) { return ADJACENT ? (i < 4 ? at : at2) / 2 + (i & 3) : at + i; };
    auto counts = [&](int i) __attribute__((always_inline)) {
        return SHAPE != HEAD_OVERLAP || (ADJACENT ? 2 * (i & 3) >= (i < 4 ? twice : twice2) : i >= twice);
    };
    const float per_channel = 1.f / (float)p.D;
    PairTurn turn[8];
    Pairs<DT, WHOLE> gains;
    float sum_a[BACKWARD ? 8 : 1], sum_b[BACKWARD ? 8 : 1];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int pair = pair_at(i);
        turn[i] = on && pair < half ? p.table[pair] : PairTurn{0.f, 0.f, 0, 0};
        if (BACKWARD) sum_a[BACKWARD ? i : 0] = sum_b[BACKWARD ? i : 0] = 0.f;
    }
    gains.clear();
    if (on && gain != nullptr) gains.load((const char*)gain, at, count, at2, count2);

    const int shares = (in.heads + TOGETHER - 1) / TOGETHER;     // groups of heads of a row
    const int64_t items = p.rows * shares, step = blocks * (ROPE_THREADS >> p.lanes_log2);
    const int64_t start = block * (ROPE_THREADS >> p.lanes_log2) + (threadIdx.x >> p.lanes_log2);
    // whole wavefronts stay together for the exchanges: the last round's spare groups work on nothing
    const int64_t rounds = (items + step - 1) / step;
    for (int64_t n = 0; n < rounds; ++n) {
        const int64_t item = start + n * step;
        const bool there = on && item < items;
        const int64_t row = there ? (shares == 1 ? item : item / shares) : 0;
        const int share = there ? (int)(item - row * shares) : 0;           // heads share, share + shares, ...: neighbouring lanes, neighbouring heads
        Pairs<DT, WHOLE> value[TOGETHER], slope[BACKWARD ? TOGETHER : 1];
#pragma unroll
        for (int h = 0; h < TOGETHER; ++h) {
            if (!BACKWARD && h * shares >= in.heads) break;    // no lane has one (backward: the branch costs a third of the wavefronts)
            const int head = share + h * shares;
            value[h].clear();
            if (BACKWARD) slope[BACKWARD ? h : 0].clear();
            if (there && head < in.heads) {
                if (!BACKWARD || gain != nullptr) value[h].load(in.data + row * in.row + head * in.head, at, count, at2, count2);
                if (BACKWARD) slope[BACKWARD ? h : 0].load(grad.data + row * grad.row + head * grad.head, at, count, at2, count2);
            }
        }
        float place[SC_AXES_MAX];
#pragma unroll
        for (int x = 0; x < SC_AXES_MAX; ++x) place[x] = there && x < p.axes ? (float)p.pos[row * p.ld_pos + x] : 0.f;
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int axis = turn[i].axis;
            turn_of<DT>(turn[i], axis == 0 ? place[0] : axis == 1 ? place[1] : axis == 2 ? place[2] : place[3], c[i], s[i]);
        }
        float gain_a[8], gain_b[8];
        gains.template take<ADJACENT>(gain_a, gain_b);
#pragma unroll
        for (int h = 0; h < TOGETHER; ++h) {
            if (!BACKWARD && h * shares >= in.heads) break;
            const int head = share + h * shares;
            float a[8], b[8];
            value[h].template take<ADJACENT>(a, b);
            float scale = 1.f;
            if (gain != nullptr) {
                float squares = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) squares = counts(i) ? fmaf(a[i], a[i], fmaf(b[i], b[i], squares)) : squares;
                scale = rsqrtf(fmaf(sum_of_lanes(squares, p.lanes_log2), per_channel, p.eps));
                if (BACKWARD && !(there && head < in.heads)) scale = 0.f;          // infinite for eps = 0: its zeros would be NaN in the gain's sums
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    a[i] *= scale;                      // the unit row
                    b[i] *= scale;
                }
            }
            float x[8], y[8];
            if constexpr (!BACKWARD) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float u = gain != nullptr ? a[i] * gain_a[i] : a[i], v = gain != nullptr ? b[i] * gain_b[i] : b[i];
                    x[i] = u * c[i] - v * s[i];
                    y[i] = u * s[i] + v * c[i];
                }
            } else {
                float ga[8], gb[8];
                slope[h].template take<ADJACENT>(ga, gb);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = ga[i] * c[i] + gb[i] * s[i];
                    y[i] = gb[i] * c[i] - ga[i] * s[i];
                }
                if (gain != nullptr) {
                    float along = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {        // a head that is not there has zeros for its gradient and its unit row
                        sum_a[i] = fmaf(x[i], a[i], sum_a[i]);
                        sum_b[i] = fmaf(y[i], b[i], sum_b[i]);
                        x[i] *= gain_a[i];
                        y[i] *= gain_b[i];
                        along = counts(i) ? fmaf(x[i], a[i], fmaf(y[i], b[i], along)) : along;
                    }
                    along = sum_of_lanes(along, p.lanes_log2) * per_channel;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = (x[i] - a[i] * along) * scale;
                        y[i] = (y[i] - b[i] * along) * scale;
                    }
                }
            }
            if (there && head < in.heads) store_pairs<DT, ADJACENT, WHOLE>(out.data + row * out.row + head * out.head, at, count, at2, count2, x, y);
        }
    }
    if constexpr (BACKWARD) {                           // the workgroup's share of the gain's gradient, groups of lanes in order
        // Lanes write eight words apart and meet in the same banks: 1.8 of 2.4 M LDS cycles of the 110545 rows above, once at the end of a workgroup, a thirtieth of its time.
        if (p.partial[which] == nullptr) return;
        __shared__ float sums[ROPE_THREADS * 2 * PAIRS_A_LANE];
        const int groups = ROPE_THREADS >> p.lanes_log2, width = 2 * PAIRS_A_LANE * lanes;
        float* mine = sums + (threadIdx.x >> p.lanes_log2) * width;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = pair_at(i);                // below 8 lanes
            if (on && pair < half && counts(i)) {
                mine[pair] = sum_a[i];
                mine[width / 2 + pair] = sum_b[i];
            }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < p.D; j += ROPE_THREADS) {
            const int pair = ADJACENT ? j >> 1 : j < half ? j : j - half;
            const int side = ADJACENT ? j & 1 : j >= half;
            float total = 0.f;
            for (int g = 0; g < groups; ++g) total += sums[g * width + side * (width / 2) + pair];
            p.partial[which][block * p.D + j] = total;
        }
    }
}

// Gradients of the gains: sums over the workgroups' shares, every 64th by one of 64 threads, in a fixed order.
template <int DT>
__global__ void __launch_bounds__(1024)
k_gain_join(const float* __restrict__ q, int q_blocks, void* __restrict__ dq, const float* __restrict__ k, int k_blocks, void* __restrict__ dk, int D) {
    __shared__ float sums[64][16];
    const float* src = blockIdx.y ? k : q;
    void* dst = blockIdx.y ? dk : dq;
    const int blocks = blockIdx.y ? k_blocks : q_blocks;
    if (dst == nullptr) return;
    const int j = blockIdx.x * 16 + (threadIdx.x & 15), which = threadIdx.x >> 4;
    float total = 0.f;
    if (j < D) {
#pragma unroll 8
        for (int b = which; b < blocks; b += 64) total += src[(int64_t)b * D + j];
    }
    sums[which][threadIdx.x & 15] = total;
    __syncthreads();
    if (which != 0 || j >= D) return;
    total = 0.f;
#pragma unroll
    for (int w = 0; w < 64; ++w) total += sums[w][threadIdx.x];
    store_elem<DT>(dst, j, total);
}

// Workgroups for the heads of queries or of keys: all that there is work for, up to a limit that keeps every compute unit full; each goes on
// with further rows and loads the table once.
int rope_blocks(int64_t rows, int heads, int lanes_log2, int together) {
    if (heads == 0) return 0;
    const int64_t items = rows * ((heads + together - 1) / together), each = ROPE_THREADS >> lanes_log2;
    const int64_t blocks = (items + each - 1) / each;
    return (int)(blocks < ROPE_BLOCKS_MAX ? blocks : ROPE_BLOCKS_MAX);
}
int lanes_log2(int D) {
    int log2 = 0;
    while ((PAIRS_A_LANE << log2) < D / 2) ++log2;
    return log2;
}
constexpr int FORWARD_TOGETHER = 4, BACKWARD_TOGETHER = 2;

Heads heads_of(const sc_heads* h, int dtype) {
    const int size = dtype == SC_F32 ? 4 : 2;
    return Heads{(char*)h->data, h->row * size, h->head * size, h->heads};
}
bool has_keys(const sc_heads* k) { return k != nullptr && k->heads > 0; }

int check_rope(const sc_heads* q, const sc_heads* k, int64_t rows, int D, const int32_t* d_pos, int64_t ld_pos, int axes, const void* d_table, int pairing,
               const void* gain_q, const void* gain_k, float eps, const sc_heads* q_out, const sc_heads* k_out, int dtype) {
    if (dtype != SC_F32 && dtype != SC_F16 && dtype != SC_BF16) return SC_EINVAL;
    if (rows < 0 || rows > SC_N_MAX || D < 2 || D > SC_HEAD_MAX || D % 2 != 0 || axes < 1 || axes > SC_AXES_MAX || ld_pos < axes) return SC_EINVAL;
    if (pairing != SC_PAIRS_HALVES && pairing != SC_PAIRS_ADJACENT) return SC_EINVAL;
    if (d_pos == nullptr || ((uintptr_t)d_pos & 3) != 0 || d_table == nullptr || !aligned16(d_table) || !(eps >= 0.f)) return SC_EINVAL;
    const uintptr_t off = dtype == SC_F32 ? 3 : 1;
    if (((uintptr_t)gain_q & off) != 0 || ((uintptr_t)gain_k & off) != 0) return SC_EINVAL;
    if (!heads_ok(q, dtype) || !heads_ok(q_out, dtype) || q->heads < 1 || q_out->heads != q->heads) return SC_EINVAL;
    if (has_keys(k) && (!heads_ok(k, dtype) || !heads_ok(k_out, dtype) || k_out->heads != k->heads)) return SC_EINVAL;
    if (!heads_apart(q_out, rows, D) || (has_keys(k) && !heads_apart(k_out, rows, D))) return SC_EINVAL;
    return SC_OK;
}

template <bool BACKWARD>
int launch_rope(const Rope& p, int pairing, int dtype, hipStream_t s) {
    constexpr int TOGETHER = BACKWARD ? BACKWARD_TOGETHER : FORWARD_TOGETHER;
    const dim3 grid((unsigned)(p.blocks[0] + p.blocks[1]));
    const int kid = BACKWARD ? KID_ROPE_GRAD : KID_ROPE;
    const int side = pairing == SC_PAIRS_ADJACENT ? p.D : p.D / 2;
    const int shape = side % 8 == 0 ? HEAD_EVEN : side > 8 ? HEAD_OVERLAP : HEAD_SMALL;
#define SC_ROPE_SHAPE(DT, ADJACENT)                                                                                                     \
    (shape == HEAD_EVEN ? k_rope<DT, ADJACENT, BACKWARD, TOGETHER, HEAD_EVEN>                                                            \
                        : shape == HEAD_OVERLAP ? k_rope<DT, ADJACENT, BACKWARD, TOGETHER, HEAD_OVERLAP> : k_rope<DT, ADJACENT, BACKWARD, TOGETHER, HEAD_SMALL>)
#define SC_ROPE(DT)                                                                                                                     \
    do {                                                                                                                                \
        const auto kernel = pairing == SC_PAIRS_ADJACENT ? SC_ROPE_SHAPE(DT, true) : SC_ROPE_SHAPE(DT, false);                          \
        SC_LAUNCH(kid, kernel, grid, dim3(ROPE_THREADS), 0, s, p);                                                                      \
    } while (0)
    if (dtype == SC_F32) SC_ROPE(SC_F32);
    else if (dtype == SC_F16) SC_ROPE(SC_F16);
    else SC_ROPE(SC_BF16);
#undef SC_ROPE
#undef SC_ROPE_SHAPE
    return SC_OK;
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" size_t sc_rope_table_bytes(int D) { return D < 2 || D > SC_HEAD_MAX || D % 2 != 0 ? 0 : (size_t)(D / 2) * sizeof(PairTurn); }

extern "C" int sc_rope_table(int D, int axes, const int32_t* h_pairs, double base, void* d_table, size_t table_bytes, void* stream) {
    const size_t need = sc_rope_table_bytes(D);
    if (need == 0 || axes < 1 || axes > SC_AXES_MAX || h_pairs == nullptr || !(base > 0.0) || base > 1e300 || d_table == nullptr || !aligned16(d_table))
        return SC_EINVAL;
    RopeSections sections{};
    int64_t sum = 0;
    for (int a = 0; a < axes; ++a) {
        if (h_pairs[a] < 0) return SC_EINVAL;
        sections.pairs[a] = h_pairs[a];
        sum += h_pairs[a];
    }
    if (sum > D / 2) return SC_EINVAL;
    if (table_bytes < need) return SC_ECAP;
    SC_LAUNCH(KID_ROPE_TABLE, k_rope_table, dim3(1), dim3(512), 0, (hipStream_t)stream, (PairTurn*)d_table, D / 2, axes, sections, base);
    return SC_OK;
}

extern "C" int sc_qk_rope_fwd(const sc_heads* q, const sc_heads* k, int64_t rows, int D, const int32_t* d_pos, int64_t ld_pos, int axes,
                              const void* d_table, int pairing, const void* d_gain_q, const void* d_gain_k, float eps, const sc_heads* q_out,
                              const sc_heads* k_out, int dtype, void* stream) {
    const int rc = check_rope(q, k, rows, D, d_pos, ld_pos, axes, d_table, pairing, d_gain_q, d_gain_k, eps, q_out, k_out, dtype);
    if (rc != SC_OK) return rc;
    if (rows == 0) return SC_OK;
    Rope p{};
    p.in[0] = heads_of(q, dtype);
    p.out[0] = heads_of(q_out, dtype);
    if (has_keys(k)) {
        p.in[1] = heads_of(k, dtype);
        p.out[1] = heads_of(k_out, dtype);
    }
    p.gain[0] = d_gain_q;
    p.gain[1] = d_gain_k;
    p.rows = rows;
    p.pos = d_pos;
    p.ld_pos = ld_pos;
    p.axes = axes;
    p.D = D;
    p.table = (const PairTurn*)d_table;
    p.eps = eps;
    p.lanes_log2 = lanes_log2(D);
    for (int w = 0; w < 2; ++w) p.blocks[w] = rope_blocks(rows, p.in[w].heads, p.lanes_log2, FORWARD_TOGETHER);
    return launch_rope<false>(p, pairing, dtype, (hipStream_t)stream);
}

extern "C" size_t sc_qk_rope_workspace_bytes(int64_t rows, int q_heads, int k_heads, int D) {
    if (rows < 0 || rows > SC_N_MAX || q_heads < 1 || q_heads > SC_GROUPS_MAX || k_heads < 0 || k_heads > SC_GROUPS_MAX || sc_rope_table_bytes(D) == 0) return 0;
    const int log2 = lanes_log2(D);
    return (size_t)(rope_blocks(rows, q_heads, log2, BACKWARD_TOGETHER) + rope_blocks(rows, k_heads, log2, BACKWARD_TOGETHER)) * D * sizeof(float);
}

extern "C" int sc_qk_rope_bwd(const sc_heads* dq_out, const sc_heads* dk_out, const sc_heads* q, const sc_heads* k, int64_t rows, int D,
                              const int32_t* d_pos, int64_t ld_pos, int axes, const void* d_table, int pairing, const void* d_gain_q,
                              const void* d_gain_k, float eps, const sc_heads* dq, const sc_heads* dk, void* d_dgain_q, void* d_dgain_k, int dtype,
                              void* d_workspace, size_t workspace_bytes, void* stream) {
    int rc = check_rope(dq_out, dk_out, rows, D, d_pos, ld_pos, axes, d_table, pairing, d_gain_q, d_gain_k, eps, dq, dk, dtype);
    if (rc != SC_OK) return rc;
    const bool keys = has_keys(dk_out);
    if (d_gain_q != nullptr && (!heads_ok(q, dtype) || q->heads != dq_out->heads)) return SC_EINVAL;
    if (keys && d_gain_k != nullptr && (!heads_ok(k, dtype) || k->heads != dk_out->heads)) return SC_EINVAL;
    const uintptr_t off = dtype == SC_F32 ? 3 : 1;
    if (((uintptr_t)d_dgain_q & off) != 0 || ((uintptr_t)d_dgain_k & off) != 0) return SC_EINVAL;
    if ((d_dgain_q != nullptr && d_gain_q == nullptr) || (d_dgain_k != nullptr && (d_gain_k == nullptr || !keys))) return SC_EINVAL;
    const int log2 = lanes_log2(D);
    const bool gains = d_dgain_q != nullptr || d_dgain_k != nullptr;
    if (gains && rows > 0) {
        if (d_workspace == nullptr || !aligned16(d_workspace)) return SC_EINVAL;
        if (workspace_bytes < sc_qk_rope_workspace_bytes(rows, dq_out->heads, keys ? dk_out->heads : 0, D)) return SC_ECAP;
    }
    Rope p{};
    p.grad[0] = heads_of(dq_out, dtype);
    p.out[0] = heads_of(dq, dtype);
    if (d_gain_q != nullptr) p.in[0] = heads_of(q, dtype);
    p.in[0].heads = dq_out->heads;
    if (keys) {
        p.grad[1] = heads_of(dk_out, dtype);
        p.out[1] = heads_of(dk, dtype);
        if (d_gain_k != nullptr) p.in[1] = heads_of(k, dtype);
        p.in[1].heads = dk_out->heads;
    }
    p.gain[0] = d_gain_q;
    p.gain[1] = d_gain_k;
    p.rows = rows;
    p.pos = d_pos;
    p.ld_pos = ld_pos;
    p.axes = axes;
    p.D = D;
    p.table = (const PairTurn*)d_table;
    p.eps = eps;
    p.lanes_log2 = log2;
    for (int w = 0; w < 2; ++w) p.blocks[w] = rope_blocks(rows, p.in[w].heads, log2, BACKWARD_TOGETHER);
    if (d_dgain_q != nullptr) p.partial[0] = (float*)d_workspace;
    if (d_dgain_k != nullptr) p.partial[1] = (float*)d_workspace + (int64_t)p.blocks[0] * D;
    hipStream_t s = (hipStream_t)stream;
    if (rows > 0) {
        rc = launch_rope<true>(p, pairing, dtype, s);
        if (rc != SC_OK) return rc;
    }
    if (gains) {                                        // no rows: zeros
        const dim3 grid((unsigned)((D + 15) / 16), 2);
#define SC_GAIN_JOIN(DT) SC_LAUNCH(KID_GAIN_JOIN, k_gain_join<DT>, grid, dim3(1024), 0, s, p.partial[0], p.blocks[0], d_dgain_q, p.partial[1], p.blocks[1], d_dgain_k, D)
        if (dtype == SC_F32) SC_GAIN_JOIN(SC_F32);
        else if (dtype == SC_F16) SC_GAIN_JOIN(SC_F16);
        else SC_GAIN_JOIN(SC_BF16);
#undef SC_GAIN_JOIN
    }
    return SC_OK;
}
