// Linear layers and layers whose weights differ by group of rows, forward and backward: argument checks, the gradient of the
// activation, and the sums of a weight gradient's parts.  The products themselves are in sc_product.h; a linear layer is one group.
#include "sc_product.h"

namespace sc {
namespace {

// dpre[p][n] = dy[row(p)][n] act'(pre[p][n]), rounded once to the rows' type: the matrix cores take it as an operand.  A pass over three
// arrays, bound by memory: 110545 x 512 bf16 GELU, 340 MB in 60 us, 5.6 TB/s; both products that follow read the result, which the last-level cache holds unless it is larger.
template <int DT>
__global__ void __launch_bounds__(256)
k_act_grad(const void* __restrict__ grad, int64_t ldg, int64_t grad_rows, const int32_t* __restrict__ list, const void* __restrict__ pre,
           int64_t ldp, int act, void* __restrict__ out, int64_t ldo, int64_t n, int N, int rows_each) {
    const int chunks = (N + 7) / 8;
    const int64_t first = (int64_t)blockIdx.x * rows_each;
    for (int t = threadIdx.x; t < rows_each * chunks; t += 256) {
        const int r = t / chunks, col = (t - r * chunks) * 8;
        const int64_t e = first + r;
        if (e >= n) break;
        int64_t row = e;
        if (list != nullptr) row = list[e];
        const int there = N - col < 8 ? N - col : 8;
        float g[8], v[8];
        const bool ok = row >= 0 && row < grad_rows;
        if (ok) load8<DT>(grad, row * ldg + col, there, g);
        load8<DT>(pre, e * ldp + col, there, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ok ? g[j] * slope<DT>(v[j], act) : 0.f;
        store8<DT>(out, e * ldo + col, there, v);
    }
}

// The same by units of a group's entries (bias_log2), with the sums of the unit's gradients before the rounding, which a bias takes: the sums of rounded values are off by half
// as much again.  A thread keeps to its eight channels, `wide` threads side by side, and walks the unit's rows; their sums meet in LDS, in a fixed order.  110545 x 512 bf16
// GELU 63 us (60 without sums; one row at a time 66), 64 x 512 5.5 (4.0).
template <int DT>
__global__ void __launch_bounds__(512)
k_act_grad_sums(const void* __restrict__ grad, int64_t ldg, int64_t grad_rows, const int32_t* __restrict__ list, const void* __restrict__ pre, int64_t ldp, int act,
                void* __restrict__ out, int64_t ldo, const int32_t* __restrict__ starts, int groups, int64_t n, int N, int wide, int col_blocks, float* __restrict__ sums) {
    constexpr int ROWS = 1 << bias_log2(false, TILE_16_32);
    extern __shared__ __align__(16) float row_sums[];  // eight a thread
    const uint32_t block = blockIdx.y * gridDim.x + blockIdx.x, unit = block / (uint32_t)col_blocks;
    const Part part = find_part<false>(starts, groups, n, ROWS, unit);
    if (part.g < 0) return;                            // the whole workgroup
    const int threads = (int)blockDim.x, step = threads / wide, width = wide * 8;
    const int first_col = (int)(block - unit * (uint32_t)col_blocks) * width, first_row = (int)threadIdx.x / wide;
    int col = first_col + ((int)threadIdx.x - first_row * wide) * 8, there = N - col < 8 ? N - col : 8;
    // the last chunk reaches back over the one before it: the same values, stored by both and summed by one
    const bool on = there > 0 && first_row < step;
    const int twice = on && there < 8 && N >= 8 ? 8 - there : 0;
    col -= twice;
    there += twice;
    float sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = 0.f;
    if (on) {
        int64_t e = part.first + first_row;
        const auto row_of = [&](int64_t at) __attribute__((always_inline)) {
            const int64_t row = list != nullptr ? list[at] : at;
            return row < grad_rows ? row : -1;
        };
        for (; N >= 8 && e + step < part.last; e += 2 * step) {          // two rows on their way at a time
            Eight<DT> g[2], x[2];
            int64_t row[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                row[k] = row_of(e + k * step);
                g[k].load(grad, (row[k] >= 0 ? row[k] : 0) * ldg + col);
                x[k].load(pre, (e + k * step) * ldp + col);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float a[8], v[8];
                g[k].to_floats(a);
                x[k].to_floats(v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = row[k] >= 0 ? a[j] * slope<DT>(v[j], act) : 0.f;
                    sum[j] += v[j];
                }
                store8<DT>(out, (e + k * step) * ldo + col, 8, v);
            }
        }
        for (; e < part.last; e += step) {
            const int64_t row = row_of(e);
            float g[8], v[8];
            if (row >= 0) load8<DT>(grad, row * ldg + col, there, g);
            load8<DT>(pre, e * ldp + col, there, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = row >= 0 ? g[j] * slope<DT>(v[j], act) : 0.f;
                sum[j] += v[j];
            }
            store8<DT>(out, e * ldo + col, there, v);
        }
    }
    if (twice == 0) {
        reinterpret_cast<float4*>(row_sums)[threadIdx.x * 2] = make_float4(sum[0], sum[1], sum[2], sum[3]);
        reinterpret_cast<float4*>(row_sums)[threadIdx.x * 2 + 1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
    } else {
#pragma unroll
        for (int j = 1; j < 8; ++j)
            if (j >= twice) row_sums[threadIdx.x * 8 + j - twice] = sum[j];
    }
    __syncthreads();
    // of every column, shares of the rows by as many threads as there are for it, then the shares in order
    const int shares = width < threads ? threads / width : 1, share = shares == 1 ? 0 : (int)threadIdx.x / width;
    float* const at = sums + (part.first / ROWS + part.g) * N + first_col;
    for (int j = (int)threadIdx.x - share * width; j < width && share < shares; j += threads) {
        float total = 0.f;
#pragma unroll 8
        for (int r = share; r < step; r += shares) total += row_sums[r * width + j];
        if (shares == 1) {
            if (first_col + j < N) at[j] = total;
        } else {
            sum[0] = total;
        }
    }
    if (shares == 1) return;
    __syncthreads();
    if (share < shares) row_sums[threadIdx.x] = sum[0];
    __syncthreads();
    if ((int)threadIdx.x >= width || first_col + (int)threadIdx.x >= N) return;
    float total = 0.f;
    for (int k = 0; k < shares; ++k) total += row_sums[k * width + threadIdx.x];
    at[threadIdx.x] = total;
}

// Sums of the parts of a group, in a fixed order.  LANES threads take 4 LANES consecutive values, 256 / LANES of them every so many'th part each, then their sums:
// few parts many values a workgroup, many parts many loads in flight.  Bound by the trip to memory: 124 parts of 129 x 512 sums, 33 MB, 8.0 us; 16 groups of
// 513 x 2048, of which the largest have parts, 11.5 us (16.6 with workgroups for the groups that have one part, too).
template <int DT, int LANES>
__global__ void __launch_bounds__(256)
k_product_join(const float* __restrict__ partial, const int32_t* __restrict__ starts, int groups, int64_t n, int64_t per, int M, int N,
               void* __restrict__ out, void* __restrict__ out_bias, int64_t slots, int64_t blocks_each) {
    constexpr int SHARES = 256 / LANES;
    __shared__ float4 sums[SHARES][LANES];
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int nth = (int)(block / blocks_each);        // of the groups that have several parts
    const int64_t values = (int64_t)(M + 1) * N;
    const int lane = threadIdx.x & 63;
    int64_t slot = 0;
    int g = 0, parts = 0;
    if (starts == nullptr) {
        if (nth == 0) parts = (int)((n + per - 1) / per);
    } else {
        int seen = 0;
        for (int g0 = 0; g0 < groups && seen <= nth; g0 += WAVE) {
            const int at = g0 + lane;
            int64_t lo = 0, hi = 0;
            if (at < groups) {
                lo = starts[at];
                hi = starts[at + 1];
                lo = lo < 0 ? 0 : lo > n ? n : lo;
                hi = hi < lo ? lo : hi > n ? n : hi;
            }
            const uint32_t len = (uint32_t)(hi - lo), step = (uint32_t)per;
            const int count = (int)(len / step + (len % step != 0));
            const uint64_t several = __ballot(count > 1), mine = (uint64_t)1 << lane;
            const int rank = seen + __popcll(several & (mine - 1));       // of this lane's group among those
            const uint64_t found = __ballot(count > 1 && rank == nth);
            int before = count > 1 && rank < nth ? count : 0;
#pragma unroll
            for (int d = 1; d < WAVE; d <<= 1) before += __shfl_xor(before, d);
            slot += before;
            if (found != 0) {
                g = g0 + __builtin_ctzll(found);
                parts = __shfl(count, g - g0);
            }
            seen += __popcll(several);
        }
    }
    if (parts <= 1 || slot + parts > slots) return;    // no more such groups: the product itself has written the others; starts that do not ascend
    const int64_t first = (block - (int64_t)nth * blocks_each) * (4 * LANES), at = first + 4 * (threadIdx.x % LANES);
    const int which = threadIdx.x / LANES;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* src = partial + slot * values + at;
    if (at + 4 <= values) {
#pragma unroll 8
        for (int s = which; s < parts; s += SHARES) {
            const uint4 v = load_chunk(src + s * values);
            sum.x += __builtin_bit_cast(float, v.x);
            sum.y += __builtin_bit_cast(float, v.y);
            sum.z += __builtin_bit_cast(float, v.z);
            sum.w += __builtin_bit_cast(float, v.w);
        }
    } else {
        for (int s = which; s < parts; s += SHARES) {
            if (at < values) sum.x += src[s * values];
            if (at + 1 < values) sum.y += src[s * values + 1];
            if (at + 2 < values) sum.z += src[s * values + 2];
        }
    }
    sums[which][threadIdx.x % LANES] = sum;
    __syncthreads();
    const int64_t weights = (int64_t)M * N;
    for (int t = threadIdx.x; t < 4 * LANES; t += 256) {
        const int64_t mine = first + t;
        if (mine >= values) return;
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < SHARES; ++w) total += reinterpret_cast<const float*>(&sums[w][0])[t];
        if (mine < weights) store_elem<DT>(out, g * weights + mine, total);
        else if (out_bias != nullptr) store_elem<DT>(out_bias, g * (int64_t)N + mine - weights, total);
    }
}

int elem(int dtype) { return dtype == SC_F32 ? 4 : 2; }
bool dtype_ok(int dtype) { return dtype == SC_F32 || dtype == SC_F16 || dtype == SC_BF16; }
bool aligned_to(const void* p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }
bool channels_ok(int C) { return C >= 1 && C <= SC_CHANNELS_MAX; }
// `n` rows `ld` elements apart; no rows need no memory
bool rows_ok(const void* p, int64_t n, int64_t ld, int C, int dtype) {
    return (p != nullptr || n == 0) && aligned_to(p, elem(dtype)) && ld >= C && ld <= SC_LD_MAX;
}
int launch(int dtype, int mode, const Product& p, hipStream_t s) {
    const int cus = compute_units();
    if (dtype == SC_F32) return launch_product_f32(mode, p, cus, s);
    if (dtype == SC_F16) return launch_product_f16(mode, p, cus, s);
    return launch_product_bf16(mode, p, cus, s);
}

struct Entries {                   // what tells a grouped layer from a linear one
    const int32_t* starts;
    int groups;
    int64_t n;
    const int32_t* rows;
    int64_t x_rows;
    const int32_t* grad_rows;
    int64_t grad_n;
};

int forward(const void* x, int64_t ldx, const Entries& e, const void* weight, const void* bias, int act, const void* residual, int64_t ldr, void* y,
            int64_t ldy, void* pre, int64_t ldp, int C_in, int C_out, int dtype_in, int dtype_out, hipStream_t s) {
    if (!channels_ok(C_in) || !channels_ok(C_out) || !dtype_ok(dtype_in) || (dtype_out != SC_F32 && dtype_out != dtype_in)) return SC_EINVAL;
    if (act < SC_ACT_NONE || act > SC_ACT_SILU) return SC_EINVAL;
    if (e.n < 0 || e.n > SC_ENTRIES_MAX || e.x_rows < 0 || e.x_rows > SC_N_MAX || e.groups < 1 || e.groups > SC_GROUPS_MAX) return SC_EINVAL;
    if (weight == nullptr || !aligned_to(weight, elem(dtype_in)) || !aligned_to(bias, elem(dtype_in))) return SC_EINVAL;
    if (!rows_ok(x, e.x_rows, ldx, C_in, dtype_in) || !rows_ok(y, e.n, ldy, C_out, dtype_out)) return SC_EINVAL;
    if (residual != nullptr && !rows_ok(residual, e.n, ldr, C_out, dtype_out)) return SC_EINVAL;
    if (pre != nullptr && !rows_ok(pre, e.n, ldp, C_out, dtype_out)) return SC_EINVAL;
    if (e.n == 0) return SC_OK;
    Product p{};
    p.a = x;
    p.lda = ldx;
    p.a_rows = e.x_rows;
    p.a_list = e.rows;
    p.b = weight;
    p.ldb = C_out;
    p.starts = e.starts;
    p.groups = e.groups;
    p.n = e.n;
    p.N = C_out;
    p.K = C_in;
    p.bias = bias;
    p.act = act;
    p.residual = residual;
    p.ldr = ldr;
    p.pre = pre;
    p.ldp = ldp;
    p.out = y;
    p.ldo = ldy;
    p.out_f32 = dtype_out == SC_F32 && dtype_in != SC_F32;
    return launch(dtype_in, PRODUCT_FWD, p, s);
}

// The gradient ahead of the activation: rows 64 bytes aligned, whatever their channels.
int64_t grad_pitch(int C_out, int dtype) { return (int64_t)align_up((size_t)C_out * elem(dtype), 64) / elem(dtype); }
size_t grad_bytes(int64_t n, int C_out, int dtype) { return align_up((size_t)n * grad_pitch(C_out, dtype) * elem(dtype), 256); }
size_t partial_bytes(int64_t n, int C_in, int C_out) {
    return (size_t)weight_slots(n, weight_part(n, C_in, C_out)) * (C_in + 1) * C_out * sizeof(float);
}
// ... and the bias' sums: of 32-bit rows the gradient is not rounded.  `linear`: row_tile knows it by no groups
size_t bias_bytes(int64_t n, int groups, bool linear, int C_in, int C_out, int dtype) {
    if (dtype == SC_F32 || n == 0) return 0;
    const int64_t apart = bias_units(n, groups, bias_log2(false, TILE_16_32)), cus = compute_units();
    const int64_t inside = act_in_product(n, groups, C_in, C_out, cus) ? bias_units(n, groups, bias_log2(true, row_tile(n, linear ? 0 : groups, C_in, C_out, false, false, cus))) : 0;
    return (size_t)(apart > inside ? apart : inside) * C_out * sizeof(float);
}
size_t workspace_bytes(int64_t n, int groups, bool linear, int C_in, int C_out, int dtype) {
    if (n < 0 || n > SC_ENTRIES_MAX || groups < 1 || groups > SC_GROUPS_MAX || !channels_ok(C_in) || !channels_ok(C_out) || !dtype_ok(dtype)) return 0;
    return grad_bytes(n, C_out, dtype) + partial_bytes(n, C_in, C_out) + bias_bytes(n, groups, linear, C_in, C_out, dtype);
}

int backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const Entries& e, const void* weight, const void* pre, int64_t ldp, int act,
             void* dx, int64_t lddx, void* dweight, void* dbias, int C_in, int C_out, int dtype, void* workspace, size_t bytes, hipStream_t s) {
    if (!channels_ok(C_in) || !channels_ok(C_out) || !dtype_ok(dtype)) return SC_EINVAL;
    if (act < SC_ACT_NONE || act > SC_ACT_SILU) return SC_EINVAL;
    if (e.n < 0 || e.n > SC_ENTRIES_MAX || e.x_rows < 0 || e.x_rows > SC_N_MAX || e.grad_n < 0 || e.grad_n > SC_N_MAX || e.groups < 1 ||
        e.groups > SC_GROUPS_MAX)
        return SC_EINVAL;
    const int size = elem(dtype);
    if (dx == nullptr && dweight == nullptr && dbias == nullptr) return SC_EINVAL;
    if (!rows_ok(dy, e.grad_n, lddy, C_out, dtype)) return SC_EINVAL;
    if (act != SC_ACT_NONE && !rows_ok(pre, e.n, ldp, C_out, dtype)) return SC_EINVAL;
    if (dx != nullptr && (!rows_ok(dx, e.n, lddx, C_in, dtype) || weight == nullptr || !aligned_to(weight, size))) return SC_EINVAL;
    if (dweight != nullptr && (!aligned_to(dweight, size) || !rows_ok(x, e.x_rows, ldx, C_in, dtype))) return SC_EINVAL;
    if (!aligned_to(dbias, size)) return SC_EINVAL;
    const bool sums = dweight != nullptr || dbias != nullptr;
    const size_t own = act != SC_ACT_NONE ? grad_bytes(e.n, C_out, dtype) : 0;
    const size_t parts = sums ? partial_bytes(e.n, C_in, C_out) : 0;
    const bool sums_apart = dbias != nullptr && act != SC_ACT_NONE && dtype != SC_F32 && e.n > 0;
    const size_t need = own + parts + (sums && act != SC_ACT_NONE ? bias_bytes(e.n, e.groups, e.starts == nullptr, C_in, C_out, dtype) : 0);
    if (need > 0 && (workspace == nullptr || !aligned16(workspace))) return SC_EINVAL;
    if (need > bytes) return SC_ECAP;
    if (e.n == 0 && !sums) return SC_OK;

    const void* grad = dy;
    const int64_t pitch = grad_pitch(C_out, dtype);
    int64_t ldg = lddy, grad_rows = e.grad_n;
    const int32_t* grad_list = e.grad_rows;
    float* const bias_terms = sums_apart ? (float*)((char*)workspace + own + parts) : nullptr;
    const bool fused = act != SC_ACT_NONE && e.n > 0 && dx != nullptr && e.grad_n > 0 && act_in_product(e.n, e.groups, C_in, C_out, compute_units());
    const RowTile tile = fused ? row_tile(e.n, e.starts == nullptr ? 0 : e.groups, C_in, C_out, false, false, compute_units()) : TILE_16_32;
    const int log2 = bias_log2(fused, tile);
    if (sums_apart && !fused) {
        const int64_t chunks = (C_out + 7) / 8, most = e.starts == nullptr ? bias_units(e.n - 1, 1, log2) : bias_units(e.n, e.groups < e.n ? e.groups : e.n, log2);
        const int64_t wide = sum_columns(most, chunks), col_blocks = (chunks + wide - 1) / wide, blocks = most * col_blocks;
        if (blocks > INT32_MAX) return SC_EINVAL;
        const unsigned threads = (unsigned)sum_threads(wide);
        const dim3 grid((unsigned)grid_columns(blocks), (unsigned)grid_rows(blocks));
#define SC_ACT_GRAD(DT)                                                                                                                                       \
    SC_LAUNCH(KID_ACT_GRAD, k_act_grad_sums<DT>, grid, dim3(threads), threads * 8 * sizeof(float), s, dy, lddy, e.grad_n, e.grad_rows, pre, ldp, act, workspace, pitch, e.starts, e.groups, \
              e.n, C_out, (int)wide, (int)col_blocks, bias_terms)
        if (dtype == SC_F16) SC_ACT_GRAD(SC_F16);
        else SC_ACT_GRAD(SC_BF16);
#undef SC_ACT_GRAD
    } else if (act != SC_ACT_NONE && e.n > 0 && !fused) {
        const int chunks = (C_out + 7) / 8, each = (int)act_grad_rows(e.n, chunks);
        const dim3 grid((unsigned)((e.n + each - 1) / each));
#define SC_ACT_GRAD(DT) SC_LAUNCH(KID_ACT_GRAD, k_act_grad<DT>, grid, dim3(256), 0, s, dy, lddy, e.grad_n, e.grad_rows, pre, ldp, act, workspace, pitch, e.n, C_out, each)
        if (dtype == SC_F32) SC_ACT_GRAD(SC_F32);
        else if (dtype == SC_F16) SC_ACT_GRAD(SC_F16);
        else SC_ACT_GRAD(SC_BF16);
#undef SC_ACT_GRAD
    }
    auto after_activation = [&] {
        grad = workspace;
        ldg = pitch;
        grad_rows = e.n;
        grad_list = nullptr;
    };
    if (act != SC_ACT_NONE && !fused) after_activation();
    if (dx != nullptr && e.n > 0) {
        Product p{};
        p.a = grad;
        p.lda = ldg;
        p.a_rows = grad_rows;
        p.a_list = grad_list;
        p.b = weight;
        p.ldb = C_out;
        p.starts = e.starts;
        p.groups = e.groups;
        p.n = e.n;
        p.N = C_in;
        p.K = C_out;
        p.out = dx;
        p.ldo = lddx;
        p.pre = const_cast<void*>(pre);
        p.ldp = ldp;
        p.act = act;
        p.kept = workspace;
        p.ldk = pitch;
        p.bias_sums = bias_terms;
        const int rc = launch(dtype, fused ? PRODUCT_DX_ACT : PRODUCT_DX, p, s);
        if (rc != SC_OK) return rc;
        if (fused) after_activation();
    }
    if (sums) {
        Product p{};
        p.a = x;
        p.lda = ldx;
        p.a_rows = e.x_rows;
        p.a_list = e.rows;
        p.b = grad;
        p.ldb = ldg;
        p.b_rows = grad_rows;
        p.b_list = grad_list;
        p.starts = e.starts;
        p.groups = e.groups;
        p.n = e.n;
        p.M = dweight != nullptr ? C_in : 0;
        p.N = C_out;
        p.per = weight_part(e.n, C_in, C_out);
        p.units = e.starts == nullptr ? (e.n > p.per ? (e.n + p.per - 1) / p.per : 1) : e.n / p.per + e.groups;
        p.out = dweight;
        p.out_bias = dbias;
        p.bias_sums = bias_terms;
        p.bias_log2 = log2;
        p.partial = (float*)((char*)workspace + own);
        p.slots = weight_slots(e.n, p.per);
        int rc = launch(dtype, PRODUCT_DW, p, s);
        if (rc != SC_OK) return rc;
        if (e.n > p.per) {
            // 1024 values a workgroup leave most of the chip idle below some thousands of them (narrow / wide: 27 groups of 64 x 64 5 / 10 us)
            const int64_t values = (int64_t)(p.M + 1) * p.N;
            const int64_t cut = e.groups < e.n / p.per ? e.groups : e.n / p.per;       // groups that can have several parts
            const bool many = (values + 1023) / 1024 * cut < 2048;
            const int64_t wide = many ? 64 : 1024, each = (values + wide - 1) / wide, blocks = each * cut;
            if (blocks > INT32_MAX) return SC_EINVAL;
            const dim3 grid((unsigned)grid_columns(blocks), (unsigned)grid_rows(blocks));
#define SC_JOIN(DT)                                                                                                                             \
    do {                                                                                                                                        \
        if (many) SC_LAUNCH(KID_PRODUCT_JOIN, (k_product_join<DT, 16>), grid, dim3(256), 0, s, p.partial, e.starts, e.groups, e.n, p.per, p.M,  \
                            p.N, dweight, dbias, p.slots, each);                                                                                \
        else SC_LAUNCH(KID_PRODUCT_JOIN, (k_product_join<DT, 256>), grid, dim3(256), 0, s, p.partial, e.starts, e.groups, e.n, p.per, p.M, p.N, \
                       dweight, dbias, p.slots, each);                                                                                          \
    } while (0)
            if (dtype == SC_F32) SC_JOIN(SC_F32);
            else if (dtype == SC_F16) SC_JOIN(SC_F16);
            else SC_JOIN(SC_BF16);
#undef SC_JOIN
        }
    }
    return SC_OK;
}

}  // namespace
}  // namespace sc

using namespace sc;

extern "C" int sc_linear_fwd(const void* d_x, int64_t ldx, int64_t rows, const void* d_weight, const void* d_bias, int act, const void* d_residual,
                             int64_t ld_residual, void* d_y, int64_t ldy, void* d_pre, int64_t ld_pre, int C_in, int C_out, int dtype_in,
                             int dtype_out, void* stream) {
    if (rows < 0 || rows > SC_N_MAX) return SC_EINVAL;
    const Entries e{nullptr, 1, rows, nullptr, rows, nullptr, rows};
    return forward(d_x, ldx, e, d_weight, d_bias, act, d_residual, ld_residual, d_y, ldy, d_pre, ld_pre, C_in, C_out, dtype_in, dtype_out,
                   (hipStream_t)stream);
}

extern "C" size_t sc_linear_workspace_bytes(int64_t rows, int C_in, int C_out, int dtype) {
    return rows > SC_N_MAX ? 0 : workspace_bytes(rows, 1, true, C_in, C_out, dtype);
}

extern "C" int sc_linear_bwd(const void* d_dy, int64_t lddy, const void* d_x, int64_t ldx, int64_t rows, const void* d_weight, const void* d_pre,
                             int64_t ld_pre, int act, void* d_dx, int64_t lddx, void* d_dweight, void* d_dbias, int C_in, int C_out, int dtype,
                             void* d_workspace, size_t bytes, void* stream) {
    if (rows < 0 || rows > SC_N_MAX) return SC_EINVAL;
    const Entries e{nullptr, 1, rows, nullptr, rows, nullptr, rows};
    return backward(d_dy, lddy, d_x, ldx, e, d_weight, d_pre, ld_pre, act, d_dx, lddx, d_dweight, d_dbias, C_in, C_out, dtype, d_workspace, bytes,
                    (hipStream_t)stream);
}

extern "C" int sc_grouped_fwd(const void* d_x, int64_t ldx, int64_t x_rows, const int32_t* d_rows, int64_t n, const int32_t* d_starts, int groups,
                              const void* d_weight, const void* d_bias, int act, void* d_y, int64_t ldy, void* d_pre, int64_t ld_pre, int C_in,
                              int C_out, int dtype_in, int dtype_out, void* stream) {
    if (d_starts == nullptr || !aligned_to(d_starts, 4) || !aligned_to(d_rows, 4)) return SC_EINVAL;
    const Entries e{d_starts, groups, n, d_rows, x_rows, nullptr, 0};
    return forward(d_x, ldx, e, d_weight, d_bias, act, nullptr, 0, d_y, ldy, d_pre, ld_pre, C_in, C_out, dtype_in, dtype_out, (hipStream_t)stream);
}

extern "C" size_t sc_grouped_workspace_bytes(int64_t n, int groups, int C_in, int C_out, int dtype) {
    return workspace_bytes(n, groups, false, C_in, C_out, dtype);
}

extern "C" int sc_grouped_bwd(const void* d_dy, int64_t lddy, int64_t dy_rows, const int32_t* d_grad_rows, const void* d_x, int64_t ldx, int64_t x_rows,
                              const int32_t* d_rows, int64_t n, const int32_t* d_starts, int groups, const void* d_weight, const void* d_pre,
                              int64_t ld_pre, int act, void* d_dx, int64_t lddx, void* d_dweight, void* d_dbias, int C_in, int C_out, int dtype,
                              void* d_workspace, size_t bytes, void* stream) {
    if (d_starts == nullptr || !aligned_to(d_starts, 4) || !aligned_to(d_rows, 4) || !aligned_to(d_grad_rows, 4)) return SC_EINVAL;
    const Entries e{d_starts, groups, n, d_rows, x_rows, d_grad_rows, dy_rows};
    return backward(d_dy, lddy, d_x, ldx, e, d_weight, d_pre, ld_pre, act, d_dx, lddx, d_dweight, d_dbias, C_in, C_out, dtype, d_workspace, bytes,
                    (hipStream_t)stream);
}
