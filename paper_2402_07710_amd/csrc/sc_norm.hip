// Group norm with an activation over packed scenes, channels last, forward and backward.
//
//     u = (x - mean) / sqrt(var + eps),  y = act(u gain + bias)        mean, var: over a scene's rows and a group's channels
//     backward: dz = dy act'(u gain + bias),  dbias = sum dz,  dgain = sum dz u        over all rows
//               dx = (dz gain - mean(dz gain) - u mean(dz gain u)) / sqrt(var + eps)   means as above
//
// Memory is the bound: x is read for the sums and again for the result, backward dy too.  A workgroup takes some rows of a scene, all channels of them, eight channels
// a thread, and leaves sums of every channel; they are joined for every scene and group in 64 bits, in the order of the rows.
// Deviations are summed about the workgroup's own first row, so they are as exact for channels far from zero as for others: sums of n squares about a row
// of the set are at most n + 1 times those about the mean.
#include "sc_product.h"
#include "sc_scenes.h"

namespace sc {
namespace {

constexpr int NORM_THREADS = 256, JOIN_THREADS = 1024, CHUNK = 8;
constexpr int SLICE = NORM_THREADS * CHUNK;          // channels that a workgroup has at most

struct Norm {
    const char *x, *dy;
    char *y;                           // backward: dx
    int64_t ldx, ldy, lddy;            // bytes
    int64_t rows;
    const int32_t* starts;
    int scenes, C, groups, channels;   // channels of a group
    const void *gain, *bias;
    void *dgain, *dbias;
    float eps;
    int act;
    float2* stats;                     // [scene][group]: mean, 1 / deviation
    float2* sums;                      // [unit][C]: mean and squares about it, or backward the sums of dz and of dz u
    float2* means;                     // backward: [scene][group]
    int per, per_log2;                 // rows of a unit
    int64_t units;
};

// The rows of a unit: first of them, how many, and of which scene.
struct NormUnit {
    int64_t first;
    int rows, scene;
};
__device__ inline NormUnit unit_of(const Norm& p, int64_t u) {
    int64_t first = 0;
    int count = 0, scene = 0;
    const int tile = __builtin_amdgcn_readfirstlane(find_scene(p.starts, p.scenes, p.rows, 1, p.per_log2, u, p.units, first, count, scene).tile);
    if (tile < 0) return NormUnit{0, 0, 0};
    first = uniform64(first) + (int64_t)tile * p.per;
    const int left = __builtin_amdgcn_readfirstlane(count) - tile * p.per;
    return NormUnit{first, left < p.per ? left : p.per, __builtin_amdgcn_readfirstlane(scene)};
}
// Where a thread stands in a slice of channels: its chunk, and its first row of those that the workgroup takes at a time.
struct Place {
    int channel, count;                // of the chunk: first, and how many there are
    int row, step;                     // step 0: the thread has nothing to do
    __device__ Place(const Norm& p, int slice) {
        const int width = p.C - slice * SLICE < SLICE ? p.C - slice * SLICE : SLICE, chunks = (width + CHUNK - 1) / CHUNK;
        step = NORM_THREADS / chunks;
        row = (int)threadIdx.x / chunks;
        channel = slice * SLICE + ((int)threadIdx.x - row * chunks) * CHUNK;
        count = p.C - channel < CHUNK ? p.C - channel : CHUNK;
        if (row >= step) row = INT32_MAX / 2;
    }
};
template <int DT>
__device__ inline void load_values(const void* values, int channel, int count, float otherwise, float (&v)[8]) {
    if (values == nullptr) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = otherwise;
    } else {
        load8<DT>(values, channel, count, v);
    }
}
// Sums of a workgroup's threads that have the same channels, of two numbers a channel; the first `width` threads ... end up with a channel each in turn.
template <class F>
__device__ inline void join_threads(const float (&a)[8], const float (&b)[8], int width, F&& take) {
    __shared__ float shared[2][NORM_THREADS * CHUNK];
    const int chunks = (width + CHUNK - 1) / CHUNK, step = NORM_THREADS / chunks, row = (int)threadIdx.x / chunks;
    const int line = chunks * CHUNK, at = row * line + ((int)threadIdx.x - row * chunks) * CHUNK;
    if (row < step) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            shared[0][at + j] = a[j];
            shared[1][at + j] = b[j];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += NORM_THREADS) {
        float x = 0.f, y = 0.f;
        for (int r = 0; r < step; ++r) {
            x += shared[0][r * line + c];
            y += shared[1][r * line + c];
        }
        take(c, x, y);
    }
}

template <int DT>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm_sums(const Norm p) {
    const NormUnit unit = unit_of(p, blockIdx.x);
    if (unit.rows == 0) return;
    const int slice = blockIdx.y;
    const Place at(p, slice);
    float pivot[8], sum[8], square[8];
    const char* const base = p.x + unit.first * p.ldx;
    load8<DT>(base, at.channel, at.count, pivot);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = square[j] = 0.f;
#pragma unroll 4
    for (int r = at.row; r < unit.rows; r += at.step) {
        float v[8];
        load8<DT>(base + r * p.ldx, at.channel, at.count, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = v[j] - pivot[j];
            sum[j] += d;
            square[j] = fmaf(d, d, square[j]);
        }
    }
    const int width = p.C - slice * SLICE < SLICE ? p.C - slice * SLICE : SLICE;
    join_threads(sum, square, width, [&](int c, float s, float q) {
        const float n = (float)unit.rows, mean = s / n;
        p.sums[(int64_t)blockIdx.x * p.C + slice * SLICE + c] = make_float2(load_elem<DT>(base, slice * SLICE + c) + mean, fmaxf(q - s * mean, 0.f));
    });
}

// Two sums over the threads of a workgroup, the same in all of them, in the order of lanes and wavefronts.
template <int THREADS>
__device__ inline void sum_of_threads(double& a, double& b) {
    __shared__ double shared[2][THREADS / WAVE];
#pragma unroll
    for (int d = 1; d < WAVE; d <<= 1) {
        a += __shfl_xor(a, d);
        b += __shfl_xor(b, d);
    }
    if (THREADS == WAVE) return;
    if ((threadIdx.x & 63) == 0) {
        shared[0][threadIdx.x >> 6] = a;
        shared[1][threadIdx.x >> 6] = b;
    }
    __syncthreads();
    a = b = 0.0;
#pragma unroll
    for (int w = 0; w < THREADS / WAVE; ++w) {
        a += shared[0][w];
        b += shared[1][w];
    }
}
// A scene's rows and the units that hold them.
__device__ inline void scene_units_of(const Norm& p, int scene, int64_t& first_unit, int& rows) {
    int64_t first = 0;
    scene_rows(p.starts, nullptr, p.rows, scene, first, rows);
    first_unit = first / p.per + scene;
}

// A scene and a group of THREADS threads: one workgroup's, or one wavefront's of the four in a workgroup where there are many of them.
template <int THREADS>
__device__ inline int pair_of_threads() { return THREADS == WAVE ? (int)(blockIdx.x * 4 + (threadIdx.x >> 6)) : (int)blockIdx.x; }
// Mean and deviation of a scene's group from its units' sums.
template <int THREADS>
__global__ void __launch_bounds__(THREADS == WAVE ? 256 : THREADS)
k_norm_join(const Norm p) {
    const int pair = pair_of_threads<THREADS>(), tid = (int)threadIdx.x % THREADS;
    if (pair >= p.scenes * p.groups) return;
    const int scene = pair / p.groups, group = pair - scene * p.groups;
    int64_t unit = 0;
    int rows = 0;
    scene_units_of(p, scene, unit, rows);
    const int units = (rows + p.per - 1) / p.per;
    const float2* const sums = p.sums + unit * p.C + group * p.channels;
    const float pivot = units > 0 ? sums[0].x : 0.f;
    double sum = 0.0, square = 0.0;
    const int64_t items = (int64_t)units * p.channels;
#pragma unroll 4
    for (int64_t i = tid; i < items; i += THREADS) {
        const int u = (int)((uint32_t)i / (uint32_t)p.channels), c = (int)(i - (int64_t)u * p.channels);
        const float2 s = sums[(int64_t)u * p.C + c];
        const double n = rows - u * p.per < p.per ? rows - u * p.per : p.per, d = (double)s.x - pivot;
        sum += n * d;
        square += s.y + n * d * d;
    }
    sum_of_threads<THREADS>(sum, square);
    if (tid != 0) return;
    const double n = (double)rows * p.channels, mean = rows > 0 ? sum / n : 0.0, var = rows > 0 ? square / n - mean * mean : 0.0;
    p.stats[pair] = make_float2((float)(pivot + mean), (float)(1.0 / sqrt((var > 0.0 ? var : var != var ? var : 0.0) + (double)p.eps)));
}

// mean, 1 / deviation, gain and bias of a thread's channels
template <int DT>
struct Channels {
    float mean[8], scale[8], gain[8], bias[8];
    int group[8];
    __device__ Channels(const Norm& p, const Place& at, int scene) {
        load_values<DT>(p.gain, at.channel, at.count, 1.f, gain);
        load_values<DT>(p.bias, at.channel, at.count, 0.f, bias);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = at.channel + j < p.C ? at.channel + j : p.C - 1;
            group[j] = c / p.channels;
            const float2 s = p.stats[(int64_t)scene * p.groups + group[j]];
            mean[j] = s.x;
            scale[j] = s.y;
        }
    }
};

template <int DT>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm(const Norm p) {
    const NormUnit unit = unit_of(p, p.units - 1 - blockIdx.x);       // the rows read last are the likeliest to be in the caches still
    if (unit.rows == 0) return;
    const Place at(p, blockIdx.y);
    if (at.row >= unit.rows) return;
    const Channels<DT> ch(p, at, unit.scene);
    const char* const x = p.x + unit.first * p.ldx;
    char* const y = p.y + unit.first * p.ldy;
    float scale[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) scale[j] = ch.scale[j] * ch.gain[j];
#pragma unroll 4
    for (int r = at.row; r < unit.rows; r += at.step) {
        float v[8];
        load8<DT>(x + r * p.ldx, at.channel, at.count, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j] - ch.mean[j], scale[j], ch.bias[j]);
        activate8<DT>(v, p.act);
        store8<DT>(y + r * p.ldy, at.channel, at.count, v);
    }
}

// Few rows: a workgroup has a scene's group to itself, and its rows stay in the caches between the passes.
template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_norm_few(const Norm p) {
    const int scene = blockIdx.x / (unsigned)p.groups, group = blockIdx.x - scene * p.groups;
    int64_t first = 0;
    int rows = 0;
    scene_rows(p.starts, nullptr, p.rows, scene, first, rows);
    const char* const x = p.x + first * p.ldx;
    char* const y = p.y + first * p.ldy;
    const int c0 = group * p.channels, items = rows * p.channels;
    const float pivot = rows > 0 ? load_elem<DT>(x, c0) : 0.f;
    double sum = 0.0, square = 0.0;
#pragma unroll 8
    for (int i = threadIdx.x; i < items; i += THREADS) {
        const int r = i / p.channels;
        const double d = (double)load_elem<DT>(x + r * p.ldx, c0 + i - r * p.channels) - pivot;
        sum += d;
        square += d * d;
    }
    sum_of_threads<THREADS>(sum, square);
    const double mean = rows > 0 ? sum / items : 0.0, var = rows > 0 ? square / items - mean * mean : 0.0;
    const float2 s = make_float2((float)(pivot + mean), (float)(1.0 / sqrt((var > 0.0 ? var : var != var ? var : 0.0) + (double)p.eps)));
    if (p.stats != nullptr && threadIdx.x == 0) p.stats[blockIdx.x] = s;
#pragma unroll 8
    for (int i = threadIdx.x; i < items; i += THREADS) {
        const int r = i / p.channels, c = c0 + i - r * p.channels;
        const float gain = p.gain != nullptr ? load_elem<DT>(p.gain, c) : 1.f, bias = p.bias != nullptr ? load_elem<DT>(p.bias, c) : 0.f;
        const float v = fmaf(load_elem<DT>(x + r * p.ldx, c) - s.x, s.y * gain, bias);
        store_elem<DT>(y + r * p.ldy, c, activate<DT>(v, p.act));
    }
}

// dz and u of a thread's chunk
template <int DT>
__device__ inline void gradient_of(const Norm& p, const Channels<DT>& ch, const char* x, const char* dy, const Place& at, float (&u)[8], float (&dz)[8]) {
    load8<DT>(x, at.channel, at.count, u);
    load8<DT>(dy, at.channel, at.count, dz);
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = (u[j] - ch.mean[j]) * ch.scale[j];
    if (p.act == SC_ACT_NONE) return;
    if (p.act == SC_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) dz[j] *= slope<DT>(fmaf(u[j], ch.gain[j], ch.bias[j]), SC_ACT_RELU);
    } else if (p.act == SC_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) dz[j] *= slope<DT>(fmaf(u[j], ch.gain[j], ch.bias[j]), SC_ACT_GELU);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) dz[j] *= slope<DT>(fmaf(u[j], ch.gain[j], ch.bias[j]), SC_ACT_SILU);
    }
}
template <int DT>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm_grad_sums(const Norm p) {
    const int slice = blockIdx.y, width = p.C - slice * SLICE < SLICE ? p.C - slice * SLICE : SLICE;
    float2* const sums = p.sums + (int64_t)blockIdx.x * p.C + slice * SLICE;
    const NormUnit unit = unit_of(p, blockIdx.x);
    if (unit.rows == 0) {                                              // counts in the sums over all units
        for (int c = threadIdx.x; c < width; c += NORM_THREADS) sums[c] = make_float2(0.f, 0.f);
        return;
    }
    const Place at(p, slice);
    const Channels<DT> ch(p, at, unit.scene);
    float sum[8], along[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = along[j] = 0.f;
#pragma unroll 2
    for (int r = at.row; r < unit.rows; r += at.step) {
        float u[8], dz[8];
        gradient_of<DT>(p, ch, p.x + (unit.first + r) * p.ldx, p.dy + (unit.first + r) * p.lddy, at, u, dz);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[j] += dz[j];
            along[j] = fmaf(dz[j], u[j], along[j]);
        }
    }
    join_threads(sum, along, width, [&](int c, float a, float b) { sums[c] = make_float2(a, b); });
}
// The gradients of 16 channels' gain and bias from the sums of all units, by a workgroup.
template <int DT, int THREADS>
__device__ inline void join_gains(const Norm& p, int first) {
    constexpr int SHARES = THREADS / 16;
    __shared__ double shared[2][SHARES][16];
    const int c = first + (threadIdx.x & 15), which = threadIdx.x >> 4;
    double sum = 0.0, along = 0.0;
    if (c < p.C) {
#pragma unroll 8
        for (int64_t u = which; u < p.units; u += SHARES) {
            const float2 s = p.sums[u * p.C + c];
            sum += s.x;
            along += s.y;
        }
    }
    shared[0][which][threadIdx.x & 15] = sum;
    shared[1][which][threadIdx.x & 15] = along;
    __syncthreads();
    if (which != 0 || c >= p.C) return;
    sum = along = 0.0;
#pragma unroll 8
    for (int w = 0; w < SHARES; ++w) {
        sum += shared[0][w][threadIdx.x];
        along += shared[1][w][threadIdx.x];
    }
    if (p.dbias != nullptr) store_elem<DT>(p.dbias, c, (float)sum);
    if (p.dgain != nullptr) store_elem<DT>(p.dgain, c, (float)along);
}
// The means of a scene's group, and in the workgroups behind `pair_blocks` the gradients of the gains.
template <int DT, int THREADS>
__global__ void __launch_bounds__(THREADS == WAVE ? 256 : THREADS)
k_norm_grad_join(const Norm p, int pair_blocks) {
    if ((int)blockIdx.x >= pair_blocks) {
        join_gains<DT, THREADS == WAVE ? 256 : THREADS>(p, ((int)blockIdx.x - pair_blocks) * 16);
        return;
    }
    const int pair = pair_of_threads<THREADS>(), tid = (int)threadIdx.x % THREADS;
    if (pair >= p.scenes * p.groups) return;
    const int scene = pair / p.groups, group = pair - scene * p.groups;
    int64_t unit = 0;
    int rows = 0;
    scene_units_of(p, scene, unit, rows);
    const int units = (rows + p.per - 1) / p.per;
    const float2* const sums = p.sums + unit * p.C + group * p.channels;
    double sum = 0.0, along = 0.0;
    const int64_t items = (int64_t)units * p.channels;
#pragma unroll 4
    for (int64_t i = tid; i < items; i += THREADS) {
        const int u = (int)((uint32_t)i / (uint32_t)p.channels), c = (int)(i - (int64_t)u * p.channels);
        const float2 s = sums[(int64_t)u * p.C + c];
        const double gain = p.gain != nullptr ? load_elem<DT>(p.gain, group * p.channels + c) : 1.f;
        sum += gain * s.x;
        along += gain * s.y;
    }
    sum_of_threads<THREADS>(sum, along);
    const double n = (double)rows * p.channels;
    if (tid == 0) p.means[pair] = rows > 0 ? make_float2((float)(sum / n), (float)(along / n)) : make_float2(0.f, 0.f);
}
template <int DT>
__global__ void __launch_bounds__(NORM_THREADS)
k_norm_grad(const Norm p) {
    const NormUnit unit = unit_of(p, p.units - 1 - blockIdx.x);
    if (unit.rows == 0) return;
    const Place at(p, blockIdx.y);
    if (at.row >= unit.rows) return;
    const Channels<DT> ch(p, at, unit.scene);
    float mean[8], along[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float2 m = p.means[(int64_t)unit.scene * p.groups + ch.group[j]];
        mean[j] = m.x;
        along[j] = m.y;
    }
#pragma unroll 2
    for (int r = at.row; r < unit.rows; r += at.step) {
        float u[8], dz[8];
        gradient_of<DT>(p, ch, p.x + (unit.first + r) * p.ldx, p.dy + (unit.first + r) * p.lddy, at, u, dz);
#pragma unroll
        for (int j = 0; j < 8; ++j) dz[j] = (fmaf(dz[j], ch.gain[j], -mean[j]) - u[j] * along[j]) * ch.scale[j];
        store8<DT>(p.y + (unit.first + r) * p.ldy, at.channel, at.count, dz);
    }
}

bool sizes_ok(int64_t rows, int scenes, int C, int groups) {
    return rows >= 0 && rows <= SC_N_MAX && scenes >= 1 && scenes <= SC_SCENES_MAX && C >= 1 && C <= SC_CHANNELS_MAX && groups >= 1 && groups <= C && C % groups == 0 &&
           (int64_t)scenes * groups <= SC_NORM_PAIRS_MAX;
}
bool rows_ok(const void* p, int64_t ld, int C, int dtype, int64_t rows) {
    return (rows == 0 || p != nullptr) && ((uintptr_t)p & (dtype == SC_F32 ? 3 : 1)) == 0 && ld >= C && ld <= SC_LD_MAX;
}
int check_norm(int64_t rows, const int32_t* starts, int scenes, int C, int groups, const void* gain, const void* bias, int act, int dtype) {
    if (dtype != SC_F32 && dtype != SC_F16 && dtype != SC_BF16) return SC_EINVAL;
    if (!sizes_ok(rows, scenes, C, groups) || act < SC_ACT_NONE || act > SC_ACT_SILU) return SC_EINVAL;
    if (((uintptr_t)starts & 3) != 0 || (starts == nullptr && scenes != 1)) return SC_EINVAL;
    const uintptr_t off = dtype == SC_F32 ? 3 : 1;
    return ((uintptr_t)gain & off) != 0 || ((uintptr_t)bias & off) != 0 ? SC_EINVAL : SC_OK;
}
size_t up16(size_t n) { return (n + 15) / 16 * 16; }
int slices_of(int C) { return (C + SLICE - 1) / SLICE; }

template <int DT>
int launch_norm(const Norm& p, bool few, hipStream_t s) {
    const int pairs = p.scenes * p.groups;
    if (few) {
        if (norm_few_threads(p.rows, p.channels, p.scenes) == 256) SC_LAUNCH(KID_NORM, (k_norm_few<DT, 256>), dim3((unsigned)pairs), dim3(256), 0, s, p);
        else SC_LAUNCH(KID_NORM, (k_norm_few<DT, 1024>), dim3((unsigned)pairs), dim3(1024), 0, s, p);
        return SC_OK;
    }
    const dim3 grid((unsigned)p.units, (unsigned)slices_of(p.C));
    SC_LAUNCH(KID_NORM_SUMS, k_norm_sums<DT>, grid, dim3(NORM_THREADS), 0, s, p);
    if (norm_join_by_wavefronts(pairs)) SC_LAUNCH(KID_NORM_JOIN, k_norm_join<WAVE>, dim3((unsigned)(pairs + 3) / 4), dim3(256), 0, s, p);
    else SC_LAUNCH(KID_NORM_JOIN, k_norm_join<JOIN_THREADS>, dim3((unsigned)pairs), dim3(JOIN_THREADS), 0, s, p);
    SC_LAUNCH(KID_NORM, k_norm<DT>, grid, dim3(NORM_THREADS), 0, s, p);
    return SC_OK;
}
template <int DT>
int launch_norm_grad(const Norm& p, hipStream_t s) {
    const int pairs = p.scenes * p.groups;
    const dim3 grid((unsigned)p.units, (unsigned)slices_of(p.C));
    SC_LAUNCH(KID_NORM_SUMS, k_norm_grad_sums<DT>, grid, dim3(NORM_THREADS), 0, s, p);
    const int gains = p.dgain != nullptr || p.dbias != nullptr ? (p.C + 15) / 16 : 0, by_wavefronts = (pairs + 3) / 4;
    if (norm_join_by_wavefronts(pairs))
        SC_LAUNCH(KID_NORM_JOIN, (k_norm_grad_join<DT, WAVE>), dim3((unsigned)(by_wavefronts + gains)), dim3(256), 0, s, p, by_wavefronts);
    else
        SC_LAUNCH(KID_NORM_JOIN, (k_norm_grad_join<DT, JOIN_THREADS>), dim3((unsigned)(pairs + gains)), dim3(JOIN_THREADS), 0, s, p, pairs);
    if (p.y != nullptr) SC_LAUNCH(KID_NORM_GRAD, k_norm_grad<DT>, grid, dim3(NORM_THREADS), 0, s, p);
    return SC_OK;
}
}  // namespace
}  // namespace sc

using namespace sc;

extern "C" size_t sc_group_norm_workspace_bytes(int64_t rows, int scenes, int C, int groups) {
    if (!sizes_ok(rows, scenes, C, groups)) return 0;
    const int64_t units = scene_units(rows, scenes, norm_rows(rows, C));
    return up16((size_t)units * C * sizeof(float2)) + up16((size_t)scenes * groups * sizeof(float2));
}

extern "C" int sc_group_norm_fwd(const void* d_x, int64_t ldx, int64_t rows, const int32_t* d_starts, int scenes, int C, int groups, const void* d_gain,
                                 const void* d_bias, float eps, int act, void* d_y, int64_t ldy, float* d_stats, int dtype, void* d_workspace, size_t workspace_bytes,
                                 void* stream) {
    const int rc = check_norm(rows, d_starts, scenes, C, groups, d_gain, d_bias, act, dtype);
    if (rc != SC_OK) return rc;
    if (!rows_ok(d_x, ldx, C, dtype, rows) || !rows_ok(d_y, ldy, C, dtype, rows) || ((uintptr_t)d_stats & 7) != 0 || !(eps > 0.f) || eps > 3.0e38f) return SC_EINVAL;
    if (d_workspace == nullptr || !aligned16(d_workspace)) return SC_EINVAL;
    if (workspace_bytes < sc_group_norm_workspace_bytes(rows, scenes, C, groups)) return SC_ECAP;
    const int size = dtype == SC_F32 ? 4 : 2;
    Norm p{};
    p.x = (const char*)d_x;
    p.y = (char*)d_y;
    p.ldx = ldx * size;
    p.ldy = ldy * size;
    p.rows = rows;
    p.starts = d_starts;
    p.scenes = scenes;
    p.C = C;
    p.groups = groups;
    p.channels = C / groups;
    p.gain = d_gain;
    p.bias = d_bias;
    p.eps = eps;
    p.act = act;
    p.per = norm_rows(rows, C);
    p.per_log2 = __builtin_ctz(p.per);
    p.units = scene_units(rows, scenes, p.per);
    p.sums = (float2*)d_workspace;
    p.stats = d_stats != nullptr ? (float2*)d_stats : (float2*)((char*)d_workspace + up16((size_t)p.units * C * sizeof(float2)));
    const bool few = norm_few(rows, p.channels) && (int64_t)scenes * groups <= NORM_FEW_PAIRS_MAX;
    hipStream_t s = (hipStream_t)stream;
    return dtype == SC_F32 ? launch_norm<SC_F32>(p, few, s) : dtype == SC_F16 ? launch_norm<SC_F16>(p, few, s) : launch_norm<SC_BF16>(p, few, s);
}

extern "C" int sc_group_norm_bwd(const void* d_dy, int64_t lddy, const void* d_x, int64_t ldx, int64_t rows, const int32_t* d_starts, int scenes, int C, int groups,
                                 const void* d_gain, const void* d_bias, int act, const float* d_stats, void* d_dx, int64_t lddx, void* d_dgain, void* d_dbias, int dtype,
                                 void* d_workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_norm(rows, d_starts, scenes, C, groups, d_gain, d_bias, act, dtype);
    if (rc != SC_OK) return rc;
    const uintptr_t off = dtype == SC_F32 ? 3 : 1;
    if (!rows_ok(d_x, ldx, C, dtype, rows) || !rows_ok(d_dy, lddy, C, dtype, rows) || d_stats == nullptr || ((uintptr_t)d_stats & 7) != 0) return SC_EINVAL;
    if (d_dx == nullptr && d_dgain == nullptr && d_dbias == nullptr) return SC_EINVAL;
    if (d_dx != nullptr && !rows_ok(d_dx, lddx, C, dtype, rows)) return SC_EINVAL;
    if (((uintptr_t)d_dgain & off) != 0 || ((uintptr_t)d_dbias & off) != 0) return SC_EINVAL;
    if (d_workspace == nullptr || !aligned16(d_workspace)) return SC_EINVAL;
    if (workspace_bytes < sc_group_norm_workspace_bytes(rows, scenes, C, groups)) return SC_ECAP;
    const int size = dtype == SC_F32 ? 4 : 2;
    Norm p{};
    p.x = (const char*)d_x;
    p.dy = (const char*)d_dy;
    p.y = (char*)d_dx;
    p.ldx = ldx * size;
    p.lddy = lddy * size;
    p.ldy = lddx * size;
    p.rows = rows;
    p.starts = d_starts;
    p.scenes = scenes;
    p.C = C;
    p.groups = groups;
    p.channels = C / groups;
    p.gain = d_gain;
    p.bias = d_bias;
    p.dgain = d_dgain;
    p.dbias = d_dbias;
    p.act = act;
    p.stats = (float2*)const_cast<float*>(d_stats);
    p.per = norm_rows(rows, C);
    p.per_log2 = __builtin_ctz(p.per);
    p.units = scene_units(rows, scenes, p.per);
    p.sums = (float2*)d_workspace;
    p.means = (float2*)((char*)d_workspace + up16((size_t)p.units * C * sizeof(float2)));
    hipStream_t s = (hipStream_t)stream;
    return dtype == SC_F32 ? launch_norm_grad<SC_F32>(p, s) : dtype == SC_F16 ? launch_norm_grad<SC_F16>(p, s) : launch_norm_grad<SC_BF16>(p, s);
}
