// Rows packed scene by scene: which scene a unit of work belongs to (sc_attention.h, sc_norm.hip).
#pragma once

#include "sc_internal.h"

namespace sc {

struct Scene {
    int64_t q0, k0;                    // first rows
    int nq, nk;
    int tile;                          // of the scene's columns; -1: none
};
__device__ inline int64_t clamp_row(int64_t v, int64_t rows) { return v < 0 ? 0 : v > rows ? rows : v; }

// Unit u of the scenes' columns cut into tiles of 2^log2 columns, `per` columns a row.  Scene s has the units from A(s) = start(s) per / 2^log2 + s on: at least as many as
// it has tiles, one too many at most, so the host knows how many units there can be without the starts (`units`), and the device finds a unit's scene by a search
// 63 wide: one trip to memory up to 63 scenes; with more of them the first one looks about the place that scenes of equal length would give, and mostly finds it there, else two
// more do up to 3969.  Called by whole wavefronts.  Starts that do not ascend give wrong scenes, but never rows outside [0, rows).
__device__ inline Scene find_scene(const int32_t* __restrict__ starts, int scenes, int64_t rows, int per, int log2, int64_t u, int64_t units, int64_t& first, int& count, int& scene) {
    Scene found{0, 0, 0, 0, -1};
    const int lane = threadIdx.x & 63;
    scene = 0;
    if (starts == nullptr) {
        first = 0;
        count = (int)rows;
        if (u << log2 < rows * per) found.tile = (int)u;
        return found;
    }
    int lo = 0, hi = scenes;
    bool guess = scenes > 63;
    if (guess) {
        lo = (int)((float)u / (float)units * (float)scenes) - 31;
        lo = lo < 0 ? 0 : lo > scenes - 63 ? scenes - 63 : lo;
        hi = lo + 63;
    }
    for (;;) {
        const int step = (hi - lo + 62) / 63, s = lo + lane * step;
        int start = 0;
        bool below = false;
        if (s < hi || (s == hi && step == 1)) {
            start = (int)clamp_row(starts[s], rows);
            below = ((int64_t)start * per >> log2) + s <= u;
        }
        const uint64_t vote = __ballot(below);
        if (guess && ((vote & 1) == 0 || (vote >> 63 != 0 && hi < scenes))) {      // before these, or behind them
            guess = false;
            if ((vote & 1) == 0) hi = lo;
            else lo = hi;
            if ((vote & 1) == 0) lo = 0;
            else hi = scenes;
            if (lo >= hi) return found;
            continue;
        }
        int n = __popcll(vote);
        if (step == 1 && n > hi - lo) n = hi - lo;
        if (n == 0) return found;
        if (step == 1) {
            const int begin = __builtin_amdgcn_readlane(start, n - 1), stop = __builtin_amdgcn_readlane(start, n);
            scene = lo + n - 1;
            first = begin;
            count = stop > begin ? stop - begin : 0;
            const int64_t nth = u - (((int64_t)begin * per >> log2) + scene);
            if (nth >= 0 && nth << log2 < (int64_t)count * per) found.tile = (int)nth;
            return found;
        }
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
}
__device__ inline void scene_rows(const int32_t* __restrict__ starts, const int32_t* __restrict__ lens, int64_t rows, int scene, int64_t& first, int& count) {
    if (starts == nullptr) {
        first = 0;
        count = (int)rows;
    } else {
        first = clamp_row(starts[scene], rows);
        const int64_t stop = clamp_row(starts[scene + 1], rows);
        count = (int)(stop > first ? stop - first : 0);
    }
    if (lens != nullptr) {
        const int n = lens[scene];
        count = n < 0 ? 0 : n < count ? n : count;
    }
}
__device__ inline int64_t uniform64(int64_t v) {
    return ((int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}
}  // namespace sc
