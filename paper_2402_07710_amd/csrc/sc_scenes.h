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

// Unit u of the scenes' columns cut into tiles of `tile` columns, `per` columns a row.  Scene s has the units from A(s) = start(s) per / tile + s on: at least as many as
// it has tiles, one too many at most, so the host knows how many units there can be without the starts, and the device finds a unit's scene by a search
// 64 wide, one trip to memory up to 64 scenes and two up to 4096.  Called by whole wavefronts.  Starts that do not ascend give wrong scenes, but never rows outside [0, rows).
__device__ inline Scene find_scene(const int32_t* __restrict__ starts, int scenes, int64_t rows, int per, int tile, int64_t u, int64_t& first, int& count, int& scene) {
    Scene none{0, 0, 0, 0, -1};
    const int lane = threadIdx.x & 63;
    scene = 0;
    if (starts == nullptr) {
        first = 0;
        count = (int)rows;
        if (u * tile >= rows * per) return none;
        none.tile = (int)u;
        return none;
    }
    int lo = 0, hi = scenes;
    int64_t at_lo = 0;
    bool found = false;
    while (!found || hi - lo > 1) {
        const int step = (hi - lo + 63) / 64;
        const int s = lo + lane * step;
        int64_t at = 0;
        bool below = false;
        if (s < hi) {
            at = clamp_row(starts[s], rows) * per / tile + s;
            below = at <= u;
        }
        const int n = __popcll(__ballot(below));
        if (n == 0) return none;
        at_lo = ((int64_t)__builtin_amdgcn_readlane((int)(at >> 32), n - 1) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)at, n - 1);
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
        found = true;
    }
    scene = lo;
    first = clamp_row(starts[lo], rows);
    const int64_t stop = clamp_row(starts[lo + 1], rows);
    count = (int)(stop > first ? stop - first : 0);
    const int64_t nth = u - at_lo;
    if (nth < 0 || nth * tile >= (int64_t)count * per) return none;
    none.tile = (int)nth;
    return none;
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
