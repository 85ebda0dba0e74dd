// Sides of the lines between the tiles of products of rows in sc_rules.h, and what the launches take for granted of the rules: the
// program prints the first thing that does not hold and ends with 1.
#include <cmath>
#include <cstdio>
#include <random>

#include "sc_rules.h"

using namespace sc;

// a row of few workgroups, ordinary layers, large ones; 256 compute units
static_assert(row_tile(1, 0, 4096, 1024, true, true, 256) == TILE_16_32_DEEP && row_tile(128, 0, 2048, 2048, true, true, 256) == TILE_16_32, "few rows");
static_assert(row_tile(1024, 0, 256, 256, true, true, 256) == TILE_16_32 && row_tile(512, 0, 1024, 1024, true, true, 256) == TILE_32_64, "hundreds of rows");
static_assert(row_tile(2048, 0, 1024, 1024, true, true, 256) == TILE_64_64_DEEP && row_tile(8192, 0, 512, 128, true, true, 256) == TILE_64_64, "thousands");
static_assert(row_tile(53373, 0, 256, 64, true, true, 256) == TILE_128_64 && row_tile(200000, 0, 32, 128, true, true, 256) == TILE_128_32, "narrow");
static_assert(row_tile(110545, 0, 256, 256, true, true, 256) == TILE_128_128_SHORT && row_tile(110545, 0, 128, 512, true, true, 256) == TILE_128_128, "long");
static_assert(row_tile(32768, 0, 512, 512, true, true, 256) == TILE_LARGE && row_tile(32768, 0, 512, 512, true, false, 256) == TILE_128_128, "large: 16-bit only");
static_assert(row_tile(8192, 0, 1024, 1024, true, true, 256) == TILE_128_128, "large: two workgroups per compute unit");
static_assert(row_tile(53373, 8, 512, 128, true, true, 256) == TILE_128_128_SHORT && row_tile(53373, 8, 256, 1024, false, true, 256) == TILE_LARGE &&
              row_tile(53373, 8, 128, 512, false, true, 256) == TILE_128_128, "groups");
static_assert(row_tile(1024, 0, 256, 256, true, true, 64) == TILE_32_64 && row_tile(2048, 0, 256, 256, true, true, 64) == TILE_64_64, "per compute unit");
static_assert(product_run(1, 64) == 1 && product_run(2048, 4) == 4 && product_run(64, 8) == 8 && product_run(8, 16) == 2, "runs");
static_assert(weight_tile(64, 64) == WEIGHTS_64_64 && weight_tile(32, 2048) == WEIGHTS_64_64 && weight_tile(64, 65) == WEIGHTS_64_128 &&
              weight_tile(256, 64) == WEIGHTS_128_64 && weight_tile(65, 65) == WEIGHTS_128_128, "weight tiles");
static_assert(weight_part(4000, 256, 256) == 128 && weight_part(53373, 128, 128) == 256 && weight_part(53373, 64, 64) == 128 && weight_part(110545, 128, 512) == 896, "parts");
static_assert(act_in_product(300000, 1, 32, 128, 256) && !act_in_product(53373, 1, 64, 256, 256) && act_in_product(1000, 1, 64, 256, 256) && !act_in_product(64, 1, 512, 512, 256), "slopes");
static_assert(act_grad_rows(3192, 20) == 13 && act_grad_rows(110545, 64) == 32 && act_grad_rows(1, 1000) == 1, "rows of a workgroup");

#define HOLDS(what)                                                                                     \
    if (!(what)) {                                                                                      \
        std::printf("%s: n %lld groups %lld c_in %lld c_out %lld\n", #what, (long long)n, (long long)groups, (long long)c_in, (long long)c_out); \
        return 1;                                                                                       \
    }

int main() {
    std::mt19937_64 rng(1);
    auto up_to = [&](int64_t most) { return 1 + (int64_t)(std::exp2(std::uniform_real_distribution<>(0, std::log2((double)most))(rng)) - 1); };
    for (int i = 0; i < 20000; ++i) {
        const int64_t n = up_to(i % 4 ? 3000000 : 2147483647), groups = i % 3 ? up_to(65536) : 1, c_in = up_to(i % 5 ? 700 : 65536), c_out = up_to(i % 7 ? 700 : 65536);
        const int64_t part = weight_part(n, c_in, c_out), slots = weight_slots(n, part);
        HOLDS(part >= 128 && part % 64 == 0 && slots >= 0);
        // groups that are cut have room for their parts, the sizes that need most of it among them: one entry more than a part
        int64_t left = n, taken = 0;
        for (int64_t g = 0; g < groups && left > 0; ++g) {
            const int64_t most = i % 2 ? part + 1 : up_to(left), e = g + 1 == groups ? left : most < left ? most : left, parts = (e + part - 1) / part;
            taken += parts > 1 ? parts : 0;
            left -= e;
        }
        HOLDS(taken <= slots);
        // the rows of a workgroup of the activation's gradient
        const int64_t chunks = (c_out + 7) / 8, rows = act_grad_rows(n, chunks);
        HOLDS(rows >= 1 && (rows * chunks <= 2048 || rows == 1) && (n + rows - 1) / rows <= 2147483647);
        // slopes inside the product: only the tiles that have it
        if (act_in_product(n, groups, c_in, c_out, 256)) {
            const RowTile t = row_tile(n, groups, c_in, c_out, false, false, 256), linear = row_tile(n, 0, c_in, c_out, false, false, 256);
            HOLDS(t == TILE_16_32 || t == TILE_32_64 || t == TILE_128_32);
            HOLDS(groups > 1 || linear == TILE_16_32 || linear == TILE_32_64 || linear == TILE_128_32);
        }
        const bool forward = rng() & 1, half = rng() & 1;
        const RowTile t = row_tile(n, i % 3 ? groups : 0, c_out, c_in, forward, half, 256);
        HOLDS(t != TILE_LARGE || half);
        HOLDS(t != TILE_128_128_SHORT || forward);
        HOLDS(product_run(n, c_out) >= 1 && product_run(n, c_out) <= c_out);
    }
    return 0;
}
