// What the kernels of attention and of the group norm take for granted of the rules in sc_rules.h, and sides of their lines: the program
// prints the first thing that does not hold and ends with 1.
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>

#include "sc_rules.h"

using namespace sc;

static_assert(attention_shape(8, 1, 8, 77, 64) == ATTENTION_FEW && attention_shape(32, 8, 4, 262144, 256) == ATTENTION_WIDE, "few rows, and few over long caches");
static_assert(attention_shape(53373, 1112, 8, 53373, 64) == ATTENTION_SHORT_64 && attention_shape(2048, 42, 8, 2048, 128) == ATTENTION_SHORT &&
              attention_shape(65536, 3, 4, 16384, 256) == ATTENTION_WIDE, "windows, sequences");
static_assert(attention_parts(ATTENTION_FEW, 8, 1, 8, 77, false) == 1 && attention_parts(ATTENTION_WIDE, 32, 8, 4, 262144, false) == 31 &&
              attention_parts(ATTENTION_WIDE, 65536, 64, 8, 262144, false) == 1, "parts");
static_assert(attention_grad_alone(110545, 2303, 8, 110545, 64, false) && !attention_grad_alone(65536, 4, 4, 16384, 128, false) && attention_grad_alone(4503, 7, 2, 1501, 128, true), "alone");
static_assert(norm_rows(261574, 64) == 256 && norm_rows(110545, 256) == 64 && norm_rows(3001, 45) == 64 && norm_rows(67108864, 8) <= 67108864, "rows of a unit");
static_assert(norm_few(33, 8) && !norm_few(261574, 8), "few rows");
static_assert(norm_few_threads(898, 8, 1) == 1024 && norm_few_threads(33, 8, 1) == 256 && norm_few_threads(1000, 8, 16) == 256, "threads of a group");

#define HOLDS(what)                                                                            \
    if (!(what)) {                                                                             \
        std::printf("%s: rows %lld scenes %lld\n", #what, (long long)rows, (long long)scenes);  \
        return 1;                                                                              \
    }

int main() {
    std::mt19937_64 rng(3);
    auto up_to = [&](int64_t most) { return 1 + (int64_t)(std::exp2(std::uniform_real_distribution<>(0, std::log2((double)most))(rng)) - 1); };
    for (int i = 0; i < 20000; ++i) {
        const int64_t rows = up_to(67108864), scenes = up_to(i % 3 ? 4096 : 67108864), heads = up_to(64), per = up_to(16), keys = up_to(67108864);
        const int bytes = 64 << rng() % 5;
        const bool f32 = rng() & 1;
        const AttentionShape shape = attention_shape(rows * per, scenes, heads, keys, bytes);
        const int parts = attention_parts(shape, rows * per, scenes, heads, keys, f32);
        HOLDS(parts >= 1 && parts <= ATTENTION_PARTS_MAX && attention_part_keys(f32) > 0);
        const bool alone = attention_grad_alone(rows * per, scenes, heads, keys, bytes, f32);
        const int grad_parts = attention_grad_parts(alone, keys, scenes, heads, rows * per, f32);
        HOLDS(grad_parts >= 1 && grad_parts <= ATTENTION_GRAD_PARTS_MAX && attention_part_rows(alone, f32) > 0);
        const int chunk_rows = norm_rows(rows, (int)up_to(65536));
        HOLDS(chunk_rows >= 1 && (chunk_rows & (chunk_rows - 1)) == 0 && rows / chunk_rows <= 4096 + 65536);
    }
    // a scene's units, from its start's on, hold its tiles and end where the next one's begin
    for (int i = 0; i < 2000; ++i) {
        const int64_t scenes = up_to(200), per = up_to(12), tile = (int64_t)1 << (2 + rng() % 8);
        std::vector<int64_t> starts{(int64_t)(rng() % 50)};
        for (int64_t s = 0; s < scenes; ++s) starts.push_back(starts.back() + (rng() % 4 ? (int64_t)(rng() % 300) : 0));
        const int64_t rows = starts.back() + (int64_t)(rng() % 9);
        for (int64_t s = 0; s < scenes; ++s) {
            const int64_t first = starts[s] * per / tile + s, next = starts[s + 1] * per / tile + s + 1;
            HOLDS(next - first >= ((starts[s + 1] - starts[s]) * per + tile - 1) / tile);
            HOLDS(next <= scene_units(rows * per, scenes, tile));
        }
    }
    // columns' rows by a multiplication
    for (uint64_t per = 2; per <= 65536; per = per < 300 ? per + 1 : per * 3 / 2) {
        const int64_t rows = (int64_t)per, scenes = 0;
        int log2 = 1;
        while ((uint64_t)1 << log2 < per) ++log2;
        const uint64_t magic = (((uint64_t)1 << (31 + log2)) + per - 1) / per;
        HOLDS(magic < (uint64_t)1 << 32);
        for (int i = 0; i < 2000; ++i) {
            const uint64_t c = i == 0 ? 2147483647u : i % 2 ? rng() % 2147483648u : (rng() % (2147483648u / per)) * per + (i % 4 ? 0 : per - 1);
            if (c < 2147483648u) HOLDS((c * magic >> 32) >> (log2 - 1) == c / per);
        }
    }
    return 0;
}
