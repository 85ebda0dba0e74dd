// Units by which a bias' gradient is summed ahead of its rounding: every unit of every group has a place of its own inside what is set aside for them, and a part of a
// weight gradient is a whole number of units.  The program prints the first thing that does not hold and ends with 1.
#include <cstdio>
#include <random>
#include <vector>

#include "sc_rules.h"

using namespace sc;

static_assert(bias_log2(true, TILE_16_32) == 2 && bias_log2(true, TILE_32_64) == 2 && bias_log2(true, TILE_128_32) == 5 && bias_log2(false, TILE_16_32) == 6, "units");
static_assert(sum_columns(1, 64) == 4 && sum_columns(47, 128) == 8 && sum_columns(128, 64) == 16 && sum_columns(266, 64) == 32 && sum_columns(5000, 3) == 3, "columns");
static_assert(sum_threads(4) == 256 && sum_threads(8) == 512 && sum_threads(32) == 512 && sum_threads(20) == 448 && sum_threads(24) == 384 && sum_threads(3) == 192 && sum_threads(1) == 64, "threads");

int main() {
    std::mt19937_64 rng(2);
    for (int round = 0; round < 3000; ++round) {
        const int groups = 1 + (int)(rng() % (round % 5 ? 40 : 1));
        std::vector<int64_t> starts{(int64_t)(rng() % 7)};
        for (int g = 0; g < groups; ++g) starts.push_back(starts.back() + (rng() % 3 ? rng() % (round % 2 ? 700 : 9) : 0));
        const int64_t n = starts.back() + rng() % 5;
        for (const int log2 : {2, 5, 6}) {
            std::vector<char> taken(bias_units(n, groups, log2), 0);
            for (int g = 0; g < groups; ++g)
                for (int64_t e = starts[g]; e < starts[g + 1]; e += 1 << log2) {
                    const int64_t at = (e >> log2) + g;
                    if (at >= (int64_t)taken.size() || taken[at]++) {
                        std::printf("entry %lld of group %d of %d, units of %d: place %lld of %lld\n", (long long)e, g, groups, 1 << log2, (long long)at, (long long)taken.size());
                        return 1;
                    }
                }
        }
        const int64_t c_in = 1 + rng() % 700, c_out = 1 + rng() % 700, part = weight_part(n, c_in, c_out);
        if (part % 64 != 0) {
            std::printf("a part of %lld\n", (long long)part);
            return 1;
        }
        const int64_t chunks = 1 + rng() % 300, wide = sum_columns(1 + rng() % 3000, chunks);
        if (wide < 1 || wide > 32 || wide > chunks || sum_threads(wide) > 512 || sum_threads(wide) < wide) {
            std::printf("%lld of %lld chunks\n", (long long)wide, (long long)chunks);
            return 1;
        }
    }
    return 0;
}
