// Parts of a weight gradient at the largest sizes that the calls take: a part's entries have to fit the 32 bits in which the kernels divide by them, and a group
// that one part holds must not seem to have several.  The program prints the first thing that does not hold and ends with 1.
#include <cstdio>
#include <initializer_list>

#include "sc_rules.h"

using namespace sc;

int main() {
    struct Size {
        int64_t n, c_in, c_out;
    };
    const Size sizes[] = {{2147483647, 4096, 4096}, {536870912, 8192, 8192}, {8388608, 65536, 65536}, {9000000, 65536, 65536}, {2147483647, 65536, 65536},
                          {2147483647, 1, 1}, {2147483647, 128, 128}, {200, 65536, 65536}, {129, 4096, 4096}, {128, 64, 64}, {1, 65536, 1}};
    for (const Size& s : sizes) {
        const int64_t part = weight_part(s.n, s.c_in, s.c_out), slots = weight_slots(s.n, part);
        const uint32_t step = (uint32_t)part;
        const bool fits = step == part && part >= 128 && part % 64 == 0;
        // the parts that the kernels count of groups of all entries, of half of them, of one
        bool counted = fits;
        for (const int64_t e : {s.n, s.n / 2, (int64_t)1})
            counted = counted && (int64_t)((uint32_t)e / step + ((uint32_t)e % step != 0)) == (e + part - 1) / part && (e > part || (e + part - 1) / part <= 1);
        if (!counted || (s.n <= part) != (slots == 0)) {
            std::printf("%lld x %lld x %lld: parts of %lld, %lld slots\n", (long long)s.n, (long long)s.c_in, (long long)s.c_out, (long long)part, (long long)slots);
            return 1;
        }
    }
    return 0;
}
