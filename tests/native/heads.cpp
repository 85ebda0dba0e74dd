// heads_meet() of sc_heads.h against sets of elements: it never says that operands meet which have no element in common, finds all that do of those with the same
// strides, and all that begin at the same place.  The program prints the first case that does not hold and ends with 1.
#include <cstdio>
#include <random>
#include <set>

#include "sc_heads.h"

using namespace sc;

int main() {
    std::mt19937_64 rng(5);
    auto below = [&](int64_t n) { return (int64_t)(rng() % (uint64_t)n); };
    int met = 0, apart = 0, missed = 0;
    for (int i = 0; i < 200000; ++i) {
        const int dtype = i % 2 ? SC_F32 : SC_F16, size = dtype == SC_F32 ? 4 : 2;
        const int D = 1 + (int)below(6);
        sc_heads a{}, b{};
        const int64_t a_rows = below(5), b_rows = below(5);
        a.heads = (int32_t)(1 + below(4));
        b.heads = (int32_t)(1 + below(4));
        auto strides = [&](sc_heads& h) {
            h.head = i % 3 == 0 ? below(12) : D * (1 + below(4));                       // of inputs that share elements, of slices
            h.row = i % 3 == 0 ? below(40) : i % 3 == 1 ? h.head * (1 + below(6)) : D * below(8);
        };
        strides(a);
        strides(b);
        const bool alike = i % 5 < 3;
        if (alike) {
            b.row = a.row;
            b.head = a.head;
        }
        const int64_t first = 1000 + below(60) * (i % 7 ? D : 1), second = 1000 + below(60) * (i % 7 ? D : 1);
        a.data = (void*)(uintptr_t)(first * size);
        b.data = (void*)(uintptr_t)(second * size);
        std::set<int64_t> elements;
        for (int64_t r = 0; r < a_rows; ++r)
            for (int64_t h = 0; h < a.heads; ++h)
                for (int64_t c = 0; c < D; ++c) elements.insert(first + r * a.row + h * a.head + c);
        bool common = false;
        for (int64_t r = 0; r < b_rows; ++r)
            for (int64_t h = 0; h < b.heads; ++h)
                for (int64_t c = 0; c < D; ++c) common = common || elements.count(second + r * b.row + h * b.head + c) != 0;
        const bool says = heads_meet(&a, a_rows, &b, b_rows, D, dtype);
        if (says != heads_meet(&b, b_rows, &a, a_rows, D, dtype) || (says && !common) || (common && !says && (alike || first == second))) {
            std::printf("says %d, has %d: rows %d heads %d strides %d %d at %d, rows %d heads %d strides %d %d at %d, D %d\n", says, common, (int)a_rows, a.heads, (int)a.row,
                        (int)a.head, (int)first, (int)b_rows, b.heads, (int)b.row, (int)b.head, (int)second, D);
            return 1;
        }
        met += says;
        apart += !common;
        missed += common && !says;
    }
    std::printf("%d meet, %d do not, %d not found\n", met, apart, missed);
    return met > 10000 && apart > 10000 ? 0 : 1;       // a twentieth of the cases each, or they say little
}
