// Checks of heads given from outside, for the calls that take queries and keys (sc_rope.hip, sc_attention.hip).
#pragma once

#include "sc_internal.h"

namespace sc {

inline bool heads_ok(const sc_heads* h, int dtype) {
    const int size = dtype == SC_F32 ? 4 : 2;
    return h != nullptr && h->data != nullptr && ((uintptr_t)h->data & (uintptr_t)(size - 1)) == 0 && h->heads >= 0 && h->heads <= SC_GROUPS_MAX &&
           h->row >= 0 && h->head >= 0 && h->row <= INT32_MAX * (int64_t)64 && h->head <= INT32_MAX * (int64_t)64;
}
// No element of an output belongs to two heads.  Mostly the heads of a row lie within it, or the rows of a head within that; rows and heads that
// interleave otherwise are gone through.
inline bool heads_apart(const sc_heads* h, int64_t rows, int D) {
    const int64_t row = h->row, head = h->head, heads = h->heads;
    if ((rows > 1 && row < D) || (heads > 1 && head < D)) return false;
    if (rows <= 1 || heads <= 1 || row >= head * (heads - 1) + D || head >= row * (rows - 1) + D) return true;
    for (int64_t j = 1; j < heads; ++j)                // row i and head j of another: i row - j head
        for (int64_t i = j * head / row; i <= j * head / row + 1; ++i)
            if (i > 0 && i < rows && i * row - j * head < D && j * head - i * row < D) return false;
    return true;
}

}  // namespace sc
