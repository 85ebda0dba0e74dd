// Checks of heads given from outside, for the calls that take queries and keys (sc_rope.hip, sc_attention.hip).
#pragma once

#include <stdint.h>

#include "sc.h"

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
// Both are the same elements, in the same places.
inline bool heads_same(const sc_heads* a, const sc_heads* b, int64_t rows) {
    return a->data == b->data && a->heads == b->heads && (rows <= 1 || a->row == b->row) && (a->heads <= 1 || a->head == b->head);
}
// Some element belongs to both, for certain: of operands of the same strides all that meet, which takes as many steps as they have heads; of others those that begin at the same
// place.  Operands of tensors of their own, and slices of one row next to each other, take none.
inline bool heads_meet(const sc_heads* a, int64_t a_rows, const sc_heads* b, int64_t b_rows, int D, int dtype) {
    if (a_rows <= 0 || b_rows <= 0 || a->heads <= 0 || b->heads <= 0) return false;
    if (a->data == b->data) return true;
    if ((uintptr_t)a->data > (uintptr_t)b->data) return heads_meet(b, b_rows, a, a_rows, D, dtype);
    const int64_t apart = (int64_t)(((uintptr_t)b->data - (uintptr_t)a->data) / (dtype == SC_F32 ? 4 : 2));       // of an a and a b in elements: apart + rows row + heads head
    if (apart >= (a_rows - 1) * a->row + (a->heads - 1) * a->head + D) return false;
    const int64_t row = a_rows > 1 ? a->row : b->row, head = a->heads > 1 ? a->head : b->head;
    if ((b_rows > 1 && b->row != row) || (b->heads > 1 && b->head != head)) return false;
    const int64_t a_wide = (a->heads - 1) * head + D, b_wide = (b->heads - 1) * head + D;
    if (row > 0 && apart % row >= a_wide && apart % row + b_wide <= row) return false;                           // next to each other in a row
    for (int64_t h = 1 - a->heads; h < b->heads; ++h) {
        const int64_t at = apart + h * head, back = row > 0 ? (at >= 0 ? at / row : -((row - 1 - at) / row)) : 0;       // a row of a behind b's by so many is next, or one more
        for (int64_t r = back; r <= back + 1; ++r) {
            const int64_t there = r < 1 - b_rows ? 1 - b_rows : r > a_rows - 1 ? a_rows - 1 : r, way = at - there * row;
            if (way < D && -way < D) return true;
        }
    }
    return false;
}

}  // namespace sc
