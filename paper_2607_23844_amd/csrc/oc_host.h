// Host-side checks shared by the C-ABI sources: the thread's error message and
// the checks that every entry point makes.
#pragma once
#include "../../include/oc.h"
#include "oc_ops.h"
#include <cstddef>
#include <cstdint>

namespace oc {

oc_status record_error(oc_status s, const char *msg);
oc_status failf(oc_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
oc_status valid_shape(const oc_shape *sh);
oc_status valid_ws(const void *ws, size_t ws_bytes, size_t need);
// checks rope (NULL: nothing to do) and fills g
oc_status make_rope(const oc_shape *sh, const oc_rope *rope, RopeGeom &g);

inline bool is_aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// [a, a + na) and [b, b + nb) share a byte (NULL shares none)
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return a && b && na && nb && x < y + nb && y < x + na;
}

// The same of rows: n rows of na (nb) bytes, lda (ldb) apart.  Rows of equal
// strides may lie between each other (columns of one buffer).
inline bool rows_overlap(const void *a, size_t na, size_t lda, const void *b, size_t nb, size_t ldb, size_t n) {
    if (n == 0 || !overlaps(a, (n - 1) * lda + na, b, (n - 1) * ldb + nb)) return false;
    if (lda != ldb) return true;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    const size_t off = y >= x ? (y - x) % lda : (lda - (x - y) % lda) % lda;   // b's column in a's rows
    return off < na || off + nb > lda;
}

}  // namespace oc
