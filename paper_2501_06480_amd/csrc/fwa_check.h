// Argument checks that the entry points share (host only).
#pragma once

#include <stdint.h>

#include "../../include/fwa.h"

namespace fwa {
namespace check {

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Row stride of a strided tensor, in elements: at least C, rows 16-byte aligned, and small enough
// that the byte offsets inside one window fit 32 bits with room to spare.
inline int check_row_stride(int64_t ld, int C, int dtype) {
    const int64_t per16 = dtype == FWA_F32 ? 4 : 8;
    if (ld < C) return FWA_ERR_SHAPE;
    if (ld % per16 != 0) return FWA_ERR_ALIGN;
    if (ld > (int64_t)1 << 20) return FWA_ERR_UNSUPPORTED;
    return FWA_OK;
}

// A row-strided [N, L, C] tensor as the bytes it touches: rows of `width` bytes every `ld` bytes.
struct Span {
    uintptr_t base;
    uint64_t ld, width, rows;
    uintptr_t end() const { return base + (rows - 1) * ld + width; }
};
inline Span span_of(const void* p, int64_t N, int L, int C, int64_t ld, int dtype) {
    const uint64_t e = dtype == FWA_F32 ? 4 : 2;
    return Span{reinterpret_cast<uintptr_t>(p), (uint64_t)ld * e, (uint64_t)C * e, (uint64_t)N * (uint64_t)L};
}
// Whether two such tensors share a byte.  Tensors whose extents are disjoint do not.  With equal row
// strides (the views of one fused [N, L, 3, heads, d] buffer) the test is exact: rows interleave
// without touching iff the bases differ, modulo the stride, by at least a row width either way (that of
// the tensor that starts first, then that of the other).
// Extents that intersect under different strides are reported as overlapping (conservative).
inline bool overlaps(const Span& a, const Span& b) {
    if (a.end() <= b.base || b.end() <= a.base) return false;
    if (a.ld != b.ld) return true;
    const Span& low = a.base <= b.base ? a : b;
    const Span& high = a.base <= b.base ? b : a;
    const uint64_t d = (high.base - low.base) % a.ld;
    return d < low.width || a.ld - d < high.width;
}

}  // namespace check
}  // namespace fwa
