// Shared parts of the operators on a paged cache (fwa_page_append.hip, fwa_page_forward.hip).
#pragma once

#include "fwa_internal.h"
#include "fwa_page_index.h"
#include "fwa_sequence.h"

namespace fwa {

__device__ __forceinline__ int page_offset_of(const PageArgs& a, int n) { return page_offset(seq_constant(a.offsets, n), a.rows); }
__device__ __forceinline__ int page_length_of(const PageArgs& a, int n) { return page_length(seq_constant(a.lengths, n)); }

}  // namespace fwa
