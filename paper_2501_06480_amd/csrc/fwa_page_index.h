// Where the operators on a paged cache read and write: plain arithmetic on what the caller's tables hold, whatever that is, so that no table
// leads outside the cache.  No HIP in here: a test on the CPU runs the same functions over tables of all kinds.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define FWA_PAGE_FN __host__ __device__ __forceinline__
#else
#define FWA_PAGE_FN inline
#endif

namespace fwa {

constexpr int kPageRows = 16;        // a page is a multiple of this many rows: the loads of 16 rows of a tile have one page
constexpr int kPageFarthest = 1 << 29;  // older tokens that a sequence is taken to have at most, so that sums with new ones do not overflow

// An entry of the offsets, cut off at the rows that there are.
FWA_PAGE_FN int page_offset(int entry, int rows) { return entry < 0 ? 0 : (entry > rows ? rows : entry); }
// Older tokens of a sequence.
FWA_PAGE_FN int page_length(int entry) { return entry < 0 ? 0 : (entry > kPageFarthest ? kPageFarthest : entry); }
// New tokens of a sequence between two offsets that are cut off already.
FWA_PAGE_FN int page_count(int begin, int end, int most) { return end <= begin ? 0 : (end - begin < most ? end - begin : most); }
// Keys of a sequence that the table has room for: places 0 .. keys - 1 have an entry.
FWA_PAGE_FN int page_keys(int length, int count, int width, int page_size) {
    const int room = width * page_size;
    return length + count < room ? length + count : room;
}
FWA_PAGE_FN bool page_exists(int page, int pages) { return (uint32_t)page < (uint32_t)pages; }
// Rows of the cache that a group of `group` keys from `key` on has: 0 where the page is none.
FWA_PAGE_FN int page_group(int key, int keys, int group, bool exists) {
    const int left = keys - key;
    return !exists || left <= 0 ? 0 : (left < group ? left : group);
}
// Bytes from the base of a head to a row of a page.
FWA_PAGE_FN uint64_t page_place(uint32_t page, uint32_t slot, uint32_t page_bytes, uint32_t token_bytes) { return (uint64_t)page * page_bytes + (uint64_t)slot * token_bytes; }
// Bytes from there that the loads of `rows` rows may touch.
FWA_PAGE_FN uint32_t page_bytes_of(int rows, uint32_t token_bytes, uint32_t row_bytes) { return rows > 0 ? (uint32_t)(rows - 1) * token_bytes + row_bytes : 0u; }

}  // namespace fwa
