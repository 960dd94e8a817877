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
// A way over the keys of a sequence in steps, without a division for each: an entry of its row of the table, and a row of that page.  A step is given as the
// entries and rows that it is long, fewer rows than a page has.  What is looked up ahead of its use may lie behind the last entry, which stands for it then.
struct PageSpot {
    int index, slot;
};
FWA_PAGE_FN void page_advance(PageSpot& p, int index, int slot, int page_size) {
    p.index += index;
    p.slot += slot;
    if (p.slot >= page_size) {
        p.slot -= page_size;
        ++p.index;
    }
}
FWA_PAGE_FN int page_entry(int index, int width) { return index < width ? index : width - 1; }
// Bytes from the base of a head to a row of a page.
FWA_PAGE_FN uint64_t page_place(uint32_t page, uint32_t slot, uint32_t page_bytes, uint32_t token_bytes) { return (uint64_t)page * page_bytes + (uint64_t)slot * token_bytes; }
// Bytes from there that the loads of `rows` rows may touch.
FWA_PAGE_FN uint32_t page_bytes_of(int rows, uint32_t token_bytes, uint32_t row_bytes) { return rows > 0 ? (uint32_t)(rows - 1) * token_bytes + row_bytes : 0u; }

// Sharing out the keys of sequences with a block of rows each.  A sequence is as many units as its keys have tiles, or one if it has none; all
// sequences, one behind the other, are cut into ranges of `per` units, one for each worker.  A worker leaves its part of a sequence in one of two
// places, 0 for the sequence that its range begins in, 1 for a later one that it begins and does not finish, of which there is one at most, the last
// of its range.  A sequence of several parts has those of the worker that begins it, and of place 0 of the workers behind it.
FWA_PAGE_FN int page_units(int rows, int tiles) { return rows == 0 ? 0 : (tiles > 0 ? tiles : 1); }
// units of a worker, a multiple of `turn` (the waves that share out a worker's tiles)
FWA_PAGE_FN int page_share(int total, int workers, int least, int turn) {
    const int per = (total + workers - 1) / workers, more = per > least ? per : least;
    return (more + turn - 1) / turn * turn;
}
struct PagePart {
    int from, to;  // units of the sequence
    int place;     // -1: all of it, no part
    int parts;     // of a sequence of several that this worker begins, else 0
};
// The part of a sequence of `units` units from unit `at` of all on that the worker of units lo .. lo + per - 1 has; the two meet.
FWA_PAGE_FN PagePart page_part(int at, int units, int lo, int per) {
    PagePart p;
    p.from = lo > at ? lo - at : 0;
    p.to = lo + per - at < units ? lo + per - at : units;
    p.parts = at >= lo && p.to < units ? 1 + (units - p.to + per - 1) / per : 0;
    p.place = at >= lo && p.to == units ? -1 : (at > lo ? 1 : 0);
    return p;
}

// Sharing out the keys of blocks whose sequences have different numbers of keys: parts of about one length, as many as a target.  A block of `tiles`
// tiles of keys is this many parts of up to `length`, one if it has `alone` or fewer:
FWA_PAGE_FN int page_parts(int tiles, int length, int alone) { return tiles <= alone ? 1 : (tiles + length - 1) / length; }
// The length begins with what all blocks together have for each part, and grows while there are more parts than the target.  The first alone keeps
// them below the target and the blocks together.
FWA_PAGE_FN int page_length_first(int total, int target, int least) {
    const int length = (int)(((uint32_t)total + (uint32_t)target - 1u) / (uint32_t)target);
    return length > least ? length : least;
}
FWA_PAGE_FN int page_length_next(int length) { return length + 1 + length / 32; }
// Parts that a block has room for, of the `parts` that its sequence's tiles make: its jobs lie one behind the other, this one being the `split`-th, and there
// are `jobs` in all.  Offsets that fall bring more than the launch has; a block that would reach beyond it is cut into fewer parts, so that each part that the
// join reads is one that a workgroup leaves.
FWA_PAGE_FN int page_parts_room(int parts, int job, int split, int jobs) {
    const int room = jobs - (job - split);
    return parts < room ? parts : room;
}
// Tiles of part `split` of a block whose sequence has up to `most` parts a block; parts: how many this one has, all of them one behind the other.
struct PageCut {
    int from, to, parts;
};
FWA_PAGE_FN PageCut page_cut(int tiles, int length, int alone, int most, int split) {
    const int wanted = page_parts(tiles, length, alone), parts = wanted < most ? wanted : most;
    const int per = (int)((uint32_t)(tiles + parts - 1) / (uint32_t)parts);
    PageCut c;
    c.parts = tiles > 0 ? (int)((uint32_t)(tiles + per - 1) / (uint32_t)per) : 1;
    c.from = split * per;
    c.to = c.from + per < tiles ? c.from + per : tiles;
    return c;
}

}  // namespace fwa
