// Attention of new tokens over a paged cache: O = softmax(scale Q K^T) V, the keys and values of a sequence in the rows of its pages, the new
// tokens of all sequences one behind the other.
//
// As fwa_sequence_forward.hip: one pass over the keys with a running reference and sum per row, S^T = K Q^T and O^T += V^T P^T, tiles of K and V
// through LDS.  What differs: the rows of a workgroup are those of all heads that share the keys, token by token, so that a tile is
// loaded once for all of them and single tokens fill a block as far as they can; the loads of 16 rows of a tile go to one page, whose number is
// looked up by the scalar unit two tiles ahead; how many rows and keys a sequence has is known on the device alone.
#include "fwa_internal.h"
#include "fwa_page_index.h"
#include "fwa_sequence.h"

#include <type_traits>

namespace fwa {
namespace {

// A row's reference moves when a score exceeds it by more than this, as in the attention of whole sequences.
constexpr float kSlack = 6.f;
// Rows (new tokens times heads of a group) up to which the waves of a workgroup share out the keys: a block of 32, or of fp32 data, whose products take
// longer than their tiles' way, two, since of 128 rows' waves half would have none (45 sequences of 5 tokens on up to 14834 keys, 3 heads of 32 with 8 of
// queries each: 375 us in a block of 128 rows, 182 in two of 32; bf16, 8000 keys: 53 and 62).
constexpr int few_rows(int dtype) { return dtype == 0 ? 64 : 32; }
// Tiles of a wave from which an even share of all keys is worth finding, which takes a workgroup about 3 us (32 sequences of 4096 to 8192 keys, 8
// heads of 128, bf16, 250 tiles a wave: 158 us in parts of each sequence, 150 in even shares; 8 sequences of 1000 to 2000, 2 heads of 64, 2 tiles a
// wave: 16.5 and 18.3), and sequences up to which it is: each lane adds up 16 of them at most.
constexpr double kWorth = 8.0;
constexpr int kMostShared = 1024;
constexpr int kLengths = 16;  // lengths of parts that are tried at most
// Tiles of a part up to which blocks of different sequences are cut for one workgroup on each CU and not two, if they are few enough to make four parts
// each (4 sequences with up to 140 new tokens on 18000, one head: 35 us with two, 28 with one; 52 with up to 23 on 12000, 3 heads: 76 and 163).
constexpr int kShort = 16;

// How a call is laid out on the device.
struct PagePlan {
    int keys;         // the waves of a workgroup share out the keys, not the rows
    int rows;         // of a block
    int group;        // heads of queries per head of keys
    int each;         // blocks of each sequence, 0: as many as it has, found by a search
    int blocks;
    // The keys of a block may be shared out among workgroups: `splits` of them for each block; parts of about one length of all blocks, `target` for each
    // head of the keys; or `workers` for each, evenly over all sequences.  1, 0 and 0 otherwise.
    int splits, target, workers;
    int alone, least; // tiles up to which a block is not shared out, and that a part has at least
    int lane_sequences;  // that a lane adds up for the workers
    unsigned grid;
    FastDiv by_kv, by_splits, by_each, by_group, by_sub;
    size_t slots;     // rows of parts: [block][kv][split][rows], [part][kv][rows] or [worker][kv][2][rows]
    float* part_o;    // [D] each, not divided by the sum
    float* part_ml;   // [2] each
    int* joins;       // [block, part or worker][kv][8]: parts (0: nothing to join), first token, row of the block's first, rows of the sequence, rows of
                      // parts: the first part's, the second's, from one to the next
    int joined;       // blocks, parts or workers
    bool many;        // blocks of rows may have many parts
};

// A block of a sequence's rows (token-major: row r is token r / group, head r % group of the group).
struct PageBlock {
    int n, row0, rows;  // sequence, first row, rows of the sequence
    int begin;          // first new token
    int start, klen;    // place of token 0, keys
    int kend;           // keys up to this one are seen by a row of the block
};

// What is known of a sequence from its entries in the tables, its blocks left open.  Of more new tokens than the caller told of, the first are all there are.
__device__ __forceinline__ void page_sequence(const PageArgs& a, const PagePlan& plan, int n, int offset, int next_offset, int length, PageBlock& b) {
    b.n = n;
    b.begin = page_offset(offset, a.rows);
    const int count = page_count(b.begin, page_offset(next_offset, a.rows), a.most);
    b.rows = count * plan.group;
    b.start = page_length(length);
    b.klen = page_keys(b.start, count, a.width, a.page_size);
}
__device__ __forceinline__ void page_sequence(const PageArgs& a, const PagePlan& plan, int n, PageBlock& b) {
    page_sequence(a, plan, n, seq_constant(a.offsets, n), seq_constant(a.offsets, n + 1), seq_constant(a.lengths, n), b);
}
__device__ __forceinline__ void page_place_block(const PageArgs& a, const PagePlan& plan, int within, int rows, PageBlock& b) {
    b.row0 = within * rows;
    const int last_row = b.rows - b.row0 < rows ? b.rows - 1 : b.row0 + rows - 1;
    const int last = b.start + (int)fastdiv((uint32_t)last_row, plan.by_group);
    b.kend = a.causal && last + 1 < b.klen ? last + 1 : b.klen;
}
// Sequence n begins at block offsets[n] group / ROWS + n, so that none shares a block with another and a few blocks have no rows.
template <int ROWS>
__device__ __forceinline__ int page_first_block(const PagePlan& plan, int offset, int n) {
    return (int)((uint32_t)offset * (uint32_t)plan.group / (uint32_t)ROWS) + n;
}
// The block with this number; false: it has no rows
template <int ROWS>
__device__ __forceinline__ bool page_block(const PageArgs& a, const PagePlan& plan, int block, PageBlock& b) {
    int within;
    if (plan.each > 0) {
        const int n = (int)fastdiv((uint32_t)block, plan.by_each);
        within = block - n * plan.each;
        page_sequence(a, plan, n, b);
    } else {
        // the last sequence that begins at or in front of this block, 64 candidates at a time, each lane with all that is known of its own
        const int lane = (int)(threadIdx.x & 63u);
        int lo = 0, size = a.N;
        for (;;) {
            const int step = (size + 63) / 64, at = lo + lane * step, n = at < a.N ? at : a.N - 1;
            const int offset = a.offsets[n], next_offset = a.offsets[n + 1], length = a.lengths[n];
            const int f = page_first_block<ROWS>(plan, page_offset(offset, a.rows), at);
            const int count = __popcll(__ballot(at < lo + size && f <= block));
            if (count == 0) return false;
            lo += (count - 1) * step;
            if (step == 1) {
                within = block - __builtin_amdgcn_readlane(f, count - 1);
                page_sequence(a, plan, lo, __builtin_amdgcn_readlane(offset, count - 1), __builtin_amdgcn_readlane(next_offset, count - 1),
                              __builtin_amdgcn_readlane(length, count - 1), b);
                break;
            }
            size = step < a.N - lo ? step : a.N - lo;
        }
    }
    if (within < 0 || (long long)within * ROWS >= b.rows) return false;
    page_place_block(a, plan, within, ROWS, b);
    return true;
}

// Sum of x over the lanes up to this one
template <int CONTROL, int ROW_MASK>
__device__ __forceinline__ int page_scan_step(int x) { return x + __builtin_amdgcn_update_dpp(0, x, CONTROL, ROW_MASK, 0xf, false); }
__device__ __forceinline__ int page_scan(int x) {
    // from 1, 2, 4 and 8 lanes back within a row of 16; from the last lane of rows 0 and 2 to rows 1 and 3; of row 1 to rows 2 and 3
    x = page_scan_step<0x111, 0xf>(x);
    x = page_scan_step<0x112, 0xf>(x);
    x = page_scan_step<0x114, 0xf>(x);
    x = page_scan_step<0x118, 0xf>(x);
    x = page_scan_step<0x142, 0xa>(x);
    return page_scan_step<0x143, 0xc>(x);
}
// Parts of blocks of different sequences, of about one length: those of sequences of one block first, then those of the others, from a sequence's last
// block on.  Each lane has a sequence.
struct PageJob {
    int split, parts, length;  // of the block; most parts of a block of the sequence; tiles of a part
};
template <int ROWS, int KT>
__device__ __forceinline__ bool page_job(const PageArgs& a, const PagePlan& plan, int job, PageBlock& b, PageJob& j) {
    const int lane = (int)(threadIdx.x & 63u), n = lane < a.N ? lane : a.N - 1;
    const int offset = a.offsets[n], next_offset = a.offsets[n + 1], length = a.lengths[n];
    const int from = page_offset(offset, a.rows), count = lane < a.N ? page_count(from, page_offset(next_offset, a.rows), a.most) : 0;
    const int blocks = (int)(((uint32_t)count * (uint32_t)plan.group + ROWS - 1u) / ROWS);
    const int tiles = (page_keys(page_length(length), count, a.width, a.page_size) + KT - 1) / KT;
    const int work = __builtin_amdgcn_readlane(page_scan(blocks * tiles), 63), half = (plan.target + 1) / 2;
    const int target = work <= kShort * half && 4 * __builtin_amdgcn_readlane(page_scan(blocks), 63) <= half ? half : plan.target;
    j.length = page_length_first(work, target, plan.least);
    int parts = page_parts(tiles, j.length, plan.alone);
    for (int turn = 0; turn < kLengths && __builtin_amdgcn_readlane(page_scan(blocks * parts), 63) > target; ++turn) {
        j.length = page_length_next(j.length);
        parts = page_parts(tiles, j.length, plan.alone);
    }
    const int one = blocks == 1 ? parts : 0, many = blocks > 1 ? blocks * parts : 0, ones = page_scan(one), all = page_scan(many);
    const int first = blocks > 1 ? __builtin_amdgcn_readlane(ones, 63) + all - many : ones - one;
    const unsigned long long mine = __ballot(first <= job && job < first + blocks * parts);
    if (mine == 0) return false;
    const int who = (int)__builtin_ctzll(mine), within = job - __builtin_amdgcn_readlane(first, who);
    j.parts = __builtin_amdgcn_readlane(parts, who);
    const int turn = (int)((uint32_t)within / (uint32_t)j.parts);
    j.split = within - turn * j.parts;
    page_sequence(a, plan, who, __builtin_amdgcn_readlane(offset, who), __builtin_amdgcn_readlane(next_offset, who), __builtin_amdgcn_readlane(length, who), b);
    page_place_block(a, plan, __builtin_amdgcn_readlane(blocks, who) - 1 - turn, ROWS, b);
    return true;
}

// A worker's way through its range of the keys of all sequences.
template <int ROWS, int KT, int TURN>
struct PageWalk {
    int lo, per, total, at, units;  // its range; first unit of the sequence that it is in, and its units
    // to the sequence that its range begins in; false: it has nothing to do.  Each wave finds this by itself, a lane adding up a few sequences.
    __device__ __forceinline__ bool begin(const PageArgs& a, const PagePlan& plan, int worker, PageBlock& b) {
        const int first = (int)(threadIdx.x & 63u) * plan.lane_sequences;
        int mine = 0;
        for (int n = first; n < first + plan.lane_sequences && n < a.N; ++n) {
            const int from = page_offset(a.offsets[n], a.rows), count = page_count(from, page_offset(a.offsets[n + 1], a.rows), a.most);
            mine += page_units(count, (page_keys(page_length(a.lengths[n]), count, a.width, a.page_size) + KT - 1) / KT);
        }
        const int upto = page_scan(mine);
        total = __builtin_amdgcn_readlane(upto, 63);
        per = page_share(total, plan.workers, plan.least, TURN);
        if ((long long)worker * per >= total) return false;
        lo = worker * per;
        const int owner = (int)__builtin_ctzll(__ballot(upto > lo));
        at = __builtin_amdgcn_readlane(upto, owner) - __builtin_amdgcn_readlane(mine, owner);
        units = 0;
        for (int n = owner * plan.lane_sequences;; ++n) {
            enter(a, plan, n, b);
            if (at + units > lo || n >= a.N - 1) return true;
        }
    }
    __device__ __forceinline__ void enter(const PageArgs& a, const PagePlan& plan, int n, PageBlock& b) {
        at += units;
        page_sequence(a, plan, n, b);
        page_place_block(a, plan, 0, ROWS, b);
        units = page_units(b.rows, (b.klen + KT - 1) / KT);
    }
    // to the next sequence of its range; false: there is none
    __device__ __forceinline__ bool next(const PageArgs& a, const PagePlan& plan, PageBlock& b) {
        if (at + units >= lo + per || at + units >= total) return false;
        int n = b.n;
        do enter(a, plan, ++n, b);
        while (units == 0 && n < a.N - 1);
        return true;
    }
};

// 16 rows of a tile of V (the `half`-th), as the operand of a product over them: 32 channels in each of v.
template <class T, int D>
__device__ __forceinline__ void page_values(const SeqColumnReader<T, D>& reader, u32x4 (&v)[D / 32], uint32_t tile, int half) {
    constexpr int RB = D * SeqSize<T>::value;
    tile += (uint32_t)(16 * RB * half);
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        const uint32_t first = reader.at ^ (uint32_t)(64 * b), second = first ^ (seq_swizzle<RB>(8u) << 4);
        const uint2 p = seq_lds_tr(tile + first), q = seq_lds_tr(tile + second + 8u * RB);
        v[b] = u32x4{p.x, p.y, q.x, q.y};
    }
}
// Half `h` of a tile of weights, rounded: the operand of a product over its 16 keys.  The matrix instruction has both operands in the data's
// type, so a weight loses up to half a step of it, once; the sums are of the weights as they were.  Outputs are off by 2.3e-3 of their size in all (bf16; 1.7e-3 with
// weights in 32 bits; half: 2.8e-4, 2.1e-4).  A second product, of what the rounding leaves, would be half as many matrix instructions again.
template <class T>
__device__ __forceinline__ u32x4 page_weights(const f32x16& w, int h) {
    constexpr bool F16 = __is_same(T, SeqF16);
    return u32x4{pack_e<F16>(w[8 * h], w[8 * h + 1]), pack_e<F16>(w[8 * h + 2], w[8 * h + 3]),
                 pack_e<F16>(w[8 * h + 4], w[8 * h + 5]), pack_e<F16>(w[8 * h + 6], w[8 * h + 7])};
}

// Waits until a wave has what it reads from LDS, so that loads may write there; until no more than N of its loads are on their way, which end in
// their order.
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void loads_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// A wave's loads of a tile: its rows in groups of 16 (or 8) that lie in one page each.
template <int RB, int KT, int WAVES>
struct PageLoader {
    static constexpr int kRows = KT / WAVES, kGroup = kRows < kPageRows ? kRows : kPageRows, kGroups = kRows / kGroup, kLoads = kGroup * RB / 1024;
    static_assert(kLoads >= 1 && kLoads * 1024 == kGroup * RB, "a group is a whole number of loads");
    uint32_t off[kLoads];
    uint32_t to;    // of the wave's rows in the tile
    int row;
    __device__ __forceinline__ void init(uint32_t wave, uint32_t lane, uint32_t token_bytes) {
        row = (int)wave * kRows;
        to = wave * (uint32_t)(kRows * RB);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t at = (uint32_t)i * 1024u + lane * 16u, r = at / RB, place = (at % RB) / 16u;
            off[i] = r * token_bytes + ((place ^ seq_swizzle<RB>((uint32_t)row + r)) * 16u);
        }
    }
    __device__ __forceinline__ void issue(const u32x4& source, uint32_t lds, int group) const {
        seq_loads_to_lds<kLoads, 1024>(source, off, lds + to + (uint32_t)(group * kGroup * RB));
    }
    __device__ __forceinline__ void zero(uint32_t lds, int group, uint32_t lane) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(lds + to + (uint32_t)(group * kGroup * RB) + (uint32_t)i * 1024u + lane * 16u) = u32x4{0u, 0u, 0u, 0u};
    }
};

// Two forms.  Rows: the W waves of a workgroup have 32 rows each and share the tiles, two of K and of V, so that one is on its way while the other is
// read.  KEYS: all have the same 32 rows and every W-th tile each, in one place for each wave without a barrier, and join what they have at the end; a
// tile's loads follow its reads, beside softmax and products (two places each: 10.6 us for 300 sequences of 100 keys, 7.5 with one, which leaves a CU
// room for more workgroups; 155 and 151 for 128 of up to 2000).  Workgroups share out the keys of a block besides where blocks are few.
// Rows: bound by what a tile takes of all units and by the clock: 2048 tokens on 6001, 16 heads of 128 on 4, bf16: 127 to 132 us, 890 to 930 TFLOP/s,
// matrix units 42, vector units 38 and LDS 32 per cent busy at the 2.1 GHz that the clock falls to (2.4 where memory bounds; a product of 8192^3 reaches
// 1260 TFLOP/s).  Leaving out the loads, or the exponentials, gains a tenth each, and no order of instructions gains any (scores a tile ahead of the
// weights: the same; 64 rows a wave, 8 waves, tiles of 32 keys: slower).  Of single tokens beside chunks (16 sequences, two of them with 500 new tokens: 54 us): one wave of four works for a
// token's block, and parts are whole numbers of tiles in one round of workgroups.  Keys: bound by the reads of the cache (814 MB in 133 to 147 us, 5.5
// to 6.1 TB/s) or, for short ones, by a chain of loads, tables, pages, keys, of about 1 us each, behind the launch (4 tokens on 700, 12 heads of 64: 8.1 us).
template <class T, int D, int W, int KT, bool KEYS, bool WALKS, int OCC>
__global__ void __launch_bounds__(64 * W, OCC) page_forward_kernel(PageArgs a, PagePlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, KS = KT / 32, SUB = KT / kPageRows;
    constexpr bool F32 = __is_same(T, SeqF32);
    constexpr int ROWS = KEYS ? 32 : 32 * W, TURN = KEYS ? W : 1;  // of a workgroup; from a wave's tile to its next one
    constexpr uint32_t kTile = KT * RB;
    using Loader = PageLoader<RB, KT, KEYS ? 1 : W>;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u;
    const uint32_t base = lds_offset(lds) + (KEYS ? wave * 2u * kTile : 0u);

    // workgroup -> head of the keys (neighbours, so that each XCD has few of them), and a part of a block of rows, the last ones of which have most
    // keys, or a share of all sequences.  Rounds of as many workgroups as there are CUs go forwards and backwards in turn, so that a CU's come to one sum.
    uint32_t id = blockIdx.x;
    const uint32_t round = id >> 8;
    if (!KEYS && (round & 1u) && 256u * round + 256u <= gridDim.x) id = 512u * round + 248u - id + 2u * (id & 7u);
    const uint32_t rest = fastdiv(id, plan.by_kv), hk = id - rest * plan.by_kv.d;
    const uint32_t turn = fastdiv(rest, plan.by_splits), split = rest - turn * plan.by_splits.d;
    const uint32_t block = WALKS || plan.target > 0 ? turn : (uint32_t)plan.blocks - 1u - turn, unit = block * (uint32_t)a.KV + hk;
    PageBlock b;
    PageWalk<ROWS, KT, TURN> walk;
    PageJob job = {};
    bool any;
    if constexpr (WALKS) any = walk.begin(a, plan, (int)block, b);
    else if (!KEYS && plan.target > 0) any = page_job<ROWS, KT>(a, plan, (int)block, b, job);
    else any = page_block<ROWS>(a, plan, (int)block, b);
    if (!any) {
        if (plan.joined > 0 && split == 0 && threadIdx.x == 0) plan.joins[8 * (size_t)unit] = 0;
        return;
    }
    Loader load;
    load.init(KEYS ? 0u : wave, lane, (uint32_t)(a.token_stride * E));
    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    SeqColumnReader<T, D> column_reader;
    column_reader.init(hi, c);

    for (;;) {
    const int tiles = (b.kend + KT - 1) / KT;
    int t0 = 0, t1 = tiles, several = 0;
    uint32_t slot0 = 0u, second = 0u;  // rows of parts: where this one goes, and the second one of a block whose first it is
    bool whole = true;
    if constexpr (WALKS) {
        const PagePart p = page_part(walk.at, walk.units, walk.lo, walk.per);
        t0 = p.from;
        t1 = p.to < tiles ? p.to : tiles;
        whole = p.place < 0;
        several = p.parts;
        slot0 = (2u * unit + (p.place > 0 ? 1u : 0u)) * ROWS;
        second = 2u * (unit + (uint32_t)a.KV) * ROWS;
    } else if (!KEYS && plan.target > 0) {
        const PageCut cut = page_cut(tiles, job.length, plan.alone, page_parts_room(job.parts, (int)block, job.split, plan.blocks), job.split);
        if (job.split >= cut.parts) {
            if (threadIdx.x == 0) plan.joins[8 * (size_t)unit] = 0;
            return;
        }
        t0 = cut.from;
        t1 = cut.to;
        whole = cut.parts == 1;
        several = job.split == 0 && !whole ? cut.parts : 0;
        slot0 = unit * ROWS;
        second = slot0 + (uint32_t)a.KV * ROWS;
    } else if (plan.splits > 1) {
        int per = (int)fastdiv((uint32_t)(tiles + plan.splits - 1), plan.by_splits);
        if (per < plan.least) per = plan.least;
        const int parts = tiles <= plan.alone ? 1 : (tiles + per - 1) / per;
        if ((int)split >= parts) return;
        whole = parts == 1;
        t0 = whole ? 0 : (int)split * per;
        t1 = whole || t0 + per > tiles ? tiles : t0 + per;
        several = split == 0 && !whole ? parts : 0;
        slot0 = (unit * (uint32_t)plan.splits + split) * ROWS;
        second = slot0 + ROWS;
    }

    const int G = plan.group, klen = b.klen;
    const size_t head_at = (size_t)hk * (size_t)a.head_stride * E;
    const char* const kp = static_cast<const char*>(a.k) + head_at;
    const char* const vp = static_cast<const char*>(a.v) + head_at;
    const uint32_t token_bytes = (uint32_t)(a.token_stride * E);
    const uint32_t page_bytes = (uint32_t)(a.page_stride * E);
    const int32_t* const page_row = a.table + (size_t)b.n * a.width;

    // Pages are looked up two tiles ahead of their use, so that nothing waits for the scalar loads, and in steps from group to group, without a
    // division: a group's place is an entry of the table and a row of that page.
    const int page_size = a.page_size, last_index = klen > 0 ? (int)fastdiv((uint32_t)(klen - 1) / (uint32_t)kPageRows, plan.by_sub) : 0;
    auto place_of = [&](int key) {
        const int index = (int)fastdiv((uint32_t)key / (uint32_t)kPageRows, plan.by_sub);
        return PageSpot{index, key - index * page_size};
    };
    // (entries behind the sequence's last are read and not used)
    auto find = [&](int index) { return seq_constant(page_row, page_entry(index, a.width)); };
    struct Group {
        int page, slot;
    };
    struct Groups {
        Group g[Loader::kGroups];
    };
    // what one wave's tiles are apart, and groups of a tile
    constexpr int kStride = TURN * KT;
    const PageSpot stride = place_of(kStride);
    const int mine0 = KEYS ? t0 + (int)wave : t0;
    PageSpot ahead = place_of(mine0 * KT + load.row);
    auto look = [&]() {
        Groups r;
        PageSpot p = ahead;
#pragma unroll
        for (int g = 0; g < Loader::kGroups; ++g) {
            r.g[g] = Group{find(p.index), p.slot};
            if (g + 1 < Loader::kGroups) page_advance(p, 0, Loader::kGroup, page_size);
        }
        page_advance(ahead, stride.index, stride.slot, page_size);
        return r;
    };
    // rows of a tile of K or V from the first of this wave's on, of which there are `left`
    auto issue = [&](const Groups& r, const char* from, int left, uint32_t to) {
#pragma unroll
        for (int g = 0; g < Loader::kGroups; ++g) {
            const int rows = page_group(g * Loader::kGroup, left, Loader::kGroup, page_exists(r.g[g].page, a.pages));
            const uint64_t at = rows > 0 ? page_place((uint32_t)r.g[g].page, (uint32_t)r.g[g].slot, page_bytes, token_bytes) : 0u;
            // Rows that no load fills hold zeros: their weights are zero, and zero times whatever else LDS may hold need not be.
            if (rows < Loader::kGroup) {
                load.zero(to, g, lane);
                lds_reads_done();  // or its writes
            }
            load.issue(lds_source(from + at, page_bytes_of(rows, token_bytes, RB)), to, g);
        }
    };
    int left = klen - mine0 * KT - load.row;  // in the tile that is asked for next
    const uint32_t k_at = base, v_at = base + kTile;  // the first of two tiles each, 2 kTile apart
    // Groups of a tile whose page is none, looked up only where the part has any.
    auto missing = [&](int t) {
        uint32_t bad = 0u;
#pragma unroll
        for (int j = 0; j < SUB; ++j) bad |= page_exists(find((int)fastdiv((uint32_t)(t * SUB + j), plan.by_sub)), a.pages) ? 0u : 1u << j;
        return bad;
    };

    Groups next = {}, after = {};
    if (mine0 < t1) {
        next = look();
        issue(next, kp, left, k_at);
        issue(next, vp, left, v_at);
        left -= kStride;
        next = look();
    }
    bool holes = false;
    if (t0 < t1) {
        const int from = place_of(t0 * KT).index, to = place_of(t1 * KT - 1).index;
        for (int x = from; x <= to && x <= last_index; x += 64) {
            const int at = x + (int)lane;
            holes = holes || !page_exists(page_row[at < last_index ? at : last_index], a.pages);
        }
        holes = __any(holes);
    }

    // the row of this lane: token, head of the group, whether there is one
    const int row = b.row0 + (KEYS ? 0 : 32 * (int)wave) + (int)c;
    const bool exists = row < b.rows;
    const int token = exists ? (int)fastdiv((uint32_t)row, plan.by_group) : 0, member = exists ? row - token * G : 0;
    const int pos = b.start + token, limit = a.causal && pos + 1 < klen ? pos + 1 : klen;
    u32x4 qf[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) qf[s] = u32x4{0u, 0u, 0u, 0u};
    if (exists && a.scale != 0.f) {  // with a scale of zero the queries are zero: a shut out score times zero would be no score
        const char* const qp = static_cast<const char*>(a.q) + ((size_t)(b.begin + token) * a.ldq + (size_t)(hk * G + member) * D) * E + 16u * hi;
#pragma unroll
        for (int s = 0; s < NC; ++s) qf[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
        // a negative scale goes into the queries, so that the largest product is the largest score
        if (a.scale < 0.f) {
            constexpr uint32_t kSign = F32 ? 0x80000000u : 0x80008000u;
#pragma unroll
            for (int s = 0; s < NC; ++s) qf[s] ^= kSign;
        }
    }
    // tiles with a key that a row of the block does not see: from mask0 on
    int mask0 = klen / KT;
    if (a.causal) {
        const int to = (b.start + (int)fastdiv((uint32_t)b.row0, plan.by_group) + 1) / KT;
        mask0 = to < mask0 ? to : mask0;
    }

    // tiles from here on show the rows of this wave nothing
    int wave_end = t1;
    if constexpr (!KEYS) {
        const int first_row = b.row0 + 32 * (int)wave, last_row = first_row + 31 < b.rows ? first_row + 31 : b.rows - 1;
        const int last = b.start + (int)fastdiv((uint32_t)last_row, plan.by_group), end = a.causal && last + 1 < klen ? last + 1 : klen;
        wave_end = first_row < b.rows ? (end + KT - 1) / KT : 0;
    }

    f32x16 o[NB];
#pragma unroll
    for (int x = 0; x < NB; ++x) seq_zero(o[x]);
    float top_at = -__builtin_inff(), sum = 0.f;
    const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e;

    // The reference of a tile of scores: what no key has is shut out, and the reference follows the largest score so far.  Returns what is added to a score.
    auto refer = [&](f32x16 (&s)[KS], int t) {
        const uint32_t bad = holes ? missing(t) : 0u;
        if (t >= mask0 || bad != 0u) {
            const int room = limit - t * KT - 4 * (int)hi;
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const bool seen = 32 * k + 8 * (r / 4) + r % 4 < room && !((bad >> (2 * k + r / 8)) & 1u);
                    s[k][r] = seen ? s[k][r] : -__builtin_inff();
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][r]);
        top = seq_max_halves(top) * scale;
        if (__any(top > top_at + kSlack)) {
            const float to = top > top_at + kSlack ? top : top_at, f = to == top_at ? 1.f : __builtin_amdgcn_exp2f(top_at - to);
            top_at = to;
            sum *= f;
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[x][r] *= f;
        }
        return top_at == -__builtin_inff() ? 0.f : -top_at;
    };
    constexpr int kTileLoads = Loader::kLoads * Loader::kGroups;
    // Tile t, in the buffers of its parity.  Rows: the loads of the next one go to the other buffers in front of everything else.  Keys: they go to the
    // same place as soon as a wave has read it, of 16-bit data all into registers in front of the softmax, of fp32 K in front of it and V behind.
    auto step = [&](auto parity, int t) {
        const uint32_t B = parity;
        const uint32_t kt = k_at + B * 2u * kTile, vt = v_at + B * 2u * kTile;
        if constexpr (KEYS && F32) loads_left<kTileLoads>();  // those of V may be on their way still
        else lds_loads_done();
        if constexpr (!KEYS) {
            __syncthreads();
            if (t + TURN < t1) {
                issue(next, kp, left, k_at + (B ^ 1u) * 2u * kTile);
                issue(next, vp, left, v_at + (B ^ 1u) * 2u * kTile);
            }
            left -= kStride;
            if (t >= wave_end) {
                next = look();
                return;
            }
        }

        f32x16 s[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) seq_zero(s[k]);
        u32x4 v[2 * KS][NB];
        if constexpr (F32) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int x = 0; x < NC; ++x) s[k] = seq_dot<T>(row_reader.read(kt, x, k), qf[x], s[k]);
            if constexpr (KEYS) {
                lds_reads_done();
                if (t + TURN < t1) issue(next, kp, left, k_at);
            }
        } else {
            u32x4 f[KS][NC];
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int k = 0; k < KS; ++k) f[k][x] = row_reader.read(kt, x, k);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < NC; ++x)
#pragma unroll
                for (int k = 0; k < KS; ++k) s[k] = seq_dot<T>(f[k][x], qf[x], s[k]);
#pragma unroll
            for (int h = 0; h < 2 * KS; ++h) page_values<T, D>(column_reader, v[h], vt, h);
            if constexpr (KEYS) {
                lds_reads_done();
                if (t + TURN < t1) {
                    issue(next, kp, left, k_at);
                    issue(next, vp, left, v_at);
                }
                left -= kStride;
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        after = look();
        const float minus = refer(s, t);
        auto weights = [&](int k) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[k][r] = __builtin_amdgcn_exp2f(fmaf(s[k][r], scale, minus));
                sum += s[k][r];
            }
        };
        if constexpr (F32) {
            if constexpr (KEYS) {
                if (t + TURN < t1) loads_left<kTileLoads>();
                else lds_loads_done();
            }
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                weights(k);
                column_reader.accumulate(o, vt, k, s[k]);
            }
        } else {
            weights(0);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const u32x4 w = page_weights<T>(s[k], h);
#pragma unroll
                    for (int x = 0; x < NB; ++x) o[x] = seq_dot<T>(v[2 * k + h][x], w, o[x]);
                }
                if (k + 1 < KS) weights(k + 1);
            }
        }
        if constexpr (KEYS && F32) {
            lds_reads_done();
            if (t + TURN < t1) issue(next, vp, left, v_at);
            left -= kStride;
        }
        next = after;
    };
    if constexpr (KEYS) {
        for (int t = mine0; t < t1; t += TURN) step(std::integral_constant<uint32_t, 0>{}, t);
    } else {
        for (int t = mine0; t < t1; t += 2) {
            step(std::integral_constant<uint32_t, 0>{}, t);
            if (t + 1 < t1) step(std::integral_constant<uint32_t, 1>{}, t + 1);
        }
    }

    sum = seq_sum_halves(sum);
    if constexpr (KEYS && W > 1) {
        // sums of all waves through LDS, rows 4 floats apart from a multiple of the banks; the last wave has them, the others are done
        constexpr uint32_t kRow = 4u * (D + 4);
        const uint32_t all = lds_offset(lds), sums = all + W * 32u * kRow;
        __syncthreads();
        if (hi == 0) *(__attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * wave + c)) = f32x2{top_at, sum};
        __syncthreads();
        float top = -__builtin_inff(), total = 0.f, mine = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, (*(const __attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * w + c)))[0]);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const f32x2 x = *(const __attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * w + c));
            const float f = x[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(x[0] - top);  // a part without weight may have no reference
            total += f * x[1];
            if (w == (int)wave) mine = f;
        }
        if (wave != W - 1) {
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(all + kRow * (32u * wave + c) + 4u * (32 * x + 8 * q + 4 * hi)) =
                        f32x4{o[x][4 * q] * mine, o[x][4 * q + 1] * mine, o[x][4 * q + 2] * mine, o[x][4 * q + 3] * mine};
        }
        __syncthreads();
        if (wave == W - 1) {
#pragma unroll
        for (int x = 0; x < NB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[x][r] *= mine;
#pragma unroll
        for (int w = 0; w < W - 1; ++w)
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 y = seq_lds_f32x4(all + kRow * (32u * w + c) + 4u * (32 * x + 8 * q + 4 * hi));
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[x][4 * q + e] += y[e];
                }
        top_at = top;
        sum = total;
        }
    }
    if (exists && !(KEYS && wave != W - 1)) {
        if (!whole) {
            const size_t slot = (size_t)slot0 + (KEYS ? 0 : 32 * wave) + c;
            float* const to = plan.part_o + slot * D;
            if (sum != 0.f)  // nothing reads a part without weight
#pragma unroll
                for (int x = 0; x < NB; ++x)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        *reinterpret_cast<f32x4*>(to + 32 * x + 8 * q + 4 * hi) = f32x4{o[x][4 * q], o[x][4 * q + 1], o[x][4 * q + 2], o[x][4 * q + 3]};
            if (hi == 0) *reinterpret_cast<f32x2*>(plan.part_ml + 2 * slot) = f32x2{top_at, sum};
        } else {
            const bool some = sum != 0.f;  // NaN too
            const float f = some ? 1.f / sum : 0.f;
            const size_t at = (size_t)(b.begin + token), head = hk * G + member;
            char* const to = static_cast<char*>(a.o) + (at * a.ldo + head * D) * E;
#pragma unroll
            for (int x = 0; x < NB; ++x)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float y[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] = some ? o[x][4 * q + e] * f : 0.f;
                    seq_store4<T>(to, 32 * x + 8 * q + 4 * hi, y[0], y[1], y[2], y[3]);
                }
            if (a.stats && hi == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * (at * a.H + head)) = f32x2{some ? top_at : -__builtin_inff(), some ? log2f(sum) : 0.f};
        }
    }
    bool more = false;
    if constexpr (WALKS) more = walk.next(a, plan, b);
    if (!more) {  // a sequence of several parts that a worker begins is its last one
        if (plan.joined > 0 && split == 0 && threadIdx.x == 0) {
            int* const to = plan.joins + 8 * (size_t)unit;
            *reinterpret_cast<i32x4*>(to) = i32x4{several, b.begin, b.row0, b.rows};
            *reinterpret_cast<i32x4*>(to + 4) = i32x4{(int)slot0, (int)second, WALKS ? 2 * a.KV * ROWS : !KEYS && plan.target > 0 ? a.KV * ROWS : ROWS, 0};
        }
        return;
    }
    __syncthreads();  // the tiles and sums in LDS are done with, and the next sequence's may come
    }
}

// Joins the parts of blocks whose keys are shared out.  MANY: a thread has four channels of a row, 16 parts at a time, for blocks of few rows or of
// many parts (one sequence of 32768 keys: 39 us in all, 58 with two at a time; 4 sequences with up to 140 new tokens on 18000, one head: 35 and 75);
// otherwise of some of a workgroup's 32 rows, with the loads of all on the way together (512 blocks of 128 rows of 128 channels, 33 MB: 8.9 us, 10.4
// with a row).  Few rows: 4 us, a launch and two loads one behind the other.
template <class T, int D, int ROWS, bool MANY>
__global__ void __launch_bounds__(256) page_join_kernel(PageArgs a, PagePlan plan) {
    constexpr int E = SeqSize<T>::value, kThreads = D / 4, kRows = 256 / kThreads, kMine = MANY ? 1 : 32 / kRows, kTurns = ROWS / (kRows * kMine);
    constexpr int kAtOnce = MANY ? 16 : 8 / kMine;  // parts of a row
    const uint32_t unit = blockIdx.x / kTurns, turn = blockIdx.x - unit * kTurns, hk = unit - fastdiv(unit, plan.by_kv) * plan.by_kv.d;
    const i32x4 known = *reinterpret_cast<const i32x4*>(plan.joins + 8 * (size_t)unit), rows = *reinterpret_cast<const i32x4*>(plan.joins + 8 * (size_t)unit + 4);
    const int parts = known[0], channel = 4 * (int)(threadIdx.x % kThreads);
    const uint32_t slot0 = (uint32_t)(kRows * kMine) * turn + threadIdx.x / kThreads;
    if (parts == 0 || known[2] + (int)slot0 >= known[3]) return;
    const size_t first = (uint32_t)rows[0], second = (uint32_t)rows[1], step = (uint32_t)rows[2];
    float top[kMine], l[kMine];
    f32x4 o[kMine];
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        top[m] = -__builtin_inff();
        l[m] = 0.f;
        o[m] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // rows that there are not are those of the first again; a part without weight was not written, and whatever is in its place is not used
    for (int s0 = 0; s0 < parts; s0 += kAtOnce) {
        f32x2 ml[kMine][kAtOnce];
        f32x4 x[kMine][kAtOnce];
#pragma unroll
        for (int m = 0; m < kMine; ++m)
#pragma unroll
            for (int s = 0; s < kAtOnce; ++s) {
                const int p = s0 + s < parts ? s0 + s : s0;
                const uint32_t slot = known[2] + (int)slot0 + m * kRows < known[3] ? slot0 + m * kRows : slot0;
                const size_t part = (p == 0 ? first : second + (size_t)(p - 1) * step) + slot;
                ml[m][s] = *reinterpret_cast<const f32x2*>(plan.part_ml + 2 * part);
                x[m][s] = *reinterpret_cast<const f32x4*>(plan.part_o + part * D + channel);
            }
#pragma unroll
        for (int m = 0; m < kMine; ++m) {
            float to = top[m];
#pragma unroll
            for (int s = 0; s < kAtOnce; ++s) to = fmaxf(to, ml[m][s][0]);
            const float f = l[m] == 0.f ? 0.f : __builtin_amdgcn_exp2f(top[m] - to);
            top[m] = to;
            l[m] *= f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[m][e] *= f;
#pragma unroll
            for (int s = 0; s < kAtOnce; ++s) {
                if (s0 + s >= parts || ml[m][s][1] == 0.f) continue;
                const float w = __builtin_amdgcn_exp2f(ml[m][s][0] - to);
                l[m] += w * ml[m][s][1];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[m][e] += w * x[m][s][e];
            }
        }
    }
#pragma unroll
    for (int m = 0; m < kMine; ++m) {
        const int r = known[2] + (int)slot0 + m * kRows;
        if (r >= known[3]) continue;
        const int token = (int)fastdiv((uint32_t)r, plan.by_group);
        const size_t row = (size_t)(known[1] + token), head = hk * plan.group + (r - token * plan.group);
        const bool any = l[m] != 0.f;
        const float f = any ? 1.f / l[m] : 0.f;
        char* const to = static_cast<char*>(a.o) + (row * a.ldo + head * D) * E;
        seq_store4<T>(to, channel, o[m][0] * f, o[m][1] * f, o[m][2] * f, o[m][3] * f);
        if (a.stats && channel == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * (row * a.H + head)) = f32x2{any ? top[m] : -__builtin_inff(), any ? log2f(l[m]) : 0.f};
    }
}

// Tiles, waves, and waves of a SIMD that the registers are held to, as in the attention of whole sequences.
constexpr int page_tile_keys(int row_bytes, bool keys) { return row_bytes >= 512 || keys ? 32 : 64; }
constexpr int page_waves(int row_bytes, bool keys) { return keys ? seq_keys_waves(row_bytes) : 4; }
// Workgroups of a CU that share out all keys: as many as hide the loads of a wave's one tile (fp32 heads of 128, 16 sequences of up to 4000 keys, 8 heads:
// two 124 us, four 112; bf16, 32 of up to 8192: 150 and 153).
constexpr int page_walkers(int row_bytes) { return row_bytes >= 512 ? 4 : 2; }
constexpr int page_occupancy(int row_bytes, bool keys) { return row_bytes == 128 && !keys ? 3 : 1; }

template <class T, int D, bool KEYS, bool WALKS>
hipError_t launch(const PageArgs& a, const PagePlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value, W = page_waves(RB, KEYS), KT = page_tile_keys(RB, KEYS), ROWS = KEYS ? 32 : 32 * W;
    constexpr size_t tiles = (size_t)KT * RB * (KEYS ? 2 * W : 4), sums = KEYS && W > 1 ? (size_t)W * 32 * (4 * (D + 4) + 8) : 0, lds = tiles > sums ? tiles : sums;
    auto* const kernel = &page_forward_kernel<T, D, W, KT, KEYS, WALKS, page_occupancy(RB, KEYS)>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(plan.grid), dim3(64 * W), lds, s, a, plan);
    e = hipGetLastError();
    if (e != hipSuccess || plan.joined == 0) return e;
    const unsigned units = (unsigned)plan.joined * (unsigned)a.KV;
    if (KEYS || plan.many) hipLaunchKernelGGL((page_join_kernel<T, D, ROWS, true>), dim3(units * (unsigned)(ROWS / (256 / (D / 4)))), dim3(256), 0, s, a, plan);
    else hipLaunchKernelGGL((page_join_kernel<T, D, ROWS, false>), dim3(units * (unsigned)(ROWS / 32)), dim3(256), 0, s, a, plan);
    return hipGetLastError();
}

// Microseconds that blocks of rows of up to `tiles` tiles take in `splits` parts each: tiles of one workgroup on a CU or of two, the join's launch, its
// reads of the parts and their writes.  Measured over drawn calls; what counts is the difference between few splits and many.
double page_rows_time(const PageArgs& a, int rows, double blocks, long long tiles, long long splits, int cus) {
    const double one = a.dtype == 0 ? (a.D == 32 ? 2.3 : 4.0) : 0.8 + a.D / 256.0, two = a.dtype == 0 ? (a.D == 32 ? 3.6 : 7.0) : 0.9 + a.D / 98.0;
    const double n = blocks * (double)splits, rounds = (double)(long long)((n + 2.0 * cus - 1.0) / (2.0 * cus));
    return (double)((tiles + splits - 1) / splits) * (n <= cus ? one : two * rounds) + (splits > 1 ? 5.0 + n * rows * a.D * 8.0 / 7.0e6 + (double)splits / 16.0 : 0.0);
}

// How a call is laid out, from what the host knows: the waves share out the keys where no sequence has more than a few rows.  Where there are too few
// blocks for the device, its workgroups share out the keys besides, and a second launch joins the parts, but for caches that are too short to be
// worth that: the join takes as long as about `alone` tiles (704 keys, 6 tiles a wave: 9.0 us whole, 10.4 in parts of two).  Parts are no shorter
// than `least` tiles of a wave (8 sequences of up to 2000 keys: two tiles 16.5 us, four 18.1; fp32 rows, whose tiles take four times as long, one
// tile 14.5 us, four 20.1; 26 sequences of up to 370 fp32 keys, 3 heads of 64: two 24 us, one 14).  How many: of blocks of sequences with the same number
// of new tokens as many as make one or two workgroups for each CU, whichever page_rows_time has as the shorter (2048 tokens on 6001: two 131 us, four 142;
// 9 sequences of 612, one head: one 21, two 26), four where the keys are all there is to do.  Blocks of sequences that bring different numbers, up to
// 64 of them, are cut into parts of one length, no more than one or two for each CU, which the device finds from all lengths (two chunks of 500 beside
// 14 tokens: 63 us, 70 with as many parts for each block; 16 chunks of 61: 49 and 65; causal prompts of one length cut like that: 101 whole, 118 to
// 160 in parts).
bool page_plan(const PageArgs& a, PagePlan& f) {
    const int size = a.dtype == 0 ? 4 : 2, RB = a.D * size, G = a.H / a.KV, cus = cu_count();
    const long long most_rows = (long long)a.most * G, capacity = (long long)a.width * a.page_size;
    f = PagePlan{};
    f.keys = most_rows <= few_rows(a.dtype);
    const int KT = page_tile_keys(RB, f.keys), W = page_waves(RB, f.keys);
    f.rows = f.keys ? 32 : 32 * W;
    f.group = G;
    // blocks: a number for each sequence, or as many as the rows fill and one more for each sequence
    const long long each = (most_rows + f.rows - 1) / f.rows, all = (long long)a.rows * G / f.rows + a.N;
    f.each = each * a.N <= all ? (int)each : 0;
    const long long blocks = f.each ? each * a.N : all;
    const double base = (double)blocks * a.KV;
    if (base * 64.0 * W > 4.0e9) return false;  // threads of a launch
    f.blocks = (int)blocks;
    f.splits = 1;
    const long long tiles = (capacity + KT - 1) / KT;
    const bool slow = a.dtype == 0 && RB >= 256;  // a wave's tile takes 2 us or more of fp32 products
    f.alone = f.keys ? (slow ? 2 : 6) * W : a.dtype == 0 ? 1 : 4;
    f.least = f.keys ? (slow ? 1 : 2) * W : a.dtype == 0 ? 1 : 2;
    if (tiles > f.alone) {
        const bool same = (long long)a.N * a.most == a.rows;  // all sequences have the same number of new tokens
        const int fit = page_walkers(RB);
        if (f.keys && f.each == 1 && a.N <= kMostShared && base < 2.0 * fit * cus && fit * cus / a.KV >= 2 && base * (double)tiles >= kWorth * W * fit * cus && (double)a.N * (double)tiles < 1.0e9) {
            f.workers = fit * cus / a.KV;
            f.lane_sequences = (a.N + 63) / 64;
        } else if (!f.keys && !same && a.N <= 64 && base < 2.0 * cus && base * (double)tiles > 1.0 * cus * f.least && (double)blocks * (double)tiles < 1.0e9) {
            f.target = 2 * cus > a.KV ? 2 * cus / a.KV : 1;
            f.blocks += f.target;
        } else {
            const long long most = tiles / f.least < 64 ? tiles / f.least : 64;
            auto cut = [&](double wanted) { const long long x = (long long)(wanted * cus / base); return x < most ? x : most; };
            long long splits = 1;
            if (f.keys) {
                splits = cut(4.0);
            } else {
                for (const double wanted : {1.0, 2.0, 4.0})
                    if ((wanted < 4.0 || !same) && cut(wanted) > splits && page_rows_time(a, f.rows, base, tiles, cut(wanted), cus) < page_rows_time(a, f.rows, base, tiles, splits, cus))
                        splits = cut(wanted);
            }
            f.splits = splits < 1 ? 1 : splits > 64 ? 64 : (int)splits;
        }
    }
    f.many = f.target > 0 ? f.target >= 4 * blocks : f.splits >= 4;
    f.joined = f.workers > 0 ? f.workers : f.splits > 1 || f.target > 0 ? f.blocks : 0;
    f.grid = (unsigned)(f.workers > 0 ? f.workers : f.blocks * f.splits) * (unsigned)a.KV;
    f.slots = f.workers > 0 ? (size_t)f.workers * a.KV * 2 * f.rows : f.joined > 0 ? (size_t)f.blocks * a.KV * f.splits * f.rows : 0;
    f.by_kv = make_fastdiv((uint32_t)a.KV);
    f.by_splits = make_fastdiv((uint32_t)f.splits);
    f.by_each = make_fastdiv(f.each > 0 ? (uint32_t)f.each : 1u);
    f.by_group = make_fastdiv((uint32_t)G);
    f.by_sub = make_fastdiv((uint32_t)(a.page_size / kPageRows));
    return true;
}
size_t page_workspace(const PagePlan& p, const PageArgs& a) {
    return p.slots * (size_t)(a.D + 2) * sizeof(float) + (size_t)p.joined * a.KV * 8 * sizeof(int);
}

template <class T, int D>
hipError_t launch(const PageArgs& a, const PagePlan& p, hipStream_t s) {
    if (p.workers > 0) return launch<T, D, true, true>(a, p, s);
    return p.keys ? launch<T, D, true, false>(a, p, s) : launch<T, D, false, false>(a, p, s);
}
template <class T>
hipError_t launch(const PageArgs& a, const PagePlan& p, hipStream_t s) {
    if (a.D == 32) return launch<T, 32>(a, p, s);
    if (a.D == 64) return launch<T, 64>(a, p, s);
    return launch<T, 128>(a, p, s);
}

}  // namespace

bool page_forward_fits(const PageArgs& a) {
    PagePlan p;
    return page_plan(a, p);
}

size_t page_forward_workspace(const PageArgs& a) {
    PagePlan p;
    return page_plan(a, p) ? page_workspace(p, a) : 0;
}

hipError_t launch_page_forward(const PageArgs& a, void* workspace, size_t workspace_bytes, hipStream_t s) {
    PagePlan p;
    // the layout goes by what the workspace's query knows too: not by pointers, strides of rows, scale or causality
    if (!page_plan(a, p) || page_workspace(p, a) > (workspace ? workspace_bytes : 0)) return hipErrorInvalidValue;
    if (p.joined > 0) {
        p.part_o = static_cast<float*>(workspace);
        p.part_ml = p.part_o + p.slots * (size_t)a.D;
        p.joins = reinterpret_cast<int*>(p.part_ml + 2 * p.slots);
    }
    if (a.dtype == 0) return launch<SeqF32>(a, p, s);
    return a.dtype == 1 ? launch<SeqBf16>(a, p, s) : launch<SeqF16>(a, p, s);
}

}  // namespace fwa
