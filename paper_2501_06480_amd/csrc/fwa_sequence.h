// Shared parts of the kernels for attention over whole sequences (fwa_sequence_forward.hip, fwa_sequence_backward.hip).
//
// Products run on the 32 x 32 matrix instructions.  Lane (hi, c), hi = lane >> 5, c = lane & 31, supplies row resp. column c of an
// operand and receives column c of the result, rows 8 (r / 4) + 4 hi + r % 4 of it in register r = 0..15.  A tile of scores is
// always formed such that the index a later product sums over runs over the registers: its 16 values per lane are then an operand of
// that product as they stand, k-slots in the order of the registers, and the probabilities never go through LDS.  The other operand
// of the later product is read from LDS in the same order: 16-bit data by the transposing read, fp32 data a row at a time.
#pragma once

#include "fwa_device.h"
#include "fwa_internal.h"

namespace fwa {

typedef float f32x16 __attribute__((ext_vector_type(16)));

struct SeqBf16 {};
struct SeqF16 {};
struct SeqF32 {};
template <class T>
struct SeqSize { static constexpr int value = 2; };
template <>
struct SeqSize<SeqF32> { static constexpr int value = 4; };

// One step of a product whose operands have their k-slots along a row of memory: 32 bytes of each row, lane (hi, c) holding
// bytes 16 hi .. 16 hi + 15 of row c.
template <class T>
__device__ __forceinline__ f32x16 seq_dot(const u32x4& a, const u32x4& b, f32x16 c) {
    if constexpr (__is_same(T, SeqBf16)) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
    } else if constexpr (__is_same(T, SeqF16)) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
        return c;
    }
}

// Tiles in LDS: rows of RB bytes, one behind the other; within a row the 16-byte chunk c stands at place c ^ seq_swizzle(row), so that
// both the reads of one chunk of 16 rows and the transposing reads of 64 bytes of 8 rows meet every bank equally often.
template <int RB>
__device__ __forceinline__ constexpr uint32_t seq_swizzle(uint32_t row) {
    if constexpr (RB == 64) return (row >> 2) & 3u;
    else if constexpr (RB == 128) return ((row & 2u) << 1) | ((row >> 2) & 3u);
    else return ((row & 3u) << 2) | ((row >> 2) & 3u);
}

// N loads of load_to_lds() (fwa_device.h, and its wait states) one behind the other, 16 bytes a lane each, to LDS places STEP bytes apart: the
// descriptor is old enough for all once it is for the first, and m0 is put back once.
template <int N, int STEP>
__device__ __forceinline__ void seq_loads_to_lds(const u32x4& r, const uint32_t* off, uint32_t lds_off) {
    uint32_t saved;
    if constexpr (N == 1) {
        load_to_lds(r, off[0], lds_off);
    } else if constexpr (N == 2) {
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %4, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, %5\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %4, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved) : "s"(lds_off), "v"(off[0]), "v"(off[1]), "s"(r), "i"(STEP) : "memory", "scc");
    } else {
        static_assert(N % 4 == 0, "one, two or a multiple of four loads");
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 2\n\tbuffer_load_dwordx4 %2, %6, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, %7\n\ts_nop 0\n\tbuffer_load_dwordx4 %3, %6, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, %7\n\ts_nop 0\n\tbuffer_load_dwordx4 %4, %6, 0 offen lds\n\t"
                     "s_add_u32 m0, m0, %7\n\ts_nop 0\n\tbuffer_load_dwordx4 %5, %6, 0 offen lds\n\ts_mov_b32 m0, %0"
                     : "=&s"(saved) : "s"(lds_off), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(r), "i"(STEP) : "memory", "scc");
        if constexpr (N > 4) seq_loads_to_lds<N - 4, STEP>(r, off + 4, lds_off + 4u * STEP);
    }
}

// The loads of one tile of ROWS rows by WAVES waves: wave-uniform descriptor, 1024 bytes of LDS per load.
template <int RB, int ROWS, int WAVES>
struct SeqLoader {
    static constexpr int kLoads = ROWS * RB / 1024 / WAVES;
    static_assert(kLoads >= 1 && kLoads * 1024 * WAVES == ROWS * RB, "a tile is a whole number of loads per wave");
    uint32_t off[kLoads];
    uint32_t to;
    __device__ __forceinline__ void init(uint32_t wave, uint32_t lane, uint32_t row_bytes) {
        to = wave * 1024u;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint32_t at = ((uint32_t)i * WAVES + wave) * 1024u + lane * 16u;
            const uint32_t row = at / RB, place = (at % RB) / 16u;
            off[i] = row * row_bytes + ((place ^ seq_swizzle<RB>(row)) * 16u);
        }
    }
    // rows from the source's base on, as many as its bytes reach; `lds` = the tile's place
    __device__ __forceinline__ void issue(const u32x4& source, uint32_t lds) const { seq_loads_to_lds<kLoads, 1024 * WAVES>(source, off, lds + to); }
};
// The source of a tensor's tiles, in four scalar registers from tile to tile.
__device__ __forceinline__ u32x4 seq_source(const void* base) { return lds_source(base, 0u); }
__device__ __forceinline__ void seq_advance(u32x4& source, uint64_t bytes) {
    const uint64_t at = (((uint64_t)source[1] << 32) | source[0]) + bytes;
    source[0] = (uint32_t)at;
    source[1] = (uint32_t)(at >> 32);
}
// Bytes from the first of `rows` rows to the end of the last, of at most `most` rows (scalar: the rows of a tile that exist).
template <int RB>
__device__ __forceinline__ uint32_t seq_tile_bytes(int rows, int most, uint32_t row_bytes) {
    const int n = rows < most ? rows : most;
    return n > 0 ? (uint32_t)(n - 1) * row_bytes + RB : 0u;
}

__device__ __forceinline__ u32x4 seq_lds_b128(uint32_t at) {
    return *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)at;
}
__device__ __forceinline__ float seq_lds_f32(uint32_t at) {
    return *(const __attribute__((address_space(3))) float*)(uintptr_t)at;
}
__device__ __forceinline__ f32x4 seq_lds_f32x4(uint32_t at) {
    return *(const __attribute__((address_space(3))) f32x4*)(uintptr_t)at;
}
__device__ __forceinline__ void seq_lds_put(uint32_t at, float x) {
    *(__attribute__((address_space(3))) float*)(uintptr_t)at = x;
}
__device__ __forceinline__ uint2 seq_lds_tr(uint32_t at) {
    typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
    const v4i16 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(uintptr_t)at);
    return __builtin_bit_cast(uint2, v);
}

// Where lane (hi, c) finds chunk 2 s + hi of row c of a tile: place() ^ 32 s, plus 32 RB for the next 32 rows.
template <int RB>
struct SeqRowReader {
    uint32_t at;
    __device__ __forceinline__ void init(uint32_t hi, uint32_t c) { at = c * RB + ((hi ^ seq_swizzle<RB>(c)) << 4); }
    __device__ __forceinline__ u32x4 read(uint32_t tile, int s, int block) const {
        return seq_lds_b128(tile + (at ^ (uint32_t)(32 * s)) + (uint32_t)(32 * RB * block));
    }
};

// Sums over the rows of a tile in LDS: acc[b] += X[rows of the block][channels 32 b ..]^T  times the 32 x 32 tile in `w`, whose registers run
// over the rows.
template <class T, int D>
struct SeqColumnReader {
    static constexpr int RB = D * SeqSize<T>::value;
    uint32_t at;
    __device__ __forceinline__ void init(uint32_t hi, uint32_t c) {
        if constexpr (__is_same(T, SeqF32)) {
            // row 4 hi, channel c
            at = 4u * hi * RB + (((c >> 2) ^ seq_swizzle<RB>(4u * hi)) << 4) + 4u * (c & 3u);
        } else {
            // lane r of 16 passes row 4 hi + (r >> 2), channels 16 (c >> 4) + 4 (r & 3) ..
            const uint32_t r = c & 15u, row = 4u * hi + (r >> 2), chunk = 2u * (c >> 4) + ((r & 3u) >> 1);
            at = row * RB + ((chunk ^ seq_swizzle<RB>(row)) << 4) + 8u * (r & 1u);
        }
    }
    __device__ __forceinline__ void accumulate(f32x16 (&acc)[D / 32], uint32_t tile, int block, const f32x16& w) const {
        tile += (uint32_t)(32 * RB * block);
        if constexpr (__is_same(T, SeqF32)) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const uint32_t row = 8u * (r / 4) + r % 4;  // and 4 hi, in `at`
                const float x = w[r];
#pragma unroll
                for (int b = 0; b < D / 32; ++b) {
                    const uint32_t flip = (seq_swizzle<RB>(row) << 4) ^ (uint32_t)(128 * b);
                    acc[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(seq_lds_f32(tile + (at ^ flip) + row * RB), x, acc[b], 0, 0, 0);
                }
            }
        } else {
            constexpr bool F16 = __is_same(T, SeqF16);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const u32x4 x = {pack_e<F16>(w[8 * t], w[8 * t + 1]), pack_e<F16>(w[8 * t + 2], w[8 * t + 3]),
                                 pack_e<F16>(w[8 * t + 4], w[8 * t + 5]), pack_e<F16>(w[8 * t + 6], w[8 * t + 7])};
#pragma unroll
                for (int b = 0; b < D / 32; ++b) {
                    const uint32_t first = at ^ (uint32_t)(64 * b), second = first ^ (seq_swizzle<RB>(8u) << 4);
                    const uint2 p = seq_lds_tr(tile + first + (uint32_t)(16 * t) * RB);
                    const uint2 q = seq_lds_tr(tile + second + (uint32_t)(16 * t + 8) * RB);
                    acc[b] = seq_dot<T>(u32x4{p.x, p.y, q.x, q.y}, x, acc[b]);
                }
            }
        }
    }
};

// max / sum of a value over the two lanes (0, c), (1, c)
__device__ __forceinline__ float seq_max_halves(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = s[0], b = s[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}
__device__ __forceinline__ float seq_sum_halves(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const uint32_t a = s[0], b = s[1];
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}

__device__ __forceinline__ void seq_zero(f32x16& x) {
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = 0.f;
}

// One entry of the table in base-2 units.  Finite values keep finite in these units: the type's lowest value, which stands for a mask in
// many programs, would otherwise turn into an infinity, and a row of nothing else would be empty instead of uniform.
__device__ __forceinline__ float seq_bias_log2(float b) {
    if (!(fabsf(b) < __builtin_inff())) return b;  // infinities and NaN
    return fminf(fmaxf(b * kLog2e, -3.4e38f), 3.4e38f);
}
// The bias of distance key - query for a head's row of the table; entries of the map outside the table add nothing.
__device__ __forceinline__ float seq_bias_at(const float* row, const int32_t* buckets, int nb, int far, int distance) {
    const int at = distance < -far ? -far : (distance > far ? far : distance);
    const uint32_t b = (uint32_t)buckets[far + at];
    return b < (uint32_t)nb ? seq_bias_log2(row[b]) : 0.f;
}

// Positions are int32 of the caller's; beyond these bounds every distance is cut off at `far` and every comparison decided, so they are
// cut there and sums of a position and a row cannot overflow.
constexpr int kSeqFarthest = 1 << 29;
// (Read through the constant address space: no kernel writes them, and the scalar unit's loads do not queue behind a tile's.)
__device__ __forceinline__ int seq_constant(const int32_t* p, long long n) {
    return ((const __attribute__((address_space(4))) int32_t*)(uintptr_t)p)[n];
}
__device__ __forceinline__ int seq_length(const int32_t* lengths, long long n, int most) {
    if (lengths == nullptr) return most;
    const int x = seq_constant(lengths, n);
    return x < 0 ? 0 : (x > most ? most : x);
}
__device__ __forceinline__ int seq_start(const int32_t* starts, long long n) {
    if (starts == nullptr) return 0;
    const int x = seq_constant(starts, n);
    return x < -kSeqFarthest ? -kSeqFarthest : (x > kSeqFarthest ? kSeqFarthest : x);
}

// Tiles of `size` keys from key 0 on that have a pair with a distance between -far and far, of queries at the positions first .. last:
// t0 .. t1 - 1.  Tiles in front of t0 lie at or beyond -far altogether, those from t1 on at or beyond far.  Without a table all count as the
// latter.
__device__ __forceinline__ void seq_near_tiles(bool table, int first, int last, int far, int size, int& t0, int& t1) {
    t0 = t1 = 0;
    if (!table) return;
    const int x = first - far - size + 1, y = far + last + size - 1;
    t0 = x < 0 ? 0 : x / size + 1;
    t1 = y < 0 ? 0 : y / size;
    if (t1 < t0) t1 = t0;
}

// Tiles of `size` rows from row 0 on that start below row x: ceil(x / size), at least 0.
__device__ __forceinline__ int seq_tiles_up_to(int x, int size) { return x > 0 ? (x + size - 1) / size : 0; }

// A thread's entry of the bias by distance of the tiles to come, for workgroups with a thread for each entry: the map a tile ahead of the table,
// both ahead of their use, so that neither is waited for.  Entries outside the table are 0.
struct SeqBiasAhead {
    uint32_t column, of;  // column of the tile after next; that of `value`
    float value;
    __device__ __forceinline__ void find(const int32_t* buckets, int far, int distance) {
        const int at = distance < -far ? -far : (distance > far ? far : distance);
        column = (uint32_t)buckets[far + at];
    }
    __device__ __forceinline__ void fetch(const float* row, int nb) {
        of = column;
        value = row[column < (uint32_t)nb ? column : 0u];
    }
    __device__ __forceinline__ float get(int nb) const { return of < (uint32_t)nb ? seq_bias_log2(value) : 0.f; }
};

// Four neighbouring channels of a row, rounded to the type.
template <class T>
__device__ __forceinline__ void seq_store4(char* row, uint32_t channel, float a, float b, float c, float d) {
    if constexpr (__is_same(T, SeqF32)) {
        *reinterpret_cast<f32x4*>(row + channel * 4u) = f32x4{a, b, c, d};
    } else {
        constexpr bool F16 = __is_same(T, SeqF16);
        *reinterpret_cast<uint2*>(row + channel * 2u) = uint2{pack_e<F16>(a, b), pack_e<F16>(c, d)};
    }
}

// Which workgroup has which part of which head of which sequence.  Workgroups go to the 8 XCDs in turn, each with an L2 of its own, and an XCD's to its
// 32 CUs.  Heads are dealt to the XCDs in turn, whole ones, whose keys then stay in one L2, and each sequence's to all XCDs, since sequences differ in
// length (contiguous ranges of all heads of all sequences left the CUs of most XCDs idle: encoder of 4 ragged sequences, 16 heads, 102 us against 91).
// Few heads that 8 does not divide are dealt by parts.  Causal parts differ in size: every second round of an XCD's 32 goes backwards,
// so that a CU's parts come to one sum.
struct SeqDeal {
    uint32_t units, each, per_xcd, heads;
    int whole, snake;
    FastDiv by_each, by_heads;
};
inline unsigned seq_deal(SeqDeal& d, long long sequences, int heads, long long each, bool snake) {
    const long long units = sequences * heads;
    d.units = (uint32_t)units;
    d.each = (uint32_t)each;
    d.heads = (uint32_t)heads;
    d.whole = units % 8 == 0 || units >= 64;
    d.per_xcd = (uint32_t)((units + 7) / 8 * each);
    d.snake = snake;
    d.by_each = make_fastdiv(d.each > 0 ? d.each : 1u);
    d.by_heads = make_fastdiv((uint32_t)heads);
    return (unsigned)(d.whole ? 8LL * d.per_xcd : units * each);
}
// false: nothing to do
__device__ __forceinline__ bool seq_dealt(const SeqDeal& d, uint32_t block, uint32_t& sequence, uint32_t& head, uint32_t& part) {
    uint32_t unit;
    if (d.whole) {
        uint32_t at = block >> 3;
        const uint32_t round = at >> 5;
        if (d.snake && (round & 1u) && 32u * round + 32u <= d.per_xcd) at = 64u * round + 31u - at;
        const uint32_t turn = fastdiv(at, d.by_each);
        part = at - turn * d.each;
        unit = 8u * turn + (block & 7u);
        if (unit >= d.units) return false;
    } else {
        unit = fastdiv(block, d.by_each);
        part = block - unit * d.each;
    }
    sequence = fastdiv(unit, d.by_heads);
    head = unit - sequence * d.heads;
    return true;
}

// How a forward call is laid out on the device.
struct SeqPlan {
    int group;           // heads of queries per head of keys
    int packed;          // one block has the rows of a whole group (few rows: group * Lq <= 32)
    int keys;            // the waves of a workgroup share out the keys, not the rows
    int waves, blocks, splits;
    unsigned grid;
    SeqDeal deal;
    uint32_t bias_entries;
    FastDiv by_splits;
    size_t rows;         // N * H * Lq
    float* part_o;       // [splits][rows][D], not divided by the sum
    float* part_ml;      // [splits][rows][2]
};

}  // namespace fwa
