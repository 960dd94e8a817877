// Rotation of pairs of channels by their positions, as fwa_rotary.hip and fwa_page_append.hip have it.
//
// Pair p of a head is turned by the angle position[axis of p] * frequency[p]: (a, b) -> (a c - b s, b c + a s).  A unit of work is V pairs of one
// head of one row: two vectors of V elements.  Channels behind the pairs are copied, 2 V a unit.  Cosine and sine are formed once for all heads of a
// row and read from LDS, V pairs as 8 V bytes in a row.
#pragma once

#include "fwa_internal.h"
#include "fwa_sequence.h"

namespace fwa {

// V neighbouring elements as they stand in memory: 16, 8 or, an element at a time, 4 or 2 bytes.
template <class T, int V>
struct RotaryVector {
    static constexpr int kBytes = V * SeqSize<T>::value, kWords = kBytes >= 4 ? kBytes / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const char* p) {
        if constexpr (kBytes == 16) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = x[i];
        } else if constexpr (kBytes == 8) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            w[0] = x.x;
            w[1] = x.y;
        } else if constexpr (kBytes == 4) {
            w[0] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            w[0] = *reinterpret_cast<const uint16_t*>(p);
        }
    }
    __device__ __forceinline__ void store(char* p) const {
        if constexpr (kBytes == 16) *reinterpret_cast<u32x4*>(p) = u32x4{w[0], w[1], w[2], w[3]};
        else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = uint2{w[0], w[1]};
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (__is_same(T, SeqF32)) {
            const uint32_t x = w[i];
            return __builtin_bit_cast(float, x);
        } else {
            const uint32_t x = i % 2 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
            if constexpr (__is_same(T, SeqBf16)) return __builtin_bit_cast(float, x << 16);
            else return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
        }
    }
    // all elements, rounded to the type
    __device__ __forceinline__ void set(const float* x) {
        if constexpr (__is_same(T, SeqF32)) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i] = __builtin_bit_cast(uint32_t, x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = pack_e<__is_same(T, SeqF16)>(x[2 * i], V == 1 ? 0.f : x[2 * i + 1]);
        }
    }
};

// Cosine and sine of position * frequency.  The product is formed in 64 bits and reduced to a part of one turn there: a position of 2^20 times a
// frequency of 1 has 20 bits of whole turns in front of the angle, of which 32 bits would leave 4; what is left of the reduction's error is 2^-25
// turns, from the fraction's rounding, which the functions of 32 bits need (fp32 data at positions from 10^6: the whole rotation is off by 4.9e-8 of its
// size, 3.7e-8 with cosines formed in 64 bits; 16-bit data hide it).
__device__ __forceinline__ f32x2 rotary_turn(int position, float frequency, bool inverse) {
    constexpr double kPerTurn = 0.15915494309189533577;  // 1 / (2 pi)
    double turns = (double)position * ((double)frequency * kPerTurn);
    turns -= __builtin_rint(turns);
    float s, c;
    sincospif(2.f * (float)turns, &s, &c);
    return f32x2{c, inverse ? -s : s};
}
// In the place of the cosine of a pair that is not turned: no cosine is this.
constexpr float kRotaryStays = 2.f;
// Where the two vectors of unit `u` of a head begin, in channels; the second may not exist for channels that are copied.  Of either kind of pairs a
// unit has V channels of each half of the rotated part, so that neighbouring threads have neighbouring vectors (a single element's interleaved pair
// has its two channels).
struct RotaryUnit {
    int first, second;
    bool turned, both;
};
template <int V>
__device__ __forceinline__ RotaryUnit rotary_unit(int u, int pairs, int d, bool interleaved) {
    RotaryUnit r;
    r.turned = u * V < pairs;
    if (r.turned && !(V == 1 && interleaved)) {
        r.first = u * V;
        r.second = pairs + u * V;
    } else {
        r.first = r.turned ? 2 * u : 2 * pairs + 2 * V * (u - pairs / V);
        r.second = r.first + V;
    }
    r.both = r.second < d;
    return r;
}

// The V pairs of the two vectors of unit `u`, `table` = cosine and sine of the row's pairs in LDS.
template <class T, int V>
__device__ __forceinline__ void rotary_apply(RotaryVector<T, V>& x, RotaryVector<T, V>& y, const f32x2* table, int u, int pairs, bool interleaved) {
    float a[V], b[V];
    // of interleaved pairs the first half is in x, the second in y
    const bool apart = V == 1 || !interleaved;
    const f32x2* const low = table + (apart ? u * V : u * (V / 2));
    const f32x2* const high = apart ? low + V / 2 : low + pairs / 2;
    f32x2 t[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = V == 1 || i < V / 2 ? low[i] : high[i - V / 2];
    auto each = [&](auto pair) {
        if (apart) {
#pragma unroll
            for (int i = 0; i < V; ++i) pair(a[i], b[i], x.get(i), y.get(i), t[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                pair(a[2 * i], a[2 * i + 1], x.get(2 * i), x.get(2 * i + 1), t[i]);
                pair(b[2 * i], b[2 * i + 1], y.get(2 * i), y.get(2 * i + 1), t[V / 2 + i]);
            }
        }
    };
    each([](float& p, float& q, float first, float second, const f32x2& at) {
        p = fmaf(first, at[0], -(second * at[1]));
        q = fmaf(second, at[0], first * at[1]);
    });
    // A pair that is not turned stays as it is: times one and zero, an infinity or NaN of one channel would reach the other.  Looked for in all pairs of the
    // threads that are here together, and put back (append of 1 to 512 tokens of 24 sequences, 36 heads of 64 in all: 13.0 us without, 13.1 so, 13.4 with a selection for
    // each pair).
    float largest = t[0][0];
#pragma unroll
    for (int i = 1; i < V; ++i) largest = fmaxf(largest, t[i][0]);
    if (__any(largest == kRotaryStays))
        each([](float& p, float& q, float first, float second, const f32x2& at) {
            p = at[0] == kRotaryStays ? first : p;
            q = at[0] == kRotaryStays ? second : q;
        });
    x.set(a);
    y.set(b);
}

// Elements of a vector: 16 bytes where widths and pairs are whole vectors, half of that (16-bit data, heads of 72 channels for
// instance), or single elements, which are bound by their instructions (2 x 6272 rows of 16 heads of 80 with 10 pairs, bf16: 64 MB in 24.2 us, vector units 63
// per cent busy).
inline int rotary_vector(int dtype, int d, int pairs) {
    const int most = dtype == 0 ? 4 : 8;
    if (d % most == 0 && pairs % most == 0) return most;
    return dtype != 0 && d % 4 == 0 && pairs % 4 == 0 ? 4 : 1;
}
// units of a head
inline int rotary_units(int d, int pairs, int V) { return pairs / V + (d - 2 * pairs + 2 * V - 1) / (2 * V); }

// Units of a workgroup: 256 threads with two each, or for small calls 128 threads with one each, more workgroups with fewer cosines for each (64 windows of 49
// rows of 3 heads of 32: kernel 5.6 us with 512 units, 3.6 with 128).
struct RotaryShape {
    static constexpr int kLarge = 512, kSmall = 128;
};
inline bool rotary_small(long long total) { return total <= 256 * RotaryShape::kLarge; }
// Rows that a workgroup's units may touch, of `each` units a row.
inline int rotary_rows(long long each, int units) { return (int)((units - 1) / each) + 2; }

// Cosines and sines of `rows` rows into LDS, pairs of a row one behind the other.  A thread has one pair of every so many rows, so that its axis and
// frequency are loaded once, and the positions of four rows at a time.  position(r, axis) is that of row r on an axis of the row's.
template <int THREADS, class Position>
__device__ __forceinline__ void rotary_turns(f32x2* turns, uint32_t rows, int pairs, int axes, const float* frequencies, const int32_t* axis_of, bool inverse,
                                             Position position) {
    uint32_t wide = 1u;  // threads for a row's pairs: a power of two
    while (wide < (uint32_t)pairs && wide < THREADS) wide *= 2u;
    const uint32_t first = threadIdx.x & (wide - 1u), step = THREADS / wide;
    for (uint32_t p = first; p < (uint32_t)pairs; p += wide) {
        const uint32_t axis = axis_of ? (uint32_t)axis_of[p] : 0u;
        const float f = frequencies[p];
        const bool turned = axis < (uint32_t)axes;
        for (uint32_t r0 = threadIdx.x / wide; r0 < rows; r0 += 4u * step) {
            int at[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t r = r0 + k * step;
                at[k] = turned && r < rows ? position(r, axis) : 0;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t r = r0 + k * step;
                if (r < rows) turns[r * (uint32_t)pairs + p] = turned ? rotary_turn(at[k], f, inverse) : f32x2{kRotaryStays, 0.f};
            }
        }
    }
}

}  // namespace fwa
