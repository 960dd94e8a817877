// Gradients of the attention of whole sequences, from q, k, v, o, d_o and the forward's row statistics; the probabilities are formed
// again.  Two kernels, each with the sums of its outputs in registers, so that no gradient needs atomics and every result is the same
// from run to run:
//   rows   a wave has 32 queries and walks the keys: dQ, the row sums delta = sum_j P dP, the sums of dS by distance for the table
//   keys   a wave has 32 keys and walks the queries (of all heads that share them): dK, dV
// Scores and dP = dO V^T are formed in both (14 instead of 10 flops per channel of a pair); the alternative, dQ added up in memory over the
// blocks of keys, has no fixed order.  Both products of a tile use its P and dS as they stand in registers (fwa_sequence.h).
#include "fwa_sequence.h"

#include <type_traits>

namespace fwa {
namespace {

struct BackPlan {
    int group, keys, waves, key_waves, row_blocks, key_blocks, splits;
    unsigned row_grid, key_grid;
    SeqDeal row_deal, key_deal;
    uint32_t row_bias, key_bias;
    FastDiv by_splits;
    int key_least;       // tiles of a part of a block of keys: a block has as many parts as that makes, `splits` at most
    int row_waves;       // waves with rows per head of a sequence: ceil(Lq / 32)
    float* delta;        // [N, H, Lq]
    float* ends;         // [H][N * row_waves][2]: sums of dS at and beyond -far and far
    float* lines;        // [H][2 far + 1]: sums of dS by distance
    float* parts;        // [H][offsets][chunks][kLine]: the same of an offset of blocks
    int low_offset, offsets, chunks, items;
    FastDiv by_offsets, by_chunks, by_table_blocks;
    float* part_kv;      // [splits][2][N, Lk, KV, D]
};

constexpr float kDead = __builtin_inff();
// Half data: P and dS are taken 2^6 times as large and the sums divided again, since a probability of 2^-14 and less (keys by the
// thousand) has fewer bits in that type; dS beyond 1023 overflows.
template <class T>
constexpr float seq_lift() { return __is_same(T, SeqF16) ? 6.f : 0.f; }
// Rows that see few keys: one of these may have nearly all the weight, dP - delta cancels, and the rounding of o would show (bf16, rows of up to 128 keys of
// width 128: elements of dQ up to 1.4e-2 off, now within half a step of each dS).  There a walk in front of the other forms delta from the same products as
// dP (70 sequences of 128 tokens, 8 heads of 128, bf16: whole backward 74 us with it, 68 without).  At every width and in both forms up to this many
// keys, which the first block of a causal call has; waves that share out the keys take it up to two tiles each, where there are more of them.
constexpr int kFewKeys = 128;

// Whether no query of a sequence sees more than one key: its weight is one and stays so, and all but dV is exactly zero, which products and their
// differences need not be to the last bit (and in half data need not be finite).
__device__ __forceinline__ bool seq_lone(bool causal, int start, int qlen, int klen) {
    return klen <= 1 || (causal && start + qlen <= 1);
}
// Whether a row's statistics are those of a row without a key; a row of NaN alone has (-inf, NaN).
__device__ __forceinline__ bool seq_dead(const f32x2& stat) { return stat[0] == -__builtin_inff() && stat[1] == 0.f; }
// a sum that is not fused with a product it takes in: the two forms of the rows kernel give the same bits
__device__ __forceinline__ float plain_sum(float a, float b) {
#pragma clang fp contract(off)
    return a + b;
}

// Two forms, as in the forward: the waves have 32 rows each and share the tiles, or (KEYS) the same 32 rows and every W-th tile each.
// The row's sum is divided out of dQ at the end, but for half data, where it is in the exponent together with the lift: dS times a sum of thousands leaves
// that type's range.
// Bound by vector instructions between the three products and by the latency of a tile (4 ragged sequences of up to 2048 tokens, 12 heads of 64, bf16:
// 106 us, vector units 43 per cent busy, matrix units 25).
template <class T, int D, int W, int KT, bool TABLE, bool KEYS>
__global__ void __launch_bounds__(64 * W) seq_rows_kernel(SeqArgs a, BackPlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, KS = KT / 32;
    constexpr int ROWS = KEYS ? 32 : 32 * W, TURN = KEYS ? W : 1;
    constexpr uint32_t kTile = KT * RB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u, bias_bytes = 4u * plan.row_bias;
    const uint32_t base = lds_offset(lds) + (KEYS ? wave * 4u * kTile : 0u);
    const uint32_t bias_at = lds_offset(lds) + (KEYS ? 4u * W * kTile + wave * 2u * bias_bytes : 4u * kTile);

    uint32_t sequence, unit, part;
    if (!seq_dealt(plan.row_deal, blockIdx.x, sequence, unit, part)) return;
    int block = (int)part;
    const long long n = sequence;
    const int head = (int)unit, kv = head / plan.group;
    if (a.causal) block = plan.row_blocks - 1 - block;
    const int i0 = block * ROWS, i = i0 + (int)(KEYS ? c : 32u * wave + c);
    const int span_rows = a.Lq - i0 < ROWS ? a.Lq - i0 : ROWS;
    const int qlen = seq_length(a.q_len, n, a.Lq), klen = seq_length(a.k_len, n, a.Lk), start = seq_start(a.q_start, n);
    const int first = start + i0, last = first + span_rows - 1, pos = i < a.Lq ? start + i : last;

    int kend = i0 < qlen ? klen : 0;
    if (a.causal && kend > last + 1) kend = last + 1 > 0 ? last + 1 : 0;
    const int tiles = (kend + KT - 1) / KT;

    const char* const kp = static_cast<const char*>(a.k) + ((size_t)n * a.Lk * a.ldk + (size_t)kv * D) * E;
    const char* const vp = static_cast<const char*>(a.v) + ((size_t)n * a.Lk * a.ldk + (size_t)kv * D) * E;
    const uint32_t kld = (uint32_t)(a.ldk * E);
    SeqLoader<RB, KT, KEYS ? 1 : W> load;
    load.init(KEYS ? 0u : wave, lane, kld);
    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    SeqColumnReader<T, D> column_reader;
    column_reader.init(hi, c);
    // the next tile to ask for, and the rows from there on
    const int mine0 = KEYS ? (int)wave : 0;
    u32x4 next_k = seq_source(kp), next_v = seq_source(vp);
    int next_rows;
    const uint32_t whole = (KT - 1u) * kld + RB, rest = seq_tile_bytes<RB>(klen % KT, KT, kld);
    auto issue = [&](uint32_t buf) {
        next_k[2] = next_v[2] = next_rows >= KT ? whole : rest;
        load.issue(next_k, base + buf * 2u * kTile);
        load.issue(next_v, base + buf * 2u * kTile + kTile);
        seq_advance(next_k, (uint64_t)(TURN * KT) * kld);
        seq_advance(next_v, (uint64_t)(TURN * KT) * kld);
        next_rows -= TURN * KT;
    };

    const size_t row = ((size_t)n * a.H + head) * a.Lq + i;
    bool dead = true;
    constexpr bool HALF = __is_same(T, SeqF16);
    float ref = 0.f, log_sum = 0.f, rl = 0.f, delta = 0.f;  // log_sum: what the exponent takes besides the reference; rl: what is left to multiply with
    u32x4 qf[NC], gf[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) qf[s] = gf[s] = u32x4{0u, 0u, 0u, 0u};
    if (i < qlen) {
        const f32x2 stat = *reinterpret_cast<const f32x2*>(a.stats + 2 * row);
        dead = seq_dead(stat);
        ref = dead ? 0.f : stat[0];
        if (HALF && !dead) log_sum = stat[1] - seq_lift<T>();
        rl = dead ? 0.f : __builtin_amdgcn_exp2f(HALF ? -seq_lift<T>() : -stat[1]);
        const bool lone = seq_lone(a.causal, start, qlen, klen);  // dP and delta from a d_o of zero
        const size_t at_row = (size_t)n * a.Lq + i, channel = (size_t)head * D;
        const char* const qp = static_cast<const char*>(a.q) + (at_row * a.ldq + channel) * E + 16u * hi;
        const char* const gp = static_cast<const char*>(a.d_o) + (at_row * a.ldg + channel) * E + 16u * hi;
        const char* const op = static_cast<const char*>(a.o) + (at_row * a.ldo + channel) * E + 16u * hi;
        // delta as the product of d_o and the rounded output; the rounding is taken out below
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            qf[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
            if (!lone) gf[s] = *reinterpret_cast<const u32x4*>(gp + 32 * s);
            const u32x4 of = *reinterpret_cast<const u32x4*>(op + 32 * s);
            if constexpr (__is_same(T, SeqF32)) {
                const f32x4 x = __builtin_bit_cast(f32x4, of), y = __builtin_bit_cast(f32x4, gf[s]);
#pragma unroll
                for (int e = 0; e < 4; ++e) delta = fmaf(x[e], y[e], delta);
            } else if constexpr (__is_same(T, SeqF16)) {
                const f16x8 x = __builtin_bit_cast(f16x8, of), y = __builtin_bit_cast(f16x8, gf[s]);
#pragma unroll
                for (int e = 0; e < 8; ++e) delta = fmaf((float)x[e], (float)y[e], delta);
            } else {
                const bf16x8 x = as_bf16x8(of), y = as_bf16x8(gf[s]);
#pragma unroll
                for (int e = 0; e < 8; ++e) delta = fmaf((float)x[e], (float)y[e], delta);
            }
        }
    }
    delta = seq_sum_halves(delta);
    const bool some_dead = __any(dead);
    // one number for both where the reference is not large, as in the keys kernel
    const bool large = HALF && __any(fabsf(ref) > 1024.f && ref != -__builtin_inff());
    const float off_exponent = HALF ? ref + log_sum : ref;
    if (klen % KT != 0 && tiles > 0) {  // rows that no load fills: as in the forward
        for (uint32_t o = threadIdx.x * 16u; o < (KEYS ? 4u * W : 4u) * kTile; o += 64u * W * 16u) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    }

    const float* const table = a.table ? a.table + (size_t)head * a.nb : nullptr;
    const int far = a.far;
    const float below = table ? seq_bias_at(table, a.buckets, a.nb, far, -far) : 0.f, above = table ? seq_bias_at(table, a.buckets, a.nb, far, far) : 0.f;
    const bool modest = !__any(!(fabsf(below) < 256.f && fabsf(above) < 256.f));  // as in the forward
    const uint32_t entries = (uint32_t)(KT + span_rows - 1), my_bias = bias_at + 4u * ((uint32_t)(last - pos) + 4u * hi);
    const int lim = dead ? 0 : (a.causal && pos + 1 < klen ? pos + 1 : klen);
    const float scale = a.scale * kLog2e;
    int near0, near1, mask0 = klen / KT;
    seq_near_tiles(table != nullptr, first, last, far, KT, near0, near1);
    if (a.causal && first < klen) {
        const int to = first + 1 > 0 ? (first + 1) / KT : 0;
        mask0 = to < mask0 ? to : mask0;
    }
    if (some_dead) mask0 = 0;

    const uint32_t entry = KEYS ? lane : threadIdx.x;  // of the bias of a near tile: one for each thread at most
    static_assert(KT + ROWS - 1 <= (KEYS ? 64 : 64 * W), "a thread for each distance of a tile");
    SeqBiasAhead ahead = {0u, 0u, 0.f};
    auto find = [&](int t) { if (t >= near0 && t < near1) ahead.find(a.buckets, far, t * KT - last + (int)entry); };
    auto fetch = [&](int t) { if (t >= near0 && t < near1) ahead.fetch(table, a.nb); };
    // before the barrier of tile t: its bias; behind it: what the tiles that follow need
    auto begin = [&](int t, uint32_t buf) {
        if (t >= near0 && t < near1 && entry < entries) seq_lds_put(bias_at + buf * bias_bytes + 4u * entry, ahead.get(a.nb));
        lds_loads_done();
        if constexpr (!KEYS) __syncthreads();
        fetch(t + TURN);
        find(t + 2 * TURN);
        if (t + TURN < tiles) issue(buf ^ 1u);
    };
    auto start_walk = [&]() {
        find(mine0);
        fetch(mine0);
        find(mine0 + TURN);
        const size_t skip = (size_t)mine0 * KT * kld;
        next_k = seq_source(kp + skip);
        next_v = seq_source(vp + skip);
        next_rows = klen - mine0 * KT;
        if (mine0 < tiles) issue(0);
    };
    auto walk = [&](auto step) {
        if constexpr (KEYS) {
            uint32_t parity = 0;
            for (int t = mine0; t < tiles; t += TURN, parity ^= 1u) step(parity, t);
        } else {
            for (int t = 0; t < tiles; t += 2) {
                step(std::integral_constant<uint32_t, 0>{}, t);
                if (t + 1 < tiles) step(std::integral_constant<uint32_t, 1>{}, t + 1);
            }
        }
    };
    // a sum over the waves that share the rows, in the order of the waves; in a place behind the tiles, whose rows that no load fills have to keep
    // what they hold for the next walk
    auto over_waves = [&](float x) {
        if constexpr (KEYS && W > 1) {
            const uint32_t sums = lds_offset(lds) + 4u * W * kTile + 2u * W * bias_bytes;
            __syncthreads();
            if (hi == 0) seq_lds_put(sums + 4u * (32u * wave + c), x);
            __syncthreads();
            x = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) x += seq_lds_f32(sums + 4u * (32u * w + c));
        }
        return x;
    };
    // Q K^T of tile t, or, where the bias is not one value or pairs are shut out, the scores; the exponent of a weight, the row's sum (but of half
    // data) not divided out, is s mul + minus
    struct Exponent { float mul, minus; };
    auto scores = [&](auto parity, int t, f32x16 (&s)[KS]) -> Exponent {
        const uint32_t B = parity;
        const uint32_t kt = base + B * 2u * kTile;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            seq_zero(s[k]);
#pragma unroll
            for (int x = 0; x < NC; ++x) s[k] = seq_dot<T>(row_reader.read(kt, x, k), qf[x], s[k]);
        }
        const float flat = t < near0 ? below : above;
        const bool near = t >= near0 && t < near1, plain = modest && !near && t < mask0 && !large;
        if (!plain) {
            if (near) {
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] = fmaf(s[k][r], scale, seq_lds_f32(my_bias + B * bias_bytes + 4u * (32 * k + 8 * (r / 4) + r % 4)));
            } else {
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] = fmaf(s[k][r], scale, flat);
            }
            if (t >= mask0) {
                const int room = lim - t * KT - 4 * (int)hi;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] = 32 * k + 8 * (r / 4) + r % 4 < room ? s[k][r] : -__builtin_inff();
            }
            if (large) {
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] -= ref;
            }
        }
        return {plain ? scale : 1.f, plain ? flat - off_exponent : large ? -log_sum : -off_exponent};
    };

    f32x16 dq[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) seq_zero(dq[b]);
    float ds_all = 0.f, ds_below = 0.f, ds_above = 0.f, p_below = 0.f, p_above = 0.f;
    start_walk();
    if (tiles > 0 && (tiles * KT <= kFewKeys || (KEYS && tiles <= 2 * W))) {
        float sum = 0.f;
        walk([&](auto parity, int t) {
            const uint32_t B = parity;
            begin(t, B);
            f32x16 s[KS];
            const Exponent e = scores(parity, t, s);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                f32x16 dp;
                seq_zero(dp);
#pragma unroll
                for (int x = 0; x < NC; ++x) dp = seq_dot<T>(row_reader.read(base + B * 2u * kTile + kTile, x, k), gf[x], dp);
#pragma unroll
                for (int r = 0; r < 16; ++r) sum = fmaf(__builtin_amdgcn_exp2f(fmaf(s[k][r], e.mul, e.minus)), dp[r], sum);
            }
        });
        delta = rl * over_waves(seq_sum_halves(sum));
        __syncthreads();
        start_walk();
    }
    f32x16 minus_delta;
#pragma unroll
    for (int r = 0; r < 16; ++r) minus_delta[r] = -delta;
    walk([&](auto parity, int t) {
        const uint32_t B = parity;
        begin(t, B);
        f32x16 s[KS];
        const Exponent ex = scores(parity, t, s);
        float ds_tile = 0.f, p_tile = 0.f;
        // distances of the tile: all at or beyond an end, or some of them
        const int nearest = t * KT - last, furthest = t * KT + KT - 1 - first;
        const bool border = TABLE && t >= near0 && t < near1 && (nearest <= -far || furthest >= far);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            f32x16 ds = minus_delta;
#pragma unroll
            for (int x = 0; x < NC; ++x) ds = seq_dot<T>(row_reader.read(base + B * 2u * kTile + kTile, x, k), gf[x], ds);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[k][r] = __builtin_amdgcn_exp2f(fmaf(s[k][r], ex.mul, ex.minus));
                ds[r] *= s[k][r];
                ds_tile = plain_sum(ds_tile, ds[r]);
                if constexpr (TABLE) p_tile += s[k][r];
            }
            column_reader.accumulate(dq, base + B * 2u * kTile, k, ds);
            if (border) {
                int d = t * KT + 4 * (int)hi - pos;
                asm volatile("" : "+v"(d));  // a branch, not selections in every tile
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int x = d + 32 * k + 8 * (r / 4) + r % 4;
                    ds_below += x <= -far ? ds[r] : 0.f;
                    p_below += x <= -far ? s[k][r] : 0.f;
                    ds_above += x >= far && x > -far ? ds[r] : 0.f;
                    p_above += x >= far && x > -far ? s[k][r] : 0.f;
                }
            }
        }
        ds_all = plain_sum(ds_all, ds_tile);
        if constexpr (TABLE) {
            const bool is_below = t < near0, is_above = t >= near1;
            ds_below += is_below ? ds_tile : 0.f;
            p_below += is_below ? p_tile : 0.f;
            ds_above += is_above ? ds_tile : 0.f;
            p_above += is_above ? p_tile : 0.f;
        }
    });
    // The dS of a row add up to zero; what they add up to is what delta is off by, times the row's weights.  dQ of 16-bit data keeps
    // it (it is below the roundings of dS); dK and the sums by distance, which are not rounded, get the better delta.
    const float off = rl * over_waves(seq_sum_halves(ds_all));
    delta = plain_sum(delta, off);

    if constexpr (TABLE) {
        // Pairs at or beyond far in either direction, all in one column of the table each: their sums, of the wave's rows.  The others are
        // added up by distance in seq_table_kernel, with the delta that is known now.
        float sum_below = dead ? 0.f : rl * (ds_below - off * p_below), sum_above = dead ? 0.f : rl * (ds_above - off * p_above);
#pragma unroll
        for (int x = 32; x > 0; x /= 2) {
            sum_below += __shfl_xor(sum_below, x, 64);
            sum_above += __shfl_xor(sum_above, x, 64);
        }
        if constexpr (KEYS && W > 1) {  // the same in every lane: sums over the waves too
            sum_below = over_waves(sum_below);
            sum_above = over_waves(sum_above);
        }
        const int rw = KEYS ? block : block * W + (int)wave;
        if (lane == 0 && rw < plan.row_waves && (!KEYS || wave == W - 1))
            *reinterpret_cast<f32x2*>(plan.ends + 2 * (((size_t)head * a.N + n) * plan.row_waves + rw)) = f32x2{sum_below, sum_above};
    }

    if constexpr (KEYS && W > 1) {
        // dQ of all waves: rows 4 floats apart from a multiple of the banks; the last wave has it, the others are done
        constexpr uint32_t kRow = 4u * (D + 4);
        const uint32_t all = lds_offset(lds);
        __syncthreads();
        if (wave != W - 1) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(all + kRow * (32u * wave + c) + 4u * (32 * b + 8 * q + 4 * hi)) =
                        f32x4{dq[b][4 * q], dq[b][4 * q + 1], dq[b][4 * q + 2], dq[b][4 * q + 3]};
        }
        __syncthreads();
        if (wave != W - 1) return;
#pragma unroll
        for (int w = 0; w < W - 1; ++w)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 x = seq_lds_f32x4(all + kRow * (32u * w + c) + 4u * (32 * b + 8 * q + 4 * hi));
#pragma unroll
                    for (int e = 0; e < 4; ++e) dq[b][4 * q + e] += x[e];
                }
    }

    if (i >= a.Lq) return;
    if (hi == 0) plan.delta[row] = dead ? 0.f : delta;
    const float f = rl * a.scale;
    char* const to = static_cast<char*>(a.dq) + (((size_t)n * a.Lq + i) * a.lddq + (size_t)head * D) * E;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = dead ? 0.f : dq[b][4 * q + e] * f;
            seq_store4<T>(to, 32 * b + 8 * q + 4 * hi, x[0], x[1], x[2], x[3]);
        }
}

// Sums of dS by distance, -far < d < far.  Blocks of 128 queries and 64 keys whose first key stands 64 x positions behind the
// first query, x an offset, have the same distance in the same place: a workgroup adds the dS of such blocks of one head, of all
// sequences and all rows (its share of them, a chunk), up in registers, 32 queries a wave, and forms the sums along the diagonals
// once at its end.  The bias of a place is the same for all of them and stays in registers too.  Bound by latency, one tile of K and V for two
// products (4 ragged sequences of up to 2048 tokens, 12 heads of 64, far 128: 41 us; atomics on LDS along the diagonals took 265 cycles each).
constexpr int kTableRows = 128, kTableKeys = 64, kLine = 192;

template <class T, int D>
__global__ void __launch_bounds__(256) seq_table_kernel(SeqArgs a, BackPlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, KT = RB >= 512 ? 32 : kTableKeys, KS = KT / 32, HALVES = kTableKeys / KT;
    constexpr uint32_t kTile = KT * RB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t base = lds_offset(lds);
    const uint32_t lane = threadIdx.x & 63u, wave = (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u;
    uint32_t rest = fastdiv(blockIdx.x, plan.by_chunks);
    const int chunk = (int)(blockIdx.x - rest * plan.by_chunks.d);
    const int head = (int)fastdiv(rest, plan.by_offsets), kv = head / plan.group;
    const int offset = plan.low_offset + (int)(rest - (uint32_t)head * plan.by_offsets.d);
    const int far = a.far;
    const float* const table = a.table + (size_t)head * a.nb;
    const float scale = a.scale * kLog2e;

    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    const uint32_t kld = (uint32_t)(a.ldk * E);
    SeqLoader<RB, KT, 4> load;
    load.init(wave, lane, kld);

    // the bias of a place: key - row = e - 127 in the block
    const uint32_t bias_at = base + 4u * kTile;
    if (threadIdx.x < kLine - 1)
        seq_lds_put(bias_at + 4u * threadIdx.x, seq_bias_at(table, a.buckets, a.nb, far, kTableKeys * offset + (int)threadIdx.x - kTableRows + 1));
    const uint32_t my_bias = bias_at + 4u * (4u * hi + 127u - 32u * wave - c);
    f32x16 sum[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) seq_zero(sum[k]);

    // the next block of the chunk (every plan.chunks-th: sequences differ in length) with a pair in it, and its sizes
    const int end = plan.items;
    struct Block { int n, i0, qlen, klen, start, j0; };
    auto at_item = [&](int item) {
        Block x;
        x.n = (int)fastdiv((uint32_t)item, plan.by_table_blocks);
        x.i0 = kTableRows * (item - x.n * (int)plan.by_table_blocks.d);
        x.qlen = seq_length(a.q_len, x.n, a.Lq);
        x.klen = seq_length(a.k_len, x.n, a.Lk);
        x.start = seq_start(a.q_start, x.n);
        x.j0 = x.start + x.i0 + kTableKeys * offset;
        return x;
    };
    auto find = [&](int item) {
        for (; item < end; item += plan.chunks) {
            const Block x = at_item(item);
            if (x.i0 < x.qlen && x.j0 < x.klen && x.j0 + kTableKeys > 0 && !seq_lone(a.causal, x.start, x.qlen, x.klen)) break;
        }
        return __builtin_amdgcn_readfirstlane(item);
    };
    // keys in front of the first one are not loaded either: the rows' offsets count from the first key that exists, and wrap
    auto issue = [&](const Block& x, int half, uint32_t buf) {
        const int j = x.j0 + half * KT, from = j < 0 ? 0 : j;
        const int rows = x.klen - from < KT + j - from ? x.klen - from : KT + j - from;
        const size_t at = (((size_t)x.n * a.Lk + from) * a.ldk + (size_t)kv * D) * E;
        const uint32_t bytes = rows > 0 ? (uint32_t)(rows - 1) * kld + RB : 0u, shift = (uint32_t)(from - j) * kld;
        SeqLoader<RB, KT, 4> shifted = load;
#pragma unroll
        for (int i = 0; i < load.kLoads; ++i) shifted.off[i] -= shift;
        shifted.issue(lds_source(static_cast<const char*>(a.k) + at, bytes), base + buf * 2u * kTile);
        shifted.issue(lds_source(static_cast<const char*>(a.v) + at, bytes), base + buf * 2u * kTile + kTile);
    };

    // what no load fills: its scores are shut out, but zero times what LDS may hold has to be zero
    for (uint32_t o = threadIdx.x * 16u; o < 4u * kTile; o += 4096u) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();

    // the rows of a block, fetched while the one before is worked on; not the wider ones, which leave room for two waves on a SIMD that way (width 128,
    // bf16, 2 x 1023 tokens: 33 us with one)
    constexpr bool AHEAD = RB <= 128;
    struct Rows { u32x4 q[NC], g[NC]; f32x2 stat; float delta; };
    auto fetch = [&](const Block& x, Rows& to) {
        const int i = x.i0 + (int)(32u * wave + c);
        to.stat = f32x2{-__builtin_inff(), 0.f};
        to.delta = 0.f;
#pragma unroll
        for (int s = 0; s < NC; ++s) to.q[s] = to.g[s] = u32x4{0u, 0u, 0u, 0u};
        if (i < x.qlen) {
            const size_t row = ((size_t)x.n * a.H + head) * a.Lq + i, at_row = (size_t)x.n * a.Lq + i, channel = (size_t)head * D;
            to.stat = *reinterpret_cast<const f32x2*>(a.stats + 2 * row);
            to.delta = plan.delta[row];
            const char* const qp = static_cast<const char*>(a.q) + (at_row * a.ldq + channel) * E + 16u * hi;
            const char* const gp = static_cast<const char*>(a.d_o) + (at_row * a.ldg + channel) * E + 16u * hi;
#pragma unroll
            for (int s = 0; s < NC; ++s) {
                to.q[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
                to.g[s] = *reinterpret_cast<const u32x4*>(gp + 32 * s);
            }
        }
    };
    int item = find(chunk);
    Rows even, odd;
    if (item < end) {
        issue(at_item(item), 0, 0);
        if constexpr (AHEAD) fetch(at_item(item), even);
    }
    auto step = [&](auto parity, Rows& mine, Rows& other) {
        constexpr uint32_t P = decltype(parity)::value;
        const Block now = at_item(item);
        if constexpr (!AHEAD) fetch(now, mine);
        item = find(item + plan.chunks);
        const bool live = !seq_dead(mine.stat);
        const int pos = now.start + now.i0 + (int)(32u * wave + c);
        const int lim = !live ? 0 : (a.causal && pos + 1 < now.klen ? pos + 1 : now.klen);
        // reference and sum as one number where the reference is not large (as in the keys kernel; its rounding is one factor for the row)
        const bool small = !__any(live && fabsf(mine.stat[0]) > 1024.f);
        const float ref = live ? mine.stat[0] : 0.f, l = live ? mine.stat[1] : kDead;
        const float first_off = small ? ref + l : ref, then_off = small ? 0.f : l;
        const bool inside = now.j0 >= 0 && !__any(now.j0 + kTableKeys > lim);
#pragma unroll
        for (int half = 0; half < HALVES; ++half) {
            constexpr uint32_t kStart = HALVES == 1 ? P : 0u;
            const uint32_t buf = kStart ^ (uint32_t)(half & 1);
            lds_loads_done();
            __syncthreads();
            if (half + 1 < HALVES) issue(now, half + 1, buf ^ 1u);
            else if (item < end) {
                const Block next = at_item(item);
                if constexpr (AHEAD) fetch(next, other);
                issue(next, 0, buf ^ 1u);
            }
            const uint32_t kt = base + buf * 2u * kTile, vt = kt + kTile;
            const int j0 = now.j0 + half * KT + 4 * (int)hi;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int block = half * KS + k;
                f32x16 p, dp;
                seq_zero(p);
                seq_zero(dp);
#pragma unroll
                for (int x = 0; x < NC; ++x) p = seq_dot<T>(row_reader.read(kt, x, k), mine.q[x], p);
#pragma unroll
                for (int x = 0; x < NC; ++x) dp = seq_dot<T>(row_reader.read(vt, x, k), mine.g[x], dp);
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    p[r] = fmaf(p[r], scale, seq_lds_f32(my_bias + 4u * (32 * block + 8 * (r / 4) + r % 4))) - first_off;
                if (!small) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) p[r] -= then_off;
                }
                if (!inside) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int j = j0 + 32 * k + 8 * (r / 4) + r % 4;
                        p[r] = j >= 0 && j < lim ? p[r] : -__builtin_inff();
                    }
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[block][r] = fmaf(__builtin_amdgcn_exp2f(p[r]), dp[r] - mine.delta, sum[block][r]);
            }
        }
    };
    while (item < end) {
        step(std::integral_constant<uint32_t, 0>{}, even, odd);
        if (item >= end) break;
        step(std::integral_constant<uint32_t, 1>{}, AHEAD ? odd : even, even);
    }

    // Diagonals of the wave's two squares of 32: each goes through LDS, rows of keys 33 apart; a lane follows one of the 63.
    __syncthreads();
    const uint32_t square = base + wave * (33u * 32u * 4u), each = base + 4u * (33u * 32u * 4u);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int r = 0; r < 16; ++r) seq_lds_put(square + 4u * (33u * (8 * (r / 4) + 4 * hi + r % 4) + c), sum[k][r]);
        __syncthreads();
        float x = 0.f;
#pragma unroll
        for (int cc = 0; cc < 32; ++cc) {
            const int key = (int)lane - 31 + cc;
            const float y = seq_lds_f32(square + 4u * (uint32_t)(33 * (key & 31) + cc));
            x += key >= 0 && key < 32 ? y : 0.f;
        }
        seq_lds_put(each + 4u * (64u * (2u * wave + k) + lane), x);  // key - row = lane - 31 of the square; lane 63: nothing
        __syncthreads();
    }
    // place x of the line: key - row = x - 127 in the block
    if (threadIdx.x < kLine) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = (int)threadIdx.x - 96 + 32 * w - 32 * k;
                if (at >= 0 && at < 63) x += seq_lds_f32(each + 4u * (uint32_t)(64 * (2 * w + k) + at));
            }
        plan.parts[(size_t)blockIdx.x * kLine + threadIdx.x] = x;
    }
}

// Lines of one head by distance: what the offsets that meet a distance have of it, and the two ends.  5 us, the launch and one way through memory;
// one workgroup a head that forms the sums by bucket as well took 9.5, as long as the two launches.
__global__ void __launch_bounds__(256) seq_lines_kernel(SeqArgs a, BackPlan plan) {
    const int head = (int)blockIdx.y, far = a.far;
    float* const line = plan.lines + (size_t)head * (2 * (size_t)far + 1);
    if (blockIdx.x == 0) {
        const float* const ends = plan.ends + 2 * (size_t)head * a.N * plan.row_waves;
        const long long count = a.N * plan.row_waves;
        f32x2 sum = {0.f, 0.f};
        for (long long w = threadIdx.x; w < count; w += 256) {
            const f32x2 x = *reinterpret_cast<const f32x2*>(ends + 2 * w);
            sum[0] += x[0];
            sum[1] += x[1];
        }
        __shared__ float sums[2][256];
        sums[0][threadIdx.x] = sum[0];
        sums[1][threadIdx.x] = sum[1];
        for (unsigned x = 128; x > 0; x /= 2) {
            __syncthreads();
            if (threadIdx.x < x) {
                sums[0][threadIdx.x] += sums[0][threadIdx.x + x];
                sums[1][threadIdx.x] += sums[1][threadIdx.x + x];
            }
        }
        if (threadIdx.x == 0) {
            if (far == 0) line[0] = sums[0][0] + sums[1][0];
            else {
                line[0] = sums[0][0];
                line[2 * (size_t)far] = sums[1][0];
            }
        }
        return;
    }
    // four threads a distance share its chunks
    const int d = ((int)blockIdx.x - 1) * 64 + (int)(threadIdx.x >> 2) - far + 1;
    float sum = 0.f;
    if (d < far)
        for (int x = 0; x < plan.offsets; ++x) {
            const int at = d - kTableKeys * (plan.low_offset + x) + kTableRows - 1;
            if (at < 0 || at >= kTableRows + kTableKeys - 1) continue;
            const float* const src = plan.parts + ((size_t)head * plan.offsets + x) * plan.chunks * kLine + at;
            for (int w = (int)(threadIdx.x & 3u); w < plan.chunks; w += 4) sum += src[(size_t)w * kLine];
        }
    sum += __shfl_xor(sum, 1, 64);
    sum += __shfl_xor(sum, 2, 64);
    if (d < far && (threadIdx.x & 3u) == 0) line[far + d] = sum;
}

constexpr bool seq_keys_v_in_lds(int row_bytes) { return row_bytes == 256; }

// The keys kernel is bound by its reads of LDS and by the latency of a tile: four products a tile, four of their operands through LDS, on two waves a SIMD
// (4 ragged sequences of up to 2048 tokens, 12 heads of 64, bf16: 138 us, LDS 30 per cent busy, matrix units 26; 2 x 1023 causal
// tokens, 16 heads of 128 on 4: 44 us, of which 64 MB of parts).

// Tiles of queries that see a key of the block from j0 on: each of q0 .. q0 + each - 1, of every head that shares the keys.
__device__ __forceinline__ void seq_key_tiles(bool causal, int qlen, int klen, int start, int j0, int size, int& q0, int& each) {
    q0 = causal && j0 > start ? (j0 - start) / size : 0;
    const int q1 = j0 < klen ? (qlen + size - 1) / size : 0;
    each = q1 > q0 ? q1 - q0 : 0;
}
// Parts that a block of so many tiles has.
__device__ __forceinline__ int seq_key_parts(int all, const BackPlan& plan) {
    const int parts = (all + plan.key_least - 1) / plan.key_least;
    return parts < plan.splits ? parts : plan.splits;
}

template <class T, int D, int W, int QT>
__global__ void __launch_bounds__(64 * W, D * SeqSize<T>::value == 256 ? 2 : 1) seq_keys_kernel(SeqArgs a, BackPlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, QS = QT / 32;
    // Rows of 256 bytes: the block's V stays in LDS, read again for every tile of queries, where K, V and both gradients would not leave registers
    // for two waves on a SIMD.
    constexpr bool VLDS = seq_keys_v_in_lds(RB);
    constexpr uint32_t kTile = QT * RB, kStat = 16u * QT;  // of each row: exponent's addend, reference, logarithm of the sum, minus delta
    constexpr uint32_t kV = VLDS ? 32u * W * RB : 0u;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t base = lds_offset(lds), v_at = base + 4u * kTile, stat_at = v_at + kV, zero_at = stat_at + 2u * kStat, bias_at = zero_at + 4u * QT + 16u,
                   bias_bytes = 4u * plan.key_bias;
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u;

    uint32_t sequence, unit, part;
    if (!seq_dealt(plan.key_deal, blockIdx.x, sequence, unit, part)) return;
    const int block = (int)fastdiv(part, plan.by_splits), split = (int)part - block * (int)plan.by_splits.d;
    const long long n = sequence;
    const int kv = (int)unit;
    const int j0 = block * 32 * W, j = j0 + (int)(32u * wave + c), j_last = j0 + 32 * W - 1;
    const int qlen = seq_length(a.q_len, n, a.Lq), klen = seq_length(a.k_len, n, a.Lk), start = seq_start(a.q_start, n);

    // the heads that share a block's keys one after the other
    int q0, each, s0 = 0, s1;
    seq_key_tiles(a.causal, qlen, klen, start, j0, QT, q0, each);
    const int q1 = q0 + each, all = s1 = each * plan.group;
    if (plan.splits > 1) {
        const int parts = seq_key_parts(all, plan);
        if (split >= parts) return;  // the joining kernel does not read it
        const int per = (all + parts - 1) / parts;
        s0 = split * per;
        s1 = s0 + per < all ? s0 + per : all;
    }

    const uint32_t qld = (uint32_t)(a.ldq * E), gld = (uint32_t)(a.ldg * E);
    SeqLoader<RB, QT, W> load_q, load_g;
    load_q.init(wave, lane, qld);
    load_g.init(wave, lane, gld);
    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    SeqColumnReader<T, D> column_reader;
    column_reader.init(hi, c);

    // a tile: of the queries, and which of the heads
    struct Place { int g, t; };
    auto behind = [&](Place x) { return x.t + 1 == q1 ? Place{x.g + 1, q0} : Place{x.g, x.t + 1}; };
    Place now{0, q0};
    if (each > 0) {
        now.g = s0 / each;
        now.t = q0 + s0 - now.g * each;
    }
    // the next tile to ask for, and its first row in the statistics; behind the last tile of a head comes the first of the next one
    const int head0 = kv * plan.group + now.g;
    const size_t row0 = (size_t)n * a.Lq + (size_t)now.t * QT;
    u32x4 next_q = seq_source(static_cast<const char*>(a.q) + (row0 * a.ldq + (size_t)head0 * D) * E);
    u32x4 next_g = seq_source(static_cast<const char*>(a.d_o) + (row0 * a.ldg + (size_t)head0 * D) * E);
    int64_t next_row = (int64_t)(((size_t)n * a.H + head0) * a.Lq) + (int64_t)now.t * QT;
    const int64_t back = (int64_t)(each > 0 ? each - 1 : 0) * QT;
    const uint64_t on_q = (uint64_t)QT * qld, on_g = (uint64_t)QT * gld, over_q = (uint64_t)(D * E - back * (int64_t)qld), over_g = (uint64_t)(D * E - back * (int64_t)gld);
    const uint32_t whole_q = (QT - 1u) * qld + RB, whole_g = (QT - 1u) * gld + RB;
    const uint32_t rest_q = qlen % QT ? seq_tile_bytes<RB>(qlen % QT, QT, qld) : whole_q, rest_g = qlen % QT ? seq_tile_bytes<RB>(qlen % QT, QT, gld) : whole_g;
    auto issue = [&](const Place& x, uint32_t buf) {
        const bool last = x.t + 1 == q1;
        next_q[2] = last ? rest_q : whole_q;
        next_g[2] = last ? rest_g : whole_g;
        load_q.issue(next_q, base + buf * 2u * kTile);
        load_g.issue(next_g, base + buf * 2u * kTile + kTile);
        seq_advance(next_q, last ? over_q : on_q);
        seq_advance(next_g, last ? over_g : on_g);
        next_row += last ? a.Lq - back : (int64_t)QT;
    };

    u32x4 kf[NC], vf[VLDS ? 1 : NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) {
        kf[s] = u32x4{0u, 0u, 0u, 0u};
        if constexpr (!VLDS) vf[s] = u32x4{0u, 0u, 0u, 0u};
    }
    const uint32_t kld = (uint32_t)(a.ldk * E);
    if (j < klen) {
        const size_t from = (((size_t)n * a.Lk + j) * a.ldk + (size_t)kv * D) * E + 16u * hi;
        const char* const kp = static_cast<const char*>(a.k) + from;
        const char* const vp = static_cast<const char*>(a.v) + from;
#pragma unroll
        for (int s = 0; s < NC; ++s) {
            kf[s] = *reinterpret_cast<const u32x4*>(kp + 32 * s);
            if constexpr (!VLDS) vf[s] = *reinterpret_cast<const u32x4*>(vp + 32 * s);
        }
    }
    if ((qlen % QT != 0 || (VLDS && j_last >= klen)) && s0 < s1) {
        for (uint32_t o = threadIdx.x * 16u; o < 4u * kTile + kV; o += 64u * W * 16u) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    if constexpr (VLDS) {
        if (s0 < s1) {
            SeqLoader<RB, 32 * W, W> load_v;
            load_v.init(wave, lane, kld);
            load_v.issue(lds_source(static_cast<const char*>(a.v) + (((size_t)n * a.Lk + j0) * a.ldk + (size_t)kv * D) * E, seq_tile_bytes<RB>(klen - j0, 32 * W, kld)), v_at);
        }
    }

    f32x16 dk[NB], dv[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        seq_zero(dk[b]);
        seq_zero(dv[b]);
    }
    const int far = a.far;
    const float scale = a.scale * kLog2e;
    for (uint32_t e = threadIdx.x; e < (uint32_t)QT; e += 64u * W) seq_lds_put(zero_at + 4u * e, 0.f);

    // tiles of queries as the keys of this block see them: near0 .. near1 - 1 with distances between -far and far (those before are at or
    // beyond far, those behind at or beyond -far); causality shuts pairs out up to mask1 - 1, the end of the keys in every tile
    int near0 = 0, near1 = 0, mask1 = a.causal ? seq_tiles_up_to(j_last - start, QT) : 0;
    if (a.table) {
        near0 = seq_tiles_up_to(j0 - start - far - QT + 1, QT);
        near1 = seq_tiles_up_to(j_last - start + far, QT);
        if (near1 < near0) near1 = near0;
    }
    if (j_last >= klen) mask1 = 1 << 30;
    const int from_row = j < klen ? (a.causal ? j - start : -(1 << 30)) : 1 << 30;  // query from which on the lane's key is seen
    float below = 0.f, above = 0.f;
    bool modest = true;
    int ends_of = -1;  // the head whose they are
    auto ends = [&](int g) {
        if (!a.table || g == ends_of) return;
        ends_of = g;
        const float* const row = a.table + (size_t)(kv * plan.group + g) * a.nb;
        below = seq_bias_at(row, a.buckets, a.nb, far, -far);
        above = seq_bias_at(row, a.buckets, a.nb, far, far);
        modest = fabsf(below) < 256.f && fabsf(above) < 256.f;
    };

    // a thread's row of the statistics, and entry of the bias, of the tiles to come
    f32x2 stat_ahead = {0.f, 0.f};
    float delta_ahead = 0.f;
    bool row_ahead = false;
    auto fetch_stats = [&](const Place& x) {
        const int i = x.t * QT + (int)threadIdx.x;
        row_ahead = threadIdx.x < (uint32_t)QT && i < qlen;
        if (row_ahead) {
            const float *stats = a.stats + 2 * next_row, *deltas = plan.delta + next_row;
            asm volatile("" : "+s"(stats), "+s"(deltas));  // in scalar registers, without an address of each thread's from tile to tile
            stat_ahead = reinterpret_cast<const f32x2*>(stats)[threadIdx.x];
            delta_ahead = deltas[threadIdx.x];
        }
    };
    SeqBiasAhead ahead = {0u, 0u, 0.f};
    auto is_near = [&](int t) { return t >= near0 && t < near1; };
    auto find = [&](const Place& x) { if (W == 4 && is_near(x.t)) ahead.find(a.buckets, far, j_last - start - x.t * QT - (int)threadIdx.x); };
    auto fetch = [&](const Place& x) { if (W == 4 && is_near(x.t)) ahead.fetch(a.table + (size_t)(kv * plan.group + x.g) * a.nb, a.nb); };

    Place next = behind(now);
    if (s0 < s1) {
        fetch_stats(now);
        issue(now, 0);
        find(now);
        fetch(now);
        if (s0 + 1 < s1) find(next);
    }
    auto step = [&](auto parity, int s) {
        constexpr uint32_t B = decltype(parity)::value;
        const uint32_t qt = base + B * 2u * kTile, gt = qt + kTile, stat = stat_at + B * kStat;
        const bool near = is_near(now.t);
        ends(now.g);
        const float flat = now.t < near0 ? above : below;
        if (near) {
            if constexpr (W == 4) {
                if (threadIdx.x < (uint32_t)(QT + 32 * W - 1)) seq_lds_put(bias_at + B * bias_bytes + 4u * threadIdx.x, ahead.get(a.nb));
            } else {
                for (uint32_t e = threadIdx.x; e < (uint32_t)(QT + 32 * W - 1); e += 64u * W)
                    seq_lds_put(bias_at + B * bias_bytes + 4u * e,
                                seq_bias_at(a.table + (size_t)(kv * plan.group + now.g) * a.nb, a.buckets, a.nb, far, j_last - start - now.t * QT - (int)e));
            }
        }
        if (threadIdx.x < (uint32_t)QT) {
            const bool live = row_ahead && !seq_dead(stat_ahead);
            const float ref = live ? stat_ahead[0] : 0.f, l = live ? stat_ahead[1] - seq_lift<T>() : kDead;
            seq_lds_put(stat + 4u * threadIdx.x, flat - (ref + l));
            seq_lds_put(stat + 4u * (QT + threadIdx.x), ref);
            seq_lds_put(stat + 4u * (2 * QT + threadIdx.x), l);
            seq_lds_put(stat + 4u * (3 * QT + threadIdx.x), live ? -delta_ahead : 0.f);
        }
        // Reference and sum as one number, for the exponent's one fused operation: of 16-bit data, whose own rounding is the larger one while the
        // reference is not
        if (wave == 0) {
            const bool large = __any(threadIdx.x < (uint32_t)QT && row_ahead && fabsf(stat_ahead[0]) > 1024.f && stat_ahead[0] != -__builtin_inff());
            if (lane == 0) seq_lds_put(zero_at + 4u * QT + 4u * B, large ? 1.f : 0.f);
        }
        lds_loads_done();
        __syncthreads();
        const Place after = behind(next);
        if (s + 1 < s1) {
            fetch_stats(next);
            fetch(next);
            if (s + 2 < s1) find(after);
            issue(next, B ^ 1u);
        }
        // places formed anew in each tile: kept, they and others go to scratch, and what comes back from there waits for the loads of the next
        // tile (57 us against 45, 2 x 1023 tokens, 4 heads of keys of 128)
        if constexpr (VLDS) asm volatile("" : "+v"(row_reader.at), "+v"(column_reader.at));
        const int first = now.t * QT;
        bool plain = !__is_same(T, SeqF32) && modest && !near && now.t >= mask1;
        if (plain) plain = __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, seq_lds_f32(zero_at + 4u * QT + 4u * B))) == 0;

        f32x16 p[QS];
#pragma unroll
        for (int k = 0; k < QS; ++k) {
            seq_zero(p[k]);
#pragma unroll
            for (int x = 0; x < NC; ++x) p[k] = seq_dot<T>(row_reader.read(qt, x, k), kf[x], p[k]);
        }
        if (!plain) {
            if (near) {
                uint32_t my_bias = bias_at + B * bias_bytes + 4u * ((uint32_t)(j_last - j) + 4u * hi);
                asm volatile("" : "+v"(my_bias));  // one address and offsets, not 16 addresses kept from tile to tile
#pragma unroll
                for (int k = 0; k < QS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) p[k][r] = fmaf(p[k][r], scale, seq_lds_f32(my_bias + 4u * (32 * k + 8 * (r / 4) + r % 4)));
            } else {
#pragma unroll
                for (int k = 0; k < QS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) p[k][r] = fmaf(p[k][r], scale, flat);
            }
            if (now.t < mask1) {
                const int room = from_row - first - 4 * (int)hi;
#pragma unroll
                for (int k = 0; k < QS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) p[k][r] = 32 * k + 8 * (r / 4) + r % 4 >= room ? p[k][r] : -__builtin_inff();
            }
            // the reference first: it cancels against the score however large a bias made both
#pragma unroll
            for (int k = 0; k < QS; ++k)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t rows = stat + 4u * (QT + 32 * k + 8 * q) + 16u * hi;
                    const f32x4 ref = seq_lds_f32x4(rows), l = seq_lds_f32x4(rows + 4u * QT);
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[k][4 * q + e] = (p[k][4 * q + e] - ref[e]) - l[e];
                }
        }
        const float mul = plain ? scale : 1.f;
        const uint32_t addend = plain ? stat : zero_at;
#pragma unroll
        for (int k = 0; k < QS; ++k) {
            f32x16 ds;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 minus_delta = seq_lds_f32x4(stat + 4u * (3 * QT + 32 * k + 8 * q) + 16u * hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) ds[4 * q + e] = minus_delta[e];
            }
#pragma unroll
            for (int x = 0; x < NC; ++x) {
                if constexpr (VLDS) ds = seq_dot<T>(row_reader.read(gt, x, k), row_reader.read(v_at + 32u * RB * wave, x, 0), ds);
                else ds = seq_dot<T>(row_reader.read(gt, x, k), vf[x], ds);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 add = seq_lds_f32x4(addend + 4u * (32 * k + 8 * q) + 16u * hi);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 4 * q + e;
                    p[k][r] = __builtin_amdgcn_exp2f(fmaf(p[k][r], mul, add[e]));
                    ds[r] *= p[k][r];
                }
            }
            column_reader.accumulate(dv, gt, k, p[k]);
            column_reader.accumulate(dk, qt, k, ds);
        }
        now = next;
        next = after;
    };
    for (int s = s0; s < s1; s += 2) {
        step(std::integral_constant<uint32_t, 0>{}, s);
        if (s + 1 < s1) step(std::integral_constant<uint32_t, 1>{}, s + 1);
    }

    if (j >= a.Lk) return;
    const float down = __builtin_amdgcn_exp2f(-seq_lift<T>());
    const bool lone = seq_lone(a.causal, start, qlen, klen);
    const float fk = lone ? 0.f : a.scale * down;
    const size_t row = (size_t)n * a.Lk + j;
    if (lone) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) dk[b][r] = dv[b][r] != dv[b][r] ? dv[b][r] : 0.f;  // NaN where P is
    }
    if (j >= klen) {  // padding has nothing of a row of NaN either
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            seq_zero(dk[b]);
            seq_zero(dv[b]);
        }
    }
    if (plan.splits > 1) {
        const size_t values = (size_t)a.N * a.Lk * a.KV * D, to = (row * a.KV + kv) * D;
        float* const into = plan.part_kv + (size_t)split * 2 * values + to;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t ch = 32 * b + 8 * q + 4 * hi;
                *reinterpret_cast<f32x4*>(into + ch) = f32x4{dk[b][4 * q], dk[b][4 * q + 1], dk[b][4 * q + 2], dk[b][4 * q + 3]};
                *reinterpret_cast<f32x4*>(into + values + ch) = f32x4{dv[b][4 * q], dv[b][4 * q + 1], dv[b][4 * q + 2], dv[b][4 * q + 3]};
            }
        return;
    }
    const size_t to = (row * a.lddk + (size_t)kv * D) * E;
    char* const dkp = static_cast<char*>(a.dk) + to;
    char* const dvp = static_cast<char*>(a.dv) + to;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t ch = 32 * b + 8 * q + 4 * hi;
            seq_store4<T>(dkp, ch, dk[b][4 * q] * fk, dk[b][4 * q + 1] * fk, dk[b][4 * q + 2] * fk, dk[b][4 * q + 3] * fk);
            seq_store4<T>(dvp, ch, dv[b][4 * q] * down, dv[b][4 * q + 1] * down, dv[b][4 * q + 2] * down, dv[b][4 * q + 3] * down);
        }
}

// Joins the parts of dK and dV: a thread has four channels of a key of one of the two.  Bound by the reads (2 x 1023 tokens, 4 heads of 128:
// 64 MB in 12 us).
template <class T, int D>
__global__ void __launch_bounds__(256) seq_join_keys_kernel(SeqArgs a, BackPlan plan) {
    constexpr int E = SeqSize<T>::value;
    const size_t values = (size_t)a.N * a.Lk * a.KV * D, at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= 2 * values) return;
    const bool is_dv = at >= values;
    const size_t in = is_dv ? at - values : at, row = in / ((size_t)a.KV * D), channel = in - row * ((size_t)a.KV * D);
    const size_t n = row / a.Lk;
    const int j = (int)(row - n * a.Lk);
    int q0, each;
    seq_key_tiles(a.causal, seq_length(a.q_len, n, a.Lq), seq_length(a.k_len, n, a.Lk), seq_start(a.q_start, n), j & -(32 * plan.key_waves),
                  seq_backward_rows(D * E), q0, each);
    const int parts = seq_key_parts(each * plan.group, plan);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < parts; ++s) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(plan.part_kv + (size_t)s * 2 * values + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += x[e];
    }
    const float f = __builtin_amdgcn_exp2f(-seq_lift<T>()) * (is_dv ? 1.f : a.scale);
    char* const to = static_cast<char*>(is_dv ? a.dv : a.dk) + row * a.lddk * E;
    seq_store4<T>(to, (uint32_t)channel, sum[0] * f, sum[1] * f, sum[2] * f, sum[3] * f);
}

template <class Kernel>
hipError_t start(Kernel* kernel, dim3 grid, int block, size_t lds, hipStream_t s, const SeqArgs& a, const BackPlan& plan) {
    if (grid.x == 0) return hipSuccess;  // no queries, or no keys
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(block), lds, s, a, plan);
    return hipGetLastError();
}

template <class T, int D>
hipError_t launch_table(const SeqArgs& a, const BackPlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value;
    const size_t tiles = 4 * (size_t)(RB >= 512 ? 32 : kTableKeys) * RB + kLine * 4, squares = 4 * 33 * 32 * 4 + 8 * 64 * 4;
    hipError_t e = start(&seq_table_kernel<T, D>, dim3((unsigned)(a.H * plan.offsets * plan.chunks)), 256, tiles > squares ? tiles : squares, s, a, plan);
    if (e != hipSuccess) return e;
    e = start(&seq_lines_kernel, dim3(1u + (unsigned)((2 * a.far - 1 + 63) / 64), (unsigned)a.H), 256, 0, s, a, plan);
    if (e != hipSuccess) return e;
    return launch_bucket_sums(plan.lines, nullptr, a.buckets, a.dtable, a.H, a.nb, a.far, 1, s);
}

template <class T, int D, int W, int KT, bool KEYS>
hipError_t launch_rows(const SeqArgs& a, const BackPlan& plan, hipStream_t s) {
    constexpr size_t tiles = 4 * (size_t)KT * D * SeqSize<T>::value * (KEYS ? W : 1), sums = KEYS && W > 1 ? (size_t)W * 32 * 4 * (D + 4) : 0;
    constexpr size_t over_waves = KEYS && W > 1 ? sizeof(float) * 32 * W : 0;
    const size_t bias = 2 * sizeof(float) * plan.row_bias * (KEYS ? W : 1), ahead = tiles + bias + over_waves, lds = ahead > sums ? ahead : sums;
    return a.dtable ? start(&seq_rows_kernel<T, D, W, KT, true, KEYS>, dim3(plan.row_grid), 64 * W, lds, s, a, plan)
                    : start(&seq_rows_kernel<T, D, W, KT, false, KEYS>, dim3(plan.row_grid), 64 * W, lds, s, a, plan);
}
template <class T, int D, int W>
hipError_t launch_keys(const SeqArgs& a, const BackPlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value, KT = seq_backward_rows(RB);
    const size_t tiles = 4 * (size_t)KT * RB + (seq_keys_v_in_lds(RB) ? 32 * W * RB : 0), bias = 2 * sizeof(float) * plan.key_bias;
    return start(&seq_keys_kernel<T, D, W, KT>, dim3(plan.key_grid), 64 * W, tiles + 36 * KT + 16 + bias, s, a, plan);
}
template <class T, int D>
hipError_t launch(const SeqArgs& a, const BackPlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value;
    hipError_t e = plan.keys ? launch_rows<T, D, seq_keys_waves(RB), 32, true>(a, plan, s) : launch_rows<T, D, 4, seq_backward_rows(RB), false>(a, plan, s);
    if (e != hipSuccess) return e;
    if (a.dtable) {
        e = launch_table<T, D>(a, plan, s);
        if (e != hipSuccess) return e;
    }
    e = plan.key_waves == 1 ? launch_keys<T, D, 1>(a, plan, s) : launch_keys<T, D, 4>(a, plan, s);
    if (e != hipSuccess || plan.splits == 1 || a.Lk == 0) return e;
    const size_t threads = (size_t)a.N * a.Lk * a.KV * D / 2, blocks = (threads + 255) / 256;
    hipLaunchKernelGGL((seq_join_keys_kernel<T, D>), dim3((unsigned)blocks), dim3(256), 0, s, a, plan);
    return hipGetLastError();
}
template <class T>
hipError_t launch(const SeqArgs& a, const BackPlan& plan, hipStream_t s) {
    if (a.D == 32) return launch<T, 32>(a, plan, s);
    if (a.D == 64) return launch<T, 64>(a, plan, s);
    return launch<T, 128>(a, plan, s);
}

// Too few blocks of keys for the device: their queries are shared out, in parts of one size, two workgroups a CU, no part smaller than two tiles (four:
// 28 us against 25.5, fp32, 4 x 515 tokens, 3 heads of 32).  Where a block's tiles are known to begin at the diagonal, those near the end
// have fewer parts (as many parts for each block, of different sizes: 62 us against 57, 2 x 1023 tokens, 4 heads of keys of 128).
void share_keys(const SeqArgs& a, BackPlan& p, int size, int key_block, double blocks, bool diagonal) {
    const int cus = cu_count();
    const long long tiles = (a.Lq + size - 1) / size, all = tiles * p.group;
    p.splits = 1;
    p.key_least = all > 1 ? (int)all : 1;
    if (blocks > cus || all < 4) return;
    const double wanted = 2.0 * cus / (double)(a.N * a.KV);  // parts, of the blocks of one head
    auto parts = [&](long long least) {
        if (!diagonal) return (double)p.key_blocks * (double)((all + least - 1) / least);
        double sum = 0;
        for (int b = 0; b < p.key_blocks; ++b) {
            const long long q0 = (long long)b * key_block / size, own = tiles > q0 ? (tiles - q0) * p.group : 0;
            sum += (double)((own + least - 1) / least);
        }
        return sum;
    };
    long long least = (all + 15) / 16;
    if (least < 2) least = 2;
    while (least < all && parts(least) > wanted) least += least / 16 + 1;
    p.key_least = (int)least;
    p.splits = (int)((all + least - 1) / least);
}

bool back_plan(const SeqArgs& a, BackPlan& p) {
    const int cus = cu_count();
    p.group = a.H / a.KV;
    const int RB = a.D * (a.dtype == 0 ? 4 : 2), KT = seq_backward_rows(RB);
    // rows: as in the forward
    p.keys = (double)a.N * a.H * ((a.Lq + 127) / 128) < cus;
    p.waves = p.keys ? seq_keys_waves(RB) : 4;
    p.key_waves = a.Lk <= 32 ? 1 : 4;
    const int block = p.keys ? 32 : 32 * p.waves, key_block = 32 * p.key_waves;
    p.row_blocks = (a.Lq + block - 1) / block;
    p.key_blocks = (a.Lk + key_block - 1) / key_block;
    p.row_waves = (a.Lq + 31) / 32;
    const double rows = (double)a.N * a.H * p.row_blocks, keys = (double)a.N * a.KV * p.key_blocks;
    share_keys(a, p, KT, key_block, keys, a.causal && a.q_start == nullptr);
    // threads of a launch
    if ((rows + 8.0 * p.row_blocks) * 64 * p.waves > 4.0e9 || (keys + 8.0 * p.key_blocks) * p.splits * 64 * p.key_waves > 4.0e9) return false;
    p.row_grid = seq_deal(p.row_deal, a.N, a.H, p.row_blocks, a.causal && p.row_blocks > 1);
    p.key_grid = seq_deal(p.key_deal, a.N, a.KV, (long long)p.key_blocks * p.splits, a.causal && p.key_blocks > 1 && p.splits == 1);
    p.by_splits = make_fastdiv((uint32_t)p.splits);
    p.row_bias = a.table ? (uint32_t)((p.keys ? 32 : KT) + block - 1) : 0u;
    p.key_bias = a.table ? (uint32_t)(KT + key_block - 1) : 0u;

    // offsets of blocks with distances between -far and far, and, where all start at 0, with a pair in them
    const int blocks = (a.Lq + kTableRows - 1) / kTableRows;
    auto down = [](long long x, int y) { return (int)(x >= 0 ? x / y : -((y - 1 - x) / y)); };  // floor
    int low = down(-(long long)a.far - kTableKeys + 1, kTableKeys) + 1, high = down((long long)a.far + kTableRows - 2, kTableKeys);
    if (a.q_start == nullptr) {
        const int most = down((long long)a.Lk - 1, kTableKeys), least = -(((blocks > 0 ? blocks - 1 : 0) * kTableRows + kTableKeys - 1) / kTableKeys);
        high = high < most ? high : most;
        low = low > least ? low : least;
    }
    if (a.causal && high > (kTableRows - 1) / kTableKeys) high = (kTableRows - 1) / kTableKeys;
    p.low_offset = low;
    p.offsets = high >= low ? high - low + 1 : 0;
    if (a.far == 0) p.offsets = 0;  // every distance is at an end
    const long long items = a.N * blocks;
    p.items = (int)items;
    // four workgroups a CU
    long long chunks = 4LL * cus / ((long long)a.H * (p.offsets > 0 ? p.offsets : 1));
    if (chunks > items) chunks = items;
    p.chunks = chunks < 1 ? 1 : (int)chunks;
    p.by_offsets = make_fastdiv((uint32_t)(p.offsets > 0 ? p.offsets : 1));
    p.by_chunks = make_fastdiv((uint32_t)p.chunks);
    p.by_table_blocks = make_fastdiv((uint32_t)(blocks > 0 ? blocks : 1));
    return true;
}

size_t padded(size_t floats) { return (floats * sizeof(float) + 255) & ~(size_t)255; }
size_t padded_ends(const SeqArgs& a, const BackPlan& p) { return padded((size_t)a.H * a.N * p.row_waves * 2); }
size_t padded_lines(const SeqArgs& a) { return padded((size_t)a.H * (2 * (size_t)a.far + 1)); }
// whatever the starts and causality leave of the offsets: as many workgroups as fill the device, or one for every offset
size_t table_bytes(const SeqArgs& a, const BackPlan& p) {
    const size_t every = (size_t)a.H * ((2 * (size_t)a.far + kTableRows + kTableKeys) / kTableKeys + 1), fill = 4 * (size_t)cu_count();
    return padded_ends(a, p) + padded_lines(a) + padded((every > fill ? every : fill) * kLine);
}

}  // namespace

bool seq_backward_fits(const SeqArgs& a) {
    BackPlan p;
    return back_plan(a, p);
}

// workspace: delta, the parts of dK and dV, the sums of dS by distance
size_t seq_backward_workspace(const SeqArgs& a, bool want_dtable) {
    BackPlan p, other;
    SeqArgs b = a;
    b.causal = 1;  // of the two ways to share the keys out the one with more parts
    b.q_start = nullptr;
    if (!back_plan(a, p) || !back_plan(b, other)) return 0;
    size_t bytes = padded((size_t)a.N * a.H * a.Lq);
    const int splits = p.splits > other.splits ? p.splits : other.splits;
    if (splits > 1) bytes += padded((size_t)splits * 2 * a.N * a.Lk * a.KV * a.D);
    if (want_dtable) bytes += table_bytes(a, p);
    return bytes;
}

hipError_t launch_sequence_backward(const SeqArgs& a, void* workspace, hipStream_t s) {
    BackPlan p;
    if (!back_plan(a, p)) return hipErrorInvalidValue;
    char* ws = static_cast<char*>(workspace);
    p.delta = reinterpret_cast<float*>(ws);
    ws += padded((size_t)a.N * a.H * a.Lq);
    p.part_kv = reinterpret_cast<float*>(ws);
    if (p.splits > 1) ws += padded((size_t)p.splits * 2 * a.N * a.Lk * a.KV * a.D);
    p.ends = reinterpret_cast<float*>(ws);
    ws += padded_ends(a, p);
    p.lines = reinterpret_cast<float*>(ws);
    ws += padded_lines(a);
    p.parts = reinterpret_cast<float*>(ws);
    if (a.dtype == 0) return launch<SeqF32>(a, p, s);
    return a.dtype == 1 ? launch<SeqBf16>(a, p, s) : launch<SeqF16>(a, p, s);
}

}  // namespace fwa
