// Attention of whole sequences: O = softmax(scale Q K^T + B) V for any number of queries and keys, with the bias B by buckets of the
// distance between them, and its split form for few rows.
//
// One pass over the keys with a running reference r >= max - 6 and sum of 2^(s - r) per row (s in base-2 units), so scores
// exist for one tile of keys at a time.  A wave has 32 rows of queries; it forms S^T = K Q^T (keys over the registers, a row per lane, so
// a row's maximum and sum are in-lane but for one exchange) and O^T += V^T P^T with the probabilities as they stand.  K and V come in
// tiles through LDS, two of each so that the next are on their way during the products.
#include "fwa_sequence.h"

#include <type_traits>

namespace fwa {
namespace {

// A row's reference moves when a score exceeds it by more than this: weights are at most 2^6 then, and the sums of a row are
// scaled anew a few times instead of at every tile.  Their type's precision is relative; half data reach 2^15.
constexpr float kSlack = 6.f;

// Waves per SIMD that the registers are held to: rows of 128 bytes come to a few registers more than three waves have otherwise (encoder of 4 x 2048
// tokens, 12 heads: 82 us with two, 68 with three).
[[maybe_unused]] constexpr int seq_forward_waves(int row_bytes, bool keys) { return row_bytes == 128 && !keys ? 3 : 1; }

// Two forms.  Rows: the W waves of a workgroup have 32 rows each and share the tiles.  KEYS: all have the same 32 rows and every W-th tile each,
// in buffers of their own without a barrier, and join what they have at the end: W times the parallel work where rows are few, for W
// times the loads of K and V.
// Rows: bound by the latency of a tile, its reads of LDS and the softmax between the two products, on two or three waves a SIMD; the matrix units
// are busy 14 to 29 per cent of the time (4 ragged sequences of up to 2048 tokens, 16 heads of 64, bf16: 71 us, 640 TFLOP/s;
// 4001 causal tokens, 16 heads of 128, half: 109 us in a kernel trace, 97 and 680 TFLOP/s in calls one behind the other).  Tiles of 32 keys, more buffers, scores a tile ahead and workgroups of 64 rows were slower.
// Keys: bound by the reads of the cache (16 sequences of up to 8192 keys, 8 heads of 128: 410 MB in 86 us, 4.8 TB/s) or, for short
// ones, by the launch and the latency of a tile or two (10 us).
template <class T, int D, int W, int KT, bool KEYS>
__global__ void __launch_bounds__(64 * W, seq_forward_waves(D * SeqSize<T>::value, KEYS)) seq_forward_kernel(SeqArgs a, SeqPlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, KS = KT / 32;
    constexpr int ROWS = KEYS ? 32 : 32 * W, TURN = KEYS ? W : 1;  // of a workgroup; from a wave's tile to its next one
    constexpr uint32_t kTile = KT * RB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u, slot = KEYS ? c : 32u * wave + c;
    const uint32_t bias_bytes = 4u * plan.bias_entries;
    const uint32_t base = lds_offset(lds) + (KEYS ? wave * 4u * kTile : 0u);
    const uint32_t bias_at = lds_offset(lds) + (KEYS ? 4u * W * kTile + wave * 2u * bias_bytes : 4u * kTile);

    // workgroup -> sequence, head (or group of heads that share keys), block of rows, split of the keys
    uint32_t sequence, unit, part;
    if (!seq_dealt(plan.deal, blockIdx.x, sequence, unit, part)) return;
    int block = (int)fastdiv(part, plan.by_splits);
    const int split = (int)part - block * (int)plan.by_splits.d;
    const long long n = sequence;
    const int hk = (int)unit;  // head, or head of the keys where the rows of a group are packed
    if (a.causal) block = plan.blocks - 1 - block;             // those with most keys first
    const bool packed = KEYS && plan.packed;
    const int G = plan.group, i0 = block * ROWS;
    const int kv = packed ? hk : hk / G;
    int head = hk, i = i0 + (int)slot, g = 0;
    if (packed) {
        g = (int)slot / a.Lq;
        i = (int)slot - g * a.Lq;
        head = hk * G + g;
    }
    const int span_rows = packed ? a.Lq : (a.Lq - i0 < ROWS ? a.Lq - i0 : ROWS);
    const bool exists = packed ? g < G : i < a.Lq;
    const int qlen = seq_length(a.q_len, n, a.Lq), klen = seq_length(a.k_len, n, a.Lk), start = seq_start(a.q_start, n);
    const int first = start + i0, last = first + span_rows - 1, pos = exists ? start + i : last;
    if (!exists) { head = packed ? hk * G : hk; g = 0; }

    int kend = i0 < qlen ? klen : 0;
    if (a.causal && kend > last + 1) kend = last + 1 > 0 ? last + 1 : 0;
    const int tiles = (kend + KT - 1) / KT, per = (tiles + plan.splits - 1) / plan.splits;
    const int t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

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
    const int mine0 = KEYS ? t0 + (int)wave : t0;
    const size_t skip = (size_t)mine0 * KT * kld;
    u32x4 next_k = seq_source(kp + skip), next_v = seq_source(vp + skip);
    int next_rows = klen - mine0 * KT;
    const uint32_t whole = (KT - 1u) * kld + RB, rest = seq_tile_bytes<RB>(klen % KT, KT, kld);
    auto issue = [&](uint32_t buf) {
        next_k[2] = next_v[2] = next_rows >= KT ? whole : rest;
        load.issue(next_k, base + buf * 2u * kTile);
        load.issue(next_v, base + buf * 2u * kTile + kTile);
        seq_advance(next_k, (uint64_t)(TURN * KT) * kld);
        seq_advance(next_v, (uint64_t)(TURN * KT) * kld);
        next_rows -= TURN * KT;
    };

    const float* const table = a.table ? a.table + (size_t)head * a.nb : nullptr;
    const int far = a.far;
    // tiles whose distances are not all cut off: near0 .. near1 - 1; tiles with a pair that a length or causality shuts out: from mask0 on
    int near0 = 0, near1 = 0, mask0 = klen / KT;
    seq_near_tiles(a.table != nullptr, first, last, far, KT, near0, near1);
    if (a.causal && first < klen) {
        const int to = first + 1 > 0 ? (first + 1) / KT : 0;
        mask0 = to < mask0 ? to : mask0;
    }
    // the bias of a near tile, by distance, for each head of the block; a thread's entry is looked up ahead where each has one
    const uint32_t span = (uint32_t)(KT + span_rows - 1), entries = packed ? span * G : span;
    const uint32_t my_bias = bias_at + 4u * ((uint32_t)g * span + (uint32_t)(last - pos) + 4u * hi);
    const float* const group_table = a.table + (size_t)(packed ? hk * G : hk) * a.nb;
    const uint32_t entry = KEYS ? lane : threadIdx.x, entry_head = packed && entry < entries ? entry / span : 0u;
    const bool one_each = entries <= (KEYS ? 64u : 64u * W);
    const float* const entry_table = KEYS ? group_table + (size_t)entry_head * a.nb : group_table;
    const int entry_distance = (int)(entry - entry_head * span) - last;
    SeqBiasAhead ahead = {0u, 0u, 0.f};
    auto find = [&](int t) { if (one_each && t >= near0 && t < near1) ahead.find(a.buckets, far, t * KT + entry_distance); };
    auto fetch = [&](int t) { if (one_each && t >= near0 && t < near1) ahead.fetch(entry_table, a.nb); };
    find(mine0);

    u32x4 qf[NC];
#pragma unroll
    for (int s = 0; s < NC; ++s) qf[s] = u32x4{0u, 0u, 0u, 0u};
    if (exists && i < qlen) {
        const char* const qp = static_cast<const char*>(a.q) + (((size_t)n * a.Lq + i) * a.ldq + (size_t)head * D) * E + 16u * hi;
#pragma unroll
        for (int s = 0; s < NC; ++s) qf[s] = *reinterpret_cast<const u32x4*>(qp + 32 * s);
        // a negative scale goes into the queries, so that the largest product is the largest score
        if (a.scale < 0.f) {
            constexpr uint32_t kSign = __is_same(T, SeqF32) ? 0x80000000u : 0x80008000u;
#pragma unroll
            for (int s = 0; s < NC; ++s) qf[s] ^= kSign;
        }
    }
    const float below = table ? seq_bias_at(table, a.buckets, a.nb, far, -far) : 0.f, above = table ? seq_bias_at(table, a.buckets, a.nb, far, far) : 0.f;
    fetch(mine0);
    find(mine0 + TURN);
    // A bias that is one value for the tile joins the reference in the exponent's one fused operation; a large one, beside which the score would
    // lose its bits in the sum and not in the difference, is added first, as everywhere else.
    const bool modest = !__any(!(fabsf(below) < 256.f && fabsf(above) < 256.f));
    // Rows of the last tile that no load fills hold zeros, or the finite rows of an earlier tile: their weights are zero, and zero times
    // whatever else LDS may hold need not be.
    if (klen % KT != 0 && t0 < t1) {
        for (uint32_t o = threadIdx.x * 16u; o < (KEYS ? 4u * W : 4u) * kTile; o += 64u * W * 16u) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    if (mine0 < t1) issue(0);

    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) seq_zero(o[b]);
    float m = -__builtin_inff(), l = 0.f;
    const int lim = a.causal && pos + 1 < klen ? pos + 1 : klen;
    const float scale = fabsf(a.scale) * kLog2e;

    auto step = [&](auto parity, int t) {
        const uint32_t B = parity;
        const uint32_t kt = base + B * 2u * kTile, vt = kt + kTile;
        const int j0 = t * KT;
        const bool near = t >= near0 && t < near1;
        if (near) {
            if (one_each) {
                if (entry < entries) seq_lds_put(bias_at + B * bias_bytes + 4u * entry, ahead.get(a.nb));
            } else {
                for (uint32_t e = entry; e < entries; e += KEYS ? 64u : 64u * W) {
                    const uint32_t ge = e / span;
                    seq_lds_put(bias_at + B * bias_bytes + 4u * e, seq_bias_at(group_table + (size_t)ge * a.nb, a.buckets, a.nb, far, j0 - last + (int)(e - ge * span)));
                }
            }
        }
        lds_loads_done();
        if constexpr (!KEYS) __syncthreads();
        fetch(t + TURN);
        find(t + 2 * TURN);
        if (t + TURN < t1) issue(B ^ 1u);

        f32x16 s[KS];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            seq_zero(s[k]);
#pragma unroll
            for (int x = 0; x < NC; ++x) s[k] = seq_dot<T>(row_reader.read(kt, x, k), qf[x], s[k]);
        }
        // exponent of a weight: s mul + add - reference
        const float flat = t < near0 ? below : above;
        const bool plain = modest && !near && t < mask0;
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
                const int room = lim - j0 - 4 * (int)hi;
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[k][r] = 32 * k + 8 * (r / 4) + r % 4 < room ? s[k][r] : -__builtin_inff();
            }
        }
        const float mul = plain ? scale : 1.f, add = plain ? flat : 0.f;
        float top = s[0][0];
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[k][r]);
        top = fmaf(seq_max_halves(top), mul, add);
        // the reference follows the largest score so far
        if (__any(top > m + kSlack)) {
            const float to = top > m + kSlack ? top : m, f = to == m ? 1.f : __builtin_amdgcn_exp2f(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[b][r] *= f;
        }
        const float minus = m == -__builtin_inff() ? add : add - m;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[k][r] = __builtin_amdgcn_exp2f(fmaf(s[k][r], mul, minus));
                l += s[k][r];
            }
            column_reader.accumulate(o, vt, k, s[k]);
        }
    };
    if constexpr (KEYS) {  // few tiles: less code to fetch before fewer additions for addresses
        uint32_t parity = 0;
        for (int t = mine0; t < t1; t += TURN, parity ^= 1u) step(parity, t);
    } else {
        for (int t = mine0; t < t1; t += 2) {
            step(std::integral_constant<uint32_t, 0>{}, t);
            if (t + 1 < t1) step(std::integral_constant<uint32_t, 1>{}, t + 1);
        }
    }

    l = seq_sum_halves(l);
    if constexpr (KEYS && W > 1) {
        // sums of all waves through LDS, rows 4 floats apart from a multiple of the banks; the last wave has them, the others are done
        constexpr uint32_t kRow = 4u * (D + 4);
        const uint32_t all = lds_offset(lds), sums = all + W * 32u * kRow;
        __syncthreads();
        if (hi == 0) *(__attribute__((address_space(3))) f32x2*)(uintptr_t)(sums + 8u * (32u * wave + c)) = f32x2{m, l};
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
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *(__attribute__((address_space(3))) f32x4*)(uintptr_t)(all + kRow * (32u * wave + c) + 4u * (32 * b + 8 * q + 4 * hi)) =
                        f32x4{o[b][4 * q] * mine, o[b][4 * q + 1] * mine, o[b][4 * q + 2] * mine, o[b][4 * q + 3] * mine};
        }
        __syncthreads();
        if (wave != W - 1) return;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[b][r] *= mine;
#pragma unroll
        for (int w = 0; w < W - 1; ++w)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 x = seq_lds_f32x4(all + kRow * (32u * w + c) + 4u * (32 * b + 8 * q + 4 * hi));
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][4 * q + e] += x[e];
                }
        m = top;
        l = total;
    }
    if (!exists) return;
    if (i >= qlen) { m = -__builtin_inff(); l = 0.f; }
    const size_t row = ((size_t)n * a.H + head) * a.Lq + i;
    if (plan.splits > 1) {
        const size_t mine = (size_t)split * plan.rows + row;
        float* const to = plan.part_o + mine * D;
        if (l != 0.f)  // nothing reads a part without weight
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(to + 32 * b + 8 * q + 4 * hi) = f32x4{o[b][4 * q], o[b][4 * q + 1], o[b][4 * q + 2], o[b][4 * q + 3]};
        if (hi == 0) *reinterpret_cast<f32x2*>(plan.part_ml + 2 * mine) = f32x2{m, l};
        return;
    }
    const bool any = l != 0.f;  // NaN too
    const float f = any ? 1.f / l : 0.f;
    char* const to = static_cast<char*>(a.o) + (((size_t)n * a.Lq + i) * a.ldo + (size_t)head * D) * E;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = any ? o[b][4 * q + e] * f : 0.f;
            seq_store4<T>(to, 32 * b + 8 * q + 4 * hi, x[0], x[1], x[2], x[3]);
        }
    if (a.stats && hi == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{any ? m : -__builtin_inff(), any ? log2f(l) : 0.f};
}

// Joins the parts of the split form: a thread has four channels of a row.  512 rows of 128 channels in 2 parts: 4.7 us, mostly the launch.
template <class T, int D>
__global__ void __launch_bounds__(256) seq_join_kernel(SeqArgs a, SeqPlan plan) {
    constexpr int E = SeqSize<T>::value, kThreads = D / 4;
    const size_t row = (size_t)blockIdx.x * (256 / kThreads) + threadIdx.x / kThreads;
    const int channel = 4 * (int)(threadIdx.x % kThreads);
    if (row >= plan.rows) return;
    float top = -__builtin_inff();
    for (int s = 0; s < plan.splits; ++s) top = fmaxf(top, plan.part_ml[2 * ((size_t)s * plan.rows + row)]);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < plan.splits; ++s) {
        const size_t part = (size_t)s * plan.rows + row;
        const f32x2 ml = *reinterpret_cast<const f32x2*>(plan.part_ml + 2 * part);
        if (ml[1] == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(ml[0] - top);
        const f32x4 x = *reinterpret_cast<const f32x4*>(plan.part_o + part * D + channel);
        l += f * ml[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f * x[e];
    }
    const size_t head_row = row / a.Lq, n = head_row / a.H;
    const size_t i = row - head_row * a.Lq, head = head_row - n * a.H;
    const bool any = l != 0.f;
    const float f = any ? 1.f / l : 0.f;
    char* const to = static_cast<char*>(a.o) + ((n * a.Lq + i) * a.ldo + head * D) * E;
    seq_store4<T>(to, channel, o[0] * f, o[1] * f, o[2] * f, o[3] * f);
    if (a.stats && channel == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{any ? top : -__builtin_inff(), any ? log2f(l) : 0.f};
}

template <class T, int D, int W, int KT, bool KEYS>
hipError_t launch(const SeqArgs& a, SeqPlan& plan, hipStream_t s) {
    constexpr size_t tiles = 4 * (size_t)KT * D * SeqSize<T>::value * (KEYS ? W : 1), sums = KEYS && W > 1 ? (size_t)W * 32 * (4 * (D + 4) + 8) : 0;
    const size_t bias = 2 * sizeof(float) * plan.bias_entries * (KEYS ? W : 1), lds = tiles + bias > sums ? tiles + bias : sums;
    auto* const kernel = &seq_forward_kernel<T, D, W, KT, KEYS>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(plan.grid), dim3(64 * W), lds, s, a, plan);
    e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    const size_t per = 256 / (D / 4), blocks = (plan.rows + per - 1) / per;
    hipLaunchKernelGGL((seq_join_kernel<T, D>), dim3((unsigned)blocks), dim3(256), 0, s, a, plan);
    return hipGetLastError();
}
template <class T, int D>
hipError_t launch(const SeqArgs& a, SeqPlan& plan, hipStream_t s) {
    constexpr int RB = D * SeqSize<T>::value;
    return plan.keys ? launch<T, D, seq_keys_waves(RB), seq_forward_keys(RB, true), true>(a, plan, s) : launch<T, D, 4, seq_forward_keys(RB, false), false>(a, plan, s);
}
template <class T>
hipError_t launch(const SeqArgs& a, SeqPlan& plan, hipStream_t s) {
    if (a.D == 32) return launch<T, 32>(a, plan, s);
    if (a.D == 64) return launch<T, 64>(a, plan, s);
    return launch<T, 128>(a, plan, s);
}

}  // namespace

bool seq_forward_plan(const SeqArgs& a, SeqPlan& p) {
    const int size = a.dtype == 0 ? 4 : 2, cus = cu_count();
    p.group = a.H / a.KV;
    p.packed = (long long)p.group * a.Lq <= 32;
    const int RB = a.D * size;
    const double heads = (double)a.N * (p.packed ? a.KV : a.H);
    // Less than a workgroup of 128 rows for each CU: the waves share out the keys instead, and where that still leaves CUs without work, workgroups
    // do too, no more of them than leaves each wave four tiles: a tile costs about 1 us where little runs, joining parts in memory 4.  (One for each CU, causal, 2 x 1023 tokens, 16 heads of 128: 33 us with rows, 46 with
    // keys, which load each tile four times as often; 37 with workgroups of 64 rows.)
    p.keys = p.packed || heads * ((a.Lq + 127) / 128) < cus;
    p.waves = p.keys ? seq_keys_waves(RB) : 4;
    const int KT = seq_forward_keys(RB, p.keys), rows = p.keys ? 32 : 128;
    p.blocks = p.packed ? 1 : (a.Lq + rows - 1) / rows;
    const double base = heads * p.blocks;
    long long splits = 1;
    if (p.keys) {
        const int tiles = (a.Lk + KT - 1) / KT;
        splits = (long long)(2.0 * cus / (base > 1 ? base : 1));
        if (splits > tiles / (4 * p.waves)) splits = tiles / (4 * p.waves);
        if (splits > 64) splits = 64;
    }
    p.splits = splits < 1 ? 1 : (int)splits;
    if ((base * p.splits + 8.0 * p.blocks * p.splits) * 64.0 * p.waves > 4.0e9) return false;  // threads of a launch
    p.grid = seq_deal(p.deal, a.N, p.packed ? a.KV : a.H, (long long)p.blocks * p.splits, a.causal && p.blocks > 1);
    p.by_splits = make_fastdiv((uint32_t)p.splits);
    p.rows = (size_t)a.N * a.H * a.Lq;
    p.bias_entries = a.table == nullptr ? 0 : p.packed ? (uint32_t)(p.group * (KT + a.Lq - 1)) : (uint32_t)(KT + rows - 1);
    return true;
}

bool seq_forward_fits(const SeqArgs& a) {
    SeqPlan p;
    return seq_forward_plan(a, p);
}

size_t seq_forward_workspace(const SeqArgs& a) {
    SeqPlan p;
    if (!seq_forward_plan(a, p) || p.splits == 1) return 0;
    return (size_t)p.splits * p.rows * (a.D + 2) * sizeof(float);
}

hipError_t launch_sequence_forward(const SeqArgs& a, void* workspace, hipStream_t s) {
    SeqPlan p;
    if (!seq_forward_plan(a, p)) return hipErrorInvalidValue;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o ? p.part_o + (size_t)p.splits * p.rows * a.D : nullptr;
    if (a.dtype == 0) return launch<SeqF32>(a, p, s);
    return a.dtype == 1 ? launch<SeqBf16>(a, p, s) : launch<SeqF16>(a, p, s);
}

}  // namespace fwa
