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

template <class T, int D, int W, int KT>
__global__ void __launch_bounds__(64 * W) seq_forward_kernel(SeqArgs a, SeqPlan plan) {
    constexpr int E = SeqSize<T>::value, RB = D * E, NC = RB / 32, NB = D / 32, KS = KT / 32;
    constexpr uint32_t kTile = KT * RB;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const uint32_t base = lds_offset(lds), bias_at = base + 4u * kTile;
    const uint32_t lane = threadIdx.x & 63u, wave = W == 1 ? 0u : (uint32_t)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t hi = lane >> 5, c = lane & 31u, slot = 32u * wave + c;

    // workgroup -> sequence, head (or group of heads that share keys), block of rows, split of the keys
    uint32_t unit, part;
    if (!seq_dealt(plan.deal, blockIdx.x, unit, part)) return;
    int block = (int)fastdiv(part, plan.by_splits);
    const int split = (int)part - block * (int)plan.by_splits.d;
    const long long n = fastdiv(unit, plan.by_heads);
    const int hk = (int)(unit - (uint32_t)n * plan.by_heads.d);  // head, or head of the keys where the rows of a group are packed
    if (a.causal) block = plan.blocks - 1 - block;             // those with most keys first
    const int G = plan.group, i0 = block * 32 * W;
    const int kv = plan.packed ? hk : hk / G;
    int head = hk, i = i0 + (int)slot, g = 0;
    if (plan.packed) {
        g = (int)slot / a.Lq;
        i = (int)slot - g * a.Lq;
        head = hk * G + g;
    }
    const int span_rows = plan.packed ? a.Lq : (a.Lq - i0 < 32 * W ? a.Lq - i0 : 32 * W);
    const bool exists = plan.packed ? g < G : i < a.Lq;
    const int qlen = seq_length(a.q_len, n, a.Lq), klen = seq_length(a.k_len, n, a.Lk), start = seq_start(a.q_start, n);
    const int first = start + i0, last = first + span_rows - 1, pos = exists ? start + i : last;
    if (!exists) { head = plan.packed ? hk * G : hk; g = 0; }

    int kend = i0 < qlen ? klen : 0;
    if (a.causal && kend > last + 1) kend = last + 1 > 0 ? last + 1 : 0;
    const int tiles = (kend + KT - 1) / KT, per = (tiles + plan.splits - 1) / plan.splits;
    const int t0 = split * per, t1 = t0 + per < tiles ? t0 + per : tiles;

    const char* const kp = static_cast<const char*>(a.k) + ((size_t)n * a.Lk * a.ldk + (size_t)kv * D) * E;
    const char* const vp = static_cast<const char*>(a.v) + ((size_t)n * a.Lk * a.ldk + (size_t)kv * D) * E;
    const uint32_t kld = (uint32_t)(a.ldk * E);

    SeqLoader<RB, KT, W> load;
    load.init(wave, lane, kld);
    SeqRowReader<RB> row_reader;
    row_reader.init(hi, c);
    SeqColumnReader<T, D> column_reader;
    column_reader.init(hi, c);
    // addresses of the next tile to ask for, and the rows from there on
    const size_t skip = (size_t)t0 * KT * kld;
    uintptr_t next_k = reinterpret_cast<uintptr_t>(kp) + skip, next_v = reinterpret_cast<uintptr_t>(vp) + skip;
    int next_rows = klen - t0 * KT;
    auto issue = [&](uint32_t buf) {
        const uint32_t bytes = seq_tile_bytes<RB>(next_rows, KT, kld);
        load.issue(next_k, bytes, base + buf * 2u * kTile);
        load.issue(next_v, bytes, base + buf * 2u * kTile + kTile);
        next_k += KT * kld;
        next_v += KT * kld;
        next_rows -= KT;
    };

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
    // Rows of the last tile that no load fills hold zeros, or the finite rows of an earlier tile: their weights are zero, and zero times
    // whatever else LDS may hold need not be.
    if (klen % KT != 0 && t0 < t1) {
        for (uint32_t o = threadIdx.x * 16u; o < 4u * kTile; o += 64u * W * 16u) *reinterpret_cast<u32x4*>(lds + o) = u32x4{0u, 0u, 0u, 0u};
        __syncthreads();
    }
    if (t0 < t1) issue(0);

    const float* const table = a.table ? a.table + (size_t)head * a.nb : nullptr;
    const int far = a.far;
    const float below = table ? seq_bias_at(table, a.buckets, a.nb, far, -far) : 0.f, above = table ? seq_bias_at(table, a.buckets, a.nb, far, far) : 0.f;
    // A bias that is one value for the tile joins the reference in the exponent's one fused operation; a large one, beside which the score would
    // lose its bits in the sum and not in the difference, is added first, as everywhere else.
    const bool modest = !__any(!(fabsf(below) < 256.f && fabsf(above) < 256.f));
    // tiles whose distances are not all cut off: near0 .. near1 - 1; tiles with a pair that a length or causality shuts out: from mask0 on
    int near0 = 0, near1 = 0, mask0 = klen / KT;
    seq_near_tiles(a.table != nullptr, first, last, far, KT, near0, near1);
    if (a.causal && first < klen) {
        const int to = first + 1 > 0 ? (first + 1) / KT : 0;
        mask0 = to < mask0 ? to : mask0;
    }
    const uint32_t span = (uint32_t)(KT + span_rows - 1), entries = plan.packed ? span * G : span, bias_bytes = 4u * plan.bias_entries;
    const uint32_t my_bias = bias_at + 4u * ((uint32_t)g * span + (uint32_t)(last - pos) + 4u * hi);
    const float* const group_table = a.table + (size_t)(plan.packed ? hk * G : hk) * a.nb;

    f32x16 o[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) seq_zero(o[b]);
    float m = -__builtin_inff(), l = 0.f;
    const int lim = a.causal && pos + 1 < klen ? pos + 1 : klen;
    const float scale = fabsf(a.scale) * kLog2e;

    SeqBiasAhead ahead = {0u, 0u, 0.f};
    if constexpr (W == 4) {
        if (t0 >= near0 && t0 < near1) {
            ahead.find(a.buckets, far, t0 * KT - last + (int)threadIdx.x);
            ahead.fetch(group_table, a.nb);
        }
        if (t0 + 1 >= near0 && t0 + 1 < near1) ahead.find(a.buckets, far, (t0 + 1) * KT - last + (int)threadIdx.x);
    }
    auto step = [&](auto parity, int t) {
        constexpr uint32_t B = decltype(parity)::value;
        const uint32_t kt = base + B * 2u * kTile, vt = kt + kTile;
        const int j0 = t * KT;
        const bool near = t >= near0 && t < near1;
        if (near) {
            if constexpr (W == 4) {
                if (threadIdx.x < entries) seq_lds_put(bias_at + B * bias_bytes + 4u * threadIdx.x, ahead.get(a.nb));
            } else {
                for (uint32_t e = threadIdx.x; e < entries; e += 64u * W) {
                    const uint32_t ge = plan.packed ? e / span : 0u;
                    seq_lds_put(bias_at + B * bias_bytes + 4u * e,
                                seq_bias_at(group_table + (size_t)ge * a.nb, a.buckets, a.nb, far, j0 - last + (int)(e - ge * span)));
                }
            }
        }
        lds_loads_done();
        __syncthreads();
        if constexpr (W == 4) {
            if (t + 1 >= near0 && t + 1 < near1) ahead.fetch(group_table, a.nb);
            if (t + 2 >= near0 && t + 2 < near1) ahead.find(a.buckets, far, j0 + 2 * KT - last + (int)threadIdx.x);
        }
        if (t + 1 < t1) issue(B ^ 1u);

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
    for (int t = t0; t < t1; t += 2) {
        step(std::integral_constant<uint32_t, 0>{}, t);
        if (t + 1 < t1) step(std::integral_constant<uint32_t, 1>{}, t + 1);
    }

    l = seq_sum_halves(l);
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

// Joins the parts of the split form: a thread has four channels of a row.
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

template <class T, int D, int W>
hipError_t launch(const SeqArgs& a, SeqPlan& plan, hipStream_t s) {
    constexpr int KT = seq_forward_keys(D * SeqSize<T>::value, W);
    const size_t lds = 4 * (size_t)KT * D * SeqSize<T>::value + 2 * sizeof(float) * plan.bias_entries;
    auto* const kernel = &seq_forward_kernel<T, D, W, KT>;
    hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(plan.grid), dim3(64 * W), lds, s, a, plan);
    e = hipGetLastError();
    if (e != hipSuccess || plan.splits == 1) return e;
    const size_t per = 256 / (D / 4), blocks = (plan.rows + per - 1) / per;
    hipLaunchKernelGGL((seq_join_kernel<T, D>), dim3((unsigned)blocks), dim3(256), 0, s, a, plan);
    return hipGetLastError();
}
template <class T>
hipError_t launch(const SeqArgs& a, SeqPlan& plan, hipStream_t s) {
    if (plan.waves == 1) {
        if (a.D == 32) return launch<T, 32, 1>(a, plan, s);
        if (a.D == 64) return launch<T, 64, 1>(a, plan, s);
        return launch<T, 128, 1>(a, plan, s);
    }
    if (a.D == 32) return launch<T, 32, 4>(a, plan, s);
    if (a.D == 64) return launch<T, 64, 4>(a, plan, s);
    return launch<T, 128, 4>(a, plan, s);
}

}  // namespace

bool seq_forward_plan(const SeqArgs& a, SeqPlan& p) {
    const int size = a.dtype == 0 ? 4 : 2, cus = cu_count();
    p.group = a.H / a.KV;
    p.packed = (long long)p.group * a.Lq <= 32;
    p.waves = p.packed || a.Lq <= 32 ? 1 : 4;
    const int KT = seq_forward_keys(a.D * size, p.waves);
    p.blocks = p.packed ? 1 : (a.Lq + 32 * p.waves - 1) / (32 * p.waves);
    const double base = (double)a.N * (p.packed ? a.KV : a.H) * p.blocks;
    // Workgroups that fill the device: a wave of its own each (four to five on a CU by LDS), or four waves each (two to four).
    // Fewer than that share out the keys, no more than leaves each two tiles.
    const double want = (p.waves == 1 ? 4.0 : 2.0) * cus;
    const int tiles = (a.Lk + KT - 1) / KT;
    long long splits = (long long)(want / (base > 1 ? base : 1));
    if (splits > tiles / 2) splits = tiles / 2;
    if (splits > 64) splits = 64;
    p.splits = splits < 1 ? 1 : (int)splits;
    if ((base * p.splits + 8.0 * p.blocks * p.splits) * 64.0 * p.waves > 4.0e9) return false;  // threads of a launch
    p.grid = seq_deal(p.deal, (long long)a.N * (p.packed ? a.KV : a.H), (long long)p.blocks * p.splits, a.causal && p.blocks > 1);
    p.by_splits = make_fastdiv((uint32_t)p.splits);
    p.by_heads = make_fastdiv((uint32_t)(p.packed ? a.KV : a.H));
    p.rows = (size_t)a.N * a.H * a.Lq;
    p.bias_entries = a.table == nullptr ? 0 : p.packed ? (uint32_t)(p.group * (KT + a.Lq - 1)) : (uint32_t)(KT + 32 * p.waves - 1);
    return true;
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
