// Append of new tokens to a paged cache: each token's keys, rotated by its position, and values go to their rows of the pages, and its queries are rotated
// besides.  Tokens of several sequences stand one behind the other; a token's sequence is found from the offsets.
#include "fwa_internal.h"
#include "fwa_page_index.h"
#include "fwa_rotary.h"

namespace fwa {
namespace {

struct AppendPlan {
    FastDiv by_each, by_units, by_page;
    int heads, units, rows;  // heads of queries, keys and values together; units of a head; rows in LDS
    int sample, samples;     // one of so many offsets is looked at first, and how many there are of these
    long long total;
};

// What a workgroup knows of a row that its units touch.
struct AppendRow {
    int place;        // in the sequence; the default position.  -1: a row of no sequence
    int sequence;     // and then, in its place, the entry of the table
};
constexpr uint32_t kNowhere = 0xffffffffu;

// Units as in the rotary kernel, a token's heads of queries, keys and values one behind the other, with their vectors on the way while the places are
// looked up: sequence and length in LDS (or, of more sequences than threads, from a sample of the offsets in LDS on), then the page, beside the
// cosines. Bound by memory for long calls (4001 tokens of 24 heads of 128, half: kernel 11.8 us for 49 MB, 4.2 TB/s, fp32 19.7 for 98, 5.0 TB/s; 6439 of 36
// of 64, bf16: 13.0 for 59), by its chain of loads for short ones (16 tokens: 3.9 us).
template <class T, int V, int UNITS, int THREADS>
__global__ void __launch_bounds__(THREADS) page_append_kernel(PageArgs a, AppendPlan plan) {
    constexpr int E = SeqSize<T>::value, U = UNITS / THREADS;
    extern __shared__ __attribute__((aligned(16))) f32x2 turns[];
    __shared__ int samples[THREADS + 1], lengths[THREADS];
    AppendRow* const known = reinterpret_cast<AppendRow*>(turns + (size_t)plan.rows * a.pairs);
    const uint32_t u0 = blockIdx.x * (uint32_t)UNITS, end = plan.total - u0 < UNITS ? (uint32_t)plan.total : u0 + UNITS;
    const uint32_t row0 = fastdiv(u0, plan.by_each), rows = fastdiv(end - 1u, plan.by_each) - row0 + 1u;
    if ((int)threadIdx.x < plan.samples) {
        const uint32_t n = threadIdx.x * (uint32_t)plan.sample;
        samples[threadIdx.x] = a.offsets[n];
        if (plan.sample == 1) {
            lengths[threadIdx.x] = a.lengths[n];
            if ((int)threadIdx.x == plan.samples - 1) samples[plan.samples] = a.offsets[n + 1u];
        }
    }
    RotaryVector<T, V> x[U], y[U];
    RotaryUnit at[U];
    uint32_t row[U], head[U], unit[U];
    bool on[U], turned[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t u = u0 + (uint32_t)(THREADS * i) + threadIdx.x;
        on[i] = u < end;
        if (!on[i]) continue;
        row[i] = fastdiv(u, plan.by_each);
        const uint32_t rest = u - row[i] * plan.by_each.d;
        head[i] = fastdiv(rest, plan.by_units);
        unit[i] = rest - head[i] * plan.by_units.d;
        // values are not turned, and their channels go by the same units
        at[i] = rotary_unit<V>((int)unit[i], a.pairs, a.D, a.interleaved);
        turned[i] = at[i].turned && head[i] < (uint32_t)(a.H + a.KV);
        const char* from;
        if (head[i] < (uint32_t)a.H) from = static_cast<const char*>(a.q) + ((size_t)row[i] * a.ldq + (size_t)head[i] * a.D) * E;
        else if (head[i] < (uint32_t)(a.H + a.KV)) from = static_cast<const char*>(a.new_k) + ((size_t)row[i] * a.ldk + (size_t)(head[i] - a.H) * a.D) * E;
        else from = static_cast<const char*>(a.new_v) + ((size_t)row[i] * a.ldv + (size_t)(head[i] - a.H - a.KV) * a.D) * E;
        x[i].load(from + (size_t)at[i].first * E);
        if (at[i].both) y[i].load(from + (size_t)at[i].second * E);
    }
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < rows; r += THREADS) {
        const int t = (int)(row0 + r);
        // the last sequence that begins at or in front of t: of the samples, then of the offsets behind it
        int lo = 0, hi = plan.samples;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (samples[mid] <= t) lo = mid;
            else hi = mid;
        }
        int n = lo * plan.sample, begin, finish, length;
        if (plan.sample == 1) {
            begin = samples[n];
            finish = samples[n + 1];
            length = lengths[n];
        } else {
            int to = n + plan.sample < a.N ? n + plan.sample : a.N;
            while (to - n > 1) {
                const int mid = (n + to) / 2;
                if (a.offsets[mid] <= t) n = mid;
                else to = mid;
            }
            begin = a.offsets[n];
            finish = a.offsets[n + 1];
            length = a.lengths[n];
        }
        known[r] = AppendRow{begin <= t && t < finish ? page_length(length) + (t - page_offset(begin, a.rows)) : -1, n};
    }
    __syncthreads();
    // the page of a row is on its way while the cosines are formed
    uint32_t page = kNowhere;
    const bool looks = threadIdx.x < rows;
    auto look = [&](uint32_t r) {
        const AppendRow k = known[r];
        const uint32_t index = k.place < 0 ? ~0u : fastdiv((uint32_t)k.place, plan.by_page);
        return index < (uint32_t)a.width ? (uint32_t)a.table[(size_t)k.sequence * a.width + index] : kNowhere;
    };
    if (looks) page = look(threadIdx.x);
    rotary_turns<THREADS>(turns, rows, a.pairs, a.axes, a.frequencies, a.axis_of, false, [&](uint32_t r, uint32_t axis) {
        return a.positions ? a.positions[(size_t)(row0 + r) * a.axes + axis] : known[r].place;
    });
    __syncthreads();
    if (looks) known[threadIdx.x].sequence = (int)page;
    for (uint32_t r = threadIdx.x + THREADS; r < rows; r += THREADS) known[r].sequence = (int)look(r);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (!on[i]) continue;
        const AppendRow k = known[row[i] - row0];
        if (k.place < 0) continue;
        if (turned[i]) rotary_apply<T, V>(x[i], y[i], turns + (size_t)(row[i] - row0) * a.pairs, (int)unit[i], a.pairs, a.interleaved);
        char* to;
        if (head[i] < (uint32_t)a.H) {
            to = static_cast<char*>(a.o) + ((size_t)row[i] * a.ldo + (size_t)head[i] * a.D) * E;
        } else {
            if (!page_exists(k.sequence, a.pages)) continue;
            const bool key = head[i] < (uint32_t)(a.H + a.KV);
            const uint32_t h = head[i] - a.H - (key ? 0 : a.KV), slot = (uint32_t)k.place - fastdiv((uint32_t)k.place, plan.by_page) * plan.by_page.d;
            to = static_cast<char*>(key ? a.k : a.v) + (size_t)h * a.head_stride * E +
                 page_place((uint32_t)k.sequence, slot, (uint32_t)(a.page_stride * E), (uint32_t)(a.token_stride * E));
        }
        x[i].store(to + (size_t)at[i].first * E);
        if (at[i].both) y[i].store(to + (size_t)at[i].second * E);
    }
}

template <class T, int V, int UNITS, int THREADS>
hipError_t launch(const PageArgs& a, AppendPlan plan, hipStream_t s) {
    plan.rows = rotary_rows((long long)plan.heads * plan.units, UNITS);
    plan.sample = (a.N + THREADS - 1) / THREADS;
    plan.samples = (a.N + plan.sample - 1) / plan.sample;
    const size_t lds = (sizeof(f32x2) * a.pairs + sizeof(AppendRow)) * (size_t)plan.rows;
    auto* const kernel = &page_append_kernel<T, V, UNITS, THREADS>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((plan.total + UNITS - 1) / UNITS)), dim3(THREADS), lds, s, a, plan);
    return hipGetLastError();
}
template <class T, int V>
hipError_t launch(const PageArgs& a, const AppendPlan& plan, hipStream_t s) {
    // Four units a thread where that leaves two workgroups for each CU: half as many searches (6439 tokens of 36 heads of 64, 0.9 million units,
    // bf16: calls one behind the other 15.0 us with two, 13.1 with four; a rotation of 0.2 million units, 7.6 and 8.1).
    if (rotary_small(plan.total)) return launch<T, V, RotaryShape::kSmall, RotaryShape::kSmall>(a, plan, s);
    return plan.total <= 512 * 1024 ? launch<T, V, RotaryShape::kLarge, 256>(a, plan, s) : launch<T, V, 2 * RotaryShape::kLarge, 256>(a, plan, s);
}

}  // namespace

bool page_append_fits(const PageArgs& a) {
    return (double)a.rows * (a.H + 2 * a.KV) * rotary_units(a.D, a.pairs, rotary_vector(a.dtype, a.D, a.pairs)) < 2.0e9;
}

hipError_t launch_page_append(const PageArgs& a, hipStream_t s) {
    const int V = rotary_vector(a.dtype, a.D, a.pairs);
    AppendPlan plan;
    plan.heads = a.H + 2 * a.KV;
    plan.units = rotary_units(a.D, a.pairs, V);
    const long long each = (long long)plan.heads * plan.units;
    plan.total = a.rows * each;
    plan.by_each = make_fastdiv((uint32_t)each);
    plan.by_units = make_fastdiv((uint32_t)plan.units);
    plan.by_page = make_fastdiv((uint32_t)a.page_size);
    if (a.dtype == 0) return V == 4 ? launch<SeqF32, 4>(a, plan, s) : launch<SeqF32, 1>(a, plan, s);
    if (a.dtype == 1) return V == 8 ? launch<SeqBf16, 8>(a, plan, s) : V == 4 ? launch<SeqBf16, 4>(a, plan, s) : launch<SeqBf16, 1>(a, plan, s);
    return V == 8 ? launch<SeqF16, 8>(a, plan, s) : V == 4 ? launch<SeqF16, 4>(a, plan, s) : launch<SeqF16, 1>(a, plan, s);
}

}  // namespace fwa
