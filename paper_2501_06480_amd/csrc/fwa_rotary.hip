// Rotary positions with several axes: y = x with each pair of a head's channels turned by position * frequency, and the inverse, its adjoint.
#include "fwa_rotary.h"

namespace fwa {
namespace {

struct RotaryPlan {
    FastDiv by_each, by_units, by_period;
    int units, rows;      // of a head; of cosines and sines in LDS
    long long total;
};

// A workgroup has its units one behind the other, whatever rows they belong to: memory is read and written in order, and each thread has its four
// vectors on the way while the workgroup forms the cosines and sines of the rows they touch, each once.  Bound by memory: 2 x 6272 rows of 16 heads
// of 128, bf16, 103 MB in 20.6 us, 5.0 TB/s, as a copy; 64 windows of 49 rows of 3 heads of 32: 3.6 us, the launch and three loads one behind the
// other (axis, position, LDS).
template <class T, int V, int UNITS, int THREADS>
__global__ void __launch_bounds__(THREADS) rotary_kernel(RotaryArgs a, RotaryPlan plan) {
    constexpr int E = SeqSize<T>::value, U = UNITS / THREADS;
    extern __shared__ __attribute__((aligned(16))) f32x2 turns[];
    const uint32_t u0 = blockIdx.x * (uint32_t)UNITS, end = plan.total - u0 < UNITS ? (uint32_t)plan.total : u0 + UNITS;
    const uint32_t row0 = fastdiv(u0, plan.by_each), rows = fastdiv(end - 1u, plan.by_each) - row0 + 1u;
    RotaryVector<T, V> x[U], y[U];
    RotaryUnit at[U];
    uint32_t row[U], head[U], unit[U];
    bool on[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
        const uint32_t u = u0 + (uint32_t)(THREADS * i) + threadIdx.x;
        on[i] = u < end;
        if (!on[i]) continue;
        row[i] = fastdiv(u, plan.by_each);
        const uint32_t rest = u - row[i] * plan.by_each.d;
        head[i] = fastdiv(rest, plan.by_units);
        unit[i] = rest - head[i] * plan.by_units.d;
        at[i] = rotary_unit<V>((int)unit[i], a.pairs, a.d, a.interleaved);
        const char* const from = static_cast<const char*>(a.x) + ((size_t)row[i] * a.ldx + (size_t)head[i] * a.d) * E;
        x[i].load(from + (size_t)at[i].first * E);
        if (at[i].both) y[i].load(from + (size_t)at[i].second * E);
    }
    rotary_turns<THREADS>(turns, rows, a.pairs, a.axes, a.frequencies, a.axis_of, a.inverse, [&](uint32_t r, uint32_t axis) {
        const uint32_t global = row0 + r, place = global - fastdiv(global, plan.by_period) * plan.by_period.d;
        return a.positions[(size_t)place * a.axes + axis];
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < U; ++i) {
        if (!on[i]) continue;
        if (at[i].turned) rotary_apply<T, V>(x[i], y[i], turns + (size_t)(row[i] - row0) * a.pairs, (int)unit[i], a.pairs, a.interleaved);
        char* const to = static_cast<char*>(a.y) + ((size_t)row[i] * a.ldy + (size_t)head[i] * a.d) * E;
        x[i].store(to + (size_t)at[i].first * E);
        if (at[i].both) y[i].store(to + (size_t)at[i].second * E);
    }
}

template <class T, int V, int UNITS, int THREADS>
hipError_t launch(const RotaryArgs& a, RotaryPlan plan, hipStream_t s) {
    plan.rows = rotary_rows((long long)a.heads * plan.units, UNITS);
    const size_t lds = sizeof(f32x2) * (size_t)plan.rows * a.pairs;
    auto* const kernel = &rotary_kernel<T, V, UNITS, THREADS>;
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((plan.total + UNITS - 1) / UNITS)), dim3(THREADS), lds, s, a, plan);
    return hipGetLastError();
}
template <class T, int V>
hipError_t launch(const RotaryArgs& a, const RotaryPlan& plan, hipStream_t s) {
    return rotary_small(plan.total) ? launch<T, V, RotaryShape::kSmall, RotaryShape::kSmall>(a, plan, s) : launch<T, V, RotaryShape::kLarge, 256>(a, plan, s);
}

}  // namespace

bool rotary_fits(long long rows, int heads, int d, int pairs, int dtype) {
    return (double)rows * heads * rotary_units(d, pairs, rotary_vector(dtype, d, pairs)) < 2.0e9;
}

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s) {
    const int V = rotary_vector(a.dtype, a.d, a.pairs);
    RotaryPlan plan;
    plan.units = rotary_units(a.d, a.pairs, V);
    const long long each = (long long)a.heads * plan.units;
    plan.total = a.rows * each;
    plan.by_each = make_fastdiv((uint32_t)each);
    plan.by_units = make_fastdiv((uint32_t)plan.units);
    plan.by_period = make_fastdiv((uint32_t)a.period);
    if (a.dtype == 0) return V == 4 ? launch<SeqF32, 4>(a, plan, s) : launch<SeqF32, 1>(a, plan, s);
    if (a.dtype == 1) return V == 8 ? launch<SeqBf16, 8>(a, plan, s) : V == 4 ? launch<SeqBf16, 4>(a, plan, s) : launch<SeqBf16, 1>(a, plan, s);
    return V == 8 ? launch<SeqF16, 8>(a, plan, s) : V == 4 ? launch<SeqF16, 4>(a, plan, s) : launch<SeqF16, 1>(a, plan, s);
}

}  // namespace fwa
