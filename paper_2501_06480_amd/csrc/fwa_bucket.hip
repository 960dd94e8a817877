// Relative position bias by buckets: pair (i, j) of a 1-D sequence reads column m[far + clamp(j - i - q0, -far, far)] of its head's row
// of the table, q0 the position of the first query.  The gather writes it out for all pairs; the scatter, its adjoint, adds a
// gradient up over the pairs of each bucket: along the diagonals first, where all pairs have one distance, then over the distances
// of a bucket.  Every sum has a fixed order.
#include "fwa_device.h"
#include "fwa_internal.h"

namespace fwa {
namespace {

constexpr int kGatherElements = 8192;  // of the bias per workgroup, in whole rows

// The distances that a workgroup's rows meet are looked up once and kept in LDS; four neighbouring elements of its part of the
// bias, which lies in memory without gaps, are one store.  Bound by the writes: 16 heads of 2048 x 2048 in fp32, 268 MB, 40.6 us (6.6 TB/s; a fill
// reaches 6.9); small calls by the launch, 2.9 us.
template <bool BF16>
__global__ void __launch_bounds__(256)
bucket_gather_kernel(const float* __restrict__ table, const int32_t* __restrict__ buckets, void* __restrict__ bias, int nb, int far, int Lq, FastDiv by_Lk,
                     int q0, int rows, FastDiv by_parts) {
    extern __shared__ float line[];
    const uint32_t h = fastdiv(blockIdx.x, by_parts), part = blockIdx.x - h * by_parts.d;
    const int Lk = (int)by_Lk.d, i0 = (int)part * rows, n = Lq - i0 < rows ? Lq - i0 : rows;
    // distances of the part: from -(i0 + n - 1) - q0 on, Lk + n - 1 of them; those of `line` are cut off at far
    const int lowest = -(i0 + n - 1) - q0, highest = Lk - 1 - i0 - q0;
    const int from = lowest < -far ? -far : (lowest > far ? far : lowest), to = highest > far ? far : (highest < -far ? -far : highest);
    for (int e = (int)threadIdx.x; e <= to - from; e += 256) {
        const uint32_t b = (uint32_t)buckets[far + from + e];
        line[e] = b < (uint32_t)nb ? table[(size_t)h * nb + b] : 0.f;
    }
    __syncthreads();
    // the part starts at an element that four need not divide: stores of four start at the first one that they do
    const size_t first = ((size_t)h * Lq + i0) * Lk;
    const uint32_t count = (uint32_t)n * (uint32_t)Lk, head = (uint32_t)((4u - (first & 3u)) & 3u);
    auto at = [&](uint32_t r, uint32_t j) -> float {
        const int d = (int)j - (i0 + (int)r) - q0;
        return line[(d < from ? from : (d > to ? to : d)) - from];
    };
    auto one = [&](uint32_t e) {
        const uint32_t r = fastdiv(e, by_Lk);
        const float x = at(r, e - r * (uint32_t)Lk);
        if constexpr (BF16) static_cast<uint16_t*>(bias)[first + e] = (uint16_t)pack_bf16(x, 0.f);
        else static_cast<float*>(bias)[first + e] = x;
    };
    if (threadIdx.x < head && threadIdx.x < count) one(threadIdx.x);
    const uint32_t fours = count > head ? (count - head) / 4u : 0u;
    for (uint32_t f = threadIdx.x; f < fours; f += 256) {
        const uint32_t e = head + 4u * f;
        uint32_t r = fastdiv(e, by_Lk), j = e - r * (uint32_t)Lk;
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            x[u] = at(r, j);
            if (++j == (uint32_t)Lk) { j = 0; ++r; }
        }
        if constexpr (BF16) *reinterpret_cast<uint2*>(static_cast<uint16_t*>(bias) + first + e) = uint2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
        else *reinterpret_cast<f32x4*>(static_cast<float*>(bias) + first + e) = f32x4{x[0], x[1], x[2], x[3]};
    }
    const uint32_t tail = head + 4u * fours + threadIdx.x;
    if (tail < count) one(tail);
}

// A workgroup has `rows` rows of a head.  A thread follows one diagonal through them, so that neighbours read neighbours; diagonals at
// or beyond far on either side go into one sum each.  Its result is a line of 2 far + 1 sums by distance, zero where it has no pair.  Bound by the
// reads: 12 heads of 1500 x 2047, 147 MB, 30 us (4.9 TB/s).
template <int ROWS>
__global__ void __launch_bounds__(256)
bucket_diagonals_kernel(const float* __restrict__ dbias, float* __restrict__ parts, int far, int Lq, int Lk, int q0, FastDiv by_parts) {
    const uint32_t h = fastdiv(blockIdx.x, by_parts), part = blockIdx.x - h * by_parts.d;
    const int i0 = (int)part * ROWS, n = Lq - i0 < ROWS ? Lq - i0 : ROWS;
    const float* const src = dbias + ((size_t)h * Lq + i0) * Lk;
    float* const line = parts + (size_t)blockIdx.x * (2 * (size_t)far + 1);
    const int lowest = -(i0 + n - 1) - q0, count = Lk + n - 1;
    float below = 0.f, above = 0.f;
    for (int base = 0; base < count; base += 256) {
        const int e = base + (int)threadIdx.x, d = lowest + e;
        float sum = 0.f;
        // row r of the part meets the diagonal at column e - (n - 1) + r
        const int j = e - (n - 1);
#pragma unroll
        for (int r0 = 0; r0 < ROWS; r0 += 8) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int r = r0 + u;
                x[u] = r < n && j + r >= 0 && j + r < Lk ? src[(size_t)r * Lk + (j + r)] : 0.f;
            }
            sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        if (e < count) {
            if (d <= -far) below += sum;
            else if (d >= far) above += sum;
            else line[far + d] = sum;
        }
    }
    const int highest = lowest + count - 1;
    for (int d = 1 - far + (int)threadIdx.x; d < far; d += 256)
        if (d < lowest || d > highest) line[far + d] = 0.f;
    __shared__ float ends[2][4];
#pragma unroll
    for (int m = 32; m > 0; m /= 2) {
        below += __shfl_xor(below, m, 64);
        above += __shfl_xor(above, m, 64);
    }
    if ((threadIdx.x & 63u) == 0) {
        ends[0][threadIdx.x >> 6] = below;
        ends[1][threadIdx.x >> 6] = above;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        below = (ends[0][0] + ends[0][1]) + (ends[0][2] + ends[0][3]);
        above = (ends[1][0] + ends[1][1]) + (ends[1][2] + ends[1][3]);
        if (far == 0) line[0] = below + above;
        else {
            line[0] = below;
            line[2 * (size_t)far] = above;
        }
    }
}

// Lines of one head [count][width] -> their sum [width]: 16 threads take the lines of a column in turns.  12 heads, 47 lines of 2049: 4.7 us,
// the launch and one way through memory.
__global__ void __launch_bounds__(1024) bucket_lines_kernel(const float* __restrict__ parts, float* __restrict__ lines, int count, int width) {
    __shared__ float sums[16][64];
    const int col = (int)(blockIdx.x * 64 + (threadIdx.x & 63u)), slice = (int)(threadIdx.x >> 6);
    const float* const src = parts + (size_t)blockIdx.y * count * width;
    float sum = 0.f;
    if (col < width) {
        int p = slice;
        for (; p + 48 < count; p += 64) {
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = src[(size_t)(p + 16 * u) * width + col];
            sum += (x[0] + x[1]) + (x[2] + x[3]);
        }
        for (; p < count; p += 16) sum += src[(size_t)p * width + col];
    }
    sums[slice][threadIdx.x & 63u] = sum;
    __syncthreads();
    if (slice == 0 && col < width) {
        float x = 0.f;
#pragma unroll
        for (int u = 0; u < 16; ++u) x += sums[u][threadIdx.x];
        lines[(size_t)blockIdx.y * width + col] = x;
    }
}

// Lines by distance [heads][count][width] -> sums by bucket [heads][nb], a workgroup a head: the lines are added up into LDS, a thread a distance (or
// several threads, each every so many lines, where distances are few), then a wave takes four buckets through all distances.  (A wave a
// bucket straight from memory, its loads behind the comparison with the map: 13.5 us for 12 heads, 64 buckets and 2049 distances, behind 4.8 for
// the lines; as two launches of 4 to 5 us each for few.)
__global__ void __launch_bounds__(1024)
bucket_sums_kernel(const float* __restrict__ lines, const int32_t* __restrict__ buckets, float* __restrict__ dtable, int nb, int count, int width) {
    extern __shared__ float line[];
    const float* const src = lines + (size_t)blockIdx.x * count * width;
    const int slices = width < 1024 ? 1024 / width : 1;
    const int slice = slices > 1 ? (int)threadIdx.x / width : 0, col0 = slices > 1 ? (int)threadIdx.x % width : (int)threadIdx.x;
    if (slice < slices)
        for (int col = col0; col < width; col += 1024) {
            float sum = 0.f;
            int p = slice;
            for (; p + 7 * slices < count; p += 8 * slices) {
                float x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = src[(size_t)(p + u * slices) * width + col];
                sum += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            }
            for (; p < count; p += slices) sum += src[(size_t)p * width + col];
            line[slice * width + col] = sum;
        }
    __syncthreads();
    if (slices > 1) {
        float sum = 0.f;
        if ((int)threadIdx.x < width)
            for (int s = 0; s < slices; ++s) sum += line[s * width + (int)threadIdx.x];
        __syncthreads();
        if ((int)threadIdx.x < width) line[threadIdx.x] = sum;
        __syncthreads();
    }
    for (int b0 = 4 * (int)(threadIdx.x >> 6); b0 < nb; b0 += 64) {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int d = (int)(threadIdx.x & 63u); d < width; d += 64) {
            const int b = buckets[d] - b0;
            const float x = line[d];
#pragma unroll
            for (int u = 0; u < 4; ++u) sum[u] += b == u ? x : 0.f;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
#pragma unroll
            for (int m = 32; m > 0; m /= 2) sum[u] += __shfl_xor(sum[u], m, 64);
            if ((threadIdx.x & 63u) == 0 && b0 + u < nb) dtable[(size_t)blockIdx.x * nb + b0 + u] = sum[u];
        }
    }
}

// Rows per workgroup of the diagonals: 32 keep the lines small beside the gradient; fewer where those would leave CUs without work.
int diagonal_rows(int heads, int Lq) { return (long long)heads * Lq >= 32LL * 2 * cu_count() ? 32 : 8; }
// Lines that a head's one workgroup adds up itself: 16 values a thread at most; more are added up by many workgroups first.
bool few_lines(int far, long long count) { return count * (2LL * far + 1) <= 16384; }

}  // namespace

hipError_t launch_bucket_gather(const float* table, const int32_t* buckets, void* bias, int heads, int nb, int far, int Lq, int Lk, int q_start, bool bf16,
                                hipStream_t s) {
    int rows = Lk >= kGatherElements ? 1 : (kGatherElements / Lk < Lq ? kGatherElements / Lk : Lq);
    while ((long long)heads * ((Lq + rows - 1) / rows) > 0xffffffLL) rows *= 2;  // a launch has fewer than 2^32 threads
    const int parts = (Lq + rows - 1) / rows;
    const long long met = (long long)Lk + rows - 1, all = 2LL * far + 1;
    const size_t lds = (size_t)(met < all ? met : all) * sizeof(float);
    const long long grid = (long long)heads * parts;
    const FastDiv by_Lk = make_fastdiv((uint32_t)Lk), by_parts = make_fastdiv((uint32_t)parts);
    const void* const fn = bf16 ? reinterpret_cast<const void*>(&bucket_gather_kernel<true>) : reinterpret_cast<const void*>(&bucket_gather_kernel<false>);
    const hipError_t e = allow_lds(fn, lds);
    if (e != hipSuccess) return e;
    if (bf16) hipLaunchKernelGGL(bucket_gather_kernel<true>, dim3((unsigned)grid), dim3(256), lds, s, table, buckets, bias, nb, far, Lq, by_Lk, q_start, rows, by_parts);
    else hipLaunchKernelGGL(bucket_gather_kernel<false>, dim3((unsigned)grid), dim3(256), lds, s, table, buckets, bias, nb, far, Lq, by_Lk, q_start, rows, by_parts);
    return hipGetLastError();
}

// [heads][count][2 far + 1] sums by distance -> [heads][nb]; `lines` has room for one line a head where there are more than a few
size_t bucket_lines_bytes(int heads, int far, long long count) {
    return count > 1 && !few_lines(far, count) ? (size_t)heads * (2 * (size_t)far + 1) * sizeof(float) : 0;
}
hipError_t launch_bucket_sums(const float* parts, float* lines, const int32_t* buckets, float* dtable, int heads, int nb, int far, long long count, hipStream_t s) {
    const int width = 2 * far + 1;
    if (count > 1 && !few_lines(far, count)) {
        hipLaunchKernelGGL(bucket_lines_kernel, dim3((unsigned)((width + 63) / 64), (unsigned)heads), dim3(1024), 0, s, parts, lines, (int)count, width);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        parts = lines;
        count = 1;
    }
    const size_t lds = (size_t)(width < 1024 ? 1024 : width) * sizeof(float);
    const hipError_t e = allow_lds(reinterpret_cast<const void*>(&bucket_sums_kernel), lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(bucket_sums_kernel, dim3((unsigned)heads), dim3(1024), lds, s, parts, buckets, dtable, nb, (int)count, width);
    return hipGetLastError();
}

size_t bucket_scatter_workspace(int heads, int far, int Lq) {
    const int rows = diagonal_rows(heads, Lq);
    const long long parts = (Lq + rows - 1) / rows;
    return (size_t)heads * parts * (2 * (size_t)far + 1) * sizeof(float) + bucket_lines_bytes(heads, far, parts);
}

hipError_t launch_bucket_scatter(const float* dbias, const int32_t* buckets, float* dtable, int heads, int nb, int far, int Lq, int Lk, int q_start,
                                 float* workspace, hipStream_t s) {
    const int rows = diagonal_rows(heads, Lq), parts = (Lq + rows - 1) / rows;
    const long long grid = (long long)heads * parts;
    if (grid > 0xffffffLL) return hipErrorInvalidValue;
    const FastDiv by_parts = make_fastdiv((uint32_t)parts);
    if (rows == 32) hipLaunchKernelGGL(bucket_diagonals_kernel<32>, dim3((unsigned)grid), dim3(256), 0, s, dbias, workspace, far, Lq, Lk, q_start, by_parts);
    else hipLaunchKernelGGL(bucket_diagonals_kernel<8>, dim3((unsigned)grid), dim3(256), 0, s, dbias, workspace, far, Lq, Lk, q_start, by_parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_bucket_sums(workspace, workspace + (size_t)grid * (2 * (size_t)far + 1), buckets, dtable, heads, nb, far, parts, s);
}

}  // namespace fwa
