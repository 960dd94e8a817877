// Internal declarations shared by the HIP translation units of libfwa.
// Nothing here is part of the public ABI (see include/fwa.h for that).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <atomic>

namespace fwa {

constexpr int kHeadDim = 32;   // head width of every path but the wide-head kernels
constexpr int kMaxWideL = 64;  // wide-head kernels (head widths 64, 128, 256): the tile of one window
constexpr int kMaxL = 256;     // 16 key blocks of 16 rows
constexpr int kMaxBackwardL = 64;  // backward: largest window whose score tile stays on chip (and that has dBias)
constexpr int kWavesPerBlock = 4;

struct FwdArgs {
    const void* q;
    const void* k;
    const void* v;
    void* o;
    const void* bias;    // [heads, L, L], fp32 or (bias_bf16) bf16, or nullptr
    int bias_bf16;
    const float* mask;   // [nW, L, L] or nullptr
    const int32_t* labels;  // [nW, L] region labels standing for the mask, or nullptr; never together with mask
    float mask_value;       // what labels that differ add to a score
    long long N;
    int L;
    int C;
    int heads;
    int nW;
    float scale;
    int ldq;             // elements between consecutive token rows of q, k, v (C when contiguous)
    int ldo;             // the same for o
    int f16;             // the 16-bit data are IEEE half, not bf16 (wide-head kernels only)
};

struct BwdArgs {
    const void* q;
    const void* k;
    const void* v;
    const void* d_o;
    void* dq;
    void* dk;
    void* dv;
    float* dbias;        // [heads, L, L] or nullptr
    float* partial;      // workspace for per-slot dS sums, or nullptr
    const void* bias;    // as in FwdArgs
    int bias_bf16;
    const float* mask;
    const int32_t* labels;  // as in FwdArgs
    float mask_value;
    long long N;
    int L;
    int C;
    int heads;
    int nW;
    float scale;
    int slots;           // number of partial-sum slots per head in `partial`
    int per_window;      // cooperative kernel for L <= 64: the mask is formed or fetched per window (a period that
                         // no slot count is a multiple of); only the bias stays in registers
    int ldq;             // elements between consecutive token rows of q, k, v (C when contiguous)
    int ldg;             // the same for d_o
    int ldd;             // the same for dq, dk, dv
    int f16;             // the 16-bit data are IEEE half, not bf16 (wide-head kernels only)
};

// Whether the scores get a mask, in either form, and its period over the windows (1 without one).
template <class Args>
inline bool has_mask(const Args& a) { return a.mask != nullptr || a.labels != nullptr; }
template <class Args>
inline int mask_period(const Args& a) { return has_mask(a) ? a.nW : 1; }

// Compute units of the current device, asked from the runtime once per device (256 on MI355X; the
// same figure stands in when no device answers, e.g. a workspace-size query on a machine without a
// GPU).  Workgroup counts of the persistent kernels and dBias slot counts are derived from it.
int cu_count();

// Lifts the 64 KB limit on dynamic LDS for kernel `fn` on the current device (to the 160 KB of a
// compute unit), once per kernel and device; a no-op for requests of at most 64 KB.  Lock-free: two
// threads racing through a kernel's first call merely ask the runtime twice.
hipError_t allow_lds(const void* fn, size_t lds_bytes);

// Each returns a hipError_t from the launch (hipSuccess when enqueued).
hipError_t launch_forward_bf16(const FwdArgs& a, hipStream_t s);
hipError_t launch_forward_f32(const FwdArgs& a, hipStream_t s);
hipError_t launch_forward_f32_rows(const FwdArgs& a, hipStream_t s);
int staged_heads_per_block(int L, int heads);
hipError_t launch_forward_bf16_staged(const FwdArgs& a, hipStream_t s);
bool forward_wide_supported(int L, int head_dim);
hipError_t launch_forward_bf16_wide(const FwdArgs& a, hipStream_t s);
hipError_t launch_backward_bf16(const BwdArgs& a, hipStream_t s);
hipError_t launch_backward_f32(const BwdArgs& a, hipStream_t s);
int backward_slots(long long N, int heads, int nW, int L, bool mask, bool labels, bool dbias);
int coop_window_slots(long long N, int heads, int L, bool dense, bool dbias);
int backward_max_slots(long long N, int heads);
int coop_slots(long long N, int heads, int nW);
hipError_t launch_backward_bf16_coop(const BwdArgs& a, hipStream_t s);
hipError_t launch_backward_bf16_large(const BwdArgs& a, hipStream_t s);
hipError_t launch_backward_bf16_fused(const BwdArgs& a, hipStream_t s, bool forced, long long windows, bool& taken);
// Workgroups of `fn` one CU holds (LDS and registers decide), asked once per kernel
hipError_t workgroups_per_cu(const void* fn, unsigned block, size_t lds, std::atomic<int>& once, int& per_cu);
hipError_t launch_backward_bf16_wide(const BwdArgs& a, hipStream_t s);
int backward_wide_slots(long long N, int heads);
hipError_t launch_dbias_reduce(const BwdArgs& a, hipStream_t s, bool key_on_lane = false);
int backward_large_slots(long long N, int heads, int L);
hipError_t launch_zero_f32(float* dst, size_t count, hipStream_t s);
hipError_t launch_widen_bf16(const void* src, float* dst, size_t count, hipStream_t s);
hipError_t launch_bias_gather(const float* table, float* bias, int heads, int k, hipStream_t s);
hipError_t launch_bias_scatter(const float* dbias, float* dtable, int heads, int k, hipStream_t s);

// Attention of whole sequences (fwa_sequence_*.hip).
struct SeqArgs {
    const void* q;       // [N, Lq, H * D]
    const void* k;       // [N, Lk, KV * D]
    const void* v;
    void* o;             // forward: out; backward: in
    float* stats;        // [N, H, Lq, 2]: reference and base-2 logarithm of the sum of each row, or nullptr (forward only)
    const void* d_o;
    void* dq;
    void* dk;
    void* dv;
    float* dtable;       // [H, nb] or nullptr
    const float* table;  // [H, nb] or nullptr
    const int32_t* buckets;  // [2 far + 1]
    const int32_t* q_len;    // [N] or nullptr
    const int32_t* k_len;
    const int32_t* q_start;
    long long N;
    int Lq, Lk, H, KV, D;
    int nb, far;
    int causal;
    int dtype;           // 0 fp32, 1 bf16, 2 half
    float scale;
    long long ldq, ldk, ldo, ldg, lddq, lddk;  // elements between rows of q; of k and v; of o; of d_o; of dq; of dk and dv
};

// Waves of a workgroup that share out the keys, two tiles each of K and V a wave in 64 KB of LDS, and keys per tile of the forward.
constexpr int seq_keys_waves(int row_bytes) { return row_bytes >= 512 ? 1 : row_bytes >= 256 ? 2 : 4; }
constexpr int seq_forward_keys(int row_bytes, bool keys) { return row_bytes >= 512 || keys ? 32 : 64; }
// Keys resp. queries per tile of the backward.
constexpr int seq_backward_rows(int row_bytes) { return row_bytes >= 256 ? 32 : 64; }

hipError_t launch_sequence_forward(const SeqArgs& a, void* workspace, hipStream_t s);
bool seq_forward_fits(const SeqArgs& a);  // a launch holds the call's workgroups
size_t seq_forward_workspace(const SeqArgs& a);
hipError_t launch_sequence_backward(const SeqArgs& a, void* workspace, hipStream_t s);
bool seq_backward_fits(const SeqArgs& a);
size_t seq_backward_workspace(const SeqArgs& a, bool want_dtable);
hipError_t launch_bucket_gather(const float* table, const int32_t* buckets, void* bias, int heads, int nb, int far, int Lq, int Lk, int q_start, bool bf16,
                                hipStream_t s);
size_t bucket_lines_bytes(int heads, int far, long long count);
hipError_t launch_bucket_sums(const float* parts, float* lines, const int32_t* buckets, float* dtable, int heads, int nb, int far, long long count, hipStream_t s);
size_t bucket_scatter_workspace(int heads, int far, int Lq);
hipError_t launch_bucket_scatter(const float* dbias, const int32_t* buckets, float* dtable, int heads, int nb, int far, int Lq, int Lk, int q_start,
                                 float* workspace, hipStream_t s);

// Rotary positions (fwa_rotary.hip).
struct RotaryArgs {
    const void* x;       // [rows, heads * d]
    void* y;
    long long rows;
    int heads, d, dtype;
    long long ldx, ldy;
    const int32_t* positions;  // [period, axes]: row r has those of r mod period
    long long period;
    int axes;
    const float* frequencies;  // [pairs], radians a position
    const int32_t* axis_of;    // [pairs] or nullptr: all the first
    int pairs;
    int interleaved, inverse;
};
bool rotary_fits(long long rows, int heads, int d, int pairs, int dtype);
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s);

// A paged cache and the new tokens of a call, packed one sequence behind the other (fwa_page_*.hip).
struct PageArgs {
    void* k;             // row t % page_size of page p of head h: k + p page_stride + (t % page_size) token_stride + h head_stride elements
    void* v;
    long long page_stride, token_stride, head_stride;
    int pages, page_size, width;
    const int32_t* table;    // [N, width]
    const int32_t* offsets;  // [N + 1]
    const int32_t* lengths;  // [N]: tokens in the cache in front of the new ones
    int N, rows;             // sequences, new tokens in all
    int H, KV, D, dtype;
    const void* q;           // [rows, H * D]
    void* o;
    long long ldq, ldo;
    // attention
    float* stats;        // [rows, H, 2] or nullptr
    int most;            // new tokens of a sequence that count, as rows and as keys
    int causal;
    float scale;
    // append: o is the rotated q
    const void* new_k;   // [rows, KV * D]
    const void* new_v;
    long long ldk, ldv;
    const int32_t* positions;  // [rows, axes], or nullptr: the place in the sequence
    int axes;
    const float* frequencies;
    const int32_t* axis_of;
    int pairs, interleaved;
};
bool page_append_fits(const PageArgs& a);
hipError_t launch_page_append(const PageArgs& a, hipStream_t s);
bool page_forward_fits(const PageArgs& a);
size_t page_forward_workspace(const PageArgs& a);
hipError_t launch_page_forward(const PageArgs& a, void* workspace, size_t workspace_bytes, hipStream_t s);

}  // namespace fwa
