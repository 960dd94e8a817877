/*
 * fwa.h -- C ABI of the Flash Window Attention library for AMD MI355X (gfx950).
 *
 * The library computes fused, batched short-sequence attention over
 * window-partitioned tensors (paper Section 2.1, eq. 1-4):
 *
 *     O[n, :, head h] = softmax(scale * Q_nh K_nh^T + B[h] + M[n mod nW]) V_nh
 *
 * with the whole L x L score/probability tile kept on chip and Q, K, V, O
 * crossing device memory exactly once (paper Algorithm 1), and its backward
 * (paper Algorithm 2) which recomputes P on chip and needs nothing saved from
 * the forward.  The paper's equations carry no scale, bias or mask; they are
 * additive extensions: scale multiplies QK^T before B and M are added.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Every pointer is a DEVICE pointer owned by the caller.  The library
 *    never allocates, frees or synchronises; it enqueues kernels on `stream`
 *    (a hipStream_t passed as void*; NULL = the default stream) and returns.
 *  - Tensors are contiguous, row-major.  Q, K, V, O, dO, dQ, dK, dV are
 *    [N, L, C]; head h owns channels [h*d, (h+1)*d) with d = C / heads.
 *    Supported: d == 32 with 1 <= L <= 256; d == 64, 128, 256 with
 *    1 <= L <= 64 (the feature-dimension loop of paper eq. 5-6; the shapes of
 *    its Section 3.1 benchmark), in fp32 and bf16 (half: the wider heads only,
 *    see dtype).  N >= 0 (N == 0 is a no-op).
 *  - dtype is FWA_F32 (fp32 data, sums and softmax; products with 24
 *    significant bits of every value, subnormal ones included, by the fp32
 *    matrix instruction or by bf16 ones on exact three-part splits; infinities,
 *    NaN and overflow as in fp32 arithmetic), FWA_BF16 (bf16 data,
 *    bf16 matrix-core products with fp32 accumulation, fp32 softmax, one final
 *    round-to-nearest-even to bf16) or FWA_F16 (IEEE half data, handled like
 *    bf16 with half products; head widths 64, 128 and 256 only, i.e. the
 *    shapes and the precision of the paper's Section 3 comparisons;
 *    FWA_ERR_UNSUPPORTED at head width 32).  With half data every intermediate
 *    that enters a matrix product -- P, dS -- must stay inside the half range.
 *  - mask and dbias are always fp32; bias is fp32, or bf16 through the
 *    *_labels entry points (bias_dtype).
 *  - Base pointers must be 16-byte aligned.  No output may share a byte with an
 *    input or with another output (FWA_ERR_ALIAS).  For row-strided tensors of
 *    one stride -- the q/k/v or dq/dk/dv views of one fused buffer -- the test is
 *    exact: rows may interleave.  Tensors of different strides whose address
 *    extents intersect are rejected even if their rows happen not to touch.
 *  - The return value is FWA_OK or an error code; on error nothing has been
 *    launched.
 *  - Calls are thread-safe.  The only state the library keeps is per kernel and
 *    device, behind atomics: whether the runtime has been told that the kernel
 *    may use more than 64 KB of LDS (hipFuncSetAttribute), how many of its
 *    workgroups fit a compute unit, and the device's compute-unit count.  These
 *    are asked on the first call that needs them, so a caller that records calls
 *    into a HIP graph makes one call of the same shape outside the capture first.
 *    (fwa_backward_noalloc also shares one scratch array per device: see there.)
 */
#ifndef FWA_H
#define FWA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { FWA_F32 = 0, FWA_BF16 = 1, FWA_F16 = 2 };

enum {
    FWA_OK = 0,
    FWA_ERR_NULL = 1,        /* a required pointer is NULL                          */
    FWA_ERR_SHAPE = 2,       /* negative N, L < 1, C % heads != 0, N % nW != 0, ... */
    FWA_ERR_UNSUPPORTED = 3, /* head dim, L, dtype or dbias outside the ranges above */
    FWA_ERR_ALIGN = 4,       /* a base pointer is not 16-byte aligned               */
    FWA_ERR_WORKSPACE = 5,   /* workspace missing or smaller than required          */
    FWA_ERR_LAUNCH = 6,      /* the HIP runtime refused the launch                  */
    FWA_ERR_ALIAS = 7        /* an output shares memory with another argument       */
};

/*
 * Forward pass (paper Algorithm 1; eq. 2-4).
 *   q, k, v : in,  [N, L, C], dtype
 *   o       : out, [N, L, C], dtype, fully overwritten
 *   bias    : NULL, or in [heads, L, L] fp32 (already gathered per token pair)
 *   mask    : NULL, or in [nW, L, L] fp32, added to the scores of window n as
 *             mask[n % nW]; requires nW >= 1 and N % nW == 0.  nW is ignored
 *             when mask is NULL.
 */
int fwa_forward(const void* q, const void* k, const void* v, void* o,
                int64_t N, int L, int C, int heads, float scale,
                const float* bias, const float* mask, int nW,
                int dtype, void* stream);

/*
 * The same with row strides: token row (n, l) of q, k and v starts ld_qkv elements after row
 * (n, l) - 1 (window n begins at row n*L), and likewise ld_o for o; ld == C is the contiguous
 * case above.  This reads Q, K, V in place out of a fused projection output [N, L, 3, heads, d]
 * (q = base, k = base + C, v = base + 2C elements, ld_qkv = 3C), saving the permute and copy in
 * front of the kernel.  Strides must be >= C and keep rows 16-byte aligned (FWA_ERR_SHAPE /
 * FWA_ERR_ALIGN otherwise).
 */
int fwa_forward_strided(const void* q, const void* k, const void* v, void* o,
                        int64_t N, int L, int C, int heads, float scale,
                        int64_t ld_qkv, int64_t ld_o,
                        const float* bias, const float* mask, int nW,
                        int dtype, void* stream);

/*
 * Backward pass (paper Algorithm 2).  Inputs are Q, K, V and dO only.
 * Supported: FWA_BF16 and FWA_F16 in every shape the forward takes them;
 * FWA_F32 for L <= 64 without dbias (FWA_ERR_UNSUPPORTED otherwise).
 *   d_o        : in,  [N, L, C], dtype
 *   dq, dk, dv : out, [N, L, C], dtype, fully overwritten
 *   dbias      : NULL, or out [heads, L, L] fp32 = sum over all N windows of
 *                dS; overwritten, not accumulated.  The mask gets no gradient.
 *   workspace  : device scratch of at least fwa_backward_workspace_bytes(...)
 *                bytes, 16-byte aligned.  It holds per-workgroup partial sums
 *                of dbias and, for L > 64, the fp32 copy of a bf16 bias
 *                (fwa_backward_labels).  It
 *                may be NULL when dbias is NULL, unless L > 64 and the bias is
 *                bf16.  Contents on entry are ignored and undefined on exit.
 * Results are bit-reproducible from run to run for fixed arguments.
 * For L > 64 a row that finite additive terms of about -1.2e7 or less shut to every key enters dk, dv and
 * dbias with up to L times its weight (fp32 cannot hold the logarithm of its sum beside such a maximum);
 * its dq is not affected, nor is anything where its d_o is zero.
 */
int fwa_backward(const void* q, const void* k, const void* v, const void* d_o,
                 void* dq, void* dk, void* dv, float* dbias,
                 int64_t N, int L, int C, int heads, float scale,
                 const float* bias, const float* mask, int nW,
                 int dtype, void* workspace, size_t workspace_bytes, void* stream);

/* The same with row strides (see fwa_forward_strided): ld_qkv for q, k, v; ld_do for d_o;
 * ld_dqkv for dq, dk, dv, so that the three gradients can be written straight into a fused
 * [N, L, 3, heads, d] gradient buffer. */
int fwa_backward_strided(const void* q, const void* k, const void* v, const void* d_o,
                         void* dq, void* dk, void* dv, float* dbias,
                         int64_t N, int L, int C, int heads, float scale,
                         int64_t ld_qkv, int64_t ld_do, int64_t ld_dqkv,
                         const float* bias, const float* mask, int nW,
                         int dtype, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Forward and backward with the shift mask given as region labels instead of a dense tile,
 * and optionally a bf16 bias
 * (paper Section 2.1: shifted blocks mask attention between tokens that were not neighbours
 * before the cyclic shift; the labels name the regions of the shifted token map):
 *   labels     : NULL (no mask), or in [nW, L] int32; the scores of window n receive
 *                M[i][j] = labels[n % nW][i] == labels[n % nW][j] ? 0 : mask_value,
 *                formed inside the kernels.  This reads L * 4 bytes per window position
 *                instead of L * L * 4.  Requires nW >= 1 and N % nW == 0; 16-byte aligned.
 *   mask_value : what a pair of tokens with different labels adds to its score (-100 in
 *                the Swin Transformer); ignored when labels is NULL.
 *   bias       : NULL, or in [heads, L, L] of type bias_dtype: FWA_F32 as everywhere else, or
 *                FWA_BF16 (half the bytes; the values are used as they are, i.e. the result is
 *                that of the fp32 call on the same values).  dbias stays fp32.
 * Everything else (shapes, strides, dtype, workspace, error codes, supported ranges) is as in
 * fwa_forward_strided / fwa_backward_strided, and the results are those of the same call with
 * the dense mask written out from the labels: bit for bit while nW is small enough for a
 * workgroup to keep one mask tile for life (nW <= 256 / heads-per-workgroup, roughly, and
 * for the backward above 64 tokens as long as a number of workgroups that is a multiple of nW
 * leaves less than about a quarter of the device idle), and to
 * within a rounding of the additive term beyond, where the dense form reads each window's
 * mask tile and this form makes it from the window's labels.
 */
int fwa_forward_labels(const void* q, const void* k, const void* v, void* o,
                       int64_t N, int L, int C, int heads, float scale,
                       int64_t ld_qkv, int64_t ld_o,
                       const void* bias, int bias_dtype, const int32_t* labels, float mask_value, int nW,
                       int dtype, void* stream);

int fwa_backward_labels(const void* q, const void* k, const void* v, const void* d_o,
                        void* dq, void* dk, void* dv, float* dbias,
                        int64_t N, int L, int C, int heads, float scale,
                        int64_t ld_qkv, int64_t ld_do, int64_t ld_dqkv,
                        const void* bias, int bias_dtype, const int32_t* labels, float mask_value, int nW,
                        int dtype, void* workspace, size_t workspace_bytes, void* stream);

/*
 * fwa_backward for callers that cannot allocate: code under HIP graph capture, serving loops,
 * harnesses that forbid hipMalloc.  It is fwa_backward without the workspace arguments: the
 * workspace (dBias partial sums) lives in an array of
 * FWA_NOALLOC_SCRATCH_BYTES bytes inside the library's code object, of which every device the
 * library runs on holds its own copy until the process ends.  The call itself allocates and frees
 * nothing, and runs the same kernels with the same results, bit for bit, as fwa_backward.
 *   - A call whose workspace would exceed the array returns FWA_ERR_WORKSPACE.  Every bf16 call
 *     with L <= 64, head width 32 and at most 1024 heads fits (at most 3 x compute-units tiles of
 *     16 KB = 12 MiB); large windows with dbias mostly do not.  Without dbias no scratch is used at all.
 *   - All calls on one device share that device's array, which keeps the previous call's contents;
 *     the kernels overwrite every element they later read, so nothing needs clearing.  Calls that
 *     overlap in time on one device (two streams, two threads) race on it: serialise them.
 *   - The array's device address is looked up on the first call on each device
 *     (hipGetSymbolAddress, no allocation).
 */
#define FWA_NOALLOC_SCRATCH_BYTES (16u * 1024u * 1024u)
int fwa_backward_noalloc(const void* q, const void* k, const void* v, const void* d_o,
                         void* dq, void* dk, void* dv, float* dbias,
                         int64_t N, int L, int C, int heads, float scale,
                         const float* bias, const float* mask, int nW,
                         int dtype, void* stream);

/* Bytes of workspace that suffice for any backward call with these arguments
 * (0 if none is needed; for L > 64 the size includes room for the fp32 copy of
 * a bf16 bias whether or not one will be passed).  Returns 0 for arguments
 * fwa_backward would reject. */
size_t fwa_backward_workspace_bytes(int64_t N, int L, int C, int heads, int dtype, int want_dbias);

/*
 * Relative-position bias helpers for k x k windows (L = k*k).  Token i sits
 * at (i / k, i % k); pair (i, j) maps to table column
 * (y_i - y_j + k - 1) * (2k - 1) + (x_i - x_j + k - 1).  The paper only says
 * its baseline follows Swin Transformer; this is that published indexing.
 *   fwa_bias_gather : table [heads, (2k-1)^2] -> bias [heads, L, L]
 *   fwa_bias_scatter: dbias [heads, L, L] -> dtable [heads, (2k-1)^2]
 *                     (adjoint of the gather; overwritten; fixed summation
 *                     order, bit-reproducible)
 * All fp32 device pointers.  Requires heads >= 1 and 1 <= k <= 16.
 */
int fwa_bias_gather(const float* table, float* bias, int heads, int k, void* stream);
int fwa_bias_scatter(const float* dbias, float* dtable, int heads, int k, void* stream);

/*
 * Relative-position bias by buckets for 1-D sequences.  The distance key - query of a pair, cut off at -far and
 * far, names a column of the table:
 *   bias[h][i][j] = table[h][ buckets[far + clamp(j - (q_start + i), -far, far)] ],   i < Lq, j < Lk
 *   table   : [heads, columns] fp32
 *   buckets : [2 far + 1] int32; an entry outside [0, columns) adds nothing and gets no gradient
 *   q_start : position of query 0 on the axis of the keys
 * fwa_bucket_gather  : table -> bias [heads, Lq, Lk], fp32 or (bias_dtype FWA_BF16, rounded once) bf16: the bias of
 *                      fwa_forward and fwa_backward where Lq == Lk <= 256, or a dense one for other code
 * fwa_bucket_scatter : dbias [heads, Lq, Lk] fp32 -> dtable [heads, columns], its adjoint: overwritten, fixed summation
 *                      order, bit-reproducible.  `workspace` is device scratch of at least
 *                      fwa_bucket_scatter_workspace_bytes(...) bytes, 16-byte aligned.
 * heads <= 2^15, columns <= 2^16, far <= FWA_BUCKET_MAX_FAR, Lq and Lk from 0 to 2^24, heads * Lq <= 2^28.  table and buckets
 * need 4-byte alignment only.  No dimension of zero launches anything but the zeros of dtable.
 */
#define FWA_BUCKET_MAX_FAR 8192
int fwa_bucket_gather(const float* table, const int32_t* buckets, void* bias, int heads, int columns, int far,
                      int Lq, int Lk, int64_t q_start, int bias_dtype, void* stream);
int fwa_bucket_scatter(const float* dbias, const int32_t* buckets, float* dtable, int heads, int columns, int far,
                       int Lq, int Lk, int64_t q_start, void* workspace, size_t workspace_bytes, void* stream);
size_t fwa_bucket_scatter_workspace_bytes(int heads, int columns, int far, int Lq, int Lk);

/*
 * Attention of whole sequences: any number of queries and keys, scores never in memory.
 *   O[n, i, head h] = sum_j P[i][j] V[n, j, head g],  P = softmax_j(scale * Q_ih . K_jg + B[h][i][j]),  g = h / (heads / kv_heads)
 * over the keys j that query i sees.
 *   q, o      : [N, Lq, heads * d], rows ld_q resp. ld_o elements apart (sequence n begins at row n * Lq)
 *   k, v      : [N, Lk, kv_heads * d], rows ld_kv elements apart; kv_heads divides heads
 *   d         : 32, 64 or 128; dtype FWA_F32, FWA_BF16 or FWA_F16.  Lq and Lk from 0 to 2^24, heads <= 2^15, heads * Lq <= 2^28,
 *               row strides <= 2^20 elements, N * heads * (max(Lq, Lk) / 128 + 1) up to about 15 million (a launch's workgroups).
 *   table, buckets, columns, far : the bias B by buckets, formed inside the kernels, as in fwa_bucket_gather (with the
 *               q_start below for each sequence); table NULL: none, the other three are ignored
 *   q_lengths : NULL, or [N] int32: queries from q_lengths[n] on are padding; their rows of o are zero
 *   k_lengths : NULL, or [N] int32: keys from k_lengths[n] on are not seen, whatever memory holds there.  Both lengths are cut
 *               off at 0 and at Lq resp. Lk.
 *   q_start   : NULL (0), or [N] int32: position of query 0 of sequence n on the axis of its keys
 *   causal    : nonzero: query i sees the keys j <= q_start[n] + i only
 *   stats     : NULL, or out [N, heads, Lq, 2] fp32: for each row a reference r and log2 of sum_j 2^(s_j - r), s the scores
 *               in base-2 units (times log2 e); their sum times ln 2 is the logarithm of the row's sum.  (-inf, 0) for a row
 *               without a key.
 *   workspace : device scratch of at least fwa_sequence_forward_workspace_bytes(...) bytes (0 for most calls; few rows against
 *               many keys are shared out over the keys and joined), 16-byte aligned
 * A row that sees no key, or whose scores are all -inf, gives zeros.  Table values of -inf shut pairs out; the lowest finite value
 * counts as such (a row of nothing else is uniform).  Inside the lengths q, k, v and d_o are expected to be finite: an
 * infinity or NaN in a key's row may reach queries that causality keeps from seeing it, and one in a query's row the gradients of
 * keys that it does not see.  Neither reaches padding or heads that do not share the keys.  The statistics of a row of NaN alone are (-inf, NaN).
 * Arithmetic: fp32 data in fp32 throughout; 16-bit data are multiplied as they are, sums, softmax and statistics are fp32, P and
 * (backward) dS are rounded once to the data's type in front of the product they enter.
 * Lengths, starts, table and buckets need 4-byte alignment only.
 */
int fwa_sequence_forward(const void* q, const void* k, const void* v, void* o, float* stats,
                         int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, float scale,
                         int64_t ld_q, int64_t ld_kv, int64_t ld_o,
                         const float* table, const int32_t* buckets, int columns, int far,
                         const int32_t* q_lengths, const int32_t* k_lengths, const int32_t* q_start, int causal,
                         int dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t fwa_sequence_forward_workspace_bytes(int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, int dtype);

/*
 * Its gradients, with the probabilities formed again from stats.
 *   o, stats   : what the forward of the same arguments wrote
 *   d_o        : in, like o, rows ld_do apart
 *   dq, dk, dv : out, like q, k, v, rows ld_dq resp. ld_dkv apart, fully overwritten (padding with zeros)
 *   dtable     : NULL, or out [heads, columns] fp32: the gradient of the table, overwritten; its terms are not rounded to the
 *                data's type
 *   workspace  : at least fwa_sequence_backward_workspace_bytes(...) bytes, 16-byte aligned
 * Bit-reproducible from run to run.  With half data dS beyond 1023 overflows.  dq of 16-bit data in rows of more than 128 keys
 * takes over half a step of the data's type of sum |d_o o|, from o as it is stored, in delta.
 */
int fwa_sequence_backward(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* stats,
                          void* dq, void* dk, void* dv, float* dtable,
                          int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, float scale,
                          int64_t ld_q, int64_t ld_kv, int64_t ld_o, int64_t ld_do, int64_t ld_dq, int64_t ld_dkv,
                          const float* table, const int32_t* buckets, int columns, int far,
                          const int32_t* q_lengths, const int32_t* k_lengths, const int32_t* q_start, int causal,
                          int dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t fwa_sequence_backward_workspace_bytes(int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, int far, int dtype,
                                             int want_dtable);

/*
 * Rotary positions with several axes (time, height and width of a video; row and column of an image; one for text).  Pair p of every head's
 * channels is turned by the angle positions[r][axis_of[p]] * frequencies[p]:
 *   (a, b) -> (a cos - b sin, b cos + a sin),  channels p and p + pairs, or (interleaved nonzero) 2 p and 2 p + 1
 * Channels from 2 pairs on stay as they are.
 *   x           : in,  [rows, heads * d], rows ld_x elements apart
 *   y           : out, like x, rows ld_y apart; may be x itself (the same address and stride), else no byte of it
 *   positions   : [position_rows, axes] int32; row r of x has row r mod position_rows of them (position_rows = L for all sequences of [N, L])
 *   frequencies : [pairs] fp32, radians a position
 *   axis_of     : [pairs] int32, or NULL: all pairs the first axis.  A pair with an axis outside [0, axes) stays as it is.
 *   inverse     : nonzero: by the negative angle, which is the inverse, and the gradient of x from that of y
 * d from 1 to 512, 0 <= pairs <= d / 2, axes <= 16, dtype FWA_F32, FWA_BF16 or FWA_F16, rows * heads * d / 2 below 2e9.  Angles are formed in 64 bits and
 * reduced to a turn there, so far positions lose nothing (2^20 of frequency 1: 1e-7 of the result, as near ones); the rotation is fp32, rounded once.
 * positions, frequencies and axis_of need 4-byte alignment only.
 */
int fwa_rotary(const void* x, void* y, int64_t rows, int heads, int d, int64_t ld_x, int64_t ld_y, const int32_t* positions,
               int64_t position_rows, int axes, const float* frequencies, const int32_t* axis_of, int pairs, int interleaved, int inverse,
               int dtype, void* stream);

/*
 * A paged cache: keys and values of N sequences in pages of page_size rows.  The token at place t of sequence n lies in row t % page_size of
 * page page_table[n][t / page_size].
 *   k_pages, v_pages : [pages, page_size, kv_heads, d]; row r of page p of head h begins p * page_stride + r * token_stride + h * head_stride
 *                      elements behind the base, so pages with a head's rows together ([pages, kv_heads, page_size, d]) are meant as well.  The strides, one set
 *                      for both, are multiples of 16 bytes (FWA_ERR_ALIGN), reach no element twice (FWA_ERR_SHAPE), token_stride <= 2^20,
 *                      page_stride <= 2^29 elements.  Keys and values may interleave in one buffer.
 *   page_size        : a multiple of 16, at most 65536; width * page_size <= 2^29; the whole cache of any size
 *   page_table       : [N, width] int32.  An entry outside [0, pages) is no page: nothing is stored there and its keys are not seen.
 *   offsets          : [N + 1] int32, not falling: the new tokens of sequence n are rows offsets[n] .. offsets[n + 1] - 1 of the packed tensors
 *                      [rows, heads * d].  Rows in front of offsets[0] and from offsets[N] on are left as they were.
 *   lengths          : [N] int32: tokens of sequence n in front of the new ones; new token i has place lengths[n] + i.  Below 0 counts as 0.
 * Both calls of a step take the same tables.  d is 32, 64 or 128, dtype FWA_F32, FWA_BF16 or FWA_F16 for all tensors, rows <= 2^24,
 * N <= 2^20, rows * (heads + 2 kv_heads) <= 2^28, N * kv_heads up to about 15 million.  The tables need 4-byte alignment only.
 *
 * fwa_page_append stores the new tokens' keys, rotated, and values in their places, and rotates their queries besides.
 *   k, v       : [rows, kv_heads * d], rows ld_k resp. ld_v apart
 *   positions, axes, frequencies, axis_of, pairs, interleaved : the rotation of fwa_rotary, positions [rows, axes]; NULL: one axis, the
 *                token's place in its sequence.  pairs 0: none.
 *   q, q_out   : NULL, or [rows, heads * d]: the rotated queries; q_out may be q itself.  heads and the strides are ignored without them.
 * Tokens beyond width * page_size are not stored.  Two tokens of a call must not have one row of a page.
 */
int fwa_page_append(const void* k, const void* v, void* k_pages, void* v_pages, int64_t rows, int64_t N, int kv_heads, int d, int64_t ld_k,
                    int64_t ld_v, int64_t pages, int page_size, int64_t page_stride, int64_t token_stride, int64_t head_stride,
                    const int32_t* page_table, int width, const int32_t* offsets, const int32_t* lengths, const int32_t* positions,
                    int axes, const float* frequencies, const int32_t* axis_of, int pairs, int interleaved, const void* q, void* q_out,
                    int heads, int64_t ld_q, int64_t ld_q_out, int dtype, void* stream);

/*
 * Attention of the new tokens over the cache that already holds them: token i of sequence n sees the keys at places up to lengths[n] + i
 * (causal nonzero) or all lengths[n] + new ones, of those within width * page_size whose page exists.
 *   q, o      : [rows, heads * d], rows ld_q resp. ld_o apart; kv_heads divides heads
 *   most_new  : no sequence has more new tokens.  Of one that has, the first most_new are all there are: the others are not computed, their
 *               rows are left as they were, and (causal zero) nobody sees their keys, whatever the cache holds.  The smaller this is, the
 *               better the call can be laid out (1 for single tokens); rows is always enough.
 *   stats     : NULL, or out [rows, heads, 2] fp32, the row statistics as in fwa_sequence_forward
 *   workspace : device scratch of at least fwa_page_forward_workspace_bytes(...) bytes, 16-byte aligned.  It goes by the arguments on the host, the
 *               lengths and offsets are read on the device alone: a captured call may be replayed with others.
 * A row that sees no key gives zeros.  Arithmetic as in fwa_sequence_forward; infinities and NaN in rows of the cache from lengths[n] + new
 * on are never read, those in a key's row that causality shuts out may reach the rows that do not see it.
 * Bit-reproducible from run to run.
 */
int fwa_page_forward(const void* q, const void* k_pages, const void* v_pages, void* o, float* stats, int64_t rows, int64_t N, int heads,
                     int kv_heads, int d, float scale, int64_t ld_q, int64_t ld_o, int64_t pages, int page_size, int64_t page_stride,
                     int64_t token_stride, int64_t head_stride, const int32_t* page_table, int width, const int32_t* offsets,
                     const int32_t* lengths, int most_new, int causal, int dtype, void* workspace, size_t workspace_bytes, void* stream);
size_t fwa_page_forward_workspace_bytes(int64_t rows, int64_t N, int heads, int kv_heads, int d, int page_size, int width, int most_new,
                                        int dtype);

/* Static, NUL-terminated description of an error code. */
const char* fwa_status_string(int code);

#ifdef __cplusplus
}
#endif
#endif /* FWA_H */
