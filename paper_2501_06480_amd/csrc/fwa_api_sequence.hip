// extern "C" entry points of the bias by buckets and of the attention of whole sequences: argument validation and dispatch.
// Every check happens before any HIP call, so an error never launches work.
#include "../../include/fwa.h"
#include "fwa_check.h"
#include "fwa_internal.h"

namespace {

using namespace fwa::check;

constexpr int kMostRows = 1 << 24, kMostHeads = 1 << 15, kMostColumns = 1 << 16, kFarthest = 1 << 29;

inline bool odd_word(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
inline Span flat(const void* p, uint64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), bytes, bytes, 1}; }

int check_buckets(int heads, int columns, int far) {
    if (heads < 1 || columns < 1 || far < 0) return FWA_ERR_SHAPE;
    if (heads > kMostHeads || columns > kMostColumns || far > FWA_BUCKET_MAX_FAR) return FWA_ERR_UNSUPPORTED;
    return FWA_OK;
}
int check_pairs(int heads, int Lq, int Lk) {
    if (Lq < 0 || Lk < 0) return FWA_ERR_SHAPE;
    return Lq > kMostRows || Lk > kMostRows || (int64_t)heads * Lq > 1 << 28 ? FWA_ERR_UNSUPPORTED : FWA_OK;
}
int clamped(int64_t q_start) { return (int)(q_start < -kFarthest ? -kFarthest : (q_start > kFarthest ? kFarthest : q_start)); }

// What forward, backward and the workspace queries share; fills in the sizes.
int check_sequence(fwa::SeqArgs& a, int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, int dtype) {
    if (N < 0 || heads < 1 || kv_heads < 1 || d < 1 || heads % kv_heads != 0) return FWA_ERR_SHAPE;
    const int rc = check_pairs(heads, Lq, Lk);
    if (rc != FWA_OK) return rc;
    if (dtype != FWA_F32 && dtype != FWA_BF16 && dtype != FWA_F16) return FWA_ERR_UNSUPPORTED;
    if (d != 32 && d != 64 && d != 128) return FWA_ERR_UNSUPPORTED;
    if (heads > kMostHeads) return FWA_ERR_UNSUPPORTED;
    // one launch per kernel: fewer than 2^32 threads
    if ((double)N * heads * ((Lq > Lk ? Lq : Lk) / 128 + 1.0) * 256.0 > 3.9e9) return FWA_ERR_UNSUPPORTED;
    a.N = N; a.Lq = Lq; a.Lk = Lk; a.H = heads; a.KV = kv_heads; a.D = d; a.dtype = dtype;
    return FWA_OK;
}
int check_terms(fwa::SeqArgs& a, const float* table, const int32_t* buckets, int columns, int far, const int32_t* q_lengths, const int32_t* k_lengths,
                const int32_t* q_start, int causal, float scale) {
    a.table = table; a.buckets = table ? buckets : nullptr; a.nb = 0; a.far = 0;
    if (table) {
        const int rc = check_buckets(a.H, columns, far);
        if (rc != FWA_OK) return rc;
        if (!buckets) return FWA_ERR_NULL;
        a.nb = columns; a.far = far;
    }
    if (odd_word(table) || odd_word(a.buckets) || odd_word(q_lengths) || odd_word(k_lengths) || odd_word(q_start)) return FWA_ERR_ALIGN;
    a.q_len = q_lengths; a.k_len = k_lengths; a.q_start = q_start; a.causal = causal != 0; a.scale = scale;
    return FWA_OK;
}

// The tensors of a call as the bytes that they touch; no output may share one with an input or with another output.
struct Touched {
    Span ins[16], outs[8];
    int ni = 0, no = 0;
    void in(const Span& s) { ins[ni++] = s; }
    void out(const Span& s) { outs[no++] = s; }
    // what all sequence calls read besides their tensors
    void terms(const fwa::SeqArgs& a) {
        if (a.table) {
            in(flat(a.table, (uint64_t)a.H * a.nb * 4));
            in(flat(a.buckets, (2 * (uint64_t)a.far + 1) * 4));
        }
        for (const int32_t* p : {a.q_len, a.k_len, a.q_start})
            if (p && a.N > 0) in(flat(p, (uint64_t)a.N * 4));
    }
    bool shared() const {
        for (int x = 0; x < no; ++x) {
            for (int y = 0; y < ni; ++y)
                if (overlaps(outs[x], ins[y])) return true;
            for (int y = x + 1; y < no; ++y)
                if (overlaps(outs[x], outs[y])) return true;
        }
        return false;
    }
};

}  // namespace

extern "C" {

int fwa_bucket_gather(const float* table, const int32_t* buckets, void* bias, int heads, int columns, int far, int Lq, int Lk, int64_t q_start,
                      int bias_dtype, void* stream) {
    int rc = check_buckets(heads, columns, far);
    if (rc == FWA_OK) rc = check_pairs(heads, Lq, Lk);
    if (rc != FWA_OK) return rc;
    if (bias_dtype != FWA_F32 && bias_dtype != FWA_BF16) return FWA_ERR_UNSUPPORTED;
    if (Lq == 0 || Lk == 0) return FWA_OK;
    if (!table || !buckets || !bias) return FWA_ERR_NULL;
    if (odd_word(table) || odd_word(buckets) || misaligned(bias)) return FWA_ERR_ALIGN;
    const Span out = flat(bias, (uint64_t)heads * Lq * Lk * (bias_dtype == FWA_F32 ? 4 : 2));
    if (overlaps(out, flat(table, (uint64_t)heads * columns * 4)) || overlaps(out, flat(buckets, (2 * (uint64_t)far + 1) * 4))) return FWA_ERR_ALIAS;
    return fwa::launch_bucket_gather(table, buckets, bias, heads, columns, far, Lq, Lk, clamped(q_start), bias_dtype == FWA_BF16,
                                     static_cast<hipStream_t>(stream)) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

size_t fwa_bucket_scatter_workspace_bytes(int heads, int columns, int far, int Lq, int Lk) {
    if (check_buckets(heads, columns, far) != FWA_OK || check_pairs(heads, Lq, Lk) != FWA_OK || Lq == 0 || Lk == 0) return 0;
    return fwa::bucket_scatter_workspace(heads, far, Lq);
}

int fwa_bucket_scatter(const float* dbias, const int32_t* buckets, float* dtable, int heads, int columns, int far, int Lq, int Lk, int64_t q_start,
                       void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_buckets(heads, columns, far);
    if (rc == FWA_OK) rc = check_pairs(heads, Lq, Lk);
    if (rc != FWA_OK) return rc;
    if (!dtable) return FWA_ERR_NULL;
    if (misaligned(dtable)) return FWA_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (Lq == 0 || Lk == 0)  // the sum over no pairs: dtable is still overwritten
        return fwa::launch_zero_f32(dtable, (size_t)heads * columns, st) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
    if (!dbias || !buckets) return FWA_ERR_NULL;
    if (misaligned(dbias) || odd_word(buckets) || misaligned(workspace)) return FWA_ERR_ALIGN;
    const Span out = flat(dtable, (uint64_t)heads * columns * 4);
    if (overlaps(out, flat(dbias, (uint64_t)heads * Lq * Lk * 4)) || overlaps(out, flat(buckets, (2 * (uint64_t)far + 1) * 4))) return FWA_ERR_ALIAS;
    if (!workspace || workspace_bytes < fwa_bucket_scatter_workspace_bytes(heads, columns, far, Lq, Lk)) return FWA_ERR_WORKSPACE;
    return fwa::launch_bucket_scatter(dbias, buckets, dtable, heads, columns, far, Lq, Lk, clamped(q_start), static_cast<float*>(workspace), st) == hipSuccess
               ? FWA_OK : FWA_ERR_LAUNCH;
}

size_t fwa_sequence_forward_workspace_bytes(int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, int dtype) {
    fwa::SeqArgs a = {};
    if (check_sequence(a, N, Lq, Lk, heads, kv_heads, d, dtype) != FWA_OK || N == 0 || Lq == 0) return 0;
    return fwa::seq_forward_workspace(a);
}

int fwa_sequence_forward(const void* q, const void* k, const void* v, void* o, float* stats, int64_t N, int Lq, int Lk, int heads, int kv_heads, int d,
                         float scale, int64_t ld_q, int64_t ld_kv, int64_t ld_o, const float* table, const int32_t* buckets, int columns, int far,
                         const int32_t* q_lengths, const int32_t* k_lengths, const int32_t* q_start, int causal, int dtype, void* workspace,
                         size_t workspace_bytes, void* stream) {
    fwa::SeqArgs a = {};
    int rc = check_sequence(a, N, Lq, Lk, heads, kv_heads, d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_q, heads * d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_kv, kv_heads * d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_o, heads * d, dtype);
    if (rc == FWA_OK) rc = check_terms(a, table, buckets, columns, far, q_lengths, k_lengths, q_start, causal, scale);
    if (rc != FWA_OK) return rc;
    if (N == 0 || Lq == 0) return FWA_OK;
    if (!q || !o || (Lk > 0 && (!k || !v))) return FWA_ERR_NULL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(o) || misaligned(stats) || misaligned(workspace)) return FWA_ERR_ALIGN;
    Touched touched;
    touched.terms(a);
    touched.in(span_of(q, N, Lq, heads * d, ld_q, dtype));
    if (Lk > 0) {
        touched.in(span_of(k, N, Lk, kv_heads * d, ld_kv, dtype));
        touched.in(span_of(v, N, Lk, kv_heads * d, ld_kv, dtype));
    }
    touched.out(span_of(o, N, Lq, heads * d, ld_o, dtype));
    if (stats) touched.out(flat(stats, (uint64_t)N * heads * Lq * 8));
    if (touched.shared()) return FWA_ERR_ALIAS;
    if (!fwa::seq_forward_fits(a)) return FWA_ERR_UNSUPPORTED;
    const size_t need = fwa::seq_forward_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FWA_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.o = o; a.stats = stats;
    a.ldq = ld_q; a.ldk = ld_kv; a.ldo = ld_o;
    return fwa::launch_sequence_forward(a, workspace, static_cast<hipStream_t>(stream)) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

size_t fwa_sequence_backward_workspace_bytes(int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, int far, int dtype, int want_dtable) {
    fwa::SeqArgs a = {};
    if (check_sequence(a, N, Lq, Lk, heads, kv_heads, d, dtype) != FWA_OK || N == 0) return 0;
    if (want_dtable && (far < 0 || far > FWA_BUCKET_MAX_FAR)) return 0;
    a.far = want_dtable ? far : 0;
    return fwa::seq_backward_workspace(a, want_dtable != 0);
}

int fwa_sequence_backward(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* stats, void* dq, void* dk, void* dv,
                          float* dtable, int64_t N, int Lq, int Lk, int heads, int kv_heads, int d, float scale, int64_t ld_q, int64_t ld_kv, int64_t ld_o,
                          int64_t ld_do, int64_t ld_dq, int64_t ld_dkv, const float* table, const int32_t* buckets, int columns, int far,
                          const int32_t* q_lengths, const int32_t* k_lengths, const int32_t* q_start, int causal, int dtype, void* workspace,
                          size_t workspace_bytes, void* stream) {
    fwa::SeqArgs a = {};
    int rc = check_sequence(a, N, Lq, Lk, heads, kv_heads, d, dtype);
    if (rc != FWA_OK) return rc;
    const int C = heads * d, CK = kv_heads * d;
    for (const int64_t ld : {ld_q, ld_o, ld_do, ld_dq})
        if (rc == FWA_OK) rc = check_row_stride(ld, C, dtype);
    for (const int64_t ld : {ld_kv, ld_dkv})
        if (rc == FWA_OK) rc = check_row_stride(ld, CK, dtype);
    if (rc == FWA_OK) rc = check_terms(a, table, buckets, columns, far, q_lengths, k_lengths, q_start, causal, scale);
    if (rc != FWA_OK) return rc;
    if (dtable && !table) return FWA_ERR_NULL;
    if (misaligned(dtable)) return FWA_ERR_ALIGN;
    Touched touched;
    touched.terms(a);
    if (dtable) touched.out(flat(dtable, (uint64_t)heads * columns * 4));
    if (touched.shared()) return FWA_ERR_ALIAS;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (N == 0)  // no pairs: dtable is still overwritten
        return !dtable || fwa::launch_zero_f32(dtable, (size_t)heads * columns, st) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
    if (Lq > 0 && (!q || !o || !d_o || !stats || !dq)) return FWA_ERR_NULL;
    if (Lk > 0 && (!k || !v || !dk || !dv)) return FWA_ERR_NULL;
    if (misaligned(q) || misaligned(k) || misaligned(v) || misaligned(o) || misaligned(d_o) || misaligned(stats) || misaligned(dq) || misaligned(dk) ||
        misaligned(dv) || misaligned(workspace))
        return FWA_ERR_ALIGN;
    if (Lq > 0) {
        touched.in(span_of(q, N, Lq, C, ld_q, dtype));
        touched.in(span_of(o, N, Lq, C, ld_o, dtype));
        touched.in(span_of(d_o, N, Lq, C, ld_do, dtype));
        touched.in(flat(stats, (uint64_t)N * heads * Lq * 8));
        touched.out(span_of(dq, N, Lq, C, ld_dq, dtype));
    }
    if (Lk > 0) {
        touched.in(span_of(k, N, Lk, CK, ld_kv, dtype));
        touched.in(span_of(v, N, Lk, CK, ld_kv, dtype));
        touched.out(span_of(dk, N, Lk, CK, ld_dkv, dtype));
        touched.out(span_of(dv, N, Lk, CK, ld_dkv, dtype));
    }
    if (touched.shared()) return FWA_ERR_ALIAS;
    if (!fwa::seq_backward_fits(a)) return FWA_ERR_UNSUPPORTED;
    const size_t need = fwa::seq_backward_workspace(a, dtable != nullptr);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FWA_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.o = const_cast<void*>(o); a.d_o = d_o; a.stats = const_cast<float*>(stats);
    a.dq = dq; a.dk = dk; a.dv = dv; a.dtable = dtable;
    a.ldq = ld_q; a.ldk = ld_kv; a.ldo = ld_o; a.ldg = ld_do; a.lddq = ld_dq; a.lddk = ld_dkv;
    return fwa::launch_sequence_backward(a, workspace, st) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

}  // extern "C"
