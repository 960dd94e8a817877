// Marshalling between torch tensors and the C ABI of libfwa: argument checks, output allocation, the current stream,
// one call.  Nothing is computed here and nothing is kept from call to call.  The same steps in Python took 9 us for a
// forward and 45 us for the forward and backward of a fused qkv tensor (nine views, two dozen attribute reads, two
// calls through ctypes), more than the kernels of the smaller calls run.  The autograd nodes below are native for the
// same reason: a Python function's bookkeeping, and the interpreter that its backward has to enter from the engine's
// thread, left a training step of the smaller calls waiting for the host (stage 3 of Swin-T at batch 128: 92 us a step, 74
// as native nodes, 66 of them kernels).
//
// Each function returns the outputs, or the library's error code as an int for the Python layer to raise.
#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/utils/pybind.h>

#include <optional>
#include <string>

#include "../../include/fwa.h"

namespace py = pybind11;

namespace {

using OptTensor = std::optional<at::Tensor>;

[[noreturn]] void type_error(const std::string& s) { throw py::type_error(s); }
[[noreturn]] void value_error(const std::string& s) { throw py::value_error(s); }

int dtype_code(const at::Tensor& t) {
    switch (t.scalar_type()) {
        case at::kFloat: return FWA_F32;
        case at::kBFloat16: return FWA_BF16;
        case at::kHalf: return FWA_F16;
        default: type_error("unsupported tensor dtype");
    }
}

void need_gpu(const at::Tensor& t, const char* name) {
    if (!t.is_cuda()) type_error(std::string(name) + " must be a GPU tensor (there is no CPU path)");
}
void need_like(const at::Tensor& t, const char* name, const at::Tensor& q) {
    if (t.sizes() != q.sizes() || t.scalar_type() != q.scalar_type() || t.device() != q.device())
        value_error(std::string(name) + " must match q in shape, dtype and device");
}
const void* dense_ptr(const at::Tensor& t, const char* name, bool f32) {
    need_gpu(t, name);
    if (!t.is_contiguous()) value_error(std::string(name) + " must be contiguous");
    if (f32 && t.scalar_type() != at::kFloat) type_error(std::string(name) + " must be float32");
    return t.data_ptr();
}

// An [N, L, C] tensor whose channels are contiguous and whose token rows are evenly spaced: its device pointer and the
// row stride in elements (C when contiguous).
struct Rows {
    void* p;
    int64_t ld;
};
std::optional<int64_t> row_stride(const at::Tensor& t) {
    const int64_t N = t.size(0), L = t.size(1), C = t.size(2);
    if (t.is_contiguous()) return C;
    const int64_t s0 = t.stride(0), s1 = t.stride(1), s2 = t.stride(2);
    if ((C > 1 && s2 != 1) || (L > 1 && s1 < C) || (N > 1 && s0 != L * s1)) return std::nullopt;
    return L > 1 ? s1 : (N > 1 ? s0 : C);
}
Rows rows_of(const at::Tensor& t, const char* name, const at::Tensor* like) {
    need_gpu(t, name);
    if (t.dim() != 3) value_error(std::string(name) + " must be [N, L, C]");
    if (like) need_like(t, name, *like);
    const std::optional<int64_t> ld = row_stride(t);
    if (!ld) value_error(std::string(name) + ": channels must be contiguous and token rows evenly spaced");
    return {t.data_ptr(), *ld};
}

// The additive terms: bias [heads, L, L] fp32 or bf16, and a dense mask [nW, L, L] or int32 labels [nW, L].
struct Terms {
    const void* bias = nullptr;
    int bias_dtype = FWA_F32;
    const float* mask = nullptr;
    const int32_t* labels = nullptr;
    int nW = 0;
    bool labels_entry() const { return labels != nullptr || bias_dtype == FWA_BF16; }
};
Terms terms_of(const OptTensor& bias, const OptTensor& mask, const OptTensor& labels, int64_t heads, int64_t L) {
    Terms t;
    if (bias) {
        if (bias->dim() != 3 || bias->size(0) != heads || bias->size(1) != L || bias->size(2) != L)
            value_error("bias must be [heads, L, L]");
        if (bias->scalar_type() == at::kBFloat16) t.bias_dtype = FWA_BF16;
        t.bias = dense_ptr(*bias, "bias", t.bias_dtype == FWA_F32);
    }
    if (mask) {
        if (mask->dim() != 3 || mask->size(1) != L || mask->size(2) != L) value_error("mask must be [nW, L, L]");
        if (t.bias_dtype == FWA_BF16)
            value_error("a bf16 bias goes with a mask given as labels (or with no mask), not with a dense mask");
        if (labels) value_error("give the mask either as a dense tensor or as labels, not both");
        t.mask = static_cast<const float*>(dense_ptr(*mask, "mask", true));
        t.nW = (int)mask->size(0);
    }
    if (labels) {
        need_gpu(*labels, "labels");
        if (labels->scalar_type() != at::kInt || labels->dim() != 2 || labels->size(1) != L || !labels->is_contiguous())
            value_error("labels must be a contiguous int32 tensor [nW, L]");
        t.labels = labels->data_ptr<int32_t>();
        t.nW = (int)labels->size(0);
    }
    return t;
}

// Lets other Python threads run during a launch; the autograd engine's threads do not hold the interpreter to begin with.
struct Nogil {
    std::optional<py::gil_scoped_release> released;
    Nogil() { if (PyGILState_Check()) released.emplace(); }
};

void* stream_of(std::optional<uintptr_t> handle, const at::Tensor& t) {
    return handle ? reinterpret_cast<void*>(*handle) : static_cast<void*>(c10::hip::getCurrentHIPStream(t.device().index()).stream());
}

void need_3d(const at::Tensor& q) {
    if (q.dim() != 3) value_error("q must be [N, L, C]");
}

int call_forward(Rows q, Rows k, Rows v, Rows o, const at::Tensor& like, int64_t N, int64_t L, int64_t C, int heads, float scale,
                 const Terms& t, float mask_value, void* stream) {
    if (!(q.ld == k.ld && q.ld == v.ld)) value_error("q, k and v must share one row stride");
    const int dtype = dtype_code(like);
    const c10::DeviceGuard guard(like.device());
    const Nogil nogil;
    if (t.labels_entry())
        return fwa_forward_labels(q.p, k.p, v.p, o.p, N, (int)L, (int)C, heads, scale, q.ld, o.ld, t.bias, t.bias_dtype,
                                  t.labels, mask_value, t.nW, dtype, stream);
    return fwa_forward_strided(q.p, k.p, v.p, o.p, N, (int)L, (int)C, heads, scale, q.ld, o.ld,
                               static_cast<const float*>(t.bias), t.mask, t.nW, dtype, stream);
}

int run_forward(at::Tensor& o, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int heads, float scale, const OptTensor& bias,
                const OptTensor& mask, const OptTensor& out, std::optional<uintptr_t> stream, const OptTensor& labels, float mask_value) {
    need_3d(q);
    const int64_t N = q.size(0), L = q.size(1), C = q.size(2);
    need_gpu(q, "q");
    o = out ? *out : at::empty(q.sizes(), q.options());
    const Terms t = terms_of(bias, mask, labels, heads, L);
    return call_forward(rows_of(q, "q", nullptr), rows_of(k, "k", &q), rows_of(v, "v", &q), rows_of(o, "out", &q), q, N, L, C, heads,
                        scale, t, mask_value, stream_of(stream, q));
}
py::object forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int heads, float scale, const OptTensor& bias,
                   const OptTensor& mask, const OptTensor& out, std::optional<uintptr_t> stream, const OptTensor& labels, float mask_value) {
    at::Tensor o;
    const int rc = run_forward(o, q, k, v, heads, scale, bias, mask, out, stream, labels, mask_value);
    return rc == FWA_OK ? py::cast(o) : py::cast(rc);
}

// q, k, v as the three slices of a contiguous [N, L, 3, heads, d] tensor: slice_of relies on need_qkv
void need_qkv(const at::Tensor& qkv) {
    if (qkv.dim() != 5 || qkv.size(2) != 3 || !qkv.is_contiguous()) value_error("qkv must be a contiguous [N, L, 3, heads, d] tensor");
    need_gpu(qkv, "qkv");
}
Rows slice_of(const at::Tensor& qkv, int which) {
    const int64_t C = qkv.size(3) * qkv.size(4);
    return {static_cast<char*>(qkv.data_ptr()) + which * C * qkv.element_size(), 3 * C};
}

// The library's code, and the output where that is FWA_OK
int run_forward_qkv(at::Tensor& o, const at::Tensor& qkv, float scale, const OptTensor& bias, const OptTensor& mask, const OptTensor& labels,
                    float mask_value) {
    need_qkv(qkv);
    const int64_t N = qkv.size(0), L = qkv.size(1), heads = qkv.size(3), C = heads * qkv.size(4);
    o = at::empty({N, L, C}, qkv.options());
    const Terms t = terms_of(bias, mask, labels, heads, L);
    return call_forward(slice_of(qkv, 0), slice_of(qkv, 1), slice_of(qkv, 2), {o.data_ptr(), C}, qkv, N, L, C, (int)heads, scale, t,
                        mask_value, stream_of(std::nullopt, qkv));
}
py::object forward_qkv(const at::Tensor& qkv, float scale, const OptTensor& bias, const OptTensor& mask, const OptTensor& labels,
                       float mask_value) {
    at::Tensor o;
    const int rc = run_forward_qkv(o, qkv, scale, bias, mask, labels, mask_value);
    return rc == FWA_OK ? py::cast(o) : py::cast(rc);
}

// The workspace of a call when the caller gives none: needed for dBias, and above 64 tokens for the fp32 copy of a bf16 bias
at::Tensor workspace_for(const at::Tensor& like, int64_t N, int64_t L, int64_t C, int heads, bool want_dbias, const Terms& t) {
    if (!want_dbias && !(t.bias_dtype == FWA_BF16 && L > 64)) return at::Tensor();
    const size_t need = fwa_backward_workspace_bytes(N, (int)L, (int)C, heads, dtype_code(like), want_dbias);
    return need ? at::empty({(int64_t)need}, like.options().dtype(at::kByte)) : at::Tensor();
}

int call_backward(const Rows (&r)[7], const at::Tensor& like, const at::Tensor& dbias, int64_t N, int64_t L, int64_t C, int heads,
                  float scale, const Terms& t, float mask_value, const at::Tensor& ws, void* stream) {
    if (!(r[0].ld == r[1].ld && r[0].ld == r[2].ld)) value_error("q, k and v must share one row stride");
    if (!(r[4].ld == r[5].ld && r[4].ld == r[6].ld)) value_error("dq, dk and dv must share one row stride");
    const int dtype = dtype_code(like);
    float* const db = dbias.defined() ? dbias.data_ptr<float>() : nullptr;
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.nbytes() : 0;
    const c10::DeviceGuard guard(like.device());
    const Nogil nogil;
    if (t.labels_entry())
        return fwa_backward_labels(r[0].p, r[1].p, r[2].p, r[3].p, r[4].p, r[5].p, r[6].p, db, N, (int)L, (int)C, heads, scale,
                                   r[0].ld, r[3].ld, r[4].ld, t.bias, t.bias_dtype, t.labels, mask_value, t.nW, dtype, wp, wb, stream);
    return fwa_backward_strided(r[0].p, r[1].p, r[2].p, r[3].p, r[4].p, r[5].p, r[6].p, db, N, (int)L, (int)C, heads, scale,
                                r[0].ld, r[3].ld, r[4].ld, static_cast<const float*>(t.bias), t.mask, t.nW, dtype, wp, wb, stream);
}

at::Tensor dbias_like(const at::Tensor& q, int64_t heads, int64_t L, bool want) {
    return want ? at::empty({heads, L, L}, q.options().dtype(at::kFloat)) : at::Tensor();
}
py::object or_none(const at::Tensor& t) { return t.defined() ? py::cast(t) : py::none(); }

struct Grads {
    at::Tensor q, k, v, bias;  // of the fused tensor: q alone
};

int run_backward(Grads& d, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& d_o, int heads, float scale,
                 const OptTensor& bias, const OptTensor& mask, bool want_dbias, const OptTensor& workspace,
                 std::optional<uintptr_t> stream, const OptTensor& dq_out, const OptTensor& dk_out, const OptTensor& dv_out,
                 const OptTensor& labels, float mask_value) {
    need_3d(q);
    const int64_t N = q.size(0), L = q.size(1), C = q.size(2);
    need_gpu(q, "q");
    d.q = dq_out ? *dq_out : at::empty(q.sizes(), q.options());
    d.k = dk_out ? *dk_out : at::empty(q.sizes(), q.options());
    d.v = dv_out ? *dv_out : at::empty(q.sizes(), q.options());
    d.bias = dbias_like(q, heads, L, want_dbias);
    const Terms t = terms_of(bias, mask, labels, heads, L);
    const at::Tensor ws = workspace ? *workspace : workspace_for(q, N, L, C, heads, want_dbias, t);
    const Rows r[7] = {rows_of(q, "q", nullptr), rows_of(k, "k", &q), rows_of(v, "v", &q), rows_of(d_o, "d_o", &q),
                       rows_of(d.q, "dq", &q), rows_of(d.k, "dk", &q), rows_of(d.v, "dv", &q)};
    return call_backward(r, q, d.bias, N, L, C, heads, scale, t, mask_value, ws, stream_of(stream, q));
}
py::object backward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& d_o, int heads, float scale,
                    const OptTensor& bias, const OptTensor& mask, bool want_dbias, const OptTensor& workspace,
                    std::optional<uintptr_t> stream, const OptTensor& dq_out, const OptTensor& dk_out, const OptTensor& dv_out,
                    const OptTensor& labels, float mask_value) {
    Grads d;
    const int rc = run_backward(d, q, k, v, d_o, heads, scale, bias, mask, want_dbias, workspace, stream, dq_out, dk_out, dv_out, labels, mask_value);
    if (rc != FWA_OK) return py::cast(rc);
    return py::make_tuple(d.q, d.k, d.v, or_none(d.bias));
}

int run_backward_qkv(Grads& d, const at::Tensor& qkv, const at::Tensor& d_o, float scale, const OptTensor& bias, const OptTensor& mask,
                     bool want_dbias, const OptTensor& labels, float mask_value) {
    need_qkv(qkv);
    const int64_t N = qkv.size(0), L = qkv.size(1), heads = qkv.size(3), C = heads * qkv.size(4);
    need_gpu(d_o, "d_o");
    if (d_o.dim() != 3 || d_o.size(0) != N || d_o.size(1) != L || d_o.size(2) != C || d_o.scalar_type() != qkv.scalar_type() ||
        d_o.device() != qkv.device())
        value_error("d_o must match q in shape, dtype and device");
    d.q = at::empty(qkv.sizes(), qkv.options());
    d.bias = dbias_like(qkv, heads, L, want_dbias);
    const Terms t = terms_of(bias, mask, labels, heads, L);
    const at::Tensor ws = workspace_for(qkv, N, L, C, (int)heads, want_dbias, t);
    const Rows r[7] = {slice_of(qkv, 0), slice_of(qkv, 1), slice_of(qkv, 2), rows_of(d_o, "d_o", nullptr),
                       slice_of(d.q, 0), slice_of(d.q, 1), slice_of(d.q, 2)};
    return call_backward(r, qkv, d.bias, N, L, C, (int)heads, scale, t, mask_value, ws, stream_of(std::nullopt, qkv));
}
py::object backward_qkv(const at::Tensor& qkv, const at::Tensor& d_o, float scale, const OptTensor& bias, const OptTensor& mask,
                        bool want_dbias, const OptTensor& labels, float mask_value) {
    Grads d;
    const int rc = run_backward_qkv(d, qkv, d_o, scale, bias, mask, want_dbias, labels, mask_value);
    if (rc != FWA_OK) return py::cast(rc);
    return py::make_tuple(d.q, or_none(d.bias));
}

py::object bias_gather(const at::Tensor& table, int k, std::optional<uintptr_t> stream) {
    if (table.dim() != 2 || table.size(1) != (2LL * k - 1) * (2LL * k - 1)) value_error("table must be [heads, (2k-1)^2]");
    const float* const src = static_cast<const float*>(dense_ptr(table, "table", true));
    const at::Tensor bias = at::empty({table.size(0), (int64_t)k * k, (int64_t)k * k}, table.options());
    float* const dst = bias.data_ptr<float>();
    void* const st = stream_of(stream, table);
    int rc;
    {
        const c10::DeviceGuard guard(table.device());
        const py::gil_scoped_release nogil;
        rc = fwa_bias_gather(src, dst, (int)table.size(0), k, st);
    }
    return rc == FWA_OK ? py::cast(bias) : py::cast(rc);
}

py::object bias_scatter(const at::Tensor& dbias, int k, std::optional<uintptr_t> stream) {
    if (dbias.dim() != 3 || dbias.size(1) != (int64_t)k * k || dbias.size(2) != (int64_t)k * k)
        value_error("dbias must be [heads, k*k, k*k]");
    const float* const src = static_cast<const float*>(dense_ptr(dbias, "dbias", true));
    const at::Tensor dtable = at::empty({dbias.size(0), (2LL * k - 1) * (2LL * k - 1)}, dbias.options());
    float* const dst = dtable.data_ptr<float>();
    void* const st = stream_of(stream, dbias);
    int rc;
    {
        const c10::DeviceGuard guard(dbias.device());
        const py::gil_scoped_release nogil;
        rc = fwa_bias_scatter(src, dst, (int)dbias.size(0), k, st);
    }
    return rc == FWA_OK ? py::cast(dtable) : py::cast(rc);
}

// ------------------------------------------------------------------ bias by buckets, attention of whole sequences

void need_same_device(const at::Tensor& t, const char* name, const at::Tensor& like) {
    need_gpu(t, name);
    if (t.device() != like.device()) value_error(std::string(name) + " must be on the device of the other tensors");
}

// The map from distances to columns: contiguous int32 [2 far + 1]
struct Buckets {
    const int32_t* p;
    int far;
};
Buckets buckets_of(const at::Tensor& t, const at::Tensor& like) {
    need_same_device(t, "buckets", like);
    if (t.scalar_type() != at::kInt || t.dim() != 1 || t.size(0) % 2 != 1 || !t.is_contiguous())
        value_error("buckets must be a contiguous int32 tensor [2 far + 1]");
    if (t.size(0) > 0x7fffffff) value_error("buckets is too long");
    return {t.data_ptr<int32_t>(), (int)(t.size(0) / 2)};
}
int to_int(int64_t x, const char* name) {
    if (x < -0x7fffffff || x > 0x7fffffff) value_error(std::string(name) + " is out of range");
    return (int)x;
}

int run_bucket_gather(at::Tensor& bias, const at::Tensor& table, const at::Tensor& buckets, int64_t Lq, int64_t Lk, int64_t q_start, bool bf16,
                      const OptTensor& out, std::optional<uintptr_t> stream) {
    if (table.dim() != 2) value_error("table must be [heads, columns]");
    if (Lq < 0 || Lk < 0) value_error("Lq and Lk must not be negative");
    const float* const src = static_cast<const float*>(dense_ptr(table, "table", true));
    const Buckets b = buckets_of(buckets, table);
    const at::ScalarType type = bf16 ? at::kBFloat16 : at::kFloat;
    if (out) {
        need_same_device(*out, "out", table);
        if (out->dim() != 3 || out->size(0) != table.size(0) || out->size(1) != Lq || out->size(2) != Lk || out->scalar_type() != type || !out->is_contiguous())
            value_error("out must be a contiguous [heads, Lq, Lk] tensor of the type asked for");
    }
    bias = out ? *out : at::empty({table.size(0), Lq, Lk}, table.options().dtype(type));
    void* const dst = bias.data_ptr();
    void* const st = stream_of(stream, table);
    const c10::DeviceGuard guard(table.device());
    const Nogil nogil;
    return fwa_bucket_gather(src, b.p, dst, to_int(table.size(0), "heads"), to_int(table.size(1), "columns"), b.far, to_int(Lq, "Lq"), to_int(Lk, "Lk"), q_start,
                             bf16 ? FWA_BF16 : FWA_F32, st);
}
py::object bucket_gather(const at::Tensor& table, const at::Tensor& buckets, int64_t Lq, int64_t Lk, int64_t q_start, bool bf16, const OptTensor& out,
                         std::optional<uintptr_t> stream) {
    at::Tensor bias;
    const int rc = run_bucket_gather(bias, table, buckets, Lq, Lk, q_start, bf16, out, stream);
    return rc == FWA_OK ? py::cast(bias) : py::cast(rc);
}

int run_bucket_scatter(at::Tensor& dtable, const at::Tensor& dbias, const at::Tensor& buckets, int64_t columns, int64_t q_start, const OptTensor& workspace,
                       std::optional<uintptr_t> stream) {
    if (dbias.dim() != 3) value_error("dbias must be [heads, Lq, Lk]");
    if (columns < 1) value_error("columns must be positive");
    const float* const src = static_cast<const float*>(dense_ptr(dbias, "dbias", true));
    const Buckets b = buckets_of(buckets, dbias);
    const int heads = to_int(dbias.size(0), "heads"), Lq = to_int(dbias.size(1), "Lq"), Lk = to_int(dbias.size(2), "Lk"), nb = to_int(columns, "columns");
    dtable = at::empty({dbias.size(0), columns}, dbias.options());
    const size_t need = fwa_bucket_scatter_workspace_bytes(heads, nb, b.far, Lq, Lk);
    if (workspace) need_same_device(*workspace, "workspace", dbias);
    const at::Tensor ws = workspace ? *workspace : need ? at::empty({(int64_t)need}, dbias.options().dtype(at::kByte)) : at::Tensor();
    float* const dst = dtable.data_ptr<float>();
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.nbytes() : 0;
    void* const st = stream_of(stream, dbias);
    const c10::DeviceGuard guard(dbias.device());
    const Nogil nogil;
    return fwa_bucket_scatter(src, b.p, dst, heads, nb, b.far, Lq, Lk, q_start, wp, wb, st);
}
py::object bucket_scatter(const at::Tensor& dbias, const at::Tensor& buckets, int64_t columns, int64_t q_start, const OptTensor& workspace,
                          std::optional<uintptr_t> stream) {
    at::Tensor dtable;
    const int rc = run_bucket_scatter(dtable, dbias, buckets, columns, q_start, workspace, stream);
    return rc == FWA_OK ? py::cast(dtable) : py::cast(rc);
}

// What the calls of a sequence attention have in common, besides the tensors of their directions.
struct Sequence {
    int64_t N, Lq, Lk;
    int heads, kv_heads, d, dtype;
    float scale;
    const float* table = nullptr;
    const int32_t* buckets = nullptr;
    int columns = 0, far = 0;
    const int32_t *q_lengths = nullptr, *k_lengths = nullptr, *q_start = nullptr;
    int causal;
};
const int32_t* per_sequence(const OptTensor& t, const char* name, const at::Tensor& q) {
    if (!t) return nullptr;
    need_same_device(*t, name, q);
    if (t->scalar_type() != at::kInt || t->dim() != 1 || t->size(0) != q.size(0) || !t->is_contiguous())
        value_error(std::string(name) + " must be a contiguous int32 tensor [N]");
    return t->data_ptr<int32_t>();
}
Sequence sequence_of(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int64_t heads, double scale, const OptTensor& table, const OptTensor& buckets,
                     const OptTensor& q_lengths, const OptTensor& k_lengths, const OptTensor& q_start, bool causal) {
    need_gpu(q, "q");
    if (q.dim() != 3) value_error("q must be [N, Lq, heads * d]");
    if (heads < 1 || q.size(2) % heads != 0 || q.size(2) == 0) value_error("the channels of q must be a multiple of heads");
    Sequence s;
    s.N = q.size(0);
    s.Lq = to_int(q.size(1), "Lq");
    s.heads = to_int(heads, "heads");
    s.d = to_int(q.size(2) / heads, "d");
    for (const auto& t : {std::make_pair(&k, "k"), std::make_pair(&v, "v")}) {
        need_same_device(*t.first, t.second, q);
        if (t.first->dim() != 3 || t.first->size(0) != s.N || t.first->scalar_type() != q.scalar_type())
            value_error(std::string(t.second) + " must be [N, Lk, kv_heads * d] of the type of q");
    }
    if (v.sizes() != k.sizes()) value_error("k and v must have one shape");
    if (k.size(2) == 0 || k.size(2) % s.d != 0 || heads % (k.size(2) / s.d) != 0) value_error("the channels of k must be kv_heads * d, kv_heads a divisor of heads");
    s.Lk = to_int(k.size(1), "Lk");
    s.kv_heads = (int)(k.size(2) / s.d);
    s.dtype = dtype_code(q);
    s.scale = (float)scale;
    s.causal = causal;
    if (table.has_value() != buckets.has_value()) value_error("table and buckets go together");
    if (table) {
        if (table->dim() != 2 || table->size(0) != heads) value_error("table must be [heads, columns]");
        s.table = static_cast<const float*>(dense_ptr(*table, "table", true));
        need_same_device(*table, "table", q);
        const Buckets b = buckets_of(*buckets, q);
        s.buckets = b.p;
        s.far = b.far;
        s.columns = to_int(table->size(1), "columns");
    }
    s.q_lengths = per_sequence(q_lengths, "q_lengths", q);
    s.k_lengths = per_sequence(k_lengths, "k_lengths", q);
    s.q_start = per_sequence(q_start, "q_start", q);
    return s;
}
at::Tensor scratch(size_t bytes, const at::Tensor& like) {
    return bytes ? at::empty({(int64_t)bytes}, like.options().dtype(at::kByte)) : at::Tensor();
}
void need_one_stride(const Rows& k, const Rows& v, const char* names, int64_t N, int64_t L) {
    if (k.ld != v.ld && N * L > 1) value_error(std::string(names) + " must share one row stride");
}

int run_sequence_forward(at::Tensor& o, at::Tensor& stats, bool want_stats, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int64_t heads, double scale,
                         const OptTensor& table, const OptTensor& buckets, const OptTensor& q_lengths, const OptTensor& k_lengths, const OptTensor& q_start,
                         bool causal, const OptTensor& out, const OptTensor& workspace, std::optional<uintptr_t> stream) {
    const Sequence s = sequence_of(q, k, v, heads, scale, table, buckets, q_lengths, k_lengths, q_start, causal);
    o = out ? *out : at::empty(q.sizes(), q.options());
    if (want_stats) stats = at::empty({s.N, heads, s.Lq, 2}, q.options().dtype(at::kFloat));
    const Rows rq = rows_of(q, "q", nullptr), rk = rows_of(k, "k", nullptr), rv = rows_of(v, "v", nullptr), ro = rows_of(o, "out", &q);
    need_one_stride(rk, rv, "k and v", s.N, s.Lk);
    if (workspace) need_same_device(*workspace, "workspace", q);
    const at::Tensor ws = workspace ? *workspace
                                    : scratch(fwa_sequence_forward_workspace_bytes(s.N, (int)s.Lq, (int)s.Lk, s.heads, s.kv_heads, s.d, s.dtype), q);
    float* const sp = stats.defined() ? stats.data_ptr<float>() : nullptr;
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.nbytes() : 0;
    void* const st = stream_of(stream, q);
    const c10::DeviceGuard guard(q.device());
    const Nogil nogil;
    return fwa_sequence_forward(rq.p, rk.p, rv.p, ro.p, sp, s.N, (int)s.Lq, (int)s.Lk, s.heads, s.kv_heads, s.d, s.scale, rq.ld, rk.ld, ro.ld, s.table, s.buckets,
                                s.columns, s.far, s.q_lengths, s.k_lengths, s.q_start, s.causal, s.dtype, wp, wb, st);
}
py::object sequence_forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int64_t heads, double scale, const OptTensor& table,
                            const OptTensor& buckets, const OptTensor& q_lengths, const OptTensor& k_lengths, const OptTensor& q_start, bool causal,
                            bool want_stats, const OptTensor& out, const OptTensor& workspace, std::optional<uintptr_t> stream) {
    at::Tensor o, stats;
    const int rc = run_sequence_forward(o, stats, want_stats, q, k, v, heads, scale, table, buckets, q_lengths, k_lengths, q_start, causal, out, workspace, stream);
    if (rc != FWA_OK) return py::cast(rc);
    if (want_stats) return py::make_tuple(o, stats);
    return py::cast(o);
}

int run_sequence_backward(Grads& d, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& o, const at::Tensor& stats, const at::Tensor& d_o,
                          int64_t heads, double scale, const OptTensor& table, const OptTensor& buckets, const OptTensor& q_lengths, const OptTensor& k_lengths,
                          const OptTensor& q_start, bool causal, bool want_dtable, const OptTensor& dq_out, const OptTensor& dk_out, const OptTensor& dv_out,
                          const OptTensor& workspace, std::optional<uintptr_t> stream) {
    const Sequence s = sequence_of(q, k, v, heads, scale, table, buckets, q_lengths, k_lengths, q_start, causal);
    if (want_dtable && !table) value_error("the gradient of a table needs the table");
    need_same_device(stats, "stats", q);
    if (stats.scalar_type() != at::kFloat || stats.dim() != 4 || stats.size(0) != s.N || stats.size(1) != heads || stats.size(2) != s.Lq || stats.size(3) != 2 ||
        !stats.is_contiguous())
        value_error("stats must be the contiguous float32 tensor [N, heads, Lq, 2] of the forward");
    d.q = dq_out ? *dq_out : at::empty(q.sizes(), q.options());
    d.k = dk_out ? *dk_out : at::empty(k.sizes(), k.options());
    d.v = dv_out ? *dv_out : at::empty(v.sizes(), v.options());
    if (want_dtable) d.bias = at::empty({heads, (int64_t)s.columns}, q.options().dtype(at::kFloat));
    const Rows rq = rows_of(q, "q", nullptr), rk = rows_of(k, "k", nullptr), rv = rows_of(v, "v", nullptr), ro = rows_of(o, "o", &q), rg = rows_of(d_o, "d_o", &q);
    const Rows rdq = rows_of(d.q, "dq", &q), rdk = rows_of(d.k, "dk", nullptr), rdv = rows_of(d.v, "dv", nullptr);
    for (const auto& t : {std::make_pair(&d.k, "dk"), std::make_pair(&d.v, "dv")})
        if (t.first->sizes() != k.sizes() || t.first->scalar_type() != k.scalar_type() || t.first->device() != k.device())
            value_error(std::string(t.second) + " must match k in shape, dtype and device");
    need_one_stride(rk, rv, "k and v", s.N, s.Lk);
    need_one_stride(rdk, rdv, "dk and dv", s.N, s.Lk);
    if (workspace) need_same_device(*workspace, "workspace", q);
    const at::Tensor ws = workspace ? *workspace
                                    : scratch(fwa_sequence_backward_workspace_bytes(s.N, (int)s.Lq, (int)s.Lk, s.heads, s.kv_heads, s.d, s.far, s.dtype, want_dtable), q);
    float* const dt = d.bias.defined() ? d.bias.data_ptr<float>() : nullptr;
    const float* const sp = stats.data_ptr<float>();
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.nbytes() : 0;
    void* const st = stream_of(stream, q);
    const c10::DeviceGuard guard(q.device());
    const Nogil nogil;
    return fwa_sequence_backward(rq.p, rk.p, rv.p, ro.p, rg.p, sp, rdq.p, rdk.p, rdv.p, dt, s.N, (int)s.Lq, (int)s.Lk, s.heads, s.kv_heads, s.d, s.scale, rq.ld, rk.ld,
                                 ro.ld, rg.ld, rdq.ld, rdk.ld, s.table, s.buckets, s.columns, s.far, s.q_lengths, s.k_lengths, s.q_start, s.causal, s.dtype, wp, wb, st);
}
py::object sequence_backward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& o, const at::Tensor& stats, const at::Tensor& d_o,
                             int64_t heads, double scale, const OptTensor& table, const OptTensor& buckets, const OptTensor& q_lengths, const OptTensor& k_lengths,
                             const OptTensor& q_start, bool causal, bool want_dtable, const OptTensor& dq_out, const OptTensor& dk_out, const OptTensor& dv_out,
                             const OptTensor& workspace, std::optional<uintptr_t> stream) {
    Grads d;
    const int rc = run_sequence_backward(d, q, k, v, o, stats, d_o, heads, scale, table, buckets, q_lengths, k_lengths, q_start, causal, want_dtable, dq_out, dk_out,
                                         dv_out, workspace, stream);
    if (rc != FWA_OK) return py::cast(rc);
    return py::make_tuple(d.q, d.k, d.v, or_none(d.bias));
}

// ------------------------------------------------------------------ rotary positions, paged cache

// Rows of [N, L, C], or of packed [T, C]
Rows any_rows_of(const at::Tensor& t, const char* name, const at::Tensor* like) {
    need_gpu(t, name);
    if (t.dim() == 3) return rows_of(t, name, like);
    if (t.dim() != 2) value_error(std::string(name) + " must be [N, L, C] or [T, C]");
    if (like) need_like(t, name, *like);
    const int64_t T = t.size(0), C = t.size(1);
    if (t.is_contiguous()) return {t.data_ptr(), C};
    if ((C > 1 && t.stride(1) != 1) || (T > 1 && t.stride(0) < C)) value_error(std::string(name) + ": channels must be contiguous and token rows evenly spaced");
    return {t.data_ptr(), T > 1 ? t.stride(0) : C};
}

// The rotation's tables
struct Rotation {
    const int32_t* positions = nullptr;
    const float* frequencies = nullptr;
    const int32_t* axis_of = nullptr;
    int axes = 1, pairs = 0;
};
Rotation rotation_of(const OptTensor& positions, const OptTensor& frequencies, const OptTensor& axis_of, const at::Tensor& like) {
    Rotation r;
    if (!frequencies) {
        if (positions || axis_of) value_error("positions and axis_of go with frequencies");
        return r;
    }
    need_same_device(*frequencies, "frequencies", like);
    if (frequencies->scalar_type() != at::kFloat || frequencies->dim() != 1 || !frequencies->is_contiguous())
        value_error("frequencies must be a contiguous float32 tensor [pairs]");
    r.frequencies = frequencies->data_ptr<float>();
    r.pairs = to_int(frequencies->size(0), "pairs");
    if (positions) {
        need_same_device(*positions, "positions", like);
        if (positions->scalar_type() != at::kInt || positions->dim() < 2 || !positions->is_contiguous())
            value_error("positions must be a contiguous int32 tensor with the axes last");
        r.positions = positions->data_ptr<int32_t>();
        r.axes = to_int(positions->size(-1), "axes");
    }
    if (axis_of) {
        need_same_device(*axis_of, "axis_of", like);
        if (axis_of->scalar_type() != at::kInt || axis_of->dim() != 1 || axis_of->size(0) != frequencies->size(0) || !axis_of->is_contiguous())
            value_error("axis_of must be a contiguous int32 tensor [pairs]");
        r.axis_of = axis_of->data_ptr<int32_t>();
    }
    return r;
}

int run_rotary(at::Tensor& y, const at::Tensor& x, int64_t heads, const at::Tensor& positions, const at::Tensor& frequencies, const OptTensor& axis_of, bool interleaved,
               bool inverse, const OptTensor& out, std::optional<uintptr_t> stream) {
    need_gpu(x, "x");
    if (x.dim() != 2 && x.dim() != 3) value_error("x must be [N, L, heads * d] or [T, heads * d]");
    if (heads < 1 || x.size(-1) == 0 || x.size(-1) % heads != 0) value_error("the channels of x must be a multiple of heads");
    const Rotation r = rotation_of(positions, frequencies, axis_of, x);
    const bool shared = positions.dim() == 2;
    if (positions.dim() > x.dim() || positions.size(-2) != x.size(-2) || (!shared && positions.size(0) != x.size(0)))
        value_error("positions must be [L, axes] or [N, L, axes], of packed rows [T, axes]");
    const int64_t rows = x.dim() == 3 ? x.size(0) * x.size(1) : x.size(0);
    const Rows rx = any_rows_of(x, "x", nullptr);
    y = out ? *out : at::empty(x.sizes(), x.options());
    const Rows ry = any_rows_of(y, "out", &x);
    if (rows == 0) return FWA_OK;
    const int dtype = dtype_code(x);
    void* const st = stream_of(stream, x);
    const c10::DeviceGuard guard(x.device());
    const Nogil nogil;
    return fwa_rotary(rx.p, ry.p, rows, to_int(heads, "heads"), to_int(x.size(-1) / heads, "d"), rx.ld, ry.ld, r.positions, shared ? positions.size(0) : rows, r.axes,
                      r.frequencies, r.axis_of, r.pairs, interleaved, inverse, dtype, st);
}
py::object rotary(const at::Tensor& x, int64_t heads, const at::Tensor& positions, const at::Tensor& frequencies, const OptTensor& axis_of, bool interleaved, bool inverse,
                  const OptTensor& out, std::optional<uintptr_t> stream) {
    at::Tensor y;
    const int rc = run_rotary(y, x, heads, positions, frequencies, axis_of, interleaved, inverse, out, stream);
    return rc == FWA_OK ? py::cast(y) : py::cast(rc);
}

// Cache and tables of a call with packed rows
struct Pages {
    void *k, *v;
    int64_t N, rows, pages, page_stride, token_stride, head_stride;
    int kv_heads, d, page_size, width;
    const int32_t *table, *offsets, *lengths;
};
Pages pages_of(const at::Tensor& like, const char* name, const at::Tensor& k_pages, const at::Tensor& v_pages, const at::Tensor& page_table, const at::Tensor& offsets,
               const at::Tensor& lengths) {
    need_gpu(like, name);
    if (like.dim() != 2) value_error(std::string(name) + " must be packed rows [T, channels]");
    for (const auto& t : {std::make_pair(&k_pages, "k_pages"), std::make_pair(&v_pages, "v_pages")}) {
        need_same_device(*t.first, t.second, like);
        if (t.first->dim() != 4 || t.first->scalar_type() != like.scalar_type())
            value_error(std::string(t.second) + " must be [pages, page_size, kv_heads, d] of the type of " + name);
        if (t.first->size(3) > 1 && t.first->stride(3) != 1) value_error(std::string(t.second) + ": channels must be contiguous");
    }
    if (k_pages.sizes() != v_pages.sizes()) value_error("k_pages and v_pages must have one shape");
    for (int i = 0; i < 3; ++i)
        if (k_pages.size(i) > 1 && k_pages.stride(i) != v_pages.stride(i)) value_error("k_pages and v_pages must share their strides");
    for (const auto& t : {std::make_pair(&page_table, "page_table"), std::make_pair(&offsets, "offsets"), std::make_pair(&lengths, "lengths")}) {
        need_same_device(*t.first, t.second, like);
        if (t.first->scalar_type() != at::kInt || !t.first->is_contiguous()) value_error(std::string(t.second) + " must be a contiguous int32 tensor");
    }
    if (lengths.dim() != 1) value_error("lengths must be [N]");
    Pages p;
    p.N = lengths.size(0);
    if (offsets.dim() != 1 || offsets.size(0) != p.N + 1) value_error("offsets must be [N + 1]");
    if (page_table.dim() != 2 || page_table.size(0) != p.N) value_error("page_table must be [N, width]");
    p.rows = like.size(0);
    p.pages = k_pages.size(0);
    p.page_size = to_int(k_pages.size(1), "page_size");
    p.kv_heads = to_int(k_pages.size(2), "kv_heads");
    p.d = to_int(k_pages.size(3), "d");
    p.width = to_int(page_table.size(1), "width");
    // a stride that no element needs may be anything
    p.head_stride = p.kv_heads > 1 ? k_pages.stride(2) : p.d;
    p.token_stride = p.page_size > 1 ? k_pages.stride(1) : p.d;
    p.page_stride = p.pages > 1 ? k_pages.stride(0) : 0;
    p.k = k_pages.data_ptr();
    p.v = v_pages.data_ptr();
    p.table = page_table.data_ptr<int32_t>();
    p.offsets = offsets.data_ptr<int32_t>();
    p.lengths = lengths.data_ptr<int32_t>();
    return p;
}

py::object page_append(const at::Tensor& k, const at::Tensor& v, const at::Tensor& k_pages, const at::Tensor& v_pages, const at::Tensor& page_table,
                       const at::Tensor& offsets, const at::Tensor& lengths, const OptTensor& frequencies, const OptTensor& positions, const OptTensor& axis_of,
                       bool interleaved, const OptTensor& q, const OptTensor& q_out, std::optional<uintptr_t> stream) {
    const Pages p = pages_of(k, "k", k_pages, v_pages, page_table, offsets, lengths);
    const Rows rk = any_rows_of(k, "k", nullptr), rv = any_rows_of(v, "v", &k);
    if (p.d < 1 || k.size(1) != (int64_t)p.kv_heads * p.d) value_error("the channels of k must be kv_heads * d");
    const Rotation r = rotation_of(positions, frequencies, axis_of, k);
    if (positions && (positions->dim() != 2 || positions->size(0) != p.rows)) value_error("positions must be [T, axes]");
    if (q_out && !q) value_error("q_out goes with q");
    at::Tensor y;
    Rows rq = {nullptr, 0}, ry = {nullptr, 0};
    int64_t heads = 0;
    if (q) {
        need_same_device(*q, "q", k);
        if (q->dim() != 2 || q->size(0) != p.rows || q->scalar_type() != k.scalar_type() || q->size(1) == 0 || q->size(1) % p.d != 0)
            value_error("q must be [T, heads * d] of the type of k");
        heads = q->size(1) / p.d;
        rq = any_rows_of(*q, "q", nullptr);
        y = q_out ? *q_out : at::empty(q->sizes(), q->options());
        ry = any_rows_of(y, "q_out", &*q);
    }
    const int dtype = dtype_code(k);
    void* const st = stream_of(stream, k);
    int rc;
    {
        const c10::DeviceGuard guard(k.device());
        const Nogil nogil;
        rc = fwa_page_append(rk.p, rv.p, p.k, p.v, p.rows, p.N, p.kv_heads, p.d, rk.ld, rv.ld, p.pages, p.page_size, p.page_stride, p.token_stride, p.head_stride, p.table,
                             p.width, p.offsets, p.lengths, r.positions, r.axes, r.frequencies, r.axis_of, r.pairs, interleaved, p.rows ? rq.p : nullptr, ry.p, (int)heads,
                             rq.ld, ry.ld, dtype, st);
    }
    if (rc != FWA_OK) return py::cast(rc);
    return or_none(y);
}

py::object page_forward(const at::Tensor& q, const at::Tensor& k_pages, const at::Tensor& v_pages, const at::Tensor& page_table, const at::Tensor& offsets,
                        const at::Tensor& lengths, int64_t heads, double scale, int64_t most_new, bool causal, bool want_stats, const OptTensor& out,
                        const OptTensor& workspace, std::optional<uintptr_t> stream) {
    const Pages p = pages_of(q, "q", k_pages, v_pages, page_table, offsets, lengths);
    if (heads < 1 || p.kv_heads < 1 || heads % p.kv_heads != 0 || q.size(1) != heads * p.d)
        value_error("the channels of q must be heads * d, heads a multiple of kv_heads");
    const Rows rq = any_rows_of(q, "q", nullptr);
    const at::Tensor o = out ? *out : at::empty(q.sizes(), q.options());
    const Rows ro = any_rows_of(o, "out", &q);
    at::Tensor stats;
    if (want_stats) stats = at::empty({p.rows, heads, 2}, q.options().dtype(at::kFloat));
    const int dtype = dtype_code(q), H = to_int(heads, "heads"), most = to_int(most_new < 0 || most_new > p.rows ? p.rows : most_new, "most_new");
    const c10::DeviceGuard guard(q.device());
    if (workspace) need_same_device(*workspace, "workspace", q);
    const at::Tensor ws = workspace ? *workspace : scratch(fwa_page_forward_workspace_bytes(p.rows, p.N, H, p.kv_heads, p.d, p.page_size, p.width, most, dtype), q);
    float* const sp = stats.defined() ? stats.data_ptr<float>() : nullptr;
    void* const wp = ws.defined() ? ws.data_ptr() : nullptr;
    const size_t wb = ws.defined() ? (size_t)ws.nbytes() : 0;
    void* const st = stream_of(stream, q);
    int rc;
    {
        const Nogil nogil;
        rc = fwa_page_forward(rq.p, p.k, p.v, ro.p, sp, p.rows, p.N, H, p.kv_heads, p.d, (float)scale, rq.ld, ro.ld, p.pages, p.page_size, p.page_stride, p.token_stride,
                              p.head_stride, p.table, p.width, p.offsets, p.lengths, most, causal, dtype, wp, wb, st);
    }
    if (rc != FWA_OK) return py::cast(rc);
    if (want_stats) return py::make_tuple(o, stats);
    return py::cast(o);
}

// ------------------------------------------------------------------ autograd
// The two differentiable calls as native nodes.  What they save goes through the engine's saved variables (version counters,
// saved-tensor hooks); an error in the backward reaches Python as the exception that the direct call raises.
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

OptTensor opt(const at::Tensor& t) { return t.defined() ? OptTensor(t) : OptTensor(); }
at::Tensor or_undefined(const OptTensor& t) { return t ? *t : at::Tensor(); }

// a contiguous tensor at an address that the library takes: the gradient of a part of a larger tensor may start at any of its elements
at::Tensor aligned(const at::Tensor& t) {
    const at::Tensor c = t.contiguous();
    return reinterpret_cast<uintptr_t>(c.data_ptr()) & 15u ? c.clone() : c;
}

std::string entry_name(const char* what, const OptTensor& bias, const OptTensor& labels) {
    return std::string(what) + (labels || (bias && bias->scalar_type() == at::kBFloat16) ? "_labels" : "_strided");
}

// `body`, with whatever it raises left as a Python error that may cross the engine's threads
template <class Body>
variable_list with_python_errors(Body body) {
    try {
        return body();
    } catch (py::builtin_exception& e) {
        const py::gil_scoped_acquire gil;
        e.set_error();
        python_error err;
        err.persist();
        throw err;
    }
}
[[noreturn]] void raise_status(int rc, const std::string& entry) {
    const py::gil_scoped_acquire gil;
    const py::object type = py::module_::import("paper_2501_06480_amd.binding").attr("FwaError");
    PyErr_SetObject(type.ptr(), type(rc, entry).ptr());
    python_error err;
    err.persist();
    throw err;
}

// a gradient of the bias that this shape and type do not have is refused in front of the forward
void need_dbias(const at::Tensor& q, int64_t N, int64_t L, int64_t C, int64_t heads, const OptTensor& bias) {
    if (!bias || !bias->requires_grad() || N == 0) return;
    if (fwa_backward_workspace_bytes(N, (int)L, (int)C, (int)heads, dtype_code(q), 1) != 0) return;
    PyErr_SetString(PyExc_NotImplementedError, "the gradient of the bias is not available for this shape and dtype");
    throw py::error_already_set();
}

struct Attention : torch::autograd::Function<Attention> {
    static at::Tensor forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const OptTensor& bias,
                              const OptTensor& mask, const OptTensor& labels, int64_t heads, double scale, double mask_value) {
        ctx->save_for_backward({q, k, v, or_undefined(bias), or_undefined(mask), or_undefined(labels)});
        ctx->saved_data["heads"] = heads;
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["mask_value"] = mask_value;
        at::Tensor o;
        const int rc = run_forward(o, q, k, v, (int)heads, (float)scale, bias, mask, std::nullopt, std::nullopt, labels, (float)mask_value);
        if (rc != FWA_OK) raise_status(rc, entry_name("fwa_forward", bias, labels));
        return o;
    }
    static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
        return with_python_errors([&]() -> variable_list {
            const variable_list s = ctx->get_saved_variables();
            Grads d;
            const int rc = run_backward(d, s[0], s[1], s[2], grads[0].contiguous(), (int)ctx->saved_data["heads"].toInt(),
                                        (float)ctx->saved_data["scale"].toDouble(), opt(s[3]), opt(s[4]), s[3].defined() && ctx->needs_input_grad(3),
                                        std::nullopt, std::nullopt, std::nullopt, std::nullopt, std::nullopt, opt(s[5]),
                                        (float)ctx->saved_data["mask_value"].toDouble());
            if (rc != FWA_OK) raise_status(rc, entry_name("fwa_backward", opt(s[3]), opt(s[5])));
            return {d.q, d.k, d.v, d.bias, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};
struct AttentionQKV : torch::autograd::Function<AttentionQKV> {
    static at::Tensor forward(AutogradContext* ctx, const at::Tensor& qkv, const OptTensor& bias, const OptTensor& mask,
                              const OptTensor& labels, double scale, double mask_value) {
        ctx->save_for_backward({qkv, or_undefined(bias), or_undefined(mask), or_undefined(labels)});
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["mask_value"] = mask_value;
        at::Tensor o;
        const int rc = run_forward_qkv(o, qkv, (float)scale, bias, mask, labels, (float)mask_value);
        if (rc != FWA_OK) raise_status(rc, entry_name("fwa_forward", bias, labels));
        return o;
    }
    static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
        return with_python_errors([&]() -> variable_list {
            const variable_list s = ctx->get_saved_variables();
            Grads d;
            // a saved-tensor hook may have handed the fused tensor back in another layout
            const int rc = run_backward_qkv(d, s[0].contiguous(), grads[0].contiguous(), (float)ctx->saved_data["scale"].toDouble(), opt(s[1]), opt(s[2]),
                                            s[1].defined() && ctx->needs_input_grad(1), opt(s[3]), (float)ctx->saved_data["mask_value"].toDouble());
            if (rc != FWA_OK) raise_status(rc, entry_name("fwa_backward", opt(s[1]), opt(s[3])));
            return {d.q, d.bias, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};

at::Tensor attention(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int heads, double scale, const OptTensor& bias,
                     const OptTensor& mask, const OptTensor& labels, double mask_value) {
    need_3d(q);
    need_dbias(q, q.size(0), q.size(1), q.size(2), heads, bias);
    return Attention::apply(q, k, v, bias, mask, labels, (int64_t)heads, scale, mask_value);
}
at::Tensor attention_qkv(const at::Tensor& qkv, double scale, const OptTensor& bias, const OptTensor& mask, const OptTensor& labels, double mask_value) {
    need_qkv(qkv);
    need_dbias(qkv, qkv.size(0), qkv.size(1), qkv.size(3) * qkv.size(4), qkv.size(3), bias);
    return AttentionQKV::apply(qkv, bias, mask, labels, scale, mask_value);
}

struct BucketBias : torch::autograd::Function<BucketBias> {
    static at::Tensor forward(AutogradContext* ctx, const at::Tensor& table, const at::Tensor& buckets, int64_t Lq, int64_t Lk, int64_t q_start, bool bf16) {
        ctx->save_for_backward({buckets});
        ctx->saved_data["columns"] = table.dim() == 2 ? table.size(1) : 0;
        ctx->saved_data["q_start"] = q_start;
        at::Tensor bias;
        const int rc = run_bucket_gather(bias, table, buckets, Lq, Lk, q_start, bf16, std::nullopt, std::nullopt);
        if (rc != FWA_OK) raise_status(rc, "fwa_bucket_gather");
        return bias;
    }
    static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
        return with_python_errors([&]() -> variable_list {
            const variable_list s = ctx->get_saved_variables();
            at::Tensor dtable;
            const int rc = run_bucket_scatter(dtable, aligned(grads[0].to(at::kFloat)), s[0].contiguous(), ctx->saved_data["columns"].toInt(),
                                              ctx->saved_data["q_start"].toInt(), std::nullopt, std::nullopt);
            if (rc != FWA_OK) raise_status(rc, "fwa_bucket_scatter");
            return {dtable, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};
// Saved tensors may come back from a hook in another layout, or at another address, than they were saved in: those the call does not take are copied.
at::Tensor saved_rows(const at::Tensor& t) {
    const std::optional<int64_t> ld = row_stride(t);
    return ld && (*ld * t.element_size()) % 16 == 0 && (reinterpret_cast<uintptr_t>(t.data_ptr()) & 15u) == 0 ? t : aligned(t);
}
struct SequenceAttention : torch::autograd::Function<SequenceAttention> {
    static at::Tensor forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const OptTensor& table, const OptTensor& buckets,
                              const OptTensor& q_lengths, const OptTensor& k_lengths, const OptTensor& q_start, int64_t heads, double scale, bool causal) {
        at::Tensor o, stats;
        const int rc = run_sequence_forward(o, stats, true, q, k, v, heads, scale, table, buckets, q_lengths, k_lengths, q_start, causal, std::nullopt, std::nullopt,
                                            std::nullopt);
        if (rc != FWA_OK) raise_status(rc, "fwa_sequence_forward");
        ctx->save_for_backward({q, k, v, o, stats, or_undefined(table), or_undefined(buckets), or_undefined(q_lengths), or_undefined(k_lengths), or_undefined(q_start)});
        ctx->saved_data["heads"] = heads;
        ctx->saved_data["scale"] = scale;
        ctx->saved_data["causal"] = causal;
        return o;
    }
    static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
        return with_python_errors([&]() -> variable_list {
            const variable_list s = ctx->get_saved_variables();
            const auto dense = [&](int i) { return s[i].defined() ? OptTensor(aligned(s[i])) : OptTensor(); };
            at::Tensor k = saved_rows(s[1]), v = saved_rows(s[2]);
            if (row_stride(k) != row_stride(v)) {
                k = aligned(k);  // one stride for both
                v = aligned(v);
            }
            Grads d;
            const int rc = run_sequence_backward(d, saved_rows(s[0]), k, v, saved_rows(s[3]), aligned(s[4]), aligned(grads[0]), ctx->saved_data["heads"].toInt(),
                                                 ctx->saved_data["scale"].toDouble(), dense(5), dense(6), dense(7), dense(8), dense(9),
                                                 ctx->saved_data["causal"].toBool(), s[5].defined() && ctx->needs_input_grad(3), std::nullopt, std::nullopt,
                                                 std::nullopt, std::nullopt, std::nullopt);
            if (rc != FWA_OK) raise_status(rc, "fwa_sequence_backward");
            return {d.q, d.k, d.v, d.bias, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};
at::Tensor bucket_bias(const at::Tensor& table, const at::Tensor& buckets, int64_t Lq, int64_t Lk, int64_t q_start, bool bf16) {
    return BucketBias::apply(table, buckets, Lq, Lk, q_start, bf16);
}
at::Tensor sequence_attention(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, int64_t heads, double scale, const OptTensor& table,
                              const OptTensor& buckets, const OptTensor& q_lengths, const OptTensor& k_lengths, const OptTensor& q_start, bool causal) {
    return SequenceAttention::apply(q, k, v, table, buckets, q_lengths, k_lengths, q_start, heads, scale, causal);
}

struct Rotary : torch::autograd::Function<Rotary> {
    static at::Tensor forward(AutogradContext* ctx, const at::Tensor& x, const at::Tensor& positions, const at::Tensor& frequencies, const OptTensor& axis_of, int64_t heads,
                              bool interleaved, bool inverse) {
        ctx->save_for_backward({positions, frequencies, or_undefined(axis_of)});
        ctx->saved_data["call"] = 4 * heads + 2 * interleaved + inverse;
        at::Tensor y;
        const int rc = run_rotary(y, x, heads, positions, frequencies, axis_of, interleaved, inverse, std::nullopt, std::nullopt);
        if (rc != FWA_OK) raise_status(rc, "fwa_rotary");
        return y;
    }
    static variable_list backward(AutogradContext* ctx, const variable_list& grads) {
        return with_python_errors([&]() -> variable_list {
            const variable_list s = ctx->get_saved_variables();
            const int64_t call = ctx->saved_data["call"].toInt();
            const at::Tensor dy = aligned(grads[0]), positions = s[0].contiguous(), frequencies = s[1].contiguous();
            const OptTensor axis_of = s[2].defined() ? OptTensor(s[2].contiguous()) : OptTensor();
            at::Tensor dx;
            if (at::GradMode::is_enabled() && dy.requires_grad()) {  // a gradient that is to be differentiated again
                dx = Rotary::apply(dy, positions, frequencies, axis_of, call / 4, (call & 2) != 0, (call & 1) == 0);
            } else {
                const int rc = run_rotary(dx, dy, call / 4, positions, frequencies, axis_of, (call & 2) != 0, (call & 1) == 0, std::nullopt, std::nullopt);
                if (rc != FWA_OK) raise_status(rc, "fwa_rotary");
            }
            return {dx, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};
at::Tensor rotary_node(const at::Tensor& x, int64_t heads, const at::Tensor& positions, const at::Tensor& frequencies, const OptTensor& axis_of, bool interleaved,
                       bool inverse) {
    return Rotary::apply(x, positions, frequencies, axis_of, heads, interleaved, inverse);
}

}  // namespace

PYBIND11_MODULE(_fwa_torch, m) {
    m.def("forward", &forward);
    m.def("forward_qkv", &forward_qkv);
    m.def("backward", &backward);
    m.def("backward_qkv", &backward_qkv);
    m.def("attention", torch::wrap_pybind_function(&attention));
    m.def("attention_qkv", torch::wrap_pybind_function(&attention_qkv));
    m.def("bias_gather", &bias_gather);
    m.def("bias_scatter", &bias_scatter);
    m.def("bucket_gather", &bucket_gather);
    m.def("bucket_scatter", &bucket_scatter);
    m.def("sequence_forward", &sequence_forward);
    m.def("sequence_backward", &sequence_backward);
    m.def("bucket_bias", torch::wrap_pybind_function(&bucket_bias));
    m.def("sequence_attention", torch::wrap_pybind_function(&sequence_attention));
    m.def("rotary", &rotary);
    m.def("page_append", &page_append);
    m.def("page_forward", &page_forward);
    m.def("rotary_node", torch::wrap_pybind_function(&rotary_node));
}
