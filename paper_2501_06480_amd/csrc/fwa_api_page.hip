// extern "C" entry points of the rotary positions and of the operators on a paged cache: argument validation and dispatch.
// Every check happens before any HIP call, so an error never launches work.
#include "../../include/fwa.h"
#include "fwa_check.h"
#include "fwa_internal.h"

namespace {

using namespace fwa::check;

constexpr int64_t kMostRows = 1 << 24, kMostKeys = 1 << 29, kMostPages = 0x7fffffff;
constexpr int kMostHeads = 1 << 15, kMostWidth = 512, kMostAxes = 16, kMostSequences = 1 << 20, kMostPageRows = 1 << 16;

inline bool odd_word(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
inline bool known_type(int dtype) { return dtype == FWA_F32 || dtype == FWA_BF16 || dtype == FWA_F16; }
inline Span flat(const void* p, uint64_t bytes) { return Span{reinterpret_cast<uintptr_t>(p), bytes, bytes, 1}; }

// Positions, frequencies and pairs of a rotation of heads of d channels.
int check_rotation(int d, const int32_t* positions, int axes, const float* frequencies, const int32_t* axis_of, int pairs) {
    if (pairs < 0 || pairs > d / 2 || axes < 1) return FWA_ERR_SHAPE;
    if (axes > kMostAxes) return FWA_ERR_UNSUPPORTED;
    if (pairs > 0 && !frequencies) return FWA_ERR_NULL;
    return odd_word(positions) || odd_word(frequencies) || odd_word(axis_of) ? FWA_ERR_ALIGN : FWA_OK;
}

struct Touched {
    Span ins[12], outs[4];
    int ni = 0, no = 0;
    void in(const Span& s) { ins[ni++] = s; }
    void words(const void* p, int64_t count) { if (p && count > 0) in(flat(p, (uint64_t)count * 4)); }
    void out(const Span& s) { outs[no++] = s; }
    bool shared() const {
        for (int x = 0; x < no; ++x)
            for (int y = 0; y < ni; ++y)
                if (overlaps(outs[x], ins[y])) return true;
        for (int x = 0; x < no; ++x)
            for (int y = x + 1; y < no; ++y)
                if (overlaps(outs[x], outs[y])) return true;
        return false;
    }
};

// A cache's dimensions from the innermost outwards, as a tensor that reaches no element twice has them.
struct Dim {
    int64_t stride, size;
};
void cache_dims(const fwa::PageArgs& a, Dim (&dims)[3]) {
    dims[0] = {a.head_stride, a.KV};
    dims[1] = {a.token_stride, a.page_size};
    dims[2] = {a.page_stride, a.pages};
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2 - i; ++j)
            if (dims[j].size > 1 && (dims[j + 1].size <= 1 || dims[j + 1].stride < dims[j].stride)) { const Dim x = dims[j]; dims[j] = dims[j + 1]; dims[j + 1] = x; }
}
uint64_t cache_bytes(const fwa::PageArgs& a) {
    const uint64_t last = (uint64_t)(a.pages - 1) * a.page_stride + (uint64_t)(a.page_size - 1) * a.token_stride + (uint64_t)(a.KV - 1) * a.head_stride + a.D;
    return last * (a.dtype == FWA_F32 ? 4 : 2);
}
// Whether keys and values share a byte: the same strides, so for each dimension and what lies inside it the test of rows is exact; one that shows
// them apart is enough.
bool caches_overlap(const fwa::PageArgs& a) {
    const uint64_t e = a.dtype == FWA_F32 ? 4 : 2;
    const uintptr_t k = reinterpret_cast<uintptr_t>(a.k), v = reinterpret_cast<uintptr_t>(a.v);
    if (!overlaps(flat(a.k, cache_bytes(a)), flat(a.v, cache_bytes(a)))) return false;
    Dim dims[3];
    cache_dims(a, dims);
    uint64_t inside = (uint64_t)a.D;  // elements from the first to the last of what lies inside a dimension
    for (int i = 0; i < 3; ++i) {
        if (dims[i].size <= 1) continue;
        // places of the dimensions from here on outwards are multiples of this one's stride
        bool even = true;
        for (int j = i + 1; j < 3; ++j) even = even && (dims[j].size <= 1 || dims[j].stride % dims[i].stride == 0);
        if (even) {
            const uint64_t step = (uint64_t)dims[i].stride * e, width = inside * e, apart = (k < v ? v - k : k - v) % step;
            if (apart >= width && step - apart >= width) return false;
        }
        inside += (uint64_t)(dims[i].size - 1) * dims[i].stride;
    }
    return true;
}

// What append and attention share; fills in the sizes and the tables.
int check_pages(fwa::PageArgs& a, int64_t rows, int64_t N, int heads, int kv_heads, int d, int64_t pages, int page_size, int64_t page_stride, int64_t token_stride,
                int64_t head_stride, int width, int dtype) {
    if (rows < 0 || N < 0 || heads < 0 || kv_heads < 1 || d < 1 || heads % kv_heads != 0 || pages < 0 || page_size < 1 || width < 0) return FWA_ERR_SHAPE;
    if (!known_type(dtype) || (d != 32 && d != 64 && d != 128) || heads > kMostHeads || kv_heads > kMostHeads) return FWA_ERR_UNSUPPORTED;
    if (rows > kMostRows || N > kMostSequences || rows * (heads + 2LL * kv_heads) > 1 << 28) return FWA_ERR_UNSUPPORTED;
    if (page_size % 16 != 0 || page_size > kMostPageRows || pages > kMostPages || (int64_t)width * page_size > kMostKeys) return FWA_ERR_UNSUPPORTED;
    const int64_t per16 = dtype == FWA_F32 ? 4 : 8;
    if (page_stride < 0 || token_stride < 0 || head_stride < 0) return FWA_ERR_SHAPE;
    if (page_stride % per16 != 0 || token_stride % per16 != 0 || head_stride % per16 != 0) return FWA_ERR_ALIGN;
    if (token_stride > (int64_t)1 << 20 || page_stride > (int64_t)1 << 29 || head_stride > (int64_t)1 << 40) return FWA_ERR_UNSUPPORTED;
    a.rows = (int)rows; a.N = (int)N; a.H = heads; a.KV = kv_heads; a.D = d; a.dtype = dtype;
    a.pages = (int)pages; a.page_size = page_size; a.width = width;
    a.page_stride = page_stride; a.token_stride = token_stride; a.head_stride = head_stride;
    Dim dims[3];
    cache_dims(a, dims);
    int64_t inside = d;
    for (const Dim& x : dims) {
        if (x.size <= 1) continue;
        if (x.stride < inside) return FWA_ERR_SHAPE;
        if (x.size - 1 > ((int64_t)1 << 60) / x.stride) return FWA_ERR_UNSUPPORTED;
        inside += (x.size - 1) * x.stride;
    }
    return FWA_OK;
}
int check_tables(fwa::PageArgs& a, const int32_t* page_table, const int32_t* offsets, const int32_t* lengths) {
    if (!offsets || !lengths || (!page_table && a.width > 0)) return FWA_ERR_NULL;
    if (odd_word(page_table) || odd_word(offsets) || odd_word(lengths)) return FWA_ERR_ALIGN;
    a.table = page_table; a.offsets = offsets; a.lengths = lengths;
    return FWA_OK;
}
void read_tables(Touched& t, const fwa::PageArgs& a) {
    t.words(a.table, (int64_t)a.N * a.width);
    t.words(a.offsets, (int64_t)a.N + 1);
    t.words(a.lengths, a.N);
}

int check_attention(fwa::PageArgs& a, int64_t rows, int64_t N, int heads, int kv_heads, int d, int64_t pages, int page_size, int64_t page_stride, int64_t token_stride,
                    int64_t head_stride, int width, int most_new, int dtype) {
    if (heads < 1 || most_new < 0) return FWA_ERR_SHAPE;
    const int rc = check_pages(a, rows, N, heads, kv_heads, d, pages, page_size, page_stride, token_stride, head_stride, width, dtype);
    a.most = most_new < a.rows ? most_new : a.rows;
    return rc;
}

}  // namespace

extern "C" {

int fwa_rotary(const void* x, void* y, int64_t rows, int heads, int d, int64_t ld_x, int64_t ld_y, const int32_t* positions, int64_t position_rows, int axes,
               const float* frequencies, const int32_t* axis_of, int pairs, int interleaved, int inverse, int dtype, void* stream) {
    if (rows < 0 || heads < 1 || d < 1 || position_rows < 1) return FWA_ERR_SHAPE;
    if (!known_type(dtype) || heads > kMostHeads || d > kMostWidth || rows > 0x7fffffff) return FWA_ERR_UNSUPPORTED;
    int rc = check_row_stride(ld_x, heads * d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_y, heads * d, dtype);
    if (rc == FWA_OK) rc = check_rotation(d, positions, axes, frequencies, axis_of, pairs);
    if (rc != FWA_OK) return rc;
    if (!fwa::rotary_fits(rows, heads, d, pairs, dtype)) return FWA_ERR_UNSUPPORTED;
    if (rows == 0) return FWA_OK;
    if (!x || !y || (pairs > 0 && !positions)) return FWA_ERR_NULL;
    if (misaligned(x) || misaligned(y)) return FWA_ERR_ALIGN;
    if (position_rows > rows) position_rows = rows;
    Touched touched;
    if (x != y || ld_x != ld_y) touched.in(span_of(x, 1, (int)rows, heads * d, ld_x, dtype));  // in place: every element is read before it is written
    touched.words(pairs > 0 ? positions : nullptr, position_rows * axes);
    touched.words(frequencies, pairs);
    touched.words(axis_of, pairs);
    touched.out(span_of(y, 1, (int)rows, heads * d, ld_y, dtype));
    if (touched.shared()) return FWA_ERR_ALIAS;
    fwa::RotaryArgs a = {};
    a.x = x; a.y = y; a.rows = rows; a.heads = heads; a.d = d; a.dtype = dtype; a.ldx = ld_x; a.ldy = ld_y;
    a.positions = positions; a.period = position_rows; a.axes = axes; a.frequencies = frequencies; a.axis_of = axis_of;
    a.pairs = pairs; a.interleaved = interleaved != 0; a.inverse = inverse != 0;
    return fwa::launch_rotary(a, static_cast<hipStream_t>(stream)) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

int fwa_page_append(const void* k, const void* v, void* k_pages, void* v_pages, int64_t rows, int64_t N, int kv_heads, int d, int64_t ld_k, int64_t ld_v, int64_t pages,
                    int page_size, int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* page_table, int width, const int32_t* offsets,
                    const int32_t* lengths, const int32_t* positions, int axes, const float* frequencies, const int32_t* axis_of, int pairs, int interleaved, const void* q,
                    void* q_out, int heads, int64_t ld_q, int64_t ld_q_out, int dtype, void* stream) {
    fwa::PageArgs a = {};
    if (q && heads < 1) return FWA_ERR_SHAPE;
    int rc = check_pages(a, rows, N, q ? heads : 0, kv_heads, d, pages, page_size, page_stride, token_stride, head_stride, width, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_k, kv_heads * d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_v, kv_heads * d, dtype);
    if (rc == FWA_OK && q) rc = check_row_stride(ld_q, heads * d, dtype);
    if (rc == FWA_OK && q) rc = check_row_stride(ld_q_out, heads * d, dtype);
    if (rc == FWA_OK) rc = check_rotation(d, positions, positions ? axes : 1, frequencies, axis_of, pairs);
    if (rc != FWA_OK) return rc;
    a.axes = positions ? axes : 1;
    a.pairs = pairs; a.interleaved = interleaved != 0;
    if (!fwa::page_append_fits(a)) return FWA_ERR_UNSUPPORTED;
    if (rows == 0 || N == 0) return FWA_OK;
    if (!k || !v || (q && !q_out) || (pages > 0 && (!k_pages || !v_pages))) return FWA_ERR_NULL;
    rc = check_tables(a, page_table, offsets, lengths);
    if (rc != FWA_OK) return rc;
    if (misaligned(k) || misaligned(v) || misaligned(k_pages) || misaligned(v_pages) || misaligned(q) || misaligned(q_out)) return FWA_ERR_ALIGN;
    a.k = k_pages; a.v = v_pages; a.new_k = k; a.new_v = v; a.ldk = ld_k; a.ldv = ld_v;
    a.q = q; a.o = q_out; a.ldq = ld_q; a.ldo = ld_q_out;
    a.positions = positions; a.frequencies = frequencies; a.axis_of = axis_of;
    Touched touched;
    read_tables(touched, a);
    touched.in(span_of(k, 1, (int)rows, kv_heads * d, ld_k, dtype));
    touched.in(span_of(v, 1, (int)rows, kv_heads * d, ld_v, dtype));
    touched.words(positions, rows * a.axes);
    touched.words(frequencies, pairs);
    touched.words(axis_of, pairs);
    if (q && (q != q_out || ld_q != ld_q_out)) touched.in(span_of(q, 1, (int)rows, heads * d, ld_q, dtype));
    if (q) touched.out(span_of(q_out, 1, (int)rows, heads * d, ld_q_out, dtype));
    if (pages > 0) {
        if (caches_overlap(a)) return FWA_ERR_ALIAS;
        // apart from each other as shown, so one after the other against the rest
        Touched other = touched;
        touched.out(flat(k_pages, cache_bytes(a)));
        other.out(flat(v_pages, cache_bytes(a)));
        if (other.shared()) return FWA_ERR_ALIAS;
    }
    if (touched.shared()) return FWA_ERR_ALIAS;
    return fwa::launch_page_append(a, static_cast<hipStream_t>(stream)) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

size_t fwa_page_forward_workspace_bytes(int64_t rows, int64_t N, int heads, int kv_heads, int d, int page_size, int width, int most_new, int dtype) {
    fwa::PageArgs a = {};
    // The cache's strides are not known here and do not matter: heads one behind the other in one page, whose distance to the next is none.
    const int rc = check_attention(a, rows, N, heads, kv_heads, d, 1, page_size, 0, d, (int64_t)page_size * d, width, most_new, dtype);
    if (rc != FWA_OK || rows == 0 || N == 0 || a.most == 0) return 0;
    return fwa::page_forward_workspace(a);
}

int fwa_page_forward(const void* q, const void* k_pages, const void* v_pages, void* o, float* stats, int64_t rows, int64_t N, int heads, int kv_heads, int d, float scale,
                     int64_t ld_q, int64_t ld_o, int64_t pages, int page_size, int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* page_table,
                     int width, const int32_t* offsets, const int32_t* lengths, int most_new, int causal, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
    fwa::PageArgs a = {};
    int rc = check_attention(a, rows, N, heads, kv_heads, d, pages, page_size, page_stride, token_stride, head_stride, width, most_new, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_q, heads * d, dtype);
    if (rc == FWA_OK) rc = check_row_stride(ld_o, heads * d, dtype);
    if (rc != FWA_OK) return rc;
    if (rows == 0 || N == 0 || a.most == 0) return FWA_OK;
    if (!q || !o || (pages > 0 && (!k_pages || !v_pages))) return FWA_ERR_NULL;
    rc = check_tables(a, page_table, offsets, lengths);
    if (rc != FWA_OK) return rc;
    if (misaligned(q) || misaligned(o) || misaligned(k_pages) || misaligned(v_pages) || misaligned(stats) || misaligned(workspace)) return FWA_ERR_ALIGN;
    Touched touched;
    read_tables(touched, a);
    touched.in(span_of(q, 1, (int)rows, heads * d, ld_q, dtype));
    if (pages > 0) {
        touched.in(flat(k_pages, cache_bytes(a)));
        touched.in(flat(v_pages, cache_bytes(a)));
    }
    touched.out(span_of(o, 1, (int)rows, heads * d, ld_o, dtype));
    if (stats) touched.out(flat(stats, (uint64_t)rows * heads * 8));
    if (touched.shared()) return FWA_ERR_ALIAS;
    if (!fwa::page_forward_fits(a)) return FWA_ERR_UNSUPPORTED;
    const size_t need = fwa::page_forward_workspace(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FWA_ERR_WORKSPACE;
    a.q = q; a.k = const_cast<void*>(k_pages); a.v = const_cast<void*>(v_pages); a.o = o; a.stats = stats;
    a.ldq = ld_q; a.ldo = ld_o; a.causal = causal != 0; a.scale = scale;
    return fwa::launch_page_forward(a, workspace, workspace_bytes, static_cast<hipStream_t>(stream)) == hipSuccess ? FWA_OK : FWA_ERR_LAUNCH;
}

}  // extern "C"
