// C ABI of the paged key-value cache: handle and argument checks.  All device memory is the caller's.
#include <atomic>
#include <cstring>
#include <new>

#include "d3_error.h"
#include "pages.h"
#include "strided.h"

using namespace d3;

namespace {

constexpr size_t kAlign = 256;
constexpr int kMostTokens = 1 << 30;       // rows of one call
// a launch has fewer than 2^32 threads: an append has 8 a row and head (of the heads' own grid dimension), a fill 64 a row and head
constexpr int kMostAppendTokens = 1 << 28, kMostFillHeads = 1 << 25;

size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
int elem_bytes(int dtype) { return dtype == D3_F32 ? 4 : 2; }
bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int check_desc(const d3_pages_desc* d) {
    if (!d) return fail(D3_EINVAL, "pages desc is NULL");
    if (d->n_layers < 1 || d->n_layers > 4096) return fail(D3_ESHAPE, "pages: n_layers must be in [1, 4096] (got %d)", d->n_layers);
    if (d->n_kv_heads < 1 || d->n_heads < 1 || d->n_heads > 65535) return fail(D3_ESHAPE, "pages: n_heads must be in [1, 65535], n_kv_heads positive (got %d, %d)", d->n_heads, d->n_kv_heads);
    if (d->n_heads % d->n_kv_heads != 0) return fail(D3_ESHAPE, "pages: n_heads (%d) must be a multiple of n_kv_heads (%d)", d->n_heads, d->n_kv_heads);
    if (d->head_dim != 64 && d->head_dim != 128) return fail(D3_ESHAPE, "pages: head_dim must be 64 or 128 (got %d)", d->head_dim);
    if (d->kv_dtype == D3_BF16) return fail(D3_EINVAL, "pages: kv_dtype D3_BF16 is not offered (an 8-bit mantissa, see d3_model_desc); use D3_F16 (same bytes) or D3_F32");
    if (d->kv_dtype != D3_F32 && d->kv_dtype != D3_F16 && d->kv_dtype != D3_I8 && d->kv_dtype != D3_E4M3) return fail(D3_EINVAL, "pages: kv_dtype must be D3_F32, D3_F16, D3_I8 or D3_E4M3 (got %d)", d->kv_dtype);
    if (d->page_rows < 16 || d->page_rows > 1024 || (d->page_rows & (d->page_rows - 1)) != 0) return fail(D3_ESHAPE, "pages: page_rows must be a power of two in [16, 1024] (got %d)", d->page_rows);
    if (d->n_pages < 1 || (int64_t)d->n_pages * d->page_rows > INT32_MAX) return fail(D3_ESHAPE, "pages: n_pages must be positive and n_pages * page_rows below 2^31 (got %d, %d)", d->n_pages, d->page_rows);
    if (d->max_batch < 1 || d->max_batch > kPagesMaxSeqs) return fail(D3_ESHAPE, "pages: max_batch must be in [1, %d] (got %d)", kPagesMaxSeqs, d->max_batch);
    if (d->max_pages < 1 || (int64_t)d->max_pages * d->page_rows > kMostTokens || (int64_t)d->max_pages * d->max_batch > INT32_MAX)
        return fail(D3_ESHAPE, "pages: max_pages must be positive, max_pages * page_rows at most 2^30 and max_pages * max_batch below 2^31 (got %d)", d->max_pages);
    // the attention counts its pieces of work in 32 bits
    const int64_t chunks = ((int64_t)d->max_pages * d->page_rows + paged_turn_rows(d->head_dim, d->kv_dtype) - 1) / paged_turn_rows(d->head_dim, d->kv_dtype);
    const int64_t per_chunk = (int64_t)d->n_kv_heads * paged_head_tiles(d->n_heads / d->n_kv_heads) * d->max_batch;
    if (chunks + kPagedOverhead > INT32_MAX / per_chunk)
        return fail(D3_ESHAPE, "pages: %d sequences of up to %d pages are more rows than one attention launch counts", d->max_batch, d->max_pages);
    return D3_OK;
}

// offsets behind the partial outputs; returns the whole size
size_t layout(const d3_pages_desc& d, size_t* part_ml, size_t* tickets) {
    const int group = d.n_heads / d.n_kv_heads;
    const size_t partials = 2 * (size_t)kPagedMaxRuns * (group < kPagedHeads ? group : kPagedHeads);
    *part_ml = align_up(partials * d.head_dim * 4);
    *tickets = *part_ml + align_up(partials * 2 * 4);
    return *tickets + align_up(((size_t)d.max_batch * d.n_kv_heads * paged_head_tiles(group) + 2 * kPagedMaxRuns) * 4);
}

int check_layers(const d3_pages* p, const char* who, int32_t layer, int32_t n) {
    if (n < 1 || layer < 0 || layer > p->desc.n_layers - n) return fail(D3_ERANGE, "%s: layers [%d, %d + %d) are outside the %d of the pool", who, layer, layer, n, p->desc.n_layers);
    return D3_OK;
}
int check_batch(const d3_pages* p, const char* who, int32_t B) {
    if (B < 1 || B > p->desc.max_batch) return fail(D3_ESHAPE, "%s: B must be in [1, %d] (got %d)", who, p->desc.max_batch, B);
    return D3_OK;
}
int check_tokens(const char* who, int32_t n) {
    if (n < 0 || n > kMostTokens) return fail(D3_EINVAL, "%s: the number of rows must be in [0, 2^30] (got %d)", who, n);
    return D3_OK;
}
int check_dtype(const char* who, int32_t dtype) {
    if (dtype != D3_F32 && dtype != D3_BF16 && dtype != D3_F16) return fail(D3_EINVAL, "%s: dtype must be D3_F32, D3_BF16 or D3_F16 (got %d)", who, dtype);
    return D3_OK;
}

}  // namespace

#define D3_HIP(expr)                                                                              \
    do {                                                                                          \
        hipError_t e_ = (hipError_t)(expr);                                                       \
        if (e_ != hipSuccess) return fail(D3_EDEVICE, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)
#define D3_CHECK(expr)                  \
    do {                                \
        const int rc_ = (expr);         \
        if (rc_ != D3_OK) return rc_;   \
    } while (0)

namespace {
// Compute units of a gfx950 device, asked once per device (the properties take longer than the rest of d3_pages_create).
int device_cus(const char* who, int dev, int* n_cu) {
    constexpr int kMaxDevices = 64;
    static std::atomic<int> known[kMaxDevices];
    if (dev < 0 || dev >= kMaxDevices) return fail(D3_EDEVICE, "%s: device index %d is outside [0, %d)", who, dev, kMaxDevices);
    *n_cu = known[dev].load(std::memory_order_relaxed);
    if (*n_cu > 0) return D3_OK;
    hipDeviceProp_t prop;
    D3_HIP(hipGetDeviceProperties(&prop, dev));
    if (strncmp(prop.gcnArchName, "gfx950", 6) != 0) return fail(D3_EDEVICE, "%s: built for gfx950, device is %s", who, prop.gcnArchName);
    *n_cu = prop.multiProcessorCount;
    known[dev].store(*n_cu, std::memory_order_relaxed);
    return D3_OK;
}
}  // namespace

extern "C" size_t d3_pages_workspace_size(const d3_pages_desc* desc) {
    if (check_desc(desc) != D3_OK) return 0;
    size_t ml, tickets;
    return layout(*desc, &ml, &tickets);
}

namespace {
int create(const char* who, d3_pages** out, const d3_pages_desc* desc, void* k_pages, void* v_pages, float* k_scales, float* v_scales, void* workspace, size_t workspace_bytes) {
    if (!k_pages || !v_pages || !workspace) return fail(D3_EINVAL, "%s: pool or workspace is NULL", who);
    if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(D3_EINVAL, "%s: the pools must be 16-byte aligned", who);
    if (reinterpret_cast<uintptr_t>(workspace) % kAlign != 0) return fail(D3_EINVAL, "%s: workspace must be %zu-byte aligned", who, kAlign);
    size_t part_ml, tickets;
    const size_t need = layout(*desc, &part_ml, &tickets);
    if (workspace_bytes < need) return fail(D3_EINVAL, "%s: workspace has %zu bytes, %zu needed", who, workspace_bytes, need);
    int dev = 0, n_cu = 0;
    D3_HIP(hipGetDevice(&dev));
    D3_CHECK(device_cus(who, dev, &n_cu));
    d3_pages* p = new (std::nothrow) d3_pages();
    if (!p) return fail(D3_EINVAL, "%s: out of host memory", who);
    p->desc = *desc;
    p->k = static_cast<char*>(k_pages); p->v = static_cast<char*>(v_pages); p->ws = static_cast<char*>(workspace);
    p->ks = k_scales; p->vs = v_scales;
    p->dev = dev; p->n_cu = n_cu;
    p->part_ml = part_ml; p->tickets = tickets;
    hipError_t e = hipMemset(p->ws + tickets, 0, need - tickets);              // arrival counters start at 0
    if (e == hipSuccess) e = hipStreamSynchronize(nullptr);                   // calls may come on any stream
    if (e != hipSuccess) { delete p; return fail(D3_EDEVICE, "%s: hipMemset failed: %s", who, hipGetErrorString(e)); }
    *out = p;
    return D3_OK;
}
}  // namespace

extern "C" int d3_pages_create(d3_pages** out, const d3_pages_desc* desc, void* k_pages, void* v_pages, void* workspace, size_t workspace_bytes) {
    if (!out) return fail(D3_EINVAL, "d3_pages_create: out is NULL");
    *out = nullptr;
    D3_CHECK(check_desc(desc));
    if (kv_elem_bytes(desc->kv_dtype) == 1) return fail(D3_EINVAL, "d3_pages_create: pools of 8 bits have scales (d3_pages_create_scaled)");
    return create("d3_pages_create", out, desc, k_pages, v_pages, nullptr, nullptr, workspace, workspace_bytes);
}

extern "C" int d3_pages_create_scaled(d3_pages** out, const d3_pages_desc* desc, void* k_pages, void* v_pages, float* k_scales, float* v_scales, void* workspace, size_t workspace_bytes) {
    if (!out) return fail(D3_EINVAL, "d3_pages_create_scaled: out is NULL");
    *out = nullptr;
    D3_CHECK(check_desc(desc));
    if (kv_elem_bytes(desc->kv_dtype) != 1) return fail(D3_EINVAL, "d3_pages_create_scaled: only pools of 8 bits (D3_I8, D3_E4M3) have scales (d3_pages_create)");
    if (!k_scales || !v_scales) return fail(D3_EINVAL, "d3_pages_create_scaled: scales are NULL");
    if (!aligned16(k_scales) || !aligned16(v_scales)) return fail(D3_EINVAL, "d3_pages_create_scaled: the scales must be 16-byte aligned");
    return create("d3_pages_create_scaled", out, desc, k_pages, v_pages, k_scales, v_scales, workspace, workspace_bytes);
}

extern "C" int d3_pages_destroy(d3_pages* pages) {
    delete pages;
    return D3_OK;
}

extern "C" int d3_pages_reserve(d3_pages* pages, int32_t B, const int32_t* added, const int32_t* rows_in, int32_t* rows_out, int32_t* tables,
                                int32_t* free_pages, const int32_t* n_free_in, int32_t* n_free_out, int32_t max_tokens, int32_t* starts,
                                int32_t* slots, int32_t* positions, void* hip_stream) {
    if (!pages || !added || !rows_in || !rows_out || !tables || !free_pages || !n_free_in || !n_free_out || !starts || (!slots && max_tokens > 0))
        return fail(D3_EINVAL, "d3_pages_reserve: NULL argument");
    D3_CHECK(check_batch(pages, "d3_pages_reserve", B));
    D3_CHECK(check_tokens("d3_pages_reserve", max_tokens));
    ReserveArgs a{};
    a.B = B; a.max_pages = pages->desc.max_pages; a.n_pages = pages->desc.n_pages; a.page_shift = __builtin_ctz(pages->desc.page_rows); a.max_tokens = max_tokens;
    a.added = added; a.rows_in = rows_in; a.n_free_in = n_free_in;
    a.rows_out = rows_out; a.n_free_out = n_free_out; a.tables = tables; a.free_pages = free_pages;
    a.starts = starts; a.slots = slots; a.positions = positions;
    const OnDevice on(pages->dev);
    D3_HIP(launch_pages_reserve(a, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}

extern "C" int d3_pages_live(d3_pages* pages, int32_t B, const int32_t* rows, const int32_t* starts, int32_t* live, void* hip_stream) {
    if (!pages || !rows || !starts || !live) return fail(D3_EINVAL, "d3_pages_live: NULL argument");
    D3_CHECK(check_batch(pages, "d3_pages_live", B));
    const OnDevice on(pages->dev);
    D3_HIP(launch_pages_live(rows, starts, pages->desc.max_pages * pages->desc.page_rows, B, live, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}

extern "C" int d3_pages_append(d3_pages* pages, int32_t layer, int32_t n_layers, int32_t n, const int32_t* slots, const void* k, const void* v, int32_t dtype,
                               int64_t token_stride, int64_t head_stride, int64_t layer_stride, const float* rope_cs, void* hip_stream) {
    if (!pages) return fail(D3_EINVAL, "d3_pages_append: pages is NULL");
    D3_CHECK(check_tokens("d3_pages_append", n));
    D3_CHECK(check_layers(pages, "d3_pages_append", layer, n_layers));
    D3_CHECK(check_dtype("d3_pages_append", dtype));
    if (n > kMostAppendTokens) return fail(D3_ESHAPE, "d3_pages_append: %d rows are more than one launch counts (%d)", n, kMostAppendTokens);
    if (n == 0) return D3_OK;
    if (!slots || !k || !v) return fail(D3_EINVAL, "d3_pages_append: NULL argument");
    const int unit = 16 / elem_bytes(dtype);
    if (!aligned16(k) || !aligned16(v) || token_stride % unit != 0 || head_stride % unit != 0 || layer_stride % unit != 0)
        return fail(D3_EINVAL, "d3_pages_append: k, v and their strides must be multiples of 16 bytes");
    if (!aligned16(rope_cs)) return fail(D3_EINVAL, "d3_pages_append: rope_cs must be 16-byte aligned");
    const d3_pages_desc& d = pages->desc;
    AppendArgs a{};
    a.n = n; a.n_layers = n_layers; a.H_kv = d.n_kv_heads; a.hd = d.head_dim; a.page_shift = __builtin_ctz(d.page_rows); a.n_slots = pages->n_slots();
    a.slots = slots; a.k = k; a.v = v; a.dtype = dtype;
    a.token_stride = token_stride; a.head_stride = head_stride; a.layer_stride = layer_stride;
    a.rope_cs = reinterpret_cast<const float2*>(rope_cs);
    a.pool_bytes = pages->pool_bytes();
    a.k_pages = pages->k + layer * a.pool_bytes; a.v_pages = pages->v + layer * a.pool_bytes;
    a.k_scales = pages->ks + layer * pages->layer_scales(); a.v_scales = pages->vs + layer * pages->layer_scales(); a.scale_bytes = pages->layer_scales() * 4;
    const OnDevice on(pages->dev);
    D3_HIP(launch_pages_append(a, d.kv_dtype, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}

extern "C" int d3_pages_read(d3_pages* pages, int32_t layer, int32_t n_layers, int32_t n, const int32_t* slots, void* k, void* v, int32_t dtype, int64_t token_stride, int64_t head_stride,
                             int64_t layer_stride, void* hip_stream) {
    if (!pages) return fail(D3_EINVAL, "d3_pages_read: pages is NULL");
    D3_CHECK(check_tokens("d3_pages_read", n));
    D3_CHECK(check_layers(pages, "d3_pages_read", layer, n_layers));
    D3_CHECK(check_dtype("d3_pages_read", dtype));
    if (n > kMostAppendTokens) return fail(D3_ESHAPE, "d3_pages_read: %d rows are more than one launch counts (%d)", n, kMostAppendTokens);
    if (n == 0) return D3_OK;
    if (!slots || !k || !v) return fail(D3_EINVAL, "d3_pages_read: NULL argument");
    const int unit = 16 / elem_bytes(dtype);
    if (!aligned16(k) || !aligned16(v) || token_stride % unit != 0 || head_stride % unit != 0 || layer_stride % unit != 0)
        return fail(D3_EINVAL, "d3_pages_read: k, v and their strides must be multiples of 16 bytes");
    const d3_pages_desc& d = pages->desc;
    const intptr_t apart = (reinterpret_cast<intptr_t>(v) - reinterpret_cast<intptr_t>(k)) / elem_bytes(dtype);
    if (apart == 0 || rows_overlap(d.head_dim, {{n, token_stride}, {d.n_kv_heads, head_stride}, {n_layers, layer_stride}}, apart))
        return fail(D3_EINVAL, "d3_pages_read: rows of k and v must not lie on each other (strides of row, head and layer %lld, %lld, %lld, v %lld elements behind k)", (long long)token_stride, (long long)head_stride,
                    (long long)layer_stride, (long long)apart);
    ReadArgs a{};
    a.n = n; a.n_layers = n_layers; a.H_kv = d.n_kv_heads; a.hd = d.head_dim; a.page_shift = __builtin_ctz(d.page_rows); a.n_slots = pages->n_slots();
    a.slots = slots; a.k = k; a.v = v; a.dtype = dtype;
    a.token_stride = token_stride; a.head_stride = head_stride; a.layer_stride = layer_stride;
    a.pool_bytes = pages->pool_bytes(); a.scale_bytes = pages->layer_scales() * 4;
    a.k_pages = pages->k + layer * a.pool_bytes; a.v_pages = pages->v + layer * a.pool_bytes;
    a.k_scales = pages->ks + layer * pages->layer_scales(); a.v_scales = pages->vs + layer * pages->layer_scales();
    const OnDevice on(pages->dev);
    D3_HIP(launch_pages_read(a, d.kv_dtype, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}

extern "C" int d3_pages_attention(d3_pages* pages, int32_t layer, int32_t B, const void* q, const void* k_new, const void* v_new, int32_t dtype, int64_t q_stride,
                                  int64_t kv_stride, const float* rope_cs, const int32_t* tables, const int32_t* rows, float scale, void* out,
                                  int64_t out_stride, void* hip_stream) {
    if (!pages || !q || !tables || !rows || !out) return fail(D3_EINVAL, "d3_pages_attention: NULL argument");
    if (!k_new != !v_new) return fail(D3_EINVAL, "d3_pages_attention: k_new and v_new come together or not at all");
    D3_CHECK(check_batch(pages, "d3_pages_attention", B));
    D3_CHECK(check_layers(pages, "d3_pages_attention", layer, 1));
    D3_CHECK(check_dtype("d3_pages_attention", dtype));
    const int unit = 16 / elem_bytes(dtype);
    if (!aligned16(q) || !aligned16(k_new) || !aligned16(v_new) || q_stride % unit != 0 || (k_new && kv_stride % unit != 0))
        return fail(D3_EINVAL, "d3_pages_attention: q, k_new, v_new and their strides must be multiples of 16 bytes");
    if (!aligned16(rope_cs)) return fail(D3_EINVAL, "d3_pages_attention: rope_cs must be 16-byte aligned");
    if (!(scale - scale == 0.f)) return fail(D3_EINVAL, "d3_pages_attention: scale must be finite");
    PagedAttnArgs a = paged_attn_args(pages, layer, B);
    a.q = q; a.k_new = k_new; a.v_new = v_new; a.dtype = dtype;
    a.q_stride = q_stride; a.kv_stride = kv_stride; a.out_stride = out_stride;
    a.rope_cs = reinterpret_cast<const float2*>(rope_cs);
    a.tables = tables; a.rows = rows; a.out = out;
    if (scale != 0.f) a.scale = scale;
    const OnDevice on(pages->dev);
    D3_HIP(launch_attention_paged(a, pages->desc.head_dim, pages->desc.kv_dtype, pages->n_cu, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}

extern "C" int d3_pages_fill(d3_pages* pages, int32_t n, const int32_t* slots, int32_t src, int32_t first, int32_t n_layers, void* hip_stream) {
    if (!pages) return fail(D3_EINVAL, "d3_pages_fill: pages is NULL");
    D3_CHECK(check_tokens("d3_pages_fill", n));
    if (n_layers == 0 || n == 0) return D3_OK;
    D3_CHECK(check_layers(pages, "d3_pages_fill", first, n_layers));
    if (src >= pages->desc.n_layers || (src >= first && src < first + n_layers))
        return fail(D3_ERANGE, "d3_pages_fill: source layer %d must be one of the pool's and outside [%d, %d)", src, first, first + n_layers);
    if (!slots) return fail(D3_EINVAL, "d3_pages_fill: NULL argument");
    if ((int64_t)n * pages->desc.n_kv_heads > kMostFillHeads) return fail(D3_ESHAPE, "d3_pages_fill: %d rows of %d KV heads are more than one launch counts (%d heads of rows)", n, pages->desc.n_kv_heads, kMostFillHeads);
    const d3_pages_desc& d = pages->desc;
    PagesFillArgs a{};
    a.n = n; a.H_kv = d.n_kv_heads; a.hd = d.head_dim; a.page_shift = __builtin_ctz(d.page_rows); a.by_heads = Divisor(d.n_kv_heads); a.first = first; a.n_layers = n_layers; a.src = src < 0 ? -1 : src;
    a.n_slots = pages->n_slots();
    a.slots = slots; a.k_pages = pages->k; a.v_pages = pages->v; a.pool_bytes = pages->pool_bytes();
    a.k_scales = pages->ks; a.v_scales = pages->vs; a.scale_bytes = pages->layer_scales() * 4;
    const OnDevice on(pages->dev);
    D3_HIP(launch_pages_fill(a, d.kv_dtype, static_cast<hipStream_t>(hip_stream)));
    return D3_OK;
}
