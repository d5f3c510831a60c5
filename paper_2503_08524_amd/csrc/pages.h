// The paged key-value cache: handle, kernel arguments and launch wrappers.
//
// A page holds page_rows rows of every KV head.  Keys are [page][head][row][dim]; values [page][head][row / R][dim][row % R] with
// R = 16 bytes / element (16 of 8 bits, 8 fp16, 4 fp32): R consecutive rows of one dim are the 16 bytes that a lane of the matrix cores wants of V
// when it weighs rows, as 16 bytes of a row are what it wants of K, so both go from memory to the matrix cores without passing through LDS.
#pragma once
#include "d3_common.h"

#include "../../include/d3.h"

namespace d3 {

constexpr int kPagesMaxSeqs = 4096;        // sequences of a call
constexpr int kPagedHeads = 16;            // query heads of one workgroup: the columns of a matrix instruction
constexpr int kPagedMaxWgs = 512;          // workgroups of an attention launch, four waves each
constexpr int kPagedMaxRuns = 4 * kPagedMaxWgs;
constexpr int kPagedOverhead = 1;          // what beginning and ending a (sequence, heads) costs a workgroup, in chunks

// As a pool holds a value.
template <typename T> __device__ __forceinline__ T held(float v);
template <> __device__ __forceinline__ float held<float>(float v) { return v; }
template <> __device__ __forceinline__ f16_t held<f16_t>(float v) { return (f16_t)(v != v ? v : fminf(fmaxf(v, -65504.f), 65504.f)); }

struct ReserveArgs {
    int B, max_pages, n_pages, page_shift, max_tokens;
    const int32_t *added, *rows_in, *n_free_in;
    int32_t *rows_out, *n_free_out, *tables, *free_pages, *starts, *slots, *positions;
};
int launch_pages_reserve(const ReserveArgs& a, hipStream_t s);
// Rows of a sequence as a step counts them: none where a reserve with these starts (optional) gave it none.
__device__ __forceinline__ int live_rows(const int32_t* rows, const int32_t* starts, int max_rows, int b) {
    const int n = min(max(rows[b], 0), max_rows);
    return starts && starts[b] == starts[b + 1] ? 0 : n;
}
int launch_pages_live(const int32_t* rows, const int32_t* starts, int max_rows, int B, int32_t* live, hipStream_t s);

struct AppendArgs {
    int n, n_layers, H_kv, hd, page_shift;
    long long n_slots;                     // n_pages * page_rows
    const int32_t* slots;
    const void *k, *v;                     // [layer][token][head][dim] by the strides, in elements
    int dtype;                             // d3_dtype of k and v
    long long token_stride, head_stride, layer_stride;
    const float2* rope_cs;                 // optional [n][hd / 2]
    void *k_pages, *v_pages;               // the first layer's pools
    size_t pool_bytes;                     // of a layer
    float *k_scales, *v_scales;            // 8-bit pools: the first layer's scales, [page][H_kv][page_rows]
    size_t scale_bytes;                    // of a layer
};
int launch_pages_append(const AppendArgs& a, int kv_dtype, hipStream_t s);
int launch_pages_append8(const AppendArgs& a, int kv_dtype, hipStream_t s);     // D3_I8, D3_E4M3

struct ReadArgs {                          // as AppendArgs, the other way round
    int n, n_layers, H_kv, hd, page_shift;
    long long n_slots;
    const int32_t* slots;
    void *k, *v;
    int dtype;
    long long token_stride, head_stride, layer_stride;
    const void *k_pages, *v_pages;
    size_t pool_bytes;
    const float *k_scales, *v_scales;
    size_t scale_bytes;
};
int launch_pages_read(const ReadArgs& a, int kv_dtype, hipStream_t s);

struct PagesFillArgs {
    int n, H_kv, hd, page_shift, first, n_layers, src;     // src < 0: zeros
    Divisor by_heads;                      // H_kv
    long long n_slots;
    const int32_t* slots;
    void *k_pages, *v_pages;               // layer 0
    size_t pool_bytes;
    float *k_scales, *v_scales;            // 8-bit pools, layer 0
    size_t scale_bytes;
};
int launch_pages_fill(const PagesFillArgs& a, int kv_dtype, hipStream_t s);

struct PagedAttnArgs {
    const void *q, *k_new, *v_new;         // [B][H][hd], [B][H_kv][hd] by the strides, in elements; k_new, v_new NULL: every row is in its page
    int dtype;                             // d3_dtype of q, k_new, v_new and out
    long long q_stride, kv_stride, out_stride;
    const float2* rope_cs;                 // optional [B][hd / 2]: q and k_new turn by it
    const int32_t *tables, *rows;          // [B][table_stride] pages; rows of each sequence, the new one included
    int table_stride, max_rows;            // rows a table has room for
    int B, H_kv, group, n_pages, page_shift;
    float scale;                           // of the scores
    void *k_pages, *v_pages;               // this layer's pools
    void* out;
    bf16_t* out_split;                     // optional split copy
    SplitForm out_form;
    float *part_o, *part_ml;               // [2 * runs][min(group, 16)][hd], [..][2]
    int* tickets;                          // [B][H_kv * tiles], then [2 * runs], zero between launches
    Divisor by_runs, by_waves;             // set by launch_attention_paged: its workgroups and their waves
    float *k_scales, *v_scales;            // this layer's scales of 8-bit rows (last: ahead of what every launch takes they cost the others 0.2 us of 9)
    float scale_part;                      // scale log2(e) = scale_part * 2^scale_exp, set by launch_attention_paged8
    int scale_exp;
};
int launch_attention_paged(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s);
int launch_attention_paged8(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s);    // D3_I8, D3_E4M3
// rows of a wave's turn: 16 loads of 16 bytes a lane
inline int paged_turn_rows(int hd, int kv_dtype) { return 16 * 64 * 16 / (2 * hd * kv_elem_bytes(kv_dtype)); }
inline int paged_head_tiles(int group) { return (group + kPagedHeads - 1) / kPagedHeads; }

}  // namespace d3

struct d3_pages {
    d3_pages_desc desc;
    char *k, *v, *ws;
    float *ks, *vs;                        // scales of 8-bit pools
    int dev, n_cu;
    size_t part_ml, tickets;               // byte offsets into the workspace; the partial outputs are first
    size_t pool_bytes() const {
        return (size_t)desc.n_pages * desc.n_kv_heads * desc.page_rows * desc.head_dim * d3::kv_elem_bytes(desc.kv_dtype);
    }
    bool scaled() const { return d3::kv_elem_bytes(desc.kv_dtype) == 1; }
    size_t layer_scales() const { return scaled() ? (size_t)desc.n_pages * desc.n_kv_heads * desc.page_rows : 0; }
    long long n_slots() const { return (long long)desc.n_pages * desc.page_rows; }
};

namespace d3 {
// One layer's attention on the handle's pools: what launch_attention_paged needs of the handle.
inline PagedAttnArgs paged_attn_args(const d3_pages* p, int layer, int B) {
    const d3_pages_desc& d = p->desc;
    PagedAttnArgs a{};
    a.B = B; a.H_kv = d.n_kv_heads; a.group = d.n_heads / d.n_kv_heads;
    a.scale = 1.f / sqrtf((float)d.head_dim);
    a.n_pages = d.n_pages; a.page_shift = __builtin_ctz(d.page_rows);
    a.table_stride = d.max_pages; a.max_rows = d.max_pages * d.page_rows;
    a.k_pages = p->k + (size_t)layer * p->pool_bytes(); a.v_pages = p->v + (size_t)layer * p->pool_bytes();
    a.k_scales = p->ks + layer * p->layer_scales(); a.v_scales = p->vs + layer * p->layer_scales();
    a.part_o = reinterpret_cast<float*>(p->ws); a.part_ml = reinterpret_cast<float*>(p->ws + p->part_ml);
    a.tickets = reinterpret_cast<int*>(p->ws + p->tickets);
    return a;
}
// The device a handle was made on is current while this lives (the caller may have another one current).
struct OnDevice {
    int before = -1;
    explicit OnDevice(int dev) {
        int now = dev;
        if (hipGetDevice(&now) == hipSuccess && now != dev && hipSetDevice(dev) == hipSuccess) before = now;
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};
}  // namespace d3
