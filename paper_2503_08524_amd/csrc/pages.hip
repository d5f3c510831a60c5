// Kernels of the paged cache beside its attention: page tables and slot maps from request lengths, rows into pages, the missing-state fill on pages.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace d3 {

namespace {

// ---------------- page tables and slot maps ----------------
// One workgroup: sums over the sequences (a wave's by row shifts, no LDS; the waves' through LDS), then pages and tokens found in those sums by bisection.  A chain of round trips
// bounds it: requests in, sums, pages of the stack, tables, slots (8 sequences 2.5 us, 256 with 20000 new rows 6.2 and 3.4 for the slots).
__device__ __forceinline__ unsigned long long shifted64(unsigned long long v, int which) {
    unsigned lo, hi;
#define D3_SHIFT(ctrl, rows) lo = __builtin_amdgcn_update_dpp(0, (unsigned)v, ctrl, rows, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (unsigned)(v >> 32), ctrl, rows, 0xf, false)
    switch (which) {
        case 0: D3_SHIFT(0x111, 0xf); break;
        case 1: D3_SHIFT(0x112, 0xf); break;
        case 2: D3_SHIFT(0x114, 0xf); break;
        case 3: D3_SHIFT(0x118, 0xf); break;
        case 4: D3_SHIFT(0x142, 0xa); break;
        default: D3_SHIFT(0x143, 0xc);
    }
#undef D3_SHIFT
    return (unsigned long long)hi << 32 | lo;
}
// Sum over the threads before this one, and over all; `red`: a word per wave.
template <int THREADS>
__device__ __forceinline__ unsigned long long scan_block(unsigned long long v, unsigned long long* red, unsigned long long* all) {
    constexpr int WAVES = THREADS / 64;
    unsigned long long s = v;
#pragma unroll
    for (int k = 0; k < 6; ++k) s += shifted64(s, k);
    const unsigned long long last = (unsigned long long)__builtin_amdgcn_readlane((unsigned)(s >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)s, 63);
    if constexpr (WAVES == 1) {
        *all = last;
        return s - v;
    }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) red[wave] = s;
    __syncthreads();
    unsigned long long before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const unsigned long long x = red[w];
        if (w < wave) before += x;
        sum += x;
    }
    *all = sum;
    return before + s - v;
}
// the last of v[0 .. n - 1], not decreasing, that is at most x (v[0] is)
__device__ __forceinline__ int last_at_most(const int* v, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (v[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// slot and position of new row t of the call; `tables` and `rows` as they are after it
__device__ __forceinline__ void write_token(const ReserveArgs& a, const int* starts, int t) {
    int slot = -1, p = -1;
    if (t < starts[a.B]) {
        const int b = last_at_most(starts, a.B, t);                 // sequences that got nothing share their start with the next one
        p = a.rows_out[b] - starts[b + 1] + t;
        const int page = a.tables[(size_t)b * a.max_pages + (p >> a.page_shift)];
        if ((unsigned)page < (unsigned)a.n_pages) slot = (page << a.page_shift) + (p & ((1 << a.page_shift) - 1));
    }
    a.slots[t] = slot;
    if (a.positions) a.positions[t] = p;
}

// THREADS * EACH sequences at most, EACH consecutive ones a thread
template <int THREADS, int EACH>
__global__ __launch_bounds__(THREADS) void pages_reserve_kernel(ReserveArgs a, int write_tokens) {
    constexpr int MOST = THREADS * EACH;
    __shared__ int starts[MOST + 1], page_at[MOST + 1], back_at[MOST + 1], page_first[MOST];
    __shared__ unsigned long long red[3][THREADS / 64];
    const int tid = threadIdx.x, b0 = tid * EACH, cap = a.max_pages << a.page_shift;
    auto pages_of = [&](int rows) { return (int)(((unsigned)rows + (1u << a.page_shift) - 1) >> a.page_shift); };
    int rows[EACH], need[EACH], back[EACH], add[EACH];
    long long asked[EACH];
    unsigned long long mine = 0, all;
    const int free_in = a.n_free_in[0];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int b = b0 + j;
        add[j] = b < a.B ? a.added[b] : 0;
        rows[j] = b < a.B ? a.rows_in[b] : 0;
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        rows[j] = min(max(rows[j], 0), cap);
        back[j] = add[j] < 0 ? pages_of(rows[j]) : 0;
        if (add[j] < 0) rows[j] = 0;
        asked[j] = add[j] > 0 && (long long)rows[j] + add[j] <= cap ? add[j] : 0;
        mine += asked[j];
    }
    // what of it fits max_tokens, the pages that needs, and the pages that come back: two sums in one word, neither passes 2^31
    unsigned long long before = scan_block<THREADS>(mine, red[0], &all), both = 0;
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        before += asked[j];
        if (before > (unsigned long long)a.max_tokens) asked[j] = 0;
        need[j] = pages_of(rows[j] + (int)asked[j]) - pages_of(rows[j]);
        both += (unsigned long long)need[j] << 32 | (unsigned)back[j];
    }
    before = scan_block<THREADS>(both, red[1], &all);
    const long long wanted = all >> 32, returned = (unsigned)all;
    const int n_free = min(max(free_in, 0), a.n_pages), avail = (int)min((long long)n_free + returned, (long long)a.n_pages);
    int need_before = (int)(before >> 32), back_before = (int)(unsigned)before;
    both = 0;
    int granted[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        granted[j] = need[j] == 0 || need_before + need[j] <= avail ? (int)asked[j] : 0;       // a refusal for pages refuses all behind it that need some
        need_before += need[j];
        if (granted[j] == 0) need[j] = 0;
        both += (unsigned long long)need[j] << 32 | (unsigned)granted[j];
    }
    before = scan_block<THREADS>(both, red[2], &all);
    const int taken = (int)(all >> 32), tokens = (int)(unsigned)all;
    int start = (int)(unsigned)before, page = (int)(before >> 32);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
        const int b = b0 + j;
        if (b >= a.B) break;
        starts[b] = start; page_at[b] = page; back_at[b] = back_before;
        page_first[b] = pages_of(rows[j]);
        a.starts[b] = start;
        a.rows_out[b] = rows[j] + granted[j];
        start += granted[j]; page += need[j]; back_before += back[j];
    }
    if (tid == 0) {
        starts[a.B] = tokens; page_at[a.B] = taken; back_at[a.B] = (int)returned;
        a.starts[a.B] = tokens;
    }
    __syncthreads();                                                // (also: everybody has read n_free_in, which may be n_free_out)
    if (tid == 0) {
        a.n_free_out[0] = avail - taken;
        a.n_free_out[1] = (int)max(wanted - avail, 0ll);
    }
    if (avail > n_free) {
        constexpr int RUN = THREADS == 64 ? 8 : 1;                  // pages of a thread, side by side (a whole workgroup has threads enough: 256 requests 9.7 us, with 8 pages a thread 14)
        for (int x0 = tid * RUN; x0 < avail - n_free; x0 += THREADS * RUN) {
            int b = last_at_most(back_at, a.B, x0), page[RUN];
#pragma unroll
            for (int k = 0; k < RUN; ++k) {
                const int x = min(x0 + k, avail - n_free - 1);
                while (back_at[b + 1] <= x) ++b;
                page[k] = a.tables[(size_t)b * a.max_pages + x - back_at[b]];
            }
#pragma unroll
            for (int k = 0; k < RUN; ++k) if (x0 + k < avail - n_free) a.free_pages[n_free + x0 + k] = page[k];
        }
        __syncthreads();
    }
    for (int x = tid; x < taken; x += THREADS) {
        const int b = last_at_most(page_at, a.B, x);
        a.tables[(size_t)b * a.max_pages + page_first[b] + x - page_at[b]] = a.free_pages[avail - 1 - x];
    }
    if (!write_tokens) return;
    __syncthreads();
    for (int t = tid; t < a.max_tokens; t += THREADS) write_token(a, starts, t);
}

// the tokens alone, behind the kernel above
__global__ __launch_bounds__(256) void pages_slots_kernel(ReserveArgs a) {
    __shared__ int starts[kPagesMaxSeqs + 1];
    for (int b = threadIdx.x; b <= a.B; b += 256) starts[b] = a.starts[b];
    __syncthreads();
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t < a.max_tokens) write_token(a, starts, t);
}

__global__ __launch_bounds__(256) void pages_live_kernel(const int32_t* rows, const int32_t* starts, int max_rows, int B, int32_t* live) {
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b < B) live[b] = live_rows(rows, starts, max_rows, b);
}

// ---------------- rows into pages ----------------
// E adjacent elements, 16 bytes of S or T at a time
template <int E, typename S> __device__ __forceinline__ void load_many(const S* p, float (&y)[E]) {
    constexpr int N = 16 / sizeof(S);
#pragma unroll
    for (int e = 0; e < E; e += N) {
        S t[N];
        const uint4 v = *reinterpret_cast<const uint4*>(p + e);
        __builtin_memcpy(t, &v, 16);
#pragma unroll
        for (int j = 0; j < N; ++j) { if constexpr (std::is_same<S, bf16_t>::value) y[e + j] = bf16_to_f32(t[j]); else y[e + j] = (float)t[j]; }
    }
}
template <int E, typename T> __device__ __forceinline__ void store_many(T* p, const float (&y)[E]) {
    T t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) t[e] = held<T>(y[e]);
    if constexpr (E * sizeof(T) == 8) {
        uint2 v;
        __builtin_memcpy(&v, t, 8);
        *reinterpret_cast<uint2*>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < E; e += 16 / sizeof(T)) {
            uint4 v;
            __builtin_memcpy(&v, t + e, 16);
            *reinterpret_cast<uint4*>(p + e) = v;
        }
    }
}
// N = 1 or 2 adjacent elements
template <int N, typename S> __device__ __forceinline__ void load_few(const S* p, float (&y)[N]) {
    if constexpr (N == 2 && sizeof(S) == 4) { const float2 v = *reinterpret_cast<const float2*>(p); y[0] = v.x; y[1] = v.y; }
    else if constexpr (N == 2) {
        const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
        S t[2];
        __builtin_memcpy(t, &v, 4);
#pragma unroll
        for (int e = 0; e < 2; ++e) { if constexpr (std::is_same<S, bf16_t>::value) y[e] = bf16_to_f32(t[e]); else y[e] = (float)t[e]; }
    } else if constexpr (std::is_same<S, bf16_t>::value) y[0] = bf16_to_f32(*p);
    else y[0] = (float)*p;
}

// grid: (32 tokens, KV head, layer and half: keys or values); a wave has 8 tokens.
// A key is a row of its page: 16 bytes of the lower half and their partners per thread.
// Of a value's dims R rows lie side by side in 16 bytes.  A lane has one or two dims: where a token is row 0 of a unit of R rows that follow each other in
// `slots`, its wave loads those R rows (whole lines each) and writes the unit's 16 bytes per dim, for all of them, also those of the next wave's tokens;
// only rows of units that the call does not fill are written element by element.  What each token is, is one wave's business: bits of a mask.
// Bound by memory: 8 layers x 1024 rows of 8 heads of 128, fp32, 30.5 us = 4.4 TB/s moved (a large copy 4.7); 512 rows of 32 heads, fp32 to fp16 with rotation, 6.7 us.  Through LDS,
// 64 tokens a workgroup, the values took 52 and 28 us.
constexpr int kAppendTokens = 32;

template <typename S, typename T, int HD>
__global__ __launch_bounds__(256) void pages_append_kernel(AppendArgs a) {
    constexpr int R = 16 / sizeof(T), DL = HD / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = blockIdx.y, layer = blockIdx.z >> 1;
    const bool values = blockIdx.z & 1;
    const S* src = static_cast<const S*>(values ? a.v : a.k) + layer * a.layer_stride + h * a.head_stride;
    const size_t head_elems = (size_t)HD << a.page_shift;
    auto pool_at = [&](void* pool, int slot) {                      // the head's rows of the slot's page
        return reinterpret_cast<T*>(static_cast<char*>(pool) + layer * a.pool_bytes) + ((size_t)(slot >> a.page_shift) * a.H_kv + h) * head_elems;
    };
    const int row_mask = (1 << a.page_shift) - 1;
    auto slot_at = [&](int t) {
        const int slot = t >= 0 && t < a.n ? a.slots[t] : -1;
        return slot < a.n_slots ? slot : -1;
    };
    if (!values) {
        constexpr int E = 16 / sizeof(S), PER = HD / (2 * E);      // threads of a token, each with one load of either half
#pragma unroll
        for (int x0 = 0; x0 < kAppendTokens * PER; x0 += 256) {
            const int x = x0 + tid, t = blockIdx.x * kAppendTokens + x / PER, j = x % PER * E, slot = x < kAppendTokens * PER ? slot_at(t) : -1;
            if (slot < 0) continue;
            float lo[E], hi[E];
            const S* row = src + t * a.token_stride;
            load_many<E, S>(row + j, lo);
            load_many<E, S>(row + j + HD / 2, hi);
            if (a.rope_cs) {
                const float2* c = a.rope_cs + (size_t)t * (HD / 2) + j;
                float2 cs[E];
#pragma unroll
                for (int e = 0; e < E; ++e) cs[e] = c[e];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x0 = lo[e], x1 = hi[e];
                    lo[e] = x0 * cs[e].x - x1 * cs[e].y;
                    hi[e] = x1 * cs[e].x + x0 * cs[e].y;
                }
            }
            T* to = pool_at(a.k_pages, slot) + (slot & row_mask) * HD + j;
            store_many<E, T>(to, lo);
            store_many<E, T>(to + HD / 2, hi);
        }
        return;
    }
    const int t0 = blockIdx.x * kAppendTokens + wave * 8;          // this wave's tokens are t0 .. t0 + 7: lanes R - 1 .. R + 6 of the ones it looks at
    const int slot = lane < 8 + 2 * (R - 1) ? slot_at(t0 - (R - 1) + lane) : -1;
    const unsigned valid = (unsigned)__ballot(slot >= 0), begins = (unsigned)__ballot(slot >= 0 && slot % R == 0);
    const int after = __shfl_down(slot, 1, 64);
    const unsigned follows = (unsigned)__ballot(slot >= 0 && after == slot + 1);        // the next token is the next row
    unsigned firsts = begins, covered = 0;
#pragma unroll
    for (int e = 0; e < R - 1; ++e) firsts &= follows >> e;
#pragma unroll
    for (int e = 0; e < R; ++e) covered |= firsts << e;
    const unsigned own = 0xffu << (R - 1);
    for (unsigned left = firsts & own; left; left &= left - 1) {
        const int x = __builtin_ctz(left), at = __builtin_amdgcn_readlane(slot, x);
        const S* row = src + (long long)(t0 - (R - 1) + x) * a.token_stride + lane * DL;
        float y[R][DL];
#pragma unroll
        for (int e = 0; e < R; ++e) load_few<DL, S>(row + e * a.token_stride, y[e]);
        T* to = pool_at(a.v_pages, at) + ((at & row_mask) / R * HD + lane * DL) * R;
#pragma unroll
        for (int d = 0; d < DL; ++d) {
            T unit[R];
#pragma unroll
            for (int e = 0; e < R; ++e) unit[e] = held<T>(y[e][d]);
            uint4 v;
            __builtin_memcpy(&v, unit, 16);
            *reinterpret_cast<uint4*>(to + d * R) = v;
        }
    }
    for (unsigned left = valid & ~covered & own; left; left &= left - 1) {
        const int x = __builtin_ctz(left), at = __builtin_amdgcn_readlane(slot, x);
        float y[DL];
        load_few<DL, S>(src + (long long)(t0 - (R - 1) + x) * a.token_stride + lane * DL, y);
        T* to = pool_at(a.v_pages, at) + ((at & row_mask) / R * HD + lane * DL) * R + at % R;
#pragma unroll
        for (int d = 0; d < DL; ++d) to[d * R] = held<T>(y[d]);
    }
}

// ---------------- missing-state fill on pages ----------------
// A wave has one (token, KV head): 16 bytes of the key in the first lanes, one or two elements of the value in each, read once from the source block
// and written into a few of the dropped ones (grid.y).  40 blocks of 8 rows of 8 heads, fp32, 4.5 us: little more than a launch, though the values, four bytes in every 16, write 6.5 MB
// for 2.6.
template <typename T, int HD>
__global__ __launch_bounds__(256) void pages_fill_kernel(PagesFillArgs a, int layers_each) {
    constexpr int R = 16 / sizeof(T), DL = HD / 64;
    const int lane = threadIdx.x & 63, unit = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= a.n * a.H_kv) return;
    const int t = a.by_heads.of(unit), head = unit - t * a.H_kv, slot = a.slots[t];
    if (slot < 0 || slot >= a.n_slots) return;
    const int row = slot & ((1 << a.page_shift) - 1);
    const size_t base = (((size_t)(slot >> a.page_shift) * a.H_kv + head) << a.page_shift) * HD;
    const int l0 = a.first + blockIdx.y * layers_each, l1 = min(l0 + layers_each, a.first + a.n_layers);
    const bool has_key = lane < HD / R;
    char* k_at = static_cast<char*>(a.k_pages) + (base + (size_t)row * HD + (has_key ? lane : 0) * R) * sizeof(T);
    char* v_at = static_cast<char*>(a.v_pages) + (base + (size_t)(row / R * HD + lane * DL) * R + row % R) * sizeof(T);
    uint4 kv = make_uint4(0, 0, 0, 0);
    T vv[DL] = {};
    if (a.src >= 0) {
        kv = *reinterpret_cast<const uint4*>(k_at + a.src * a.pool_bytes);
#pragma unroll
        for (int d = 0; d < DL; ++d) vv[d] = *reinterpret_cast<const T*>(v_at + a.src * a.pool_bytes + d * 16);
    }
    if constexpr (sizeof(T) == 1) {                                 // the row's scales: of the key in lane 0, of the value in lane 1
        if (lane < 2) {
            char* s_at = reinterpret_cast<char*>((lane == 0 ? a.k_scales : a.v_scales) + base / HD + row);
            const float scale = a.src >= 0 ? *reinterpret_cast<const float*>(s_at + a.src * a.scale_bytes) : 0.f;
            for (int l = l0; l < l1; ++l) *reinterpret_cast<float*>(s_at + l * a.scale_bytes) = scale;
        }
    }
    for (int l = l0; l < l1; ++l) {
        if (has_key) *reinterpret_cast<uint4*>(k_at + l * a.pool_bytes) = kv;
#pragma unroll
        for (int d = 0; d < DL; ++d) *reinterpret_cast<T*>(v_at + l * a.pool_bytes + d * 16) = vv[d];
    }
}

template <typename T>
int launch_fill(const PagesFillArgs& a, hipStream_t s) {
    // Blocks to a wave: one where all of them are few enough to be resident at once (each block is then one store away from its source); where there are more, several, that share their loads.
    // us by 1, 4, 8, all blocks of a wave, fp16: 8 units 8 blocks 2.2 2.9 3.9 3.8, 80 blocks 2.4 3.1 4.1 22; 32 units 32 blocks 2.6 3.2 4.2 9.9, 80 blocks 3.9 3.8 4.8 22; 128 units 8 blocks 2.6 3.3 4.3
    // 4.2, 32 blocks 5.2 4.7 5.4 11; 256 units 8 blocks 3.4 3.7 4.7 4.7, 32 blocks 8.0 7.0 7.0 12; 512 units 8 blocks 5.4 4.8 5.5 5.6, 32 blocks 12.5 11.6 10.9 13.3; 1024 units 32 blocks 18.7 20.2 18.8 20.0;
    // 4096 units 32 blocks 95.8 100.4 100.4 99.3; 16384 units 32 blocks 520 516 520 510, 80 blocks 1285 1275 1286 1253.
    const int units = a.n * a.H_kv, each = (long long)units * a.n_layers <= 2048 ? 1 : units >= 4096 ? a.n_layers : units >= 512 ? 8 : 4;
    const dim3 grid((units + 3) / 4, (a.n_layers + each - 1) / each);
    if (a.hd == 64) hipLaunchKernelGGL((pages_fill_kernel<T, 64>), grid, dim3(256), 0, s, a, each);
    else hipLaunchKernelGGL((pages_fill_kernel<T, 128>), grid, dim3(256), 0, s, a, each);
    return (int)hipGetLastError();
}

template <typename S, typename T>
int launch_append(const AppendArgs& a, hipStream_t s) {
    const dim3 grid((a.n + kAppendTokens - 1) / kAppendTokens, a.H_kv, 2 * a.n_layers);
    if (a.hd == 64) hipLaunchKernelGGL((pages_append_kernel<S, T, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((pages_append_kernel<S, T, 128>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <typename T>
int launch_append_to(const AppendArgs& a, hipStream_t s) {
    return a.dtype == D3_F32 ? launch_append<float, T>(a, s) : a.dtype == D3_BF16 ? launch_append<bf16_t, T>(a, s) : launch_append<f16_t, T>(a, s);
}

}  // namespace

int launch_pages_reserve(const ReserveArgs& a, hipStream_t s) {
    // Few tokens: by the same workgroup; many: by a launch of their own over the chip.  us by one launch / two: 2048 tokens of 1, 64, 1024 sequences 4.5 / 5.9, 5.7 / 6.8, 6.2 / 7.6; 4096 tokens
    // 5.1 / 6.0, 7.2 / 6.8, 8.2 / 7.8; a token each of 4096 sequences 11.9 / 13.9, two each 16.5 / 13.8.
    const bool few = a.max_tokens <= std::max(3500, a.B);
    // One wave where it has few rounds to go: 1, 8, 64 sequences, us by one wave / a workgroup, a token each 2.1 / 3.9, 2.3 / 4.0, 2.5 / 4.2; 256 tokens in all 2.9 / 4.0, 3.9 / 4.5, 4.3 / 4.2; 512
    // 3.7 / 4.1, 5.5 / 4.5, 6.6 / 4.3.  Pages that come back cost it a round for 512: full tables of 8192 entries, one of 2, 8, 64 sequences ends 11.1 / 5.2, 4.8 / 4.6, 3.8 / 4.8, all of 1, 8, 64
    // 19 / 5.5, 22 / 7.3, 25 / 9.0.  A step gains 1.7 us, so four steps or fewer pay for one that ends, ten for all.  Tables of 65536 entries: one ends 73 / 12.9, 22 / 7.7, 5.4 / 5.0, all 136 / 18, 160 / 32, 182 / 46.
    if (a.B <= 64 && a.max_tokens <= 256 && (long long)a.B * a.max_pages <= 8192) hipLaunchKernelGGL((pages_reserve_kernel<64, 1>), dim3(1), dim3(64), 0, s, a, 1);
    else if (a.B <= 1024) hipLaunchKernelGGL((pages_reserve_kernel<1024, 1>), dim3(1), dim3(1024), 0, s, a, few ? 1 : 0);
    else hipLaunchKernelGGL((pages_reserve_kernel<1024, kPagesMaxSeqs / 1024>), dim3(1), dim3(1024), 0, s, a, few ? 1 : 0);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || few) return (int)e;
    hipLaunchKernelGGL(pages_slots_kernel, dim3((a.max_tokens + 255) / 256), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

int launch_pages_live(const int32_t* rows, const int32_t* starts, int max_rows, int B, int32_t* live, hipStream_t s) {
    hipLaunchKernelGGL(pages_live_kernel, dim3((B + 255) / 256), dim3(256), 0, s, rows, starts, max_rows, B, live);
    return (int)hipGetLastError();
}

int launch_pages_append(const AppendArgs& a, int kv_dtype, hipStream_t s) {
    if (kv_elem_bytes(kv_dtype) == 1) return launch_pages_append8(a, kv_dtype, s);
    return kv_dtype == D3_F32 ? launch_append_to<float>(a, s) : launch_append_to<f16_t>(a, s);
}

int launch_pages_fill(const PagesFillArgs& a, int kv_dtype, hipStream_t s) {
    if (kv_elem_bytes(kv_dtype) == 1) return launch_fill<uint8_t>(a, s);
    return kv_dtype == D3_F32 ? launch_fill<float>(a, s) : launch_fill<f16_t>(a, s);
}

}  // namespace d3
