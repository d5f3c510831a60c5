// Decode attention over a paged cache: one new token per sequence,
//   o[b][h] = sum_j w_j V[j] / sum_j w_j,   w_j = exp(scale * q[b][h] . K[j]),   j over the rows of sequence b,
// each sequence with a length and a list of pages of its own.
//
// Work: the rows of every (sequence, KV head, 16 query heads) are cut into chunks of 64 KB of keys and values, all chunks laid end to end, and
// every workgroup (or wave, see attn_paged_kernel) takes an equal run of them, whatever the lengths: it may end one sequence, take others whole and begin another.  The host
// knows no lengths, so a launch can be captured once and replayed while sequences grow.  A run that covers a (sequence, heads) whole writes the
// result; else it publishes (max, sum, unnormalised output), and the run that arrives last joins them.
//
// Rows of 8 bits (codes8.h) come with a scale for each row: see attention_paged8.hip for what they add.
//
// Both contractions run on the matrix cores with the query heads of a KV head as one matrix dimension, straight from the registers that the
// loads fill (see pages.h for the layout of the values):
//   scores  D[row][head] = K[row][dim] q[head][dim]: a lane (i = lane % 16, g = lane / 16) loads 16 bytes of row i and ends with the scores of head i for
//           R rows that are consecutive in the cache, because row i of the instruction is cache row R (i / 4) + 4 t + i % 4 of its tile t;
//   outputs D[dim][head] += V[dim][row] w[row][head]: a lane loads the 16 bytes that hold R rows of dim i, the very rows whose weights of head i it has.
// So the head stays with lane % 16 throughout, the running maximum and sum of a softmax are the lane's own, and of what is read or weighed nothing passes through LDS before the
// four waves of a workgroup are merged at the end of a run (q does, once, to leave the registers to the rows in flight: 16 loads of 16 bytes a lane).
//
// Bound by memory where there is much of it: 32 x 2304 rows of 32 heads, fp16, 189 us = 6.4 TB/s (a pure read 6.7); 48 requests of 1 to 32768 rows of 8 heads 109 us, 6.0 TB/s.  Matrix
// and vector units are at 8 and 13 % there, so one form serves 1 to 16 query heads a KV head and both types.  Small launches are a chain of round trips: one row 5.5 us, 640 rows of 32 heads, five
// runs a head, 9.2 us: lengths 0.4, place found 0.3, tables and q 1.4, rows 1.7, turn 0.7, merge 0.7, publish, arrive and join 2.4.
#pragma once
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "codes8.h"
#include "pages.h"

namespace d3 {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

template <typename T, int HD>
struct PagedShape {
    static constexpr int ES = sizeof(T);
    static constexpr int R = 16 / ES;              // rows of a V unit
    static constexpr int RS = ES == 1 ? 4 : ES == 2 ? 3 : 2;       // R = 2^RS
    static constexpr int KT = R / 4;               // row tiles of a group of rows
    static constexpr int RG = 4 * R;               // rows of a group: one matrix instruction's worth of weights
    static constexpr int NK = HD * ES / 64;        // 16-byte loads per lane of a row tile of K
    static constexpr int ND = HD / 16;             // ... of a group's V: tiles of 16 dims
    static constexpr int U = 16 / (KT * NK + ND);  // groups of a turn: 16 loads in flight per lane
    static constexpr int TR = U * RG;              // rows of a wave's turn
    static constexpr int CH = 4 * TR;              // rows of a chunk, a turn of each wave
    static constexpr int QE = 16 / ES;             // elements of q beside a 16-byte piece of K
    static constexpr int QP = ES == 2 ? 2 * NK : ES == 1 ? 4 * NK : NK;       // 16-byte pieces of a lane's q in LDS: fp16 halves, or fp32
    // Weights are in (0, 1]; times 2^15 before they become fp16 halves, so that small ones keep their digits (fp16 counts in steps of 2^-24 at the bottom).
    static constexpr float SHIFT = ES == 2 ? 15.f : 0.f;
};

template <typename T, int HD>
struct __align__(16) PagedShared {
    float o[4][kPagedHeads][HD + 4];               // per wave: unnormalised outputs (rows 4 words apart in the banks)
    float m[kPagedHeads][4], l[kPagedHeads][4];    // per wave: running max and sum of each head
    T new_k[4][HD], new_v[4][HD];                  // per wave: the newest row as the pool holds it
    int is_last;
};

constexpr int kJoin = 16;      // partial results that one workgroup joins at a time, all of their loads in flight together
constexpr int kLeastUnit = -110;       // 8 bits: the smallest unit of weights, so that what brings them to it and back is a normal number
constexpr int kAgent = 16;     // buffer accesses at agent scope (past the XCD's own L2, like st_agent and ld_agent)

// Activations as they lie in memory (A: float, or the bits of a 16-bit type) and as fp32.  The two are apart so that all loads are requested before the first conversion waits.
template <int N, typename A>
struct ActVec {
    uint4 w[N * sizeof(A) >= 16 ? N * sizeof(A) / 16 : 1];         // N = 4 of 16 bits: half of it
    __device__ __forceinline__ void load(const A* p) {
        if constexpr (N * sizeof(A) >= 16) {
#pragma unroll
            for (int j = 0; j < (int)(N * sizeof(A) / 16); ++j) w[j] = *reinterpret_cast<const uint4*>(p + j * (16 / sizeof(A)));
        } else {
            const uint2 t = *reinterpret_cast<const uint2*>(p);
            w[0].x = t.x; w[0].y = t.y;
        }
    }
    __device__ __forceinline__ void get(int dtype, float (&y)[N]) const {
        A h[16 / sizeof(A) * sizeof(w) / 16];
        __builtin_memcpy(h, w, sizeof(w));
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (sizeof(A) == 4) y[e] = h[e];
            else y[e] = dtype == D3_BF16 ? bf16_to_f32(h[e]) : (float)__builtin_bit_cast(_Float16, h[e]);
        }
    }
};
template <typename A> __device__ __forceinline__ float act_f32(A v, int dtype) {
    if constexpr (sizeof(A) == 4) return v;
    else return dtype == D3_BF16 ? bf16_to_f32(v) : (float)__builtin_bit_cast(_Float16, v);
}
// four consecutive ones; `whole`: they lie on a multiple of their size
__device__ __forceinline__ void store_act4(void* p, long long at, int dtype, const float (&v)[4], bool whole) {
    if (dtype == D3_F32) {
        float* f = static_cast<float*>(p) + at;
        if (whole) *reinterpret_cast<float4*>(f) = make_float4(v[0], v[1], v[2], v[3]);
        else { f[0] = v[0]; f[1] = v[1]; f[2] = v[2]; f[3] = v[3]; }
        return;
    }
    uint2 w;
    if (dtype == D3_BF16) w = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
    else {
        typedef _Float16 half4 __attribute__((ext_vector_type(4)));
        w = __builtin_bit_cast(uint2, half4{(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]});
    }
    uint16_t* h = static_cast<uint16_t*>(p) + at;
    if (whole) *reinterpret_cast<uint2*>(h) = w;
    else { h[0] = (uint16_t)w.x; h[1] = (uint16_t)(w.x >> 16); h[2] = (uint16_t)w.y; h[3] = (uint16_t)(w.y >> 16); }
}

// x = hi + lo
__device__ __forceinline__ void split_half8(const float (&x)[8], half8& hi, half8& lo) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef _Float16 half2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
        const half2 h = __builtin_convertvector((f32x2{x[e], x[e + 1]}), half2);
        const half2 l = __builtin_convertvector((f32x2{x[e] - (float)h[0], x[e + 1] - (float)h[1]}), half2);
        hi[e] = h[0]; hi[e + 1] = h[1];
        lo[e] = l[0]; lo[e + 1] = l[1];
    }
}

// 16 codes as two operands
template <typename T>
__device__ __forceinline__ void decode16(const uint4& w, half8 (&y)[2]) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        half2_t lo, hi;
        decode4<T>(in[j], lo, hi);
        y[j / 2][j % 2 * 4] = lo[0]; y[j / 2][j % 2 * 4 + 1] = lo[1];
        y[j / 2][j % 2 * 4 + 2] = hi[0]; y[j / 2][j % 2 * 4 + 3] = hi[1];
    }
}
// st_agent, ld_agent of two adjacent floats
__device__ __forceinline__ void st_agent2(float* p, float x, float y) {
    __hip_atomic_store(reinterpret_cast<unsigned long long*>(p), (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 ld_agent2(const float* p) {
    const unsigned long long v = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}

__device__ __forceinline__ int scan_wave(int v) {                  // inclusive: within rows of 16 lanes, then over the rows
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);
    return v + __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);
}

// x / d where the quotient is below 2^20 (an estimate that is one off at most, and a correction): a division is 40 dependent instructions.
__device__ __forceinline__ int small_quotient(int x, int d) {
    int q = (int)((float)x * __builtin_amdgcn_rcpf((float)d));
    const int r = x - q * d;
    q += r >= d ? 1 : r < 0 ? -1 : 0;
    return __builtin_amdgcn_readfirstlane(q);
}

// Equal runs of `total` units: the first `more` workgroups have one more.  (Of the two workgroups on a compute unit the one that came first gets its loads first, so what is longer
// belongs to the first 256; runs that differ by turns took 24.0 instead of 22.6 us for 8 x 1152 rows of 8 KV heads, fp32.)
struct Runs {
    int per, more;
    __device__ Runs(int total, const Divisor& by) : per(by.of(total)), more(total - per * by.d) {}
    __device__ int begin(int w) const { return w * per + min(w, more); }
    __device__ int of(int x, int none = 0) const {                 // the run that unit x is in; none: 0, which the compiler need not know
        const int larger = more * (per + 1), each = per + none;
        return x < larger ? small_quotient(x, each + 1) : more + small_quotient(x - larger, max(each, 1));    // per = 0: every unit is below `larger`
    }
};

// What the first loads need of the arguments, requested together (see attn_take_args).
__device__ __forceinline__ void paged_take_args(const PagedAttnArgs& a) {
    asm volatile("" :: "s"(a.q), "s"(a.k_new), "s"(a.v_new), "s"(a.q_stride), "s"(a.kv_stride), "s"(a.rope_cs), "s"(a.tables), "s"(a.rows), "s"(a.table_stride),
                       "s"(a.max_rows), "s"(a.B), "s"(a.H_kv), "s"(a.group), "s"(a.n_pages), "s"(a.page_shift), "s"(a.k_pages), "s"(a.v_pages));
    asm volatile("" :: "s"(a.dtype), "s"(a.scale), "s"(a.out), "s"(a.out_stride), "s"(a.out_split), "s"(a.out_form.lo), "s"(a.part_o), "s"(a.part_ml), "s"(a.tickets), "s"(a.by_runs.d), "s"(a.by_runs.m));
}

// What is known of the lengths before the work is divided.
struct Lengths {
    int chunks, turns, live;                                        // chunks (four waves' turns) and turns (one's) of all sequences; sequences that have rows
    float shortest;                                                 // rows of the shortest of these (to 24 bits)
    int own;                                                        // the length of sequence `lane`
};
template <typename P, typename Length>
__device__ __forceinline__ Lengths take_lengths(int B, int lane, Length length) {
    Lengths n = {0, 0, 0, 0x1p30f, lane < B ? length(lane) : 0};
    auto take = [&](int len) {
        n.chunks += (len + P::CH - 1) / P::CH;
        n.turns += (len + P::TR - 1) / P::TR;
        n.live += __popcll(__ballot(len > 0));
        n.shortest = fminf(n.shortest, len > 0 ? (float)len : 0x1p30f);
    };
    take(n.own);
    for (int b0 = 64; b0 < B; b0 += 512) {                          // eight of a lane's in flight (3000 sequences of one KV head 65 -> 52 us)
        int len[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) len[j] = length(min(b0 + j * 64 + lane, B - 1));
#pragma unroll
        for (int j = 0; j < 8; ++j) take(b0 + j * 64 + lane < B ? len[j] : 0);
    }
    n.chunks = __builtin_amdgcn_readlane(scan_wave(n.chunks), 63);
    n.turns = __builtin_amdgcn_readlane(scan_wave(n.turns), 63);
    n.shortest = -reduce_row(reduce_row_pairs(reduce_halves(-n.shortest, MaxOp()), MaxOp()), MaxOp());
    n.shortest = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(n.shortest)));
    return n;
}

// T: the pool's type; A: float, or the bits of a 16-bit type (q, k_new, v_new).  WAVES: a chunk is one wave's turn and a run a wave's; else a chunk is a turn of each of the four waves of a
// workgroup, whose run it is.
template <typename T, int HD, typename A, bool WAVES, typename Length>
__device__ __forceinline__ void attn_paged_runs(const PagedAttnArgs& a, PagedShared<T, HD>& sh, const Lengths& lengths, Length length) {
    typedef PagedShape<T, HD> P;
    constexpr int R = P::R, KT = P::KT, RG = P::RG, NK = P::NK, ND = P::ND, U = P::U, QE = P::QE, CH = WAVES ? P::TR : P::CH;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int H = a.H_kv * a.group, tiles = (a.group + kPagedHeads - 1) / kPagedHeads, HH = a.H_kv * tiles, GP = min(a.group, kPagedHeads);
    const Divisor& by_runs = WAVES ? a.by_waves : a.by_runs;

    // ---- this run of units, and where it begins ----
    // A (sequence, heads) counts as its chunks, and where runs are longer than the shortest one, i.e. may hold several, as `over` more: what beginning
    // and ending it costs (48 requests of 1 to 32768 rows 130 -> 110 us).  Elsewhere that would only make runs uneven (20480 rows, 32 heads: 160 chunks are 10 a workgroup; 57.8 us, with `over` 62.3).
    auto chunks_of = [&](int len) { return (len + CH - 1) / CH; };
    const int chunks_in_all = WAVES ? lengths.turns : lengths.chunks;
    const int over = (float)(chunks_in_all * HH) > (float)by_runs.d * (float)chunks_of((int)lengths.shortest) ? kPagedOverhead : 0, total = (chunks_in_all + lengths.live * over) * HH;
    if (lengths.live < a.B) {
        for (int b = blockIdx.x; b < a.B; b += gridDim.x) {         // a sequence without rows: zeros
            if (length(b) > 0) continue;
            const float zero[4] = {0.f, 0.f, 0.f, 0.f};
            for (int e = tid * 4; e < H * HD; e += 1024) {
                store_act4(a.out, b * a.out_stride + e, a.dtype, zero, false);
                if (a.out_split) store_split4(a.out_split + b * a.out_form.pitch(H * HD), e, zero, a.out_form.lo);
            }
        }
    }
    if (total == 0) return;
    const Runs runs(total, by_runs);
    const int run = WAVES ? blockIdx.x * 4 + wave : blockIdx.x, end = runs.begin(run + 1);
    int u = runs.begin(run);
    if (u >= end) return;
    int b = 0, seq_begin = 0, len = 0;                              // the sequence of unit u, its first unit and its rows
    auto units_of = [&](int len) { return len > 0 ? (chunks_of(len) + over) * HH : 0; };
    if (a.B <= 64) {
        const int n = units_of(lengths.own), upto = scan_wave(n);
        b = __builtin_ctzll(__ballot(upto > u));
        seq_begin = __builtin_amdgcn_readlane(upto, b) - __builtin_amdgcn_readlane(n, b);
        len = __builtin_amdgcn_readlane(lengths.own, b);
    } else {
        for (int b0 = 0, before = 0;; b0 += 512) {                  // a lane has eight sequences one after the other
            int n = 0, lens[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) lens[j] = length(min(b0 + lane * 8 + j, a.B - 1));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (b0 + lane * 8 + j >= a.B) lens[j] = 0;
                n += units_of(lens[j]);
            }
            const int upto = before + scan_wave(n);
            const unsigned long long past = __ballot(upto > u);
            if (past) {
                const int at = __builtin_ctzll(past);
                seq_begin = __builtin_amdgcn_readlane(upto - n, at);
                b = b0 + at * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) {                       // (the one that holds u, then no longer another)
                    const int x = __builtin_amdgcn_readlane(lens[j], at), here = units_of(x);
                    if (len == 0 && here > u - seq_begin) len = x;
                    if (len == 0) { seq_begin += here; ++b; }
                }
                break;
            }
            before = __builtin_amdgcn_readlane(upto, 63);
        }
    }

    const int block_shift = a.page_shift - P::RS, block_mask = (1 << block_shift) - 1;      // blocks of R rows
    const size_t head_bytes = ((size_t)HD * P::ES) << a.page_shift, page_bytes = head_bytes * a.H_kv;
    const bool out_whole = reinterpret_cast<uintptr_t>(a.out) % 16 == 0 && a.out_stride % 4 == 0;

    while (u < end) {
        // 8 bits: what the loads of a (sequence, heads) need of the lane's number is computed here, not ahead of all of them, where it would be kept and others spilled
        int self = tid, zero = 0;
        if constexpr (P::ES == 1) {
            asm volatile("" : "+v"(self));
            asm volatile("" : "+s"(zero));
        }
        const int lane = self & 63, i = lane & 15, g = lane >> 4;
        const int chunks = chunks_of(len), per_head = chunks + over, hh = small_quotient(u - seq_begin, per_head), head_begin = seq_begin + hh * per_head;
        const int c0 = max(u - head_begin - over, 0), c1 = min(chunks, end - head_begin - over);
        const int next = min(end, head_begin + per_head);
        if (c1 <= 0) return;                                        // the run ends in what this one counts more
        const int kvh = tiles == 1 ? hh : small_quotient(hh, tiles + zero), h0 = (hh - kvh * tiles) * kPagedHeads, nh = min(kPagedHeads, a.group - h0);
        const bool whole = c0 == 0 && c1 == chunks;
        const int newest = len - 1, last_block = newest / R;
        const int* tab = a.tables + (size_t)b * a.table_stride;
        char* Kh = static_cast<char*>(a.k_pages) + kvh * head_bytes;
        char* Vh = static_cast<char*>(a.v_pages) + kvh * head_bytes;
        float *Ks = nullptr, *Vs = nullptr;                         // scales of the head's rows, a page's page_rows * H_kv apart
        if constexpr (P::ES == 1) {
            Ks = a.k_scales + ((size_t)kvh << a.page_shift);
            Vs = a.v_scales + ((size_t)kvh << a.page_shift);
        }
        // This wave's turns: rows first, first + CH, ... last, in a circle that begins at another place in every workgroup.  (Sequences whose pages lie a power of two apart, 64 pages
        // each, are at the same place of their memory channels in every row; workgroups that walk them in step meet there.)
        const int row0 = WAVES ? 0 : wave * P::TR, first = c0 * CH + row0, turns = c1 - c0 - ((c1 - 1) * CH + row0 >= len ? 1 : 0), last = first + (turns - 1) * CH;
        int r = first;
        if (turns >= 4) r += (run - small_quotient(run, turns) * turns) * CH;       // (a few turns do not meet for long)
        auto after = [&](int row) { return row == last ? first : row + CH; };

        uint4 kr[U][KT][NK], vr[U][ND];
        float ksr[U], vsr[U];                                       // 8 bits: scales of row `lane` of each group, which are rows 16 g + i
        // pages of the blocks of R rows that a lane loads of K and of V; blocks past the last are read as the last
        auto load_pages = [&](int row, int (&pk)[U], int (&pv)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                pk[x] = tab[min((row + x * RG) / R + (i >> 2), last_block) >> block_shift];
                pv[x] = tab[min((row + x * RG) / R + g, last_block) >> block_shift];
            }
        };
        auto present = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
        auto scale_at = [&](const float* scales, int page, int blk) {
            return scales + ((size_t)(present(page) ? page : 0) * a.H_kv << a.page_shift) + (blk & block_mask) * R + i;
        };
        auto issue_k = [&](int row, const int (&pk)[U], const int (&pv)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int blk = min((row + x * RG) / R + (i >> 2), last_block) & block_mask;
                const char* p = Kh + (present(pk[x]) ? pk[x] : 0) * page_bytes + (blk * R + (i & 3)) * (HD * P::ES) + g * 16;
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int k = 0; k < NK; ++k) kr[x][t][k] = __builtin_bit_cast(uint4, load_stream16(p + t * 4 * HD * P::ES + k * 64));
                if constexpr (P::ES == 1) ksr[x] = *scale_at(Ks, pv[x], min((row + x * RG) / R + g, last_block));
            }
        };
        auto issue_v = [&](int row, const int (&pv)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int blk = min((row + x * RG) / R + g, last_block) & block_mask;
                const char* p = Vh + (present(pv[x]) ? pv[x] : 0) * page_bytes + blk * (HD * 16) + i * 16;
#pragma unroll
                for (int d = 0; d < ND; ++d) vr[x][d] = __builtin_bit_cast(uint4, load_stream16(p + d * 256));
                if constexpr (P::ES == 1) vsr[x] = *scale_at(Vs, pv[x], min((row + x * RG) / R + g, last_block));
            }
        };
        // the wave whose turn has the newest row rounds it as the pool does, and puts it into its page
        const bool fresh = a.k_new && c1 == chunks && (WAVES || (newest / P::TR & 3) == wave);
        float m = -INFINITY, l = 0.f;
        // 8 bits: a weight goes into the products with its row's scale, w = exp2(score - m) * scale, in units of 2^(unit - 16) where 2^unit is more than the largest so far, as fp16 halves need it.  unit is a
        // whole number: what brings sums from one to another is exact.
        int unit_w = kLeastUnit;
        float new_ks = 0.f, new_vs = 0.f;
        f32x4 acc[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (turns > 0) {
            int pk[U], pv[U], pk1[U], pv1[U], new_page = 0;
            load_pages(r, pk, pv);
            if (fresh) new_page = tab[last_block >> block_shift];
            float qf[NK][QE];
            ActVec<QE, A> qa[NK];
#pragma unroll
            for (int k = 0; k < NK; ++k) qa[k].load(static_cast<const A*>(a.q) + b * a.q_stride + (long long)(kvh * a.group + h0 + min(i, nh - 1)) * HD + k * 4 * QE + g * QE);
            // a lane has dims k * 4 QE + g * QE ... of q, k < NK: those half a head away, with which they turn, among them (of one piece, 64 dims in 8 bits, they are lane ^ 32's)
            constexpr int NC = NK == 1 ? 1 : NK / 2;
            ActVec<2 * QE, float> cs[NC];
            if (a.rope_cs) {
#pragma unroll
                for (int k = 0; k < NC; ++k) cs[k].load(reinterpret_cast<const float*>(a.rope_cs + (size_t)b * (HD / 2) + (NK == 1 ? (g & 1) * QE : k * 4 * QE + g * QE)));
            }
            load_pages(after(r), pk1, pv1);
            A nk[2], nv[2];                                         // dims `lane` and lane + HD / 2 of the newest row
            float2 ncs = {1.f, 0.f};
            uint4 unit[2];                                          // and the values beside it: R rows share 16 bytes
            char* unit_at = Vh;
            if (fresh) {
                const long long at = b * a.kv_stride + (long long)kvh * HD + lane % (HD / 2);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    nk[e] = static_cast<const A*>(a.k_new)[at + e * (HD / 2)];
                    nv[e] = static_cast<const A*>(a.v_new)[at + e * (HD / 2)];
                }
                if (a.rope_cs) ncs = a.rope_cs[(size_t)b * (HD / 2) + lane % (HD / 2)];
                unit_at += (size_t)(present(new_page) ? new_page : 0) * page_bytes + ((last_block & block_mask) * HD + lane % (HD / 2)) * 16;
#pragma unroll
                for (int e = 0; e < 2; ++e) unit[e] = *reinterpret_cast<const uint4*>(unit_at + e * (HD * 8));
            }
            __builtin_amdgcn_sched_barrier(0);
            issue_k(r, pk, pv);
            issue_v(r, pv);
            __builtin_amdgcn_sched_barrier(0);
            if (P::ES == 1 && fresh) {
                if constexpr (P::ES == 1) {                         // (with hd 64 the lanes of the upper half do as those of the lower)
                    float y[2] = {act_f32(nk[0], a.dtype), act_f32(nk[1], a.dtype)}, z[2] = {act_f32(nv[0], a.dtype), act_f32(nv[1], a.dtype)};
                    if (a.rope_cs) turned(y[0], y[1], ncs);
                    auto most = [&](const float (&x)[2]) {
                        const MaxMagnitude op;
                        return reduce_halves(reduce_row_pairs(reduce_row(op(magnitude(x[0]), magnitude(x[1])), op), op), op);
                    };
                    const RowScale sk = row_scale<T>(most(y)), sv = row_scale<T>(most(z));
                    new_ks = sk.scale; new_vs = sv.scale;
                    const float yk[2] = {y[0] * sk.inv, y[1] * sk.inv}, zv[2] = {z[0] * sv.inv, z[1] * sv.inv};
                    uint32_t kc[1], vc[1];
                    encode<T, 2>(yk, kc);
                    encode<T, 2>(zv, vc);
                    const bool put = h0 == 0 && present(new_page);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int d = lane % (HD / 2) + e * (HD / 2);
                        const T kt = {(uint8_t)(kc[0] >> 8 * e)}, vt = {(uint8_t)(vc[0] >> 8 * e)};
                        sh.new_k[wave][d] = kt; sh.new_v[wave][d] = vt;
                        if (put) {
                            reinterpret_cast<T*>(Kh + new_page * page_bytes)[(newest & ((1 << a.page_shift) - 1)) * HD + d] = kt;
                            uint32_t rows[4];
                            __builtin_memcpy(rows, &unit[e], 16);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t at = 0xffu << (newest % 4 * 8);
                                if (newest % R / 4 == j) rows[j] = (rows[j] & ~at) | (vt.bits * 0x01010101u & at);
                            }
                            __builtin_memcpy(unit_at + e * (HD * 8), rows, 16);
                        }
                    }
                    if (put && lane == 0) {
                        const size_t at = ((size_t)new_page * a.H_kv << a.page_shift) + (newest & ((1 << a.page_shift) - 1));
                        Ks[at] = new_ks;
                        Vs[at] = new_vs;
                    }
                }
            }
            if constexpr (P::ES > 1) if (fresh) {
                if (lane < HD / 2) {
                    const float k0 = act_f32(nk[0], a.dtype), k1 = act_f32(nk[1], a.dtype);
                    const float y[2] = {k0 * ncs.x - k1 * ncs.y, k1 * ncs.x + k0 * ncs.y}, z[2] = {act_f32(nv[0], a.dtype), act_f32(nv[1], a.dtype)};
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int d = lane + e * (HD / 2);
                        const T kt = held<T>(y[e]), vt = held<T>(z[e]);
                        sh.new_k[wave][d] = kt; sh.new_v[wave][d] = vt;
                        if (h0 == 0 && present(new_page)) {
                            reinterpret_cast<T*>(Kh + new_page * page_bytes)[(newest & ((1 << a.page_shift) - 1)) * HD + d] = kt;
                            T rows[R];
                            __builtin_memcpy(rows, &unit[e], 16);
#pragma unroll
                            for (int j = 0; j < R; ++j) if (newest % R == j) rows[j] = vt;
                            // whole lines (two bytes of every 16 would be 5 us of 190 with 1024 of these)
                            __builtin_memcpy(unit_at + e * (HD * 8), rows, 16);
                        }
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < NK; ++k) qa[k].get(a.dtype, qf[k]);
            if (a.rope_cs) {
#pragma unroll
                for (int k = 0; k < NC; ++k) {
                    float c[2 * QE];
                    cs[k].get(D3_F32, c);
#pragma unroll
                    for (int e = 0; e < QE; ++e) {
                        if constexpr (NK == 1) {
                            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(qf[0][e]), __float_as_uint(qf[0][e]), false, false);
                            const float lo = __uint_as_float(both[0]), hi = __uint_as_float(both[1]);
                            qf[0][e] = g < 2 ? lo * c[2 * e] - hi * c[2 * e + 1] : hi * c[2 * e] + lo * c[2 * e + 1];
                        } else {
                            const float lo = qf[k][e], hi = qf[k + NC][e];
                            qf[k][e] = lo * c[2 * e] - hi * c[2 * e + 1];
                            qf[k + NC][e] = hi * c[2 * e] + lo * c[2 * e + 1];
                        }
                    }
                }
            }
            // q as fp16 halves hi + lo, scaled by a power of two that puts its largest element at 2^14: 22 bits of it
            float mul = P::ES == 1 ? a.scale_part : a.scale * 1.4426950408889634f;    // scores are kept in units of log2(e): every exponential is one hardware exp2
            bool far = false;
            // In LDS from here on (where this wave puts its outputs in the end): in registers it would leave too few for the rows in flight.
            uint4* const q_lds = reinterpret_cast<uint4*>(sh.o[wave]) + lane;
            if constexpr (P::ES <= 2) {
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int e = 0; e < QE; ++e) top = fmaxf(top, fabsf(qf[k][e]));
                top = reduce_halves(reduce_row_pairs(top, MaxOp()), MaxOp());
                const int ex = 15 - __builtin_amdgcn_frexp_expf(top);
#pragma unroll
                for (int k = 0; k < NK; ++k) {
#pragma unroll
                    for (int e = 0; e < QE; ++e) qf[k][e] = __builtin_ldexpf(qf[k][e], ex);
#pragma unroll
                    for (int e = 0; e < QE; e += 8) {
                        float part[8];
                        half8 hi, lo;
                        __builtin_memcpy(part, &qf[k][e], 32);
                        split_half8(part, hi, lo);
                        const int at = (k * QE + e) / 4;            // hi at piece 2 (k QE + e) / 8, lo behind it
                        q_lds[at * 64] = __builtin_bit_cast(uint4, hi);
                        q_lds[(at + 1) * 64] = __builtin_bit_cast(uint4, lo);
                    }
                }
                if constexpr (P::ES == 1) {
                    // Codes have at most 2^31 in a product with q, and scales of rows 2^121: with 2^-120 to 2^95 ahead of the row's scale (all there is to it, but for queries or a scale far from one) mul is a normal
                    // number and only a score that is too large for fp32 overflows.  The rest, `far`, goes by head into LDS, where sums come at the end, and is left out where no head has any.
                    const int all = a.scale_exp - ex, near = min(max(all, -120), 95);
                    mul = __builtin_ldexpf(mul, near);
                    far = __any(all != near);
                    if (g == 0) sh.l[i][wave] = __int_as_float(all - near);
                } else mul = __builtin_ldexpf(mul, -ex);
            } else {
#pragma unroll
                for (int k = 0; k < NK; ++k) __builtin_memcpy(&q_lds[k * 64], qf[k], 16);
            }
            static_assert(P::QP * 64 * 16 <= sizeof(sh.o[0]), "");

            auto turn = [&](auto more_) {
                constexpr bool MORE = decltype(more_)::value;       // another turn follows
                const int next_r = after(r);
                const bool tail = r + P::TR >= len;                 // holds the newest row, or rows past it
                const bool with_new = fresh && tail && r <= newest;
                bool absent = false;                                // a page that is none: its rows do not count
#pragma unroll
                for (int x = 0; x < U; ++x) absent = absent || !present(pv[x]);
                absent = __any(absent);
                if (with_new) {                                     // the newest row's key takes its place among the rows
#pragma unroll
                    for (int x = 0; x < U; ++x)
#pragma unroll
                        for (int t = 0; t < KT; ++t) {
                            if (newest - r - x * RG - R * (i >> 2) - (i & 3) != 4 * t) continue;
#pragma unroll
                            for (int k = 0; k < NK; ++k) __builtin_memcpy(&kr[x][t][k], &sh.new_k[wave][k * 4 * QE + g * QE], 16);
                        }
                }
                const uint4* q_at = q_lds;
                int none = 0;                                       // (read again in every turn: the compiler cannot know that it is 0)
                asm volatile("" : "+v"(none));
                q_at += none;
                uint4 qr[P::QP];
#pragma unroll
                for (int k = 0; k < P::QP; ++k) qr[k] = q_at[k * 64];
                float s[U][R];
                if constexpr (P::ES == 1) {
                    // hi and lo in one sum a tile, a group's tiles side by side; mul ahead of the row's scale
#pragma unroll
                    for (int x = 0; x < U; ++x) {
                        if (with_new && r + x * RG + lane == newest) ksr[x] = new_ks;
                        f32x4 d[KT] = {};
#pragma unroll
                        for (int k = 0; k < NK; ++k) {
                            half8 kv[KT][2];
#pragma unroll
                            for (int t = 0; t < KT; ++t) decode16<T>(kr[x][t][k], kv[t]);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int t = 0; t < KT; ++t) d[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv[t][e / 2], __builtin_bit_cast(half8, qr[4 * k + e]), d[t], 0, 0, 0);
                        }
                        of_rows(ksr[x], [&](int e, float scale) { s[x][e] = d[e / 4][e % 4] * mul * scale; });
                    }
                    if (far) {
                        const int more = __float_as_int(sh.l[lane & 15][wave]);
#pragma unroll
                        for (int x = 0; x < U; ++x)
#pragma unroll
                            for (int e = 0; e < R; ++e) s[x][e] = __builtin_ldexpf(s[x][e], more);
                    }
                } else
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        f32x4 d = {0.f, 0.f, 0.f, 0.f}, d1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < NK; ++k) {
                            if constexpr (P::ES == 2) {
                                const half8 kv = __builtin_bit_cast(half8, kr[x][t][k]);
                                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, __builtin_bit_cast(half8, qr[2 * k]), d, 0, 0, 0);
                                d1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, __builtin_bit_cast(half8, qr[2 * k + 1]), d1, 0, 0, 0);
                            } else {
                                const f32x4 kv = __builtin_bit_cast(f32x4, kr[x][t][k]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if (e & 1) d1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], __builtin_bit_cast(f32x4, qr[k])[e], d1, 0, 0, 0);
                                    else d = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], __builtin_bit_cast(f32x4, qr[k])[e], d, 0, 0, 0);
                                }
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[x][4 * t + j] = (d[j] + d1[j]) * mul;
                    }
                __builtin_amdgcn_sched_barrier(0);
                int pk2[U], pv2[U];
                if constexpr (MORE) {
                    load_pages(after(next_r), pk2, pv2);
                    issue_k(next_r, pk1, pv1);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (tail || absent) {
#pragma unroll
                    for (int x = 0; x < U; ++x) {
                        const int left = present(pv[x]) ? len - r - x * RG - R * g : 0;         // of the lane's R rows those that count
#pragma unroll
                        for (int e = 0; e < R; ++e) if (e >= left) s[x][e] = -INFINITY;
                    }
                }
                // ---- running softmax of head i over the lane's rows (and, for the maximum, those of the other lanes that have the head) ----
                float top = s[0][0];
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int e = 0; e < R; ++e) top = fmaxf(top, s[x][e]);
                top = fmaxf(m, reduce_halves(reduce_row_pairs(top, MaxOp()), MaxOp()));
                float kept = 1.f;                                   // 8 bits: what the sums keep, 1/2 to 1 times a power of two that goes to l and to the unit
                if constexpr (P::ES == 1) {                         // (beside the exponentials, without a branch of its own)
                    const float grown = m > -INFINITY ? fminf(top - m, 1e6f) : 0.f, whole = floorf(grown);
                    kept = __builtin_amdgcn_exp2f(whole - grown);
                    l = __builtin_ldexpf(l * kept, -(int)whole);
                    unit_w -= (int)whole;
                    m = top;
                } else if (__any(top > m)) {
                    const float f = top > m ? __builtin_amdgcn_exp2f(m - top) : 1.f;
                    l *= f;
#pragma unroll
                    for (int d = 0; d < ND; ++d) acc[d] *= f;
                    m = top;
                }
                const float sub = m > -INFINITY ? m - P::SHIFT : 0.f;
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int e = 0; e < R; ++e) {
                        s[x][e] = __builtin_amdgcn_exp2f(s[x][e] - sub);
                        l += s[x][e];
                    }
                if constexpr (P::ES == 1) {
                    float most = 0.f;
#pragma unroll
                    for (int x = 0; x < U; ++x) {
                        if (with_new && r + x * RG + lane == newest) vsr[x] = new_vs;
                        if ((tail || absent) && (!present(pv[x]) || r + x * RG + lane >= len)) vsr[x] = 0.f;       // (of a row that does not count: anything)
                        of_rows(vsr[x], [&](int e, float scale) {
                            s[x][e] *= scale;
                            most = fmaxf(most, fabsf(s[x][e]));
                        });
                    }
                    most = reduce_halves(reduce_row_pairs(most, MaxOp()), MaxOp());
                    // the largest weight becomes 65504 at most (fp16's largest) and 32752 at least
                    const int larger = max(max(unit_w, most > 0.f ? __builtin_amdgcn_frexp_expf(most * (1.f + 0x1p-11f)) : kLeastUnit), kLeastUnit);
                    if (__any(kept < 1.f || larger > unit_w)) {
                        const float f = __builtin_ldexpf(kept, unit_w - larger);
#pragma unroll
                        for (int d = 0; d < ND; ++d) acc[d] *= f;
                        unit_w = larger;
                    }
                    const float by = __builtin_ldexpf(1.f, 16 - unit_w);
#pragma unroll
                    for (int x = 0; x < U; ++x)
#pragma unroll
                        for (int e = 0; e < R; ++e) s[x][e] *= by;
                }
                if (tail || absent) {
                    // Rows that do not count hold anything: 0 times it must be 0.  Bits of a lane's R rows in the four words of a unit, the same in all its units.
                    constexpr int PER = 4 / P::ES;                  // rows of a word
                    constexpr uint32_t ROW = PER == 4 ? 0xffu : PER == 2 ? 0xffffu : 0xffffffffu;
#pragma unroll
                    for (int x = 0; x < U; ++x) {
                        const int left = present(pv[x]) ? len - r - x * RG - R * g : 0, fresh_at = newest - r - x * RG - R * g;
                        uint32_t counts[4], fresh_bits[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            if constexpr (P::ES == 1) {             // bytes 0 .. left - 1, and byte fresh_at, of 16
                                const int n = max(left - 4 * j, 0);
                                counts[j] = n >= 4 ? ~0u : (1u << (8 * n & 31)) - 1;
                                fresh_bits[j] = fresh_at >> 2 == j ? 0xffu << (8 * fresh_at & 31) : 0u;
                                continue;
                            }
                            counts[j] = fresh_bits[j] = 0;
#pragma unroll
                            for (int e = 0; e < PER; ++e) {
                                counts[j] |= j * PER + e < left ? ROW << (8 * P::ES * e) : 0u;
                                fresh_bits[j] |= j * PER + e == fresh_at ? ROW << (8 * P::ES * e) : 0u;
                            }
                        }
                        if (with_new) {                             // the newest row's value takes its place
#pragma unroll
                            for (int d = 0; d < ND; ++d) {
                                uint32_t own = 0;
                                __builtin_memcpy(&own, &sh.new_v[wave][d * 16 + i], P::ES);
                                if (PER == 2) own |= own << 16;
                                if (PER == 4) own = __builtin_amdgcn_perm(own, own, 0u);
                                vr[x][d].x = (fresh_bits[0] & own) | (~fresh_bits[0] & vr[x][d].x);
                                vr[x][d].y = (fresh_bits[1] & own) | (~fresh_bits[1] & vr[x][d].y);
                                vr[x][d].z = (fresh_bits[2] & own) | (~fresh_bits[2] & vr[x][d].z);
                                vr[x][d].w = (fresh_bits[3] & own) | (~fresh_bits[3] & vr[x][d].w);
                            }
                        }
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            vr[x][d].x &= counts[0]; vr[x][d].y &= counts[1]; vr[x][d].z &= counts[2]; vr[x][d].w &= counts[3];
                        }
                    }
                }
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    if constexpr (P::ES == 1) {
                        __builtin_amdgcn_sched_barrier(0);
                        half8 ph[2], pl[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float part[8];
                            __builtin_memcpy(part, &s[x][8 * e], 32);
                            split_half8(part, ph[e], pl[e]);
                        }
#pragma unroll
                        for (int d0 = 0; d0 < ND; d0 += 4) {        // four sums side by side: a product waits for the one before it of its own sum
                            half8 v[4][2];
#pragma unroll
                            for (int d = 0; d < 4; ++d) decode16<T>(vr[x][d0 + d], v[d]);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int d = 0; d < 4; ++d) acc[d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[d][e / 2], e % 2 ? pl[e / 2] : ph[e / 2], acc[d0 + d], 0, 0, 0);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    } else if constexpr (P::ES == 2) {
                        half8 ph, pl;
                        split_half8(s[x], ph, pl);
#pragma unroll
                        for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, vr[x][d]), ph, acc[d], 0, 0, 0);
#pragma unroll
                        for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, vr[x][d]), pl, acc[d], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < R; ++e)
#pragma unroll
                            for (int d = 0; d < ND; ++d) acc[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(f32x4, vr[x][d])[e], s[x][e], acc[d], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (MORE) {
                    issue_v(next_r, pv1);
                    r = next_r;
#pragma unroll
                    for (int x = 0; x < U; ++x) { pv[x] = pv1[x]; pk1[x] = pk2[x]; pv1[x] = pv2[x]; }
                }
            };
            for (int more = turns; more > 1; --more) turn(std::true_type());
            turn(std::false_type());
            if constexpr (P::ES == 1) {
                const float f = __builtin_ldexpf(1.f, unit_w - 16);
#pragma unroll
                for (int d = 0; d < ND; ++d) acc[d] *= f;
            }
            l = reduce_halves(reduce_row_pairs(l, AddOp()), AddOp());
        }

        // ---- merge the waves ----
        asm volatile("" ::: "memory");                              // outputs take the place of q
        // From here on addresses are computed where they are used (the compiler cannot know that `none` and `still` are 0 and tid): ahead of the loop over (sequence, heads), where it
        // would compute them, every launch waits for them before its first load, and they spill.
        int none = 0, still = tid;
        asm volatile("" : "+s"(none));
        asm volatile("" : "+v"(still));
        const int H_ = H + none, HH_ = HH + none, GP_ = GP + none;
        if (const int i = still & 15, g = (still & 63) >> 4; !WAVES && i < nh) {
            if (g == 0) { sh.m[i][wave] = m; sh.l[i][wave] = l; }
#pragma unroll
            for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(&sh.o[wave][i][d * 16 + g * 4]) = acc[d];
        }
        if (!WAVES) __syncthreads();
        // Partial results of a (sequence, heads) are those of runs w0 .. w1.  A run has at most two: in slot 2 run of the one that it begins in, in the next of the one that it ends in.
        int w0 = run, parts = 1;
        if (!whole) {
            w0 = runs.of(head_begin + over, P::ES == 1 ? none : 0);
            parts = runs.of(head_begin + per_head - 1, P::ES == 1 ? none : 0) - w0 + 1;
        }
        const unsigned before = runs.begin(w0) < head_begin ? 1 : 0;
        auto slot_of = [&](int k) { return 2u * (w0 + k) + (k == 0 ? before : 0); };
        const int items = nh * (HD / 4);                            // a thread has four dims of a head
        auto finish = [&](int h, int t, const float (&o)[4], float sum) {
            const float by = sum == 0.f ? 0.f : 1.f / sum;          // no row counted: zeros
            const float v[4] = {o[0] * by, o[1] * by, o[2] * by, o[3] * by};
            const int e = (kvh * a.group + h0 + h) * HD + t;
            store_act4(a.out, b * a.out_stride + e, a.dtype, v, out_whole);
            if (a.out_split) store_split4(a.out_split + b * a.out_form.pitch(H_ * HD), e, v, a.out_form.lo);
        };
        // 16 bytes an access (two of 8, a head at a time: 64 x 1000 rows of one KV head, 16 query heads, 19.1 us; so 15.6); 32-bit offsets, the partial results of all runs are 32 MiB at most
        const auto part_buf = __builtin_amdgcn_make_buffer_rsrc(a.part_o + none, 0, 2 * by_runs.d * GP_ * (HD * 4), 0x00027000);
        auto part_ml_at = [&](unsigned slot, int h) { return reinterpret_cast<float*>(reinterpret_cast<char*>(a.part_ml) + (slot * GP_ + h) * 8u); };
        auto publish_o = [&](unsigned slot, int h, int t, const float (&o)[4]) {
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{o[0], o[1], o[2], o[3]}), part_buf, (h * HD + t) * 4, slot * GP_ * (HD * 4), kAgent);
        };
        auto publish_ml = [&](unsigned slot, int h, float M, float L) { st_agent2(part_ml_at(slot, h), M, L); };
        if constexpr (!WAVES) {
            for (int idx = still; idx < items; idx += 256) {
                const int h = idx / (HD / 4), t = idx % (HD / 4) * 4;
                const f32x4 ms = *reinterpret_cast<const f32x4*>(sh.m[h]), ls = *reinterpret_cast<const f32x4*>(sh.l[h]);
                f32x4 x[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) x[w] = *reinterpret_cast<const f32x4*>(&sh.o[w][h][t]);
                const float M = fmaxf(fmaxf(ms[0], ms[1]), fmaxf(ms[2], ms[3]));
                float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float f = ms[w] > -INFINITY ? __builtin_amdgcn_exp2f(ms[w] - M) : 0.f;
                    L += ls[w] * f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] += x[w][e] * f;
                }
                if (whole) finish(h, t, o, L);
                else {
                    publish_o(slot_of(run - w0), h, t, o);
                    if (t == 0) publish_ml(slot_of(run - w0), h, M, L);
                }
            }
        } else if (const int i = still & 15, g = (still & 63) >> 4; i < nh) {       // a lane has the head, four dims of each tile
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const float o[4] = {acc[d][0], acc[d][1], acc[d][2], acc[d][3]};
                if (whole) finish(i, d * 16 + g * 4, o, l);
                else publish_o(slot_of(run - w0), i, d * 16 + g * 4, o);
            }
            if (!whole && g == 0) publish_ml(slot_of(run - w0), i, m, l);
        }
        auto join_all = [&](auto threads_) {
            constexpr int THREADS = decltype(threads_)::value, ITEMS = kPagedHeads * (HD / 4) / THREADS;
            const int self = still & (THREADS - 1), column = THREADS == 64 ? wave : 0;
            // The run that arrives last joins them; more than kJoin in two rounds: the last of every kJoin joins these, the last of all joins what they give.
            auto arrive = [&](int* ticket, int of) {
                wait_stores();
                if constexpr (THREADS == 256) {
                    __syncthreads();
                    if (still == 0) {
                        sh.is_last = atomicAdd(ticket, 1) == of - 1;
                        if (sh.is_last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // all arrived: leave it clean
                    }
                    __syncthreads();
                    return sh.is_last != 0;
                } else {
                    int is_last = 0;
                    if (self == 0) {
                        is_last = atomicAdd(ticket, 1) == of - 1;
                        if (is_last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    }
                    is_last = __builtin_amdgcn_readfirstlane(is_last);
                    asm volatile("" ::: "memory");
                    return is_last != 0;
                }
            };
            // done(h, t, o, M, L) of every item of this thread, four dims from t on of head h: J partial results of N items in flight
            auto join = [&](auto flight, auto items_at_once, int first, int step, int count, auto done) {
                constexpr int J = decltype(flight)::value, N = decltype(items_at_once)::value;
                auto some = [&](int begin) {
                    int at[N], h[N];
                    float M[N], L[N], o[N][4];
#pragma unroll
                    for (int n = 0; n < N; ++n) {
                        const int idx = min(begin + n * THREADS, items - 1);
                        h[n] = idx / (HD / 4); at[n] = idx * 16;
                        M[n] = -INFINITY; L[n] = o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
                    }
                    for (int k0 = 0; k0 < count; k0 += J) {
                        float2 ml[N][J];
                        f32x4 x[N][J];
#pragma unroll
                        for (int k = 0; k < J; ++k) {
                            const unsigned slot = slot_of(first + min(k0 + k, count - 1) * step);
#pragma unroll
                            for (int n = 0; n < N; ++n) {
                                ml[n][k] = ld_agent2(part_ml_at(slot, h[n]));
                                x[n][k] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part_buf, at[n], slot * GP_ * (HD * 4), kAgent));
                            }
                        }
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            float top = M[n];
#pragma unroll
                            for (int k = 0; k < J; ++k) {
                                if (k0 + k >= count) { ml[n][k] = make_float2(-INFINITY, 0.f); x[n][k] = f32x4{0.f, 0.f, 0.f, 0.f}; }
                                top = fmaxf(top, ml[n][k].x);
                            }
                            const float keep = M[n] > -INFINITY ? __builtin_amdgcn_exp2f(M[n] - top) : 0.f;
                            L[n] *= keep;
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[n][e] *= keep;
#pragma unroll
                            for (int k = 0; k < J; ++k) {
                                const float f = ml[n][k].x > -INFINITY ? __builtin_amdgcn_exp2f(ml[n][k].x - top) : 0.f;
                                L[n] += ml[n][k].y * f;
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[n][e] += x[n][k][e] * f;
                            }
                            M[n] = top;
                        }
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) if (begin + n * THREADS < items) done(h[n], at[n] / 4 % HD, o[n], M[n], L[n]);
                };
                if constexpr (THREADS == 256) {                     // N is all there are
                    if (self < items) some(self);
                } else {
#pragma unroll 1
                    for (int idx = self; idx < items; idx += 64) some(idx);
                }
            };
            // All loads of a round go out together whether there are as many parts or not, so a round is one of three widths.  One sequence, 32 heads, fp16 (four sequences, 8 KV heads of 8, fp32), us by
            // the width: 2 to 4 parts 4 wide 8.0 (8.6), 5 wide 8.0 (8.7), 8 wide 8.4 (8.9), 16 wide 8.6 (9.6); 5 parts, 4 wide in 16, 8.8 8.2 8.5 8.8 (9.8 8.9 9.0 9.8); 6 to 8 parts, 5 and 8 wide against
            // 16, 8.2 to 8.4 against 8.7 to 8.9 (9.2 to 9.6 against 10.0 to 10.3); 9 to 16 in two rounds of 8 are up to 0.4 us slower than in one of 16.
            auto join_some = [&](int first, int step, int count, auto done) {
                typedef std::integral_constant<int, 1> One;
                typedef std::integral_constant<int, 5> Five;
                if constexpr (THREADS == 64) join(Five(), One(), first, step, count, done);
                else if (ITEMS > 1 && items > THREADS) join(std::integral_constant<int, 8>(), std::integral_constant<int, 2>(), first, step, count, done);
                else if (count <= 5) join(Five(), One(), first, step, count, done);
                else if (count <= 8) join(std::integral_constant<int, 8>(), One(), first, step, count, done);
                else join(std::integral_constant<int, kJoin>(), One(), first, step, count, done);
            };
            const int sets = (parts + kJoin - 1) / kJoin, first = (run - w0) / kJoin * kJoin, count = min(kJoin, parts - first);
            bool mine = true;
            if (sets > 1 && count > 1) {
                mine = arrive(&a.tickets[a.B * HH_ + (int)slot_of(first)], count);
                if (mine) {                                         // what they give goes into the first one's slot: a thread's dims as it has read them, maxima and sums once all have
                    join_some(first, 1, count, [&](int h, int t, const float (&o)[4], float M, float L) {
                        publish_o(slot_of(first), h, t, o);
                        if (t == 0) { sh.m[h][column] = M; sh.l[h][column] = L; }
                    });
                    if (THREADS == 256) __syncthreads();
                    if (self < nh) publish_ml(slot_of(first), self, sh.m[self][column], sh.l[self][column]);
                }
            }
            const int left = sets > 1 ? sets : parts;
            if (mine && arrive(&a.tickets[b * HH_ + hh], left)) {
                auto last = [&](int h, int t, const float (&o)[4], float, float L) { finish(h, t, o, L); };
                join_some(0, sets > 1 ? kJoin : 1, left, last);
            }
        };
        if (!whole) {
            if constexpr (WAVES) join_all(std::integral_constant<int, 64>());
            else join_all(std::integral_constant<int, 256>());
        }
        u = next;
        if (u < end) {
            if (!WAVES) __syncthreads();                            // the merge has read what the next (sequence, heads) will write
            if (u == seq_begin + per_head * HH) {                   // all heads of this sequence: the next one that has rows
                seq_begin = u;
                do len = __builtin_amdgcn_readfirstlane(length(++b)); while (len == 0);      // there is one: u < end <= total
            }
        }
    }
}

// MANY: there are as many (sequence, heads) as waves, or nearly.  If those that have rows are as many, and have three chunks or less on average, every wave takes runs of its own: no merge of four,
// no wave without rows where they are few, q prepared once instead of four times.  us a pass, runs of workgroups and of waves: 256 sequences of 30 / 100 / 200 / 500 rows of 8 KV heads, 32 query heads
// 23.0 14.5 / 34.2 26.5 / 46.7 44.3 / 95.8 96.3; 128 x 100 rows of 32 heads 63.0 50.2; 512 x 64 of 8, 64 query heads 47.5 38.1; lengths of 1 to 2048, 256 x 8 KV heads, 32 query heads (2.6 chunks) 72.9 67.9.
// Above that the few long sequences are shared by so many waves that it turns: 1 to 4096 (4.3 chunks) 106.3 111.3, 1 to 32768 with 64 query heads 517 556.  With fewer (sequence, heads) than waves every
// wave has parts of them, to be joined: 7/8 as many, 200 rows, 64 query heads 47.6 55.1; 15/16 48.8 51.2, but 7/8 of 1 to 1000 rows, 32 query heads, 46.6 38.6.
__host__ __device__ inline int nearly(int waves) { return waves - waves / 16; }

template <typename T, int HD, typename A, bool MANY>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(PagedAttnArgs a) {
    __shared__ PagedShared<T, HD> sh;
    paged_take_args(a);
    if constexpr (sizeof(T) == 1) asm volatile("" :: "s"(a.k_scales), "s"(a.v_scales), "s"(a.scale_part), "s"(a.scale_exp));
    auto length = [&](int b) { return min(max(a.rows[b], 0), a.max_rows); };
    const Lengths n = take_lengths<PagedShape<T, HD>>(a.B, threadIdx.x & 63, length);
    if constexpr (MANY) {
        if (n.chunks <= 3 * n.live && n.live * a.H_kv * ((a.group + kPagedHeads - 1) / kPagedHeads) >= nearly((int)a.by_waves.d))
            return attn_paged_runs<T, HD, A, true>(a, sh, n, length);
    }
    attn_paged_runs<T, HD, A, false>(a, sh, n, length);
}

template <typename T, int HD, bool MANY>
int launch_many(const PagedAttnArgs& a, int n, hipStream_t s) {
    if (a.dtype == D3_F32) hipLaunchKernelGGL((attn_paged_kernel<T, HD, float, MANY>), dim3(n), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((attn_paged_kernel<T, HD, uint16_t, MANY>), dim3(n), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <typename T, int HD>
int launch(PagedAttnArgs a, int n_cu, hipStream_t s) {
    const long long heads = (long long)a.B * a.H_kv * paged_head_tiles(a.group), most = heads * ((a.max_rows + PagedShape<T, HD>::CH - 1) / PagedShape<T, HD>::CH);
    // as many workgroups as are resident, two per compute unit
    const int resident = std::min(2 * n_cu, kPagedMaxWgs), n = (int)std::min<long long>(most, resident);
    a.by_runs = Divisor(n);
    a.by_waves = Divisor(4 * n);
    a.scale_part = std::frexp(a.scale, &a.scale_exp) * 1.4426950408889634f;
    return heads >= nearly(4 * resident) ? launch_many<T, HD, true>(a, n, s) : launch_many<T, HD, false>(a, n, s);
}

}  // namespace

}  // namespace d3
