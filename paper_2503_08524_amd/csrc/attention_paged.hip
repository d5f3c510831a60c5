// Decode attention over a paged cache: one new token per sequence,
//   o[b][h] = sum_j w_j V[j] / sum_j w_j,   w_j = exp(scale * q[b][h] . K[j]),   j over the rows of sequence b,
// each sequence with a length and a list of pages of its own.
//
// Work: the rows of every (sequence, KV head, 16 query heads) are cut into chunks of 64 KB of keys and values, all chunks laid end to end, and
// every workgroup takes an equal run of them, whatever the lengths: it may end one sequence, take others whole and begin another.  The host
// knows no lengths, so a launch can be captured once and replayed while sequences grow.  A run that covers a (sequence, heads) whole writes the
// result; else it publishes (max, sum, unnormalised output), and the run that arrives last joins them.
//
// Both contractions run on the matrix cores with the query heads of a KV head as one matrix dimension, straight from the registers that the
// loads fill (see pages.h for the layout of the values):
//   scores  D[row][head] = K[row][dim] q[head][dim]: a lane (i = lane % 16, g = lane / 16) loads 16 bytes of row i and ends with the scores of head i for
//           R rows that are consecutive in the cache, because row i of the instruction is cache row R (i / 4) + 4 t + i % 4 of its tile t;
//   outputs D[dim][head] += V[dim][row] w[row][head]: a lane loads the 16 bytes that hold R rows of dim i, the very rows whose weights of head i it has.
// So the head stays with lane % 16 throughout, the running maximum and sum of a softmax are the lane's own, and nothing passes through LDS before the
// four waves of a workgroup are merged at the end of a run.
#include <algorithm>
#include <type_traits>

#include "pages.h"

namespace d3 {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

template <typename T, int HD>
struct PagedShape {
    static constexpr int ES = sizeof(T);
    static constexpr int R = 16 / ES;              // rows of a V unit
    static constexpr int KT = R / 4;               // row tiles of a group of rows
    static constexpr int RG = 4 * R;               // rows of a group: one matrix instruction's worth of weights
    static constexpr int NK = HD * ES / 64;        // 16-byte loads per lane of a row tile of K
    static constexpr int ND = HD / 16;             // ... of a group's V: tiles of 16 dims
    static constexpr int U = 16 / (KT * NK + ND);  // groups of a turn: 16 loads in flight per lane
    static constexpr int TR = U * RG;              // rows of a wave's turn
    static constexpr int CH = 4 * TR;              // rows of a chunk, a turn of each wave
    static constexpr int QE = 16 / ES;             // elements of q beside a 16-byte piece of K
    // Weights are in (0, 1]; times 2^15 before they become fp16 halves, so that small ones keep their digits (fp16 counts in steps of 2^-24 at the bottom).
    static constexpr float SHIFT = ES == 2 ? 15.f : 0.f;
};

template <int HD>
struct PagedShared {
    float m[kPagedHeads][4], l[kPagedHeads][4];    // per wave: running max and sum of each head
    float o[4][kPagedHeads][HD + 4];               // per wave: unnormalised outputs (rows 4 words apart in the banks)
    int is_last;
};

// N consecutive activations
template <int N>
__device__ __forceinline__ void load_act(const void* p, long long at, int dtype, float (&y)[N]) {
    if (dtype == D3_F32) {
        const float* f = static_cast<const float*>(p) + at;
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const float4 t = *reinterpret_cast<const float4*>(f + e);
            y[e] = t.x; y[e + 1] = t.y; y[e + 2] = t.z; y[e + 3] = t.w;
        }
        return;
    }
    uint32_t w[N / 2];
    const uint16_t* h = static_cast<const uint16_t*>(p) + at;
    if constexpr (N == 8) {
        const uint4 t = *reinterpret_cast<const uint4*>(h);
        w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
    } else {
        const uint2 t = *reinterpret_cast<const uint2*>(h);
        w[0] = t.x; w[1] = t.y;
    }
#pragma unroll
    for (int e = 0; e < N; e += 2) {
        if (dtype == D3_BF16) { y[e] = bf16_lo(w[e / 2]); y[e + 1] = bf16_hi(w[e / 2]); }
        else {
            y[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)w[e / 2]);
            y[e + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[e / 2] >> 16));
        }
    }
}
__device__ __forceinline__ float load_act1(const void* p, long long at, int dtype) {
    if (dtype == D3_F32) return static_cast<const float*>(p)[at];
    const uint16_t h = static_cast<const uint16_t*>(p)[at];
    return dtype == D3_BF16 ? bf16_to_f32(h) : (float)__builtin_bit_cast(_Float16, h);
}
__device__ __forceinline__ void store_act(void* p, long long at, int dtype, float v) {
    if (dtype == D3_F32) static_cast<float*>(p)[at] = v;
    else if (dtype == D3_BF16) static_cast<uint16_t*>(p)[at] = (uint16_t)bf16_pair(v, 0.f);
    else static_cast<_Float16*>(p)[at] = (_Float16)v;
}

__device__ __forceinline__ int scan_wave(int v) {                  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const int below = __shfl_up(v, o, 64);
        if (lane >= o) v += below;
    }
    return v;
}

// Equal runs of `total` chunks: the first `over` workgroups have one more.
struct Runs {
    int per, over;
    __device__ Runs(int total, int n) : per((int)((unsigned)total / (unsigned)n)), over(total - per * n) {}
    __device__ int begin(int w) const { return w * per + min(w, over); }
    __device__ int of(int x) const {                               // the run that chunk x is in
        const int larger = over * (per + 1);
        return x < larger ? x / (per + 1) : over + (x - larger) / per;      // per = 0: every chunk is below `larger`
    }
};

template <typename T, int HD>
__global__ __launch_bounds__(256, 2) void attn_paged_kernel(PagedAttnArgs a) {
    typedef PagedShape<T, HD> P;
    constexpr int R = P::R, KT = P::KT, RG = P::RG, NK = P::NK, ND = P::ND, U = P::U, QE = P::QE;
    __shared__ PagedShared<HD> sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = lane & 15, g = lane >> 4;
    const int H = a.H_kv * a.group, tiles = (a.group + kPagedHeads - 1) / kPagedHeads, HH = a.H_kv * tiles, GP = min(a.group, kPagedHeads);
    auto length = [&](int b) { return min(max(a.rows[b], 0), a.max_rows); };

    // ---- this workgroup's run of chunks, and where it begins ----
    auto chunks_of = [&](int b) { return b < a.B ? (length(b) + P::CH - 1) / P::CH * HH : 0; };
    int n = chunks_of(lane), upto = scan_wave(n), total = __builtin_amdgcn_readlane(upto, 63);
    const int total64 = total;
    for (int b0 = 64; b0 < a.B; b0 += 64) total += __builtin_amdgcn_readlane(scan_wave(chunks_of(b0 + lane)), 63);
    for (int b = blockIdx.x; b < a.B; b += gridDim.x) {             // a sequence without rows: zeros
        if (length(b) > 0) continue;
        for (int e = tid; e < H * HD; e += 256) {
            store_act(a.out, b * a.out_stride + e, a.dtype, 0.f);
            if (a.out_split) store_split1(a.out_split + b * a.out_form.pitch(H * HD), e, 0.f, a.out_form.lo);
        }
    }
    const Runs runs(total, gridDim.x);
    const int run = blockIdx.x, end = runs.begin(run + 1);
    int u = runs.begin(run);
    if (u >= end) return;
    int b = 0, seq_begin = 0;                                       // the sequence of chunk u, and its first chunk
    {
        int before = 0, b0 = 0, here = total64;
        while (u >= before + here) {
            before += here; b0 += 64;
            n = chunks_of(b0 + lane); upto = scan_wave(n); here = __builtin_amdgcn_readlane(upto, 63);
        }
        const int at = __builtin_ctzll(__ballot(before + upto > u));
        b = b0 + at;
        seq_begin = before + __builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at);
    }

    const int block_shift = a.page_shift - (R == 8 ? 3 : 2), block_mask = (1 << block_shift) - 1;      // blocks of R rows
    const size_t head_bytes = ((size_t)HD * P::ES) << a.page_shift, page_bytes = head_bytes * a.H_kv;

    while (u < end) {
        const int len = __builtin_amdgcn_readfirstlane(length(b));
        const int per_head = (len + P::CH - 1) / P::CH, hh = (u - seq_begin) / per_head, head_begin = seq_begin + hh * per_head;
        const int c0 = u - head_begin, c1 = min(per_head, c0 + end - u);
        const int kvh = hh / tiles, h0 = (hh - kvh * tiles) * kPagedHeads, nh = min(kPagedHeads, a.group - h0);
        const bool whole = c0 == 0 && c1 == per_head;
        const int newest = len - 1, last_block = newest / R;
        const int* tab = a.tables + (size_t)b * a.table_stride;
        char* Kh = static_cast<char*>(a.k_pages) + kvh * head_bytes;
        char* Vh = static_cast<char*>(a.v_pages) + kvh * head_bytes;
        const int rend = min(c1 * P::CH, len);
        int r = c0 * P::CH + wave * P::TR;                          // first row of this wave's turn

        uint4 kr[U][KT][NK], vr[U][ND];
        // pages of the blocks of R rows that a lane loads of K and of V; blocks past the last are read as the last
        auto load_pages = [&](int row, int (&pk)[U], int (&pv)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                pk[x] = tab[min((row + x * RG) / R + (i >> 2), last_block) >> block_shift];
                pv[x] = tab[min((row + x * RG) / R + g, last_block) >> block_shift];
            }
        };
        auto present = [&](int page) { return (unsigned)page < (unsigned)a.n_pages; };
        auto issue_k = [&](int row, const int (&pk)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int blk = min((row + x * RG) / R + (i >> 2), last_block) & block_mask;
                const char* p = Kh + (present(pk[x]) ? pk[x] : 0) * page_bytes + (blk * R + (i & 3)) * (HD * P::ES) + g * 16;
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int k = 0; k < NK; ++k) kr[x][t][k] = __builtin_bit_cast(uint4, load_stream16(p + t * 4 * HD * P::ES + k * 64));
            }
        };
        auto issue_v = [&](int row, const int (&pv)[U]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int blk = min((row + x * RG) / R + g, last_block) & block_mask;
                const char* p = Vh + (present(pv[x]) ? pv[x] : 0) * page_bytes + blk * (HD * 16) + i * 16;
#pragma unroll
                for (int d = 0; d < ND; ++d) vr[x][d] = __builtin_bit_cast(uint4, load_stream16(p + d * 256));
            }
        };
        // dims of piece k that this lane has of q and of a new key: k * 4 QE + g * QE ...; those half a head away are the lane's too
        auto rotated = [&](float (&y)[NK][QE]) {
#pragma unroll
            for (int k = 0; k < NK / 2; ++k) {
                const float2* cs = a.rope_cs + (size_t)b * (HD / 2) + k * 4 * QE + g * QE;
#pragma unroll
                for (int e = 0; e < QE; ++e) {
                    const float2 t = cs[e];
                    const float lo = y[k][e], hi = y[k + NK / 2][e];
                    y[k][e] = lo * t.x - hi * t.y;
                    y[k + NK / 2][e] = hi * t.x + lo * t.y;
                }
            }
        };

        float m = -INFINITY, l = 0.f;
        f32x4 acc[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (r < rend) {
            int pk[U], pv[U], pk1[U], pv1[U];
            load_pages(r, pk, pv);
            load_pages(r + P::CH, pk1, pv1);
            float qf[NK][QE];
#pragma unroll
            for (int k = 0; k < NK; ++k) load_act<QE>(a.q, b * a.q_stride + (long long)(kvh * a.group + h0 + min(i, nh - 1)) * HD + k * 4 * QE + g * QE, a.dtype, qf[k]);
            issue_k(r, pk);
            issue_v(r, pv);
            if (a.rope_cs) rotated(qf);
            // q as fp16 halves hi + lo, scaled by a power of two that puts its largest element at 2^14: 22 bits of it
            float mul = a.scale * 1.4426950408889634f;               // scores are kept in units of log2(e): every exponential is one hardware exp2
            half8 qh[NK], ql[NK];
            if constexpr (P::ES == 2) {
                float top = 0.f;
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int e = 0; e < QE; ++e) top = fmaxf(top, fabsf(qf[k][e]));
                top = reduce_halves(reduce_row_pairs(top, MaxOp()), MaxOp());
                const int ex = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0;
#pragma unroll
                for (int k = 0; k < NK; ++k)
#pragma unroll
                    for (int e = 0; e < QE; ++e) {
                        const float v = ldexpf(qf[k][e], ex);
                        qh[k][e] = (_Float16)v;
                        ql[k][e] = (_Float16)(v - (float)qh[k][e]);
                    }
                mul = ldexpf(mul, -ex);
            }

            auto turn = [&](auto more_) {
                constexpr bool MORE = decltype(more_)::value;
                const bool tail = !MORE && r + P::TR >= len;        // holds the newest row, or rows past it
                bool absent = false;                                // a page that is none: its rows do not count
#pragma unroll
                for (int x = 0; x < U; ++x) absent = absent || !present(pv[x]);
                absent = __any(absent);
                if (!MORE && tail && a.k_new) {                     // the newest row's key takes its place among the rows
                    float y[NK][QE];
#pragma unroll
                    for (int k = 0; k < NK; ++k) load_act<QE>(a.k_new, b * a.kv_stride + (long long)kvh * HD + k * 4 * QE + g * QE, a.dtype, y[k]);
                    if (a.rope_cs) rotated(y);
                    uint4 nk[NK];
#pragma unroll
                    for (int k = 0; k < NK; ++k) {
                        T h[QE];
#pragma unroll
                        for (int e = 0; e < QE; ++e) h[e] = held<T>(y[k][e]);
                        __builtin_memcpy(&nk[k], h, 16);
                    }
#pragma unroll
                    for (int x = 0; x < U; ++x)
#pragma unroll
                        for (int t = 0; t < KT; ++t) {
                            if (r + x * RG + R * (i >> 2) + 4 * t + (i & 3) != newest) continue;
#pragma unroll
                            for (int k = 0; k < NK; ++k) kr[x][t][k] = nk[k];
                        }
                    const int page = tab[last_block >> block_shift];
                    if (h0 == 0 && i == 0 && newest >= r && present(page)) {       // and its place in the cache
                        char* to = Kh + page * page_bytes + (newest & ((1 << a.page_shift) - 1)) * (HD * P::ES) + g * 16;
#pragma unroll
                        for (int k = 0; k < NK; ++k) *reinterpret_cast<uint4*>(to + k * 64) = nk[k];
                    }
                }
                float s[U][R];
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int t = 0; t < KT; ++t) {
                        f32x4 d = {0.f, 0.f, 0.f, 0.f}, d1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < NK; ++k) {
                            if constexpr (P::ES == 2) {
                                const half8 kv = __builtin_bit_cast(half8, kr[x][t][k]);
                                d = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, qh[k], d, 0, 0, 0);
                                d1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv, ql[k], d1, 0, 0, 0);
                            } else {
                                const f32x4 kv = __builtin_bit_cast(f32x4, kr[x][t][k]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    if (e & 1) d1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], qf[k][e], d1, 0, 0, 0);
                                    else d = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[e], qf[k][e], d, 0, 0, 0);
                                }
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[x][4 * t + j] = (d[j] + d1[j]) * mul;
                    }
                __builtin_amdgcn_sched_barrier(0);
                int pk2[U], pv2[U];
                if constexpr (MORE) {
                    load_pages(r + 2 * P::CH, pk2, pv2);
                    issue_k(r + P::CH, pk1);
                }
                __builtin_amdgcn_sched_barrier(0);
                if ((!MORE && tail) || absent) {
#pragma unroll
                    for (int x = 0; x < U; ++x)
#pragma unroll
                        for (int e = 0; e < R; ++e)
                            if (!present(pv[x]) || r + x * RG + R * g + e >= len) s[x][e] = -INFINITY;
                }
                // ---- running softmax of head i over the lane's rows (and, for the maximum, those of the other lanes that have the head) ----
                float top = s[0][0];
#pragma unroll
                for (int x = 0; x < U; ++x)
#pragma unroll
                    for (int e = 0; e < R; ++e) top = fmaxf(top, s[x][e]);
                top = fmaxf(m, reduce_halves(reduce_row_pairs(top, MaxOp()), MaxOp()));
                if (__any(top > m)) {
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
                if ((!MORE && tail) || absent) {                    // rows that do not count hold anything: 0 times it must be 0
#pragma unroll
                    for (int x = 0; x < U; ++x) {
                        const int row0 = r + x * RG + R * g;
#pragma unroll
                        for (int d = 0; d < ND; ++d) {
                            T v[R];
                            __builtin_memcpy(v, &vr[x][d], 16);
                            T own{};
                            if (!MORE && a.k_new && newest >= row0 && newest < row0 + R) own = held<T>(load_act1(a.v_new, b * a.kv_stride + (long long)kvh * HD + d * 16 + i, a.dtype));
#pragma unroll
                            for (int e = 0; e < R; ++e) {
                                if (!MORE && a.k_new && row0 + e == newest) v[e] = own;
                                if (!present(pv[x]) || row0 + e >= len) v[e] = (T)0.f;
                            }
                            __builtin_memcpy(&vr[x][d], v, 16);
                            if (!MORE && a.k_new && h0 == 0 && newest >= row0 && newest < row0 + R && present(pv[x])) {
                                char* to = Vh + pv[x] * page_bytes + (last_block & block_mask) * (HD * 16) + (d * 16 + i) * 16 + (newest - row0) * P::ES;
                                *reinterpret_cast<T*>(to) = own;
                            }
                        }
                    }
                }
#pragma unroll
                for (int x = 0; x < U; ++x) {
                    if constexpr (P::ES == 2) {
                        half8 ph, pl;
#pragma unroll
                        for (int e = 0; e < R; ++e) {
                            ph[e] = (_Float16)s[x][e];
                            pl[e] = (_Float16)(s[x][e] - (float)ph[e]);
                        }
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
                    issue_v(r + P::CH, pv1);
#pragma unroll
                    for (int x = 0; x < U; ++x) { pv[x] = pv1[x]; pk1[x] = pk2[x]; pv1[x] = pv2[x]; }
                }
            };
            for (; r + P::CH < rend; r += P::CH) turn(std::true_type());
            turn(std::false_type());
            l = reduce_halves(reduce_row_pairs(l, AddOp()), AddOp());
        }

        // ---- merge the waves ----
        if (i < nh) {
            if (g == 0) { sh.m[i][wave] = m; sh.l[i][wave] = l; }
#pragma unroll
            for (int d = 0; d < ND; ++d) *reinterpret_cast<f32x4*>(&sh.o[wave][i][d * 16 + g * 4]) = acc[d];
        }
        __syncthreads();
        auto finish = [&](int h, int t, float o, float sum) {
            const float v = sum == 0.f ? 0.f : o / sum;             // no row counted: zeros
            const int e = (kvh * a.group + h0 + h) * HD + t;
            store_act(a.out, b * a.out_stride + e, a.dtype, v);
            if (a.out_split) store_split1(a.out_split + b * a.out_form.pitch(H * HD), e, v, a.out_form.lo);
        };
        // this run's partials: a run has at most two, of the (sequence, heads) that it begins in and of the one that it ends in
        const size_t slot = 2 * (size_t)run + (u == runs.begin(run) ? 0 : 1);
        for (int idx = tid; idx < nh * HD; idx += 256) {
            const int h = idx / HD, t = idx % HD;
            float M = sh.m[h][0];
#pragma unroll
            for (int w = 1; w < 4; ++w) M = fmaxf(M, sh.m[h][w]);
            float L = 0.f, o = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = sh.m[h][w] > -INFINITY ? exp2f(sh.m[h][w] - M) : 0.f;
                L += sh.l[h][w] * f;
                o += sh.o[w][h][t] * f;
            }
            if (whole) { finish(h, t, o, L); continue; }
            st_agent(&a.part_o[(slot * GP + h) * HD + t], o);
            if (t == 0) { st_agent(&a.part_ml[(slot * GP + h) * 2], M); st_agent(&a.part_ml[(slot * GP + h) * 2 + 1], L); }
        }
        if (!whole) {                                               // the run that arrives last joins them all
            const int w0 = runs.of(head_begin), w1 = runs.of(head_begin + per_head - 1);
            wait_stores();
            __syncthreads();
            if (tid == 0) {
                int* ticket = &a.tickets[b * HH + hh];
                sh.is_last = atomicAdd(ticket, 1) == w1 - w0;
                if (sh.is_last) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // all arrived: leave it clean
            }
            __syncthreads();
            if (sh.is_last) {
                const size_t s0 = 2 * (size_t)w0 + (runs.begin(w0) >= head_begin ? 0 : 1);     // begins here, or in what is before
                for (int idx = tid; idx < nh * HD; idx += 256) {
                    const int h = idx / HD, t = idx % HD;
                    float M = -INFINITY, L = 0.f, o = 0.f;
                    constexpr int RND = 8;                           // partials in flight
                    for (int w = w0; w <= w1; w += RND) {
                        float ms[RND], ls[RND], os[RND];
#pragma unroll
                        for (int k = 0; k < RND; ++k) {
                            const int ww = min(w + k, w1);
                            const size_t p = (ww == w0 ? s0 : 2 * (size_t)ww) * GP + h;
                            ms[k] = ld_agent(&a.part_ml[p * 2]);
                            ls[k] = ld_agent(&a.part_ml[p * 2 + 1]);
                            os[k] = ld_agent(&a.part_o[p * HD + t]);
                        }
                        float top = M;
#pragma unroll
                        for (int k = 0; k < RND; ++k) if (w + k <= w1) top = fmaxf(top, ms[k]);
                        const float keep = M > -INFINITY ? exp2f(M - top) : 0.f;
                        L *= keep; o *= keep;
#pragma unroll
                        for (int k = 0; k < RND; ++k) {
                            if (w + k > w1) break;
                            const float f = ms[k] > -INFINITY ? exp2f(ms[k] - top) : 0.f;
                            L += ls[k] * f;
                            o += os[k] * f;
                        }
                        M = top;
                    }
                    finish(h, t, o, L);
                }
            }
        }
        u += c1 - c0;
        if (u < end) {
            __syncthreads();                                        // the merge has read what the next (sequence, heads) will write
            if (u == seq_begin + per_head * HH) {                   // all heads of this sequence: the next one that has rows
                seq_begin = u;
                do ++b; while (length(b) == 0);                     // there is one: u < end <= total
            }
        }
    }
}

template <typename T, int HD>
int launch(const PagedAttnArgs& a, int n_cu, hipStream_t s) {
    const long long most = (long long)a.B * a.H_kv * paged_head_tiles(a.group) * ((a.max_rows + PagedShape<T, HD>::CH - 1) / PagedShape<T, HD>::CH);
    // as many workgroups as are resident, two per compute unit
    const int n = (int)std::min<long long>(most, std::min(2 * n_cu, kPagedMaxWgs));
    hipLaunchKernelGGL((attn_paged_kernel<T, HD>), dim3(n), dim3(256), 0, s, a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_attention_paged(const PagedAttnArgs& a, int hd, int kv_dtype, int n_cu, hipStream_t s) {
    if (kv_dtype == D3_F32) return hd == 64 ? launch<float, 64>(a, n_cu, s) : launch<float, 128>(a, n_cu, s);
    if (kv_dtype == D3_F16) return hd == 64 ? launch<f16_t, 64>(a, n_cu, s) : launch<f16_t, 128>(a, n_cu, s);
    return (int)hipErrorInvalidValue;
}

}  // namespace d3
