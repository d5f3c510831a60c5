// Rows into pages of 8 bits, quantised as they are written (codes8.h), and rows out of pages of any type.  Both move every byte once and are bound by memory, or by a launch where there are few rows: see kTokens.
#include <algorithm>
#include <type_traits>

#include "codes8.h"
#include "pages.h"

namespace d3 {

namespace {

// ---------------- rows of activations ----------------
// N adjacent elements of S (float, f16_t, bf16_t) at once, 2 to 16 bytes a load
template <int N, typename S>
struct Vec {
    static constexpr int BYTES = N * sizeof(S), WORDS = (BYTES + 3) / 4;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const void* p) {
        if constexpr (BYTES == 1) w[0] = *static_cast<const uint8_t*>(p);
        else if constexpr (BYTES == 2) w[0] = *static_cast<const uint16_t*>(p);
        else if constexpr (BYTES == 4) w[0] = *static_cast<const uint32_t*>(p);
        else if constexpr (BYTES == 8) { const uint2 t = *static_cast<const uint2*>(p); w[0] = t.x; w[1] = t.y; }
        else {
#pragma unroll
            for (int j = 0; j < WORDS; j += 4) {
                const uint4 t = *reinterpret_cast<const uint4*>(static_cast<const char*>(p) + 4 * j);
                w[j] = t.x; w[j + 1] = t.y; w[j + 2] = t.z; w[j + 3] = t.w;
            }
        }
    }
    __device__ __forceinline__ void store(void* p) const {
        if constexpr (BYTES == 2) *static_cast<uint16_t*>(p) = (uint16_t)w[0];
        else if constexpr (BYTES == 4) *static_cast<uint32_t*>(p) = w[0];
        else if constexpr (BYTES == 8) *static_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else {
            static_assert(BYTES % 16 == 0, "");
#pragma unroll
            for (int j = 0; j < WORDS; j += 4) *reinterpret_cast<uint4*>(static_cast<char*>(p) + 4 * j) = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
        }
    }
    // as fp32: values, or codes
    __device__ __forceinline__ void get(float (&y)[N]) const {
        if constexpr (sizeof(S) == 4) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = __uint_as_float(w[e]);
        } else if constexpr (sizeof(S) == 2) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const uint32_t bits = w[e / 2] >> (e % 2 * 16) & 0xffffu;
                if constexpr (std::is_same<S, bf16_t>::value) y[e] = bf16_to_f32(bits);
                else y[e] = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
            }
        } else {
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                half2_t h[2];
                decode4<S>(w[j], h[0], h[1]);
#pragma unroll
                for (int e = 0; e < 4 && 4 * j + e < N; ++e) y[4 * j + e] = (float)h[e / 2][e % 2];
            }
        }
    }
    // rounded to nearest even
    __device__ __forceinline__ void put(const float (&y)[N]) {
        if constexpr (sizeof(S) == 4) {
#pragma unroll
            for (int e = 0; e < N; ++e) w[e] = __float_as_uint(y[e]);
        } else {
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                const float a = y[2 * j], b = 2 * j + 1 < N ? y[2 * j + 1] : 0.f;
                if constexpr (std::is_same<S, bf16_t>::value) w[j] = bf16_pair(a, b);
                else w[j] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)a, (_Float16)b});
            }
        }
    }
};

// code * scale, rounded to fp32 whatever it is rounded to next (else the compiler takes the instruction that rounds to fp16 at once, and outputs of one type would differ from fp32 ones rounded later)
__device__ __forceinline__ float value_of(float code, float scale) {
    float y = code * scale;
    asm("" : "+v"(y));
    return y;
}

// the largest magnitude of N lanes side by side (N = 4, 8, 16)
template <int N> __device__ __forceinline__ float reduce_lanes(float v) {
    const MaxMagnitude op;
#define D3_FROM(ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
    v = op(v, D3_FROM(0xb1));                                       // lanes l ^ 1
    v = op(v, D3_FROM(0x4e));                                       // l ^ 2
    if (N >= 8) v = op(v, D3_FROM(0x141));                          // mirrored within 8
    if (N >= 16) v = op(v, D3_FROM(0x140));                         // within 16
#undef D3_FROM
    return v;
}
// Of 16 rows at once, a lane's part of each in m: lane l gets that of row l % 16.  In each of four steps a lane keeps half of its rows and takes its partner's part of these (15 exchanges; row by row it is 96);
// the lanes l ^ 8, l ^ 7, l ^ 2 and l ^ 1 that they exchange with make up the 16 side by side, and two steps more the wave.
__device__ __forceinline__ float reduce_rows16(const float (&m)[16], int lane) {
    const MaxMagnitude op;
    float a[8], b[4], c[2];
#define D3_FROM(v, ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
#define D3_HALF(to, from, n, bit, ctrl)                                          \
    _Pragma("unroll") for (int e = 0; e < n; ++e) {                              \
        const float keep = lane & bit ? from[e + n] : from[e], give = lane & bit ? from[e] : from[e + n]; \
        to[e] = op(keep, D3_FROM(give, ctrl));                                   \
    }
    D3_HALF(a, m, 8, 8, 0x128)
    D3_HALF(b, a, 4, 4, 0x141)
    D3_HALF(c, b, 2, 2, 0x4e)
    const float keep = lane & 1 ? c[1] : c[0], give = lane & 1 ? c[0] : c[1];
    const float d = op(keep, D3_FROM(give, 0xb1));
#undef D3_HALF
#undef D3_FROM
    return reduce_halves(reduce_row_pairs(d, op), op);
}

__device__ __forceinline__ unsigned long long lane_of(unsigned long long v, int lane) {
    return (unsigned long long)(unsigned)__builtin_amdgcn_readlane((unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)v, lane);
}

// The tokens that a wave looks at for its own WN, R - 1 before them (lane 0 is the first of these) to R - 1 behind, as the slots of values lie in units of R rows.
template <int R, int WN>
struct Units {
    int slot;
    unsigned long long firsts, singles;                             // own tokens that are row 0 of a unit filled by the R tokens from there on; own tokens in no such unit (of this or the wave before)
    template <typename F> __device__ __forceinline__ Units(int lane, int t0, F slot_at) {
        slot = lane < WN + 2 * (R - 1) ? slot_at(t0 - (R - 1) + lane) : -1;
        const unsigned long long valid = __ballot(slot >= 0), begins = __ballot(slot >= 0 && slot % R == 0);
        const int after = __shfl_down(slot, 1, 64);
        unsigned long long run = __ballot(slot >= 0 && lane < 63 && after == slot + 1), covered;        // the next token is the next row; then the next R - 1 are
        run &= run >> 1;
        if (R > 4) run &= run >> 2;
        if (R > 8) run &= run >> 4;
        firsts = covered = begins & run & run >> (R / 2 - 1);
#pragma unroll
        for (int n = 1; n < R; n *= 2) covered |= covered << n;
        constexpr unsigned long long own = ((1ull << WN) - 1) << (R - 1);
        firsts &= own;
        singles = (valid & ~covered & own) >> (R - 1);
    }
};

// ---------------- rows into pages ----------------
// grid: (64 tokens, KV head, layer and half: keys or values).
// A key is a row of its page: 16 bytes of the source's lower half and their partners per thread, the row's magnitude from the threads beside it.
// Values: a wave has 16 tokens, a lane one or two dims of all of them; where 16 tokens fill a unit of 16 rows it writes the unit's 16 bytes per dim, elsewhere bytes.
// Workgroups of 16 / 32 / 64 tokens, us (the shortest of 30 launches): 512 rows of 32 heads, fp32 to e4m3 with rotation, 10.7 / 8.3 / 7.1; 8 layers x 1024 rows of 8 heads 26.0 / 24.1 / 17.8 (4.7 TB/s, a large copy's rate); 1024 rows of 40 heads,
// fp16 to i8, 15.8 / 12.8 / 10.5; read, 4 layers x 2304 rows of 32 heads, i8 to fp16, 55 / 47 / 40 (the first of a series, 5.7 TB/s; from the third on 46 to 48, 4.8 TB/s: the 151 MB that the one before has written are then presumably still on their way from the memory-side cache): workgroups begin one after the other, and the loads of four rounds are in flight together.
constexpr int kTokens = 64, kValueTokens = kTokens / 4;

template <typename S, typename T, int HD>
__global__ __launch_bounds__(256) void pages_append8_kernel(AppendArgs a) {
    constexpr int R = 16, DL = HD / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = blockIdx.y, layer = blockIdx.z >> 1;
    const bool values = blockIdx.z & 1;
    const S* src = static_cast<const S*>(values ? a.v : a.k) + layer * a.layer_stride + h * a.head_stride;
    const int row_mask = (1 << a.page_shift) - 1;
    auto rows_at = [&](int slot) { return ((size_t)(slot >> a.page_shift) * a.H_kv + h) << a.page_shift; };      // rows before the head's of the slot's page
    char* pool = static_cast<char*>(values ? a.v_pages : a.k_pages) + layer * a.pool_bytes;
    float* scales = reinterpret_cast<float*>(reinterpret_cast<char*>(values ? a.v_scales : a.k_scales) + layer * a.scale_bytes);
    auto slot_at = [&](int t) {
        const int slot = t >= 0 && t < a.n ? a.slots[t] : -1;
        return slot < a.n_slots ? slot : -1;
    };
    if (!values) {
        constexpr int E = 16 / sizeof(S), PER = HD / (2 * E), ROUNDS = (kTokens * PER + 255) / 256;      // threads of a token, each with one load of either half
        int slot[ROUNDS];
        Vec<E, S> lo[ROUNDS], hi[ROUNDS];
        Vec<2 * E, float> cs[ROUNDS];
        const int j = tid % PER * E;
#pragma unroll
        for (int x = 0; x < ROUNDS; ++x) {
            const int t = blockIdx.x * kTokens + (x * 256 + tid) / PER, from = min(t, a.n - 1);
            slot[x] = x * 256 + tid < kTokens * PER ? slot_at(t) : -1;
            lo[x].load(src + from * a.token_stride + j);
            hi[x].load(src + from * a.token_stride + j + HD / 2);
            if (a.rope_cs) cs[x].load(a.rope_cs + (size_t)from * (HD / 2) + j);
        }
#pragma unroll
        for (int x = 0; x < ROUNDS; ++x) {
            float y0[E], y1[E], c[2 * E];
            lo[x].get(y0);
            hi[x].get(y1);
            if (a.rope_cs) {
                cs[x].get(c);
#pragma unroll
                for (int e = 0; e < E; ++e) turned(y0[e], y1[e], make_float2(c[2 * e], c[2 * e + 1]));
            }
            float most = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) most = MaxMagnitude()(most, MaxMagnitude()(magnitude(y0[e]), magnitude(y1[e])));
            const RowScale s = row_scale<T>(reduce_lanes<PER>(most));
#pragma unroll
            for (int e = 0; e < E; ++e) { y0[e] *= s.inv; y1[e] *= s.inv; }
            Vec<E / 4, float> w0, w1;
            encode<T, E>(y0, w0.w);
            encode<T, E>(y1, w1.w);
            if (slot[x] < 0) continue;
            const size_t row = rows_at(slot[x]) + (slot[x] & row_mask);
            w0.store(pool + row * HD + j);
            w1.store(pool + row * HD + j + HD / 2);
            if (j == 0) scales[row] = s.scale;
        }
        return;
    }
    const int t0 = (blockIdx.x * 4 + wave) * kValueTokens;
    if (t0 >= a.n) return;
    // the rows of the wave's own tokens, requested beside their slots; those of a unit that begins among them, where it does not begin with the first
    Vec<DL, S> v[R];
    auto load_rows = [&](int first) {
#pragma unroll
        for (int e = 0; e < R; ++e) v[e].load(src + min(first + e, a.n - 1) * a.token_stride + lane * DL);
    };
    load_rows(t0);
    const int own = lane < R ? slot_at(t0 + lane) : -1;
    const Units<R, kValueTokens> units(lane, t0, slot_at);
    const int unit_at = units.firsts ? __builtin_ctzll(units.firsts) - (R - 1) : 0;        // one at most: units begin 16 tokens apart
#pragma unroll 1
    for (int pass = units.singles ? 0 : 1; pass < (units.firsts ? 2 : 1); ++pass) {
        if (pass == 1 && unit_at != 0) load_rows(t0 + unit_at);
        float y[R][DL], most[R];
#pragma unroll
        for (int e = 0; e < R; ++e) {
            v[e].get(y[e]);
            most[e] = magnitude(y[e][0]);
            if (DL == 2) most[e] = MaxMagnitude()(most[e], magnitude(y[e][DL - 1]));
        }
        const RowScale s = row_scale<T>(reduce_rows16(most, lane));                    // of row lane % 16
        of_rows(s.inv, [&](int e, float inv) {
#pragma unroll
            for (int d = 0; d < DL; ++d) y[e][d] *= inv;
        });
        Vec<4, float> w[DL];
#pragma unroll
        for (int d = 0; d < DL; ++d) {
            float z[R];
#pragma unroll
            for (int e = 0; e < R; ++e) z[e] = y[e][d];
            encode<T, R>(z, w[d].w);
        }
        if (pass == 1) {
            const int at = __builtin_amdgcn_readlane(units.slot, R - 1 + unit_at);
            const size_t row = rows_at(at) + (at & row_mask);
#pragma unroll
            for (int d = 0; d < DL; ++d) w[d].store(pool + row * HD + (lane * DL + d) * R);
            if (lane < R) scales[row + lane] = s.scale;
        } else {
            const unsigned long long row = rows_at(own) + (own & row_mask), at = (row & ~(unsigned long long)(R - 1)) * HD + own % R;       // (means nothing where the token is none)
#pragma unroll
            for (int e = 0; e < R; ++e) {
                if (!(units.singles >> e & 1)) continue;
                char* to = pool + lane_of(at, e) + lane * (DL * R);
#pragma unroll
                for (int d = 0; d < DL; ++d) to[d * R] = (char)(w[d].w[e / 4] >> (8 * (e % 4)));
            }
            if (units.singles >> lane & 1) scales[row] = s.scale;          // (no bits from R on)
        }
    }
}

// ---------------- rows out of pages ----------------
// grid as above.  Where R tokens are a unit of R rows, a wave reads the unit's 16 bytes per dim and writes the R rows; elsewhere it reads elements.
template <typename T, typename D, int HD>
__global__ __launch_bounds__(256) void pages_read_kernel(ReadArgs a) {
    constexpr int R = 16 / sizeof(T), DL = HD / 64, WN = kValueTokens;
    constexpr bool SCALED = sizeof(T) == 1;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = blockIdx.y, layer = blockIdx.z >> 1;
    const bool values = blockIdx.z & 1;
    D* out = static_cast<D*>(values ? a.v : a.k) + layer * a.layer_stride + h * a.head_stride;
    const int row_mask = (1 << a.page_shift) - 1;
    auto rows_at = [&](int slot) { return ((size_t)(slot >> a.page_shift) * a.H_kv + h) << a.page_shift; };
    const char* pool = static_cast<const char*>(values ? a.v_pages : a.k_pages) + layer * a.pool_bytes;
    const float* scales = reinterpret_cast<const float*>(reinterpret_cast<const char*>(values ? a.v_scales : a.k_scales) + layer * a.scale_bytes);
    auto slot_at = [&](int t) {
        const int slot = t >= 0 && t < a.n ? a.slots[t] : -1;
        return slot < a.n_slots ? slot : -1;
    };
    if (!values) {
        constexpr int E = 16 / sizeof(D), PER = HD / E, ROUNDS = (kTokens * PER + 255) / 256;
        int slot[ROUNDS];
        Vec<E, T> in[ROUNDS];
        float scale[ROUNDS];
        const int j = tid % PER * E;
#pragma unroll
        for (int x = 0; x < ROUNDS; ++x) slot[x] = x * 256 + tid < kTokens * PER ? slot_at(blockIdx.x * kTokens + (x * 256 + tid) / PER) : -1;
#pragma unroll
        for (int x = 0; x < ROUNDS; ++x) {
            const int from = max(slot[x], 0);
            const size_t row = rows_at(from) + (from & row_mask);
            in[x].load(pool + (row * HD + j) * sizeof(T));
            if (SCALED) scale[x] = scales[row];
        }
#pragma unroll
        for (int x = 0; x < ROUNDS; ++x) {
            float y[E];
            in[x].get(y);
            if (SCALED) {
#pragma unroll
                for (int e = 0; e < E; ++e) y[e] = value_of(y[e], scale[x]);
            }
            Vec<E, D> w;
            w.put(y);
            if (slot[x] >= 0) w.store(out + (blockIdx.x * kTokens + (x * 256 + tid) / PER) * a.token_stride + j);
        }
        return;
    }
    const int t0 = (blockIdx.x * 4 + wave) * WN;
    if (t0 >= a.n) return;
    const int own = lane < WN ? slot_at(t0 + lane) : -1;
    const Units<R, WN> units(lane, t0, slot_at);
    for (unsigned long long left = units.firsts; left; left &= left - 1) {
        const int x = __builtin_ctzll(left), at = __builtin_amdgcn_readlane(units.slot, x);
        const size_t row = rows_at(at) + (at & row_mask);
        Vec<R, T> in[DL];
        float scale[R], y[DL][R];
#pragma unroll
        for (int d = 0; d < DL; ++d) in[d].load(pool + row * HD * sizeof(T) + (lane * DL + d) * 16);
        if (SCALED) {
#pragma unroll
            for (int e = 0; e < R; ++e) scale[e] = scales[row + e];
        }
#pragma unroll
        for (int d = 0; d < DL; ++d) in[d].get(y[d]);
        D* to = out + (long long)(t0 - (R - 1) + x) * a.token_stride + lane * DL;
#pragma unroll
        for (int e = 0; e < R; ++e) {
            float z[DL];
#pragma unroll
            for (int d = 0; d < DL; ++d) z[d] = SCALED ? value_of(y[d][e], scale[e]) : y[d][e];
            Vec<DL, D> w;
            w.put(z);
            w.store(to + e * a.token_stride);
        }
    }
    if (!units.singles) return;
    Vec<1, T> in[WN][DL];
    float scale = 0.f;                                              // of row `lane`
    const int from = max(own, 0);                                   // (tokens that are in a unit, or none, are loaded too)
    const unsigned long long row = rows_at(from) + (from & row_mask), at = ((row & ~(unsigned long long)(R - 1)) * HD + from % R) * sizeof(T);
    if (SCALED) scale = scales[row];
#pragma unroll
    for (int e = 0; e < WN; ++e) {
        const char* p = pool + lane_of(at, e) + lane * (DL * 16);
#pragma unroll
        for (int d = 0; d < DL; ++d) in[e][d].load(p + d * 16);
    }
#pragma unroll
    for (int e = 0; e < WN; ++e) {
        if (!(units.singles >> e & 1)) continue;
        const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(scale), e));
        float z[DL];
#pragma unroll
        for (int d = 0; d < DL; ++d) {
            float y[1];
            in[e][d].get(y);
            z[d] = SCALED ? value_of(y[0], by) : y[0];
        }
        Vec<DL, D> w;
        w.put(z);
        w.store(out + (t0 + e) * a.token_stride + lane * DL);
    }
}

template <typename S, typename T>
int launch_append(const AppendArgs& a, hipStream_t s) {
    const dim3 grid((a.n + kTokens - 1) / kTokens, a.H_kv, 2 * a.n_layers);
    if (a.hd == 64) hipLaunchKernelGGL((pages_append8_kernel<S, T, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((pages_append8_kernel<S, T, 128>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <typename T>
int launch_append_to(const AppendArgs& a, hipStream_t s) {
    return a.dtype == D3_F32 ? launch_append<float, T>(a, s) : a.dtype == D3_BF16 ? launch_append<bf16_t, T>(a, s) : launch_append<f16_t, T>(a, s);
}
template <typename T, typename D>
int launch_read(const ReadArgs& a, hipStream_t s) {
    const dim3 grid((a.n + kTokens - 1) / kTokens, a.H_kv, 2 * a.n_layers);
    if (a.hd == 64) hipLaunchKernelGGL((pages_read_kernel<T, D, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((pages_read_kernel<T, D, 128>), grid, dim3(256), 0, s, a);
    return (int)hipGetLastError();
}
template <typename T>
int launch_read_from(const ReadArgs& a, hipStream_t s) {
    return a.dtype == D3_F32 ? launch_read<T, float>(a, s) : a.dtype == D3_BF16 ? launch_read<T, bf16_t>(a, s) : launch_read<T, f16_t>(a, s);
}

}  // namespace

int launch_pages_append8(const AppendArgs& a, int kv_dtype, hipStream_t s) {
    return kv_dtype == D3_I8 ? launch_append_to<i8_t>(a, s) : launch_append_to<e4m3_t>(a, s);
}

int launch_pages_read(const ReadArgs& a, int kv_dtype, hipStream_t s) {
    switch (kv_dtype) {
        case D3_F32: return launch_read_from<float>(a, s);
        case D3_F16: return launch_read_from<f16_t>(a, s);
        case D3_I8: return launch_read_from<i8_t>(a, s);
        default: return launch_read_from<e4m3_t>(a, s);
    }
}

}  // namespace d3
