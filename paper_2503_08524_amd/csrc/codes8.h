// A row of a head (a key after its rotation, a value) in 8 bits: hd codes and one fp32 scale.  With a the row's largest magnitude and Q the largest code (127 for D3_I8, whole numbers; 448 for D3_E4M3)
//   scale = a / Q,   code = x * (Q / a) to nearest even,   and it stands for code * scale.
// a counts as 3e38 at most (an infinity is held as that); below 2^-100 the row is held as zeros (scale 0), which keeps both quotients normal numbers; a row with a NaN has the scale NaN and reads as NaN throughout.
//
// The block that shares a scale is one row of one head.  Rows come one at a time and in any order of slots, and are copied one at a time between blocks of the model; a scale over several would have
// to be rewritten with every row under it whenever a larger one came: a second rounding, other results for another order of calls, a race between calls that write neighbours, and what a page's last
// owner left would count.  Four bytes beside 128 (3 %) buy rows that do not know of each other, and a factor per row is one multiplication of a score or of a weight.
//
// Half a step: i8 2^-8 of the row's largest value (a / 254); e4m3 2^-4 of the value itself, 2^-10 a / 448 near zero.  Relative to the norm of rows of normal values (hd 128): i8 6.5e-3, e4m3 2.6e-2; where one dim is 50
// times the others, i8 leaves these two or three codes and e4m3 as many digits as before.
#pragma once
#include "d3_common.h"

namespace d3 {

struct i8_t { uint8_t bits; };             // two's complement
struct e4m3_t { uint8_t bits; };           // sign, 4 bits of exponent, 3 of mantissa, bias 7; no infinities

constexpr float kScaledMost = 3e38f, kScaledLeast = 0x1p-100f;
template <typename T> struct MostCode { static constexpr float value = 0.f; };
template <> struct MostCode<i8_t> { static constexpr float value = 127.f; };
template <> struct MostCode<e4m3_t> { static constexpr float value = 448.f; };

// Of magnitudes (sign cleared), as their bits: a NaN is the largest and stays.
struct MaxMagnitude {
    __device__ __forceinline__ float operator()(float a, float b) const { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }
};
__device__ __forceinline__ float magnitude(float x) { return __uint_as_float(__float_as_uint(x) & 0x7fffffffu); }

// f(e, v of lane e) of the 16 lanes of this lane's row of lanes: an operand of the instruction that uses it
template <int E = 0, typename F>
__device__ __forceinline__ void of_rows(float v, F f) {
    if constexpr (E < 16) {
        f(E, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x150 + E, 0xf, 0xf, false)));
        of_rows<E + 1>(v, f);
    }
}

struct RowScale { float scale, inv; };     // value = code * scale, code = value * inv
template <typename T>
__device__ __forceinline__ RowScale row_scale(float most) {
    const float a = fminf(most, kScaledMost);
    RowScale s = {a / MostCode<T>::value, MostCode<T>::value / a};
    if (a < kScaledLeast) s = {0.f, 0.f};
    if (most != most) s = {most, 0.f};
    return s;
}

// Products and sums of a rotation are rounded each, not contracted: a key has the same codes whichever kernel turned it, and those that separate operations give.
__device__ __forceinline__ void turned(float& lo, float& hi, float2 cs) {
#pragma clang fp contract(off)
    const float a = lo * cs.x, b = hi * cs.y, c = hi * cs.x, d = lo * cs.y;
    lo = a - b;
    hi = c + d;
}

// N codes (2 or a multiple of 4) of values x already multiplied by inv, in order from the lowest byte.  The bounds are for infinities.  Whole numbers: the last byte of 1.5 2^23 + x is x to nearest even, as long as
// the product that x is has been rounded by itself.
template <typename T, int N>
__device__ __forceinline__ void encode(const float (&x)[N], uint32_t (&w)[(N + 3) / 4]) {
#pragma clang fp contract(off)
    constexpr float Q = MostCode<T>::value;
    constexpr int PER = N < 4 ? N : 4;
#pragma unroll
    for (int j = 0; j < (N + 3) / 4; ++j) {
        float y[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) y[e] = __builtin_amdgcn_fmed3f(x[4 * j + e], -Q, Q);
        if constexpr (Q == 127.f) {
            uint32_t b[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) b[e] = __float_as_uint(y[e] + 12582912.f);
            w[j] = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
            if constexpr (PER == 4) w[j] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), w[j], 0x05040100u);
        } else {
            w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            if constexpr (PER == 4) w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w[j], true);
        }
    }
}

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
// The four codes of a word as fp16, which holds every code of either type.  i8: the bytes with their signs turned over are the last digits of 1024 + 0 ... 1024 + 255.
template <typename T>
__device__ __forceinline__ void decode4(uint32_t w, half2_t& lo, half2_t& hi) {
    if constexpr (MostCode<T>::value == 127.f) {
        w ^= 0x80808080u;
        const half2_t base = {(_Float16)1152.f, (_Float16)1152.f};
        lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04010400u)) - base;
        hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, w, 0x04030402u)) - base;
    } else {
        lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
        hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true);
    }
}

}  // namespace d3
