// Device-side building blocks of the 8-bit operators (include/lutq.h: form, rounding).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lutq_mx4_device.hpp"

namespace lutq {
namespace fp8 {

using mx4::bf16x2;
using mx4::Eight;
using mx4::f16x2;
using mx4::f32x2;
using mx4::f32x4;
using mx4::i32x8;
using mx4::kBF16;
using mx4::kF16;
using mx4::kF32;
using mx4::pair;
using mx4::round_pair;
using mx4::u32x2;
using mx4::u32x4;

template <int SRC> __device__ __forceinline__ void to_floats(const Eight<SRC>& x, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (SRC == kF32) v[j] = pair<float>(x.v[j / 4][j % 4]);
        else if constexpr (SRC == kBF16) v[j] = pair<float>(j & 1 ? x.v[0][j / 2] & 0xffff0000u : x.v[0][j / 2] << 16);
        else v[j] = (float)pair<f16x2>(x.v[0][j / 2])[j & 1];
    }
}

// Magnitudes as bit patterns, which order as integers, a NaN above infinity above every number.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t largest(const float (&v)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) a = max(a, magnitude(v[j]));
    return a;
}
// The largest over the sixteen lanes of a row (quad_perm 1 0 3 2 and 2 3 0 1, row_ror 4 and 8).
__device__ __forceinline__ uint32_t largest_of_sixteen(uint32_t a) {
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true));
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true));
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x124, 0xf, 0xf, true));
    return max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x128, 0xf, 0xf, true));
}

// A block's scale and what its values are multiplied with, from its largest magnitude.  One division each, rounded to the nearest, and at
// least 2^-110: 448 / 2^-110 is still a number.  A block that is not finite has no scale, and codes of 0.
struct Scale { float scale, inverse; bool bad; };
constexpr uint32_t kFloorBits = (127u - 110u) << 23, kInfBits = 0x7f800000u;
__device__ __forceinline__ Scale scale_of(uint32_t bits) {
    const float a = __builtin_bit_cast(float, max(bits, kFloorBits));
    const bool bad = bits >= kInfBits;
    return {bad ? __builtin_nanf("") : a / 448.0f, bad ? 0.0f : 448.0f / a, bad};
}
// The least power of two that is at least a / 448 = a / (1.75 * 2^8): the exponent of a less eight, one more where its mantissa is
// above 1.75.
__device__ __forceinline__ Scale power_of_two_scale_of(uint32_t bits) {
    const uint32_t e = ((max(bits, kFloorBits) + 0x1fffffu) >> 23) - 8u;
    const bool bad = bits >= kInfBits;
    return {bad ? __builtin_nanf("") : __builtin_bit_cast(float, e << 23), bad ? 0.0f : __builtin_bit_cast(float, (254u - e) << 23), bad};
}

// Eight values to codes, in order: rounded to the nearest, ties to the even code.  (At most 448 (1 + 2^-23) comes here, which rounds to 448.)
__device__ __forceinline__ u32x2 to_codes(const float (&v)[8], const Scale& s) {
    u32x2 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h] * s.inverse, v[4 * h + 1] * s.inverse, 0, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2] * s.inverse, v[4 * h + 3] * s.inverse, c, true);
        r[h] = s.bad ? 0u : (uint32_t)c;
    }
    return r;
}

// Eight codes back to 16-bit values: the product with the scale in 32 bits, rounded to the nearest.
__device__ __forceinline__ u32x4 from_codes(u32x2 c, float scale, bool bf16) {
    u32x4 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[h], true);
        r[2 * h] = round_pair(a[0] * scale, a[1] * scale, bf16);
        r[2 * h + 1] = round_pair(b[0] * scale, b[1] * scale, bf16);
    }
    return r;
}

// The sums over 128 columns of the codes of sixteen rows of W times sixteen of X.  Lane 16 o + i holds row i of either, the same 32 columns of both
// in any order; its four sums are rows 4 o .. 4 o + 3 of W, row i of X.  (The instruction's own scales are 1.)
__device__ __forceinline__ f32x4 product(const i32x8& w, const i32x8& x, const f32x4& acc) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, 0, 127, 0, 127);
}
// The same with scales that are powers of two, as the biased exponents in the low bytes of the words given.
__device__ __forceinline__ f32x4 scaled_product(const i32x8& w, const i32x8& x, const f32x4& acc, uint32_t we, uint32_t xe) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, acc, 0, 0, 0, (int)we, 0, (int)xe);
}
// It adds eight neighbours' products (of a lane's columns) in fewer bits than fp32 has: what lies below 2^-13 of the power of two of the largest
// is cut off, 2^-18 of the sum of magnitudes on random codes.  The 16-bit instruction does not (2^-30), at half the rate: the same sums of
// the codes as 16-bit numbers, which hold them exactly.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
struct Wide { u32x4 v[4]; };
// Pair `n` of the sixteen that a lane's 32 codes make, into its place.
__device__ __forceinline__ void widen_pair(Wide& to, const i32x8& c, int n) {
    const uint32_t four = (uint32_t)c[n >> 1];
    const f16x2 h = n & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, 1.0f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(four, 1.0f, false);
    to.v[n >> 2][n & 3] = __builtin_bit_cast(uint32_t, h);
}
__device__ __forceinline__ Wide widen(const i32x8& c) {
    Wide r;
#pragma unroll
    for (int n = 0; n < 16; ++n) widen_pair(r, c, n);
    return r;
}
// Quarter q of the product: 32 of the columns.
__device__ __forceinline__ f32x4 product(const Wide& w, const Wide& x, const f32x4& acc, int q) {
    const u32x4 a = w.v[q], b = x.v[q];
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 product(const Wide& w, const Wide& x, f32x4 acc) {
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = product(w, x, acc, q);
    return acc;
}
__device__ __forceinline__ i32x8 operand(u32x4 a, u32x4 b) {
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// The gate's activation g sigma(z), z = g, or 2 sqrt(2 / pi) (g + 0.044715 g^3) (gelu in its tanh form), and its derivative
// sigma + g sigma (1 - sigma) z'.  exp and the reciprocal are the hardware's: sigma is off by some steps of 2^-24 relative to it, and by about |z| as
// many, since z log2 e is rounded before the power of two is taken ((16 + 8 |z|) 2^-24 holds everywhere); beyond the ends it is 0 or 1.
enum Activation { kSilu = 0, kGelu = 1 };
__device__ __forceinline__ float sigma(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }
__device__ __forceinline__ float argument(float g, int act) { return act == kSilu ? g : 1.5957691216057308f * (g + 0.044715f * g * g * g); }
__device__ __forceinline__ float activated(float g, int act) { return g * sigma(argument(g, act)); }
__device__ __forceinline__ void activated(float g, int act, float& f, float& slope) {
    const float s = sigma(argument(g, act)), rest = 1.0f - s;
    f = g * s;
    // (Beyond the ends f rest is 0 and stays it, whatever g is: z' by itself passes fp32's largest number from |g| = 5e19 on, and 0 times that would be no
    // number.  Holding g at +-64 for it instead takes one instruction more, 159 us for 147 at 4096 x 14336.)
    const float t = f * rest;
    slope = act == kSilu ? s + t : s + 1.5957691216057308f * (t + 0.134145f * (t * g * g));
}

}  // namespace fp8
}  // namespace lutq
