// Device-side building blocks of the microscaled 4-bit operators (include/lutq.h: form, rounding, layout).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lutq {
namespace mx4 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How values are held outside the 4-bit form.
enum Source { kF32 = 0, kF16 = 1, kBF16 = 2 };

// What eight neighbouring values are loaded as.
template <int SRC> struct Eight { u32x4 v[SRC == kF32 ? 2 : 1]; };

// The largest magnitude so far, as a bit pattern: magnitudes order as integers, a NaN above infinity above every number.  16-bit
// values are compared two at a time, `a` holds one maximum per half.
template <int SRC> __device__ __forceinline__ void max_bits(uint32_t v, uint32_t& a) {
    if constexpr (SRC == kF32) {
        a = max(a, v & 0x7fffffffu);
    } else {
        const u16x2 m = __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, v & 0x7fff7fffu));
        a = __builtin_bit_cast(uint32_t, m);
    }
}

// The exponent byte of a block from its largest magnitude: the biased fp32 exponent less two (6 = 1.5 * 2^2 is the largest
// code), at least 0.  A biased exponent of 0 or 1 stands for magnitudes below 2^-125, whose byte is 0 by the rule; 255 stays.
template <int SRC> __device__ __forceinline__ uint32_t exponent_byte(uint32_t a) {
    uint32_t b = a;
    if constexpr (SRC != kF32) {
        const uint32_t h = max(a & 0xffffu, a >> 16);
        b = SRC == kBF16 ? h << 16 : __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)h));
    }
    b >>= 23;
    return b == 255u ? 255u : b < 2u ? 0u : b - 2u;
}

// The power of two as the conversion instructions take it: they read the exponent field only, 0 as 2^-127.
__device__ __forceinline__ float power_of(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// (by value: a cast of a vector's element in place reads the vector's first one)
template <typename T> __device__ __forceinline__ T pair(uint32_t v) { return __builtin_bit_cast(T, v); }

// Eight values to a word of codes, in order: one instruction per pair divides by the power of two, rounds to the nearest (ties to the
// even code) and keeps 6 beyond it.
template <int SRC> __device__ __forceinline__ uint32_t to_codes(const Eight<SRC>& x, float power) {
    uint32_t r = 0;
    if constexpr (SRC == kF32) {
        const f32x4 a = __builtin_bit_cast(f32x4, x.v[0]), b = __builtin_bit_cast(f32x4, x.v[1]);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a[0], a[1], power, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a[2], a[3], power, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, b[0], b[1], power, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, b[2], b[3], power, 3);
    } else if constexpr (SRC == kF16) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair<f16x2>(x.v[0][0]), power, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair<f16x2>(x.v[0][1]), power, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair<f16x2>(x.v[0][2]), power, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, pair<f16x2>(x.v[0][3]), power, 3);
    } else {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair<bf16x2>(x.v[0][0]), power, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair<bf16x2>(x.v[0][1]), power, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair<bf16x2>(x.v[0][2]), power, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, pair<bf16x2>(x.v[0][3]), power, 3);
    }
    return r;
}

// The exponent byte of the block that this lane's quad holds, and the lane's word of codes.
template <int SRC> __device__ __forceinline__ uint32_t quantize_eight(const Eight<SRC>& x, uint32_t& e) {
    uint32_t a = 0;
#pragma unroll
    for (int j = 0; j < (SRC == kF32 ? 8 : 4); ++j) max_bits<SRC>(x.v[j / 4][j % 4], a);
    // (quad_perm 1 0 3 2 and 2 3 0 1)
    max_bits<SRC>((uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xb1, 0xf, 0xf, true), a);
    max_bits<SRC>((uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4e, 0xf, 0xf, true), a);
    e = exponent_byte<SRC>(a);
    const uint32_t c = to_codes<SRC>(x, power_of(e));
    return e == 255u ? 0u : c;
}

// A word of codes back to eight 16-bit values.
template <bool BF16> __device__ __forceinline__ u32x4 from_codes(uint32_t c, float power) {
    u32x4 r;
    if constexpr (BF16) {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, power, 3));
    } else {
        r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, power, 0));
        r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, power, 1));
        r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, power, 2));
        r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, power, 3));
    }
    return r;
}

// Two sums to a word of the 16-bit type, rounded to the nearest even.
__device__ __forceinline__ uint32_t round_pair(float a, float b, bool bf16) {
    if (bf16) { const bf16x2 r = {(__bf16)a, (__bf16)b}; return __builtin_bit_cast(uint32_t, r); }
    const f16x2 r = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, r);
}

// acc[n, m] += W X^T of 16 rows of weights, 16 rows of activations and 128 columns.  Lane 16 o + i holds row i, columns
// 32 o .. 32 o + 31 of either factor and their exponent, in byte SW (SX) of the word given; acc is rows 4 o .. 4 o + 3 of W, row i of X.
template <int SW, int SX>
__device__ __forceinline__ f32x4 product(u32x4 w, u32x4 x, f32x4 acc, uint32_t we, uint32_t xe) {
    const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    const i32x8 b = {(int)x[0], (int)x[1], (int)x[2], (int)x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, SW, (int)we, SX, (int)xe);
}

}  // namespace mx4
}  // namespace lutq
