// Microscaled numbers: blocks of 32 neighbouring values of a row share a power of two, 2^(s - 127) for the scale byte s, and are held as 8-bit (e4m3:
// 1, 1.125, ... up to 448) or 4-bit (e2m1: 0, 0.5, 1, 1.5, 2, 3, 4, 6) floating point numbers of its multiples.
//   s: the smallest with which no value of the block lies behind the largest element (so nothing saturates and every element is
//      off by at most half a step), kept where the smallest element is a normal bf16 and the largest a finite one: what a block stands for
//      is exact in bf16.  (Rounding the largest value's exponent down instead, so that it may lie up to 2^-3 behind the largest element, e4m3, or a third,
//      e2m1, and is cut off there, would make the other steps of such blocks half as long.)
//   elements: the nearest, ties to the even one, the value's sign kept; a block with an infinity or a NaN has scale 255 and is NaN.
#pragma once
#include "lotts_common.h"

namespace lotts {

constexpr int kMxBlock = 32;
constexpr unsigned kMxNaN = 255;

struct E4M3 {
    static constexpr int kExponent = 8;               // of the largest element, 1.75 * 2^8
    static constexpr unsigned kFraction = 0x600000;   // of the largest element
    static constexpr int kLo = 10, kHi = 246;         // 2^-9 * 2^-117 = 2^-126; 448 * 2^119 < 2^128
};
struct E2M1 {
    static constexpr int kExponent = 2;               // 1.5 * 2^2
    static constexpr unsigned kFraction = 0x400000;
    static constexpr int kLo = 2, kHi = 252;          // 2^-1 * 2^-125 = 2^-126; 6 * 2^125 < 2^128
};

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 mx_bf16x8 __attribute__((ext_vector_type(8)));
typedef float mx_f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned mx_u32x4 __attribute__((ext_vector_type(4)));

// Scale byte of a block from the largest magnitude's bits.
template <class E>
__device__ __forceinline__ unsigned mx_scale(unsigned largest) {
    const int s = (int)(largest >> 23) - E::kExponent + ((largest & 0x7fffff) > E::kFraction);
    return largest >= 0x7f800000u ? kMxNaN : (unsigned)min(max(s, E::kLo), E::kHi);
}
__device__ __forceinline__ float mx_power(unsigned s) { return __uint_as_float(s << 23); }
// What the values of a block are multiplied with: 2^(127 - s).  Exact, so the element is rounded once.
__device__ __forceinline__ float mx_inverse(unsigned s) { return mx_power(254 - min(s, 253u)); }

// Largest magnitude's bits (an infinity's and a NaN's are larger than any number's) of a lane's eight values and its three neighbours': four lanes hold a block.
__device__ __forceinline__ unsigned mx_largest(const float (&x)[8]) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    m = max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, false));   // quad_perm 1 0 3 2
    return max(m, (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, false));  // quad_perm 2 3 0 1
}

// Eight values of a block with scale s: as e4m3, 8 bytes; as e2m1, 4 bytes, the lower half of a byte first.
__device__ __forceinline__ uint2 mx_to_e4m3(const float (&x)[8], unsigned s) {
    const float inv = mx_inverse(s);
    int w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = fminf(fmaxf(x[i * 4 + j] * inv, -448.f), 448.f);  // (beyond 448 with the largest scale only)
        w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w[i], true);
    }
    const bool nan = s == kMxNaN;
    return make_uint2(nan ? 0x7f7f7f7fu : (unsigned)w[0], nan ? 0x7f7f7f7fu : (unsigned)w[1]);
}
__device__ __forceinline__ unsigned mx_to_e2m1(const float (&x)[8], unsigned s) {
    const float inv = mx_inverse(s);
    unsigned w = 0;  // (the conversion ends at 6)
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0] * inv, x[1] * inv, 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2] * inv, x[3] * inv, 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4] * inv, x[5] * inv, 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6] * inv, x[7] * inv, 1.0f, 3);
    return s == kMxNaN ? 0 : w;
}

// Eight elements as bf16, exact under the scales that are written here; under others (below 2^-126 bf16 has fewer bits) the nearest, ties to the even one, infinite
// from 2^128 on.  Scale 255 makes every element NaN.
__device__ __forceinline__ mx_bf16x8 mx_of_e2m1(unsigned w, unsigned s) {
    const float scale = mx_power(s);
    const mx_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1),
                    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return mx_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ mx_bf16x8 mx_of_e4m3(unsigned lo, unsigned hi, unsigned s) {
    const float scale = mx_power(s);
    const mx_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                    c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return mx_bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// Four e4m3 elements as fp32, exact under any scale, infinite from 2^128 on.
__device__ __forceinline__ float4 mx_f32_of_e4m3(unsigned w, unsigned s) {
    const mx_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, mx_power(s), false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, mx_power(s), true);
    return make_float4(a[0], a[1], b[0], b[1]);
}

// Eight bf16 or fp32 values, 16-byte aligned.
template <typename T>
struct MxSource;
template <>
struct MxSource<__bf16> {
    mx_bf16x8 v;
    __device__ __forceinline__ void load(const void* p) { v = *static_cast<const mx_bf16x8*>(p); }
    __device__ __forceinline__ void values(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
};
template <>
struct MxSource<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const void* p) {
        a = static_cast<const float4*>(p)[0];
        b = static_cast<const float4*>(p)[1];
    }
    __device__ __forceinline__ void values(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
};

}  // namespace lotts
