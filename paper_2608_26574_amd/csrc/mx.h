// Device-side helpers of the microscaled (MX) kernels.
//
// OCP microscaling: 32 consecutive values share a scale 2^(c - 127), c one
// byte (E8M0; 255 = NaN), the elements are E4M3 (DARD_MX_FP8) or E2M1
// (DARD_MX_FP4, two to a byte, the even one in the low nibble).  The scale's
// exponent is floor(log2(largest magnitude)) - emax, emax the exponent of the
// element type's largest value (448: 8, 6: 2), so scaled magnitudes are below
// 2^(emax + 1) and only those past the largest value saturate.
#pragma once

#include "common.h"

namespace dard {

constexpr int kMxBlock = 32;

template <int F> struct Mx;   // element format
template <> struct Mx<DARD_MX_FP8> {
    static constexpr int kEmax = 8, kMant = 3, kEmin = -6;
    static constexpr float kTop = 448.f;
    static constexpr int kMfma = 0;   // operand format code of the scaled matrix instructions
};
template <> struct Mx<DARD_MX_FP4> {
    static constexpr int kEmax = 2, kMant = 1, kEmin = 0;
    static constexpr float kTop = 6.f;
    static constexpr int kMfma = 4;
};

typedef int intx8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Largest of a value over the four lanes of a quad (two quad permutations).
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    const uint32_t a = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true);   // lanes 1 0 3 2
    v = v > a ? v : a;
    const uint32_t b = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true);   // lanes 2 3 0 1
    return v > b ? v : b;
}

// Scale code of a block whose largest magnitude has float32 exponent field E
// (255: the block holds an infinity or a NaN and reads as NaN).
template <int F> __device__ __forceinline__ uint32_t mx_scale(uint32_t E) {
    if (E == 255u) return 255u;
    return E > (uint32_t)Mx<F>::kEmax ? E - Mx<F>::kEmax : 0u;
}

// Eight scaled values (already within the element type's range, or clamped
// here) to element codes, little-endian: 8 bytes (FP8) or 4 (FP4, in x).  The
// hardware conversions round to nearest even; beyond 448 the E4M3 one gives
// NaN, hence the clamp.
template <int F> __device__ __forceinline__ uint2 mx_encode8(const float (&t)[8]) {
    float c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = fminf(fmaxf(t[i], -Mx<F>::kTop), Mx<F>::kTop);
    if constexpr (F == DARD_MX_FP8) {
        int a = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
        a = __builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], a, true);
        int b = __builtin_amdgcn_cvt_pk_fp8_f32(c[4], c[5], 0, false);
        b = __builtin_amdgcn_cvt_pk_fp8_f32(c[6], c[7], b, true);
        return make_uint2((uint32_t)a, (uint32_t)b);
    } else {
        uint32_t a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, c[0], c[1], 1.0f, 0);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, c[2], c[3], 1.0f, 1);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, c[4], c[5], 1.0f, 2);
        a = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(a, c[6], c[7], 1.0f, 3);
        return make_uint2(a, 0u);
    }
}

// The scale as a float operand of the hardware conversions, which read its
// exponent field alone (0 stands for 2^-127, 255 makes every value NaN).
__device__ __forceinline__ float mx_scale_f(uint32_t code) { return __uint_as_float(code << 23); }

// Two E2M1 codes (byte SEL of x) times a scale as two bf16 values: exact.
template <int SEL> __device__ __forceinline__ uint32_t fp4x2_to_bf16x2(uint32_t x, float scale) {
    const bf16x2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, scale, SEL);
    return __builtin_bit_cast(uint32_t, r);
}

// The float32 value of an E4M3 or E2M1 code (the low byte / nibble of c).
template <int F> __device__ __forceinline__ float mx_value(uint32_t c) {
    if constexpr (F == DARD_MX_FP8) {
        return __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
    } else {
        return __uint_as_float((uint32_t)fp4x2_to_bf16x2<0>(c & 15u, 1.0f) << 16);
    }
}

// Eight consecutive values as floats; p only as aligned as its element.
__device__ __forceinline__ void ld_8(const float* p, float (&v)[8]) {
    const floatx4 a = ld_f4(p), b = ld_f4(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
}
__device__ __forceinline__ void ld_8(const bf16_t* p, float (&v)[8]) {
    typedef uint32_t u4 __attribute__((ext_vector_type(4), aligned(2)));
    const u4 w = *reinterpret_cast<const u4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

}  // namespace dard
