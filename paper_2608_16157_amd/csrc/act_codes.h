// 8-bit form of activations and gradients (ft_act_codes_t): device helpers shared by the kernels that
// write it and the products that read it; internal.
//
// A block of 128 values with largest finite magnitude a takes the scale 2^e, e the smallest integer with
// 448 * 2^e >= a (0 for a = 0, clamped to [-127, 127]), and the codes e4m3fn(v / 2^e), rounded to
// nearest, ties to even; values that are not finite take a NaN code.
#pragma once

#include "ftmoe_device.h"

namespace ftmoe {

typedef int i32x8_vec_t __attribute__((ext_vector_type(8)));
typedef short i16x2_vec_t __attribute__((ext_vector_type(2)));

// magnitude bits of v for the block maximum: those of non-negative floats order as integers, and what is
// not finite does not count
__device__ __forceinline__ uint32_t act_mag_bits(float v) {
    const uint32_t u = __float_as_uint(v) & 0x7FFFFFFFu;
    return u < 0x7F800000u ? u : 0u;
}

// e + 127 (the e8m0 byte) of a block whose largest magnitude has the bits u.  a = 1.m * 2^x and 448 =
// 1.75 * 2^8, so e = x - 8, one more if 1.m > 1.75; a subnormal a clamps to -127 in any case.
__device__ __forceinline__ int act_scale_byte(uint32_t u) {
    const int byte = static_cast<int>(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return u == 0 ? 127 : max(byte, 0);   // u is finite: byte <= 247
}

// The scaled conversions read their scale operand's exponent field as an e8m0 byte (0: 2^-127): measured
// equal to rounding v * 2^-e in one step, ties to even, for every bf16 value and exponent, subnormal
// codes included.
__device__ __forceinline__ float act_scale_operand(int byte) {
    return __uint_as_float(static_cast<uint32_t>(byte) << 23);
}

// four codes in one word, v0 in the low byte
__device__ __forceinline__ uint32_t act_codes4(float v0, float v1, float v2, float v3, float scale) {
    i16x2_vec_t r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v0, v1, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v2, v3, scale, true);
    return __builtin_bit_cast(uint32_t, r);
}

// four values of one word of codes, times the scale (exact in float32: 4 significant bits)
typedef float f32x2_vec_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void act_values4(uint32_t w, float scale, float *v) {
    const f32x2_vec_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, false);
    const f32x2_vec_t hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, scale, true);
    v[0] = lo[0];
    v[1] = lo[1];
    v[2] = hi[0];
    v[3] = hi[1];
}

// eight codes times a power of two -> eight bf16 (exact: 4 significant bits)
__device__ __forceinline__ bf16x8_t act_bf16x8(uint32_t w0, uint32_t w1, float scale) {
    auto pk = [](bf16x2_vec_t v) { return __builtin_bit_cast(uint32_t, v); };
    return as_bf16x8(u32x4_t{pk(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false)),
                             pk(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true)),
                             pk(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false)),
                             pk(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true))});
}

// eight consecutive elements of a bf16 or float32 row (16-byte aligned)
__device__ __forceinline__ void load8(const uint16_t *p, float *v) {
    const uint4 r = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float *p, float *v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float4 r = reinterpret_cast<const float4 *>(p)[i];
        v[4 * i] = r.x;
        v[4 * i + 1] = r.y;
        v[4 * i + 2] = r.z;
        v[4 * i + 3] = r.w;
    }
}

// Values as they come from memory, with signalling NaNs made quiet.  Results of arithmetic are quiet already.
template <int N>
__device__ __forceinline__ void quiet(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_canonicalizef(v[i]);
}

// max(m, |a|, |b|) in one instruction.  The compiler takes four: it clears the signs and quiets the operands
// first.  A quiet NaN drops out.  A signalling one would take the maximum so far with it (it makes that a quiet NaN,
// which the next step drops), so values of memory go through quiet() before.
__device__ __forceinline__ float max3_abs(float m, float a, float b) {
    float r;
    asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(r) : "v"(m), "v"(a), "v"(b));
    return r;
}

// Largest finite magnitude of N values (N even).  The plain maximum first: only what is not finite reaches the
// bits of infinity, and then the values are looked at again one by one.
template <int N>
__device__ __forceinline__ uint32_t mag_of(const float *v) {
    float f = 0.0f;
#pragma unroll
    for (int i = 0; i < N; i += 2) f = max3_abs(f, v[i], v[i + 1]);
    uint32_t m = __float_as_uint(f);
    if (m >= 0x7F800000u) {
        m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) m = max(m, act_mag_bits(v[i]));
    }
    return m;
}

// a block's 128 values: 8 in each of the 16 lanes of a lane row, or 16 in each of the 8 lanes of half of one
__device__ __forceinline__ uint32_t block_mag16(const float *v) { return row_max_u32(mag_of<8>(v)); }
__device__ __forceinline__ uint32_t eight_max_u32(uint32_t m) {
    m = max(m, dpp_u32<0xB1>(m));       // quad_perm: lane ^ 1
    m = max(m, dpp_u32<0x4E>(m));       // quad_perm: lane ^ 2
    return max(m, dpp_u32<0x141>(m));   // row_half_mirror: 7 - lane
}
__device__ __forceinline__ uint32_t block_mag8(const float *v) { return eight_max_u32(mag_of<16>(v)); }

// float32 -> bf16, round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t f32_to_bf16_any(float f) {
    const uint32_t u = __float_as_uint(f);
    return f != f ? 0x7FC0u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// two of them in one instruction, a in the low half; a NaN keeps its sign and payload, made quiet
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

}  // namespace ftmoe
