// The two low-bit formats of the serving operators and the storage types around them.
// 8 bits: e4m3 codes times 2^e, e per block; 4 bits: e2m1 codes times 2^e, e per 32 values.  A scale is kept
// as the byte e + 127, which is what the scaled matrix instructions take and, shifted by 23, the float32 2^e.
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_fp16.h>
#include <stdint.h>
#include "nnv.h"

namespace nnv {

template <int DT> struct Elem;
template <> struct Elem<NNV_F32> { typedef float type; };
template <> struct Elem<NNV_F16> { typedef _Float16 type; };
template <> struct Elem<NNV_BF16> { typedef __bf16 type; };
template <int DT, int N> using ElemVec = typename Elem<DT>::type __attribute__((ext_vector_type(N)));

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr uint32_t kInfBits = 0x7f800000u;

// 2^e of a scale byte.
__device__ static inline float scale_of_byte(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }
// 2^-e; bytes are 1 .. 253, so that both are normal numbers.
__device__ static inline float inverse_of_byte(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// Scale byte of a block of e4m3 codes from the bits of its largest magnitude: the smallest e with amax <= 448 * 2^e, which
// is 1.75 * 2^(e + 8).  Magnitudes compare as their bits do; of a block that holds an infinity or a NaN any scale will do.
__device__ static inline uint32_t e4m3_scale_byte(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);      // e + 127
    return (uint32_t)(e < 1 ? 1 : e);
}

// Four values divided by the block's scale as e4m3 codes.  The division is exact and stays within +-448, so the conversion rounds
// once and never saturates; what is not finite becomes the format's NaN.
__device__ static inline uint32_t e4m3_code4(float a, float b, float c, float d, float inverse) {
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, v, true);
}
__device__ static inline uint32_t e4m3_nan_where(uint32_t codes, float a, float b, float c, float d) {
    auto bad = [](float v, int at) { return (__builtin_bit_cast(uint32_t, v) & kInfBits) == kInfBits ? 0x7fu << at : 0u; };
    const uint32_t set = bad(a, 0) | bad(b, 8) | bad(c, 16) | bad(d, 24);
    return codes | set;
}

// Largest scale bytes of the 4-bit format: what the codes stand for stays finite in the cache's 16-bit type (6 * 2^125; 6 * 2^13).
template <int DT> constexpr uint32_t kMostE2m1Byte = DT == NNV_F16 ? 127 + 13 : 127 + 125;

// Scale byte of 32 values from the bits of their largest (finite) magnitude: the smallest e with amax < 7 * 2^e = 1.75 * 2^(e + 2).
template <int DT> __device__ static inline uint32_t e2m1_scale_byte(uint32_t amax_bits) {
    const int e = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7fffffu) >= 0x600000u ? 1 : 0);
    return (uint32_t)(e < 1 ? 1 : e > (int)kMostE2m1Byte<DT> ? (int)kMostE2m1Byte<DT> : e);
}

// What the 4-bit format can take of a value: a NaN counts as 0, an infinity as the largest float32.
__device__ static inline float e2m1_input(float v) {
    const uint32_t a = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    if (a < kInfBits) return v;
    return a > kInfBits ? 0.f : __builtin_copysignf(3.4028234663852886e38f, v);
}

// Rounds to the neighbour of odd last bit where the value is not a float32: a later rounding to a few bits is then that of the value itself.
__device__ static inline float float_odd(double x) {
    const float f = (float)x;
    const double back = (double)f;
    if (back == x || !(__builtin_fabs(x) < 3.4028234663852886e38)) return f;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (__builtin_fabs(back) > __builtin_fabs(x)) u -= 1;
    return __builtin_bit_cast(float, u | 1u);
}

}  // namespace nnv
