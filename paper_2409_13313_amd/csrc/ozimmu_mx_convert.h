// Element types and block conversion of the microscaled 4-bit form, shared by the kernels.
#pragma once
#include "ozimmu_mx.h"

namespace mxk {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

template <int TYPE> struct Elem;
template <> struct Elem<F32> { typedef uint32_t Bits; };
template <> struct Elem<BF16> { typedef uint16_t Bits; };
template <> struct Elem<F16> { typedef uint16_t Bits; };

// Largest magnitude of N elements (N even) as an integer: magnitudes are ordered as their bits are, NaN above infinity.
// (16-bit types: two at a time.)  f32_bits() makes such an integer the bits of the FP32 value.
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
template <int TYPE, int N> __device__ inline uint32_t max_magnitude(const typename Elem<TYPE>::Bits* x)
{
    if constexpr (TYPE == F32) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t a = x[i] & 0x7fffffffu;
            m = a > m ? a : m;
        }
        return m;
    } else {
        v2u16 m = {0, 0};
#pragma unroll
        for (int i = 0; i < N; i += 2)
            m = __builtin_elementwise_max(m, __builtin_bit_cast(v2u16, ((uint32_t)x[i] | (uint32_t)x[i + 1] << 16) & 0x7fff7fffu));
        return m[0] > m[1] ? m[0] : m[1];
    }
}
template <int TYPE> __device__ inline uint32_t f32_bits(uint32_t magnitude)
{
    if constexpr (TYPE == F32) return magnitude;
    if constexpr (TYPE == BF16) return magnitude << 16;
    if constexpr (TYPE == F16) return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)magnitude));
}

// scale byte of a block whose largest magnitude has these bits: floor(log2) - 2, biased, at least 0; 255 for infinities and NaN
__device__ inline uint32_t scale_byte(uint32_t amax)
{
    const uint32_t e = amax >> 23;  // (0 for subnormals: their scale is the least one anyway)
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
// that scale as an FP32 value (2^-127 is subnormal; the NaN block's codes are made with some finite scale)
__device__ inline float scale_value(uint32_t b) { return __uint_as_float(b == 0u ? 0x00400000u : (b == 255u ? 0x7f000000u : b << 23)); }

// 8 elements -> 8 codes.  The conversion instruction divides by the (power of two) scale, rounds to nearest even and saturates.
template <int TYPE> __device__ inline uint32_t codes8(const typename Elem<TYPE>::Bits* x, float scale)
{
    uint32_t r = 0;
    if constexpr (TYPE == F32) {
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(x[0]), __uint_as_float(x[1]), scale, 0);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(x[2]), __uint_as_float(x[3]), scale, 1);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(x[4]), __uint_as_float(x[5]), scale, 2);
        r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, __uint_as_float(x[6]), __uint_as_float(x[7]), scale, 3);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = (uint32_t)x[2 * i] | (uint32_t)x[2 * i + 1] << 16;
        if constexpr (TYPE == BF16) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[0]), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[1]), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[2]), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[3]), scale, 3);
        } else {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2h, w[0]), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2h, w[1]), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2h, w[2]), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, __builtin_bit_cast(v2h, w[3]), scale, 3);
        }
    }
    return r;
}

// 8 codes -> 8 elements, rounded where the type cannot hold code times scale.  The conversion instruction multiplies by the power of two
// whose exponent bits the scale has; a NaN is put in here.
template <int TYPE> __device__ inline void values8(uint32_t codes, uint32_t b, typename Elem<TYPE>::Bits* x)
{
    const float s = scale_value(b);
    if constexpr (TYPE == F32) {
        typedef float v2f __attribute__((ext_vector_type(2)));
        const v2f v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3)};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = b == 255u ? 0x7fc00000u : __float_as_uint(v[e / 2][e % 2]);
    } else {
        uint32_t w[4];
        if constexpr (TYPE == BF16) {
            w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
            w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
            w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
            w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
        } else {
            w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 0));
            w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 1));
            w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 2));
            w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 3));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = b == 255u ? (TYPE == BF16 ? 0x7fc07fc0u : 0x7e007e00u) : w[i];
            x[2 * i] = (uint16_t)w[i];
            x[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
}

// FP32 -> element, one rounding (nearest even)
template <int TYPE> __device__ inline typename Elem<TYPE>::Bits from_float(float v)
{
    if constexpr (TYPE == F32) return __float_as_uint(v);
    if constexpr (TYPE == BF16) return __builtin_bit_cast(uint16_t, (__bf16)v);
    if constexpr (TYPE == F16) return __builtin_bit_cast(uint16_t, (_Float16)v);
}
template <int TYPE> __device__ inline float to_float(typename Elem<TYPE>::Bits x)
{
    if constexpr (TYPE == F32) return __uint_as_float(x);
    if constexpr (TYPE == BF16) return __uint_as_float((uint32_t)x << 16);
    if constexpr (TYPE == F16) return (float)__builtin_bit_cast(_Float16, x);
}

// N consecutive elements from any element address in as few loads as the hardware needs (dword loads take any alignment);
// those at and behind `left` are zeros
template <int TYPE, int N> __device__ inline void load_row(const typename Elem<TYPE>::Bits* p, int64_t left, typename Elem<TYPE>::Bits* x)
{
    if (left >= N) {
        __builtin_memcpy(x, p, N * sizeof(*x));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < left ? p[i] : 0;
    }
}
template <int TYPE, int N> __device__ inline void store_row(typename Elem<TYPE>::Bits* p, int64_t left, const typename Elem<TYPE>::Bits* x)
{
    if (left >= N) {
        __builtin_memcpy(p, x, N * sizeof(*x));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) p[i] = x[i];
    }
}

}  // namespace mxk
