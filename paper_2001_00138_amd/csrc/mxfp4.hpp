// MXFP4 on the device: blocks of 32 values that share a power of two, four bits a value.
//
// Scale byte b stands for 2^(b-127), 255 for a block that held something not finite (its values are NaN); a code's
// low three bits select 0, 0.5, 1, 1.5, 2, 3, 4, 6 and bit 3 is the sign.  b - 127 = floor(log2(largest magnitude)) - 2, at
// least -127, so that the largest value becomes 4 to 8 units (above 6 it becomes 6); the conversion instructions
// divide by the power of two and round to the nearest code, ties to the even one.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "element.hpp"

namespace patdnn {

typedef int int32x8 __attribute__((ext_vector_type(8)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef _Float16 halfx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bfloatx2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));

constexpr uint32_t kNanScale = 255;

// Largest magnitude of V values, as the bits of a float: magnitudes order like unsigned integers, what is not finite above the others.
template <int V>
__device__ __forceinline__ uint32_t largest(const Pack<float, V>& a)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, __float_as_uint(a.v[i]) & 0x7fffffffu);
    return m;
}
template <class T, int V>
__device__ __forceinline__ uint32_t largest(const Pack<T, V>& a)
{
    static_assert(sizeof(T) == 2 && V % 2 == 0, "two-byte elements in pairs");
    ushortx2 m = {0, 0};
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        uint32_t both = (uint32_t)__builtin_bit_cast(unsigned short, a.v[i]) | (uint32_t)__builtin_bit_cast(unsigned short, a.v[i + 1]) << 16;
        m = __builtin_elementwise_max(m, __builtin_bit_cast(ushortx2, both & 0x7fff7fffu));
    }
    const unsigned short top = m[0] > m[1] ? m[0] : m[1];
    return __float_as_uint(to_float(__builtin_bit_cast(T, top)));
}

// Scale byte for a block whose largest magnitude has these bits.  (A subnormal one is below 2^-126: byte 0.)
__device__ __forceinline__ uint32_t scale_byte(uint32_t largest_bits)
{
    const uint32_t e = largest_bits >> 23;
    return e == 255 ? kNanScale : e > 2 ? e - 2 : 0;
}

// The scale operand of the conversion instructions, which read its exponent field only.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight values to codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t encode8(const Pack<float, 8>& a, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a.v[0], a.v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a.v[2], a.v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a.v[4], a.v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, a.v[6], a.v[7], scale, 3);
}
__device__ __forceinline__ uint32_t encode8(const Pack<_Float16, 8>& a, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, halfx2{a.v[0], a.v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, halfx2{a.v[2], a.v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, halfx2{a.v[4], a.v[5]}, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(r, halfx2{a.v[6], a.v[7]}, scale, 3);
}
__device__ __forceinline__ uint32_t encode8(const Pack<__bf16, 8>& a, float scale)
{
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bfloatx2{a.v[0], a.v[1]}, scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bfloatx2{a.v[2], a.v[3]}, scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bfloatx2{a.v[4], a.v[5]}, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, bfloatx2{a.v[6], a.v[7]}, scale, 3);
}

// Eight values from p on, those from `left` on (of the row) zero.
template <class T>
__device__ __forceinline__ Pack<T, 8> load8(const T* p, int left)
{
    Pack<T, 8> a;
    if (left >= 8) {
        a = load_pack<T, 8>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) a.v[i] = i < left ? p[i] : T(0.0f);
    }
    return a;
}

// Product of 16 rows of 128 codes with 16 others, added to c: lane l holds block l / 16 of row l % 16 on either side
// and gets rows 4 * (l / 16) + i of the first, column l % 16 of the second.  The scales are the low bytes.
__device__ __forceinline__ floatx4 multiply(const uint4& a, const uint4& b, floatx4 c, uint32_t scale_a, uint32_t scale_b)
{
    const int32x8 va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, 0, (int)scale_a, 0, (int)scale_b);
}

}  // namespace patdnn
