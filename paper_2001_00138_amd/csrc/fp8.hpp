// Eight-bit floating point (e4m3: 448 the largest, no infinity) in blocks of 128 values that share a power of two.
//
// Scale byte b stands for 2^(b-127), 255 for a block that held something not finite (its values are NaN).  b - 127 is the
// smallest exponent, at least -127, with which the block's largest magnitude is at most 448 units; values are divided by it, which is
// exact, and rounded to the nearest code, ties to even.  Powers of two cost no precision in a floating format, and the matrix
// instruction applies them itself.
#pragma once

#include "mxfp4.hpp"

namespace patdnn {

// Scale byte for a block whose largest magnitude has these bits: 448 is 1.75 * 2^8.
__device__ __forceinline__ uint32_t fp8_scale_byte(uint32_t largest_bits)
{
    const int e = (int)(largest_bits >> 23), b = e - 8 + ((largest_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e == 255 ? kNanScale : (uint32_t)max(b, 0);
}
// 2^(127-b): units in a value.  A block that is not finite (b = 255) gets 0 here and its codes are cleared.
__device__ __forceinline__ float fp8_inverse(uint32_t byte) { return __uint_as_float(byte == kNanScale ? 0u : (254 - byte) << 23); }
// 2^(b-127); byte 0 is the subnormal 2^-127.
__device__ __forceinline__ float fp8_unit(uint32_t byte)
{
    return byte == kNanScale ? __builtin_nanf("") : __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// Four values to codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t fp8_encode4(float a, float b, float c, float d, float inverse)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, low, true);
}
__device__ __forceinline__ uint2 fp8_encode8(const float (&v)[8], uint32_t byte)
{
    const float inverse = fp8_inverse(byte);
    const uint2 r = make_uint2(fp8_encode4(v[0], v[1], v[2], v[3], inverse), fp8_encode4(v[4], v[5], v[6], v[7], inverse));
    return byte == kNanScale ? make_uint2(0u, 0u) : r;
}
__device__ __forceinline__ void fp8_decode4(uint32_t codes, float unit, float (&v)[4])
{
    const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    v[0] = a[0] * unit, v[1] = a[1] * unit, v[2] = b[0] * unit, v[3] = b[1] * unit;
}

// Largest of eight magnitudes, as the bits of a float.
__device__ __forceinline__ uint32_t largest8(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    return m;
}
template <int CONTROL>
__device__ __forceinline__ uint32_t moved(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CONTROL, 0xf, 0xf, false);
}
// Largest over sixteen neighbouring lanes, in all of them: neighbours, pairs, then halves and wholes mirrored.
__device__ __forceinline__ uint32_t largest_of_16_lanes(uint32_t v)
{
    v = max(v, moved<0xb1>(v));
    v = max(v, moved<0x4e>(v));
    v = max(v, moved<0x141>(v));
    return max(v, moved<0x140>(v));
}

// Product of 16 rows of 128 codes with 16 others, added to c, with fp32's precision: lane l holds 32 codes of row l % 16 on either side (which 32 does not matter, so long as both
// sides deal them to the four lanes of a row alike: the scale is the same for all), and gets rows 4 * (l / 16) + i of the first, column l % 16 of the second.  Codes become
// bfloat16, multiplied by their scales on the way, and go through four bfloat16 instructions, whose products and sums are fp32's: half the rate of the fp8 instruction.
// Exact but for values below 2^-126, which have bfloat16's subnormals left, and of 2^128 and more, which are infinite; a scale of NaN makes
// NaN of any code.  unit: the scale's byte where a float's exponent is.
typedef __bf16 bfloatx8 __attribute__((ext_vector_type(8)));
struct Wide {
    bfloatx8 v[4];
};
__device__ __forceinline__ Wide fp8_widen(const int32x8& a, uint32_t unit)
{
    const float s = __uint_as_float(unit);
    Wide w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bfloatx2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)a[2 * i], s, false), q = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)a[2 * i], s, true);
        const bfloatx2 r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)a[2 * i + 1], s, false), t = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)a[2 * i + 1], s, true);
        w.v[i] = bfloatx8{p[0], p[1], q[0], q[1], r[0], r[1], t[0], t[1]};
    }
    return w;
}
__device__ __forceinline__ floatx4 multiply_wide(const Wide& a, const Wide& b, floatx4 c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ int32x8 both_halves(const uint4& a, const uint4& b)
{
    return int32x8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// Eight neighbouring results of a row, `left` of them inside it.
template <class T>
__device__ __forceinline__ void store8(T* to, int left, const float (&v)[8])
{
    Pack<T, 8> p;
#pragma unroll
    for (int i = 0; i < 8; ++i) p.v[i] = from_float<T>(v[i]);
    if (left >= 8) {
        store_pack<T, 8>(to, p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) to[i] = p.v[i];
    }
}
template <class T>
__device__ __forceinline__ void load8_floats(const T* p, int left, float (&v)[8])
{
    const Pack<T, 8> a = load8(p, left);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_float(a.v[i]);
}

}  // namespace patdnn
