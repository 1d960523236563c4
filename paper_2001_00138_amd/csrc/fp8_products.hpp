// What the kernels of products of fp8 codes share.
#pragma once

#include "fp8.hpp"
#include "linear.hpp"

namespace patdnn {

// Gradients of the two projections g and u from that of h = act(g) u.  SiLU's slope, with s = 1 / (1 + exp(-z)), is s (1 + z (1 - s)) = s + z s (1 - s).
template <int ACT>
__device__ __forceinline__ void gated_gradients(float g, float u, float dh, float& dg, float& du)
{
    float value = g, slope = 1.0f;
    if (ACT == kActRelu) {
        value = activate<kActRelu>(g);
        slope = g <= 0.0f ? 0.0f : 1.0f;
    } else if (ACT == kActSilu) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-g));
        value = g * s;
        slope = s + value * (1.0f - s);
    }
    dg = dh * u * slope;
    du = dh * value;
}
__device__ __forceinline__ void gated_gradients_as(int act, float g, float u, float dh, float& dg, float& du)
{
    if (act == kActSilu) gated_gradients<kActSilu>(g, u, dh, dg, du);
    else if (act == kActRelu) gated_gradients<kActRelu>(g, u, dh, dg, du);
    else gated_gradients<kActNone>(g, u, dh, dg, du);
}
__device__ __forceinline__ float load_as(const void* from, long long at, int type)
{
    return type == kF32 ? static_cast<const float*>(from)[at]
           : type == kF16 ? static_cast<float>(static_cast<const _Float16*>(from)[at])
                          : static_cast<float>(static_cast<const __bf16*>(from)[at]);
}

// One result: row m, column n.  a, b: its sums (b: of the second projection).
template <int KIND>
__device__ __forceinline__ void finish_one(const ProductShape& s, const ProductTensors& t, int m, int n, float a, float b)
{
    const long long at = m * s.out_row + n;
    if (KIND == kLinear) {
        store_as(t.out, at, s.out_type, activate_as(t.bias ? a + t.bias[n] : a, s.act));
    } else if (KIND == kGated) {
        store_as(t.out, at, s.out_type, activate_as(a, s.act) * b);
    } else {
        float dg, du;
        gated_gradients_as(s.act, a, b, load_as(t.dh, m * s.dh_row + n, s.dh_type), dg, du);
        store_as(t.out, at, s.out_type, dg);
        store_as(t.out2, at, s.out_type, du);
    }
}

// Many rows (kernel_fp8_tiles.hip).
bool product_tiles_fit(const ProductShape& s);
size_t product_tiles_workspace_bytes(const ProductShape& s);
hipError_t launch_product_tiles(const ProductShape& s, const ProductTensors& t, float* partial, hipStream_t stream);

}  // namespace patdnn
