// What the two files of the linear layer's kernels share.
#pragma once

#include "kernels.hpp"
#include "mxfp4.hpp"
#include "operators.hpp"

namespace patdnn {

__device__ __forceinline__ void store_as(void* out, long long at, int type, float v)
{
    if (type == kF32) static_cast<float*>(out)[at] = v;
    else if (type == kF16) static_cast<_Float16*>(out)[at] = static_cast<_Float16>(v);
    else static_cast<__bf16*>(out)[at] = static_cast<__bf16>(v);
}
__device__ __forceinline__ float activate_as(float z, int act)
{
    return act == kActRelu ? activate<kActRelu>(z) : act == kActSilu ? activate<kActSilu>(z) : z;
}

// Sixteen neighbouring results.
template <class T>
__device__ __forceinline__ void store_sixteen(void* out, long long at, const float (&z)[16])
{
    constexpr int kRun = 16 / (int)sizeof(T);
#pragma unroll
    for (int i = 0; i < 16; i += kRun) {
        Pack<T, kRun> p;
#pragma unroll
        for (int e = 0; e < kRun; ++e) p.v[e] = from_float<T>(z[i + e]);
        store_pack<T, kRun>(static_cast<T*>(out) + at + i, p);
    }
}

// The same into a tensor of any type, `left` of them inside the row.
__device__ __forceinline__ void store_results(void* out, long long at, int type, int left, const float (&z)[16])
{
    if (left >= 16) {
        if (type == kF32) store_sixteen<float>(out, at, z);
        else if (type == kF16) store_sixteen<_Float16>(out, at, z);
        else store_sixteen<__bf16>(out, at, z);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (i < left) store_as(out, at + i, type, z[i]);
    }
}
__device__ __forceinline__ void finish_sixteen(float (&z)[16], int act)
{
    if (act == kActRelu) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = activate<kActRelu>(z[i]);
    } else if (act == kActSilu) {
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = activate<kActSilu>(z[i]);
    }
}

// Many rows of few values (kernel_linear_short.hip): x, of any type, in registers.
bool short_fits(const LinearShape& s);
hipError_t launch_short(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                        hipStream_t stream);

// The tiled kernel (kernel_linear_tiles.hip), codes times codes.  Which shape it takes, and along how many slices of k.
struct TilePlan {
    int shape = -1;                                      // -1: not this kernel
    int slices = 1;
};
TilePlan tile_plan(const LinearShape& s);
size_t tile_workspace_bytes(const LinearShape& s, const TilePlan& p);
hipError_t launch_tiles(const LinearShape& s, const TilePlan& p, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales,
                        const float* bias, void* out, float* partial, hipStream_t stream);

}  // namespace patdnn
