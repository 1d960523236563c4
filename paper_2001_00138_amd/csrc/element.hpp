// Element types of the operators around the convolutions (fp32, binary16, bfloat16): loads to fp32, stores
// rounded once to the nearest (ties to even), and the activations.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace patdnn {

enum { kF32 = 0, kF16 = 1, kBF16 = 2, kMxfp4 = 3, kFp8 = 4 };         // the PATDNN_F32... of patdnn.h
enum { kActNone = 0, kActRelu = 1, kActSilu = 2 };       // the PATDNN_ACT_...

inline size_t element_bytes(int type) { return type == kF32 ? 4 : 2; }

// V elements side by side, moved with one access, which needs no more alignment than the elements have: gfx950's vector memory
// instructions take any address.
template <class T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[V];
};

template <class T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T* p)
{
    return *reinterpret_cast<const Pack<T, V>*>(p);
}
template <class T, int V>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& a)
{
    *reinterpret_cast<Pack<T, V>*>(p) = a;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(_Float16 v) { return static_cast<float>(v); }
__device__ __forceinline__ float to_float(__bf16 v) { return static_cast<float>(v); }
template <class T>
__device__ __forceinline__ T from_float(float v)
{
    return static_cast<T>(v);
}

// z / (1 + exp(-z)): the exponential overflows to infinity for z < -88, where the quotient is the -0 that it should be.
// The hardware's exponential, of -z log2(e) rounded to fp32, and reciprocal: for z far below zero the result is off by |z| 2^-24 of itself, as much as the
// rounding of z before it makes (at most 1.2e-6 of 4e-8 at z = -20), and by a few 2^-24 elsewhere.  A second part of the argument would be three operations more
// an element, and z's own rounding would stay.
template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if (ACT == kActRelu) return z <= 0.0f ? 0.0f : z;                    // NaN stays NaN
    if (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.0f + __expf(-z));
    return z;
}

// Calls f with a value of the element type `type` and with the activation as a compile-time constant.
template <class F>
auto with_type(int type, F&& f)
{
    return type == kF32 ? f(float{}) : type == kF16 ? f(_Float16{}) : f(__bf16{});
}
template <int N>
struct Const {
    static constexpr int value = N;
};
template <class F>
auto with_act(int act, F&& f)
{
    return act == kActRelu ? f(Const<kActRelu>{}) : act == kActSilu ? f(Const<kActSilu>{}) : f(Const<kActNone>{});
}

}  // namespace patdnn
