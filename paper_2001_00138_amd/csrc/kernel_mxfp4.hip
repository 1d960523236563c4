// MXFP4: quantisation of rows of values, and back.
//
// A lane takes eight adjacent values, so four lanes share a block: it is read, its largest magnitude joined over the four
// lanes, and it is written as four bytes a lane and one byte of scale.  Bytes bound it: each value is read once.
// 200704 x 256 fp16, eight tensors in turn (from and to memory): quantised in 26 us and read back in 40, 5.0 and 3.3 TB/s; one tensor again and again, of
// which the last-level cache keeps a part, 22 and 27; in a program that alternates them 53 us.
#include "kernels.hpp"
#include "mxfp4.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;

// How lanes are laid over rows of `lanes` runs of eight values: a workgroup takes `across` runs of each of `down` rows.
struct Spread {
    int lanes, across, down, blocks_across;
    FastDiv by_across, by_blocks;
};
Spread spread_of(const Mxfp4Shape& s)
{
    Spread p{};
    p.lanes = (int)mxfp4_pieces(s.cols) * 16;
    p.across = std::min(p.lanes, kThreads);
    p.down = kThreads / p.across;
    p.blocks_across = (p.lanes + p.across - 1) / p.across;
    p.by_across = make_fast_div((uint32_t)p.across);
    p.by_blocks = make_fast_div((uint32_t)p.blocks_across);
    return p;
}
long long blocks_of(const Mxfp4Shape& s)
{
    const Spread p = spread_of(s);
    return p.blocks_across * ceil_div(s.rows, p.down);
}

// This thread's row and run; false if it has none.
__device__ __forceinline__ bool place_of(const Mxfp4Shape& s, const Spread& p, int& row, int& run)
{
    const int down = (int)fast_div(threadIdx.x, p.by_across), across = (int)threadIdx.x - down * p.across;
    const uint32_t above = fast_div(blockIdx.x, p.by_blocks);
    row = (int)above * p.down + down;
    run = (int)(blockIdx.x - above * (uint32_t)p.blocks_across) * p.across + across;
    return down < p.down && row < s.rows && run < p.lanes;
}

template <class T>
__global__ __launch_bounds__(kThreads) void quantize_kernel(Mxfp4Shape s, Spread p, const T* __restrict__ x,
                                                            uint32_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    int row, run;
    const bool mine = place_of(s, p, row, run);
    Pack<T, 8> a;
    uint32_t top = 0;
    if (mine) {
        a = load8(x + (long long)row * s.row + run * 8, s.cols - run * 8);
        top = largest(a);
    }
    // four lanes of a block are neighbours in a wavefront: runs of a row and workgroup start at multiples of 16
    top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
    if (!mine) return;
    const uint32_t byte = scale_byte(top);
    codes[(long long)row * p.lanes + run] = byte == kNanScale ? 0u : encode8(a, scale_of(byte));
    if (run % 4 == 0) scales[((long long)row * p.lanes + run) / 4] = (uint8_t)byte;
}

template <class T>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Mxfp4Shape s, Spread p, const uint32_t* __restrict__ codes,
                                                              const uint8_t* __restrict__ scales, T* __restrict__ out)
{
    int row, run;
    if (!place_of(s, p, row, run)) return;
    const int left = s.cols - run * 8;
    if (left <= 0) return;
    const uint32_t c = codes[(long long)row * p.lanes + run], byte = scales[((long long)row * p.lanes + run) / 4];
    const float scale = scale_of(byte);
    const floatx2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1),
                          __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3)};
    T* to = out + (long long)row * s.row + run * 8;
    Pack<T, 8> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = from_float<T>(byte == kNanScale ? __builtin_nanf("") : v[i / 2][i % 2]);
    if (left >= 8) {
        store_pack<T, 8>(to, r);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) to[i] = r.v[i];
    }
}

}  // namespace

bool mxfp4_fits(const Mxfp4Shape& s) { return mxfp4_pieces(s.cols) * 128 <= INT32_MAX - 128 && blocks_of(s) <= kMostBlocks; }

hipError_t launch_mxfp4_quantize(const Mxfp4Shape& s, const void* x, uint8_t* codes, uint8_t* scales, hipStream_t stream)
{
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((quantize_kernel<T>), dim3((unsigned)blocks_of(s)), dim3(kThreads), 0, stream, s, spread_of(s), static_cast<const T*>(x), reinterpret_cast<uint32_t*>(codes), scales);
    });
    return hipGetLastError();
}

hipError_t launch_mxfp4_dequantize(const Mxfp4Shape& s, const uint8_t* codes, const uint8_t* scales, void* out, hipStream_t stream)
{
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((dequantize_kernel<T>), dim3((unsigned)blocks_of(s)), dim3(kThreads), 0, stream, s, spread_of(s), reinterpret_cast<const uint32_t*>(codes), scales, static_cast<T*>(out));
    });
    return hipGetLastError();
}

}  // namespace patdnn
