// Order of channels: NCHW <-> channels last, with a change of element type on the way.
//
// Per image the channels and the pixels are the rows and columns of a matrix that is transposed.  Nothing is
// computed, so the copy's bytes bound it: each is to be read and written once, in whole cache lines on both
// sides.  A workgroup takes a tile through LDS: it reads runs along the one order and writes runs along the other.
// Runs of four elements a lane where both ends of the runs are aligned to them, single elements otherwise: a wavefront
// still reads 128 or 256 adjacent bytes then.
#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;

struct Launch {
    TransposeShape s;
    int row_tiles, col_tiles;
    FastDiv per_batch, per_row;          // col_tiles * row_tiles, col_tiles
};

// Tile of TR rows x TC columns of the input; VI / VO elements an access of the input / output.
template <class Ti, class To, int TR, int TC, int VI, int VO>
__global__ __launch_bounds__(kThreads) void transpose_kernel(Launch L, const Ti* __restrict__ in, To* __restrict__ out)
{
    constexpr int kPitch = TR + (sizeof(To) == 4 ? 1 : 2);       // an odd number of banks from column to column
    __shared__ To tile[TC][kPitch];
    const uint32_t b = blockIdx.x;
    const uint32_t batch = fast_div(b, L.per_batch), in_batch = b - batch * (uint32_t)(L.row_tiles * L.col_tiles);
    const uint32_t rt = fast_div(in_batch, L.per_row), ct = in_batch - rt * (uint32_t)L.col_tiles;
    const int r0 = (int)rt * TR, c0 = (int)ct * TC;
    const int rows = min(TR, L.s.rows - r0), cols = min(TC, L.s.cols - c0);
    {
        constexpr int kLanes = TC / VI, kStep = kThreads / kLanes, kTimes = TR / kStep;
        const int c = (int)(threadIdx.x % kLanes) * VI, r = (int)(threadIdx.x / kLanes);
        const Ti* src = in + (long long)batch * L.s.in_batch + (long long)(r0 + r) * L.s.in_row + c0 + c;
        Pack<Ti, VI> v[kTimes];
#pragma unroll
        for (int k = 0; k < kTimes; ++k)
            if (r + k * kStep < rows && c < cols) v[k] = load_pack<Ti, VI>(src + (long long)k * kStep * L.s.in_row);
#pragma unroll
        for (int k = 0; k < kTimes; ++k)
            if (r + k * kStep < rows && c < cols)
#pragma unroll
                for (int i = 0; i < VI; ++i) tile[c + i][r + k * kStep] = from_float<To>(to_float(v[k].v[i]));
    }
    __syncthreads();
    {
        constexpr int kLanes = TR / VO, kStep = kThreads / kLanes, kTimes = TC / kStep;
        const int r = (int)(threadIdx.x % kLanes) * VO, c = (int)(threadIdx.x / kLanes);
        To* dst = out + (long long)batch * L.s.out_batch + (long long)(c0 + c) * L.s.out_row + r0 + r;
#pragma unroll
        for (int k = 0; k < kTimes; ++k)
            if (c + k * kStep < cols && r < rows) {
                Pack<To, VO> v;
#pragma unroll
                for (int i = 0; i < VO; ++i) v.v[i] = tile[c + k * kStep][r + i];
                store_pack<To, VO>(dst + (long long)k * kStep * L.s.out_row, v);
            }
    }
}

constexpr int kTileSide = 64;

bool runs_of_four(const void* p, int type, int run, long long row, long long batch)
{
    return (run | row | batch) % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (4 * element_bytes(type)) == 0;
}

}  // namespace

bool transpose_fits(const TransposeShape& s)
{
    const long long tiles = (long long)((s.rows + kTileSide - 1) / kTileSide) * ((s.cols + kTileSide - 1) / kTileSide);
    return tiles <= kMostBlocks && tiles * s.batch <= kMostBlocks;
}

hipError_t launch_transpose(const TransposeShape& s, const void* in, void* out, hipStream_t stream)
{
    Launch L{s, (s.rows + kTileSide - 1) / kTileSide, (s.cols + kTileSide - 1) / kTileSide, {}, {}};
    L.per_batch = make_fast_div((uint32_t)(L.row_tiles * L.col_tiles));
    L.per_row = make_fast_div((uint32_t)L.col_tiles);
    const dim3 grid((unsigned)((long long)L.row_tiles * L.col_tiles * s.batch));
    const bool vi = runs_of_four(in, s.in_type, s.cols, s.in_row, s.in_batch), vo = runs_of_four(out, s.out_type, s.rows, s.out_row, s.out_batch);
    with_type(s.in_type, [&](auto ti) {
        with_type(s.out_type, [&](auto to) {
            using Ti = decltype(ti);
            using To = decltype(to);
            const Ti* src = static_cast<const Ti*>(in);
            To* dst = static_cast<To*>(out);
            if (vi && vo) hipLaunchKernelGGL((transpose_kernel<Ti, To, kTileSide, kTileSide, 4, 4>), grid, dim3(kThreads), 0, stream, L, src, dst);
            else if (vi) hipLaunchKernelGGL((transpose_kernel<Ti, To, kTileSide, kTileSide, 4, 1>), grid, dim3(kThreads), 0, stream, L, src, dst);
            else if (vo) hipLaunchKernelGGL((transpose_kernel<Ti, To, kTileSide, kTileSide, 1, 4>), grid, dim3(kThreads), 0, stream, L, src, dst);
            else hipLaunchKernelGGL((transpose_kernel<Ti, To, kTileSide, kTileSide, 1, 1>), grid, dim3(kThreads), 0, stream, L, src, dst);
        });
    });
    return hipGetLastError();
}

}  // namespace patdnn
