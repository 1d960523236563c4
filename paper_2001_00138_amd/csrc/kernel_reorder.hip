// Order of channels: NCHW <-> channels last, with a change of element type on the way.
//
// Per image the channels and the pixels are the rows and columns of a matrix that is transposed.  Nothing is
// computed, so the copy's bytes bound it: each is to be read and written once, in whole cache lines on both
// sides.  A workgroup takes a tile through LDS: it reads runs along the one order and writes runs along the other.
// Lanes move four elements at a time, whatever they are aligned to, and single ones where a tile's rows end inside four.
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

constexpr int kTileSide = 64, kRun = 4;

template <class Ti, class To>
__global__ __launch_bounds__(kThreads) void transpose_kernel(Launch L, const Ti* __restrict__ in, To* __restrict__ out)
{
    constexpr int kPitch = kTileSide + (sizeof(To) == 4 ? 1 : 2);        // an odd number of banks from column to column
    constexpr int kLanes = kTileSide / kRun, kStep = kThreads / kLanes, kTimes = kTileSide / kStep;
    __shared__ To tile[kTileSide][kPitch];
    const uint32_t b = blockIdx.x;
    const uint32_t batch = fast_div(b, L.per_batch), in_batch = b - batch * (uint32_t)(L.row_tiles * L.col_tiles);
    const uint32_t rt = fast_div(in_batch, L.per_row), ct = in_batch - rt * (uint32_t)L.col_tiles;
    const int r0 = (int)rt * kTileSide, c0 = (int)ct * kTileSide;
    const int rows = min(kTileSide, L.s.rows - r0), cols = min(kTileSide, L.s.cols - c0);
    const int run = (int)(threadIdx.x % kLanes) * kRun, line = (int)(threadIdx.x / kLanes);
    {
        const Ti* src = in + (long long)batch * L.s.in_batch + (long long)(r0 + line) * L.s.in_row + c0 + run;
        Pack<Ti, kRun> v[kTimes];
        const int left = cols - run;
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
            const Ti* p = src + (long long)k * kStep * L.s.in_row;
            if (line + k * kStep >= rows) continue;
            if (left >= kRun) v[k] = load_pack<Ti, kRun>(p);
            else
#pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (i < left) v[k].v[i] = p[i];
        }
#pragma unroll
        for (int k = 0; k < kTimes; ++k)
            if (line + k * kStep < rows)
#pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (i < left) tile[run + i][line + k * kStep] = from_float<To>(to_float(v[k].v[i]));
    }
    __syncthreads();
    {
        To* dst = out + (long long)batch * L.s.out_batch + (long long)(c0 + line) * L.s.out_row + r0 + run;
        const int left = rows - run;
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
            if (line + k * kStep >= cols) continue;
            To* p = dst + (long long)k * kStep * L.s.out_row;
            Pack<To, kRun> v;
#pragma unroll
            for (int i = 0; i < kRun; ++i) v.v[i] = tile[line + k * kStep][run + i];
            if (left >= kRun) store_pack<To, kRun>(p, v);
            else
#pragma unroll
                for (int i = 0; i < kRun; ++i)
                    if (i < left) p[i] = v.v[i];
        }
    }
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
    with_type(s.in_type, [&](auto ti) {
        with_type(s.out_type, [&](auto to) {
            using Ti = decltype(ti);
            using To = decltype(to);
            const Ti* src = static_cast<const Ti*>(in);
            To* dst = static_cast<To*>(out);
            hipLaunchKernelGGL((transpose_kernel<Ti, To>), grid, dim3(kThreads), 0, stream, L, src, dst);
        });
    });
    return hipGetLastError();
}

}  // namespace patdnn
