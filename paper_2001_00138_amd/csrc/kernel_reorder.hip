// Order of channels: NCHW <-> channels last, with a change of element type on the way.
//
// Per image the channels and the pixels are the rows and columns of a matrix that is transposed.  Nothing is
// computed, so the copy's bytes bound it: each is to be read and written once, in whole cache lines on both
// sides.  A workgroup takes a tile through LDS: it reads runs along the one order and writes runs along the other.
// Lanes move four elements at a time, whatever they are aligned to, and single ones where a tile's rows end inside four.
//
// 64 x 64x224x224 fp16 144 us, 5.7 TB/s; 48 x 203x61x45 fp16 -> fp32 to NCHW 47 us, 3.4 TB/s (a fourth tile of eleven channels, cache lines
// written in two parts).
#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;

struct Launch {
    TransposeShape s;
    int row_tiles, col_tiles;
    uint32_t tiles;
    bool grouped;
    FastDiv per_batch, per_row;          // col_tiles * row_tiles, col_tiles
};

constexpr int kRun = 4;

// Tile of TR rows x TC columns of the input.
template <class Ti, class To, int TR, int TC>
__global__ __launch_bounds__(kThreads) void transpose_kernel(Launch L, const Ti* __restrict__ in, To* __restrict__ out)
{
    constexpr int kPitch = TR + (sizeof(To) == 4 ? 1 : 2);               // an odd number of banks from column to column
    __shared__ To tile[TC][kPitch];
    // Workgroups go to the eight XCDs in turn; grouped, each XCD takes a run of tiles.
    const uint32_t xcd = blockIdx.x & 7, q = L.tiles >> 3;
    const uint32_t b = L.grouped ? xcd * q + min(xcd, L.tiles & 7) + (blockIdx.x >> 3) : blockIdx.x;
    const uint32_t batch = fast_div(b, L.per_batch), in_batch = b - batch * (uint32_t)(L.row_tiles * L.col_tiles);
    const uint32_t rt = fast_div(in_batch, L.per_row), ct = in_batch - rt * (uint32_t)L.col_tiles;
    const int r0 = (int)rt * TR, c0 = (int)ct * TC;
    const int rows = min(TR, L.s.rows - r0), cols = min(TC, L.s.cols - c0);
    {
        constexpr int kLanes = TC / kRun, kStep = kThreads / kLanes, kTimes = TR / kStep;
        const int run = (int)(threadIdx.x % kLanes) * kRun, line = (int)(threadIdx.x / kLanes);
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
        constexpr int kLanes = TR / kRun, kStep = kThreads / kLanes, kTimes = TC / kStep;
        const int run = (int)(threadIdx.x % kLanes) * kRun, line = (int)(threadIdx.x / kLanes);
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

// Square tiles, unless one side is short (64 x 3x224x224 fp32 -> fp16: 45 us with square ones, 25 with 32 x 128).
struct TileSize {
    int rows, cols;
};
TileSize tile_of(const TransposeShape& s)
{
    return s.rows <= 32 ? TileSize{32, 128} : s.cols <= 32 ? TileSize{128, 32} : TileSize{64, 64};
}

}  // namespace

bool transpose_fits(const TransposeShape& s)
{
    const TileSize t = tile_of(s);
    const long long tiles = (((long long)s.rows + t.rows - 1) / t.rows) * (((long long)s.cols + t.cols - 1) / t.cols);
    return tiles <= kMostBlocks && tiles * s.batch <= kMostBlocks;
}

hipError_t launch_transpose(const TransposeShape& s, const void* in, void* out, hipStream_t stream)
{
    const TileSize t = tile_of(s);
    Launch L{s, (s.rows - 1) / t.rows + 1, (s.cols - 1) / t.cols + 1, 0, false, {}, {}};
    // Rows that end inside a cache line: neighbouring tiles share lines, which should meet in one L2 (48 x 203x61x45 fp16 -> fp32: 58 us
    // without, 49 so; aligned rows spread better over all channels of memory, 64 x 64x224x224 fp16: 143 us without, 159 so).
    L.grouped = (s.in_row * (long long)element_bytes(s.in_type)) % 128 != 0 || (s.out_row * (long long)element_bytes(s.out_type)) % 128 != 0;
    L.tiles = (uint32_t)L.row_tiles * (uint32_t)L.col_tiles * (uint32_t)s.batch;
    L.per_batch = make_fast_div((uint32_t)(L.row_tiles * L.col_tiles));
    L.per_row = make_fast_div((uint32_t)L.col_tiles);
    with_type(s.in_type, [&](auto ti) {
        with_type(s.out_type, [&](auto to) {
            using Ti = decltype(ti);
            using To = decltype(to);
            const Ti* src = static_cast<const Ti*>(in);
            To* dst = static_cast<To*>(out);
            if (t.rows == 32) hipLaunchKernelGGL((transpose_kernel<Ti, To, 32, 128>), dim3(L.tiles), dim3(kThreads), 0, stream, L, src, dst);
            else if (t.cols == 32) hipLaunchKernelGGL((transpose_kernel<Ti, To, 128, 32>), dim3(L.tiles), dim3(kThreads), 0, stream, L, src, dst);
            else hipLaunchKernelGGL((transpose_kernel<Ti, To, 64, 64>), dim3(L.tiles), dim3(kThreads), 0, stream, L, src, dst);
        });
    });
    return hipGetLastError();
}

}  // namespace patdnn
