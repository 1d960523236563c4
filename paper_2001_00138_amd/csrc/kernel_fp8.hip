// fp8 codes with a power of two for each block of 128: quantisation in four layouts, and back.
//
// Bytes bound all of it: each value is read once and its code written once.
//
// Blocks along the rows of x: sixteen neighbouring lanes share a block, eight values each.
// Everything else goes by tiles of 128 x 128 values of x, a workgroup each: a thread holds eight values of each of eight neighbouring
// rows, so that a column's codes are eight neighbouring bytes of it when the matrix is turned; turned bytes go through LDS, and rows of 128
// bytes leave it.
//
// From memory: 16384 x 4096 bf16, blocks along the rows: 39.5 us, 5.1 TB/s (fp32 61 us, 5.5).  12288 x 4096 bf16, squares: 33 us, 4.6 TB/s; turned: 36 us, 4.2 TB/s; back to bf16
// 37 us, 4.1 TB/s (29.5 of codes that have just been written).  8111 x 4500 bf16, turned: 30.5 us, 3.6 TB/s (its rows begin inside cache lines).
#include "fp8.hpp"
#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;

// How lanes are laid over rows of `lanes` runs of eight values: a workgroup takes `across` runs of each of `down` rows.
struct Spread {
    int lanes, across, down, blocks_across;
    FastDiv by_across, by_blocks;
};
Spread spread_of(const Fp8Shape& s)
{
    Spread p{};
    p.lanes = (int)fp8_pieces(s.cols) * 16;
    p.across = std::min(p.lanes, kThreads);
    p.down = kThreads / p.across;
    p.blocks_across = (p.lanes + p.across - 1) / p.across;
    p.by_across = make_fast_div((uint32_t)p.across);
    p.by_blocks = make_fast_div((uint32_t)p.blocks_across);
    return p;
}
long long run_blocks(const Fp8Shape& s)
{
    const Spread p = spread_of(s);
    return p.blocks_across * ceil_div(s.rows, p.down);
}
bool by_tiles(const Fp8Shape& s) { return s.squares || s.transposed; }
long long tile_count(const Fp8Shape& s) { return ceil_div(s.rows, 128) * ceil_div(s.cols, 128); }

// This thread's row and run; false if it has none.
__device__ __forceinline__ bool place_of(const Fp8Shape& s, const Spread& p, int& row, int& run)
{
    const int down = (int)fast_div(threadIdx.x, p.by_across), across = (int)threadIdx.x - down * p.across;
    const uint32_t above = fast_div(blockIdx.x, p.by_blocks);
    row = (int)above * p.down + down;
    run = (int)(blockIdx.x - above * (uint32_t)p.blocks_across) * p.across + across;
    return down < p.down && row < s.rows && run < p.lanes;
}

template <class T>
__global__ __launch_bounds__(kThreads) void fp8_rows_kernel(Fp8Shape s, Spread p, const T* __restrict__ x, uint2* __restrict__ codes,
                                                            uint8_t* __restrict__ scales)
{
    int row, run;
    // (a block's sixteen lanes have a row and a run together or not at all: rows are multiples of sixteen runs)
    if (!place_of(s, p, row, run)) return;
    float v[8];
    load8_floats(x + (long long)row * s.row + run * 8, s.cols - run * 8, v);
    const uint32_t byte = fp8_scale_byte(largest_of_16_lanes(largest8(v)));
    const long long at = (long long)row * p.lanes + run;
    codes[at] = fp8_encode8(v, byte);
    if (run % 16 == 0) scales[at / 16] = (uint8_t)byte;
}

// A tile: rows r0 ... and columns c0 ... of x.
template <class T, bool SQUARES, bool TRANSPOSED>
__global__ __launch_bounds__(kThreads) void fp8_tiles_kernel(int rows, int cols, long long pitch, FastDiv by_across, const T* __restrict__ x,
                                                             uint8_t* __restrict__ codes, uint8_t* __restrict__ scales)
{
    __shared__ uint4 turned[TRANSPOSED ? 128 * 8 : 1];                   // [column][16 rows], the eights of rows dealt by column
    __shared__ uint32_t tops[4][SQUARES ? 1 : 128];
    const int across = (cols + 127) / 128, down = (rows + 127) / 128;
    const int tr = (int)fast_div(blockIdx.x, by_across), tc = (int)blockIdx.x - tr * across;
    const int run = (int)threadIdx.x & 15, line = (int)threadIdx.x >> 4, wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63;
    const int row = tr * 128 + line * 8, col = tc * 128 + run * 8;
    Pack<T, 8> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = load8(x + (long long)min(row + i, rows - 1) * pitch + col, row + i < rows ? cols - col : 0);
    uint32_t byte[SQUARES ? 1 : 8];
    if (SQUARES) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, largest(v[i]));
        top = largest_of_16_lanes(top);
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        if (lane == 0) tops[wave][0] = top;
        __syncthreads();
        byte[0] = fp8_scale_byte(max(max(tops[0][0], tops[1][0]), max(tops[2][0], tops[3][0])));
    } else {
        uint32_t top[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) top[j] = max(top[j], __float_as_uint(to_float(v[i].v[j])) & 0x7fffffffu);
            top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 16, 64));
            top[j] = max(top[j], (uint32_t)__shfl_xor((int)top[j], 32, 64));
        }
        if (lane < 16)
#pragma unroll
            for (int j = 0; j < 8; ++j) tops[wave][run * 8 + j] = top[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = run * 8 + j;
            byte[SQUARES ? 0 : j] = fp8_scale_byte(max(max(tops[0][c], tops[1][c]), max(tops[2][c], tops[3][c])));
        }
    }
    if constexpr (!TRANSPOSED) {
        const long long out_pitch = (long long)across * 128;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = to_float(v[i].v[j]);
            if (row + i < rows) *reinterpret_cast<uint2*>(codes + (row + i) * out_pitch + col) = fp8_encode8(f, byte[0]);
        }
        if (threadIdx.x == 0) scales[(long long)tr * across + tc] = (uint8_t)byte[0];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = to_float(v[i].v[j]);
            const int c = run * 8 + j;
            reinterpret_cast<uint2*>(&turned[c * 8 + (line >> 1 ^ (run & 7))])[line & 1] = fp8_encode8(f, byte[SQUARES ? 0 : j]);
        }
        __syncthreads();
        const long long out_pitch = (long long)down * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = i * kThreads + (int)threadIdx.x, c = at >> 3, chunk = at & 7;
            if (tc * 128 + c < cols)
                *reinterpret_cast<uint4*>(codes + (tc * 128 + c) * out_pitch + tr * 128 + chunk * 16) = turned[c * 8 + (chunk ^ (c >> 3 & 7))];
        }
        if (SQUARES) {
            if (threadIdx.x == 0) scales[(long long)tc * down + tr] = (uint8_t)byte[0];
        } else if (line == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (col + j < cols) scales[(long long)(col + j) * down + tr] = (uint8_t)byte[SQUARES ? 0 : j];
        }
    }
}

template <class T>
__global__ __launch_bounds__(kThreads) void fp8_values_kernel(Fp8Shape s, Spread p, const uint2* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                              T* __restrict__ out)
{
    int row, run;
    if (!place_of(s, p, row, run)) return;
    const int left = s.cols - run * 8;
    if (left <= 0) return;
    const uint2 c = codes[(long long)row * p.lanes + run];
    const float unit = fp8_unit(scales[(long long)(s.squares ? row >> 7 : row) * (p.lanes / 16) + run / 16]);
    float a[4], b[4], v[8];
    fp8_decode4(c.x, unit, a);
    fp8_decode4(c.y, unit, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[i + 4] = b[i];
    store8(out + (long long)row * s.row + run * 8, left, v);
}

}  // namespace

bool fp8_fits(const Fp8Shape& s, bool quantize)
{
    return fp8_pieces(s.cols) * 128 <= INT32_MAX - 128 && fp8_pieces(s.rows) * 128 <= INT32_MAX - 128 &&
           (quantize && by_tiles(s) ? tile_count(s) : run_blocks(s)) <= kMostBlocks;
}

hipError_t launch_fp8_quantize(const Fp8Shape& s, const void* x, uint8_t* codes, uint8_t* scales, hipStream_t stream)
{
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        const T* from = static_cast<const T*>(x);
        if (!by_tiles(s)) {
            hipLaunchKernelGGL((fp8_rows_kernel<T>), dim3((unsigned)run_blocks(s)), dim3(kThreads), 0, stream, s, spread_of(s), from,
                               reinterpret_cast<uint2*>(codes), scales);
            return;
        }
        const int rows = s.transposed ? s.cols : s.rows, cols = s.transposed ? s.rows : s.cols;       // of x
        const FastDiv across = make_fast_div((uint32_t)((cols + 127) / 128));
        const dim3 grid((unsigned)tile_count(s));
        if (!s.transposed) hipLaunchKernelGGL((fp8_tiles_kernel<T, true, false>), grid, dim3(kThreads), 0, stream, rows, cols, s.row, across, from, codes, scales);
        else if (s.squares) hipLaunchKernelGGL((fp8_tiles_kernel<T, true, true>), grid, dim3(kThreads), 0, stream, rows, cols, s.row, across, from, codes, scales);
        else hipLaunchKernelGGL((fp8_tiles_kernel<T, false, true>), grid, dim3(kThreads), 0, stream, rows, cols, s.row, across, from, codes, scales);
    });
    return hipGetLastError();
}

hipError_t launch_fp8_dequantize(const Fp8Shape& s, const uint8_t* codes, const uint8_t* scales, void* out, hipStream_t stream)
{
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL((fp8_values_kernel<T>), dim3((unsigned)run_blocks(s)), dim3(kThreads), 0, stream, s, spread_of(s),
                           reinterpret_cast<const uint2*>(codes), scales, static_cast<T*>(out));
    });
    return hipGetLastError();
}

}  // namespace patdnn
