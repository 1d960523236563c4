// Root-mean-square norm of rows, with the residual's addition before it and an output of values or of fp8 codes; and its gradients.
//
// Forward, a row: s = x + residual, r = 1 / sqrt(mean(s^2) + eps), y = gamma s r.  Backward, with d = gamma dy:
//   ds = dsum + r (d - s r^2 mean(d s)),  dgamma = sum over rows of dy s r.
// Bytes bound both: a row is read once and kept in registers between its sum and its results (up to kHeld runs of eight values a
// lane); longer rows are read again.  y comes from the sum as it is in fp32, not from its rounded copy that is stored.
//
// Short rows share a wavefront or have one each; longer ones take up to sixteen wavefronts, which join their sums through LDS in their order, so
// results repeat bit for bit.  Backward, a workgroup takes several rows, a stride apart, and keeps its sums of dgamma in registers; they are
// joined, again in a fixed order, by a second launch.
//
// 16384 x 4096 bf16 (from memory): codes with the residual 105 us, 4.5 TB/s; backward 112 us with its joining, 4.8 TB/s, 103 without gamma's gradient.
#include "fp8.hpp"
#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

struct Codes {};                                         // y as fp8

// A row's lanes (16, 32, 64 or whole wavefronts), how many runs of eight values each has (0: as many as it takes, rows are read twice), and
// how many rows share a workgroup.
struct Plan {
    int lanes, runs, rows;
};
// Most runs that a lane holds: four are 32 registers; backward two, beside as many of dy, gamma and the sums of dgamma (with four the compiler spills).
constexpr int kHeld = 4, kHeldBackward = 2;
Plan plan_of(const RmsShape& s, bool backward)
{
    const int runs = s.cols > INT32_MAX - 128 ? INT32_MAX / 8 : (int)(s.y_type == kFp8 && !backward ? fp8_pieces(s.cols) * 16 : ((long long)s.cols + 7) / 8);
    Plan p{};
    if (runs <= 64) {
        p.lanes = runs <= 16 ? 16 : runs <= 32 ? 32 : 64;
        p.runs = 1;
        p.rows = 256 / p.lanes;
        return p;
    }
    p.rows = 1;
    // One run a lane is fastest, but for workgroups whose wavefronts the four SIMDs do not share evenly (16384 x 5120 bf16 forward: 137 us with ten, 124 with two runs on
    // five; 8192 columns 94 with one, 98 with two; 12288: 77 with two, 84 with four), and backward for so many that a CU has one workgroup (8192 x 8192: 133 and 120).
    if (backward) p.runs = runs <= 768 ? 1 : runs <= 1024 * kHeldBackward ? kHeldBackward : 0;
    else p.runs = runs <= 512 || (runs <= 1024 && (runs + 63) / 64 % 4 == 0) ? 1 : runs <= 2048 ? 2 : runs <= 1024 * kHeld ? kHeld : 0;
    p.lanes = p.runs ? ((runs + p.runs - 1) / p.runs + 63) / 64 * 64 : 1024;
    return p;
}

// Sum over a row's lanes, in all of them.  `slot`: a word of LDS for each wavefront, not in use since the barrier before.
__device__ __forceinline__ float row_sum(float v, int lanes, float* slot)
{
    const int most = min(lanes, 64);
    for (int d = 1; d < most; d <<= 1) v += __shfl_xor(v, d, 64);
    if (lanes <= 64) return v;
    const int wave = (int)threadIdx.x >> 6, waves = lanes >> 6;
    if (((int)threadIdx.x & 63) == 0) slot[wave] = v;
    __syncthreads();
    float sum = 0.0f;
    for (int i = 0; i < waves; ++i) sum += slot[i];
    return sum;
}

template <class Y>
__device__ __forceinline__ void put(const RmsShape& s, int pieces, int row, int run, const float (&y)[8], void* out, uint8_t* scales)
{
    if constexpr (std::is_same_v<Y, Codes>) {
        const uint32_t byte = fp8_scale_byte(largest_of_16_lanes(largest8(y)));
        if (run >= pieces * 16) return;
        const long long at = (long long)row * pieces * 16 + run;
        static_cast<uint2*>(out)[at] = fp8_encode8(y, byte);
        if (run % 16 == 0) scales[at / 16] = (uint8_t)byte;
    } else {
        if (run * 8 < s.cols) store8(static_cast<Y*>(out) + (long long)row * s.y_row + run * 8, s.cols - run * 8, y);
    }
}

// gamma of a run; behind the row's end zero, so that codes there are.
__device__ __forceinline__ void load_gamma(const float* gamma, int run, int cols, float (&g)[8])
{
    if (gamma) {
        load8_floats(gamma + run * 8, cols - run * 8, g);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    }
}

template <class T, class Y, int RUNS>
__global__ __launch_bounds__(1024) void rms_kernel(RmsShape s, int lanes, int rows, const T* __restrict__ x, const T* residual,
                                                   const float* __restrict__ gamma, T* sum, void* __restrict__ y, uint8_t* __restrict__ scales,
                                                   float* __restrict__ rstd)
{
    __shared__ float slots[2][16];
    const int group = rows > 1 ? (int)threadIdx.x / lanes : 0, l = (int)threadIdx.x - group * lanes;
    const long long r = (long long)blockIdx.x * rows + group;
    if (r >= s.rows) return;                                             // (only where rows share a workgroup, which has no barrier)
    const int row = (int)r, pieces = (s.cols + 127) / 128;
    const T* x_at = x + r * s.x_row;
    const T* residual_at = residual ? residual + r * s.residual_row : nullptr;
    auto load = [&](int run, float(&v)[8]) {
        const int left = s.cols - run * 8;
        load8_floats(x_at + run * 8, left, v);
        if (residual_at) {
            float add[8];
            load8_floats(residual_at + run * 8, left, add);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += add[j];
        }
    };
    auto keep = [&](int run, const float(&v)[8]) {
        if (sum && run * 8 < s.cols) store8(sum + r * s.sum_row + run * 8, s.cols - run * 8, v);
    };
    auto finish = [&](int run, float(&v)[8], float scale) {
        float g[8];
        load_gamma(gamma, run, s.cols, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = v[j] * scale * g[j];
        put<Y>(s, pieces, row, run, v, y, scales);
    };
    // 1 / sqrt(mean + eps) from this lane's sum of squares; again(factor): that of the values times a power of two.  A sum may pass fp32's range where the mean does not: it is made again in
    // units of 2^16 (columns are fewer than 2^32), from which a mean beyond the range is infinite and its root 0.  Squares below the range are lost: they count where neither the mean nor eps is
    // 2^-100, and are made again in units of 2^-80 (no value is 2^-34 then, whose square times 2^31 columns stays in range).  (All lanes of a row have the same sum.)
    auto root = [&](float total, auto again) {
        float mean = row_sum(total, lanes, slots[0]) / (float)s.cols;
        const bool over = mean == __builtin_inff(), under = mean < 0x1p-100f && s.eps < 0x1p-100f;
        float scale;
        if (over || under) {
            mean = row_sum(again(over ? 0x1p-16f : 0x1p80f), lanes, slots[1]) / (float)s.cols;
            scale = over ? 1.0f / sqrtf(mean * 0x1p32f + s.eps) : 0x1p80f / sqrtf(mean + s.eps * 0x1p80f * 0x1p80f);
        } else {
            scale = 1.0f / sqrtf(mean + s.eps);
        }
        if (rstd && l == 0) rstd[r] = scale;
        return scale;
    };
    if constexpr (RUNS > 0) {
        float v[RUNS][8], total = 0.0f;
#pragma unroll
        for (int i = 0; i < RUNS; ++i) load(l + i * lanes, v[i]);
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            keep(l + i * lanes, v[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) total += v[i][j] * v[i][j];
        }
        const float scale = root(total, [&](float factor) {
            float sum2 = 0.0f;
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum2 += (v[i][j] * factor) * (v[i][j] * factor);
            return sum2;
        });
#pragma unroll
        for (int i = 0; i < RUNS; ++i) finish(l + i * lanes, v[i], scale);
    } else {
        // sum may be residual itself, so it is written after the second reading
        const int runs = pieces * 16;
        float v[8];
        auto squares = [&](float factor) {
            float sum2 = 0.0f;
            for (int run = l; run < runs; run += lanes) {
                load(run, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) sum2 += (v[j] * factor) * (v[j] * factor);
            }
            return sum2;
        };
        const float scale = root(squares(1.0f), squares);
        for (int run = l; run < runs; run += lanes) {
            load(run, v);
            keep(run, v);
            finish(run, v, scale);
        }
    }
}

// RUNS > 0: dx, and the workgroup's sums of dgamma in partial[workgroup][cols].  RUNS == 0: dx only.
template <class T, class Y, int RUNS>
__global__ __launch_bounds__(1024) void rms_backward_kernel(RmsShape s, int lanes, int rows, int row_step, const Y* __restrict__ dy, const T* dsum,
                                                            const T* __restrict__ x, const float* __restrict__ rstd, const float* __restrict__ gamma,
                                                            T* dx, float* __restrict__ partial)
{
    __shared__ float slots[2][16];
    const int group = rows > 1 ? (int)threadIdx.x / lanes : 0, l = (int)threadIdx.x - group * lanes;
    const float per = 1.0f / (float)s.cols;
    int turn = 0;
    if constexpr (RUNS == 0) {
        for (long long r = blockIdx.x; r < s.rows; r += row_step, turn ^= 1) {
            const float scale = rstd[r];
            float d[8], v[8], g[8], dot = 0.0f;
            auto load = [&](int run) {
                const int left = s.cols - run * 8;
                load8_floats(dy + r * s.y_row + run * 8, left, d);
                load8_floats(x + r * s.x_row + run * 8, left, v);
                load_gamma(gamma, run, s.cols, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] *= g[j], v[j] *= scale;
            };
            for (int run = l; run * 8 < s.cols; run += lanes) {
                load(run);
#pragma unroll
                for (int j = 0; j < 8; ++j) dot += d[j] * v[j];
            }
            const float back = scale * (row_sum(dot, lanes, slots[turn]) * per);
            for (int run = l; run * 8 < s.cols; run += lanes) {
                load(run);
                const int left = s.cols - run * 8;
                float add[8] = {};
                if (dsum) load8_floats(dsum + r * s.residual_row + run * 8, left, add);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[j] = scale * d[j] - back * v[j] + add[j];
                store8(dx + r * s.sum_row + run * 8, left, d);
            }
        }
    } else {
        __shared__ float share[256 * 8];
        float g[RUNS][8], sums[RUNS][8];
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            load_gamma(gamma, l + i * lanes, s.cols, g[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[i][j] = 0.0f;
        }
        for (long long r = (long long)blockIdx.x * rows + group; r < s.rows; r += row_step, turn ^= 1) {
            // all of the row is on its way before any of it is waited for (asking for the next one too takes registers that more workgroups use better)
            Pack<Y, 8> of_dy[RUNS];
            Pack<T, 8> of_x[RUNS], of_dsum[RUNS];
            const float scale = rstd[r];
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int run = l + i * lanes, left = s.cols - run * 8;
                of_dy[i] = load8(dy + r * s.y_row + run * 8, left);
                of_x[i] = load8(x + r * s.x_row + run * 8, left);
                if (dsum) of_dsum[i] = load8(dsum + r * s.residual_row + run * 8, left);
            }
            float d[RUNS][8], dot = 0.0f;
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float xh = to_float(of_x[i].v[j]) * scale, of_y = to_float(of_dy[i].v[j]);
                    sums[i][j] += of_y * xh;
                    d[i][j] = of_y * g[i][j];
                    dot += d[i][j] * xh;
                }
            const float back = scale * (row_sum(dot, lanes, slots[turn]) * per);
#pragma unroll
            for (int i = 0; i < RUNS; ++i) {
                const int run = l + i * lanes, left = s.cols - run * 8;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    d[i][j] = scale * d[i][j] - back * (to_float(of_x[i].v[j]) * scale);
                    if (dsum) d[i][j] += to_float(of_dsum[i].v[j]);
                }
                if (left > 0) store8(dx + r * s.sum_row + run * 8, left, d[i]);
            }
        }
        if (!partial) return;
        float* to = partial + (long long)blockIdx.x * s.cols;
        if (rows == 1) {
#pragma unroll
            for (int i = 0; i < RUNS; ++i)
                if ((l + i * lanes) * 8 < s.cols) store8(to + (l + i * lanes) * 8, s.cols - (l + i * lanes) * 8, sums[i]);
            return;
        }
        // rows that share a workgroup: their sums in the order of the groups
#pragma unroll
        for (int j = 0; j < 8; ++j) share[threadIdx.x * 8 + j] = sums[0][j];
        __syncthreads();
        for (int c = (int)threadIdx.x; c < s.cols; c += (int)blockDim.x) {
            float v = 0.0f;
            for (int k = 0; k < rows; ++k) v += share[(k * lanes) * 8 + c];
            to[c] = v;
        }
    }
}

// dgamma[c] = the sum of partial[0 ... count)[c]: 32 columns a workgroup, its 32 half wavefronts each a part of the rows, eight on their way at a time.
__global__ __launch_bounds__(1024) void rms_join_kernel(int cols, int count, const float* __restrict__ partial, float* __restrict__ dgamma)
{
    __shared__ float sums[32][32];
    const int lane = (int)threadIdx.x & 31, part = (int)threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    const int per = (count + 31) / 32, first = part * per, last = min(first + per, count);
    float v = 0.0f;
    if (c < cols)
#pragma unroll 8
        for (int k = first; k < last; ++k) v += partial[(long long)k * cols + c];
    sums[part][lane] = v;
    __syncthreads();
    if (part || c >= cols) return;
    for (int k = 1; k < 32; ++k) v += sums[k][lane];
    dgamma[c] = v;
}

// dgamma of rows that are not held: partial[slab][c] over the rows of a slab, 256 columns a workgroup.
template <class T, class Y>
__global__ __launch_bounds__(256) void rms_gamma_kernel(RmsShape s, int slab_rows, const Y* __restrict__ dy, const T* __restrict__ x,
                                                        const float* __restrict__ rstd, float* __restrict__ partial)
{
    const long long c = (long long)blockIdx.x * 256 + threadIdx.x;
    if (c >= s.cols) return;
    const long long first = (long long)blockIdx.y * slab_rows, last = min(first + slab_rows, (long long)s.rows);
    float v = 0.0f;
    for (long long r = first; r < last; ++r) v += to_float(dy[r * s.y_row + c]) * (to_float(x[r * s.x_row + c]) * rstd[r]);
    partial[(long long)blockIdx.y * s.cols + c] = v;
}

// Most wavefronts a CU of the backward pass, whose workgroups keep sums of dgamma: all of them run at once, and every CU has as many (16384 x 4096 bf16 with 16, 24 and
// 32: 120, 109 and 133 us); at least two rows each.
constexpr int kBackwardWaves = 24, kBackwardWaves2 = 16; // with one run a lane, with two
constexpr int kSlabs = 64;
// Rows of partial sums of dgamma.
int partial_rows(const RmsShape& s)
{
    const Plan p = plan_of(s, true);
    if (!p.runs) return std::min(kSlabs, s.rows);
    const int each = std::max(1, (p.runs == 1 ? kBackwardWaves : kBackwardWaves2) * 64 / (p.lanes * p.rows));
    return (int)std::min<long long>(256 * each, ceil_div(s.rows, 2 * p.rows));
}

}  // namespace

// A grid has fewer than 2^32 threads: a workgroup for a row, or for several; backward, 64 threads for a column that is summed in slabs.
constexpr int kMostBackwardColumns = (1 << 26) - 1024;
bool rms_fits(const RmsShape& s, bool backward)
{
    if (s.cols > (backward ? kMostBackwardColumns : INT32_MAX - 8 * 1024 - 128)) return false;
    const Plan p = plan_of(s, backward);
    return backward || ceil_div(s.rows, p.rows) <= kMostBlocks * 256 / std::max(256, p.lanes);
}

size_t rms_workspace_floats(const RmsShape& s) { return s.rows ? (size_t)partial_rows(s) * (size_t)s.cols : 0; }

hipError_t launch_rms(const RmsShape& s, const void* x, const void* residual, const float* gamma, void* sum, void* y, uint8_t* y_scales, float* rstd,
                      hipStream_t stream)
{
    const Plan p = plan_of(s, false);
    const dim3 grid((unsigned)ceil_div(s.rows, p.rows)), block((unsigned)(p.lanes * p.rows));
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        auto run = [&](auto of_y, auto runs) {
            hipLaunchKernelGGL((rms_kernel<T, decltype(of_y), decltype(runs)::value>), grid, block, 0, stream, s, p.lanes, p.rows, static_cast<const T*>(x),
                               static_cast<const T*>(residual), gamma, static_cast<T*>(sum), y, y_scales, rstd);
        };
        auto with_runs = [&](auto of_y) {
            if (p.runs == 1) run(of_y, Const<1>{});
            else if (p.runs == 2) run(of_y, Const<2>{});
            else if (p.runs == kHeld) run(of_y, Const<kHeld>{});
            else run(of_y, Const<0>{});
        };
        if (s.y_type == kFp8) with_runs(Codes{});
        else with_type(s.y_type, with_runs);
    });
    return hipGetLastError();
}

hipError_t launch_rms_backward(const RmsShape& s, const void* dy, const void* dsum, const void* x, const float* rstd, const float* gamma, void* dx,
                               float* dgamma, float* workspace, hipStream_t stream)
{
    const Plan p = plan_of(s, true);
    const int count = s.rows ? partial_rows(s) : 0;
    float* const partial = dgamma ? workspace : nullptr;
    if (s.rows) {
        // (rows that are not held: as many workgroups as fit a grid many times over)
        const int groups = p.runs ? count : (int)std::min<long long>(1 << 16, s.rows);
        const dim3 grid((unsigned)groups), block((unsigned)(p.lanes * p.rows));
        with_type(s.type, [&](auto t) {
            using T = decltype(t);
            with_type(s.y_type, [&](auto of_y) {
                using Y = decltype(of_y);
                auto run = [&](auto runs) {
                    hipLaunchKernelGGL((rms_backward_kernel<T, Y, decltype(runs)::value>), grid, block, 0, stream, s, p.lanes, p.rows, groups * p.rows,
                                       static_cast<const Y*>(dy), static_cast<const T*>(dsum), static_cast<const T*>(x), rstd, gamma, static_cast<T*>(dx),
                                       partial);
                };
                if (p.runs == 1) run(Const<1>{});
                else if (p.runs == kHeldBackward) run(Const<kHeldBackward>{});
                else {
                    run(Const<0>{});
                    if (partial)
                        hipLaunchKernelGGL((rms_gamma_kernel<T, Y>), dim3((unsigned)((s.cols + 255ll) / 256), (unsigned)count), dim3(256), 0, stream, s,
                                           (s.rows + count - 1) / count, static_cast<const Y*>(dy), static_cast<const T*>(x), rstd, partial);
                }
            });
        });
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (!dgamma) return hipSuccess;
    hipLaunchKernelGGL(rms_join_kernel, dim3((unsigned)((s.cols + 31ll) / 32)), dim3(1024), 0, stream, s.cols, count, partial, dgamma);
    return hipGetLastError();
}

}  // namespace patdnn
