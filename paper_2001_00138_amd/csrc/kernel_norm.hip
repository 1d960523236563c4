// Group norm with an activation, channels last, forward and backward.
//
// Per image and group of channels, over all pixels (M values): mean mu, variance var = mean of (x - mu)^2,
// r = 1 / sqrt(var + eps), xh = (x - mu) r, z = gamma xh + beta, y = act(z).  Backward, with dz = dy act'(z):
//   dbeta = sum of dz and dgamma = sum of dz xh over images and pixels, per channel;
//   dx = r (gamma dz - (A + xh B) / M), A and B the sums of gamma dz and gamma dz xh over the group.
//
// Where a workgroup can hold the pixels of some whole groups in its registers it reads them once and needs no second launch (the
// "held" kernels below).  Otherwise what is normalised is read twice, once for the sums and once to apply them: a workgroup takes a
// slab of pixels and a chunk of channels that holds whole groups (or a part of one group, if that has more than
// kChunk channels); a lane keeps V adjacent channels and walks the slab's pixels, so that lanes read whole cache
// lines and channels need no shuffling.  Slabs leave their sums in the workspace; the second launch adds them up
// in the order of the slabs - the result does not depend on which workgroup came first - and applies them.
//
// Statistics are fp32.  What is held has its mean taken first and then the squared distances from it; where values are seen once, every lane runs
// Welford's update (mean and sum of squared distances from it), and partial results are joined by Chan's formula: none of them
// subtracts large squares from each other, so values far from zero keep their variance.  With ReLU z is rounded after each of its four operations, forward and backward alike, so
// that the two agree about the sign that decides its gradient.
//
// Bytes bound it, and for SiLU in two-byte types nearly as much the vector ALU, whose exponential and reciprocal take four cycles each.  64 x 56x56x256:
// forward fp16 with SiLU 58 us, 3.5 TB/s of the bytes that it cannot do without (held; a workgroup's 16 wavefronts fill a CU's registers, so
// that loads, arithmetic and stores of a CU overlap little); backward bf16 118 us, 2.6 TB/s, x and dy read twice at 4.3 TB/s; backward
// fp32 154 us, 4.0 TB/s (held).
#include <type_traits>

#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 256;          // most channels of a chunk
constexpr int kAhead = 4;            // pixels a lane has in flight

struct Geometry {
    NormShape s;
    int cpg;                         // channels per group
    int chunk, chunks, per_group;    // channels of a chunk, chunks of an image, chunks of a group (1: a chunk holds whole groups)
    int slab, slabs;                 // pixels of a slab, slabs of an image
    int tx, ty;                      // lanes side by side over channels, and over pixels
    int join;                        // lanes that join the sums of one group (a power of two up to 64)
    int runs, full, last_runs, last_full;        // pixels that the first `full` rows of lanes have, the others one less; of the last slab
    int width, parts;                // channels of a chunk that is whole, and how often a workgroup has a lane for each
    float m;                         // pixels * cpg.  (Divided by: a product with the rounded 1 / m would make the mean of equal values another one.)
    FastDiv by_slabs, by_chunks, by_tx, by_cpg, by_width;
};

// What a workgroup works on.
struct Place {
    int n, c0, width, g0, groups, part;      // image, first channel and channels, first group and groups, its place among a group's partial sums
    int p0, p1;                              // pixels
};
__device__ __forceinline__ Place place_of(const Geometry& G, uint32_t block)
{
    Place w;
    const uint32_t above = fast_div(block, G.by_slabs), slab = block - above * (uint32_t)G.slabs;
    const uint32_t n = fast_div(above, G.by_chunks), q = above - n * (uint32_t)G.chunks;
    w.n = (int)n;
    if (G.per_group == 1) {
        w.c0 = (int)q * G.chunk;
        w.width = min(G.chunk, G.s.c - w.c0);
        w.g0 = (int)fast_div((uint32_t)w.c0, G.by_cpg);
        w.groups = (int)fast_div((uint32_t)w.width, G.by_cpg);
        w.part = (int)slab;
    } else {
        w.g0 = (int)q / G.per_group;
        const int j = (int)q - w.g0 * G.per_group;
        w.c0 = w.g0 * G.cpg + j * G.chunk;
        w.width = min(G.chunk, G.cpg - j * G.chunk);
        w.groups = 1;
        w.part = (int)slab * G.per_group + j;
    }
    w.p0 = (int)slab * G.slab;
    w.p1 = min(w.p0 + G.slab, G.s.pixels);
    return w;
}

__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    for (int d = lanes >> 1; d > 0; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// count, mean and squared distances of `entries` partial results, joined by the `lanes` lanes of which this is one.
// entry(i, n, mean, m2) gives the i-th.
template <class F>
__device__ __forceinline__ void join_stats(int entries, int lane, int lanes, F&& entry, float& mean, float& m2)
{
    float n = 0.0f, total = 0.0f;
    for (int i = lane; i < entries; i += lanes) {
        float ni, mi, si;
        entry(i, ni, mi, si);
        n += ni;
        total += ni * mi;
    }
    n = lanes_sum(n, lanes);
    mean = lanes_sum(total, lanes) / n;
    float s = 0.0f;
    for (int i = lane; i < entries; i += lanes) {
        float ni, mi, si;
        entry(i, ni, mi, si);
        const float d = mi - mean;
        s += si + ni * d * d;
    }
    m2 = lanes_sum(s, lanes);
}

template <class T, int V>
__device__ __forceinline__ void widen(const Pack<T, V>& a, float (&f)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_float(a.v[i]);
}

// Calls f(values) for every ty-th pixel of the slab from p on, kAhead loads in flight.
template <class T, int V, class F>
__device__ __forceinline__ void walk(const T* p, long long step, int count, F&& f)
{
    int k = 0;
    for (; k + kAhead <= count; k += kAhead) {
        Pack<T, V> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = load_pack<T, V>(p + u * step);
        __builtin_amdgcn_sched_barrier(0);               // all of them before the first is used
        p += kAhead * step;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            float x[V];
            widen(v[u], x);
            f(x);
        }
    }
    for (; k < count; ++k, p += step) {
        float x[V];
        widen(load_pack<T, V>(p), x);
        f(x);
    }
}

// ---- forward ----

template <class T, int V>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(Geometry G, const T* __restrict__ x, float* __restrict__ parts)
{
    __shared__ float s_mean[kThreads * V], s_m2[kThreads * V];
    const Place w = place_of(G, blockIdx.x);
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx;
    const int c = tx * V;
    const int pitch = G.tx * V;
    if (ty < G.ty && c < w.width) {
        const int first = w.p0 + ty, count = first < w.p1 ? (w.p1 - first + G.ty - 1) / G.ty : 0;
        float mean[V], m2[V], n = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) mean[i] = m2[i] = 0.0f;
        walk<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel, count, [&](const float (&v)[V]) {
            n += 1.0f;
            const float share = __builtin_amdgcn_rcpf(n);        // (off by 2^-23 of a step that moves the mean by less than a deviation / n)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = v[i] - mean[i];
                mean[i] = fmaf(d, share, mean[i]);
                m2[i] = fmaf(d, v[i] - mean[i], m2[i]);
            }
        });
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s_mean[ty * pitch + c + i] = mean[i];
            s_m2[ty * pitch + c + i] = m2[i];
        }
    }
    __syncthreads();
    // per group of the chunk: the rows of lanes and the group's channels
    const int lane = (int)threadIdx.x & (G.join - 1), per = G.per_group == 1 ? G.cpg : w.width;
    const FastDiv by_per = G.per_group == 1 ? G.by_cpg : FastDiv{0, 0};
    for (int g = (int)threadIdx.x / G.join; g < w.groups; g += kThreads / G.join) {
        float mean, m2;
        join_stats(per * G.ty, lane, G.join, [&](int i, float& ni, float& mi, float& si) {
            const int row = G.per_group == 1 ? (int)fast_div((uint32_t)i, by_per) : i / per;
            const int at = row * pitch + g * per + (i - row * per), pixels = w.p1 - w.p0;
            ni = (float)(pixels == G.slab ? G.runs - (row >= G.full) : G.last_runs - (row >= G.last_full));
            mi = s_mean[at];
            si = s_m2[at];
        }, mean, m2);
        if (lane == 0) {
            float* to = parts + (((long long)w.n * G.s.groups + w.g0 + g) * (G.slabs * G.per_group) + w.part) * 2;
            to[0] = mean;
            to[1] = m2;
        }
    }
}

// Number of values that the part-th partial result of a group counts.
__device__ __forceinline__ float part_count(const Geometry& G, int part)
{
    int slab = part, width = G.cpg;
    if (G.per_group > 1) {
        slab = part / G.per_group;
        width = min(G.chunk, G.cpg - (part - slab * G.per_group) * G.chunk);
    }
    return (float)min(G.slab, G.s.pixels - slab * G.slab) * (float)width;
}

// xh and z of the comment at the top, rounded after each operation.
__device__ __forceinline__ float centred(float x, float mean)
{
#pragma clang fp contract(off)
    return x - mean;
}
__device__ __forceinline__ float affine(float d, float rstd, float gamma, float beta)
{
#pragma clang fp contract(off)
    return d * rstd * gamma + beta;
}

// Without ReLU nothing jumps where z is 0: (x - mean) scale + beta with scale = rstd gamma, as the backward pass has it.  (x scale + (beta - mean scale)
// would be an operation less, but rounds at the size of mean scale: values far from zero would lose what x - mean keeps.)
// (binary16: x * 1 - mean takes x as it is stored, with a 1 that the compiler does not know; in fp32 x would be widened first.  64 x 56x56x256 with SiLU:
// 50.4 us with five tensors in turn, 51.9 widened.)
template <class T, int ACT>
__device__ __forceinline__ float apply_one(float x, float mean, float rstd, float gamma, float beta, float scale)
{
    float one = 1.0f;
    if (std::is_same_v<T, _Float16>) asm("" : "+s"(one));
    const float d = std::is_same_v<T, _Float16> ? fmaf(x, one, -mean) : centred(x, mean);
    return activate<ACT>(ACT == kActRelu ? affine(d, rstd, gamma, beta) : fmaf(d, scale, beta));
}

template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(Geometry G, const T* __restrict__ x, const float* __restrict__ gamma,
                                                              const float* __restrict__ beta, const float* __restrict__ parts,
                                                              T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    __shared__ float s_mean[kChunk], s_rstd[kChunk];
    const Place w = place_of(G, blockIdx.x);
    {
        const int lane = (int)threadIdx.x & (G.join - 1), entries = G.slabs * G.per_group;
        for (int g = (int)threadIdx.x / G.join; g < w.groups; g += kThreads / G.join) {
            const long long at = (long long)w.n * G.s.groups + w.g0 + g;
            const float* from = parts + at * entries * 2;
            float mean, m2;
            join_stats(entries, lane, G.join, [&](int i, float& ni, float& mi, float& si) {
                ni = part_count(G, i);
                mi = from[2 * i];
                si = from[2 * i + 1];
            }, mean, m2);
            if (lane == 0) {
                const float rstd = 1.0f / sqrtf(m2 / G.m + G.s.eps);
                s_mean[g] = mean;
                s_rstd[g] = rstd;
                if (w.part == 0) {
                    if (mean_out) mean_out[at] = mean;
                    if (rstd_out) rstd_out[at] = rstd;
                }
            }
        }
    }
    __syncthreads();
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx;
    const int c = tx * V, first = w.p0 + ty;
    if (ty >= G.ty || c >= w.width || first >= w.p1) return;
    float mean[V], rstd[V], ga[V], be[V], scale[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0;
        mean[i] = s_mean[g];
        rstd[i] = s_rstd[g];
        ga[i] = gamma ? gamma[w.c0 + c + i] : 1.0f;
        be[i] = beta ? beta[w.c0 + c + i] : 0.0f;
        scale[i] = rstd[i] * ga[i];
    }
    T* to = y + w.n * G.s.y_image + first * G.s.y_pixel + w.c0 + c;
    walk<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel, (w.p1 - first + G.ty - 1) / G.ty, [&](const float (&v)[V]) {
        Pack<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.v[i] = from_float<T>(apply_one<T, ACT>(v[i], mean[i], rstd[i], ga[i], be[i], scale[i]));
        store_pack<T, V>(to, r);
        to += G.ty * G.s.y_pixel;
    });
}

// ---- held in registers ----

// A workgroup holds all pixels of `chunk` channels (whole groups) of one image: lane (ty, tx) has channels tx V ... of pixels ty, ty + G.ty, ...
struct Held {
    NormShape s;
    int cpg, chunk, chunks, tx, ty, join;
    int span, entries;                                   // channels of a lane that are joined before others see them; what a row of lanes adds to a group
    int folded, lanes;                                   // a group's lanes in a row are a power of two (`lanes`), and the rows too: sums fold by exchange
    int runs, full;                                      // runs that the first `full` rows of lanes have, the others one less
    float m;
    int parts;                                           // into which the backward kernel cuts the rows of lanes where it adds columns up
    FastDiv by_chunks, by_tx, by_cpg, by_entries, by_chunk;
};

// Most runs that a lane holds, so that nothing spills: of 16 bytes, of eight, of fewer.
constexpr int held_runs(int run_bytes) { return run_bytes >= 16 ? 16 : run_bytes == 8 ? 24 : 32; }

__device__ __forceinline__ uint32_t held_block(uint32_t total)
{
    // neighbouring chunks share cache lines: each XCD (workgroups go to the eight in turn) takes a run of them
    const uint32_t xcd = blockIdx.x & 7, q = total >> 3, rest = total & 7;
    return xcd * q + min(xcd, rest) + (blockIdx.x >> 3);
}

// Registers that hold a run.  used(sum) keeps the compiler from holding the values that it widened the run to as well, once `sum`
// has them.
template <class T, int V>
struct Kept {
    static constexpr int kWords = V * sizeof(T) >= 4 ? V * (int)sizeof(T) / 4 : 1;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (V * sizeof(T) >= 4) {
            struct __attribute__((packed, aligned(sizeof(T)))) Words {
                uint32_t w[kWords];
            };
            const Words a = *reinterpret_cast<const Words*>(p);
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = a.w[i];
        } else {
            w[0] = *reinterpret_cast<const unsigned short*>(p);
        }
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0;
    }
    __device__ __forceinline__ float at(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
        else return to_float(__builtin_bit_cast(T, (unsigned short)(i & 1 ? w[i / 2] >> 16 : w[i / 2])));
    }
    template <int N>
    __device__ __forceinline__ void used(float (&sum)[N])
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                if (j + 1 < N) asm volatile("" : "+v"(w[i]), "+v"(sum[j]), "+v"(sum[j + 1 < N ? j + 1 : j]));
                else asm volatile("" : "+v"(w[i]), "+v"(sum[j]));
            }
    }
};

// Sum over a workgroup of what its lanes have for their group: over the lanes of a wavefront by exchange, over the wavefronts
// through s_part.
__device__ __forceinline__ float fold(const Held& G, float v, int c, int groups, int wave, int waves, float* s_part)
{
    for (int d = 1; d < G.lanes; d *= 2) v += __shfl_xor(v, d, 64);
    for (int d = G.tx; d < 64; d *= 2) v += __shfl_xor(v, d, 64);
    const int g = c < groups * G.cpg ? (int)fast_div((uint32_t)c, G.by_cpg) : 0;
    if (((int)threadIdx.x & 63) < G.tx && c < groups * G.cpg) s_part[wave * groups + g] = v;       // the wavefront's first row of lanes
    __syncthreads();
    v = 0.0f;
    for (int k = 0; k < waves; ++k) v += s_part[k * groups + g];
    return v;
}

// ONE: the V channels of a lane are of one group.
template <class T, int V, int R, bool ONE>
__global__ __launch_bounds__(1024) void norm_held_kernel(Held G, const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                                                         T* __restrict__ y, float* __restrict__ mean_out, float* __restrict__ rstd_out)
{
    extern __shared__ float shared[];                    // per lane (ONE) or lane and channel: mean, m2; then per group: mean, rstd
    const uint32_t block = held_block(gridDim.x);
    const uint32_t n = fast_div(block, G.by_chunks);
    const int c0 = (int)(block - n * (uint32_t)G.chunks) * G.chunk, width = min(G.chunk, G.s.c - c0);
    const int groups = (int)fast_div((uint32_t)width, G.by_cpg), g0 = (int)fast_div((uint32_t)c0, G.by_cpg);
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx, c = tx * V;
    const bool mine = ty < G.ty && c < width;
    const int pitch = G.tx * V / G.span, all = G.ty * pitch;
    float* s_mean = shared;
    float* s_m2 = shared + all;
    float* g_mean = s_m2 + all;
    float* g_rstd = g_mean + groups;
    const int count = mine ? G.runs - (ty >= G.full) : 0;
    // Without branches, so that all loads are on their way together: what a lane reads past its runs counts as nothing.
    Kept<T, V> kept[R];
    // (It is of its own group all the same, so that something not finite stays in there.)
    const T* from = x + n * G.s.x_image + c0 + (c < width ? c : 0);
    if (count) from += ty * G.s.x_pixel;
    const long long step = G.ty * G.s.x_pixel;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        kept[k].load(from);
        from += k + 1 < count ? step : 0;                // past its last run a lane reads that one again
    }
    float mean[ONE ? 1 : V], rstd[ONE ? 1 : V], ga[V], be[V];
    {
        // sums, then squared distances from a mean, of what the lane holds, per channel or over its channels.  Folded: the group's mean
        // (two sums over the workgroup); otherwise the lane's own, and lanes are joined by Chan's formula.
        constexpr int N = ONE ? (V > 1 ? 2 : 1) : V, M = ONE ? 1 : V;
        float sum[N], m2[N];
#pragma unroll
        for (int i = 0; i < N; ++i) sum[i] = m2[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k < G.runs) {
                const float counts = k < count ? 1.0f : 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i % N] = fmaf(counts, kept[k].at(i), sum[i % N]);
            }
            kept[k].used(sum);
        }
        if (ONE && N > 1) sum[0] += sum[N - 1];
        float* s_part = shared;                          // folded: per wavefront and group; two of them, for the sums and for the squares
        const int wave = (int)threadIdx.x >> 6, waves = (int)blockDim.x >> 6;
        const bool folded = ONE && G.folded;
        if (folded) {
            sum[0] = fold(G, sum[0], c, groups, wave, waves, s_part) / G.m;
        } else {
            const float many = (float)max(1, ONE ? count * V : count);
#pragma unroll
            for (int i = 0; i < M; ++i) sum[i] /= many;
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k < G.runs) {
                const float counts = k < count ? 1.0f : 0.0f;
                float from_mean[M];
#pragma unroll
                for (int i = 0; i < M; ++i) from_mean[i] = -counts * sum[i];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = fmaf(counts, kept[k].at(i), from_mean[ONE ? 0 : i]);
                    m2[i % N] = fmaf(d, d, m2[i % N]);
                }
            }
            kept[k].used(m2);
        }
        if (ONE && N > 1) m2[0] += m2[N - 1];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            ga[i] = gamma && count ? gamma[c0 + c + i] : 1.0f;
            be[i] = beta && count ? beta[c0 + c + i] : 0.0f;
        }
        if (folded) {
            m2[0] = fold(G, m2[0], c, groups, wave, waves, s_part + waves * groups);
            mean[0] = sum[0];
            rstd[0] = 1.0f / sqrtf(m2[0] / G.m + G.s.eps);
            const int g = (int)fast_div((uint32_t)c, G.by_cpg);
            if (ty == 0 && count && c == g * G.cpg) {
                const long long at = (long long)n * G.s.groups + g0 + g;
                if (mean_out) mean_out[at] = mean[0];
                if (rstd_out) rstd_out[at] = rstd[0];
            }
        } else {
            if constexpr (!ONE) {
                // channels of one group, equally many values each: pairs, then pairs of pairs
                auto pair = [&](int i, int d) {
                    const float mid = 0.5f * (sum[i] + sum[i + d]), off = sum[i] - mid;
                    m2[i] += m2[i + d] + 2.0f * (float)(count * d) * off * off;
                    sum[i] = mid;
                };
                if (G.span >= 2)
#pragma unroll
                    for (int i = 0; i < V; i += 2) pair(i, 1);
                if (G.span >= 4)
#pragma unroll
                    for (int i = 0; i + 2 < V; i += 4) pair(i, 2);
            }
            if (mine) {
                int at = ty * pitch + tx * (pitch / G.tx);
#pragma unroll
                for (int i = 0; i < M; ++i)
                    if (ONE || (i & (G.span - 1)) == 0) {
                        s_mean[at] = sum[i];
                        s_m2[at] = m2[i];
                        ++at;
                    }
            }
            __syncthreads();
            const int lane = (int)threadIdx.x & (G.join - 1);
            for (int g = (int)threadIdx.x / G.join; g < groups; g += (int)blockDim.x / G.join) {
                float mean_g, m2_g;
                join_stats(G.entries * G.ty, lane, G.join, [&](int i, float& ni, float& mi, float& si) {
                    const int row = (int)fast_div((uint32_t)i, G.by_entries), at = row * pitch + g * G.entries + (i - row * G.entries);
                    ni = (float)((G.runs - (row >= G.full)) * G.span);
                    mi = s_mean[at];
                    si = s_m2[at];
                }, mean_g, m2_g);
                if (lane == 0) {
                    const float rstd_g = 1.0f / sqrtf(m2_g / G.m + G.s.eps);
                    const long long at = (long long)n * G.s.groups + g0 + g;
                    g_mean[g] = mean_g;
                    g_rstd[g] = rstd_g;
                    if (mean_out) mean_out[at] = mean_g;
                    if (rstd_out) rstd_out[at] = rstd_g;
                }
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const int g = count ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0;
                mean[i] = g_mean[g];
                rstd[i] = g_rstd[g];
            }
        }
    }
    if (count == 0) return;
    T* to = y + n * G.s.y_image + ty * G.s.y_pixel + c0 + c;
    const long long y_step = G.ty * G.s.y_pixel;
    auto apply = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        float scale[V];
#pragma unroll
        for (int i = 0; i < V; ++i) scale[i] = rstd[ONE ? 0 : i] * ga[i];
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < count) {
                Pack<T, V> r;
#pragma unroll
                for (int i = 0; i < V; ++i) r.v[i] = from_float<T>(apply_one<T, ACT>(kept[k].at(i), mean[ONE ? 0 : i], rstd[ONE ? 0 : i], ga[i], be[i], scale[i]));
                store_pack<T, V>(to, r);
                to += y_step;
                __builtin_amdgcn_sched_barrier(0);       // one run's values at a time
            }
    };
    if (G.s.act == kActRelu) apply(Const<kActRelu>{});
    else if (G.s.act == kActSilu) apply(Const<kActSilu>{});
    else apply(Const<kActNone>{});
}

// ---- backward ----

// One channel's constants and what the backward pass makes of one value: dz, and d = x - mean, so that xh = d rstd.
//   dx = rstd (gamma dz - A/M - xh B/M) = dz scale - (shift + d slope)   with scale = rstd gamma, shift = rstd A/M, slope = rstd^2 B/M.
struct Channel {
    float mean, rstd, gamma, beta, scale;
    __device__ __forceinline__ void set(float m, float r, float g, float b) { mean = m, rstd = r, gamma = g, beta = b, scale = r * g; }
    template <int ACT>
    __device__ __forceinline__ void slopes(float x, float dy, float& dz, float& d) const
    {
        d = centred(x, mean);
        dz = dy;
        if (ACT == kActRelu) dz = affine(d, rstd, gamma, beta) <= 0.0f ? 0.0f : dy;       // the forward pass's z
        if (ACT == kActSilu) {
            const float z = fmaf(d, scale, beta), s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
            dz = dy * (s * fmaf(z, 1.0f - s, 1.0f));
        }
    }
};

// Calls f(x, dy) for every ty-th pixel of the slab.
template <class T, int V, class F>
__device__ __forceinline__ void walk2(const T* p, long long step, const T* q, long long qstep, int count, F&& f)
{
    constexpr int kTwo = kAhead / 2;
    int k = 0;
    for (; k + kTwo <= count; k += kTwo) {
        Pack<T, V> a[kTwo], b[kTwo];
#pragma unroll
        for (int u = 0; u < kTwo; ++u) {
            a[u] = load_pack<T, V>(p + u * step);
            b[u] = load_pack<T, V>(q + u * qstep);
        }
        p += kTwo * step;
        q += kTwo * qstep;
#pragma unroll
        for (int u = 0; u < kTwo; ++u) {
            float x[V], d[V];
            widen(a[u], x);
            widen(b[u], d);
            f(x, d);
        }
    }
    for (; k < count; ++k, p += step, q += qstep) {
        float x[V], d[V];
        widen(load_pack<T, V>(p), x);
        widen(load_pack<T, V>(q), d);
        f(x, d);
    }
}

// Sums over a slab's pixels: parts [image][slab][2][channel], dz first, then dz xh.
template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_back_sums_kernel(Geometry G, const T* __restrict__ dy, const T* __restrict__ x,
                                                                  const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                                  const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                  float* __restrict__ parts)
{
    __shared__ float s_a[kThreads * V], s_b[kThreads * V];
    const Place w = place_of(G, blockIdx.x);
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx;
    const int c = tx * V, pitch = G.tx * V;
    if (ty < G.ty && c < w.width) {
        const int first = w.p0 + ty, count = first < w.p1 ? (w.p1 - first + G.ty - 1) / G.ty : 0;
        Channel ch[V];
        float a[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const long long g = (long long)w.n * G.s.groups + w.g0 + (G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0);
            ch[i].set(mean_in[g], rstd_in[g], gamma ? gamma[w.c0 + c + i] : 1.0f, beta ? beta[w.c0 + c + i] : 0.0f);
            a[i] = b[i] = 0.0f;
        }
        walk2<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel,
                    dy + w.n * G.s.dy_image + first * G.s.dy_pixel + w.c0 + c, G.ty * G.s.dy_pixel, count, [&](const float (&v)[V], const float (&d)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float dz, off;
                ch[i].template slopes<ACT>(v[i], d[i], dz, off);
                a[i] += dz;
                b[i] = fmaf(dz, off, b[i]);
            }
        });
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s_a[ty * pitch + c + i] = a[i];
            s_b[ty * pitch + c + i] = b[i] * ch[i].rstd;
        }
    }
    __syncthreads();
    const int slab = w.p0 / G.slab;
    float* to = parts + ((long long)w.n * G.slabs + slab) * 2 * G.s.c + w.c0;
    for (int i = (int)threadIdx.x; i < w.width; i += kThreads) {
        float a = 0.0f, b = 0.0f;
        for (int k = 0; k < G.ty; ++k) {
            a += s_a[k * pitch + i];
            b += s_b[k * pitch + i];
        }
        to[i] = a;
        to[G.s.c + i] = b;
    }
}

// Sums over images (and slabs) of parts [row][2][channel] -> dbeta, dgamma, kParamChannels channels a workgroup.
constexpr int kParamChannels = 16;
__device__ __forceinline__ void add_params(int channels, long long rows, int first, const float* __restrict__ parts, float* s_a, float* s_b,
                                           float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    constexpr int kRows = kThreads / kParamChannels;
    const int i = (int)threadIdx.x % kParamChannels, row = (int)threadIdx.x / kParamChannels, c = first + i;
    float a = 0.0f, b = 0.0f;
    if (c < channels)
        for (long long k = row; k < rows; k += kRows) {
            a += parts[k * 2 * channels + c];
            b += parts[(k * 2 + 1) * channels + c];
        }
    s_a[threadIdx.x] = a;
    s_b[threadIdx.x] = b;
    __syncthreads();
    if (row == 0 && c < channels) {
        for (int k = 1; k < kRows; ++k) {
            a += s_a[k * kParamChannels + i];
            b += s_b[k * kParamChannels + i];
        }
        if (dbeta) dbeta[c] = a;
        if (dgamma) dgamma[c] = b;
    }
}

__global__ __launch_bounds__(kThreads) void norm_params_kernel(int channels, int images, const float* __restrict__ parts, float* __restrict__ dgamma,
                                                               float* __restrict__ dbeta)
{
    __shared__ float s_a[kThreads], s_b[kThreads];
    add_params(channels, images, (int)blockIdx.x * kParamChannels, parts, s_a, s_b, dgamma, dbeta);
}

// Runs of dy that the kernel below keeps in LDS, with room for r.
constexpr int held_in_lds(int r) { return r > 8 ? 9 : 0; }
// Most runs of x and dy that a lane holds.  Two-byte values: eight runs take as long as reading twice where thirteen do not fit the registers any
// more.  And where a lane's channels are of several groups, with statistics for each.
constexpr int held_back_runs(int type_bytes) { return type_bytes == 4 ? 13 : 8; }
constexpr int held_back_mixed_runs(int type_bytes) { return type_bytes == 4 ? 8 : 4; }

// The backward pass of what norm_held_kernel does.  x and dy are both held: R runs of either, of dy the first held_in_lds(R) in LDS.
// sums_a, sums_b: dz and dz xh over an image's pixels, per channel, images 2 * channels floats apart.
template <class T, int V, int R, bool ONE>
__global__ __launch_bounds__(1024) void norm_back_held_kernel(Held G, const T* __restrict__ dy, const T* __restrict__ x, const float* __restrict__ mean_in,
                                                              const float* __restrict__ rstd_in, const float* __restrict__ gamma,
                                                              const float* __restrict__ beta, T* __restrict__ dx, float* __restrict__ sums_a, float* __restrict__ sums_b)
{
    constexpr int kInLds = held_in_lds(R), M = ONE ? 1 : V;
    using Run = Kept<T, V>;
    extern __shared__ float shared[];
    const uint32_t block = held_block(gridDim.x);
    const uint32_t n = fast_div(block, G.by_chunks);
    const int c0 = (int)(block - n * (uint32_t)G.chunks) * G.chunk, width = min(G.chunk, G.s.c - c0);
    const int groups = (int)fast_div((uint32_t)width, G.by_cpg), g0 = (int)fast_div((uint32_t)c0, G.by_cpg);
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx, c = tx * V;
    const bool mine = ty < G.ty && c < width;
    const int threads = (int)blockDim.x, wave = (int)threadIdx.x >> 6, waves = threads >> 6;
    const int count = mine ? G.runs - (ty >= G.full) : 0;
    const int inside = c < width ? c : 0;
    Run* const s_dy = reinterpret_cast<Run*>(shared) + threadIdx.x;      // [run][thread]
    float* const s = shared + kInLds * threads * Run::kWords;
    // As in the forward kernel: no branches, what a lane reads past its runs counts as nothing.
    Run kx[R], kd[R - kInLds];
    {
        const T* px = x + n * G.s.x_image + c0 + inside;
        const T* pd = dy + n * G.s.dy_image + c0 + inside;
        if (count) px += ty * G.s.x_pixel, pd += ty * G.s.dy_pixel;
        const long long x_step = G.ty * G.s.x_pixel, d_step = G.ty * G.s.dy_pixel;
        Run first[kInLds ? kInLds : 1];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k < kInLds) first[k < kInLds ? k : 0].load(pd);
            else kd[k < kInLds ? 0 : k - kInLds].load(pd);
            pd += k + 1 < count ? d_step : 0;
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            kx[k].load(px);
            px += k + 1 < count ? x_step : 0;
        }
#pragma unroll
        for (int k = 0; k < kInLds; ++k) s_dy[k * threads] = first[k];      // read by this thread only
    }
    float mean[M], rstd[M], ga[V], be[V], a[V], b[V];
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const long long g = (long long)n * G.s.groups + g0 + (int)fast_div((uint32_t)(inside + i), G.by_cpg);
        mean[i] = mean_in[g];
        rstd[i] = rstd_in[g];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        ga[i] = gamma ? gamma[c0 + inside + i] : 1.0f;
        be[i] = beta ? beta[c0 + inside + i] : 0.0f;
        a[i] = b[i] = 0.0f;
    }
    auto channel = [&](int i) {
        Channel ch;
        ch.set(mean[ONE ? 0 : i], rstd[ONE ? 0 : i], ga[i], be[i]);
        return ch;
    };
    // dz and d of a run; the branch on the activation is inside so that the runs stay in the same registers
    auto slopes = [&](const Run& x_run, const Run& d_run, float (&dz)[V], float (&off)[V]) {
        auto each = [&](auto act) {
#pragma unroll
            for (int i = 0; i < V; ++i) channel(i).template slopes<decltype(act)::value>(x_run.at(i), d_run.at(i), dz[i], off[i]);
        };
        if (G.s.act == kActRelu) each(Const<kActRelu>{});
        else if (G.s.act == kActSilu) each(Const<kActSilu>{});
        else each(Const<kActNone>{});
    };
#pragma unroll
    for (int k = 0; k < R; ++k) {
        if (k < G.runs) {
            Run d = k < kInLds ? s_dy[k * threads] : kd[k < kInLds ? 0 : k - kInLds];
            if (k >= count) d.clear();
            float dz[V], off[V];
            slopes(kx[k], d, dz, off);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                a[i] += dz[i];
                b[i] = fmaf(dz[i], off[i], b[i]);
            }
        }
        kx[k].used(b);
        if (k >= kInLds) kd[k < kInLds ? 0 : k - kInLds].used(a);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) b[i] *= rstd[ONE ? 0 : i];

    float* const to_a = sums_a + (long long)n * 2 * G.s.c + c0;
    float* const to_b = sums_b + (long long)n * 2 * G.s.c + c0;
    float shift[M], slope[M];                            // of Channel's comment
    if (ONE && G.folded) {
        // over the rows of lanes of a wavefront by exchange, then the wavefronts; a group's sums likewise
        float ag = 0.0f, bg = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            for (int d = G.tx; d < 64; d *= 2) {
                a[i] += __shfl_xor(a[i], d, 64);
                b[i] += __shfl_xor(b[i], d, 64);
            }
            ag = fmaf(ga[i], a[i], ag);
            bg = fmaf(ga[i], b[i], bg);
        }
        for (int d = 1; d < G.lanes; d *= 2) {
            ag += __shfl_xor(ag, d, 64);
            bg += __shfl_xor(bg, d, 64);
        }
        float* const s_group = s;                        // [wave][2][group]
        float* const s_channel = s + waves * 2 * groups; // [wave][2][channel]
        const int g = (int)fast_div((uint32_t)inside, G.by_cpg);
        if (((int)threadIdx.x & 63) < G.tx && c < width) {
            s_group[(wave * 2) * groups + g] = ag;
            s_group[(wave * 2 + 1) * groups + g] = bg;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s_channel[(wave * 2) * G.chunk + c + i] = a[i];
                s_channel[(wave * 2 + 1) * G.chunk + c + i] = b[i];
            }
        }
        __syncthreads();
        ag = bg = 0.0f;
        for (int k = 0; k < waves; ++k) {
            ag += s_group[(k * 2) * groups + g];
            bg += s_group[(k * 2 + 1) * groups + g];
        }
        for (int i = (int)threadIdx.x; i < 2 * G.chunk; i += threads) {
            const int half = i >= G.chunk, at = i - half * G.chunk;
            float v = 0.0f;
            for (int k = 0; k < waves; ++k) v += s_channel[(k * 2 + half) * G.chunk + at];
            if (at < width) (half ? to_b : to_a)[at] = v;
        }
        shift[0] = rstd[0] * (ag / G.m);
        slope[0] = rstd[0] * rstd[0] * (bg / G.m);
    } else {
        const int pitch = G.tx * V, all = G.ty * pitch;
        float* const s_a = s;                            // [row of lanes][channel]
        float* const s_b = s + all;
        if (ty < G.ty) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s_a[ty * pitch + c + i] = a[i];
                s_b[ty * pitch + c + i] = b[i];
            }
        }
        __syncthreads();
        // columns: in parts of the rows, then the parts; the totals, weighted with gamma, stay in the first row
        float* const s_part = s + 2 * all;               // [part][2][channel]
        const int part = (int)fast_div(threadIdx.x, G.by_chunk);
        for (int i = part < G.parts ? (int)threadIdx.x - part * pitch : pitch; i < pitch; i += threads) {
            float pa = 0.0f, pb = 0.0f;
            for (int k = part; k < G.ty; k += G.parts) {
                pa += s_a[k * pitch + i];
                pb += s_b[k * pitch + i];
            }
            s_part[(part * 2) * pitch + i] = pa;
            s_part[(part * 2 + 1) * pitch + i] = pb;
        }
        __syncthreads();
        for (int i = (int)threadIdx.x; i < width; i += threads) {
            float pa = 0.0f, pb = 0.0f;
            for (int k = 0; k < G.parts; ++k) {
                pa += s_part[(k * 2) * pitch + i];
                pb += s_part[(k * 2 + 1) * pitch + i];
            }
            to_a[i] = pa;
            to_b[i] = pb;
            const float weight = gamma ? gamma[c0 + i] : 1.0f;
            s_a[i] = weight * pa;
            s_b[i] = weight * pb;
        }
        __syncthreads();
        float* const g_a = s_part;                       // per group
        float* const g_b = s_part + groups;
        const int lane = (int)threadIdx.x & (G.join - 1);
        for (int g = (int)threadIdx.x / G.join; g < groups; g += threads / G.join) {
            float ag = 0.0f, bg = 0.0f;
            for (int i = lane; i < G.cpg; i += G.join) {
                ag += s_a[g * G.cpg + i];
                bg += s_b[g * G.cpg + i];
            }
            ag = lanes_sum(ag, G.join);
            bg = lanes_sum(bg, G.join);
            if (lane == 0) {
                g_a[g] = ag / G.m;
                g_b[g] = bg / G.m;
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const int g = (int)fast_div((uint32_t)(inside + i), G.by_cpg);
            shift[i] = rstd[i] * g_a[g];
            slope[i] = rstd[i] * rstd[i] * g_b[g];
        }
    }
    if (count == 0) return;
    T* out = dx + n * G.s.y_image + ty * G.s.y_pixel + c0 + c;
    const long long step = G.ty * G.s.y_pixel;
#pragma unroll
    for (int k = 0; k < R; ++k)
        if (k < count) {
            const Run d = k < kInLds ? s_dy[k * threads] : kd[k < kInLds ? 0 : k - kInLds];
            float dz[V], off[V];
            slopes(kx[k], d, dz, off);
            Pack<T, V> r;
#pragma unroll
            for (int i = 0; i < V; ++i)
                r.v[i] = from_float<T>(fmaf(dz[i], channel(i).scale, -fmaf(off[i], slope[ONE ? 0 : i], shift[ONE ? 0 : i])));
            store_pack<T, V>(out, r);
            out += step;
            __builtin_amdgcn_sched_barrier(0);           // one run's values at a time
        }
}

// The first `param_blocks` workgroups add the slabs of all images up to dgamma and dbeta, the others apply.
template <class T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void norm_back_apply_kernel(Geometry G, int param_blocks, const T* __restrict__ dy, const T* __restrict__ x,
                                                                   const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                                   const float* __restrict__ gamma, const float* __restrict__ beta,
                                                                   const float* __restrict__ parts, T* __restrict__ dx,
                                                                   float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float s_a[kThreads], s_b[kThreads];
    if ((int)blockIdx.x < param_blocks) {
        add_params(G.s.c, (long long)G.s.n * G.slabs, (int)blockIdx.x * kParamChannels, parts, s_a, s_b, dgamma, dbeta);
        return;
    }
    const Place w = place_of(G, blockIdx.x - (uint32_t)param_blocks);
    const float* from = parts + (long long)w.n * G.slabs * 2 * G.s.c;
    __shared__ float g_a[kChunk], g_b[kChunk];           // per group of the chunk: A / M, B / M
    if (G.per_group == 1) {
        // channels side by side, the slabs in as many parts as there are lanes for (kThreads >= kChunk)
        const int part = (int)fast_div(threadIdx.x, G.by_width), i = (int)threadIdx.x - part * G.width;
        float a = 0.0f, b = 0.0f;
        if (part < G.parts && i < w.width) {
            const float* p = from + (long long)part * 2 * G.s.c + w.c0 + i;
            const long long step = (long long)G.parts * 2 * G.s.c;
#pragma unroll 4
            for (int k = part; k < G.slabs; k += G.parts, p += step) {
                a += p[0];
                b += p[G.s.c];
            }
        }
        s_a[threadIdx.x] = a;
        s_b[threadIdx.x] = b;
        __syncthreads();
        if (part == 0 && i < w.width) {
            for (int k = 1; k < G.parts; ++k) {
                a += s_a[k * G.width + i];
                b += s_b[k * G.width + i];
            }
            const float ga = gamma ? gamma[w.c0 + i] : 1.0f;
            s_a[i] = ga * a;
            s_b[i] = ga * b;
        }
        __syncthreads();
        const int lane = (int)threadIdx.x & (G.join - 1);
        for (int g = (int)threadIdx.x / G.join; g < w.groups; g += kThreads / G.join) {
            float a = 0.0f, b = 0.0f;
            for (int i = lane; i < G.cpg; i += G.join) {
                a += s_a[g * G.cpg + i];
                b += s_b[g * G.cpg + i];
            }
            a = lanes_sum(a, G.join);
            b = lanes_sum(b, G.join);
            if (lane == 0) {
                g_a[g] = a / G.m;
                g_b[g] = b / G.m;
            }
        }
    } else {
        float a = 0.0f, b = 0.0f;
        for (int i = (int)threadIdx.x; i < G.cpg; i += kThreads) {
            const int c = w.g0 * G.cpg + i;
            float ca = 0.0f, cb = 0.0f;
            for (int k = 0; k < G.slabs; ++k) {
                ca += from[(long long)k * 2 * G.s.c + c];
                cb += from[((long long)k * 2 + 1) * G.s.c + c];
            }
            const float ga = gamma ? gamma[c] : 1.0f;
            a = fmaf(ga, ca, a);
            b = fmaf(ga, cb, b);
        }
        a = lanes_sum(a, 64);
        b = lanes_sum(b, 64);
        if ((threadIdx.x & 63) == 0) {
            s_a[threadIdx.x >> 6] = a;
            s_b[threadIdx.x >> 6] = b;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int k = 1; k < kThreads / 64; ++k) {
                a += s_a[k];
                b += s_b[k];
            }
            g_a[0] = a / G.m;
            g_b[0] = b / G.m;
        }
    }
    __syncthreads();
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx;
    const int c = tx * V, first = w.p0 + ty;
    if (ty >= G.ty || c >= w.width || first >= w.p1) return;
    Channel ch[V];
    float shift[V], slope[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0;
        const long long at = (long long)w.n * G.s.groups + w.g0 + g;
        ch[i].set(mean_in[at], rstd_in[at], gamma ? gamma[w.c0 + c + i] : 1.0f, beta ? beta[w.c0 + c + i] : 0.0f);
        shift[i] = ch[i].rstd * g_a[g];
        slope[i] = ch[i].rstd * ch[i].rstd * g_b[g];
    }
    T* to = dx + w.n * G.s.y_image + first * G.s.y_pixel + w.c0 + c;
    walk2<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel,
                dy + w.n * G.s.dy_image + first * G.s.dy_pixel + w.c0 + c, G.ty * G.s.dy_pixel, (w.p1 - first + G.ty - 1) / G.ty,
                [&](const float (&v)[V], const float (&d)[V]) {
        Pack<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float dz, off;
            ch[i].template slopes<ACT>(v[i], d[i], dz, off);
            r.v[i] = from_float<T>(fmaf(dz, ch[i].scale, -fmaf(off, slope[i], shift[i])));
        }
        store_pack<T, V>(to, r);
        to += G.ty * G.s.y_pixel;
    });
}

// ---- launches ----

// Chunks and slabs go by the sizes alone (the workspace's size does too).
Geometry geometry_of(const NormShape& s, bool backward)
{
    Geometry G{};
    G.s = s;
    G.cpg = s.c / s.groups;
    if (G.cpg > kChunk) {
        G.chunk = kChunk;
        G.per_group = (G.cpg + kChunk - 1) / kChunk;
        G.chunks = s.groups * G.per_group;
    } else {
        // whole groups, and a multiple of eight channels if there is one, so that lanes have whole runs
        int unit = G.cpg;
        while (unit % 8 && unit + G.cpg <= kChunk) unit += G.cpg;
        if (unit % 8) unit = G.cpg;
        G.chunk = std::min(kChunk / unit * unit, s.c);
        G.per_group = 1;
        G.chunks = (s.c + G.chunk - 1) / G.chunk;
    }
    // Four workgroups a CU if the slabs keep 32 pixels, backward 64: every workgroup of the second launch adds up all slabs of its image, backward
    // per channel (16 x 112x112x64 in groups of two, fp16: 26 us, 37 with twice the slabs; its backward pass in bf16 41 and 103).
    const long long want = 4 * 256 / std::max<long long>(1, (long long)s.n * G.chunks);
    const int least = backward ? 64 : 32, most = (int)std::min<long long>(backward ? 64 : 128, (s.pixels + least - 1) / least);
    G.slabs = (int)std::max<long long>(1, std::min<long long>(want, most));
    G.slab = (s.pixels + G.slabs - 1) / G.slabs;
    G.slabs = (int)ceil_div(s.pixels, G.slab);
    G.m = (float)((double)s.pixels * G.cpg);
    return G;
}

// Elements that a lane moves with one access: up to 16 bytes of them, and the channels (of a chunk, of a part of a group) a multiple.
int run_of(const NormShape& s)
{
    int v = 16 / (int)element_bytes(s.type);
    while (s.c % v) v /= 2;
    return v;
}
int run_of(const Geometry& G)
{
    int v = run_of(G.s);
    while ((G.chunks > 1 && G.chunk % v) || (G.per_group > 1 && G.cpg % v)) v /= 2;
    return v;
}

void finish(Geometry& G, int v)
{
    G.tx = (std::min(G.chunk, G.s.c) + v - 1) / v;
    G.ty = kThreads / G.tx;
    G.width = std::min(G.chunk, G.s.c);
    G.parts = kThreads / G.width;
    G.by_width = make_fast_div((uint32_t)G.width);
    const int last = G.s.pixels - (G.slabs - 1) * G.slab;
    G.runs = (G.slab + G.ty - 1) / G.ty;
    G.full = G.slab - (G.runs - 1) * G.ty;
    G.last_runs = (last + G.ty - 1) / G.ty;
    G.last_full = last - (G.last_runs - 1) * G.ty;
    G.by_slabs = make_fast_div((uint32_t)G.slabs);
    G.by_chunks = make_fast_div((uint32_t)G.chunks);
    G.by_tx = make_fast_div((uint32_t)G.tx);
    G.by_cpg = make_fast_div((uint32_t)G.cpg);
    const int groups = G.per_group == 1 ? G.chunk / G.cpg : 1;
    G.join = 64;
    while (G.join > 1 && groups * G.join > kThreads) G.join /= 2;
}

template <class F>
void with_run(int v, F&& f)
{
    v == 8 ? f(Const<8>{}) : v == 4 ? f(Const<4>{}) : v == 2 ? f(Const<2>{}) : f(Const<1>{});
}

// The held kernel's geometry for lanes of `v` channels, up to `most` runs a lane; false if the pixels do not fit.
bool held_of(const NormShape& s, int v, int most, bool backward, Held& H, int& threads, int& runs)
{
    H = Held{};
    H.s = s;
    H.cpg = s.c / s.groups;
    H.chunk = H.cpg;
    while (H.chunk % v && H.chunk < s.c) H.chunk += H.cpg;
    auto fits = [&](int chunk) { return chunk % v == 0 && chunk / v <= 1024 && (s.pixels + 1024 / (chunk / v) - 1) / (1024 / (chunk / v)) <= most; };
    if (!fits(H.chunk)) return false;
    // Few bytes a pixel and many pixels: most of each cache line is fetched for others.  (1 x 112x112x64 in groups of two channels, fp16: 29 us
    // held and 17 in two launches; 64 of them 89 and 69; at 56x56 11 and 15, 18 and 29.  Backward 32 x 90x90x128 in groups of four, fp32: 183 and 163.)
    if (H.chunk * element_bytes(s.type) < 32 && s.pixels > (backward ? 4096 : 8192)) return false;
    // 64 adjacent bytes a pixel, as long as every CU has a workgroup
    while (H.chunk * element_bytes(s.type) < 64 && H.chunk * 2 <= s.c && fits(H.chunk * 2) && (long long)s.n * (s.c / (H.chunk * 2)) >= 256) H.chunk *= 2;
    H.chunks = (int)ceil_div(s.c, H.chunk);
    if ((long long)s.n * H.chunks > kMostBlocks / 4) return false;
    H.tx = H.chunk / v;
    // Every lane has one run where there are few workgroups; where there are many, four (eight where x and dy are held), and several
    // workgroups share a CU.  (64 x 14x14x1024 fp16: 34 us with one run a lane, 16 with four.)
    const long long need = (long long)H.tx * s.pixels / ((long long)s.n * H.chunks < 512 ? 1 : std::min(most, backward ? 8 : 4));
    threads = (int)std::max<long long>((H.tx + 63) / 64 * 64, std::min<long long>(1024, (need + 63) / 64 * 64));
    // `need` is rounded down, and so are the rows of lanes: more lanes where that leaves runs without room (1024 have room: fits())
    while ((s.pixels + threads / H.tx - 1) / (threads / H.tx) > most) threads += 64;
    H.ty = threads / H.tx;
    runs = H.runs = (s.pixels + H.ty - 1) / H.ty;
    H.full = s.pixels - (H.runs - 1) * H.ty;
    H.m = (float)((double)s.pixels * H.cpg);
    H.by_chunks = make_fast_div((uint32_t)H.chunks);
    H.by_tx = make_fast_div((uint32_t)H.tx);
    H.by_cpg = make_fast_div((uint32_t)H.cpg);
    H.span = H.cpg % v == 0 ? v : v % H.cpg == 0 && H.cpg <= 4 ? H.cpg : 1;
    H.entries = H.lanes = H.cpg / H.span;
    auto power = [](int i) { return (i & (i - 1)) == 0; };
    H.folded = H.cpg % v == 0 && H.tx <= 64 && power(H.tx) && power(H.lanes);
    H.by_entries = make_fast_div((uint32_t)H.entries);
    H.parts = std::max(1, threads / H.chunk);
    H.by_chunk = make_fast_div((uint32_t)H.chunk);
    H.join = 64;
    while (H.join > 1 && H.chunk / H.cpg * H.join > threads) H.join /= 2;
    return true;
}

size_t held_lds(const Held& H, int v, int threads)
{
    const size_t groups = (size_t)H.chunk / H.cpg;
    return (H.folded ? (size_t)threads / 64 * groups : (size_t)H.ty * H.tx * v / H.span + groups) * 2 * sizeof(float);
}

template <class T, int V, int R, bool ONE>
hipError_t launch_held(const Held& H, int threads, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                       hipStream_t stream)
{
    static std::atomic<uint64_t> allowed{0};
    const size_t lds = held_lds(H, V, threads);
    if (lds > 64 * 1024)
        if (const hipError_t e = allow_big_lds(reinterpret_cast<const void*>(norm_held_kernel<T, V, R, ONE>), allowed); e != hipSuccess) return e;
    hipLaunchKernelGGL((norm_held_kernel<T, V, R, ONE>), dim3((unsigned)(H.s.n * H.chunks)), dim3((unsigned)threads), lds, stream, H,
                       static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd);
    return hipGetLastError();
}

// The backward kernel's LDS: held runs of dy; where sums fold, per wavefront those of groups and channels, else those of every lane and
// of the parts of the rows.
size_t held_back_lds(const Held& H, int v, int threads, int in_lds, size_t run_bytes)
{
    const size_t groups = (size_t)H.chunk / H.cpg;
    const size_t floats = H.folded ? (size_t)threads / 64 * 2 * (groups + H.chunk) : 2 * (size_t)H.ty * H.chunk + std::max<size_t>(2 * (size_t)H.parts * H.chunk, 2 * groups);
    return (size_t)in_lds * threads * run_bytes + floats * sizeof(float);
}

template <class T, int V, int R, bool ONE>
hipError_t launch_held_back(const Held& H, int threads, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma,
                            const float* beta, void* dx, float* sums_a, float* sums_b, hipStream_t stream)
{
    static std::atomic<uint64_t> allowed{0};
    const size_t lds = held_back_lds(H, V, threads, held_in_lds(R), sizeof(Kept<T, V>));
    if (lds > 64 * 1024)
        if (const hipError_t e = allow_big_lds(reinterpret_cast<const void*>(norm_back_held_kernel<T, V, R, ONE>), allowed); e != hipSuccess) return e;
    hipLaunchKernelGGL((norm_back_held_kernel<T, V, R, ONE>), dim3((unsigned)(H.s.n * H.chunks)), dim3((unsigned)threads), lds, stream, H,
                       static_cast<const T*>(dy), static_cast<const T*>(x), mean, rstd, gamma, beta, static_cast<T*>(dx),
                       sums_a, sums_b);
    return hipGetLastError();
}

int param_blocks_of(const NormShape& s) { return (s.c + kParamChannels - 1) / kParamChannels; }

// What a call launches: the held kernel for lanes of `v` channels with room for `room` runs, or (v = 0) two launches.
struct Plan {
    Held H{};
    int v = 0, threads = 0, runs = 0, room = 0;
    bool one = false;                                    // the kernels' ONE
};
Plan plan_of(const NormShape& s)
{
    Plan p;
    for (int v = run_of(s); v > 0; v /= 2) {
        const int most = held_runs(v * (int)element_bytes(s.type));
        if (!held_of(s, v, most, false, p.H, p.threads, p.runs)) continue;
        p.v = v;
        p.one = p.H.cpg % v == 0;
        p.room = p.runs <= 2 ? 2 : p.runs <= most / 4 ? most / 4 : p.runs <= most / 2 ? most / 2 : p.runs <= most * 3 / 4 + 1 ? most * 3 / 4 + 1 : most;
        break;
    }
    return p;
}

// Held where lanes have whole runs of 16 bytes, and sums fold or pixels are few: the other way to add columns up costs more than reading
// twice (8 x 56x56x64 in groups of two, fp32: 23 us and 15).
Plan back_plan_of(const NormShape& s)
{
    Plan p;
    const int bytes = (int)element_bytes(s.type), v = 16 / bytes, most = held_back_runs(bytes);
    if (run_of(s) != v) return p;
    p.one = s.c / s.groups % v == 0;
    // more constants a lane: fewer runs
    if (!held_of(s, v, p.one ? most : held_back_mixed_runs(bytes), true, p.H, p.threads, p.runs)) return p;
    p.room = p.runs <= 2 ? 2 : p.runs <= 4 ? 4 : p.runs <= 8 ? 8 : most;
    if (!p.one && p.room > held_back_mixed_runs(bytes)) return p;          // no such kernel (nor does held_of ask for it)
    // (64 x 56x56x256 bf16, 32 bytes a pixel: 135 us held, 118 in two launches)
    if ((!p.H.folded && (s.pixels > 1024 || p.runs > 8)) || (p.H.chunk * bytes < 64 && (long long)s.n * p.H.chunks >= 256) ||
        held_back_lds(p.H, v, p.threads, held_in_lds(p.room), 16) > 160 * 1024)
        return p;
    p.v = v;
    return p;
}

}  // namespace

// For tests: lanes' channels (0: two launches), runs, room for runs, whether lanes keep to one group, threads, rows of lanes, channels of a chunk, bytes of LDS.
void norm_plan_numbers(const NormShape& s, bool backward, int32_t (&out)[8])
{
    const Plan p = backward ? back_plan_of(s) : plan_of(s);
    const size_t lds = !p.v ? 0 : backward ? held_back_lds(p.H, p.v, p.threads, held_in_lds(p.room), 16) : held_lds(p.H, p.v, p.threads);
    const int32_t numbers[8] = {p.v, p.runs, p.room, p.one, p.threads, p.H.ty, p.H.chunk, (int32_t)lds};
    std::copy(numbers, numbers + 8, out);
}

bool norm_fits(const NormShape& s)
{
    // 32-bit sums here and in the kernels go past the pixels and channels by as much as a workgroup has lanes
    if (s.pixels > kMostNormLength || s.c > kMostNormLength) return false;
    const Geometry G = geometry_of(s, false);
    return (long long)s.n * G.chunks <= kMostBlocks && (long long)s.n * G.chunks * G.slabs + param_blocks_of(s) <= kMostBlocks;
}

size_t norm_workspace_floats(const NormShape& s, bool backward)
{
    if (s.n == 0) return 0;
    const Geometry G = geometry_of(s, backward);
    return backward ? (size_t)s.n * G.slabs * 2 * s.c : (size_t)s.n * s.groups * G.slabs * G.per_group * 2;
}

hipError_t launch_norm(const NormShape& s, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                       float* workspace, hipStream_t stream)
{
    if (const Plan p = plan_of(s); p.v) {
        hipError_t e = hipErrorInvalidValue;
        with_type(s.type, [&](auto t) {
            using T = decltype(t);
            with_run(p.v, [&](auto run) {
                constexpr int V = decltype(run)::value;
                if constexpr (V * sizeof(T) <= 16) {
                    constexpr int kMost = held_runs(V * sizeof(T));
                    auto with_room = [&](auto r) {
                        constexpr int R = decltype(r)::value;
                        if constexpr (V > 1)
                            if (!p.one) {
                                e = launch_held<T, V, R, false>(p.H, p.threads, x, gamma, beta, y, mean, rstd, stream);
                                return;
                            }
                        e = launch_held<T, V, R, true>(p.H, p.threads, x, gamma, beta, y, mean, rstd, stream);
                    };
                    if (p.room == 2) with_room(Const<2>{});
                    else if (p.room == kMost / 4) with_room(Const<kMost / 4>{});
                    else if (p.room == kMost / 2) with_room(Const<kMost / 2>{});
                    else if (p.room == kMost * 3 / 4 + 1) with_room(Const<kMost * 3 / 4 + 1>{});
                    else with_room(Const<kMost>{});
                }
            });
        });
        return e;
    }
    Geometry G = geometry_of(s, false);
    const int v = run_of(G);
    finish(G, v);
    const dim3 grid((unsigned)(s.n * G.chunks * G.slabs));
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        with_run(v, [&](auto run) {
            constexpr int V = decltype(run)::value;
            if constexpr (V * sizeof(T) <= 16) {
                hipLaunchKernelGGL((norm_stats_kernel<T, V>), grid, dim3(kThreads), 0, stream, G, static_cast<const T*>(x), workspace);
                with_act(s.act, [&](auto act) {
                    hipLaunchKernelGGL((norm_apply_kernel<T, V, decltype(act)::value>), grid, dim3(kThreads), 0, stream, G, static_cast<const T*>(x),
                                       gamma, beta, workspace, static_cast<T*>(y), mean, rstd);
                });
            }
        });
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormShape& s, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma,
                                const float* beta, void* dx, float* dgamma, float* dbeta, float* workspace, hipStream_t stream)
{
    hipError_t e = hipErrorInvalidValue;
    if (s.n == 0) {                                      // sums over nothing
        if (dgamma && (e = launch_fill_zero(dgamma, (size_t)s.c, stream)) != hipSuccess) return e;
        if (dbeta && (e = launch_fill_zero(dbeta, (size_t)s.c, stream)) != hipSuccess) return e;
        return hipSuccess;
    }
    if (const Plan p = back_plan_of(s); p.v) {
        // one image: its sums are dbeta and dgamma
        float* const sums_a = s.n == 1 && dbeta ? dbeta : workspace;
        float* const sums_b = s.n == 1 && dgamma ? dgamma : workspace + s.c;
        with_type(s.type, [&](auto t) {
            using T = decltype(t);
            constexpr int V = 16 / (int)sizeof(T), kMost = held_back_runs(sizeof(T)), kMixed = held_back_mixed_runs(sizeof(T));
            auto with_room = [&](auto r) {
                constexpr int R = decltype(r)::value;
                if (p.one) e = launch_held_back<T, V, R, true>(p.H, p.threads, dy, x, mean, rstd, gamma, beta, dx, sums_a, sums_b, stream);
                else if constexpr (R <= kMixed) e = launch_held_back<T, V, R, false>(p.H, p.threads, dy, x, mean, rstd, gamma, beta, dx, sums_a, sums_b, stream);
            };
            if (p.room == 2) with_room(Const<2>{});
            else if (p.room == 4) with_room(Const<4>{});
            else if (p.room == 8) with_room(Const<8>{});
            else with_room(Const<kMost>{});
        });
        if (e == hipSuccess && s.n > 1 && (dgamma || dbeta)) {
            hipLaunchKernelGGL(norm_params_kernel, dim3((unsigned)param_blocks_of(s)), dim3(kThreads), 0, stream, s.c, s.n, workspace, dgamma, dbeta);
            e = hipGetLastError();
        }
        return e;
    }
    Geometry G = geometry_of(s, true);
    const int v = run_of(G);
    finish(G, v);
    const unsigned blocks = (unsigned)(s.n * G.chunks * G.slabs);
    const int params = dgamma || dbeta ? param_blocks_of(s) : 0;
    with_type(s.type, [&](auto t) {
        using T = decltype(t);
        with_run(v, [&](auto run) {
            constexpr int V = decltype(run)::value;
            if constexpr (V * sizeof(T) <= 16)
                with_act(s.act, [&](auto act) {
                    constexpr int ACT = decltype(act)::value;
                    hipLaunchKernelGGL((norm_back_sums_kernel<T, V, ACT>), dim3(blocks), dim3(kThreads), 0, stream, G, static_cast<const T*>(dy),
                                       static_cast<const T*>(x), mean, rstd, gamma, beta, workspace);
                    hipLaunchKernelGGL((norm_back_apply_kernel<T, V, ACT>), dim3(blocks + (unsigned)params), dim3(kThreads), 0, stream, G, params,
                                       static_cast<const T*>(dy), static_cast<const T*>(x), mean, rstd, gamma, beta, workspace,
                                       static_cast<T*>(dx), dgamma, dbeta);
                });
        });
    });
    return hipGetLastError();
}

}  // namespace patdnn
