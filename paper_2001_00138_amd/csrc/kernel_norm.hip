// Group norm with an activation, channels last, forward and backward.
//
// Per image and group of channels, over all pixels (M values): mean mu, variance var = mean of (x - mu)^2,
// r = 1 / sqrt(var + eps), xh = (x - mu) r, z = gamma xh + beta, y = act(z).  Backward, with dz = dy act'(z):
//   dbeta = sum of dz and dgamma = sum of dz xh over images and pixels, per channel;
//   dx = r (gamma dz - (A + xh B) / M), A and B the sums of gamma dz and gamma dz xh over the group.
//
// Both read what they normalise twice, once for the sums and once to apply them: two launches.  A workgroup takes a
// slab of pixels and a chunk of channels that holds whole groups (or a part of one group, if that has more than
// kChunk channels); a lane keeps V adjacent channels and walks the slab's pixels, so that lanes read whole cache
// lines and channels need no shuffling.  Slabs leave their sums in the workspace; the second launch adds them up
// in the order of the slabs - the result does not depend on which workgroup came first - and applies them.
//
// Statistics are fp32.  Every lane runs Welford's update (mean and sum of squared distances from it), and partial results
// are joined by Chan's formula: neither subtracts large squares from each other, so values far from zero keep
// their variance.  z is rounded after each of its four operations, forward and backward alike, so that the two agree about
// the sign that decides ReLU's gradient.
#include "kernels.hpp"
#include "operators.hpp"

namespace patdnn {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 256;          // most channels of a chunk
constexpr int kMostSlabs = 128;
constexpr int kAhead = 4;            // pixels a lane has in flight

struct Geometry {
    NormShape s;
    int cpg;                         // channels per group
    int chunk, chunks, per_group;    // channels of a chunk, chunks of an image, chunks of a group (1: a chunk holds whole groups)
    int slab, slabs;                 // pixels of a slab, slabs of an image
    int tx, ty;                      // lanes side by side over channels, and over pixels
    int join;                        // lanes that join the sums of one group (a power of two up to 64)
    float inv_m;                     // 1 / (pixels * cpg)
    FastDiv by_slabs, by_chunks, by_tx, by_cpg;
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
            const float share = __builtin_amdgcn_rcpf(n);
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
            const int at = row * pitch + g * per + (i - row * per), left = w.p1 - w.p0 - row;
            ni = left > 0 ? (float)((left + G.ty - 1) / G.ty) : 0.0f;
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
__device__ __forceinline__ float normalised(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }
__device__ __forceinline__ float affine(float xh, float gamma, float beta) { return __fadd_rn(__fmul_rn(xh, gamma), beta); }

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
                const float rstd = 1.0f / sqrtf(m2 * G.inv_m + G.s.eps);
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
    float mean[V], rstd[V], ga[V], be[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0;
        mean[i] = s_mean[g];
        rstd[i] = s_rstd[g];
        ga[i] = gamma ? gamma[w.c0 + c + i] : 1.0f;
        be[i] = beta ? beta[w.c0 + c + i] : 0.0f;
    }
    T* to = y + w.n * G.s.y_image + first * G.s.y_pixel + w.c0 + c;
    walk<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel, (w.p1 - first + G.ty - 1) / G.ty, [&](const float (&v)[V]) {
        Pack<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) r.v[i] = from_float<T>(activate<ACT>(affine(normalised(v[i], mean[i], rstd[i]), ga[i], be[i])));
        store_pack<T, V>(to, r);
        to += G.ty * G.s.y_pixel;
    });
}

// ---- backward ----

// dz and xh of one value.
template <int ACT>
__device__ __forceinline__ void slopes(float x, float dy, float mean, float rstd, float gamma, float beta, float& dz, float& xh)
{
    xh = normalised(x, mean, rstd);
    dz = dy;
    if (ACT == kActNone) return;
    const float z = affine(xh, gamma, beta);
    if (ACT == kActRelu) {
        dz = z <= 0.0f ? 0.0f : dy;
    } else {
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-z));
        dz = dy * (s * fmaf(z, 1.0f - s, 1.0f));
    }
}

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
        float mean[V], rstd[V], ga[V], be[V], a[V], b[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const long long g = (long long)w.n * G.s.groups + w.g0 + (G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0);
            mean[i] = mean_in[g];
            rstd[i] = rstd_in[g];
            ga[i] = gamma ? gamma[w.c0 + c + i] : 1.0f;
            be[i] = beta ? beta[w.c0 + c + i] : 0.0f;
            a[i] = b[i] = 0.0f;
        }
        walk2<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel,
                    dy + w.n * G.s.dy_image + first * G.s.dy_pixel + w.c0 + c, G.ty * G.s.dy_pixel, count, [&](const float (&v)[V], const float (&d)[V]) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float dz, xh;
                slopes<ACT>(v[i], d[i], mean[i], rstd[i], ga[i], be[i], dz, xh);
                a[i] += dz;
                b[i] = fmaf(dz, xh, b[i]);
            }
        });
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s_a[ty * pitch + c + i] = a[i];
            s_b[ty * pitch + c + i] = b[i];
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

constexpr int kParamChannels = 16;       // channels of a workgroup that adds up dgamma and dbeta

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
        constexpr int kRows = kThreads / kParamChannels;
        const int i = (int)threadIdx.x % kParamChannels, row = (int)threadIdx.x / kParamChannels;
        const int c = (int)blockIdx.x * kParamChannels + i;
        float a = 0.0f, b = 0.0f;
        if (c < G.s.c)
            for (long long k = row; k < (long long)G.s.n * G.slabs; k += kRows) {
                a += parts[k * 2 * G.s.c + c];
                b += parts[(k * 2 + 1) * G.s.c + c];
            }
        s_a[threadIdx.x] = a;
        s_b[threadIdx.x] = b;
        __syncthreads();
        if (row == 0 && c < G.s.c) {
            for (int k = 1; k < kRows; ++k) {
                a += s_a[k * kParamChannels + i];
                b += s_b[k * kParamChannels + i];
            }
            if (dbeta) dbeta[c] = a;
            if (dgamma) dgamma[c] = b;
        }
        return;
    }
    const Place w = place_of(G, blockIdx.x - (uint32_t)param_blocks);
    const float* from = parts + (long long)w.n * G.slabs * 2 * G.s.c;
    __shared__ float g_a[kChunk], g_b[kChunk];           // per group of the chunk: A / M, B / M
    if (G.per_group == 1) {
        if ((int)threadIdx.x < w.width) {                // kThreads >= kChunk
            const int c = w.c0 + (int)threadIdx.x;
            float a = 0.0f, b = 0.0f;
            for (int k = 0; k < G.slabs; ++k) {
                a += from[(long long)k * 2 * G.s.c + c];
                b += from[((long long)k * 2 + 1) * G.s.c + c];
            }
            const float ga = gamma ? gamma[c] : 1.0f;
            s_a[threadIdx.x] = ga * a;
            s_b[threadIdx.x] = ga * b;
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
                g_a[g] = a * G.inv_m;
                g_b[g] = b * G.inv_m;
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
            g_a[0] = a * G.inv_m;
            g_b[0] = b * G.inv_m;
        }
    }
    __syncthreads();
    const int ty = (int)fast_div(threadIdx.x, G.by_tx), tx = (int)threadIdx.x - ty * G.tx;
    const int c = tx * V, first = w.p0 + ty;
    if (ty >= G.ty || c >= w.width || first >= w.p1) return;
    float mean[V], rstd[V], ga[V], be[V], ma[V], mb[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = G.per_group == 1 ? (int)fast_div((uint32_t)(c + i), G.by_cpg) : 0;
        mean[i] = mean_in[(long long)w.n * G.s.groups + w.g0 + g];
        rstd[i] = rstd_in[(long long)w.n * G.s.groups + w.g0 + g];
        ga[i] = gamma ? gamma[w.c0 + c + i] : 1.0f;
        be[i] = beta ? beta[w.c0 + c + i] : 0.0f;
        ma[i] = g_a[g];
        mb[i] = g_b[g];
    }
    T* to = dx + w.n * G.s.y_image + first * G.s.y_pixel + w.c0 + c;
    walk2<T, V>(x + w.n * G.s.x_image + first * G.s.x_pixel + w.c0 + c, G.ty * G.s.x_pixel,
                dy + w.n * G.s.dy_image + first * G.s.dy_pixel + w.c0 + c, G.ty * G.s.dy_pixel, (w.p1 - first + G.ty - 1) / G.ty,
                [&](const float (&v)[V], const float (&d)[V]) {
        Pack<T, V> r;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float dz, xh;
            slopes<ACT>(v[i], d[i], mean[i], rstd[i], ga[i], be[i], dz, xh);
            r.v[i] = from_float<T>(rstd[i] * (__fsub_rn(__fmul_rn(dz, ga[i]), ma[i]) - xh * mb[i]));
        }
        store_pack<T, V>(to, r);
        to += G.ty * G.s.y_pixel;
    });
}

// ---- launches ----

// Chunks and slabs go by the sizes alone (the workspace's size does too).
Geometry geometry_of(const NormShape& s)
{
    Geometry G{};
    G.s = s;
    G.cpg = s.c / s.groups;
    if (G.cpg > kChunk) {
        G.chunk = kChunk;
        G.per_group = (G.cpg + kChunk - 1) / kChunk;
        G.chunks = s.groups * G.per_group;
    } else {
        // whole groups, and a multiple of eight channels if there is one, so that the lanes' runs stay aligned
        int unit = G.cpg;
        while (unit % 8 && unit + G.cpg <= kChunk) unit += G.cpg;
        if (unit % 8) unit = G.cpg;
        G.chunk = std::min(kChunk / unit * unit, s.c);
        G.per_group = 1;
        G.chunks = (s.c + G.chunk - 1) / G.chunk;
    }
    // eight workgroups a CU if the slabs keep 32 pixels
    const long long want = 8 * 256 / std::max<long long>(1, (long long)s.n * G.chunks);
    const int most = (int)std::min<long long>(kMostSlabs, (s.pixels + 31) / 32);
    G.slabs = (int)std::max<long long>(1, std::min<long long>(want, most));
    G.slab = (s.pixels + G.slabs - 1) / G.slabs;
    G.slabs = (s.pixels + G.slab - 1) / G.slab;
    G.inv_m = (float)(1.0 / ((double)s.pixels * G.cpg));
    return G;
}

// Elements that a lane moves with one access: as many as everything is aligned to.
int run_of(const Geometry& G, const void* const* pointers, const long long* strides, int count)
{
    const int bytes = (int)element_bytes(G.s.type);
    uint64_t all = 0;
    for (int i = 0; i < count; ++i) all |= reinterpret_cast<uintptr_t>(pointers[i]) / bytes;
    for (int i = 0; i < 2 * count; ++i) all |= (uint64_t)strides[i];
    all |= (uint64_t)G.s.c;
    if (G.chunks > 1) all |= (uint64_t)G.chunk;
    if (G.per_group > 1) all |= (uint64_t)G.cpg;
    int v = 16 / bytes;
    while (all % (uint64_t)v) v /= 2;
    return v;
}

void finish(Geometry& G, int v)
{
    G.tx = (std::min(G.chunk, G.s.c) + v - 1) / v;
    G.ty = kThreads / G.tx;
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

int param_blocks_of(const NormShape& s) { return (s.c + kParamChannels - 1) / kParamChannels; }

}  // namespace

bool norm_fits(const NormShape& s)
{
    const Geometry G = geometry_of(s);
    return (long long)s.n * G.chunks <= kMostBlocks && (long long)s.n * G.chunks * G.slabs + param_blocks_of(s) <= kMostBlocks;
}

size_t norm_workspace_floats(const NormShape& s, bool backward)
{
    if (s.n == 0) return 0;
    const Geometry G = geometry_of(s);
    return backward ? (size_t)s.n * G.slabs * 2 * s.c : (size_t)s.n * s.groups * G.slabs * G.per_group * 2;
}

hipError_t launch_norm(const NormShape& s, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                       float* workspace, hipStream_t stream)
{
    Geometry G = geometry_of(s);
    const void* pointers[] = {x, y};
    const long long strides[] = {s.x_image, s.x_pixel, s.y_image, s.y_pixel};
    const int v = run_of(G, pointers, strides, 2);
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
    hipError_t e;
    if (s.n == 0) {                                      // sums over nothing
        if (dgamma && (e = launch_fill_zero(dgamma, (size_t)s.c, stream)) != hipSuccess) return e;
        if (dbeta && (e = launch_fill_zero(dbeta, (size_t)s.c, stream)) != hipSuccess) return e;
        return hipSuccess;
    }
    Geometry G = geometry_of(s);
    const void* pointers[] = {x, dx, dy};
    const long long strides[] = {s.x_image, s.x_pixel, s.y_image, s.y_pixel, s.dy_image, s.dy_pixel};
    const int v = run_of(G, pointers, strides, 3);
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
