// Linear layers on MXFP4 weights, many rows of few values (pointwise layers of up to 512 channels): bound by the bytes of x and of the output.
//
// A wavefront takes 16, 32 or 64 rows of x, all of their k: it reads them once, in whole cache lines, quantises them (four lanes share a block of 32 values)
// and turns the codes over in LDS of its own, from which a lane reads one block of one row, what the matrix instruction wants of it.  Then it
// multiplies them with one set of 64 outputs after the other; the weights are small and come from the caches.  Nothing waits for other wavefronts,
// and there is no launch before.  The weights' rows are dealt to the instruction's rows so that a lane's results for four tiles are sixteen
// neighbouring outputs.
//
// 50176 x 128 -> 512 fp16 with SiLU 23 us, 2.8 TB/s; 200704 x 64 -> 256 fp16 34 us, 3.8 TB/s (every wavefront reads, computes and stores in turn, and
// there are only two to four a SIMD).
#include <type_traits>

#include "linear.hpp"

namespace patdnn {

namespace {

struct Codes {};                                         // x is MXFP4 already

constexpr int kWaves = 4;                                // wavefronts of a workgroup

struct Args {
    LinearShape s;
    int pieces, sets, splits;                            // of 128 along k; of 64 outputs; workgroups that share them
    FastDiv by_splits;
};

// P pieces of 128 along k, kRowTiles tiles of 16 rows a wavefront.
template <class X, int P, int kRowTiles>
__global__ __launch_bounds__(64 * kWaves) void linear_short_kernel(Args A, const void* __restrict__ x, const uint8_t* __restrict__ x_scales,
                                                                   const uint8_t* __restrict__ w, const uint8_t* __restrict__ w_scales,
                                                                   const float* __restrict__ bias, void* __restrict__ out)
{
    // (scalar: a matrix instruction in a branch that only masks lanes out would be executed)
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int r = lane & 15, kb = lane >> 4;
    const uint32_t block = __builtin_amdgcn_readfirstlane((int)fast_div(blockIdx.x, A.by_splits)), split = blockIdx.x - block * (uint32_t)A.splits;
    const int m0 = ((int)block * kWaves + wave) * 16 * kRowTiles;
    if (m0 >= A.s.rows) return;
    // [tile][piece][row][64 bytes], a row's 16-byte chunks at their place xor row / 2 (banks); then scales [tile][piece][row][4]
    __shared__ char s_x[kWaves][kRowTiles * P * (1024 + 64)];
    char* const codes = s_x[wave];
    uint8_t* const scales = reinterpret_cast<uint8_t*>(codes + kRowTiles * P * 1024);
    // As many tiles at a time as keep sixteen loads on their way.  (The loop is not unrolled: each wavefront runs most of its code once, and the
    // instruction cache counts.)
    constexpr int kMost = P == 1 ? 4 : P == 2 ? 2 : 1, kTogether = kMost < kRowTiles ? kMost : kRowTiles;
#pragma unroll 1
    for (int j0 = 0; j0 < kRowTiles; j0 += kTogether) {
        if constexpr (std::is_same_v<X, Codes>) {
            uint4 v[kTogether][P];
            Pack<uint32_t, P> byte[kTogether];
#pragma unroll
            for (int t = 0; t < kTogether; ++t) {
                const long long row = (long long)min(m0 + (j0 + t) * 16 + r, A.s.rows - 1) * P;          // rows past the end: the last one, not stored
#pragma unroll
                for (int p = 0; p < P; ++p) v[t][p] = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + (row + p) * 64 + kb * 16);
                byte[t] = load_pack<uint32_t, P>(reinterpret_cast<const uint32_t*>(x_scales) + row);
            }
#pragma unroll
            for (int t = 0; t < kTogether; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    *reinterpret_cast<uint4*>(codes + ((j0 + t) * P + p) * 1024 + r * 64 + (kb ^ (r >> 1 & 3)) * 16) = v[t][p];
                    scales[((j0 + t) * P + p) * 64 + r * 4 + kb] = (uint8_t)(byte[t].v[p] >> (8 * kb));
                }
        } else {
            const int run = lane & 15;                                   // eight values of a row; lane / 16: one of four rows
            Pack<X, 8> v[kTogether][P][4];
#pragma unroll
            for (int t = 0; t < kTogether; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const X* at = static_cast<const X*>(x) + (long long)min(m0 + (j0 + t) * 16 + i * 4 + kb, A.s.rows - 1) * A.s.x_row + run * 8;
#pragma unroll
                    for (int p = 0; p + 1 < P; ++p) v[t][p][i] = load_pack<X, 8>(at + p * 128);
                    // the last piece may end early
                    const int left = A.s.in - (P - 1) * 128 - run * 8;
                    if (P * 128 <= A.s.in) v[t][P - 1][i] = load_pack<X, 8>(at + (P - 1) * 128);
                    else v[t][P - 1][i] = load8(at + (P - 1) * 128, left);
                }
#pragma unroll
            for (int t = 0; t < kTogether; ++t)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int at = (j0 + t) * P + p;
                        uint32_t top = largest(v[t][p][i]);
                        top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
                        top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
                        const uint32_t byte = scale_byte(top);
                        *reinterpret_cast<uint32_t*>(codes + at * 1024 + (i * 4 + kb) * 64 + ((run >> 2) ^ (i * 2 + (kb >> 1) & 3)) * 16 + (run & 3) * 4) =
                            byte == kNanScale ? 0u : encode8(v[t][p][i], scale_of(byte));
                        if ((run & 3) == 0) scales[at * 64 + (i * 4 + kb) * 4 + (run >> 2)] = (uint8_t)byte;
                    }
        }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                   // the wavefront's own: no barrier
    const char* const b_at = codes + r * 64 + (kb ^ (r >> 1 & 3)) * 16;
    const uint8_t* const sb_at = scales + r * 4 + kb;
    const int last = A.s.out - 1;
    for (int set = (int)split; set < A.sets; set += A.splits) {
        const int n0 = set * 64, n = n0 + kb * 16;
        uint4 a[4][P];
        Pack<uint32_t, P> sa[4];                         // four scales a piece, of which a lane's is the kb-th byte
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long row = (long long)min(n0 + (r >> 2) * 16 + i * 4 + (r & 3), last) * P;
#pragma unroll
            for (int p = 0; p < P; ++p) a[i][p] = *reinterpret_cast<const uint4*>(w + (row + p) * 64 + kb * 16);
            sa[i] = load_pack<uint32_t, P>(reinterpret_cast<const uint32_t*>(w_scales) + row);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int p = 0; p < P; ++p) sa[i].v[p] >>= 8 * kb;
        float add[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) add[i] = bias ? bias[min(n + i, last)] : 0.0f;
#pragma unroll 1
        for (int j = 0; j < kRowTiles; ++j) {
            floatx4 acc[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const uint4 b = *reinterpret_cast<const uint4*>(b_at + (j * P + p) * 1024);
                const uint32_t sb = sb_at[(j * P + p) * 64];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i] = multiply(a[i][p], b, acc[i], sa[i].v[p], sb);
            }
            const int m = m0 + j * 16 + r;
            float z[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = acc[i / 4][i % 4] + add[i];
            finish_sixteen(z, A.s.act);
            if (m < A.s.rows && n < A.s.out) store_results(out, m * A.s.out_row + n, A.s.out_type, A.s.out - n, z);
        }
    }
}

template <class X, int P, int kRowTiles>
hipError_t launch_tiles_of(Args A, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                           hipStream_t stream)
{
    // Where rows are few, several workgroups share the outputs, and each quantises the rows for itself.
    const long long blocks = (A.s.rows + kWaves * 16 * kRowTiles - 1) / (kWaves * 16 * kRowTiles);
    A.splits = (int)std::max<long long>(1, std::min<long long>(A.sets, (kRowTiles == 1 || P == 1 ? 1024 : 512) / blocks));
    A.by_splits = make_fast_div((uint32_t)A.splits);
    hipLaunchKernelGGL((linear_short_kernel<X, P, kRowTiles>), dim3((unsigned)(blocks * A.splits)), dim3(64 * kWaves), 0, stream, A, x, x_scales, w, w_scales,
                       bias, out);
    return hipGetLastError();
}

template <class X, int P>
hipError_t launch_pieces(const Args& A, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                         hipStream_t stream)
{
    // Few rows a wavefront where there is little work (784 x 256 -> 1024 fp16: 5 us, 7 and 11 with 32 and 64 rows), many where the weights
    // are read most (15516 x 352 -> 4772: 64 us, 98 and 73 with 16 and 32), else 32 (50176 x 128 -> 512: 22, 25 and 22 with 16 and 64).
    const long long work = (long long)((A.s.rows + 63) / 64) * A.sets;
    return work <= 1024                    ? launch_tiles_of<X, P, 1>(A, x, x_scales, w, w_scales, bias, out, stream)
           : A.sets >= 32 && work >= 8192 ? launch_tiles_of<X, P, 4>(A, x, x_scales, w, w_scales, bias, out, stream)
                                           : launch_tiles_of<X, P, 2>(A, x, x_scales, w, w_scales, bias, out, stream);
}

template <class X>
hipError_t launch_type(const Args& A, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                       hipStream_t stream)
{
    return A.pieces == 1   ? launch_pieces<X, 1>(A, x, x_scales, w, w_scales, bias, out, stream)
           : A.pieces == 2 ? launch_pieces<X, 2>(A, x, x_scales, w, w_scales, bias, out, stream)
           : A.pieces == 3 ? launch_pieces<X, 3>(A, x, x_scales, w, w_scales, bias, out, stream)
                           : launch_pieces<X, 4>(A, x, x_scales, w, w_scales, bias, out, stream);
}

}  // namespace

// Longer rows only where there are many: few workgroups would quantise the same ones too often (3136 x 512 -> 2048 fp16: 21 us, 16 through tiles).
bool short_fits(const LinearShape& s)
{
    const long long pieces = mxfp4_pieces(s.in);
    return s.rows >= 64 && (pieces <= 2 || (pieces <= 4 && s.rows >= 8192));
}

hipError_t launch_short(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                        hipStream_t stream)
{
    const Args A{s, (int)mxfp4_pieces(s.in), (s.out + 63) / 64, 1, {}};
    if (s.x_type == kMxfp4) return launch_type<Codes>(A, x, x_scales, w, w_scales, bias, out, stream);
    hipError_t e = hipSuccess;
    with_type(s.x_type, [&](auto t) { e = launch_type<decltype(t)>(A, x, x_scales, w, w_scales, bias, out, stream); });
    return e;
}

}  // namespace patdnn
