// Linear layers on MXFP4 weights, on the scaled matrix instructions.
//
// out[m][n] = act(bias[n] + sum over k of x[m][k] w[n][k]).  The instruction multiplies 16 rows of 128 codes with 16
// others and applies the scales of their blocks of 32 itself; a lane holds one block of one row, 16 bytes, which is how
// rows lie in memory.  The weights are the instruction's first operand, so that a lane's four results are
// neighbours along n.  Sums are fp32.
//
// This kernel reads both operands straight from memory: a wavefront takes a range of k for a set of NT x MT tiles of 16 x 16 outputs,
// and the workgroup's wavefronts add their sums up in LDS, in the order of the ranges.
#include <type_traits>

#include "linear.hpp"

namespace patdnn {

namespace {

struct Codes {};                                         // x is MXFP4 already

struct Args {
    LinearShape s;
    int pieces;                                          // of 128 along k
    int n_tiles, m_tiles;                                // workgroups over the outputs
    bool whole_runs;                                     // rows of x in runs of 16 bytes
    FastDiv by_n;
};

// This lane's block of 32 values of row m: codes and scale byte.
template <class X>
__device__ __forceinline__ void block_of(const Args& A, const void* x, const uint8_t* x_scales, int m, int piece, int kb, uint4& codes, uint32_t& scale)
{
    if constexpr (std::is_same_v<X, Codes>) {
        const long long row = (long long)m * A.pieces + piece;
        codes = *reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + row * 64 + kb * 16);
        scale = x_scales[row * 4 + kb];
    } else {
        const int k = piece * 128 + kb * 32;
        const X* p = static_cast<const X*>(x) + (long long)m * A.s.x_row + k;
        Pack<X, 8> a[4];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = load8(p + 8 * i, A.s.in - k - 8 * i, A.whole_runs);
            top = max(top, largest(a[i]));
        }
        scale = scale_byte(top);
        const float unit = scale_of(scale);
        const bool fine = scale != kNanScale;
        codes = make_uint4(fine ? encode8(a[0], unit) : 0u, fine ? encode8(a[1], unit) : 0u, fine ? encode8(a[2], unit) : 0u,
                           fine ? encode8(a[3], unit) : 0u);
    }
}

template <class X, int NT, int MT>
__global__ __launch_bounds__(NT * MT > 1 ? 256 : 1024) void linear_direct_kernel(Args A, const void* __restrict__ x, const uint8_t* __restrict__ x_scales,
                                                             const uint8_t* __restrict__ w, const uint8_t* __restrict__ w_scales,
                                                             const float* __restrict__ bias, void* __restrict__ out)
{
    extern __shared__ float sums[];                      // [wavefront][tile][lane][4]
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, waves = (int)blockDim.x >> 6;
    const int r = lane & 15, kb = lane >> 4;
    const uint32_t mt = fast_div(blockIdx.x, A.by_n), nt = blockIdx.x - mt * (uint32_t)A.n_tiles;
    const int n0 = (int)nt * 16 * NT, m0 = (int)mt * 16 * MT;
    floatx4 acc[NT][MT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    const int per = (A.pieces + waves - 1) / waves;
    const int last = min(A.pieces, (wave + 1) * per);
    // rows past the end are read as the last one, and their results dropped
    for (int piece = wave * per; piece < last; ++piece) {
        uint4 a[NT], b[MT];
        uint32_t sa[NT], sb[MT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const long long row = (long long)min(n0 + i * 16 + r, A.s.out - 1) * A.pieces + piece;
            a[i] = *reinterpret_cast<const uint4*>(w + row * 64 + kb * 16);
            sa[i] = w_scales[row * 4 + kb];
        }
#pragma unroll
        for (int j = 0; j < MT; ++j) block_of<X>(A, x, x_scales, min(m0 + j * 16 + r, A.s.rows - 1), piece, kb, b[j], sb[j]);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[i][j] = multiply(a[i], b[j], acc[i][j], sa[i], sb[j]);
    }
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) *reinterpret_cast<floatx4*>(sums + ((wave * NT * MT + i * MT + j) * 64 + lane) * 4) = acc[i][j];
    __syncthreads();
    for (int t = (int)threadIdx.x; t < NT * MT * 256; t += (int)blockDim.x) {
        const int nl = t % (NT * 16), ml = t / (NT * 16);
        const int n = n0 + nl, m = m0 + ml;
        if (n >= A.s.out || m >= A.s.rows) continue;
        const int tile = (nl >> 4) * MT + (ml >> 4), at = (tile * 64 + ((nl & 15) >> 2) * 16 + (ml & 15)) * 4 + (nl & 3);
        float z = 0.0f;
        for (int k = 0; k < waves; ++k) z += sums[k * NT * MT * 256 + at];
        if (bias) z += bias[n];
        store_as(out, (long long)m * A.s.out_row + n, A.s.out_type, activate_as(z, A.s.act));
    }
}

// Rows up to which x is quantised where it is multiplied; above, once for all workgroups, in the workspace.
constexpr int kDirectRows = 16;

template <class X, int NT, int MT>
hipError_t launch_direct(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias,
                         void* out, hipStream_t stream)
{
    Args A{s, (int)mxfp4_pieces(s.in), (s.out + 16 * NT - 1) / (16 * NT), (s.rows + 16 * MT - 1) / (16 * MT), false, {}};
    A.by_n = make_fast_div((uint32_t)A.n_tiles);
    if (s.x_type != kMxfp4)
        A.whole_runs = reinterpret_cast<uintptr_t>(x) % 16 == 0 && (s.rows == 1 || s.x_row * (long long)element_bytes(s.x_type) % 16 == 0);
    const int waves = std::min(NT * MT > 1 ? 4 : 16, A.pieces);
    hipLaunchKernelGGL((linear_direct_kernel<X, NT, MT>), dim3((unsigned)((long long)A.n_tiles * A.m_tiles)), dim3((unsigned)waves * 64),
                       (size_t)waves * NT * MT * 1024, stream, A, x, x_scales, w, w_scales, bias, out);
    return hipGetLastError();
}

}  // namespace

bool linear_fits(const LinearShape& s)
{
    return mxfp4_pieces(s.in) * 128 <= INT32_MAX - 128 && (long long)((s.rows + 15) / 16) * ((s.out + 15) / 16) <= kMostBlocks / 4 &&
           mxfp4_fits(Mxfp4Shape{s.rows, s.in, kF32, s.in});
}

namespace {

// The workspace: codes and scales of x where it is quantised beforehand, then the slices' sums.
struct Room {
    bool quantised_here;
    TilePlan plan;
    size_t scales_at, sums_at, bytes;
};
Room room_of(const LinearShape& s)
{
    Room r{};
    r.quantised_here = s.x_type != kMxfp4 && s.rows > kDirectRows;
    r.plan = tile_plan(s);
    const size_t blocks = r.quantised_here ? (size_t)s.rows * (size_t)mxfp4_pieces(s.in) * 4 : 0;
    r.scales_at = blocks * 16;
    r.sums_at = (r.scales_at + blocks + 15) / 16 * 16;
    r.bytes = r.sums_at + tile_workspace_bytes(s, r.plan);
    return r;
}

}  // namespace

size_t linear_workspace_bytes(const LinearShape& s) { return room_of(s).bytes; }

hipError_t launch_linear(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias,
                         void* out, void* workspace, hipStream_t stream)
{
    const Room room = room_of(s);
    uint8_t* work = static_cast<uint8_t*>(workspace);
    if (s.x_type != kMxfp4 && !room.quantised_here) {
        hipError_t e = hipSuccess;
        with_type(s.x_type, [&](auto t) { e = launch_direct<decltype(t), 1, 1>(s, x, nullptr, w, w_scales, bias, out, stream); });
        return e;
    }
    if (room.quantised_here) {
        const hipError_t e = launch_mxfp4_quantize(Mxfp4Shape{s.rows, s.in, s.x_type, s.x_row}, x, work, work + room.scales_at, stream);
        if (e != hipSuccess) return e;
        x = work;
        x_scales = work + room.scales_at;
    }
    if (room.plan.shape >= 0)
        return launch_tiles(s, room.plan, x, x_scales, w, w_scales, bias, out, reinterpret_cast<float*>(work + room.sums_at), stream);
    return launch_direct<Codes, 1, 1>(s, x, x_scales, w, w_scales, bias, out, stream);
}

}  // namespace patdnn
