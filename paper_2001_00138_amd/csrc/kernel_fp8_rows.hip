// Products of fp8 codes, few rows of x: linear layers, and the gated pair of projections with its gradients.
//
// sum over k of x[m][k] w[n][k], 16 rows of 128 codes with 16 others at a time; sums are fp32.  There is time for the bfloat16 instructions, so sums have fp32's precision
// whatever the result's type (1 x 12288 -> 4096, three matrices in turn, which the last-level cache holds: 11.2 us with the fp8 instruction, 11.1 so).
// The weights are the first operand, so that a lane's four results are neighbours along n.
//
// The weights' bytes count, and every CU should have loads on their way all the time.  A workgroup takes 16 outputs (of both projections); its wavefronts take
// pieces of 128 values of k in turn, straight from memory to registers, and add their sums up in LDS, in their order.
//
// From memory (twenty matrices in turn): 1 x 12288 -> 4096 12.1 us, 4.2 TB/s of weights, eight rows 14.9; gated 1 x 4096 -> 12288 21.1 us, 4.8 TB/s, codes 23.1.
#include "fp8_products.hpp"

namespace patdnn {

namespace {

constexpr int kRows = 16;                                // rows of x a workgroup
constexpr int kAhead = 2;                                // pieces of weights that a wavefront asks for together (one to four are alike)

struct Args {
    ProductShape s;
    ProductTensors t;
    int pieces, row_tiles;                               // of 128 along k; of kRows rows of x
    FastDiv by_tiles;
};

template <int KIND>
__global__ __launch_bounds__(1024) void product_rows_kernel(Args A)
{
    constexpr int kSides = KIND == kLinear ? 1 : 2;
    extern __shared__ float sums[];                      // [wavefront][projection][lane][4]
    // (the wavefront's number in a scalar register: a matrix instruction in a branch that only masks lanes out would be executed)
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const int r = lane & 15, kb = lane >> 4;
    const uint32_t block = fast_div(blockIdx.x, A.by_tiles), m_tile = blockIdx.x - block * (uint32_t)A.row_tiles;
    const int n0 = (int)block * 16, m0 = (int)m_tile * kRows, rows = min(kRows, A.s.rows - m0);
    // rows past the end are read as the last one, and their results dropped
    const long long n_row = min(n0 + r, A.s.out - 1), m_row = m0 + min(r, rows - 1);
    const long long n_at = n_row * A.pieces * 128 + kb * 16, ns_at = (A.s.squares ? n_row >> 7 : n_row) * A.pieces;
    const uint8_t* w_at[2] = {A.t.w + n_at, A.t.w2 + n_at};
    const uint8_t* ws_at[2] = {A.t.w_scales + ns_at, A.t.w2_scales + ns_at};
    const uint8_t* x_at = A.t.x + m_row * A.pieces * 128 + kb * 16;
    const uint8_t* xs_at = A.t.x_scales + m_row * A.pieces;

    auto load = [](const uint8_t* p) { return both_halves(*reinterpret_cast<const uint4*>(p), *reinterpret_cast<const uint4*>(p + 64)); };
    floatx4 acc[kSides];
#pragma unroll
    for (int k = 0; k < kSides; ++k) acc[k] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int first = wave; first < A.pieces; first += kAhead * waves) {
        int32x8 a[kAhead][kSides], b[kAhead];
        uint32_t sa[kAhead][kSides], sb[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int piece = min(first + i * waves, A.pieces - 1);      // past the end: the last one, which is not multiplied
#pragma unroll
            for (int k = 0; k < kSides; ++k) {
                a[i][k] = load(w_at[k] + piece * 128);
                sa[i][k] = ws_at[k][piece];
            }
            b[i] = load(x_at + piece * 128);
            sb[i] = xs_at[piece];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (first + i * waves >= A.pieces) break;
#pragma unroll
            for (int k = 0; k < kSides; ++k) acc[k] = multiply_wide(fp8_widen(a[i][k], sa[i][k] << 23), fp8_widen(b[i], sb[i] << 23), acc[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kSides; ++k) *reinterpret_cast<floatx4*>(sums + ((wave * kSides + k) * 64 + lane) * 4) = acc[k];
    __syncthreads();
    for (int t = (int)threadIdx.x; t < rows * 16; t += (int)blockDim.x) {
        const int nl = t & 15, ml = t >> 4, n = n0 + nl;
        if (n >= A.s.out) continue;
        const int at = ((nl >> 2) * 16 + ml) * 4 + (nl & 3);
        float z[2] = {0.0f, 0.0f};
        for (int i = 0; i < waves; ++i)
#pragma unroll
            for (int k = 0; k < kSides; ++k) z[k] += sums[(i * kSides + k) * 256 + at];
        finish_one<KIND>(A.s, A.t, m0 + ml, n, z[0], z[1]);
    }
}

long long workgroups_of(const ProductShape& s) { return (s.rows + kRows - 1ll) / kRows * ((s.out + 15ll) / 16); }

template <int KIND>
hipError_t launch_rows(const ProductShape& s, const ProductTensors& t, hipStream_t stream)
{
    Args A{s, t, (int)fp8_pieces(s.in), (s.rows + kRows - 1) / kRows, {}};
    A.by_tiles = make_fast_div((uint32_t)A.row_tiles);
    const int waves = std::min(16, A.pieces);
    hipLaunchKernelGGL((product_rows_kernel<KIND>), dim3((unsigned)workgroups_of(s)), dim3((unsigned)waves * 64),
                       (size_t)waves * (KIND == kLinear ? 1024 : 2048), stream, A);
    return hipGetLastError();
}

// Whether the call is for this kernel and not for tiles: up to 16 rows, but linear layers on the fp8 instruction's sums from 1.25 * 2^30 products on, with nine rows or more: there tiles, which
// read x less often, are faster (us here and in tiles, weights from memory: 16 rows 8192 -> 8192 23.6 and 25.1, 16384 -> 8192 44.3 and 40.6; twelve 22.1 and 25.0, 41.6 and 39.8; nine rows
// 16384 -> 8192 37.6 and 43.1, 16384 -> 16384 70.7 and 69.6).  The gated pair, whose tiles of 64 rows of x multiply twice as much for nothing, has no such size (16 rows 4096 -> 6144 17.5 and 20.8,
// codes 19.9 and 19.5; 8192 -> 16384 63 and 61, codes 65.9 and 66.8).
bool by_rows(const ProductShape& s)
{
    if (!product_tiles_fit(s)) return true;
    return s.rows <= 8 || (s.rows <= kRows && (s.kind != kLinear || s.out_type == kF32 || (long long)s.in * s.out * s.rows < 5ll << 28));
}

// The workspace: slices' sums of the tiles; h in fp32, where codes are made of it by a launch of their own.
bool codes_apart(const ProductShape& s) { return s.kind == kGated && s.out_type == kFp8 && by_rows(s); }

}  // namespace

bool product_fits(const ProductShape& s)
{
    return fp8_pieces(s.in) * 128 <= INT32_MAX - 128 && s.rows <= INT32_MAX - 256 && ceil_div(s.out, 16) <= kMostBlocks / 4 &&
           (!by_rows(s) || workgroups_of(s) <= kMostBlocks / 4) &&
           (!codes_apart(s) || fp8_fits(Fp8Shape{s.rows, s.out, kF32, false, false, s.out}, true));
}

size_t product_workspace_bytes(const ProductShape& s)
{
    return !by_rows(s) ? product_tiles_workspace_bytes(s) : codes_apart(s) ? (size_t)s.rows * (size_t)s.out * 4 : 0;
}

hipError_t launch_product(const ProductShape& shape, const ProductTensors& tensors, void* workspace, hipStream_t stream)
{
    if (!by_rows(shape)) return launch_product_tiles(shape, tensors, static_cast<float*>(workspace), stream);
    ProductShape s = shape;
    ProductTensors t = tensors;
    const bool apart = codes_apart(s);
    if (apart) {
        s.out_type = kF32;
        s.out_row = s.out;
        t.out = workspace;
    }
    const hipError_t e = s.kind == kLinear  ? launch_rows<kLinear>(s, t, stream)
                         : s.kind == kGated ? launch_rows<kGated>(s, t, stream)
                                            : launch_rows<kGatedBackward>(s, t, stream);
    if (e != hipSuccess || !apart) return e;
    return launch_fp8_quantize(Fp8Shape{s.rows, s.out, kF32, false, false, s.out}, workspace, static_cast<uint8_t*>(tensors.out), tensors.out_scales, stream);
}

}  // namespace patdnn
