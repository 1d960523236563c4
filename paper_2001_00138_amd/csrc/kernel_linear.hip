// Linear layers on MXFP4 weights, on the scaled matrix instructions.
//
// out[m][n] = act(bias[n] + sum over k of x[m][k] w[n][k]).  The instruction multiplies 16 rows of 128 codes with 16
// others and applies the scales of their blocks of 32 itself; a lane holds one block of one row, 16 bytes, which is how
// rows lie in memory.  The weights are the instruction's first operand, so that a lane's four results are
// neighbours along n.  Sums are fp32.
//
// Few rows, or few outputs: the weights' bytes count, and every CU should have loads on their way all the time.  A workgroup takes 16 outputs; its wavefronts
// take pieces of 128 values of k in turn and add their sums up in LDS, in their order.  A wavefront asks for its first weights, then x is
// quantised into LDS by all of them (every workgroup does that for itself: there is no launch before), and then weights stream through registers.
//
// Two pieces at a time: the sixteen wavefronts of a workgroup, and with few registers two workgroups a CU, have enough loads on their way, and asking
// for more before x is there only delays it and asks for the last pieces again (fp16, us with 2, 4 and 8 pieces: 1 x 25088 -> 4096 13.5, 14.1 and 16.2;
// 4 x 4096 -> 4096 5.3, 7.0 and 10.5; 1 x 8192 -> 8192 12.5, 10.7 and 19.0; 1 x 25088 -> 16384 48, 51 and 63; with eight wavefronts 14.7, 6.0, 11.9
// and 52 at 2 pieces).  1 x 25088 -> 4096: 13.4 us, 4.1 TB/s of weights; the launch, the first load's latency and the joining of the sums are not
// hidden by anything.
#include <type_traits>

#include "linear.hpp"

namespace patdnn {

namespace {

struct Codes {};                                         // x is MXFP4 already

constexpr int kRows = 16;                                // most rows of x here: the matrix instruction's
constexpr int kAhead = 2;                                // pieces of weights that a wavefront asks for together
constexpr int kRowsLds = 128 * 1024;                     // most bytes of x in LDS

struct Args {
    LinearShape s;
    int pieces, row_tiles;                               // of 128 along k; of kRows rows of x
    FastDiv by_tiles, by_lanes;                          // row_tiles; runs of eight values in a row of x
};

template <class X>
__global__ __launch_bounds__(1024) void linear_rows_kernel(Args A, const void* __restrict__ x, const uint8_t* __restrict__ x_scales,
                                                           const uint8_t* __restrict__ w, const uint8_t* __restrict__ w_scales,
                                                           const float* __restrict__ bias, void* __restrict__ out)
{
    constexpr bool kStored = std::is_same_v<X, Codes>;
    extern __shared__ char lds[];                        // sums [wavefront][lane][4]; then x: codes [row][pieces * 64 + 16] (rows in other banks), scales [row][pieces * 4]
    // (the wavefront's number in a scalar register: a matrix instruction in a branch that only masks lanes out would be executed)
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const int r = lane & 15, kb = lane >> 4;
    const uint32_t block = fast_div(blockIdx.x, A.by_tiles), m_tile = blockIdx.x - block * (uint32_t)A.row_tiles;
    const int n0 = (int)block * 16, m0 = (int)m_tile * kRows, rows = min(kRows, A.s.rows - m0);
    // rows past the end are read as the last one, and their results dropped
    const long long n_row = (long long)min(n0 + r, A.s.out - 1) * A.pieces, m_row = (long long)(m0 + min(r, rows - 1)) * A.pieces;
    const uint8_t* w_at = w + n_row * 64 + kb * 16;
    const uint8_t* ws_at = w_scales + n_row * 4 + kb;
    const uint8_t* x_at = static_cast<const uint8_t*>(x) + m_row * 64 + kb * 16;       // of codes
    const uint8_t* xs_at = x_scales + m_row * 4 + kb;

    uint4 a[kAhead], b[kStored ? kAhead : 1];
    uint32_t sa[kAhead], sb[kStored ? kAhead : 1];
    auto ask = [&](int first) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int piece = min(first + i * waves, A.pieces - 1);      // past the end: the last one, which is not multiplied
            a[i] = *reinterpret_cast<const uint4*>(w_at + piece * 64);
            sa[i] = ws_at[piece * 4];
            if constexpr (kStored) {
                b[i] = *reinterpret_cast<const uint4*>(x_at + piece * 64);
                sb[i] = xs_at[piece * 4];
            }
        }
    };
    ask(wave);
    const int pitch = A.pieces * 64 + 16;
    char* const s_codes = lds + waves * 1024;
    uint8_t* const s_scales = reinterpret_cast<uint8_t*>(s_codes) + rows * pitch;
    if constexpr (!kStored) {
        // a block's four lanes are neighbours; rows are multiples of 16 runs of eight values long
        const int runs = A.pieces * 16;
        for (int i = (int)threadIdx.x; i < (rows * runs + 63) / 64 * 64; i += (int)blockDim.x) {
            const int row = (int)fast_div((uint32_t)i, A.by_lanes), run = i - row * runs;
            Pack<X, 8> v;
            uint32_t top = 0;
            if (row < rows) {
                v = load8(static_cast<const X*>(x) + (long long)(m0 + row) * A.s.x_row + run * 8, A.s.in - run * 8);
                top = largest(v);
            }
            top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
            top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
            if (row < rows) {
                const uint32_t byte = scale_byte(top);
                *reinterpret_cast<uint32_t*>(s_codes + row * pitch + run * 4) = byte == kNanScale ? 0u : encode8(v, scale_of(byte));
                if (run % 4 == 0) s_scales[i / 4] = (uint8_t)byte;
            }
        }
        __syncthreads();
    }
    const int x_row = min(r, rows - 1);
    const char* s_code_at = s_codes + x_row * pitch + kb * 16;
    const uint8_t* s_scale_at = s_scales + x_row * A.pieces * 4 + kb;
    floatx4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int first = wave; first < A.pieces; first += kAhead * waves) {
        if (first != wave) ask(first);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int piece = first + i * waves;
            if (piece >= A.pieces) break;
            if constexpr (kStored) acc = multiply(a[i], b[i], acc, sa[i], sb[i]);
            else acc = multiply(a[i], *reinterpret_cast<const uint4*>(s_code_at + piece * 64), acc, sa[i], s_scale_at[piece * 4]);
        }
    }
    float* sums = reinterpret_cast<float*>(lds);
    *reinterpret_cast<floatx4*>(sums + (wave * 64 + lane) * 4) = acc;
    __syncthreads();
    for (int t = (int)threadIdx.x; t < rows * 16; t += (int)blockDim.x) {
        const int nl = t & 15, ml = t >> 4, n = n0 + nl;
        if (n >= A.s.out) continue;
        const int at = ((nl >> 2) * 16 + ml) * 4 + (nl & 3);
        float z = 0.0f;
        for (int k = 0; k < waves; ++k) z += sums[k * 256 + at];
        if (bias) z += bias[n];
        store_as(out, (long long)(m0 + ml) * A.s.out_row + n, A.s.out_type, activate_as(z, A.s.act));
    }
}

template <class X>
hipError_t launch_rows(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias,
                       void* out, hipStream_t stream)
{
    Args A{s, (int)mxfp4_pieces(s.in), (s.rows + kRows - 1) / kRows, {}, {}};
    A.by_tiles = make_fast_div((uint32_t)A.row_tiles);
    A.by_lanes = make_fast_div((uint32_t)A.pieces * 16);
    size_t x_bytes = 0;
    if constexpr (!std::is_same_v<X, Codes>) x_bytes = (size_t)std::min(s.rows, kRows) * (A.pieces * 68 + 16);
    const int waves = std::min(16, A.pieces);
    const size_t lds = (size_t)waves * 1024 + x_bytes;
    static std::atomic<uint64_t> allowed{0};
    if (lds > 64 * 1024)
        if (const hipError_t e = allow_big_lds(reinterpret_cast<const void*>(linear_rows_kernel<X>), allowed); e != hipSuccess) return e;
    hipLaunchKernelGGL((linear_rows_kernel<X>), dim3((unsigned)((long long)((s.out + 15) / 16) * A.row_tiles)), dim3((unsigned)waves * 64), lds, stream,
                       A, x, x_scales, w, w_scales, bias, out);
    return hipGetLastError();
}

long long workgroups_of(const LinearShape& s) { return (s.rows + kRows - 1ll) / kRows * ((s.out + 15ll) / 16); }

// Whether codes are multiplied here and not in tiles: up to four rows, and while a CU has at most one workgroup and k is no longer than 64 pieces (codes
// -> fp16, us here and in tiles: 16 x 4096 -> 4096 6.2 and 9.1, 48 x 4096 -> 1000 6.0 and 9.0, 256 x 4100 -> 256 4.5 and 9.5, 3000 x 8192 -> 16 9.1 and
// 10.1; above: 77 x 2048 -> 1000 9.2 and 6.2, 5 x 2048 -> 6000 7.1 and 5.6, 16 x 12288 -> 4096 12.9 and 12.1, 8 x 25088 -> 1000 16.5 and 13.4).
bool by_rows(const LinearShape& s) { return s.rows <= 4 || (workgroups_of(s) <= 256 && mxfp4_pieces(s.in) <= 64); }

// Whether x is quantised where it is multiplied, by every workgroup for itself.  That is less than a launch up to some 400 pieces (fp16, us in one
// launch and in two: 12 x 4096 -> 1000 7.3 and 7.7, 16 x 4096 8.5 and 8.0; 128 x 2048 -> 500 6.4 and 8.0; 2 x 25088 -> 4096 15.2 and 16.3, 4 x 25088 19.2
// and 17.2); from five rows on also while a CU has at most one workgroup or all of them together have few weights to read (63 x 512 -> 4096 5.7 and 5.8,
// 77 x 1024 -> 1000 6.1 and 7.3, 32 x 1024 -> 4096 6.2 and 6.5; 48 x 1024 -> 4096 8.0 and 6.6, 5 x 1024 -> 16384 7.1 and 6.8).  One row always is:
// 1 x 25088 -> 4096 13.3 and 15.3.
bool in_one_launch(const LinearShape& s)
{
    if (s.x_type == kMxfp4) return false;
    const long long pieces = mxfp4_pieces(s.in), rows = std::min(s.rows, kRows);
    if (rows * (pieces * 68 + 16) > kRowsLds || (s.rows > 1 && rows * pieces > 400)) return false;
    return s.rows <= 4 || workgroups_of(s) <= 256 || workgroups_of(s) * pieces <= 4096;
}

}  // namespace

namespace {

// The workspace: codes and scales of x where it is quantised in a launch of its own, then the slices' sums.
struct Room {
    bool quantised_here;
    TilePlan plan;
    size_t scales_at, sums_at, bytes;
};
Room room_of(const LinearShape& s)
{
    Room r{};
    if (short_fits(s)) return r;
    r.quantised_here = s.x_type != kMxfp4 && !in_one_launch(s);
    if (!by_rows(s)) r.plan = tile_plan(s);
    // (more than kRows rows: room for the codes whichever way the call takes, so that a change of that choice is no caller's concern)
    const size_t blocks = r.quantised_here || (s.x_type != kMxfp4 && s.rows > kRows) ? (size_t)s.rows * (size_t)mxfp4_pieces(s.in) * 4 : 0;
    r.scales_at = blocks * 16;
    r.sums_at = (r.scales_at + blocks + 15) / 16 * 16;
    r.bytes = r.sums_at + tile_workspace_bytes(s, r.plan);
    return r;
}

}  // namespace

// Outputs that one row can have (a workgroup for 16 of them), whatever the rows; rows that 32-bit sums of a tile's end do not pass (so the kernel of short
// rows has fewer than 2^24 workgroups, of 128 rows and more); and the grids of what is launched.
bool linear_fits(const LinearShape& s)
{
    if (mxfp4_pieces(s.in) * 128 > INT32_MAX - 128 || ceil_div(s.out, 16) > kMostBlocks / 4 || s.rows > INT32_MAX - 256) return false;
    if (short_fits(s)) return true;
    const Room room = room_of(s);
    return (!room.quantised_here || mxfp4_fits(Mxfp4Shape{s.rows, s.in, s.x_type, s.x_row})) &&
           (room.plan.shape >= 0 || workgroups_of(s) <= kMostBlocks / 4);
}

size_t linear_workspace_bytes(const LinearShape& s) { return room_of(s).bytes; }

hipError_t launch_linear(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias,
                         void* out, void* workspace, hipStream_t stream)
{
    if (short_fits(s)) return launch_short(s, x, x_scales, w, w_scales, bias, out, stream);
    const Room room = room_of(s);
    uint8_t* work = static_cast<uint8_t*>(workspace);
    if (s.x_type != kMxfp4 && !room.quantised_here) {
        hipError_t e = hipSuccess;
        with_type(s.x_type, [&](auto t) { e = launch_rows<decltype(t)>(s, x, nullptr, w, w_scales, bias, out, stream); });
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
    return launch_rows<Codes>(s, x, x_scales, w, w_scales, bias, out, stream);
}

}  // namespace patdnn
