// Linear layers on MXFP4 weights, many rows: tiles of BN outputs x BM rows, both operands through LDS.
//
// A workgroup walks k in stages of 128 values, 64 bytes a row.  Four stages are in LDS: while one is multiplied, up to three are on their
// way, straight from memory to LDS.  The scales come four stages at a time: each thread fetches the 16 bytes of one row and transposes
// them (bytes of one block position side by side), so that a lane's four scales are one 32-bit word, whose byte the
// matrix instruction selects.
//
// LDS holds 16-byte chunks; a chunk of a row stands at its place xor a number that depends on the row, chosen so that the
// eight lanes that are served in one cycle find theirs in different banks (8192^3: 305 us with a choice that suits sixteen, 290 so).  A wavefront
// reads the next stage's x and half of its weights while it multiplies.  The weights' rows of a wavefront are dealt to the instruction's
// rows so that a lane's results for four tiles are sixteen neighbouring outputs: whole runs are stored without going
// through LDS.
//
// 8192 x 8192 values, 8192 outputs, bf16: 290 us, 3.8 PFLOP/s.  The matrix cores are busy 48 % of the cycles, at 1.75 GHz of 2.4 (which points to the
// card's power, but was not shown: with fewer LDS conflicts the clock fell from 1.85 GHz, and all wavefronts together still waited as long).
#include "linear.hpp"

namespace patdnn {

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct Args {
    LinearShape s;
    int pieces;                                          // stages along k
    int tiles_n, tiles_m, slices, slice_pieces;          // slices of k, whole groups of four stages each
    bool wide_scales;                                    // rows of scales in whole aligned runs of 16 bytes
    FastDiv by_tiles, by_band, by_last;                  // tiles of a slice, of a band, rows of tiles of the last band
};
constexpr int kBand = 8;                                 // rows of tiles that are taken side by side
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Moves 16 (4) bytes a lane from memory to LDS: lane l's to lds + 16 l (4 l), the start from m0, which the compiler keeps for itself and finds as it
// was (the load reads it as it is issued).  Not waited for: s_waitcnt vmcnt counts it.
__device__ __forceinline__ void fetch16(intx4 buffer, uint32_t lds, uint32_t lane_offset, uint32_t offset)
{
    uint32_t kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds), "v"(lane_offset), "s"(buffer), "s"(offset) : "memory");
}
__device__ __forceinline__ void fetch4(intx4 buffer, uint32_t lds, uint32_t lane_offset, uint32_t offset)
{
    uint32_t kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds), "v"(lane_offset), "s"(buffer), "s"(offset) : "memory");
}
template <int OUTSTANDING>
__device__ __forceinline__ void wait_fetches()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OUTSTANDING) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ intx4 buffer_of(const void* p)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return intx4{uniform((int)(uint32_t)a), uniform((int)(uint32_t)(a >> 32) & 0xffff), -1, 0x00020000};
}

template <int STEP>
__device__ __forceinline__ floatx4 multiply_step(const uint4& a, const uint4& b, floatx4 c, uint32_t sa, uint32_t sb)
{
    const int32x8 va = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, vb = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(va, vb, c, 4, 4, STEP, (int)sa, STEP, (int)sb);
}

// BN x BM outputs x rows on WN x WM wavefronts.
template <int BN, int BM, int WN, int WM>
struct Tile {
    static constexpr int kWaves = WN * WM, kThreads = 64 * kWaves, kRows = BN + BM;
    static constexpr int kTN = BN / WN / 16, kTM = BM / WM / 16;         // matrix tiles of a wavefront
    static constexpr int kFetches = kRows / 16 / kWaves;                 // of 16 rows, per wavefront and stage
    static constexpr int kStage = kRows * 64, kStages = 4;
    static constexpr int kScales = kStages * kStage, kRaw = kScales + kRows * 16, kLds = kRaw + kRows * 16;
    static_assert(kTN % 4 == 0 && BN % 64 == 0 && BM % 64 == 0 && kRows % (16 * kWaves) == 0 && BN % (16 * kFetches) == 0 && kRows <= kThreads, "shape");
};

template <int BN, int BM, int WN, int WM>
__global__ __launch_bounds__(64 * WN * WM) void linear_tiles_kernel(Args A, const uint8_t* __restrict__ x, const uint8_t* __restrict__ x_scales,
                                                                    const uint8_t* __restrict__ w, const uint8_t* __restrict__ w_scales,
                                                                    const float* __restrict__ bias, void* __restrict__ out, float* __restrict__ partial)
{
    using S = Tile<BN, BM, WN, WM>;
    extern __shared__ char lds[];
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int r = lane & 15, kb = lane >> 4;
    // Which tile: workgroups go to the eight XCDs in turn, each takes a run of tiles, kBand rows of them at a time.
    int slice, tn, tm;
    {
        const int tiles = A.tiles_n * A.tiles_m, all = tiles * A.slices;
        const int xcd = (int)blockIdx.x & 7, q = all >> 3, rest = all & 7;
        int t = xcd * q + min(xcd, rest) + ((int)blockIdx.x >> 3);
        slice = uniform((int)fast_div((uint32_t)t, A.by_tiles));
        t -= slice * tiles;
        const int band = uniform((int)fast_div((uint32_t)t, A.by_band)), in_band = t - band * kBand * A.tiles_n, height = min(kBand, A.tiles_m - band * kBand);
        tn = uniform(height == kBand ? in_band / kBand : (int)fast_div((uint32_t)in_band, A.by_last));
        tm = band * kBand + in_band - tn * height;
    }
    const int n0 = tn * BN, m0 = tm * BM;
    const int first = slice * A.slice_pieces, pieces = min(A.slice_pieces, A.pieces - first);

    // What this wavefront fetches: rows past the end are those of the last one.
    const long long pitch = (long long)A.pieces * 64;
    const int fetch_row = wave * S::kFetches * 16;                       // its first row in LDS
    const bool of_w = fetch_row < BN;
    const intx4 data = buffer_of((of_w ? w + n0 * pitch : x + m0 * pitch) + first * 64);
    const int data_last = of_w ? A.s.out - 1 - n0 : A.s.rows - 1 - m0;
    uint32_t data_at[S::kFetches];
#pragma unroll
    for (int i = 0; i < S::kFetches; ++i) {
        const int sixteen = wave * S::kFetches + i, row = sixteen * 16 + (lane >> 2) - (of_w ? 0 : BN);
        const int swap = of_w ? (lane >> 3 & 1) + (sixteen & 1) * 2 : lane >> 3 & 3;
        data_at[i] = (uint32_t)(min(row, data_last) * pitch) + (uint32_t)(((lane & 3) ^ swap) * 16);
    }
    const int scale_row = wave * 64;                                     // 64 rows' scales, if that many are left
    const bool scales_of_w = scale_row < BN, fetches_scales = scale_row < S::kRows;
    const intx4 scales = buffer_of((scales_of_w ? w_scales + n0 * (pitch / 16) : x_scales + m0 * (pitch / 16)) + first * 4);
    const uint32_t scale_at = (uint32_t)(min(scale_row + lane - (scales_of_w ? 0 : BN), scales_of_w ? A.s.out - 1 - n0 : A.s.rows - 1 - m0) * (pitch / 16));
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

    auto fetch_stage = [&](int stage) {
#pragma unroll
        for (int i = 0; i < S::kFetches; ++i)
            fetch16(data, lds0 + (uint32_t)((stage & 3) * S::kStage + (fetch_row + i * 16) * 64), data_at[i], (uint32_t)stage * 64);
    };
    // Scales of stages 4 group ... 4 group + 3, of this wavefront's 64 rows: [row][stage] words, or [stage][row] where rows are not in runs.
    auto fetch_scales = [&](int group) {
        if (!fetches_scales) return;
        const uint32_t to = lds0 + (uint32_t)(S::kRaw + scale_row * 16);
        if (A.wide_scales) fetch16(scales, to, scale_at, (uint32_t)group * 16);
        else
#pragma unroll
            for (int p = 0; p < 4; ++p) fetch4(scales, to + (uint32_t)p * 256, scale_at, (uint32_t)min(group * 4 + p, pieces - 1) * 4);
    };
    auto turn_scales = [&]() {
        if (!fetches_scales) return;
        uint32_t d[4];
        if (A.wide_scales) {
            const uint4 v = *reinterpret_cast<const uint4*>(lds + S::kRaw + (scale_row + lane) * 16);
            d[0] = v.x, d[1] = v.y, d[2] = v.z, d[3] = v.w;
        } else {
#pragma unroll
            for (int p = 0; p < 4; ++p) d[p] = *reinterpret_cast<const uint32_t*>(lds + S::kRaw + scale_row * 16 + p * 256 + lane * 4);
        }
        const uint32_t a = __builtin_amdgcn_perm(d[1], d[0], 0x05010400), b = __builtin_amdgcn_perm(d[3], d[2], 0x05010400);
        const uint32_t c = __builtin_amdgcn_perm(d[1], d[0], 0x07030602), e = __builtin_amdgcn_perm(d[3], d[2], 0x07030602);
        const uint4 v = make_uint4(__builtin_amdgcn_perm(b, a, 0x05040100), __builtin_amdgcn_perm(b, a, 0x07060302),
                                   __builtin_amdgcn_perm(e, c, 0x05040100), __builtin_amdgcn_perm(e, c, 0x07060302));
        *reinterpret_cast<uint4*>(lds + S::kScales + (scale_row + lane) * 16) = v;
    };

    const int wn = wave % WN, wm = wave / WN;
    const int a_row = wn * (16 * S::kTN) + (r >> 2) * 16 + (r & 3), b_row = BN + wm * (16 * S::kTM) + r;
    const char* a_at = lds + a_row * 64 + (kb ^ (r >> 1 & 3)) * 16;
    const char* b_at = lds + b_row * 64 + (kb ^ (r >> 1 & 3)) * 16;
    const char* sa_at = lds + S::kScales + a_row * 16 + kb * 4;
    const char* sb_at = lds + S::kScales + b_row * 16 + kb * 4;

    floatx4 acc[S::kTN][S::kTM];
#pragma unroll
    for (int i = 0; i < S::kTN; ++i)
#pragma unroll
        for (int j = 0; j < S::kTM; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t sa[S::kTN], sb[S::kTM];
    // Registers of a stage: the rows of x and the first half of the weights' are read a stage ahead, the second half under the first one's products.
    constexpr int kHalf = S::kTN / 2;
    uint4 b[2][S::kTM], low[2][kHalf];
    auto read_a = [&](int step, int i) { return *reinterpret_cast<const uint4*>(a_at + step * S::kStage + ((i >> 2) * 64 + (i & 3) * 4) * 64); };
    auto read_ahead = [&](int step, int set) {
#pragma unroll
        for (int j = 0; j < S::kTM; ++j) b[set][j] = *reinterpret_cast<const uint4*>(b_at + step * S::kStage + j * 16 * 64);
#pragma unroll
        for (int i = 0; i < kHalf; ++i) low[set][i] = read_a(step, i);
    };

    fetch_scales(0);
    for (int t = 0; t < min(3, pieces); ++t) fetch_stage(t);
    if (pieces >= 3) wait_fetches<2 * S::kFetches>();
    else wait_fetches<0>();
    turn_scales();
    meet();
    read_ahead(0, 0);

    auto stage = [&](auto step, int t) {
        constexpr int STEP = decltype(step)::value, SET = STEP & 1;
        // the next stage has arrived once no more than the one after it is on its way
        if (t + 2 < pieces) wait_fetches<S::kFetches>();
        else wait_fetches<0>();
        meet();
        if (STEP == 0) {
#pragma unroll
            for (int i = 0; i < S::kTN; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(sa_at + ((i >> 2) * 64 + (i & 3) * 4) * 16);
#pragma unroll
            for (int j = 0; j < S::kTM; ++j) sb[j] = *reinterpret_cast<const uint32_t*>(sb_at + j * 16 * 16);
            if (t + 4 < pieces) fetch_scales((t >> 2) + 1);
        }
        if (t + 3 < pieces) fetch_stage(t + 3);
        uint4 high[kHalf];
#pragma unroll
        for (int i = 0; i < kHalf; ++i) high[i] = read_a(STEP, kHalf + i);
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
#pragma unroll
            for (int j = 0; j < S::kTM; ++j) acc[i][j] = multiply_step<STEP>(low[SET][i], b[SET][j], acc[i][j], sa[i], sb[j]);
        if (t + 1 < pieces) read_ahead((STEP + 1) & 3, SET ^ 1);
#pragma unroll
        for (int i = 0; i < kHalf; ++i)
#pragma unroll
            for (int j = 0; j < S::kTM; ++j)
                acc[kHalf + i][j] = multiply_step<STEP>(high[i], b[SET][j], acc[kHalf + i][j], sa[kHalf + i], sb[j]);
        // fetched three stages ago, so it is there; the last ones' words were read at their first stage
        if (STEP == 3 && t + 1 < pieces) turn_scales();
    };
    for (int t = 0; t < pieces; t += 4) {
        stage(Const<0>{}, t);
        if (t + 1 < pieces) stage(Const<1>{}, t + 1);
        if (t + 2 < pieces) stage(Const<2>{}, t + 2);
        if (t + 3 < pieces) stage(Const<3>{}, t + 3);
    }

    // A lane's results: row m0 + ... + r of x, for each four tiles sixteen neighbouring outputs.
    const int type = A.slices > 1 ? kF32 : A.s.out_type, act = A.slices > 1 ? kActNone : A.s.act;
    void* to = A.slices > 1 ? static_cast<void*>(partial + (long long)slice * A.s.rows * A.s.out) : out;
    const long long out_row = A.slices > 1 ? A.s.out : A.s.out_row;
#pragma unroll
    for (int g = 0; g < S::kTN / 4; ++g) {
        const int n = n0 + wn * (16 * S::kTN) + g * 64 + kb * 16;
        float add[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) add[i] = A.slices == 1 && bias && n + i < A.s.out ? bias[n + i] : 0.0f;
#pragma unroll
        for (int j = 0; j < S::kTM; ++j) {
            const int m = m0 + wm * (16 * S::kTM) + j * 16 + r;
            if (m >= A.s.rows || n >= A.s.out) continue;
            float z[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = acc[g * 4 + i / 4][j][i % 4] + add[i];
            finish_sixteen(z, act);
            store_results(to, m * out_row + n, type, A.s.out - n, z);
        }
    }
}

// Adds the slices up in their order; bias, activation, type.
__global__ __launch_bounds__(256) void linear_join_kernel(LinearShape s, int slices, const float* __restrict__ partial, const float* __restrict__ bias,
                                                          void* __restrict__ out, FastDiv by_out_blocks)
{
    const uint32_t m = fast_div(blockIdx.x, by_out_blocks);
    const int n = (int)(blockIdx.x - m * (uint32_t)((s.out + 255) / 256)) * 256 + (int)threadIdx.x;
    if (n >= s.out) return;
    const long long stride = (long long)s.rows * s.out;
    const float* p = partial + (long long)m * s.out + n;
    float z = 0.0f;
    for (int k = 0; k < slices; ++k) z += p[k * stride];
    if (bias) z += bias[n];
    store_as(out, (long long)m * s.out_row + n, s.out_type, activate_as(z, s.act));
}

template <int BN, int BM, int WN, int WM>
hipError_t launch_shape(Args A, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias, void* out,
                        float* partial, hipStream_t stream)
{
    using S = Tile<BN, BM, WN, WM>;
    A.tiles_n = (A.s.out + BN - 1) / BN;
    A.tiles_m = (A.s.rows + BM - 1) / BM;
    A.by_tiles = make_fast_div((uint32_t)(A.tiles_n * A.tiles_m));
    A.by_band = make_fast_div((uint32_t)(kBand * A.tiles_n));
    A.by_last = make_fast_div((uint32_t)(A.tiles_m % kBand ? A.tiles_m % kBand : kBand));
    static std::atomic<uint64_t> allowed{0};
    const hipError_t e = allow_big_lds(reinterpret_cast<const void*>(linear_tiles_kernel<BN, BM, WN, WM>), allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((linear_tiles_kernel<BN, BM, WN, WM>), dim3((unsigned)(A.tiles_n * A.tiles_m * A.slices)), dim3(S::kThreads), S::kLds, stream,
                       A, static_cast<const uint8_t*>(x), x_scales, w, w_scales, bias, out, partial);
    return hipGetLastError();
}

struct ShapeSize {
    int bn, bm;
};
constexpr ShapeSize kShapes[] = {{256, 256}, {128, 128}, {64, 64}};

}  // namespace

TilePlan tile_plan(const LinearShape& s)
{
    TilePlan p;
    const long long pieces = mxfp4_pieces(s.in);
    if (pieces * 64 * 256 > INT32_MAX) return p;         // offsets in a tile are 32-bit
    auto tiles = [&](int i) { return (long long)((s.out + kShapes[i].bn - 1) / kShapes[i].bn) * ((s.rows + kShapes[i].bm - 1) / kShapes[i].bm); };
    // The largest tiles that give every CU one (k = 4096, 4096 outputs: 512 rows 12.6, 16 and 32 us with tiles of 64, 128 and 256; 1024 rows 24, 18
    // and 33; 8192 rows of 8192 values and outputs take the largest).
    p.shape = tiles(0) >= 256 ? 0 : tiles(1) >= 256 ? 1 : 2;
    if (tiles(p.shape) > kMostBlocks / 4) p.shape = -1;
    // Few tiles are cut along k where a slice keeps 20 stages: adding slices up is a launch of its own (64 x 25088 -> 4096: 43 us in one, 19 in four
    // and 20 in eight slices; 256 x 4096 -> 4096 10 in one and 17 in two).
    else if (p.shape == 2) p.slices = (int)std::max<long long>(1, std::min<long long>(std::min<long long>(16, pieces / 20), 512 / tiles(2)));
    return p;
}

size_t tile_workspace_bytes(const LinearShape& s, const TilePlan& p)
{
    return p.shape >= 0 && p.slices > 1 ? (size_t)p.slices * (size_t)s.rows * (size_t)s.out * 4 : 0;
}

hipError_t launch_tiles(const LinearShape& s, const TilePlan& p, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales,
                        const float* bias, void* out, float* partial, hipStream_t stream)
{
    Args A{};
    A.s = s;
    A.pieces = (int)mxfp4_pieces(s.in);
    A.slice_pieces = (((A.pieces + 3) / 4 + p.slices - 1) / p.slices) * 4;
    A.slices = (A.pieces + A.slice_pieces - 1) / A.slice_pieces;
    A.wide_scales = A.pieces % 4 == 0 && (reinterpret_cast<uintptr_t>(x_scales) | reinterpret_cast<uintptr_t>(w_scales)) % 16 == 0;
    hipError_t e = p.shape == 0   ? launch_shape<256, 256, 2, 4>(A, x, x_scales, w, w_scales, bias, out, partial, stream)
                   : p.shape == 1 ? launch_shape<128, 128, 2, 2>(A, x, x_scales, w, w_scales, bias, out, partial, stream)
                                  : launch_shape<64, 64, 1, 4>(A, x, x_scales, w, w_scales, bias, out, partial, stream);
    if (e == hipSuccess && A.slices > 1) {
        const int across = (s.out + 255) / 256;
        hipLaunchKernelGGL(linear_join_kernel, dim3((unsigned)((long long)across * s.rows)), dim3(256), 0, stream, s, A.slices, partial, bias, out,
                           make_fast_div((uint32_t)across));
        e = hipGetLastError();
    }
    return e;
}

}  // namespace patdnn
