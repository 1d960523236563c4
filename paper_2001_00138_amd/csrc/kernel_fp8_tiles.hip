// Products of fp8 codes, many rows of x: tiles of BN of the weights' rows x BM rows of x, both operands through LDS.
//
// A workgroup walks k in stages of 128 codes.  NS stages are in LDS, and arrive straight from memory.  A wavefront holds a stage's operands in two halves each;
// it multiplies them in an order that turns round from stage to stage, so that each half is read from LDS while another two are multiplied
// and none is held twice.  Half-way through a stage everything of it is in registers: there the workgroup meets, the stage's place in LDS is
// given to the stage NS ahead, and reading the next one begins under the second half of the products.
//
// LDS holds 16-byte chunks, eight a row; a chunk of a row stands at its place xor a number that depends on the row, chosen so that the eight lanes
// that are served in one cycle find theirs in different banks.  The weights' rows of a wavefront are dealt to the instruction's rows so that a lane's
// results for four tiles are sixteen neighbouring outputs.  For the gated pair, each 64 rows of the first projection's are followed by the same 64 of the second's,
// so that one lane has both sums of an output, and a workgroup whose result is codes all 128 outputs that share a scale.
//
// 8192 x 8192 values, 8192 outputs, bf16: 424 to 515 us by the card's clock, 465 (2.36 PFLOP/s) in the middle of a series; the matrix cores are busy 64 % of its 818 thousand cycles.
// (In the shortest series 407, and 335 there without the fetches.)  fp32: 890 to 910 us.  Gated, 8192 x 4096 -> 12288: codes 680 to 745 us, bf16 710, fp32 1490; its gradients in bf16 785 to 830.
#include "fp8_products.hpp"

namespace patdnn {

namespace {

typedef int intx4 __attribute__((ext_vector_type(4)));

struct Args {
    ProductShape s;
    ProductTensors t;
    float* partial;                                      // [slice][row][sums], of calls in slices
    int pieces;                                          // stages
    int tiles_n, tiles_m, slices, slice_pieces;          // slices of k
    FastDiv by_tiles, by_band, by_last;                  // tiles of a slice, of a band, rows of tiles of the last band
};
constexpr int kGatedCodes = 3;                          // kGated with codes as its result
constexpr int kBand = 8;                                 // rows of tiles that are taken side by side
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Moves 16 bytes a lane from memory to LDS: lane l's to lds + 16 l, the start from m0, which the compiler keeps for itself and finds as it
// was (the load reads it as it is issued).  Not waited for: s_waitcnt vmcnt counts it.
__device__ __forceinline__ void fetch16(intx4 buffer, uint32_t lds, uint32_t lane_offset, uint32_t offset)
{
    uint32_t kept;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(kept) : "s"(lds), "v"(lane_offset), "s"(buffer), "s"(offset) : "memory");
}
template <int OUTSTANDING>
__device__ __forceinline__ void wait_fetches()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(OUTSTANDING) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Product of 16 rows of 128 codes with 16 others, added to c, by the fp8 instruction: operands and sums as multiply_wide has them, the scales are bytes BYTE_A and BYTE_B of the operands.
//
// The instruction adds eight neighbouring products in a fixed width: below 2^-13 of the power of two of the largest they are cut off (found by
// putting single products beside a large one; so do its other shapes and the unscaled ones).  Sums of normal values are off by 1.5e-5 of their
// size then, a thirtieth of half a spacing of binary16 (2^-11) and less of the others' but 250 times fp32's, so results in fp32 are not made by it.
//
// The sums are kept where they are, in the accumulation registers: the compiler would give them new ones with every product, and move them back in
// every round, for which there is no room.  What it does not see here it need not see: the operands were waited for before; a result is read by another
// product no sooner than three behind it, and by other instructions only after let_settle().  (The wait is for scales that a vector instruction has just moved.)
template <int BYTE_A, int BYTE_B>
__device__ __forceinline__ void multiply_in_place(const int32x8& a, const int32x8& b, floatx4& c, uint32_t sa, uint32_t sb)
{
    asm("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
        : "+a"(c) : "v"(a), "v"(b), "v"(sa), "v"(sb), "n"(BYTE_A & 1), "n"(BYTE_B & 1), "n"(BYTE_A >> 1), "n"(BYTE_B >> 1));
}
// (the bytes' places are constants once the loops around are unrolled)
__device__ __forceinline__ void multiply_tile(const int32x8& a, const int32x8& b, floatx4& c, uint32_t sa, uint32_t sb, int byte_a, int byte_b)
{
    auto with_b = [&](auto i, auto j) { multiply_in_place<decltype(i)::value, decltype(j)::value>(a, b, c, sa, sb); };
    auto with_a = [&](auto i) { byte_b == 0 ? with_b(i, Const<0>{}) : byte_b == 1 ? with_b(i, Const<1>{}) : byte_b == 2 ? with_b(i, Const<2>{}) : with_b(i, Const<3>{}); };
    byte_a == 0 ? with_a(Const<0>{}) : byte_a == 1 ? with_a(Const<1>{}) : byte_a == 2 ? with_a(Const<2>{}) : with_a(Const<3>{});
}
// The last products' results may be read 20 wait states after them; these are 24.
template <int N, int M>
__device__ __forceinline__ void let_settle(floatx4 (&acc)[N][M])
{
    asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < M; ++j) asm volatile("" : "+a"(acc[i][j]));
}

// BN x BM rows of the weights and of x, on WN x WM wavefronts, NS stages in LDS.
template <int BN, int BM, int WN, int WM, int NS>
struct Tile {
    static constexpr int kWaves = WN * WM, kThreads = 64 * kWaves, kRows = BN + BM;
    static constexpr int kTN = BN / WN / 16, kTM = BM / WM / 16;         // matrix tiles of a wavefront
    static constexpr int kHN = kTN / 2, kHM = kTM > 1 ? kTM / 2 : 1, kPart = kHN / 2;    // of a half, of a part of one
    static constexpr int kFetches = kRows / 8 / kWaves;                  // of 8 rows, per wavefront and stage
    static constexpr int kWords = (kRows + kThreads - 1) / kThreads;     // of scales, per thread
    // Scales of a stage: a word for a lane's four neighbouring tiles of the weights, one for as many of x.
    static constexpr int kGroupsN = kTN / 4, kGroupsM = (kTM + 3) / 4, kScaleStage = BN + WM * kGroupsM * 64;
    static constexpr int kStage = kRows * 128, kScales = NS * kStage, kLds = kScales + 8 * kScaleStage;
    static_assert(kTN % 4 == 0 && (kTM == 1 || kTM % 2 == 0) && kRows % (8 * kWaves) == 0 && BN % 64 == 0 && BM % 16 == 0, "shape");
    static_assert(NS == 2 || NS == 4, "stages by their place in a group of four");
};

// SLICED: sums of a slice of k go to A.partial.  D: dh's type.  (What is decided here and not in the kernel is what would cost it registers.)
// WAVES: of a SIMD, for which the compiler has to leave registers.
template <int KIND, bool EXACT, int BN, int BM, int WN, int WM, int NS, int WAVES, bool SLICED, class D>
__global__ __launch_bounds__(64 * WN * WM, WAVES) void product_tiles_kernel(Args A)
{
    using S = Tile<BN, BM, WN, WM, NS>;
    constexpr bool kTwo = KIND != kLinear;
    constexpr int kOut = kTwo ? BN / 2 : BN;                             // outputs of a workgroup
    static_assert(!kTwo || S::kTN == 8, "a wavefront has 64 rows of each projection");
    extern __shared__ char lds[];
    const int lane = (int)threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int r = lane & 15, kb = lane >> 4;
    // Which tile: workgroups go to the eight XCDs in turn, each takes a run of tiles, kBand rows of them at a time.
    int slice = 0, tn, tm;
    {
        const int tiles = A.tiles_n * A.tiles_m, all = SLICED ? tiles * A.slices : tiles, xcd = (int)blockIdx.x & 7, q = all >> 3, rest = all & 7;
        int t = xcd * q + min(xcd, rest) + ((int)blockIdx.x >> 3);
        if (SLICED) {
            slice = uniform((int)fast_div((uint32_t)t, A.by_tiles));
            t -= slice * tiles;
        }
        const int band = uniform((int)fast_div((uint32_t)t, A.by_band)), in_band = t - band * kBand * A.tiles_n, height = min(kBand, A.tiles_m - band * kBand);
        tn = uniform(height == kBand ? in_band / kBand : (int)fast_div((uint32_t)in_band, A.by_last));
        tm = band * kBand + in_band - tn * height;
    }
    const int n0 = tn * kOut, m0 = tm * BM, first_piece = SLICED ? slice * A.slice_pieces : 0;
    const int pieces = SLICED ? min(A.slice_pieces, A.pieces - first_piece) : A.pieces;
    const long long pitch = (long long)A.pieces * 128;

    // A row of LDS: whose it is (0, 1: of the weights; 2: of x), and which row behind the tile's first.
    auto side_of = [&](int row) { return row >= BN ? 2 : kTwo ? row >> 6 & 1 : 0; };
    auto row_of = [&](int row) { return row >= BN ? row - BN : kTwo ? (row >> 7) * 64 + (row & 63) : row; };
    const int w_last = A.s.out - 1 - n0, x_last = A.s.rows - 1 - m0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    // The wavefronts fetch eight rows each, of one side, and so on.  What lies past a side's end the buffer's own check keeps from being read (it compares a lane's part of the
    // offset with what the scalar part leaves, which is never past the last row); what stands in LDS there reaches only results that are dropped.
    constexpr int kTogether = 8 * S::kWaves;
    static_assert(BN % kTogether == 0 && BM % kTogether == 0 && (!kTwo || 64 % kTogether == 0), "rows that are fetched together are of one side");
    auto buffer_of_side = [&](int side) {
        const uint64_t p = (uint64_t)((side == 2 ? A.t.x + m0 * pitch : (side == 1 ? A.t.w2 : A.t.w) + n0 * pitch) + first_piece * 128);
        const long long bytes = ((long long)(side == 2 ? x_last : w_last) + 1) * pitch - first_piece * 128;
        return intx4{uniform((int)(uint32_t)p), uniform((int)(p >> 32 & 0xffff)), uniform((int)(uint32_t)min(bytes, 0xffffffffll)), 0x00020000};
    };
    const intx4 from_w = buffer_of_side(0), from_w2 = buffer_of_side(kTwo ? 1 : 0), from_x = buffer_of_side(2);
    // a lane's row of the eight, and its chunk's place
    const int w_at = (lane >> 3) * (int)pitch + ((lane & 7) ^ ((lane >> 3 & 3) | (wave >> 1 & 1) << 2)) * 16;
    const int x_at = (lane >> 3) * (int)pitch + ((lane & 7) ^ (lane >> 3)) * 16;
    auto fetch = [&](int i, int t) {
        const int side = side_of(i * kTogether), first = i * kTogether + wave * 8, row = min(row_of(i * kTogether) + wave * 8, side == 2 ? x_last : w_last);
        fetch16(side == 2 ? from_x : side == 1 ? from_w2 : from_w, lds0 + (uint32_t)((t & (NS - 1)) * S::kStage + first * 128), (uint32_t)(side == 2 ? x_at : w_at),
                (uint32_t)(row * (int)pitch + min(t, pieces - 1) * 128));
    };
    // Scales of a group of four stages, four bytes for each row of LDS: in a register for three stages, then in LDS, where two groups have a place.
    // There a word is what a lane needs for four tiles: the matrix instruction selects its byte.
    const uint8_t* scales_at[S::kWords];
#pragma unroll
    for (int k = 0; k < S::kWords; ++k) {
        const int row = min(k * S::kThreads + (int)threadIdx.x, S::kRows - 1), side = side_of(row);
        const uint8_t* from = side == 2 ? A.t.x_scales : kTwo && side == 1 ? A.t.w2_scales : A.t.w_scales;
        const int at = side == 2 ? m0 + min(row_of(row), x_last) : n0 + min(row_of(row), w_last);
        scales_at[k] = from + (long long)(side != 2 && A.s.squares ? at >> 7 : at) * A.pieces + first_piece;
    }
    uint32_t words[S::kWords];
    // (four bytes that lie in the row: in its last group those before it come along, and are shifted out)
    auto fetch_scales = [&](int t) {
        const int at = min(t, pieces - 4);
#pragma unroll
        for (int k = 0; k < S::kWords; ++k) words[k] = __builtin_bit_cast(uint32_t, load_pack<uint8_t, 4>(scales_at[k] + at));
    };
    auto put_scales = [&](int group, int shift) {
#pragma unroll
        for (int k = 0; k < S::kWords; ++k) {
            const int row = min(k * S::kThreads + (int)threadIdx.x, S::kRows - 1), m = row - BN;
            const int at = row < BN ? (row & ~63) + ((row >> 4 & 3) * 4 + (row & 3)) * 4 + (row >> 2 & 3)
                                    : BN + (m / (16 * S::kTM) * S::kGroupsM + (m / 16 % S::kTM) / 4) * 64 + (m & 15) * 4 + (m / 16 % S::kTM) % 4;
#pragma unroll
            for (int i = 0; i < 4; ++i) lds[S::kScales + ((group & 1) * 4 + i) * S::kScaleStage + at] = (char)(words[k] >> shift >> (8 * i));
        }
    };

    const int wn = wave % WN, wm = wave / WN;
    const int a_row = wn * (16 * S::kTN) + (r >> 2) * 16 + (r & 3), b_row = BN + wm * (16 * S::kTM) + r;
    // A lane's two chunks are kb and kb + 4, four chunks apart or four back.  (Four addresses that go from stage to stage: left to itself the compiler keeps one for
    // each tile of each stage, which do not fit the registers.)
    uint32_t from[4];
    {
        const uint32_t a_at = lds0 + (uint32_t)(a_row * 128 + (kb ^ ((r & 3) | (r >> 2 & 1) << 2)) * 16), b_at = lds0 + (uint32_t)(b_row * 128 + (kb ^ (r & 7)) * 16);
        from[0] = a_at, from[1] = lds0 + ((a_at - lds0) ^ 64), from[2] = b_at, from[3] = lds0 + ((b_at - lds0) ^ 64);
    }
    auto go_on = [&](int by) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            from[i] += (uint32_t)by;
            asm volatile("" : "+v"(from[i]));
        }
    };
    auto chunks = [&](int first, int at) {
        typedef const __attribute__((address_space(3))) intx4* lds_chunk;
        const intx4 p = *(lds_chunk)(from[first] + (uint32_t)at), q = *(lds_chunk)(from[first + 1] + (uint32_t)at);
        return int32x8{p[0], p[1], p[2], p[3], q[0], q[1], q[2], q[3]};
    };

    floatx4 acc[S::kTN][S::kTM];
#pragma unroll
    for (int i = 0; i < S::kTN; ++i)
#pragma unroll
        for (int j = 0; j < S::kTM; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t sa[S::kGroupsN], sb[S::kGroupsM], next_sa[S::kGroupsN], next_sb[S::kGroupsM];
    int32x8 a[2][S::kHN], b[2][S::kHM];                  // halves; of a single tile of x: two stages
    // (part: two of a half's four tiles)
    auto read_a = [&](int half, int part) {
#pragma unroll
        for (int i = part * S::kPart; i < (part + 1) * S::kPart; ++i) {
            const int tile = half * S::kHN + i;
            a[half][i] = chunks(0, ((tile >> 2) * 64 + (tile & 3) * 4) * 128);
        }
    };
    auto read_scales = [&](int t) {
        const char* at = lds + S::kScales + (t & 7) * S::kScaleStage + r * 4;
#pragma unroll
        for (int g = 0; g < S::kGroupsN; ++g) next_sa[g] = *reinterpret_cast<const uint32_t*>(at + wn * (16 * S::kTN) + g * 64);
#pragma unroll
        for (int g = 0; g < S::kGroupsM; ++g) next_sb[g] = *reinterpret_cast<const uint32_t*>(at + BN + (wm * S::kGroupsM + g) * 64);
    };
    auto read_b = [&](int half) {
#pragma unroll
        for (int j = 0; j < S::kHM; ++j) b[half][j] = chunks(2, (S::kTM > 1 ? half * S::kHM + j : 0) * 16 * 128);
    };

    if (pieces >= 4) {
        fetch_scales(0);
    } else {
#pragma unroll
        for (int k = 0; k < S::kWords; ++k) {
            words[k] = 0;
            for (int i = 0; i < pieces; ++i) words[k] |= (uint32_t)scales_at[k][i] << (8 * i);
        }
    }
    for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int i = 0; i < S::kFetches; ++i) fetch(i, t);
    put_scales(0, 0);
    wait_fetches<0>();
    meet();
    read_scales(0);
    read_a(0, 0);
    read_a(0, 1);
    read_b(0);

    // Stage t, at place STEP of its group of four; LOOP: a whole group.  No branches: around them the compiler would move products, and hold their operands
    // longer.  Behind the last stage it is fetched again, and what LDS holds is read and not used.
    auto stage = [&](auto step, auto loop, int t) {
        constexpr int STEP = decltype(step)::value, LOOP = decltype(loop)::value, F = STEP & 1, HERE = STEP & (NS - 1), NEXT = (STEP + 1) & (NS - 1);
#pragma unroll
        for (int g = 0; g < S::kGroupsN; ++g) sa[g] = next_sa[g];
#pragma unroll
        for (int g = 0; g < S::kGroupsM; ++g) sb[g] = next_sb[g];
        if (STEP == 0 && LOOP) fetch_scales(t + 4);
        // The fetches of the stage NS ahead are issued between the products behind the meeting, from number `done` on: together they would hold those up.
        constexpr int kProducts = S::kHN * S::kTM, kEach = (S::kFetches + kProducts - 1) / kProducts;
        auto fetch_behind = [&](int done) {
#pragma unroll
            for (int i = done * kEach; i < min((done + 1) * kEach, S::kFetches); ++i) {
                fetch(i, t + NS);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        auto multiply = [&](int ha, int part, int hb, int done = -1000) {
#pragma unroll
            for (int i = part * S::kPart; i < (part + 1) * S::kPart; ++i)
#pragma unroll
                for (int j = 0; j < S::kHM; ++j) {
                    const int n = ha * S::kHN + i, m = (S::kTM > 1 ? hb * S::kHM : 0) + j;
                    if (done >= 0) fetch_behind(done + (i - part * S::kPart) * S::kHM + j);
                    multiply_tile(a[ha][i], b[hb][j], acc[n][m], sa[n / 4], sb[m / 4], n % 4, m % 4);
                }
        };
        // (in bfloat16 a tile of x is made once a stage, one of the weights where it is multiplied with all of x's)
        Wide wide[EXACT ? S::kTM : 1];
        auto widen_b = [&](int hb) {
#pragma unroll
            for (int j = 0; j < S::kHM; ++j) {
                const int m = (S::kTM > 1 ? hb * S::kHM : 0) + j;
                wide[EXACT ? m : 0] = fp8_widen(b[hb][j], (sb[m / 4] >> (8 * (m % 4)) & 255) << 23);
            }
        };
        auto multiply_half = [&](int ha) {
#pragma unroll
            for (int i = 0; i < S::kHN; ++i) {
                const int n = ha * S::kHN + i;
                const Wide w = fp8_widen(a[ha][i], (sa[n / 4] >> (8 * (n % 4)) & 255) << 23);
#pragma unroll
                for (int m = 0; m < S::kTM; ++m) acc[n][m] = multiply_wide(w, wide[EXACT ? m : 0], acc[n][m]);
            }
        };
        // What is read takes the place of what has been multiplied.  (The compiler would read earlier, and spill.)
        auto phase = [] { __builtin_amdgcn_sched_barrier(0); };
        auto next_stage = [&] {
            // it has arrived once no more than those behind it are on their way
            wait_fetches<(NS - 2) * S::kFetches>();
            if (STEP == 3) put_scales((t >> 2) + 1, 8 * max(0, min(t + 5 - pieces, 3)));
            meet();
            go_on((NEXT - HERE) * S::kStage);
            read_scales(t + 1);
        };
        if (S::kTM > 1) read_b(F ^ 1);
        read_a(1, 0);
        if constexpr (EXACT) {
            read_a(1, 1);
            widen_b(F);
            if (S::kTM > 1) widen_b(F ^ 1);
            multiply_half(0);
            next_stage();
#pragma unroll
            for (int i = 0; i < S::kFetches; ++i) fetch(i, t + NS);
            read_a(0, 0);
            read_a(0, 1);
            multiply_half(1);
            read_b(F ^ 1);
        } else {
            multiply(0, 0, F);
            multiply(0, 1, F);
            phase();
            if (S::kTM > 1) multiply(0, 0, F ^ 1);
            phase();
            read_a(1, 1);
            if (S::kTM > 1) multiply(0, 1, F ^ 1);
            phase();
            next_stage();
            read_a(0, 0);
            constexpr int kOf = S::kPart * S::kHM, kBefore = S::kTM > 1 ? 2 * kOf : 0;
            if (S::kTM > 1) {
                multiply(1, 0, F ^ 1, 0);
                multiply(1, 1, F ^ 1, kOf);
            }
            phase();
            read_b(F ^ 1);
            multiply(1, 0, F, kBefore);
            phase();
            read_a(0, 1);
            multiply(1, 1, F, kBefore + kOf);
            phase();
        }
    };
    int t = 0;
    for (; t + 4 <= pieces; t += 4) {
        stage(Const<0>{}, Const<1>{}, t);
        stage(Const<1>{}, Const<1>{}, t + 1);
        stage(Const<2>{}, Const<1>{}, t + 2);
        stage(Const<3>{}, Const<1>{}, t + 3);
    }
    if (t < pieces) stage(Const<0>{}, Const<0>{}, t);
    if (t + 1 < pieces) stage(Const<1>{}, Const<0>{}, t + 1);
    if (t + 2 < pieces) stage(Const<2>{}, Const<0>{}, t + 2);
    wait_fetches<0>();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (!EXACT) let_settle(acc);

    // A lane's results: row m0 + ... + r of x, sixteen neighbouring outputs for each four tiles (and their other sums four tiles on).
    constexpr int kGroups = kTwo ? 1 : S::kTN / 4;
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int n = n0 + wn * (kOut / WN) + g * 64 + kb * 16, left = A.s.out - n;
        float add[16];
        if constexpr (SLICED) {
            float* to = A.partial + ((long long)slice * A.s.rows + m0) * (kTwo ? 2ll : 1ll) * A.s.out + n;
#pragma unroll
            for (int j = 0; j < S::kTM; ++j) {
                const int m = wm * (16 * S::kTM) + j * 16 + r;
                if (m0 + m >= A.s.rows || left <= 0) continue;
#pragma unroll
                for (int side = 0; side < (kTwo ? 2 : 1); ++side) {
                    float z[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[i] = acc[(g + side) * 4 + i / 4][j][i % 4];
                    store_results(to, ((long long)m * (kTwo ? 2 : 1) + side) * A.s.out, kF32, left, z);
                }
            }
            continue;
        }
        if (KIND == kLinear)
#pragma unroll
            for (int i = 0; i < 16; ++i) add[i] = A.t.bias && i < left ? A.t.bias[n + i] : 0.0f;
        if constexpr (KIND == kGatedCodes) {
            // the largest of a row's 128 outputs is that of its lanes in the two wavefronts that have them
            static_assert(WN == 2, "128 outputs in two wavefronts");
            uint32_t* tops = reinterpret_cast<uint32_t*>(lds);           // [wn][row]
            __syncthreads();
#pragma unroll
            for (int j = 0; j < S::kTM; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                uint32_t top = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float h = i < left ? activate_as(acc[g * 4 + i / 4][j][i % 4], A.s.act) * acc[(g + (kTwo ? 1 : 0)) * 4 + i / 4][j][i % 4] : 0.0f;
                    acc[g * 4 + i / 4][j][i % 4] = h;
                    top = max(top, __float_as_uint(h) & 0x7fffffffu);
                }
                top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
                if (kb == 0) tops[wn * BM + wm * (16 * S::kTM) + j * 16 + r] = top;
            }
            __syncthreads();
            const int out_pieces = (A.s.out + 127) / 128;
#pragma unroll
            for (int j = 0; j < S::kTM; ++j) {
                __builtin_amdgcn_sched_barrier(0);
                const int at = wm * (16 * S::kTM) + j * 16 + r, m = m0 + at;
                if (m >= A.s.rows) continue;
                const uint32_t byte = fp8_scale_byte(max(tops[at], tops[BM + at]));
                const float inverse = fp8_inverse(byte);
                uint32_t c[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const floatx4 h = acc[g * 4 + i][j];
                    c[i] = byte == kNanScale ? 0u : fp8_encode4(h[0], h[1], h[2], h[3], inverse);
                }
                *reinterpret_cast<uint4*>(static_cast<uint8_t*>(A.t.out) + ((long long)m * out_pieces + tn) * 128 + wn * 64 + kb * 16) =
                    make_uint4(c[0], c[1], c[2], c[3]);
                if (wn == 0 && kb == 0) A.t.out_scales[(long long)m * out_pieces + tn] = (uint8_t)byte;
            }
            continue;
        }
        auto sums = [&](int side, int j, float(&z)[16]) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = acc[(g + side) * 4 + i / 4][j][i % 4];
        };
        if constexpr (KIND == kGatedBackward) {
            auto one = [&](int j, const Pack<D, 8>& d0, const Pack<D, 8>& d1) {
                const int m = m0 + wm * (16 * S::kTM) + j * 16 + r;
                if (m >= A.s.rows || left <= 0) return;
                float z[16], y[16];
                sums(0, j, z);
                sums(kTwo ? 1 : 0, j, y);
                auto gradients = [&](auto act) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float gate = z[i], up = y[i];
                        gated_gradients<decltype(act)::value>(gate, up, to_float(i < 8 ? d0.v[i % 8] : d1.v[i % 8]), z[i], y[i]);
                    }
                };
                if (A.s.act == kActSilu) gradients(Const<kActSilu>{});
                else if (A.s.act == kActRelu) gradients(Const<kActRelu>{});
                else gradients(Const<kActNone>{});
                store_results(A.t.out, m * A.s.out_row + n, A.s.out_type, left, z);
                store_results(A.t.out2, m * A.s.out_row + n, A.s.out_type, left, y);
            };
            auto dh_at = [&](int j) {
                const long long m = min(m0 + wm * (16 * S::kTM) + j * 16 + r, A.s.rows - 1);
                return static_cast<const D*>(A.t.dh) + m * A.s.dh_row + n;
            };
            if (n0 + kOut <= A.s.out) {
                // dh is on its way before it is waited for: all of it, or in 32 bits two tiles ahead
                constexpr int kMost = sizeof(D) == 4 ? 2 : 4, kDeep = S::kTM < kMost ? S::kTM : kMost;
                Pack<D, 8> d[S::kTM][2];
                auto ask = [&](int j) { d[j][0] = load_pack<D, 8>(dh_at(j)), d[j][1] = load_pack<D, 8>(dh_at(j) + 8); };
#pragma unroll
                for (int j = 0; j < kDeep; ++j) ask(j);
#pragma unroll
                for (int j = 0; j < S::kTM; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
                    one(j, d[j][0], d[j][1]);
                    if (j + kDeep < S::kTM) ask(j + kDeep);
                }
            } else {
#pragma unroll
                for (int j = 0; j < S::kTM; ++j) {
                    __builtin_amdgcn_sched_barrier(0);
                    one(j, load8(dh_at(j), left), load8(dh_at(j) + 8, left - 8));
                }
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < S::kTM; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            const int m = m0 + wm * (16 * S::kTM) + j * 16 + r;
            if (m >= A.s.rows || left <= 0) continue;
            float z[16];
            sums(0, j, z);
            if (KIND == kLinear) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] += add[i];
                finish_sixteen(z, A.s.act);
            } else {
                float y[16];
                sums(kTwo ? 1 : 0, j, y);
                finish_sixteen(z, A.s.act);
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] *= y[i];
            }
            store_results(A.t.out, m * A.s.out_row + n, A.s.out_type, left, z);
        }
    }
}

// Adds the slices up in their order, and makes the results: 256 outputs of a row a workgroup.
template <int KIND>
__global__ __launch_bounds__(256) void product_join_kernel(ProductShape s, ProductTensors t, const float* __restrict__ partial, int slices, FastDiv by_out_blocks)
{
    constexpr int kSides = KIND == kLinear ? 1 : 2;
    __shared__ uint32_t tops[4];
    const uint32_t m = fast_div(blockIdx.x, by_out_blocks);
    const int n = (int)(blockIdx.x - m * (uint32_t)((s.out + 255) / 256)) * 256 + (int)threadIdx.x;
    const long long stride = (long long)s.rows * kSides * s.out;
    float z[2] = {0.0f, 0.0f};
    if (n < s.out) {
        const float* p = partial + (long long)m * kSides * s.out + n;
#pragma unroll 4
        for (int k = 0; k < slices; ++k)
#pragma unroll
            for (int i = 0; i < kSides; ++i) z[i] += p[k * stride + i * s.out];
    }
    if constexpr (KIND == kGatedCodes) {
        const float h = n < s.out ? activate_as(z[0], s.act) * z[1] : 0.0f;
        uint32_t top = largest_of_16_lanes(__float_as_uint(h) & 0x7fffffffu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
        const int wave = (int)threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) tops[wave] = top;
        __syncthreads();
        const int pieces = (s.out + 127) / 128;
        if (n >= pieces * 128) return;
        const uint32_t byte = fp8_scale_byte(max(tops[wave], tops[wave ^ 1]));
        const uint32_t code = byte == kNanScale ? 0u : fp8_encode4(h, 0.0f, 0.0f, 0.0f, fp8_inverse(byte));
        static_cast<uint8_t*>(t.out)[(long long)m * pieces * 128 + n] = (uint8_t)code;
        if (n % 128 == 0) t.out_scales[(long long)m * pieces + n / 128] = (uint8_t)byte;
    } else if (n < s.out) {
        finish_one<KIND>(s, t, (int)m, n, z[0], z[1]);
    }
}

// CUT: whether a plan cuts such tiles along k.
template <int KIND, bool EXACT, int BN, int BM, int WN, int WM, int NS, bool CUT, int WAVES = 1>
hipError_t launch_shape(Args A, hipStream_t stream)
{
    using S = Tile<BN, BM, WN, WM, NS>;
    constexpr int kOut = KIND == kLinear ? BN : BN / 2;
    A.tiles_n = (A.s.out + kOut - 1) / kOut;
    A.tiles_m = (A.s.rows + BM - 1) / BM;
    A.by_tiles = make_fast_div((uint32_t)(A.tiles_n * A.tiles_m));
    A.by_band = make_fast_div((uint32_t)(kBand * A.tiles_n));
    A.by_last = make_fast_div((uint32_t)(A.tiles_m % kBand ? A.tiles_m % kBand : kBand));
    auto launch = [&](auto sliced, auto of_dh) {
        constexpr auto kernel = product_tiles_kernel<KIND, EXACT, BN, BM, WN, WM, NS, WAVES, decltype(sliced)::value != 0, decltype(of_dh)>;
        static std::atomic<uint64_t> allowed{0};
        if (const hipError_t e = allow_big_lds(reinterpret_cast<const void*>(kernel), allowed); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)(A.tiles_n * A.tiles_m * A.slices)), dim3(S::kThreads), S::kLds, stream, A);
        return hipGetLastError();
    };
    if (A.slices == 1) {
        if constexpr (KIND == kGatedBackward) return with_type(A.s.dh_type, [&](auto of_dh) { return launch(Const<0>{}, of_dh); });
        else return launch(Const<0>{}, float{});
    }
    if constexpr (!CUT) return hipErrorInvalidValue;
    else if (const hipError_t e = launch(Const<1>{}, float{}); e != hipSuccess) return e;
    const int across = (A.s.out + 255) / 256;
    hipLaunchKernelGGL((product_join_kernel<KIND>), dim3((unsigned)((long long)across * A.s.rows)), dim3(256), 0, stream, A.s, A.t, A.partial, A.slices,
                       make_fast_div((uint32_t)across));
    return hipGetLastError();
}

// Tiles of bn outputs x bm rows.
long long tiles_of(const ProductShape& s, int bn, int bm) { return ceil_div(s.out, bn) * ceil_div(s.rows, bm); }

// The shape, outputs x rows, and slices of k of a call.
struct Plan {
    int outputs, rows, slices, slice_pieces;
};
Plan plan_of(const ProductShape& s)
{
    const bool exact = s.out_type == kF32;
    const int pieces = (int)fp8_pieces(s.in);
    // The largest tiles that three of four CUs get one of (256 x 4096 -> 12288, 192 tiles of 128^2: 23.5 us, 32 with 64^2; 512 x 4096 -> 4096, 128 of them: 25.9
    // and 19.5; gated 512 x 4096 -> 12288, 192 of 256 rows: 54 and 63).  Results in fp32 stop at 128 rows.  The gated pair's
    // next are of 64 outputs, or 128 for the scale that they share (1003 x 2000 -> 3000, 192 tiles of 128 rows: 18 us, 30 with 64 rows), by 128 rows also with fewer
    // tiles where k is long enough to be cut (600 x 12288 -> 1000, 80 tiles: 46 us, 69 by 64 rows uncut; 500 x 700 -> 2000, 128 of them: 11 and 9).
    constexpr long long kEnough = 192;
    Plan p{};
    if (s.kind == kLinear)
        p = !exact && tiles_of(s, 256, 256) >= kEnough ? Plan{256, 256} : tiles_of(s, 128, 128) >= kEnough ? Plan{128, 128} : Plan{64, 64};
    else if (!exact && tiles_of(s, 128, 256) >= kEnough) p = Plan{128, 256};
    else if (s.out_type == kFp8) p = Plan{128, tiles_of(s, 128, 128) >= kEnough ? 128 : 64};
    else p = Plan{64, tiles_of(s, 64, 128) >= (pieces >= 64 ? 64 : kEnough) ? 128 : 64};
    // Fewer tiles than CUs are cut along k, into slices of eight stages and more (four in fp32, whose take longer): adding them up is a launch of its own, whose
    // bytes cost what it saves where there are many rows (us in 1, 2, 4 and 8 slices: 32 x 4096 -> 4096 14.8, 12.3, 11.0, 12.5; 128 x 4096 -> 4096 15.1, 14.9, 17.0,
    // 22.7; 64 x 12288 -> 4096 36, 23, 17.7, 17.7; gated codes 256 x 12288 -> 4096 77, 54, 62, 89).  Linear layers' long slices of the smallest tiles pay up to twice as many
    // (256 x 12288 -> 4096 37, 33, 37).  The largest tiles are whole.
    const long long tiles = tiles_of(s, p.outputs, p.rows);
    long long slices = p.rows == 256 ? 1 : std::max<long long>(1, std::min<long long>(pieces / (exact ? 4 : 8), 256 / tiles));
    if (s.kind == kLinear && p.rows == 64) slices = std::max<long long>(slices, std::min<long long>(pieces / 24, 512 / tiles));
    p.slice_pieces = (int)((pieces + slices - 1) / slices);
    p.slices = (pieces + p.slice_pieces - 1) / p.slice_pieces;
    return p;
}

}  // namespace

bool product_tiles_fit(const ProductShape& s)
{
    // offsets in a tile are 32-bit; the smallest tiles are 64 x 64
    return fp8_pieces(s.in) * 128 * 256 <= INT32_MAX && tiles_of(s, 64, 64) <= kMostBlocks / 4;
}

size_t product_tiles_workspace_bytes(const ProductShape& s)
{
    const Plan p = plan_of(s);
    return p.slices > 1 ? (size_t)p.slices * (size_t)s.rows * (size_t)s.out * (s.kind == kLinear ? 4 : 8) : 0;
}

hipError_t launch_product_tiles(const ProductShape& s, const ProductTensors& t, float* partial, hipStream_t stream)
{
    const Plan p = plan_of(s);
    Args A{};
    A.s = s;
    A.t = t;
    A.partial = partial;
    A.pieces = (int)fp8_pieces(s.in);
    A.slices = p.slices;
    A.slice_pieces = p.slice_pieces;
    const bool exact = s.out_type == kF32;
    if (s.kind == kLinear) {
        if (exact) return p.rows == 128 ? launch_shape<kLinear, true, 128, 128, 2, 2, 2, false, 2>(A, stream) : launch_shape<kLinear, true, 64, 64, 1, 4, 2, true>(A, stream);
        if (p.rows == 256) return launch_shape<kLinear, false, 256, 256, 2, 4, 2, false>(A, stream);
        if (p.rows == 64) return launch_shape<kLinear, false, 64, 64, 1, 4, 4, true>(A, stream);
        // A workgroup that has its CU to itself takes four stages; two on a CU cover each other's waits, and the LDS has room for them with two stages only
        // (us with two and four: 1024 x 12288 -> 4096, 256 tiles, 77.7 and 61.6; 2048 x 4096 -> 4096, 512 of them, 37.8 and 43.1; fp32's products are long enough for two:
        // 99.8 and 97.4, 67.5 and 78.1).
        return tiles_of(s, 128, 128) <= 256 ? launch_shape<kLinear, false, 128, 128, 2, 2, 4, false>(A, stream) : launch_shape<kLinear, false, 128, 128, 2, 2, 2, false>(A, stream);
    }
    auto run = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
        if (p.rows == 256) return launch_shape<KIND, false, 256, 256, 2, 4, 2, false>(A, stream);
        if constexpr (KIND == kGatedCodes) {
            return p.rows == 128 ? launch_shape<KIND, false, 256, 128, 2, 4, 2, false>(A, stream) : launch_shape<KIND, false, 256, 64, 2, 4, 2, true>(A, stream);
        } else if (const bool alone = tiles_of(s, 64, 128) * p.slices <= 256; exact) {
            if (p.rows == 64) return launch_shape<KIND, true, 128, 64, 1, 4, 2, true>(A, stream);
            // (registers for two workgroups on a CU where there are as many, 4096 x 4096 -> 8192 backward: 521 us, 576 in tiles of 256 x 128; else as many as the
            // compiler likes: 777 x 1500 -> 2100 23.0, 25.1 with those for two)
            return alone ? launch_shape<KIND, true, 128, 128, 1, 4, 2, true>(A, stream) : launch_shape<KIND, true, 128, 128, 1, 4, 2, false, 2>(A, stream);
        } else {
            if (p.rows == 64) return launch_shape<KIND, false, 128, 64, 1, 4, 2, true>(A, stream);
            // (four stages as above, where k is long enough to make up for their start: 512 x 4096 -> 4096, 256 tiles, 26.2 us with two and 21.5 with four;
            // 777 x 1500 -> 2100 11.4 and 11.8; 1003 x 2000 -> 3000, 376 tiles, 19.4 and 24.4)
            return alone && A.pieces >= 16 ? launch_shape<KIND, false, 128, 128, 1, 4, 4, true>(A, stream) : launch_shape<KIND, false, 128, 128, 1, 4, 2, false>(A, stream);
        }
    };
    return s.kind == kGatedBackward ? run(Const<kGatedBackward>{}) : s.out_type == kFp8 ? run(Const<kGatedCodes>{}) : run(Const<kGated>{});
}

}  // namespace patdnn
