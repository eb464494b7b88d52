// 8-bit products on tiles of 256 rows by up to 256 columns: 2 x 2 waves of 128 x 128 (8 x 8 MFMA tiles of 16 x 16, all 256 accumulator registers, one
// wave per SIMD).  A K tile is 64 MFMAs a wave, 32 cycles each, and 128 KB out of the LDS for the four of them, half of what it delivers
// in that time.
//
// LDS: two stages of one K tile, 32 KB of each operand, 16 positions a fragment; chunk h of position 16 f + c at slot h ^ (c / 2), and lane (c, q) reads chunks
// q and q + 4 (fp8_gemm.hip).  A's rows stand in their order; B's so that a lane ends with eight neighbouring columns and its three neighbours with those
// beside them, 64 bytes a row: fragment 2 s + h of 64 columns has the columns 32 s + 8 (c / 4) + 4 h + c % 4.  Beside them the 512 scale
// bytes, a dword each, four fragments' of a lane together.  All of it is written by direct global ->
// LDS loads (scales byte by byte: they start anywhere), so that the loads in flight can be counted.  Rows past the edge are clamped to the last one.
//
// A K tile in quarters, halves of A against halves of B, a half's registers read again as soon as its last quarter is done; of B the half that
// the tile before ended without comes first (P, then Q):
//     A0 x P   while Q is read             A0 x Q   while A1 is read            a barrier: A0, P and scales of kt + 1 have landed
//     A1 x Q   while A0 of kt + 1 is read  A1 x P   while its P and scales are  a barrier: Q and A1 of kt + 1 have landed
// A barrier also says that every wave has read what the two quarters before it read, whose place the loads for two K tiles on then take: A0, P and
// scales in a tile's first quarter, Q and A1 in its third.  So a load has a K tile and a quarter at least; with the loads behind the first barrier only,
// three quarters, 4096 x 4096 x 11008 took 167 us.  Past the last K tile the loads repeat one piece of the first, so that
// the counts hold.
//
// Workgroups stay (one per CU) and walk the output tiles: the first two K tiles of the next one are requested before this one's outputs are
// stored.  Stores are of whole lines, eight rows' at a time, for which lanes eight apart exchange halves: a CU takes a tile's 128 KB in 5000 cycles so, in 8000
// by stores of sixteen half lines (8192 x 8192 x 1024 80.2 -> 78.6 us, 16 experts' weight gradients 4096 x 2048 from 16384 rows 155 -> 150).  Which tiles there are
// for how many rows of an expert is counted once, into the LDS.
//
// What bounds it: long contractions the matrix instructions (4096 x 4096 x 11008 127 us, 2.9 PFLOP/s, 2290 cycles a K tile of which 2048 are MFMAs; 8192^3 360 us, 3.05
// PFLOP/s; the power limit lowers the clock to 2 GHz), short ones what is not them: of 8192 x 8192 x 1024 (79 us, 1.7 PFLOP/s) a tile takes 35000 cycles, 23000 for
// eight K tiles, of which the first wait for memory, 8000 for the stores, which all CUs do at once, 3000 to find and request the next tile.
#include <atomic>
#include <type_traits>

#include "fp8_gemm.h"

namespace nvfp4 {
namespace f8w {

constexpr int BM = 256, KT = FP8_BLOCK;
// Weight gradients of so many tiles an expert are walked expert by expert, each over all XCDs (contractions differ in length as the tokens do); else an XCD takes a
// band of the experts' tiles, whose operands its L2 then keeps.  us, band / each: 16 experts' 4096 x 2048 with 300 to 2281 of 16384 rows (128 tiles) 241 / 187; 64 experts'
// 1024 x 1024 with 23 to 3016 of 32768 (24 tiles) 75 / 83.
constexpr int SPREAD = 64;
// FB: fragments of 16 columns of a wave; the workgroup's tile is 256 x 32 FB
template <int FB, int OUT_DT>
struct Geom {
    static constexpr int BN = 32 * FB, HB = FB / 2;                     // fragments of a half of B
    static constexpr int STAGE = (BM + BN) * KT, SCALES = 4 * 512;     // of a K tile; scale bytes: a dword for each of 8 fragments a wave
    static constexpr int SCALES0 = 2 * STAGE, GROUPS0 = SCALES0 + 2 * SCALES, LDS_BYTES = GROUPS0 + 2 * 4 * (MAX_EXPERTS + 2);
    static constexpr int FIRST = 4 + HB + 2, SECOND = HB + 4;           // loads of a wave and K tile: A0, P and scales; Q and A1
    static constexpr int STORES = (OUT_DT == NVFP4_F32 ? 8 : 4) * FB;  // of a wave, for an output inside
};

// Column of the tile that position c of fragment f of the waves `part` holds: a lane ends with columns of one row that fill 16 bytes.  Waves have whole
// lines of the output, of 96 columns all but the last 32.
template <int FB>
__device__ __forceinline__ int columns_of(int part, int f)
{
    return FB == 6 && f >= 4 ? 128 + 32 * part : 16 * (FB == 6 ? 4 : FB) * part;
}
template <int OUT_DT, int FB>
__device__ __forceinline__ int column(int part, int f, int c)
{
    return columns_of<FB>(part, f) + (FB == 6 && f >= 4 ? -64 : 0) + (OUT_DT == NVFP4_F32 ? 16 * f + c : 32 * (f >> 1) + 8 * (c >> 2) + 4 * (f & 1) + (c & 3));
}

// x of the lanes c < 8 and y of c + 8 in the others; and y of the lanes c >= 8, x of c + 8 in the others: of two halves of 16 rows' lines, the lines of eight rows each
__device__ __forceinline__ void exchange(uint32_t &x, uint32_t &y)
{
    constexpr int ROTATE_8 = 0x128;
    const uint32_t t = __builtin_amdgcn_update_dpp(x, y, ROTATE_8, 0xf, 0xc, false);
    y = __builtin_amdgcn_update_dpp(y, x, ROTATE_8, 0xf, 0x3, false);
    x = t;
}

// As assembly, so that the 64 accumulators stay where they are (gemm_mx.hip).  What the compiler does not know about it: an operand must not have been
// written by the vector ALU in the two instructions before (they come from LDS reads), and the last result must not be read for 11 wait
// states.
__device__ __forceinline__ void mfma(f8g::float4v_t &acc, const f8g::int8v_t &b, const f8g::int8v_t &a, uint32_t sb, uint32_t sa)
{
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0]" : "+a"(acc) : "v"(b), "v"(a), "v"(sb), "v"(sa));
}

// Assembly because the compiler takes a direct-to-LDS load for a possible writer of all of the LDS and would wait for it before the next LDS
// read; here a stage is read behind an explicit wait and barrier only.
template <int TO>
__device__ __forceinline__ void load(uint32_t dst, uint32_t off, const uint8_t *base)
{
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" : : "s"(dst), "n"(TO), "v"(off), "s"(base) : "memory", "scc", "m0");
}

template <int TO>
__device__ __forceinline__ void load_byte(uint32_t dst, uint32_t off, const uint8_t *base)
{
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %2, %3" : : "s"(dst), "n"(TO), "v"(off), "s"(base) : "memory", "scc", "m0");
}

template <int I, int N, class F>
__device__ __forceinline__ void each(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<I + 1, N>(f);
    }
}

}  // namespace f8w

template <int MODE, int OUT_DT, int FB>
__global__ __launch_bounds__(256) void fp8_gemm_wide_kernel(Fp8GemmArgs P)
{
    using namespace f8g;
    using G = f8w::Geom<FB, OUT_DT>;
    constexpr int BM = f8w::BM, BN = G::BN, HB = G::HB, STAGE = G::STAGE, ALL = G::FIRST + G::SECOND;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;
    const int64_t pitch = (int64_t)P.blocks * KT;

    // ---- which tiles there are.  Groups' first rows (clamped, ascending) and, for the experts' product, their first tile rows, with the rows of no expert
    // as one more group.
    const int ntx = (int)((P.N + BN - 1) / BN);
    int *const group_row = reinterpret_cast<int *>(lds + G::GROUPS0), *const group_tile = group_row + MAX_EXPERTS + 2;
    int nty = (int)((P.M + BM - 1) / BM);
    constexpr bool DIVIDED = MODE == FP8_DIVIDED;
    if (MODE == FP8_EXPERTS || MODE == FP8_EXPERTS_DW) {
        const int total = MODE == FP8_EXPERTS ? (int)P.M : P.total, groups = P.groups + (MODE == FP8_EXPERTS ? 1 : 0);
        if (wave == 0) {
            int row = 0, tiles = 0;
            for (int e0 = 0; e0 <= groups; e0 += 64) {
                // (an offset below an earlier one counts as that one, so that groups do not overlap)
                const int e = e0 + lane;
                int a = e <= P.groups ? P.offsets[e] : total;
                a = a < 0 ? 0 : a > total ? total : a;
#pragma unroll
                for (int d = 1; d < 64; d <<= 1) {
                    const int up = __shfl_up(a, d);
                    if (lane >= d) a = a > up ? a : up;
                }
                a = a > row ? a : row;
                if (e <= groups) group_row[e] = a;
                if (MODE == FP8_EXPERTS) {
                    // tiles of the group before, which ends here
                    int before = __shfl_up(a, 1);
                    before = lane == 0 ? row : before;
                    int n = e == 0 || e > groups ? 0 : (int)(((unsigned)(a - before) + BM - 1) / BM);  // (up to 2^31 - 1 rows)
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) {
                        const int up = __shfl_up(n, d);
                        if (lane >= d) n += up;
                    }
                    if (e <= groups) group_tile[e] = tiles + n;
                    tiles += __shfl(n, 63);
                }
                row = __shfl(a, 63);
            }
        }
        __syncthreads();
        if (MODE == FP8_EXPERTS) nty = __builtin_amdgcn_readfirstlane(group_tile[groups]);
    }
    // An output without a contraction (rows of no expert, an expert without rows) is one K tile of whatever is there, stored as zeros: `keep` is a mask.
    auto find = [&](int id, uint32_t &keep) -> Tile {
        Tile T;
        keep = ~0u;
        int ty, tx, e = 0;
        if (MODE == FP8_EXPERTS_DW && ntx * nty >= f8w::SPREAD) {
            e = id / (ntx * nty);
            tile_coords(id - e * ntx * nty, ntx, nty, ty, tx);
        } else {
            tile_coords(id, ntx, MODE == FP8_EXPERTS_DW || DIVIDED ? nty * P.groups : nty, ty, tx);
            if (MODE == FP8_EXPERTS_DW || DIVIDED) {
                e = ty / nty;
                ty -= e * nty;
            }
        }
        T.k0 = 0;
        T.count = P.blocks;
        T.b0 = T.out = 0;
        int left;
        if constexpr (MODE == FP8_EXPERTS) {
            int n = 0;
            for (int e0 = 0; e0 <= P.groups; e0 += 64) n += __popcll(__ballot(e0 + lane <= P.groups && group_tile[e0 + lane <= P.groups ? e0 + lane : 0] <= ty));
            e = __builtin_amdgcn_readfirstlane(n - 1);
            const int row = __builtin_amdgcn_readfirstlane(group_row[e] + (ty - group_tile[e]) * BM), end = __builtin_amdgcn_readfirstlane(group_row[e + 1]);
            T.m0 = row;
            left = end - row;
            if (e < P.groups) {
                T.b0 = e * P.N;
            } else {  // rows of no expert
                keep = 0;
                T.count = 1;
            }
        } else {
            if (MODE == FP8_EXPERTS_DW) {
                const int row = __builtin_amdgcn_readfirstlane(group_row[e]), rows = __builtin_amdgcn_readfirstlane(group_row[e + 1]) - row;
                T.k0 = row / KT + e;
                T.count = rows > 0 ? (rows + KT - 1) / KT : 1;
                keep = rows > 0 ? ~0u : 0u;
                T.out = e * P.M;
            }
            if (DIVIDED) {
                // (a part has a K tile at least)
                T.k0 = (int)((int64_t)P.blocks * e / P.groups);
                T.count = (int)((int64_t)P.blocks * (e + 1) / P.groups) - T.k0;
                T.out = ((int64_t)e * nty + ty) * ntx + tx;
            }
            T.m0 = (int64_t)ty * BM;
            left = P.M - T.m0 < BM ? (int)(P.M - T.m0) : BM;
        }
        T.n0 = (int64_t)tx * BN;
        T.rows = left < BM ? left : BM;
        T.cols = (int)(P.N - T.n0 < BN ? P.N - T.n0 : BN);
        return T;
    };

    // ---- global -> LDS.  Half h of A is positions 64 h .. + 63 of each 128, of B 16 HB h .. of each 16 FB; a wave's instructions fill 8
    // positions each, half of one of the two parts.
    uint32_t offA[8], offB[FB], offSA, offSB;  // [half][instruction]
    const int part = wave >> 1, side = wave & 1;
    // K tile that is requested next
    const uint8_t *pA, *pB, *pSA, *pSB;
    int64_t step, stepSA, stepSB;
    auto uniform = [](const uint8_t *p) -> const uint8_t * {
        const uint64_t v = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return reinterpret_cast<const uint8_t *>(((uint64_t)hi << 32) | lo);
    };
    auto point_to = [&](const Tile &T) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int in = 32 * side + 8 * (i & 3) + (lane >> 3), row = 128 * part + 64 * (i >> 2) + in;
            offA[i] = (uint32_t)((row < T.rows ? row : T.rows - 1) * pitch) + ((lane & 7) ^ ((in & 15) >> 1)) * 16;
        }
#pragma unroll
        for (int i = 0; i < FB; ++i) {
            const int in = 16 * HB * (i / HB) + 8 * HB * side + 8 * (i % HB) + (lane >> 3), col = f8w::column<OUT_DT, FB>(part, in >> 4, in & 15);
            offB[i] = (uint32_t)((col < T.cols ? col : T.cols - 1) * pitch) + ((lane & 7) ^ ((in & 15) >> 1)) * 16;
        }
        // dword 4 c + f of the wave's 64: position c of fragment 4 side + f of a part (of B those there are)
        const int f = 4 * side + (lane & 3), row = 128 * part + 16 * f + (lane >> 2), col = f8w::column<OUT_DT, FB>(part, f < FB ? f : FB - 1, lane >> 2);
        offSA = row < T.rows ? row : T.rows - 1;
        offSB = col < T.cols ? col : T.cols - 1;
        pA = uniform(P.A + T.m0 * pitch + (int64_t)T.k0 * KT);
        pB = uniform(P.B + (T.b0 + T.n0) * pitch + (int64_t)T.k0 * KT);
        pSA = uniform(P.A_scales + T.k0 * P.a_rows + T.m0);
        pSB = uniform(P.B_scales + T.k0 * P.b_rows + T.b0 + T.n0);
        step = KT;
        stepSA = P.a_rows;
        stepSB = P.b_rows;
        asm volatile("s_nop 4");  // (a lane read's register as an address, five wait states later)
    };
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds, dstA = __builtin_amdgcn_readfirstlane(lds0 + (128 * part + 32 * side) * KT),
                   dstB = __builtin_amdgcn_readfirstlane(lds0 + (BM + 16 * FB * part + 8 * HB * side) * KT),
                   dstS = __builtin_amdgcn_readfirstlane(lds0 + G::SCALES0 + wave * 256);
    // load i of a K tile: of the first ones (A0, P = half ST of B, scales) and of the second (Q, A1)
    auto request_first = [&](auto st, auto i) {
        constexpr int S = decltype(st)::value, I = decltype(i)::value;
        if constexpr (I < 4) f8w::load<S * STAGE + I * 1024>(dstA, offA[I], pA);
        else if constexpr (I < 4 + HB) f8w::load<S * STAGE + S * HB * 2048 + (I - 4) * 1024>(dstB, offB[HB * S + I - 4], pB);
        else if constexpr (I == 4 + HB) f8w::load_byte<S * G::SCALES>(dstS, offSA, pSA);
        else f8w::load_byte<S * G::SCALES + 1024>(dstS, offSB, pSB);
    };
    auto request_second = [&](auto st, auto i) {
        constexpr int S = decltype(st)::value, I = decltype(i)::value;
        if constexpr (I < HB) f8w::load<S * STAGE + (1 - S) * HB * 2048 + I * 1024>(dstB, offB[HB * (1 - S) + I], pB);
        else f8w::load<S * STAGE + 8192 + (I - HB) * 1024>(dstA, offA[4 + I - HB], pA);
    };
    auto advance = [&]() {
        pA += step;
        pB += step;
        pSA += stepSA;
        pSB += stepSB;
    };
    auto past_end = [&]() {
#pragma unroll
        for (int i = 0; i < 8; ++i) offA[i] = 0;
#pragma unroll
        for (int i = 0; i < FB; ++i) offB[i] = 0;
        offSA = offSB = 0;
        pA = P.A;
        pB = P.B;
        pSA = P.A_scales;
        pSB = P.B_scales;
        step = stepSA = stepSB = 0;
    };
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    // K tiles 0 and 1 of an output tile
    auto request_start = [&](const Tile &T) {
        point_to(T);
        f8w::each<0, G::FIRST>([&](auto i) { request_first(I0{}, i); });
        f8w::each<0, G::SECOND>([&](auto i) { request_second(I0{}, i); });
        advance();
        if (T.count < 2) past_end();
        f8w::each<0, G::FIRST>([&](auto i) { request_first(I1{}, i); });
        f8w::each<0, G::SECOND>([&](auto i) { request_second(I1{}, i); });
        advance();
    };

    // ---- LDS -> registers: fragment f of the wave's rows of A, of its columns
    const int s0 = (q ^ (c >> 1)) << 4;
    const uint8_t *baseA[2][2], *baseB[2][2];  // [stage][half of the row]
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            baseA[s][h] = lds + s * STAGE + (wm * 128 + c) * KT + (s0 ^ (64 * h));
            baseB[s][h] = lds + s * STAGE + (BM + wn * 16 * FB + c) * KT + (s0 ^ (64 * h));
            uint32_t v = (uint32_t)(uintptr_t)(lds_ptr_t)baseA[s][h], w = (uint32_t)(uintptr_t)(lds_ptr_t)baseB[s][h];
            asm volatile("" : "+v"(v), "+v"(w));  // (an LDS instruction's constant does not reach the second stage: bases that the compiler keeps)
            baseA[s][h] = (const uint8_t *)(lds_ptr_t)(uintptr_t)v;
            baseB[s][h] = (const uint8_t *)(lds_ptr_t)(uintptr_t)w;
        }
    const uint8_t *baseSA = lds + G::SCALES0 + (wm * 128 + 4 * c) * 4, *baseSB = lds + G::SCALES0 + 1024 + (wn * 128 + 4 * c) * 4;
    // everything but the last n loads (and stores) has landed and all of the wave's LDS reads are done; then the same of every wave
#define NVFP4_F8W_WAIT(n) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(n) : "memory");
#define NVFP4_F8W_BARRIER               \
    __builtin_amdgcn_s_barrier(); \
    asm volatile("" ::: "memory");

    const int tiles = ntx * nty * (MODE == FP8_EXPERTS_DW || DIVIDED ? P.groups : 1);
    int id = (int)blockIdx.x;
    if (id >= tiles) return;
    uint32_t keep, next_keep = 0;
    Tile T = find(id, keep);
    request_start(T);
    NVFP4_F8W_WAIT(ALL)
    while (true) {
        // here: K tile 0 has landed, as far as this wave is concerned
        float4v_t acc[8][FB];
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
            for (int b = 0; b < FB; ++b) acc[a][b] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};
        Codes A[8], B[FB];
        bool beyond = false;  // (exact sums) a block that bf16 does not hold
        auto read_a = [&](int st, int f, int h) { (h ? A[f].hi : A[f].lo) = *reinterpret_cast<const u32x4_t *>(baseA[st][h] + 16 * f * KT); };
        auto read_b = [&](int st, int f, int h) { (h ? B[f].hi : B[f].lo) = *reinterpret_cast<const u32x4_t *>(baseB[st][h] + 16 * f * KT); };
        // scales of fragments 4 i .. 4 i + 3 of the wave's part of A and of B, of tiles of either stage
        u32x4_t SA[2][2], SB[2][2];
        auto read_scales = [&](int st, int i) {
            (i < 2 ? SA[st][i & 1] : SB[st][i & 1]) = *reinterpret_cast<const u32x4_t *>((i < 2 ? baseSA : baseSB) + st * G::SCALES + (i & 1) * 256);
        };
            int kt = 0;
        // stage ST, which is also the half P of B
        auto tile = [&](auto stage) {
            constexpr int ST = decltype(stage)::value;
            using HP = std::integral_constant<int, ST>;
            using HQ = std::integral_constant<int, 1 - ST>;
            if (kt + 2 >= T.count) past_end();
            asm volatile("s_nop 1");  // (accumulators that were just cleared: two instructions between that and the MFMAs)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (exact_sums(OUT_DT)) {
                // Halves as bf16: of A the one that is multiplied, of B both.  The compiler arranges what is between the barriers.
                Expanded EA[4], EB[FB];
                auto expand_a = [&](int h) {
#pragma unroll
                    for (int f = 0; f < 4; ++f) EA[f] = expand(A[4 * h + f], SA[ST][h][f]);
                };
                auto expand_b = [&](int h) {
#pragma unroll
                    for (int f = HB * h; f < HB * h + HB; ++f) EB[f] = expand(B[f], SB[ST][f >> 2][f & 3]);
                };
                auto quarter = [&](int ha, int hb) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int f = HB * hb; f < HB * hb + HB; ++f)
#pragma unroll
                            for (int a = 0; a < 4; ++a) multiply(acc[4 * ha + a][f], EB[f], EA[a], i);
                };
                // Blocks that bf16 does not hold, in a tile with scale bytes that may be such.  (A0 and P are in registers, and their places others' to write; Q and A1
                // stay until the barrier.)
                uint32_t least_a = ~0u, most_a = 0, least_b = ~0u, most_b = 0;
#pragma unroll
                for (int f = 0; f < 8; ++f) extend(least_a, most_a, SA[ST][f >> 2][f & 3]);
#pragma unroll
                for (int f = 0; f < FB; ++f) extend(least_b, most_b, SB[ST][f >> 2][f & 3]);
                if (__builtin_expect(suspects(least_a, most_a, least_b, most_b), 0)) {
                    auto there = [&](const uint8_t *const (&base)[2], int f) -> Codes {
                        return {*reinterpret_cast<const u32x4_t *>(base[0] + 16 * f * KT), *reinterpret_cast<const u32x4_t *>(base[1] + 16 * f * KT)};
                    };
#pragma unroll
                    for (int f = 0; f < 8; ++f) beyond |= (f < 4 ? A[f] : there(baseA[ST], f)).beyond(SA[ST][f >> 2][f & 3]);
#pragma unroll
                    for (int f = 0; f < FB; ++f) beyond |= (f / HB == ST ? B[f] : there(baseB[ST], f)).beyond(SB[ST][f >> 2][f & 3]);
                }
                f8w::each<0, G::FIRST>([&](auto i) { request_first(stage, i); });
                expand_a(0);
                expand_b(ST);
#pragma unroll
                for (int i = 0; i < 2 * HB; ++i) read_b(ST, HB * (1 - ST) + (i >> 1), i & 1);
                quarter(0, ST);
#pragma unroll
                for (int i = 0; i < 8; ++i) read_a(ST, 4 + (i >> 1), i & 1);
                expand_b(1 - ST);
                quarter(0, 1 - ST);
                NVFP4_F8W_WAIT(ALL)
                NVFP4_F8W_BARRIER
                f8w::each<0, G::SECOND>([&](auto i) { request_second(stage, i); });
                expand_a(1);
#pragma unroll
                for (int i = 0; i < 8; ++i) read_a(1 - ST, i >> 1, i & 1);
                quarter(1, 1 - ST);
#pragma unroll
                for (int i = 0; i < 2 * HB; ++i) read_b(1 - ST, HB * (1 - ST) + (i >> 1), i & 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) read_scales(1 - ST, i);
                quarter(1, ST);
                advance();
                NVFP4_F8W_WAIT(ALL)
                NVFP4_F8W_BARRIER
                ++kt;
                return;
            }
            // MFMA j of a quarter: along a row of tiles and back along the next, one operand changes at a time
            auto quarter = [&](auto ha, auto hb, auto &&between) {
                f8w::each<0, 4 * HB>([&](auto j) {
                    constexpr int J = decltype(j)::value, r = J / HB, i = r & 1 ? HB - 1 - J % HB : J % HB;
                    constexpr int a = 4 * decltype(ha)::value + r, b = HB * decltype(hb)::value + i;
                    f8w::mfma(acc[a][b], B[b].all(), A[a].all(), SB[ST][b >> 2][b & 3], SA[ST][a >> 2][a & 3]);
                    __builtin_amdgcn_sched_barrier(0);
                    between(j);
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            // what goes between the MFMAs, N things from MFMA `from` on, spread over those that are left
            auto spread = [&](auto j, auto from, auto n, auto &&f) {
                constexpr int J = decltype(j)::value, F = decltype(from)::value, N = decltype(n)::value, L = 4 * HB - F;
                if constexpr (J >= F) f8w::each<(J - F) * N / L, (J - F + 1) * N / L>(f);
            };
            using F0 = std::integral_constant<int, 0>;
            using FH = std::integral_constant<int, 2 * HB>;
            using Frags = std::integral_constant<int, 8>;
            quarter(I0{}, HP{}, [&](auto j) {
                if constexpr (decltype(j)::value < 2 * HB) read_b(ST, HB * (1 - ST) + (decltype(j)::value >> 1), decltype(j)::value & 1);
                spread(j, F0{}, std::integral_constant<int, G::FIRST>{}, [&](auto i) { request_first(stage, i); });
            });
            quarter(I0{}, HQ{}, [&](auto j) { spread(j, F0{}, Frags{}, [&](auto i) { read_a(ST, 4 + (decltype(i)::value >> 1), decltype(i)::value & 1); }); });
            NVFP4_F8W_WAIT(ALL)
            NVFP4_F8W_BARRIER
            __builtin_amdgcn_sched_barrier(0);
            quarter(I1{}, HQ{}, [&](auto j) {
                spread(j, F0{}, Frags{}, [&](auto i) { read_a(1 - ST, decltype(i)::value >> 1, decltype(i)::value & 1); });
                spread(j, F0{}, std::integral_constant<int, G::SECOND>{}, [&](auto i) { request_second(stage, i); });
            });
            advance();
            quarter(I1{}, HP{}, [&](auto j) {
                if constexpr (decltype(j)::value < 2 * HB) read_b(1 - ST, HB * (1 - ST) + (decltype(j)::value >> 1), decltype(j)::value & 1);
                spread(j, FH{}, std::integral_constant<int, 4>{}, [&](auto i) { read_scales(1 - ST, decltype(i)::value); });
            });
            NVFP4_F8W_WAIT(ALL)
            NVFP4_F8W_BARRIER
            ++kt;
        };
        NVFP4_F8W_BARRIER
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_a(0, f, h);
                if (f < HB) read_b(0, f, h);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) read_scales(0, i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        NVFP4_F8W_BARRIER
        while (kt + 2 <= T.count) {
            tile(I0{});
            tile(I1{});
        }
        if (kt < T.count) tile(I0{});
        // Every wave has read all that it needed: the next tile's loads may follow (behind this one's past its end, to the same places, of which each
        // has one wave that loads it).
        id += (int)gridDim.x;
        Tile next = T;
        if (id < tiles) {
            next = find(id, next_keep);
            request_start(next);
        }
        asm volatile("s_nop 15" ::: "memory");
        // The next tile's first K tile has landed when its second and what was stored behind that (STORES inside the output, as few as none at its
        // edge) are all that is outstanding.
        auto store = [&](auto inside, auto streamed) {
            int at_lane = lane;
            asm volatile("" : "+v"(at_lane));  // (or the addresses are computed before the K loop and kept)
            const int c = at_lane & 15, q = at_lane >> 4;
            constexpr bool IN = decltype(inside)::value != 0, STREAMED = decltype(streamed)::value != 0;
            // words of row 16 a + c that fill 64 bytes in four lanes (bf16: fragments 2 s and 2 s + 1; binary32: fragment s)
            auto words = [&](int a, int s) -> u32x4_t {
                if constexpr (OUT_DT == NVFP4_F32) return __builtin_bit_cast(u32x4_t, acc[a][s]) & keep;
                float v[8];
                // (reads that stay behind the wait states and leave the accumulators alone)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if constexpr (exact_sums(OUT_DT)) v[i] = acc[a][2 * s + (i >> 2)][i & 3];
                    else asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[i]) : "a"(acc[a][2 * s + (i >> 2)][i & 3]));
                }
                return to_bf16(v) & keep;
            };
            constexpr int EACH = OUT_DT == NVFP4_F32 ? 16 : 32, N = 16 * FB / EACH;  // columns of such 64 bytes; how many
#pragma unroll
            for (int a = 0; a < 8; ++a) {
                const int64_t top = T.out + T.m0 + wm * 128 + 16 * a;
                auto col_of = [&](int s) { return f8w::columns_of<FB>(wn, s * EACH / 16) + (FB == 6 && s * EACH >= 64 ? s * EACH - 64 : s * EACH); };
                auto one = [&](int s) {
                    const int row = wm * 128 + 16 * a + c, col = col_of(s) + q * (EACH / 4);
                    const u32x4_t w = words(a, s);
                    if (IN || (row < T.rows && col < T.cols)) store_lane<OUT_DT, STREAMED>(P.out, (top + c) * P.ldc + T.n0 + col, w, IN ? 16 : T.cols - col);
                };
#pragma unroll
                for (int s = 0; s < N; s += 2) {
                    if (!IN || s + 1 == N) {
                        one(s);
                        if (s + 1 < N) one(s + 1);
                        continue;
                    }
                    u32x4_t w = words(a, s), x = words(a, s + 1);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t lo = w[i], hi = x[i];
                        f8w::exchange(lo, hi);
                        w[i] = lo;
                        x[i] = hi;
                    }
                    const int64_t at = (top + (c & 7)) * P.ldc + T.n0 + col_of(s) + (c >> 3) * EACH + q * (EACH / 4);
                    store_lane<OUT_DT, STREAMED>(P.out, at, w, 16);
                    store_lane<OUT_DT, STREAMED>(P.out, at + 8 * P.ldc, x, 16);
                }
            }
            NVFP4_F8W_WAIT(ALL + (decltype(inside)::value != 0 ? G::STORES : 0))
        };
        bool again = false;
        if constexpr (exact_sums(OUT_DT)) again = keep != 0 && __ballot(beyond) != 0;  // (what no row holds may be anything)
        if (__builtin_expect(again, 0)) {
#pragma unroll 1
            for (int f = 0; f < 8 * FB; ++f) {
                const int row = wm * 128 + 16 * (f / FB) + c, s = f8w::column<OUT_DT, FB>(wn, f % FB, c), col = f8w::column<OUT_DT, FB>(wn, f % FB, 4 * q);
                const int64_t ra = T.m0 + (row < T.rows ? row : T.rows - 1), rb = T.b0 + T.n0 + (s < T.cols ? s : T.cols - 1);
                const float4v_t v = multiply_codes(P, P.B + rb * pitch + q * 16, P.B_scales + rb, P.A + ra * pitch + q * 16, P.A_scales + ra, T.k0, 1, T.k0 + T.count);
                if (DIVIDED) reinterpret_cast<float4v_t *>(P.partial)[(T.out * 4 + wave) * (8 * FB * 64) + f * 64 + lane] = v;
                else
                    for (int i = 0; i < 4; ++i)
                        if (row < T.rows && col + i < T.cols) store_one<OUT_DT>(P.out, (T.out + T.m0 + row) * P.ldc + T.n0 + col + i, v[i]);
            }
            NVFP4_F8W_WAIT(ALL)
        } else if constexpr (DIVIDED) {
            // as they are, a fragment's 64 lanes together; fragments past the last row are nobody's
            float4v_t *const to = reinterpret_cast<float4v_t *>(P.partial) + (T.out * 4 + wave) * (8 * FB * 64) + lane;
#pragma unroll
            for (int a = 0; a < 8; ++a) {
                if (wm * 128 + 16 * a >= T.rows) continue;
#pragma unroll
                for (int b = 0; b < FB; ++b) {
                    float4v_t v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (exact_sums(OUT_DT)) v[i] = acc[a][b][i];
                        else asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v[i]) : "a"(acc[a][b][i]));
                    }
                    to[(a * FB + b) * 64] = v;
                }
            }
            NVFP4_F8W_WAIT(ALL)
        } else if (T.rows != BM || T.cols != BN) store(I0{}, I0{});
        else if (P.stream) store(I1{}, I1{});
        else store(I1{}, I0{});
        if (id >= tiles) break;
        T = next;
        keep = next_keep;
    }
#undef NVFP4_F8W_BARRIER
#undef NVFP4_F8W_WAIT
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads past the end, before the workgroup's LDS is another's)
}

// out = the sums of the parts in their order.  A lane has two fragments' places beside each other, eight columns of a row.
template <int OUT_DT, int FB>
__global__ __launch_bounds__(256) void fp8_gemm_join_kernel(Fp8GemmArgs P, int ntx, int nty)
{
    using namespace f8g;
    constexpr int HB = FB / 2;
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    // pair s of fragments, fragment row a, wave and tile of this wave of the grid
    int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int s = id % HB, a = id / HB % 8, wave = id / (8 * HB) % 4, tile = id / (32 * HB);
    if (tile >= ntx * nty) return;
    const int ty = tile / ntx, tx = tile - ty * ntx, wm = wave >> 1, wn = wave & 1;
    const int64_t row = (int64_t)ty * f8w::BM + wm * 128 + 16 * a + c, col0 = (int64_t)tx * 32 * FB;
    if (row - c >= P.M) return;
    const float4v_t *from = reinterpret_cast<const float4v_t *>(P.partial) + ((int64_t)tile * 4 + wave) * (8 * FB * 64) + (a * FB + 2 * s) * 64 + lane;
    const int64_t part = (int64_t)ntx * nty * (32 * FB * 64);
    float4v_t v[2] = {from[0], from[64]};
    for (int p = 1; p < P.groups; p += 4) {
        float4v_t w[4][2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float4v_t *const at = from + (p + u < P.groups ? p + u : p) * part;
            w[u][0] = at[0];
            w[u][1] = at[64];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p + u < P.groups) {
                v[0] += w[u][0];
                v[1] += w[u][1];
            }
    }
    if (row >= P.M) return;
    if constexpr (OUT_DT == NVFP4_F32) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t col = col0 + f8w::column<OUT_DT, FB>(wn, 2 * s + h, 4 * q);
            if (col < P.N) store_lane<OUT_DT, false>(P.out, row * P.ldc + col, __builtin_bit_cast(u32x4_t, v[h]), P.N - col < 16 ? (int)(P.N - col) : 16);
        }
    } else {
        const float both[8] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
        const int64_t col = col0 + f8w::column<OUT_DT, FB>(wn, 2 * s, 4 * q);
        if (col < P.N) store_lane<OUT_DT, false>(P.out, row * P.ldc + col, to_bf16(both), P.N - col < 16 ? (int)(P.N - col) : 16);
    }
}

// Of the current device; a multiple of 8, so that a workgroup's tiles stay on its XCD's part of the walk
int64_t compute_units()
{
    static std::atomic<int> known[64];
    int device = 0, n = 0;
    if (hipGetDevice(&device) != hipSuccess) return 256;
    if (device >= 0 && device < 64 && (n = known[device].load(std::memory_order_relaxed)) != 0) return n;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || n < 8) n = 256;
    n = n / 8 * 8;
    if (device >= 0 && device < 64) known[device].store(n, std::memory_order_relaxed);
    return n;
}

template <int MODE, int OUT_DT, int FB>
static hipError_t launch_wide(const Fp8GemmArgs &P, hipStream_t st)
{
    using G = f8w::Geom<FB, OUT_DT>;
    auto *k = fp8_gemm_wide_kernel<MODE, OUT_DT, FB>;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, G::LDS_BYTES);
    if (once != hipSuccess) return once;
    const int64_t tiles = f8g::tiles<MODE == FP8_DIVIDED ? FP8_DENSE : MODE>(P, f8w::BM, G::BN) * (MODE == FP8_DIVIDED ? P.groups : 1), cus = compute_units();
    k<<<dim3((unsigned)(tiles < cus ? tiles : cus)), 256, G::LDS_BYTES, st>>>(P);
    if (MODE == FP8_DIVIDED) {
        const int ntx = (int)((P.N + G::BN - 1) / G::BN), nty = (int)((P.M + f8w::BM - 1) / f8w::BM);
        fp8_gemm_join_kernel<OUT_DT, FB><<<dim3((unsigned)(ntx * nty * 4 * FB)), 256, 0, st>>>(P, ntx, nty);
    }
    return hipGetLastError();
}

// Time of a K tile on every CU, us, by the tile's width (4096 x 4096 x 4096 and 2048 x 4096 x 4096, where tiles are one round and fewer than the CUs)
constexpr double K_TILE_128 = 0.67, K_TILE_192 = 0.92, K_TILE_256 = 1.2, K_TILE_F32 = 1.85;

// The tile's width: fewest rounds of the CUs, weighted by what a round takes.  us, 128 / 192 / 256 columns: 777 x 12288 x 4096 57 / 45 / 54, 4096 x 4096 x 4096
// 64 / 76 / 54, 2048 x 4096 x 4096 30 / 36 / 44, 2048 x 11008 x 4096 100 / 86 / 100, 4096 x 11008 x 4096 186 / 158 / 146, 3000 x 3000 x 1024 21 / 16 / 18,
// experts 4096 x 2 of 8, 4096 x 4096 134 / 144 / 139, 8192 x 2 of 16, 4096 x 2048 168 / 166 / 146.
static int width_of(const Fp8GemmArgs &P, int mode, int out_dt, double *cost)
{
    // (an expert's last tile of rows is half full on average)
    const int64_t cus = compute_units(), rows = mode == FP8_EXPERTS ? P.M / 256 + (P.groups + 1) / 2 : (P.M + 255) / 256 * (mode == FP8_EXPERTS_DW ? P.groups : 1);
    const double k_tile[3] = {K_TILE_128, K_TILE_192, K_TILE_256};
    int best = 4;
    *cost = 1e30;
    for (int fb = 4; fb <= (exact_sums(out_dt) ? 4 : 8); fb += 2) {
        const double c = (double)((rows * ((P.N + 32 * fb - 1) / (32 * fb)) + cus - 1) / cus) * (exact_sums(out_dt) ? K_TILE_F32 : k_tile[fb / 2 - 2]);
        if (c < *cost) {
            *cost = c;
            best = fb;
        }
    }
    return best;
}

double fp8_gemm_wide_cost(const Fp8GemmArgs &P, int mode, int out_dt)
{
    double cost;
    width_of(P, mode, out_dt, &cost);
    return cost;
}

// A dense product with fewer tiles than CUs: the tiles' width and in how many parts of at least PART K tiles the contraction goes to a workgroup each.  The sums of the
// parts leave as binary32 and are added by a second kernel: START, JOIN and JOIN_BYTES (a us, written and read) are what that costs, K tiles take longer than with all CUs
// at work.  us, whole / divided: 512 x 4096 x 11008 71 / 36, 1000 x 4096 x 11008 75 / 53, 256 x 4096 x 11008 43 / 27, 128 x 4096 x 11008 35 / 24, 1000 x 1024 x 8192 32 / 21,
// 512 x 4096 x 4096 24 / 21, binary32 1000 x 4096 x 4096 60 / 46; where this rule does not divide, 128 x 1024 x 8192 13.9 / 15.3, binary32 256 x 1024 x 8192 17.6 / 23.3.
constexpr int PART = 4, MOST_PARTS = 16;
constexpr double START = 3.0, JOIN = 5.0, JOIN_BYTES = 6e6, FEW_128 = 0.8, FEW_192 = 1.0, FEW_256 = 1.25;
static int divided_width(const Fp8GemmArgs &P, int out_dt, int *parts, size_t *bytes, double *cost)
{
    const int64_t cus = compute_units(), rows = (P.M + 255) / 256;
    const double k_tile[3] = {FEW_128, FEW_192, FEW_256};
    int best = 4;
    *parts = 1;
    *bytes = 0;
    *cost = 1e30;
    for (int fb = 4; fb <= (exact_sums(out_dt) ? 4 : 8); fb += 2) {
        const int64_t tiles = rows * ((P.N + 32 * fb - 1) / (32 * fb));
        for (int n = 1; n <= MOST_PARTS && n * tiles <= cus && (n == 1 || n * PART <= P.blocks); ++n) {
            const double c = (P.blocks + n - 1) / n * (exact_sums(out_dt) ? K_TILE_F32 : k_tile[fb / 2 - 2]) + START +
                             (n == 1 ? 0.0 : JOIN + 2.0 * n * (tiles / rows * 32 * fb) * ((P.M + 15) / 16 * 16) * 4 / JOIN_BYTES);
            if (c < *cost) {
                *cost = c;
                best = fb;
                *parts = n;
                *bytes = n == 1 ? 0 : (size_t)n * tiles * (256 * 32 * fb * 4);
            }
        }
    }
    return best;
}

int fp8_gemm_parts(const Fp8GemmArgs &P, int out_dt, double below, size_t *bytes, double *cost)
{
    int parts;
    if (below < START + JOIN + PART * FEW_128) return 1;  // (small products: no search)
    divided_width(P, out_dt, &parts, bytes, cost);
    return parts;
}

int fp8_gemm_wide_cols(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt)
{
    double cost;
    int parts;
    size_t bytes;
    return 32 * (mode == FP8_DIVIDED ? divided_width(P, out_dt, &parts, &bytes, &cost) : width_of(P, mode, out_dt, &cost));
}

template <int MODE>
static hipError_t launch_width(const Fp8GemmArgs &P, int out_dt, int cols, hipStream_t st)
{
    if (out_dt == NVFP4_F32) return launch_wide<MODE, NVFP4_F32, 4>(P, st);
    if (exact_sums(out_dt)) return launch_wide<MODE, NVFP4_BF16_EXACT, 4>(P, st);
    return cols == 128 ? launch_wide<MODE, NVFP4_BF16, 4>(P, st) : cols == 192 ? launch_wide<MODE, NVFP4_BF16, 6>(P, st) : launch_wide<MODE, NVFP4_BF16, 8>(P, st);
}

hipError_t launch_fp8_gemm_wide(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, int cols, hipStream_t st)
{
    if (mode == FP8_DIVIDED) return launch_width<FP8_DIVIDED>(P, out_dt, cols, st);
    return mode == FP8_DENSE ? launch_width<FP8_DENSE>(P, out_dt, cols, st)
           : mode == FP8_EXPERTS ? launch_width<FP8_EXPERTS>(P, out_dt, cols, st) : launch_width<FP8_EXPERTS_DW>(P, out_dt, cols, st);
}

}  // namespace nvfp4
