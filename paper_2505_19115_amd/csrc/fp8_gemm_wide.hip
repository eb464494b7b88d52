// 8-bit products with bf16 outputs on 256 x 256 tiles: 2 x 2 waves of 128 x 128 (8 x 8 MFMA tiles of 16 x 16, all 256 accumulator registers, one
// wave per SIMD).  A K tile is 64 MFMAs a wave, 32 cycles each, and 128 KB out of the LDS for the four of them, half of what it delivers
// in that time.
//
// LDS: two stages of one K tile, 32 KB of each operand, placed as in fp8_gemm.hip (row 64 g + 4 c + j at position 64 g + 16 j + c, chunk h at slot h ^ (c / 2)), and
// its 512 scale bytes, a dword each in the rows' order, so that a lane's four fragments' come in one read.  All of it is written by direct global ->
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
#include <type_traits>

#include "fp8_gemm.h"

namespace nvfp4 {
namespace f8w {

constexpr int BM = 256, BN = 256, KT = FP8_BLOCK;
constexpr int STAGE = (BM + BN) * KT, SCALES = (BM + BN) * 4, SCALES0 = 2 * STAGE, LDS_BYTES = SCALES0 + 2 * SCALES;
constexpr int FIRST = 10, SECOND = 8;  // loads of a wave and K tile: A0, P and scales; Q and A1

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

template <int MODE>
__global__ __launch_bounds__(256) void fp8_gemm_wide_kernel(Fp8GemmArgs P)
{
    using namespace f8g;
    constexpr int BM = f8w::BM, BN = f8w::BN, STAGE = f8w::STAGE;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;
    const Tile T = find_tile<MODE>(P, blockIdx.x, BM, BN);
    if (T.rows <= 0) return;
    const int64_t pitch = (int64_t)P.blocks * KT;

    // ---- global -> LDS: instruction u of four of a half fills 8 of the wave's 32 positions of it.  (Half h: positions 64 h .. + 63 of
    // each 128.)
    uint32_t offA[8], offB[8];  // [half][u]
    const int first = 128 * (wave >> 1), second = 32 * (wave & 1);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int in = second + 8 * (i & 3) + (lane >> 3), at = in & 15, row = first + 64 * (i >> 2) + 4 * at + (in >> 4), chunk = (lane & 7) ^ (at >> 1);
        offA[i] = (uint32_t)((row < T.rows ? row : T.rows - 1) * pitch) + chunk * 16;
        offB[i] = (uint32_t)((row < T.cols ? row : T.cols - 1) * pitch) + chunk * 16;
    }
    const int srow = wave * 64 + lane;
    uint32_t offSA = srow < T.rows ? srow : T.rows - 1, offSB = srow < T.cols ? srow : T.cols - 1;
    auto uniform = [](const uint8_t *p) -> const uint8_t * {
        const uint64_t v = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return reinterpret_cast<const uint8_t *>(((uint64_t)hi << 32) | lo);
    };
    // K tile that is requested next
    const uint8_t *pA = uniform(P.A + T.m0 * pitch + (int64_t)T.k0 * KT), *pB = uniform(P.B + (T.b0 + T.n0) * pitch + (int64_t)T.k0 * KT);
    const uint8_t *pSA = uniform(P.A_scales + T.k0 * P.a_rows + T.m0), *pSB = uniform(P.B_scales + T.k0 * P.b_rows + T.b0 + T.n0);
    int64_t step = KT, stepSA = P.a_rows, stepSB = P.b_rows;
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds, dst = __builtin_amdgcn_readfirstlane(lds0 + (first + second) * KT),
                   dstS = __builtin_amdgcn_readfirstlane(lds0 + f8w::SCALES0 + wave * 256);
    // load i of a K tile: of the first ones (A0, P = half ST of B, scales) and of the second (Q, A1)
    auto request_first = [&](auto st, auto i) {
        constexpr int S = decltype(st)::value, I = decltype(i)::value;
        if constexpr (I < 4) f8w::load<S * STAGE + I * 1024>(dst, offA[I], pA);
        else if constexpr (I < 8) f8w::load<S * STAGE + BM * KT + S * 8192 + (I - 4) * 1024>(dst, offB[4 * S + I - 4], pB);
        else if constexpr (I == 8) f8w::load_byte<S * f8w::SCALES>(dstS, offSA, pSA);
        else f8w::load_byte<S * f8w::SCALES + 4 * BM>(dstS, offSB, pSB);
    };
    auto request_second = [&](auto st, auto i) {
        constexpr int S = decltype(st)::value, I = decltype(i)::value;
        if constexpr (I < 4) f8w::load<S * STAGE + BM * KT + (1 - S) * 8192 + I * 1024>(dst, offB[4 * (1 - S) + I], pB);
        else f8w::load<S * STAGE + 8192 + (I - 4) * 1024>(dst, offA[I], pA);
    };
    auto advance = [&]() {
        pA += step;
        pB += step;
        pSA += stepSA;
        pSB += stepSB;
    };
    auto past_end = [&]() {
#pragma unroll
        for (int i = 0; i < 8; ++i) offA[i] = offB[i] = 0;
        offSA = offSB = 0;
        pA = P.A;
        pB = P.B;
        pSA = P.A_scales;
        pSB = P.B_scales;
        step = stepSA = stepSB = 0;
    };

    // ---- LDS -> registers: fragment f of the wave's 128 rows of an operand
    const int s0 = (q ^ (c >> 1)) << 4;
    const uint8_t *baseA[2][2], *baseB[2][2];  // [stage][half of the row]
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            baseA[s][h] = lds + s * STAGE + (wm * 128 + c) * KT + (s0 ^ (64 * h));
            baseB[s][h] = lds + s * STAGE + (BM + wn * 128 + c) * KT + (s0 ^ (64 * h));
            uint32_t v = (uint32_t)(uintptr_t)(lds_ptr_t)baseA[s][h], w = (uint32_t)(uintptr_t)(lds_ptr_t)baseB[s][h];
            asm volatile("" : "+v"(v), "+v"(w));  // (an LDS instruction's constant does not reach the second stage: bases that the compiler keeps)
            baseA[s][h] = (const uint8_t *)(lds_ptr_t)(uintptr_t)v;
            baseB[s][h] = (const uint8_t *)(lds_ptr_t)(uintptr_t)w;
        }
    Codes A[8], B[8];
    auto read_a = [&](int st, int f, int h) { (h ? A[f].hi : A[f].lo) = *reinterpret_cast<const u32x4_t *>(baseA[st][h] + 16 * f * KT); };
    auto read_b = [&](int st, int f, int h) { (h ? B[f].hi : B[f].lo) = *reinterpret_cast<const u32x4_t *>(baseB[st][h] + 16 * f * KT); };

    float4v_t acc[8][8];
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 8; ++b) acc[a][b] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};

    // scales of fragments 4 i .. 4 i + 3 of the wave's part of A and of B, of tiles of either stage
    u32x4_t SA[2][2], SB[2][2];
    const uint8_t *baseSA = lds + f8w::SCALES0 + (wm * 128 + 4 * c) * 4, *baseSB = lds + f8w::SCALES0 + (BM + wn * 128 + 4 * c) * 4;
    auto read_scales = [&](int st, int i) {
        (i < 2 ? SA[st][i & 1] : SB[st][i & 1]) = *reinterpret_cast<const u32x4_t *>((i < 2 ? baseSA : baseSB) + st * f8w::SCALES + (i & 1) * 256);
    };
    // everything but the last n loads has landed and all of the wave's LDS reads are done; then the same of every wave
#define NVFP4_F8W_BARRIER(n)                                                    \
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(n) : "memory"); \
    __builtin_amdgcn_s_barrier();                                               \
    asm volatile("" ::: "memory");
    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    if (T.count > 0) {
        f8w::each<0, f8w::FIRST>([&](auto i) { request_first(I0{}, i); });
        f8w::each<0, f8w::SECOND>([&](auto i) { request_second(I0{}, i); });
        advance();
        if (T.count < 2) past_end();
        f8w::each<0, f8w::FIRST>([&](auto i) { request_first(I1{}, i); });
        f8w::each<0, f8w::SECOND>([&](auto i) { request_second(I1{}, i); });
        advance();
        NVFP4_F8W_BARRIER(f8w::FIRST + f8w::SECOND)
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_a(0, f, h);
                read_b(0, f, h);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) read_scales(0, i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    int kt = 0;
    // stage ST, which is also the half P of B
    auto tile = [&](auto stage) {
        constexpr int ST = decltype(stage)::value;
        using HP = std::integral_constant<int, ST>;
        using HQ = std::integral_constant<int, 1 - ST>;
        if (kt + 2 >= T.count) past_end();
        __builtin_amdgcn_sched_barrier(0);
        // MFMA j of a quarter: along a row of tiles and back along the next, one operand changes at a time
        auto quarter = [&](auto ha, auto hb, auto &&between) {
            f8w::each<0, 16>([&](auto j) {
                constexpr int J = decltype(j)::value, r = J >> 2, i = r & 1 ? 3 - (J & 3) : J & 3;
                constexpr int a = 4 * decltype(ha)::value + r, b = 4 * decltype(hb)::value + i;
                f8w::mfma(acc[a][b], B[b].all(), A[a].all(), SB[ST][b >> 2][b & 3], SA[ST][a >> 2][a & 3]);
                __builtin_amdgcn_sched_barrier(0);
                between(j);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        quarter(I0{}, HP{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_b(ST, 4 * (1 - ST) + (J >> 1), J & 1);
            if constexpr (J >= 16 - f8w::FIRST) request_first(stage, std::integral_constant<int, J - (16 - f8w::FIRST)>{});
        });
        quarter(I0{}, HQ{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_a(ST, 4 + (J >> 1), J & 1);
        });
        NVFP4_F8W_BARRIER(f8w::FIRST + f8w::SECOND)
        __builtin_amdgcn_sched_barrier(0);
        quarter(I1{}, HQ{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_a(1 - ST, J >> 1, J & 1);
            if constexpr (J >= 8) request_second(stage, std::integral_constant<int, J - 8>{});
        });
        advance();
        quarter(I1{}, HP{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_b(1 - ST, 4 * (1 - ST) + (J >> 1), J & 1);
            if constexpr (J >= 8 && J < 12) read_scales(1 - ST, J - 8);
        });
        NVFP4_F8W_BARRIER(f8w::FIRST + f8w::SECOND)
        ++kt;
    };
    while (kt + 2 <= T.count) {
        tile(I0{});
        tile(I1{});
    }
    if (kt < T.count) tile(I0{});
#undef NVFP4_F8W_BARRIER
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (the loads past the end, before the workgroup's LDS is another's)
    asm volatile("s_nop 15" ::: "memory");
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int b = 0; b < 8; ++b) asm volatile("" : "+a"(acc[a][b]));
#pragma unroll
    for (int a = 0; a < 8; ++a)
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const int row = wm * 128 + 64 * (a >> 2) + 4 * c + (a & 3), col = wn * 128 + 64 * g + 16 * q;
            float v[16];
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * i + b] = acc[a][4 * g + b][i];
            if (row < T.rows && col < T.cols) store_sixteen<NVFP4_BF16>(P.out, (T.out + T.m0 + row) * P.ldc + T.n0 + col, v, T.cols - col);
        }
}

template <int MODE>
static hipError_t launch_wide(const Fp8GemmArgs &P, hipStream_t st)
{
    auto *k = fp8_gemm_wide_kernel<MODE>;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, f8w::LDS_BYTES);
    if (once != hipSuccess) return once;
    k<<<dim3((unsigned)f8g::tiles<MODE>(P, f8w::BM, f8w::BN)), 256, f8w::LDS_BYTES, st>>>(P);
    return hipGetLastError();
}

bool fp8_gemm_is_wide(const Fp8GemmArgs &P, int mode)
{
    const int64_t ntx = (P.N + 255) / 256;
    if (mode == FP8_DENSE) return ntx * ((P.M + 255) / 256) >= 128;
    if (mode == FP8_EXPERTS) return ntx * (P.M / 256) >= 128 && P.M >= 128 * (int64_t)P.groups;
    return ntx * ((P.M + 255) / 256) * P.groups >= 128;
}

hipError_t launch_fp8_gemm_wide(const Fp8GemmArgs &P, Fp8Mode mode, hipStream_t st)
{
    return mode == FP8_DENSE ? launch_wide<FP8_DENSE>(P, st) : mode == FP8_EXPERTS ? launch_wide<FP8_EXPERTS>(P, st) : launch_wide<FP8_EXPERTS_DW>(P, st);
}

}  // namespace nvfp4
