// 8-bit products with bf16 outputs on 256 x 256 tiles: 2 x 2 waves of 128 x 128 (8 x 8 MFMA tiles of 16 x 16, all 256 accumulator registers, one
// wave per SIMD).  A K tile is 64 MFMAs a wave, 32 cycles each, and 128 KB out of the LDS for the four of them, half of what it delivers
// in that time.
//
// LDS: two stages of one K tile, 32 KB of each operand, placed as in fp8_gemm.hip (row 64 g + 4 c + j at position 64 g + 16 j + c, chunk h at slot h ^ (c / 2)),
// written by direct global -> LDS loads whose lanes choose which chunk they fetch.  Rows past the edge are clamped to the last one.
//
// A K tile in quarters, halves of A against halves of B, a half's registers read again as soon as its last quarter is done; of B the half that
// the tile before ended without comes first (P, then Q):
//     A0 x P   while Q is read             A0 x Q   while A1 is read
//     ONE barrier, with every load of tile kt + 1 landed and this tile's stage read by every wave
//     A1 x Q   while A0 of kt + 1 is read  A1 x P   while Q of kt + 1 is read, the next tile's P;    tile kt + 2 is requested meanwhile
#include <type_traits>

#include "fp8_gemm.h"

namespace nvfp4 {
namespace f8w {

constexpr int BM = 256, BN = 256, KT = FP8_BLOCK;
constexpr int STAGE = (BM + BN) * KT, LDS_BYTES = 2 * STAGE;

// As assembly, so that the 64 accumulators stay where they are (gemm_mx.hip).  What the compiler does not know about it: an operand must not have been
// written by the vector ALU in the two instructions before (they come from LDS reads), and the last result must not be read for 11 wait
// states.  BA, BB: bytes of the scale registers.
template <int BB, int BA>
__device__ __forceinline__ void mfma(f8g::float4v_t &acc, const f8g::int8v_t &b, const f8g::int8v_t &a, uint32_t sb, uint32_t sa)
{
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%6,0] op_sel_hi:[%7,%8,0]"
                 : "+a"(acc)
                 : "v"(b), "v"(a), "v"(sb), "v"(sa), "n"(BB & 1), "n"(BA & 1), "n"(BB >> 1), "n"(BA >> 1));
}

// Assembly because the compiler takes a direct-to-LDS load for a possible writer of all of the LDS and would wait for it before the next LDS
// read; here a stage is read behind an explicit wait and barrier only.
template <int TO>
__device__ __forceinline__ void load(uint32_t dst, uint32_t off, const uint8_t *base)
{
    asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" : : "s"(dst), "n"(TO), "v"(off), "s"(base) : "memory", "scc", "m0");
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

    // ---- global -> LDS: instruction u of a wave fills positions 64 wave + 8 u .. + 7
    uint32_t offA[8], offB[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        const int at = (u & 1) * 8 + (lane >> 3), row = 64 * wave + 4 * at + (u >> 1), chunk = (lane & 7) ^ (at >> 1);
        offA[u] = (uint32_t)((row < T.rows ? row : T.rows - 1) * pitch) + chunk * 16;
        offB[u] = (uint32_t)((row < T.cols ? row : T.cols - 1) * pitch) + chunk * 16;
    }
    auto uniform = [](const uint8_t *p) -> const uint8_t * {
        const uint64_t v = reinterpret_cast<uint64_t>(p);
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
        return reinterpret_cast<const uint8_t *>(((uint64_t)hi << 32) | lo);
    };
    const uint8_t *pA = uniform(P.A + T.m0 * pitch + (int64_t)T.k0 * KT), *pB = uniform(P.B + (T.b0 + T.n0) * pitch + (int64_t)T.k0 * KT);  // next to be requested
    typedef __attribute__((address_space(3))) void *lds_ptr_t;
    const uint32_t dst = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_ptr_t)lds + wave * 8192);
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

    // scale bytes of the wave's rows in a K tile
    struct Scales {
        uint32_t a[2], b[2];
    };
    const int64_t sa0 = T.m0 + (wm * 128 < T.rows ? wm * 128 : 0), sb0 = T.b0 + T.n0 + (wn * 128 < T.cols ? wn * 128 : 0);
    const int sa1 = wm * 128 + 64 < T.rows ? 64 : 0, sb1 = wn * 128 + 64 < T.cols ? 64 : 0;  // (parts past the edge: the first bytes, for results that nobody stores)
    auto scales = [&](int kt) -> Scales {
        return {{four_scales(P.A_scales, P.a_rows, P.blocks, T.k0 + kt, sa0, c), four_scales(P.A_scales, P.a_rows, P.blocks, T.k0 + kt, sa0 + sa1, c)},
                {four_scales(P.B_scales, P.b_rows, P.blocks, T.k0 + kt, sb0, c), four_scales(P.B_scales, P.b_rows, P.blocks, T.k0 + kt, sb0 + sb1, c)}};
    };
    auto there = [](Scales &s) { asm volatile("" : "+v"(s.a[0]), "+v"(s.a[1]), "+v"(s.b[0]), "+v"(s.b[1])); };
    auto request = [&](auto st, auto i) {  // load i of 16 of a K tile
        constexpr int S = decltype(st)::value, U = decltype(i)::value & 7;
        if constexpr (decltype(i)::value < 8) {
            f8w::load<S * STAGE + U * 1024>(dst, offA[U], pA);
        } else {
            f8w::load<S * STAGE + BM * KT + U * 1024>(dst, offB[U], pB);
        }
    };
    Scales now, next;
    if (T.count > 0) {
        f8w::each<0, 16>([&](auto i) { request(std::integral_constant<int, 0>{}, i); });
        pA += KT;
        pB += KT;
        now = scales(0);
        if (T.count > 1) {
            f8w::each<0, 16>([&](auto i) { request(std::integral_constant<int, 1>{}, i); });
            pA += KT;
            pB += KT;
            next = scales(1);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        there(now);
        __syncthreads();
#pragma unroll
        for (int f = 0; f < 4; ++f)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                read_a(0, f, h);
                read_b(0, f, h);
            }
    }
    int kt = 0;
    // stage ST; P: the half of B that is there already
    auto tile = [&](auto stage) {
        constexpr int ST = decltype(stage)::value, Pb = ST, Qb = 1 - ST;
        // (the scales may just have been copied from register to register: two instructions between that and the MFMAs)
        asm volatile("s_nop 1" : "+v"(now.a[0]), "+v"(now.a[1]), "+v"(now.b[0]), "+v"(now.b[1]));
        __builtin_amdgcn_sched_barrier(0);
        auto one = [&](auto ia, auto ib) {
            constexpr int a = decltype(ia)::value, b = decltype(ib)::value;
            f8w::mfma<(b & 3), (a & 3)>(acc[a][b], B[b].all(), A[a].all(), now.b[b >> 2], now.a[a >> 2]);
        };
        // MFMA j of a quarter: along a row of tiles and back along the next, one operand changes at a time
        auto quarter = [&](auto ha, auto hb, auto &&between) {
            f8w::each<0, 16>([&](auto j) {
                constexpr int J = decltype(j)::value, r = J >> 2, i = r & 1 ? 3 - (J & 3) : J & 3;
                one(std::integral_constant<int, 4 * decltype(ha)::value + r>{}, std::integral_constant<int, 4 * decltype(hb)::value + i>{});
                __builtin_amdgcn_sched_barrier(0);
                between(j);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        using H0 = std::integral_constant<int, 0>;
        using H1 = std::integral_constant<int, 1>;
        using HP = std::integral_constant<int, Pb>;
        using HQ = std::integral_constant<int, Qb>;
        quarter(H0{}, HP{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_b(ST, 4 * Qb + (J >> 1), J & 1);
        });
        quarter(H0{}, HQ{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_a(ST, 4 + (J >> 1), J & 1);
        });
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        there(next);
        const bool more = kt + 2 < T.count;
        Scales later = next;
        if (more) later = scales(kt + 2);
        __builtin_amdgcn_sched_barrier(0);
        quarter(H1{}, HQ{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_a(1 - ST, J >> 1, J & 1);
            if (more) request(stage, j);
        });
        quarter(H1{}, HP{}, [&](auto j) {
            constexpr int J = decltype(j)::value;
            if constexpr (J < 8) read_b(1 - ST, 4 * Qb + (J >> 1), J & 1);
        });
        pA += KT;
        pB += KT;
        now = next;
        next = later;
        ++kt;
    };
    while (kt + 2 <= T.count) {
        tile(std::integral_constant<int, 0>{});
        tile(std::integral_constant<int, 1>{});
    }
    if (kt < T.count) tile(std::integral_constant<int, 0>{});
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
