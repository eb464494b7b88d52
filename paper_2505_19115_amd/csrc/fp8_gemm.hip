// Products of quantized 8-bit operands ("NT": both stored with the contraction axis contiguous),
//     out[i, j] = sum_b 2^(sA[b,i] - 127) 2^(sB[b,j] - 127) sum_{k in b} cA[i,k] cB[j,k],
// on v_mfma_scale_f32_16x16x128_f8f6f4, which takes 128 contraction elements of 16 rows of each operand with the rows' scale bytes: one
// instruction is one block, and the scales cost nothing.  Products of codes are exact, sums are binary32.
//
// One body serves the dense product, the experts' (rows of A divided among weights) and the experts' weight gradients (a contraction
// divided among outputs): they differ in which rows and K tiles a workgroup's tile covers (Tile).
//
// Which row of a tile stands where.  Scales are block-major, so the bytes of a tile's rows are contiguous, and a lane can fetch the bytes of
// four fragments in one dword if these fragments' rows alternate: fragment j (of four) of rows 64 g .. 64 g + 63 has the rows 64 g + 4 c + j,
// c = 0 .. 15, and the instruction picks byte j.  The first MFMA operand is B's, whose fragments' rows become accumulator rows, so a lane
// (c, q) ends with 16 consecutive columns 64 g + 16 q .. + 15 of the output rows 64 g' + 4 c + j'.
#include "experts.h"

namespace nvfp4 {
namespace f8g {

typedef int int8v_t __attribute__((ext_vector_type(8)));
typedef float float4v_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2v_t __attribute__((ext_vector_type(2)));

constexpr int KT = FP8_BLOCK;

// What a workgroup multiplies: rows m0 .. m0 + rows - 1 of A (and of the output that starts at out) against rows n0 .. n0 + cols - 1 of B,
// K tiles k0 .. k0 + count - 1; b0 + column is a row of B.  rows <= 0: nothing.
struct Tile {
    int64_t m0, n0, b0, out;
    int rows, cols, k0, count;
};

template <int MODE>
__device__ __forceinline__ Tile find_tile(const Fp8GemmArgs &P, unsigned id, int BM, int BN)
{
    Tile T;
    const int ntx = (int)((P.N + BN - 1) / BN);
    T.k0 = 0;
    T.count = P.blocks;
    T.b0 = 0;
    T.out = 0;
    int ty = (int)(id / (unsigned)ntx), tx = (int)(id % (unsigned)ntx);
    int64_t left;
    if (MODE == FP8_EXPERTS) {
        // rows past the last expert's are a group of their own, with no K tile: zeros
        const int e = group_of_slot(P.offsets, P.groups + 1, (int32_t)P.M, BM, ty);
        if (e < 0) {
            T.rows = 0;
            return T;
        }
        RowGroup g;
        if (e < P.groups) {
            g = row_group(P.offsets, e, (int32_t)P.M);
        } else {
            int32_t a = P.offsets[P.groups];
            a = a < 0 ? 0 : a > (int32_t)P.M ? (int32_t)P.M : a;
            g = {a, (int32_t)P.M - a};
            T.count = 0;
        }
        const int b = ty - (g.first / BM + e);
        left = b < 0 ? 0 : (int64_t)g.count - (int64_t)b * BM;
        T.m0 = g.first + (int64_t)b * BM;
        T.b0 = e < P.groups ? e * P.N : 0;
    } else {
        if (MODE == FP8_EXPERTS_DW) {
            const int nty = (int)((P.M + BM - 1) / BM), e = ty / nty;
            ty -= e * nty;
            const RowGroup g = row_group(P.offsets, e, P.total);
            T.k0 = g.first / KT + e;
            T.count = (g.count + KT - 1) / KT;
            T.out = e * P.M;
        }
        T.m0 = (int64_t)ty * BM;
        left = P.M - T.m0;
    }
    T.n0 = (int64_t)tx * BN;
    T.rows = (int)(left < BM ? left : BM);
    T.cols = (int)(P.N - T.n0 < BN ? P.N - T.n0 : BN);
    return T;
}

// Sixteen columns of one row from a lane's accumulators v[4 i + j] = column 4 i + j.  Rows of the output start at any element.
template <int OUT_DT>
__device__ __forceinline__ void store_sixteen(void *out, int64_t at, const float (&v)[16], int n)
{
    if (OUT_DT == NVFP4_F32) {
        struct __attribute__((packed, aligned(4))) P { u32x4_t w; };
        float *const p = reinterpret_cast<float *>(out) + at;
        if (n >= 16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x4_t w = {__float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3])};
                reinterpret_cast<P *>(p)[i].w = w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < n) p[i] = v[i];
        }
    } else {
        struct __attribute__((packed, aligned(2))) P { u32x4_t w; };
        uint16_t *const p = reinterpret_cast<uint16_t *>(out) + at;
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2v_t f = {v[2 * i], v[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
        }
        if (n >= 16) {
            const u32x4_t lo = {w[0], w[1], w[2], w[3]}, hi = {w[4], w[5], w[6], w[7]};
            reinterpret_cast<P *>(p)[0].w = lo;
            reinterpret_cast<P *>(p)[1].w = hi;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}

}  // namespace f8g

// 128 x 128 tiles: 2 x 2 waves of 64 x 64, two LDS stages of one K tile, filled through registers.
// LDS: a row's 128 bytes are eight chunks of 16; tile row 64 g + 4 c + j stands at position 64 g + 16 j + c, its chunk h at slot
// h ^ ((c / 2) % 8), and lane (c, q) takes chunks q and q + 4 of its rows, of both operands alike: the sixteen lanes that the LDS serves at
// a time read sixteen different pieces of its 256-byte period.
template <int MODE, int OUT_DT>
__global__ __launch_bounds__(256, 2) void fp8_gemm_kernel(Fp8GemmArgs P)
{
    using namespace f8g;
    constexpr int BM = 128, BN = 128, STAGE = (BM + BN) * KT;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, q = lane >> 4;
    const int wm = wave >> 1, wn = wave & 1;
    const Tile T = find_tile<MODE>(P, blockIdx.x, BM, BN);
    if (T.rows <= 0) return;
    const int64_t pitch = (int64_t)P.blocks * KT;

    // thread t stages chunk t % 8 of positions t / 8 + 32 u; rows past the edge repeat the last one
    const uint8_t *pa[4], *pb[4];
    int to[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int p = (tid >> 3) + 32 * u, row = (p & 64) + 4 * (p & 15) + ((p >> 4) & 3), chunk = tid & 7;
        to[u] = p * KT + ((chunk ^ ((p >> 1) & 7)) << 4);
        pa[u] = P.A + (T.m0 + (row < T.rows ? row : T.rows - 1)) * pitch + (int64_t)T.k0 * KT + chunk * 16;
        pb[u] = P.B + (T.b0 + T.n0 + (row < T.cols ? row : T.cols - 1)) * pitch + (int64_t)T.k0 * KT + chunk * 16;
    }
    u32x4_t ga[4], gb[4];
    auto fetch = [&](int kt) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            ga[u] = *reinterpret_cast<const u32x4_t *>(pa[u] + (int64_t)kt * KT);
            gb[u] = *reinterpret_cast<const u32x4_t *>(pb[u] + (int64_t)kt * KT);
        }
    };
    auto stash = [&](int st) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            *reinterpret_cast<u32x4_t *>(lds + st * STAGE + to[u]) = ga[u];
            *reinterpret_cast<u32x4_t *>(lds + st * STAGE + BM * KT + to[u]) = gb[u];
        }
    };
    // the bytes of rows 4 c .. 4 c + 3 of the wave's 64, clamped one by one at the edge
    auto scales = [&](const uint8_t *s, int64_t rows, int64_t first, int have, int kt) -> uint32_t {
        const uint8_t *p = s + (int64_t)(T.k0 + kt) * rows + first;
        uint32_t w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = 4 * c + j < have ? 4 * c + j : have - 1;
            w |= (uint32_t)p[r < 0 ? 0 : r] << (8 * j);
        }
        return w;
    };
    float4v_t acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int ma = wm * 64 < T.rows ? wm * 64 : 0, nb = wn * 64 < T.cols ? wn * 64 : 0;  // (a wave past the edge computes what nobody stores)
    if (T.count > 0) {
        fetch(0);
        stash(0);
    }
    __syncthreads();
    for (int kt = 0; kt < T.count; ++kt) {
        const bool more = kt + 1 < T.count;
        if (more) fetch(kt + 1);
        const uint32_t sa = scales(P.A_scales, P.a_rows, T.m0 + ma, T.rows - ma, kt);
        const uint32_t sb = scales(P.B_scales, P.b_rows, T.b0 + T.n0 + nb, T.cols - nb, kt);
        const uint8_t *const base = lds + (kt & 1) * STAGE + c * KT, *const A = base + wm * 64 * KT, *const B = base + (BM + wn * 64) * KT;
        const int s0 = (q ^ (c >> 1)) << 4, s1 = ((q + 4) ^ (c >> 1)) << 4;
        int8v_t fa[4], fb[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x4_t a0 = *reinterpret_cast<const u32x4_t *>(A + 16 * j * KT + s0), a1 = *reinterpret_cast<const u32x4_t *>(A + 16 * j * KT + s1);
            const u32x4_t b0 = *reinterpret_cast<const u32x4_t *>(B + 16 * j * KT + s0), b1 = *reinterpret_cast<const u32x4_t *>(B + 16 * j * KT + s1);
            fa[j] = int8v_t{(int)a0[0], (int)a0[1], (int)a0[2], (int)a0[3], (int)a1[0], (int)a1[1], (int)a1[2], (int)a1[3]};
            fb[j] = int8v_t{(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
        }
#define NVFP4_F8_MFMA(a, b) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[b], fa[a], acc[a][b], 0, 0, b, sb, a, sa);
#define NVFP4_F8_MFMA_ROW(a) NVFP4_F8_MFMA(a, 0) NVFP4_F8_MFMA(a, 1) NVFP4_F8_MFMA(a, 2) NVFP4_F8_MFMA(a, 3)
        NVFP4_F8_MFMA_ROW(0) NVFP4_F8_MFMA_ROW(1) NVFP4_F8_MFMA_ROW(2) NVFP4_F8_MFMA_ROW(3)
#undef NVFP4_F8_MFMA_ROW
#undef NVFP4_F8_MFMA
        if (more) stash((kt + 1) & 1);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int row = wm * 64 + 4 * c + a, col = wn * 64 + 16 * q;
        float v[16];
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * i + b] = acc[a][b][i];
        if (row < T.rows && col < T.cols) store_sixteen<OUT_DT>(P.out, (T.out + T.m0 + row) * P.ldc + T.n0 + col, v, T.cols - col);
    }
}

template <int MODE>
static hipError_t launch(const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    constexpr int BM = 128, BN = 128, LDS = 2 * (BM + BN) * FP8_BLOCK;
    const int64_t ntx = (P.N + BN - 1) / BN, nty = (P.M + BM - 1) / BM;
    const int64_t tiles = ntx * (MODE == FP8_EXPERTS ? P.M / BM + P.groups + 1 : MODE == FP8_EXPERTS_DW ? nty * P.groups : nty);
    auto *k = out_dt == NVFP4_F32 ? fp8_gemm_kernel<MODE, NVFP4_F32> : fp8_gemm_kernel<MODE, NVFP4_BF16>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (e != hipSuccess) return e;
    k<<<dim3((unsigned)tiles), 256, LDS, st>>>(P);
    return hipGetLastError();
}

hipError_t launch_fp8_gemm(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, hipStream_t st)
{
    return mode == FP8_DENSE ? launch<FP8_DENSE>(P, out_dt, st) : mode == FP8_EXPERTS ? launch<FP8_EXPERTS>(P, out_dt, st) : launch<FP8_EXPERTS_DW>(P, out_dt, st);
}

}  // namespace nvfp4
