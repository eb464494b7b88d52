// 8-bit products of few rows (generation: a token of each of a few sequences; an expert with a handful of tokens).  Such a product reads B
// once and does little else, so nothing is staged: a workgroup has 16 columns and up to 64 rows, its waves divide the K tiles (wave w takes w, w + NW, ...), and
// every lane loads its own codes, 32 of a row and K tile, a batch of K tiles at a time.  The waves' sums are added through the LDS
// in the waves' order.
#include "fp8_gemm.h"

namespace nvfp4 {

// MT: fragments of 16 rows of A.  U: K tiles of a batch.
template <int MODE, int OUT_DT, int MT, int U, int NW>
__global__ __launch_bounds__(64 * NW) void fp8_gemm_thin_kernel(Fp8GemmArgs P)
{
    using namespace f8g;
    __shared__ float4v_t sums[NW][MT][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
    const Tile T = find_tile<MODE>(P, blockIdx.x, 16 * MT, 16);
    if (T.rows <= 0) return;
    const int64_t pitch = (int64_t)P.blocks * KT;
    const int64_t brow = T.b0 + T.n0 + (c < T.cols ? c : T.cols - 1);
    const uint8_t *const pb = P.B + brow * pitch + q * 16;
    const uint8_t *pa[MT];
    int64_t arow[MT];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int r = 16 * a + c;
        arow[a] = T.m0 + (r < T.rows ? r : T.rows - 1);
        pa[a] = P.A + arow[a] * pitch + q * 16;
    }
    float4v_t acc[MT];
#pragma unroll
    for (int a = 0; a < MT; ++a) acc[a] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int kt = wave; kt < T.count; kt += NW * U) {
        Codes fb[U], fa[U][MT];
        uint32_t sb[U], sa[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (past the last K tile: the last once more, and not multiplied)
            const int64_t k = kt + u * NW < T.count ? kt + u * NW : T.count - 1;
            fb[u].lo = *reinterpret_cast<const u32x4_t *>(pb + k * KT);
            fb[u].hi = *reinterpret_cast<const u32x4_t *>(pb + k * KT + 64);
            sb[u] = P.B_scales[k * P.b_rows + brow];
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                fa[u][a].lo = *reinterpret_cast<const u32x4_t *>(pa[a] + k * KT);
                fa[u][a].hi = *reinterpret_cast<const u32x4_t *>(pa[a] + k * KT + 64);
                sa[u][a] = P.A_scales[k * P.a_rows + arow[a]];
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kt + u * NW < T.count) {
                if constexpr (OUT_DT == NVFP4_F32) {
                    const Expanded b = expand(fb[u], sb[u]);
#pragma unroll
                    for (int a = 0; a < MT; ++a) multiply(acc[a], b, expand(fa[u][a], sa[u][a]));
                } else {
#pragma unroll
                    for (int a = 0; a < MT; ++a)
                        acc[a] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u].all(), fa[u][a].all(), acc[a], 0, 0, 0, sb[u], 0, sa[u][a]);
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a) sums[wave][a][lane] = acc[a];
    __syncthreads();
    // lane (c, q) of a wave: row c of fragment a, columns 4 q .. 4 q + 3
    for (int a = wave; a < MT; a += NW) {
        float4v_t s = sums[0][a][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += sums[w][a][lane];
        const int row = 16 * a + c, n = T.cols - 4 * q;
        const int64_t at = (T.out + T.m0 + row) * P.ldc + T.n0 + 4 * q;
        if (row < T.rows && n > 0) store_four<OUT_DT>(P.out, at, s, n);
    }
}

template <int MODE, int MT, int U, int NW>
static hipError_t launch_thin(const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    auto *k = out_dt == NVFP4_F32 ? fp8_gemm_thin_kernel<MODE, NVFP4_F32, MT, U, NW> : fp8_gemm_thin_kernel<MODE, NVFP4_BF16, MT, U, NW>;
    k<<<dim3((unsigned)f8g::tiles<MODE>(P, 16 * MT, 16)), 64 * NW, 0, st>>>(P);
    return hipGetLastError();
}

bool fp8_gemm_is_thin(const Fp8GemmArgs &P, int mode)
{
    return mode == FP8_DENSE ? P.M <= 64 : P.M <= 16 * (int64_t)P.groups;
}

hipError_t launch_fp8_gemm_thin(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, hipStream_t st)
{
    if (mode == FP8_EXPERTS) return launch_thin<FP8_EXPERTS, 1, 4, 8>(P, out_dt, st);
    if (P.M <= 16) return launch_thin<FP8_DENSE, 1, 4, 8>(P, out_dt, st);
    if (P.M <= 32) return launch_thin<FP8_DENSE, 2, 4, 8>(P, out_dt, st);
    return launch_thin<FP8_DENSE, 4, 2, 8>(P, out_dt, st);
}

}  // namespace nvfp4
