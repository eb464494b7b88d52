// 8-bit products of few rows (generation: a token of each of a few sequences; an expert with a handful of tokens).  Such a product reads B
// once and does little else, so nothing is staged: a workgroup has 16 columns and up to 64 rows, its waves divide the K tiles (wave w takes w, w + NW, ...), and
// every lane loads its own codes, 32 of a row and K tile, a batch of K tiles at a time.  The waves' sums are added through the LDS
// in the waves' order.
//
// What bounds it: loads in flight, and the first of them, which an expert's product asks for behind its offsets.  16 x 11008 x 4096 11.6 us, 3.9 TB/s; 16 x 16384 x
// 4096 15.7 us, 4.3 TB/s; 8 experts of 2048 x 4096, 16 rows 18.7 us, 3.6 TB/s (10.5, 12.8 and 17 where the last cache level has the weights); a token's 2 of them 7.0 us, where one 4096 x 4096 takes 5.1.  Without effect: lanes that load
// whole lines; slower: streaming loads (16 x 11008 x 4096 12.8 us), the experts' products on more columns (20 us) or more waves (20 us).
#include "fp8_gemm.h"

namespace nvfp4 {

// MT, TN: fragments of 16 rows of A and of 16 columns.  U: K tiles of a batch (a wave without so many loads its last once more and does not multiply it).
template <int MODE, int OUT_DT, int MT, int TN, int U, int NW>
// (the experts' binary32 outputs: registers for as many waves a SIMD as hide the loads; 64 x 8 of 64 experts, 1024 x 2048, 37.6 us for 42.9 with one less)
__global__ __launch_bounds__(64 * NW, MODE == FP8_EXPERTS && exact_sums(OUT_DT) ? (U == 4 ? 3 : U == 2 ? 4 : 5) : 1) void fp8_gemm_thin_kernel(Fp8GemmArgs P)
{
    using namespace f8g;
    __shared__ float4v_t sums[NW][MT * TN][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, q = lane >> 4;
    const Tile T = find_tile<MODE>(P, workgroup(), 16 * MT, 16 * TN);
    if (T.rows <= 0) return;
    const int64_t pitch = (int64_t)P.blocks * KT;
    // (rows past the edge repeat the last one)
    const uint8_t *pb[TN], *psb[TN], *pa[MT], *psa[MT];
#pragma unroll
    for (int b = 0; b < TN; ++b) {
        const int r = 16 * b + c;
        const int64_t row = T.b0 + T.n0 + (r < T.cols ? r : T.cols - 1);
        pb[b] = P.B + row * pitch + q * 16;
        psb[b] = P.B_scales + row;
    }
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int r = 16 * a + c;
        const int64_t row = T.m0 + (r < T.rows ? r : T.rows - 1);
        pa[a] = P.A + row * pitch + q * 16;
        psa[a] = P.A_scales + row;
    }
    float4v_t acc[MT][TN];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < TN; ++b) acc[a][b] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t least_a = ~0u, most_a = 0, least_b = ~0u, most_b = 0;  // (exact sums) scale bytes
    for (int kt = wave; kt < T.count; kt += NW * U) {
        Codes fb[U][TN], fa[U][MT];
        uint32_t sb[U][TN], sa[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (past the last K tile: the last once more, and not multiplied)
            const int64_t k = kt + u * NW < T.count ? kt + u * NW : T.count - 1;
#pragma unroll
            for (int b = 0; b < TN; ++b) {
                fb[u][b].lo = *reinterpret_cast<const u32x4_t *>(pb[b] + k * KT);
                fb[u][b].hi = *reinterpret_cast<const u32x4_t *>(pb[b] + k * KT + 64);
                sb[u][b] = psb[b][k * P.b_rows];
            }
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                fa[u][a].lo = *reinterpret_cast<const u32x4_t *>(pa[a] + k * KT);
                fa[u][a].hi = *reinterpret_cast<const u32x4_t *>(pa[a] + k * KT + 64);
                sa[u][a] = psa[a][k * P.a_rows];
            }
        }
        __builtin_amdgcn_sched_barrier(0);  // (all of a batch's loads first)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kt + u * NW < T.count) {
                if constexpr (exact_sums(OUT_DT)) {
                    Expanded ea[MT];
#pragma unroll
                    for (int a = 0; a < MT; ++a) ea[a] = expand(fa[u][a], sa[u][a]);
#pragma unroll
                    for (int b = 0; b < TN; ++b) {
                        const Expanded eb = expand(fb[u][b], sb[u][b]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int a = 0; a < MT; ++a) multiply(acc[a][b], eb, ea[a], i);
                    }
                } else {
#pragma unroll
                    for (int b = 0; b < TN; ++b)
#pragma unroll
                        for (int a = 0; a < MT; ++a)
                            acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[u][b].all(), fa[u][a].all(), acc[a][b], 0, 0, 0, sb[u][b], 0, sa[u][a]);
                }
            }
        }
        if constexpr (exact_sums(OUT_DT)) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int a = 0; a < MT; ++a) extend(least_a, most_a, sa[u][a]);
#pragma unroll
                for (int b = 0; b < TN; ++b) extend(least_b, most_b, sb[u][b]);
            }
        }
    }
    // blocks that bf16 does not hold, or of zeros: which, from memory (looked at above, codes would stay in registers longer)
    bool beyond = false;
    if (exact_sums(OUT_DT) && __builtin_expect(suspects(least_a, most_a, least_b, most_b), 0)) {
#pragma unroll 1
        for (int f = 0; f < MT + TN; ++f) {
            const int r = 16 * (f < MT ? f : f - MT) + c;
            const int64_t row = f < MT ? T.m0 + (r < T.rows ? r : T.rows - 1) : T.b0 + T.n0 + (r < T.cols ? r : T.cols - 1);
            beyond |= any_beyond((f < MT ? P.A : P.B) + row * pitch + q * 16, (f < MT ? P.A_scales : P.B_scales) + row, f < MT ? P.a_rows : P.b_rows, wave, NW, T.count);
        }
    }
    if (exact_sums(OUT_DT) && __builtin_expect(__ballot(beyond) != 0, 0)) {
#pragma unroll 1
        for (int f = 0; f < MT * TN; ++f) {
            const int r = 16 * (f / TN) + c, s = 16 * (f % TN) + c;
            const int64_t ra = T.m0 + (r < T.rows ? r : T.rows - 1), rb = T.b0 + T.n0 + (s < T.cols ? s : T.cols - 1);
            sums[wave][f][lane] = multiply_codes(P, P.B + rb * pitch + q * 16, P.B_scales + rb, P.A + ra * pitch + q * 16, P.A_scales + ra, wave, NW, T.count);
        }
    } else {
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int b = 0; b < TN; ++b) sums[wave][TN * a + b][lane] = acc[a][b];
    }
    __syncthreads();
    // lane (c, q) of a wave: row c of fragment a, columns 4 q .. 4 q + 3 of fragment b
    for (int f = wave; f < MT * TN; f += NW) {
        float4v_t s = sums[0][f][lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += sums[w][f][lane];
        const int row = 16 * (f / TN) + c, col = 16 * (f % TN) + 4 * q;
        if (row < T.rows && col < T.cols) store_four<OUT_DT>(P.out, (T.out + T.m0 + row) * P.ldc + T.n0 + col, s, T.cols - col);
    }
}

template <int MODE, int MT, int TN, int U, int NW>
static hipError_t launch_batches(const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    auto *k = out_dt == NVFP4_F32    ? fp8_gemm_thin_kernel<MODE, NVFP4_F32, MT, TN, U, NW>
              : out_dt == NVFP4_BF16 ? fp8_gemm_thin_kernel<MODE, NVFP4_BF16, MT, TN, U, NW>
                                     : fp8_gemm_thin_kernel<MODE, NVFP4_BF16_EXACT, MT, TN, U, NW>;
    k<<<launch_grid(f8g::tiles<MODE>(P, 16 * MT, 16 * TN)), 64 * NW, 0, st>>>(P);
    return hipGetLastError();
}

// (batches of no more K tiles than a wave has: 64 experts of 1024 x 2048 with 2 tokens each, 16 K tiles, 64 us in batches of 4 by 8 waves, 30 by 4)
static int batch_of(const Fp8GemmArgs &P, int most, int waves) { return most >= 4 && P.blocks >= 4 * waves ? 4 : most >= 2 && P.blocks >= 2 * waves ? 2 : 1; }
template <int MODE, int MT, int TN, int U, int NW>
static hipError_t launch_thin(const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    const int batch = batch_of(P, U, NW);
    if (batch == 4) return launch_batches<MODE, MT, TN, U < 4 ? U : 4, NW>(P, out_dt, st);
    if (batch == 2) return launch_batches<MODE, MT, TN, U < 2 ? U : 2, NW>(P, out_dt, st);
    return launch_batches<MODE, MT, TN, 1, NW>(P, out_dt, st);
}

// Shapes of a workgroup's output, rows and columns in 16s, and its largest batch.  What bounds these kernels is what a CU's loads bring, (MT + TN) * 16 rows of a K tile at
// 36 GB/s: the fewest rounds of the CUs times that.  us, 16 rows, 48 columns at most / 64: 16384 x 4096 18.3 / 15.5, 28672 x 4096 32.5 / 28.3, 12288 x 4096 13.0 / 12.1.
namespace f8t {
struct Shape {
    int mt, tn, u;
};
constexpr Shape SHAPES[] = {{1, 1, 4}, {1, 2, 4}, {1, 3, 4}, {1, 4, 4}, {2, 1, 4}, {2, 2, 2}, {2, 3, 2}, {2, 4, 2}, {4, 2, 2}, {4, 3, 1}, {4, 4, 1}};
constexpr int N_SHAPES = sizeof(SHAPES) / sizeof(SHAPES[0]), WAVES = 8;
constexpr Shape EXPERTS = {1, 2, 4};
constexpr int EXPERTS_WAVES = 4;
constexpr double PER_16_ROWS = 0.057;  // us

inline int64_t workgroups(const Fp8GemmArgs &P, Shape s)
{
    return (P.M + 16 * s.mt - 1) / (16 * s.mt) * ((P.N + 16 * s.tn - 1) / (16 * s.tn));
}
}  // namespace f8t

static int shape_of(const Fp8GemmArgs &P, double *cost)
{
    const int64_t cus = compute_units();
    int best = 0;
    *cost = 1e30;
    for (int i = 0; i < f8t::N_SHAPES; ++i) {
        const f8t::Shape s = f8t::SHAPES[i];
        const double c = (double)((f8t::workgroups(P, s) + cus - 1) / cus) * (s.mt + s.tn) * f8t::PER_16_ROWS;
        if (c < *cost) {
            *cost = c;
            best = i;
        }
    }
    return best;
}

double fp8_gemm_thin_cost(const Fp8GemmArgs &P)
{
    double cost;
    shape_of(P, &cost);
    return cost;
}

void fp8_gemm_thin_choice(const Fp8GemmArgs &P, Fp8Mode mode, Fp8Choice *c)
{
    double cost;
    const f8t::Shape s = mode == FP8_EXPERTS ? f8t::EXPERTS : f8t::SHAPES[shape_of(P, &cost)];
    c->rows = 16 * s.mt;
    c->cols = 16 * s.tn;
    c->parts = batch_of(P, s.u, mode == FP8_EXPERTS ? f8t::EXPERTS_WAVES : f8t::WAVES);
}

template <int I>
static hipError_t launch_shape(const Fp8Choice &c, const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    constexpr f8t::Shape S = f8t::SHAPES[I];
    if (c.rows == 16 * S.mt && c.cols == 16 * S.tn) return launch_thin<FP8_DENSE, S.mt, S.tn, S.u, f8t::WAVES>(P, out_dt, st);
    if constexpr (I + 1 < f8t::N_SHAPES) return launch_shape<I + 1>(c, P, out_dt, st);
    return hipErrorInvalidValue;
}

hipError_t launch_fp8_gemm_thin(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, const Fp8Choice &c, hipStream_t st)
{
    if (mode == FP8_EXPERTS) return launch_thin<FP8_EXPERTS, f8t::EXPERTS.mt, f8t::EXPERTS.tn, f8t::EXPERTS.u, f8t::EXPERTS_WAVES>(P, out_dt, st);
    return launch_shape<0>(c, P, out_dt, st);
}

}  // namespace nvfp4
