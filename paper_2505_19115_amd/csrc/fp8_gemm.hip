// Products of quantized 8-bit operands ("NT": both stored with the contraction axis contiguous),
//     out[i, j] = sum_b 2^(sA[b,i] - 127) 2^(sB[b,j] - 127) sum_{k in b} cA[i,k] cB[j,k],
// on v_mfma_scale_f32_16x16x128_f8f6f4, which takes 128 contraction elements of 16 rows of each operand with the rows' scale bytes: one
// instruction is one block, and the scales cost nothing.  What its sums lose, and what binary32 outputs take in its place: fp8_gemm.h.
//
// Each kernel's one body serves the dense product, the experts' (rows of A divided among weights) and the experts' weight gradients (a contraction
// divided among outputs): they differ in which rows and K tiles a workgroup's tile covers (Tile).  The kernel here has tiles of 128 x 128 and serves what is
// too short or too small for the larger tiles of fp8_gemm_wide.hip and too much for fp8_gemm_thin.hip.
//
// Which row of a tile stands where.  Scales are block-major, so the bytes of a tile's rows are contiguous, and a lane can fetch the bytes of
// four fragments in one dword if these fragments' rows alternate: fragment j (of four) of rows 64 g .. 64 g + 63 has the rows 64 g + 4 c + j,
// c = 0 .. 15, and the instruction picks byte j.  The first MFMA operand is B's, whose fragments' rows become accumulator rows, so a lane
// (c, q) ends with 16 consecutive columns 64 g + 16 q .. + 15 of the output rows 64 g' + 4 c + j'.
#include "fp8_gemm.h"

namespace nvfp4 {

// 128 x 128 tiles: 2 x 2 waves of 64 x 64, two LDS stages of one K tile, filled through registers; two workgroups a CU, one of which computes while
// the other waits at its barrier.  What bounds it is latency, of the loads before the first K tile and of a barrier each: 300 x 700 x 500 4.8 us, 2000 x 2000 x
// 2000 16 (0.99 PFLOP/s).
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
    const Tile T = find_tile<MODE>(P, workgroup(), BM, BN);
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
    float4v_t acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = float4v_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int ma = wm * 64 < T.rows ? wm * 64 : 0, nb = wn * 64 < T.cols ? wn * 64 : 0;  // (a wave past the edge computes what nobody stores)
    bool beyond = false;
    if (T.count > 0) {
        fetch(0);
        stash(0);
    }
    __syncthreads();
    for (int kt = 0; kt < T.count; ++kt) {
        const bool more = kt + 1 < T.count;
        if (more) fetch(kt + 1);
        const uint32_t sa = four_scales(P.A_scales, P.a_rows, P.blocks, T.k0 + kt, T.m0 + ma, c);
        const uint32_t sb = four_scales(P.B_scales, P.b_rows, P.blocks, T.k0 + kt, T.b0 + T.n0 + nb, c);
        const uint8_t *const base = lds + (kt & 1) * STAGE + c * KT, *const A = base + wm * 64 * KT, *const B = base + (BM + wn * 64) * KT;
        const int s0 = (q ^ (c >> 1)) << 4, s1 = ((q + 4) ^ (c >> 1)) << 4;
        auto read = [&](const uint8_t *p, int j) -> Codes {
            return {*reinterpret_cast<const u32x4_t *>(p + 16 * j * KT + s0), *reinterpret_cast<const u32x4_t *>(p + 16 * j * KT + s1)};
        };
        if constexpr (exact_sums(OUT_DT)) {
            // (blocks of the rows that there are)
            if (__builtin_expect(__ballot(far_bytes(sa, sb)) != 0, 0)) {
                uint32_t least_a = ~0u, most_a = 0, least_b = ~0u, most_b = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (4 * c + j < T.rows - ma) extend(least_a, most_a, (sa >> (8 * j)) & 255);
                    if (4 * c + j < T.cols - nb) extend(least_b, most_b, (sb >> (8 * j)) & 255);
                }
                if (suspects(least_a, most_a, least_b, most_b)) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        beyond |= 4 * c + j < T.rows - ma && read(A, j).beyond((sa >> (8 * j)) & 255);
                        beyond |= 4 * c + j < T.cols - nb && read(B, j).beyond((sb >> (8 * j)) & 255);
                    }
                }
            }
            Expanded fa[4];
#pragma unroll
            for (int a = 0; a < 4; ++a) fa[a] = expand(read(A, a), (sa >> (8 * a)) & 255);
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const Expanded fb = expand(read(B, b), (sb >> (8 * b)) & 255);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int a = 0; a < 4; ++a) multiply(acc[a][b], fb, fa[a], i);
            }
        } else {
            int8v_t fa[4], fb[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                fa[j] = read(A, j).all();
                fb[j] = read(B, j).all();
            }
#define NVFP4_F8_MFMA(a, b) acc[a][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb[b], fa[a], acc[a][b], 0, 0, b, sb, a, sa);
#define NVFP4_F8_MFMA_ROW(a) NVFP4_F8_MFMA(a, 0) NVFP4_F8_MFMA(a, 1) NVFP4_F8_MFMA(a, 2) NVFP4_F8_MFMA(a, 3)
            NVFP4_F8_MFMA_ROW(0) NVFP4_F8_MFMA_ROW(1) NVFP4_F8_MFMA_ROW(2) NVFP4_F8_MFMA_ROW(3)
#undef NVFP4_F8_MFMA_ROW
#undef NVFP4_F8_MFMA
        }
        if (more) stash((kt + 1) & 1);
        __syncthreads();
    }
    if (exact_sums(OUT_DT) && __builtin_expect(__ballot(beyond) != 0, 0)) {
#pragma unroll 1
        for (int f = 0; f < 16; ++f) {
            const int r = ma + 4 * c + (f >> 2), s = nb + 4 * c + (f & 3);
            const int64_t ra = T.m0 + (r < T.rows ? r : T.rows - 1), rb = T.b0 + T.n0 + (s < T.cols ? s : T.cols - 1);
            const float4v_t v = multiply_codes(P, P.B + rb * pitch + q * 16, P.B_scales + rb, P.A + ra * pitch + q * 16, P.A_scales + ra, T.k0, 1, T.k0 + T.count);
            const int row = wm * 64 + 4 * c + (f >> 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = wn * 64 + 16 * q + 4 * i + (f & 3);
                if (row < T.rows && col < T.cols) store_one<OUT_DT>(P.out, (T.out + T.m0 + row) * P.ldc + T.n0 + col, v[i]);
            }
        }
        return;
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
static hipError_t launch_tiles(const Fp8GemmArgs &P, int out_dt, hipStream_t st)
{
    constexpr int BM = 128, BN = 128, LDS = 2 * (BM + BN) * FP8_BLOCK;
    auto *k = out_dt == NVFP4_F32 ? fp8_gemm_kernel<MODE, NVFP4_F32> : out_dt == NVFP4_BF16 ? fp8_gemm_kernel<MODE, NVFP4_BF16> : fp8_gemm_kernel<MODE, NVFP4_BF16_EXACT>;
    k<<<launch_grid(f8g::tiles<MODE>(P, BM, BN)), 256, LDS, st>>>(P);
    return hipGetLastError();
}

// Per K tile: us of a round of these tiles, two workgroups a CU (128 x 40000 x 4096, 313 of these tiles or 209 of 256 x 192: 56.6 / 50.2 us, binary32 and 256 x 128 85 / 117)
constexpr double K_TILE_BF16 = 0.95, K_TILE_F32 = 2.2;

static double tiles_cost(int64_t tiles, int out_dt)
{
    const int64_t slots = 2 * compute_units();
    return (double)((tiles + slots - 1) / slots) * (exact_sums(out_dt) ? K_TILE_F32 : K_TILE_BF16);
}
// (expanding codes for binary32: 2000 x 2000 x 2000 44 / 34, 1056 x 2080 x 2784 36 / 43)
static double thin_cost(const Fp8GemmArgs &P, int out_dt) { return fp8_gemm_thin_cost(P) * (exact_sums(out_dt) ? 1.3 : 1.0); }

// Parts of the contraction of a dense product (1: not divided), where that is quicker than every kernel that does not divide it (3 and 2.5 us: their start) by more
// than the host takes for the second launch: 16 x 64 x 12288 and 64 x 128 x 12288 would gain 1 us of 13 on the GPU alone.
// us, binary32, whole / divided: 384 x 6016 x 7296 75 / 62, 200 x 5000 x 4096 31 / 26, 777 x 1025 x 8192 34 / 32, 512 x 1000 x 8064 25.6 / 26.1.
constexpr double SECOND_LAUNCH = 3.0;
static int parts_of(const Fp8GemmArgs &P, int out_dt, size_t *bytes)
{
    if (P.M > 0 && P.N > 0 && P.blocks > 0) {
        const double tiles = tiles_cost(f8g::tiles<FP8_DENSE>(P, 128, 128), out_dt) * P.blocks + 3.0, thin = thin_cost(P, out_dt) * P.blocks + 2.5;
        const double whole = tiles < thin ? tiles : thin;
        double cost;
        const int parts = fp8_gemm_parts(P, out_dt, whole - SECOND_LAUNCH, bytes, &cost);
        if (parts > 1 && cost < whole - SECOND_LAUNCH) return parts;
    }
    *bytes = 0;
    return 1;
}

size_t fp8_gemm_workspace(const Fp8GemmArgs &P, int out_dt)
{
    size_t bytes;
    parts_of(P, out_dt, &bytes);
    return bytes;
}

template <int MODE>
static Fp8Choice choose(const Fp8GemmArgs &P, int out_dt, bool scratch)
{
    Fp8Choice c{Fp8Choice::TILES, 128, 128, 1, false};
    // Outputs past what the last cache level holds leave by streaming stores: 256 MB of weight gradients (8192 x 2 of 16, 4096 x 2048) 175 -> 155 us,
    // but 86 MB (4096 x 11008 x 4096) 154 -> 160, 128 MB the same.
    c.stream = (MODE == FP8_EXPERTS_DW ? P.groups : 1) * P.M * P.ldc * out_bytes(out_dt) >= ((int64_t)256 << 20);
    const int64_t mine = f8g::tiles<MODE>(P, 128, 128), slots = 2 * compute_units();
    const double cost = tiles_cost(mine, out_dt);
    const double wide = P.blocks > 0 ? fp8_gemm_wide_cost(P, MODE, out_dt) : 1e30;
    auto few_rows = [&]() {
        c.kernel = Fp8Choice::FEW_ROWS;
        fp8_gemm_thin_choice(P, (Fp8Mode)MODE, &c);
        return c;
    };
    // An expert's few rows: 8 on average for bf16, 16 for binary32 (us, few rows / tiles: 64 tokens, 8 of 64, 1024 x 2048 38 / 40 and 39 / 68; 128 tokens 51 / 41 and
    // 51 / 68; 64 tokens, 2 of 8, 4096 x 4096 51 / 30 and 52 / 74)
    if (MODE == FP8_EXPERTS && P.M <= (exact_sums(out_dt) ? 16 : 8) * (int64_t)P.groups) return few_rows();
    if (MODE == FP8_DENSE) {
        size_t bytes;
        c.parts = scratch ? parts_of(P, out_dt, &bytes) : 1;
        if (c.parts > 1) {
            c.kernel = Fp8Choice::DIVIDED;
            c.rows = 256;
            c.cols = fp8_gemm_wide_cols(P, FP8_DIVIDED, out_dt);
            return c;
        }
        const double thin = thin_cost(P, out_dt);
        if (thin < cost && thin < wide) return few_rows();
    }
    // A short contraction in few tiles: the larger ones take 1 to 2 us more to begin and end (experts 300 tokens, 3 of 10, 500 x 700 8.7 / 10.5, their weight
    // gradients 7.1 / 8.5)
    const int32_t count = MODE == FP8_EXPERTS_DW ? P.blocks / P.groups : P.blocks;
    if (wide < cost && !(count <= 6 && mine <= slots / 2)) {
        c.kernel = Fp8Choice::WIDE;
        c.rows = 256;
        c.cols = fp8_gemm_wide_cols(P, (Fp8Mode)MODE, out_dt);
    }
    return c;
}

Fp8Choice fp8_gemm_choice(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, bool scratch)
{
    return mode == FP8_DENSE ? choose<FP8_DENSE>(P, out_dt, scratch) : mode == FP8_EXPERTS ? choose<FP8_EXPERTS>(P, out_dt, scratch) : choose<FP8_EXPERTS_DW>(P, out_dt, scratch);
}

hipError_t launch_fp8_gemm(const Fp8GemmArgs &args, Fp8Mode mode, int out_dt, hipStream_t st)
{
    Fp8GemmArgs P = args;
    const Fp8Choice c = fp8_gemm_choice(P, mode, out_dt, P.partial != nullptr);
    P.stream = c.stream;
    if (c.kernel == Fp8Choice::FEW_ROWS) return launch_fp8_gemm_thin(P, mode, out_dt, c, st);
    if (c.kernel == Fp8Choice::WIDE) return launch_fp8_gemm_wide(P, mode, out_dt, c.cols, st);
    if (c.kernel == Fp8Choice::DIVIDED) {
        P.groups = c.parts;
        return launch_fp8_gemm_wide(P, FP8_DIVIDED, out_dt, c.cols, st);
    }
    return mode == FP8_DENSE ? launch_tiles<FP8_DENSE>(P, out_dt, st) : mode == FP8_EXPERTS ? launch_tiles<FP8_EXPERTS>(P, out_dt, st) : launch_tiles<FP8_EXPERTS_DW>(P, out_dt, st);
}

}  // namespace nvfp4
