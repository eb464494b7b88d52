// Products of a bf16 or binary32 tensor with a packed 4-bit weight,
//     out[i, j] = g sum_k x[i, k] c[j, k] s[j, k / B]
// on the bf16 matrix instruction: a code times its scale byte has at most 6 significant bits (E2M1 2, E4M3 4) and is exact in bf16, and so are the products in the
// instruction's binary32 sums.  A binary32 x is the sum of three bf16 numbers (8 bits of its 24 each, cut off), which are multiplied one after the other.
// What bounds the products of few rows is reading W once.
// Tile: 16 rows of W are the instruction's A, 16 rows of x its B.  Lane (q, r) of a wave takes the 32 codes 32 q .. 32 q + 31 of a K tile of 128 of row r, 16
// bytes, and the same 32 elements of x: the order of the contraction inside a K tile is free, as long as both operands have it.
#include "gemm_w4.h"

namespace nvfp4 {

// 16 rows of the output by 16 TN columns a workgroup; its NW waves take the K tiles in turn, and their sums are added through the LDS in the waves' order.
template <int XDT, int SC, int TN, int NW, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void gemm_w4_kernel(W4Args P, int out_dt)
{
    using namespace w4;
    constexpr int MT = 1, ROWS = 16 * MT, COLS = 16 * TN, XSZ = Elem<XDT>::BYTES;
    __shared__ float sums[NW][ROWS][COLS + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, r = lane & 15;
    // workgroups side by side take the same columns
    const unsigned column = workgroup() / P.slots, slot = workgroup() - column * P.slots;
    const int64_t n0 = (int64_t)column * COLS;
    if (n0 >= P.N) return;
    int64_t m0 = (int64_t)slot * ROWS, count = P.rows - m0;
    int e = 0;
    if (GROUPED) {
        const f8g::RowTile t = f8g::row_tile(P.offsets, P.groups, (int32_t)P.rows, ROWS, (int)slot);
        if (t.group < 0) return;
        e = t.group;
        m0 = t.row;
        count = t.left;
    }
    if (count > ROWS) count = ROWS;
    const bool none = GROUPED && e == P.groups;  // rows of no group
    const int shift = SC == TWO_E4M3 ? 4 : 31 - __builtin_clz((unsigned)P.block);
    const uint8_t *codes[TN], *scales[TN], *x[MT];
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        int64_t row = n0 + t * 16 + r;
        row = (row < P.N ? row : P.N - 1) + (none ? 0 : e) * P.N;
        codes[t] = P.codes + row * (P.K >> 1) + q * 16;
        scales[t] = P.scales + row * (P.K >> shift);
    }
    bool row_there[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        int64_t row = t * 16 + r;
        row_there[t] = row < count && !none;
        row = row_there[t] ? m0 + row : 0;
        if (GROUPED && P.order && row_there[t]) {
            const int32_t pair = P.order[row];
            row = pair < 0 ? -1 : pair / P.top_k;
            row_there[t] = row >= 0 && row < P.x_rows;
            if (!row_there[t]) row = 0;
        }
        x[t] = P.x + (row * P.ldx + q * 32) * XSZ;
    }
    float4v_t acc[MT][TN];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = float4v_t{0, 0, 0, 0};
    const int tiles = none ? 0 : (int)((P.K + 127) >> 7);
    for (int kt = wave; kt < tiles; kt += NW) {
        const int64_t k = (int64_t)kt * 128;
        const bool there = k + q * 32 < P.K;
        Codes<SC> a[TN];
        Elems<XDT> b[MT];
#pragma unroll
        for (int t = 0; t < TN; ++t) a[t].load(codes[t] + (k >> 1), scales[t] + ((k + q * 32) >> shift), there);
#pragma unroll
        for (int t = 0; t < MT; ++t) b[t].load(x[t] + k * XSZ, there && row_there[t]);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            bf16x8_t fb[MT][Elems<XDT>::PIECES];
#pragma unroll
            for (int i = 0; i < MT; ++i) b[i].part(p, fb[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const bf16x8_t fa = a[j].part(p);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int s = 0; s < Elems<XDT>::PIECES; ++s) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, fb[i][s], acc[i][j], 0, 0, 0);
            }
        }
    }
    // lane (q, r) has columns 4 q .. 4 q + 3 of row r
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) *reinterpret_cast<float4v_t *>(&sums[wave][i * 16 + r][j * 16 + q * 4]) = acc[i][j];
    __syncthreads();
    const float g = P.g ? P.g[none ? 0 : e * P.g_step] : 1.0f;
    for (int id = threadIdx.x; id < ROWS * COLS; id += 64 * NW) {
        const int m = id / COLS, n = id % COLS;
        if (m >= count || n0 + n >= P.N) continue;
        float s = sums[0][m][n];
        for (int w = 1; w < NW; ++w) s += sums[w][m][n];
        s = none ? 0.0f : s * g;
        if (out_dt == NVFP4_BF16) Elem<NVFP4_BF16>::store(P.out + ((m0 + m) * P.ldc + n0 + n) * 2, s);
        else Elem<NVFP4_F32>::store(P.out + ((m0 + m) * P.ldc + n0 + n) * 4, s);
    }
}

namespace w4 {

template <int XDT, int SC>
static hipError_t few_rows(W4Args P, int out_dt, hipStream_t st)
{
    constexpr int TN = 1, NW = 8;
    const int64_t cols = (P.N + 16 * TN - 1) / (16 * TN);
    if (P.groups > 0) {
        P.slots = (uint32_t)(P.rows / 16 + (P.rows < P.groups + 1 ? P.rows : P.groups + 1));
        gemm_w4_kernel<XDT, SC, TN, NW, true><<<launch_grid(cols * P.slots), 64 * NW, 0, st>>>(P, out_dt);
    } else {
        P.slots = 1;
        gemm_w4_kernel<XDT, SC, TN, NW, false><<<launch_grid(cols * P.slots), 64 * NW, 0, st>>>(P, out_dt);
    }
    return hipGetLastError();
}

}  // namespace w4

hipError_t launch_gemm_w4(const W4Args &P, int x_dt, int out_dt, hipStream_t st)
{
    using namespace w4;
    W4Tile t;
    if (w4_takes_tiles(P, x_dt, &t)) return launch_gemm_w4_tiles(P, x_dt, out_dt, t, st);
    if (x_dt == NVFP4_BF16)
        return P.scale == NVFP4_SCALE_E8M0 ? few_rows<NVFP4_BF16, ONE_E8M0>(P, out_dt, st)
               : P.block == 16             ? few_rows<NVFP4_BF16, TWO_E4M3>(P, out_dt, st)
                                           : few_rows<NVFP4_BF16, ONE_E4M3>(P, out_dt, st);
    return P.scale == NVFP4_SCALE_E8M0 ? few_rows<NVFP4_F32, ONE_E8M0>(P, out_dt, st)
           : P.block == 16             ? few_rows<NVFP4_F32, TWO_E4M3>(P, out_dt, st)
                                       : few_rows<NVFP4_F32, ONE_E4M3>(P, out_dt, st);
}

}  // namespace nvfp4
