// Products of a bf16 or binary32 tensor with a packed 4-bit weight,
//     out[i, j] = g sum_k x[i, k] c[j, k] s[j, k / B]
// on the bf16 matrix instruction: a code times its scale byte has at most 6 significant bits (E2M1 2, E4M3 4) and is exact in bf16, and so are the products in the
// instruction's binary32 sums.  A binary32 x is the sum of three bf16 numbers (8 bits of its 24 each, cut off), which are multiplied one after the other.
// What bounds the products of few rows is reading W once.
// Tile: 16 rows of W are the instruction's A, 16 rows of x its B.  Lane (q, r) of a wave takes the 32 codes 32 q .. 32 q + 31 of a K tile of 128 of row r, 16
// bytes, and the same 32 elements of x: the order of the contraction inside a K tile is free, as long as both operands have it.
#include "gemm_w4.h"

namespace nvfp4 {

// 16 rows of the output by 16 columns a workgroup; its NW waves take the K tiles in turn, the codes of BATCH of them requested at a time and x of the next one, and their sums are
// added through the LDS in the waves' order.  us, from memory, NW 4 / 8: 1 x 4096 x 11008 NVFP4 16.3 / 12.9, MXFP4 15.2 / 11.2, 16 x 12288 x 4096 19.8 / 19.7, 4 x 11008 x 2048 8.2 / 9.0, 16 tokens x 2
// of 8 experts 4096 x 2048 MXFP4 19.8 / 24.2, 1 x 2 6.8 / 7.1, 8 x 2 of 64 1024 x 1024 7.6 / 9.9: eight where there are few columns.  The floor of the first is 4.8 us.  What the rest goes to: a batch of codes is asked for
// at the top of the loop and waited for at once, because x, asked for behind it, is needed first and loads come in their order; between two batches nothing is on its way.  K = 11008 is three such
// waits for each of eight waves, and one more a K tile for x (1 x 256 x 12288, 1.7 MB, takes 11.7).  Tried: twelve K tiles' codes at a time and x of four (12.3, experts 25), four waves on columns
// of their own instead of parts of the contraction (experts 25).
template <int XDT, int SC, int NW, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void gemm_w4_kernel(W4Args P, int out_dt)
{
    using namespace w4;
    constexpr int BATCH = 4, ROWS = 16, COLS = 16, XSZ = Elem<XDT>::BYTES;
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
    int64_t w_row = n0 + r;
    w_row = (w_row < P.N ? w_row : P.N - 1) + (none ? 0 : e) * P.N;
    const uint8_t *const codes = P.codes + w_row * (P.K >> 1), *const scales = P.scales + w_row * (P.K >> shift);
    // W's first batch is on its way before an order says which rows of x there are
    const int tiles = none ? 0 : (int)((P.K + 127) >> 7);
    Codes<SC> a[BATCH];
    auto load_w = [&](int kt) {
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            const int64_t k = (int64_t)(kt + u * NW) * 128 + q * 32;
            if (kt + u * NW < tiles) a[u].load(codes + (k < P.K ? k >> 1 : 0), scales + (k < P.K ? k >> shift : 0), true);
        }
    };
    load_w(wave);
    const uint8_t *x;
    bool row_there = r < count && !none;
    {
        int64_t row = row_there ? m0 + r : 0;
        if (GROUPED && P.order && row_there) {
            const int32_t pair = P.order[row];
            row = pair < 0 ? -1 : pair / P.top_k;
            row_there = row >= 0 && row < P.x_rows;
            if (!row_there) row = 0;
        }
        x = P.x + (row * P.ldx + q * 32) * XSZ;
    }
    // (the same in every wave: lane r asks for row r)  Rows that are not there become zeros whatever W and g hold
    const uint64_t rows_there = __ballot(row_there);
    float4v_t acc = {0, 0, 0, 0};
    for (int kt = wave; kt < tiles; kt += NW * BATCH) {
        if (kt != wave) load_w(kt);
        Elems<XDT> b[2];
        auto load_x = [&](int u) {
            const int64_t k = (int64_t)(kt + u * NW) * 128;
            b[u & 1].load(x + k * XSZ, row_there && k + q * 32 < P.K);
        };
        load_x(0);
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (kt + u * NW >= tiles) break;
            if (u + 1 < BATCH) load_x(u + 1);
            const bool there = (int64_t)(kt + u * NW) * 128 + q * 32 < P.K;  // (past the end came some codes of the row)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[u].w[i] = there ? a[u].w[i] : 0;
            a[u].s = there ? a[u].s : 0;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                bf16x8_t fb[Elems<XDT>::PIECES];
                b[u & 1].part(p, fb);
                const bf16x8_t fa = a[u].part(p);
#pragma unroll
                for (int s = 0; s < Elems<XDT>::PIECES; ++s) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa, fb[s], acc, 0, 0, 0);
            }
        }
    }
    // lane (q, r) has columns 4 q .. 4 q + 3 of row r
    *reinterpret_cast<float4v_t *>(&sums[wave][r][q * 4]) = acc;
    __syncthreads();
    const float g = P.g ? P.g[none ? 0 : e * P.g_step] : 1.0f;
    for (int id = threadIdx.x; id < ROWS * COLS; id += 64 * NW) {
        const int m = id / COLS, n = id % COLS;
        if (m >= count || n0 + n >= P.N) continue;
        float s = sums[0][m][n];
        for (int w = 1; w < NW; ++w) s += sums[w][m][n];
        s = rows_there >> m & 1 ? s * g : 0.0f;
        if (out_dt == NVFP4_BF16) Elem<NVFP4_BF16>::store(P.out + ((m0 + m) * P.ldc + n0 + n) * 2, s);
        else Elem<NVFP4_F32>::store(P.out + ((m0 + m) * P.ldc + n0 + n) * 4, s);
    }
}

namespace w4 {

template <int XDT, int SC, int NW>
static hipError_t divided(W4Args P, int64_t slots, int out_dt, hipStream_t st)
{
    P.slots = (uint32_t)slots;
    const dim3 grid = launch_grid((P.N + 15) / 16 * slots);
    if (P.groups > 0) gemm_w4_kernel<XDT, SC, NW, true><<<grid, 64 * NW, 0, st>>>(P, out_dt);
    else gemm_w4_kernel<XDT, SC, NW, false><<<grid, 64 * NW, 0, st>>>(P, out_dt);
    return hipGetLastError();
}

constexpr int64_t MANY = 512;  // workgroups that fill the CUs with four waves each
static int64_t row_slots(const W4Args &P) { return P.groups > 0 ? P.rows / 16 + (P.rows < P.groups + 1 ? P.rows : P.groups + 1) : 1; }
static bool four_waves(const W4Args &P) { return (P.N + 15) / 16 * row_slots(P) >= MANY; }
template <int XDT, int SC>
static hipError_t few_rows(const W4Args &P, int out_dt, hipStream_t st)
{
    return four_waves(P) ? divided<XDT, SC, 4>(P, row_slots(P), out_dt, st) : divided<XDT, SC, 8>(P, row_slots(P), out_dt, st);
}

}  // namespace w4

W4Choice gemm_w4_choice(const W4Args &P, int x_dt)
{
    W4Tile t;
    if (w4_takes_tiles(P, x_dt, &t)) return {w4_takes_direct(P, x_dt) ? W4Choice::DIRECT : W4Choice::STAGED, 16 * t.rows16, 64 * t.cols16, 4};
    return {W4Choice::FEW_ROWS, 16, 16, w4::four_waves(P) ? 4 : 8};
}

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
