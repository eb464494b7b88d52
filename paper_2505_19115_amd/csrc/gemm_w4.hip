// Products of a bf16 or binary32 tensor with a packed 4-bit weight,
//     out[i, j] = g sum_k x[i, k] c[j, k] s[j, k / B]
// on the bf16 matrix instruction: a code times its scale byte has at most 6 significant bits (E2M1 2, E4M3 4) and is exact in bf16, and so are the products in the
// instruction's binary32 sums.  A binary32 x is the sum of three bf16 numbers (8 bits of its 24 each, cut off), which are multiplied one after the other.
// What bounds the products of few rows is reading W once.
// Tile: 16 rows of W are the instruction's A, 16 rows of x its B.  Lane (q, r) of a wave takes the 32 codes 32 q .. 32 q + 31 of a K tile of 128 of row r, 16
// bytes, and the same 32 elements of x: the order of the contraction inside a K tile is free, as long as both operands have it.
#include <type_traits>

#include "layer_ops.h"

namespace nvfp4 {
namespace w4 {

using namespace layer;

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float float4v_t __attribute__((ext_vector_type(4)));

// How a lane's 32 codes are scaled: two E4M3 bytes, one, or one E8M0 byte
enum Scaling { TWO_E4M3, ONE_E4M3, ONE_E8M0 };

union Frag {
    uint32_t w[4];
    bf16x8_t v;
};

// 8 codes times their scale in bf16 (exact)
__device__ __forceinline__ bf16x8_t expand_e4m3(uint32_t codes, float s)
{
    Frag f;
    auto two = [&](float2v_t p) {
        const float2v_t v = {p[0] * s, p[1] * s};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
    };
    f.w[0] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0));
    f.w[1] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1));
    f.w[2] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2));
    f.w[3] = two(__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3));
    return f.v;
}
__device__ __forceinline__ bf16x8_t expand_e8m0(uint32_t codes, float s)
{
    Frag f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return f.v;
}

// A lane's 32 codes of a K tile
template <int SC>
struct Codes {
    u32x4_t w;
    uint32_t s;
    __device__ __forceinline__ void load(const uint8_t *codes, const uint8_t *scales, bool there)
    {
        w = there ? *reinterpret_cast<const u32x4_t *>(codes) : u32x4_t{0, 0, 0, 0};
        s = !there ? 0 : SC == TWO_E4M3 ? *reinterpret_cast<const uint16_t *>(scales) : *scales;
    }
    __device__ __forceinline__ bf16x8_t part(int p) const
    {
        if (SC == ONE_E8M0) return expand_e8m0(w[p], __uint_as_float(s << 23));
        return expand_e4m3(w[p], SC == TWO_E4M3 && p >= 2 ? __builtin_amdgcn_cvt_f32_fp8((int)s, 1) : __builtin_amdgcn_cvt_f32_fp8((int)s, 0));
    }
};

// 32 elements of a row of x as they come
template <int XDT>
struct Elems {
    static constexpr int W = XDT == NVFP4_BF16 ? 4 : 8;
    struct __attribute__((packed, aligned(Elem<XDT>::BYTES))) Q { u32x4_t w; };
    u32x4_t w[W];
    __device__ __forceinline__ void load(const uint8_t *p, bool there)
    {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = there ? reinterpret_cast<const Q *>(p)[i].w : u32x4_t{0, 0, 0, 0};
    }
    // part p (8 elements) into its bf16 pieces, which add up to it
    static constexpr int PIECES = XDT == NVFP4_BF16 ? 1 : 3;
    __device__ __forceinline__ void part(int p, bf16x8_t (&out)[PIECES]) const
    {
        Frag f[PIECES];
        if constexpr (XDT == NVFP4_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f[0].w[i] = w[p][i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t top[3][2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float rest = __uint_as_float(w[2 * p + (i >> 1)][(2 * i + k) & 3]);
#pragma unroll
                    for (int s = 0; s < 3; ++s) {
                        top[s][k] = __float_as_uint(rest) & 0xFFFF0000u;
                        const float cut = __uint_as_float(top[s][k]);
                        rest = rest == cut ? 0.0f : rest - cut;  // (an infinity has no rest)
                    }
                }
#pragma unroll
                for (int s = 0; s < 3; ++s) f[s].w[i] = top[s][0] >> 16 | top[s][1];
            }
        }
#pragma unroll
        for (int s = 0; s < PIECES; ++s) out[s] = f[s].v;
    }
};

}  // namespace w4

// 16 MT rows of the output by 16 TN columns a workgroup; its NW waves take the K tiles in turn, and their sums are added through the LDS in the waves' order.
template <int XDT, int SC, int MT, int TN, int NW, bool GROUPED>
__global__ __launch_bounds__(64 * NW) void gemm_w4_kernel(W4Args P, int out_dt)
{
    using namespace w4;
    constexpr int ROWS = 16 * MT, COLS = 16 * TN, XSZ = Elem<XDT>::BYTES;
    __shared__ float sums[NW][ROWS][COLS + 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, r = lane & 15;
    // workgroups side by side take the same columns
    const unsigned column = workgroup() / P.slots, slot = workgroup() - column * P.slots;
    const int64_t n0 = (int64_t)column * COLS;
    if (n0 >= P.N) return;
    int64_t m0 = (int64_t)slot * ROWS, count = P.rows - m0;
    int e = 0;
    if (GROUPED) {
        e = group_of_slot(P.offsets, P.groups + 1, (int32_t)P.rows, ROWS, (int)slot);
        int32_t first = P.offsets[e], last = e < P.groups ? P.offsets[e + 1] : (int32_t)P.rows;
        first = first < 0 ? 0 : first > P.rows ? (int32_t)P.rows : first;
        last = last < first ? first : last > P.rows ? (int32_t)P.rows : last;
        m0 = first + ((int64_t)slot - (first / ROWS + e)) * ROWS;
        count = last - m0;
        if (count <= 0) return;
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

template <int XDT, int SC, int MT, bool GROUPED>
static hipError_t run(W4Args P, int out_dt, hipStream_t st)
{
    constexpr int TN = MT >= 4 ? 2 : 1, NW = MT >= 4 ? 4 : 8;
    P.slots = (uint32_t)(GROUPED ? P.rows / (16 * MT) + P.groups + 1 : (P.rows + 16 * MT - 1) / (16 * MT));
    const int64_t cols = (P.N + 16 * TN - 1) / (16 * TN);
    gemm_w4_kernel<XDT, SC, MT, TN, NW, GROUPED><<<launch_grid(cols * P.slots), 64 * NW, 0, st>>>(P, out_dt);
    return hipGetLastError();
}

template <int XDT, int SC>
static hipError_t by_rows(const W4Args &P, int out_dt, hipStream_t st)
{
    const int64_t rows = P.groups > 0 ? P.rows / P.groups : P.rows;
    if (P.groups > 0) {
        if (rows <= 16) return run<XDT, SC, 1, true>(P, out_dt, st);
        return run<XDT, SC, 4, true>(P, out_dt, st);
    }
    if (rows <= 16) return run<XDT, SC, 1, false>(P, out_dt, st);
    return run<XDT, SC, 4, false>(P, out_dt, st);
}

}  // namespace w4

hipError_t launch_gemm_w4(const W4Args &P, int x_dt, int out_dt, hipStream_t st)
{
    using namespace w4;
    if (x_dt == NVFP4_BF16)
        return P.scale == NVFP4_SCALE_E8M0 ? by_rows<NVFP4_BF16, ONE_E8M0>(P, out_dt, st)
               : P.block == 16             ? by_rows<NVFP4_BF16, TWO_E4M3>(P, out_dt, st)
                                           : by_rows<NVFP4_BF16, ONE_E4M3>(P, out_dt, st);
    return P.scale == NVFP4_SCALE_E8M0 ? by_rows<NVFP4_F32, ONE_E8M0>(P, out_dt, st)
           : P.block == 16             ? by_rows<NVFP4_F32, TWO_E4M3>(P, out_dt, st)
                                       : by_rows<NVFP4_F32, ONE_E4M3>(P, out_dt, st);
}

}  // namespace nvfp4
