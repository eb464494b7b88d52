// What the kernels of 8-bit products share: which rows and K tiles a workgroup's tile covers, scale bytes, fragments, and the way out.
#pragma once
#include <type_traits>
#include "experts.h"
#include "kernels.h"

namespace nvfp4 {
namespace f8g {

typedef int int8v_t __attribute__((ext_vector_type(8)));
typedef float float4v_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2v_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int KT = FP8_BLOCK;

// What a workgroup multiplies: rows m0 .. m0 + rows - 1 of A (and of the output that starts at out) against rows n0 .. n0 + cols - 1 of B,
// K tiles k0 .. k0 + count - 1; b0 + column is a row of B.  rows <= 0: nothing.
struct Tile {
    int64_t m0, n0, b0, out;
    int rows, cols, k0, count;
};

// Tiles of a launch; of the experts' product the most there can be: every group of rows (the rows of no expert are one) may have one that is not full.
template <int MODE>
__host__ __device__ inline int64_t tile_rows(const Fp8GemmArgs &P, int BM)
{
    return MODE == FP8_EXPERTS ? P.M / BM + (P.M < P.groups + 1 ? P.M : P.groups + 1) : (P.M + BM - 1) / BM * (MODE == FP8_EXPERTS_DW ? P.groups : 1);
}
template <int MODE>
inline int64_t tiles(const Fp8GemmArgs &P, int BM, int BN) { return (P.N + BN - 1) / BN * tile_rows<MODE>(P, BM); }

// Tile `n` of those that the groups of rows have one after the other, step rows each: its group (`groups` for the rows of no expert, -1: there are not so many), first
// row and the rows from there on to the group's end.  Every wave asks for itself.  (With a place for each tile that a group might have, found from
// its first row alone, a launch had as many workgroups with nothing to do as there are experts: a token's two of 32 experts, 2048 x 4096, took 35 us, of 8 15.)
struct RowTile {
    int group, row, left;
};
__device__ __forceinline__ RowTile row_tile(const int32_t *offsets, int groups, int32_t total, int step, int n)
{
    const int lane = (int)(threadIdx.x & 63);
    int before = 0;
    for (int e0 = 0; e0 <= groups; e0 += 64) {
        const int e = e0 + lane;
        int32_t a = 0, b = 0;
        if (e <= groups) {
            a = offsets[e];
            b = e < groups ? offsets[e + 1] : total;
            a = a < 0 ? 0 : a > total ? total : a;
            b = b < a ? a : b > total ? total : b;
        }
        const int mine = (int)(((unsigned)(b - a) + (unsigned)step - 1) / (unsigned)step);  // (up to 2^31 - 1 rows)
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(upto, d);
            if (lane >= d) upto += up;
        }
        const uint64_t past = __ballot(before + upto > n);
        if (past) {
            const int l = __builtin_ctzll(past);
            const int row = a + (n - (before + upto - mine)) * step;
            return {e0 + l, __builtin_amdgcn_readlane(row, l), __builtin_amdgcn_readlane(b - row, l)};
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}

template <int MODE>
__device__ __forceinline__ Tile find_tile(const Fp8GemmArgs &P, unsigned id, int BM, int BN)
{
    Tile T;
    const int ntx = (int)((P.N + BN - 1) / BN), nty = (int)tile_rows<MODE>(P, BM);
    T.k0 = 0;
    T.count = P.blocks;
    T.b0 = 0;
    T.out = 0;
    if (id >= (unsigned)ntx * (unsigned)nty) {
        T.rows = 0;
        return T;
    }
    int ty, tx;
    tile_coords((int)id, ntx, nty, ty, tx);
    int64_t left;
    if (MODE == FP8_EXPERTS) {
        // rows past the last expert's are a group of their own, with no K tile: zeros
        const RowTile r = row_tile(P.offsets, P.groups, (int32_t)P.M, BM, ty);
        if (r.group < 0) {
            T.rows = 0;
            return T;
        }
        if (r.group == P.groups) T.count = 0;
        else T.b0 = r.group * P.N;
        T.m0 = r.row;
        left = r.left;
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

// Scale bytes of four neighbouring rows, rows 4 c .. 4 c + 3 of `have` that start at `first`, of K tile `kt` of all the operand's: one load, at any
// byte.  The array ends with the last K tile's last row; a load that would pass it is moved back.  (Rows past the tile's get some byte.)
__device__ __forceinline__ uint32_t four_scales(const uint8_t *scales, int64_t rows, int blocks, int kt, int64_t first, int c)
{
    struct __attribute__((packed)) Four { uint32_t w; };
    const int64_t at = kt * rows + first, left = blocks * rows - at;  // (bytes from the first row's on, at least one)
    const uint8_t *const p = scales + at;
    if (left >= 64) return reinterpret_cast<const Four *>(p + 4 * c)->w;
    if (at + left < 4) {  // an operand of one to three bytes
        uint32_t w = 0;
        for (int j = 0; j < 4; ++j)
            if (4 * c + j < left) w |= (uint32_t)p[4 * c + j] << (8 * j);
        return w;
    }
    const int l = (int)left, from = 4 * c + 4 <= l ? 4 * c : l - 4, off = 4 * c - from;
    return off >= 4 ? 0x7F7F7F7Fu : reinterpret_cast<const Four *>(p + from)->w >> (8 * off);
}

// Two ways to multiply a K tile of two fragments of 16 rows, of which a lane holds 32 codes each.
//   bf16 outputs: v_mfma_scale_f32_16x16x128_f8f6f4, one instruction, scales included.  It adds the products in groups of eight neighbours and cuts each
//     off at 2^-13 of the power of two under its group's largest (the other 8-bit forms lose as much), and adds the groups in binary32: what is lost is at
//     most 7 2^-13 = 8.5e-4 of sum |a||b|, reached only where single products stand far above the seven beside them, and 1.5e-5 of the result's norm for
//     normal data, where rounding to bf16 takes 1.7e-3 of the norm.
//   binary32 outputs, and bf16 ones of such sums (NVFP4_BF16_EXACT): the codes become bf16, scale included (v_cvt_scalef32_pk_bf16_fp8), for v_mfma_f32_16x16x32_bf16, whose sums
//     are binary32 (1e-7 of the norm), at half the rate and for 32 conversions a lane.  That is exact for scale bytes LEAST .. MOST: below, the smallest codes
//     need bits under bf16's least subnormal 2^-133, above, 448 * 2^(byte - 127) passes its largest number (a finite tensor's byte is 247 from
//     1.75 * 2^127 on, torch.finfo(torch.bfloat16).min among them).  A wave that meets a block beyond these sums its outputs by multiply_codes().
//     Bits are lost of the lower ones only against scale bytes above LARGE: against others a product is off by less than 2^-126, and blocks of zeros, which have byte 0,
//     cost nothing.
constexpr uint32_t LEAST = 3, MOST = 246, LARGE = 126;
struct Codes {
    u32x4_t lo, hi;  // chunks q and q + 4 of a row's eight
    __device__ __forceinline__ bool any() const
    {
        return ((lo[0] | lo[1] | lo[2] | lo[3] | hi[0] | hi[1] | hi[2] | hi[3]) & 0x7F7F7F7Fu) != 0;
    }
    // whether bf16 may not hold these codes with this scale
    __device__ __forceinline__ bool beyond(uint32_t byte) const { return byte > MOST || (byte < LEAST && any()); }
    __device__ __forceinline__ int8v_t all() const
    {
        return int8v_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    }
};
__device__ __forceinline__ Codes codes_at(const uint8_t *p) { return {*reinterpret_cast<const u32x4_t *>(p), *reinterpret_cast<const u32x4_t *>(p + 64)}; }
struct Expanded {
    bf16x8_t v[4];
};
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x00400000u); }
// eight codes of step i of four
__device__ __forceinline__ bf16x8_t expand(const Codes &x, float s, int i)
{
    bf16x8_t r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = i < 2 ? x.lo[2 * i + h] : x.hi[2 * (i - 2) + h];
        const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, 1);
        r[4 * h] = a[0];
        r[4 * h + 1] = a[1];
        r[4 * h + 2] = b[0];
        r[4 * h + 3] = b[1];
    }
    return r;
}
__device__ __forceinline__ Expanded expand(const Codes &x, uint32_t byte)
{
    const float s = scale_of(byte);
    Expanded r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.v[i] = expand(x, s, i);
    return r;
}
// Whether one of eight scale bytes is outside 64 .. 191, that is has its two top bits alike: what few operations say of LEAST .. MOST
__device__ __forceinline__ bool far_bytes(uint32_t a, uint32_t b) { return (~((a ^ (a << 1)) & (b ^ (b << 1))) & 0x80808080u) != 0; }
__device__ __forceinline__ void extend(uint32_t &least, uint32_t &most, uint32_t byte)
{
    least = byte < least ? byte : least;
    most = byte > most ? byte : most;
}
// Whether codes have to be looked at for blocks that bf16 does not hold: by the wave's scale bytes of both operands
__device__ __forceinline__ bool suspects(uint32_t least_a, uint32_t most_a, uint32_t least_b, uint32_t most_b)
{
    const uint32_t least = least_a < least_b ? least_a : least_b, most = most_a > most_b ? most_a : most_b;
    if (__builtin_expect(__ballot(least < LEAST || most > MOST) == 0, 1)) return false;
    return __ballot(most > MOST) != 0 || (__ballot(least_a < LEAST) != 0 && __ballot(most_b > LARGE) != 0) || (__ballot(least_b < LEAST) != 0 && __ballot(most_a > LARGE) != 0);
}
// step i of four
__device__ __forceinline__ void multiply(float4v_t &acc, const Expanded &b, const Expanded &a, int i)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], acc, 0, 0, 0);
}

// Whether one of K tiles kt, kt + step, ... below `end` is a block that bf16 does not hold
__device__ __forceinline__ bool any_beyond(const uint8_t *codes, const uint8_t *scale, int64_t rows, int kt, int step, int end)
{
    bool beyond = false;
#pragma unroll 2
    for (; kt < end; kt += step) {
        const Codes x = codes_at(codes + (int64_t)kt * KT);
        const uint32_t byte = scale[kt * rows];
        beyond |= (byte > MOST) | ((byte < LEAST) & x.any());
    }
    return beyond;
}
// The sum of K tiles kt, kt + step, ... below `end` of one fragment of each operand, whatever the scales: a tile's codes are multiplied, whose products and sums
// binary32 holds as it holds any, and the sum takes both scales.  a, b: the lane's first chunk of its row at K tile 0; sa, sb: its row's first scale byte.
// Byte 255 is no number.  Slow, straight from memory: what a wave does again where bf16 did not hold one of its blocks.
__device__ __forceinline__ float4v_t multiply_codes(const Fp8GemmArgs &P, const uint8_t *b, const uint8_t *sb, const uint8_t *a, const uint8_t *sa, int kt, int step, int end)
{
    float4v_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (; kt < end; kt += step) {
        const Codes xb = codes_at(b + (int64_t)kt * KT), xa = codes_at(a + (int64_t)kt * KT);
        const uint32_t mine = sb[kt * P.b_rows], s = sa[kt * P.a_rows];
        float4v_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(expand(xb, 1.0f, i), expand(xa, 1.0f, i), sum, 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);  // (registers of one step: the kernels' other paths are to have as many waves as without this one)
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t r = (uint32_t)__shfl((int)mine, 4 * (int)((threadIdx.x & 63) >> 4) + i);  // acc's rows of B: positions 4 q .. 4 q + 3
            acc[i] += r == 255 || s == 255 ? __uint_as_float(0x7FC00000u) : __builtin_ldexpf(sum[i], (int)(r + s) - 254);
        }
    }
    return acc;
}

template <int OUT_DT>
__device__ __forceinline__ void store_one(void *out, int64_t at, float v)
{
    if (OUT_DT == NVFP4_F32) reinterpret_cast<float *>(out)[at] = v;
    else reinterpret_cast<__bf16 *>(out)[at] = (__bf16)v;
}

// n of four columns of one row
template <int OUT_DT>
__device__ __forceinline__ void store_four(void *out, int64_t at, const float4v_t &v, int n)
{
    if (OUT_DT == NVFP4_F32) {
        struct __attribute__((packed, aligned(4))) P { u32x4_t w; };
        float *const p = reinterpret_cast<float *>(out) + at;
        if (n >= 4) {
            reinterpret_cast<P *>(p)->w = __builtin_bit_cast(u32x4_t, v);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) p[i] = v[i];
        }
    } else {
        typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
        struct __attribute__((packed, aligned(2))) P { u32x2_t w; };
        uint16_t *const p = reinterpret_cast<uint16_t *>(out) + at;
        const float2v_t lo = {v[0], v[1]}, hi = {v[2], v[3]};
        const u32x2_t w = {__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t)), __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t))};
        if (n >= 4) {
            reinterpret_cast<P *>(p)->w = w;
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) p[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
}

__device__ __forceinline__ u32x4_t to_bf16(const float (&v)[8])
{
    u32x4_t w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2v_t f = {v[2 * i], v[2 * i + 1]};
        w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
    }
    return w;
}

// n of the four (binary32) or eight (bf16) columns of one row that fill 16 bytes
template <int OUT_DT, bool STREAMED>
__device__ __forceinline__ void store_lane(void *out, int64_t at, const u32x4_t &w, int n)
{
    typedef std::conditional_t<OUT_DT == NVFP4_F32, uint32_t, uint16_t> element_t;
    typedef u32x4_t __attribute__((aligned(2))) anywhere_t;
    constexpr int N = 16 / sizeof(element_t);
    element_t *const p = reinterpret_cast<element_t *>(out) + at;
    if (n >= N) {
        if (STREAMED) __builtin_nontemporal_store(w, reinterpret_cast<anywhere_t *>(p));
        else *reinterpret_cast<anywhere_t *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; ++i)
            if (i < n) p[i] = (element_t)(w[i * 4 / N] >> (N == 8 ? 16 * (i & 1) : 0));
    }
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


}  // namespace nvfp4
