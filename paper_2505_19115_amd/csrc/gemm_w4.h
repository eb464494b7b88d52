// What the kernels of products with packed 4-bit weights share (gemm_w4.hip): operands in registers.
#pragma once
#include <type_traits>

#include "fp8_gemm.h"
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

// For more rows than a few: tiles of 16 rows16 rows by 64 cols16 columns
struct W4Tile {
    int rows16, cols16;
};
bool w4_takes_tiles(const W4Args &P, int x_dt, W4Tile *t);
// Whether x goes to their LDS directly
bool w4_takes_direct(const W4Args &P, int x_dt);
hipError_t launch_gemm_w4_tiles(const W4Args &P, int x_dt, int out_dt, const W4Tile &t, hipStream_t st);

}  // namespace nvfp4
