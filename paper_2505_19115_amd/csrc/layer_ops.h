// Internal interface between the C ABI (api_layer.hip) and the launchers of the operators around the products: the experts' router with its balance
// loss, rows' norms, products with packed 4-bit weights.  Below: what their kernels share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/nvfp4.h"
#include "experts.h"

namespace nvfp4 {

struct RouteArgs {
    const void *logits;       // [tokens, groups] in rows of pitch ld
    int64_t tokens, ld;
    int32_t groups, top_k;
    bool renormalize;
};
hipError_t launch_moe_route(const RouteArgs &P, int dt, int32_t *experts, float *weights, hipStream_t st);
// dweights, counts, dlosses: null for none (counts and dlosses are both there or neither); experts of id_bytes
hipError_t launch_moe_route_bwd(const RouteArgs &P, int dt, const int32_t *experts, const float *dweights, const int32_t *counts, const float *dlosses, void *dlogits,
                                hipStream_t st);
size_t moe_balance_workspace(int64_t tokens, int32_t groups);
hipError_t launch_moe_balance(const RouteArgs &P, int dt, const void *experts, int id_bytes, float *losses, int32_t *counts, float *probs, void *workspace, hipStream_t st);

// y = (x - mean) rstd weight + bias of rows
struct NormArgs {
    int64_t rows, cols, ld;   // of x
    const void *weight, *bias;  // null: ones, zeros
    int wdt;
    bool center;
};
hipError_t launch_layer_norm(const NormArgs &P, int dt, const void *x, float eps, void *y, float *mean, float *rstd, hipStream_t st);
// dweight, dbias: null where not wanted (then no workspace is)
size_t layer_norm_bwd_workspace(int64_t rows, int64_t cols, int dt, bool dweight, bool dbias);
hipError_t launch_layer_norm_bwd(const NormArgs &P, int dt, const void *dy, int64_t ldy, const void *x, const float *mean, const float *rstd, void *dx, void *dweight,
                                 void *dbias, void *workspace, hipStream_t st);

// out = g x W^T of a tensor x [rows, K] and a packed W [N, K].  With offsets [groups + 1] the rows of the output are divided among `groups` weights of N rows each,
// rows past the last become zeros; with order, row r is row order[r] / top_k of x (none: zeros).
struct W4Args {
    const uint8_t *x;
    int64_t rows, x_rows, ldx, N, K;
    const uint8_t *codes, *scales;  // [(groups) N, K / 2], [(groups) N, K / block]
    const float *g;                 // one, or one a group (g_step 1)
    int32_t g_step;
    int32_t block, scale;           // as in nvfp4_format
    const int32_t *offsets, *order;
    int32_t groups, top_k;          // groups 0: one product
    uint8_t *out;
    int64_t ldc;
    uint32_t slots;                 // tiles of rows (set by launch_gemm_w4())
};
hipError_t launch_gemm_w4(const W4Args &P, int x_dt, int out_dt, hipStream_t st);
// Which kernel that is: for few rows, or tiles whose rows of x go to the LDS directly or through registers; rows and columns of a workgroup's outputs, waves that share them
struct W4Choice {
    enum Kernel { FEW_ROWS, DIRECT, STAGED } kernel;
    int rows, cols, waves;
};
W4Choice gemm_w4_choice(const W4Args &P, int x_dt);

namespace layer {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2v_t __attribute__((ext_vector_type(2)));

template <int DT>
struct Elem {
    static constexpr int BYTES = DT == NVFP4_BF16 ? 2 : 4;
    __device__ static __forceinline__ float load(const uint8_t *p)
    {
        return DT == NVFP4_BF16 ? __uint_as_float((uint32_t) * reinterpret_cast<const uint16_t *>(p) << 16) : *reinterpret_cast<const float *>(p);
    }
    __device__ static __forceinline__ void store(uint8_t *p, float v)
    {
        if (DT == NVFP4_BF16) *reinterpret_cast<__bf16 *>(p) = (__bf16)v;
        else *reinterpret_cast<float *>(p) = v;
    }
};

// N neighbouring elements (16 bytes, or 32) from any element on; of the last ones of a row the first n
template <int DT, int N>
__device__ __forceinline__ void load_run(float (&v)[N], const uint8_t *p, int n, float fill)
{
    constexpr int ESZ = Elem<DT>::BYTES;
    struct __attribute__((packed, aligned(ESZ))) Q { u32x4_t w; };
    if (n >= N) {
#pragma unroll
        for (int q = 0; q < N * ESZ / 16; ++q) {
            const u32x4_t w = reinterpret_cast<const Q *>(p)[q].w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (DT == NVFP4_BF16) {
                    v[q * 8 + 2 * i] = __uint_as_float(w[i] << 16);
                    v[q * 8 + 2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                } else {
                    v[(q * 4 + i) % N] = __uint_as_float(w[i]);
                }
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? Elem<DT>::load(p + i * ESZ) : fill;
}
template <int DT, int N>
__device__ __forceinline__ void store_run(const float (&v)[N], uint8_t *p, int n)
{
    constexpr int ESZ = Elem<DT>::BYTES;
    struct __attribute__((packed, aligned(ESZ))) Q { u32x4_t w; };
    if (n >= N) {
#pragma unroll
        for (int q = 0; q < N * ESZ / 16; ++q) {
            u32x4_t w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (DT == NVFP4_BF16) {
                    const float2v_t f = {v[q * 8 + 2 * i], v[q * 8 + 2 * i + 1]};
                    w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
                } else {
                    w[i] = __float_as_uint(v[(q * 4 + i) % N]);
                }
            }
            reinterpret_cast<Q *>(p)[q].w = w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < n) Elem<DT>::store(p + i * ESZ, v[i]);
}

// The value of the lane across, among 2^(STEP + 1) neighbours: its partner differs in bit STEP at least, and groups of 2^STEP lanes that agree
// meet the other half of theirs (data-parallel moves inside 16 lanes, the LDS crossbar past them)
template <int STEP>
__device__ __forceinline__ uint32_t across(uint32_t v)
{
    if constexpr (STEP == 0) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, false);        // lanes 1 0 3 2
    else if constexpr (STEP == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, false);   // lanes 2 3 0 1
    else if constexpr (STEP == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, false);  // 8 lanes mirrored
    else if constexpr (STEP == 3) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, false);  // 16 lanes mirrored
    else return (uint32_t)__shfl_xor((int)v, 1 << STEP);
}
// Over G neighbouring lanes, the result in all of them.  The order of the additions is the same for every lane up to commuted operands.
template <int G, int STEP = 0>
__device__ __forceinline__ float group_sum(float v)
{
    if constexpr ((1 << STEP) >= G) return v;
    else return group_sum<G, STEP + 1>(v + __uint_as_float(across<STEP>(__float_as_uint(v))));
}
template <int G, int STEP = 0>
__device__ __forceinline__ uint32_t group_most(uint32_t v)
{
    if constexpr ((1 << STEP) >= G) {
        return v;
    } else {
        const uint32_t o = across<STEP>(v);
        return group_most<G, STEP + 1>(o > v ? o : v);
    }
}

}  // namespace layer
}  // namespace nvfp4
