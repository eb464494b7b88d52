// Internal interface between the C ABI (api_experts.hip) and the launchers of the 8-bit operators and of the experts' routing.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/nvfp4.h"

namespace nvfp4 {

constexpr int FP8_BLOCK = 128;      // elements that share a scale, contraction elements of a K tile, bytes of a row of one
constexpr int MAX_EXPERTS = 512;

// A launch counts the threads along an axis in 32 bits: workgroups 0 .. n - 1 in rows of LAUNCH_ROW, the last of which may have some past n.
constexpr int64_t LAUNCH_ROW = (int64_t)1 << 22;  // (512 threads each at the most)
inline dim3 launch_grid(int64_t n) { return n <= LAUNCH_ROW ? dim3((unsigned)n) : dim3((unsigned)LAUNCH_ROW, (unsigned)((n + LAUNCH_ROW - 1) / LAUNCH_ROW)); }
__device__ __forceinline__ unsigned workgroup() { return blockIdx.y * gridDim.x + blockIdx.x; }

// A tensor to quantize in blocks of 128: rows, columns or both.  With `order` its row r is row order[r] / top_k of x (none: zeros).
// With `offsets` [groups + 1] the column blocks start anew at each group's first row.
struct Fp8QuantArgs {
    const void *x;
    int64_t batch, rows, cols, ld;  // `batch` matrices of rows x cols, one behind the other in rows of pitch ld
    const int32_t *order;
    int64_t x_rows;                 // rows of x that an order may name
    int32_t top_k;
    const int32_t *offsets;
    int32_t groups;
    uint8_t *codes_r, *scales_r;    // [batch * rows, 128 ceil(cols / 128)], [ceil(cols / 128), batch * rows]
    uint8_t *codes_c, *scales_c;    // [batch * cols, 128 slots], [slots, batch * cols]
};
// Blocks along the rows of a matrix: whole matrices, or groups of rows, each of which begins at the first free slot
// floor(first row / 128) + group (so that no slot depends on the lengths of other groups, and 128 more per group are enough).
inline int64_t fp8_slots(int64_t rows, int64_t groups) { return groups > 0 ? rows / FP8_BLOCK + groups : (rows + FP8_BLOCK - 1) / FP8_BLOCK; }
hipError_t launch_fp8_quantize(const Fp8QuantArgs &P, int dt, hipStream_t st);

// What a group of rows is: rows first .. first + count - 1 of those that the offsets divide.  Offsets come from the device: whatever they
// hold, the rows stay inside [0, total].
struct RowGroup {
    int32_t first, count;
};
__device__ __forceinline__ RowGroup row_group(const int32_t *offsets, int e, int32_t total)
{
    int32_t a = offsets[e], b = offsets[e + 1];
    a = a < 0 ? 0 : a > total ? total : a;
    b = b < a ? a : b > total ? total : b;
    return {a, b - a};
}
// Group e that slot s belongs to, where group e owns the slots from floor(first row / step) + e on: the last one that starts at or before s
// (`groups` of them; every wave asks for itself).
__device__ __forceinline__ int group_of_slot(const int32_t *offsets, int groups, int32_t total, int step, int s)
{
    int n = 0;
    for (int e0 = 0; e0 < groups; e0 += 64) {
        const int e = e0 + (int)(threadIdx.x & 63);
        int32_t a = 0;
        if (e < groups) {
            a = offsets[e];
            a = a < 0 ? 0 : a > total ? total : a;
        }
        n += __popcll(__ballot(e < groups && a / step + e <= s));
    }
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// out = A B^T of quantized operands [rows, 128 blocks].  FP8_DENSE: one product.  FP8_EXPERTS: the M rows of A and of the output are divided
// by offsets among `groups` experts, expert e's against rows e N .. e N + N - 1 of B; rows of no expert become zeros.  FP8_EXPERTS_DW: one
// M x N output for each expert, the contraction over its slots of A and B.  FP8_DIVIDED: one product, the contraction divided among `groups` workgroups a tile, whose
// sums meet in `partial`.
enum Fp8Mode { FP8_DENSE, FP8_EXPERTS, FP8_EXPERTS_DW, FP8_DIVIDED };
struct Fp8GemmArgs {
    int64_t M, N;
    int32_t blocks;                       // 128s of the operands' rows
    const uint8_t *A, *A_scales, *B, *B_scales;
    int64_t a_rows, b_rows;               // rows of the operands: pitch of their scales
    void *out;
    int64_t ldc;
    const int32_t *offsets;
    int32_t groups, total;                // total (FP8_EXPERTS_DW): the rows that the offsets divide
    float *partial;                       // FP8_DIVIDED
    int32_t stream;                       // the output leaves by nontemporal stores (set by launch_fp8_gemm())
};
// Whether results of a type come of exact products in binary32 sums (fp8_gemm.h); their bytes
constexpr bool exact_sums(int out_dt) { return out_dt != NVFP4_BF16; }
constexpr int out_bytes(int out_dt) { return out_dt == NVFP4_F32 ? 4 : 2; }
// Which kernel, the rows and columns of a workgroup's tile, K tiles of a batch (few rows) or workgroups of a tile (divided), else 1, and whether the output is streamed
struct Fp8Choice {
    enum Kernel { FEW_ROWS, TILES, WIDE, DIVIDED } kernel;
    int rows, cols, parts;
    bool stream;
};
// `scratch`: of a dense product, whether there is memory at `partial`
Fp8Choice fp8_gemm_choice(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, bool scratch);
// The kernels that launch_fp8_gemm() chooses from, with what a K tile of the contraction takes them, in us: waves that divide the contraction, for outputs of
// few tiles; 256 rows by 128 to 256 columns (binary32 outputs: 128); 128 x 128.
double fp8_gemm_thin_cost(const Fp8GemmArgs &P);
void fp8_gemm_thin_choice(const Fp8GemmArgs &P, Fp8Mode mode, Fp8Choice *c);
hipError_t launch_fp8_gemm_thin(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, const Fp8Choice &c, hipStream_t st);
double fp8_gemm_wide_cost(const Fp8GemmArgs &P, int mode, int out_dt);
int fp8_gemm_wide_cols(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt);  // of a tile
hipError_t launch_fp8_gemm_wide(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, int cols, hipStream_t st);
int64_t compute_units();
// Among how many workgroups that kernel divides a dense product's contraction to be quickest (1: not at all, or not in less than `below` us), the bytes that it then
// needs at `partial`, and its time in us
int fp8_gemm_parts(const Fp8GemmArgs &P, int out_dt, double below, size_t *bytes, double *cost);
size_t fp8_gemm_workspace(const Fp8GemmArgs &P, int out_dt);
hipError_t launch_fp8_gemm(const Fp8GemmArgs &P, Fp8Mode mode, int out_dt, hipStream_t st);

// Routing
size_t moe_sort_workspace(int64_t pairs, int32_t groups);
hipError_t launch_moe_sort(const void *experts, int id_bytes, int64_t pairs, int32_t groups, int32_t *offsets, int32_t *order, int32_t *position,
                           int32_t *workspace, hipStream_t st);
hipError_t launch_moe_gather(const void *x, int dt, int64_t x_rows, int64_t cols, int64_t ld, const int32_t *order, int32_t top_k, int64_t rows, void *out,
                             hipStream_t st);
hipError_t launch_moe_combine(const void *y, int dt, int64_t y_rows, int64_t cols, const float *weights, const int32_t *position, int64_t tokens,
                              int32_t top_k, void *out, int out_dt, hipStream_t st);
hipError_t launch_moe_combine_bwd(const void *dout, int dout_dt, const void *y, int dt, int64_t rows, int64_t cols, const float *weights, const int32_t *position,
                                  const int32_t *kept, int64_t tokens, int32_t top_k, void *dy, float *dweights, hipStream_t st);

}  // namespace nvfp4
