// C ABI of the 8-bit operators and of the experts' routing (declared in include/nvfp4.h): argument validation on the host, one launch
// function each.
#include <string.h>

#include "experts.h"

using namespace nvfp4;

namespace {

constexpr int64_t MOST_ROWS = INT32_MAX;                  // rows that offsets, orders and positions number
constexpr int64_t MOST_WIDTH = (int64_t)1 << 23;          // the products keep 32-bit byte offsets inside a tile's rows
constexpr int64_t MOST_GRID = INT32_MAX;                  // workgroups of a launch

template <class E>
inline int raw(const E &e)
{
    static_assert(sizeof(E) == sizeof(int), "C enumerations of this ABI are int-sized");
    int v;
    memcpy(&v, &e, sizeof(v));
    return v;
}
inline bool valid_dtype(int dt) { return dt == NVFP4_F32 || dt == NVFP4_BF16; }
inline bool valid_result(int dt) { return valid_dtype(dt) || dt == NVFP4_BF16_EXACT; }
inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline size_t elem(int dt) { return out_bytes(dt); }
inline nvfp4_status done(hipError_t e) { return e == hipSuccess ? NVFP4_OK : NVFP4_EHIP; }
inline int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }

// The operands and the output of a product whose sizes are above zero
nvfp4_status check_product(const uint8_t *A, const uint8_t *As, const uint8_t *B, const uint8_t *Bs, const void *out, int dt, bool operands)
{
    if (!out || (operands && (!A || !As || !B || !Bs))) return NVFP4_EINVAL;
    if (!aligned(A, 16) || !aligned(B, 16) || !aligned(out, elem(dt))) return NVFP4_EALIGN;
    return NVFP4_OK;
}

}  // namespace

extern "C" {

size_t nvfp4_fp8_codes_bytes(int64_t rows, int64_t K) { return rows > 0 && K > 0 ? (size_t)rows * FP8_BLOCK * ceil_div(K, FP8_BLOCK) : 0; }
size_t nvfp4_fp8_scales_bytes(int64_t rows, int64_t K) { return rows > 0 && K > 0 ? (size_t)rows * ceil_div(K, FP8_BLOCK) : 0; }
int64_t nvfp4_fp8_slots(int64_t rows, int64_t groups) { return rows < 0 || groups < 0 ? 0 : fp8_slots(rows, groups); }

nvfp4_status nvfp4_fp8_quantize(const void *x, nvfp4_dtype dt_, int64_t batch, int64_t rows, int64_t cols, int64_t ld,
                                const int32_t *order, int32_t top_k, int64_t x_rows, const int32_t *offsets, int32_t groups,
                                uint8_t *codes_rows, uint8_t *scales_rows, uint8_t *codes_cols, uint8_t *scales_cols,
                                void *stream)
{
    const int dt = raw(dt_);
    if (!valid_dtype(dt)) return NVFP4_EINVAL;
    if (batch < 0 || rows < 0 || cols < 0 || ld < cols || rows > MOST_ROWS || batch > MOST_ROWS || cols > MOST_WIDTH) return NVFP4_ESHAPE;
    if (!codes_rows != !scales_rows || !codes_cols != !scales_cols) return NVFP4_EINVAL;
    if (order && (top_k < 1 || x_rows < 0)) return NVFP4_EINVAL;
    if (offsets && (groups < 1 || groups > MAX_EXPERTS || !codes_cols)) return NVFP4_EINVAL;
    if ((order || offsets) && batch != 1) return NVFP4_ESHAPE;
    if (batch == 0 || rows == 0 || cols == 0) return NVFP4_OK;
    if ((!codes_rows && !codes_cols) || (!x && !(order && x_rows == 0))) return NVFP4_EINVAL;
    if (codes_cols && fp8_slots(rows, offsets ? groups : 0) > MOST_WIDTH / FP8_BLOCK) return NVFP4_ESHAPE;
    if (batch * rows > MOST_ROWS || (codes_cols && batch * cols > MOST_ROWS)) return NVFP4_ESHAPE;
    if (!aligned(x, elem(dt)) || !aligned(codes_rows, 16) || !aligned(codes_cols, 16) || !aligned(order, 4) || !aligned(offsets, 4)) return NVFP4_EALIGN;
    Fp8QuantArgs P;
    P.x = x;
    P.batch = batch;
    P.rows = rows;
    P.cols = cols;
    P.ld = ld;
    P.order = order;
    P.x_rows = x_rows;
    P.top_k = order ? top_k : 1;
    P.offsets = offsets;
    P.groups = offsets ? groups : 0;
    P.codes_r = codes_rows;
    P.scales_r = scales_rows;
    P.codes_c = codes_cols;
    P.scales_c = scales_cols;
    if (ceil_div(cols, FP8_BLOCK) * (ceil_div(rows, 4) + (offsets ? groups : 0)) * batch > MOST_GRID) return NVFP4_ESHAPE;
    return done(launch_fp8_quantize(P, dt, reinterpret_cast<hipStream_t>(stream)));
}

// Sizes of a product: within what the operands, offsets and launches count
static bool valid_sizes(Fp8Mode mode, int64_t M, int64_t N, int64_t K, int32_t groups)
{
    if (M < 0 || N < 0 || K < 0 || K % FP8_BLOCK != 0 || K > MOST_WIDTH || M > MOST_ROWS || N > MOST_ROWS) return false;
    if (mode != FP8_DENSE && (mode == FP8_EXPERTS ? groups * N : groups * M) > MOST_ROWS) return false;
    return (ceil_div(M, 16) + groups + 1) * ceil_div(N, 16) <= MOST_GRID / (mode == FP8_EXPERTS_DW ? groups : 1);
}

static nvfp4_status product(Fp8Mode mode, int64_t M, int64_t N, int64_t K, int32_t groups, const int32_t *offsets, int64_t total, const uint8_t *A_codes,
                            const uint8_t *A_scales, const uint8_t *B_codes, const uint8_t *B_scales, void *out, int out_dt, int64_t ldc, void *workspace, void *stream)
{
    if (!valid_result(out_dt)) return NVFP4_EINVAL;
    if (mode != FP8_DENSE && (groups < 1 || groups > MAX_EXPERTS || !offsets)) return NVFP4_EINVAL;
    if (ldc < N || !valid_sizes(mode, M, N, K, groups)) return NVFP4_ESHAPE;
    if (mode != FP8_DENSE && !aligned(offsets, 4)) return NVFP4_EALIGN;
    if (M == 0 || N == 0) return NVFP4_OK;
    const nvfp4_status s = check_product(A_codes, A_scales, B_codes, B_scales, out, out_dt, K > 0);
    if (s != NVFP4_OK) return s;
    Fp8GemmArgs P;
    P.M = M;
    P.N = N;
    P.blocks = (int32_t)(K / FP8_BLOCK);
    P.A = A_codes;
    P.A_scales = A_scales;
    P.B = B_codes;
    P.B_scales = B_scales;
    P.a_rows = M;
    P.b_rows = mode == FP8_EXPERTS ? groups * N : N;
    P.out = out;
    P.ldc = ldc;
    P.offsets = offsets;
    P.groups = mode == FP8_DENSE ? 0 : groups;
    P.total = (int32_t)total;
    P.partial = reinterpret_cast<float *>(workspace);
    return done(launch_fp8_gemm(P, mode, out_dt, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_fp8_gemm(int64_t M, int64_t N, int64_t K, const uint8_t *A_codes, const uint8_t *A_scales,
                            const uint8_t *B_codes, const uint8_t *B_scales, void *out, nvfp4_dtype out_dt, int64_t ldc,
                            void *stream)
{
    return product(FP8_DENSE, M, N, K, 0, nullptr, 0, A_codes, A_scales, B_codes, B_scales, out, raw(out_dt), ldc, nullptr, stream);
}

size_t nvfp4_fp8_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, nvfp4_dtype out_dt)
{
    if (!valid_result(raw(out_dt)) || M <= 0 || N <= 0 || K <= 0 || !valid_sizes(FP8_DENSE, M, N, K, 0)) return 0;
    Fp8GemmArgs P = {};
    P.M = M;
    P.N = N;
    P.blocks = (int32_t)(K / FP8_BLOCK);
    return fp8_gemm_workspace(P, raw(out_dt));
}

nvfp4_status nvfp4_fp8_gemm_ws(int64_t M, int64_t N, int64_t K, const uint8_t *A_codes, const uint8_t *A_scales,
                               const uint8_t *B_codes, const uint8_t *B_scales, void *out, nvfp4_dtype out_dt, int64_t ldc,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    const size_t need = nvfp4_fp8_gemm_workspace_bytes(M, N, K, out_dt);
    if (need > 0 && (!workspace || workspace_bytes < need)) return NVFP4_EWORKSPACE;
    if (need > 0 && !aligned(workspace, 16)) return NVFP4_EALIGN;
    return product(FP8_DENSE, M, N, K, 0, nullptr, 0, A_codes, A_scales, B_codes, B_scales, out, raw(out_dt), ldc, need > 0 ? workspace : nullptr, stream);
}

nvfp4_status nvfp4_fp8_gemm_experts(int64_t rows, int64_t N, int64_t K, int32_t groups, const int32_t *offsets,
                                    const uint8_t *A_codes, const uint8_t *A_scales, const uint8_t *B_codes,
                                    const uint8_t *B_scales, void *out, nvfp4_dtype out_dt, int64_t ldc, void *stream)
{
    return product(FP8_EXPERTS, rows, N, K, groups, offsets, rows, A_codes, A_scales, B_codes, B_scales, out, raw(out_dt), ldc, nullptr, stream);
}

nvfp4_status nvfp4_fp8_gemm_experts_dw(int64_t M, int64_t N, int64_t rows, int32_t groups, const int32_t *offsets,
                                       const uint8_t *A_codes, const uint8_t *A_scales, const uint8_t *B_codes,
                                       const uint8_t *B_scales, void *out, nvfp4_dtype out_dt, int64_t ldc, void *stream)
{
    if (rows < 0 || rows > MOST_ROWS) return NVFP4_ESHAPE;
    if (groups < 1 || groups > MAX_EXPERTS) return NVFP4_EINVAL;
    return product(FP8_EXPERTS_DW, M, N, FP8_BLOCK * fp8_slots(rows, groups), groups, offsets, rows, A_codes, A_scales, B_codes, B_scales, out, raw(out_dt), ldc,
                   nullptr, stream);
}

int nvfp4_host_fp8_gemm_kernel(int32_t call, int64_t M, int64_t N, int64_t K, int32_t groups, nvfp4_dtype out_dt, int32_t choice[5])
{
    const Fp8Mode mode = call == 2 ? FP8_EXPERTS : call == 3 ? FP8_EXPERTS_DW : FP8_DENSE;
    if (call < 0 || call > 3 || !choice || !valid_result(raw(out_dt)) || M <= 0 || N <= 0 || K < 0 || K > MOST_ROWS) return 0;
    if (mode == FP8_DENSE) groups = 0;
    else if (groups < 1 || groups > MAX_EXPERTS) return 0;
    if (mode == FP8_EXPERTS_DW) K = FP8_BLOCK * fp8_slots(K, groups);
    if (!valid_sizes(mode, M, N, K, groups)) return 0;
    Fp8GemmArgs P = {};
    P.M = M;
    P.N = N;
    P.ldc = N;
    P.blocks = (int32_t)(K / FP8_BLOCK);
    P.groups = groups;
    const Fp8Choice c = fp8_gemm_choice(P, mode, raw(out_dt), call == 1);
    choice[0] = c.kernel;
    choice[1] = c.rows;
    choice[2] = c.cols;
    choice[3] = c.parts;
    choice[4] = c.stream;
    return 1;
}

size_t nvfp4_moe_sort_workspace_bytes(int64_t pairs, int32_t groups)
{
    return pairs > 0 && pairs <= MOST_ROWS && groups >= 1 && groups <= MAX_EXPERTS ? moe_sort_workspace(pairs, groups) : 0;
}

nvfp4_status nvfp4_moe_sort(const void *experts, int32_t id_bytes, int64_t pairs, int32_t groups, int32_t *offsets,
                            int32_t *order, int32_t *position, void *workspace, size_t workspace_bytes, void *stream)
{
    if (id_bytes != 4 && id_bytes != 8) return NVFP4_EINVAL;
    if (pairs < 0 || pairs > MOST_ROWS) return NVFP4_ESHAPE;
    if (groups < 1 || groups > MAX_EXPERTS || !offsets || (pairs > 0 && (!experts || !order || !position))) return NVFP4_EINVAL;
    if (!aligned(experts, (size_t)id_bytes) || !aligned(offsets, 4) || !aligned(order, 4) || !aligned(position, 4) || !aligned(workspace, 4)) return NVFP4_EALIGN;
    const size_t need = nvfp4_moe_sort_workspace_bytes(pairs, groups);
    if (need && (!workspace || workspace_bytes < need)) return NVFP4_EWORKSPACE;
    return done(launch_moe_sort(experts, id_bytes, pairs, groups, offsets, order, position, reinterpret_cast<int32_t *>(workspace),
                                reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_moe_gather(const void *x, nvfp4_dtype dt_, int64_t x_rows, int64_t cols, int64_t ld, const int32_t *order,
                              int32_t top_k, int64_t rows, void *out, void *stream)
{
    const int dt = raw(dt_);
    if (!valid_dtype(dt) || top_k < 1) return NVFP4_EINVAL;
    if (x_rows < 0 || cols < 0 || ld < cols || rows < 0 || rows > MOST_ROWS) return NVFP4_ESHAPE;
    if (rows == 0 || cols == 0) return NVFP4_OK;
    if ((!x && x_rows > 0) || !order || !out) return NVFP4_EINVAL;
    if (!aligned(x, elem(dt)) || !aligned(out, elem(dt)) || !aligned(order, 4)) return NVFP4_EALIGN;
    return done(launch_moe_gather(x, dt, x_rows, cols, ld, order, top_k, rows, out, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_moe_combine_to(const void *y, nvfp4_dtype dt_, int64_t rows, int64_t cols, const float *weights,
                                  const int32_t *position, int64_t tokens, int32_t top_k, void *out, nvfp4_dtype out_dt_,
                                  void *stream)
{
    const int dt = raw(dt_), out_dt = raw(out_dt_);
    if (!valid_dtype(dt) || !valid_dtype(out_dt) || top_k < 1) return NVFP4_EINVAL;
    if (rows < 0 || rows > MOST_ROWS || cols < 0 || tokens < 0 || tokens > MOST_ROWS / top_k) return NVFP4_ESHAPE;
    if (tokens == 0 || cols == 0) return NVFP4_OK;
    if ((!y && rows > 0) || !position || !out) return NVFP4_EINVAL;
    if (!aligned(y, elem(dt)) || !aligned(out, elem(out_dt)) || !aligned(position, 4) || !aligned(weights, 4)) return NVFP4_EALIGN;
    return done(launch_moe_combine(y, dt, rows, cols, weights, position, tokens, top_k, out, out_dt, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_moe_combine(const void *y, nvfp4_dtype dt, int64_t rows, int64_t cols, const float *weights,
                               const int32_t *position, int64_t tokens, int32_t top_k, void *out, void *stream)
{
    return nvfp4_moe_combine_to(y, dt, rows, cols, weights, position, tokens, top_k, out, dt, stream);
}

nvfp4_status nvfp4_moe_combine_to_bwd(const void *dout, nvfp4_dtype dout_dt_, const void *y, nvfp4_dtype dt_, int64_t rows,
                                      int64_t cols, const float *weights, const int32_t *position, const int32_t *offsets,
                                      int32_t groups, int64_t tokens, int32_t top_k, void *dy, float *dweights, void *stream)
{
    const int dt = raw(dt_), dout_dt = raw(dout_dt_);
    if (!valid_dtype(dt) || !valid_dtype(dout_dt) || top_k < 1 || groups < 1 || groups > MAX_EXPERTS) return NVFP4_EINVAL;
    if (rows < 0 || rows > MOST_ROWS || cols < 0 || tokens < 0 || tokens > MOST_ROWS / top_k) return NVFP4_ESHAPE;
    if (tokens == 0 && (rows == 0 || cols == 0)) return NVFP4_OK;
    if (!offsets || (tokens > 0 && (!weights || !position || !dweights)) || (cols > 0 && ((tokens > 0 && !dout) || (rows > 0 && (!y || !dy))))) return NVFP4_EINVAL;
    if (!aligned(dout, elem(dout_dt)) || !aligned(y, elem(dt)) || !aligned(dy, elem(dt)) || !aligned(weights, 4) || !aligned(position, 4) || !aligned(offsets, 4) ||
        !aligned(dweights, 4))
        return NVFP4_EALIGN;
    return done(launch_moe_combine_bwd(dout, dout_dt, y, dt, rows, cols, weights, position, offsets + groups, tokens, top_k, dy, dweights,
                                       reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_moe_combine_bwd(const void *dout, const void *y, nvfp4_dtype dt, int64_t rows, int64_t cols,
                                   const float *weights, const int32_t *position, const int32_t *offsets, int32_t groups,
                                   int64_t tokens, int32_t top_k, void *dy, float *dweights, void *stream)
{
    return nvfp4_moe_combine_to_bwd(dout, dt, y, dt, rows, cols, weights, position, offsets, groups, tokens, top_k, dy, dweights, stream);
}

}  // extern "C"
