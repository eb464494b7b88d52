// C ABI of the operators around the products: the experts' router with its balance loss, rows' norms, products with packed 4-bit weights (declared in
// include/nvfp4.h): argument validation on the host, one launch function each.
#include <math.h>
#include <string.h>

#include "layer_ops.h"

using namespace nvfp4;

namespace {

constexpr int64_t MOST_ROWS = INT32_MAX;
constexpr int64_t MOST_WIDTH = (int64_t)1 << 23;
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
inline bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline size_t elem(int dt) { return dt == NVFP4_F32 ? 4 : 2; }
inline nvfp4_status done(hipError_t e) { return e == hipSuccess ? NVFP4_OK : NVFP4_EHIP; }

// What the three calls on router logits share
nvfp4_status check_logits(int dt, int64_t tokens, int32_t groups, int64_t ld, int32_t top_k)
{
    if (!valid_dtype(dt) || groups < 1 || groups > MAX_EXPERTS || top_k < 1 || top_k > groups) return NVFP4_EINVAL;
    if (tokens < 0 || tokens > MOST_ROWS / top_k || ld < groups) return NVFP4_ESHAPE;
    return NVFP4_OK;
}

}  // namespace

extern "C" {

nvfp4_status nvfp4_moe_route(const void *logits, nvfp4_dtype dt_, int64_t tokens, int32_t groups, int64_t ld, int32_t top_k,
                             int renormalize, int32_t *experts, float *weights, void *stream)
{
    const int dt = raw(dt_);
    const nvfp4_status s = check_logits(dt, tokens, groups, ld, top_k);
    if (s != NVFP4_OK) return s;
    if (tokens == 0) return NVFP4_OK;
    if (!logits || !experts || !weights) return NVFP4_EINVAL;
    if (!aligned(logits, elem(dt)) || !aligned(experts, 4) || !aligned(weights, 4)) return NVFP4_EALIGN;
    const RouteArgs P = {logits, tokens, ld, groups, top_k, renormalize != 0};
    return done(launch_moe_route(P, dt, experts, weights, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_moe_route_bwd(const void *logits, nvfp4_dtype dt_, int64_t tokens, int32_t groups, int64_t ld, int32_t top_k,
                                 int renormalize, const int32_t *experts, const float *dweights, const int32_t *counts,
                                 const float *dlosses, void *dlogits, void *stream)
{
    const int dt = raw(dt_);
    const nvfp4_status s = check_logits(dt, tokens, groups, ld, top_k);
    if (s != NVFP4_OK) return s;
    if (!counts != !dlosses) return NVFP4_EINVAL;
    if (tokens == 0) return NVFP4_OK;
    if (!logits || !dlogits || (!dweights && !counts) || (dweights && !experts)) return NVFP4_EINVAL;
    if (!aligned(logits, elem(dt)) || !aligned(dlogits, elem(dt)) || !aligned(experts, 4) || !aligned(dweights, 4) || !aligned(counts, 4) || !aligned(dlosses, 4)) return NVFP4_EALIGN;
    const RouteArgs P = {logits, tokens, ld, groups, top_k, renormalize != 0};
    return done(launch_moe_route_bwd(P, dt, experts, dweights, counts, dlosses, dlogits, reinterpret_cast<hipStream_t>(stream)));
}

size_t nvfp4_moe_balance_workspace_bytes(int64_t tokens, int32_t groups)
{
    return tokens > 0 && tokens <= MOST_ROWS && groups >= 1 && groups <= MAX_EXPERTS ? moe_balance_workspace(tokens, groups) : 0;
}

nvfp4_status nvfp4_moe_balance(const void *logits, nvfp4_dtype dt_, int64_t tokens, int32_t groups, int64_t ld,
                               const void *experts, int32_t id_bytes, int32_t top_k, float *losses, int32_t *counts,
                               float *probs, void *workspace, size_t workspace_bytes, void *stream)
{
    const int dt = raw(dt_);
    if (id_bytes != 4 && id_bytes != 8) return NVFP4_EINVAL;
    const nvfp4_status s = check_logits(dt, tokens, groups, ld, top_k);
    if (s != NVFP4_OK) return s;
    if (!losses || !counts || !probs || (tokens > 0 && (!logits || !experts))) return NVFP4_EINVAL;
    if (!aligned(logits, elem(dt)) || !aligned(experts, (size_t)id_bytes) || !aligned(losses, 4) || !aligned(counts, 4) || !aligned(probs, 4) || !aligned(workspace, 4)) return NVFP4_EALIGN;
    const size_t need = nvfp4_moe_balance_workspace_bytes(tokens, groups);
    if (need && (!workspace || workspace_bytes < need)) return NVFP4_EWORKSPACE;
    const RouteArgs P = {logits, tokens, ld, groups, top_k, true};
    return done(launch_moe_balance(P, dt, experts, id_bytes, losses, counts, probs, workspace, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_layer_norm(const void *x, nvfp4_dtype dt_, int64_t rows, int64_t cols, int64_t ld, const void *weight,
                              const void *bias, nvfp4_dtype weight_dt_, int center, float eps, void *y, float *mean, float *rstd,
                              void *stream)
{
    const int dt = raw(dt_), wdt = raw(weight_dt_);
    if (!valid_dtype(dt) || !valid_dtype(wdt) || !(eps >= 0.0f) || isinf(eps)) return NVFP4_EINVAL;
    if (rows < 0 || rows > MOST_ROWS || cols < 0 || cols > MOST_WIDTH || ld < cols) return NVFP4_ESHAPE;
    if (rows == 0 || cols == 0) return NVFP4_OK;
    if (!x || !y) return NVFP4_EINVAL;
    if (!aligned(x, elem(dt)) || !aligned(y, elem(dt)) || !aligned(weight, elem(wdt)) || !aligned(bias, elem(wdt)) || !aligned(mean, 4) || !aligned(rstd, 4)) return NVFP4_EALIGN;
    const NormArgs P = {rows, cols, ld, weight, bias, wdt, center != 0};
    return done(launch_layer_norm(P, dt, x, eps, y, mean, rstd, reinterpret_cast<hipStream_t>(stream)));
}

size_t nvfp4_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols, nvfp4_dtype dt_, int dweight, int dbias)
{
    const int dt = raw(dt_);
    if (!valid_dtype(dt) || rows <= 0 || rows > MOST_ROWS || cols <= 0 || cols > MOST_WIDTH) return 0;
    return layer_norm_bwd_workspace(rows, cols, dt, dweight != 0, dbias != 0);
}

nvfp4_status nvfp4_layer_norm_bwd(const void *dy, int64_t ldy, const void *x, int64_t ld, nvfp4_dtype dt_, int64_t rows, int64_t cols,
                                  const void *weight, nvfp4_dtype weight_dt_, const float *mean, const float *rstd, void *dx,
                                  void *dweight, void *dbias, void *workspace, size_t workspace_bytes, void *stream)
{
    const int dt = raw(dt_), wdt = raw(weight_dt_);
    if (!valid_dtype(dt) || !valid_dtype(wdt)) return NVFP4_EINVAL;
    if (rows < 0 || rows > MOST_ROWS || cols < 0 || cols > MOST_WIDTH || ld < cols || ldy < cols) return NVFP4_ESHAPE;
    if (cols == 0) return NVFP4_OK;
    if (rows > 0 && (!dy || !x || !rstd || !dx)) return NVFP4_EINVAL;
    if (!aligned(dy, elem(dt)) || !aligned(x, elem(dt)) || !aligned(dx, elem(dt)) || !aligned(weight, elem(wdt)) || !aligned(dweight, elem(wdt)) || !aligned(dbias, elem(wdt)) ||
        !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(workspace, 16))
        return NVFP4_EALIGN;
    const size_t need = nvfp4_layer_norm_bwd_workspace_bytes(rows, cols, dt_, dweight != nullptr, dbias != nullptr);
    if (need && (!workspace || workspace_bytes < need)) return NVFP4_EWORKSPACE;
    const NormArgs P = {rows, cols, ld, weight, nullptr, wdt, mean != nullptr};
    return done(launch_layer_norm_bwd(P, dt, dy, ldy, x, mean, rstd, dx, dweight, dbias, workspace, reinterpret_cast<hipStream_t>(stream)));
}

static bool w4_sizes(int64_t rows, int64_t N, int64_t K, int32_t groups)
{
    return rows >= 0 && rows <= MOST_ROWS && N >= 0 && N <= MOST_ROWS && (groups <= 0 || groups * N <= MOST_ROWS) && K >= 0 && K <= MOST_WIDTH && K % 32 == 0 &&
           (rows / 16 + groups + 2) * (N / 16 + 1) <= MOST_GRID;
}

static nvfp4_status product_w4(int64_t rows, int64_t N, int64_t K, int32_t groups, const int32_t *offsets, const nvfp4_format *f, const void *x, int x_dt, int64_t ldx,
                               int64_t x_rows, const int32_t *order, int32_t top_k, const uint8_t *codes, const uint8_t *scales, const float *g, int32_t g_step, void *out,
                               int out_dt, int64_t ldc, void *stream)
{
    if (!f || !valid_dtype(x_dt) || !valid_dtype(out_dt)) return NVFP4_EINVAL;
    if ((f->scale != NVFP4_SCALE_E4M3 && f->scale != NVFP4_SCALE_E8M0) || (f->tensor_scale != 0 && f->tensor_scale != 1)) return NVFP4_EINVAL;
    if (f->scale == NVFP4_SCALE_E8M0 ? f->block != 32 || f->tensor_scale : f->block != 16 && f->block != 32 && f->block != 64 && f->block != 128) return NVFP4_EUNSUPPORTED;
    if (!w4_sizes(rows, N, K, groups) || K % f->block != 0 || ldx < K || ldc < N || x_rows < 0) return NVFP4_ESHAPE;
    if (!aligned(offsets, 4) || !aligned(order, 4)) return NVFP4_EALIGN;
    if (rows == 0 || N == 0) return NVFP4_OK;
    if (!out || (K > 0 && ((!x && x_rows > 0) || !codes || !scales)) || (f->tensor_scale && !g)) return NVFP4_EINVAL;
    if (!aligned(x, elem(x_dt)) || !aligned(out, elem(out_dt)) || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(g, 4)) return NVFP4_EALIGN;
    W4Args P = {};
    P.x = reinterpret_cast<const uint8_t *>(x);
    P.rows = rows;
    P.x_rows = x_rows;
    P.ldx = ldx;
    P.N = N;
    P.K = K;
    P.codes = codes;
    P.scales = scales;
    P.g = f->tensor_scale && K > 0 ? g : nullptr;  // (a sum of nothing is 0 whatever g is)
    P.g_step = g_step;
    P.block = f->block;
    P.scale = f->scale;
    P.offsets = offsets;
    P.order = order;
    P.groups = groups;
    P.top_k = top_k;
    P.out = reinterpret_cast<uint8_t *>(out);
    P.ldc = ldc;
    return done(launch_gemm_w4(P, x_dt, out_dt, reinterpret_cast<hipStream_t>(stream)));
}

nvfp4_status nvfp4_gemm_w4(int64_t M, int64_t N, int64_t K, const nvfp4_format *f, const void *x, nvfp4_dtype x_dt, int64_t ldx,
                           const uint8_t *W_codes, const uint8_t *W_scales, const float *W_scale, void *out, nvfp4_dtype out_dt,
                           int64_t ldc, void *stream)
{
    return product_w4(M, N, K, 0, nullptr, f, x, raw(x_dt), ldx, M, nullptr, 1, W_codes, W_scales, W_scale, 0, out, raw(out_dt), ldc, stream);
}

nvfp4_status nvfp4_gemm_w4_experts(int64_t rows, int64_t N, int64_t K, int32_t groups, const int32_t *offsets, const nvfp4_format *f,
                                   const void *x, nvfp4_dtype x_dt, int64_t ldx, int64_t x_rows, const int32_t *order, int32_t top_k,
                                   const uint8_t *W_codes, const uint8_t *W_scales, const float *W_scale, int32_t W_scale_step,
                                   void *out, nvfp4_dtype out_dt, int64_t ldc, void *stream)
{
    if (groups < 1 || groups > MAX_EXPERTS || !offsets || (order && top_k < 1) || (W_scale_step != 0 && W_scale_step != 1)) return NVFP4_EINVAL;
    if (!order && x_rows < rows) return NVFP4_ESHAPE;
    return product_w4(rows, N, K, groups, offsets, f, x, raw(x_dt), ldx, x_rows, order, order ? top_k : 1, W_codes, W_scales, W_scale, W_scale_step, out, raw(out_dt), ldc, stream);
}

int nvfp4_host_gemm_w4_kernel(int64_t rows, int64_t N, int64_t K, int32_t groups, nvfp4_dtype x_dt, int x_aligned, int32_t choice[4])
{
    if (!choice || !valid_dtype(raw(x_dt)) || rows <= 0 || N <= 0 || groups < 0 || groups > MAX_EXPERTS || !w4_sizes(rows, N, K, groups)) return 0;
    W4Args P = {};
    P.x = reinterpret_cast<const uint8_t *>(x_aligned ? 16 : 18);  // (nobody follows it)
    P.rows = P.x_rows = rows;
    P.ldx = K;
    P.N = P.ldc = N;
    P.K = K;
    P.groups = groups;
    P.top_k = 1;
    const W4Choice c = gemm_w4_choice(P, raw(x_dt));
    choice[0] = c.kernel;
    choice[1] = c.rows;
    choice[2] = c.cols;
    choice[3] = c.waves;
    return 1;
}

}  // extern "C"
