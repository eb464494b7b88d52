// The experts' router: from logits [T, E] each token's top_k experts and their weights, the balance of a batch over the experts, and the gradient of the
// logits of both.
//   route    the k largest of a row, ties to the lower expert, -inf never; w_j = exp(l_j - lse), lse over the row, or over the chosen
//   balance  N rows have an entry above -inf; p = softmax(row); f_e = pairs of e / (N k), P_e = sum_t p_te / N;  E sum_e f_e P_e  and  sum_t lse_t^2 / N
//   bwd      of weights over the chosen: dl_e = w_e (dw_e - sum_i w_i dw_i);  over the row: p_e (dw_e - sum_i w_i dw_i), dw_e = 0 where e is not chosen;
//            of the balance: dL0 (E / N) p_e (f_e - sum_i f_i p_i), f taken as constants;  of lse^2: dL1 (2 / N) lse p_e
// G lanes hold a row, eight entries each, so that a row of up to 512 experts is in registers and read once.
// us, kernels alone, rows from memory / from the last cache: route 16 x 8 2.5 (a launch), 32768 x 128 bf16 k 8 11.1 / 10.5: eight rounds of some 50 instructions, where its 8 MB take 1.6; bwd
// 32768 x 128 binary32 with both gradients 17.5 / 15.8 (34 MB: 6.3 at a copy's rate; the rest exponentials and the search of the choices' lanes, 64 compares a lane); balance 32768 x 256 bf16
// 14.7 / 13.0 (17 MB: 3.2; a group of lanes asks for its next row when it is done with one) + 10 (one workgroup reads 526 KB of sums).
#include <math.h>

#include "layer_ops.h"

namespace nvfp4 {
namespace route {

using namespace layer;

constexpr int V = 8;  // entries of a lane
constexpr float NONE = -INFINITY;

// Numbers in their order as unsigned integers, zeros equal; every NaN above all of them, 0 below
__device__ __forceinline__ uint32_t key_of(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return f != f ? 0xFFFFFFFFu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k ^ ((uint32_t)((int32_t)~k >> 31) | 0x80000000u)); }
constexpr uint32_t KEY_NONE = 0x007FFFFFu;  // of -inf

template <int DT, int G>
__device__ __forceinline__ void load_row(float (&v)[V], const uint8_t *logits, int64_t ld, int64_t t, int groups, bool there)
{
    const int c = (threadIdx.x & (G - 1)) * V;
    load_run<DT, V>(v, logits + (t * ld + c) * Elem<DT>::BYTES, there ? groups - c : 0, NONE);
}

// Softmax of a row in the lanes that hold it: v becomes p (zeros without an entry above -inf); lse (0 then), and whether there is one
template <int G>
__device__ __forceinline__ bool softmax(float (&v)[V], float *lse)
{
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t k = key_of(v[i]);
        most = k > most ? k : most;
    }
    most = group_most<G>(most);
    const bool kept = most > KEY_NONE;
    const float top = kept ? of_key(most) : 0.0f;
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        v[i] = expf(v[i] - top);
        sum += v[i];
    }
    sum = group_sum<G>(sum);
    const float share = kept ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= share;
    *lse = kept ? logf(sum) + top : 0.0f;
    return kept;
}

}  // namespace route

// Each of k rounds takes the largest entry that is left: a maximum over the lane's entries, one over the row's lanes, and of the lanes that have it the
// first one (entries lie in the experts' order) gives it up.
template <int DT, int G>
__global__ __launch_bounds__(256) void moe_route_kernel(const uint8_t *logits, int64_t tokens, int groups, int64_t ld, int top_k, int renormalize, int32_t *experts,
                                                        float *weights)
{
    using namespace route;
    const int lane = threadIdx.x & 63, g = threadIdx.x & (G - 1);
    const int64_t t = (int64_t)workgroup() * (256 / G) + threadIdx.x / G;
    const bool there = t < tokens;
    float v[V];
    load_row<DT, G>(v, logits, ld, t, groups, there);
    uint32_t key[V], most = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        key[i] = g * V + i < groups ? key_of(v[i]) : 0;
        most = key[i] > most ? key[i] : most;
    }
    most = group_most<G>(most);
    const float top = most > KEY_NONE ? of_key(most) : 0.0f;
    float sum = 0.0f;
    if (!renormalize) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum += expf(v[i] - top);
        sum = group_sum<G>(sum);
    }
    extern __shared__ float staged[];  // the chosen logits: [256 / G][top_k]
    float *const mine = staged + threadIdx.x / G * top_k;
    for (int j = 0; j < top_k; ++j) {
        if (j > 0) {
            most = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) most = key[i] > most ? key[i] : most;
            most = group_most<G>(most);
        }
        const bool chosen = most > KEY_NONE;
        int first = V;
#pragma unroll
        for (int i = V - 1; i >= 0; --i)
            if (key[i] == most) first = i;
        const uint64_t have = __ballot(first < V) >> (lane & ~(G - 1));
        const bool wins = __builtin_ctzll(have) == g;
        if (wins && there) {
            experts[t * top_k + j] = chosen ? g * V + first : -1;
            mine[j] = chosen ? of_key(most) : NONE;
        }
        if (wins && chosen) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i == first) key[i] = 0;
        }
    }
    __syncthreads();
    // the row's lanes share its choices; the exponentials once, outside the rounds
    const float mark = NONE;
    if (renormalize) {
        for (int j = g; j < top_k; j += G) {
            const float l = there ? mine[j] : mark;
            const float e = l == mark ? 0.0f : expf(l - top);
            if (there && l != mark) mine[j] = e;
            if (there && l == mark) mine[j] = -1.0f;
            sum += e;
        }
        sum = group_sum<G>(sum);
    }
    if (!there) return;
    for (int j = g; j < top_k; j += G) {
        float e = mine[j];
        if (!renormalize) e = e == mark ? -1.0f : expf(e - top);
        weights[t * top_k + j] = e < 0.0f ? 0.0f : e / sum;
    }
}

template <int DT, int G>
__global__ __launch_bounds__(256) void moe_route_bwd_kernel(const uint8_t *logits, int64_t tokens, int groups, int64_t ld, int top_k, int renormalize, const int32_t *experts,
                                                            const float *dweights, const int32_t *counts, const float *dlosses, uint8_t *dlogits)
{
    using namespace route;
    const int g = threadIdx.x & (G - 1);
    const int64_t t = (int64_t)workgroup() * (256 / G) + threadIdx.x / G;
    if (t >= tokens) return;  // (whole groups of lanes)
    float l[V], d[V];
    load_row<DT, G>(l, logits, ld, t, groups, true);
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = 0.0f;
    float up[V], times[V];  // sums of dw over the choices of an entry, and how many these are
    if (dweights) {
#pragma unroll
        for (int i = 0; i < V; ++i) up[i] = times[i] = 0.0f;
        for (int j0 = 0; j0 < top_k; j0 += 8) {  // (loads of eight choices at a time)
            int at[8];
            float dw[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int64_t j = t * top_k + (j0 + u < top_k ? j0 + u : 0);
                at[u] = experts[j];
                dw[u] = dweights[j];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                at[u] = j0 + u < top_k && (unsigned)at[u] < (unsigned)groups ? at[u] - g * V : -1;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at[u] == i) {
                        up[i] += dw[u];
                        times[i] += 1.0f;
                    }
            }
        }
        if (renormalize) {
            uint32_t most = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t k = times[i] > 0.0f ? key_of(l[i]) : 0;
                most = k > most ? k : most;
            }
            most = group_most<G>(most);
            const float top = most > KEY_NONE ? of_key(most) : 0.0f;
            float w[V], sum = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                w[i] = times[i] > 0.0f ? expf(l[i] - top) : 0.0f;
                sum += w[i] * times[i];
                dot += w[i] * up[i];
            }
            sum = group_sum<G>(sum);
            dot = group_sum<G>(dot);
            if (most > KEY_NONE) {
                const float share = 1.0f / sum;
                dot *= share;
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] = w[i] * share * (up[i] - times[i] * dot);
            }
        }
    }
    if (counts || (dweights && !renormalize)) {
        float lse;
        const bool kept = softmax<G>(l, &lse);
        if (dweights && !renormalize) {
            float dot = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) dot += l[i] * up[i];
            dot = group_sum<G>(dot);
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] = l[i] * (up[i] - dot);
        }
        if (counts) {
            const int rows = counts[groups];
            const float n = rows > 1 ? (float)rows : 1.0f, per = 1.0f / (n * (float)top_k);
            float f[V], dot = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[i] = g * V + i < groups ? (float)counts[g * V + i] * per : 0.0f;
                dot += f[i] * l[i];
            }
            dot = group_sum<G>(dot);
            const float a = dlosses[0] * (float)groups / n, b = dlosses[1] * 2.0f / n * lse;
#pragma unroll
            for (int i = 0; i < V; ++i) d[i] += l[i] * (a * (f[i] - dot) + b);
        }
        // (also where what comes back is not a number: 0 times it is none either)
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] = kept ? d[i] : 0.0f;
    }
    store_run<DT, V>(d, dlogits + (t * groups + g * V) * Elem<DT>::BYTES, groups - g * V);
}

namespace route {

// Both losses and the means from the sums over all tokens; s_sums, s_counts: [groups + 1] in the LDS, behind a barrier
__device__ __forceinline__ void balance_end(const float *s_sums, const int *s_counts, int groups, int top_k, int threads, float *per_wave, float *losses, int32_t *counts, float *probs)
{
    const int tid = threadIdx.x, kept = s_counts[groups];
    const float n = kept > 1 ? (float)kept : 1.0f, per = 1.0f / (n * (float)top_k);
    float loss = 0.0f;
    for (int e = tid; e < groups; e += threads) {
        const float p = s_sums[e] / n;
        loss += (float)s_counts[e] * per * p;
        probs[e] = p;
        counts[e] = s_counts[e];
    }
    loss = group_sum<64>(loss);
    if ((tid & 63) == 0) per_wave[tid >> 6] = loss;
    __syncthreads();
    if (tid == 0) {
        loss = 0.0f;
        for (int w = 0; w < threads / 64; ++w) loss += per_wave[w];
        losses[0] = (float)groups * loss;
        losses[1] = s_sums[groups] / n;
        counts[groups] = kept;
    }
}

}  // namespace route

constexpr int BALANCE_NT = 512;

// A workgroup's tokens first .. last - 1: probabilities summed by the lanes that hold the columns, then over the workgroup's rows in their order.  What it leaves of them: probabilities
// summed and lse^2 summed [groups + 1]; pairs and tokens [groups + 1].
template <int DT, int G, typename ID>
__global__ __launch_bounds__(BALANCE_NT) void moe_balance_kernel(const uint8_t *logits, int64_t tokens, int groups, int64_t ld, int top_k, const ID *experts, int64_t part,
                                                                 float *part_sums, int32_t *part_counts, float *losses, int32_t *counts, float *probs)
{
    using namespace route;
    constexpr int NT = BALANCE_NT, ROWS = NT / G, WAVES = NT / 64;
    extern __shared__ float lds[];  // [WAVES][8 G + 1] sums, [groups + 1] counts
    constexpr int PITCH = 8 * G + 1;
    float *const sums = lds;
    int *const hist = reinterpret_cast<int *>(lds + WAVES * PITCH);
    __shared__ float per_wave[WAVES];
    const int tid = threadIdx.x, g = tid & (G - 1), wave = tid >> 6, lane = tid & 63;
    for (int e = tid; e <= groups; e += NT) hist[e] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * part, last = first + part < tokens ? first + part : tokens;
    for (int64_t i = first * top_k + tid; i < last * top_k; i += NT) {
        const ID e = experts[i];
        if (e >= 0 && e < (ID)groups) atomicAdd(&hist[(int)e], 1);
    }
    // sums of 64 rows, of 64 of these, of those: a chain of thousands of additions in a long batch would lose ten bits
    float sum[V + 1], some[V + 1], most[V + 1];  // (lse^2 behind the probabilities)
#pragma unroll
    for (int i = 0; i <= V; ++i) sum[i] = some[i] = most[i] = 0.0f;
    int kept = 0;
    unsigned step = 0;
    for (int64_t t = first + tid / G; t < last; t += ROWS) {
        float v[V], lse;
        load_row<DT, G>(v, logits, ld, t, groups, true);
        kept += softmax<G>(v, &lse);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += v[i];
        sum[V] += lse * lse;
        if ((++step & 63) == 0) {
#pragma unroll
            for (int i = 0; i <= V; ++i) {
                some[i] += sum[i];
                sum[i] = 0.0f;
            }
            if ((step & 4095) == 0) {
#pragma unroll
                for (int i = 0; i <= V; ++i) {
                    most[i] += some[i];
                    some[i] = 0.0f;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i <= V; ++i) sum[i] += some[i] + most[i];
    float squares = sum[V];
    // the wave's rows, then the waves'
#pragma unroll
    for (int d = G; d < 64; d <<= 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += __shfl_xor(sum[i], d);
        squares += __shfl_xor(squares, d);
        kept += __shfl_xor(kept, d);
    }
    if (lane < G) {
#pragma unroll
        for (int i = 0; i < V; ++i) sums[wave * PITCH + g * V + i] = sum[i];
    }
    if (lane == 0) {
        sums[wave * PITCH + 8 * G] = squares;
        atomicAdd(&hist[groups], kept);
    }
    __syncthreads();
    for (int e = tid; e <= groups; e += NT) {
        float s = 0.0f;
        const int from = e < groups ? e : 8 * G;
        for (int w = 0; w < WAVES; ++w) s += sums[w * PITCH + from];
        if (part_sums) {
            part_sums[(int64_t)blockIdx.x * (groups + 1) + e] = s;
            part_counts[(int64_t)blockIdx.x * (groups + 1) + e] = hist[e];
        } else {
            sums[from] = s;  // (of wave 0, which this thread alone has read)
        }
    }
    if (part_sums) return;
    __syncthreads();
    if (tid == 0) sums[groups] = sums[8 * G];
    __syncthreads();
    balance_end(sums, hist, groups, top_k, NT, per_wave, losses, counts, probs);
}

__global__ __launch_bounds__(1024) void moe_balance_end_kernel(const float *part_sums, const int32_t *part_counts, int parts, int groups, int top_k, float *losses,
                                                               int32_t *counts, float *probs)
{
    using namespace route;
    extern __shared__ float lds[];  // [slices][groups + 1] sums, counts
    __shared__ float per_wave[16];
    const int cells = groups + 1, tid = threadIdx.x;
    const int slices = 1024 / cells, slice = tid / cells, e = tid - slice * cells;
    float *const sums = lds;
    int *const hist = reinterpret_cast<int *>(lds + slices * cells);
    if (slice < slices) {
        float s = 0.0f;
        int c = 0;
        for (int p0 = slice; p0 < parts; p0 += 16 * slices) {  // (loads of sixteen parts at a time: one after the other took 25 us of 38)
            float v[16];
            int n[16];
#pragma unroll
            for (int u = 0; u < 16; ++u) {
                const int64_t at = (int64_t)(p0 + u * slices < parts ? p0 + u * slices : slice) * cells + e;
                v[u] = part_sums[at];
                n[u] = part_counts[at];
            }
#pragma unroll
            for (int u = 0; u < 16; ++u)
                if (p0 + u * slices < parts) {
                    s += v[u];
                    c += n[u];
                }
        }
        sums[tid] = s;
        hist[tid] = c;
    }
    __syncthreads();
    if (tid < cells) {
        float s = sums[tid];
        int c = hist[tid];
        for (int k = 1; k < slices; ++k) {
            s += sums[k * cells + tid];
            c += hist[k * cells + tid];
        }
        sums[tid] = s;
        hist[tid] = c;
    }
    __syncthreads();
    balance_end(sums, hist, groups, top_k, 1024, per_wave, losses, counts, probs);
}

// f(lanes of a row) as a constant
template <class F>
static void with_row_lanes(int groups, F &&f)
{
    if (groups <= 8) f(std::integral_constant<int, 1>{});
    else if (groups <= 16) f(std::integral_constant<int, 2>{});
    else if (groups <= 32) f(std::integral_constant<int, 4>{});
    else if (groups <= 64) f(std::integral_constant<int, 8>{});
    else if (groups <= 128) f(std::integral_constant<int, 16>{});
    else if (groups <= 256) f(std::integral_constant<int, 32>{});
    else f(std::integral_constant<int, 64>{});
}

template <int DT>
static hipError_t forward(const RouteArgs &P, int32_t *experts, float *weights, hipStream_t st)
{
    with_row_lanes(P.groups, [&](auto g) {
        constexpr int G = decltype(g)::value, ROWS = 256 / G;
        moe_route_kernel<DT, G><<<launch_grid((P.tokens + ROWS - 1) / ROWS), 256, (size_t)ROWS * P.top_k * 4, st>>>(
            reinterpret_cast<const uint8_t *>(P.logits), P.tokens, P.groups, P.ld, P.top_k, P.renormalize, experts, weights);
    });
    return hipGetLastError();
}

template <int DT>
static hipError_t backward(const RouteArgs &P, const int32_t *experts, const float *dweights, const int32_t *counts, const float *dlosses, void *dlogits, hipStream_t st)
{
    with_row_lanes(P.groups, [&](auto g) {
        constexpr int G = decltype(g)::value, ROWS = 256 / G;
        moe_route_bwd_kernel<DT, G><<<launch_grid((P.tokens + ROWS - 1) / ROWS), 256, 0, st>>>(
            reinterpret_cast<const uint8_t *>(P.logits), P.tokens, P.groups, P.ld, P.top_k, P.renormalize, experts, dweights, counts, dlosses, reinterpret_cast<uint8_t *>(dlogits));
    });
    return hipGetLastError();
}

hipError_t launch_moe_route(const RouteArgs &P, int dt, int32_t *experts, float *weights, hipStream_t st)
{
    return dt == NVFP4_BF16 ? forward<NVFP4_BF16>(P, experts, weights, st) : forward<NVFP4_F32>(P, experts, weights, st);
}

hipError_t launch_moe_route_bwd(const RouteArgs &P, int dt, const int32_t *experts, const float *dweights, const int32_t *counts, const float *dlosses, void *dlogits,
                                hipStream_t st)
{
    return dt == NVFP4_BF16 ? backward<NVFP4_BF16>(P, experts, dweights, counts, dlosses, dlogits, st) : backward<NVFP4_F32>(P, experts, dweights, counts, dlosses, dlogits, st);
}

namespace route {
constexpr int64_t MOST_PARTS = 256;
constexpr int64_t LEAST_STEPS = 4;  // rows of a group of lanes before more workgroups are worth the second launch
inline int row_lanes(int groups)
{
    int g = 1;
    while (8 * g < groups) g *= 2;
    return g;
}
// Tokens of a workgroup
inline int64_t part_of(int64_t tokens, int groups)
{
    const int64_t rows = BALANCE_NT / row_lanes(groups);
    if (tokens <= LEAST_STEPS * rows) return tokens > 0 ? tokens : 1;
    const int64_t part = (tokens + MOST_PARTS - 1) / MOST_PARTS;
    return part <= rows ? rows : (part + rows - 1) / rows * rows;
}
}  // namespace route

size_t moe_balance_workspace(int64_t tokens, int32_t groups)
{
    const int64_t part = route::part_of(tokens, groups), parts = (tokens + part - 1) / part;
    return parts > 1 ? (size_t)parts * (groups + 1) * 8 : 0;
}

template <int DT, typename ID>
static hipError_t balance(const RouteArgs &P, const ID *experts, float *losses, int32_t *counts, float *probs, void *workspace, hipStream_t st)
{
    const int64_t part = route::part_of(P.tokens, P.groups), parts = P.tokens > 0 ? (P.tokens + part - 1) / part : 1;
    const int cells = P.groups + 1;
    float *const sums = parts > 1 ? reinterpret_cast<float *>(workspace) : nullptr;
    int32_t *const hist = parts > 1 ? reinterpret_cast<int32_t *>(sums + parts * cells) : nullptr;
    with_row_lanes(P.groups, [&](auto g) {
        constexpr int G = decltype(g)::value;
        moe_balance_kernel<DT, G, ID><<<dim3((unsigned)parts), BALANCE_NT, (BALANCE_NT / 64 * (8 * G + 1) + cells) * 4, st>>>(
            reinterpret_cast<const uint8_t *>(P.logits), P.tokens, P.groups, P.ld, P.top_k, experts, part, sums, hist, losses, counts, probs);
    });
    if (parts > 1)
        moe_balance_end_kernel<<<1, 1024, 1024 / cells * cells * 8, st>>>(sums, hist, (int)parts, P.groups, P.top_k, losses, counts, probs);
    return hipGetLastError();
}

hipError_t launch_moe_balance(const RouteArgs &P, int dt, const void *experts, int id_bytes, float *losses, int32_t *counts, float *probs, void *workspace, hipStream_t st)
{
    if (dt == NVFP4_BF16)
        return id_bytes == 8 ? balance<NVFP4_BF16>(P, reinterpret_cast<const int64_t *>(experts), losses, counts, probs, workspace, st)
                             : balance<NVFP4_BF16>(P, reinterpret_cast<const int32_t *>(experts), losses, counts, probs, workspace, st);
    return id_bytes == 8 ? balance<NVFP4_F32>(P, reinterpret_cast<const int64_t *>(experts), losses, counts, probs, workspace, st)
                         : balance<NVFP4_F32>(P, reinterpret_cast<const int32_t *>(experts), losses, counts, probs, workspace, st);
}

}  // namespace nvfp4
