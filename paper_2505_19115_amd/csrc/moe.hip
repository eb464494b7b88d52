// Routing of tokens to experts: (token, choice) pairs sorted by expert, rows moved between the tokens' order and the experts', and the gradients
// of that.  pair = token * top_k + choice.
//   sort          a stable counting sort: every pair's slot is the number of pairs of smaller experts plus that of earlier pairs of its own.
//                 No atomic decides an order, so the answer is the same from call to call.
//   gather        out[slot] = x[order[slot] / top_k]
//   combine       out[t] = sum_j w[t, j] y[position[t, j]], choices in their order, binary32
//   combine_bwd   dy[position[t, j]] = w[t, j] dout[t],  dw[t, j] = sum_d dout[t, d] y[position[t, j], d]
// What bounds rows is memory, at what a copy reaches (5.3 TB/s): a wave moves a row (of a pair, or of a token with its choices) in pieces of 16 bytes a lane.
// 8192 tokens x 2 of 4096 bf16, combined 38 to 41 us (4.9 to 5.3 TB/s), binary32 rows into bf16 70 (4.8), gradient 52 to 64 (5.2 to 6.4, by what the last cache level still
// holds); 1777 x 4 of 1027 binary32 gathered 9.7 (3.8 TB/s: rows that share lines; 10.8 from memory).  The sort is bound by latency: 32 pairs of 8 experts 3.3 us in one workgroup, 262144 of 128 experts 3.2 + 9.3
// in 64 of them (128 and 256 the same), where its 4 MB take 0.8.
#include <type_traits>

#include "experts.h"

namespace nvfp4 {
namespace moe {

constexpr int WAVES = 16, NT = 64 * WAVES;
constexpr int AHEAD = 4;  // loads of pairs' experts in flight: one after the other, four of them took half of the time

// Exclusive prefix sum of one value per thread over the workgroup; *total receives the sum
__device__ __forceinline__ int prefix(int v, int *per_wave, int *total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int up = __shfl_up(s, d);
        if (lane >= d) s += up;
    }
    if (lane == 63) per_wave[wave] = s;
    __syncthreads();
    int before = 0, sum = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int n = per_wave[w];
        if (w < wave) before += n;
        sum += n;
    }
    __syncthreads();
    *total = sum;
    return before + s - v;
}

template <typename ID>
__device__ __forceinline__ int expert_of(const ID *ids, int64_t i, int64_t n, int groups)
{
    if (i >= n) return -1;
    const ID e = ids[i];
    return e >= 0 && e < (ID)groups ? (int)e : -1;
}

}  // namespace moe

// Pairs of each expert in each workgroup's part of them: counts [workgroups, groups]
template <typename ID>
__global__ __launch_bounds__(1024) void moe_count_kernel(const ID *ids, int64_t n, int groups, int64_t part, int32_t *counts)
{
    using namespace moe;
    extern __shared__ int hist[];
    for (int e = threadIdx.x; e < groups; e += NT) hist[e] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * part, last = first + part < n ? first + part : n;
    for (int64_t i = first + threadIdx.x; i < last; i += AHEAD * NT) {
        int e[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) e[u] = expert_of(ids, i + u * NT, last, groups);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (e[u] >= 0) atomicAdd(&hist[e[u]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < groups; e += NT) counts[(int64_t)blockIdx.x * groups + e] = hist[e];
}

// A workgroup places its part of the pairs.  Its waves take consecutive pieces of the part; a wave places 64 pairs at a time, a lane's rank
// among those of its expert from one ballot per bit of the expert's number.  counts: of all parts, null for one part.
template <typename ID>
__global__ __launch_bounds__(1024) void moe_place_kernel(const ID *ids, int64_t n, int groups, int64_t part, const int32_t *counts, int32_t *offsets,
                                                         int32_t *order, int32_t *position)
{
    using namespace moe;
    extern __shared__ int hist[];  // [WAVES][groups], first counts and then the next free slot; sums over the parts
    __shared__ int per_wave[WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = blockIdx.x * part, last = first + part < n ? first + part : n;
    const int64_t piece = (part / WAVES + 63) / 64 * 64, w0 = first + wave * piece, w1 = w0 + piece < last ? w0 + piece : last;
    int *const mine = hist + wave * groups;
    for (int i = tid; i < WAVES * groups; i += NT) hist[i] = 0;
    __syncthreads();
    int own[AHEAD];  // the wave's first 64 AHEAD pairs, which are placed from here
    for (int64_t i0 = w0; i0 < w1; i0 += 64 * AHEAD) {
        int e[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            e[u] = expert_of(ids, i0 + u * 64 + lane, w1, groups);
            if (i0 == w0) own[u] = e[u];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (e[u] >= 0) atomicAdd(&mine[e[u]], 1);
    }
    __syncthreads();
    // thread e: the expert's pairs of all parts, of the parts before this one, of the waves before each (groups <= NT).  The counts of many parts are
    // added by all threads, eight loads at a time: one thread an expert, one load after the other, took 15 us of 20 at 64 parts.
    int all = 0, before = 0;
    if (counts) {
        int *const sum = hist + WAVES * groups;  // [2][groups]
        for (int i = tid; i < 2 * groups; i += NT) sum[i] = 0;
        __syncthreads();
        const int cells = (int)gridDim.x * groups, own = (int)blockIdx.x * groups, per = NT / groups * groups;  // (thread's expert: the same in each step)
        if (tid < per) {
            for (int i = tid; i < cells; i += 8 * per) {
                int k[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) k[u] = i + u * per < cells ? counts[i + u * per] : 0;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    all += k[u];
                    before += i + u * per < own ? k[u] : 0;
                }
            }
            const int e = tid % groups;
            atomicAdd(&sum[e], all);
            atomicAdd(&sum[groups + e], before);
        }
        __syncthreads();
        all = tid < groups ? sum[tid] : 0;
        before = tid < groups ? sum[groups + tid] : 0;
    } else if (tid < groups) {
        for (int w = 0; w < WAVES; ++w) all += hist[w * groups + tid];
    }
    int total;
    const int start = prefix(all, per_wave, &total);
    if (tid < groups) {
        int at = start + before;
        for (int w = 0; w < WAVES; ++w) {
            const int k = hist[w * groups + tid];
            hist[w * groups + tid] = at;
            at += k;
        }
        if (blockIdx.x == 0) offsets[tid] = start;
    }
    if (blockIdx.x == 0 && tid == 0) offsets[groups] = total;
    __syncthreads();
    const int bits = 32 - __builtin_clz((unsigned)groups);
    for (int64_t i0 = w0; i0 < w1; i0 += 64 * AHEAD) {
        int expert[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) expert[u] = i0 == w0 ? own[u] : expert_of(ids, i0 + u * 64 + lane, w1, groups);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t i = i0 + u * 64 + lane;
            if (i0 + u * 64 >= w1) break;
            const int e = expert[u];
            uint64_t same = __ballot(e >= 0);
            for (int b = 0; b < bits; ++b) {
                const uint64_t ones = __ballot((e >> b) & 1);
                same &= (e >> b) & 1 ? ones : ~ones;
            }
            if (e >= 0) {
                const int rank = __popcll(same & ((1ull << lane) - 1));
                const int slot = *const_cast<volatile int *>(&mine[e]) + rank;
                if (rank == 0) atomicAdd(&mine[e], __popcll(same));  // (behind the wave's reads: LDS accesses of a wave keep their order)
                order[slot] = (int32_t)i;
                position[i] = slot;
            } else if (i < w1) {
                position[i] = -1;
            }
        }
    }
    for (int64_t i = first + tid; i < last; i += NT)
        if (i >= total) order[i] = -1;
}

namespace moe {
constexpr int64_t PART = 4096;       // pairs of a workgroup
constexpr int64_t MOST_PARTS = 256;  // (every workgroup reads the counts of all)
inline int64_t part_of(int64_t n)
{
    int64_t part = n <= 2 * PART ? (n > 0 ? n : 1) : PART;
    if ((n + part - 1) / part > MOST_PARTS) part = (n + MOST_PARTS - 1) / MOST_PARTS;
    return (part + NT - 1) / NT * NT;
}
}  // namespace moe

size_t moe_sort_workspace(int64_t pairs, int32_t groups)
{
    const int64_t part = moe::part_of(pairs), parts = (pairs + part - 1) / part;
    return parts > 1 ? (size_t)parts * groups * 4 : 0;
}

template <typename ID>
static hipError_t sort(const ID *ids, int64_t n, int32_t groups, int32_t *offsets, int32_t *order, int32_t *position, int32_t *counts, hipStream_t st)
{
    using namespace moe;
    const int64_t part = part_of(n), parts = n > 0 ? (n + part - 1) / part : 1;
    if (parts > 1) moe_count_kernel<ID><<<dim3((unsigned)parts), NT, groups * 4, st>>>(ids, n, groups, part, counts);
    moe_place_kernel<ID><<<dim3((unsigned)parts), NT, (WAVES + 2) * groups * 4, st>>>(ids, n, groups, part, parts > 1 ? counts : nullptr, offsets, order, position);
    return hipGetLastError();
}

hipError_t launch_moe_sort(const void *experts, int id_bytes, int64_t pairs, int32_t groups, int32_t *offsets, int32_t *order, int32_t *position,
                           int32_t *workspace, hipStream_t st)
{
    return id_bytes == 8 ? sort(reinterpret_cast<const int64_t *>(experts), pairs, groups, offsets, order, position, workspace, st)
                         : sort(reinterpret_cast<const int32_t *>(experts), pairs, groups, offsets, order, position, workspace, st);
}

namespace moe {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float float2v_t __attribute__((ext_vector_type(2)));

// Elements that fill 16 bytes of a row of a type; beside a narrower one, as many as it has
constexpr int per_piece(int dt) { return dt == NVFP4_BF16 ? 8 : 4; }

// N neighbouring elements of a row, from any element on
template <int DT, int N = per_piece(DT)>
struct Piece {
    static constexpr int ESZ = DT == NVFP4_BF16 ? 2 : 4, W = N * ESZ / 16;
    struct __attribute__((packed, aligned(ESZ))) P { u32x4_t w; };
    u32x4_t w[W];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int k = 0; k < W; ++k) w[k] = u32x4_t{0, 0, 0, 0};
    }
    template <bool STREAMED>
    __device__ __forceinline__ void load(const uint8_t *p)
    {
#pragma unroll
        for (int k = 0; k < W; ++k) w[k] = STREAMED ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p) + k) : reinterpret_cast<const P *>(p)[k].w;
    }
    __device__ __forceinline__ void store(uint8_t *p) const
    {
#pragma unroll
        for (int k = 0; k < W; ++k) reinterpret_cast<P *>(p)[k].w = w[k];
    }
    __device__ __forceinline__ void load_some(const uint8_t *p, int n)
    {
        zero();
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) {
                if (DT == NVFP4_BF16) w[0][(i >> 1) & 3] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
                else w[(i >> 2) % W][i & 3] = reinterpret_cast<const uint32_t *>(p)[i];
            }
    }
    __device__ __forceinline__ void store_some(uint8_t *p, int n) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) {
                if (DT == NVFP4_BF16) reinterpret_cast<uint16_t *>(p)[i] = (uint16_t)(w[0][(i >> 1) & 3] >> (16 * (i & 1)));
                else reinterpret_cast<uint32_t *>(p)[i] = w[(i >> 2) % W][i & 3];
            }
    }
    __device__ __forceinline__ float get(int i) const
    {
        return DT == NVFP4_BF16 ? __uint_as_float(i & 1 ? w[0][(i >> 1) & 3] & 0xFFFF0000u : w[0][(i >> 1) & 3] << 16) : __uint_as_float(w[(i >> 2) % W][i & 3]);
    }
    __device__ __forceinline__ void set(const float (&v)[N])
    {
        if (DT == NVFP4_BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2v_t f = {v[(2 * i) % N], v[(2 * i + 1) % N]};
                w[0][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[(i >> 2) % W][i & 3] = __float_as_uint(v[i]);
        }
    }
};

// Which row (of the launch's) a lane works on, G lanes side by side on one: the same in the wave where that is one row.
template <int G>
__device__ __forceinline__ int64_t row_of()
{
    const int64_t wave = (int64_t)workgroup() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    return G == 64 ? wave : wave * (64 / G) + (threadIdx.x & 63) / G;
}

// Walks a row in steps of U pieces of N elements a lane: body(at, n, again, whole) with the first elements of a lane's pieces, how many each has there (0: none), how many of
// them the piece before has too (a row's last piece ends with the row), and whether all pieces are there and none overlaps, which is the same in the wave.
template <int N, int U, int G, class F>
__device__ __forceinline__ void walk(int64_t cols, F &&body)
{
    const int lane = threadIdx.x & (G - 1);
    for (int64_t c0 = 0; c0 < cols; c0 += G * N * U) {
        int64_t at[U];
        int n[U], again[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + (u * G + lane) * N;
            const int left = cols - c < N ? (int)(cols - c) : N;
            again[u] = left > 0 && cols >= N ? N - left : 0;
            at[u] = c - again[u];
            n[u] = left > 0 ? left + again[u] : 0;
        }
        if (c0 + G * N * U <= cols) body(at, n, again, std::true_type{});
        else body(at, n, again, std::false_type{});
    }
}
template <bool WHOLE, bool STREAMED, int DT, int N, int U>
__device__ __forceinline__ void load(Piece<DT, N> (&v)[U], const uint8_t *row, const int64_t (&at)[U], const int (&n)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint8_t *const p = row + at[u] * Piece<DT, N>::ESZ;
        if (WHOLE || n[u] == N) v[u].template load<STREAMED>(p);
        else if (n[u] > 0) v[u].load_some(p, n[u]);
        else v[u].zero();
    }
}
template <bool WHOLE, int DT, int N, int U>
__device__ __forceinline__ void store(const Piece<DT, N> (&v)[U], uint8_t *row, const int64_t (&at)[U], const int (&n)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        uint8_t *const p = row + at[u] * Piece<DT, N>::ESZ;
        if (WHOLE || n[u] == N) v[u].store(p);
        else if (n[u] > 0) v[u].store_some(p, n[u]);
    }
}

}  // namespace moe

template <int DT, bool STREAMED, int G>
__global__ __launch_bounds__(256) void moe_gather_kernel(const uint8_t *x, int64_t x_rows, int64_t cols, int64_t ld, const int32_t *order, int32_t top_k,
                                                         int64_t rows, uint8_t *out)
{
    using namespace moe;
    constexpr int U = 2;
    const int64_t r = row_of<G>();
    if (r >= rows) return;
    const int32_t pair = order[r];
    const int64_t src = pair < 0 || pair / top_k >= x_rows ? -1 : pair / top_k;
    const uint8_t *const from = x + src * ld * Piece<DT>::ESZ;
    uint8_t *const to = out + r * cols * Piece<DT>::ESZ;
    walk<per_piece(DT), U, G>(cols, [&](const int64_t (&at)[U], const int (&n)[U], const int (&again)[U], auto whole) {
        constexpr bool W = decltype(whole)::value;
        Piece<DT> v[U];
        if (src >= 0) {
            load<W, STREAMED>(v, from, at, n);
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].zero();
        }
        store<W>(v, to, at, n);
    });
}

// G lanes for each token.  Two choices at a time: as many loads in flight.  DT: of y; OUT: of the result.
template <int DT, int OUT, bool STREAMED, int G>
__global__ __launch_bounds__(256) void moe_combine_kernel(const uint8_t *y, int64_t y_rows, int64_t cols, const float *weights, const int32_t *position,
                                                          int64_t tokens, int32_t top_k, uint8_t *out)
{
    using namespace moe;
    constexpr int U = 2, N = per_piece(DT) > per_piece(OUT) ? per_piece(DT) : per_piece(OUT);
    const int64_t t = row_of<G>(), row = cols * Piece<DT>::ESZ;
    if (t >= tokens) return;
    const int32_t *const places = position + t * top_k;
    walk<N, U, G>(cols, [&](const int64_t (&at)[U], const int (&n)[U], const int (&again)[U], auto whole) {
        constexpr bool W = decltype(whole)::value;
        float sum[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) sum[u][i] = 0.0f;
        auto add = [&](const Piece<DT, N> (&v)[U], float w) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[u][i] = __builtin_fmaf(w, v[u].get(i), sum[u][i]);
        };
        for (int j = 0; j < top_k; j += 2) {
            const int32_t p = places[j], q = j + 1 < top_k ? places[j + 1] : -1;
            const bool has_p = p >= 0 && p < y_rows, has_q = q >= 0 && q < y_rows;
            Piece<DT, N> a[U], b[U];
            if (has_p) load<W, STREAMED>(a, y + p * row, at, n);
            if (has_q) load<W, STREAMED>(b, y + q * row, at, n);
            if (has_p) add(a, weights ? weights[t * top_k + j] : 1.0f);
            if (has_q) add(b, weights ? weights[t * top_k + j + 1] : 1.0f);
        }
        Piece<OUT, N> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].set(sum[u]);
        store<W>(v, out + t * cols * Piece<OUT>::ESZ, at, n);
    });
}

// G lanes for each pair; behind them those that clear the rows of dy past the last kept pair.  DT: of y and dy; UP: of dout.
template <int DT, int UP, bool STREAMED, int G>
__global__ __launch_bounds__(256) void moe_combine_bwd_kernel(const uint8_t *dout, const uint8_t *y, int64_t rows, int64_t cols, const float *weights,
                                                              const int32_t *position, const int32_t *kept, int64_t pairs, int32_t top_k, uint8_t *dy,
                                                              float *dweights)
{
    using namespace moe;
    constexpr int U = 2, N = per_piece(DT) > per_piece(UP) ? per_piece(DT) : per_piece(UP);
    const int lane = threadIdx.x & (G - 1);
    const int64_t id = row_of<G>(), row = cols * Piece<DT>::ESZ;
    if (id >= pairs) {
        const int64_t clearing = (int64_t)gridDim.x * gridDim.y * (256 / G) - pairs;
        for (int64_t r = (kept[0] < 0 ? 0 : kept[0]) + (id - pairs); r < rows; r += clearing)
            walk<N, U, G>(cols, [&](const int64_t (&at)[U], const int (&n)[U], const int (&again)[U], auto whole) {
                Piece<DT, N> v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u].zero();
                store<decltype(whole)::value>(v, dy + r * row, at, n);
            });
        return;
    }
    const int32_t p = position[id];
    if (p < 0 || p >= rows) {
        if (lane == 0) dweights[id] = 0.0f;
        return;
    }
    const uint8_t *const up = dout + id / top_k * cols * Piece<UP>::ESZ, *const from = y + p * row;
    uint8_t *const to = dy + p * row;
    const float w = weights[id];
    float dot = 0.0f;
    walk<N, U, G>(cols, [&](const int64_t (&at)[U], const int (&n)[U], const int (&again)[U], auto whole) {
        constexpr bool W = decltype(whole)::value;
        Piece<UP, N> a[U];
        Piece<DT, N> b[U];
        load<W, false>(a, up, at, n);
        load<W, STREAMED>(b, from, at, n);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = w * a[u].get(i);
                if (W || i >= again[u]) dot = __builtin_fmaf(a[u].get(i), b[u].get(i), dot);
            }
            b[u].set(v);
        }
        store<W>(b, to, at, n);
    });
#pragma unroll
    for (int d = G / 2; d > 0; d >>= 1) dot += __shfl_xor(dot, d);
    if (lane == 0) dweights[id] = dot;
}

// Whether rows that are read once come by streaming loads: where they are much of what the last cache level keeps, in whole cache lines.  us, plain / streaming:
// 16384 binary32 rows of 4096 gathered 108 / 82, combined 124 / 89; 16384 bf16 rows of 4096, two a token, combined 48 / 42, gradient 69 / 56; 8192 of these, four a
// token, 20 / 22 and 27 / 27; 7108 binary32 rows of 1027, which share lines, combined 12.5 / 17.5.
constexpr int64_t STREAM_MB = 96;
static bool streams(const void *rows, int64_t n, int64_t cols, int dt)
{
    const int64_t row = cols * (dt == NVFP4_BF16 ? 2 : 4);
    return row % 128 == 0 && reinterpret_cast<uintptr_t>(rows) % 128 == 0 && n * row >= ((int64_t)STREAM_MB << 20);
}

// Lanes of a row, which has two pieces for each at a time: short rows by a wave each are bound by how fast waves begin.  us, 64 lanes / so, 10010 tokens x 6 gathered, combined,
// gradient: 64 bf16 20.4 / 7.0, 14.2 / 7.0, 28.6 / 9.5; 256 20.6 / 10.2, 15.0 / 8.3, 28.7 / 12.4; 512 20.0 / 18.4, 16.0 / 12.5, 31.2 / 25.0.
static int lanes_of(int64_t cols, int per_piece)
{
    const int64_t pieces = (cols + per_piece - 1) / per_piece;
    return pieces <= 16 ? 8 : pieces <= 32 ? 16 : pieces <= 64 ? 32 : 64;
}
// (rows of a wave's groups of lanes)
static dim3 grid_of(int64_t rows, int lanes) { return launch_grid((rows + 256 / lanes - 1) / (256 / lanes)); }

// f(streamed, lanes) of a kernel's template, as constants
template <class F>
static void with_lanes(bool s, int lanes, F &&f)
{
    if (lanes == 8) f(std::false_type{}, std::integral_constant<int, 8>{});
    else if (lanes == 16) f(std::false_type{}, std::integral_constant<int, 16>{});
    else if (lanes == 32) f(std::false_type{}, std::integral_constant<int, 32>{});
    else if (s) f(std::true_type{}, std::integral_constant<int, 64>{});
    else f(std::false_type{}, std::integral_constant<int, 64>{});
}

template <int DT>
static hipError_t gather(const void *x, int64_t x_rows, int64_t cols, int64_t ld, const int32_t *order, int32_t top_k, int64_t rows, void *out, hipStream_t st)
{
    const int lanes = lanes_of(cols, moe::per_piece(DT));
    with_lanes(top_k == 1 && ld == cols && streams(x, x_rows, cols, DT), lanes, [&](auto s, auto g) {
        moe_gather_kernel<DT, decltype(s)::value, decltype(g)::value><<<grid_of(rows, lanes), 256, 0, st>>>(reinterpret_cast<const uint8_t *>(x), x_rows, cols, ld, order, top_k, rows,
                                                                                                            reinterpret_cast<uint8_t *>(out));
    });
    return hipGetLastError();
}

template <int DT, int OUT>
static hipError_t combine(const void *y, int64_t y_rows, int64_t cols, const float *weights, const int32_t *position, int64_t tokens, int32_t top_k, void *out, hipStream_t st)
{
    const int lanes = lanes_of(cols, DT == NVFP4_BF16 || OUT == NVFP4_BF16 ? 8 : 4);
    with_lanes(streams(y, y_rows, cols, DT), lanes, [&](auto s, auto g) {
        moe_combine_kernel<DT, OUT, decltype(s)::value, decltype(g)::value><<<grid_of(tokens, lanes), 256, 0, st>>>(reinterpret_cast<const uint8_t *>(y), y_rows, cols, weights, position,
                                                                                                                    tokens, top_k, reinterpret_cast<uint8_t *>(out));
    });
    return hipGetLastError();
}

template <int DT, int UP>
static hipError_t combine_bwd(const void *dout, const void *y, int64_t rows, int64_t cols, const float *weights, const int32_t *position, const int32_t *kept, int64_t tokens,
                              int32_t top_k, void *dy, float *dweights, hipStream_t st)
{
    const int64_t pairs = tokens * top_k, clearing = rows < 256 ? rows : 256;
    const int lanes = lanes_of(cols, DT == NVFP4_BF16 || UP == NVFP4_BF16 ? 8 : 4);
    with_lanes(streams(y, rows, cols, DT), lanes, [&](auto s, auto g) {
        moe_combine_bwd_kernel<DT, UP, decltype(s)::value, decltype(g)::value><<<grid_of(pairs + clearing, lanes), 256, 0, st>>>(
            reinterpret_cast<const uint8_t *>(dout), reinterpret_cast<const uint8_t *>(y), rows, cols, weights, position, kept, pairs, top_k, reinterpret_cast<uint8_t *>(dy), dweights);
    });
    return hipGetLastError();
}

hipError_t launch_moe_gather(const void *x, int dt, int64_t x_rows, int64_t cols, int64_t ld, const int32_t *order, int32_t top_k, int64_t rows, void *out,
                             hipStream_t st)
{
    return dt == NVFP4_BF16 ? gather<NVFP4_BF16>(x, x_rows, cols, ld, order, top_k, rows, out, st) : gather<NVFP4_F32>(x, x_rows, cols, ld, order, top_k, rows, out, st);
}

hipError_t launch_moe_combine(const void *y, int dt, int64_t y_rows, int64_t cols, const float *weights, const int32_t *position, int64_t tokens,
                              int32_t top_k, void *out, int out_dt, hipStream_t st)
{
    auto *f = dt == NVFP4_BF16 ? (out_dt == NVFP4_BF16 ? combine<NVFP4_BF16, NVFP4_BF16> : combine<NVFP4_BF16, NVFP4_F32>)
                               : (out_dt == NVFP4_BF16 ? combine<NVFP4_F32, NVFP4_BF16> : combine<NVFP4_F32, NVFP4_F32>);
    return f(y, y_rows, cols, weights, position, tokens, top_k, out, st);
}

hipError_t launch_moe_combine_bwd(const void *dout, int dout_dt, const void *y, int dt, int64_t rows, int64_t cols, const float *weights, const int32_t *position,
                                  const int32_t *kept, int64_t tokens, int32_t top_k, void *dy, float *dweights, hipStream_t st)
{
    auto *f = dt == NVFP4_BF16 ? (dout_dt == NVFP4_BF16 ? combine_bwd<NVFP4_BF16, NVFP4_BF16> : combine_bwd<NVFP4_BF16, NVFP4_F32>)
                               : (dout_dt == NVFP4_BF16 ? combine_bwd<NVFP4_F32, NVFP4_BF16> : combine_bwd<NVFP4_F32, NVFP4_F32>);
    return f(dout, y, rows, cols, weights, position, kept, tokens, top_k, dy, dweights, st);
}

}  // namespace nvfp4
