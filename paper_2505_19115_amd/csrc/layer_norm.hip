// Rows normalised, and the gradients of that.
//   forward   m = mean x (or 0), r = 1 / sqrt(mean (x - m)^2 + eps), y = (x - m) r w + b
//   backward  h = (x - m) r, u = dy w:  dx = r (u - mean u - h mean(u h)) (mean u where m is taken off),  dw = sum over rows of dy h,  db = of dy
// What bounds both is memory.  T threads hold a row in registers, U pieces of 16 bytes each, so that x (and dy) are read once and deviations come
// from the mean, not from a difference of sums.  In the backward pass a thread keeps its columns from row to row: the weight stays in registers, the
// sums for dw and db too; they meet in the LDS at the end, each workgroup leaves one row of sums, and a second kernel adds these in order.
// us, kernels alone, rows from memory: forward 2049 x 2785 binary32 11.7 (3.9 TB/s; 9.9 where the last cache has them), 8192 x 4096 bf16 25.8 (5.2); backward 8192 x 4096 bf16 71 + 5 (2.9 TB/s,
// and 16 MB of sums written and read; 54 + 5 from the cache), 65536 rows of 96 bf16 21 + 4 (1.8 TB/s: half of the lanes' second pieces lie past the row's end).  What holds the bf16 gradient
// back: load_run() unpacks a piece in the branch that loads it, so that the compiler waits for each 16 bytes of x and dy before it asks for the next, four times a row; and 134 registers
// of 256 threads leave a CU one workgroup of eight waves.  (Of the binary32 forms the one of 1024 threads spills 3 registers of 128.)  Tried: the next row's loads before this row's work (8192 x 4096
// 56, 65536 x 96 30 from the cache), with loads that wait for one another all the same.
#include <type_traits>

#include "layer_ops.h"

namespace nvfp4 {
namespace norm {

using namespace layer;

constexpr int per_piece(int dt) { return dt == NVFP4_BF16 ? 8 : 4; }

// Sum over the T threads of a row, in all of them.  per_wave: LDS of T / 64 floats a row, free again behind the caller's next barrier
template <int T>
__device__ __forceinline__ float row_sum(float v, float *per_wave)
{
    if constexpr (T <= 64) {
        return group_sum<T>(v);
    } else {
        v = group_sum<64>(v);
        const int wave = (threadIdx.x & (T - 1)) >> 6;
        if ((threadIdx.x & 63) == 0) per_wave[wave] = v;
        __syncthreads();
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < T / 64; ++w) s += per_wave[w];
        return s;
    }
}

template <int N>
__device__ __forceinline__ void load_weight(float (&w)[N], const uint8_t *p, int wdt, int64_t c, int n, float fill)
{
    if (!p) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = fill;
    } else if (wdt == NVFP4_BF16) {
        if constexpr (N == 8) {
            load_run<NVFP4_BF16, N>(w, p + c * 2, n, 0.0f);
        } else {
            struct __attribute__((packed, aligned(2))) Q { uint32_t w[2]; };
            if (n >= N) {
                const Q q = *reinterpret_cast<const Q *>(p + c * 2);
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] = __uint_as_float(i & 1 ? q.w[(i >> 1) & 1] & 0xFFFF0000u : q.w[(i >> 1) & 1] << 16);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) w[i] = i < n ? Elem<NVFP4_BF16>::load(p + (c + i) * 2) : 0.0f;
            }
        }
    } else {
        load_run<NVFP4_F32, N>(w, p + c * 4, n, 0.0f);
    }
}

}  // namespace norm

// Rows of up to T * U pieces
template <int DT, int T, int U>
__global__ __launch_bounds__(T < 256 ? 256 : T) void layer_norm_kernel(const uint8_t *x, int64_t rows, int cols, int64_t ld, const uint8_t *weight, const uint8_t *bias, int wdt,
                                                                       int center, float eps, uint8_t *y, float *mean, float *rstd)
{
    using namespace norm;
    constexpr int NT = T < 256 ? 256 : T, N = per_piece(DT), ESZ = Elem<DT>::BYTES;
    __shared__ float per_wave[2][T > 64 ? T / 64 : 1];
    const int g = threadIdx.x & (T - 1);
    const int64_t r = (int64_t)workgroup() * (NT / T) + threadIdx.x / T;
    if (r >= rows) return;  // (whole waves' rows, or whole groups of lanes)
    float v[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) load_run<DT, N>(v[u], x + (r * ld + (u * T + g) * N) * ESZ, cols - (u * T + g) * N, 0.0f);
    float m = 0.0f;
    if (center) {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) s += v[u][i];
        m = row_sum<T>(s, per_wave[0]) / (float)cols;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) v[u][i] = (u * T + g) * N + i < cols ? v[u][i] - m : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < N; ++i) s = __builtin_fmaf(v[u][i], v[u][i], s);
    const float scale = 1.0f / __builtin_sqrtf(row_sum<T>(s, per_wave[1]) / (float)cols + eps);
    if (g == 0) {
        if (mean) mean[r] = m;
        if (rstd) rstd[r] = scale;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int c = (u * T + g) * N, n = cols - c;
        if (n <= 0) continue;
        float w[N], b[N];
        load_weight<N>(w, weight, wdt, c, n, 1.0f);
        load_weight<N>(b, bias, wdt, c, n, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) v[u][i] = __builtin_fmaf(v[u][i] * scale, w[i], b[i]);
        store_run<DT, N>(v[u], y + (r * cols + c) * ESZ, n);
    }
}

// Rows that no workgroup's registers hold: a workgroup for a row, read three times (the mean, the deviations, the results)
template <int DT>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(const uint8_t *x, int64_t rows, int64_t cols, int64_t ld, const uint8_t *weight, const uint8_t *bias, int wdt,
                                                               int center, float eps, uint8_t *y, float *mean, float *rstd)
{
    using namespace norm;
    constexpr int N = per_piece(DT), ESZ = Elem<DT>::BYTES, STEP = 1024 * N;
    __shared__ float per_wave[2][16];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const uint8_t *const row = x + r * ld * ESZ;
    const int64_t c0 = (int64_t)threadIdx.x * N;
    auto left = [&](int64_t c) { return (int)(cols - c < N ? cols - c : N); };
    float m = 0.0f, s = 0.0f, v[N];
    if (center) {
        for (int64_t c = c0; c < cols; c += STEP) {
            load_run<DT, N>(v, row + c * ESZ, left(c), 0.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) s += v[i];
        }
        m = row_sum<1024>(s, per_wave[0]) / (float)cols;
    }
    s = 0.0f;
    for (int64_t c = c0; c < cols; c += STEP) {
        load_run<DT, N>(v, row + c * ESZ, left(c), m);
#pragma unroll
        for (int i = 0; i < N; ++i) s = __builtin_fmaf(v[i] - m, v[i] - m, s);
    }
    const float scale = 1.0f / __builtin_sqrtf(row_sum<1024>(s, per_wave[1]) / (float)cols + eps);
    if (threadIdx.x == 0) {
        if (mean) mean[r] = m;
        if (rstd) rstd[r] = scale;
    }
    for (int64_t c = c0; c < cols; c += STEP) {
        float w[N], b[N];
        load_run<DT, N>(v, row + c * ESZ, left(c), 0.0f);
        load_weight<N>(w, weight, wdt, c, left(c), 1.0f);
        load_weight<N>(b, bias, wdt, c, left(c), 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __builtin_fmaf((v[i] - m) * scale, w[i], b[i]);
        store_run<DT, N>(v, y + (r * cols + c) * ESZ, left(c));
    }
}

// Rows of up to T * U pieces; a workgroup's teams of T threads take its rows in turn.  sums: [workgroups][dw, db] rows of `cols` floats, null: not wanted.
template <int DT, int T, int U, int NT>
__global__ __launch_bounds__(NT) void layer_norm_bwd_kernel(const uint8_t *dy, int64_t ldy, const uint8_t *x, int64_t rows, int cols, int64_t ld, const uint8_t *weight, int wdt,
                                                            const float *mean, const float *rstd, uint8_t *dx, float *sum_w, float *sum_b, int64_t pitch)
{
    using namespace norm;
    constexpr int N = per_piece(DT), ESZ = Elem<DT>::BYTES, TEAMS = NT / T;
    __shared__ float per_wave[2][TEAMS][T > 64 ? T / 64 : 1][2];
    extern __shared__ float lds[];  // [cols] sums
    const int g = threadIdx.x & (T - 1), team = threadIdx.x / T;
    float w[U][N], dw[U][N], db[U][N];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        load_weight<N>(w[u], weight, wdt, (u * T + g) * N, cols - (u * T + g) * N, 1.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) dw[u][i] = db[u][i] = 0.0f;
    }
    const int64_t step = (int64_t)gridDim.x * TEAMS;
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * TEAMS; r0 < rows; r0 += step, turn ^= 1) {
        const int64_t r = r0 + team;
        const bool there = r < rows;
        float h[U][N], d[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (u * T + g) * N, n = there ? cols - c : 0;
            load_run<DT, N>(h[u], x + (r * ld + c) * ESZ, n, 0.0f);
            load_run<DT, N>(d[u], dy + (r * ldy + c) * ESZ, n, 0.0f);
        }
        const float m = there && mean ? mean[r] : 0.0f, scale = there ? rstd[r] : 0.0f;
        float su = 0.0f, sh = 0.0f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bool in = (u * T + g) * N + i < cols;
                h[u][i] = in ? (h[u][i] - m) * scale : 0.0f;
                dw[u][i] = __builtin_fmaf(d[u][i], h[u][i], dw[u][i]);
                db[u][i] += d[u][i];
                const float p = d[u][i] * (in ? w[u][i] : 0.0f);
                d[u][i] = p;
                su += p;
                sh = __builtin_fmaf(p, h[u][i], sh);
            }
        if constexpr (T <= 64) {
            su = group_sum<T>(su);
            sh = group_sum<T>(sh);
        } else {  // (two places in turn: the next row's are written while some thread reads these)
            su = group_sum<64>(su);
            sh = group_sum<64>(sh);
            const int wave = g >> 6;
            if ((threadIdx.x & 63) == 0) {
                per_wave[turn][team][wave][0] = su;
                per_wave[turn][team][wave][1] = sh;
            }
            __syncthreads();
            su = sh = 0.0f;
#pragma unroll
            for (int k = 0; k < T / 64; ++k) {
                su += per_wave[turn][team][k][0];
                sh += per_wave[turn][team][k][1];
            }
        }
        su = mean ? su / (float)cols : 0.0f;
        sh /= (float)cols;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = (u * T + g) * N, n = there ? cols - c : 0;
            if (n <= 0) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) d[u][i] = scale * (d[u][i] - su - h[u][i] * sh);
            store_run<DT, N>(d[u], dx + (r * cols + c) * ESZ, n);
        }
    }
    // the teams' sums: those of a wave across its lanes, then wave after wave through the LDS
    auto leave = [&](float (&v)[U][N], float *out) {
        if constexpr (TEAMS == 1) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = (u * T + g) * N;
                store_run<NVFP4_F32, N>(v[u], reinterpret_cast<uint8_t *>(out + blockIdx.x * pitch + c), cols - c);
            }
            return;
        }
        if constexpr (T < 64) {
#pragma unroll
            for (int k = T; k < 64; k <<= 1)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < N; ++i) v[u][i] += __shfl_xor(v[u][i], k);
        }
        constexpr int ROUNDS = T < 64 ? NT / 64 : TEAMS;
        const int turn = T < 64 ? threadIdx.x >> 6 : team;
        for (int k = 0; k < ROUNDS; ++k) {
            if (turn == k && (T >= 64 || (threadIdx.x & 63) < T)) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const int c = (u * T + g) * N + i;
                        if (c < cols) lds[c] = k == 0 ? v[u][i] : lds[c] + v[u][i];
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += NT) out[blockIdx.x * pitch + c] = lds[c];
        __syncthreads();
    };
    if (sum_w) leave(dw, sum_w);
    if (sum_b) leave(db, sum_b);
}

// Rows that no workgroup's registers hold: dx by a workgroup a row, read twice; the columns' sums by another kernel
template <int DT>
__global__ __launch_bounds__(1024) void layer_norm_bwd_long_kernel(const uint8_t *dy, int64_t ldy, const uint8_t *x, int64_t rows, int64_t cols, int64_t ld, const uint8_t *weight,
                                                                   int wdt, const float *mean, const float *rstd, uint8_t *dx)
{
    using namespace norm;
    constexpr int N = per_piece(DT), ESZ = Elem<DT>::BYTES, STEP = 1024 * N;
    __shared__ float per_wave[2][16];
    const int64_t r = workgroup();
    if (r >= rows) return;
    const float m = mean ? mean[r] : 0.0f, scale = rstd[r];
    float su = 0.0f, sh = 0.0f;
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t c = (int64_t)threadIdx.x * N; c < cols; c += STEP) {
            const int n = (int)(cols - c < N ? cols - c : N);
            float h[N], d[N], w[N];
            load_run<DT, N>(h, x + (r * ld + c) * ESZ, n, m);
            load_run<DT, N>(d, dy + (r * ldy + c) * ESZ, n, 0.0f);
            load_weight<N>(w, weight, wdt, c, n, 1.0f);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                h[i] = (h[i] - m) * scale;
                d[i] *= w[i];
                if (pass == 0) {
                    su += d[i];
                    sh = __builtin_fmaf(d[i], h[i], sh);
                } else {
                    d[i] = scale * (d[i] - su - h[i] * sh);
                }
            }
            if (pass == 1) store_run<DT, N>(d, dx + (r * cols + c) * ESZ, n);
        }
        if (pass == 0) {
            su = row_sum<1024>(su, per_wave[0]);
            sh = row_sum<1024>(sh, per_wave[1]) / (float)cols;
            su = mean ? su / (float)cols : 0.0f;
        }
    }
}

namespace norm {

// A long sum: what the roundings of its additions leave is summed beside it, so that it is right to 2 u of the terms' sizes however many they are.  An infinite sum has no rest.
struct LongSum {
    float sum = 0.0f, rest = 0.0f;
    __device__ __forceinline__ void add(float v)
    {
        const float s = sum + v, b = s - sum;
        rest += (sum - (s - b)) + (v - b);
        sum = s;
    }
    __device__ __forceinline__ float value() const { return __builtin_isfinite(sum) ? sum + rest : sum; }
};

}  // namespace norm

// A thread adds rows / parts terms of its column, thousands in a long batch: one after the other in binary32 they were off by 270 u where all were alike (8192 x 65537, four parts).
// Four rows' loads at a time pay for the additions.  us, the call, 8192 x 65537 binary32: 3180 without, 2666; 8192 x 20000 bf16 690, 490
template <int DT>
__global__ __launch_bounds__(256) void layer_norm_columns_kernel(const uint8_t *dy, int64_t ldy, const uint8_t *x, int64_t rows, int64_t cols, int64_t ld, const float *mean,
                                                                 const float *rstd, int64_t part, float *sum_w, float *sum_b, int64_t pitch)
{
    using namespace norm;
    constexpr int ESZ = Elem<DT>::BYTES;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x, first = blockIdx.y * part, last = first + part < rows ? first + part : rows;
    if (c >= cols) return;
    LongSum dw, db;
#pragma unroll 4
    for (int64_t r = first; r < last; ++r) {
        const float d = Elem<DT>::load(dy + (r * ldy + c) * ESZ), h = (Elem<DT>::load(x + (r * ld + c) * ESZ) - (mean ? mean[r] : 0.0f)) * rstd[r];
        dw.add(d * h);
        db.add(d);
    }
    if (sum_w) sum_w[blockIdx.y * pitch + c] = dw.value();
    if (sum_b) sum_b[blockIdx.y * pitch + c] = db.value();
}

// Sums over the workgroups of the first kernel, 64 columns a workgroup: SLICES waves each take every SLICES-th row, and meet in their order
constexpr int NORM_SLICES = 16;
template <int WDT>
__global__ __launch_bounds__(64 * NORM_SLICES) void layer_norm_sums_kernel(const float *sum_w, const float *sum_b, int64_t pitch, int parts, int64_t cols, uint8_t *dweight,
                                                                           uint8_t *dbias)
{
    using namespace norm;
    __shared__ float lds[NORM_SLICES][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    const float *const from = blockIdx.y == 0 ? sum_w : sum_b;
    uint8_t *const out = blockIdx.y == 0 ? dweight : dbias;
    if (!out) return;  // (the whole workgroup)
    float s = 0.0f;
    if (c < cols) {
#pragma unroll 8
        for (int p = slice; p < parts; p += NORM_SLICES) s += from[p * pitch + c];
    }
    lds[slice][lane] = s;
    __syncthreads();
    if (slice == 0 && c < cols) {
        for (int k = 1; k < NORM_SLICES; ++k) s += lds[k][lane];
        Elem<WDT>::store(out + c * Elem<WDT>::BYTES, s);
    }
}

namespace norm {

// f(threads of a row, pieces of a thread) of the forward kernel; false for rows that no workgroup holds
template <class F>
static bool with_row(int64_t pieces, F &&f)
{
    auto at = [&](auto t, auto u) { f(t, u); return true; };
    using std::integral_constant;
    if (pieces <= 8) return at(integral_constant<int, 8>{}, integral_constant<int, 1>{});
    if (pieces <= 16) return at(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    if (pieces <= 32) return at(integral_constant<int, 32>{}, integral_constant<int, 1>{});
    if (pieces <= 64) return at(integral_constant<int, 64>{}, integral_constant<int, 1>{});
    if (pieces <= 128) return at(integral_constant<int, 64>{}, integral_constant<int, 2>{});
    if (pieces <= 256) return at(integral_constant<int, 64>{}, integral_constant<int, 4>{});
    // (us, 64 threads of eight pieces / 256 of two: 128 x 4096 bf16 5.7 / 3.5, 1024 rows 6.6 / 4.8, 8192 rows 31.8 / 21.2, 32768 rows 193 / 96; 32768 x 2304 129 / 67; binary32 128 x 2048 4.4 / 3.2,
    // 32768 rows 101 / 92: eight pieces take 170 registers and their loads go out one behind the other)
    if (pieces <= 512) return at(integral_constant<int, 256>{}, integral_constant<int, 2>{});
    if (pieces <= 1024) return at(integral_constant<int, 256>{}, integral_constant<int, 4>{});
    if (pieces <= 2048) return at(integral_constant<int, 256>{}, integral_constant<int, 8>{});
    if (pieces <= 4096) return at(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
    return false;
}

// Of the backward kernel: threads of a row; the pieces of a thread are 2 (bf16) or 4 (binary32) at most, 16 columns
inline int bwd_threads(int64_t cols, int dt)
{
    const int64_t pieces = (cols + per_piece(dt) - 1) / per_piece(dt), u = dt == NVFP4_BF16 ? 2 : 4;
    int t = 8;
    while (t * u < pieces) t *= 2;
    return t;
}
constexpr int BWD_NT = 512, MOST_BWD_THREADS = 1024;
constexpr int64_t BWD_PARTS = 512;  // sums of so many workgroups
inline int64_t bwd_parts(int64_t rows, int64_t cols, int dt)
{
    const int t = bwd_threads(cols, dt);
    if (t > MOST_BWD_THREADS) {
        const int64_t by_columns = (cols + 255) / 256, want = (1024 + by_columns - 1) / by_columns;
        return rows < want ? rows : want;
    }
    const int64_t teams = t < BWD_NT ? BWD_NT / t : 1, all = (rows + teams - 1) / teams;
    return all < BWD_PARTS ? all : BWD_PARTS;
}

}  // namespace norm

size_t layer_norm_bwd_workspace(int64_t rows, int64_t cols, int dt, bool dweight, bool dbias)
{
    return (size_t)norm::bwd_parts(rows, cols, dt) * (size_t)cols * 4 * ((dweight ? 1 : 0) + (dbias ? 1 : 0));
}

template <int DT>
static hipError_t forward(const NormArgs &P, const uint8_t *x, float eps, uint8_t *y, float *mean, float *rstd, hipStream_t st)
{
    const uint8_t *const w = reinterpret_cast<const uint8_t *>(P.weight), *const b = reinterpret_cast<const uint8_t *>(P.bias);
    const bool held = norm::with_row((P.cols + norm::per_piece(DT) - 1) / norm::per_piece(DT), [&](auto t, auto u) {
        constexpr int T = decltype(t)::value, U = decltype(u)::value, NT = T < 256 ? 256 : T;
        layer_norm_kernel<DT, T, U><<<launch_grid((P.rows + NT / T - 1) / (NT / T)), NT, 0, st>>>(x, P.rows, (int)P.cols, P.ld, w, b, P.wdt, P.center, eps, y, mean, rstd);
    });
    if (!held) layer_norm_long_kernel<DT><<<launch_grid(P.rows), 1024, 0, st>>>(x, P.rows, P.cols, P.ld, w, b, P.wdt, P.center, eps, y, mean, rstd);
    return hipGetLastError();
}

template <int DT>
static hipError_t backward(const NormArgs &P, const uint8_t *dy, int64_t ldy, const uint8_t *x, const float *mean, const float *rstd, uint8_t *dx, uint8_t *dweight, uint8_t *dbias,
                           float *workspace, hipStream_t st)
{
    using namespace norm;
    const uint8_t *const w = reinterpret_cast<const uint8_t *>(P.weight);
    const int64_t parts = bwd_parts(P.rows, P.cols, DT);
    float *const sum_w = dweight ? workspace : nullptr, *const sum_b = dbias ? workspace + (dweight ? parts * P.cols : 0) : nullptr;
    if (P.rows == 0) {
        // (the sums of nothing are left to the second kernel)
    } else if (const int t = bwd_threads(P.cols, DT); t > MOST_BWD_THREADS) {
        layer_norm_bwd_long_kernel<DT><<<launch_grid(P.rows), 1024, 0, st>>>(dy, ldy, x, P.rows, P.cols, P.ld, w, P.wdt, mean, rstd, dx);
        if (sum_w || sum_b)
            layer_norm_columns_kernel<DT><<<dim3((unsigned)((P.cols + 255) / 256), (unsigned)parts), 256, 0, st>>>(dy, ldy, x, P.rows, P.cols, P.ld, mean, rstd,
                                                                                                                   (P.rows + parts - 1) / parts, sum_w, sum_b, P.cols);
    } else {
        auto run = [&](auto threads) {
            constexpr int T = decltype(threads)::value, NT = T < BWD_NT ? BWD_NT : T, U = DT == NVFP4_BF16 ? 2 : 4;
            layer_norm_bwd_kernel<DT, T, U, NT><<<dim3((unsigned)parts), NT, T < NT ? (size_t)P.cols * 4 : 0, st>>>(dy, ldy, x, P.rows, (int)P.cols, P.ld, w, P.wdt, mean, rstd, dx, sum_w, sum_b, P.cols);
        };
        if (t == 8) run(std::integral_constant<int, 8>{});
        else if (t == 16) run(std::integral_constant<int, 16>{});
        else if (t == 32) run(std::integral_constant<int, 32>{});
        else if (t == 64) run(std::integral_constant<int, 64>{});
        else if (t == 128) run(std::integral_constant<int, 128>{});
        else if (t == 256) run(std::integral_constant<int, 256>{});
        else if (t == 512) run(std::integral_constant<int, 512>{});
        else run(std::integral_constant<int, 1024>{});
    }
    if (dweight || dbias) {  // (zeros where there are no rows)
        const dim3 grid((unsigned)((P.cols + 63) / 64), 2);
        if (P.wdt == NVFP4_BF16) layer_norm_sums_kernel<NVFP4_BF16><<<grid, 64 * NORM_SLICES, 0, st>>>(sum_w, sum_b, P.cols, (int)parts, P.cols, dweight, dbias);
        else layer_norm_sums_kernel<NVFP4_F32><<<grid, 64 * NORM_SLICES, 0, st>>>(sum_w, sum_b, P.cols, (int)parts, P.cols, dweight, dbias);
    }
    return hipGetLastError();
}

hipError_t launch_layer_norm(const NormArgs &P, int dt, const void *x, float eps, void *y, float *mean, float *rstd, hipStream_t st)
{
    auto *f = dt == NVFP4_BF16 ? forward<NVFP4_BF16> : forward<NVFP4_F32>;
    return f(P, reinterpret_cast<const uint8_t *>(x), eps, reinterpret_cast<uint8_t *>(y), mean, rstd, st);
}

hipError_t launch_layer_norm_bwd(const NormArgs &P, int dt, const void *dy, int64_t ldy, const void *x, const float *mean, const float *rstd, void *dx, void *dweight,
                                 void *dbias, void *workspace, hipStream_t st)
{
    auto *f = dt == NVFP4_BF16 ? backward<NVFP4_BF16> : backward<NVFP4_F32>;
    return f(P, reinterpret_cast<const uint8_t *>(dy), ldy, reinterpret_cast<const uint8_t *>(x), mean, rstd, reinterpret_cast<uint8_t *>(dx), reinterpret_cast<uint8_t *>(dweight),
             reinterpret_cast<uint8_t *>(dbias), reinterpret_cast<float *>(workspace), st);
}

}  // namespace nvfp4
