// Quantization to 8 bits: E4M3 codes with one power-of-two scale (an E8M0 byte) per 128 elements along the axis that a product contracts,
//     a = max|x| of the block,  e = the smallest exponent with a <= 448 * 2^e (at least -127),  byte = e + 127,  code = E4M3(x * 2^-e),
// ties to the even code.  Everything but the code's rounding is exact, so the codes are a function of the input's bits alone; a block
// with an infinity or a NaN becomes NaN codes, so that the product shows it.  The scale is a power of two because that is what the
// matrix instruction applies by itself: a product with binary32 scales would need a multiply-add per output and 128 elements.
//
// What bounds it is memory: 2 or 4 bytes per element in, 1 out (2 where both sides are wanted, from one read).  bf16 4096 x 11008, rows 24.2 us (5.6
// TB/s, what a copy reaches), both sides 35 (5.2) where the last cache level still has the tensor, 37 to 42 (4.3 to 4.8) from memory: the columns' codes leave in pieces of 128
// bytes, a column pitch apart; 16 matrices 4096 x 2048 both sides 91 (5.9); 8192 x 2048 gathered to 16384 rows, both sides by expert 32 to 36 (3.7 to 4.2 TB/s with the rows
// read twice); 16 x 4096 3.0, latency.
#include "experts.h"

namespace nvfp4 {
namespace f8 {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Eight neighbouring elements as they came, in W words.  Rows start at any multiple of an element: the memory pipe takes wide loads at any such
// address (ragged pitches cost requests, not instructions).  Magnitudes are compared as integers, NaN above infinity above every number,
// bf16 ones two at a time.
template <int DT>
struct Eight {
    static constexpr bool HALF = DT == NVFP4_BF16;
    static constexpr int W = HALF ? 4 : 8, ESZ = HALF ? 2 : 4;
    uint32_t w[W];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    template <bool STREAMED>
    __device__ __forceinline__ void load(const uint8_t *p)
    {
        struct __attribute__((packed, aligned(ESZ))) P { u32x4_t w; };
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const u32x4_t v = STREAMED ? __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(p) + i) : reinterpret_cast<const P *>(p)[i].w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
        }
    }
    __device__ __forceinline__ void load_some(const uint8_t *p, int n)
    {
        zero();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) {
                if (HALF) w[i >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i] << (16 * (i & 1));
                else w[i % W] = reinterpret_cast<const uint32_t *>(p)[i];
            }
    }
    // without the first n (0 .. 8), zeros behind the others
    __device__ __forceinline__ void drop(int n)
    {
#pragma unroll
        for (int step = W / 2; step > 0; step /= 2) {
            const bool on = (n & (HALF ? 2 * step : step)) != 0;
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = on ? (i + step < W ? w[(i + step) % W] : 0u) : w[i];
        }
        if (HALF) {
            const bool on = (n & 1) != 0;
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = on ? w[i] >> 16 | (i + 1 < W ? w[(i + 1) % W] << 16 : 0u) : w[i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = n >= 8 ? 0u : w[i];
    }
    // binary32 bits of element i
    __device__ __forceinline__ uint32_t bits(int i) const { return HALF ? (i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16) : w[i % W]; }
    __device__ __forceinline__ float value(int i) const { return __uint_as_float(bits(i)); }
    __device__ __forceinline__ static uint32_t magnitudes(uint32_t v) { return v & (HALF ? 0x7FFF7FFFu : 0x7FFFFFFFu); }
    __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b)
    {
        typedef unsigned short u16x2_t __attribute__((ext_vector_type(2)));
        return HALF ? __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2_t, a), __builtin_bit_cast(u16x2_t, b))) : umax(a, b);
    }
    // the largest magnitude's bits
    __device__ __forceinline__ uint32_t largest() const
    {
        uint32_t m = magnitudes(w[0]);
#pragma unroll
        for (int i = 1; i < W; ++i) m = larger(m, magnitudes(w[i]));
        return HALF ? umax(m << 16, m & 0xFFFF0000u) : m;
    }
};

// maximum over the 16 lanes of a row of lanes
__device__ __forceinline__ uint32_t max16(uint32_t m)
{
    m = umax(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0xB1, 0xF, 0xF, false));   // quad: 1 0 3 2
    m = umax(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x4E, 0xF, 0xF, false));   // quad: 2 3 0 1
    m = umax(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x141, 0xF, 0xF, false));  // half row mirrored
    m = umax(m, (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x140, 0xF, 0xF, false));  // row mirrored
    return m;
}

constexpr uint32_t NOT_FINITE = 0x7F800000u;

// Scale byte of a block whose largest magnitude has the bits m: 448 = 1.75 * 2^8
__device__ __forceinline__ uint32_t scale_byte(uint32_t m)
{
    if (m >= NOT_FINITE) return 127;
    const int e = (int)(m >> 23) - 8 + ((m & 0x7FFFFFu) > 0x600000u);
    return e > 0 ? (uint32_t)e : 0u;
}
// 2^-e; of a block that is not finite NaN, which makes every code one
__device__ __forceinline__ float inverse_scale(uint32_t m, uint32_t byte) { return __uint_as_float(m >= NOT_FINITE ? 0x7FC00000u : (254u - byte) << 23); }

__device__ __forceinline__ uint32_t four_codes(float a, float b, float c, float d, float q)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * q, b * q, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c * q, d * q, w, true);
    return (uint32_t)w;
}
template <int DT>
__device__ __forceinline__ u32x2_t eight_codes(const Eight<DT> &x, float q)
{
    return u32x2_t{four_codes(x.value(0), x.value(1), x.value(2), x.value(3), q), four_codes(x.value(4), x.value(5), x.value(6), x.value(7), q)};
}

}  // namespace f8

// Elements col .. col + 7 of N rows r0, r0 + step, ..., of which there are `have` (rows past these, and rows that an order does not name, are zeros).
// Loads do not branch: a row that is not there reads the first one instead, a piece past the row's end what ends with the row (rows of eight elements and more).  us, pieces
// at an end element by element / so: 11274 x 1223 bf16, rows 14.5 / 11.5, both sides 18.5 / 18.0; 60000 x 263 both sides 24.8 / 21.9.
template <int DT, bool STREAMED, int N>
__device__ __forceinline__ void load_rows(const Fp8QuantArgs &P, f8::Eight<DT> (&x)[N], int64_t r0, int have, int64_t col, bool whole)
{
    constexpr int ESZ = f8::Eight<DT>::ESZ;
    const uint8_t *const base = reinterpret_cast<const uint8_t *>(P.x) + col * ESZ;
    if (P.order ? P.x_rows == 0 : false) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].zero();
        return;
    }
    int64_t src[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        src[i] = i < have ? r0 + i : -1;
        if (P.order) {
            const int32_t pair = P.order[i < have ? r0 + i : 0];
            const int64_t at = pair / P.top_k;
            src[i] = i < have && pair >= 0 && at < P.x_rows ? at : -1;
        }
    }
    if (whole) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].template load<STREAMED>(base + (src[i] < 0 ? 0 : src[i]) * P.ld * ESZ);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int k = 0; k < f8::Eight<DT>::W; ++k) x[i].w[k] = src[i] < 0 ? 0u : x[i].w[k];
    } else if (P.cols >= 8) {
        const int64_t at = col < P.cols - 8 ? col : P.cols - 8;
        const int past = col - at < 8 ? (int)(col - at) : 8;
        const uint8_t *const from = reinterpret_cast<const uint8_t *>(P.x) + at * ESZ;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].template load<false>(from + (src[i] < 0 ? 0 : src[i]) * P.ld * ESZ);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].drop(src[i] < 0 ? 8 : past);
    } else {
        const int64_t left = P.cols - col;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (src[i] < 0 || left <= 0) x[i].zero();
            else x[i].load_some(base + src[i] * P.ld * ESZ, (int)left);
        }
    }
}

// Rows alone.  16 lanes hold a block, a wave four groups of RPG consecutive rows each: as many loads in flight, and their scale bytes are
// neighbours in the block-major scales.
template <int DT, bool STREAMED, int RPG>
__global__ __launch_bounds__(256) void fp8_quantize_rows_kernel(Fp8QuantArgs P, int64_t rows, int blocks, unsigned across)
{
    using namespace f8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane & 15;
    const unsigned id = workgroup(), up = id / across;
    const int kb = __builtin_amdgcn_readfirstlane((int)(id - up * across) * 4 + wave);
    if (kb >= blocks) return;
    const int64_t r0 = ((int64_t)up * 4 + (lane >> 4)) * RPG;
    const int64_t col = (int64_t)kb * FP8_BLOCK + in * 8;
    Eight<DT> x[RPG];
    load_rows<DT, STREAMED, RPG>(P, x, r0, (int)(rows - r0 < RPG ? rows - r0 : RPG), col, (int64_t)(kb + 1) * FP8_BLOCK <= P.cols);
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < RPG; ++i) {
        const uint32_t m = max16(x[i].largest()), byte = scale_byte(m);
        const u32x2_t w = eight_codes(x[i], inverse_scale(m, byte));
        if (r0 + i < rows) *reinterpret_cast<u32x2_t *>(P.codes_r + (r0 + i) * blocks * FP8_BLOCK + col) = w;
        if (in == i) mine = byte;
    }
    if (in < RPG && r0 + in < rows) P.scales_r[(int64_t)kb * rows + r0 + in] = (uint8_t)mine;
}

// Columns, or both sides from one read: a workgroup takes 128 rows (a column block: of one matrix, or of one group of rows) by 128 columns,
// a thread 8 rows by 8 columns of them, all in registers.  Codes of the column side turn through the LDS into rows of 128 bytes.
template <int DT, bool STREAMED, bool ROWS>
__global__ __launch_bounds__(256) void fp8_quantize_tile_kernel(Fp8QuantArgs P, int col_tiles, int slots)
{
    using namespace f8;
    constexpr int PITCH = FP8_BLOCK + 16;  // (16-byte reads of neighbouring columns start in other banks)
    __shared__ __attribute__((aligned(16))) uint8_t turned[FP8_BLOCK * PITCH];
    __shared__ uint32_t top[4][FP8_BLOCK];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 15, rg = tid >> 4;
    const unsigned id = workgroup();
    const int tile = (int)(id % (unsigned)col_tiles);
    const int at = (int)(id / (unsigned)col_tiles);
    int64_t row0;  // of all matrices' rows
    int count, slot, matrix = 0;
    if (P.offsets) {
        slot = at;
        const int e = group_of_slot(P.offsets, P.groups, (int32_t)P.rows, FP8_BLOCK, slot);
        if (e < 0) return;
        const RowGroup g = row_group(P.offsets, e, (int32_t)P.rows);
        const int b = slot - (g.first / FP8_BLOCK + e);
        if (b < 0) return;
        count = g.count - b * FP8_BLOCK;
        row0 = g.first + (int64_t)b * FP8_BLOCK;
    } else {
        matrix = at / slots;
        if (matrix >= P.batch) return;
        slot = at - matrix * slots;
        count = (int)(P.rows - (int64_t)slot * FP8_BLOCK < FP8_BLOCK ? P.rows - (int64_t)slot * FP8_BLOCK : FP8_BLOCK);
        row0 = matrix * P.rows + (int64_t)slot * FP8_BLOCK;
    }
    if (count <= 0) return;
    const int64_t col = (int64_t)tile * FP8_BLOCK + cg * 8;
    Eight<DT> x[8];
    load_rows<DT, STREAMED, 8>(P, x, row0 + rg * 8, count - rg * 8, col, (int64_t)(tile + 1) * FP8_BLOCK <= P.cols);
    // columns' largest magnitudes: of the thread's rows, of the wave's, of all
#pragma unroll
    for (int j = 0; j < Eight<DT>::W; ++j) {
        uint32_t m = Eight<DT>::magnitudes(x[0].w[j]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = Eight<DT>::larger(m, Eight<DT>::magnitudes(x[i].w[j]));
        m = Eight<DT>::larger(m, (uint32_t)__shfl_xor((int)m, 16));
        m = Eight<DT>::larger(m, (uint32_t)__shfl_xor((int)m, 32));
        if (lane < 16) {
            if (Eight<DT>::HALF) {
                top[wave][cg * 8 + (2 * j & 7)] = m << 16;
                top[wave][cg * 8 + (2 * j & 7) + 1] = m & 0xFFFF0000u;
            } else {
                top[wave][cg * 8 + j] = m;
            }
        }
    }
    if (ROWS) {
        const int64_t rows = P.batch * P.rows, pitch = (int64_t)col_tiles * FP8_BLOCK;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = max16(x[i].largest()), byte = scale_byte(m);
            const u32x2_t w = eight_codes(x[i], inverse_scale(m, byte));
            if (rg * 8 + i < count) *reinterpret_cast<u32x2_t *>(P.codes_r + (row0 + rg * 8 + i) * pitch + col) = w;
            if (cg == i) mine = byte;
        }
        if (cg < 8 && rg * 8 + cg < count) P.scales_r[tile * rows + row0 + rg * 8 + cg] = (uint8_t)mine;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = umax(m, top[w][cg * 8 + j]);
        const uint32_t byte = scale_byte(m);
        const float q = inverse_scale(m, byte);
        const u32x2_t w = {four_codes(x[0].value(j), x[1].value(j), x[2].value(j), x[3].value(j), q), four_codes(x[4].value(j), x[5].value(j), x[6].value(j), x[7].value(j), q)};
        *reinterpret_cast<u32x2_t *>(turned + (cg * 8 + j) * PITCH + rg * 8) = w;
    }
    const int64_t out_rows = P.batch * P.cols, out0 = matrix * P.cols + (int64_t)tile * FP8_BLOCK, pitch = (int64_t)slots * FP8_BLOCK;
    const int ncols = (int)(P.cols - (int64_t)tile * FP8_BLOCK < FP8_BLOCK ? P.cols - (int64_t)tile * FP8_BLOCK : FP8_BLOCK);
    if (tid < ncols) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) m = umax(m, top[w][tid]);
        P.scales_c[(int64_t)slot * out_rows + out0 + tid] = (uint8_t)scale_byte(m);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int c = u * 32 + (tid >> 3), piece = (tid & 7) * 16;
        if (c < ncols)
            *reinterpret_cast<u32x4_t *>(P.codes_c + (out0 + c) * pitch + (int64_t)slot * FP8_BLOCK + piece) =
                *reinterpret_cast<const u32x4_t *>(turned + c * PITCH + piece);
    }
}

template <int DT, bool STREAMED>
static hipError_t launch(const Fp8QuantArgs &P, hipStream_t st)
{
    const int64_t tiles = (P.cols + FP8_BLOCK - 1) / FP8_BLOCK;
    if (!P.codes_c) {
        const int64_t rows = P.batch * P.rows, across = (tiles + 3) / 4;
        // few rows: one a group of lanes, so that more waves load
        const int rpg = STREAMED || rows * tiles >= 32 * 1024 ? 8 : 1;
        const dim3 grid = launch_grid(across * ((rows + 4 * rpg - 1) / (4 * rpg)));
        if (rpg == 8) fp8_quantize_rows_kernel<DT, STREAMED, 8><<<grid, 256, 0, st>>>(P, rows, (int)tiles, (unsigned)across);
        else fp8_quantize_rows_kernel<DT, false, 1><<<grid, 256, 0, st>>>(P, rows, (int)tiles, (unsigned)across);
        return hipGetLastError();
    }
    const int64_t slots = fp8_slots(P.rows, P.offsets ? P.groups : 0);
    const dim3 grid = launch_grid(tiles * slots * P.batch);
    if (P.codes_r) fp8_quantize_tile_kernel<DT, STREAMED, true><<<grid, 256, 0, st>>>(P, (int)tiles, (int)slots);
    else fp8_quantize_tile_kernel<DT, STREAMED, false><<<grid, 256, 0, st>>>(P, (int)tiles, (int)slots);
    return hipGetLastError();
}

hipError_t launch_fp8_quantize(const Fp8QuantArgs &P, int dt, hipStream_t st)
{
    // Tensors past what the last cache level holds come by streaming loads (they need 16-byte aligned rows).  us, both sides: 65536 x 2048 bf16 111 / 93, 16384 x 8192
    // binary32 (rows) 126 / 116; 8192 x 8192 bf16 50 / 51, 4096 x 11008 binary32 49 / 58.
    const int64_t esz = dt == NVFP4_BF16 ? 2 : 4;
    const bool s = !P.order && P.ld * esz % 16 == 0 && reinterpret_cast<uintptr_t>(P.x) % 16 == 0 && P.batch * P.rows * P.cols * esz >= ((int64_t)256 << 20);
    return dt == NVFP4_BF16 ? (s ? launch<NVFP4_BF16, true>(P, st) : launch<NVFP4_BF16, false>(P, st)) : s ? launch<NVFP4_F32, true>(P, st) : launch<NVFP4_F32, false>(P, st);
}

}  // namespace nvfp4
