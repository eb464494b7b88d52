// Quantization to 8 bits: E4M3 codes with one power-of-two scale (an E8M0 byte) per 128 elements along the axis that a product contracts,
//     a = max|x| of the block,  e = the smallest exponent with a <= 448 * 2^e (at least -127),  byte = e + 127,  code = E4M3(x * 2^-e),
// ties to the even code.  Everything but the code's rounding is exact, so the codes are a function of the input's bits alone; a block
// with an infinity or a NaN becomes NaN codes, so that the product shows it.  The scale is a power of two because that is what the
// matrix instruction applies by itself: a product with binary32 scales would need a multiply-add per output and 128 elements.
//
// What bounds it is memory: 2 or 4 bytes per element in, 1 out (2 where both sides are wanted, from one read).
#include "experts.h"

namespace nvfp4 {
namespace f8 {

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// Eight neighbouring elements as binary32 bits.  Rows start at any multiple of an element: the memory pipe takes wide loads at any such
// address (ragged pitches cost requests, not instructions).
template <int DT>
struct Eight {
    uint32_t v[8];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0;
    }
    __device__ __forceinline__ void load(const void *row, int64_t col)
    {
        if (DT == NVFP4_BF16) {
            struct __attribute__((packed, aligned(2))) P { u32x4_t w; };
            const u32x4_t w = reinterpret_cast<const P *>(reinterpret_cast<const uint16_t *>(row) + col)->w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = w[i] << 16;
                v[2 * i + 1] = w[i] & 0xFFFF0000u;
            }
        } else {
            struct __attribute__((packed, aligned(4))) P { u32x4_t w; };
            const P *p = reinterpret_cast<const P *>(reinterpret_cast<const float *>(row) + col);
            const u32x4_t lo = p[0].w, hi = p[1].w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i] = lo[i];
                v[4 + i] = hi[i];
            }
        }
    }
    __device__ __forceinline__ void load_some(const void *row, int64_t col, int n)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i >= n ? 0u : DT == NVFP4_BF16 ? (uint32_t)reinterpret_cast<const uint16_t *>(row)[col + i] << 16 : reinterpret_cast<const uint32_t *>(row)[col + i];
    }
    __device__ __forceinline__ void load_upto(const void *row, int64_t col, int64_t cols)
    {
        if (col + 8 <= cols) load(row, col);
        else if (col < cols) load_some(row, col, (int)(cols - col));
        else zero();
    }
};

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// (magnitudes as integers: NaN above infinity above every number)
template <int DT>
__device__ __forceinline__ uint32_t largest(const Eight<DT> &x)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = umax(m, x.v[i] & 0x7FFFFFFFu);
    return m;
}

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

__device__ __forceinline__ uint32_t four_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float q)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(a) * q, __uint_as_float(b) * q, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(c) * q, __uint_as_float(d) * q, w, true);
    return (uint32_t)w;
}

}  // namespace f8

// Row of x behind row r, -1 for none
__device__ __forceinline__ int64_t source_row(const Fp8QuantArgs &P, int64_t r)
{
    if (!P.order) return r;
    const int32_t pair = P.order[r];
    const int64_t at = pair < 0 ? -1 : pair / P.top_k;
    return at < P.x_rows ? at : -1;
}

// Rows alone.  16 lanes hold a block, a wave four groups of RPG consecutive rows each: as many loads in flight, and their scale bytes are
// neighbours in the block-major scales.
template <int DT, int RPG>
__global__ __launch_bounds__(256) void fp8_quantize_rows_kernel(Fp8QuantArgs P, int64_t rows, int blocks, unsigned across)
{
    using namespace f8;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, in = lane & 15;
    const unsigned up = blockIdx.x / across;
    const int kb = (int)(blockIdx.x - up * across) * 4 + wave;
    if (kb >= blocks) return;
    const int64_t r0 = ((int64_t)up * 4 + (lane >> 4)) * RPG;
    const int64_t col = (int64_t)kb * FP8_BLOCK + in * 8;
    Eight<DT> x[RPG];
#pragma unroll
    for (int i = 0; i < RPG; ++i) {
        const int64_t src = r0 + i < rows ? source_row(P, r0 + i) : -1;
        if (src < 0) x[i].zero();
        else x[i].load_upto(reinterpret_cast<const uint8_t *>(P.x) + src * P.ld * (DT == NVFP4_BF16 ? 2 : 4), col, P.cols);
    }
    uint32_t mine = 0;
#pragma unroll
    for (int i = 0; i < RPG; ++i) {
        const uint32_t m = max16(largest(x[i])), byte = scale_byte(m);
        const float q = inverse_scale(m, byte);
        const u32x2_t w = {four_codes(x[i].v[0], x[i].v[1], x[i].v[2], x[i].v[3], q), four_codes(x[i].v[4], x[i].v[5], x[i].v[6], x[i].v[7], q)};
        if (r0 + i < rows) *reinterpret_cast<u32x2_t *>(P.codes_r + (r0 + i) * blocks * FP8_BLOCK + col) = w;
        if (in == i) mine = byte;
    }
    if (in < RPG && r0 + in < rows) P.scales_r[(int64_t)kb * rows + r0 + in] = (uint8_t)mine;
}

// Columns, or both sides from one read: a workgroup takes 128 rows (a column block: of one matrix, or of one group of rows) by 128 columns,
// a thread 8 rows by 8 columns of them, all in registers.  Codes of the column side turn through the LDS into rows of 128 bytes.
template <int DT, bool ROWS>
__global__ __launch_bounds__(256) void fp8_quantize_tile_kernel(Fp8QuantArgs P, int col_tiles, int slots)
{
    using namespace f8;
    constexpr int PITCH = FP8_BLOCK + 16;  // (16-byte reads of neighbouring columns start in other banks)
    __shared__ __attribute__((aligned(16))) uint8_t turned[FP8_BLOCK * PITCH];
    __shared__ uint32_t top[4][FP8_BLOCK];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cg = tid & 15, rg = tid >> 4;
    const int tile = (int)(blockIdx.x % (unsigned)col_tiles);
    const int at = (int)(blockIdx.x / (unsigned)col_tiles);
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
        slot = at - matrix * slots;
        count = (int)(P.rows - (int64_t)slot * FP8_BLOCK < FP8_BLOCK ? P.rows - (int64_t)slot * FP8_BLOCK : FP8_BLOCK);
        row0 = matrix * P.rows + (int64_t)slot * FP8_BLOCK;
    }
    if (count <= 0) return;
    const int64_t col = (int64_t)tile * FP8_BLOCK + cg * 8;
    Eight<DT> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t src = rg * 8 + i < count ? source_row(P, row0 + rg * 8 + i) : -1;
        if (src < 0) x[i].zero();
        else x[i].load_upto(reinterpret_cast<const uint8_t *>(P.x) + src * P.ld * (DT == NVFP4_BF16 ? 2 : 4), col, P.cols);
    }
    // columns' largest magnitudes: of the thread's rows, of the wave's, of all
    uint32_t colmax[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = umax(m, x[i].v[j] & 0x7FFFFFFFu);
        m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
        m = umax(m, (uint32_t)__shfl_xor((int)m, 32));
        colmax[j] = m;
    }
    if (lane < 16) {
#pragma unroll
        for (int j = 0; j < 8; ++j) top[wave][cg * 8 + j] = colmax[j];
    }
    if (ROWS) {
        const int64_t rows = P.batch * P.rows, pitch = (int64_t)col_tiles * FP8_BLOCK;
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t m = max16(largest(x[i])), byte = scale_byte(m);
            const float q = inverse_scale(m, byte);
            const u32x2_t w = {four_codes(x[i].v[0], x[i].v[1], x[i].v[2], x[i].v[3], q), four_codes(x[i].v[4], x[i].v[5], x[i].v[6], x[i].v[7], q)};
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
        const u32x2_t w = {four_codes(x[0].v[j], x[1].v[j], x[2].v[j], x[3].v[j], q), four_codes(x[4].v[j], x[5].v[j], x[6].v[j], x[7].v[j], q)};
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

hipError_t launch_fp8_quantize(const Fp8QuantArgs &P, int dt, hipStream_t st)
{
    const int64_t tiles = (P.cols + FP8_BLOCK - 1) / FP8_BLOCK;
    if (!P.codes_c) {
        const int64_t rows = P.batch * P.rows, across = (tiles + 3) / 4;
        // few rows: one a group of lanes, so that more waves load
        const int rpg = rows * tiles >= 32 * 1024 ? 8 : 1;
        const dim3 grid((unsigned)(across * ((rows + 4 * rpg - 1) / (4 * rpg))));
        auto *k = dt == NVFP4_BF16 ? (rpg == 8 ? fp8_quantize_rows_kernel<NVFP4_BF16, 8> : fp8_quantize_rows_kernel<NVFP4_BF16, 1>)
                                   : (rpg == 8 ? fp8_quantize_rows_kernel<NVFP4_F32, 8> : fp8_quantize_rows_kernel<NVFP4_F32, 1>);
        k<<<grid, 256, 0, st>>>(P, rows, (int)tiles, (unsigned)across);
        return hipGetLastError();
    }
    const int64_t slots = fp8_slots(P.rows, P.offsets ? P.groups : 0);
    const dim3 grid((unsigned)(tiles * slots * P.batch));
    auto *k = dt == NVFP4_BF16 ? (P.codes_r ? fp8_quantize_tile_kernel<NVFP4_BF16, true> : fp8_quantize_tile_kernel<NVFP4_BF16, false>)
                               : (P.codes_r ? fp8_quantize_tile_kernel<NVFP4_F32, true> : fp8_quantize_tile_kernel<NVFP4_F32, false>);
    k<<<grid, 256, 0, st>>>(P, (int)tiles, (int)slots);
    return hipGetLastError();
}

}  // namespace nvfp4
