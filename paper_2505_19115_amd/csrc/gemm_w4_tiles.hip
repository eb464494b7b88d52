// Products with packed 4-bit weights for more rows than a few (gemm_w4.hip): a workgroup's tile is 16 MT rows of x by 64 TN rows of W, 16 TN for each of its four waves, two or
// more workgroups a CU where there are as many.  W goes from memory into the registers of the one wave that multiplies with it, a K tile of 128 ahead, which expands its codes there, a
// quarter of a K tile ahead of the products: nothing of W is in the LDS, and each code is expanded once a tile (16 vector instructions for 8 codes with E4M3 scales, 4 with E8M0).
// x goes through the LDS, two stages of a K tile, where all waves read it, a fragment at a time, three ahead.  bf16 rows on 16-byte boundaries go there by direct global -> LDS
// loads, other rows through registers, binary32 ones as three bf16 pieces.
// What bounds it: 4096^3 NVFP4 125 us (1.1 PFLOP/s, MXFP4 112; the instruction alone reaches 1.96 with two waves a SIMD), of which the expansion is a sixth, the rest waits: for the K
// tile's loads, which a tile alone on its CU waits 0.4 us for, and at its barrier.  Tried: 32 x 32 x 16 products on one wave a SIMD, W through the LDS two K tiles ahead, one barrier a K tile
// behind its last read (777 x 12288 x 4096 104 us, 92 here; 4096^3 144).  Tiles of 128 x 256 take all 256 registers and spill 2 to 6 of them (NVFP4; wider blocks by expert).
// LDS image of a stage: row after row of 256 bytes, sixteen pieces of 16; piece c of row r stands at c ^ place(r), which spreads the rows that a fragment's
// read is served with together over the banks (kernels.h).
#include "gemm_w4.h"

namespace nvfp4 {
namespace w4 {

// Assembly because the compiler takes a direct-to-LDS load for a possible writer of all of the LDS and would wait for it before the next LDS read; here a
// stage is read behind an explicit wait and barrier only.  16 bytes a lane, side by side from dst on.
__device__ __forceinline__ void load_lds(uint32_t dst, uint32_t off, const uint8_t *base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(dst)), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ int place(int row) { return (row & 3) | quad_xor((row >> 2) & 3) << 2; }
// All loads have come, as the compiler knows then too (vmcnt 0, the other counters as they are)
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }
__device__ __forceinline__ void barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
template <int I, int N, class F>
__device__ __forceinline__ void each(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<I + 1, N>(f);
    }
}

template <int MT, int PIECES>
constexpr int STAGE = MT * 16 * 256 * PIECES;

}  // namespace w4

// DIRECT: x is bf16 with rows on 16-byte boundaries; a tile of its rows (with order: all of them) spans less than 2^32 bytes
template <int XDT, int SC, int MT, int TN, bool GROUPED, bool DIRECT>
__global__ __launch_bounds__(256, 2) void gemm_w4_tiles_kernel(W4Args P, int out_dt)
{
    using namespace w4;
    constexpr int BM = 16 * MT, BN = 64 * TN, XSZ = Elem<XDT>::BYTES, PIECES = Elems<XDT>::PIECES, STG = STAGE<MT, PIECES>;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];  // [2][pieces][rows][256]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, r = lane & 15;
    const int ntx = (int)((P.N + BN - 1) / BN), nty = (int)P.slots;
    if (workgroup() >= (unsigned)ntx * (unsigned)nty) return;
    int ty, tx;
    tile_coords((int)workgroup(), ntx, nty, ty, tx);
    int64_t m0 = (int64_t)ty * BM, left = P.rows - m0;
    int e = 0;
    if (GROUPED) {
        const f8g::RowTile t = f8g::row_tile(P.offsets, P.groups, (int32_t)P.rows, BM, ty);
        if (t.group < 0) return;
        e = t.group;
        m0 = t.row;
        left = t.left;
    }
    const int rows = (int)(left < BM ? left : BM);
    const bool none = GROUPED && e == P.groups;  // rows of no group
    const int64_t n0 = (int64_t)tx * BN + wave * (16 * TN);

    // ---- W.  Offsets from the wave's first row, which its rows do not take past 32 bits; rows past the edge repeat the last one.
    const int shift = SC == TWO_E4M3 ? 4 : 31 - __builtin_clz((unsigned)P.block);
    const int64_t first_row = (none ? 0 : e * P.N) + (n0 < P.N ? n0 : P.N - 1), more_rows = n0 < P.N ? P.N - 1 - n0 : 0;
    const uint8_t *const codes = P.codes + first_row * (P.K >> 1), *const scales = P.scales + first_row * (P.K >> shift);
    uint32_t code_at[TN], scale_at[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const uint32_t row = (uint32_t)(j * 16 + r < more_rows ? j * 16 + r : more_rows);
        code_at[j] = row * (uint32_t)(P.K >> 1);
        scale_at[j] = row * (uint32_t)(P.K >> shift);
    }
    auto load_w = [&](Codes<SC> (&c)[TN], int kt) {
        uint32_t k = (uint32_t)kt * 128 + q * 32;
        k = k < P.K ? k : 0;  // (past the end some codes of the row, which cut() clears)
#pragma unroll
        for (int j = 0; j < TN; ++j) c[j].load(codes + (code_at[j] + (k >> 1)), scales + (scale_at[j] + (k >> shift)), true);
    };
    auto cut = [&](Codes<SC> (&c)[TN], int kt) {
        if ((kt + 1) * 128 <= P.K) return;
        const bool there = kt * 128 + q * 32 < P.K;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) c[j].w[i] = there ? c[j].w[i] : 0;
            c[j].s = there ? c[j].s : 0;
        }
    };

    // ---- x.  Which row of it stands in row `row` of the tile, or a number below zero: rows past the end repeat the last one (what comes of them is not stored), rows that
    // an order does not name any of become zeros at the end.
    auto source = [&](int row) -> int64_t {
        row = row < rows ? row : rows - 1;
        if (!GROUPED || !P.order) return m0 + row;
        const int32_t pair = P.order[m0 + row];
        const int32_t from = pair < 0 ? -1 : pair / P.top_k;
        return from < P.x_rows ? from : -1;
    };
    auto row_of = [&](int row) {
        const int64_t from = source(row);
        return from < 0 ? 0 : from;
    };
    const bool some = !none && P.x_rows > 0;
    // direct loads: instruction i of a wave brings rows 4 (MT wave + i) .. + 3, a lane the piece that belongs at its place
    uint32_t off[DIRECT ? MT : 1];
    const int64_t base_row = GROUPED && P.order ? 0 : m0;
    const uint8_t *const base = P.x + base_row * P.ldx * XSZ;
    if (DIRECT && some) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int row = (wave * MT + i) * 4 + (lane >> 4);
            off[i] = (uint32_t)((row_of(row) - base_row) * P.ldx * 2) + (((lane & 15) ^ place(row)) << 4);
        }
    }
    // through registers: a thread brings piece tid % 16 of rows tid / 16 + 16 i
    const uint8_t *from[DIRECT ? 1 : MT];
    if (!DIRECT && some) {
#pragma unroll
        for (int i = 0; i < MT; ++i) from[i] = P.x + (row_of((tid >> 4) + 16 * i) * P.ldx + (tid & 15) * 8) * XSZ;
    }
    struct Piece8 {
        u32x4_t w[XDT == NVFP4_BF16 ? 1 : 2];
    };
    struct __attribute__((packed, aligned(XSZ))) Q { u32x4_t w; };
    auto fetch = [&](const uint8_t *row, int64_t k) {  // 8 elements of a row, zeros past K
        Piece8 s;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(s.w) / 16); ++i) s.w[i] = k + (tid & 15) * 8 < P.K ? reinterpret_cast<const Q *>(row + k * XSZ)[i].w : u32x4_t{0, 0, 0, 0};
        return s;
    };
    auto put = [&](int stage, int i, const Piece8 &s) {
        const int row = (tid >> 4) + 16 * i;
        uint8_t *const at = lds + stage * STG + row * 256 + (((tid & 15) ^ place(row)) << 4);
        if constexpr (XDT == NVFP4_BF16) {
            *reinterpret_cast<u32x4_t *>(at) = s.w[0];
        } else {
            Elems<XDT> x;
            x.w[0] = s.w[0];
            x.w[1] = s.w[1];
            bf16x8_t f[PIECES];
            x.part(0, f);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) *reinterpret_cast<bf16x8_t *>(at + p * (BM * 256)) = f[p];
        }
    };
    const int tiles = some ? (int)((P.K + 127) >> 7) : 0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    Piece8 held[DIRECT ? 1 : MT];
    // x of K tile kt into stage kt % 2: begun here, finished by end()
    auto begin = [&](int kt) {
        const int64_t k = (int64_t)kt * 128;
        if constexpr (DIRECT) {
            if (k + 128 <= P.K) {
#pragma unroll
                for (int i = 0; i < MT; ++i) load_lds(lds0 + (kt & 1) * STG + (wave * MT + i) * 1024, off[i], base + k * 2);
            } else {  // the last K tile, where it is not a whole one
#pragma unroll 1
                for (int i = 0; i < MT; ++i) put(kt & 1, i, fetch(P.x + (row_of((tid >> 4) + 16 * i) * P.ldx + (tid & 15) * 8) * XSZ, k));
            }
        } else {
#pragma unroll
            for (int i = 0; i < MT; ++i) held[i] = fetch(from[i], k);
        }
    };
    auto end = [&](int kt) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < MT; ++i) put(kt & 1, i, held[i]);
        }
        wait_loads();
        barrier();
    };

    float4v_t acc[MT][TN];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = float4v_t{0, 0, 0, 0};
    if (tiles > 0) {
        // 4 MT fragments of x a K tile, AHEAD of them on their way, TN products (of each piece) with each; the codes of the next quarter are expanded beside these
        constexpr int AHEAD = PIECES == 1 ? 3 : 1, RING = AHEAD + 1, FRAGS = 4 * MT;
        Codes<SC> a[TN], next[TN];
        load_w(a, 0);
        begin(0);
        end(0);
        cut(a, 0);
        for (int kt = 0; kt < tiles; ++kt) {
            const uint8_t *const stage = lds + (kt & 1) * STG + r * 256;
            if (kt + 1 < tiles) {
                load_w(next, kt + 1);
                begin(kt + 1);
            }
            bf16x8_t fa[2][TN], fb[RING][PIECES];
            auto read = [&](auto at) {
                constexpr int t = decltype(at)::value, p = t / MT, i = t % MT;
#pragma unroll
                for (int s = 0; s < PIECES; ++s) fb[t % RING][s] = *reinterpret_cast<const bf16x8_t *>(stage + s * (BM * 256) + i * 4096 + (((4 * q + p) ^ place(r)) << 4));
            };
            each<0, AHEAD>(read);
#pragma unroll
            for (int j = 0; j < TN; ++j) fa[0][j] = a[j].part(0);
            __builtin_amdgcn_sched_barrier(0);
            each<0, FRAGS>([&](auto step) {
                constexpr int t = decltype(step)::value, p = t / MT, i = t % MT;
                if constexpr (t + AHEAD < FRAGS) read(std::integral_constant<int, t + AHEAD>{});
#pragma unroll
                for (int s = 0; s < PIECES; ++s)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fa[p & 1][j], fb[t % RING][s], acc[i][j], 0, 0, 0);
                if constexpr (p < 3) {
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        if (j * MT / TN == i) fa[(p + 1) & 1][j] = a[j].part(p + 1);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
            if (kt + 1 < tiles) {
                end(kt + 1);
#pragma unroll
                for (int j = 0; j < TN; ++j) a[j] = next[j];
                cut(a, kt + 1);
            }
        }
    }
    // lane (q, r) has columns 4 q .. 4 q + 3 of row r
    const float g = P.g && !none ? P.g[e * P.g_step] : 1.0f;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int row = i * 16 + r;
        const bool zero = none || (GROUPED && P.order && row < rows && source(row) < 0);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + j * 16 + q * 4;
            if (row >= rows || n >= P.N) continue;
            float v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = zero ? 0.0f : acc[i][j][c] * g;
            const int64_t at = (m0 + row) * P.ldc + n;
            if (n + 4 <= P.N) {
                if (out_dt == NVFP4_BF16) {
                    struct __attribute__((packed, aligned(2))) H { uint32_t w[2]; } h;
                    const float2v_t lo = {v[0], v[1]}, hi = {v[2], v[3]};
                    h.w[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t));
                    h.w[1] = __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t));
                    *reinterpret_cast<H *>(P.out + at * 2) = h;
                } else {
                    store_run<NVFP4_F32, 4>(v, P.out + at * 4, 4);
                }
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (n + c < P.N) {
                        if (out_dt == NVFP4_BF16) Elem<NVFP4_BF16>::store(P.out + (at + c) * 2, v[c]);
                        else Elem<NVFP4_F32>::store(P.out + (at + c) * 4, v[c]);
                    }
            }
        }
    }
}

namespace w4 {

static int64_t tile_rows(const W4Args &P, int bm)
{
    return P.groups > 0 ? P.rows / bm + (P.rows < P.groups + 1 ? P.rows : P.groups + 1) : (P.rows + bm - 1) / bm;
}

template <int XDT, int SC, int MT, int TN, bool GROUPED, bool DIRECT>
static hipError_t run(W4Args P, int out_dt, hipStream_t st)
{
    constexpr int LDS = 2 * STAGE<MT, Elems<XDT>::PIECES>;
    auto *k = gemm_w4_tiles_kernel<XDT, SC, MT, TN, GROUPED, DIRECT>;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(k), hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
    if (once != hipSuccess) return once;
    P.slots = (uint32_t)tile_rows(P, 16 * MT);
    k<<<launch_grid((P.N + 64 * TN - 1) / (64 * TN) * P.slots), 256, LDS, st>>>(P, out_dt);
    return hipGetLastError();
}

template <int XDT, int SC, bool GROUPED, bool DIRECT>
static hipError_t by_tile(const W4Args &P, int out_dt, const W4Tile &t, hipStream_t st)
{
    auto with = [&](auto m, auto n) { return run<XDT, SC, decltype(m)::value, decltype(n)::value, GROUPED, DIRECT>(P, out_dt, st); };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    const integral_constant<int, 8> eight;
    if constexpr (XDT == NVFP4_F32) return t.cols16 == 1 ? with(two, one) : t.cols16 == 2 ? with(two, two) : with(two, four);
    else if constexpr (!DIRECT) return t.rows16 == 2 ? with(two, one) : t.cols16 == 1 ? with(four, one) : with(eight, two);
    else if (t.rows16 == 8) return t.cols16 == 4 ? with(eight, four) : t.cols16 == 2 ? with(eight, two) : with(eight, one);
    else return t.rows16 == 7 ? with(integral_constant<int, 7>{}, integral_constant<int, 3>{}) : t.rows16 == 4 ? with(four, one) : with(two, one);
}

template <int XDT, int SC>
static hipError_t by_form(const W4Args &P, int out_dt, const W4Tile &t, hipStream_t st)
{
    if constexpr (XDT == NVFP4_BF16) {
        if (w4_takes_direct(P, XDT)) return P.groups > 0 ? by_tile<XDT, SC, true, true>(P, out_dt, t, st) : by_tile<XDT, SC, false, true>(P, out_dt, t, st);
    }
    return P.groups > 0 ? by_tile<XDT, SC, true, false>(P, out_dt, t, st) : by_tile<XDT, SC, false, false>(P, out_dt, t, st);
}

// A K tile of a CU's only tile and of each more, us (NVFP4; that is less than the sum, since up to seven small tiles share a CU): bf16 x by direct loads, bf16 through registers,
// binary32.  us, 16 rows16 x 64 cols16 as 8,4 / 7,3 / 8,2 / 8,1 / 4,1 / 2,1: 4096 x 4096 x 4096 126 / 158 / 129 / 160 / 199 / 292, 777 x 12288 x 4096 128 / 94 / 108, 2000 x 2048 x 2048
// 45 / 37 / 28 / 23 / 30 / 47, 128 x 12288 x 4096 80 / 60 / 46 / 30 / 28 / 32, 300 x 2048 x 2048 43 / 32 / 24 / 16 / 12 / 13, 65 x 1024 x 4096 74 / 55 / 42 / 27 / 20 / 17; binary32 2,4 / 2,2 /
// 2,1: 777 x 12288 x 4096 307 / 329 / 446, 4096 x 4096 x 4096 477 / 524 / 713, 2000 x 2048 x 2048 68 / 82 / 114, 1280 x 1920 x 2048 63 / 59 / 76, 256 x 4096 x 11008 232 / 162 / 154,
// 64 x 12288 x 4096 97 / 66 / 59, 64 x 4096 x 4096 93 / 62 / 51.  MXFP4 takes up to 25 % less in each: of eleven sizes the tile chosen is the best one or within 10 % of it.
struct TileCost {
    W4Tile tile;
    double first, more;
};
constexpr TileCost DIRECT_TILES[] = {{{2, 1}, 0.42, 0.28}, {{4, 1}, 0.5, 0.3}, {{8, 1}, 0.82, 0.5}, {{8, 2}, 1.4, 0.88}, {{7, 3}, 1.75, 1.0}, {{8, 4}, 2.3, 1.45}};
constexpr TileCost STAGED_TILES[] = {{{2, 1}, 0.78, 0.3}, {{4, 1}, 1.1, 0.4}, {{8, 2}, 2.2, 1.1}};
constexpr TileCost F32_TILES[] = {{{2, 1}, 1.25, 0.68}, {{2, 2}, 1.95, 0.95}, {{2, 4}, 2.8, 1.7}};

template <int N>
static W4Tile cheapest(const W4Args &P, const TileCost (&of)[N])
{
    const int64_t cus = compute_units();
    W4Tile best = of[0].tile;
    double least = 1e30;
    for (const TileCost &c : of) {
        // (an expert's last tile of rows is half full on average)
        const int64_t bm = 16 * c.tile.rows16, bn = 64 * c.tile.cols16, rows = P.groups > 0 ? P.rows / bm + (P.groups + 1) / 2 : (P.rows + bm - 1) / bm;
        const int64_t a_cu = (rows * ((P.N + bn - 1) / bn) + cus - 1) / cus;
        const double cost = c.first + (double)(a_cu - 1) * c.more;
        if (cost < least) {
            least = cost;
            best = c.tile;
        }
    }
    return best;
}

}  // namespace w4

bool w4_takes_direct(const W4Args &P, int x_dt)
{
    const int64_t span = P.order ? P.x_rows : 16 * 8;  // (rows of a tile; with an order any row of x may be one)
    return x_dt == NVFP4_BF16 && reinterpret_cast<uintptr_t>(P.x) % 16 == 0 && P.ldx % 8 == 0 && P.ldx < ((int64_t)1 << 31) / (span > 0 ? span : 1);
}

// More rows than one fragment has, of experts on average.  us, the kernel for few rows / tiles: 16 x 4096 x 11008 19 / 55, 16 x 12288 x 4096 26 / 24, 33 x 4096 x 4096 (four fragments of rows) 21 / 20,
// 64 x 12288 x 4096 45 / 28, binary32 16 x 4096 x 11008 35 / 135, 64 x 12288 x 4096 93 / 59.  (Few columns and a long contraction lose by it: 17 x 4096 x 11008 58 where 16 rows take 18,
// since nothing divides a tile's contraction.)
bool w4_takes_tiles(const W4Args &P, int x_dt, W4Tile *t)
{
    using namespace w4;
    if ((P.groups > 0 ? P.rows / P.groups : P.rows) <= 16) return false;
    *t = x_dt == NVFP4_F32 ? cheapest(P, F32_TILES) : w4_takes_direct(P, x_dt) ? cheapest(P, DIRECT_TILES) : cheapest(P, STAGED_TILES);
    return true;
}

hipError_t launch_gemm_w4_tiles(const W4Args &P, int x_dt, int out_dt, const W4Tile &t, hipStream_t st)
{
    using namespace w4;
    if (x_dt == NVFP4_BF16)
        return P.scale == NVFP4_SCALE_E8M0 ? by_form<NVFP4_BF16, ONE_E8M0>(P, out_dt, t, st)
               : P.block == 16             ? by_form<NVFP4_BF16, TWO_E4M3>(P, out_dt, t, st)
                                           : by_form<NVFP4_BF16, ONE_E4M3>(P, out_dt, t, st);
    return P.scale == NVFP4_SCALE_E8M0 ? by_form<NVFP4_F32, ONE_E8M0>(P, out_dt, t, st)
           : P.block == 16             ? by_form<NVFP4_F32, TWO_E4M3>(P, out_dt, t, st)
                                       : by_form<NVFP4_F32, ONE_E4M3>(P, out_dt, t, st);
}

}  // namespace nvfp4
