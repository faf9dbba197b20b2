// Products of 8-bit block matrices in tiles: Y = A B^T, and the gated block H = act(X Wg^T) * (X Wu^T).
#include "pvq_fp8_dev.h"

using namespace pvq_fp8_dev;

namespace {

// ---- matrix instructions ---------------------------------------------------------------------------------------------
// A lane holds 32 codes of one row (lane % 16) of an operand: those of quarter lane / 16 of a block of 128.  Which codes of
// the block a quarter is does not matter, as long as both operands agree.  The result's rows are the first operand's.

// 8-bit instruction: 16 x 16 x 128 with both scales multiplied in.  Its adders align eight products at a time to the largest and
// keep about 14 bits below it, so that sums of Gaussian terms are 3.3e-5 of their size off: a sixtieth of bfloat16's rounding.
__device__ inline f32x4 multiply_codes(i32x8 a, uint32_t ea, i32x8 b, uint32_t eb, f32x4 c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, (int)ea, 0, (int)eb);
}

// bfloat16 instruction: four of 16 x 16 x 32 on the decoded values, which are exact; sums rounded as float32 sums are.
struct wide_codes { bf16x8 part[4]; };
__device__ inline wide_codes widen(i32x8 a, uint32_t e)
{
    wide_codes w;
    const float scale = scale_of(e & 255u);
#pragma unroll
    for (int i = 0; i < 4; i++) w.part[i] = bf16x8_of_codes((uint32_t)a[2 * i], (uint32_t)a[2 * i + 1], scale);
    return w;
}
__device__ inline f32x4 multiply_wide(const wide_codes &a, const wide_codes &b, f32x4 c)
{
#pragma unroll
    for (int i = 0; i < 4; i++) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.part[i], b.part[i], c, 0, 0, 0);
    return c;
}

// ---- loads into LDS --------------------------------------------------------------------------------------------------
// 1 KiB a wave: lane i's 16 bytes from `base` + `offset` to `lds` + 16 i.  The compiler does not count these loads: they are
// waited for by hand (all_loads) in front of the barrier behind which they are read.
__device__ inline void load_to_lds(const void *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ inline void all_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// A tile row is a block of codes, 128 bytes in eight chunks; chunk c of row r lies at place c ^ (r % 8), so that the
// sixteen rows that an instruction's operand takes at one chunk number lie in all banks.
__device__ inline uint32_t chunk_at(uint32_t row, uint32_t chunk) { return row * kFp8Block + ((chunk ^ (row & 7)) << 4); }

__device__ inline i32x8 read_operand(const uint8_t *tile, uint32_t row, uint32_t quarter)
{
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, 2 * quarter)), hi = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, 2 * quarter + 1));
    return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

struct tile_args {
    fp8_blocks a, b, up;         // up: the gated block's second weights
    fp8_matrix y;                // (data null: the gated block's result goes to hc, he)
    float *work;                 // split: the parts' sums
    int act;
    uint8_t *hc, *he, *gc, *ge, *uc, *ue;
    int64_t n;
    int tiles_m, tiles_n, parts, blocks_a_part;
    bool vec;
};

// Tiles of the result in bands of 8 rows of tiles, down a band's columns one after the other: the workgroups of a chiplet
// at work at one time share few rows of A and B in its L2.
__device__ inline void tile_of(const tile_args &t, int id, int &tm, int &tn)
{
    constexpr int kBand = 8;
    const int per = kBand * t.tiles_n, band = id / per, rows = min(kBand, t.tiles_m - band * kBand), in = id - band * per;
    // (in scalar registers, as are the addresses that follow from them)
    tm = __builtin_amdgcn_readfirstlane(band * kBand + in % rows);
    tn = __builtin_amdgcn_readfirstlane(in / rows);
}

// TM x TN tiles, WM x WN waves.  GATED: the tile's TN columns are TN / 2 hidden units of the gate weights and the same of the up
// weights, and a wave has both for its units.  WIDE: on the bfloat16 instruction.
template <int TM, int TN, int WM, int WN, bool GATED, bool WIDE>
__global__ __launch_bounds__(WM *WN *kWave) void tile_kernel(tile_args t)
{
    constexpr int kWaves = WM * WN, FM = TM / WM / 16, FN = TN / WN / 16, kStage = (TM + TN) * kFp8Block;
    constexpr int kCols = GATED ? TN / 2 : TN;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16;
    int tm, tn;
    tile_of(t, chiplet_order(blockIdx.x, gridDim.x), tm, tn);
    const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * kCols;
    const int part = blockIdx.y;
    const int kb0 = part * t.blocks_a_part, kb1 = min(kb0 + t.blocks_a_part, (int)t.a.blocks());
    const uint32_t row_bytes = (uint32_t)t.a.code_row();

    // rows past the end are the last row once more, whose results nobody stores
    const int64_t m_last = t.a.rows - 1 - m0, n_last = t.n - 1 - n0;
    const uint8_t *a_base = t.a.codes + m0 * row_bytes, *b_base = t.b.codes + n0 * row_bytes, *u_base = GATED ? t.up.codes + n0 * row_bytes : nullptr;
    // wave-loads of eight rows: first A's, then B's, dealt out over the waves
    constexpr int kLoads = (TM + TN) / 8 / kWaves;
    static_assert((TM / 8) % kWaves == 0 && (TN / 8) % kWaves == 0, "whole loads");
    uint32_t offset[kLoads];
    const uint8_t *base[kLoads];
    const uint32_t in_row = lane / 8, chunk = ((lane % 8) ^ in_row) << 4;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int tile_row = (i * kWaves + wave) * 8;
        if (i < TM / 8 / kWaves) {
            base[i] = a_base;
            offset[i] = (uint32_t)min((int64_t)(tile_row + in_row), m_last) * row_bytes + chunk;
        } else {
            int row = tile_row - TM;
            const bool up = GATED && row >= kCols;
            if (up) row -= kCols;
            base[i] = up ? u_base : b_base;
            offset[i] = (uint32_t)min((int64_t)(row + in_row), n_last) * row_bytes + chunk;
        }
    }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    auto load_stage = [&](int kb, int stage) {
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            load_to_lds(base[i] + (int64_t)kb * kFp8Block, offset[i], lds0 + stage * kStage + (uint32_t)((i * kWaves + wave) * 8 * kFp8Block));
    };
    // exponents of the lane's operand rows, four blocks a word
    const uint32_t exp_row = (uint32_t)t.a.exp_row();
    uint32_t a_exp[FM], b_exp[FN];
    auto load_exps = [&](int kb) {
#pragma unroll
        for (int f = 0; f < FM; f++) {
            const int64_t row = min((int64_t)(wm * FM * 16 + f * 16 + r16), m_last);
            a_exp[f] = *reinterpret_cast<const uint32_t *>(t.a.exps + (m0 + row) * exp_row + (kb & ~3));
        }
#pragma unroll
        for (int f = 0; f < FN; f++) {
            const bool up = GATED && f >= FN / 2;
            const int col = GATED ? wn * FN * 8 + (f % (FN / 2)) * 16 + r16 : wn * FN * 16 + f * 16 + r16;
            const int64_t row = min((int64_t)col, n_last);
            b_exp[f] = *reinterpret_cast<const uint32_t *>((up ? t.up.exps : t.b.exps) + (n0 + row) * exp_row + (kb & ~3));
        }
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    if (kb0 < kb1) {
        load_stage(kb0, 0);
        load_exps(kb0);
    }
    for (int kb = kb0; kb < kb1; kb++) {
        const int stage = (kb - kb0) & 1;
        all_loads();
        __syncthreads();
        if (kb + 1 < kb1) load_stage(kb + 1, stage ^ 1);
        if ((kb & 3) == 0 && kb != kb0) load_exps(kb);
        const uint8_t *at = lds + stage * kStage, *bt = at + TM * kFp8Block;
        const int shift = 8 * (kb & 3);
        if constexpr (WIDE) {
            wide_codes bw[FN];
#pragma unroll
            for (int j = 0; j < FN; j++) {
                const int row = GATED ? (j / (FN / 2)) * kCols + wn * FN * 8 + (j % (FN / 2)) * 16 + r16 : wn * FN * 16 + j * 16 + r16;
                bw[j] = widen(read_operand(bt, row, quarter), b_exp[j] >> shift);
            }
#pragma unroll
            for (int i = 0; i < FM; i++) {
                const wide_codes aw = widen(read_operand(at, wm * FM * 16 + i * 16 + r16, quarter), a_exp[i] >> shift);
#pragma unroll
                for (int j = 0; j < FN; j++) acc[i][j] = multiply_wide(bw[j], aw, acc[i][j]);
            }
        } else {
            i32x8 bw[FN];
#pragma unroll
            for (int j = 0; j < FN; j++) {
                const int row = GATED ? (j / (FN / 2)) * kCols + wn * FN * 8 + (j % (FN / 2)) * 16 + r16 : wn * FN * 16 + j * 16 + r16;
                bw[j] = read_operand(bt, row, quarter);
            }
#pragma unroll
            for (int i = 0; i < FM; i++) {
                const i32x8 aw = read_operand(at, wm * FM * 16 + i * 16 + r16, quarter);
#pragma unroll
                for (int j = 0; j < FN; j++) acc[i][j] = multiply_codes(bw[j], b_exp[j] >> shift, aw, a_exp[i] >> shift, acc[i][j]);
            }
        }
    }

    // a lane has four neighbouring columns of one row: columns 4 quarter .. of a fragment, row lane % 16
    const int64_t rows = t.a.rows;
    if constexpr (!GATED) {
        fp8_matrix y = t.y;
        if (t.parts > 1) y = fp8_matrix{t.work + (int64_t)part * rows * t.n, PVQ_F32, t.n};
        const bool vec = t.parts > 1 ? t.n % 4 == 0 : t.vec;
#pragma unroll
        for (int i = 0; i < FM; i++) {
            const int64_t row = m0 + wm * FM * 16 + i * 16 + r16;
            if (row >= rows) continue;
#pragma unroll
            for (int j = 0; j < FN; j++) {
                const int64_t col = n0 + wn * FN * 16 + j * 16 + 4 * quarter;
                if (vec) store4<true>(y, row, col, t.n - col, acc[i][j]);
                else store4<false>(y, row, col, t.n - col, acc[i][j]);
            }
        }
    } else {
        constexpr int FH = FN / 2;
        f32x4 h[FM][FH];
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FH; j++)
#pragma unroll
                for (int e = 0; e < 4; e++) h[i][j][e] = act_value(t.act, acc[i][j][e]) * acc[i][j + FH][e];
        if (t.y.data) {
#pragma unroll
            for (int i = 0; i < FM; i++) {
                const int64_t row = m0 + wm * FM * 16 + i * 16 + r16;
                if (row >= rows) continue;
#pragma unroll
                for (int j = 0; j < FH; j++) {
                    const int64_t col = n0 + wn * FN * 8 + j * 16 + 4 * quarter;
                    if (t.vec) store4<true>(t.y, row, col, t.n - col, h[i][j]);
                    else store4<false>(t.y, row, col, t.n - col, h[i][j]);
                }
            }
        }
        // to blocks: the tile's hidden units are one block, of which the WN waves of a row of tiles hold a part each
        if constexpr (kCols == kFp8Block) {
            const int64_t code_row = (t.n + kFp8Block - 1) / kFp8Block * kFp8Block, out_exp_row = (code_row / kFp8Block + 3) / 4 * 4;
            uint32_t *tops = reinterpret_cast<uint32_t *>(lds);          // [what][row of the tile][WN]
            auto to_blocks = [&](int what, uint8_t *codes, uint8_t *exps, auto value) {
                if (!codes) return;
                __syncthreads();
#pragma unroll
                for (int i = 0; i < FM; i++) {
                    uint32_t top = 0;
#pragma unroll
                    for (int j = 0; j < FH; j++)
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            if (n0 + wn * FN * 8 + j * 16 + 4 * quarter + e < t.n) top = max(top, finite_bits(value(i, j)[e]));
                    top = max(top, (uint32_t)__shfl_xor((int)top, 16));
                    top = max(top, (uint32_t)__shfl_xor((int)top, 32));
                    if (quarter == 0) tops[(wm * FM * 16 + i * 16 + r16) * WN + wn] = top;
                }
                __syncthreads();
#pragma unroll
                for (int i = 0; i < FM; i++) {
                    const int in = wm * FM * 16 + i * 16 + r16;
                    const int64_t row = m0 + in;
                    uint32_t top = 0;
#pragma unroll
                    for (int w = 0; w < WN; w++) top = max(top, tops[in * WN + w]);
                    const uint32_t e = exponent_of(top);
                    const float inverse = scale_of(254 - e);
                    if (row >= rows) continue;
#pragma unroll
                    for (int j = 0; j < FH; j++) {
                        const int64_t col = n0 + wn * FN * 8 + j * 16 + 4 * quarter;
                        f32x4 v = value(i, j);
#pragma unroll
                        for (int q = 0; q < 4; q++) if (col + q >= t.n) v[q] = 0.0f;
                        *reinterpret_cast<uint32_t *>(codes + row * code_row + col) = codes4(v[0], v[1], v[2], v[3], inverse);
                    }
                    if (wn == 0 && quarter == 0) {
                        uint8_t *p = exps + row * out_exp_row;
                        p[tn] = (uint8_t)e;
                        if (tn == t.tiles_n - 1)
                            for (int64_t b = tn + 1; b < out_exp_row; b++) p[b] = 0;
                    }
                }
            };
            to_blocks(0, t.gc, t.ge, [&](int i, int j) { return acc[i][j]; });
            to_blocks(1, t.uc, t.ue, [&](int i, int j) { return acc[i][j + FH]; });
            to_blocks(2, t.hc, t.he, [&](int i, int j) { return h[i][j]; });
        }
    }
}

template <int TM, int TN, int WM, int WN, bool GATED, bool WIDE>
hipError_t launch_tile(tile_args &t, hipStream_t s)
{
    constexpr int kLds = 2 * (TM + TN) * kFp8Block, kCols = GATED ? TN / 2 : TN;
    const auto kernel = &tile_kernel<TM, TN, WM, WN, GATED, WIDE>;
    if (kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
    }
    t.tiles_m = (int)((t.a.rows + TM - 1) / TM);
    t.tiles_n = (int)((t.n + kCols - 1) / kCols);
    t.blocks_a_part = (int)((t.a.blocks() + t.parts - 1) / t.parts);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_m * t.tiles_n), (unsigned)t.parts), dim3(WM * WN * kWave), kLds, s, t);
    return hipGetLastError();
}

bool vector_rows(const fp8_matrix &y)
{
    const int size = y.dtype == PVQ_F32 ? 4 : 2;
    return (uintptr_t)y.data % (4 * size) == 0 && y.ld % 4 == 0;
}

}  // namespace

size_t fp8_product_work(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t fp8_launch_product(const fp8_product_args &p, hipStream_t s)
{
    tile_args t{};
    t.a = p.a; t.b = p.b; t.y = p.y; t.work = p.work; t.n = p.b.rows; t.parts = 1;
    t.vec = vector_rows(p.y);
    const bool wide = p.y.dtype == PVQ_F32;
    if (wide) return launch_tile<128, 128, 2, 2, false, true>(t, s);
    return launch_tile<128, 128, 2, 2, false, false>(t, s);
}

hipError_t fp8_launch_gated(const fp8_gated_args &g, hipStream_t s)
{
    tile_args t{};
    t.a = g.x; t.b = g.gate; t.up = g.up; t.y = g.h; t.act = g.act; t.n = g.gate.rows; t.parts = 1;
    t.hc = g.hc; t.he = g.he; t.gc = g.gc; t.ge = g.ge; t.uc = g.uc; t.ue = g.ue;
    t.vec = g.h.data && vector_rows(g.h);
    // Kept products are codes of sums of 32 bits: what the 8-bit instructions are off would change one code of 2000, which is as
    // much again as the roundings of the gradients to bfloat16 (dX 3.0e-3 off instead of 2.3e-3).
    if (g.gc || (g.h.data && g.h.dtype == PVQ_F32)) return launch_tile<128, 256, 2, 4, true, true>(t, s);
    return launch_tile<128, 256, 2, 4, true, false>(t, s);
}
