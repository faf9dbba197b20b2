// Products of 8-bit block matrices in tiles: Y = A B^T, and the gated block H = act(X Wg^T) * (X Wu^T).
#include "pvq_fp8_tile.h"

#include <type_traits>

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

// A tile row is a block of codes, 128 bytes in eight chunks; chunk c of row r lies at place c ^ (r / 2 % 8), so that
// what sixteen lanes read at one chunk number of sixteen rows lies in all 64 banks.
__device__ inline uint32_t chunk_at(uint32_t row, uint32_t chunk) { return row * kFp8Block + ((chunk ^ (row >> 1 & 7)) << 4); }

__device__ inline i32x8 read_operand(const uint8_t *tile, uint32_t row, uint32_t quarter)
{
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, quarter)), hi = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, 4 + quarter));
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
    int vec;                     // what y's rows are aligned to: 8 values, 4 or 1
};

// The tile's sums, or what the gated block makes of them, to memory.  A lane has four neighbouring columns of one row: columns 4 quarter .. of
// a fragment, row lane % 16.
// ACCUMULATION: the sums are in accumulation registers.
template <int TM, int TN, int WM, int WN, bool GATED, bool ACCUMULATION>
__device__ inline void store_tile(const tile_args &t, uint8_t *lds, f32x4 (&acc)[TM / WM / 16][TN / WN / 16], int tm, int tn, int part)
{
    constexpr int FM = TM / WM / 16, FN = TN / WN / 16, kCols = GATED ? TN / 2 : TN;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16;
    const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * kCols;
    const int64_t rows = t.a.rows;
    constexpr int FH = GATED ? FN / 2 : FN;           // the fragments of a row of results
    fp8_matrix y = t.y;
    if (!GATED && t.parts > 1) y = fp8_matrix{t.work + (int64_t)part * rows * t.n, PVQ_F32, t.n};
    const int64_t col0 = n0 + wn * FH * 16;
    // (what the gated block makes is formed where it is wanted, twice for blocks: all of it at once would not fit beside the sums)
    auto sum = [&](int i, int j) {
        if constexpr (ACCUMULATION) return read_sums(acc[i][j]);
        else return acc[i][j];
    };
    auto result = [&](int i, int j) {
        f32x4 v = sum(i, j);
        if constexpr (GATED) {
            const f32x4 u = sum(i, j + FH);
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = act_value(t.act, v[e]) * u[e];
        }
        return v;
    };
    const int vec = !GATED && t.parts > 1 ? (t.n % 8 == 0 ? 8 : t.n % 4 == 0 ? 4 : 1) : t.vec;
    if (y.data) store_fragments<FM, FH>(y, vec, rows, t.n, m0 + wm * FM * 16, col0, result);
    if constexpr (GATED) {
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
            to_blocks(0, t.gc, t.ge, sum);
            to_blocks(1, t.uc, t.ue, [&](int i, int j) { return sum(i, j + FH); });
            to_blocks(2, t.hc, t.he, result);
        }
    }
}

// TM x TN tiles, WM x WN waves.  GATED: the tile's TN columns are TN / 2 hidden units of the gate weights and the same of the up
// weights, and a wave has both for its units.  WIDE: on the bfloat16 instruction.
//
// Two stages of LDS, each a block of 128 of the tile's rows of A and B.  The waves are two groups, one of each on every SIMD, half
// a step apart: while one reads its operands of a block from LDS, all of them, the other's matrix instructions run, and they
// change places at a barrier.  (2048 x 28672 x 8192, gated, on the 8-bit instruction: 787 us; all eight in step, which read at the same time
// and multiply at the same time, 1155.)  A block's loads are under way for two such halves.
template <int TM, int TN, int WM, int WN, bool GATED, bool WIDE>
__global__ __launch_bounds__(WM *WN *kWave) void tile_kernel(tile_args t)
{
    constexpr int kWaves = WM * WN, FM = TM / WM / 16, FN = TN / WN / 16, kStage = (TM + TN) * kFp8Block;
    constexpr int kCols = GATED ? TN / 2 : TN;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / WN, wn = wave % WN, r16 = lane % 16, quarter = lane / 16, group = wave / (kWaves / 2);
    int tm, tn;
    tile_of(t.tiles_m, t.tiles_n, chiplet_order(blockIdx.x, gridDim.x), tm, tn);
    const int64_t m0 = (int64_t)tm * TM, n0 = (int64_t)tn * kCols;
    const int part = blockIdx.y;
    const int kb0 = part * t.blocks_a_part, kb1 = min(kb0 + t.blocks_a_part, (int)t.a.blocks());
    const uint32_t row_bytes = (uint32_t)t.a.code_row(), exp_row = (uint32_t)t.a.exp_row();

    // rows past the end are the last row once more, whose results nobody stores
    const int64_t m_last = t.a.rows - 1 - m0, n_last = t.n - 1 - n0;
    // wave-loads of eight rows: first A's, then B's, dealt out over the waves
    constexpr int kLoads = (TM + TN) / 8 / kWaves;
    static_assert((TM / 8) % kWaves == 0 && (kCols / 8) % kWaves == 0, "whole loads");
    uint32_t offset[kLoads];
    const uint8_t *base[kLoads];
    const uint32_t in_row = lane / 8, chunk = ((lane % 8) ^ ((wave * 8 + in_row) >> 1 & 7)) << 4;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int first = i * kWaves * 8;                                      // where this load's rows of all waves begin
        const int tile_row = first + wave * 8 + in_row;
        if (first < TM) {
            base[i] = t.a.codes + m0 * row_bytes;
            offset[i] = (uint32_t)min((int64_t)tile_row, m_last) * row_bytes + chunk;
        } else {
            const bool up = first >= TM + kCols;
            base[i] = (up ? t.up.codes : t.b.codes) + n0 * row_bytes;
            offset[i] = (uint32_t)min((int64_t)(tile_row - TM - (up ? kCols : 0)), n_last) * row_bytes + chunk;
        }
    }
    // exponents, a word of four blocks for each of the tile's rows, by the first waves, 64 rows each
    constexpr int kExpBytes = (TM + TN) * 4, kExpWaves = (TM + TN) / kWave;
    static_assert(kExpWaves <= kWaves && TM % kWave == 0 && kCols % kWave == 0, "whole waves");
    const int exp_first = wave * kWave;
    const bool exp_a = exp_first < TM, exp_up = exp_first >= TM + kCols;
    const uint8_t *exp_base = exp_a ? t.a.exps + m0 * exp_row : (exp_up ? t.up.exps : t.b.exps) + n0 * exp_row;
    const uint32_t exp_offset = (uint32_t)min((int64_t)(exp_first + lane - (exp_a ? 0 : exp_up ? TM + kCols : TM)), exp_a ? m_last : n_last) * exp_row;

    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    // one of the wave's loads of a block, its exponents with the first.  Past the last block it is the last once more, to a place
    // that nobody reads any more: no load is under a condition.  (A word of exponents is loaded with each of its four blocks.)
    auto load_piece = [&](int kb, int i) {
        const int from = min(kb, kb1 - 1);
        load_to_lds(base[i] + (int64_t)from * kFp8Block, offset[i], lds0 + ((kb - kb0) & 1) * kStage + (uint32_t)((i * kWaves + wave) * 8 * kFp8Block));
        if (i == 0 && (kExpWaves == kWaves || wave < kExpWaves))
            load_words_to_lds(exp_base + (from & ~3), exp_offset, lds0 + 2 * kStage + ((kb >> 2) & 1) * kExpBytes + wave * kWave * 4);
    };
    auto load_stage = [&](int kb) {
#pragma unroll
        for (int i = 0; i < kLoads; i++) load_piece(kb, i);
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    uint32_t a_exp[FM], b_exp[FN];
    i32x8 a_op[FM], b_op[FN];
    // the tile row of the lane's row of an operand of B
    auto b_row = [&](int j) { return GATED ? (j / (FN / 2)) * kCols + wn * FN * 8 + (j % (FN / 2)) * 16 + r16 : wn * FN * 16 + j * 16 + r16; };
    // (behind: what follows the reads of each operand of A)
    auto read_stage = [&](int kb, auto behind) {
        const uint8_t *at = lds + ((kb - kb0) & 1) * kStage, *bt = at + TM * kFp8Block;
#pragma unroll
        for (int j = 0; j < FN; j++) b_op[j] = read_operand(bt, b_row(j), quarter);
#pragma unroll
        for (int i = 0; i < FM; i++) {
            a_op[i] = read_operand(at, wm * FM * 16 + i * 16 + r16, quarter);
            behind(i);
        }
        if ((kb & 3) == 0 || kb == kb0) {
            const uint32_t *exps = reinterpret_cast<const uint32_t *>(lds + 2 * kStage + ((kb >> 2) & 1) * kExpBytes);
            const int shift = 8 * (kb & 3);
#pragma unroll
            for (int i = 0; i < FM; i++) a_exp[i] = exps[wm * FM * 16 + i * 16 + r16] >> shift;
#pragma unroll
            for (int j = 0; j < FN; j++) b_exp[j] = exps[TM + b_row(j)] >> shift;
        } else {
#pragma unroll
            for (int i = 0; i < FM; i++) a_exp[i] >>= 8;
#pragma unroll
            for (int j = 0; j < FN; j++) b_exp[j] >>= 8;
        }
    };
    // (behind: what follows the instructions of each operand of A)
    auto multiply = [&](auto behind) {
        __builtin_amdgcn_s_setprio(1);
        if constexpr (WIDE) {
#pragma unroll
            for (int h = 0; h < 4; h++) {
                bf16x8 bw[FN];
#pragma unroll
                for (int j = 0; j < FN; j++) bw[j] = bf16x8_of_codes((uint32_t)b_op[j][2 * h], (uint32_t)b_op[j][2 * h + 1], scale_of(b_exp[j] & 255u));
#pragma unroll
                for (int i = 0; i < FM; i++) {
                    const bf16x8 aw = bf16x8_of_codes((uint32_t)a_op[i][2 * h], (uint32_t)a_op[i][2 * h + 1], scale_of(a_exp[i] & 255u));
#pragma unroll
                    for (int j = 0; j < FN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[j], aw, acc[i][j], 0, 0, 0);
                    if ((h * FM + i) % 4 == 3) behind((h * FM + i) / 4);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < FM; i++) {
#pragma unroll
                for (int j = 0; j < FN; j++) acc[i][j] = multiply_codes(b_op[j], b_exp[j], a_op[i], a_exp[i], acc[i][j]);
                behind(i);
            }
        }
        // (no instructions: these keep the products on this side of what follows)
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) asm volatile("" : "+v"(acc[i][j]));
        __builtin_amdgcn_s_setprio(0);
    };
    // Loads are issued between the reads (the first group) and between the matrix instructions (the second): issued in a row they
    // hold up what the wave does next for as long as the address unit takes for all of them.
    auto piece_behind = [&](int kb, int pieces) {
        return [=, &load_piece](int i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < kLoads; k++)
                if (k * pieces / kLoads == i) load_piece(kb, k);
            __builtin_amdgcn_sched_barrier(0);
        };
    };
    auto nothing = [](int) {};

    if (kb0 < kb1) {
        load_stage(kb0);
        all_loads();
        barrier();
        if (group == 0) {
            // the stage of the next block is free for its loads: both groups have read what it held.  What this group loads is waited
            // for behind the instructions of this block, half a step before it is read.
            for (int kb = kb0; kb < kb1; kb++) {
                read_stage(kb, piece_behind(kb + 1, FM));
                all_reads();
                barrier();
                multiply(nothing);
                all_loads();
                barrier();
            }
            barrier();
        } else {
            load_stage(kb0 + 1);
            barrier();
            for (int kb = kb0; kb < kb1; kb++) {
                read_stage(kb, nothing);
                all_reads();
                all_loads();
                barrier();
                multiply(piece_behind(kb + 2, FM));
                barrier();
            }
            all_loads();
        }
    }

    store_tile<TM, TN, WM, WN, GATED, false>(t, lds, acc, tm, tn, part);
}

// Tiles of 256 x 256 on the 8-bit instruction by four waves of 128 x 128, one to a SIMD.  Of what bounds these products LDS comes first: a
// block of 128 of a tile is 64 KB that are written at 64 bytes a cycle and 256 KB / (waves' tile side / 64) that are read at 128, beside 2048
// cycles of matrix instructions.  Eight waves of 128 x 64 read 192 KB (2560 cycles in all), four of 128 x 128 128 KB (2048).
//
// A wave alone on its SIMD has nobody to fill in for it, so its own instructions are laid out: a block's products come in two
// halves, of the upper and the lower 64 rows of the wave's part of A, with a barrier in front of each.
//   first half   products of the upper rows; reads the lower rows' operands; loads B and the upper rows of the next block but one, whose
//                place everybody has read
//   second half  products of the lower rows; reads all of B (into a second set of registers) and the upper rows of the next block; loads
//                the lower rows of the next block but one
// Each load has a step and a half to arrive (with one barrier and a single step 1.6 us a step where operands come from beyond L2).
template <bool GATED>
__global__ __launch_bounds__(256) void big_tile_kernel(tile_args t)
{
    constexpr int kTile = 256, kWaves = 4, F = 8, H = F / 2, kCols = GATED ? kTile / 2 : kTile;
    constexpr int kPlane = kTile * kFp8Block;         // LDS: A's two stages, B's two stages, the words of exponents of two runs of four blocks
    constexpr int kExps = 4 * kPlane, kExpBytes = 2 * kTile * 4;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / 2, wn = wave % 2, r16 = lane % 16, quarter = lane / 16;
    int tm, tn;
    tile_of(t.tiles_m, t.tiles_n, chiplet_order(blockIdx.x, gridDim.x), tm, tn);
    const int64_t m0 = (int64_t)tm * kTile, n0 = (int64_t)tn * kCols;
    const int part = blockIdx.y;
    const int kb0 = part * t.blocks_a_part, kb1 = min(kb0 + t.blocks_a_part, (int)t.a.blocks());       // (kb0 a multiple of four)
    const uint32_t row_bytes = (uint32_t)t.a.code_row(), exp_row = (uint32_t)t.a.exp_row();

    // The tile's rows as buffers that end with the matrix: what rows past the end bring does not matter, their results are not stored.  A load
    // is eight rows, 1 KiB; load i of wave w is rows 32 i + 8 w ..: first A's, then B's (the gate's, the up weights').
    auto rows_of = [&](const uint8_t *plane, uint32_t row, int64_t first, int64_t rows, int most) {
        return make_buffer(plane + first * row, min(rows - first, (int64_t)most) * row);
    };
    const buffer_t a_codes = rows_of(t.a.codes, row_bytes, m0, t.a.rows, kTile), b_codes = rows_of(t.b.codes, row_bytes, n0, t.n, kCols);
    const buffer_t u_codes = GATED ? rows_of(t.up.codes, row_bytes, n0, t.n, kCols) : b_codes;
    const uint32_t in_row = lane / 8, chunk = ((lane % 8) ^ ((wave * 8 + in_row) >> 1 & 7)) << 4;
    const uint32_t offset = (wave * 8 + in_row) * row_bytes + chunk;
    // words of four exponents, 64 rows a load: rows 64 w .. of A, then of B
    const buffer_t a_exps = rows_of(t.a.exps, exp_row, m0, t.a.rows, kTile);
    const buffer_t b_exps = rows_of(GATED && wave >= 2 ? t.up.exps : t.b.exps, exp_row, n0, t.n, kCols);
    const uint32_t exp_offset = lane * exp_row;

    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    const uint32_t to0 = lds0 + wave * 8 * kFp8Block, exp_to0 = lds0 + kExps + wave * kWave * 4;
    // Past the last block it is the last once more, to a place that nobody reads any more: no load is under a condition, and each wait
    // knows how many were issued behind those that it waits for.
    auto load_rows = [&](int kb, bool b, int i) {      // rows 32 i + 8 w .. of A or of B
        const buffer_t codes = !b ? a_codes : GATED && i >= 4 ? u_codes : b_codes;
        load_to_lds(codes, offset, (uint32_t)min(kb, kb1 - 1) * kFp8Block + (b ? 32 * i % kCols : 32 * i) * row_bytes,
                    to0 + (b ? 2 : 0) * kPlane + (kb & 1) * kPlane + (uint32_t)(i * 32 * kFp8Block));
    };
    auto load_exps = [&](int kb, bool b) {             // the words of four blocks
        load_words_to_lds(b ? b_exps : a_exps, exp_offset, (uint32_t)(min(kb, kb1 - 1) & ~3) + (b ? wave % (kCols / kWave) : wave) * kWave * exp_row,
                          exp_to0 + ((kb >> 2) & 1) * kExpBytes + (b ? kExpBytes / 2 : 0));
    };
    constexpr int kFirst = 12, kSecond = 4;
    auto load_first = [&](int kb, int piece) {         // B and the upper rows of both halves of A
        if (piece < 8) load_rows(kb, true, piece);
        else if (piece < kFirst) load_rows(kb, false, (piece - 8) % 2 + (piece - 8) / 2 * 4);
    };
    auto load_second = [&](int kb, int piece) {
        if (piece < kSecond) load_rows(kb, false, 2 + piece % 2 + piece / 2 * 4);
    };

    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < F; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    i32x8 a_upper[H], a_lower[H], b_op[2][F];
    uint32_t a_exp[F], b_exp[F];
    auto b_row = [&](int j) { return GATED ? (j / H) * kCols + wn * 64 + (j % H) * 16 + r16 : wn * 128 + j * 16 + r16; };
    auto read_a = [&](int stage, int i) { return read_operand(lds + stage * kPlane, wm * 128 + i * 16 + r16, quarter); };
    auto read_b = [&](int stage, int j) { return read_operand(lds + (2 + stage) * kPlane, b_row(j), quarter); };

    // one block; AT: its number modulo four
    auto step = [&](auto AT, int kb) {
        constexpr int at = decltype(AT)::value, stage = at & 1;
        // the next four blocks' exponents come with the second of these: two loads more
        constexpr int kExpLoads = at == 1 ? 2 : 0, kBehind = kFirst + kSecond + kExpLoads;
        if constexpr (at == 0) {
            const uint32_t *exps = reinterpret_cast<const uint32_t *>(lds + kExps + ((kb >> 2) & 1) * kExpBytes);
#pragma unroll
            for (int i = 0; i < F; i++) a_exp[i] = exps[wm * 128 + i * 16 + r16];
#pragma unroll
            for (int j = 0; j < F; j++) b_exp[j] = exps[kTile + b_row(j)];
        }
#pragma unroll
        for (int i = 0; i < H; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated<at>(acc[i][j], b_op[stage][j], b_exp[j], a_upper[i], a_exp[i]);
                const int slot = i * F + j;
                if (slot % 2 == 0 && slot / 2 < H) a_lower[slot / 2] = read_a(stage, H + slot / 2);
                if (slot % 2 == 1) load_first(kb + 2, slot / 2);
                if (kExpLoads && (slot == 26 || slot == 28)) load_exps(kb + 3, slot == 28);
                __builtin_amdgcn_sched_barrier(0);
            }
        all_reads();
        loads_but<kBehind>();                    // B and the upper rows of the next block are there
        barrier();
#pragma unroll
        for (int i = 0; i < H; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated<at>(acc[H + i][j], b_op[stage][j], b_exp[j], a_lower[i], a_exp[H + i]);
                const int slot = i * F + j;
                if (slot < F) b_op[stage ^ 1][slot] = read_b(stage ^ 1, slot);
                else if (slot < F + H) a_upper[slot - F] = read_a(stage ^ 1, slot - F);
                if (slot % 2 == 1) load_second(kb + 2, slot / 2);
                __builtin_amdgcn_sched_barrier(0);
            }
        all_reads();
        loads_but<kBehind>();                    // the lower rows of the next block are there
        barrier();
    };

    if (kb0 < kb1) {
        load_exps(kb0, false);
        load_exps(kb0, true);
#pragma unroll
        for (int i = 0; i < kFirst; i++) load_first(kb0, i);
#pragma unroll
        for (int i = 0; i < kSecond; i++) load_second(kb0, i);
#pragma unroll
        for (int i = 0; i < kFirst; i++) load_first(kb0 + 1, i);
#pragma unroll
        for (int i = 0; i < kSecond; i++) load_second(kb0 + 1, i);
        loads_but<kFirst + kSecond>();
        barrier();
#pragma unroll
        for (int j = 0; j < F; j++) b_op[0][j] = read_b(0, j);
#pragma unroll
        for (int i = 0; i < H; i++) a_upper[i] = read_a(0, i);
        all_reads();
        barrier();
        int kb = kb0;
        for (; kb + 4 <= kb1; kb += 4) {
            step(std::integral_constant<int, 0>{}, kb);
            step(std::integral_constant<int, 1>{}, kb + 1);
            step(std::integral_constant<int, 2>{}, kb + 2);
            step(std::integral_constant<int, 3>{}, kb + 3);
        }
        if (kb < kb1) {
            step(std::integral_constant<int, 0>{}, kb);
            if (kb + 1 < kb1) step(std::integral_constant<int, 1>{}, kb + 1);
            if (kb + 2 < kb1) step(std::integral_constant<int, 2>{}, kb + 2);
        }
        all_loads();
    }
    sums_are_there();
    store_tile<kTile, kTile, 2, 2, GATED, true>(t, lds, acc, tm, tn, part);
}

template <bool GATED>
hipError_t launch_big_tile(tile_args &t, hipStream_t s)
{
    constexpr int kTile = 256, kLds = 2 * 2 * kTile * (kFp8Block + 4), kCols = GATED ? kTile / 2 : kTile;
    const auto kernel = &big_tile_kernel<GATED>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    t.tiles_m = (int)((t.a.rows + kTile - 1) / kTile);
    t.tiles_n = (int)((t.n + kCols - 1) / kCols);
    t.blocks_a_part = (int)((t.a.blocks() + t.parts - 1) / t.parts + 3) / 4 * 4;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_m * t.tiles_n), (unsigned)t.parts), dim3(256), kLds, s, t);
    return hipGetLastError();
}
template <int TM, int TN, int WM, int WN, bool GATED, bool WIDE>
hipError_t launch_tile(tile_args &t, hipStream_t s)
{
    constexpr int kLds = 2 * (TM + TN) * (kFp8Block + 4), kCols = GATED ? TN / 2 : TN;
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

}  // namespace

size_t fp8_product_work(int64_t, int64_t, int64_t, int) { return 0; }

hipError_t fp8_launch_product(const fp8_product_args &p, hipStream_t s)
{
    tile_args t{};
    t.a = p.a; t.b = p.b; t.y = p.y; t.work = p.work; t.n = p.b.rows; t.parts = 1;
    t.vec = row_alignment(p.y);
    const bool wide = p.y.dtype == PVQ_F32;
    if (wide) return launch_tile<256, 128, 4, 2, false, true>(t, s);
    return launch_big_tile<false>(t, s);
}

hipError_t fp8_launch_gated(const fp8_gated_args &g, hipStream_t s)
{
    tile_args t{};
    t.a = g.x; t.b = g.gate; t.up = g.up; t.y = g.h; t.act = g.act; t.n = g.gate.rows; t.parts = 1;
    t.hc = g.hc; t.he = g.he; t.gc = g.gc; t.ge = g.ge; t.uc = g.uc; t.ue = g.ue;
    t.vec = row_alignment(g.h);
    // Kept products are codes of sums of 32 bits: what the 8-bit instructions are off would change one code of 2000, which is as
    // much again as the roundings of the gradients to bfloat16 (dX 3.0e-3 off instead of 2.3e-3).
    if (g.gc || (g.h.data && g.h.dtype == PVQ_F32)) return launch_tile<128, 256, 2, 4, true, true>(t, s);
    return launch_big_tile<true>(t, s);
}
