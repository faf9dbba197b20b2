// Sums of a tile of 256 x 256 on the bfloat16 matrix instruction, from 8-bit blocks that are decoded, exactly, on their way into LDS:
//   out(i, j) = sum over r of A(i, r) B(r, j)
// for products whose sums are to be those of 32 bits, and for the gradients.
#pragma once

#include "pvq_fp8_tile.h"

namespace pvq_fp8_dev {

constexpr int kWideTile = 256, kWideStep = 64, kWideLds = 4 * kWideTile * kWideStep * 2;

enum wide_kind {
    WIDE_PRODUCT,        // A and B in blocks along the sum: A(i, r) = a[i][r], B(r, j) = b[j][r]
    WIDE_INPUT_GRAD,     // A(i, r) = dy[i][r], B(r, j) = b[r][j]; a term for each piece of each dY, one after the other
    WIDE_WEIGHT_GRAD,    // A(i, r) = dy[r][i], B(r, j) = b[r][j]; a term for each piece of an output's dY
};

// Tiles of 256 x 256, low ones of 128 x 256, or small ones of 64 x 64 (pvq_fp8_small.h), whichever take less: a step of a low tile is 64 matrix
// instructions less but the same codes to decode.
struct wide_tiles {
    int rows, cols, parts;
    double us;
};
inline wide_tiles wide_plan(int64_t rows, int64_t cols, int64_t depth, int terms, int outputs)
{
    const int64_t steps = (depth + kWideStep - 1) / kWideStep * terms, values = rows * cols * outputs;
    auto tiles = [&](int r, int c) { return (rows + r - 1) / r * ((cols + c - 1) / c) * outputs; };
    wide_tiles best{256, 256, 1, 0.0}, low{128, 256, 1, 0.0}, small{64, 64, 1, 0.0};
    best.parts = fp8_parts(tiles(256, 256), steps, kWideStepUs, values, &best.us);
    low.parts = fp8_parts(tiles(128, 256), steps, kLowStepUs, values, &low.us);
    small.parts = fp8_small_parts(tiles(64, 64), steps, values, false, &small.us);
    if (low.us < best.us) best = low;
    return small.us < best.us ? small : best;
}

struct wide_args {
    fp8_bf16 dy[4];                  // of the pairs, each in its pieces, all of one stride; how their rows lie: fp8_bf16
    fp8_blocks a, b[2];              // b: of the pairs; the gate's and the up weights
    fp8_matrix out[2];
    int64_t rows, cols, depth;       // of the output, and of the sum (one term's); GATED: cols are hidden units
    int terms, pieces;               // of the sum, and of a pair's dY
    int tiles_i, tiles_j;
    int parts, steps_a_part;         // of a split sum, whose parts go to work
    int units;                       // tiles of all parts of all outputs

    // these tiles of that many outputs
    void use(const wide_tiles &plan, int outputs)
    {
        parts = plan.parts;
        tiles_i = (int)((rows + plan.rows - 1) / plan.rows);
        tiles_j = (int)((cols + plan.cols - 1) / plan.cols);
        steps_a_part = (int)(((depth + kWideStep - 1) / kWideStep * terms + parts - 1) / parts);
        units = tiles_i * tiles_j * outputs * parts;
    }
    float *work;
};

// The term that a step belongs to (four at most; behind the last step whatever follows), and whose dY and whose blocks it takes.
template <int KIND>
__device__ inline int term_of(int step, int steps_a_term)
{
    if constexpr (KIND == WIDE_PRODUCT) return 0;
    return (step >= steps_a_term) + (step >= 2 * steps_a_term) + (step >= 3 * steps_a_term);
}
template <int KIND>
__device__ inline const fp8_bf16 &dy_of(const wide_args &t, int term, int out_of) { return t.dy[KIND == WIDE_INPUT_GRAD ? term : (out_of * t.pieces + term) & 3]; }
template <int KIND>
__device__ inline bool second_pair(const wide_args &t, int term, int out_of) { return KIND == WIDE_INPUT_GRAD ? term >= t.pieces : out_of != 0; }

// Where a step's part of an operand's tile starts, and how many bytes of the matrix are left there, the upper word below zero where none are: what
// lies behind is zero.  (Of 64 bits compared whole the vector unit does it, between matrix instructions.)
struct source {
    const uint8_t *p;
    uint32_t left;
    int32_t left_up;
};
__device__ inline source source_of(const void *base, int64_t row, int64_t rows, int64_t row_bytes, int64_t at)
{
    const int64_t left = (rows - 1) * row + row_bytes - at;
    return source{(const uint8_t *)base + at, (uint32_t)left, (int32_t)(left >> 32)};
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t take(source &s, uint32_t step)       // the buffer of a step, and on to the next, `step` bytes on
{
    asm("" : "+s"(s.left_up));
    const uint32_t left = s.left_up > 0 ? ~0u : s.left_up < 0 ? 0u : s.left;
    const auto r = __builtin_amdgcn_make_buffer_rsrc((void *)s.p, 0, left, 0x00020000);
    s.p += step;
    s.left_up -= s.left < step;
    s.left -= step;
    return r;
}

// A tile, or a part of its sum: steps first .. last of output out_of at i0, j0.
struct wide_unit {
    int64_t i0, j0;
    int out_of, part, first, last;
    __device__ int steps() const { return max(last - first + 1, 1); }       // (of none: one of zeros)
};

// The sums of a workgroup's units, t the kernel's first argument, and what becomes of each: done(unit, acc).  Four waves of 128 x 128, one to a SIMD, as for products on the 8-bit instruction
// (pvq_fp8_product.hip): LDS is written 64 KB and read 128 KB for 64 of the sum, 1500 of the 2048 cycles of matrix instructions.  Both operands come
// through registers, codes to be decoded once for the four waves, dY as it is.
//
// A step is 64 of the sum, two halves of 32.  While the first half's 64 instructions run, the second half's operands are read, which empties the
// stage; behind the step's barrier, while the second half's run, the next step's first operands are read from the other stage, then what was fetched
// a step ago is put into the empty one.  One operand's codes are decoded in the first half, the other's in the second, and either is fetched again as
// soon as its registers are free: a wave alone on its SIMD has about three instructions to issue beside each matrix instruction, and what does not fit
// holds the next one up (all of it in the second half: 478 us for dX of 2048 x 2 x 14336 x 4096, now 420; where the loads are, worked out in one place
// at the start of a step: 10 % more).
//
// GATED (WIDE_PRODUCT): the tile's 256 columns are 128 hidden units of the gate weights and the same of the up weights; a wave has both for its 64.
//
// A workgroup has units blockIdx.x, blockIdx.x + gridDim.x .. and goes from one to the next without a pause: three steps ahead of the products, its loads
// are the next unit's when one ends, and between two steps the sums are stored from where they are.  (GATED: one unit, and done may use LDS.)
// dW of 64 x 16384 x 4096, four tiles of one step to a workgroup, 38 us; with a workgroup to each tile, stored by way of LDS, 50; 576 tokens 85 and 97.
template <int KIND, bool GATED, int FI, typename UNIT, typename DONE>
__device__ __forceinline__ void wide_sums(const wide_args &t, uint8_t *lds, int units, UNIT unit_of, DONE done)
{
    constexpr int F = 8, kPlane = kWideTile * kWideStep * 2, kPieces = 8, kSlots = FI * F;       // LDS: A's two stages, B's two stages
    static_assert(FI == 8 || (FI == 4 && !GATED), "rows");
    constexpr bool A_ALONG = KIND != WIDE_WEIGHT_GRAD, B_ALONG = KIND == WIDE_PRODUCT, A_CODES = KIND == WIDE_PRODUCT;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wi = wave / 2, wj = wave % 2, r16 = lane % 16, quarter = lane / 16;
    const int steps_a_term = (int)((t.depth + kWideStep - 1) / kWideStep);

    // Strides in bytes (the same for all terms and outputs).  A lane's piece is eight values of a row; an operand whose rows run along the sum has eight
    // lanes to a row, one whose rows run across it 32 (A of 128 columns 16), and piece p is 32 or 8 (16) rows behind piece p - 1.
    const uint32_t a_row = A_CODES ? (uint32_t)t.a.code_row() : (uint32_t)t.dy[0].ld * 2, b_row = (uint32_t)t.b[0].code_row();
    const uint32_t ae_row = (uint32_t)t.a.exp_row(), be_row = (uint32_t)t.b[0].exp_row();
    constexpr int kALanes = 4 * FI;        // to a row of A that runs across the sum
    const uint32_t along_row = tid / 8, along_col = tid % 8 * 8, across_row = tid / 32, across_col = tid % 32 * 8, a_across_row = tid / kALanes, a_across_col = tid % kALanes * 8;
    const uint32_t a_at = (A_ALONG ? along_row * a_row + along_col * (A_CODES ? 1 : 2) : a_across_row * a_row + a_across_col * 2), a_next = (A_ALONG ? 32 : 256 / kALanes) * a_row;
    const uint32_t b_at = B_ALONG ? along_row * b_row + along_col : across_row * b_row + across_col, b_next = (B_ALONG ? 32 : 8) * b_row;
    const uint32_t be_at = B_ALONG ? along_row * be_row : across_row * be_row + across_col / kFp8Block, be_next = (B_ALONG ? 32 : 8) * be_row;
    const uint32_t ae_at = along_row * ae_row, ae_next = 32 * ae_row;

    u32x4 ra[FI];                    // (codes: the first two words, and the exponent)
    u32x2 rb[kPieces];
    uint32_t re[kPieces];
    bf16x8 decoded[kPieces];         // A's codes, or else B's, for the next half
    source a_src, b_src, u_src, ae_src, be_src, ue_src;
    auto stop = [&] { a_src.left_up = b_src.left_up = u_src.left_up = ae_src.left_up = be_src.left_up = ue_src.left_up = -1; };
    // where the loads are
    wide_unit ahead = unit_of(blockIdx.x);
    int ahead_u = blockIdx.x, step = ahead.first, ahead_left = 0;      // (steps to the end of the unit or of a term)
    auto start = [&] {                  // at the first step, and where another term begins
        const wide_args &t = argument<wide_args>();
        const int term = term_of<KIND>(step, steps_a_term);
        const bool second = second_pair<KIND>(t, term, ahead.out_of);
        const int64_t i0 = ahead.i0, j0 = ahead.j0;
        const int64_t r0 = (int64_t)(step - term * steps_a_term) * kWideStep;
        const fp8_blocks b = {second ? t.b[1].codes : t.b[0].codes, second ? t.b[1].exps : t.b[0].exps, 0, 0};
        if constexpr (A_CODES) {
            a_src = source_of(t.a.codes, a_row, t.rows, a_row, i0 * a_row + r0);
            ae_src = source_of(t.a.exps, ae_row, t.rows, ae_row, i0 * ae_row + step / 2);
        } else {
            // (dY's last row to the end of its last 16 bytes: a load that is not whole would bring nothing)
            const int64_t row_end = ((A_ALONG ? (t.depth + kWideStep - 1) / kWideStep * kWideStep : t.rows) * 2 + 15) / 16 * 16;
            const uint16_t *y = dy_of<KIND>(t, term, ahead.out_of).data;
            a_src = A_ALONG ? source_of(y, a_row, t.rows, row_end, i0 * a_row + r0 * 2) : source_of(y, a_row, t.depth, row_end, r0 * a_row + i0 * 2);
        }
        if constexpr (B_ALONG) {
            b_src = source_of(t.b[0].codes, b_row, t.cols, b_row, j0 * b_row + r0);
            be_src = source_of(t.b[0].exps, be_row, t.cols, be_row, j0 * be_row + step / 2);
            u_src = GATED ? source_of(t.b[1].codes, b_row, t.cols, b_row, j0 * b_row + r0) : b_src;
            ue_src = GATED ? source_of(t.b[1].exps, be_row, t.cols, be_row, j0 * be_row + step / 2) : be_src;
        } else {
            b_src = source_of(b.codes, b_row, t.depth, b_row, r0 * b_row + j0);
            be_src = source_of(b.exps, be_row, t.depth, be_row, r0 * be_row + j0 / kFp8Block);
        }
        if (step > ahead.last) stop();
        ahead_left = max((KIND == WIDE_PRODUCT ? ahead.last + 1 : min((term + 1) * steps_a_term, ahead.last + 1)) - step, 1);
    };
    __amdgpu_buffer_rsrc_t a_from, b_from, u_from, ae_from, be_from, ue_from;
    // (rows along the sum: an exponent is that of two steps)
    const uint32_t a_step = A_CODES ? kWideStep : A_ALONG ? kWideStep * 2 : kWideStep * a_row, b_step = B_ALONG ? kWideStep : kWideStep * b_row;
    auto aim_a = [&](int what) {
        if (what == 0) a_from = take(a_src, a_step);
        if (what == 1 && A_CODES) ae_from = take(ae_src, step & 1);
    };
    auto aim_b = [&](int what) {
        if (what == 0) b_from = take(b_src, b_step);
        if (what == 1) be_from = take(be_src, B_ALONG ? step & 1 : kWideStep * be_row);
        if (what == 2 && GATED) u_from = take(u_src, b_step);
        if (what == 3 && GATED) ue_from = take(ue_src, step & 1);
    };
    auto go_on = [&](int steps) {                 // behind so many; on to the next term or unit; behind the last unit there are steps of zeros
        ahead_left -= steps;
        if (ahead_left) return;
        if (step > ahead.last) {
            ahead_u += gridDim.x;
            if (GATED || ahead_u >= units) {
                stop();
                ahead_left = 1 << 30;
                return;
            }
            ahead = unit_of(ahead_u);
            step = ahead.first;
        }
        start();
    };
    auto fetch_a = [&](int p) {
        if constexpr (A_CODES) {
            const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(a_from, a_at, p * a_next, 0));
            ra[p][0] = w[0]; ra[p][1] = w[1];
            ra[p][2] = __builtin_amdgcn_raw_buffer_load_b8(ae_from, ae_at, p * ae_next, 0);
        } else ra[p] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(a_from, a_at, p * a_next, 0));
    };
    auto fetch_b = [&](int p) {
        const bool up = GATED && p >= kPieces / 2;
        const int in = up ? p - kPieces / 2 : p;
        rb[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(up ? u_from : b_from, b_at, in * b_next, 0));
        re[p] = __builtin_amdgcn_raw_buffer_load_b8(up ? ue_from : be_from, be_at, in * be_next, 0);
    };

    // Rows across the sum lie in LDS as in memory, [r][256 columns] (or 128), in pieces of sixteen columns; the transposing read gives a lane four neighbouring r
    // of one column.  Piece c of row r lies at place c ^ f(r), f = r % 4 + 4 (r / 8 % 2): the eight rows that 32 lanes read at once lie in different
    // banks.  Rows along the sum: [row][64 r], chunk c (eight r) of row i at place c ^ (i / 2 % 8).
    const uint32_t across_to = across_row * 512 + (((across_col / 16) ^ (across_row & 3)) << 5) + across_col % 16 * 2, across_odd = across_to ^ (4 << 5);
    const uint32_t along_to = along_row * 128 + (((along_col / 8) ^ (along_row / 2 & 7)) << 4);
    const uint32_t a_across_to = a_across_row * kALanes * 16 + (((a_across_col / 16) ^ (a_across_row & 3) ^ (FI == 4 ? a_across_row / 8 * 4 : 0)) << 5) + a_across_col % 16 * 2;
    auto place_a = [&](int p) { return p * 4096 + (A_ALONG ? along_to : FI == 8 && p & 1 ? a_across_to ^ (4 << 5) : a_across_to); };
    auto place_b = [&](int p) { return p * 4096 + (B_ALONG ? along_to : p & 1 ? across_odd : across_to); };
    auto decode = [&](int p) {
        if constexpr (A_CODES) decoded[p] = bf16x8_of_codes(ra[p][0], ra[p][1], scale_of(ra[p][2]));
        else decoded[p] = bf16x8_of_codes(rb[p][0], rb[p][1], scale_of(re[p]));
    };
    auto put_a = [&](uint32_t stage, int p) {
        uint8_t *to = lds + stage + place_a(p);
        if constexpr (A_CODES) *reinterpret_cast<bf16x8 *>(to) = decoded[p];
        else *reinterpret_cast<u32x4 *>(to) = ra[p];
    };
    auto put_b = [&](uint32_t stage, int p) {
        bf16x8 *to = reinterpret_cast<bf16x8 *>(lds + stage + 2 * kPlane + place_b(p));
        if constexpr (A_CODES) *to = bf16x8_of_codes(rb[p][0], rb[p][1], scale_of(re[p]));
        else *to = decoded[p];
    };
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t sub = lane % 16, f = sub / 4 | (quarter & 1) << 2, row_of = 8 * quarter + sub / 4;
    auto read_across = [&](uint32_t plane, int row_bytes, int column, int h) {       // sixteen columns from 16 * column on
        const uint8_t *from = lds + plane + h * 32 * row_bytes + (column / 8) * 256 + (((column % 8) ^ f) << 5) + row_of * row_bytes + (sub % 4) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * row_bytes));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_along = [&](uint32_t plane, int row, int h) {           // sixteen rows from `row` on
        return *reinterpret_cast<const bf16x8 *>(lds + plane + (row + r16) * 128 + (((4 * h + quarter) ^ (r16 >> 1)) << 4));
    };
    auto read_a = [&](uint32_t stage, int i, int h) { return A_ALONG ? read_along(stage, (wi * FI + i) * 16, h) : read_across(stage, kALanes * 16, wi * FI + i, h); };
    auto read_b = [&](uint32_t stage, int j, int h) {
        return B_ALONG ? read_along(stage + 2 * kPlane, GATED ? (j / 4) * 128 + wj * 64 + (j % 4) * 16 : wj * 128 + j * 16, h) : read_across(stage + 2 * kPlane, 512, wj * 8 + j, h);
    };

    f32x4 acc[FI][F];
    bf16x8 a_op[2][FI], b_op[2][F];

    auto fetch_all = [&] {
#pragma unroll
        for (int i = 0; i < 4; i++) { aim_a(i); aim_b(i); }
        step++;
        go_on(1);
#pragma unroll
        for (int p = 0; p < kPieces; p++) {
            if (p < FI) fetch_a(p);
            fetch_b(p);
        }
    };
    // the reads of a half's operands behind its predecessor's first 32 instructions
    auto read_behind = [&](uint32_t stage, int slot, int h) {
        if (slot % 2 == 0 && slot / 2 < F) b_op[h][slot / 2] = read_b(stage, slot / 2, h);
        if (slot % 2 == 0 && slot / 2 >= F && slot / 2 < F + FI) a_op[h][slot / 2 - F] = read_a(stage, slot / 2 - F, h);
    };
    // which piece's turn it is behind an instruction: the first one's behind `from`, the next `every` on
    auto piece_of = [](int slot, int from, int every, int pieces) { return slot >= from && (slot - from) % every == 0 && (slot - from) / every < pieces ? (slot - from) / every : -1; };
    wide_unit now = ahead;
    int u = blockIdx.x, left = now.steps();
    start();
    {
        // (the second step's on its way while the first is waited for)
        u32x4 a[2][FI];
        u32x2 b[2][kPieces];
        uint32_t e[2][kPieces];
#pragma unroll
        for (int s = 0; s < 2; s++) {
            fetch_all();
#pragma unroll
            for (int p = 0; p < FI; p++) a[s][p] = ra[p];
#pragma unroll
            for (int p = 0; p < kPieces; p++) { b[s][p] = rb[p]; e[s][p] = re[p]; }
        }
#pragma unroll
        for (int s = 0; s < 2; s++) {
#pragma unroll
            for (int p = 0; p < FI; p++) ra[p] = a[s][p];
#pragma unroll
            for (int p = 0; p < kPieces; p++) { rb[p] = b[s][p]; re[p] = e[s][p]; }
#pragma unroll
            for (int p = 0; p < kPieces; p++) {
                if (!A_CODES || p < FI) decode(p);
                if (p < FI) put_a(s * kPlane, p);
                put_b(s * kPlane, p);
            }
        }
    }
    fetch_all();
    all_reads();
    barrier();
#pragma unroll
    for (int j = 0; j < F; j++) b_op[0][j] = read_b(0, j, 0);
#pragma unroll
    for (int i = 0; i < FI; i++) a_op[0][i] = read_a(0, i, 0);
    no_sums(acc);
    // (stages by the offset of their planes, 0 or kPlane: one body for all steps, whose sums stay where they are)
    // In runs without a condition, until either the products or the loads come to an end of theirs.
    uint32_t stage = 0;
    for (;;) {
        const int run = min(left, ahead_left);
        int more = run;
        do {
#pragma unroll
            for (int i = 0; i < FI; i++)
#pragma unroll
                for (int j = 0; j < F; j++) {
                    multiply_accumulated(acc[i][j], b_op[0][j], a_op[0][i]);
                    const int slot = i * F + j;
                    read_behind(stage, slot, 1);
                    const int aim = piece_of(slot, FI == 8 ? 5 : 1, FI == 8 ? 8 : 4, GATED ? 4 : 2);
                    if (aim >= 0) {
                        if (A_CODES) aim_a(aim);
                        else aim_b(aim);
                    }
                    const int piece = piece_of(slot, FI == 8 ? 33 : 17, FI == 8 ? 4 : 2, A_CODES ? FI : kPieces);
                    if (piece >= 0) {
                        decode(piece);
                        if (A_CODES) fetch_a(piece);
                        else fetch_b(piece);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            all_reads();
            barrier();
#pragma unroll
            for (int i = 0; i < FI; i++)
#pragma unroll
                for (int j = 0; j < F; j++) {
                    multiply_accumulated(acc[i][j], b_op[1][j], a_op[1][i]);
                    const int slot = i * F + j;
                    read_behind(stage ^ kPlane, slot, 0);
                    const int aim = piece_of(slot, FI == 8 ? 5 : 1, FI == 8 ? 8 : 4, GATED ? 4 : 2);        // (before the fetches below)
                    if (aim >= 0) {
                        if (A_CODES) aim_b(aim);
                        else aim_a(aim);
                    }
                    if (slot == 31) step++;
                    const int piece = piece_of(slot, FI == 8 ? 33 : 25, FI == 8 ? 4 : 2, FI), piece_b = piece_of(slot, FI == 8 ? 35 : 9, FI == 8 ? 4 : 2, kPieces);
                    if (piece >= 0) {
                        put_a(stage, piece);
                        if (!A_CODES) fetch_a(piece);
                    }
                    if (piece_b >= 0) {
                        put_b(stage, piece_b);
                        if (A_CODES) fetch_b(piece_b);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            stage ^= kPlane;
        } while (--more);
        go_on(run);
        left -= run;
        if (left) continue;
        if constexpr (GATED) break;
        sums_are_there();
        done(now, acc);
        u += gridDim.x;
        if (u >= units) break;
        now = unit_of(u);
        left = now.steps();
        no_sums(acc);
    }
    all_reads();
    if constexpr (GATED) {
        sums_are_there();
        done(now, acc);
    }
}

// Unit u of `tiles` tiles, in each of the outputs' parts one after the other.
template <bool GATED, int FI>
__device__ inline wide_unit wide_unit_of(const wide_args &t, int u)
{
    const int tiles = t.tiles_i * t.tiles_j, of = u / tiles, steps = (int)((t.depth + kWideStep - 1) / kWideStep) * t.terms;
    int ti, tj;
    tile_of(t.tiles_i, t.tiles_j, chiplet_order(u % tiles, tiles), ti, tj);
    const int part = of % t.parts, first = part * t.steps_a_part;
    return {(int64_t)ti * 32 * FI, (int64_t)tj * (GATED ? kWideTile / 2 : kWideTile), of / t.parts, part, first, min(first + t.steps_a_part, steps) - 1};
}

}  // namespace pvq_fp8_dev
