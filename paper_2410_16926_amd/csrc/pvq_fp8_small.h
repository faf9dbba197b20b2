// The sums of pvq_fp8_wide.h in tiles of 64 x 64, for matrices too small to fill the card with large ones.
#pragma once

#include "pvq_fp8_wide.h"

namespace pvq_fp8_dev {

constexpr int kSmallTile = 64, kSmallPlane = kSmallTile * kWideStep * 2, kSmallLds = 4 * kSmallPlane;

// Four waves of 32 x 32.  A step is 64 of the sum, and little but waiting and the instructions of one wave a SIMD: a thread's sixteen values of either operand
// are fetched four steps ahead (six or eight: longer to start, 2 to 8 % more), decoded and put into one of two stages; one barrier a step, 0.3 us alone on a unit, 0.21 of several
// that take turns (where a step starts worked out anew each time, 0.35 to 0.45).  64 x 1500 x 1500 10.5 us, in large tiles 23; the gated block of 64 x 1500 x 1500 with G and U
// kept 13 and 43; but it reads four times what large tiles do: 333 x 3001 x 11008 69 us, in tiles of 128 x 256 46.
// dY's rows may start anywhere: they are loaded as they lie, what is behind their end by elements.
template <int KIND, bool GATED>
__device__ __forceinline__ void small_sums(const wide_args &t, uint8_t *lds, const wide_unit &u, f32x4 (&acc)[2][2])
{
    constexpr bool A_ALONG = KIND != WIDE_WEIGHT_GRAD, B_ALONG = KIND == WIDE_PRODUCT, A_CODES = KIND == WIDE_PRODUCT;
    constexpr int kAhead = 4;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wi = wave / 2, wj = wave % 2, r16 = lane % 16, quarter = lane / 16;
    const int row = tid / 4, from = tid % 4 * 16;               // a thread's sixteen values of 64 x 64
    const int steps_a_term = (int)((t.depth + kWideStep - 1) / kWideStep);
    struct piece {
        u32x4 a[A_CODES ? 1 : 2], b;
        uint32_t ae, be;
    };
    // Strides in bytes, a thread's place in a step, and where the next step to be fetched starts
    const uint32_t a_row = A_CODES ? (uint32_t)t.a.code_row() : 0, ae_row = A_CODES ? (uint32_t)t.a.exp_row() : 0, b_row = (uint32_t)t.b[0].code_row(), be_row = (uint32_t)t.b[0].exp_row();
    const int b_in = GATED ? row % 32 : row;                    // GATED: the gate's 32 units, then the up weights'
    const uint32_t a_at = row * a_row + from, ae_at = row * ae_row, b_at = b_in * b_row + from, be_at = b_in * be_row;
    source a_src{}, ae_src{}, b_src{}, be_src{};
    const uint16_t *y = nullptr;
    int64_t y_left = 0;                                         // of dY's row (along) or rows (across) from a thread's own on
    const int64_t y_cols = u.i0 + from < t.rows ? t.rows - u.i0 - from : 0;
    int step = u.first, term_end = 0;
    auto start = [&] {
        const int term = term_of<KIND>(step, steps_a_term);
        const bool second = second_pair<KIND>(t, term, u.out_of);
        term_end = (term + 1) * steps_a_term;
        const int64_t r0 = (int64_t)(step - term * steps_a_term) * kWideStep;
        const fp8_blocks b = second || (GATED && wave >= 2) ? t.b[1] : t.b[0];
        if constexpr (A_CODES) {
            a_src = source_of(t.a.codes, a_row, t.rows, a_row, u.i0 * a_row + r0);
            ae_src = source_of(t.a.exps, ae_row, t.rows, ae_row, u.i0 * ae_row + r0 / kFp8Block);
        } else {
            y = dy_of<KIND>(t, term, u.out_of).data + ((A_ALONG ? u.i0 : r0) + row) * t.dy[0].ld + (A_ALONG ? r0 : u.i0) + from;
            y_left = A_ALONG ? (u.i0 + row < t.rows ? t.depth - r0 - from : 0) : t.depth - r0 - row;
        }
        b_src = B_ALONG ? source_of(b.codes, b_row, b.rows, b_row, u.j0 * b_row + r0) : source_of(b.codes, b_row, t.depth, b_row, r0 * b_row + u.j0);
        be_src = B_ALONG ? source_of(b.exps, be_row, b.rows, be_row, u.j0 * be_row + r0 / kFp8Block) : source_of(b.exps, be_row, t.depth, be_row, r0 * be_row + u.j0 / kFp8Block);
    };
    start();
    // the next step, zeros behind the unit's last
    auto fetch = [&](piece &p) {
        if (KIND != WIDE_PRODUCT && step == term_end) start();
        if (step > u.last) { a_src.left_up = ae_src.left_up = b_src.left_up = be_src.left_up = -1; y_left = 0; }
        auto codes = [&](source &c, source &e, uint32_t c_step, uint32_t e_step, uint32_t c_at, uint32_t e_at, u32x4 &w, uint32_t &byte) {
            w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(take(c, c_step), c_at, 0, 0));
            byte = __builtin_amdgcn_raw_buffer_load_b8(take(e, e_step), e_at, 0, 0);
        };
        if constexpr (A_CODES) codes(a_src, ae_src, kWideStep, step & 1, a_at, ae_at, p.a[0], p.ae);
        else {
            const int64_t count = A_ALONG ? y_left : y_left > 0 ? y_cols : 0;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                p.a[h] = u32x4{0, 0, 0, 0};
                if (count >= 8 * h + 8) p.a[h] = reinterpret_cast<const unaligned<u32x4, 2> *>(y + 8 * h)->v;
                else if (count > 8 * h) {
#pragma unroll
                    for (int e = 0; e < 7; e++)
                        if (8 * h + e < count) p.a[h][e / 2] |= (uint32_t)y[8 * h + e] << 16 * (e % 2);
                }
            }
            y += A_ALONG ? (int64_t)kWideStep : kWideStep * t.dy[0].ld;
            y_left -= kWideStep;
        }
        codes(b_src, be_src, B_ALONG ? kWideStep : kWideStep * b_row, B_ALONG ? step & 1 : kWideStep * be_row, b_at, be_at, p.b, p.be);
        step++;
    };
    // LDS: rows of 64 values.  Along the sum, chunk c (eight values) of row r lies at place c ^ (r / 2 % 8); across it, piece c (sixteen) at place
    // c ^ (r / 2 % 2 + 2 (r / 8 % 2)): what lanes read at one time lies in different banks.
    auto across_place = [](int r, int c) { return r * 128 + ((c ^ ((r >> 1 & 1) | (r >> 2 & 2))) << 5); };
    auto along_place = [](int r, int c) { return r * 128 + ((c ^ (r >> 1 & 7)) << 4); };
    auto put = [&](uint8_t *to, bool along, bf16x8 lo, bf16x8 hi) {
        *reinterpret_cast<bf16x8 *>(to + (along ? along_place(row, from / 8) : across_place(row, from / 16))) = lo;
        *reinterpret_cast<bf16x8 *>(to + (along ? along_place(row, from / 8 + 1) : across_place(row, from / 16) + 16)) = hi;
    };
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    auto read = [&](const uint8_t *plane, bool along, int first, int h) {        // sixteen rows (or columns) from `first` on
        if (along) return *reinterpret_cast<const bf16x8 *>(plane + along_place(first + r16, 4 * h + quarter));
        const int r = h * 32 + 8 * quarter + lane % 16 / 4;
        const uint8_t *at = plane + across_place(r, first / 16) + lane % 4 * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(at + 4 * 128));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };

#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 2; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    piece p[kAhead];
    if (u.first > u.last) return;
#pragma unroll
    for (int s = 0; s < kAhead; s++) fetch(p[s]);
    for (int at = u.first; at <= u.last; at += kAhead) {
#pragma unroll
        for (int s = 0; s < kAhead; s++) {
            if (at + s > u.last) break;
            uint8_t *a = lds + s % 2 * 2 * kSmallPlane, *b = a + kSmallPlane;
            if constexpr (A_CODES) put(a, true, bf16x8_of_codes(p[s].a[0][0], p[s].a[0][1], scale_of(p[s].ae)), bf16x8_of_codes(p[s].a[0][2], p[s].a[0][3], scale_of(p[s].ae)));
            else put(a, A_ALONG, __builtin_bit_cast(bf16x8, p[s].a[0]), __builtin_bit_cast(bf16x8, p[s].a[1]));
            put(b, B_ALONG, bf16x8_of_codes(p[s].b[0], p[s].b[1], scale_of(p[s].be)), bf16x8_of_codes(p[s].b[2], p[s].b[3], scale_of(p[s].be)));
            fetch(p[s]);
            all_reads();
            barrier();
#pragma unroll
            for (int h = 0; h < 2; h++) {
                bf16x8 a_op[2], b_op[2];
#pragma unroll
                for (int i = 0; i < 2; i++) a_op[i] = read(a, A_ALONG, wi * 32 + i * 16, h);
#pragma unroll
                for (int j = 0; j < 2; j++) b_op[j] = read(b, B_ALONG, GATED ? j * 32 + wj * 16 : wj * 32 + j * 16, h);
#pragma unroll
                for (int i = 0; i < 2; i++)
#pragma unroll
                    for (int j = 0; j < 2; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b_op[j], a_op[i], acc[i][j], 0, 0, 0);
            }
        }
    }
}

// A unit's sums, and what becomes of each lane's four neighbouring columns: store(row, col, acc[i][0], acc[i][1]) of one row, GATED of the gate's and the up
// weights' products; otherwise the second sixteen columns behind the first.
template <int KIND, bool GATED, typename STORE>
__device__ __forceinline__ void small_tile(const wide_args &t, uint8_t *lds, STORE store)
{
    const int tiles = t.tiles_i * t.tiles_j, of = blockIdx.x / tiles, steps = (int)((t.depth + kWideStep - 1) / kWideStep) * t.terms;
    int ti, tj;
    tile_of(t.tiles_i, t.tiles_j, chiplet_order(blockIdx.x % tiles, tiles), ti, tj);
    const int part = of % t.parts, first = part * t.steps_a_part;
    const wide_unit u{(int64_t)ti * kSmallTile, (int64_t)tj * (GATED ? kSmallTile / 2 : kSmallTile), of / t.parts, part, first, min(first + t.steps_a_part, steps) - 1};
    f32x4 acc[2][2];
    small_sums<KIND, GATED>(t, lds, u, acc);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int64_t row = u.i0 + wave / 2 * 32 + i * 16 + lane % 16, col = u.j0 + wave % 2 * (GATED ? 16 : 32) + lane / 16 * 4;
        if (row < t.rows) store(u, row, col, acc[i][0], acc[i][1]);
    }
}

// four values to a matrix of `cols` columns
__device__ inline void store_four(const fp8_matrix &y, int64_t row, int64_t col, int64_t cols, f32x4 s)
{
    const float v[4] = {s[0], s[1], s[2], s[3]};
    if (col < cols) store_values(y, row, col, cols - col, v);
}

}  // namespace pvq_fp8_dev
