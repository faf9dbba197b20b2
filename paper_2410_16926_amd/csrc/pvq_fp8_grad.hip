// Products of the backward pass: a bfloat16 matrix times an 8-bit block matrix along the blocks' rows.
#include "pvq_fp8_tile.h"

using namespace pvq_fp8_dev;

namespace {

struct grad_args {
    fp8_bf16 dy[2];
    fp8_blocks b[2];
    fp8_matrix out[2];
    int64_t rows, cols, depth;       // of the output, and of the sum (one term's)
    int terms;                       // terms of the sum
    int tiles_i, tiles_j;
    int parts, steps_a_part;         // of a split sum, whose parts go to work
    float *work;
    int vec;                         // what the outputs' rows are aligned to: 8 values, 4 or 1
};

constexpr int kStep = 64;            // of the sum at a time

// Eight bfloat16 of a row from column c on, zeros from `cols` on; rows start at any element.
__device__ inline u32x4 load8_bf16(const uint16_t *row, int64_t c, int64_t cols)
{
    if (c + 8 <= cols) {
        struct __attribute__((packed, aligned(2))) any { u32x4 w; };
        return reinterpret_cast<const any *>(row + c)->w;
    }
    u32x4 w = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (c + i < cols) w[i / 2] |= (uint32_t)row[c + i] << (16 * (i & 1));
    return w;
}

// out(i, j) = sum_r A(i, r) B(r, j), B in blocks along j, decoded to bfloat16 on the way into LDS.
// ACROSS == false: A(i, r) = dY[i][r] (dX = dY W); true: A(i, r) = dY[r][i] (dW = dY^T X).
// An operand whose rows run across the sum lies in LDS as in memory, [r][columns], in pieces of 32 bytes; the transposing
// LDS read gives a lane four neighbouring r of one column.  Piece p of row r lies at place p ^ (r % 4) (of a run of four), so that the
// four rows of such a read lie in different banks.
template <int T>
__device__ inline uint32_t across_at(uint32_t r, uint32_t col) { return r * (2 * T) + ((((col >> 4) ^ (r & 3)) << 5) | ((col & 15) << 1)); }

// dY[i][r] rows: 64 values of r, 128 bytes in eight chunks; chunk c of row i at place c ^ (i % 8)
__device__ inline uint32_t along_at(uint32_t i, uint32_t chunk) { return i * (2 * kStep) + ((chunk ^ (i & 7)) << 4); }

template <int T>
__device__ inline bf16x8 read_across(const uint8_t *tile, uint32_t r, uint32_t col)
{
    // lane % 16 gives the read its row and columns, and gets column lane % 16 of the sixteen
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t sub = threadIdx.x % 16, row = r + sub / 4, c = col + 4 * (sub % 4);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + across_at<T>(row, c)));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(tile + across_at<T>(row + 4, c)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <int TI, int TJ, int WI, int WJ, bool ACROSS>
__global__ __launch_bounds__(WI *WJ *kWave) void grad_kernel(grad_args t)
{
    constexpr int kThreads = WI * WJ * kWave, FI = TI / WI / 16, FJ = TJ / WJ / 16;
    constexpr int kA = TI * kStep * 2, kB = TJ * kStep * 2;
    constexpr int kPiecesA = TI * kStep / 8 / kThreads, kPiecesB = TJ * kStep / 16 / kThreads;
    extern __shared__ __align__(16) uint8_t lds[];
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wi = wave / WJ, wj = wave % WJ, r16 = lane % 16, quarter = lane / 16;
    const int id = chiplet_order(blockIdx.x, gridDim.x);
    const int64_t i0 = (int64_t)(id % t.tiles_i) * TI, j0 = (int64_t)(id / t.tiles_i) * TJ;
    const int out_of = blockIdx.y;
    const int steps_a_term = (int)((t.depth + kStep - 1) / kStep), steps = steps_a_term * t.terms;

    u32x4 ra[kPiecesA], rb[kPiecesB];
    float sb[kPiecesB];
    auto fetch = [&](int step) {
        const int term = step / steps_a_term + out_of;
        const int64_t r0 = (int64_t)(step % steps_a_term) * kStep;
        const fp8_bf16 &dy = t.dy[term];
        const fp8_blocks &b = t.b[term];
#pragma unroll
        for (int p = 0; p < kPiecesA; p++) {
            const int piece = p * kThreads + tid;
            if constexpr (ACROSS) {
                const int r = piece / (TI / 8);
                const int64_t i = i0 + (piece % (TI / 8)) * 8;
                ra[p] = r0 + r < t.depth && i < t.rows ? load8_bf16(dy.data + (r0 + r) * dy.ld, i, t.rows) : u32x4{0, 0, 0, 0};
            } else {
                const int64_t i = min(i0 + piece / (kStep / 8), t.rows - 1), r = r0 + (piece % (kStep / 8)) * 8;
                ra[p] = r < t.depth ? load8_bf16(dy.data + i * dy.ld, r, t.depth) : u32x4{0, 0, 0, 0};
            }
        }
#pragma unroll
        for (int p = 0; p < kPiecesB; p++) {
            const int piece = p * kThreads + tid;
            const int64_t r = r0 + piece / (TJ / 16), j = j0 + (piece % (TJ / 16)) * 16;
            const bool in = r < t.depth && j < b.code_row();
            rb[p] = in ? *reinterpret_cast<const u32x4 *>(b.codes + r * b.code_row() + j) : u32x4{0, 0, 0, 0};
            sb[p] = in ? scale_of(b.exps[r * b.exp_row() + j / kFp8Block]) : 1.0f;
        }
    };
    auto put = [&](int stage) {
        uint8_t *at = lds + stage * (kA + kB), *bt = at + kA;
#pragma unroll
        for (int p = 0; p < kPiecesA; p++) {
            const int piece = p * kThreads + tid;
            if constexpr (ACROSS) *reinterpret_cast<u32x4 *>(at + across_at<TI>(piece / (TI / 8), (piece % (TI / 8)) * 8)) = ra[p];
            else *reinterpret_cast<u32x4 *>(at + along_at(piece / (kStep / 8), piece % (kStep / 8))) = ra[p];
        }
#pragma unroll
        for (int p = 0; p < kPiecesB; p++) {
            const int piece = p * kThreads + tid;
            uint8_t *to = bt + across_at<TJ>(piece / (TJ / 16), (piece % (TJ / 16)) * 16);
            *reinterpret_cast<bf16x8 *>(to) = bf16x8_of_codes(rb[p][0], rb[p][1], sb[p]);
            *reinterpret_cast<bf16x8 *>(to + 16) = bf16x8_of_codes(rb[p][2], rb[p][3], sb[p]);
        }
    };

    f32x4 acc[FI][FJ];
#pragma unroll
    for (int i = 0; i < FI; i++)
#pragma unroll
        for (int j = 0; j < FJ; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    fetch(0);
    put(0);
    for (int step = 0; step < steps; step++) {
        __syncthreads();
        const int stage = step & 1;
        if (step + 1 < steps) fetch(step + 1);
        const uint8_t *at = lds + stage * (kA + kB), *bt = at + kA;
#pragma unroll
        for (int h = 0; h < kStep / 32; h++) {
            bf16x8 bf[FJ];
#pragma unroll
            for (int j = 0; j < FJ; j++) bf[j] = read_across<TJ>(bt, 32 * h + 8 * quarter, wj * FJ * 16 + j * 16);
#pragma unroll
            for (int i = 0; i < FI; i++) {
                bf16x8 af;
                if constexpr (ACROSS) af = read_across<TI>(at, 32 * h + 8 * quarter, wi * FI * 16 + i * 16);
                else af = *reinterpret_cast<const bf16x8 *>(at + along_at(wi * FI * 16 + i * 16 + r16, 4 * h + quarter));
#pragma unroll
                for (int j = 0; j < FJ; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[j], af, acc[i][j], 0, 0, 0);
            }
        }
        if (step + 1 < steps) put(stage ^ 1);
    }
    store_fragments<FI, FJ>(t.out[out_of], t.vec, t.rows, t.cols, i0 + wi * FI * 16, j0 + wj * FJ * 16, [&](int i, int j) { return acc[i][j]; });
}

// Tiles of 256 x 256 by four waves of 128 x 128, one to a SIMD, as for products on the 8-bit instruction (pvq_fp8_product.hip): LDS is
// written 64 KB and read 128 KB for 64 of the sum, 1500 of the 2048 cycles of matrix instructions.  Both operands come through registers, B's codes
// to be decoded once for the four waves, dY as it is.
//
// A step is 64 of the sum, two halves of 32.  While the first half's 64 instructions run, the second half's operands are read, which empties the
// stage; behind the step's barrier, while the second half's run, the next step's first operands are read from the other stage, then what was fetched
// a step ago is put into the empty one, and the step after that is fetched.
//
// dY's rows are aligned to 16 bytes (others go to grad_kernel).
template <bool ACROSS>
__global__ __launch_bounds__(256) void big_grad_kernel(grad_args t)
{
    constexpr int kTile = 256, F = 8, kPlane = kTile * kStep * 2, kPieces = 8;
    extern __shared__ __align__(16) uint8_t lds[];               // A's two stages, B's two stages
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int wi = wave / 2, wj = wave % 2, r16 = lane % 16, quarter = lane / 16;
    int ti, tj;
    tile_of(t.tiles_i, t.tiles_j, chiplet_order(blockIdx.x, gridDim.x), ti, tj);
    const int64_t i0 = (int64_t)ti * kTile, j0 = (int64_t)tj * kTile;
    const int out_of = blockIdx.y / t.parts, part = blockIdx.y % t.parts;
    const int steps_a_term = (int)((t.depth + kStep - 1) / kStep);
    const int first = part * t.steps_a_part, last = min(first + t.steps_a_part, steps_a_term * t.terms) - 1;

    const uint32_t ld = (uint32_t)t.dy[0].ld * 2, code_row = (uint32_t)t.b[0].code_row(), exp_row = (uint32_t)t.b[0].exp_row();   // (the same for both)
    // a lane's piece: eight of dY (16 bytes) and eight codes; piece p of either is `*_next` bytes behind piece p - 1
    const uint32_t a_at = ACROSS ? (tid / 32) * ld + (tid % 32) * 16 : (tid / 8) * ld + (tid % 8) * 16, a_next = (ACROSS ? 8 : 32) * ld;
    const uint32_t b_at = (tid / 32) * code_row + (tid % 32) * 8, e_at = (tid / 32) * exp_row + tid % 32 / 16;

    u32x4 ra[kPieces];
    u32x2 rb[kPieces];
    uint32_t re[kPieces];
    __amdgpu_buffer_rsrc_t a_from, b_from, e_from;
    // Buffers that start with the step's part of the tile and end with the matrix: what lies behind, and everything of a step behind the last,
    // is zero.
    int tail = 8;                                                 // of the lane's eight of a row of dY, how many belong to the sum
    auto aim = [&](int step) {
        const int term = step >= steps_a_term ? 1 : 0;
        const bool second = (term | out_of) != 0;
        const int64_t r0 = (int64_t)(step - term * steps_a_term) * kStep;
        const uint16_t *y = second ? t.dy[1].data : t.dy[0].data;
        const uint8_t *codes = second ? t.b[1].codes : t.b[0].codes, *exps = second ? t.b[1].exps : t.b[0].exps;
        auto buffer = [&](const void *base, int64_t row, int64_t rows, int64_t cols, int64_t at) {
            const int64_t left = step <= last ? min((rows - 1) * row + cols - at, (int64_t)0xFFFFFFFF) : 0;
            return __builtin_amdgcn_make_buffer_rsrc((void *)((const uint8_t *)base + at), 0, (uint32_t)left, 0x00020000);
        };
        // (dY's last row to the end of its last 16 bytes: a load that is not whole would bring nothing)
        const int64_t row_end = ((ACROSS ? t.rows : t.depth) * 2 + 15) / 16 * 16;
        a_from = ACROSS ? buffer(y, ld, t.depth, row_end, r0 * ld + i0 * 2) : buffer(y, ld, t.rows, row_end, i0 * ld + r0 * 2);
        b_from = buffer(codes, code_row, t.depth, code_row, r0 * code_row + j0);
        e_from = buffer(exps, exp_row, t.depth, exp_row, r0 * exp_row + j0 / kFp8Block);
        tail = (int)min(t.depth - r0 - (tid % 8) * 8, (int64_t)8);
    };
    auto fetch_a = [&](int p) { ra[p] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(a_from, a_at, p * a_next, 0)); };
    auto fetch_b = [&](int p) {
        rb[p] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b_from, b_at, p * 8 * code_row, 0));
        re[p] = __builtin_amdgcn_raw_buffer_load_b8(e_from, e_at, p * 8 * exp_row, 0);
    };

    // An operand whose rows run across the sum lies in LDS as in memory, [r][256 columns], in pieces of sixteen columns; the transposing
    // read gives a lane four neighbouring r of one column.  Piece c of row r lies at place c ^ f(r), f = r % 4 + 4 (r / 8 % 2): the eight rows that 32
    // lanes read at once lie in different banks.  dY whose rows run along the sum: [i][64 r], chunk c of row i at place c ^ (i / 2 % 8).
    const uint32_t across_to = (tid / 32) * 512 + (((tid % 32 / 2) ^ (tid / 32 & 3)) << 5) + (tid % 2) * 16, across_odd = across_to ^ (4 << 5);
    const uint32_t along_to = (tid / 8) * 128 + (((tid % 8) ^ (tid / 16 & 7)) << 4);
    // what lies behind the end of dY's row must not count, not even times zero
    uint32_t keep[4];
    auto keep_tail = [&]() {
#pragma unroll
        for (int e = 0; e < 4; e++) keep[e] = 2 * e + 1 < tail ? ~0u : 2 * e < tail ? 0xFFFFu : 0u;
    };
    // (stages by the offset of their planes, 0 or kPlane: one body for all steps, whose sums stay where they are)
    auto put_a = [&](uint32_t stage, int p) {
        u32x4 v = ra[p];
        if constexpr (!ACROSS) {
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] &= keep[e];
        }
        *reinterpret_cast<u32x4 *>(lds + stage + p * 4096 + (ACROSS ? (p & 1 ? across_odd : across_to) : along_to)) = v;
    };
    auto put_b = [&](uint32_t stage, int p) {
        *reinterpret_cast<bf16x8 *>(lds + stage + 2 * kPlane + p * 4096 + (p & 1 ? across_odd : across_to)) = bf16x8_of_codes(rb[p][0], rb[p][1], scale_of(re[p]));
    };
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const uint32_t sub = lane % 16, f = sub / 4 | (quarter & 1) << 2, row_at = (8 * quarter + sub / 4) * 512 + (sub % 4) * 8;
    auto read_across = [&](uint32_t plane, int column, int h) {       // sixteen columns from 16 * column on
        const uint8_t *from = lds + plane + h * 32 * 512 + (column / 8) * 256 + (((column % 8) ^ f) << 5) + row_at;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(from + 4 * 512));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_a = [&](uint32_t stage, int i, int h) {
        if constexpr (ACROSS) return read_across(stage, wi * 8 + i, h);
        else return *reinterpret_cast<const bf16x8 *>(lds + stage + (wi * 128 + i * 16 + r16) * 128 + (((4 * h + quarter) ^ (r16 >> 1)) << 4));
    };
    auto read_b = [&](uint32_t stage, int j, int h) { return read_across(stage + 2 * kPlane, wj * 8 + j, h); };

    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < F; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    bf16x8 a_op[2][F], b_op[2][F];

    auto fetch_all = [&](int step) {
        aim(step);
#pragma unroll
        for (int p = 0; p < kPieces; p++) { fetch_a(p); fetch_b(p); }
    };
    auto put_all = [&](uint32_t stage) {
        keep_tail();
#pragma unroll
        for (int p = 0; p < kPieces; p++) { put_a(stage, p); put_b(stage, p); }
    };
    auto step_of = [&](int step, uint32_t stage) {
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated(acc[i][j], b_op[0][j], a_op[0][i]);
                const int slot = i * F + j;
                if (slot % 2 == 0 && slot / 2 < F) b_op[1][slot / 2] = read_b(stage, slot / 2, 1);
                if (slot % 2 == 0 && slot / 2 >= F && slot / 2 < 2 * F) a_op[1][slot / 2 - F] = read_a(stage, slot / 2 - F, 1);
                __builtin_amdgcn_sched_barrier(0);
            }
        all_reads();
        barrier();
        keep_tail();
        aim(step + 3);
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated(acc[i][j], b_op[1][j], a_op[1][i]);
                const int slot = i * F + j;
                if (slot % 2 == 0 && slot / 2 < F) b_op[0][slot / 2] = read_b(stage ^ kPlane, slot / 2, 0);
                if (slot % 2 == 0 && slot / 2 >= F && slot / 2 < 2 * F) a_op[0][slot / 2 - F] = read_a(stage ^ kPlane, slot / 2 - F, 0);
                if (slot >= 32 && slot % 4 == 1) { put_a(stage, (slot - 32) / 4); fetch_a((slot - 32) / 4); }
                if (slot >= 32 && slot % 4 == 3) { put_b(stage, (slot - 32) / 4); fetch_b((slot - 32) / 4); }
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    if (first <= last) {
        fetch_all(first);
        put_all(0);
        fetch_all(first + 1);
        put_all(kPlane);
        fetch_all(first + 2);
        all_reads();
        barrier();
#pragma unroll
        for (int j = 0; j < F; j++) b_op[0][j] = read_b(0, j, 0);
#pragma unroll
        for (int i = 0; i < F; i++) a_op[0][i] = read_a(0, i, 0);
        uint32_t stage = 0;
        for (int step = first; step <= last; step++, stage ^= kPlane) step_of(step, stage);
    }
    sums_are_there();
    fp8_matrix out = t.out[out_of];
    if (t.parts > 1) out = fp8_matrix{t.work + (int64_t)blockIdx.y * t.rows * t.cols, PVQ_F32, t.cols};
    const int vec = t.parts > 1 ? (t.cols % 8 == 0 ? 8 : t.cols % 4 == 0 ? 4 : 1) : t.vec;
    store_fragments<F, F>(out, vec, t.rows, t.cols, i0 + wi * 128, j0 + wj * 128, [&](int i, int j) { return read_sums(acc[i][j]); });
}

template <bool ACROSS>
hipError_t launch_big_grad(grad_args &t, int outputs, hipStream_t s)
{
    constexpr int kTile = 256, kLds = 4 * kTile * kStep * 2;
    const auto kernel = &big_grad_kernel<ACROSS>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    t.tiles_i = (int)((t.rows + kTile - 1) / kTile);
    t.tiles_j = (int)((t.cols + kTile - 1) / kTile);
    t.vec = std::min(row_alignment(t.out[0]), outputs == 1 ? 8 : row_alignment(t.out[1]));
    t.steps_a_part = (int)((((t.depth + kStep - 1) / kStep) * t.terms + t.parts - 1) / t.parts);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_i * t.tiles_j), (unsigned)(outputs * t.parts)), dim3(256), kLds, s, t);
    return hipGetLastError();
}

// whether dY's rows can be read 16 bytes at a time, and a tile's lie within 32-bit offsets
bool aligned_rows(const fp8_grad_args &g)
{
    for (int i = 0; i < g.pairs; i++)
        if ((uintptr_t)g.dy[i].data % 16 || g.dy[i].ld % 8 || g.dy[i].ld > 1 << 22) return false;
    return true;
}

template <int TI, int TJ, int WI, int WJ, bool ACROSS>
hipError_t launch_grad(grad_args &t, int outputs, hipStream_t s)
{
    constexpr int kLds = 2 * (TI + TJ) * kStep * 2;
    const auto kernel = &grad_kernel<TI, TJ, WI, WJ, ACROSS>;
    if (kLds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
        if (e != hipSuccess) return e;
    }
    t.tiles_i = (int)((t.rows + TI - 1) / TI);
    t.tiles_j = (int)((t.cols + TJ - 1) / TJ);
    t.vec = std::min(row_alignment(t.out[0]), outputs == 1 ? 8 : row_alignment(t.out[1]));
    hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_i * t.tiles_j), (unsigned)outputs), dim3(WI * WJ * kWave), kLds, s, t);
    return hipGetLastError();
}

}  // namespace

size_t fp8_input_grad_work(int64_t, int64_t, int64_t, int, int) { return 0; }
size_t fp8_weight_grad_work(int64_t, int64_t, int64_t, int, int) { return 0; }

hipError_t fp8_launch_input_grad(const fp8_grad_args &g, hipStream_t s)
{
    grad_args t{};
    for (int i = 0; i < g.pairs; i++) { t.dy[i] = g.dy[i]; t.b[i] = g.b[i]; }
    t.out[0] = g.out[0];
    t.rows = g.dy[0].rows; t.cols = g.b[0].cols; t.depth = g.dy[0].cols; t.terms = g.pairs;
    t.parts = 1;
    if (aligned_rows(g) && t.rows > 128 && t.cols > 128) return launch_big_grad<false>(t, 1, s);
    return launch_grad<128, 128, 2, 2, false>(t, 1, s);
}

hipError_t fp8_launch_weight_grad(const fp8_grad_args &g, hipStream_t s)
{
    grad_args t{};
    for (int i = 0; i < g.pairs; i++) { t.dy[i] = g.dy[i]; t.b[i] = g.b[i]; t.out[i] = g.out[i]; }
    t.rows = g.dy[0].cols; t.cols = g.b[0].cols; t.depth = g.dy[0].rows; t.terms = 1;
    t.parts = 1;
    if (aligned_rows(g) && t.rows > 128 && t.cols > 128) return launch_big_grad<true>(t, g.pairs, s);
    return launch_grad<128, 128, 2, 2, true>(t, g.pairs, s);
}
