// Products of the backward pass: a bfloat16 matrix times an 8-bit block matrix along the blocks' rows.
#include "pvq_fp8_dev.h"

using namespace pvq_fp8_dev;

namespace {

struct grad_args {
    fp8_bf16 dy[2];
    fp8_blocks b[2];
    fp8_matrix out[2];
    int64_t rows, cols, depth;       // of the output, and of the sum (one term's)
    int terms;                       // terms of the sum
    int tiles_i, tiles_j;
    bool vec;
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
    // a lane has four neighbouring columns of one row
    const fp8_matrix out = t.out[out_of];
#pragma unroll
    for (int i = 0; i < FI; i++) {
        const int64_t row = i0 + wi * FI * 16 + i * 16 + r16;
        if (row >= t.rows) continue;
#pragma unroll
        for (int j = 0; j < FJ; j++) {
            const int64_t col = j0 + wj * FJ * 16 + j * 16 + 4 * quarter;
            if (t.vec) store4<true>(out, row, col, t.cols - col, acc[i][j]);
            else store4<false>(out, row, col, t.cols - col, acc[i][j]);
        }
    }
}

bool vector_rows(const fp8_matrix &y)
{
    const int size = y.dtype == PVQ_F32 ? 4 : 2;
    return (uintptr_t)y.data % (4 * size) == 0 && y.ld % 4 == 0;
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
    t.vec = vector_rows(t.out[0]) && (outputs == 1 || vector_rows(t.out[1]));
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
    return launch_grad<128, 128, 2, 2, false>(t, 1, s);
}

hipError_t fp8_launch_weight_grad(const fp8_grad_args &g, hipStream_t s)
{
    grad_args t{};
    for (int i = 0; i < g.pairs; i++) { t.dy[i] = g.dy[i]; t.b[i] = g.b[i]; t.out[i] = g.out[i]; }
    t.rows = g.dy[0].cols; t.cols = g.b[0].cols; t.depth = g.dy[0].rows; t.terms = 1;
    return launch_grad<128, 128, 2, 2, true>(t, g.pairs, s);
}
