// 8-bit blocks: to and from floats, and the element-wise half of the gated block's backward pass.  All of it is bound by memory.
#include "pvq_fp8_dev.h"

using namespace pvq_fp8_dev;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kItem = 4 * kFp8Block;          // a wave's values at a time: 8 a lane, four blocks, one word of exponents

template <int T> struct element { using type = uint16_t; };
template <> struct element<PVQ_F32> { using type = float; };

template <int T>
__device__ inline float to_float(typename element<T>::type v)
{
    if constexpr (T == PVQ_F32) return v;
    else if constexpr (T == PVQ_F16) return (float)__builtin_bit_cast(_Float16, v);
    else return __uint_as_float((uint32_t)v << 16);
}

// eight values of a row from column c on, zeros from column `cols` on
template <int T>
__device__ inline void load8(const typename element<T>::type *row, int64_t c, int64_t cols, float (&v)[8])
{
    using E = typename element<T>::type;
    if (c + 8 <= cols) {
        union { u32x4 w[sizeof(E) / 2]; E e[8]; } u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; i++) u.w[i] = reinterpret_cast<const unaligned<u32x4, sizeof(E)> *>(row + c)[i].v;
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = to_float<T>(u.e[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = c + i < cols ? to_float<T>(row[c + i]) : 0.0f;
}

template <int T>
__global__ __launch_bounds__(kThreads) void encode_kernel(const typename element<T>::type *X, int64_t rows, int64_t cols, int64_t ldx,
                                                          uint8_t *codes, uint8_t *exps, int64_t code_row, int64_t exp_row, int tiles)
{
    const int lane = threadIdx.x % kWave;
    const int64_t items = rows * tiles, step = (int64_t)gridDim.x * kWaves;
    for (int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); item < items; item += step) {
        const int64_t row = item / tiles;
        const int64_t tile = item - row * tiles, c = tile * kItem + 8 * lane;
        float v[8];
        load8<T>(X + row * ldx, c, cols, v);
        const uint32_t e = block_exponent(v);
        if (c < code_row) store_codes8(codes + row * code_row + c, e, v);
        uint32_t word = 0;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if ((tile * 4 + i) * kFp8Block < code_row) word |= (uint32_t)__builtin_amdgcn_readlane((int)e, 16 * i) << (8 * i);
        if (lane == 0) *reinterpret_cast<uint32_t *>(exps + row * exp_row + tile * 4) = word;
    }
}

__global__ __launch_bounds__(kThreads) void decode_kernel(fp8_blocks b, fp8_matrix y, int tiles)
{
    const int lane = threadIdx.x % kWave;
    const int64_t items = b.rows * tiles, step = (int64_t)gridDim.x * kWaves, code_row = b.code_row(), exp_row = b.exp_row();
    for (int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); item < items; item += step) {
        const int64_t row = item / tiles;
        const int64_t c = (item - row * tiles) * kItem + 8 * lane;
        if (c >= b.cols) continue;
        const u32x2 w = *reinterpret_cast<const u32x2 *>(b.codes + row * code_row + c);
        const float scale = scale_of(b.exps[row * exp_row + c / kFp8Block]);
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], true);
            v[4 * h] = lo[0] * scale; v[4 * h + 1] = lo[1] * scale; v[4 * h + 2] = hi[0] * scale; v[4 * h + 3] = hi[1] * scale;
        }
        store_values(y, row, c, b.cols - c, v);
    }
}

// What the rounding of a value to bfloat16 left of it, exactly (nothing of an infinity or a NaN, or of what becomes one).
__device__ inline float left_of(float v, uint32_t rounded) { return (rounded & 0x7F80u) == 0x7F80u ? 0.0f : v - __uint_as_float(rounded << 16); }

// One lane a run of eight: dG = dH U act'(G) and dU = dH act(G), and with two pieces what their roundings left.
template <int ACT, int PIECES>
__global__ __launch_bounds__(kThreads) void slopes_kernel(fp8_bf16 dh, fp8_blocks g, fp8_blocks u, uint16_t *dg, uint16_t *du,
                                                          int64_t ld)
{
    const int64_t runs = ld / 8, total = dh.rows * runs, n = dh.cols, code_row = g.code_row(), exp_row = g.exp_row(), piece = dh.rows * ld;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / runs, c = (i - row * runs) * 8;
        u32x4 wg[PIECES] = {}, wu[PIECES] = {};
        if (c < n) {
            float d[8];
            load8<PVQ_BF16>(dh.data + row * dh.ld, c, n, d);
            const u32x2 cg = *reinterpret_cast<const u32x2 *>(g.codes + row * code_row + c), cu = *reinterpret_cast<const u32x2 *>(u.codes + row * code_row + c);
            const float sg = scale_of(g.exps[row * exp_row + c / kFp8Block]), su = scale_of(u.exps[row * exp_row + c / kFp8Block]);
#pragma unroll
            for (int p = 0; p < 4; p++) {
                const f32x2 a = p & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(cg[p / 2], true) : __builtin_amdgcn_cvt_pk_f32_fp8(cg[p / 2], false);
                const f32x2 b = p & 1 ? __builtin_amdgcn_cvt_pk_f32_fp8(cu[p / 2], true) : __builtin_amdgcn_cvt_pk_f32_fp8(cu[p / 2], false);
                float og[2], ou[2];
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    float value, slope;
                    act_slope<ACT>(a[j] * sg, value, slope);
                    const bool in = c + 2 * p + j < n;
                    og[j] = in ? d[2 * p + j] * (b[j] * su) * slope : 0.0f;
                    ou[j] = in ? d[2 * p + j] * value : 0.0f;
                }
                wg[0][p] = bf16_pair(og[0], og[1]);
                wu[0][p] = bf16_pair(ou[0], ou[1]);
                if constexpr (PIECES == 2) {
                    wg[1][p] = bf16_pair(left_of(og[0], wg[0][p] & 0xFFFFu), left_of(og[1], wg[0][p] >> 16));
                    wu[1][p] = bf16_pair(left_of(ou[0], wu[0][p] & 0xFFFFu), left_of(ou[1], wu[0][p] >> 16));
                }
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; i++) {
            *reinterpret_cast<u32x4 *>(dg + i * piece + row * ld + c) = wg[i];
            *reinterpret_cast<u32x4 *>(du + i * piece + row * ld + c) = wu[i];
        }
    }
}

// four neighbouring sums a lane; a part's rows follow one another without a gap
__global__ __launch_bounds__(kThreads) void join_kernel(const float *work, int parts, int64_t rows, int64_t cols, fp8_matrix out)
{
    const int64_t runs = (cols + 3) / 4, total = rows * runs, part = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / runs, c = (i - row * runs) * 4, count = cols - c;
        const float *p = work + row * cols + c;
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < parts; k++, p += part)
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (j < count) sum[j] += p[j];
        const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
        store_values(out, row, c, count, v);
    }
}

// The parts' sums of G and U, [part][G, U][rows][cols], added, and what the gated block makes of them: sixteen lanes a block.
__global__ __launch_bounds__(kThreads) void gated_join_kernel(const float *work, int parts, int64_t rows, int64_t cols, gated_out out)
{
    const int64_t blocks = (cols + kFp8Block - 1) / kFp8Block, items = rows * blocks, item = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / 16;
    const bool there = item < items;                             // (the others come along: the lanes of a block work together)
    const int64_t row = there ? item / blocks : 0, block = there ? item - row * blocks : 0, c = block * kFp8Block + threadIdx.x % 16 * 8;
    float g[8] = {}, u[8] = {};
    for (int p = 0; p < parts; p++) {
        float a[8], b[8];
        const float *from = work + (int64_t)p * 2 * rows * cols + row * cols;
        load8<PVQ_F32>(from, c, cols, a);
        load8<PVQ_F32>(from + rows * cols, c, cols, b);
#pragma unroll
        for (int i = 0; i < 8; i++) { g[i] += a[i]; u[i] += b[i]; }
    }
    if (out.act == PVQ_SILU) store_gated8<PVQ_SILU>(out, row, cols, block, c, there, g, u);
    else store_gated8<PVQ_GELU>(out, row, cols, block, c, there, g, u);
}

// A lane eight values, loaded as they lie: 1030 x 20603 in 14 us (by elements 28).
__global__ __launch_bounds__(kThreads) void align_kernel(fp8_bf16 from, uint16_t *to, int64_t ld)
{
    const int64_t runs = ld / 8, total = from.rows * runs;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / runs, c = (i - row * runs) * 8;
        const uint16_t *p = from.data + row * from.ld + c;
        u32x4 w = {0, 0, 0, 0};
        if (c + 8 <= from.cols) w = reinterpret_cast<const unaligned<u32x4, 2> *>(p)->v;
        else {
#pragma unroll
            for (int e = 0; e < 7; e++)
                if (c + e < from.cols) w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
        }
        *reinterpret_cast<u32x4 *>(to + row * ld + c) = w;
    }
}

unsigned grid_for(int64_t work, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min(work, most)); }

template <int T>
hipError_t launch_encode(const void *X, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes, uint8_t *exps, hipStream_t s)
{
    using E = typename element<T>::type;
    const fp8_blocks b{codes, exps, rows, cols};
    const int tiles = (int)((b.blocks() + 3) / 4);
    const unsigned grid = grid_for((rows * tiles + kWaves - 1) / kWaves, 256 * 8 * 4);
    hipLaunchKernelGGL(encode_kernel<T>, dim3(grid), dim3(kThreads), 0, s, (const E *)X, rows, cols, ldx, codes, exps, b.code_row(), b.exp_row(), tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t fp8_launch_encode(const void *X, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes, uint8_t *exps, hipStream_t s)
{
    if (dtype == PVQ_F32) return launch_encode<PVQ_F32>(X, rows, cols, ldx, codes, exps, s);
    if (dtype == PVQ_F16) return launch_encode<PVQ_F16>(X, rows, cols, ldx, codes, exps, s);
    return launch_encode<PVQ_BF16>(X, rows, cols, ldx, codes, exps, s);
}

hipError_t fp8_launch_decode(const fp8_blocks &b, const fp8_matrix &y, hipStream_t s)
{
    const int tiles = (int)((b.blocks() + 3) / 4);
    const unsigned grid = grid_for((b.rows * tiles + kWaves - 1) / kWaves, 256 * 8 * 4);
    hipLaunchKernelGGL(decode_kernel, dim3(grid), dim3(kThreads), 0, s, b, y, tiles);
    return hipGetLastError();
}

hipError_t fp8_launch_gated_slopes(const fp8_bf16 &dh, const fp8_blocks &g, const fp8_blocks &u, int act, uint16_t *dg, uint16_t *du, int pieces,
                                   int64_t ld, hipStream_t s)
{
    const unsigned grid = grid_for((dh.rows * (ld / 8) + kThreads - 1) / kThreads, 256 * 8 * 4);
    const auto kernel = act == PVQ_SILU ? pieces == 1 ? &slopes_kernel<PVQ_SILU, 1> : &slopes_kernel<PVQ_SILU, 2>
                                        : pieces == 1 ? &slopes_kernel<PVQ_GELU, 1> : &slopes_kernel<PVQ_GELU, 2>;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, s, dh, g, u, dg, du, ld);
    return hipGetLastError();
}

hipError_t fp8_launch_join(const float *work, int parts, int64_t rows, int64_t cols, const fp8_matrix &out, hipStream_t s)
{
    const unsigned grid = grid_for((rows * ((cols + 3) / 4) + kThreads - 1) / kThreads, 256 * 8 * 4);
    hipLaunchKernelGGL(join_kernel, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, out);
    return hipGetLastError();
}

hipError_t fp8_launch_gated_join(const float *work, int parts, const fp8_gated_args &a, hipStream_t s)
{
    const int64_t rows = a.x.rows, cols = a.gate.rows;
    const gated_out out{a.h, a.act, a.hc, a.he, a.gc, a.ge, a.uc, a.ue};
    const unsigned grid = (unsigned)((rows * ((cols + kFp8Block - 1) / kFp8Block) * 16 + kThreads - 1) / kThreads);
    hipLaunchKernelGGL(gated_join_kernel, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, out);
    return hipGetLastError();
}

hipError_t fp8_launch_align(const fp8_bf16 &from, uint16_t *to, int64_t ld, hipStream_t s)
{
    const unsigned grid = grid_for((from.rows * (ld / 8) + kThreads - 1) / kThreads, 256 * 8 * 4);
    hipLaunchKernelGGL(align_kernel, dim3(grid), dim3(kThreads), 0, s, from, to, ld);
    return hipGetLastError();
}
