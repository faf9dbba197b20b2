// 8-bit blocks: to and from floats, and the element-wise half of the gated block's backward pass.  All of it is bound by memory.
#include "pvq_fp8_dev.h"

using namespace pvq_fp8_dev;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
constexpr int kItem = 4 * kFp8Block;          // a wave's values at a time: 8 a lane, four blocks, one word of exponents

// the largest of a block's sixteen lanes, in all of them (rotations inside a row of sixteen)
__device__ inline uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
}

template <int T> struct element { using type = uint16_t; };
template <> struct element<PVQ_F32> { using type = float; };

template <int T>
__device__ inline float to_float(typename element<T>::type v)
{
    if constexpr (T == PVQ_F32) return v;
    else if constexpr (T == PVQ_F16) return (float)__builtin_bit_cast(_Float16, v);
    else return __uint_as_float((uint32_t)v << 16);
}

// eight values of a row from column c on, zeros from column `cols` on; VEC: 16-byte aligned rows
template <int T, bool VEC>
__device__ inline void load8(const typename element<T>::type *row, int64_t c, int64_t cols, float (&v)[8])
{
    using E = typename element<T>::type;
    if (VEC && c + 8 <= cols) {
        union { u32x4 w[sizeof(E) / 2]; E e[8]; } u;
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; i++) u.w[i] = reinterpret_cast<const u32x4 *>(row + c)[i];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = to_float<T>(u.e[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = c + i < cols ? to_float<T>(row[c + i]) : 0.0f;
}

// A wave's item of four blocks, whose largest magnitudes are `top`: the lane's eight codes, and the blocks' exponents in one word.
__device__ inline void store_codes(uint8_t *codes, uint8_t *exps, int64_t tile, int64_t c, int64_t code_row, int lane, const float (&v)[8], uint32_t top)
{
    const uint32_t e = exponent_of(top);
    const float inverse = scale_of(254 - e);
    if (c < code_row) {
        const u32x2 w = {codes4(v[0], v[1], v[2], v[3], inverse), codes4(v[4], v[5], v[6], v[7], inverse)};
        *reinterpret_cast<u32x2 *>(codes + c) = w;
    }
    uint32_t word = 0;
#pragma unroll
    for (int i = 0; i < 4; i++)
        if ((tile * 4 + i) * kFp8Block < code_row) word |= (uint32_t)__builtin_amdgcn_readlane((int)e, 16 * i) << (8 * i);
    if (lane == 0) *reinterpret_cast<uint32_t *>(exps + tile * 4) = word;
}

template <int T, bool VEC>
__global__ __launch_bounds__(kThreads) void encode_kernel(const typename element<T>::type *X, int64_t rows, int64_t cols, int64_t ldx,
                                                          uint8_t *codes, uint8_t *exps, int64_t code_row, int64_t exp_row, int tiles)
{
    const int lane = threadIdx.x % kWave;
    const int64_t items = rows * tiles, step = (int64_t)gridDim.x * kWaves;
    for (int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); item < items; item += step) {
        const int64_t row = item / tiles;
        const int64_t tile = item - row * tiles, c = tile * kItem + 8 * lane;
        float v[8];
        load8<T, VEC>(X + row * ldx, c, cols, v);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, finite_bits(v[i]));
        store_codes(codes + row * code_row, exps + row * exp_row, tile, c, code_row, lane, v, block_max(top));
    }
}

template <bool VEC>
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
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[h], true);
            if (c + 4 * h < b.cols)
                store4<VEC>(y, row, c + 4 * h, b.cols - c - 4 * h, f32x4{lo[0] * scale, lo[1] * scale, hi[0] * scale, hi[1] * scale});
        }
    }
}

// One lane a run of eight: dG = dH U act'(G) and dU = dH act(G).
template <bool VEC>
__global__ __launch_bounds__(kThreads) void slopes_kernel(fp8_bf16 dh, fp8_blocks g, fp8_blocks u, int act, uint16_t *dg, uint16_t *du,
                                                          int64_t ld)
{
    const int64_t runs = ld / 8, total = dh.rows * runs, n = dh.cols, code_row = g.code_row(), exp_row = g.exp_row();
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / runs, c = (i - row * runs) * 8;
        u32x4 wg = {0, 0, 0, 0}, wu = {0, 0, 0, 0};
        if (c < n) {
            float d[8];
            load8<PVQ_BF16, VEC>(dh.data + row * dh.ld, c, n, d);
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
                    act_slope(act, a[j] * sg, value, slope);
                    const bool in = c + 2 * p + j < n;
                    og[j] = in ? d[2 * p + j] * (b[j] * su) * slope : 0.0f;
                    ou[j] = in ? d[2 * p + j] * value : 0.0f;
                }
                wg[p] = bf16_pair(og[0], og[1]);
                wu[p] = bf16_pair(ou[0], ou[1]);
            }
        }
        *reinterpret_cast<u32x4 *>(dg + row * ld + c) = wg;
        *reinterpret_cast<u32x4 *>(du + row * ld + c) = wu;
    }
}

// four neighbouring sums a lane; a part's rows follow one another without a gap
template <bool VEC>
__global__ __launch_bounds__(kThreads) void join_kernel(const float *work, int parts, int64_t rows, int64_t cols, fp8_matrix out)
{
    const int64_t runs = (cols + 3) / 4, total = rows * runs, part = rows * cols;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= total) return;
    const int64_t row = i / runs, c = (i - row * runs) * 4, count = cols - c;
    const float *p = work + row * cols + c;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = 0; k < parts; k++, p += part)
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (j < count) sum[j] += p[j];
    store4<VEC>(out, row, c, count, sum);
}

// The parts' sums of G and U, [part][G, U][rows][cols], added, and what the gated block makes of them; a wave's items as in encode_kernel.
template <bool VEC>
__global__ __launch_bounds__(kThreads) void gated_join_kernel(const float *work, int parts, int64_t rows, int64_t cols, int act, fp8_matrix h,
                                                              uint8_t *hc, uint8_t *he, uint8_t *gc, uint8_t *ge, uint8_t *uc, uint8_t *ue, int tiles)
{
    const int lane = threadIdx.x % kWave;
    const int64_t items = rows * tiles, step = (int64_t)gridDim.x * kWaves, code_row = (cols + kFp8Block - 1) / kFp8Block * kFp8Block, exp_row = (int64_t)tiles * 4;
    for (int64_t item = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave); item < items; item += step) {
        const int64_t row = item / tiles, tile = item - row * tiles, c = tile * kItem + 8 * lane;
        float g[8] = {}, u[8] = {}, v[8];
        for (int p = 0; p < parts; p++) {
            float a[8], b[8];
            const float *from = work + (int64_t)p * 2 * rows * cols + row * cols;
            load8<PVQ_F32, VEC>(from, c, cols, a);
            load8<PVQ_F32, VEC>(from + rows * cols, c, cols, b);
#pragma unroll
            for (int i = 0; i < 8; i++) { g[i] += a[i]; u[i] += b[i]; }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = act_value(act, g[i]) * u[i];
        if (h.data)
#pragma unroll
            for (int i = 0; i < 8; i += 4)
                if (c + i < cols) store4<false>(h, row, c + i, cols - c - i, f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]});
        auto to_blocks = [&](uint8_t *codes, uint8_t *exps, const float (&w)[8]) {
            if (!codes) return;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) top = max(top, finite_bits(w[i]));
            store_codes(codes + row * code_row, exps + row * exp_row, tile, c, code_row, lane, w, block_max(top));
        };
        to_blocks(gc, ge, g);
        to_blocks(uc, ue, u);
        to_blocks(hc, he, v);
    }
}

// a lane eight values
__global__ __launch_bounds__(kThreads) void align_kernel(fp8_bf16 from, uint16_t *to, int64_t ld)
{
    const int64_t runs = ld / 8, total = from.rows * runs;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
        const int64_t row = i / runs, c = (i - row * runs) * 8;
        const uint16_t *p = from.data + row * from.ld + c;
        u32x4 w = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (c + e < from.cols) w[e / 2] |= (uint32_t)p[e] << (16 * (e & 1));
        *reinterpret_cast<u32x4 *>(to + row * ld + c) = w;
    }
}

unsigned grid_for(int64_t work, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min(work, most)); }

bool aligned_rows(const void *p, int64_t ld, int size, int bytes) { return (uintptr_t)p % bytes == 0 && (ld * size) % bytes == 0; }

template <int T>
hipError_t launch_encode(const void *X, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes, uint8_t *exps, hipStream_t s)
{
    using E = typename element<T>::type;
    const fp8_blocks b{codes, exps, rows, cols};
    const int tiles = (int)((b.blocks() + 3) / 4);
    const unsigned grid = grid_for((rows * tiles + kWaves - 1) / kWaves, 256 * 8 * 4);
    if (aligned_rows(X, ldx, sizeof(E), 16))
        hipLaunchKernelGGL((encode_kernel<T, true>), dim3(grid), dim3(kThreads), 0, s, (const E *)X, rows, cols, ldx, codes, exps, b.code_row(), b.exp_row(), tiles);
    else
        hipLaunchKernelGGL((encode_kernel<T, false>), dim3(grid), dim3(kThreads), 0, s, (const E *)X, rows, cols, ldx, codes, exps, b.code_row(), b.exp_row(), tiles);
    return hipGetLastError();
}

bool vector_rows(const fp8_matrix &y)
{
    const int size = y.dtype == PVQ_F32 ? 4 : 2;
    return aligned_rows(y.data, y.ld, size, 4 * size);
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
    if (vector_rows(y)) hipLaunchKernelGGL(decode_kernel<true>, dim3(grid), dim3(kThreads), 0, s, b, y, tiles);
    else hipLaunchKernelGGL(decode_kernel<false>, dim3(grid), dim3(kThreads), 0, s, b, y, tiles);
    return hipGetLastError();
}

hipError_t fp8_launch_gated_slopes(const fp8_bf16 &dh, const fp8_blocks &g, const fp8_blocks &u, int act, uint16_t *dg, uint16_t *du,
                                   int64_t ld, hipStream_t s)
{
    const unsigned grid = grid_for((dh.rows * (ld / 8) + kThreads - 1) / kThreads, 256 * 8 * 4);
    if (aligned_rows(dh.data, dh.ld, 2, 16)) hipLaunchKernelGGL(slopes_kernel<true>, dim3(grid), dim3(kThreads), 0, s, dh, g, u, act, dg, du, ld);
    else hipLaunchKernelGGL(slopes_kernel<false>, dim3(grid), dim3(kThreads), 0, s, dh, g, u, act, dg, du, ld);
    return hipGetLastError();
}

hipError_t fp8_launch_join(const float *work, int parts, int64_t rows, int64_t cols, const fp8_matrix &out, hipStream_t s)
{
    const unsigned grid = (unsigned)((rows * ((cols + 3) / 4) + kThreads - 1) / kThreads);
    if (vector_rows(out)) hipLaunchKernelGGL(join_kernel<true>, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, out);
    else hipLaunchKernelGGL(join_kernel<false>, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, out);
    return hipGetLastError();
}

hipError_t fp8_launch_gated_join(const float *work, int parts, const fp8_gated_args &a, hipStream_t s)
{
    const int64_t rows = a.x.rows, cols = a.gate.rows;
    const int tiles = (int)((cols + kItem - 1) / kItem);
    const unsigned grid = grid_for((rows * tiles + kWaves - 1) / kWaves, 256 * 8 * 4);
    if (cols % 4 == 0)
        hipLaunchKernelGGL(gated_join_kernel<true>, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, a.act, a.h, a.hc, a.he, a.gc, a.ge, a.uc, a.ue, tiles);
    else
        hipLaunchKernelGGL(gated_join_kernel<false>, dim3(grid), dim3(kThreads), 0, s, work, parts, rows, cols, a.act, a.h, a.hc, a.he, a.gc, a.ge, a.uc, a.ue, tiles);
    return hipGetLastError();
}

hipError_t fp8_launch_align(const fp8_bf16 &from, uint16_t *to, int64_t ld, hipStream_t s)
{
    const unsigned grid = grid_for((from.rows * (ld / 8) + kThreads - 1) / kThreads, 256 * 8 * 4);
    hipLaunchKernelGGL(align_kernel, dim3(grid), dim3(kThreads), 0, s, from, to, ld);
    return hipGetLastError();
}
