// Gradients of products: a bfloat16 matrix times an 8-bit block matrix along the blocks' rows.
#include "pvq_fp8_wide.h"

using namespace pvq_fp8_dev;

namespace {

template <int KIND>
__global__ __launch_bounds__(256) void grad_kernel(wide_args t)
{
    extern __shared__ __align__(16) uint8_t lds[];
    int ti, tj, first, last;
    tile_of(t.tiles_i, t.tiles_j, chiplet_order(blockIdx.x, gridDim.x), ti, tj);
    const int64_t i0 = (int64_t)ti * kWideTile, j0 = (int64_t)tj * kWideTile;
    const int out_of = blockIdx.y / t.parts;
    wide_steps(t, blockIdx.y % t.parts, first, last);
    f32x4 acc[8][8];
    wide_sums<KIND, false>(t, lds, i0, j0, out_of, first, last, acc);
    const fp8_matrix out = t.parts > 1 ? part_of(t.work, blockIdx.y, t.rows, t.cols) : out_of ? t.out[1] : t.out[0];
    store_plain(out, t.rows, t.cols, lds, acc, i0, j0);
}

// the parts of the sum of an output's tiles
int parts_of(int64_t rows, int64_t cols, int64_t depth, int terms, int outputs)
{
    const int64_t tiles = ((rows + kWideTile - 1) / kWideTile) * ((cols + kWideTile - 1) / kWideTile) * outputs;
    return fp8_parts(tiles, (depth + kWideStep - 1) / kWideStep * terms, kWideStepUs, rows * cols * outputs);
}

size_t work_of(int64_t rows, int64_t cols, int64_t depth, int terms, int outputs)
{
    const int parts = parts_of(rows, cols, depth, terms, outputs);
    return parts > 1 ? (size_t)parts * outputs * rows * cols * 4 : 0;
}

template <int KIND>
hipError_t launch(wide_args &t, const fp8_grad_args &g, int outputs, hipStream_t s)
{
    const auto kernel = &grad_kernel<KIND>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kWideLds);
    if (e != hipSuccess) return e;
    for (int i = 0; i < g.pairs; i++) { t.dy[i] = g.dy[i]; t.b[i] = g.b[i]; }
    for (int i = 0; i < outputs; i++) t.out[i] = g.out[i];
    t.tiles_i = (int)((t.rows + kWideTile - 1) / kWideTile);
    t.tiles_j = (int)((t.cols + kWideTile - 1) / kWideTile);
    t.work = g.work;
    t.parts = parts_of(t.rows, t.cols, t.depth, t.terms, outputs);
    t.steps_a_part = (int)(((t.depth + kWideStep - 1) / kWideStep * t.terms + t.parts - 1) / t.parts);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(t.tiles_i * t.tiles_j), (unsigned)(outputs * t.parts)), dim3(256), kWideLds, s, t);
    e = hipGetLastError();
    for (int i = 0; i < outputs && t.parts > 1 && e == hipSuccess; i++)
        e = fp8_launch_join(t.work + (int64_t)i * t.parts * t.rows * t.cols, t.parts, t.rows, t.cols, t.out[i], s);
    return e;
}

}  // namespace

size_t fp8_input_grad_work(int64_t m, int64_t n, int64_t k, int pairs) { return work_of(m, k, n, pairs, 1); }
size_t fp8_weight_grad_work(int64_t m, int64_t n, int64_t k, int pairs) { return work_of(n, k, m, 1, pairs); }

hipError_t fp8_launch_input_grad(const fp8_grad_args &g, hipStream_t s)
{
    wide_args t{};
    t.rows = g.dy[0].rows; t.cols = g.b[0].cols; t.depth = g.dy[0].cols; t.terms = g.pairs;
    return launch<WIDE_INPUT_GRAD>(t, g, 1, s);
}

hipError_t fp8_launch_weight_grad(const fp8_grad_args &g, hipStream_t s)
{
    wide_args t{};
    t.rows = g.dy[0].cols; t.cols = g.b[0].cols; t.depth = g.dy[0].rows; t.terms = 1;
    return launch<WIDE_WEIGHT_GRAD>(t, g, g.pairs, s);
}
