// Gradients of products: a bfloat16 matrix times an 8-bit block matrix along the blocks' rows.
#include "pvq_fp8_small.h"

using namespace pvq_fp8_dev;

namespace {

template <int KIND, int FI>
__global__ __launch_bounds__(256) void grad_kernel(wide_args t)
{
    extern __shared__ __align__(16) uint8_t lds[];
    wide_sums<KIND, false, FI>(t, lds, t.units, [&](int u) { return wide_unit_of<false, FI>(argument<wide_args>(), u); }, [&](const wide_unit &u, const f32x4 (&acc)[FI][8]) {
        const wide_args &t = argument<wide_args>();
        const fp8_matrix out = t.parts > 1 ? part_of(t.work, u.out_of * t.parts + u.part, t.rows, t.cols) : u.out_of ? t.out[1] : t.out[0];
        store_sums(out, t.rows, t.cols, acc, u.i0, u.j0);
    });
}

template <int KIND>
__global__ __launch_bounds__(256, 4) void small_grad_kernel(wide_args t)
{
    __shared__ __align__(16) uint8_t lds[kSmallLds];
    small_tile<KIND, false>(t, lds, [&](const wide_unit &u, int64_t row, int64_t col, f32x4 first, f32x4 second) {
        const fp8_matrix out = t.parts > 1 ? part_of(t.work, u.out_of * t.parts + u.part, t.rows, t.cols) : u.out_of ? t.out[1] : t.out[0];
        store_four(out, row, col, t.cols, first);
        store_four(out, row, col + 16, t.cols, second);
    });
}

size_t work_of(int64_t rows, int64_t cols, int64_t depth, int terms, int outputs)
{
    const int parts = wide_plan(rows, cols, depth, terms, outputs).parts;
    return parts > 1 ? (size_t)parts * outputs * rows * cols * 4 : 0;
}

template <int KIND>
hipError_t launch(wide_args &t, const fp8_grad_args &g, int outputs, hipStream_t s)
{
    for (int i = 0; i < g.pairs * g.pieces; i++) t.dy[i] = g.dy[i];
    for (int i = 0; i < g.pairs; i++) t.b[i] = g.b[i];
    t.pieces = g.pieces;
    for (int i = 0; i < outputs; i++) t.out[i] = g.out[i];
    t.work = g.work;
    const wide_tiles plan = wide_plan(t.rows, t.cols, t.depth, t.terms, outputs);
    t.use(plan, outputs);
    hipError_t e = hipSuccess;
    if (plan.rows == kSmallTile) hipLaunchKernelGGL(small_grad_kernel<KIND>, dim3((unsigned)t.units), dim3(256), 0, s, t);
    else {
        const auto kernel = plan.rows == 128 ? &grad_kernel<KIND, 4> : &grad_kernel<KIND, 8>;
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kWideLds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(t.units, 256)), dim3(256), kWideLds, s, t);
    }
    e = hipGetLastError();
    for (int i = 0; i < outputs && t.parts > 1 && e == hipSuccess; i++)
        e = fp8_launch_join(t.work + (int64_t)i * t.parts * t.rows * t.cols, t.parts, t.rows, t.cols, t.out[i], s);
    return e;
}

}  // namespace

// (a copy takes 4 us; rows that start anywhere a little more each step: dX of 333 x 3001 x 11008 in small tiles 83 us, with a copy 78)
static bool as_it_is(const wide_tiles &plan) { return plan.rows == kSmallTile && plan.us < 14.0; }
bool fp8_input_grad_as_it_is(int64_t m, int64_t n, int64_t k) { return as_it_is(wide_plan(m, k, n, 1, 1)); }
bool fp8_weight_grad_as_it_is(int64_t m, int64_t n, int64_t k) { return as_it_is(wide_plan(n, k, m, 1, 1)); }
static fp8_tiles tiles_of(const wide_tiles &t) { return {t.rows, t.parts}; }
fp8_tiles fp8_input_grad_tiles(int64_t m, int64_t n, int64_t k, int pairs, int pieces) { return tiles_of(wide_plan(m, k, n, pairs * pieces, 1)); }
fp8_tiles fp8_weight_grad_tiles(int64_t m, int64_t n, int64_t k, int pairs, int pieces) { return tiles_of(wide_plan(n, k, m, pieces, pairs)); }
size_t fp8_input_grad_work(int64_t m, int64_t n, int64_t k, int pairs, int pieces) { return work_of(m, k, n, pairs * pieces, 1); }
size_t fp8_weight_grad_work(int64_t m, int64_t n, int64_t k, int pairs, int pieces) { return work_of(n, k, m, pieces, pairs); }

hipError_t fp8_launch_input_grad(const fp8_grad_args &g, hipStream_t s)
{
    wide_args t{};
    t.rows = g.dy[0].rows; t.cols = g.b[0].cols; t.depth = g.dy[0].cols; t.terms = g.pairs * g.pieces;
    return launch<WIDE_INPUT_GRAD>(t, g, 1, s);
}

hipError_t fp8_launch_weight_grad(const fp8_grad_args &g, hipStream_t s)
{
    wide_args t{};
    t.rows = g.dy[0].cols; t.cols = g.b[0].cols; t.depth = g.dy[0].rows; t.terms = g.pieces;
    return launch<WIDE_WEIGHT_GRAD>(t, g, g.pairs, s);
}
