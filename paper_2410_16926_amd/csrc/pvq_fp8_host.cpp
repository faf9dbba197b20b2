// 8-bit blocks: the C entries, checks of their arguments.
#include "pvq_diagnostics.h"
#include "pvq_fp8.h"

namespace {

constexpr int64_t kMostCols = 1 << 22;        // a tile's rows stay within 32-bit offsets
constexpr int64_t kMostRows = 1 << 30;
constexpr int64_t kMostValues = (int64_t)1 << 41;      // of one matrix: far beyond the memory of a GPU, and what the numbers of tiles are counted for

bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }
size_t size_of(int dtype) { return dtype == PVQ_F32 ? 4 : 2; }
bool known(int dtype) { return dtype == PVQ_F32 || dtype == PVQ_F16 || dtype == PVQ_BF16; }
int status_of(hipError_t e) { return e == hipSuccess ? PVQ_OK : pvq_hip_fail(e); }

int check_shape(int64_t rows, int64_t cols)
{
    if (rows < 0 || cols < 0) return PVQ_E_INVALID_ARG;
    return cols > kMostCols || rows > kMostRows || rows * cols > kMostValues ? PVQ_E_UNSUPPORTED : PVQ_OK;
}

// a matrix of floats that no operand's row is: its columns may be as many as rows
int check_result(int64_t rows, int64_t cols) { return rows > 0 && cols > kMostValues / rows ? PVQ_E_UNSUPPORTED : PVQ_OK; }

// both planes there and aligned; an empty matrix has none
int check_blocks(const fp8_blocks &b)
{
    if (b.rows == 0 || b.cols == 0) return PVQ_OK;
    if (!b.codes || !b.exps) return PVQ_E_INVALID_ARG;
    return aligned(b.codes, 16) && aligned(b.exps, 4) ? PVQ_OK : PVQ_E_ALIGNMENT;
}

int check_matrix(const void *p, int dtype, int64_t cols, int64_t ld)
{
    if (!p || ld < cols) return PVQ_E_INVALID_ARG;
    return aligned(p, size_of(dtype)) ? PVQ_OK : PVQ_E_ALIGNMENT;
}

int check_work(const void *work, size_t have, size_t wanted)
{
    if (wanted == 0) return PVQ_OK;
    if (!work || have < wanted) return PVQ_E_INVALID_ARG;
    return aligned(work, 16) ? PVQ_OK : PVQ_E_ALIGNMENT;
}

int first_of(std::initializer_list<int> codes)
{
    for (const int rc : codes) if (rc) return rc;
    return PVQ_OK;
}

// the row stride of a workspace's bfloat16 matrices, in values
int64_t slope_row(int64_t n) { return (n + 63) / 64 * 64; }

// Of how many pieces of bfloat16 the gated block's dG and dU are.  Rounded once they are off by half a step, 2^-8, which is what a result in
// bfloat16 is off by anyway (2.3e-3 in all instead of 1.7e-3, in half the time).  A result of more bits takes a second piece, what the first left,
// and is off by 2^-16 of a slope at most: float32 gradients of 517 x 2816 x 1024 by 2.5e-6 (one piece: 1.7e-3; float32 slopes: 4e-7 to 1e-6), float16
// ones by no more than their own rounding, 2.1e-4 (1.7e-3).  2048 x 14336 x 4096 takes 1.6 ms with two pieces, 0.84 with one.
int slope_pieces(int out_dtype) { return out_dtype == PVQ_BF16 ? 1 : 2; }
constexpr int kMostPieces = 2;

// Whether the gradient kernels of large tiles can take dY as it is: rows aligned to 16 bytes, a tile's within 32-bit offsets, and where they run along
// the sum (dX) in whole steps of it.  Otherwise it is copied first, with zeros behind the rows.
bool whole_rows(const void *dY, int64_t ld, int64_t n, bool along) { return aligned(dY, 16) && ld % 8 == 0 && ld <= kMostCols && (!along || n % 64 == 0); }

// whether the kernel that streams the weights takes the gated block
bool gated_by_rows(int64_t m, bool to_blocks, int64_t k) { return fp8_rows_pay(m) && !to_blocks && k > 0; }

size_t up16(size_t v) { return (v + 15) / 16 * 16; }

size_t copy_bytes(const void *dY, int64_t ld, int64_t m, int64_t n, int64_t k, bool along)
{
    const bool as_it_is = along ? fp8_input_grad_as_it_is(m, n, k) : fp8_weight_grad_as_it_is(m, n, k);
    return as_it_is || whole_rows(dY, ld, n, along) ? 0 : up16((size_t)m * slope_row(n) * 2);
}

// a gradient's dY, copied to the front of its workspace where it has to be; the split's sums behind it
hipError_t take_dy(fp8_grad_args &a, void *work, size_t copy, hipStream_t s)
{
    a.work = (float *)((char *)work + copy);
    if (copy == 0) return hipSuccess;
    const fp8_bf16 from = a.dy[0];
    a.dy[0] = {(const uint16_t *)work, from.rows, from.cols, slope_row(from.cols)};
    return fp8_launch_align(from, (uint16_t *)work, a.dy[0].ld, s);
}

}  // namespace

extern "C" int pvq_fp8_sizes(int64_t rows, int64_t cols, size_t *code_bytes, size_t *exponent_bytes)
{
    if (const int rc = check_shape(rows, cols)) return rc;
    const fp8_blocks b{nullptr, nullptr, rows, cols};
    if (code_bytes) *code_bytes = (size_t)(rows * b.code_row());
    if (exponent_bytes) *exponent_bytes = (size_t)(rows * b.exp_row());
    return PVQ_OK;
}

extern "C" int pvq_fp8_encode(const void *X, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes, uint8_t *exponents,
                              void *stream)
{
    if (const int rc = check_shape(rows, cols)) return rc;
    if (!known(dtype)) return PVQ_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return PVQ_OK;
    if (const int rc = first_of({check_matrix(X, dtype, cols, ldx), check_blocks({codes, exponents, rows, cols})})) return rc;
    return status_of(fp8_launch_encode(X, dtype, rows, cols, ldx, codes, exponents, (hipStream_t)stream));
}

extern "C" int pvq_fp8_decode(const uint8_t *codes, const uint8_t *exponents, int64_t rows, int64_t cols, void *Y, int out_dtype, int64_t ldy,
                              void *stream)
{
    if (const int rc = check_shape(rows, cols)) return rc;
    if (!known(out_dtype)) return PVQ_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return PVQ_OK;
    const fp8_blocks b{codes, exponents, rows, cols};
    if (const int rc = first_of({check_matrix(Y, out_dtype, cols, ldy), check_blocks(b)})) return rc;
    return status_of(fp8_launch_decode(b, {Y, out_dtype, ldy}, (hipStream_t)stream));
}

extern "C" int pvq_fp8_product_work_bytes(int64_t m, int64_t n, int64_t k, int out_dtype, size_t *bytes)
{
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), check_result(m, n)})) return rc;
    if (!known(out_dtype) || !bytes) return PVQ_E_INVALID_ARG;
    *bytes = m && n && k ? fp8_product_work(m, n, k, out_dtype) : 0;
    return PVQ_OK;
}

extern "C" int pvq_fp8_product(const uint8_t *a_codes, const uint8_t *a_exponents, int64_t m, const uint8_t *b_codes,
                               const uint8_t *b_exponents, int64_t n, int64_t k, void *Y, int out_dtype, int64_t ldy, void *work,
                               size_t work_bytes, void *stream)
{
    size_t wanted = 0;
    if (const int rc = pvq_fp8_product_work_bytes(m, n, k, out_dtype, &wanted)) return rc;
    if (m == 0 || n == 0) return PVQ_OK;
    fp8_product_args a;
    a.a = {a_codes, a_exponents, m, k};
    a.b = {b_codes, b_exponents, n, k};
    a.y = {Y, out_dtype, ldy};
    a.work = (float *)work;
    if (const int rc = first_of({check_matrix(Y, out_dtype, n, ldy), check_blocks(a.a), check_blocks(a.b), check_work(work, work_bytes, wanted)})) return rc;
    if (k == 0) return status_of(fp8_launch_join(nullptr, 0, m, n, a.y, (hipStream_t)stream));
    return status_of(fp8_rows_pay(m) ? fp8_launch_product_rows(a, (hipStream_t)stream) : fp8_launch_product(a, (hipStream_t)stream));
}

extern "C" int pvq_fp8_input_grad_work_bytes(const void *dY, int64_t lddy, int64_t m, int64_t n, int64_t k, size_t *bytes)
{
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), check_shape(m, n)})) return rc;
    if (!bytes) return PVQ_E_INVALID_ARG;
    *bytes = m && n && k ? copy_bytes(dY, lddy, m, n, k, true) + fp8_input_grad_work(m, n, k, 1, 1) : 0;
    return PVQ_OK;
}

extern "C" int pvq_fp8_input_grad(const void *dY, int64_t lddy, int64_t m, const uint8_t *w_codes, const uint8_t *w_exponents, int64_t n,
                                  int64_t k, void *dX, int out_dtype, int64_t lddx, void *work, size_t work_bytes, void *stream)
{
    size_t wanted = 0;
    if (const int rc = pvq_fp8_input_grad_work_bytes(dY, lddy, m, n, k, &wanted)) return rc;
    if (!known(out_dtype)) return PVQ_E_INVALID_ARG;
    if (m == 0 || k == 0) return PVQ_OK;
    fp8_grad_args a{};
    a.pairs = a.pieces = 1;
    a.dy[0] = {(const uint16_t *)dY, m, n, lddy};
    a.b[0] = {w_codes, w_exponents, n, k};
    a.out[0] = {dX, out_dtype, lddx};
    if (const int rc = first_of({check_matrix(dX, out_dtype, k, lddx), n ? check_matrix(dY, PVQ_BF16, n, lddy) : PVQ_OK, check_blocks(a.b[0]),
                                 check_work(work, work_bytes, wanted)}))
        return rc;
    const hipStream_t s = (hipStream_t)stream;
    if (n == 0) return status_of(fp8_launch_join(nullptr, 0, m, k, a.out[0], s));
    const hipError_t e = take_dy(a, work, copy_bytes(dY, lddy, m, n, k, true), s);
    return status_of(e == hipSuccess ? fp8_launch_input_grad(a, s) : e);
}

extern "C" int pvq_fp8_weight_grad_work_bytes(const void *dY, int64_t lddy, int64_t m, int64_t n, int64_t k, size_t *bytes)
{
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), check_shape(m, n)})) return rc;
    if (!bytes) return PVQ_E_INVALID_ARG;
    *bytes = m && n && k ? copy_bytes(dY, lddy, m, n, k, false) + fp8_weight_grad_work(m, n, k, 1, 1) : 0;
    return PVQ_OK;
}

extern "C" int pvq_fp8_weight_grad(const void *dY, int64_t lddy, int64_t m, int64_t n, const uint8_t *x_codes, const uint8_t *x_exponents,
                                   int64_t k, void *dW, int out_dtype, int64_t lddw, void *work, size_t work_bytes, void *stream)
{
    size_t wanted = 0;
    if (const int rc = pvq_fp8_weight_grad_work_bytes(dY, lddy, m, n, k, &wanted)) return rc;
    if (!known(out_dtype)) return PVQ_E_INVALID_ARG;
    if (n == 0 || k == 0) return PVQ_OK;
    fp8_grad_args a{};
    a.pairs = a.pieces = 1;
    a.dy[0] = {(const uint16_t *)dY, m, n, lddy};
    a.b[0] = {x_codes, x_exponents, m, k};
    a.out[0] = {dW, out_dtype, lddw};
    if (const int rc = first_of({check_matrix(dW, out_dtype, k, lddw), m ? check_matrix(dY, PVQ_BF16, n, lddy) : PVQ_OK, check_blocks(a.b[0]),
                                 check_work(work, work_bytes, wanted)}))
        return rc;
    const hipStream_t s = (hipStream_t)stream;
    if (m == 0) return status_of(fp8_launch_join(nullptr, 0, n, k, a.out[0], s));
    const hipError_t e = take_dy(a, work, copy_bytes(dY, lddy, m, n, k, false), s);
    return status_of(e == hipSuccess ? fp8_launch_weight_grad(a, s) : e);
}

extern "C" int pvq_fp8_gated_work_bytes(int64_t m, int64_t n, int64_t k, int out_dtype, int to_blocks, size_t *bytes)
{
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), check_shape(m, n)})) return rc;
    if (!known(out_dtype) || !bytes) return PVQ_E_INVALID_ARG;
    *bytes = m && n && k && (to_blocks || !fp8_rows_pay(m)) ? std::max(fp8_gated_work(m, n, k, false, to_blocks), fp8_gated_work(m, n, k, true, to_blocks)) : 0;
    return PVQ_OK;
}

extern "C" int pvq_fp8_gated(const uint8_t *x_codes, const uint8_t *x_exponents, int64_t m, const uint8_t *gate_codes,
                             const uint8_t *gate_exponents, const uint8_t *up_codes, const uint8_t *up_exponents, int64_t n, int64_t k,
                             int activation, void *H, int out_dtype, int64_t ldh, uint8_t *h_codes, uint8_t *h_exponents, uint8_t *g_codes,
                             uint8_t *g_exponents, uint8_t *u_codes, uint8_t *u_exponents, void *work, size_t work_bytes, void *stream)
{
    const bool keep = g_codes || g_exponents || u_codes || u_exponents, encoded = h_codes || h_exponents;
    size_t wanted = 0;
    if (const int rc = pvq_fp8_gated_work_bytes(m, n, k, out_dtype, keep || encoded, &wanted)) return rc;
    if (activation != PVQ_SILU && activation != PVQ_GELU) return PVQ_E_INVALID_ARG;
    if (m == 0 || n == 0) return PVQ_OK;
    if (!H && !encoded) return PVQ_E_INVALID_ARG;
    fp8_gated_args a{};
    a.x = {x_codes, x_exponents, m, k};
    a.gate = {gate_codes, gate_exponents, n, k};
    a.up = {up_codes, up_exponents, n, k};
    a.act = activation;
    a.h = {H, out_dtype, ldh};
    a.hc = h_codes; a.he = h_exponents; a.gc = g_codes; a.ge = g_exponents; a.uc = u_codes; a.ue = u_exponents;
    a.work = (float *)work;
    if (const int rc = first_of({H ? check_matrix(H, out_dtype, n, ldh) : PVQ_OK, check_blocks(a.x), check_blocks(a.gate), check_blocks(a.up),
                                 encoded ? check_blocks({h_codes, h_exponents, m, n}) : PVQ_OK, keep ? check_blocks({g_codes, g_exponents, m, n}) : PVQ_OK,
                                 keep ? check_blocks({u_codes, u_exponents, m, n}) : PVQ_OK, check_work(work, work_bytes, wanted)}))
        return rc;
    return status_of(gated_by_rows(m, keep || encoded, k) ? fp8_launch_gated_rows(a, (hipStream_t)stream) : fp8_launch_gated(a, (hipStream_t)stream));
}

extern "C" int pvq_fp8_gated_backward_work_bytes(int64_t m, int64_t n, int64_t k, size_t *bytes)
{
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), check_shape(m, n)})) return rc;
    if (!bytes) return PVQ_E_INVALID_ARG;
    // (enough for every type of the results)
    const size_t slopes = (size_t)m * slope_row(n) * 2;
    size_t sums = 0;
    for (int pieces = 1; m && n && k && pieces <= kMostPieces; pieces++)
        sums = std::max({sums, fp8_input_grad_work(m, n, k, 2, pieces), fp8_weight_grad_work(m, n, k, 2, pieces)});
    *bytes = 2 * kMostPieces * slopes + sums;
    return PVQ_OK;
}

extern "C" int pvq_fp8_gated_backward(const void *dH, int64_t lddh, const uint8_t *x_codes, const uint8_t *x_exponents, int64_t m,
                                      const uint8_t *gate_codes, const uint8_t *gate_exponents, const uint8_t *up_codes,
                                      const uint8_t *up_exponents, int64_t n, int64_t k, const uint8_t *g_codes, const uint8_t *g_exponents,
                                      const uint8_t *u_codes, const uint8_t *u_exponents, int activation, void *dX, int64_t lddx, void *dWg,
                                      void *dWu, int64_t lddw, int out_dtype, void *work, size_t work_bytes, void *stream)
{
    size_t wanted = 0;
    if (const int rc = pvq_fp8_gated_backward_work_bytes(m, n, k, &wanted)) return rc;
    if (!known(out_dtype)) return PVQ_E_INVALID_ARG;
    if (activation != PVQ_SILU && activation != PVQ_GELU) return PVQ_E_INVALID_ARG;
    if (!dWg != !dWu || (!dX && !dWg)) return PVQ_E_INVALID_ARG;
    if (k == 0) return PVQ_OK;
    const fp8_blocks x{x_codes, x_exponents, m, k}, gate{gate_codes, gate_exponents, n, k}, up{up_codes, up_exponents, n, k};
    const fp8_blocks g{g_codes, g_exponents, m, n}, u{u_codes, u_exponents, m, n};
    if (const int rc = first_of({dX ? check_matrix(dX, out_dtype, k, lddx) : PVQ_OK, dWg ? check_matrix(dWg, out_dtype, k, lddw) : PVQ_OK,
                                 dWu ? check_matrix(dWu, out_dtype, k, lddw) : PVQ_OK, m && n ? check_matrix(dH, PVQ_BF16, n, lddh) : PVQ_OK,
                                 check_blocks(x), check_blocks(gate), check_blocks(up), check_blocks(g), check_blocks(u),
                                 check_work(work, work_bytes, wanted)}))
        return rc;
    const hipStream_t s = (hipStream_t)stream;
    hipError_t e = hipSuccess;
    if (m == 0 || n == 0) {
        // empty sums
        if (dX && m) e = fp8_launch_join(nullptr, 0, m, k, {dX, out_dtype, lddx}, s);
        if (dWg && n && e == hipSuccess) e = fp8_launch_join(nullptr, 0, n, k, {dWg, out_dtype, lddw}, s);
        if (dWu && n && e == hipSuccess) e = fp8_launch_join(nullptr, 0, n, k, {dWu, out_dtype, lddw}, s);
        return status_of(e);
    }
    const int64_t ld = slope_row(n), slopes = m * ld;
    fp8_grad_args a{};
    a.pairs = 2;
    a.pieces = slope_pieces(out_dtype);
    uint16_t *dg = (uint16_t *)work, *du = dg + a.pieces * slopes;
    for (int i = 0; i < a.pairs * a.pieces; i++) a.dy[i] = {dg + i * slopes, m, n, ld};
    a.work = (float *)(dg + 2 * kMostPieces * slopes);
    e = fp8_launch_gated_slopes({(const uint16_t *)dH, m, n, lddh}, g, u, activation, dg, du, a.pieces, ld, s);
    if (dX && e == hipSuccess) {
        a.b[0] = gate; a.b[1] = up;
        a.out[0] = {dX, out_dtype, lddx};
        e = fp8_launch_input_grad(a, s);
    }
    if (dWg && e == hipSuccess) {
        a.b[0] = x; a.b[1] = x;
        a.out[0] = {dWg, out_dtype, lddw};
        a.out[1] = {dWu, out_dtype, lddw};
        e = fp8_launch_weight_grad(a, s);
    }
    return status_of(e);
}

extern "C" int pvq_fp8_plan(int what, int64_t m, int64_t n, int64_t k, int out_dtype, int *kind, int *parts)
{
    if (m < 1 || n < 1 || k < 1 || !known(out_dtype) || !kind || !parts) return PVQ_E_INVALID_ARG;
    if (const int rc = first_of({check_shape(m, k), check_shape(n, k), what == PVQ_FP8_PRODUCT ? check_result(m, n) : check_shape(m, n)})) return rc;
    const int pieces = slope_pieces(out_dtype);
    const bool to_blocks = what == PVQ_FP8_GATED_TO_BLOCKS || what == PVQ_FP8_GATED_KEPT;
    fp8_tiles t{};
    bool by_rows = false;
    switch (what) {
    case PVQ_FP8_PRODUCT:
        by_rows = fp8_rows_pay(m);
        t = fp8_product_tiles(m, n, k, false, out_dtype == PVQ_F32, false);
        break;
    case PVQ_FP8_GATED: case PVQ_FP8_GATED_TO_BLOCKS: case PVQ_FP8_GATED_KEPT:
        by_rows = gated_by_rows(m, to_blocks, k);
        t = fp8_product_tiles(m, n, k, true, fp8_gated_is_wide(what == PVQ_FP8_GATED_KEPT, what != PVQ_FP8_GATED_TO_BLOCKS, out_dtype), to_blocks);
        break;
    case PVQ_FP8_INPUT_GRAD: t = fp8_input_grad_tiles(m, n, k, 1, 1); break;
    case PVQ_FP8_WEIGHT_GRAD: t = fp8_weight_grad_tiles(m, n, k, 1, 1); break;
    case PVQ_FP8_GATED_INPUT_GRAD: t = fp8_input_grad_tiles(m, n, k, 2, pieces); break;
    case PVQ_FP8_GATED_WEIGHT_GRADS: t = fp8_weight_grad_tiles(m, n, k, 2, pieces); break;
    default: return PVQ_E_INVALID_ARG;
    }
    *kind = by_rows ? PVQ_FP8_BY_ROWS : t.rows == 0 ? PVQ_FP8_TILES_8BIT : t.rows == 64 ? PVQ_FP8_TILES_64 : t.rows == 128 ? PVQ_FP8_TILES_128 : PVQ_FP8_TILES_256;
    *parts = by_rows ? 1 : t.parts;
    return PVQ_OK;
}
