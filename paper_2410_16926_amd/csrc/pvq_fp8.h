// 8-bit block matrices: the interface between the checks of arguments (pvq_fp8_host.cpp) and the kernels
// (pvq_fp8_blocks.hip, pvq_fp8_product.hip, pvq_fp8_rows.hip, pvq_fp8_grad.hip).  Not installed; the contract is include/pvq.h.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <stdint.h>

#include "pvq.h"

// remembers the HIP error of a call for pvq_last_hip_error and returns PVQ_E_HIP (pvq_host.cpp)
int pvq_hip_fail(hipError_t e);

constexpr int kFp8Block = 128;        // values of one exponent

// A block matrix [rows][cols]: a row of codes takes whole blocks, a row of exponents whole words.
struct fp8_blocks {
    const uint8_t *codes = nullptr, *exps = nullptr;
    int64_t rows = 0, cols = 0;
#if defined(__HIPCC__)
    __host__ __device__
#endif
    int64_t blocks() const { return (cols + kFp8Block - 1) / kFp8Block; }
#if defined(__HIPCC__)
    __host__ __device__
#endif
    int64_t code_row() const { return blocks() * kFp8Block; }
#if defined(__HIPCC__)
    __host__ __device__
#endif
    int64_t exp_row() const { return (blocks() + 3) / 4 * 4; }
};

// A matrix of floats with unit column stride.
struct fp8_matrix {
    void *data = nullptr;
    int dtype = PVQ_F32;
    int64_t ld = 0;
};

// Into how many parts the sums of `tiles` tiles of `steps` steps are split: as many as take least (us), with a workgroup to a compute unit, a launch, 3 us
// around each tile's steps, and the parts' sums (values of them) written, and read again by a kernel that adds them.
constexpr double kByteStepUs = 1.4;                    // a step of a 256 x 256 tile: 128 of the sum on the 8-bit instruction
constexpr double kWideStepUs = 1.75, kLowStepUs = 1.2;  // 64 of the sum on the bfloat16 instruction; of a tile of 128 x 256 (short runs, at full clocks: 1.45 and 0.9)
inline int fp8_parts(int64_t tiles, int64_t steps, double step_us, int64_t values, double *takes = nullptr)
{
    int best = 1;
    double least = 0.0;
    for (int parts = 1; parts <= 32 && (parts == 1 || steps >= 2 * parts); parts++) {
        const double rounds = (double)((tiles * parts + 255) / 256);
        double us = 5.0 + rounds * ((double)((steps + parts - 1) / parts) * step_us + 3.0);
        if (parts > 1) us += 4.0 + 8.0 * parts * (double)values / 4e6;
        if (parts == 1 || us < least) { best = parts; least = us; }
    }
    if (takes) *takes = least;
    return best;
}

// The same for tiles of 64 x 64 (GATED: 32 hidden units), a step 64 of the sum.  Several workgroups share a unit and fill it between each other's waits.
// join: the parts' sums go to work and are added (or taken to blocks) by a kernel of its own, however few they are.
constexpr double kSmallStepUs = 0.3, kSmallBusyUs = 0.28;      // a step of a workgroup alone on its unit, and a unit's time for it where there are several (dX; the others 0.21)
inline int fp8_small_parts(int64_t tiles, int64_t steps, int64_t values, bool join, double *takes)
{
    int best = 1;
    double least = 0.0;
    for (int parts = 1; parts <= 16 && (parts == 1 || steps >= 8 * parts); parts++) {
        const double a_part = (double)((steps + parts - 1) / parts), a_unit = (double)((tiles * parts + 255) / 256);
        double us = 6.0 + a_part * std::max(kSmallStepUs, a_unit * kSmallBusyUs) + (double)(tiles * parts) * 0.003;
        if (parts > 1 || join) us += 4.0 + 8.0 * parts * (double)values / 4e6;
        if (parts == 1 || us < least) { best = parts; least = us; }
    }
    *takes = tiles > (1 << 20) ? 1e30 : least;                      // (a launch has less than 2^32 threads)
    return best;
}

// Y = A B^T.  work: float32 sums of the parts of a split (fp8_product_work), unused without one.
struct fp8_product_args {
    fp8_blocks a, b;
    fp8_matrix y;
    float *work;
};
size_t fp8_product_work(int64_t m, int64_t n, int64_t k, int out_dtype);
// the tiles that a product or the gated block takes (rows of 0: 256 on the 8-bit instruction) and the parts of their sums
struct fp8_tiles { int rows, parts; };
fp8_tiles fp8_product_tiles(int64_t m, int64_t n, int64_t k, bool gated, bool wide, bool to_blocks);
hipError_t fp8_launch_product(const fp8_product_args &a, hipStream_t s);

// H = act(X Wg^T) * (X Wu^T); h in floats (h.data) or in blocks (hc, he), and G and U in blocks where gc, ge, uc and ue are given
struct fp8_gated_args {
    fp8_blocks x, gate, up;
    int act;
    fp8_matrix h;
    uint8_t *hc, *he, *gc, *ge, *uc, *ue;
    float *work;
};
// Whether the gated block's sums are formed on the bfloat16 instruction whatever their number: for float32 results, and with kept products.  These
// are codes of sums of 32 bits: what the 8-bit instructions are off would change one code of 2000, which is as much again as the roundings of
// the gradients to bfloat16 (dX 3.0e-3 off instead of 2.3e-3).
inline bool fp8_gated_is_wide(bool kept, bool in_floats, int out_dtype) { return kept || (in_floats && out_dtype == PVQ_F32); }
// wide: as above; to_blocks: H in blocks, or G and U kept
size_t fp8_gated_work(int64_t m, int64_t n, int64_t k, bool wide, bool to_blocks);
hipError_t fp8_launch_gated(const fp8_gated_args &a, hipStream_t s);
// ... of the parts of G and U, [parts][2][rows][cols]
hipError_t fp8_launch_gated_join(const float *work, int parts, const fp8_gated_args &a, hipStream_t s);

// Few rows of A (tokens): the kernels that stream B (pvq_fp8_rows.hip).  The entries of pvq_fp8_host.cpp choose between these and the two above.
bool fp8_rows_pay(int64_t m);
hipError_t fp8_launch_product_rows(const fp8_product_args &a, hipStream_t s);
hipError_t fp8_launch_gated_rows(const fp8_gated_args &a, hipStream_t s);

// A bf16 matrix [rows][cols] with row stride ld.  The gradients' large tiles take rows aligned to 16 bytes and strides of at most 2^22 values, dX whole 64s
// of the sum or zeros behind a row; their small tiles rows that start and end anywhere, of any stride.  pvq_fp8_host.cpp sees to it (copy_bytes,
// take_dy): what is not so is copied, but for small tiles that are faster without (fp8_input_grad_as_it_is, fp8_weight_grad_as_it_is).
struct fp8_bf16 {
    const uint16_t *data = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
};

// dX = sum over p of dY_p W_p (one output) or dW_p = dY_p^T X_p (an output each), of one or two pairs.  A dY may be given in pieces whose sum it is:
// its rounding to bfloat16 and that of what was left.
struct fp8_grad_args {
    int pairs, pieces;
    fp8_bf16 dy[4];              // pair p's piece i: dy[p * pieces + i], all of one shape and stride
    fp8_blocks b[2];
    fp8_matrix out[2];
    float *work;
};
// whether a single gradient's dY is taken with rows that start and end anywhere, by small tiles
bool fp8_input_grad_as_it_is(int64_t m, int64_t n, int64_t k);
bool fp8_weight_grad_as_it_is(int64_t m, int64_t n, int64_t k);
fp8_tiles fp8_input_grad_tiles(int64_t m, int64_t n, int64_t k, int pairs, int pieces);
fp8_tiles fp8_weight_grad_tiles(int64_t m, int64_t n, int64_t k, int pairs, int pieces);
size_t fp8_input_grad_work(int64_t m, int64_t n, int64_t k, int pairs, int pieces);
size_t fp8_weight_grad_work(int64_t m, int64_t n, int64_t k, int pairs, int pieces);
hipError_t fp8_launch_input_grad(const fp8_grad_args &a, hipStream_t s);
hipError_t fp8_launch_weight_grad(const fp8_grad_args &a, hipStream_t s);

hipError_t fp8_launch_encode(const void *X, int dtype, int64_t rows, int64_t cols, int64_t ldx, uint8_t *codes, uint8_t *exps, hipStream_t s);
hipError_t fp8_launch_decode(const fp8_blocks &b, const fp8_matrix &y, hipStream_t s);
// dG = dH U act'(G), dU = dH act(G), each in one or two pieces of bf16, [piece][rows][ld], the columns from n to ld set to zero
hipError_t fp8_launch_gated_slopes(const fp8_bf16 &dh, const fp8_blocks &g, const fp8_blocks &u, int act, uint16_t *dg, uint16_t *du, int pieces,
                                   int64_t ld, hipStream_t s);
// a bf16 matrix to rows of `ld` values that start at 16 bytes, the columns behind the last zero
hipError_t fp8_launch_align(const fp8_bf16 &from, uint16_t *to, int64_t ld, hipStream_t s);
// the sums of a split, added in order: out = sum_p work[p], work [parts][rows][cols]
hipError_t fp8_launch_join(const float *work, int parts, int64_t rows, int64_t cols, const fp8_matrix &out, hipStream_t s);
