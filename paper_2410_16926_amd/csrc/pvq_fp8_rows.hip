// Products of a few rows (tokens) with 8-bit block weights.
#include "pvq_fp8_dev.h"

using namespace pvq_fp8_dev;

namespace {

struct rows_args {
    fp8_blocks a, b, up;
    fp8_matrix y;
    int act;
};

// A workgroup takes 16 rows of the weights (of both of them, GATED) and 16 FM tokens; its waves take the blocks of 128 in
// turn, straight from memory to registers: each weight is read once and used at once.  The codes are decoded to bfloat16,
// exactly, and the waves' float32 sums meet in LDS, added in the order of the waves.
// Bound by the weights' bytes: the decoding of 32 codes a lane is 16 instructions beside 32 bytes.
template <int FM, bool GATED>
__global__ __launch_bounds__(512) void rows_kernel(rows_args t)
{
    constexpr int kMats = GATED ? 2 : 1;
    extern __shared__ __align__(16) float sums[];                 // [wave][matrix][FM][lane][4]
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int r16 = lane % 16, quarter = lane / 16;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = t.b.rows, m = t.a.rows;
    const int64_t m0 = (int64_t)blockIdx.y * (16 * FM);
    const int64_t row_bytes = t.a.code_row(), exp_row = t.a.exp_row();
    const int blocks = (int)t.a.blocks();
    const int64_t wrow = min(n0 + r16, n - 1);
    const uint8_t *w[kMats], *we[kMats], *x[FM], *xe[FM];
#pragma unroll
    for (int i = 0; i < kMats; i++) {
        const fp8_blocks &b = i ? t.up : t.b;
        w[i] = b.codes + wrow * row_bytes + quarter * 32;
        we[i] = b.exps + wrow * exp_row;
    }
#pragma unroll
    for (int i = 0; i < FM; i++) {
        const int64_t row = min(m0 + i * 16 + r16, m - 1);
        x[i] = t.a.codes + row * row_bytes + quarter * 32;
        xe[i] = t.a.exps + row * exp_row;
    }
    f32x4 acc[kMats][FM];
#pragma unroll
    for (int i = 0; i < kMats; i++)
#pragma unroll
        for (int j = 0; j < FM; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    for (int kb = wave; kb < blocks; kb += waves) {
        u32x4 wc[kMats][2], xc[FM][2];
        float ws[kMats], xs[FM];
#pragma unroll
        for (int i = 0; i < kMats; i++) {
            const u32x4 *p = reinterpret_cast<const u32x4 *>(w[i] + (int64_t)kb * kFp8Block);
            wc[i][0] = __builtin_nontemporal_load(p); wc[i][1] = __builtin_nontemporal_load(p + 1);
            ws[i] = scale_of(we[i][kb]);
        }
#pragma unroll
        for (int j = 0; j < FM; j++) {
            const u32x4 *p = reinterpret_cast<const u32x4 *>(x[j] + (int64_t)kb * kFp8Block);
            xc[j][0] = p[0]; xc[j][1] = p[1];
            xs[j] = scale_of(xe[j][kb]);
        }
#pragma unroll
        for (int h = 0; h < 4; h++) {
            bf16x8 wp[kMats];
#pragma unroll
            for (int i = 0; i < kMats; i++) wp[i] = bf16x8_of_codes(wc[i][h / 2][2 * (h & 1)], wc[i][h / 2][2 * (h & 1) + 1], ws[i]);
#pragma unroll
            for (int j = 0; j < FM; j++) {
                const bf16x8 xp = bf16x8_of_codes(xc[j][h / 2][2 * (h & 1)], xc[j][h / 2][2 * (h & 1) + 1], xs[j]);
#pragma unroll
                for (int i = 0; i < kMats; i++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wp[i], xp, acc[i][j], 0, 0, 0);
            }
        }
    }
    // lane: columns (weight rows) n0 + 4 quarter .., token m0 + 16 j + r16
#pragma unroll
    for (int i = 0; i < kMats; i++)
#pragma unroll
        for (int j = 0; j < FM; j++) *reinterpret_cast<f32x4 *>(sums + (((wave * kMats + i) * FM + j) * kWave + lane) * 4) = acc[i][j];
    __syncthreads();
    for (int j = wave; j < FM; j += waves) {
        f32x4 total[kMats];
#pragma unroll
        for (int i = 0; i < kMats; i++) {
            total[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            for (int v = 0; v < waves; v++) total[i] += *reinterpret_cast<const f32x4 *>(sums + (((v * kMats + i) * FM + j) * kWave + lane) * 4);
        }
        f32x4 out = total[0];
        if constexpr (GATED) {
#pragma unroll
            for (int e = 0; e < 4; e++) out[e] = (t.act == PVQ_SILU ? act_value<PVQ_SILU>(total[0][e]) : act_value<PVQ_GELU>(total[0][e])) * total[1][e];
        }
        const int64_t row = m0 + 16 * j + r16, col = n0 + 4 * quarter;
        if (row < m) {
            const float v[4] = {out[0], out[1], out[2], out[3]};
            store_values(t.y, row, col, n - col, v);
        }
    }
}

template <int FM, bool GATED>
hipError_t launch_rows(const rows_args &t, hipStream_t s)
{
    const int waves = 8;
    const size_t lds = (size_t)waves * (GATED ? 2 : 1) * FM * kWave * 16;
    const dim3 grid((unsigned)((t.b.rows + 15) / 16), (unsigned)((t.a.rows + 16 * FM - 1) / (16 * FM)));
    hipLaunchKernelGGL((rows_kernel<FM, GATED>), grid, dim3(waves * kWave), lds, s, t);
    return hipGetLastError();
}

template <bool GATED>
hipError_t launch_rows_of(rows_args &t, hipStream_t s)
{
    if (t.a.rows <= 16) return launch_rows<1, GATED>(t, s);
    if (t.a.rows <= 32) return launch_rows<2, GATED>(t, s);
    return launch_rows<4, GATED>(t, s);
}

}  // namespace

bool fp8_rows_pay(int64_t m) { return m <= 64; }

hipError_t fp8_launch_product_rows(const fp8_product_args &p, hipStream_t s)
{
    rows_args t{};
    t.a = p.a; t.b = p.b; t.y = p.y;
    return launch_rows_of<false>(t, s);
}

hipError_t fp8_launch_gated_rows(const fp8_gated_args &g, hipStream_t s)
{
    rows_args t{};
    t.a = g.x; t.b = g.gate; t.up = g.up; t.y = g.h; t.act = g.act;
    return launch_rows_of<true>(t, s);
}
