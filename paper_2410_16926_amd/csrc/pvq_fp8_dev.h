// Device functions of the 8-bit block kernels.
#pragma once

#include "pvq_fp8.h"

namespace pvq_fp8_dev {

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

constexpr int kWave = 64;
// What an exponent byte may be after encoding: every value of a block is then a normal number in float32 and bfloat16, or zero
// (the smallest code is 2^-9), and the scale's reciprocal is one too.
constexpr uint32_t kExpLow = 127 - 110, kExpHigh = 127 + 120;

// 2^(e - 127)
__device__ inline float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// The exponent of a block whose largest magnitude has these bits: the least s with top <= 448 * 2^s = 1.75 * 2^(s + 8).
__device__ inline uint32_t exponent_of(uint32_t top_bits)
{
    const int e = (int)(top_bits >> 23) - 8 + ((top_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)min(max(e, (int)kExpLow), (int)kExpHigh);
}

// the bits of |x|, 0 for an infinity or a NaN: what counts for a block's largest magnitude
__device__ inline uint32_t finite_bits(float x)
{
    const uint32_t b = __float_as_uint(x) & 0x7FFFFFFFu;
    return b < 0x7F800000u ? b : 0u;
}

// Four values, scaled by `inverse` (a power of two), to four codes: to nearest, ties to even; infinities and NaN to NaN.  A
// scaled value never exceeds 448, the largest code; one too small for float32's normal numbers is far below half the smallest code.
__device__ inline uint32_t codes4(float a, float b, float c, float d, float inverse)
{
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * inverse, b * inverse, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c * inverse, d * inverse, r, true);
    return (uint32_t)r;
}

__device__ inline uint32_t bf16_pair(float lo, float hi)
{
    const f32x2 pair = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(pair, bf16x2));
}

__device__ inline uint32_t f16_pair(float lo, float hi)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)lo) | ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)hi) << 16);
}

// two codes (the lower or the upper half of a word) times a power of two, exactly, in bfloat16
template <bool UPPER>
__device__ inline uint32_t bf16_of_codes(uint32_t codes, float scale)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, UPPER));
}

// eight codes to bfloat16
__device__ inline bf16x8 bf16x8_of_codes(uint32_t lo, uint32_t hi, float scale)
{
    const u32x4 w = {bf16_of_codes<false>(lo, scale), bf16_of_codes<true>(lo, scale), bf16_of_codes<false>(hi, scale), bf16_of_codes<true>(hi, scale)};
    return __builtin_bit_cast(bf16x8, w);
}

// Vectors at any element's address: loads and stores of global memory need no more alignment than that.
template <typename V, int ALIGNMENT>
struct __attribute__((packed, aligned(ALIGNMENT))) unaligned { V v; };
template <typename V>
__device__ inline void store_vector(float *p, V v) { reinterpret_cast<unaligned<V, 4> *>(p)->v = v; }
template <typename V>
__device__ inline void store_vector(uint16_t *p, V v) { reinterpret_cast<unaligned<V, 2> *>(p)->v = v; }

// Neighbouring values of a row, four or eight, to out[row][col ..], of which `count` lie inside.
template <int N>
__device__ inline void store_values(const fp8_matrix &y, int64_t row, int64_t col, int64_t count, const float (&v)[N])
{
    const int64_t at = row * y.ld + col;
    if (y.dtype == PVQ_F32) {
        float *p = reinterpret_cast<float *>(y.data) + at;
        if (count >= N) {
#pragma unroll
            for (int i = 0; i < N; i += 4) store_vector(p + i, f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]});
            return;
        }
#pragma unroll
        for (int i = 0; i < N; i++) if (i < count) p[i] = v[i];
        return;
    }
    typedef __attribute__((ext_vector_type(N / 2))) uint32_t words;
    words w;
#pragma unroll
    for (int i = 0; i < N / 2; i++) w[i] = y.dtype == PVQ_BF16 ? bf16_pair(v[2 * i], v[2 * i + 1]) : f16_pair(v[2 * i], v[2 * i + 1]);
    uint16_t *p = reinterpret_cast<uint16_t *>(y.data) + at;
    if (count >= N) { store_vector(p, w); return; }
#pragma unroll
    for (int i = 0; i < N; i++) if (i < count) p[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

// the largest of a block's sixteen lanes, in all of them (rotations inside a row of sixteen)
__device__ inline uint32_t block_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xF, 0xF, false));
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xF, 0xF, false));
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xF, 0xF, false));
}

// the exponent of a block of which each of sixteen lanes has eight values
__device__ inline uint32_t block_exponent(const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    if (__builtin_amdgcn_ballot_w64(top >= 0x7F800000u)) {             // (seldom: infinities or NaN in the wave)
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) top = max(top, finite_bits(v[i]));
    }
    return exponent_of(block_max(top));
}

// a lane's eight codes of a block
__device__ inline void store_codes8(uint8_t *to, uint32_t e, const float (&v)[8])
{
    const float inverse = scale_of(254 - e);
    *reinterpret_cast<u32x2 *>(to) = u32x2{codes4(v[0], v[1], v[2], v[3], inverse), codes4(v[4], v[5], v[6], v[7], inverse)};
}

// Activations.  sigma(x) = 1 / (1 + exp(-x)) by the hardware's 2^x and reciprocal, each off by about one place; exp(-x) may be
// infinite, sigma is 0 then.  silu(g) = g sigma(g); gelu in its tanh form, 0.5 g (1 + tanh w) = g sigma(2 w) with
// w = sqrt(2/pi) (g + 0.044715 g^3), of which nothing changes beyond |g| = 16 but the factor g.
__device__ inline float exp_minus(float x) { return __builtin_amdgcn_exp2f(x * -1.4426950408889634f); }

__device__ inline float gelu_argument(float g)
{
    const float c = fminf(fmaxf(g, -16.0f), 16.0f);
    return 1.5957691216057308f * (c + 0.044715f * c * c * c);       // 2 w
}

template <int ACT>
__device__ inline float act_value(float g)
{
    const float x = ACT == PVQ_SILU ? g : gelu_argument(g);
    return g * __builtin_amdgcn_rcpf(1.0f + exp_minus(x));
}

// act(g) and its derivative sigma + g sigma (1 - sigma) dx/dg.  1 - sigma is formed as sigma exp(-x), of full accuracy for
// large x too; where exp(-x) is infinite sigma is 0 and so is the product.
template <int ACT>
__device__ inline void act_slope(float g, float &value, float &slope)
{
    float x = g, dx = 1.0f;
    if constexpr (ACT != PVQ_SILU) {
        const float c = fminf(fmaxf(g, -16.0f), 16.0f);
        x = gelu_argument(g);
        dx = 1.5957691216057308f * (1.0f + 3.0f * 0.044715f * c * c);
    }
    const float e = exp_minus(x), s = __builtin_amdgcn_rcpf(1.0f + e);
    value = g * s;
    const float rest = s > 0.0f ? s * e : 1.0f;                      // 1 - s
    slope = s + value * rest * dx;
}

// What the gated block stores, of eight neighbouring hidden units: H in floats and in blocks, G and U in blocks.
struct gated_out {
    fp8_matrix h;                // (data null: in blocks alone)
    int act;
    uint8_t *hc, *he, *gc, *ge, *uc, *ue;      // (null: not wanted)
};

// Sixteen lanes have the units of block `block` of a row, from col on eight each; all of them come here.  Units from n on are zeros in the codes.
template <int ACT>
__device__ inline void store_gated8(const gated_out &t, int64_t row, int64_t n, int64_t block, int64_t col, bool row_there, float (&g)[8], float (&u)[8])
{
    const int64_t count = n - col, code_row = (n + kFp8Block - 1) / kFp8Block * kFp8Block, exp_row = (code_row / kFp8Block + 3) / 4 * 4;
    float h[8];
    if (count < 8) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i >= count) g[i] = u[i] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) h[i] = act_value<ACT>(g[i]) * u[i];
    if (t.h.data && row_there && count > 0) store_values(t.h, row, col, count, h);
    auto to_blocks = [&](uint8_t *codes, uint8_t *exps, const float (&v)[8]) {
        if (!codes) return;
        const uint32_t e = block_exponent(v);
        if (!row_there || block * kFp8Block >= n) return;
        store_codes8(codes + row * code_row + col, e, v);
        if (threadIdx.x % 16 == 0) {
            uint8_t *p = exps + row * exp_row;
            p[block] = (uint8_t)e;
            if ((block + 1) * kFp8Block >= n)
                for (int64_t b = block + 1; b < exp_row; b++) p[b] = 0;
        }
    };
    to_blocks(t.gc, t.ge, g);
    to_blocks(t.uc, t.ue, u);
    to_blocks(t.hc, t.he, h);
}

// The workgroup's number such that those on one chiplet (the hardware deals them out in turn over 8) are neighbours, for any
// number of them: each chiplet has its own L2.
__device__ inline int chiplet_order(int id, int total)
{
    const int each = total / 8, more = total % 8, x = id % 8, y = id / 8;
    return x * each + min(x, more) + y;
}

}  // namespace pvq_fp8_dev
