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

// Four neighbouring values of a row to out[row][col ..], of which `count` lie inside.  VEC: `out` and its rows are aligned
// to four values.
template <bool VEC>
__device__ inline void store4(const fp8_matrix &y, int64_t row, int64_t col, int64_t count, f32x4 v)
{
    const int64_t at = row * y.ld + col;
    if (y.dtype == PVQ_F32) {
        float *p = reinterpret_cast<float *>(y.data) + at;
        if (VEC && count >= 4) { *reinterpret_cast<f32x4 *>(p) = v; return; }
#pragma unroll
        for (int i = 0; i < 4; i++) if (i < count) p[i] = v[i];
        return;
    }
    const u32x2 w = y.dtype == PVQ_BF16 ? u32x2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])} : u32x2{f16_pair(v[0], v[1]), f16_pair(v[2], v[3])};
    uint16_t *p = reinterpret_cast<uint16_t *>(y.data) + at;
    if (VEC && count >= 4) { *reinterpret_cast<u32x2 *>(p) = w; return; }
#pragma unroll
    for (int i = 0; i < 4; i++) if (i < count) p[i] = (uint16_t)(w[i / 2] >> (16 * (i & 1)));
}

// The same of two fragments side by side (columns col .. and col + 16 .., a lane's four at 4 quarter of each): lanes of quarters 2 p and
// 2 p + 1 exchange halves, so that each holds eight neighbouring columns, of the left fragment or the right one.  A row's store is
// 64 bytes in a row in place of 32.  Only for what lies inside, in rows aligned to eight values; `col` is that of the left fragment.
__device__ inline void store_pair(const fp8_matrix &y, int64_t row, int64_t col, int quarter, f32x4 left, f32x4 right)
{
    const int64_t at = row * y.ld + col + 16 * (quarter & 1) + 8 * (quarter >> 1);
    if (y.dtype == PVQ_F32) {
        u32x4 lo, hi;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(left[i]), __float_as_uint(right[i]), false, false);
            lo[i] = r[0]; hi[i] = r[1];
        }
        u32x4 *p = reinterpret_cast<u32x4 *>(reinterpret_cast<float *>(y.data) + at);
        p[0] = lo; p[1] = hi;
        return;
    }
    const bool b = y.dtype == PVQ_BF16;
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const uint32_t l = b ? bf16_pair(left[2 * i], left[2 * i + 1]) : f16_pair(left[2 * i], left[2 * i + 1]);
        const uint32_t r = b ? bf16_pair(right[2 * i], right[2 * i + 1]) : f16_pair(right[2 * i], right[2 * i + 1]);
        const auto s = __builtin_amdgcn_permlane16_swap(l, r, false, false);
        w[i] = s[0]; w[2 + i] = s[1];
    }
    *reinterpret_cast<u32x4 *>(reinterpret_cast<uint16_t *>(y.data) + at) = w;
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

__device__ inline float act_value(int act, float g)
{
    const float x = act == PVQ_SILU ? g : gelu_argument(g);
    return g * __builtin_amdgcn_rcpf(1.0f + exp_minus(x));
}

// act(g) and its derivative sigma + g sigma (1 - sigma) dx/dg.  1 - sigma is formed as sigma exp(-x), of full accuracy for
// large x too; where exp(-x) is infinite sigma is 0 and so is the product.
__device__ inline void act_slope(int act, float g, float &value, float &slope)
{
    float x = g, dx = 1.0f;
    if (act != PVQ_SILU) {
        const float c = fminf(fmaxf(g, -16.0f), 16.0f);
        x = gelu_argument(g);
        dx = 1.5957691216057308f * (1.0f + 3.0f * 0.044715f * c * c);
    }
    const float e = exp_minus(x), s = __builtin_amdgcn_rcpf(1.0f + e);
    value = g * s;
    const float rest = s > 0.0f ? s * e : 1.0f;                      // 1 - s
    slope = s + value * rest * dx;
}

// The workgroup's number such that those on one chiplet (the hardware deals them out in turn over 8) are neighbours, for any
// number of them: each chiplet has its own L2.
__device__ inline int chiplet_order(int id, int total)
{
    const int each = total / 8, more = total % 8, x = id % 8, y = id / 8;
    return x * each + min(x, more) + y;
}

}  // namespace pvq_fp8_dev
