// Products of a few rows (tokens) with 8-bit block weights: bound by the weights' bytes.
#include "pvq_fp8_tile.h"

#include <type_traits>

using namespace pvq_fp8_dev;

namespace {

constexpr int kRows = 16;                 // of a set of a wave's weights
constexpr int kWaves = 8, kLdsBytes = 160 * 1024;

struct rows_args {
    fp8_blocks a, b, up;
    fp8_matrix y;
    int act;
    int parts;                            // waves that share a sum, 1, 2, 4 or 8
    int blocks_a_part;
};

// The tokens' rows that come with each block, by eights.
enum tokens_of { EIGHT = 1, SIXTEEN = 2, THIRTY_TWO = 4 };

// What a wave has in LDS: a ring of stages, each a block of 128 of its 32 rows of weights and of the tokens, and behind it the words of
// exponents of four runs of four blocks: lanes 0 .. 31 the weights' rows, 32 .. the tokens'.
template <int TOKENS>
struct ring_of {
    static constexpr int FM = TOKENS == THIRTY_TWO ? 2 : 1, kTokens = 2 * kRows * kFp8Block, kStage = kTokens + TOKENS * 1024, kExps = 4 * 64 * 4;
    static constexpr int kLoads = 4 + TOKENS, kStages = (kLdsBytes / kWaves - kExps) / kStage, kBytes = kStages * kStage + kExps;
    static_assert(kStages >= 2 && kStages <= 9 && FM <= 2, "stages");
};

// A wave takes 32 rows of the weights, two sets of 16 (GATED: 16 of the gate's and the same of the up weights), and all tokens (16 FM), or a part of
// the sum of these, alone: its loads, a KiB each of eight whole lines, go straight into its own ring of stages in LDS, several blocks ahead, and
// nobody waits for anybody until the parts' sums are added, in their order.  The codes are decoded to bfloat16, exactly.
// (Straight to registers a lane would load 16 bytes of a row of its own, sixteen lines for 256 bytes: 16 x 8192 x 28672 80 us.  Sixteen rows a wave and
// exponents with each block: 57 us, of which the tokens took 17 and the exponents 11.  Thus 48 us, the gated block of 1 x 28672 x 8192 84 to 93: 5.0 to
// 5.6 TB/s, as fast as the weights can be read; loads without the products take as long.  Weights' loads marked as used once: 4 % less or more, by shape.)
template <int TOKENS, bool GATED>
__global__ __launch_bounds__(kWaves *kWave) void rows_kernel(rows_args t)
{
    using R = ring_of<TOKENS>;
    constexpr int FM = R::FM, kStages = R::kStages;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int r16 = lane % 16, quarter = lane / 16;
    const int part = wave % t.parts;
    constexpr int kCols = GATED ? kRows : 2 * kRows;             // of the result
    const int64_t n = t.b.rows, m = t.a.rows, n0 = ((int64_t)blockIdx.x * (kWaves / t.parts) + wave / t.parts) * kCols;
    const uint32_t row_bytes = (uint32_t)t.a.code_row(), exp_row = (uint32_t)t.a.exp_row();
    const int kb0 = part * t.blocks_a_part, kb1 = min(kb0 + t.blocks_a_part, (int)t.a.blocks());       // (kb0 a multiple of four)
    const bool there = n0 < n && kb0 < kb1;

    f32x4 acc[2][FM];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < FM; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    uint8_t *mine = lds + wave * R::kBytes;
    if (there) {
        const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(mine));
        // a load: eight rows of 128 bytes, chunk c of row r at place c ^ (r / 2 % 8); rows past the end are the last one once more
        const int64_t n_last = n - 1 - n0;
        const uint32_t in_row = lane / 8;
        uint32_t w_at[4], x_at[TOKENS];
#pragma unroll
        for (int i = 0; i < 4; i++) w_at[i] = (uint32_t)min((int64_t)((GATED ? 8 * i % kRows : 8 * i) + in_row), n_last) * row_bytes + ((lane % 8 ^ ((8 * i + in_row) >> 1 & 7)) << 4);
#pragma unroll
        for (int i = 0; i < TOKENS; i++) x_at[i] = (uint32_t)min((int64_t)(8 * i + in_row), m - 1) * row_bytes + ((lane % 8 ^ ((8 * i + in_row) >> 1 & 7)) << 4);
        const uint8_t *first = t.b.codes + n0 * row_bytes, *second = GATED ? t.up.codes + n0 * row_bytes : first;
        const int64_t exp_at = lane < 32 ? (n0 + min((int64_t)(GATED ? r16 : lane), n_last)) * exp_row : min((int64_t)(lane - 32), m - 1) * exp_row;
        const uint8_t *exps = (lane < 32 ? GATED && lane >= 16 ? t.up.exps : t.b.exps : t.a.exps) + exp_at;

        auto load = [&](int kb, uint32_t to) {
            const int from = min(kb, kb1 - 1);                  // (behind the last one: once more, and nobody looks)
#pragma unroll
            for (int i = 0; i < 4; i++) load_to_lds((i < 2 ? first : second) + (int64_t)from * kFp8Block, w_at[i], lds0 + to + i * 1024);
#pragma unroll
            for (int i = 0; i < TOKENS; i++) load_to_lds(t.a.codes + (int64_t)from * kFp8Block, x_at[i], lds0 + to + R::kTokens + i * 1024);
        };
        auto load_exps = [&](int kb) {
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
                         : : "s"(lds0 + kStages * R::kStage + (kb >> 2 & 3) * 256), "v"(exps + (min(kb, kb1 - 1) & ~3)) : "memory", "m0");
        };
        // operand: 32 codes of row lane % 16, chunks lane / 16 and 4 + lane / 16
        auto codes_of = [&](const uint8_t *rows, int row, u32x4 (&c)[2]) {
#pragma unroll
            for (int h = 0; h < 2; h++) c[h] = *reinterpret_cast<const u32x4 *>(rows + row * kFp8Block + (((4 * h + quarter) ^ (row >> 1 & 7)) << 4));
        };
        auto behind = [&](uint32_t at) { return at + R::kStage == kStages * R::kStage ? 0u : at + R::kStage; };
        // Loads are issued kStages - 1 blocks ahead, a run's exponents with its first block; what may still be on its way when a block is read
        // follows from its place in its run.
        constexpr int kAhead = kStages - 1;
        uint32_t words[2], x_words[FM];
        uint32_t at = 0, to = kAhead * R::kStage;
        auto step = [&](auto AT, int kb) {
            constexpr int place = decltype(AT)::value, kRuns = (place + kAhead) / 4;          // runs that begin among the blocks ahead
            if constexpr ((place + kAhead) % 4 == 0) load_exps(kb + kAhead);
            load(kb + kAhead, to);
            loads_but<kAhead * R::kLoads + kRuns>();
            const uint8_t *stage = mine + at;
            if constexpr (place == 0) {
                const uint32_t *run = reinterpret_cast<const uint32_t *>(mine + kStages * R::kStage + (kb >> 2 & 3) * 256);
#pragma unroll
                for (int i = 0; i < 2; i++) words[i] = run[16 * i + r16];
#pragma unroll
                for (int j = 0; j < FM; j++) x_words[j] = run[32 + 16 * j + r16];
            }
            u32x4 w[2][2], x[FM][2];
#pragma unroll
            for (int i = 0; i < 2; i++) codes_of(stage + i * kRows * kFp8Block, r16, w[i]);
#pragma unroll
            for (int j = 0; j < FM; j++) codes_of(stage + R::kTokens + j * 16 * kFp8Block, TOKENS == EIGHT ? r16 % 8 : r16, x[j]);
            all_reads();                                          // (the stage may be loaded into again)
#pragma unroll
            for (int h = 0; h < 4; h++) {
                bf16x8 wp[2];
#pragma unroll
                for (int i = 0; i < 2; i++) wp[i] = bf16x8_of_codes(w[i][h / 2][2 * (h & 1)], w[i][h / 2][2 * (h & 1) + 1], scale_of(words[i] >> 8 * place & 255u));
#pragma unroll
                for (int j = 0; j < FM; j++) {
                    const bf16x8 xp = bf16x8_of_codes(x[j][h / 2][2 * (h & 1)], x[j][h / 2][2 * (h & 1) + 1], scale_of(x_words[j] >> 8 * place & 255u));
#pragma unroll
                    for (int i = 0; i < 2; i++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wp[i], xp, acc[i][j], 0, 0, 0);
                }
            }
            at = behind(at);
            to = behind(to);
        };
        load_exps(kb0);
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            if (i && i % 4 == 0) load_exps(kb0 + i);
            load(kb0 + i, i * R::kStage);
        }
        for (int kb = kb0; kb < kb1; kb += 4) {
            step(std::integral_constant<int, 0>{}, kb);
            if (kb + 1 < kb1) step(std::integral_constant<int, 1>{}, kb + 1);
            if (kb + 2 < kb1) step(std::integral_constant<int, 2>{}, kb + 2);
            if (kb + 3 < kb1) step(std::integral_constant<int, 3>{}, kb + 3);
        }
        all_loads();
    }
    // lane: columns (weight rows) 4 quarter .. of a set, token 16 j + r16
    if (t.parts > 1) {
        float *sums = reinterpret_cast<float *>(mine);
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
            for (int j = 0; j < FM; j++) *reinterpret_cast<f32x4 *>(sums + ((i * FM + j) * kWave + lane) * 4) = acc[i][j];
        __syncthreads();
        if (part) return;
        for (int p = 1; p < t.parts; p++) {
            const float *other = reinterpret_cast<const float *>(mine + p * R::kBytes);
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < FM; j++) acc[i][j] += *reinterpret_cast<const f32x4 *>(other + ((i * FM + j) * kWave + lane) * 4);
        }
    }
#pragma unroll
    for (int j = 0; j < FM; j++) {
        const int64_t row = 16 * j + r16, col = n0 + 4 * quarter;
        if (row >= m) continue;
        float v[2][4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            v[0][e] = acc[0][j][e];
            v[1][e] = acc[1][j][e];
            if constexpr (GATED) v[0][e] = (t.act == PVQ_SILU ? act_value<PVQ_SILU>(v[0][e]) : act_value<PVQ_GELU>(v[0][e])) * v[1][e];
        }
        if (col < n) store_values(t.y, row, col, n - col, v[0]);
        if (!GATED && col + kRows < n) store_values(t.y, row, col + kRows, n - col - kRows, v[1]);
    }
}

template <int TOKENS, bool GATED>
hipError_t launch_rows(rows_args &t, hipStream_t s)
{
    constexpr int kLds = kWaves * ring_of<TOKENS>::kBytes, kCols = GATED ? kRows : 2 * kRows;
    const auto kernel = &rows_kernel<TOKENS, GATED>;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
    if (e != hipSuccess) return e;
    // the parts, of whole runs of four blocks, with which a unit has the fewest blocks to take, one workgroup after the other; of as many the fewest parts
    const int64_t tiles = (t.b.rows + kCols - 1) / kCols, runs = (t.a.blocks() + 3) / 4;
    int64_t least = 0;
    for (int parts = 1; parts <= kWaves && runs >= parts; parts *= 2) {
        const int64_t groups = (tiles * parts + kWaves - 1) / kWaves, takes = (groups + 255) / 256 * ((runs + parts - 1) / parts);
        if (parts == 1 || takes < least) { least = takes; t.parts = parts; }
    }
    t.blocks_a_part = (int)((runs + t.parts - 1) / t.parts * 4);
    const int64_t a_group = kWaves / t.parts;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((tiles + a_group - 1) / a_group)), dim3(kWaves * kWave), kLds, s, t);
    return hipGetLastError();
}

template <bool GATED>
hipError_t launch_rows_of(rows_args &t, hipStream_t s)
{
    if (t.a.rows <= 8) return launch_rows<EIGHT, GATED>(t, s);
    return t.a.rows <= 16 ? launch_rows<SIXTEEN, GATED>(t, s) : launch_rows<THIRTY_TWO, GATED>(t, s);
}

}  // namespace

// Up to as many tokens as a wave's ring has room for: 32 x 8192 x 8192 20 us here, 33 in tiles 29 (32 x 28672 x 8192 59, 64 in tiles 75).
bool fp8_rows_pay(int64_t m) { return m <= 32; }

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
