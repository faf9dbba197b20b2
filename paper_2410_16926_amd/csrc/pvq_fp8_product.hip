// Products of 8-bit block matrices in tiles: Y = A B^T, and the gated block H = act(X Wg^T) * (X Wu^T).
#include "pvq_fp8_small.h"

#include <type_traits>

using namespace pvq_fp8_dev;

namespace {

// ---- on the 8-bit instruction -----------------------------------------------------------------------------------------
// A lane holds 32 codes of one row (lane % 16) of an operand: those of quarter lane / 16 of a block of 128.  Which codes of the block a quarter is does
// not matter, as long as both operands agree.  The instruction's adders align eight products at a time to the largest and keep about 14 bits
// below it, so that sums of Gaussian terms are 3.3e-5 of their size off: a sixtieth of bfloat16's rounding.

// A tile row is a block of codes, 128 bytes in eight chunks; chunk c of row r lies at place c ^ (r / 2 % 8), so that
// what sixteen lanes read at one chunk number of sixteen rows lies in all 64 banks.
__device__ inline uint32_t chunk_at(uint32_t row, uint32_t chunk) { return row * kFp8Block + ((chunk ^ (row >> 1 & 7)) << 4); }

__device__ inline i32x8 read_operand(const uint8_t *tile, uint32_t row, uint32_t quarter)
{
    const i32x4 lo = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, quarter)), hi = *reinterpret_cast<const i32x4 *>(tile + chunk_at(row, 4 + quarter));
    return i32x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

struct tile_args {
    fp8_blocks a, b, up;         // up: the gated block's second weights
    int64_t n;
    int tiles_m, tiles_n, blocks_a_part;
};

// what becomes of a tile's sums
struct tile_out {
    fp8_matrix y;                // of a product
    gated_out gated;
    int parts;                   // whose sums go to work, [part][rows][n], GATED [part][G, U][rows][n]; 0: none do
    float *work;
};

// The sums of a tile at m0, n0 (GATED: of 128 hidden units), or what the gated block makes of them, to memory.
template <bool GATED>
__device__ __forceinline__ void store_tile(const tile_out &t, int64_t rows, int64_t n, uint8_t *lds, const f32x4 (&acc)[8][8], int64_t m0, int64_t n0, int part)
{
    const bool split = t.parts > 0;
    if constexpr (!GATED) store_sums(split ? part_of(t.work, part, rows, n) : t.y, rows, n, acc, m0, n0);
    else {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), lane = threadIdx.x % kWave, chunk = lane % 16 * 2;
        const int64_t col = n0 + lane % 16 * 8;
        store_rows(lds, acc, [&](int j) { return j / 4 * 128 + wave % 2 * 64 + j % 4 * 16; }, [&](int half, auto at) {
            // sixteen lanes have the 128 hidden units of a row; a wave's rows four at a time, two times ahead
            auto rows_of = [&](auto what) {
#pragma unroll 1
                for (int r0 = wave * 4 + lane / 16; r0 < 128; r0 += 32) {
                    float g[2][8], u[2][8];
#pragma unroll
                    for (int k = 0; k < 2; k++)
#pragma unroll
                        for (int h = 0; h < 2; h++) {
                            const f32x4 a = *at(r0 + 16 * k, chunk + h), b = *at(r0 + 16 * k, 32 + chunk + h);
#pragma unroll
                            for (int e = 0; e < 4; e++) { g[k][4 * h + e] = a[e]; u[k][4 * h + e] = b[e]; }
                        }
                    what(m0 + tile_row(half, r0), g[0], u[0], m0 + tile_row(half, r0 + 16), g[1], u[1]);
                }
            };
            const gated_out &o = t.gated;
            const bool plain = o.h.data && !o.hc && !o.gc && o.h.dtype == PVQ_BF16 && n0 + 128 <= n;
            // whole rows of H in bfloat16 alone, as a prompt wants them
            auto prompt = [&](auto ACT) {
                rows_of([&](int64_t row, float (&g)[8], float (&u)[8], int64_t next_row, float (&next_g)[8], float (&next_u)[8]) {
                    u32x4 w[2];
#pragma unroll
                    for (int k = 0; k < 2; k++)
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const float *a = k ? next_g : g, *b = k ? next_u : u;
                            w[k][e] = bf16_pair(act_value<decltype(ACT)::value>(a[2 * e]) * b[2 * e], act_value<decltype(ACT)::value>(a[2 * e + 1]) * b[2 * e + 1]);
                        }
                    uint16_t *h = reinterpret_cast<uint16_t *>(o.h.data) + col;
                    if (row < rows) store_vector(h + row * o.h.ld, w[0]);
                    if (next_row < rows) store_vector(h + next_row * o.h.ld, w[1]);
                });
            };
            auto all = [&](auto ACT) {
                rows_of([&](int64_t row, float (&g)[8], float (&u)[8], int64_t next_row, float (&next_g)[8], float (&next_u)[8]) {
                    store_gated8<decltype(ACT)::value>(o, row, n, n0 / kFp8Block, col, row < rows, g, u);
                    store_gated8<decltype(ACT)::value>(o, next_row, n, n0 / kFp8Block, col, next_row < rows, next_g, next_u);
                });
            };
            if (split) {
                // (G's columns and U's are two matrices)
                const fp8_matrix to_g = part_of(t.work, 2 * part, rows, n), to_u = part_of(t.work, 2 * part + 1, rows, n);
                rows_of([&](int64_t row, float (&g)[8], float (&u)[8], int64_t next_row, float (&next_g)[8], float (&next_u)[8]) {
#pragma unroll 1
                    for (int k = 0; k < 4; k++) {
                        float v[8];
#pragma unroll
                        for (int e = 0; e < 8; e++) v[e] = k == 0 ? g[e] : k == 1 ? u[e] : k == 2 ? next_g[e] : next_u[e];
                        const int64_t r = k < 2 ? row : next_row;
                        if (r < rows && col < n) store_values(k % 2 ? to_u : to_g, r, col, n - col, v);
                    }
                });
            } else if (plain) {
                if (o.act == PVQ_SILU) prompt(std::integral_constant<int, PVQ_SILU>{});
                else prompt(std::integral_constant<int, PVQ_GELU>{});
            } else {
                if (o.act == PVQ_SILU) all(std::integral_constant<int, PVQ_SILU>{});
                else all(std::integral_constant<int, PVQ_GELU>{});
            }
        });
    }
}

// Tiles of 256 x 256 on the 8-bit instruction by four waves of 128 x 128, one to a SIMD.  Of what bounds these products LDS comes first: a
// block of 128 of a tile is 64 KB that are written at 64 bytes a cycle and 256 KB / (waves' tile side / 64) that are read at 128, beside 2048
// cycles of matrix instructions.  Eight waves of 128 x 64 read 192 KB (2560 cycles in all), four of 128 x 128 128 KB (2048).
//
// A wave alone on its SIMD has nobody to fill in for it, so its own instructions are laid out: a block's products come in two
// halves, of the upper and the lower 64 rows of the wave's part of A, with a barrier in front of each.
//   first half   products of the upper rows; reads the lower rows' operands; loads B and the upper rows of the next block but one, whose
//                place everybody has read
//   second half  products of the lower rows; reads all of B (into a second set of registers) and the upper rows of the next block; loads
//                the lower rows of the next block but one
// Each load has a step and a half to arrive (with one barrier and a single step 1.6 us a step where operands come from beyond L2; thus 1.4).
// 4096 x 8192 x 8192 201 us, 2.7 PFLOP/s; the gated block of 2048 x 28672 x 8192 700 us (1648 by eight waves that take turns with their loads).
template <bool GATED>
__global__ __launch_bounds__(256) void tile_kernel(tile_args t, tile_out out)
{
    constexpr int kTile = 256, F = 8, H = F / 2, kCols = GATED ? kTile / 2 : kTile;
    constexpr int kPlane = kTile * kFp8Block;         // LDS: A's two stages, B's two stages, the words of exponents of two runs of four blocks
    constexpr int kExps = 4 * kPlane, kExpBytes = 2 * kTile * 4;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / 2, wn = wave % 2, r16 = lane % 16, quarter = lane / 16;
    int tm, tn;
    tile_of(t.tiles_m, t.tiles_n, chiplet_order(blockIdx.x, gridDim.x), tm, tn);
    const int64_t m0 = (int64_t)tm * kTile, n0 = (int64_t)tn * kCols;
    const int part = blockIdx.y;
    const int kb0 = part * t.blocks_a_part, kb1 = min(kb0 + t.blocks_a_part, (int)t.a.blocks());       // (kb0 a multiple of four)
    const uint32_t row_bytes = (uint32_t)t.a.code_row(), exp_row = (uint32_t)t.a.exp_row();

    // The tile's rows as buffers that end with the matrix: what rows past the end bring does not matter, their results are not stored.  A load
    // is eight rows, 1 KiB; load i of wave w is rows 32 i + 8 w ..: first A's, then B's (the gate's, the up weights').
    auto rows_of = [&](const uint8_t *plane, uint32_t row, int64_t first, int64_t rows, int most) {
        return make_buffer(plane + first * row, min(rows - first, (int64_t)most) * row);
    };
    const buffer_t a_codes = rows_of(t.a.codes, row_bytes, m0, t.a.rows, kTile), b_codes = rows_of(t.b.codes, row_bytes, n0, t.n, kCols);
    const buffer_t u_codes = GATED ? rows_of(t.up.codes, row_bytes, n0, t.n, kCols) : b_codes;
    const uint32_t in_row = lane / 8, chunk = ((lane % 8) ^ ((wave * 8 + in_row) >> 1 & 7)) << 4;
    const uint32_t offset = (wave * 8 + in_row) * row_bytes + chunk;
    // words of four exponents, 64 rows a load: rows 64 w .. of A, then of B
    const buffer_t a_exps = rows_of(t.a.exps, exp_row, m0, t.a.rows, kTile);
    const buffer_t b_exps = rows_of(GATED && wave >= 2 ? t.up.exps : t.b.exps, exp_row, n0, t.n, kCols);
    const uint32_t exp_offset = lane * exp_row;

    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));
    const uint32_t to0 = lds0 + wave * 8 * kFp8Block, exp_to0 = lds0 + kExps + wave * kWave * 4;
    // Past the last block it is the last once more, to a place that nobody reads any more: no load is under a condition, and each wait
    // knows how many were issued behind those that it waits for.
    auto load_rows = [&](int kb, bool b, int i) {      // rows 32 i + 8 w .. of A or of B
        const buffer_t codes = !b ? a_codes : GATED && i >= 4 ? u_codes : b_codes;
        load_to_lds(codes, offset, (uint32_t)min(kb, kb1 - 1) * kFp8Block + (b ? 32 * i % kCols : 32 * i) * row_bytes,
                    to0 + (b ? 2 : 0) * kPlane + (kb & 1) * kPlane + (uint32_t)(i * 32 * kFp8Block));
    };
    auto load_exps = [&](int kb, bool b) {             // the words of four blocks
        load_words_to_lds(b ? b_exps : a_exps, exp_offset, (uint32_t)(min(kb, kb1 - 1) & ~3) + (b ? wave % (kCols / kWave) : wave) * kWave * exp_row,
                          exp_to0 + ((kb >> 2) & 1) * kExpBytes + (b ? kExpBytes / 2 : 0));
    };
    constexpr int kFirst = 12, kSecond = 4;
    auto load_first = [&](int kb, int piece) {         // B and the upper rows of both halves of A
        if (piece < 8) load_rows(kb, true, piece);
        else if (piece < kFirst) load_rows(kb, false, (piece - 8) % 2 + (piece - 8) / 2 * 4);
    };
    auto load_second = [&](int kb, int piece) {
        if (piece < kSecond) load_rows(kb, false, 2 + piece % 2 + piece / 2 * 4);
    };

    f32x4 acc[F][F];
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < F; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    i32x8 a_upper[H], a_lower[H], b_op[2][F];
    uint32_t a_exp[F], b_exp[F];
    auto b_row = [&](int j) { return GATED ? (j / H) * kCols + wn * 64 + (j % H) * 16 + r16 : wn * 128 + j * 16 + r16; };
    auto read_a = [&](int stage, int i) { return read_operand(lds + stage * kPlane, wm * 128 + i * 16 + r16, quarter); };
    auto read_b = [&](int stage, int j) { return read_operand(lds + (2 + stage) * kPlane, b_row(j), quarter); };

    // one block; AT: its number modulo four
    auto step = [&](auto AT, int kb) {
        constexpr int at = decltype(AT)::value, stage = at & 1;
        // the next four blocks' exponents come with the second of these: two loads more
        constexpr int kExpLoads = at == 1 ? 2 : 0, kBehind = kFirst + kSecond + kExpLoads;
        if constexpr (at == 0) {
            const uint32_t *exps = reinterpret_cast<const uint32_t *>(lds + kExps + ((kb >> 2) & 1) * kExpBytes);
            const uint32_t there = kb + 4 <= kb1 ? ~0u : (1u << 8 * (kb1 - kb)) - 1;       // blocks behind the last: 0
#pragma unroll
            for (int i = 0; i < F; i++) a_exp[i] = exps[wm * 128 + i * 16 + r16] & there;
#pragma unroll
            for (int j = 0; j < F; j++) b_exp[j] = exps[kTile + b_row(j)] & there;
        }
#pragma unroll
        for (int i = 0; i < H; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated<at>(acc[i][j], b_op[stage][j], b_exp[j], a_upper[i], a_exp[i]);
                const int slot = i * F + j;
                if (slot % 2 == 0 && slot / 2 < H) a_lower[slot / 2] = read_a(stage, H + slot / 2);
                if (slot % 2 == 1) load_first(kb + 2, slot / 2);
                if (kExpLoads && (slot == 26 || slot == 28)) load_exps(kb + 3, slot == 28);
                __builtin_amdgcn_sched_barrier(0);
            }
        all_reads();
        loads_but<kBehind>();                    // B and the upper rows of the next block are there
        barrier();
#pragma unroll
        for (int i = 0; i < H; i++)
#pragma unroll
            for (int j = 0; j < F; j++) {
                multiply_accumulated<at>(acc[H + i][j], b_op[stage][j], b_exp[j], a_lower[i], a_exp[H + i]);
                const int slot = i * F + j;
                if (slot < F) b_op[stage ^ 1][slot] = read_b(stage ^ 1, slot);
                else if (slot < F + H) a_upper[slot - F] = read_a(stage ^ 1, slot - F);
                if (slot % 2 == 1) load_second(kb + 2, slot / 2);
                __builtin_amdgcn_sched_barrier(0);
            }
        all_reads();
        loads_but<kBehind>();                    // the lower rows of the next block are there
        barrier();
    };

    if (kb0 < kb1) {
        load_exps(kb0, false);
        load_exps(kb0, true);
#pragma unroll
        for (int i = 0; i < kFirst; i++) load_first(kb0, i);
#pragma unroll
        for (int i = 0; i < kSecond; i++) load_second(kb0, i);
#pragma unroll
        for (int i = 0; i < kFirst; i++) load_first(kb0 + 1, i);
#pragma unroll
        for (int i = 0; i < kSecond; i++) load_second(kb0 + 1, i);
        loads_but<kFirst + kSecond>();
        barrier();
#pragma unroll
        for (int j = 0; j < F; j++) b_op[0][j] = read_b(0, j);
#pragma unroll
        for (int i = 0; i < H; i++) a_upper[i] = read_a(0, i);
        all_reads();
        barrier();
        // Whole runs of four: blocks behind the last take exponents of zero for both operands, a scale of 2^-254, and add nothing.  (One body for
        // all steps, whose sums stay where they are.)
        for (int kb = kb0; kb < kb1; kb += 4) {
            step(std::integral_constant<int, 0>{}, kb);
            step(std::integral_constant<int, 1>{}, kb + 1);
            step(std::integral_constant<int, 2>{}, kb + 2);
            step(std::integral_constant<int, 3>{}, kb + 3);
        }
        all_loads();
    }
    sums_are_there();
    store_tile<GATED>(out, t.a.rows, t.n, lds, acc, m0, n0, part);
}

// the same on the bfloat16 instruction
template <bool GATED, int FI>
__global__ __launch_bounds__(256) void wide_tile_kernel(wide_args t, tile_out out)
{
    extern __shared__ __align__(16) uint8_t lds[];
    wide_sums<WIDE_PRODUCT, GATED, FI>(t, lds, t.units, [&](int u) { return wide_unit_of<GATED, FI>(argument<wide_args>(), u); }, [&](const wide_unit &u, const f32x4 (&acc)[FI][8]) {
        const wide_args &t = argument<wide_args>();
        static_assert(sizeof(wide_args) % 8 == 0 && alignof(tile_out) <= 8, "where the second argument starts");
        const tile_out &out = argument<tile_out>(sizeof(wide_args));
        if constexpr (GATED) store_tile<GATED>(out, t.rows, t.cols, lds, acc, u.i0, u.j0, u.part);
        else store_sums(out.parts ? part_of(out.work, u.part, t.rows, t.cols) : out.y, t.rows, t.cols, acc, u.i0, u.j0);
    });
}

// in tiles of 64 x 64 (GATED: of 32 hidden units)
template <bool GATED>
__global__ __launch_bounds__(256, 4) void small_kernel(wide_args t, tile_out out)
{
    __shared__ __align__(16) uint8_t lds[kSmallLds];
    small_tile<WIDE_PRODUCT, GATED>(t, lds, [&](const wide_unit &u, int64_t row, int64_t col, f32x4 first, f32x4 second) {
        if constexpr (!GATED) {
            const fp8_matrix y = out.work ? part_of(out.work, u.part, t.rows, t.cols) : out.y;
            store_four(y, row, col, t.cols, first);
            store_four(y, row, col + 16, t.cols, second);
        } else if (out.work) {
            store_four(part_of(out.work, 2 * u.part, t.rows, t.cols), row, col, t.cols, first);
            store_four(part_of(out.work, 2 * u.part + 1, t.rows, t.cols), row, col, t.cols, second);
        } else {
            f32x4 h;
#pragma unroll
            for (int e = 0; e < 4; e++) h[e] = (out.gated.act == PVQ_SILU ? act_value<PVQ_SILU>(first[e]) : act_value<PVQ_GELU>(first[e])) * second[e];
            store_four(out.gated.h, row, col, t.cols, h);
        }
    });
}

// The tiles of a product, rows of 0 for those on the 8-bit instruction; join: whether the sums go to work, to be added there or taken to blocks.
struct product_plan {
    wide_tiles tiles;
    bool join;
};

product_plan plan_of(int64_t m, int64_t n, int64_t k, bool gated, bool wide, bool to_blocks)
{
    if (wide && !gated) {
        const wide_tiles t = wide_plan(m, n, k, 1, 1);
        return {t, t.parts > 1};
    }
    const int64_t values = m * n * (gated ? 2 : 1), tiles = (m + 255) / 256 * ((n + (gated ? 127 : 255)) / (gated ? 128 : 256)), steps = (k + kWideStep - 1) / kWideStep;
    wide_tiles large{wide ? 256 : 0, 256, 1, 0.0}, small{64, gated ? 32 : 64, 1, 0.0};
    // (8-bit: parts of whole runs of four blocks, the words of their exponents)
    large.parts = wide ? fp8_parts(tiles, steps, kWideStepUs, values, &large.us) : fp8_parts(tiles, (k + 4 * kFp8Block - 1) / (4 * kFp8Block), 4 * kByteStepUs, values, &large.us);
    small.parts = fp8_small_parts((m + 63) / 64 * ((n + small.cols - 1) / small.cols), steps, values, to_blocks, &small.us);
    if (to_blocks) large.us += 15.0 * (double)((tiles * large.parts + 255) / 256);              // (the codes of its epilogue)
    if (k && small.us < large.us) return {small, small.parts > 1 || to_blocks};
    return {large, large.parts > 1};
}

size_t work_of(int64_t m, int64_t n, int64_t k, bool gated, bool wide, bool to_blocks)
{
    const product_plan plan = plan_of(m, n, k, gated, wide, to_blocks);
    return plan.join ? (size_t)plan.tiles.parts * (gated ? 2 : 1) * m * n * 4 : 0;
}

// out.parts becomes 0 where there is nothing to join
template <bool GATED>
hipError_t launch_tiles(const fp8_blocks &a, const fp8_blocks &b, const fp8_blocks &up, tile_out &out, bool wide, bool to_blocks, hipStream_t s)
{
    const int64_t m = a.rows, n = b.rows, k = a.cols;
    const product_plan plan = plan_of(m, n, k, GATED, wide, to_blocks);
    constexpr int kLds = 2 * 2 * 256 * (kFp8Block + 4);
    auto allow = [](auto kernel, int bytes) { return hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
    out.parts = plan.join ? plan.tiles.parts : 0;
    if (!plan.join) out.work = nullptr;
    if (plan.tiles.rows == 0 || (GATED && plan.tiles.rows == 256)) {
        const int64_t across = (n + (GATED ? 127 : 255)) / (GATED ? 128 : 256), down = (m + 255) / 256;
        const dim3 grid((unsigned)(down * across), (unsigned)plan.tiles.parts);
        if (!wide) {
            const hipError_t e = allow(&tile_kernel<GATED>, kLds);
            if (e != hipSuccess) return e;
            const tile_args t{a, b, up, n, (int)down, (int)across, (int)(((a.blocks() + 3) / 4 + plan.tiles.parts - 1) / plan.tiles.parts * 4)};
            hipLaunchKernelGGL(tile_kernel<GATED>, grid, dim3(256), kLds, s, t, out);
            return hipGetLastError();
        }
    }
    wide_args t{};
    t.a = a; t.b[0] = b; t.b[1] = up;
    t.rows = m; t.cols = n; t.depth = k; t.terms = 1;
    wide_tiles tiles = plan.tiles;
    if (GATED && tiles.rows == 256) tiles.cols = 128;           // (hidden units)
    t.use(tiles, 1);
    if (tiles.rows == kSmallTile) {
        hipLaunchKernelGGL(small_kernel<GATED>, dim3((unsigned)t.units), dim3(256), 0, s, t, out);
        return hipGetLastError();
    }
    hipError_t e;
    if constexpr (GATED) {
        e = allow(&wide_tile_kernel<true, 8>, kWideLds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((wide_tile_kernel<true, 8>), dim3((unsigned)t.units), dim3(256), kWideLds, s, t, out);
    } else {
        const auto kernel = tiles.rows == 128 ? &wide_tile_kernel<false, 4> : &wide_tile_kernel<false, 8>;
        e = allow(kernel, kWideLds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(t.units, 256)), dim3(256), kWideLds, s, t, out);
    }
    return hipGetLastError();
}

}  // namespace

fp8_tiles fp8_product_tiles(int64_t m, int64_t n, int64_t k, bool gated, bool wide, bool to_blocks)
{
    const wide_tiles t = plan_of(m, n, k, gated, wide, to_blocks).tiles;
    return {t.rows, t.parts};
}
size_t fp8_product_work(int64_t m, int64_t n, int64_t k, int out_dtype) { return fp8_rows_pay(m) ? 0 : work_of(m, n, k, false, out_dtype == PVQ_F32, false); }
size_t fp8_gated_work(int64_t m, int64_t n, int64_t k, bool wide, bool to_blocks) { return work_of(m, n, k, true, wide, to_blocks); }

hipError_t fp8_launch_product(const fp8_product_args &p, hipStream_t s)
{
    tile_out out{};
    out.y = p.y; out.work = p.work;
    hipError_t e = launch_tiles<false>(p.a, p.b, {}, out, p.y.dtype == PVQ_F32, false, s);
    if (out.parts && e == hipSuccess) e = fp8_launch_join(p.work, out.parts, p.a.rows, p.b.rows, p.y, s);
    return e;
}

hipError_t fp8_launch_gated(const fp8_gated_args &g, hipStream_t s)
{
    tile_out out{};
    out.gated = {g.h, g.act, g.hc, g.he, g.gc, g.ge, g.uc, g.ue};
    out.work = g.work;
    hipError_t e = launch_tiles<true>(g.x, g.gate, g.up, out, fp8_gated_is_wide(g.gc != nullptr, g.h.data != nullptr, g.h.dtype), g.gc || g.hc, s);
    if (out.parts && e == hipSuccess) e = fp8_launch_gated_join(g.work, out.parts, g, s);
    return e;
}
