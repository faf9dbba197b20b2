// What the kernels with tiles of 256 x 256 share: loads into LDS, waits and barriers, sums in accumulation registers.
#pragma once

#include "pvq_fp8_dev.h"

namespace pvq_fp8_dev {

// ---- loads into LDS --------------------------------------------------------------------------------------------------
// 1 KiB a wave: lane i's 16 bytes from `base` + `offset` to `lds` + 16 i.  The compiler does not count these loads: they are
// waited for by hand (all_loads) in front of the barrier behind which they are read.
__device__ inline void load_to_lds(const void *base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// The same from a buffer of `bytes` bytes (below 4 GiB), base, size and `uniform` in scalar registers: nothing is fetched from behind its end.
typedef __attribute__((ext_vector_type(4))) uint32_t buffer_t;
__device__ inline buffer_t make_buffer(const void *base, int64_t bytes)
{
    const uint64_t p = (uint64_t)base;
    return buffer_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) & 0xFFFFu,
                    (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bytes), 0x00020000u};
}
// (these have `lds` for an operand, not in their name: no register of theirs is written)
#define PVQ_BUFFER_TO_LDS(width) "s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_" width " %1, %2, %3 offen lds"
__device__ inline void load_to_lds(buffer_t from, uint32_t offset, uint32_t uniform, uint32_t lds)
{
    asm volatile(PVQ_BUFFER_TO_LDS("dwordx4") : : "s"(lds), "v"(offset), "s"(from), "s"(uniform) : "memory", "m0");
}
__device__ inline void load_words_to_lds(buffer_t from, uint32_t offset, uint32_t uniform, uint32_t lds)     // 4 bytes a lane
{
    asm volatile(PVQ_BUFFER_TO_LDS("dword") : : "s"(lds), "v"(offset), "s"(from), "s"(uniform) : "memory", "m0");
}
#undef PVQ_BUFFER_TO_LDS
__device__ inline void all_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

// all but the last N
template <int N>
__device__ inline void loads_but() { asm volatile("s_waitcnt vmcnt(%0)" : : "i"(N) : "memory"); }
// what a wave has read from LDS is in its registers
__device__ inline void all_reads() { asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory"); }
// (matrix instructions touch no memory: nothing but the scheduling barriers keeps them on their side)
__device__ inline void barrier()
{
    asm volatile("" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" : : : "memory");
}

__device__ inline uint32_t lds_address(const void *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)p; }

// Tiles of the result in bands of 8 rows of tiles, down a band's columns one after the other: the workgroups of a chiplet
// at work at one time share few rows of A and B in its L2.
__device__ inline void tile_of(int tiles_m, int tiles_n, int id, int &tm, int &tn)
{
    constexpr int kBand = 8;
    const int per = kBand * tiles_n, band = id / per, rows = min(kBand, tiles_m - band * kBand), in = id - band * per;
    // (in scalar registers, as are the addresses that follow from them)
    tm = __builtin_amdgcn_readfirstlane(band * kBand + in % rows);
    tn = __builtin_amdgcn_readfirstlane(in / rows);
}

// ---- sums in accumulation registers ----------------------------------------------------------------------------------
// Those of 128 x 128 fill all 256, and nothing else is in them: left to the compiler, they move between the two halves of the register file in
// the loop, to make room beside the operands.  So the matrix instructions that add to them, and what reads them, are written by hand; a result is
// read behind sums_are_there, 8 passes of 4 cycles at least.
__device__ inline void sums_are_there()
{
    asm volatile("s_nop 15\n\ts_nop 15\n\ts_nop 15" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

__device__ __forceinline__ f32x4 read_sums(const f32x4 &c)
{
    f32x4 v;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        float x;
        asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(c[e]));
        v[e] = x;
    }
    return v;
}

// 8-bit instruction, 16 x 16 x 128, with byte AT of words of four exponents
template <int AT>
__device__ __forceinline__ void multiply_accumulated(f32x4 &c, i32x8 a, uint32_t ea, i32x8 b, uint32_t eb)
{
    asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%5,0] op_sel_hi:[%6,%6,0]"
                 : "+a"(c) : "v"(a), "v"(b), "v"(ea), "v"(eb), "n"(AT & 1), "n"(AT >> 1));
}

// bfloat16 instruction, 16 x 16 x 32
__device__ __forceinline__ void multiply_accumulated(f32x4 &c, bf16x8 a, bf16x8 b)
{
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}

// A kernel's argument that starts at byte `offset` of them, read anew: kept in scalar registers for what happens once a tile, arguments leave too few
// of them to the steps.
template <typename T>
__device__ __forceinline__ const T &argument(int offset = 0)
{
    auto p = (const __attribute__((address_space(4))) uint8_t *)(uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const T *)(p + offset);
}

// All sums zero, where they are.
template <int FI>
__device__ __forceinline__ void no_sums(f32x4 (&acc)[FI][8])
{
    u32x4 zero{0, 0, 0, 0};
    asm volatile("s_nop 7" : "+v"(zero));                // (written, and some instructions before the first below)
#pragma unroll
    for (int i = 0; i < FI; i++)
#pragma unroll
        for (int j = 0; j < 8; j++) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %1, 0" : "+a"(acc[i][j]) : "v"(zero));
}

// The sums of a tile of 256 x 256 to its rows, by way of LDS (128 KB of it), which everybody has read and nobody loads into any more.  A lane has
// four neighbouring columns of one row of a fragment: row lane % 16, columns 4 (lane / 16) ..; the rows are taken whole again, in short loops.  (The
// first workgroups of a launch wait for each line of instructions: stored from where the sums are, unrolled over 64 fragments for every type and
// alignment, that was 200 KB of them.)  column(j): where a wave's fragments j start.
// rows(half, at): what becomes of the upper or the lower 64 rows of both waves that are side by side; at(r, chunk) is where four columns of the
// half's row r are (row tile_row(half, r) of the tile).
__device__ inline int tile_row(int half, int r) { return r / 64 * 128 + half * 64 + r % 64; }

template <typename COLUMN, typename ROWS>
__device__ __forceinline__ void store_rows(uint8_t *lds, const f32x4 (&acc)[8][8], COLUMN column, ROWS rows)
{
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int wm = wave / 2, r16 = lane % 16, quarter = lane / 16;
    // row r of 256 columns, a KiB in 64 chunks of four; chunk c lies at place c ^ (r % 16)
    auto at = [&](int r, int chunk) { return reinterpret_cast<f32x4 *>(lds + r * 1024 + ((chunk ^ (r & 15)) << 4)); };
#pragma unroll
    for (int half = 0; half < 2; half++) {
        all_reads();                                     // (not the stores, as __syncthreads would)
        barrier();
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < 8; j++) *at(wm * 64 + i * 16 + r16, column(j) / 4 + quarter) = read_sums(acc[half * 4 + i][j]);
        all_reads();
        barrier();
        rows(half, at);
    }
}

// A tile's sums to a matrix, the tile's first at row0, col0, from where they are: LDS may hold the next tile's operands by now.  Four waves of 16 FI x 128;
// a lane has four neighbouring columns of one row of a fragment.  float32 is stored so, 16 rows of 64 bytes at a time.  Of 16-bit types two fragments'
// halves and quarters change places, after which a lane has eight neighbouring columns: 64 bytes of a row again.  (Every sum is read at one place,
// whatever the type: of reads in several branches the compiler moves some up, to where the sums need not be there yet.)
template <int FI>
__device__ __forceinline__ void store_sums(const fp8_matrix &y, int64_t rows, int64_t cols, const f32x4 (&acc)[FI][8], int64_t row0, int64_t col0)
{
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), r16 = lane % 16, quarter = lane / 16;
    row0 += wave / 2 * 16 * FI;
    col0 += wave % 2 * 128;
    const bool inside = row0 + 16 * FI <= rows && col0 + 128 <= cols, f32 = y.dtype == PVQ_F32, bf16 = y.dtype == PVQ_BF16;
    const int bytes = f32 ? 4 : 2;
    const int64_t row = row0 + r16, col = col0 + quarter * (f32 ? 4 : 8);
    uint8_t *to = reinterpret_cast<uint8_t *>(y.data) + (row * y.ld + col) * bytes;
#pragma unroll
    for (int i = 0; i < FI; i++, to += 16 * y.ld * bytes) {
        const bool there = row + 16 * i < rows;
        const int64_t left = there ? cols - col : 0;
        __builtin_amdgcn_sched_barrier(0);
        f32x4 s[8];
#pragma unroll
        for (int j = 0; j < 8; j++) s[j] = read_sums(acc[i][j]);
        if (f32) {
            float *at = reinterpret_cast<float *>(to);
            if (__builtin_expect(inside, 1)) {
#pragma unroll
                for (int j = 0; j < 8; j++) store_vector(at + 16 * j, s[j]);
                continue;
            }
#pragma unroll
            for (int j = 0; j < 8; j++) {
                if (left >= 16 * j + 4) store_vector(at + 16 * j, s[j]);
                else {
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        if (16 * j + e < left) at[16 * j + e] = s[j][e];
                }
            }
            continue;
        }
        uint32_t w[8][2];
        if (bf16) {
#pragma unroll
            for (int j = 0; j < 8; j++) { w[j][0] = bf16_pair(s[j][0], s[j][1]); w[j][1] = bf16_pair(s[j][2], s[j][3]); }
        } else {
#pragma unroll
            for (int j = 0; j < 8; j++) { w[j][0] = f16_pair(s[j][0], s[j][1]); w[j][1] = f16_pair(s[j][2], s[j][3]); }
        }
        u32x4 v[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int e = 0; e < 2; e++) {
                const auto halves = __builtin_amdgcn_permlane32_swap(w[2 * j][e], w[2 * j + 1][e], false, false);
                const auto quarters = __builtin_amdgcn_permlane16_swap(halves[0], halves[1], false, false);
                v[j][e] = quarters[0];
                v[j][2 + e] = quarters[1];
            }
        uint16_t *at = reinterpret_cast<uint16_t *>(to);
        if (__builtin_expect(inside, 1)) {
#pragma unroll
            for (int j = 0; j < 4; j++) store_vector(at + 32 * j, v[j]);
            continue;
        }
#pragma unroll
        for (int j = 0; j < 4; j++) {
            if (left >= 32 * j + 8) store_vector(at + 32 * j, v[j]);
            else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (32 * j + e < left) at[32 * j + e] = (uint16_t)(v[j][e / 2] >> 16 * (e % 2));
            }
        }
    }
}

// ... a split's, rows of `cols` sums without a gap
__device__ __forceinline__ fp8_matrix part_of(float *work, int64_t part, int64_t rows, int64_t cols) { return {work + part * rows * cols, PVQ_F32, cols}; }

}  // namespace pvq_fp8_dev
