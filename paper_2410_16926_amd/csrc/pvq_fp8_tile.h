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
__device__ inline void load_words_to_lds(const void *base, uint32_t offset, uint32_t lds)     // 4 bytes a lane
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// The same from a buffer of `bytes` bytes (below 4 GiB), base, size and `uniform` in scalar registers: nothing is fetched from behind its end.
typedef __attribute__((ext_vector_type(4))) uint32_t buffer_t;
__device__ inline buffer_t make_buffer(const void *base, int64_t bytes)
{
    const uint64_t p = (uint64_t)base;
    return buffer_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)) & 0xFFFFu,
                    (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bytes), 0x00020000u};
}
__device__ inline void load_to_lds(buffer_t from, uint32_t offset, uint32_t uniform, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(from), "s"(uniform) : "memory", "m0");
}
__device__ inline void load_words_to_lds(buffer_t from, uint32_t offset, uint32_t uniform, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" : : "s"(lds), "v"(offset), "s"(from), "s"(uniform) : "memory", "m0");
}
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

// FM x FN fragments of 16 x 16 of a result to memory, from row0 and col0 on, rows and columns the result's.  A lane has four neighbouring columns of one
// row: columns 4 (lane / 16 % 4) .. of a fragment, row lane % 16.  vec: what y's rows are aligned to, 8 values, 4 or 1.
template <int FM, int FN, typename V>
__device__ __forceinline__ void store_fragments(const fp8_matrix &y, int vec, int64_t rows, int64_t cols, int64_t row0, int64_t col0, V value)
{
    const int lane = threadIdx.x % kWave, r16 = lane % 16, quarter = lane / 16;
    if (vec == 8 && row0 + FM * 16 <= rows && col0 + FN * 16 <= cols) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j += 2) store_pair(y, row0 + i * 16 + r16, col0 + j * 16, quarter, value(i, j), value(i, j + 1));
        return;
    }
#pragma unroll
    for (int i = 0; i < FM; i++) {
        const int64_t row = row0 + i * 16 + r16;
#pragma unroll
        for (int j = 0; j < FN; j++) {
            const int64_t col = col0 + j * 16 + 4 * quarter;
            const f32x4 v = value(i, j);
            if (row >= rows) continue;
            if (vec >= 4) store4<true>(y, row, col, cols - col, v);
            else store4<false>(y, row, col, cols - col, v);
        }
    }
}

inline int row_alignment(const fp8_matrix &y)
{
    const int size = y.dtype == PVQ_F32 ? 4 : 2;
    for (const int n : {8, 4})
        if ((uintptr_t)y.data % std::min(16, n * size) == 0 && y.ld % n == 0) return n;
    return 1;
}

}  // namespace pvq_fp8_dev
