// Tiles in LDS and operands of the bf16 32 x 32 x 16 products (gfx950): copies from global memory, reads along rows and
// transposed, the products and their waits.
#ifndef PSF_LDS_H
#define PSF_LDS_H

#include <hip/hip_runtime.h>
#include <stdint.h>
#include <type_traits>
#include <utility>

namespace psf {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x8 __attribute__((ext_vector_type(8)));

// An operand fragment whose contraction index runs across rows in LDS: every group of 16 lanes reads 4 rows x 16
// columns of 16-bit values (lane s: row s / 4, columns 4 (s % 4) ..+3 at its address) and lane i gets column i, rows
// 0..3 in order.  `a` gives entries 0..3 of the fragment, `b` entries 4..7.
__device__ __forceinline__ bf16x8 read_turned(const void *a, const void *b)
{
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4 *at;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(__attribute__((address_space(3))) const void *)a);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(__attribute__((address_space(3))) const void *)b);
    return __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Two wait states at the end of a loop body that ends in products whose results the next pass reads
// first.  The compiler counts the branches between a product and its reader before it turns some of
// them round, which leaves one wait state fewer than it meant to on the turned way.
__device__ __forceinline__ void branch_wait()
{
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 1");
}

__device__ __forceinline__ bf16x8 cvt8(f32x8 v) { return __builtin_convertvector(v, bf16x8); }
__device__ __forceinline__ bf16x8 cvt8_from16(const f32x16 &v, int first)
{
    f32x8 t;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = v[first + e];
    return cvt8(t);
}

template <int... Js, class F>
__device__ __forceinline__ void static_for_impl(std::integer_sequence<int, Js...>, F &&f)
{
    (f(std::integral_constant<int, Js>{}), ...);
}
// f(integral_constant<int, 0>) ... f(integral_constant<int, N - 1>), in order
template <int N, class F>
__device__ __forceinline__ void static_for(F &&f)
{
    static_for_impl(std::make_integer_sequence<int, N>{}, f);
}

// Direct global -> LDS copy of 16 bytes per lane: lane i of the wave lands at lds_wave_base +
// 16*i.  Completion is tracked by vmcnt; callers wait before the barrier that publishes it.
__device__ __forceinline__ void dma16(const void *gsrc_lane, void *lds_wave_base)
{
    // Written as assembly so that the compiler does not tie later LDS reads to these copies
    // with a full vmcnt(0) wait; callers count the copies in flight themselves (wait_vmem_le).
    // m0 carries the LDS destination; nothing else in these kernels uses m0.
    const uint32_t lds_off = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)lds_wave_base;
    asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off"
                 :
                 : "v"(gsrc_lane), "s"(__builtin_amdgcn_readfirstlane(lds_off))
                 : "memory");
}
// Same copy with the address split into a wave-uniform base (scalar registers) and a 32-bit
// per-lane byte offset: a loop that walks the base then spends no vector instructions on it.
// The destination is given as an LDS byte address (see lds_address).
__device__ __forceinline__ void dma16_sbase(const void *gsrc_uniform, uint32_t lane_byte_off, uint32_t lds_wave_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\tglobal_load_lds_dwordx4 %0, %1"
                 :
                 : "v"(lane_byte_off), "s"(gsrc_uniform), "s"(__builtin_amdgcn_readfirstlane(lds_wave_addr))
                 : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}
__device__ __forceinline__ void wait_all_memory() { __builtin_amdgcn_s_waitcnt(0); }
// Wait until at most N vector-memory operations of this wave are outstanding (they complete in
// order, so everything older has landed); LDS/scalar counters are left alone.
template <int N>
__device__ __forceinline__ void wait_vmem_le()
{
    static_assert(N >= 0 && N < 64, "vmcnt is 6 bits");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | (0x7 << 4) | (0xF << 8) | ((N >> 4) << 14));
}

// Rows of D 16-bit values staged in LDS as they lie in memory: the 16-byte piece p of row j at p ^ row_swz(j).  Plain
// reads (one piece of 16 consecutive rows) and transposed ones (two neighbouring pieces of 4 consecutive
// rows a 16-lane group, four pieces two groups) meet every bank once, with 32 banks as with 64.  Period: 16 rows.
// With it values are read where the caller has them; a pass that laid them out first, at the rate of a copy, cost
// (us a call, with and without): 60 units of 4096, no mask 97, 87; gradients of 96 units of 4096, d = 64 838, 778, 16 units of
// 16384, d = 128 2238, 2048; causal, 24 units of 32768 807, 768.
template <int D>
__device__ __forceinline__ constexpr int row_swz(int j)
{
    static_assert(D == 64 || D == 128, "8 or 16 pieces");
    if constexpr (D == 64) return ((j & 3) << 1) ^ ((j >> 2) & 1) ^ ((j >> 2) & 2);
    else return ((j & 1) * 10) ^ ((j & 2) << 1) ^ ((j >> 2) & 1) ^ (j & 8);
}
// Where lane `lane` of a copy that moves rows of D values, 16 bytes a lane, takes its piece from.
template <int D>
__device__ __forceinline__ uint32_t row_copy_offset(int lane)
{
    constexpr int PIECES = D / 8;
    const int row = lane / PIECES;
    return (uint32_t)((row * PIECES + (lane % PIECES ^ row_swz<D>(row))) * 16);
}
// Byte offset of this lane's read for a transposed fragment of staged rows: columns 32 ct .. of the four rows that
// start at row j0 (a multiple of four) of the lane's 16-lane group.
template <int D>
__device__ __forceinline__ uint32_t row_turned_offset(int lane, int j0, int ct)
{
    const int s16 = lane & 15, j = j0 + s16 / 4, p = 4 * ct + 2 * ((lane >> 4) & 1) + (s16 % 4) / 2;
    return (uint32_t)((j * (D / 8) + (p ^ row_swz<D>(j))) * 16 + (s16 & 1) * 8);
}

}  // namespace psf
#endif
