// device.h -- helpers that the device code of more than one file uses: launches
// that a recorder can time, bf16 conversions, waits and the workgroup barrier.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace corun {

// The events to record around the next launch (nullptr: none), noted in the
// recorder of set_launch_recorder.
void launch_events(hipEvent_t *start, hipEvent_t *stop);

#define KLAUNCH(kernel, grid, block, shmem, stream, ...)                                                   \
    do {                                                                                                    \
        hipEvent_t ks_, ke_;                                                                                \
        launch_events(&ks_, &ke_);                                                                          \
        if (ks_ != nullptr)                                                                                 \
            hipExtLaunchKernelGGL(kernel, grid, block, shmem, stream, ks_, ke_, 0, __VA_ARGS__);            \
        else                                                                                                \
            hipLaunchKernelGGL(kernel, grid, block, shmem, stream, __VA_ARGS__);                            \
    } while (0)

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf2f(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// fp32 -> bf16, round to nearest even, NaN quieted: gfx950's v_cvt_pk_bf16_f32
// (bit-identical, over all 2^32 inputs, to adding 0x7fff + lsb and truncating,
// with (u >> 16) | 0x40 for NaN)
__device__ __forceinline__ uint16_t f2bf(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
// two values in one instruction: a in the low half, b in the high half
__device__ __forceinline__ uint32_t f2bf2(float a, float b)
{
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

typedef float f32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ constexpr int vmcnt_imm(int n)
{
    return (n & 15) | ((n >> 4) << 14) | (7 << 4) | (15 << 8);   // vmcnt(n), expcnt and lgkmcnt not waited
}

__device__ __forceinline__ void lds_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Transposed LDS read (gfx950 ds_read_b64_tr_b16).  Within each group of 16
// lanes, lane a + 4 q supplies the address of four 16-bit values (row q,
// elements 4 a .. 4 a + 3 of some column block); lane i of the group then
// receives element i of the block from rows 0..3.  Two such reads give a
// lane eight consecutive rows of one column: the B (or A) operand of a bf16
// MFMA whose K runs along the rows, read from row-major tiles.
typedef short s16x4_tr __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint2 lds_read_tr16(const void *lds_ptr)
{
    typedef __attribute__((address_space(3))) s16x4_tr lds_s16x4;
    const s16x4_tr v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (lds_s16x4 *)(const __attribute__((address_space(3))) void *)lds_ptr);
    return __builtin_bit_cast(uint2, v);
}

// Value tiles in LDS are token-major, 16-byte chunk c of token t (KCH
// chunks per token) at t KCH + (c ^ vtile_swz<KCH>(t)).  A transposed read
// of the attention kernels takes, per 16-lane group, 32 bytes (two chunks)
// of four consecutive tokens 4 r + 0..3, and the two groups of a half
// wavefront read either the next two chunks of the same tokens or the same
// chunks of the tokens 8 further on.  The swizzle moves the four tokens to
// four distinct 16-bank ranges (bits 2-3 of the chunk, with the token's
// parity for 128-byte rows) and those 8 tokens further to the other half of
// each range (bit 1), so the 64 lanes of a half wavefront pair touch each
// of the 64 banks once.
template <int KCH>
__device__ __forceinline__ int vtile_swz(int t)
{
    static_assert(KCH == 8 || KCH == 16, "128- or 256-byte value rows");
    if constexpr (KCH == 16) return (4 * (t & 3)) ^ (2 * ((t >> 3) & 1));
    else return (4 * ((t >> 1) & 1)) ^ (2 * ((t >> 3) & 1));
}

// Prefill attention: the key that MFMA row m of a 32-key score tile carries (bits 2
// and 3 of m swapped), and the swizzled unit of chunk c of key row r.
__device__ __forceinline__ int pf_key_of_row(int m) { return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1); }

template <int KC>
__device__ __forceinline__ int pf_swz(int r, int c)
{
    // KC 16-byte chunks per row: 16 (256-byte rows) or 8 (128-byte rows)
    if constexpr (KC == 16) return r * 16 + (c ^ (r & 15));
    else return r * 8 + (c ^ ((r >> 1) & 7));
}

}  // namespace corun
