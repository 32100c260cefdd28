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

}  // namespace corun
