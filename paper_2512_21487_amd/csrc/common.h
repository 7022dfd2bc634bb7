// Device-side helpers shared by the HIP kernels of the expert-group MoE layer.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace moe_ep {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

constexpr int kWave = 64;          // CDNA wavefront

__device__ __forceinline__ float bf16_lo(uint32_t packed) { return __uint_as_float(packed << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t packed) { return __uint_as_float(packed & 0xffff0000u); }

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// two fp32 -> two bf16 (round to nearest even) in one 32-bit word, lo in the low half:
// gfx950's v_cvt_pk_bf16_f32
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const f32x2_t v = {lo, hi};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// Between an LDS access of one lane and that of another lane of the same wavefront to the same place: a wavefront's LDS
// accesses run in program order, so nothing has to be waited for, but the compiler must keep that order.
__device__ __forceinline__ void wavefront_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// g * sigmoid(g) from the hardware's exp2 and reciprocal (about 1 ulp each: far below the bf16
// rounding of the result); exp2 saturates to +inf / 0 at the ends, which give -0 and g
__device__ __forceinline__ float silu_f(float g)
{
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.4426950408889634f));
}

// Workgroups of a launch that may have more threads than the 2^32 of one grid dimension: rows of 2^20 workgroups (a multiple of the XCDs)
inline dim3 grid_of(long long workgroups)
{
    const long long x = workgroups < 1 << 20 ? workgroups : 1 << 20;
    return dim3((unsigned)x, (unsigned)((workgroups + x - 1) / x));
}
__device__ __forceinline__ long long workgroup() { return (long long)blockIdx.y * gridDim.x + blockIdx.x; }

}  // namespace moe_ep
