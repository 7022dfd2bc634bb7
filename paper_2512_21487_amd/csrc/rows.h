// Rows of elements at any alignment and of any length, as the operators' kernels read them.
#pragma once
#include "common.h"

namespace moe_ep {

namespace {

// 16 or 8 bytes from an address that only the type of the elements aligns
typedef uint32_t u32x4_any2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float f32x4_any4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

// exp from the hardware's exp2: off by about a step of fp32 and by what the argument's own rounding makes of it
__device__ __forceinline__ float exp_f(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// 16 bytes of a row, the `left` first elements of which are there, and zeros.  A row of N elements and more: its last 16 bytes, shifted
// (an element at a time, the last K step of 1531 x 1409 x 2049 took 7 of 49 us).
template <int N, class T>
__device__ __forceinline__ u32x4_t load_part(const T* p, int left, int cols)
{
    if (left >= N) return *reinterpret_cast<const u32x4_any2*>(p);
    u32x4_t v = {0, 0, 0, 0};
    if (cols >= N) {
        if (left <= 0) return v;
        const u32x4_t u = *reinterpret_cast<const u32x4_any2*>(p - (N - left));
        const uint64_t lo = (uint64_t)u[1] << 32 | u[0], hi = (uint64_t)u[3] << 32 | u[2];
        const int drop = (N - left) * (128 / N);                     // bits, 16 .. 112
        const uint64_t a = drop < 64 ? lo >> drop | hi << (64 - drop) : hi >> (drop - 64), b = drop < 64 ? hi >> drop : 0;
        return u32x4_t{(uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32)};
    }
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        if (i >= left) continue;
        if constexpr (N == 8) v[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        else v[i] = __float_as_uint(p[i]);
    }
    return v;
}

}  // namespace

}  // namespace moe_ep
