// What the kernels share that stage tokens in LDS for many query rows (ffd_prefix.hip has the mapping).
#pragma once

#include "ffd_attend.h"

namespace ffd {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

constexpr float kSlack = 8.f;                  // growth of the maximum, in powers of two, that rescales

// Chunk order of the two kinds of rows.
__device__ __forceinline__ int key_chunk(int row, int c) { return c ^ (row & 15); }
template <bool I8>                             // 8 bits: a store takes every second chunk of two rows, which then complement
__device__ __forceinline__ int value_chunk(int row, int c) { return c ^ (((row & 3) << 2) | ((row >> 2) & 3)) ^ (I8 ? row & 1 : 0); }

__device__ __forceinline__ float halves_max(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// For loads straight to LDS written as assembly, which the compiler does not count.
__device__ __forceinline__ void wait_for_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

// x plus both bf16 values of a pair.
__device__ __forceinline__ float pair_sum(uint32_t pair, float x) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf, pair), v2bf{(__bf16)1.f, (__bf16)1.f}, x, false);
}

}  // namespace ffd
