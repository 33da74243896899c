// What the attention kernels share.
#pragma once
#include "kv_cache.h"

namespace ngemm {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void *lds_ptr;
typedef __attribute__((address_space(3))) s4 *lds_s4;

__device__ __forceinline__ f16v mfma32(F16, u4 a, u4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f16v mfma32(BF16, u4 a, u4 b, f16v c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

__device__ __forceinline__ f4 mfma16(u4 a, u4 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// Two floats rounded to nearest even, packed.
template <class E>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    typedef typename E::T T2 __attribute__((ext_vector_type(2)));
    typedef float V2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((V2){lo, hi}, T2));
}

// What lane l and lane l ^ 32 hold, both in both lanes.
__device__ __forceinline__ float max_of_halves(float x)
{
    const u2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_of_halves(float x)
{
    const u2 s = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// Work on one output that is split over workgroups: each stores its part in the workspace, and the one that finds the others' flags set joins
// them.  A flag is set to the call's own number, which no workspace holds by chance, and cleared by who joins, so that a workspace needs no
// clearing and a captured call can be replayed.  Nobody waits: whoever sets the last flag finds all of them, unless another that
// found them too has begun to clear.
// Parts and flags go through accesses of device scope, which every XCD's L2 passes on: a fence in their place writes the whole L2 back
// (measured: 124 us a call where this takes NEW).
__device__ __forceinline__ void store_part(f4 *to, f4 x)
{
    const uint64_t lo = (uint64_t)__float_as_uint(x[1]) << 32 | __float_as_uint(x[0]), hi = (uint64_t)__float_as_uint(x[3]) << 32 | __float_as_uint(x[2]);
    __hip_atomic_store((uint64_t *)to, lo, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store((uint64_t *)to + 1, hi, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f4 load_part(const f4 *from)
{
    const uint64_t lo = __hip_atomic_load((const uint64_t *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    const uint64_t hi = __hip_atomic_load((const uint64_t *)from + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return (f4){__uint_as_float((uint32_t)lo), __uint_as_float((uint32_t)(lo >> 32)), __uint_as_float((uint32_t)hi), __uint_as_float((uint32_t)(hi >> 32))};
}
// All threads of the workgroup call this after their stores, with 4 bytes of LDS; what it returns is the same in all of them.
__device__ __forceinline__ bool all_parts_stored(uint64_t *flags, int parts, int mine, uint64_t call, volatile int *shared)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // this wavefront's stores are at the device's point of coherence
    __syncthreads();
    if (threadIdx.x < 64) {
        if (threadIdx.x == 0) (void)__hip_atomic_exchange(flags + mine, call, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        bool there = true;
        for (int i = threadIdx.x; i < parts; i += 64)
            there = there && __hip_atomic_load(flags + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == call;
        there = __all(there);
        if (there)
            for (int i = threadIdx.x; i < parts; i += 64) __hip_atomic_store(flags + i, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (threadIdx.x == 0) *shared = there;
    }
    __syncthreads();
    return *shared != 0;
}

}  // namespace ngemm
