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

// Over the four lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_of_rows(float x)
{
    const u2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return max_of_halves(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}
__device__ __forceinline__ float sum_of_rows(float x)
{
    const u2 s = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return sum_of_halves(__uint_as_float(s[0]) + __uint_as_float(s[1]));
}

}  // namespace ngemm
