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

// Codes as 16-bit floats, in order: four, and 16.  A code with its sign bit turned, as the low byte under 0x64, is the float 1024 + 128 + code.
constexpr uint32_t kCodeSigns = 0x80808080u;
__device__ __forceinline__ u2 codes4_to_f16(uint32_t x, uint32_t signs = kCodeSigns)
{
    const uint32_t y = x ^ signs;
    const h2 base = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    return (u2){__builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, y, 0x04010400u)) + base),
                __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, y, 0x04030402u)) + base)};
}
__device__ __forceinline__ void codes_to_f16(u4 x, u4 (&out)[2], uint32_t signs = kCodeSigns)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const u2 y = codes4_to_f16(x[e], signs);
        out[e / 2][2 * (e % 2)] = y[0];
        out[e / 2][2 * (e % 2) + 1] = y[1];
    }
}

// Lane 16 r + K's value in all lanes 16 r .. 16 r + 15.
template <int K>
__device__ __forceinline__ float of_row(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x150 + K, 0xf, 0xf, true));
}

// Sums over a wavefront's lanes up to and with each.
template <class T>
__device__ __forceinline__ T sums_up_to(T x)
{
#define NGEMM_WITH(dpp, rows) x += __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), dpp, rows, 0xf, true))
    NGEMM_WITH(0x111, 0xf);                              // in rows of 16 lanes: the lane's 1, 2, 4, 8 before
    NGEMM_WITH(0x112, 0xf);
    NGEMM_WITH(0x114, 0xf);
    NGEMM_WITH(0x118, 0xf);
    NGEMM_WITH(0x142, 0xa);                              // rows 0 and 2 to the next
    NGEMM_WITH(0x143, 0xc);                              // row 1 to rows 2 and 3
#undef NGEMM_WITH
    return x;
}

// f(Index<0>) .. f(Index<N - 1>)
template <int I> struct Index { static constexpr int value = I; };
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled(F &&f)
{
    if constexpr (I < N) {
        f(Index<I>{});
        unrolled<N, I + 1>(f);
    }
}

}  // namespace ngemm
