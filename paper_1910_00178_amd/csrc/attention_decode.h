// Attention of one token per sequence over the 8-bit cache.
#pragma once
#include "kv_cache.h"

namespace ngemm {

struct DecodeArgs {
    CacheView cache;
    Rows q, o;
    const int32_t *lengths;
    int32_t batch, q_heads, max_length;
    float scale;
};

// A wavefront per sequence and query head, 64 tokens at a time: lanes are tokens in the first product, elements of V in the second.
template <class E>
__global__ __launch_bounds__(64) void attention_decode_kernel(const DecodeArgs a)
{
    __shared__ float q[256], p[64];
    const int b = blockIdx.x / a.q_heads, h = blockIdx.x % a.q_heads, lane = threadIdx.x, D = a.cache.head_dim;
    const int g = h / (a.q_heads / a.cache.kv_heads);
    const typename E::T *qrow = (const typename E::T *)a.q.data + b * a.q.token_stride + h * a.q.head_stride;
    for (int d = lane; d < D; d += 64) q[d] = E::get(qrow[d]) * a.scale;
    __syncthreads();
    const int length = min(a.lengths[b], a.max_length);
    float m = -__builtin_inff(), l = 0.0f, o[4] = {};
    for (int t0 = 0; t0 < length; t0 += 64) {
        const int t = t0 + lane;
        const uint8_t *block = t < length ? cache_block(a.cache, b, g, t / 16) : nullptr;
        float s = -__builtin_inff(), vs = 0.0f;
        if (block) {
            const int8_t *k = (const int8_t *)block + (t & 15) * D;
            float dot = 0.0f;
            for (int d = 0; d < D; ++d) dot += q[d] * k[d];
            const float *scales = (const float *)(block + 32 * D);
            s = dot * scales[t & 15];
            vs = scales[16 + (t & 15)];
        }
        float most = s;
        for (int x = 32; x; x /= 2) most = fmaxf(most, __shfl_xor(most, x));
        const float now = fmaxf(m, most), ref = now == -__builtin_inff() ? 0.0f : now;
        const float w = block ? expf(s - ref) : 0.0f, fall = expf(m - ref);
        float sum = w;
        for (int x = 32; x; x /= 2) sum += __shfl_xor(sum, x);
        l = l * fall + sum;
        m = now;
        __syncthreads();
        p[lane] = block ? w * vs : 0.0f;
        __syncthreads();
        for (int n = 0; n < 4; ++n) o[n] *= fall;
        for (int u = 0; u < 64 && t0 + u < length; u += 16) {
            const int8_t *v = (const int8_t *)cache_block(a.cache, b, g, (t0 + u) / 16);
            if (!v) continue;
            for (int n = 0; n < 4; ++n) {
                const int d = lane + 64 * n;
                if (d < D)
                    for (int j = 0; j < 16; ++j) o[n] += p[u + j] * v[16 * D + 16 * d + j];
            }
        }
    }
    typename E::T *out = (typename E::T *)a.o.data + b * a.o.token_stride + h * a.o.head_stride;
    for (int n = 0; n < 4; ++n) {
        const int d = lane + 64 * n;
        if (d < D) out[d] = E::put(length > 0 && l != 0.0f ? o[n] / l : 0.0f);
    }
}

}  // namespace ngemm
