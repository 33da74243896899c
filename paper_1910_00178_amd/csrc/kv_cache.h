// Device side of the 8-bit key-value cache: its addresses, and the kernels that write rows into it and read them back.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace ngemm {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));

constexpr int kBlockTokens = 16;                                 // tokens of a block, see include/ngemm.h

// One cache and the pages of a call's sequences in it.
struct CacheView {
    uint8_t *data;
    const int32_t *pages;
    int64_t pages_stride;
    int32_t num_pages, kv_heads, head_dim, page_blocks;
    __host__ __device__ int block_bytes() const { return 32 * head_dim + 8 * kBlockTokens; }
};

// The block that holds positions 16 * index .. of sequence b and a head, or null where there is none.  The page's number is checked, and
// the product of page, heads and blocks passes 32 bits in large caches.
__device__ __forceinline__ uint8_t *cache_block(const CacheView &c, int b, int head, int index)
{
    if (index < 0) return nullptr;
    const int page = index / c.page_blocks;
    if (page >= c.pages_stride) return nullptr;
    const int id = c.pages[b * c.pages_stride + page];
    if (id < 0 || id >= c.num_pages) return nullptr;
    return c.data + (((int64_t)id * c.kv_heads + head) * c.page_blocks + (index - page * c.page_blocks)) * c.block_bytes();
}

// Rows of a 16-bit or 32-bit type as floats and back, rounded to nearest even.
struct F32 {
    typedef float T;
    static __device__ __forceinline__ float get(T x) { return x; }
    static __device__ __forceinline__ T put(float x) { return x; }
};
struct F16 {
    typedef _Float16 T;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (_Float16)x; }
};
struct BF16 {
    typedef __bf16 T;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (__bf16)x; }
};

// Packed rows of one kind: element (token, head, d) lies at token * token_stride + head * head_stride + d.
struct Rows {
    void *data;
    int64_t token_stride, head_stride;
};

// The sequence that packed row `i` belongs to: the last b with offsets[b] <= i, of offsets[0 .. batch - 1].
__device__ __forceinline__ int sequence_of(const int32_t *offsets, int batch, int64_t i)
{
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (offsets[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

struct MoveArgs {
    CacheView cache;
    Rows k, v;
    const int32_t *offsets, *starts;
    int32_t batch, tokens;
};

// A wavefront per token and head: amax over the row by lane exchanges, then the codes.
template <class E>
__global__ __launch_bounds__(256) void kv_write_kernel(const MoveArgs a)
{
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 64;
    const int lane = threadIdx.x & 63, D = a.cache.head_dim;
    const int i = (int)(item / a.cache.kv_heads), head = (int)(item % a.cache.kv_heads);
    if (i >= a.tokens) return;
    const int b = sequence_of(a.offsets, a.batch, i);
    const int at = (a.starts ? a.starts[b] : 0) + i - a.offsets[b];
    uint8_t *block = at < 0 ? nullptr : cache_block(a.cache, b, head, at / kBlockTokens);
    if (!block) return;
    const int token = at % kBlockTokens;
    for (int which = 0; which < 2; ++which) {
        const Rows &r = which ? a.v : a.k;
        const typename E::T *row = (const typename E::T *)r.data + i * r.token_stride + head * r.head_stride;
        float x[4], most = 0.0f;
        bool finite = true;
        for (int n = 0; n < 4; ++n) {
            const int d = lane + 64 * n;
            x[n] = d < D ? E::get(row[d]) : 0.0f;
            finite = finite && __builtin_isfinite(x[n]);
            most = fmaxf(most, fabsf(x[n]));
        }
        finite = __all(finite);
        for (int s = 32; s; s /= 2) most = fmaxf(most, __shfl_xor(most, s));
        // relative to a power of two, so that 127 x neither overflows nor, for rows of 16-bit types, is rounded
        int e;
        (void)frexpf(most, &e);
        const float m = ldexpf(most, -e);
        for (int n = 0; n < 4; ++n) {
            const int d = lane + 64 * n;
            if (d >= D) continue;
            const int code = finite && most > 0.0f ? (int)rintf(ldexpf(x[n], -e) * 127.0f / m) : 0;
            block[which ? 16 * D + 16 * d + token : token * D + d] = (uint8_t)code;
        }
        if (lane == 0) ((float *)(block + 32 * D))[16 * which + token] = finite ? most / 127.0f : __builtin_nanf("");
    }
}

template <class E>
__global__ __launch_bounds__(256) void kv_read_kernel(const MoveArgs a)
{
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 64;
    const int lane = threadIdx.x & 63, D = a.cache.head_dim;
    const int i = (int)(item / a.cache.kv_heads), head = (int)(item % a.cache.kv_heads);
    if (i >= a.tokens) return;
    const int b = sequence_of(a.offsets, a.batch, i);
    const int at = (a.starts ? a.starts[b] : 0) + i - a.offsets[b];
    const uint8_t *block = at < 0 ? nullptr : cache_block(a.cache, b, head, at / kBlockTokens);
    const int token = at % kBlockTokens;
    for (int which = 0; which < 2; ++which) {
        const Rows &r = which ? a.v : a.k;
        typename E::T *row = (typename E::T *)r.data + i * r.token_stride + head * r.head_stride;
        const float scale = block ? ((const float *)(block + 32 * D))[16 * which + token] : 0.0f;
        for (int d = lane; d < D; d += 64) {
            const int code = block ? (int8_t)block[which ? 16 * D + 16 * d + token : token * D + d] : 0;
            row[d] = E::put((float)code * scale);
        }
    }
}

}  // namespace ngemm
