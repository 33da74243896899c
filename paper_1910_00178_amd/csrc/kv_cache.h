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
    static constexpr uint32_t kOne = 0x3c00;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (_Float16)x; }
};
struct BF16 {
    typedef __bf16 T;
    static constexpr uint32_t kOne = 0x3f80;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (__bf16)x; }
};

// Packed rows of one kind: element (token, head, d) lies at token * token_stride + head * head_stride + d.
struct Rows {
    void *data;
    int64_t token_stride, head_stride;
};

// The last b of 0 .. batch - 1 with start(b) <= x (0 if there is none), start not falling: 64 places are looked at together.
template <class F>
__device__ __forceinline__ int last_start(int batch, int x, F &&start)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = batch;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const int below = __popcll(__ballot(at < n && start(lo + at) <= x));
        const int skip = max(below - 1, 0) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

struct MoveArgs {
    CacheView cache;
    Rows k, v;
    const int32_t *offsets, *starts;
    int32_t batch, tokens;
};

// Workgroups of the kernels below: one per head and block of the cache that the new tokens of a sequence may touch.  Sequence b has
// the slots (offsets[b] + 30 b) / 16 and on, at least as many as blocks, wherever its first token stands in one.
__host__ __device__ inline int64_t move_slots(int64_t offset, int64_t b) { return (offset + 30 * b) / kBlockTokens; }

struct MoveBlock {
    uint8_t *block;          // null: no such place
    int row0, begin, end;    // packed row of the block's token 0 (tokens begin .. end - 1 exist)
};

__device__ __forceinline__ MoveBlock move_block(const MoveArgs &a, int head, int slot)
{
    const int b = last_start(a.batch, slot, [&](int x) { return (int)move_slots(a.offsets[x], x); });
    const int first = min(max(a.offsets[b], 0), a.tokens), rows = min(max(a.offsets[b + 1], first), a.tokens) - first;
    const int64_t start = a.starts ? a.starts[b] : 0;
    // blocks of the sequence, from the one that holds its first token (which may stand before position 0)
    const int64_t index = (start >> 4) + slot - (int)move_slots(a.offsets[b], b);
    MoveBlock m{nullptr, 0, 0, 0};
    const int64_t before = index * kBlockTokens - start;         // rows before the block's token 0
    if (before >= rows || before <= -kBlockTokens) return m;
    m.row0 = first + (int)before;
    m.begin = before < 0 ? (int)-before : 0;
    m.end = (int)min((int64_t)kBlockTokens, rows - before);
    if (index >= 0 && index < (1 << 28)) m.block = cache_block(a.cache, b, head, (int)index);
    return m;
}

// Eight elements of a row.
template <class E, bool VEC>
__device__ __forceinline__ void load8(const typename E::T *from, float (&x)[8])
{
    typename E::T y[8];
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(y) / 16; ++i) ((u4 *)y)[i] = ((const u4 *)from)[i];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = from[e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = E::get(y[e]);
}
template <class E, int N, bool VEC>
__device__ __forceinline__ void store(typename E::T *to, const float (&x)[N])
{
    typename E::T y[N];
#pragma unroll
    for (int e = 0; e < N; ++e) y[e] = E::put(x[e]);
    if constexpr (VEC && sizeof(y) >= 16) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(y) / 16; ++i) ((u4 *)to)[i] = ((const u4 *)y)[i];
    } else if constexpr (VEC) {
        *(u2 *)to = *(const u2 *)y;
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = y[e];
    }
}

// Over the 16 lanes of a row.
__device__ __forceinline__ float max_in_row(float x)
{
#define NGEMM_TURN(n) x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + n, 0xf, 0xf, true)))
    NGEMM_TURN(8);
    NGEMM_TURN(4);
    NGEMM_TURN(2);
    NGEMM_TURN(1);
#undef NGEMM_TURN
    return x;
}

// The four dwords' bytes as a 4 x 4 matrix, transposed.
__device__ __forceinline__ void transpose_bytes(uint32_t (&x)[4])
{
    const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
    x[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    x[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    x[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    x[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// Codes of eight elements, and the row's scale.  127 x / amax as one product is off by less than 2^-14 (three roundings and the
// reciprocal's); where that could matter for a tie, and for rows of very small numbers, the quotient is formed as the definition
// says: 127 x relative to a power of two (exact for 16-bit types), one correctly rounded division.
__device__ __forceinline__ void quantise8(const float (&x)[8], float most, bool finite, uint32_t (&codes)[2])
{
    constexpr float magic = 12582912.0f;                 // 1.5 2^23: the sum's low byte is the nearest whole number's, ties to even
    codes[0] = codes[1] = 0;
    if (!finite || most == 0.0f) return;
    const float by = 127.0f * __builtin_amdgcn_rcpf(most);
    float n[8];
    bool doubtful = most < 0x1p-100f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = x[e] * by;
        n[e] = t + magic;
        doubtful = doubtful || fabsf(t - (n[e] - magic)) > 0.5f - 0x1p-14f;
    }
    if (doubtful) {
        const int ex = __builtin_amdgcn_frexp_expf(most);
        const float m = __builtin_amdgcn_ldexpf(most, -ex);
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = __builtin_amdgcn_ldexpf(x[e], -ex) * 127.0f / m + magic;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 1]), __float_as_uint(n[4 * i]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 3]), __float_as_uint(n[4 * i + 2]), 0x0c0c0400u);
        codes[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
}

// A thread holds up to two pieces of eight elements of a token of K and of V, 16 lanes a token.  V's codes pass LDS so that a thread holds
// four tokens of four elements, whose bytes it transposes.
template <class E, bool VEC>
__global__ __launch_bounds__(256) void kv_write_kernel(const MoveArgs a)
{
    __shared__ __align__(16) uint32_t turned[16][65];
    typedef typename E::T T;
    const int head = blockIdx.x % a.cache.kv_heads, D = a.cache.head_dim, tid = threadIdx.x;
    const MoveBlock m = move_block(a, head, blockIdx.x / a.cache.kv_heads);
    if (!m.block) return;
    const int token = tid >> 4, piece = tid & 15;
    const bool there = token >= m.begin && token < m.end;
    float x[2][2][8];
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const Rows &r = which ? a.v : a.k;
        const T *row = (const T *)r.data + (m.row0 + token) * r.token_stride + head * r.head_stride;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int c = piece + 16 * n;
            if (there && 8 * c < D) {
                load8<E, VEC>(row + 8 * c, x[which][n]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[which][n][e] = 0.0f;
            }
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float most = 0.0f, odd = 0.0f;                   // odd: NaN where an element is an infinity or a NaN, else 0
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                most = fmaxf(most, fabsf(x[which][n][e]));
                odd = __builtin_fmaf(x[which][n][e], 0.0f, odd);
            }
        most = max_in_row(most);
        const bool finite = max_in_row(odd == 0.0f ? 0.0f : 1.0f) == 0.0f;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int c = piece + 16 * n;
            if (8 * c >= D) break;
            uint32_t codes[2];
            quantise8(x[which][n], most, finite, codes);
            if (which) {
                turned[token][2 * c] = codes[0];
                turned[token][2 * c + 1] = codes[1];
            } else if (there) {
                *(u2 *)(m.block + token * D + 8 * c) = (u2){codes[0], codes[1]};
            }
        }
        if (there && piece == 0) ((float *)(m.block + 32 * D))[16 * which + token] = finite ? most / 127.0f : __builtin_nanf("");
    }
    __syncthreads();
    for (int i = tid; i < D; i += 256) {                 // tokens 4 t .. 4 t + 3 of elements 4 q .. 4 q + 3
        const int t = i & 3, q = i >> 2;
        uint32_t y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = turned[4 * t + j][q];
        transpose_bytes(y);
        uint8_t *to = m.block + 16 * D + 64 * q + 4 * t;
        if (4 * t >= m.begin && 4 * t + 4 <= m.end) {
#pragma unroll
            for (int j = 0; j < 4; ++j) *(uint32_t *)(to + 16 * j) = y[j];
        } else {
            for (int u = 0; u < 4; ++u)
                if (4 * t + u >= m.begin && 4 * t + u < m.end)
#pragma unroll
                    for (int j = 0; j < 4; ++j) to[16 * j + u] = (uint8_t)(y[j] >> (8 * u));
        }
    }
}

// Four codes times a scale.
__device__ __forceinline__ void values4(uint32_t codes, float scale, float *x)
{
    const uint32_t y = codes ^ 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = ((float)(y >> (8 * e) & 255u) - 128.0f) * scale;
}

template <class E, bool VEC>
__global__ __launch_bounds__(256) void kv_read_kernel(const MoveArgs a)
{
    typedef typename E::T T;
    const int head = blockIdx.x % a.cache.kv_heads, D = a.cache.head_dim, tid = threadIdx.x;
    const MoveBlock m = move_block(a, head, blockIdx.x / a.cache.kv_heads);
    if (m.begin >= m.end) return;
    const bool block = m.block != nullptr;               // rows of places that do not exist are 0
    {
        const int token = tid >> 4;
        if (token >= m.begin && token < m.end) {
            T *row = (T *)a.k.data + (m.row0 + token) * a.k.token_stride + head * a.k.head_stride;
            const float scale = block ? ((const float *)(m.block + 32 * D))[token] : 0.0f;
            for (int c = tid & 15; 8 * c < D; c += 16) {
                const u2 codes = block ? *(const u2 *)(m.block + token * D + 8 * c) : (u2)(0u);
                float x[8];
                values4(codes[0], scale, x);
                values4(codes[1], scale, x + 4);
                store<E, 8, VEC>(row + 8 * c, x);
            }
        }
    }
    for (int i = tid; i < D; i += 256) {                 // tokens 4 t .. 4 t + 3 of elements 4 q .. 4 q + 3
        const int t = i & 3, q = i >> 2;
        uint32_t y[4] = {};
        f4 scale = (f4)(0.0f);
        if (block) {
            const uint8_t *from = m.block + 16 * D + 64 * q + 4 * t;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = *(const uint32_t *)(from + 16 * j);
            scale = *(const f4 *)(m.block + 32 * D + 64 + 16 * t);
        }
        transpose_bytes(y);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int token = 4 * t + u;
            if (token < m.begin || token >= m.end) continue;
            float x[4];
            values4(y[u], scale[u], x);
            store<E, 4, VEC>((T *)a.v.data + (m.row0 + token) * a.v.token_stride + head * a.v.head_stride + 4 * q, x);
        }
    }
}

}  // namespace ngemm
