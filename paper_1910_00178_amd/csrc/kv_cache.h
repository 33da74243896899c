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
    static constexpr uint32_t kInfinityBits = 0x7f800000;
    static __device__ __forceinline__ float of_bits(uint32_t x) { return __uint_as_float(x); }
    static __device__ __forceinline__ float get(T x) { return x; }
    static __device__ __forceinline__ T put(float x) { return x; }
};
struct F16 {
    typedef _Float16 T;
    static constexpr uint32_t kInfinityBits = 0x7c00;
    static __device__ __forceinline__ float of_bits(uint32_t x) { return (float)__builtin_bit_cast(T, (uint16_t)x); }
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (_Float16)x; }
};
struct BF16 {
    typedef __bf16 T;
    static constexpr uint32_t kInfinityBits = 0x7f80;
    static __device__ __forceinline__ float of_bits(uint32_t x) { return __uint_as_float(x << 16); }
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (__bf16)x; }
};

// Packed rows of one kind: element (token, head, d) lies at token * token_stride + head * head_stride + d.
struct Rows {
    void *data;
    int64_t token_stride, head_stride;
};

// The last b of 0 .. batch - 1 with start(arrays[0][b], b) <= x (0 if there is none), start not falling, and what the arrays hold for it (0 for
// one that is null): 64 places are looked at together, the last 64 in all arrays at once, so that a batch of up to 64 takes one trip to memory.
template <int N, class F>
__device__ __forceinline__ int find_sequence(int batch, int x, const int32_t *const (&arrays)[N], int (&values)[N], F &&start)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = batch;
    while (n > 64) {
        const int step = (n + 63) / 64, at = lane * step;
        const int below = __popcll(__ballot(at < n && start(arrays[0][lo + min(at, n - 1)], lo + at) <= x));
        const int skip = max(below - 1, 0) * step;
        lo += skip;
        n = min(step, n - skip);
    }
    const int at = lo + min(lane, n - 1);
    int found[N];
#pragma unroll
    for (int i = 0; i < N; ++i) found[i] = arrays[i] ? arrays[i][at] : 0;
    const int below = __popcll(__ballot(lane < n && start(found[0], at) <= x)), of = __builtin_amdgcn_readfirstlane(max(below - 1, 0));
#pragma unroll
    for (int i = 0; i < N; ++i) values[i] = __builtin_amdgcn_readlane(found[i], of);
    return __builtin_amdgcn_readfirstlane(lo) + of;
}

struct MoveArgs {
    CacheView cache;
    Rows k, v;
    const int32_t *offsets, *starts;
    int32_t batch, tokens;
    int32_t heads;           // of a workgroup, one after the other
};

// Workgroups of the kernels below: one per some heads and block of the cache that the new tokens of a sequence may touch.  Sequence b has
// the slots (offsets[b] + 30 b) / 16 and on, at least as many as blocks, wherever its first token stands in one.
__host__ __device__ inline int64_t move_slots(int64_t offset, int64_t b) { return (offset + 30 * b) / kBlockTokens; }

struct MoveBlock {
    int b, row0, begin, end; // sequence; packed row of the block's token 0 (tokens begin .. end - 1 exist)
    int64_t index;           // of the block in the sequence

    __device__ __forceinline__ MoveBlock(const MoveArgs &a, int slot) : row0(0), begin(0), end(0)
    {
        int of[3];
        b = find_sequence(a.batch, slot, {a.offsets, a.offsets + 1, a.starts}, of, [](int offset, int x) { return (int)move_slots(offset, x); });
        const int first = min(max(of[0], 0), a.tokens), rows = min(max(of[1], first), a.tokens) - first;
        const int64_t start = of[2];
        // blocks of the sequence, from the one that holds its first token (which may stand before position 0)
        index = (start >> 4) + slot - (int)move_slots(of[0], b);
        const int64_t before = index * kBlockTokens - start;     // rows before the block's token 0
        if (before >= rows || before <= -kBlockTokens) return;
        row0 = first + (int)before;
        begin = before < 0 ? (int)-before : 0;
        end = (int)min((int64_t)kBlockTokens, rows - before);
    }
    // head 0's; null: no such place
    __device__ __forceinline__ uint8_t *block(const MoveArgs &a) const
    {
        return index >= 0 && index < (1 << 28) ? cache_block(a.cache, b, 0, (int)index) : nullptr;
    }
};

// Eight elements of a row.
template <class E>
struct Piece {
    typename E::T x[8];
};
template <class E, bool VEC>
__device__ __forceinline__ Piece<E> load_piece(const typename E::T *from)
{
    Piece<E> p;
    if constexpr (VEC) __builtin_memcpy(p.x, __builtin_assume_aligned(from, 16), sizeof(p.x));
    else
#pragma unroll
        for (int e = 0; e < 8; ++e) p.x[e] = from[e];
    return p;
}
// The largest of their bit patterns without signs: ordered as the magnitudes are, infinities and NaN on top.
template <class E>
__device__ __forceinline__ uint32_t most_bits(const Piece<E> &p)
{
    uint32_t w[sizeof(p.x) / 4], most = 0;
    __builtin_memcpy(w, p.x, sizeof(w));
    if constexpr (sizeof(typename E::T) == 2) {
        typedef uint16_t V2 __attribute__((ext_vector_type(2)));
        V2 m = {0, 0};
#pragma unroll
        for (uint32_t x : w) m = __builtin_elementwise_max(m, __builtin_bit_cast(V2, x & 0x7fff7fffu));
        most = max((uint32_t)m[0], (uint32_t)m[1]);
    } else {
#pragma unroll
        for (uint32_t x : w) most = max(most, x & 0x7fffffffu);
    }
    return most;
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

// Over aligned groups of 16 or 8 lanes.
template <int LANES, class T>
__device__ __forceinline__ T max_of_lanes(T x)
{
#define NGEMM_WITH(dpp) x = max(x, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), dpp, 0xf, 0xf, true)))
    if constexpr (LANES == 16) NGEMM_WITH(0x140);        // lane 15 - i's
    NGEMM_WITH(0x141);                                   // of 8 lanes, lane 7 - i's
    NGEMM_WITH(0x1b);                                    // of 4, lane 3 - i's
    NGEMM_WITH(0xb1);                                    // of 2, the other's
#undef NGEMM_WITH
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

// Codes of eight elements.  127 x / amax as one product is off by less than 2^-14 (its and the factor's roundings); where that could
// matter for a tie, and for rows of very small numbers, the quotient is formed as the definition says: 127 x relative to a power
// of two (exact for 16-bit types), one correctly rounded division.
template <class E>
__device__ __forceinline__ u2 quantise(const Piece<E> &p, float most, bool finite)
{
    constexpr float magic = 12582912.0f;                 // 1.5 2^23: the sum's low byte is the nearest whole number's, ties to even
    if (!finite || most == 0.0f) return (u2)(0u);
    const float by = 127.0f * __builtin_amdgcn_rcpf(most);
    float n[8], off = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = E::get(p.x[e]);
        n[e] = __builtin_fmaf(x, by, magic);
        off = fmaxf(off, fabsf(__builtin_fmaf(x, by, magic - n[e])));
    }
    if (off > 0.5f - 0x1p-14f || most < 0x1p-100f) {
        const int ex = __builtin_amdgcn_frexp_expf(most);
        const float m = __builtin_amdgcn_ldexpf(most, -ex);
#pragma unroll
        for (int e = 0; e < 8; ++e) n[e] = __builtin_amdgcn_ldexpf(E::get(p.x[e]), -ex) * 127.0f / m + magic;
    }
    u2 codes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 1]), __float_as_uint(n[4 * i]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(n[4 * i + 3]), __float_as_uint(n[4 * i + 2]), 0x0c0c0400u);
        codes[i] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
    return codes;
}

// A thread holds N pieces of eight elements of a token of K and of V, LANES lanes a token: 8 for heads of up to 64 elements, else 16.  V's codes
// pass LDS so that a thread holds four tokens of four elements, whose bytes it transposes.
//
// Bound by memory: each row is read once, stays in registers while its maximum is found, and leaves as codes.  15800 tokens of 8 heads of 128
// (bf16): 25 us, 3.9 TB/s read and written, where a large copy reaches 4.85 (f32 26 us; rows off 16-byte multiples 26 and 29); 64 sequences of a token each
// 4.7 us, a launch and four trips to memory one behind the other (offsets, page, rows and the stores).
template <class E, int LANES, int N, bool VEC>
__global__ __launch_bounds__(16 * LANES) void kv_write_kernel(const MoveArgs a)
{
    __shared__ __align__(16) uint32_t turned[2][16][2 * LANES * N + 1];
    typedef typename E::T T;
    const int groups = (a.cache.kv_heads + a.heads - 1) / a.heads, head0 = blockIdx.x % groups * a.heads;
    const int D = a.cache.head_dim, tid = threadIdx.x;
    const MoveBlock m(a, blockIdx.x / groups);
    if (m.begin >= m.end) return;
    const int token = tid / LANES, piece = tid % LANES;
    const bool there = token >= m.begin && token < m.end;
    const int64_t head_bytes = (int64_t)a.cache.page_blocks * a.cache.block_bytes();
    Piece<E> x[2][N];
    auto load = [&](int head) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const Rows &r = which ? a.v : a.k;
            const T *row = (const T *)r.data + (m.row0 + token) * r.token_stride + head * r.head_stride;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = piece + LANES * n;
                if (there && 8 * c < D) x[which][n] = load_piece<E, VEC>(row + 8 * c);
                else x[which][n] = Piece<E>{};
            }
        }
    };
    load(head0);                                         // on their way while the place is looked up
    uint8_t *block = m.block(a);
    if (!block) return;
    block += head0 * head_bytes;
    const int end = min(head0 + a.heads, a.cache.kv_heads);
    for (int head = head0, turn = 0; head < end; ++head, turn ^= 1, block += head_bytes) {
        if (head > head0) load(head);
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            uint32_t bits = 0;
#pragma unroll
            for (int n = 0; n < N; ++n) bits = max(bits, most_bits(x[which][n]));
            bits = max_of_lanes<LANES>(bits);
            const float most = E::of_bits(bits);
            const bool finite = bits < E::kInfinityBits;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const int c = piece + LANES * n;
                if (8 * c >= D) break;
                const u2 codes = quantise<E>(x[which][n], most, finite);
                if (which) {
                    turned[turn][token][2 * c] = codes[0];
                    turned[turn][token][2 * c + 1] = codes[1];
                } else if (there) {
                    *(u2 *)(block + token * D + 8 * c) = codes;
                }
            }
            if (there && piece == 0) ((float *)(block + 32 * D))[16 * which + token] = finite ? most / 127.0f : __builtin_nanf("");
        }
        __syncthreads();                                 // (the next head writes the other half)
        for (int i = tid; i < D; i += 16 * LANES) {             // tokens 4 t .. 4 t + 3 of elements 4 q .. 4 q + 3
            const int t = i & 3, q = i >> 2;
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = turned[turn][4 * t + j][q];
            transpose_bytes(y);
            uint8_t *to = block + 16 * D + 64 * q + 4 * t;
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
}

// Four codes times a scale, as floats (the compiler would round some products to 16 bits in one step, others in two).
__device__ __forceinline__ void values4(uint32_t codes, float scale, float *x)
{
    const uint32_t y = codes ^ 0x80808080u;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = ((float)(y >> (8 * e) & 255u) - 128.0f) * scale;
        asm("" : "+v"(x[e]));
    }
}

// K: LANES lanes a token, as above.  V: a thread takes four tokens of four elements and transposes their bytes.
//
// Bound by memory: 39700 tokens of 8 heads of 128 to bf16 53 us, 4.65 TB/s; 46000 of 16 heads of 64 in 64 us, 4.5 TB/s (82 with 16 lanes a token,
// of which half had nothing); up to 4 x 1000 tokens 5.4 us.  15800 of 8 heads of 128: 21 us, 27 to rows off 16-byte multiples; to f32 27 and 31.
template <class E, int LANES, int N, bool VEC>
__global__ __launch_bounds__(16 * LANES) void kv_read_kernel(const MoveArgs a)
{
    typedef typename E::T T;
    const int groups = (a.cache.kv_heads + a.heads - 1) / a.heads, head0 = blockIdx.x % groups * a.heads;
    const int D = a.cache.head_dim, tid = threadIdx.x;
    const MoveBlock m(a, blockIdx.x / groups);
    if (m.begin >= m.end) return;
    const uint8_t *const block0 = m.block(a);
    const bool there = block0 != nullptr;                // rows of places that do not exist are 0
    const int token = tid / LANES, piece = tid % LANES, t = tid & 3, q = tid >> 2;
    for (int head = head0; head < min(head0 + a.heads, a.cache.kv_heads); ++head) {
        const uint8_t *block = block0 + head * ((int64_t)a.cache.page_blocks * a.cache.block_bytes());
        u2 k[N] = {};
        uint32_t v[4] = {};
        float k_scale = 0.0f;
        f4 v_scale = (f4)(0.0f);
        if (there) {
            k_scale = ((const float *)(block + 32 * D))[token];
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (8 * (piece + LANES * n) < D) k[n] = *(const u2 *)(block + token * D + 8 * (piece + LANES * n));
            if (tid < D) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t *)(block + 16 * D + 64 * q + 4 * t + 16 * j);
                v_scale = *(const f4 *)(block + 32 * D + 64 + 16 * t);
            }
        }
        if (token >= m.begin && token < m.end) {
            T *row = (T *)a.k.data + (m.row0 + token) * a.k.token_stride + head * a.k.head_stride;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if (8 * (piece + LANES * n) >= D) break;
                float x[8];
                values4(k[n][0], k_scale, x);
                values4(k[n][1], k_scale, x + 4);
                store<E, 8, VEC>(row + 8 * (piece + LANES * n), x);
            }
        }
        if (tid < D) {
            transpose_bytes(v);
            T *column = (T *)a.v.data + (m.row0 + 4 * t) * a.v.token_stride + head * a.v.head_stride + 4 * q;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float x[4];
                values4(v[u], v_scale[u], x);
                if (4 * t + u >= m.begin && 4 * t + u < m.end) store<E, 4, VEC>(column + u * a.v.token_stride, x);
            }
        }
    }
}

}  // namespace ngemm
