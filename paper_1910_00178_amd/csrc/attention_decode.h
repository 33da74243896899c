// Attention of one token per sequence over the 8-bit cache.
#pragma once
#include "attention_common.h"

namespace ngemm {

struct DecodeArgs {
    CacheView cache;
    Rows q, o;
    const int32_t *lengths;
    int32_t batch, q_heads, max_length;
    int32_t chunk, chunks;   // tokens of a workgroup, workgroups along a sequence
    float scale;             // of the scores, times log2 e
    f4 *parts;               // chunks > 1: [batch][q_heads][chunks] times head_dim / 4 + 1: maximum and weight, sums
    int32_t o_pieces;        // whether rows of O lie at 16-byte multiples
};

// (what the registers allow; told to the compiler, which otherwise takes some more for the rare branch of the tile loop)
constexpr int decode_waves_per_simd(int D) { return D <= 64 ? 4 : D <= 96 ? 3 : D <= 192 ? 2 : 1; }

// 16 codes as 16-bit floats, in order.  A code with its sign bit turned, as the low byte under 0x64, is the float 1024 + 128 + code.
constexpr uint32_t kCodeSigns = 0x80808080u;
__device__ __forceinline__ void codes_to_f16(u4 x, u4 (&out)[2], uint32_t signs = kCodeSigns)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t y = x[e] ^ signs;
        const h2 base = {(_Float16)-1152.0f, (_Float16)-1152.0f};
        const h2 lo = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, y, 0x04010400u)) + base;
        const h2 hi = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, y, 0x04030402u)) + base;
        out[e / 2][2 * (e % 2)] = __builtin_bit_cast(uint32_t, lo);
        out[e / 2][2 * (e % 2) + 1] = __builtin_bit_cast(uint32_t, hi);
    }
}

// Of two 16-bit floats those without a sign, else 0.
__device__ __forceinline__ uint32_t positive_halves(uint32_t x)
{
    typedef int16_t V2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(V2, x), (V2)(int16_t)0));
}

// Lane 16 r + K's value in all lanes 16 r .. 16 r + 15.
template <int K>
__device__ __forceinline__ float of_row(float x)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x150 + K, 0xf, 0xf, true));
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

// Elements d .. d + 3 of an output row (0 where nothing was seen).
template <class E>
__device__ __forceinline__ void put_row(const DecodeArgs &a, int b, int qh, int d, f4 sum, float weight)
{
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = weight == 0.0f ? 0.0f : sum[e] / weight;
    typename E::T *to = (typename E::T *)a.o.data + b * a.o.token_stride + qh * a.o.head_stride + d;
    if (a.o_pieces) store<E, 4, true>(to, x);
    else store<E, 4, false>(to, x);
}

// A wavefront takes tiles of 64 tokens = 4 blocks: S^T = K Q^T and O^T = V^T P^T on 16 x 16 x 32 matrix instructions, up to 16 heads that share
// a K/V head.  Row r of the first product's tile t is token 4 t + r % 4 of block r / 4, so that lane 16 g + h holds head h's scores of
// block g's tokens, which is what the second product wants of it: the 16 tokens of a row of V in a block are the lane's 16-byte load.
// D: head_dim, known to the compiler so that the loads of a tile are one run without branches.
// NW wavefronts of a workgroup take the chunk's tiles in turn, each with a running maximum and sum, merged through LDS at the end.
//
// Bound by reading the cache, 2 D + 8 bytes a token and K/V head, read once for all heads that share it, straight to registers: no two
// wavefronts want the same bytes.  What counts is bytes on their way, so K of the next tile and V of this one are (V asked for at the loop's
// top and not where it ends: the compiler's waits then count K and V apart).  8 sequences of 100000 to 131072 tokens (8 K/V heads of 128, 32 heads,
// bf16): the kernel alone 344 to 348 us, 5.7 to 5.8 TB/s, where a large read reaches 6.15; 64 sequences of up to 8192: 69 to 71 us, 3.9 to 4.0 TB/s, the
// workgroups' loads unequal; 32 of up to 1000 (12 heads of 64): 8.6 to 9.5 us; one of 4097: 5.7 to 5.9 us, a chain of three trips to memory (length,
// page, rows) and the tiles behind it.  A wavefront has work for 16 rows whatever the heads that share a K/V head; with one to four of them the matrix
// instructions idle, which costs nothing here.
template <class E, int D, int NW>
__global__ __launch_bounds__(NW * 64, decode_waves_per_simd(D)) void attention_decode_kernel(const DecodeArgs a)
{
    extern __shared__ __align__(16) float shared[];
    constexpr int NJ = (D + 63) / 64, DT = D / 16;
    typedef typename E::T T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane & 15, g = lane >> 4;
    const int kv_heads = a.cache.kv_heads, group = a.q_heads / kv_heads, head_tiles = (group + 15) / 16;
    int id = blockIdx.x;
    const int head_tile = id % head_tiles;
    id /= head_tiles;
    const int head = id % kv_heads;
    id /= kv_heads;
    const int b = id % a.batch, chunk = id / a.batch;
    const int heads = min(16, group - 16 * head_tile), q_head0 = head * group + 16 * head_tile;

    const int first = chunk * a.chunk;
    const int end = min(min(a.lengths[b], a.max_length), first + a.chunk);
    if (first >= end && chunk > 0) return;               // (an empty sequence's first workgroup writes its zeros)

    // the wavefront's blocks, 16 tiles ahead: lane l looks up block l % 4 of its tile l / 4
    constexpr int block_bytes = 32 * D + 128;
    const int blocks_per_page = a.cache.page_blocks;
    auto look_up = [&](int tile) {
        const int index = (first + 64 * (tile + NW * (lane >> 2))) / 16 + (lane & 3);
        const int page = index / blocks_per_page;
        int where = -1;
        if (page < a.cache.pages_stride) {               // (past the sequence's end: looked at, but masked)
            const int id = a.cache.pages[b * a.cache.pages_stride + page];
            if (id >= 0 && id < a.cache.num_pages) where = (id * kv_heads + head) * blocks_per_page + (index - page * blocks_per_page);
        }
        return where;
    };

    f4 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f4)(0.0f);
    float m = -3.0e38f, l = 0.0f;                        // the row's reference and this lane's part of the sum of its weights
    // The second product takes weight times V's scale times f, the row's factor: it follows the largest of these products, not V's scales
    // alone, so that a token of little weight does not push the others out of float16's range, however large its values.  Products so
    // small that they would lose bits all the same enter apart, so that many of them behind a large one are not lost: 11 bits of each down to 2^-38
    // of the largest.
    constexpr float kMostFactor = 0x1p120f;
    float f = kMostFactor;

    const int tiles = end > first ? (end - first + 63) / 64 : 0;
    int places = tiles > wave ? look_up(wave) : -1;
    // the rows of Q, on their way before the cache's
    u4 q[2 * NJ];
    {
        const int qh = q_head0 + min(h, heads - 1);      // (rows past the heads repeat the last one's and are not written)
        const T *row = (const T *)a.q.data + b * a.q.token_stride + qh * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < 2 * NJ; ++s) {
            const int d = 64 * (s / 2) + 16 * g + 8 * (s % 2);
            const T *from = row + (d < D ? d : 0);
            __builtin_memcpy(&q[s], from, 16);           // (one load, also where rows do not lie at 16-byte multiples)
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    // K of the next tile is on its way while this one's scores and values are worked on, V while the next one's scores are
    u4 k[4][NJ], v[DT];
    float ks = 0.0f, vs = 0.0f;
    int v_place = -1;
    const uint8_t *vb = a.cache.data;
    auto load_keys = [&](int n) {
        const int k_place = __shfl(places, 4 * n + (h >> 2));
        v_place = __shfl(places, 4 * n + g);
        const uint8_t *kb = a.cache.data + (int64_t)max(k_place, 0) * block_bytes + (h & 3) * D;
        vb = a.cache.data + (int64_t)max(v_place, 0) * block_bytes + 16 * D;
        ks = *(const float *)(vb + 16 * D + 4 * h);
        vs = *(const float *)(vb + 16 * D + 64 + 4 * h);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < NJ; ++j) k[t][j] = *(const u4 *)(kb + 4 * t * D + min(64 * j + 16 * g, D - 16));
    };
    auto load_values = [&]() {
#pragma unroll
        for (int t = 0; t < DT; ++t) v[t] = *(const u4 *)(vb + (16 * t + h) * 16);
    };
    load_keys(0);                                        // (without a tile, the first block's: so that Q alone is waited for next, whatever the wavefront has)
    __builtin_amdgcn_sched_barrier(0);

    // Q as f16, relative to a power of two for a bf16 row: its 8 bits are exact there
    float turned = 1.0f;                                 // the inverse of that power
    for (int tile = wave, n = 0; tile < tiles; tile += NW) {
        load_values();
        __builtin_amdgcn_sched_barrier(0);
        if (tile == wave) {                              // behind all requests of the first tile
            if constexpr (D % 64 != 0) {
#pragma unroll
                for (int s = 2 * NJ - 2; s < 2 * NJ; ++s) q[s] = 64 * (NJ - 1) + 16 * g < D ? q[s] : (u4)(0u);
            }
            if constexpr (!__is_same(T, _Float16)) {
                float most = 0.0f;
#pragma unroll
                for (int s = 0; s < 2 * NJ; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(fmaxf(most, fabsf(E::of_bits(q[s][e] & 0xffffu))), fabsf(E::of_bits(q[s][e] >> 16)));
                most = max_of_rows(most);
                int turn = 0;
                if (most > 0.0f && most < __builtin_inff()) turn = 15 - __builtin_amdgcn_frexp_expf(most);
                turned = __builtin_amdgcn_ldexpf(1.0f, -turn);
#pragma unroll
                for (int s = 0; s < 2 * NJ; ++s)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        q[s][e] = pack2<F16>(__builtin_amdgcn_ldexpf(E::of_bits(q[s][e] & 0xffffu), turn), __builtin_amdgcn_ldexpf(E::of_bits(q[s][e] >> 16), turn));
            }
        }
        // ---- scores ----
        const int there = v_place < 0 ? 0 : end - (first + 64 * tile + 16 * g);     // tokens of block g that count
        // (with the call's scale first, then the row's power: a score's factor is of a size between theirs, whatever those of queries and keys)
        float ks_now = h < there ? ks * a.scale : 0.0f, vs_now = h < there ? vs : 0.0f;
        // (here, so that the next tile's take the registers of this one's: moved at the loop's end, they would be waited for)
        asm volatile("" : "+v"(ks_now), "+v"(vs_now));
        f4 s[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            s[t] = (f4)(0.0f);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                u4 x[2];
                codes_to_f16(k[t][j], x);
                s[t] = mfma16(x[0], q[2 * j], s[t]);
                s[t] = mfma16(x[1], q[2 * j + 1], s[t]);
            }
        }
        const bool more = tile + NW < tiles;
        if (more) {
            if (++n == 16) {
                places = look_up(tile + NW);
                n = 0;
            }
            load_keys(n);
        }
        unrolled<16>([&](auto i) {
            constexpr int I = decltype(i)::value;
            s[I / 4][I % 4] = s[I / 4][I % 4] * (of_row<I>(ks_now) * turned);
        });
        const bool whole = __all(there >= 16);
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i >= there) s[i / 4][i % 4] = -__builtin_inff();
        }
        float most = fmaxf(fmaxf(s[0][0], s[0][1]), s[0][2]);
#pragma unroll
        for (int i = 3; i < 16; ++i) most = fmaxf(most, s[i / 4][i % 4]);
        if (__any(most > m)) {                           // weights are 1 at most, and 2^-8 or more for the largest
            most = max_of_rows(most);
            const float next = most > m ? most + 8.0f : m, fall = __builtin_amdgcn_exp2f(m - next), grown = f * __builtin_amdgcn_exp2f(next - m);
            l *= fall;
            m = next;
            // the values' sums stay: their weights' factor grows by as much as the weights fall, up to its limit
            if (tile > wave && __any(grown > kMostFactor)) {
                const float keep = grown > kMostFactor ? fall * (kMostFactor / f) : 1.0f;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= keep;
            }
            f = fminf(grown, kMostFactor);
        }
        float top = 0.0f, low = __builtin_inff();
        unrolled<16>([&](auto i) {
            constexpr int I = decltype(i)::value;
            const float x = __builtin_amdgcn_exp2f(s[I / 4][I % 4] - m);
            l += x;
            s[I / 4][I % 4] = x * of_row<I>(vs_now);
            top = fmaxf(top, s[I / 4][I % 4]);
            low = fminf(low, s[I / 4][I % 4]);
        });
        bool apart = false;
        if (__any(top * f > 0x1p15f || low * f < 0x1p-14f)) {
            if (__any(top * f > 0x1p15f)) {              // to 2^12 .. 2^13 (what has been summed then is scaled: not for every small rise)
                top = max_of_rows(top);
                const float next = top * f > 0x1p15f ? __builtin_amdgcn_ldexpf(1.0f, 13 - __builtin_amdgcn_frexp_expf(top)) : f, keep = next / f;
                if (tile > wave) {
#pragma unroll
                    for (int t = 0; t < DT; ++t) o[t] *= keep;
                }
                f = next;
            }
            if (!whole) {                                // without the tokens that do not count
                const float gap = h < there ? 0.0f : __builtin_inff();
                low = __builtin_inff();
                unrolled<16>([&](auto i) {
                    constexpr int I = decltype(i)::value;
                    low = fminf(low, s[I / 4][I % 4] + of_row<I>(gap));
                });
            }
            if (__any(low * f < 0x1p-14f)) {             // below float16's normal numbers: apart, times 2^12, and until then marked by the sign
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = s[i / 4][i % 4];
                    s[i / 4][i % 4] = x * f < 0x1p-14f ? x * -0x1p12f : x;
                }
                apart = true;
            }
        }
        u4 p[2];
#pragma unroll
        for (int i = 0; i < 16; i += 2) p[i / 8][i % 8 / 2] = pack2<F16>(s[i / 4][i % 4] * f, s[i / 4][i % 4 + 1] * f);
        if (__builtin_expect(apart, 0)) {
            u4 small[2];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t both = p[i / 4][i % 4];
                small[i / 4][i % 4] = positive_halves(both ^ 0x80008000u);
                p[i / 4][i % 4] = positive_halves(both);
            }
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                u4 x[2];
                uint32_t signs = kCodeSigns;
                asm volatile("" : "+s"(signs));          // (converted again below: all of them kept would be too many registers)
                codes_to_f16(v[t], x, signs);
                o[t] = mfma16(x[1], small[1], mfma16(x[0], small[0], o[t] * 0x1p12f)) * 0x1p-12f;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // ---- values ----
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            u4 x[2];
            codes_to_f16(v[t], x);
            o[t] = mfma16(x[0], p[0], o[t]);
            o[t] = mfma16(x[1], p[1], o[t]);
        }
    }

    // ---- the wavefronts' parts, joined in their order ----
    float *ms = shared, *ls = shared + 16 * NW, *os = shared + 32 * NW;      // [wave][16], [wave][16], [wave][heads][D]
    l = sum_of_rows(l);
    if (g == 0) ms[16 * wave + h] = m;
    __syncthreads();
    float top = m;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[16 * w + h]);
    const float fall = __builtin_amdgcn_exp2f(m - top);
    if (g == 0) ls[16 * wave + h] = l * fall;
    if (h < heads) {
        float *mine = os + (wave * heads + h) * D;
#pragma unroll
        for (int t = 0; t < DT; ++t)
            *(f4 *)(mine + 16 * t + 4 * g) = o[t] * (fall / f);
    }
    __syncthreads();
    // a thread's pieces of 4 elements
    const int row_pieces = D / 4;
    for (int i = threadIdx.x; i < heads * row_pieces; i += NW * 64) {
        const int hh = i / row_pieces, piece = i - hh * row_pieces, qh = q_head0 + hh;
        f4 sum = (f4)(0.0f);
        float weight = 0.0f, ref = -3.0e38f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            sum += *(const f4 *)(os + w * heads * D + 4 * i);
            weight += ls[16 * w + hh];
            ref = fmaxf(ref, ms[16 * w + hh]);
        }
        if (a.chunks > 1) {
            f4 *part = a.parts + (((int64_t)b * a.q_heads + qh) * a.chunks + chunk) * (row_pieces + 1);
            part[1 + piece] = sum;
            if (piece == 0) part[0] = (f4){ref, weight, 0.0f, 0.0f};
        } else {
            put_row<E>(a, b, qh, 4 * piece, sum, weight);
        }
    }
}

// The chunks of a sequence and query head, joined in an order that depends on nothing but their number.  A workgroup per sequence and
// head; groups of head_dim / 4 lanes take the chunks in turn, four at a time, and the groups' sums are added in their order.
// 3.6 to 6.3 us: a launch and two trips to memory.  (Joined by the last workgroup of a sequence to arrive instead, with a counter and device scope
// stores, a call on 4097 tokens took 20.7 us and not 11.3: every unit waits for its stores.)
constexpr int kJoinThreads = 512;

template <class E, int D>
__global__ __launch_bounds__(kJoinThreads) void attention_decode_join_kernel(const DecodeArgs a)
{
    constexpr int PIECES = D / 4, GROUPS = kJoinThreads / PIECES < 32 ? kJoinThreads / PIECES : 32;
    __shared__ f4 sums[GROUPS * PIECES];
    __shared__ float weights[GROUPS];
    const int tid = threadIdx.x, b = blockIdx.x / a.q_heads, qh = blockIdx.x % a.q_heads;
    const f4 *parts = a.parts + (int64_t)blockIdx.x * a.chunks * (PIECES + 1);
    const int length = min(a.lengths[b], a.max_length), chunks = length > 0 ? (length + a.chunk - 1) / a.chunk : 1;
    float top = -3.0e38f;
    for (int c = tid & 63; c < chunks; c += 64) top = fmaxf(top, parts[(int64_t)c * (PIECES + 1)][0]);
    top = max_of_rows(max_of_lanes<16>(top));
    const int g = tid / PIECES, piece = tid % PIECES;
    f4 sum = (f4)(0.0f);
    float weight = 0.0f;
    if (g < GROUPS) {
        for (int c = g; c < chunks; c += 4 * GROUPS) {
            f4 stats[4], x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f4 *part = parts + (int64_t)min(c + u * GROUPS, chunks - 1) * (PIECES + 1);
                stats[u] = part[0];
                x[u] = part[1 + piece];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (c + u * GROUPS >= chunks) break;
                const float fall = __builtin_amdgcn_exp2f(stats[u][0] - top);
                weight += stats[u][1] * fall;
                sum += x[u] * fall;
            }
        }
        sums[tid] = sum;
        if (piece == 0) weights[g] = weight;
    }
    __syncthreads();
    if (g > 0) return;
    for (int x = 1; x < min(GROUPS, chunks); ++x) {
        sum += sums[x * PIECES + piece];
        weight += weights[x];
    }
    put_row<E>(a, b, qh, 4 * piece, sum, weight);
}

}  // namespace ngemm
