// Norms of rows per head and their rotation by positions: rows to rows, and keys on their way into the 8-bit cache.
#pragma once
#include "kv_cache.h"

namespace ngemm {

// table [positions][dim]: the cosines and behind them the sines of a row's dim / 2 pairs; dim 0: no rotation.
struct RotationView {
    const float *table;
    int32_t positions, dim;
};

constexpr int kNoPairs = 0, kHalves = 1, kNeighbours = 2;

// A row of D elements is held by D / 16 of LANES lanes, two pieces of eight elements each.  Where its halves are paired, the lanes of the rotated
// part hold pieces l and l + dim / 16, whose elements are pairs, and the others pieces 2 l and 2 l + 1; else l and l + D / 16.
template <class E, int LANES, int PAIRS>
struct TurnedRow {
    int lane, at[2];         // elements where the pieces start
    bool there, turned[2];   // (halves: both the same)
    bool known_position = true;
    float cosines[8], sines[8];

    __device__ __forceinline__ TurnedRow(const RotationView &r, int D, int lane) : lane(lane), there(lane < D / 16)
    {
        const int apart = PAIRS == kHalves ? r.dim / 16 : D / 16;
        at[0] = 8 * (lane < apart ? lane : 2 * lane);
        at[1] = 8 * (lane < apart ? lane + apart : 2 * lane + 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) turned[i] = PAIRS != kNoPairs && there && at[i] < r.dim;
    }
    // What the table has for a position; one that it does not have makes rows NaN.
    __device__ __forceinline__ void find(const RotationView &r, int64_t position)
    {
        if constexpr (PAIRS == kNoPairs) return;
        const bool known = position >= 0 && position < r.positions;
        const float *const row = r.table + (known ? position : 0) * r.dim;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (!turned[i]) continue;
            const float *const from = row + (PAIRS == kHalves ? at[0] + 4 * i : at[i] / 2);
            const f4 c = *(const f4 *)from, s = *(const f4 *)(from + r.dim / 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                cosines[4 * i + e] = known ? c[e] : __builtin_nanf("");
                sines[4 * i + e] = s[e];
            }
        }
        known_position = known;
    }

    template <bool VEC>
    __device__ __forceinline__ void load(Piece<E> (&x)[2], const typename E::T *row) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (there) x[i] = load_piece<E, VEC>(row + at[i]);
            else x[i] = Piece<E>{};
    }
    // Sixteen elements of a vector of floats that starts anywhere.
    __device__ __forceinline__ void weights(float (&w)[16], const float *from) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = from && there ? from[at[i / 8] + i % 8] : 1.0f;
    }
    // y = x / sqrt(mean x^2 + eps) w, then the pairs turned, in floats.  Rows whose squares leave the floats' range, and those of very small
    // numbers, are taken relative to a power of two.  A row of zeros stays so.
    __device__ __forceinline__ void turn(float (&y)[16], const Piece<E> (&x)[2], bool norm, const float (&w)[16], float eps, int D) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) y[i] = E::get(x[i / 8].x[i % 8]);
        if (norm) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = __builtin_fmaf(y[i], y[i], sum);
            sum = sum_of_lanes<LANES>(sum);
            const float of_one = 1.0f / (float)D;
            float by = __builtin_amdgcn_rsqf(__builtin_fmaf(sum, of_one, eps));
            if (!(sum < 0x1p120f && sum > 0x1p-100f)) {          // (the lanes of a row agree)
                const uint32_t bits = max_of_lanes<LANES>(max(most_bits(x[0]), most_bits(x[1])));
                if (bits == 0) {
                    by = 0.0f;
                } else if (bits < E::kInfinityBits) {
                    const int ex = __builtin_amdgcn_frexp_expf(E::of_bits(bits));
                    sum = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float z = __builtin_amdgcn_ldexpf(y[i], -ex);
                        sum = __builtin_fmaf(z, z, sum);
                    }
                    sum = sum_of_lanes<LANES>(sum) * of_one;
                    // eps relative to 2^(2 ex): out of range, it counts alone
                    const float small = __builtin_amdgcn_ldexpf(__builtin_amdgcn_ldexpf(eps, -ex), -ex);
                    if (small < 0x1p120f) {
                        by = __builtin_amdgcn_rsqf(sum + small);
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = __builtin_amdgcn_ldexpf(y[i], -ex);
                    } else {
                        by = 1.0f / sqrtf(eps);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = y[i] * by * w[i];
        }
        if constexpr (PAIRS == kHalves) {
            if (turned[0])
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = y[e], b = y[8 + e];
                    y[e] = __builtin_fmaf(a, cosines[e], -(b * sines[e]));
                    y[8 + e] = __builtin_fmaf(b, cosines[e], a * sines[e]);
                }
        } else if constexpr (PAIRS == kNeighbours) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (turned[i])
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = y[8 * i + 2 * e], b = y[8 * i + 2 * e + 1];
                        y[8 * i + 2 * e] = __builtin_fmaf(a, cosines[4 * i + e], -(b * sines[4 * i + e]));
                        y[8 * i + 2 * e + 1] = __builtin_fmaf(b, cosines[4 * i + e], a * sines[4 * i + e]);
                    }
        }
        if (!known_position)
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = __builtin_nanf("");
    }
};

// One kind of rows of a call: where they come from and go to.
struct TurnedRows {
    Rows from, to;
    const float *weight;     // null: no norm
    int32_t heads;
};

struct TurnArgs {
    TurnedRows kind[2];      // Q and K
    RotationView rotation;
    const int32_t *positions;
    float eps;
    int32_t head_dim, items, chunks, chunks_q;   // items: tokens times chunks of U heads; a token's, and those of Q among them
};

// LANES lanes take U heads of a token, one item: its angles and weights are read once, and the rows are on their way together.  All of an
// item's rows are read before any is written, so outputs may stand in their inputs' places.  The sums of squares are floats, and the result is rounded to the type once.
// Bound by memory, a read and a write of every row: 9900 tokens of 32 + 8 heads of 128, bf16, 46 us = 4.4 TB/s, f32 84 us = 4.9 (a large copy: 4.9).
template <class E, int LANES, int PAIRS, int U, bool VEC>
__global__ __launch_bounds__(256) void qk_norm_rotate_kernel(const TurnArgs a)
{
    typedef typename E::T T;
    const int item = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const bool real = item < a.items;                    // (all lanes stay for the sums over lanes)
    const int token = real ? item / a.chunks : 0, chunk = real ? item - token * a.chunks : 0;
    const bool is_k = chunk >= a.chunks_q;
    const TurnedRows &k = a.kind[is_k];
    const int head0 = (is_k ? chunk - a.chunks_q : chunk) * U;
    TurnedRow<E, LANES, PAIRS> row(a.rotation, a.head_dim, threadIdx.x % LANES);
    row.there = row.there && real;
#pragma unroll
    for (int i = 0; i < 2; ++i) row.turned[i] = row.turned[i] && real;
    int position = 0;
    if constexpr (PAIRS != kNoPairs) position = a.positions[token];
    Piece<E> x[U][2];
    const T *from = (const T *)k.from.data + token * k.from.token_stride + head0 * k.from.head_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) row.template load<VEC>(x[u], from + (head0 + u < k.heads ? u : 0) * k.from.head_stride);
    float w[16];
    row.weights(w, k.weight);
    row.find(a.rotation, position);
    T *to = (T *)k.to.data + token * k.to.token_stride + head0 * k.to.head_stride;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float y[16];
        row.turn(y, x[u], k.weight != nullptr, w, a.eps, a.head_dim);
        if (row.there && head0 + u < k.heads)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float z[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = y[8 * i + e];
                store<E, 8, VEC>(to + u * k.to.head_stride + row.at[i], z);
            }
    }
}

struct TurnedMoveArgs {
    MoveArgs move;
    RotationView rotation;
    const float *weight;
    float eps;
};

// kv_write_kernel with K's rows normalised and turned in floats before their maximum is found: LANES lanes a token, two pieces each.  Codes are of the 32-bit
// results: a rounding to the type in between would be of 2^-8 in bf16, as much again as the codes' own, a 254th of the largest.
// Bound by memory where tokens are many: 17 200 tokens of 8 heads of 128, bf16, 31 us (3.4 TB/s), f32 34 (5.3 TB/s); vector instructions are next (some 21 an element of K
// and V, bf16).
template <class E, int LANES, int PAIRS, bool VEC>
__global__ __launch_bounds__(16 * LANES) void kv_write_rotated_kernel(const TurnedMoveArgs args)
{
    __shared__ __align__(16) uint32_t turned[2][16][4 * LANES + 1];
    typedef typename E::T T;
    const MoveArgs &a = args.move;
    const int groups = (a.cache.kv_heads + a.heads - 1) / a.heads, head0 = blockIdx.x % groups * a.heads;
    const int D = a.cache.head_dim, tid = threadIdx.x;
    const MoveBlock m(a, blockIdx.x / groups);
    if (m.begin >= m.end) return;
    const int token = tid / LANES;
    const bool there = token >= m.begin && token < m.end;
    const int64_t head_bytes = (int64_t)a.cache.page_blocks * a.cache.block_bytes();
    TurnedRow<E, LANES, PAIRS> row(args.rotation, D, tid % LANES);
    row.there = row.there && there;
    Piece<E> k[2], v[2];
    auto load = [&](int head) {
        row.template load<VEC>(k, (const T *)a.k.data + (m.row0 + token) * a.k.token_stride + head * a.k.head_stride);
        row.template load<VEC>(v, (const T *)a.v.data + (m.row0 + token) * a.v.token_stride + head * a.v.head_stride);
    };
    load(head0);                                         // on their way while the place is looked up
    row.find(args.rotation, m.index * kBlockTokens + (there ? token : m.begin));
    float w[16];
    row.weights(w, args.weight);
    uint8_t *block = m.block(a);
    if (!block) return;
    block += head0 * head_bytes;
    const int end = min(head0 + a.heads, a.cache.kv_heads);
    for (int head = head0, turn = 0; head < end; ++head, turn ^= 1, block += head_bytes) {
        float y[16];
        row.turn(y, k, args.weight != nullptr, w, args.eps, D);
        Piece<F32> z[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i / 8].x[i % 8] = y[i];
        const uint32_t k_bits = max_of_lanes<LANES>(max(most_bits(z[0]), most_bits(z[1])));
        const uint32_t v_bits = max_of_lanes<LANES>(max(most_bits(v[0]), most_bits(v[1])));
        const float k_most = __uint_as_float(k_bits), v_most = E::of_bits(v_bits);
        const bool k_finite = k_bits < F32::kInfinityBits, v_finite = v_bits < E::kInfinityBits;
        if (row.there) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *(u2 *)(block + token * D + row.at[i]) = quantise<F32>(z[i], k_most, k_finite);
                const u2 codes = quantise<E>(v[i], v_most, v_finite);
                turned[turn][token][row.at[i] / 4] = codes[0];
                turned[turn][token][row.at[i] / 4 + 1] = codes[1];
            }
            if (row.lane == 0) {
                ((float *)(block + 32 * D))[token] = k_finite ? k_most / 127.0f : __builtin_nanf("");
                ((float *)(block + 32 * D))[16 + token] = v_finite ? v_most / 127.0f : __builtin_nanf("");
            }
        }
        if (head + 1 < end) load(head + 1);              // on their way while this head's codes are turned and stored
        __syncthreads();                                 // (the next head writes the other half)
        store_turned<16 * LANES>(block, turned[turn], m, D);
    }
}

}  // namespace ngemm
