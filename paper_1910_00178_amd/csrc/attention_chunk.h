// Attention of several new tokens per sequence over the 8-bit cache, with or without a window.
#pragma once
#include "attention_common.h"

namespace ngemm {

constexpr int kChunkKeys = 64;                                   // of a tile

struct ChunkArgs {
    CacheView cache;
    Rows q, o;
    const int32_t *offsets, *starts;
    int32_t batch, q_heads, tokens, max_new, max_length;
    int32_t window, sinks;   // window 0: none
    float scale;             // of the scores, times log2 e
    int32_t few_rows;        // sequences of up to so many rows (new tokens times heads that share a K/V head) are attention_chunk_few_kernel's
    int32_t run, parts;      // tiles of keys of a workgroup at most, workgroups along a sequence
    int32_t slots;           // tiles of rows (attention_chunk_kernel)
    f4 *part_data;           // parts > 1: sums, maxima and weights of the parts
    int32_t o_pieces;        // whether rows of O lie at 16-byte multiples
};

// The new tokens of a sequence, and where in the sequence they stand.
struct ChunkSequence {
    int first, queries;
    int64_t start;
    __device__ __forceinline__ ChunkSequence(const ChunkArgs &a, int begin, int end, int at) : start(at)
    {
        first = min(max(begin, 0), a.tokens);
        queries = min(min(max(end, first), a.tokens) - first, a.max_new);
    }
    __device__ __forceinline__ int position(int query) const { return (int)min(max(start + query, (int64_t)-1), (int64_t)0x7ffffffe); }
};

__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1; }

// x where bit i of `bits` is set, else what `other` is.  (A choice by a value, not by a condition: conditions on single elements of a vector are
// compiled to branches, which are slow, and of the first element's one was lost.)
__device__ __forceinline__ float where_bit(uint32_t bits, int i, float x, float other) { return bits >> i & 1 ? x : other; }

// What a row sees: keys lo .. hi and those before `sinks`.
struct ChunkRow {
    int lo = 0, hi = -1;
    __device__ __forceinline__ ChunkRow() {}
    __device__ __forceinline__ ChunkRow(const ChunkArgs &a, int position)
        : lo(a.window ? max(0, position - a.window + 1) : 0), hi(min(position, a.max_length - 1)) {}
    // of the tile that starts at key0, a bit per key
    __device__ __forceinline__ uint64_t seen(int key0, int sinks) const { return low_bits(hi - key0 + 1) & (~low_bits(lo - key0) | low_bits(sinks - key0)); }
    __device__ __forceinline__ bool sees_all(int key0, int sinks) const { return key0 + kChunkKeys - 1 <= hi && (key0 >= lo || key0 + kChunkKeys <= sinks); }
};

// The tiles of keys that rows from `first` to `last` see: those of the sinks, and those of the windows.
struct ChunkTiles {
    int sink_tiles, lo_tile, count;
    __device__ __forceinline__ ChunkTiles(const ChunkArgs &a, const ChunkRow &first, const ChunkRow &last) : sink_tiles(0), lo_tile(first.lo / kChunkKeys), count(0)
    {
        if (last.hi < 0) return;
        if (a.window) sink_tiles = min((min(a.sinks, last.hi + 1) + kChunkKeys - 1) / kChunkKeys, lo_tile);
        count = sink_tiles + max(0, last.hi / kChunkKeys - lo_tile + 1);
    }
    __device__ __forceinline__ int at(int i) const { return i < sink_tiles ? i : i - sink_tiles + lo_tile; }
};

// 16 codes as 16-bit floats, in order.
__device__ __forceinline__ void codes_to(F16, u4 x, u4 (&out)[2]) { codes_to_f16(x, out); }
__device__ __forceinline__ void codes_to(BF16, u4 x, u4 (&out)[2])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(x[e] >> (8 * i));
        out[e / 2][2 * (e % 2)] = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
        out[e / 2][2 * (e % 2) + 1] = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
    }
}

__device__ __forceinline__ f4 mfma16(F16, u4 a, u4 b, f4 c) { return mfma16(a, b, c); }
__device__ __forceinline__ f4 mfma16(BF16, u4 a, u4 b, f4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

// Two floats as bf16, and what that leaves of them, as bf16 again: 16 bits of each, over all of the floats' range.
__device__ __forceinline__ u2 split2(float x, float y)
{
    const uint32_t both = pack2<BF16>(x, y);
    return (u2){both, pack2<BF16>(x - __uint_as_float(both << 16), y - __uint_as_float(both & 0xffff0000u))};
}

// Elements d .. d + 3 of an output row (0 where nothing was seen).
template <class E>
__device__ __forceinline__ void put_chunk_row(const ChunkArgs &a, int token, int qh, int d, f4 sum, float weight)
{
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = weight == 0.0f ? 0.0f : sum[e] / weight;
    typename E::T *to = (typename E::T *)a.o.data + token * a.o.token_stride + qh * a.o.head_stride + d;
    if (a.o_pieces) store<E, 4, true>(to, x);
    else store<E, 4, false>(to, x);
}

constexpr int kFewWaves = 4;

// Sequences of few rows: those of up to R tiles of 16 (new tokens times the heads that share a K/V head, heads fastest).  A wavefront takes
// tiles of 64 keys = 4 blocks: S^T = K Q^T and O^T = V^T P^T on 16 x 16 x 32 matrix instructions.  Row r of the first product's tile t is
// token 4 t + r % 4 of block r / 4, so that lane 16 g + h holds row h's scores of block g's tokens, which is what the second product wants of it.
// The weights times V's scales enter the second product as two bf16 numbers each.
template <class E, int D, int R>
__global__ __launch_bounds__(kFewWaves * 64) void attention_chunk_few_kernel(const ChunkArgs a)
{
    extern __shared__ __align__(16) float shared[];
    constexpr int NW = kFewWaves, NJ = (D + 63) / 64, DT = D / 16, ROWS = 16 * R;
    typedef typename E::T T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane & 15, g = lane >> 4;
    const int kv_heads = a.cache.kv_heads, group = a.q_heads / kv_heads;
    int id = blockIdx.x;
    const int head = id % kv_heads;
    id /= kv_heads;
    const int b = id % a.batch, part = id / a.batch;

    const ChunkSequence seq(a, a.offsets[b], a.offsets[b + 1], a.starts ? a.starts[b] : 0);
    const int rows = seq.queries * group;
    if (rows == 0 || rows > min(a.few_rows, ROWS)) return;
    const ChunkTiles list(a, ChunkRow(a, seq.position(0)), ChunkRow(a, seq.position(seq.queries - 1)));
    // parts of whole turns of the wavefronts; an empty list's first workgroup writes its zeros
    const int parts = max(1, min(a.parts, (list.count + a.run - 1) / a.run));
    const int each = ((list.count + parts - 1) / parts + NW - 1) / NW * NW;
    const int first = part * each, end = min(list.count, first + each);
    if (part > 0 && first >= end) return;

    // the wavefront's blocks, 16 tiles ahead: lane l looks up block l % 4 of its tile l / 4
    constexpr int block_bytes = 32 * D + 128;
    const int blocks_per_page = a.cache.page_blocks;
    auto look_up = [&](int i) {
        const int index = 4 * list.at(min(i + NW * (lane >> 2), max(list.count - 1, 0))) + (lane & 3), page = index / blocks_per_page;
        int where = -1;
        if (page < a.cache.pages_stride) {
            const int id = a.cache.pages[b * a.cache.pages_stride + page];
            if (id >= 0 && id < a.cache.num_pages) where = (id * kv_heads + head) * blocks_per_page + (index - page * blocks_per_page);
        }
        return where;
    };
    int places = first + wave < end ? look_up(first + wave) : -1;

    u4 q[R][2 * NJ];
    ChunkRow range[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {                        // (rows past the last repeat it and are not written)
        const int row = min(16 * r + h, rows - 1), query = row / group;
        range[r] = ChunkRow(a, seq.position(query));
        const T *from = (const T *)a.q.data + (seq.first + query) * a.q.token_stride + (head * group + row % group) * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < 2 * NJ; ++s) {
            const int d = 64 * (s / 2) + 16 * g + 8 * (s % 2);
            __builtin_memcpy(&q[r][s], from + (d < D ? d : 0), 16);
            if (d >= D) q[r][s] = (u4)(0u);
        }
    }

    f4 o[R][DT];
    float m[R], l[R];                                    // the rows' references and this lane's part of the sums of their weights
#pragma unroll
    for (int r = 0; r < R; ++r) {
        m[r] = -3.0e38f;
        l[r] = 0.0f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[r][t] = (f4)(0.0f);
    }
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
    if (first + wave < end) load_keys(0);
    for (int i = first + wave, n = 0; i < end; i += NW) {
#pragma unroll
        for (int t = 0; t < DT; ++t) v[t] = *(const u4 *)(vb + (16 * t + h) * 16);
        __builtin_amdgcn_sched_barrier(0);
        const int key0 = kChunkKeys * list.at(i);
        const bool there = v_place >= 0;
        float ks_now = ks * a.scale, vs_now = vs;
        asm volatile("" : "+v"(ks_now), "+v"(vs_now));
        f4 s[R][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int r = 0; r < R; ++r) s[r][t] = (f4)(0.0f);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                u4 x[2];
                codes_to(E{}, k[t][j], x);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    s[r][t] = mfma16(E{}, x[0], q[r][2 * j], s[r][t]);
                    s[r][t] = mfma16(E{}, x[1], q[r][2 * j + 1], s[r][t]);
                }
            }
        }
        if (i + NW < end) {
            if (++n == 16) {
                places = look_up(i + NW);
                n = 0;
            }
            load_keys(n);
        }
        u4 p[R][2], rest[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            f4 (&x)[4] = s[r];
            unrolled<16>([&](auto at) {
                constexpr int I = decltype(at)::value;
                x[I / 4][I % 4] = x[I / 4][I % 4] * of_row<I>(ks_now);
            });
            // the row's bits of the lane's block, all set in most tiles
            const bool whole = __all(there && range[r].sees_all(key0, a.sinks));
            const uint32_t seen = there ? (uint32_t)(range[r].seen(key0, a.sinks) >> (16 * g)) : 0;
            if (!whole)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e / 4][e % 4] = where_bit(seen, e, x[e / 4][e % 4], -__builtin_inff());
            float most = x[0][0];
#pragma unroll
            for (int e = 1; e < 16; ++e) most = fmaxf(most, x[e / 4][e % 4]);
            if (__any(most > m[r])) {                    // weights are 1 at most, and 2^-8 or more for the largest
                most = max_of_rows(most);
                const float next = most > m[r] ? most + 8.0f : m[r], fall = __builtin_amdgcn_exp2f(m[r] - next);
                l[r] *= fall;
                m[r] = next;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[r][t] *= fall;
            }
            unrolled<16>([&](auto at) {
                constexpr int I = decltype(at)::value;
                const float w = __builtin_amdgcn_exp2f(x[I / 4][I % 4] - m[r]);
                l[r] += w;
                x[I / 4][I % 4] = w * of_row<I>(vs_now);
            });
            if (!whole)                                  // (a hidden token's scale may be NaN)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e / 4][e % 4] = where_bit(seen, e, x[e / 4][e % 4], 0.0f);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const u2 both = split2(x[e / 4][e % 4], x[e / 4][e % 4 + 1]);
                p[r][e / 8][e % 8 / 2] = both[0];
                rest[r][e / 8][e % 8 / 2] = both[1];
            }
        }
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            u4 x[2];
            codes_to(BF16{}, v[t], x);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                o[r][t] = mfma16(BF16{}, x[0], rest[r][0], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[1], rest[r][1], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[0], p[r][0], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[1], p[r][1], o[r][t]);
            }
        }
    }

    // ---- the wavefronts' parts, joined in their order ----
    float *ms = shared, *ls = shared + ROWS * NW, *os = shared + 2 * ROWS * NW;          // [wave][row], [wave][row], [wave][rows][D]
#pragma unroll
    for (int r = 0; r < R; ++r) {
        l[r] = sum_of_rows(l[r]);
        if (g == 0) ms[ROWS * wave + 16 * r + h] = m[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = 16 * r + h;
        float top = m[r];
#pragma unroll
        for (int w = 0; w < NW; ++w) top = fmaxf(top, ms[ROWS * w + row]);
        const float fall = __builtin_amdgcn_exp2f(m[r] - top);
        if (g == 0) ls[ROWS * wave + row] = l[r] * fall;
        if (row < rows) {
            float *mine = os + (wave * rows + row) * D;
#pragma unroll
            for (int t = 0; t < DT; ++t) *(f4 *)(mine + 16 * t + 4 * g) = o[r][t] * fall;
        }
    }
    __syncthreads();
    constexpr int PIECES = D / 4;
    for (int i = threadIdx.x; i < rows * PIECES; i += NW * 64) {
        const int row = i / PIECES, piece = i % PIECES;
        f4 sum = (f4)(0.0f);
        float weight = 0.0f, ref = -3.0e38f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            sum += *(const f4 *)(os + w * rows * D + 4 * i);
            weight += ls[ROWS * w + row];
            ref = fmaxf(ref, ms[ROWS * w + row]);
        }
        if (parts > 1) {
            f4 *to = a.part_data + ((((int64_t)b * kv_heads + head) * a.parts + part) * ROWS + row) * (PIECES + 1);
            to[1 + piece] = sum;
            if (piece == 0) to[0] = (f4){ref, weight, 0.0f, 0.0f};
        } else {
            put_chunk_row<E>(a, seq.first + row / group, head * group + row % group, 4 * piece, sum, weight);
        }
    }
}

// The parts of a row, joined in an order that depends on nothing but their number.  A workgroup per row; groups of D / 4 lanes take the parts
// in turn, and the groups' sums are added in their order.
constexpr int kFewJoinThreads = 256;

template <class E, int D, int R>
__global__ __launch_bounds__(kFewJoinThreads) void attention_chunk_few_join_kernel(const ChunkArgs a)
{
    constexpr int PIECES = D / 4, ROWS = 16 * R, GROUPS = kFewJoinThreads / PIECES;
    __shared__ f4 sums[GROUPS * PIECES];
    __shared__ float weights[GROUPS];
    const int kv_heads = a.cache.kv_heads, group = a.q_heads / kv_heads, tid = threadIdx.x;
    const int row = blockIdx.x % ROWS, unit = blockIdx.x / ROWS, head = unit % kv_heads, b = unit / kv_heads;
    const ChunkSequence seq(a, a.offsets[b], a.offsets[b + 1], a.starts ? a.starts[b] : 0);
    const int rows = seq.queries * group;
    if (row >= rows || rows > min(a.few_rows, ROWS)) return;
    const ChunkTiles list(a, ChunkRow(a, seq.position(0)), ChunkRow(a, seq.position(seq.queries - 1)));
    const int parts = max(1, min(a.parts, (list.count + a.run - 1) / a.run));
    if (parts == 1) return;
    const int each = ((list.count + parts - 1) / parts + kFewWaves - 1) / kFewWaves * kFewWaves, full = (list.count + each - 1) / each;
    const f4 *from = a.part_data + ((int64_t)unit * a.parts * ROWS + row) * (PIECES + 1);
    constexpr int STEP = ROWS * (PIECES + 1);
    float top = -3.0e38f;
    for (int c = tid & 63; c < full; c += 64) top = fmaxf(top, from[(int64_t)c * STEP][0]);
    top = max_of_rows(max_of_lanes<16>(top));
    const int g = tid / PIECES, piece = tid % PIECES;
    f4 sum = (f4)(0.0f);
    float weight = 0.0f;
    if (g < GROUPS) {
        for (int c = g; c < full; c += GROUPS) {
            const f4 *part = from + (int64_t)c * STEP;
            const f4 stats = part[0], x = part[1 + piece];
            const float fall = __builtin_amdgcn_exp2f(stats[0] - top);
            weight += stats[1] * fall;
            sum += x * fall;
        }
        sums[tid] = sum;
        if (piece == 0) weights[g] = weight;
    }
    __syncthreads();
    if (g > 0) return;
    for (int x = 1; x < min(GROUPS, full); ++x) {
        sum += sums[x * PIECES + piece];
        weight += weights[x];
    }
    put_chunk_row<E>(a, seq.first + row / group, head * group + row % group, 4 * piece, sum, weight);
}

// ---- many rows ----

// DP: head_dim rounded up.
template <int DP_, int PER_CU_>
struct ChunkCfg {
    static constexpr int DP = DP_, PER_CU = PER_CU_, NW = 4, BM = 32 * NW, BN = kChunkKeys;
    static constexpr int CH = DP / 8;                            // 16-byte pieces of a row of K
    static constexpr int kTile = BN * DP * 2, kScales = 2 * kTile, kStage = 2 * kTile + 2 * BN * 4, kLds = 2 * kStage;
    static constexpr int PIECES = 4 * DP / (NW * 64) + (4 * DP % (NW * 64) != 0);        // of 16 codes of K (and of V) per thread
    static constexpr int kPart = BM * 2 * (DP / 8 + 1);          // 16-byte pieces of a part: sums, maximum and weight
    static __device__ __forceinline__ int k_swizzle(int j) { return CH % 16 == 0 ? j & 15 : CH % 8 == 0 ? (j >> 1) & 7 : (j >> 2) & 3; }
    static __device__ __forceinline__ int v_swizzle(int d) { return (d >> 1) & 7; }
};

// A tile of a sequence's rows, heads fastest, and its share of the keys.
template <class C>
struct ChunkTile {
    ChunkSequence seq;
    int group, row0, rows;
    bool there;
    // Sequence b has the slots floor(rows before it / BM) + b .. : as many as its rows need or one more.
    __device__ __forceinline__ static ChunkTile find(const ChunkArgs &a, int slot)
    {
        const int group = a.q_heads / a.cache.kv_heads;
        int of[3];
        const int b = find_sequence(a.batch, slot, {a.offsets, a.offsets + 1, a.starts}, of, [&](int offset, int x) { return offset * group / C::BM + x; });
        ChunkTile t{ChunkSequence(a, of[0], of[1], of[2]), group, (slot - (of[0] * group / C::BM + b)) * C::BM, 0, false, b};
        t.rows = t.seq.queries * group;
        t.there = t.row0 >= 0 && t.row0 < t.rows && t.rows > a.few_rows;
        return t;
    }
    int b;
    __device__ __forceinline__ ChunkRow row(const ChunkArgs &a, int r) const { return ChunkRow(a, seq.position(min(r, rows - 1) / group)); }
    __device__ __forceinline__ ChunkTiles keys(const ChunkArgs &a) const { return ChunkTiles(a, row(a, row0), row(a, row0 + C::BM - 1)); }
};

template <class E, class C, bool VEC>
__global__ __launch_bounds__(C::NW * 64, C::PER_CU * C::NW / 4) void attention_chunk_kernel(const ChunkArgs a)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    constexpr int DP = C::DP, BN = C::BN, PIECES = C::PIECES;
    constexpr bool SPLIT = __is_same(typename E::T, _Float16);   // two bf16 numbers per weight
    typedef typename E::T T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
    const int kv_heads = a.cache.kv_heads, D = a.cache.head_dim;
    const int head = blockIdx.x % kv_heads, part = blockIdx.x / kv_heads % a.parts;
    const ChunkTile<C> tile = ChunkTile<C>::find(a, a.slots - 1 - blockIdx.x / kv_heads / a.parts);
    if (!tile.there) return;
    const int group = tile.group, rows = tile.rows;
    const ChunkTiles list = tile.keys(a);
    const int parts = max(1, min(a.parts, (list.count + a.run - 1) / a.run));
    if (part >= parts) return;
    const int first = (int)((int64_t)list.count * part / parts), end = (int)((int64_t)list.count * (part + 1) / parts);

    const int row = tile.row0 + 32 * wave + col;
    const bool row_there = row < rows;
    const int query = min(row, rows - 1) / group, qhead = head * group + min(row, rows - 1) % group;
    const ChunkRow range = tile.row(a, row), wave_first = tile.row(a, tile.row0 + 32 * wave), wave_last = tile.row(a, tile.row0 + 32 * wave + 31);
    const bool wave_there = tile.row0 + 32 * wave < rows;

    // ---- the blocks of 16 tiles: lane l looks up block l % 4 of tile l / 4 ----
    const int blocks_per_page = a.cache.page_blocks, block_bytes = 32 * D + 128;
    auto look_up = [&](int i) {
        const int index = 4 * list.at(min(i + (lane >> 2), max(list.count - 1, 0))) + (lane & 3), page = index / blocks_per_page;
        int where = -1;
        if (page < a.cache.pages_stride) {
            const int id = a.cache.pages[tile.b * a.cache.pages_stride + page];
            if (id >= 0 && id < a.cache.num_pages) where = (id * kv_heads + head) * blocks_per_page + (index - page * blocks_per_page);
        }
        return where;
    };
    // ---- a tile's codes, and where they go as 16-bit floats ----
    int piece_block[PIECES], piece_at[PIECES], k_to[PIECES][2], v_to[PIECES][2];
    bool piece_there[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = i * C::NW * 64 + tid, q = p % DP, per = D / 16, token = q / per, c = 2 * (q % per);
        piece_block[i] = p / DP;
        piece_there[i] = p < 4 * DP && q < D;
        piece_at[i] = 16 * q;
        const int j = 16 * piece_block[i] + token;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            k_to[i][e] = j * DP * 2 + ((c + e) ^ C::k_swizzle(j)) * 16;
            v_to[i][e] = C::kTile + q * BN * 2 + ((2 * piece_block[i] + e) ^ C::v_swizzle(q)) * 16;
        }
    }
    u4 k_codes[PIECES], v_codes[PIECES];
    float a_scale = 0.0f;                                        // threads 0 .. 63: K's of key tid, 64 .. 127: V's
    auto load_codes = [&](int places, int n) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (!piece_there[i]) continue;
            const uint8_t *block = a.cache.data + (int64_t)max(__shfl(places, 4 * n + piece_block[i]), 0) * block_bytes;
            k_codes[i] = *(const u4 *)(block + piece_at[i]);
            v_codes[i] = *(const u4 *)(block + 16 * D + piece_at[i]);
        }
        const uint8_t *block = a.cache.data + (int64_t)max(__shfl(places, 4 * n + (lane >> 4)), 0) * block_bytes + 32 * D;
        if (wave < 2) a_scale = *(const float *)(block + 64 * wave + 4 * (lane & 15));
    };
    auto store_codes = [&](uint8_t *at) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            if (!piece_there[i]) continue;
            u4 x[2];
            codes_to(E{}, k_codes[i], x);
            *(u4 *)(at + k_to[i][0]) = x[0];
            *(u4 *)(at + k_to[i][1]) = x[1];
            codes_to(BF16{}, v_codes[i], x);
            *(u4 *)(at + v_to[i][0]) = x[0];
            *(u4 *)(at + v_to[i][1]) = x[1];
        }
        if (wave < 2) ((float *)(at + C::kScales))[tid] = wave == 0 ? a_scale * a.scale : a_scale;
    };
    if (D < DP) {                                                // elements past head_dim are 0 throughout
        for (int i = tid; i < C::kLds / 16; i += C::NW * 64) ((u4 *)lds)[i] = (u4)(0u);
        __syncthreads();
    }
    int places = first < end ? look_up(first) : -1;
    if (first < end) load_codes(places, 0);

    // ---- Q^T's operand: 8 elements of the lane's row per step ----
    u4 q[DP / 16];
    {
        const T *from = (const T *)a.q.data + (tile.seq.first + query) * a.q.token_stride + qhead * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            const int d = 16 * s + 8 * half;
            const T *at = from + (d < D ? d : 0);
            if constexpr (VEC) q[s] = *(const u4 *)at;
            else __builtin_memcpy(&q[s], at, 16);
            if (d >= D) q[s] = (u4)(0u);
        }
    }
    // the key whose scores are row `col` of the first product: so that a lane holds 8 consecutive keys' of each 16
    const int key = 16 * (col >> 4) + 8 * (col >> 2 & 1) + 4 * (col >> 3 & 1) + (col & 3);
    const int k_row = key * DP * 2, k_chunk = (half ^ C::k_swizzle(key)) * 16;
    const int v_row = C::kTile + col * BN * 2, v_chunk = (half ^ C::v_swizzle(col)) * 16;

    f16v o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = (f16v)(0.0f);
    float m = -3.0e38f, l = 0.0f;
    for (int i = first; i < end; ++i) {
        uint8_t *const at = lds + (i - first & 1) * C::kStage;
        const int n = i - first & 15;
        const uint32_t lost = (uint32_t)(__ballot(places < 0) >> (4 * n)) & 15u;         // blocks that are not there
        store_codes(at);
        if (i + 1 < end) {
            if (n == 15) places = look_up(i + 1);
            load_codes(places, n + 1 & 15);
        }
        __syncthreads();
        const int key0 = BN * list.at(i);
        if (!wave_there || key0 > wave_last.hi || (key0 + BN - 1 < wave_first.lo && key0 >= a.sinks)) continue;
        f16v s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            s[t] = (f16v)(0.0f);
#pragma unroll
            for (int u = 0; u < DP / 16; ++u) s[t] = mfma32(E{}, *(const u4 *)(at + k_row + (k_chunk ^ 32 * u) + t * 32 * DP * 2), q[u], s[t]);
        }
        const bool masked = lost || !wave_first.sees_all(key0, a.sinks) || !wave_last.sees_all(key0, a.sinks);
        // bit 32 t + 16 (e / 8) + e % 8: whether the row sees s[t][e]'s key
        uint64_t seen = ~(uint64_t)0;
        if (masked) {
            seen = range.seen(key0, a.sinks);
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (lost >> g & 1) seen &= ~((uint64_t)0xffff << (16 * g));
            seen >>= 8 * half;
        }
        const float *const scales = (const float *)(at + C::kScales) + 8 * half;
        float most = m;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f4 by = *(const f4 *)(scales + 32 * t + 16 * (e / 8) + e % 8);
#pragma unroll
                for (int x = 0; x < 4; ++x) s[t][e + x] *= by[x];
            }
        if (masked)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[t][e] = where_bit((uint32_t)(seen >> (32 * t)), 16 * (e / 8) + e % 8, s[t][e], -__builtin_inff());
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) most = fmaxf(most, s[t][e]);
        most = max_of_halves(most);
        if (__any(most > m)) {                           // weights are 1 at most, and 2^-8 or more for the largest
            const float next = most > m ? most + 8.0f : m, fall = __builtin_amdgcn_exp2f(m - next);
            l *= fall;
            m = next;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) o[t] *= fall;
        }
        u4 p[4], rest[4];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const f4 by = *(const f4 *)(scales + BN + 32 * t + 16 * (e / 8) + e % 8);
                float w[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    w[x] = __builtin_amdgcn_exp2f(s[t][e + x] - m);
                    l += w[x];
                    w[x] *= by[x];
                }
                if (masked)                              // (a hidden key's scale may be NaN)
#pragma unroll
                    for (int x = 0; x < 4; ++x) w[x] = where_bit((uint32_t)(seen >> (32 * t)), 16 * (e / 8) + e % 8 + x, w[x], 0.0f);
#pragma unroll
                for (int x = 0; x < 4; x += 2) {
                    const int u = 2 * t + e / 8, to = (e % 8 + x) / 2;
                    if constexpr (SPLIT) {
                        const u2 both = split2(w[x], w[x + 1]);
                        p[u][to] = both[0];
                        rest[u][to] = both[1];
                    } else {
                        p[u][to] = pack2<BF16>(w[x], w[x + 1]);
                    }
                }
            }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) {
                const u4 x = *(const u4 *)(at + v_row + (v_chunk ^ 32 * u) + t * 32 * BN * 2);
                if constexpr (SPLIT) o[t] = mfma32(BF16{}, x, rest[u], o[t]);
                o[t] = mfma32(BF16{}, x, p[u], o[t]);
            }
    }
    l = sum_of_halves(l);
    if (parts > 1) {
        f4 *mine = a.part_data + (int64_t)blockIdx.x * C::kPart + tid;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(4 * t + i) * C::BM * 2] = (f4){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
        mine[DP / 8 * C::BM * 2] = (f4){m, l, 0.0f, 0.0f};
        return;
    }
    // ---- O = O^T / l: 4 consecutive elements per lane and quarter, exchanged between lane halves to 8 ----
    T *out = (T *)a.o.data + (tile.seq.first + query) * a.o.token_stride + qhead * a.o.head_stride;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = l == 0.0f ? 0.0f : o[t][i + e] / l;
            const u2 s0 = __builtin_amdgcn_permlane32_swap(pack2<E>(x[0], x[1]), pack2<E>(x[4], x[5]), false, false);
            const u2 s1 = __builtin_amdgcn_permlane32_swap(pack2<E>(x[2], x[3]), pack2<E>(x[6], x[7]), false, false);
            const u4 y = {s0[0], s1[0], s0[1], s1[1]};
            const int d = 32 * t + 2 * i + 8 * half;
            if (row_there && d < D) {
                if constexpr (VEC) {
                    *(u4 *)(out + d) = y;
                } else {
                    T e8[8];
                    __builtin_memcpy(e8, &y, 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) out[d + e] = e8[e];
                }
            }
        }
}

// The parts of a tile, joined in their order: a workgroup per tile and piece of 4 elements of a lane.
template <class E, class C, bool VEC>
__global__ __launch_bounds__(C::BM * 2) void attention_chunk_join_kernel(const ChunkArgs a)
{
    constexpr int THREADS = C::BM * 2, PIECES = C::DP / 8;
    const int piece = blockIdx.x % PIECES, kv_heads = a.cache.kv_heads, head = blockIdx.x / PIECES % kv_heads, number = blockIdx.x / PIECES / kv_heads;
    const ChunkTile<C> tile = ChunkTile<C>::find(a, a.slots - 1 - number);
    const int tid = threadIdx.x, lane = tid & 63, row = tile.row0 + 32 * (tid >> 6) + (lane & 31);
    const int d = 8 * piece + 4 * (lane >> 5);                   // 32 (piece / 4) + 8 (piece % 4) + ..
    if (!tile.there || row >= tile.rows || d >= a.cache.head_dim) return;
    const int parts = max(1, min(a.parts, (tile.keys(a).count + a.run - 1) / a.run));
    if (parts == 1) return;
    const f4 *from = a.part_data + ((int64_t)number * a.parts * kv_heads + head) * C::kPart + tid;
    float top = -3.0e38f, l = 0.0f;
    f4 o = (f4)(0.0f);
    for (int p0 = 0; p0 < parts; p0 += 4) {                      // four on their way together
        f4 stats[4], x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f4 *part = from + (int64_t)min(p0 + i, parts - 1) * kv_heads * C::kPart;
            stats[i] = part[PIECES * THREADS];
            x[i] = part[piece * THREADS];
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < 4; ++i) now = fmaxf(now, stats[i][0]);
        const float fall = __builtin_amdgcn_exp2f(top - now);
        l *= fall;
        o *= fall;
        top = now;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p0 + i >= parts) break;
            const float by = __builtin_amdgcn_exp2f(stats[i][0] - top);
            l += stats[i][1] * by;
            o += x[i] * by;
        }
    }
    put_chunk_row<E>(a, tile.seq.first + row / tile.group, head * tile.group + row % tile.group, d, o, l);
}

}  // namespace ngemm
