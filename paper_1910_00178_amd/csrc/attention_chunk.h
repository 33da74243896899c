// Attention of several new tokens per sequence over the 8-bit cache, with or without a window.
#pragma once
#include "attention_common.h"

namespace ngemm {

constexpr int kChunkKeys = 64;                                   // of a tile
constexpr int kLeastTiles = 4;                                   // of keys, of a workgroup where a tile's are shared out
constexpr int kMostShared = 128;                                 // sequences of a call that are

struct ChunkArgs {
    CacheView cache;
    Rows q, o;
    const int32_t *offsets, *starts;
    int32_t batch, q_heads, tokens, max_new, max_length;
    int32_t window, sinks;   // window 0: none
    float scale;             // of the scores, times log2 e
    int32_t few_rows;        // sequences of up to so many rows (new tokens times heads that share a K/V head) are attention_chunk_few_kernel's
    int32_t slots;           // workgroups of a K/V head
    float share;             // of the device's places, where the keys are shared out: a K/V head's; else 0
    f4 *part_data;           // keys shared out: [slots][kv_heads] parts: sums, maxima and weights
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

// The number of the block that holds positions 16 * index .. of sequence b and a head, or -1 where there is none.  Without branches (a table without
// entries has been taken as one without tokens), so that loops around it have uniform ones only: sums in registers stay where they are.  (Blocks have 640 bytes or more:
// the number of one in a device's memory fits 32 bits.)
__device__ __forceinline__ int chunk_place(const ChunkArgs &a, int b, int head, int index)
{
    const int page = index / a.cache.page_blocks;
    const bool there = page < a.cache.pages_stride;
    const int id = a.cache.pages[b * a.cache.pages_stride + (there ? page : 0)];
    return there && id >= 0 && id < a.cache.num_pages ? (id * a.cache.kv_heads + head) * a.cache.page_blocks + (index - page * a.cache.page_blocks) : -1;
}

// A tile of BM of a sequence's rows (new tokens times the heads that share a K/V head, heads fastest) and a workgroup's share of its keys.  FEW: of the sequences of
// up to few_rows rows; else of the others.
template <bool FEW, int BM>
struct ChunkUnit {
    int b, first_row, queries, rows, row0, group;                // first_row: of the packed rows of tokens
    int64_t start;
    int part, parts, part0;                                      // `parts` workgroups share out the keys; of them this one, and the first one's number
    bool there;

    __device__ __forceinline__ void take(const ChunkArgs &a, int begin, int end, int at)
    {
        const ChunkSequence seq(a, begin, end, at);
        first_row = seq.first, queries = seq.queries, start = seq.start, rows = queries * group;
    }
    // (of rows that are the same in all lanes: `start` takes 64 bits, which the compiler compares in the vector unit and leaves there)
    __device__ __forceinline__ ChunkRow row_of_all(const ChunkArgs &a, int r) const
    {
        ChunkRow x = row(a, r);
        x.lo = __builtin_amdgcn_readfirstlane(x.lo), x.hi = __builtin_amdgcn_readfirstlane(x.hi);
        return x;
    }
    __device__ __forceinline__ ChunkRow row(const ChunkArgs &a, int r) const
    {
        return ChunkRow(a, (int)min(max(start + min(r, rows - 1) / group, (int64_t)-1), (int64_t)0x7ffffffe));
    }
    __device__ __forceinline__ ChunkTiles keys(const ChunkArgs &a) const { return ChunkTiles(a, row(a, row0), row(a, row0 + BM - 1)); }
    __device__ __forceinline__ bool mine(const ChunkArgs &a) const { return FEW ? rows > 0 && rows <= a.few_rows : rows > a.few_rows; }

    // Workgroup `number` of a head (JOIN: tile `number`).
    template <int JOIN>
    __device__ __forceinline__ ChunkUnit(const ChunkArgs &a, int number, Index<JOIN>) : row0(0), group(a.q_heads / a.cache.kv_heads), part(0), parts(1), part0(0)
    {
        if (FEW ? a.share == 0.0f : a.batch > kMostShared) {     // a workgroup takes all keys of its tile
            int of[3];
            if constexpr (FEW) {
                const int each = (a.few_rows + BM - 1) / BM;
                b = number / each;
                row0 = number % each * BM;
                of[0] = a.offsets[b], of[1] = a.offsets[b + 1], of[2] = a.starts ? a.starts[b] : 0;
            } else {                                             // sequence b has the slots floor(rows before it / BM) + b .. : as many as its rows need or one more
                const int group = this->group;
                b = find_sequence(a.batch, number, {a.offsets, a.offsets + 1, a.starts}, of, [group](int offset, int x) { return offset * group / BM + x; });
                row0 = (number - (of[0] * group / BM + b)) * BM;
            }
            take(a, of[0], of[1], of[2]);
            there = mine(a) && row0 >= 0 && row0 < rows;
            same_in_all_lanes();
            return;
        }
        // Up to kMostShared sequences, a lane each: tiles are numbered without gaps.  (Workgroups without a tile between others leave the units unevenly loaded:
        // 16 x 128 tokens behind 1000, a tile per unit, 88 us with them, 52 without.)  All places of the device would have the same if each tile saw what its sequence's
        // first and last ones do on average; all of a sequence's are cut into as many parts as its last one's keys take places (at most twice the places in all;
        // share 0: into one).
        constexpr int TURNS = kMostShared / 64;
        const int lane = threadIdx.x & 63;
        int of[TURNS][3] = {}, tiles[TURNS] = {}, most[TURNS] = {};
        float work = 0.0f;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            if (64 * i >= a.batch) break;
            const int at = min(64 * i + lane, a.batch - 1);
            of[i][0] = a.offsets[at], of[i][1] = a.offsets[at + 1], of[i][2] = a.starts ? a.starts[at] : 0;
            take(a, of[i][0], of[i][1], of[i][2]);
            tiles[i] = 64 * i + lane < a.batch && mine(a) ? (rows + BM - 1) / BM : 0;
            if (a.share == 0.0f) continue;
            row0 = 0;
            const int least = tiles[i] > 0 ? keys(a).count : 0;
            row0 = max(tiles[i] - 1, 0) * BM;
            most[i] = tiles[i] > 0 ? keys(a).count : 0;
            work += (float)tiles[i] * (0.5f * (float)(most[i] + max(least, 0)));
        }
        if (a.share > 0.0f) work = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sums_up_to(work)), 63));
        const float share = a.share / fmaxf(work, 1.0f);
        int tile = 0, each = 1, tiles_before = 0, parts_before = 0;
        there = false;
        b = 0;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            if (64 * i >= a.batch) break;
            // (a whole number of parts may come out as a little less)
            const int cut = max(1, min((int)((float)most[i] * share + 0x1p-8f), most[i] / kLeastTiles)), all = tiles[i] * cut;
            const int tiles_to = tiles_before + sums_up_to(tiles[i]), parts_to = a.share > 0.0f ? parts_before + sums_up_to(all) : tiles_to;
            const int begin = JOIN ? tiles_to - tiles[i] : parts_to - all, end = JOIN ? tiles_to : parts_to;
            const uint64_t here = __ballot(begin <= number && number < end);
            if (here) {
                const int l = __builtin_ctzll(here);
                take(a, __builtin_amdgcn_readlane(of[i][0], l), __builtin_amdgcn_readlane(of[i][1], l), __builtin_amdgcn_readlane(of[i][2], l));
                b = 64 * i + l;
                each = __builtin_amdgcn_readlane(cut, l);
                const int at = number - __builtin_amdgcn_readlane(begin, l);
                tile = JOIN ? at : at / each;
                part = JOIN ? 0 : at % each;
                part0 = __builtin_amdgcn_readlane(parts_to - all, l) + tile * each;
                // The longest first; of whole tiles every other four turned round: workgroups go to a chiplet's four engines in turn, and one of these would always
                // get the longest of four (64 x 512 tokens: 320 us so, 307 turned).
                const int count = __builtin_amdgcn_readlane(tiles[i], l), four = tile & ~3;
                if (each == 1 && (__builtin_amdgcn_readlane(tiles_to - tiles[i], l) + four) & 4) tile = four + min(4, count - four) - 1 - (tile & 3);
                tile = count - 1 - tile;
                there = true;
            }
            tiles_before = __builtin_amdgcn_readlane(tiles_to, 63);
            parts_before = __builtin_amdgcn_readlane(parts_to, 63);
        }
        if (!there) return;
        row0 = tile * BM;
        if (each > 1) parts = max(1, min(each, keys(a).count / kLeastTiles));
        there = part < parts && part0 >= 0 && part0 + parts <= a.slots;          // (places past the end: offsets that fall)
        same_in_all_lanes();
    }
    // (as it is, which the compiler does not see)
    __device__ __forceinline__ void same_in_all_lanes()
    {
        for (int *const x : {&b, &first_row, &queries, &rows, &row0, &part, &parts, &part0}) *x = __builtin_amdgcn_readfirstlane(*x);
        start = (int64_t)__builtin_amdgcn_readfirstlane((int)start);
        there = __builtin_amdgcn_readfirstlane(there);
    }
};

// Four codes as 16-bit floats, in order.
__device__ __forceinline__ u2 codes4_to(F16, uint32_t x) { return codes4_to_f16(x); }
__device__ __forceinline__ u2 codes4_to(BF16, uint32_t x)
{
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(x >> (8 * i));            // (whole numbers of 8 bits: the upper half is all of it)
    return (u2){__builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u),
                __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u)};
}
template <class E>
__device__ __forceinline__ void codes_to(E, u4 x, u4 (&out)[2])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const u2 y = codes4_to(E{}, x[e]);
        out[e / 2][2 * (e % 2)] = y[0];
        out[e / 2][2 * (e % 2) + 1] = y[1];
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

constexpr int few_waves_per_simd(int D, int R, int NW) { return D * R <= 128 || NW == 8 ? 2 : 1; }

// Sequences of few rows: tiles of R times 16 of them (new tokens times the heads that share a K/V head, heads fastest).  A wavefront takes
// tiles of 64 keys = 4 blocks: S^T = K Q^T and O^T = V^T P^T on 16 x 16 x 32 matrix instructions.  Row r of the first product's tile t is
// token 4 t + r % 4 of block r / 4, so that lane 16 g + h holds row h's scores of block g's tokens, which is what the second product wants of it:
// codes go from memory to registers, become floats there and meet the matrix unit, without LDS.
// A softmax in one pass: weights are exp2(s - m), the largest of them 2^4 when m was set, which it is again only where one passes 2^12.  The weights times V's scales
// enter the second product as two bf16 numbers each, 16 bits (the products are few): no fewer than attention_decode's weights have.  A bf16 number's last
// bits are lost below 2^-126, and the second's are 2^-16 of the weight: values of 2^-100 in magnitude keep all of them (weights of 1 at most lost 2^-9 of values of 2^-110).
// Bound by memory where a key is read for one tile: 32 sequences of 4 tokens behind 8000 (8 heads of 128) 97 us, 5.6 TB/s; by the chain of trips (lengths, pages, codes) in
// small calls: 32 single tokens behind 500 9 us.
template <class E, int D, int R, int NW>
__global__ __launch_bounds__(NW * 64, few_waves_per_simd(D, R, NW)) void attention_chunk_few_kernel(const ChunkArgs a)
{
    extern __shared__ __align__(16) float shared[];
    constexpr int NJ = (D + 63) / 64, DT = D / 16, ROWS = 16 * R;
    constexpr bool SHORT = few_waves_per_simd(D, R, NW) == 1;    // of registers for the vector unit
    typedef typename E::T T;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int h = lane & 15, g = lane >> 4;
    const int kv_heads = a.cache.kv_heads, head = blockIdx.x % kv_heads;
    const ChunkUnit<true, ROWS> unit(a, blockIdx.x / kv_heads, Index<0>{});
    if (!unit.there) return;
    const int group = unit.group, rows = min(unit.rows - unit.row0, ROWS), parts = unit.parts, b = unit.b;         // rows: of this tile
    const ChunkTiles list = unit.keys(a);
    // parts of whole turns of the wavefronts (the last of them may be empty)
    const int each = ((list.count + parts - 1) / parts + NW - 1) / NW * NW;
    const int first = min(list.count, unit.part * each), end = min(list.count, first + each);

    // the wavefront's blocks, 16 tiles ahead: lane l looks up block l % 4 of its tile l / 4
    constexpr int block_bytes = 32 * D + 128;
    auto look_up = [&](int i) {
        return chunk_place(a, b, head, 4 * list.at(min(i + NW * (lane >> 2), list.count - 1)) + (lane & 3));
    };
    int places = first + wave < end ? look_up(first + wave) : -1;

    u4 q[R][2 * NJ];
    ChunkRow range[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {                        // (rows past the last repeat it and are not written)
        const int row = unit.row0 + min(16 * r + h, rows - 1), query = row / group;
        range[r] = unit.row(a, row);
        const T *from = (const T *)a.q.data + (unit.first_row + query) * a.q.token_stride + (head * group + row % group) * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < 2 * NJ; ++s) {
            const int d = 64 * (s / 2) + 16 * g + 8 * (s % 2);
            __builtin_memcpy(&q[r][s], from + (d < D ? d : 0), 16);
            if (d >= D) q[r][s] = (u4)(0u);
            if constexpr (SHORT) asm volatile("" : "+a"(q[r][s]));       // (out of the vector unit's registers, which are short)
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
                asm volatile("" : "+v"(k[t][j]));        // (converted here and not before, and 16 codes at a time: all floats at once would be too many registers)
                codes_to(E{}, k[t][j], x);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    s[r][t] = mfma16(E{}, x[0], q[r][2 * j], s[r][t]);
                    s[r][t] = mfma16(E{}, x[1], q[r][2 * j + 1], s[r][t]);
                }
                __builtin_amdgcn_sched_barrier(0);
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
            if (__any(most > m[r] + 12.0f)) {            // weights are 2^12 at most, and 2^4 or more for the largest
                most = max_of_rows(most);
                const float next = most > m[r] + 12.0f ? most - 4.0f : m[r], fall = __builtin_amdgcn_exp2f(m[r] - next);
                l[r] *= fall;
                m[r] = next;
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    if constexpr (SHORT) asm volatile("" : "+a"(o[r][t]));
                    o[r][t] *= fall;
                    if constexpr (SHORT) asm volatile("" : "+a"(o[r][t]));
                }
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
            asm volatile("" : "+v"(v[t]));
            codes_to(BF16{}, v[t], x);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                o[r][t] = mfma16(BF16{}, x[0], rest[r][0], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[1], rest[r][1], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[0], p[r][0], o[r][t]);
                o[r][t] = mfma16(BF16{}, x[1], p[r][1], o[r][t]);
            }
            __builtin_amdgcn_sched_barrier(0);
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
            f4 *to = a.part_data + ((int64_t)blockIdx.x * ROWS + row) * (PIECES + 1);
            to[1 + piece] = sum;
            if (piece == 0) to[0] = (f4){ref, weight, 0.0f, 0.0f};
        } else {
            const int of = unit.row0 + row;
            put_chunk_row<E>(a, unit.first_row + of / group, head * group + of % group, 4 * piece, sum, weight);
        }
    }
}

// The parts of a tile's rows, joined in an order that depends on nothing but their number.  Lanes take D / 4 pieces of a row; with few parts a workgroup has as
// many rows as lanes allow, with many (rows_each 1) groups of lanes take the parts in turn, and the groups' sums are added in their order.
// Bound by its trips to memory (the lengths, then the parts, four on their way together): 4 - 7 us with the launch.
constexpr int kFewJoinThreads = 256;

template <class E, int D, int R>
__global__ __launch_bounds__(kFewJoinThreads) void attention_chunk_few_join_kernel(const ChunkArgs a, int rows_each, int blocks)
{
    constexpr int PIECES = D / 4, ROWS = 16 * R, SLOTS = kFewJoinThreads / PIECES;
    __shared__ f4 sums[SLOTS * PIECES];
    __shared__ float weights[SLOTS], refs[SLOTS];
    const int kv_heads = a.cache.kv_heads, tid = threadIdx.x, id = blockIdx.x / blocks, row0 = (int)blockIdx.x % blocks * rows_each;
    const int head = id % kv_heads, number = id / kv_heads;
    const ChunkUnit<true, ROWS> unit(a, number, Index<1>{});
    const int groups = SLOTS / rows_each, slot = tid / PIECES, piece = tid % PIECES;
    const int row = row0 + slot / groups, g = slot % groups, rows = min(unit.rows - unit.row0, ROWS);
    if (!unit.there || unit.parts == 1 || row0 >= rows) return;
    const f4 *from = a.part_data + (((int64_t)unit.part0 * kv_heads + head) * ROWS + min(row, rows - 1)) * (PIECES + 1);
    const int64_t step = (int64_t)kv_heads * ROWS * (PIECES + 1);
    float top = -3.0e38f, weight = 0.0f;
    f4 sum = (f4)(0.0f);
    if (slot < groups * rows_each) {
        for (int c = g; c < unit.parts; c += 4 * groups) {       // four on their way together
            f4 stats[4], x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f4 *part = from + min(c + i * groups, unit.parts - 1) * step;
                stats[i] = part[0];
                x[i] = part[1 + piece];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (c + i * groups >= unit.parts) break;
                const float now = fmaxf(top, stats[i][0]), fall = __builtin_amdgcn_exp2f(top - now), by = __builtin_amdgcn_exp2f(stats[i][0] - now);
                weight = weight * fall + stats[i][1] * by;
                sum = sum * fall + x[i] * by;
                top = now;
            }
        }
        sums[tid] = sum;
        if (piece == 0) weights[slot] = weight, refs[slot] = top;
    }
    __syncthreads();
    if (g > 0 || slot >= groups * rows_each || row >= rows) return;
    for (int x = 1; x < min(groups, unit.parts); ++x) {
        const float now = fmaxf(top, refs[slot + x]), fall = __builtin_amdgcn_exp2f(top - now), by = __builtin_amdgcn_exp2f(refs[slot + x] - now);
        weight = weight * fall + weights[slot + x] * by;
        sum = sum * fall + sums[tid + x * PIECES] * by;
        top = now;
    }
    const int of = unit.row0 + row;
    put_chunk_row<E>(a, unit.first_row + of / unit.group, head * unit.group + of % unit.group, 4 * piece, sum, weight);
}

// ---- many rows ----

// DP: head_dim rounded up; NW wavefronts of 32 rows, PER_SIMD of which share a SIMD's registers.
template <int DP_, int NW_, int PER_SIMD_>
struct ChunkCfg {
    static constexpr int DP = DP_, NW = NW_, PER_SIMD = PER_SIMD_, BM = 32 * NW, BN = kChunkKeys;
    // rows in LDS: of K (a key's elements) and of V (an element's keys), 16 bytes apart more than they are long, so that 16 consecutive ones' equal pieces
    // fall on different banks (64 of 4 bytes) without a turn of addresses
    static constexpr int kKeyRow = 2 * DP + 16, kValueRow = 2 * BN + 16;
    static constexpr int kKeys = BN * kKeyRow, kValues = DP * kValueRow, kValuesAt = 2 * kKeys, kScalesAt = kValuesAt + 2 * kValues, kScales = 2 * BN * 4;
    static constexpr int kLds = kScalesAt + 3 * kScales;         // two tiles of K, two of V, three of scales
    static constexpr int PIECES = (4 * DP + NW * 64 - 1) / (NW * 64);                    // of 16 codes of K (and of V) per thread
    static constexpr int kPart = BM * 2 * (DP / 8 + 1);          // 16-byte pieces of a part: sums, maximum and weight
};

// A tile of BM rows of a sequence: S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 matrix instructions, a wavefront 32 rows, lane c of each half row c.  Codes of 64 keys become
// 16-bit floats (exact) once for all wavefronts, on their way into LDS; K's scales meet the scores and V's the weights, in floats.  A lane holds the scores of 8 consecutive
// keys of each 16, which is the second product's operand as they lie.
// A softmax in one pass, with a reference that need not be the maximum: weights are exp2(s - m), m a score that was the largest once; a block whose weights sum up to more than 2^12 in a lane
// sets it anew.  Most blocks then have no maximum, no exchange between lanes and no sums to rescale.
// bf16 rows: weights times V's scales rounded to bf16 (2^-8 of each at most, as matrix instructions take them; the formula's error 2.4e-3 of the norm for 1.7e-3 with weights in 32 bits). f16 rows:
// two bf16 numbers, 16 bits, since one alone is less than the rows' own 11.
// Bound: per 32 x 32 scores of heads of 128 the matrix unit takes 16 instructions of 32 cycles and the vector unit some 150; one wavefront's instructions of either kind keep the other's of the
// same SIMD waiting (12 multiply-adds beside one matrix instruction: 113 - 120 cycles of two wavefronts, 67 and 65 of either alone), so a prompt of 8192 (32 heads on 8) takes
// 560 us, the matrix unit busy 45 % of the cycles, at 1.7 - 2.0 GHz. Hence what is not here: a maximum per block, conversions per wavefront, masks in tiles that all rows see.
template <class E, class C, bool VEC>
__global__ __launch_bounds__(C::NW * 64, C::PER_SIMD) void attention_chunk_kernel(const ChunkArgs a)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    constexpr int DP = C::DP, BN = C::BN, NW = C::NW, PIECES = C::PIECES, STEPS = DP / 16, DT = DP / 32;
    constexpr bool SPLIT = __is_same(typename E::T, _Float16);   // two bf16 numbers per weight
    // Codes are asked for two blocks ahead of their conversion: a prompt of 8192 554 -> 548 us, 512 tokens behind 16000 111 -> 110.  One block ahead
    // where that would take more registers than there are (tiles of 128 rows, heads of 128: prompts of 2048 61 us with it, 57 without).
    constexpr bool EARLY = DP != 128 || (!SPLIT && PIECES == 1);
    typedef typename E::T T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
    const int kv_heads = a.cache.kv_heads, D = a.cache.head_dim;
    const int head = blockIdx.x % kv_heads, number = blockIdx.x / kv_heads;
    const ChunkUnit<false, C::BM> tile(a, a.batch <= kMostShared ? number : a.slots - 1 - number, Index<0>{});
    if (!tile.there) return;
    const int group = tile.group, rows = tile.rows, parts = tile.parts;
    const ChunkTiles list(a, tile.row_of_all(a, tile.row0), tile.row_of_all(a, tile.row0 + C::BM - 1));
    const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)list.count * tile.part / parts));
    const int count = __builtin_amdgcn_readfirstlane((int)((int64_t)list.count * (tile.part + 1) / parts)) - first;

    const int row0 = tile.row0 + 32 * wave, row = min(row0 + col, rows - 1);             // the wavefront's first, the lane's
    const ChunkRow range = tile.row(a, row), row_first = tile.row_of_all(a, row0), row_last = tile.row_of_all(a, row0 + 31);

    // ---- the blocks of 16 tiles: lane l looks up block l % 4 of tile l / 4 ----
    const int block_bytes = 32 * D + 128;
    auto look_up = [&](int i) { return chunk_place(a, tile.b, head, 4 * list.at(min(first + i + (lane >> 2), list.count - 1)) + (lane & 3)); };
    // ---- a tile's codes, and where they go as 16-bit floats ----
    // (all threads store: those past the last piece others' again, those past head_dim something finite where it meets Q's zeros or becomes no output)
    int piece_block[PIECES], piece_at[PIECES], k_to[PIECES], v_to[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int p = (i * NW * 64 + tid) % (4 * DP), q = p % DP, per = D / 16, token = q < D ? q / per : 0, c = 2 * (q < D ? q % per : per);
        piece_block[i] = p / DP;
        piece_at[i] = q < D ? 16 * q : 0;
        k_to[i] = (16 * piece_block[i] + token) * C::kKeyRow + c * 16;
        v_to[i] = C::kValuesAt + q * C::kValueRow + piece_block[i] * 32;
    }
    u4 k_codes[PIECES], v_codes[PIECES], k_next[PIECES], v_next[PIECES];         // of the tile that becomes floats, and of the one behind it, on its way
    float a_scale = 0.0f;                                        // of block `wave` % 4: lanes 0 .. 15 K's, 16 .. 31 V's
    // block b of tile n of those looked up; the pieces of a wavefront are of one block mostly, which the scalar unit finds
    auto block_of = [&](int places, int b) { return a.cache.data + (int64_t)max(__builtin_amdgcn_readlane(places, b), 0) * block_bytes; };
    auto block_of_piece = [&](int places, int n, int i) {
        if constexpr (DP % 64 == 0) return block_of(places, 4 * n + (i * NW + wave) * 64 / DP % 4);
        else return a.cache.data + (int64_t)max(__shfl(places, 4 * n + piece_block[i]), 0) * block_bytes;
    };
    auto load_k = [&](int places, int n) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) k_next[i] = *(const u4 *)(block_of_piece(places, n, i) + (uint32_t)piece_at[i]);
        a_scale = *(const float *)(block_of(places, 4 * n + wave % 4) + (uint32_t)(32 * D + 4 * (lane & 31)));
    };
    auto load_v = [&](int places, int n) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) v_next[i] = *(const u4 *)(block_of_piece(places, n, i) + (uint32_t)(16 * D + piece_at[i]));
    };
    auto take = [](u4 (&codes)[PIECES], const u4 (&next)[PIECES]) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) codes[i] = next[i];
    };
    // dword x % 4 of piece x / 4, stored with the second and the fourth
    u4 out;
    auto store_step = [&](auto which, auto x, int buffer) {
        constexpr int X = decltype(x)::value, I = X / 4, W = X % 4;
        constexpr bool V = decltype(which)::value;
        u2 y;
        if constexpr (V) y = codes4_to(BF16{}, v_codes[I][W]);
        else y = codes4_to(E{}, k_codes[I][W]);
        out[2 * (W % 2)] = y[0];
        out[2 * (W % 2) + 1] = y[1];
        if constexpr (W % 2 == 1) *(u4 *)(lds + buffer * (V ? C::kValues : C::kKeys) + (V ? v_to[I] : k_to[I]) + W / 2 * 16) = out;
    };
    auto store_scales = [&](int tile_number) {
        ((float *)(lds + C::kScalesAt + tile_number % 3 * C::kScales))[(lane >> 4 & 1) * BN + 16 * (wave % 4) + (lane & 15)] = a_scale * (lane & 16 ? 1.0f : a.scale);
    };
    // elements past head_dim, and what stands for the values before the first block's, are 0
    for (int i = (D < DP ? 0 : C::kValuesAt + C::kValues) / 16 + tid; i < C::kScalesAt / 16; i += NW * 64) ((u4 *)lds)[i] = (u4)(0u);
    if (D < DP) __syncthreads();
    int places = count > 0 ? look_up(0) : -1;
    load_k(places, 0);
    load_v(places, 0);

    // ---- Q^T's operand: 8 elements of the lane's row per step ----
    u4 q[STEPS];
    const int qhead = head * group + row % group, token = tile.first_row + row / group;
    {
        const T *from = (const T *)a.q.data + token * a.q.token_stride + qhead * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int d = 16 * s + 8 * half;
            const T *at = from + (d < D ? d : 0);
            if constexpr (VEC) q[s] = *(const u4 *)at;
            else __builtin_memcpy(&q[s], at, 16);
            if (d >= D) q[s] = (u4)(0u);
            // (only the matrix unit reads it: beside the sums, out of the vector unit's registers, where a wavefront has more than these)
            if constexpr (C::PER_SIMD == 1) asm volatile("" : "+a"(q[s]));
        }
    }
    // the key whose scores are row `col` of the first product: so that a lane holds 8 consecutive keys' of each 16
    const int key = 16 * (col >> 4) + 8 * (col >> 2 & 1) + 4 * (col >> 3 & 1) + (col & 3);
    const uint8_t *const k_from = lds + key * C::kKeyRow + 16 * half, *const v_from = lds + C::kValuesAt + col * C::kValueRow + 16 * half;
    const float *const ks_from = (const float *)(lds + C::kScalesAt) + 8 * half;
    const float *const vs_from = (const float *)(lds + C::kScalesAt) + BN + 16 * (lane >> 3 & 1) + 8 * half + (lane & 7);    // lane x of 16: score x's

    f16v o[DT], s[2];
    u4 p[2][2], rest[2][2];
    f4 ks[2];                                                    // scales of K of the next four keys, and of V of the block's 16
    float vs;
    float m = -3.0e38f, l = 0.0f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[t] = (f16v)(0.0f);
#pragma unroll
    for (int u = 0; u < 2; ++u) p[1][u] = rest[1][u] = (u4)(0u);
    auto k_operand = [&](const uint8_t *at, int u) { return *(const u4 *)(at + 32 * u); };
    auto v_operand = [&](const uint8_t *at, int u, int t) { return *(const u4 *)(at + t * 32 * C::kValueRow + 32 * u); };

    // Block j of 32 keys (B: its parity): the scores of block j become weights while the matrix unit makes those of block j + 1 and takes the weights of
    // block j - 1 to the values, and codes of the next tile (of K where B is 0, of V where it is 1) become floats: 16 steps, with one of the lane's scores and a
    // share of everything else in each.
    constexpr float kMostSum = 0x1p12f;
    auto block = [&](auto parity, auto masked, int i, uint32_t lost) {
        constexpr int B = decltype(parity)::value;
        constexpr bool MASKED = decltype(masked)::value;
        const int odd = i & 1, next = i % 3 == 2 ? 0 : i % 3 + 1;
        const uint8_t *const k_at = k_from + (B == 0 ? odd : 1 - odd) * C::kKeys + (B == 0 ? 32 * C::kKeyRow : 0);           // block j + 1's
        const uint8_t *const v_at = v_from + (B == 0 ? 1 - odd : odd) * C::kValues + (B == 0 ? 64 : 0);                      // block j - 1's
        const float *const scales = ks_from + i % 3 * (C::kScales / 4) + 32 * B;
        uint32_t seen = 0;
        if constexpr (MASKED) {
            uint64_t bits = range.seen(BN * list.at(first + i), a.sinks);
#pragma unroll
            for (int g = 0; g < 4; ++g)
                if (lost >> g & 1) bits &= ~((uint64_t)0xffff << (16 * g));
            seen = (uint32_t)(bits >> (32 * B)) >> (8 * half);
        }
        // MFMAS matrix instructions over all steps but the first (their operands are on their way), scores and values in turn, operands read AHEAD
        constexpr int MFMAS = 2 * STEPS, AHEAD = 1, RING = AHEAD + 1;
        u4 k_ahead[RING], v_ahead[RING];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            k_ahead[u] = k_operand(k_at, u);
            v_ahead[u] = v_operand(v_at, u / DT, u % DT);
        }
        float sum = 0.0f, w[2];
        float vs_next = 0.0f;
        uint32_t pinned;
        __builtin_amdgcn_sched_barrier(0);
        unrolled<16>([&](auto step) {
            constexpr int N = decltype(step)::value;
            // the weights: keys 16 (N / 8) + 8 half + N % 8 of the block
            if constexpr (N % 4 == 0) {                  // four keys' scales ahead, the next block's first at last
                constexpr int G = N / 4 + 1;
                const float *from = scales + 16 * (G / 2) + 4 * (G % 2);
                if constexpr (G == 4) from = B == 0 ? scales + 32 : ks_from + next * (C::kScales / 4);
                ks[G & 1] = *(const f4 *)from;
                if constexpr (G == 4) vs_next = B == 0 ? vs_from[i % 3 * (C::kScales / 4) + 32] : vs_from[next * (C::kScales / 4)];
            }
            float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[B][N], ks[N / 4 & 1][N % 4], -m));
            // what is not seen is made 0 by its bits, whatever it is: as a weight, and times V's scale, which may be NaN
            const uint32_t keep = MASKED ? (uint32_t)__builtin_amdgcn_sbfe((int)seen, 16 * (N / 8) + N % 8, 1) : 0;
            if constexpr (MASKED) x = __uint_as_float(__float_as_uint(x) & keep);
            sum += x;
            x *= of_row<N>(vs);
            if constexpr (MASKED) x = __uint_as_float(__float_as_uint(x) & keep);
            w[N % 2] = x;
            if constexpr (N % 2 == 1) {
                if constexpr (SPLIT) {
                    const u2 both = split2(w[0], w[1]);
                    pinned = both[0];
                    rest[B][N / 8][N % 8 / 2] = both[1];
                } else {
                    pinned = pack2<BF16>(w[0], w[1]);
                }
                asm volatile("" : "+v"(pinned));         // (formed here, beside the matrix unit's work, and not where it is wanted)
                p[B][N / 8][N % 8 / 2] = pinned;
            }
            // the matrix unit's share
            constexpr int M0 = N < 1 ? 0 : (N - 1) * MFMAS / 15, M1 = N * MFMAS / 15;
            unrolled<M1 - M0>([&](auto x) {
                constexpr int M = M0 + decltype(x)::value, U = M / 2;
                if constexpr (M % 2 == 0) {
                    if constexpr (U + AHEAD < STEPS) k_ahead[(U + AHEAD) % RING] = k_operand(k_at, U + AHEAD);
                    s[1 - B] = mfma32(E{}, k_ahead[U % RING], q[U], U == 0 ? (f16v)(0.0f) : s[1 - B]);
                } else {
                    if constexpr (U + AHEAD < STEPS) v_ahead[(U + AHEAD) % RING] = v_operand(v_at, (U + AHEAD) / DT, (U + AHEAD) % DT);
                    if constexpr (SPLIT) o[U % DT] = mfma32(BF16{}, v_ahead[U % RING], rest[1 - B][U / DT], o[U % DT]);
                    o[U % DT] = mfma32(BF16{}, v_ahead[U % RING], p[1 - B][U / DT], o[U % DT]);
                }
            });
            // the next tile's codes
            unrolled<(N + 1) * 4 * PIECES / 16 - N * 4 * PIECES / 16>([&](auto x) {
                store_step(Index<B>{}, Index<N * 4 * PIECES / 16 + decltype(x)::value>{}, 1 - odd);
            });
            if constexpr (N % 2 == 1) __builtin_amdgcn_sched_barrier(0);
        });
        // Weights stay relative to what was the largest score once, as long as their sums are moderate (bf16 and float lose nothing by that).
        if (__any(sum > kMostSum)) {
            float most = m;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float x = s[B][e] * scales[16 * (e / 8) + e % 8];
                if constexpr (MASKED) x = where_bit(seen, 16 * (e / 8) + e % 8, x, -__builtin_inff());
                most = fmaxf(most, x);
            }
            most = max_of_halves(most);
            const float fall = __builtin_amdgcn_exp2f(m - most);
            m = most;
            l *= fall;
            sum = 0.0f;
#pragma unroll
            for (int t = 0; t < DT; ++t) {               // (one after the other, and not before the branch: or the registers would not do)
                if constexpr (C::PER_SIMD == 1) asm volatile("" : "+a"(o[t]));
                o[t] *= fall;
                if constexpr (C::PER_SIMD == 1) asm volatile("" : "+a"(o[t]));
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int of = 16 * (e / 8) + e % 8 + h;
                    float x = __builtin_fmaf(s[B][e + h], scales[of], -m);
                    if constexpr (MASKED) x = where_bit(seen, of, x, -__builtin_inff());
                    x = __builtin_amdgcn_exp2f(x);
                    sum += x;
                    x *= scales[BN + of];
                    if constexpr (MASKED) x = where_bit(seen, of, x, 0.0f);
                    w[h] = x;
                }
                if constexpr (SPLIT) {
                    const u2 both = split2(w[0], w[1]);
                    p[B][e / 8][e % 8 / 2] = both[0];
                    rest[B][e / 8][e % 8 / 2] = both[1];
                } else {
                    p[B][e / 8][e % 8 / 2] = pack2<BF16>(w[0], w[1]);
                }
            }
        }
        vs = vs_next;
        l += sum;
    };
    if (count > 0) {
        take(k_codes, k_next);
        take(v_codes, v_next);
        unrolled<4 * PIECES>([&](auto x) { store_step(Index<0>{}, x, 0); });
        unrolled<4 * PIECES>([&](auto x) { store_step(Index<1>{}, x, 0); });
        store_scales(0);
        uint32_t lost = (uint32_t)__ballot(places < 0) & 15u;    // blocks of the tile that are not there
        auto next = [&](int i) {                                 // (past the end: the last tile again)
            if (i < count && (i & 15) == 0) places = look_up(i);
            return min(i, count - 1) & 15;
        };
        int n = next(1);
        uint32_t lost_next = (uint32_t)(__ballot(places < 0) >> (4 * n)) & 15u;
        load_k(places, n);
        load_v(places, n);
        __syncthreads();
        ks[0] = *(const f4 *)ks_from;
        vs = vs_from[0];
#pragma unroll
        for (int u = 0; u < STEPS; ++u) s[0] = mfma32(E{}, k_operand(k_from, u), q[u], u == 0 ? (f16v)(0.0f) : s[0]);
        int i = 0;
        auto whole = [&]() {                                     // (the same in all lanes, which the compiler has to see)
            const int key0 = BN * list.at(first + i);
            return __builtin_amdgcn_readfirstlane(!lost && row_first.sees_all(key0, a.sinks) && row_last.sees_all(key0, a.sinks)) != 0;
        };
        auto step = [&](auto masked) {
            const uint32_t lost_now = lost;
            store_scales(i + 1);
            take(k_codes, k_next);
            n = next(i + 2);
            if constexpr (EARLY) load_k(places, n);
            lost = lost_next;
            lost_next = (uint32_t)(__ballot(places < 0) >> (4 * n)) & 15u;
            block(Index<0>{}, masked, i, lost_now);
            if constexpr (!EARLY) load_k(places, n);
            __syncthreads();
            take(v_codes, v_next);
            if constexpr (EARLY) load_v(places, n);
            block(Index<1>{}, masked, i, lost_now);
            if constexpr (!EARLY) load_v(places, n);
            ++i;
        };
        if (row0 >= rows) {                                      // a wavefront without rows: codes alone
            while (i < count) {
                store_scales(i + 1);
                take(k_codes, k_next);
                n = next(i + 2);
                load_k(places, n);
                unrolled<4 * PIECES>([&](auto x) { store_step(Index<0>{}, x, ~i & 1); });
                __syncthreads();
                take(v_codes, v_next);
                load_v(places, n);
                unrolled<4 * PIECES>([&](auto x) { store_step(Index<1>{}, x, ~i & 1); });
                ++i;
            }
            if (parts == 1) return;
        }
        while (i < count) {                                      // (two loops, not a choice in one: that would keep the sums twice)
            while (i < count && whole()) step(Index<0>{});
            while (i < count && !whole()) step(Index<1>{});
        }
        const uint8_t *const v_at = v_from + (count - 1 & 1) * C::kValues + 64;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                const u4 x = v_operand(v_at, u, t);
                if constexpr (SPLIT) o[t] = mfma32(BF16{}, x, rest[1][u], o[t]);
                o[t] = mfma32(BF16{}, x, p[1][u], o[t]);
            }
    }
    const float weight = sum_of_halves(l);
    if (parts > 1) {
        f4 *mine = a.part_data + (int64_t)blockIdx.x * C::kPart + tid;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(4 * t + i) * NW * 64] = (f4){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
        mine[DP / 8 * NW * 64] = (f4){m, weight, 0.0f, 0.0f};
        return;
    }
    // ---- O = O^T / l: 4 consecutive elements per lane and quarter, exchanged between lane halves to 8 ----
    int of = row0 + col;
    asm volatile("" : "+v"(of));                                 // (found again here: what is kept through the loop takes its registers)
    of = min(of, rows - 1);
    T *to = (T *)a.o.data + (tile.first_row + of / group) * a.o.token_stride + (head * group + of % group) * a.o.head_stride;
    const float by = 1.0f / weight;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = weight == 0.0f ? 0.0f : o[t][i + e] * by;
            const u2 s0 = __builtin_amdgcn_permlane32_swap(pack2<E>(x[0], x[1]), pack2<E>(x[4], x[5]), false, false);
            const u2 s1 = __builtin_amdgcn_permlane32_swap(pack2<E>(x[2], x[3]), pack2<E>(x[6], x[7]), false, false);
            const u4 y = {s0[0], s1[0], s0[1], s1[1]};
            const int d = 32 * t + 2 * i + 8 * half;
            if (row0 + col < rows && d < D) {
                if constexpr (VEC) {
                    *(u4 *)(to + d) = y;
                } else {
                    T e8[8];
                    __builtin_memcpy(e8, &y, 16);
#pragma unroll
                    for (int e = 0; e < 8; ++e) to[d + e] = e8[e];
                }
            }
        }
}

// The parts of a tile, joined in their order: `blocks` workgroups a tile, DP / 8 / blocks pieces of 4 elements of a lane each.  A launch of its own after the parts: 8 - 13 us,
// of which the trips to the lengths and to the first parts are 3; one part at a time instead of eight on their way together 20.
template <class E, class C>
__global__ __launch_bounds__(C::NW * 64) void attention_chunk_join_kernel(const ChunkArgs a, int blocks)
{
    constexpr int THREADS = C::NW * 64, PIECES = C::DP / 8;
    const int kv_heads = a.cache.kv_heads, block = blockIdx.x % blocks, head = blockIdx.x / blocks % kv_heads, number = blockIdx.x / blocks / kv_heads;
    const ChunkUnit<false, C::BM> tile(a, number, Index<1>{});
    const int tid = threadIdx.x, lane = tid & 63, row = tile.row0 + 32 * (tid >> 6) + (lane & 31), parts = tile.parts;
    if (!tile.there || parts == 1 || row >= tile.rows) return;
    const f4 *from = a.part_data + ((int64_t)tile.part0 * kv_heads + head) * C::kPart + tid;
    for (int piece = block; piece < PIECES; piece += blocks) {
        const int d = 8 * piece + 4 * (lane >> 5);               // 32 (piece / 4) + 8 (piece % 4) + ..
        if (d >= a.cache.head_dim) return;
        float top = -3.0e38f, l = 0.0f;
        f4 o = (f4)(0.0f);
        for (int p0 = 0; p0 < parts; p0 += 8) {                  // eight on their way together
            f4 stats[8], x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const f4 *part = from + (int64_t)min(p0 + i, parts - 1) * kv_heads * C::kPart;
                stats[i] = part[PIECES * THREADS];
                x[i] = part[piece * THREADS];
            }
            float now = top;
#pragma unroll
            for (int i = 0; i < 8; ++i) now = fmaxf(now, stats[i][0]);
            const float fall = __builtin_amdgcn_exp2f(top - now);
            l *= fall;
            o *= fall;
            top = now;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (p0 + i >= parts) break;
                const float by = __builtin_amdgcn_exp2f(stats[i][0] - top);
                l += stats[i][1] * by;
                o += x[i] * by;
            }
        }
        put_chunk_row<E>(a, tile.first_row + row / tile.group, head * tile.group + row % tile.group, d, o, l);
    }
}

}  // namespace ngemm
