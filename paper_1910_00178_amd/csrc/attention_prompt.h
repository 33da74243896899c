// Attention over packed rows, whole prompts and prompts behind a context.
#pragma once
#include "attention_common.h"

namespace ngemm {

struct PromptArgs {
    Rows q, k, v, o;
    const int32_t *q_offsets, *k_offsets;
    int32_t batch, q_heads, kv_heads, head_dim, q_tokens, k_tokens, causal;
    float scale;             // of the scores, times log2 e; not negative (Q's sign is turned instead)
    uint32_t q_xor;
    int32_t slots;           // workgroups of a K/V head
    float share;             // of the units, where the keys are split: a K/V head's; else 0
    f4 *parts;               // keys split: [slots][kv_heads] times kPart
};

constexpr int kLeastRun = 256;                                   // keys of a workgroup where a tile's are split
constexpr int kMostSplit = 128;                                  // sequences of a call that are

// DP: head_dim rounded up; RW groups of 32 rows, each of KS wavefronts that share out the BN keys of a tile; PER_CU workgroups to a unit.
template <int DP_, int RW_, int KS_, int BN_, int PER_CU_>
struct PromptCfg {
    static constexpr int DP = DP_, RW = RW_, KS = KS_, BN = BN_, PER_CU = PER_CU_;
    static constexpr int NW = RW * KS, BM = 32 * RW, KT = BN / 32 / KS;       // KT: 32-key blocks of a wavefront
    static constexpr int CH = DP / 8;              // CH: 16-byte chunks of a row
    static constexpr int kTile = BN * DP * 2, kStage = 2 * kTile, kFlags = 2 * kStage;
    static constexpr int LOADS = kTile / 1024 / NW;              // 1 KiB copies of K (and of V) per wavefront
    static constexpr int AHEAD = DP == 96 ? 6 : DP == 64 || DP == 192 ? 4 : DP == 256 ? 2 : 8, V_AHEAD = DP == 96 ? 3 : DP == 64 || DP == 256 ? 2 : 4;     // operands read together
    static_assert(KT * (DP / 16) % AHEAD == 0 && 2 * KT * (DP / 32) % V_AHEAD == 0, "whole groups");
    static constexpr int kPart = BM * 2 * (DP / 8 + 1);          // 16-byte pieces of a part: sums, maximum and weight
    static constexpr int kMerge = (KS - 1) * kPart * 16;
    static constexpr int kLds = (kFlags > kMerge ? kFlags : kMerge) + 16;
    static_assert(kLds >= NW * (DP + 64) * 4, "rows one by one");
    static_assert(kTile % (1024 * NW) == 0 && KT * 32 * KS == BN, "whole copies and blocks");
    // Where chunk c of key j lies: so that 16 consecutive keys' equal chunks of K, and the 64 bytes of four consecutive keys of V,
    // fall on different banks (64 banks of 4 bytes).
    static __device__ __forceinline__ int k_swizzle(int j)
    {
        return CH % 16 == 0 ? j & 15 : CH % 8 == 0 ? (j >> 1) & 7 : (j >> 2) & 3;
    }
    static __device__ __forceinline__ int v_swizzle(int j)
    {
        return CH % 16 == 0 ? (j & 3) << 2 : CH % 8 == 0 ? (j & 2) << 1 : 0;
    }
};

// Of each half of two dwords, as 16-bit numbers without sign, the larger.
__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b)
{
    typedef uint16_t V2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(V2, a), __builtin_bit_cast(V2, b)));
}

// A factor 2^weight_bits of the softmax weights and their sums, and how much weights may grow (2^weight_slack) before what they are relative to is
// raised.  The weights enter the second product in the rows' type, of which float16 loses bits below 2^-14 while their sum has
// them: with its upper range in use, all weights down to 2^-25 of a row's largest have 11 bits, and the others are off by 2^-36 of it at most.  2^13 and a slack
// of 2 take 1 to 2 % longer (8192 tokens of 32 heads of 128, f16: 569 us for 564), 2^11 takes what 1 does.
template <class E>
constexpr float weight_bits() { return __is_same(typename E::T, _Float16) ? 11.0f : 0.0f; }
template <class E>
constexpr float weight_slack() { return __is_same(typename E::T, _Float16) ? 4.0f : 8.0f; }

// Copies memory -> LDS, 16 bytes a lane from base + offset; what lies past the buffer's end becomes 0.  Written as the instruction: behind
// the builtin, the compiler lets the transposing LDS reads wait for every copy in flight, those of the next tile among them.  No
// register is written; who reads the LDS waits with copies_landed() and a barrier.
typedef uint32_t Buffer __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Buffer buffer_of(const void *from, int bytes)
{
    const uint64_t at = (uint64_t)from;
    return (Buffer){(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32)) & 0xffffu,
                    (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy_to_lds(Buffer from, uint32_t lds_at, uint32_t offset)
{
    // (M0 is the compiler's as well, for what it makes itself of LDS copies and indexes: named, so that it keeps no value there.  It warns that the
    // register is one of its reserved ones, which is the reason.  Five wait states: what a vector instruction that wrote the descriptor's registers needs; M0 needs one.)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane((int)lds_at)), "v"(offset), "s"(from) : "memory", "m0");
}
#pragma clang diagnostic pop
__device__ __forceinline__ void copies_landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A tile of a sequence's rows, which are its queries times the heads that share a K/V head, heads fastest.
template <class C>
struct PromptTile {
    int q_first, queries, row0, rows, k_first, keys, group, causal;
    int key_tiles, part, parts, part0;                           // `parts` workgroups share out the key tiles; of them this one, and the first one's number
    bool there;

    // Where a workgroup takes all keys: tile `number`.  Sequence b has the slots floor(rows before it / BM) + b .. : as many as its rows
    // need or one more.
    __device__ __forceinline__ PromptTile(const PromptArgs &a, int number) : group(a.q_heads / a.kv_heads), causal(a.causal), part(0), parts(1), part0(0)
    {
        int of[4];
        const int b = find_sequence(a.batch, number, {a.q_offsets, a.q_offsets + 1, a.k_offsets, a.k_offsets + 1}, of,
                                    [&](int offset, int x) { return offset * group / C::BM + x; });
        take(a, of);
        row0 = (number - (of[0] * group / C::BM + b)) * C::BM;
        there = row0 >= 0 && row0 < rows;
        key_tiles = tiles_of_keys(min(row0 + C::BM, rows) - 1);
    }
    // Where the keys of up to kMostSplit sequences are shared out: workgroup `number` of a head (JOIN: tile `number`).  If each tile took what its
    // sequence's last one does, which sees the most, all units would have the same; tiles that see less are cut into as many parts.
    template <int JOIN>
    __device__ __forceinline__ PromptTile(const PromptArgs &a, int number, Index<JOIN>) : group(a.q_heads / a.kv_heads), causal(a.causal)
    {
        constexpr int TURNS = kMostSplit / 64;
        const int lane = threadIdx.x & 63;
        int of[TURNS][4] = {}, tiles[TURNS] = {}, most[TURNS] = {};
        float work = 0.0f;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            if (64 * i >= a.batch) break;
            const int b = min(64 * i + lane, a.batch - 1);
            of[i][0] = a.q_offsets[b], of[i][1] = a.q_offsets[b + 1], of[i][2] = a.k_offsets[b], of[i][3] = a.k_offsets[b + 1];
            take(a, of[i]);
            tiles[i] = 64 * i + lane < a.batch ? (rows + C::BM - 1) / C::BM : 0;
            most[i] = tiles_of_keys(rows - 1);
            work += (float)tiles[i] * (float)most[i];
        }
        work = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, sums_up_to(work)), 63));
        const float share = a.share / fmaxf(work, 1.0f);
        int tile = 0, each = 1, tiles_before = 0, parts_before = 0;
        part = part0 = 0;
        there = false;
#pragma unroll
        for (int i = 0; i < TURNS; ++i) {
            if (64 * i >= a.batch) break;
            // (a whole number of parts may come out as a little less)
            const int cut = max(1, min((int)((float)most[i] * share + 0x1p-8f), most[i] / (kLeastRun / C::BN))), all = tiles[i] * cut;
            const int tiles_to = tiles_before + sums_up_to(tiles[i]), parts_to = parts_before + sums_up_to(all);
            const int begin = JOIN ? tiles_to - tiles[i] : parts_to - all, end = JOIN ? tiles_to : parts_to;
            const uint64_t here = __ballot(begin <= number && number < end);
            if (here) {
                const int l = __builtin_ctzll(here);
                const int mine[4] = {__builtin_amdgcn_readlane(of[i][0], l), __builtin_amdgcn_readlane(of[i][1], l), __builtin_amdgcn_readlane(of[i][2], l),
                                     __builtin_amdgcn_readlane(of[i][3], l)};
                take(a, mine);
                each = __builtin_amdgcn_readlane(cut, l);
                const int at = number - __builtin_amdgcn_readlane(begin, l);
                tile = JOIN ? at : at / each;
                part = JOIN ? 0 : at % each;
                part0 = __builtin_amdgcn_readlane(parts_to - all, l) + tile * each;
                tile = __builtin_amdgcn_readlane(tiles[i], l) - 1 - tile;          // the longest first
                there = true;
            }
            tiles_before = __builtin_amdgcn_readlane(tiles_to, 63);
            parts_before = __builtin_amdgcn_readlane(parts_to, 63);
        }
        row0 = tile * C::BM;
        key_tiles = there ? tiles_of_keys(min(row0 + C::BM, rows) - 1) : 0;
        parts = max(1, min(each, key_tiles / (kLeastRun / C::BN)));              // no less than kLeastRun keys a part
        there = there && part < parts && part0 >= 0 && part0 + parts <= a.slots;  // (places past the end: offsets that fall)
        // (the same in all lanes, which the compiler does not see)
        for (int *const x : {&q_first, &queries, &row0, &rows, &k_first, &keys, &key_tiles, &part, &parts, &part0}) *x = __builtin_amdgcn_readfirstlane(*x);
        there = __builtin_amdgcn_readfirstlane(there);
    }
    __device__ __forceinline__ void take(const PromptArgs &a, const int (&of)[4])
    {
        q_first = min(max(of[0], 0), a.q_tokens);
        queries = min(max(of[1], q_first), a.q_tokens) - q_first;
        rows = queries * group;
        k_first = min(max(of[2], 0), a.k_tokens);
        keys = min(max(of[3], k_first), a.k_tokens) - k_first;
    }
    __device__ __forceinline__ int tiles_of_keys(int row) const { return row < 0 ? 0 : max(0, (last_seen(row) + C::BN) / C::BN); }
    __device__ __forceinline__ int first_tile() const { return (int)((int64_t)key_tiles * part / parts); }
    __device__ __forceinline__ int end_tile() const { return (int)((int64_t)key_tiles * (part + 1) / parts); }
    // the last key that a row sees
    __device__ __forceinline__ int last_seen(int row) const { return causal ? min(row / group + keys - queries, keys - 1) : keys - 1; }
};

// The rows of a tile element by element: what a workgroup does whose keys hold an infinity or a NaN that not all of its rows see (0 times
// it would reach the others in the matrix instructions).
template <class E, class C>
__device__ __forceinline__ void prompt_rows_one_by_one(const PromptArgs &a, const PromptTile<C> &tile, int head, int first_key, int end_key, f4 *part,
                                                                 uint8_t *lds)
{
    typedef typename E::T T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.head_dim;
    float *q = (float *)lds + wave * (C::DP + 64), *p = q + C::DP;
    const T *kr = (const T *)a.k.data + tile.k_first * a.k.token_stride + head * a.k.head_stride;
    const T *vr = (const T *)a.v.data + tile.k_first * a.v.token_stride + head * a.v.head_stride;
    for (int r = wave; r < C::BM; r += C::NW) {
        const int row = min(tile.row0 + r, tile.rows - 1), token = tile.q_first + row / tile.group, qhead = head * tile.group + row % tile.group;
        const T *qr = (const T *)a.q.data + token * a.q.token_stride + qhead * a.q.head_stride;
        for (int d = lane; d < D; d += 64) q[d] = a.q_xor ? -E::get(qr[d]) : E::get(qr[d]);
        const int end = min(end_key, tile.last_seen(row) + 1);
        float m = -3.0e38f / fmaxf(a.scale, 1.0f), l = 0.0f, o[(C::DP + 63) / 64] = {};
        __builtin_amdgcn_wave_barrier();
        for (int t0 = first_key; t0 < end; t0 += 64) {
            const int t = t0 + lane;
            float s = -__builtin_inff();
            if (t < end) {
                s = 0.0f;
                for (int d = 0; d < D; ++d) s += q[d] * E::get(kr[t * a.k.token_stride + d]);
            }
            const float most = fmaxf(max_of_rows(max_of_lanes<16>(s)), m), fall = __builtin_amdgcn_exp2f((m - most) * a.scale);
            const float w = t < end ? __builtin_amdgcn_exp2f((s - most) * a.scale + weight_bits<E>()) : 0.0f;
            float sum = w;
            for (int x = 32; x; x /= 2) sum += __shfl_xor(sum, x);
            l = l * fall + sum;
            m = most;
            __builtin_amdgcn_wave_barrier();
            p[lane] = w;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int n = 0; n < (C::DP + 63) / 64; ++n) {
                const int d = lane + 64 * n;
                o[n] *= fall;
                if (d < D)
                    for (int j = 0; j < 64 && t0 + j < end; ++j) o[n] += p[j] * E::get(vr[(t0 + j) * a.v.token_stride + d]);
            }
        }
        __builtin_amdgcn_wave_barrier();
        const int place = r / 32 * 64 + r % 32;              // of the row's lower lane in a part
#pragma unroll
        for (int n = 0; n < (C::DP + 63) / 64; ++n) {
            const int d = lane + 64 * n;
            if (d >= D || tile.row0 + r >= tile.rows) continue;
            if (part) ((float *)(part + d / 8 * C::BM * 2 + place + (d / 4 & 1) * 32))[d % 4] = o[n];
            else ((T *)a.o.data)[token * a.o.token_stride + qhead * a.o.head_stride + d] = E::put(tile.last_seen(row) < 0 ? 0.0f : o[n] / l);
        }
        if (part && lane < 2) part[C::DP / 8 * C::BM * 2 + place + 32 * lane] = (f4){m, l, 0.0f, 0.0f};
    }
}

// Rows of a workgroup: the queries of a sequence times the q_heads / kv_heads heads that share a K/V head, heads fastest.  S^T = K Q^T
// and O^T = V^T P^T on 32 x 32 x 16 matrix instructions: a lane holds scores of one row (lane % 32), so the softmax needs one exchange of
// lane halves per tile, and P^T's operand is what the lane holds, rounded, with the keys in the order in which the transposing LDS
// reads deliver V.
//
// Long prompts are bound by the matrix unit and the power it draws: 8192 tokens, causal, 32 heads on 8 K/V heads of 128 (bf16) 510 to 590 us by the card
// and what runs beside it (traced launches, alone between host work, are the slow ones), 0.93 to 1.08 PFLOP/s, where a large library product of that type
// reaches 1.21; the matrix unit is busy for 51 % of the cycles, the clock falls to 2.0 GHz, LDS reads have no bank conflict.  Heads of 64: 0.99 PFLOP/s,
// 96: 1.06, 192 and 256: 1.02.  Two workgroups of four wavefronts share a unit so that one's softmax runs beside the other's products; heads of more than 128
// have no registers for that, and there two wavefronts halve a tile's keys (of more than 192 even so six registers do not fit, and one of the reloads, in tiles that are
// masked, waits for the next tile's copies as well).  Neither four tiles in LDS nor the softmax of one tile between the products of the next (535 us for 517)
// gained anything.
// Few rows behind a long context are bound by memory, with what the parts write: 96 rows each behind 3900 and 2100 keys (16 heads on 4 of 256, f16) 26.4 us, in
// which some 60 MB are read, K and V being 25 (three tiles of rows share a K/V head and mostly fetch its keys each for themselves), and 35 MB of parts written; 10.2
// for the join, which reads them.  The smallest prompts are bound by the launch: 8 of 128 tokens (12 heads of 64) 5.4 to 6.2 us.
// Rows that are not at 16-byte multiples go through registers element by element: 2048 tokens of the first heads 211 us for 53.
template <class E, class C, bool VEC>
__global__ __launch_bounds__(C::NW * 64, C::PER_CU * C::NW / 4) void attention_prompt_kernel(const PromptArgs a)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    constexpr int DP = C::DP, NW = C::NW, BN = C::BN, CH = C::CH, KT = C::KT;
    typedef typename E::T T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int half = lane >> 5, col = lane & 31, row_group = wave % C::RW, key0 = 32 * KT * (wave / C::RW);   // key0: its first of a tile
    const int head = blockIdx.x % a.kv_heads, number = blockIdx.x / a.kv_heads;
    const int group = a.q_heads / a.kv_heads, D = a.head_dim;

    const PromptTile<C> tile_of = a.share > 0.0f ? PromptTile<C>(a, number, Index<0>{}) : PromptTile<C>(a, a.slots - 1 - number);
    const int q_first = tile_of.q_first, row0 = tile_of.row0, rows = tile_of.rows;
    const int k_first = tile_of.k_first, keys = tile_of.keys;
    if (!tile_of.there) return;
    auto last_seen = [&](int row) { return tile_of.last_seen(row); };
    const int row = row0 + 32 * row_group + col;
    const bool row_there = row < rows;
    const int query = min(row, rows - 1) / group, qhead = head * group + min(row, rows - 1) % group;
    const int seen = last_seen(min(row, rows - 1));
    const int wave_first = min(row0 + 32 * row_group, rows - 1), wave_last = min(row0 + 32 * row_group + 31, rows - 1);
    const int seen_by_all = last_seen(wave_first), seen_by_any = last_seen(wave_last);
    const int group_seen_by_all = last_seen(row0);
    const int parts = tile_of.parts, first_tile = tile_of.first_tile(), tiles = tile_of.end_tile();

    const T *kbase = (const T *)a.k.data + k_first * a.k.token_stride + head * a.k.head_stride;
    const T *vbase = (const T *)a.v.data + k_first * a.v.token_stride + head * a.v.head_stride;

    // ---- copies of a tile into LDS ----
    // (where a round of copies takes whole periods of the swizzles, the lanes' offsets of all rounds differ by the same)
    constexpr bool SAME = NW * 64 % (16 * CH) == 0;
    uint32_t kv_off[2][SAME ? 1 : C::LOADS];
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (SAME ? 1 : C::LOADS); ++i) {
            const int s = (i * NW + wave) * 64 + lane, j = s / CH, p = s % CH;
            const int kc = p ^ C::k_swizzle(j), vc = p ^ C::v_swizzle(j);
            kv_off[0][i] = kc * 8 < D ? (uint32_t)(j * a.k.token_stride * 2 + kc * 16) : 0x80000000u;
            kv_off[1][i] = vc * 8 < D ? (uint32_t)(j * a.v.token_stride * 2 + vc * 16) : 0x80000000u;
        }
    }
    auto load_tile = [&](int tile, int stage) {
        const int left = min(keys - tile * BN, BN);              // rows past it, and elements past head_dim, become 0
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const T *from = which ? vbase + (int64_t)tile * BN * a.v.token_stride : kbase + (int64_t)tile * BN * a.k.token_stride;
            const int64_t stride = which ? a.v.token_stride : a.k.token_stride;
            uint8_t *to = lds + stage * C::kStage + which * C::kTile;
            if constexpr (VEC) {
                const Buffer buffer = buffer_of(from, (int)((left - 1) * stride * 2 + D * 2));
#pragma unroll
                for (int i = 0; i < C::LOADS; ++i)
                    copy_to_lds(buffer, (uint32_t)(uintptr_t)(lds_ptr)(to + (i * NW + wave) * 1024),
                                SAME ? kv_off[which][0] + i * (uint32_t)(NW * 64 / CH * stride * 2) : kv_off[which][SAME ? 0 : i]);
            } else {
                for (int i = 0; i < C::LOADS; ++i) {
                    const int s = (i * NW + wave) * 64 + lane, j = s / CH;
                    const int c = (s % CH) ^ (which ? C::v_swizzle(j) : C::k_swizzle(j));
                    T x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = j < left && c * 8 < D ? from[j * stride + c * 8 + e] : (T)0.0f;
                    __builtin_memcpy(to + s * 16, x, 16);
                }
            }
        }
    };
    __attribute__((address_space(3))) volatile int *odd_seen = (__attribute__((address_space(3))) volatile int *)(lds_ptr)(lds + C::kLds - 16);
    if (tid < 2) odd_seen[tid] = 0;
    if (first_tile < tiles) load_tile(first_tile, first_tile & 1);

    // ---- Q^T's operand: 8 elements of the lane's row per step ----
    u4 q[DP / 16];
    {
        const T *from = (const T *)a.q.data + (q_first + query) * a.q.token_stride + qhead * a.q.head_stride;
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            const int d = 16 * s + 8 * half;
            const T *at = from + (d < D ? d : 0);
            if constexpr (VEC) {
                q[s] = *(const u4 *)at;
            } else {
                T x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = at[e];
                __builtin_memcpy(&q[s], x, 16);
            }
            q[s] = d < D ? q[s] ^ a.q_xor : (u4)(0u);
        }
    }

    // ---- LDS places of the operands: a row's and, apart because of the swizzle, a chunk's ----
    const int v_token = 4 * half + ((lane & 15) >> 2);           // of 8 or 16: the transposing read's lanes give 4 elements of a key each
    const int k_row = (key0 + col) * DP * 2, v_row = C::kTile + (key0 + v_token) * DP * 2 + (lane & 1) * 8;
    int k_chunk = (half ^ C::k_swizzle(col)) * 16;
    int v_chunk = ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ C::v_swizzle(v_token)) * 16;

    f16v o[DP / 32];
#pragma unroll
    for (int t = 0; t < DP / 32; ++t) o[t] = (f16v)(0.0f);
    // m: what the weights are relative to, in units of the scores; no less than a number whose product with the scale is finite
    float m = -3.0e38f / fmaxf(a.scale, 1.0f), l = 0.0f;

    bool odd = false;
    for (int tile = first_tile; tile < tiles; ++tile) {
        const int stage = tile & 1;
        copies_landed();
        __syncthreads();
        if (tile + 1 < tiles) load_tile(tile + 1, stage ^ 1);
        const uint8_t *at = lds + stage * C::kStage;
        // (not known to stay the same: one instruction per read is cheaper than the registers of all places)
        asm volatile("" : "+v"(k_chunk), "+v"(v_chunk));
        const bool masked = tile * BN + BN - 1 > group_seen_by_all;          // for some row of the workgroup
        if (masked) {                            // a value that some row does not see must not reach it through 0 * infinity
            uint32_t most = 0;
            for (int i = 0; i < C::LOADS; ++i) {
                const u4 x = *(const u4 *)(at + C::kTile + ((i * NW + wave) * 64 + lane) * 16) & 0x7fff7fffu;
                most = max_u16(most, max_u16(max_u16(x[0], x[1]), max_u16(x[2], x[3])));
            }
            if ((most & 0xffff) >= E::kInfinityBits || (most >> 16) >= E::kInfinityBits) odd_seen[tile & 1] = 1;
            if (tid == 0) odd_seen[~tile & 1] = 0;       // read before this tile's first barrier, written behind the next tile's
            __syncthreads();
            odd = __builtin_amdgcn_readfirstlane(odd_seen[tile & 1]) != 0;
            if (odd) break;
        }
        if (tile * BN + key0 > seen_by_any) continue;
        // operands are read a group ahead of the products that take them
        f16v s[KT];
        {
            constexpr int STEPS = DP / 16, ALL = KT * STEPS, N = C::AHEAD;
            u4 ahead[2][N];
            auto read = [&](int group) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = (group * N + i) / STEPS, u = (group * N + i) % STEPS;
                    ahead[group & 1][i] = *(const u4 *)(at + k_row + (k_chunk ^ 32 * u) + t * 32 * DP * 2);
                }
            };
            read(0);
#pragma unroll
            for (int group = 0; group < ALL / N; ++group) {
                if (group + 1 < ALL / N) read(group + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = (group * N + i) / STEPS, u = (group * N + i) % STEPS;
                    s[t] = mfma32(E{}, ahead[group & 1][i], q[u], u == 0 ? (f16v)(0.0f) : s[t]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (tile * BN + key0 + 32 * KT - 1 > seen_by_all) {
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (tile * BN + key0 + 32 * t + 8 * (i / 4) + 4 * half + i % 4 > seen) s[t][i] = -__builtin_inff();
        }
        float most = m;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[t][i]);
        most = max_of_halves(most);
        if (__any((most - m) * a.scale > weight_slack<E>())) {   // most tiles leave the sums as they are
            const float fall = __builtin_amdgcn_exp2f((m - most) * a.scale);
            l *= fall;
#pragma unroll
            for (int t = 0; t < DP / 32; ++t) o[t] *= fall;
            m = most;
        }
        const float ms = m * a.scale - weight_bits<E>();
        u4 p[2 * KT];
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], a.scale, -ms));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i + 1], a.scale, -ms));
                l += x + y;
                p[2 * t + i / 8][(i % 8) / 2] = pack2<E>(x, y);
            }
        auto v_operand = [&](int t, int u) {
            const uint8_t *from = at + v_row + (v_chunk ^ 64 * t) + u * 16 * DP * 2;
            const u2 v0 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)from));
            const u2 v1 = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(from + 8 * DP * 2)));
            return (u4){v0[0], v0[1], v1[0], v1[1]};
        };
        {
            constexpr int STEPS = DP / 32, ALL = 2 * KT * STEPS, N = C::V_AHEAD;
            u4 ahead[2][N];
            auto read = [&](int group) {
#pragma unroll
                for (int i = 0; i < N; ++i) ahead[group & 1][i] = v_operand((group * N + i) % STEPS, (group * N + i) / STEPS);
            };
            read(0);
#pragma unroll
            for (int group = 0; group < ALL / N; ++group) {
                if (group + 1 < ALL / N) read(group + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int t = (group * N + i) % STEPS, u = (group * N + i) / STEPS;
                    o[t] = mfma32(E{}, ahead[group & 1][i], p[u], o[t]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    f4 *const part = parts > 1 ? a.parts + (int64_t)blockIdx.x * C::kPart : nullptr;
    if (odd) {
        copies_landed();
        __syncthreads();
        prompt_rows_one_by_one<E, C>(a, tile_of, head, first_tile * BN, tiles * BN, part, lds);
        return;
    }
    l = sum_of_halves(l);
    if constexpr (C::KS == 2) {                          // the two wavefronts of a row group, through LDS
        f4 *const there = (f4 *)lds + row_group * 64 + lane;
        copies_landed();
        __syncthreads();
        if (wave >= C::RW) {
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    there[(4 * t + i) * C::BM * 2] = (f4){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
            there[DP / 8 * C::BM * 2] = (f4){m, l, 0.0f, 0.0f};
        }
        __syncthreads();
        if (wave >= C::RW) return;
        const f4 other = there[DP / 8 * C::BM * 2];
        const float top = fmaxf(m, other[0]), mine = __builtin_amdgcn_exp2f((m - top) * a.scale), its = __builtin_amdgcn_exp2f((other[0] - top) * a.scale);
        l = l * mine + other[1] * its;
        m = top;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f4 x = there[(4 * t + i) * C::BM * 2];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[t][4 * i + e] = o[t][4 * i + e] * mine + x[e] * its;
            }
    }
    if (parts > 1) {
        f4 *mine = part + tid;
#pragma unroll
        for (int t = 0; t < DP / 32; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(4 * t + i) * C::BM * 2] = (f4){o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
        mine[DP / 8 * C::BM * 2] = (f4){m, l, 0.0f, 0.0f};
        return;
    }

    // ---- O = O^T / l: 4 consecutive elements per lane and quarter, exchanged between lane halves to 8 ----
    const float by = seen < 0 ? 0.0f : 1.0f / l;
    T *out = (T *)a.o.data + (q_first + query) * a.o.token_stride + qhead * a.o.head_stride;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; i += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = seen < 0 ? 0.0f : o[t][i + e] * by;
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

// The parts of a tile, joined in their order: a workgroup per tile and piece of 4 elements of a lane.  Bound by reading the parts: 34 MB
// (252 of 128 rows of 256 elements) 10.2 us, 3.3 TB/s.
template <class E, class C, bool VEC>
__global__ __launch_bounds__(C::BM * 2) void attention_prompt_join_kernel(const PromptArgs a)
{
    typedef typename E::T T;
    constexpr int THREADS = C::BM * 2, PIECES = C::DP / 8;
    const int piece = blockIdx.x % PIECES, head = blockIdx.x / PIECES % a.kv_heads;
    const PromptTile<C> tile(a, blockIdx.x / PIECES / a.kv_heads, Index<1>{});
    const int tid = threadIdx.x, lane = tid & 63, row = tile.row0 + 32 * (tid >> 6) + (lane & 31);
    const int d = 8 * piece + 4 * (lane >> 5);                   // 32 (piece / 4) + 8 (piece % 4) + ..
    if (!tile.there || tile.parts <= 1 || row >= tile.rows || d >= a.head_dim) return;
    const f4 *from = a.parts + ((int64_t)tile.part0 * a.kv_heads + head) * C::kPart + tid;
    float top = -3.0e38f, l = 0.0f;
    f4 o = (f4)(0.0f);
    for (int p0 = 0; p0 < tile.parts; p0 += 8) {                 // eight on their way together
        f4 stats[8], x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f4 *part = from + (int64_t)min(p0 + i, tile.parts - 1) * a.kv_heads * C::kPart;
            stats[i] = part[PIECES * THREADS];
            x[i] = part[piece * THREADS];
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < 8; ++i) now = fmaxf(now, stats[i][0]);
        const float fall = __builtin_amdgcn_exp2f((top - now) * a.scale);
        l *= fall;
        o *= fall;
        top = now;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float by = p0 + i < tile.parts ? __builtin_amdgcn_exp2f((stats[i][0] - top) * a.scale) : 0.0f;
            l += p0 + i < tile.parts ? stats[i][1] * by : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += p0 + i < tile.parts ? x[i][e] * by : 0.0f;
        }
    }
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = tile.last_seen(row) < 0 ? 0.0f : o[e] / l;
    T *out = (T *)a.o.data + (tile.q_first + row / tile.group) * a.o.token_stride + (head * tile.group + row % tile.group) * a.o.head_stride;
    store<E, 4, VEC>(out + d, x);
}

}  // namespace ngemm
