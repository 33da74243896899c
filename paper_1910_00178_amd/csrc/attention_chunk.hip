// Host side of ngemm_attention_chunk of include/ngemm.h: argument validation and launches.
#include "attention_host.h"
#include "attention_chunk.h"

#include <algorithm>
#include <cmath>

using namespace ngemm;

namespace {

constexpr int64_t kUnits = 256;
constexpr float kLog2E = 1.44269504f;
constexpr int kWideFew = 192;                                    // heads that leave registers for eight wavefronts
constexpr int64_t kFewRows = 64;                                 // of a sequence, that attention_chunk_few_kernel takes at most, in tiles of 16 or 32

// f(ChunkCfg<...>{}) for the smallest DP that holds head_dim.  `wide`: 256 rows a workgroup where there are registers for it.
template <class F>
void with_chunk_form(int64_t head_dim, bool wide, F &&f)
{
    if (head_dim <= 64) wide ? f(ChunkCfg<64, 8, 2>{}) : f(ChunkCfg<64, 4, 2>{});
    else if (head_dim <= 96) wide ? f(ChunkCfg<96, 8, 2>{}) : f(ChunkCfg<96, 4, 2>{});
    else if (head_dim <= 128) wide ? f(ChunkCfg<128, 8, 2>{}) : f(ChunkCfg<128, 4, 2>{});
    else if (head_dim <= 192) f(ChunkCfg<192, 4, 1>{});
    else f(ChunkCfg<256, 4, 1>{});
}
int64_t tile_rows(int64_t head_dim, bool wide) { return wide && head_dim <= 128 ? 256 : 128; }

// Tiles of keys that `queries` consecutive tokens of a sequence see at most.
int64_t most_tiles(int64_t queries, int64_t max_length, int64_t window, int64_t sinks)
{
    const int64_t all = (max_length + kChunkKeys - 1) / kChunkKeys;
    if (window == 0) return all;
    return std::min(all, (window + queries + kChunkKeys - 3) / kChunkKeys + 1 + (std::min(sinks, max_length) + kChunkKeys - 1) / kChunkKeys);
}

struct ChunkCut {
    int64_t few_rows = 0, few_slots = 0, slots = 0;              // 0: no sequence can have so few, or more
    int64_t few_places = 0, places = 0, few_waves = 4;           // places 0: keys are not shared out
    bool wide = false;
    size_t few_bytes = 0, bytes = 0;
};
ChunkCut chunk_cut(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t tokens, int64_t max_new, int64_t max_length,
                   int64_t window, int64_t sinks)
{
    ChunkCut cut;
    const int64_t group = q_heads / kv_heads, most_new = std::min(max_new, tokens), most_rows = most_new * group;
    // Sequences of up to 64 rows on attention_chunk_few_kernel (heads of 128, 32 on 8; us).  Up to 16 rows always: it reads a key once where a tile of 128 rows
    // would convert it into LDS for them (16 x 4 tokens behind 1000: 15 for 31).  Up to 64 where their tiles of 32 fit the device together: 16 x 16 tokens behind 1000
    // 28 for 33, 32 x 8 31 for 43; but 64 x 16 behind 500, four rounds of tiles, 66 for 42.  Among longer ones those of up to 16 alone (16 x 20 behind 1000: 35, with tiles
    // of 32 for those of up to 64 rows 39).
    const int64_t tall = (most_rows + 31) / 32;                  // tiles of 32 of a sequence
    if (most_rows > 16 && most_rows <= kFewRows && batch * tall * kv_heads <= (head_dim <= 64 ? 2 * kUnits : kUnits)) cut.few_rows = 32 * tall;
    else if (most_rows <= 16 || (group <= 16 && batch > 1)) cut.few_rows = 16;
    if (cut.few_rows > 0) {
        const int64_t height = std::min<int64_t>(cut.few_rows, 32);
        cut.few_slots = batch * (cut.few_rows / height);
        const int64_t grid = cut.few_slots * kv_heads;
        // A tile's keys by eight wavefronts of one workgroup where that fills half of the units at least: 16 x 4 tokens behind 1000 14.5, shared out and joined 19.5;
        // 32 x 4 behind 8000 97 and 107 (16 x 4 behind 8000 57 and 51).  By four of one workgroup from two workgroups a unit on: 64 x 4 behind 1000 26.5 (by eight 32),
        // 256 x 4 behind 500 52 (82).  Else shared out over workgroups: 8 x 4 behind 8000 34 (whole 54).
        // (By the sizes alone, as lengths of one kind want it: where one sequence is much longer than the others it bounds a call whose keys are whole.  Single tokens behind 300 and
        // one behind 32768: 15 sequences, shared out, 32; 16, by eight wavefronts, 190; 64, by four, 229.)
        if (grid >= kUnits / 2 && grid < 2 * kUnits && cut.few_rows <= 16 && head_dim <= kWideFew) cut.few_waves = 8;
        else if (grid < 2 * kUnits && batch <= kMostShared && most_tiles(std::min(most_new, height / group + 2), max_length, window, sinks) >= 2 * kLeastTiles) {
            cut.few_places = std::max(height / 16 * head_dim <= 128 ? 2 * kUnits : kUnits, kv_heads);
            cut.few_slots += 2 * cut.few_places / kv_heads + 4;             // (and for rounding)
            cut.few_bytes = (size_t)(cut.few_slots * kv_heads * height * (head_dim / 4 + 1) * 16);
        }
    }
    if (most_rows > cut.few_rows) {
        // 256 rows a workgroup convert a key once where two of 128 do it twice, but leave coarser pieces of work: prompts of 4096 155 us (128 rows: 169), 16 x 256 behind
        // 2000 166 (177), 512 behind 16000 111 (120); a prompt of 2048 65 (57), 64 x 256 135 (120), 64 x 512 309 (293).
        // Windows are alike, by what a row sees: of 10000 tokens, window 4096 572 (600), 1000 230 (228), 256 122 (117); 4 x 2500, window 1000 208 (199), 256 117 (110); f16 the same to 2 %.
        // Not so where keys are shared out: 2000 tokens, window 1000 49 (56), 512 35 (44).
        // (Heads of 128; those of 64 are faster with 128 rows beyond 1024 too: 4 x 2500 of 12 heads 118 (94), 10000 255 (247).)
        const int64_t seen = window > 0 ? std::min(max_length, window + sinks) : max_length - std::min(max_length, most_new) / 2;       // by a row, about
        cut.wide = tokens * group / batch >= 256 && seen > 1024;
        const int64_t height = tile_rows(head_dim, cut.wide), places = cut.wide || head_dim > 128 ? kUnits : 2 * kUnits;
        cut.slots = tokens * group / height + batch;
        const int64_t grid = std::max(batch, (tokens * group + height - 1) / height) * kv_heads;
        if (batch <= kMostShared && grid < places && most_tiles(std::min(most_new, height / group + 2), max_length, window, sinks) >= 2 * kLeastTiles) {
            cut.places = places;
            cut.slots += 2 * cut.places / kv_heads + 4;
            with_chunk_form(head_dim, cut.wide, [&](auto form) { cut.bytes = (size_t)(cut.slots * kv_heads) * decltype(form)::kPart * 16; });
        }
    }
    return cut;
}

bool sizes_ok(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t tokens, int64_t max_new, int64_t max_length, int64_t window,
              int64_t sinks)
{
    return batch >= 0 && batch <= kMaxCount && q_heads >= 1 && q_heads <= 65536 && kv_heads >= 1 && q_heads % kv_heads == 0 && head_dim_ok(head_dim) &&
           tokens >= 0 && tokens <= kMaxCount && (tokens + 256 * batch) * q_heads <= kMaxCount && max_new >= 0 && max_new <= kMaxCount && max_length >= 0 &&
           max_length <= kMaxLength && window >= 0 && window <= kMaxLength && sinks >= 0 && sinks <= kMaxLength;
}

template <class E, int D, int R, int NW> struct FewForm {};
template <class E, int D, int R, int NW>
bool launch_few(const ChunkArgs &a, int device, hipStream_t st)
{
    const auto lds = [](int rows) constexpr { return NW * (2 * 16 * R + rows * D) * 4; };
    if (!allow_lds<FewForm<E, D, R, NW>, lds(16 * R)>(device, attention_chunk_few_kernel<E, D, R, NW>)) return false;
    const int most = (int)std::min<int64_t>(16 * R, (int64_t)std::min(a.max_new, a.tokens) * (a.q_heads / a.cache.kv_heads));
    hipLaunchKernelGGL((attention_chunk_few_kernel<E, D, R, NW>), dim3((unsigned)(a.slots * a.cache.kv_heads)), dim3(NW * 64), (size_t)lds(most), st, a);
    if (a.share > 0.0f) {
        // as many rows a workgroup as leave a group of lanes no more than some 8 parts in turn, by the places that a sequence has on average
        const int lanes = kFewJoinThreads / (D / 4);
        int rows_each = 1;
        const int64_t tiles = (int64_t)a.batch * ((a.few_rows + 16 * R - 1) / (16 * R));
        while (rows_each * 2 <= std::min(lanes, 16 * R) && a.slots * rows_each <= tiles * lanes * 2) rows_each *= 2;
        const int blocks = (most + rows_each - 1) / rows_each;
        hipLaunchKernelGGL((attention_chunk_few_join_kernel<E, D, R>), dim3((unsigned)(tiles * a.cache.kv_heads * blocks)), dim3(kFewJoinThreads), 0, st, a,
                           rows_each, blocks);
    }
    return true;
}

template <class E, class C, bool VEC> struct ManyForm {};
template <class E, class C, bool VEC>
bool launch_many(const ChunkArgs &a, int device, hipStream_t st)
{
    if (!allow_lds<ManyForm<E, C, VEC>, C::kLds>(device, attention_chunk_kernel<E, C, VEC>)) return false;
    hipLaunchKernelGGL((attention_chunk_kernel<E, C, VEC>), dim3((unsigned)(a.slots * a.cache.kv_heads)), dim3(C::NW * 64), C::kLds, st, a);
    if (a.share > 0.0f) {
        // as many pieces a workgroup as leave some thousands of them: tiles that were not shared out cost little then
        const int64_t tiles = ((int64_t)a.tokens * (a.q_heads / a.cache.kv_heads) / C::BM + a.batch) * a.cache.kv_heads;
        int blocks = C::DP / 8;
        while (blocks % 2 == 0 && tiles * blocks > 2048) blocks /= 2;
        hipLaunchKernelGGL((attention_chunk_join_kernel<E, C>), dim3((unsigned)(tiles * blocks)), dim3(C::NW * 64), 0, st, a, blocks);
    }
    return true;
}

template <class E>
bool launch_chunk(ChunkArgs a, const ChunkCut &cut, bool vec, uint8_t *workspace, int device, hipStream_t st)
{
    bool ok = true;
    a.few_rows = (int32_t)cut.few_rows;
    if (cut.slots > 0) {
        a.slots = (int32_t)cut.slots, a.share = (float)cut.places / (float)a.cache.kv_heads, a.part_data = (f4 *)workspace;
        with_chunk_form(a.cache.head_dim, cut.wide, [&](auto form) {
            typedef decltype(form) C;
            ok = vec ? launch_many<E, C, true>(a, device, st) : launch_many<E, C, false>(a, device, st);
        });
    }
    if (cut.few_rows > 0 && ok) {
        a.slots = (int32_t)cut.few_slots, a.share = (float)cut.few_places / (float)a.cache.kv_heads, a.part_data = (f4 *)(workspace + cut.bytes);
        with_head_dim(a.cache.head_dim, [&](auto dim) {
            constexpr int D = decltype(dim)::value;
            if constexpr (D <= kWideFew) {
                if (cut.few_waves == 8) {
                    ok = launch_few<E, D, 1, 8>(a, device, st);
                    return;
                }
            }
            ok = cut.few_rows <= 16 ? launch_few<E, D, 1, 4>(a, device, st) : launch_few<E, D, 2, 4>(a, device, st);
        });
    }
    return ok;
}

}  // namespace

extern "C" {

size_t ngemm_attention_chunk_workspace_bytes(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t tokens, int64_t max_new,
                                             int64_t max_length, int64_t window, int64_t sinks)
{
    if (!sizes_ok(batch, q_heads, kv_heads, head_dim, tokens, max_new, max_length, window, sinks) || batch < 1 || tokens < 1 || max_new < 1) return 0;
    const ChunkCut cut = chunk_cut(batch, q_heads, kv_heads, head_dim, tokens, max_new, max_length, window, sinks);
    return cut.few_bytes + cut.bytes;
}

ngemm_status ngemm_attention_chunk(ngemm_ctx *ctx, const ngemm_kv_cache *cache, ngemm_type type, int64_t batch, int64_t q_heads, int64_t tokens,
                                   const void *Q_dev, int64_t q_token_stride, int64_t q_head_stride,
                                   const int32_t *offsets_dev, const int32_t *starts_dev, int64_t max_new, int64_t max_length,
                                   const int32_t *pages_dev, int64_t pages_stride, int64_t window, int64_t sinks, float scale,
                                   void *O_dev, int64_t o_token_stride, int64_t o_head_stride,
                                   void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!ctx_ok(ctx) || !cache_ok(cache) || cache->device != ctx->device) return NGEMM_ERR_INVALID_ARG;
    if ((type != NGEMM_F16 && type != NGEMM_BF16) || !std::isfinite(scale * kLog2E)) return NGEMM_ERR_INVALID_ARG;
    const int64_t kv_heads = cache->kv_heads, head_dim = cache->head_dim;
    if (!sizes_ok(batch, q_heads, kv_heads, head_dim, tokens, max_new, max_length, window, sinks) || pages_stride < 0 || pages_stride > kMaxCount)
        return NGEMM_ERR_BAD_SHAPE;
    if (tokens == 0 || max_new == 0) return NGEMM_OK;
    if (batch == 0) return NGEMM_ERR_BAD_SHAPE;
    if (!offsets_dev || (!pages_dev && max_length > 0)) return NGEMM_ERR_INVALID_ARG;
    const Rows q{const_cast<void *>(Q_dev), q_token_stride, q_head_stride}, o{O_dev, o_token_stride, o_head_stride};
    if (const ngemm_status s = check_rows(q, type, tokens, q_heads, head_dim, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_rows(o, type, tokens, q_heads, head_dim, true); s != NGEMM_OK) return s;
    const ChunkCut cut = chunk_cut(batch, q_heads, kv_heads, head_dim, tokens, max_new, max_length, window, sinks);
    if (std::max(cut.slots * kv_heads * (cut.places > 0 ? head_dim / 8 + 8 : 1), cut.few_slots * kv_heads * (cut.few_places > 0 ? cut.few_rows : 1)) > kMaxGroups)
        return NGEMM_ERR_BAD_SHAPE;
    const size_t need = cut.few_bytes + cut.bytes;
    if (need > 0 && !workspace_dev) return NGEMM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    if (need > 0 && ((uintptr_t)workspace_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const ChunkArgs a{view_of(cache, pages_dev, pages_stride), q, o, offsets_dev, starts_dev, (int32_t)batch, (int32_t)q_heads, (int32_t)tokens, (int32_t)max_new,
                      pages_stride > 0 ? (int32_t)max_length : 0, (int32_t)window, (int32_t)sinks, scale * kLog2E, 0, 0, 0.0f, nullptr, in_pieces(o, type)};
    const bool vec = in_pieces(q, type) && in_pieces(o, type);
    hipStream_t st = (hipStream_t)hip_stream;
    const bool ok = type == NGEMM_F16 ? launch_chunk<F16>(a, cut, vec, (uint8_t *)workspace_dev, ctx->device, st)
                                      : launch_chunk<BF16>(a, cut, vec, (uint8_t *)workspace_dev, ctx->device, st);
    return ok ? launched() : NGEMM_ERR_DEVICE;
}

}  // extern "C"
