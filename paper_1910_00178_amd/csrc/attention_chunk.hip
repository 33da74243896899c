// Host side of ngemm_attention_chunk of include/ngemm.h: argument validation and launches.
#include "attention_host.h"
#include "attention_chunk.h"

#include <algorithm>
#include <cmath>

using namespace ngemm;

namespace {

constexpr int64_t kUnits = 256;
// Rows of a sequence that attention_chunk_few_kernel takes at most: heads of more than 128 leave no registers for two tiles of 16.
constexpr int64_t few_rows_of(int64_t head_dim) { return head_dim <= 128 ? 32 : 16; }

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
    int64_t few_rows = 0;                                        // 0: no sequence can have so few
    int64_t few_run = 1, few_parts = 1, slots = 0, run = 1, parts = 1;           // slots 0: no sequence can have more
    bool wide = false;
    size_t few_bytes = 0, bytes = 0;
};
ChunkCut chunk_cut(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t tokens, int64_t max_new, int64_t max_length,
                   int64_t window, int64_t sinks)
{
    ChunkCut cut;
    const int64_t group = q_heads / kv_heads, most_new = std::min(max_new, tokens);
    const int64_t few = few_rows_of(head_dim);
    if (group <= few && (batch > 1 || most_new * group <= few)) {
        cut.few_rows = most_new * group <= 16 ? 16 : few;
        const int64_t tiles = std::max<int64_t>(1, most_tiles(std::min(most_new, cut.few_rows / group), max_length, window, sinks)), grid = batch * kv_heads;
        cut.few_run = std::max<int64_t>(std::min<int64_t>((tiles * grid / (2 * kUnits) + 3) / 4 * 4, 64), (tiles * grid / (32 * kUnits) + 4) / 4 * 4);
        cut.few_parts = (tiles + cut.few_run - 1) / cut.few_run;
        if (cut.few_parts > 1) cut.few_bytes = (size_t)(grid * cut.few_parts * cut.few_rows * (head_dim / 4 + 1) * 16);
    }
    if (most_new * group > cut.few_rows) {
        cut.wide = tokens * group / batch >= 256;
        const int64_t height = tile_rows(head_dim, cut.wide), places = cut.wide || head_dim > 128 ? kUnits : 2 * kUnits;
        cut.slots = tokens * group / height + batch;
        const int64_t tiles = std::max<int64_t>(1, most_tiles(std::min(most_new, height / group + 2), max_length, window, sinks));
        const int64_t grid = std::max(batch, (tokens * group + height - 1) / height) * kv_heads;
        cut.run = std::max<int64_t>((tiles * grid + places - 1) / places, 4);
        cut.parts = grid >= places ? 1 : (tiles + cut.run - 1) / cut.run;
        if (cut.parts == 1) cut.run = tiles;
        else
            with_chunk_form(head_dim, cut.wide, [&](auto form) { cut.bytes = (size_t)(cut.slots * kv_heads * cut.parts) * decltype(form)::kPart * 16; });
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

template <class E, int D, int R> struct FewForm {};
template <class E, int D, int R>
bool launch_few(const ChunkArgs &a, int device, hipStream_t st)
{
    const auto lds = [](int rows) constexpr { return kFewWaves * (2 * 16 * R + rows * D) * 4; };
    if (!allow_lds<FewForm<E, D, R>, lds(16 * R)>(device, attention_chunk_few_kernel<E, D, R>)) return false;
    const int most = (int)std::min<int64_t>(16 * R, (int64_t)std::min(a.max_new, a.tokens) * (a.q_heads / a.cache.kv_heads));
    const unsigned units = (unsigned)(a.batch * a.cache.kv_heads);
    hipLaunchKernelGGL((attention_chunk_few_kernel<E, D, R>), dim3(units * a.parts), dim3(kFewWaves * 64), (size_t)lds(most), st, a);
    if (a.parts > 1) hipLaunchKernelGGL((attention_chunk_few_join_kernel<E, D, R>), dim3(units * 16 * R), dim3(kFewJoinThreads), 0, st, a);
    return true;
}

template <class E, class C, bool VEC> struct ManyForm {};
template <class E, class C, bool VEC>
bool launch_many(const ChunkArgs &a, int device, hipStream_t st)
{
    if (!allow_lds<ManyForm<E, C, VEC>, C::kLds>(device, attention_chunk_kernel<E, C, VEC>)) return false;
    const unsigned units = (unsigned)(a.slots * a.cache.kv_heads);
    hipLaunchKernelGGL((attention_chunk_kernel<E, C, VEC>), dim3(units * a.parts), dim3(C::NW * 64), C::kLds, st, a);
    if (a.parts > 1) hipLaunchKernelGGL((attention_chunk_join_kernel<E, C>), dim3(units * (C::DP / 8)), dim3(C::NW * 64), 0, st, a);
    return true;
}

template <class E>
bool launch_chunk(ChunkArgs a, const ChunkCut &cut, bool vec, uint8_t *workspace, int device, hipStream_t st)
{
    bool ok = true;
    a.few_rows = (int32_t)cut.few_rows;
    if (cut.slots > 0) {
        a.run = (int32_t)cut.run, a.parts = (int32_t)cut.parts, a.slots = (int32_t)cut.slots, a.part_data = (f4 *)workspace;
        with_chunk_form(a.cache.head_dim, cut.wide, [&](auto form) {
            typedef decltype(form) C;
            ok = vec ? launch_many<E, C, true>(a, device, st) : launch_many<E, C, false>(a, device, st);
        });
    }
    if (cut.few_rows > 0 && ok) {
        a.run = (int32_t)cut.few_run, a.parts = (int32_t)cut.few_parts, a.part_data = (f4 *)(workspace + cut.bytes);
        with_head_dim(a.cache.head_dim, [&](auto dim) {
            constexpr int D = decltype(dim)::value;
            if constexpr (few_rows_of(D) > 16) {
                if (cut.few_rows > 16) {
                    ok = launch_few<E, D, 2>(a, device, st);
                    return;
                }
            }
            ok = launch_few<E, D, 1>(a, device, st);
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
    if ((type != NGEMM_F16 && type != NGEMM_BF16) || !std::isfinite(scale)) return NGEMM_ERR_INVALID_ARG;
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
    if (std::max(cut.slots * kv_heads * std::max(cut.parts, head_dim / 8 + 4), batch * kv_heads * std::max(cut.few_parts, cut.few_rows)) > kMaxGroups)
        return NGEMM_ERR_BAD_SHAPE;
    const size_t need = cut.few_bytes + cut.bytes;
    if (need > 0 && !workspace_dev) return NGEMM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    if (need > 0 && ((uintptr_t)workspace_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const ChunkArgs a{view_of(cache, pages_dev, pages_stride), q, o, offsets_dev, starts_dev, (int32_t)batch, (int32_t)q_heads, (int32_t)tokens, (int32_t)max_new,
                      pages_stride > 0 ? (int32_t)max_length : 0, (int32_t)window, (int32_t)sinks, scale * 1.44269504f, 0, 1, 1, 0, nullptr, in_pieces(o, type)};
    const bool vec = in_pieces(q, type) && in_pieces(o, type);
    hipStream_t st = (hipStream_t)hip_stream;
    const bool ok = type == NGEMM_F16 ? launch_chunk<F16>(a, cut, vec, (uint8_t *)workspace_dev, ctx->device, st)
                                      : launch_chunk<BF16>(a, cut, vec, (uint8_t *)workspace_dev, ctx->device, st);
    return ok ? launched() : NGEMM_ERR_DEVICE;
}

}  // extern "C"
