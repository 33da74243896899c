// Host side of the key-value cache and the attention calls of include/ngemm.h: argument validation and launches.
#include "attention_host.h"
#include "attention_decode.h"
#include "attention_prompt.h"

#include <algorithm>
#include <cmath>
#include <new>

using namespace ngemm;

namespace {

template <class E, int LANES, int N>
void launch_move_form(bool write, bool vec, unsigned groups, hipStream_t st, const MoveArgs &a)
{
    const dim3 grid(groups), block(16 * LANES);
    if (write && vec) hipLaunchKernelGGL((kv_write_kernel<E, LANES, N, true>), grid, block, 0, st, a);
    else if (write) hipLaunchKernelGGL((kv_write_kernel<E, LANES, N, false>), grid, block, 0, st, a);
    else if (vec) hipLaunchKernelGGL((kv_read_kernel<E, LANES, N, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((kv_read_kernel<E, LANES, N, false>), grid, block, 0, st, a);
}

template <class E>
void launch_move(bool write, bool vec, unsigned groups, hipStream_t st, const MoveArgs &a)
{
    if (a.cache.head_dim <= 64) launch_move_form<E, 8, 1>(write, vec, groups, st, a);
    else if (a.cache.head_dim <= 128) launch_move_form<E, 16, 1>(write, vec, groups, st, a);
    else launch_move_form<E, 16, 2>(write, vec, groups, st, a);
}

ngemm_status move_rows(bool write, ngemm_ctx *ctx, const ngemm_kv_cache *cache, int type, int64_t batch, int64_t tokens, Rows k, Rows v,
                       const int32_t *offsets, const int32_t *starts, const int32_t *pages, int64_t pages_stride, void *stream)
{
    MovePlan plan;
    if (const ngemm_status s = plan_move(plan, ctx, cache, type, batch, tokens, k, v, offsets, pages, pages_stride, !write); s != NGEMM_OK) return s;
    if (plan.groups == 0) return NGEMM_OK;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const MoveArgs a{view_of(cache, pages, pages_stride), k, v, offsets, starts, (int32_t)batch, (int32_t)tokens, plan.heads};
    const bool vec = in_pieces(k, type) && in_pieces(v, type);
    hipStream_t st = (hipStream_t)stream;
    if (type == NGEMM_F32) launch_move<F32>(write, vec, (unsigned)plan.groups, st, a);
    else if (type == NGEMM_F16) launch_move<F16>(write, vec, (unsigned)plan.groups, st, a);
    else launch_move<BF16>(write, vec, (unsigned)plan.groups, st, a);
    return launched();
}

// ---- one token per sequence ----

// How a sequence is cut.  Whole, by eight wavefronts, where the sequences and heads give half of the units a workgroup and no wavefront takes more than
// four tiles: the join, a launch more, mostly costs more than the split gains (calls back to back: 32 sequences of up to 1000 tokens, 12 heads of 64: 9.5 us whole,
// 12.0 in chunks; 16 of 2000, 8 K/V heads of 128: 16.7 and 17.7; 64 of 2000, 8 K/V heads of 64: 29.5 and 29.0; but 64 of 500, 8 of 128: 17.6 and 14.1; heads
// of more than 192 have no registers for it).  Else in chunks, by four wavefronts: as many as give every unit two workgroups, of 256 to 4096 tokens (8
// sequences of 100000 to 131072 tokens: 365 us, with half as long ones 374, with 1024 tokens 387, with 512 409; 16 of 8192 with heads of
// 256: 60 us, with half as long ones 66; only 64 sequences of very different lengths would rather have 1024 tokens: 71 us for 76).  The cut follows max_length, not
// the lengths, which the host does not know: one sequence of 4097 tokens takes 9.9 us where max_length says so and 23 where it says 131072.
constexpr int64_t kUnits = 256;
constexpr int kWideHeadDim = 192;

struct DecodeCut {
    int64_t waves, chunk, chunks;
    size_t bytes;
};
DecodeCut decode_cut(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_length)
{
    const int64_t group = q_heads / kv_heads, grid = batch * kv_heads * ((group + 15) / 16);
    if (grid >= kUnits / 2 && max_length > 256 && max_length <= 4 * 64 * 8 && head_dim <= kWideHeadDim)
        return DecodeCut{8, (max_length + 511) / 512 * 512, 1, 0};
    DecodeCut cut{4, std::min<int64_t>(std::max<int64_t>((max_length * grid / (2 * kUnits) + 255) / 256 * 256, 256), 4096), 1, 0};
    cut.chunks = std::max<int64_t>(1, (max_length + cut.chunk - 1) / cut.chunk);
    if (cut.chunks > 1) cut.bytes = (size_t)(batch * q_heads * cut.chunks * (head_dim / 4 + 1) * 16);
    return cut;
}

template <class E, int D, int NW> struct DecodeForm {};
template <class E, int D, int NW>
bool launch_decode_form(const DecodeArgs &a, int device, hipStream_t st)
{
    const int group = a.q_heads / a.cache.kv_heads;
    const unsigned grid = (unsigned)((int64_t)a.batch * a.cache.kv_heads * ((group + 15) / 16) * a.chunks);
    const auto lds = [](int heads) constexpr { return NW * (32 + heads * D) * 4; };
    if (!allow_lds<DecodeForm<E, D, NW>, lds(16)>(device, attention_decode_kernel<E, D, NW>)) return false;
    hipLaunchKernelGGL((attention_decode_kernel<E, D, NW>), dim3(grid), dim3(NW * 64), (size_t)lds(std::min(group, 16)), st, a);
    if (a.chunks > 1) hipLaunchKernelGGL((attention_decode_join_kernel<E, D>), dim3((unsigned)(a.batch * a.q_heads)), dim3(kJoinThreads), 0, st, a);
    return true;
}

template <class E>
bool launch_decode(const DecodeArgs &a, int64_t waves, int device, hipStream_t st)
{
    bool ok = false;
    with_head_dim(a.cache.head_dim, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if constexpr (D <= kWideHeadDim) {
            if (waves == 8) {
                ok = launch_decode_form<E, D, 8>(a, device, st);
                return;
            }
        }
        ok = launch_decode_form<E, D, 4>(a, device, st);
    });
    return ok;
}

// ---- prompts ----

constexpr int64_t kPromptRows = 128;            // of a tile in all forms

// f(PromptCfg<...>{}) for the smallest DP that holds head_dim.
template <class F>
void with_prompt_form(int64_t head_dim, F &&f)
{
    if (head_dim <= 64) f(PromptCfg<64, 4, 1, 64, 2>{});
    else if (head_dim <= 96) f(PromptCfg<96, 4, 1, 64, 2>{});
    else if (head_dim <= 128) f(PromptCfg<128, 4, 1, 64, 2>{});
    else if (head_dim <= 192) f(PromptCfg<192, 4, 2, 64, 1>{});
    else f(PromptCfg<256, 4, 2, 64, 1>{});
}

// Copies of 16-byte pieces, a tile's offsets within 31 bits.
bool rows_in_pieces(const Rows &r) { return in_pieces(r, NGEMM_BF16) && r.token_stride < (1 << 23); }

// Tiles of query rows that any lengths of the sequences can need; and where these are few and the mean context is long enough for the join (a launch
// more) to pay, the units that share out the keys, with the workgroups that this takes: a tile has as many parts as its share of the units,
// rounded down, but at least one.  Shares follow the lengths on the device: 8 rows behind 20000, 1500, 900, 500, 400 and 300 keys take 36 us, 88
// with equal shares for all; sequences of equal lengths the same either way.  Two workgroups a unit write twice the parts: 16 heads on one K/V head,
// 1144 rows, 40 us for 28; 8 rows behind 32768 keys 43 for 38; only 256 rows behind 8192 keys gain, 55 for 60.  Whether keys are split is
// decided by the mean: 8 rows behind 10000 keys take 24 us alone and 199 in a batch with 15 others behind 200 (8 K/V heads of 128).
struct PromptCut {
    int64_t tiles, slots, units;
    size_t bytes;
};
template <class C>
PromptCut prompt_cut(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t q_tokens, int64_t k_tokens)
{
    const int64_t rows = q_tokens * (q_heads / kv_heads), tiles = std::max<int64_t>(batch, (rows + C::BM - 1) / C::BM) * kv_heads;
    PromptCut cut{rows / C::BM + batch, rows / C::BM + batch, 0, 0};
    if (tiles > kUnits / 2 || k_tokens / batch < 4 * kLeastRun) return cut;
    static_assert(kUnits / 2 <= kMostSplit, "sequences");
    cut.units = kUnits;
    cut.slots += (cut.units + kv_heads - 1) / kv_heads + cut.tiles / 256 + 2;
    cut.bytes = (size_t)(cut.slots * kv_heads) * C::kPart * 16;
    return cut;
}

template <class E, class C, bool VEC> struct PromptForm {};
template <class E, class C, bool VEC>
bool launch_prompt_form(const PromptArgs &a, const PromptCut &cut, int device, hipStream_t st)
{
    if (!allow_lds<PromptForm<E, C, VEC>, C::kLds>(device, attention_prompt_kernel<E, C, VEC>)) return false;
    hipLaunchKernelGGL((attention_prompt_kernel<E, C, VEC>), dim3((unsigned)(cut.slots * a.kv_heads)), dim3(C::NW * 64), C::kLds, st, a);
    if (cut.units > 0)
        hipLaunchKernelGGL((attention_prompt_join_kernel<E, C, VEC>), dim3((unsigned)(cut.tiles * a.kv_heads * (C::DP / 8))), dim3(C::BM * 2), 0, st, a);
    return true;
}

template <class E>
bool launch_prompt(PromptArgs a, bool vec, void *workspace, int device, hipStream_t st)
{
    bool ok = false;
    with_prompt_form(a.head_dim, [&](auto form) {
        typedef decltype(form) C;
        static_assert(C::BM == kPromptRows, "one height of tiles");
        const PromptCut cut = prompt_cut<C>(a.batch, a.q_heads, a.kv_heads, a.q_tokens, a.k_tokens);
        a.slots = (int32_t)cut.slots;
        a.share = (float)cut.units / (float)a.kv_heads;
        a.parts = (f4 *)workspace;
        ok = vec ? launch_prompt_form<E, C, true>(a, cut, device, st) : launch_prompt_form<E, C, false>(a, cut, device, st);
    });
    return ok;
}

}  // namespace

extern "C" {

size_t ngemm_kv_cache_bytes(int64_t num_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim)
{
    if (num_pages < 1 || num_pages > kMaxCount || page_tokens < kBlockTokens || page_tokens > (1 << 24) || page_tokens % kBlockTokens ||
        kv_heads < 1 || kv_heads > 65536 || !head_dim_ok(head_dim))
        return 0;
    const __int128 blocks = (__int128)num_pages * kv_heads * (page_tokens / kBlockTokens);       // numbered in 31 bits
    return blocks <= kMaxCount ? (size_t)(blocks * (32 * head_dim + 8 * kBlockTokens)) : 0;
}

ngemm_status ngemm_kv_cache_create(ngemm_ctx *ctx, int64_t num_pages, int64_t page_tokens, int64_t kv_heads, int64_t head_dim,
                                   void *cache_dev, size_t cache_bytes, ngemm_kv_cache **out)
{
    if (!out) return NGEMM_ERR_INVALID_ARG;
    *out = nullptr;
    if (!ctx_ok(ctx)) return NGEMM_ERR_INVALID_ARG;
    const size_t need = ngemm_kv_cache_bytes(num_pages, page_tokens, kv_heads, head_dim);
    if (need == 0) return NGEMM_ERR_BAD_SHAPE;
    if (!cache_dev || ((uintptr_t)cache_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    if (cache_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    ngemm_kv_cache *c = new (std::nothrow) ngemm_kv_cache{kCacheMagic, ctx->device, num_pages, page_tokens, kv_heads, head_dim, (uint8_t *)cache_dev};
    if (!c) return NGEMM_ERR_DEVICE;
    *out = c;
    return NGEMM_OK;
}

ngemm_status ngemm_kv_cache_free(ngemm_kv_cache *cache)
{
    if (!cache) return NGEMM_OK;
    if (!cache_ok(cache)) return NGEMM_ERR_INVALID_ARG;
    cache->magic = 0;
    delete cache;
    return NGEMM_OK;
}

ngemm_status ngemm_kv_write(ngemm_ctx *ctx, const ngemm_kv_cache *cache, ngemm_type type, int64_t batch, int64_t tokens,
                            const void *K_dev, int64_t k_token_stride, int64_t k_head_stride,
                            const void *V_dev, int64_t v_token_stride, int64_t v_head_stride,
                            const int32_t *offsets_dev, const int32_t *starts_dev,
                            const int32_t *pages_dev, int64_t pages_stride, void *hip_stream)
{
    return move_rows(true, ctx, cache, type, batch, tokens, Rows{const_cast<void *>(K_dev), k_token_stride, k_head_stride},
                     Rows{const_cast<void *>(V_dev), v_token_stride, v_head_stride}, offsets_dev, starts_dev, pages_dev, pages_stride, hip_stream);
}

ngemm_status ngemm_kv_read(ngemm_ctx *ctx, const ngemm_kv_cache *cache, ngemm_type type, int64_t batch, int64_t tokens,
                           void *K_dev, int64_t k_token_stride, int64_t k_head_stride,
                           void *V_dev, int64_t v_token_stride, int64_t v_head_stride,
                           const int32_t *offsets_dev, const int32_t *starts_dev,
                           const int32_t *pages_dev, int64_t pages_stride, void *hip_stream)
{
    return move_rows(false, ctx, cache, type, batch, tokens, Rows{K_dev, k_token_stride, k_head_stride},
                     Rows{V_dev, v_token_stride, v_head_stride}, offsets_dev, starts_dev, pages_dev, pages_stride, hip_stream);
}

size_t ngemm_attention_decode_workspace_bytes(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim, int64_t max_length)
{
    if (batch < 1 || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || !head_dim_ok(head_dim) || max_length < 0 || max_length > kMaxLength ||
        batch > kMaxCount || q_heads > 65536 || batch * q_heads > kMaxCount)
        return 0;
    return decode_cut(batch, q_heads, kv_heads, head_dim, max_length).bytes;
}

ngemm_status ngemm_attention_decode(ngemm_ctx *ctx, const ngemm_kv_cache *cache, ngemm_type type, int64_t batch, int64_t q_heads,
                                    const void *Q_dev, int64_t q_token_stride, int64_t q_head_stride,
                                    const int32_t *lengths_dev, int64_t max_length,
                                    const int32_t *pages_dev, int64_t pages_stride, float scale,
                                    void *O_dev, int64_t o_token_stride, int64_t o_head_stride,
                                    void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!ctx_ok(ctx) || !cache_ok(cache) || cache->device != ctx->device) return NGEMM_ERR_INVALID_ARG;
    if ((type != NGEMM_F16 && type != NGEMM_BF16) || !std::isfinite(scale)) return NGEMM_ERR_INVALID_ARG;
    if (batch < 0 || batch > kMaxCount || q_heads < 1 || q_heads > 65536 || q_heads % cache->kv_heads || max_length < 0 || max_length > kMaxLength ||
        pages_stride < 0 || pages_stride > kMaxCount || batch * q_heads > kMaxCount)
        return NGEMM_ERR_BAD_SHAPE;
    if (batch == 0) return NGEMM_OK;
    if (!lengths_dev || (!pages_dev && max_length > 0)) return NGEMM_ERR_INVALID_ARG;
    const Rows q{const_cast<void *>(Q_dev), q_token_stride, q_head_stride}, o{O_dev, o_token_stride, o_head_stride};
    if (const ngemm_status s = check_rows(q, type, batch, q_heads, cache->head_dim, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_rows(o, type, batch, q_heads, cache->head_dim, true); s != NGEMM_OK) return s;
    const size_t need = ngemm_attention_decode_workspace_bytes(batch, q_heads, cache->kv_heads, cache->head_dim, max_length);
    if (need > 0 && !workspace_dev) return NGEMM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    if (need > 0 && ((uintptr_t)workspace_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const DecodeCut cut = decode_cut(batch, q_heads, cache->kv_heads, cache->head_dim, max_length);
    if (batch * q_heads * cut.chunks > kMaxGroups) return NGEMM_ERR_BAD_SHAPE;
    const DecodeArgs a{view_of(cache, pages_dev, pages_stride), q, o, lengths_dev, (int32_t)batch, (int32_t)q_heads, (int32_t)max_length,
                       (int32_t)cut.chunk, (int32_t)cut.chunks, scale * 1.44269504f, (f4 *)workspace_dev, in_pieces(o, type)};
    hipStream_t st = (hipStream_t)hip_stream;
    const bool ok = type == NGEMM_F16 ? launch_decode<F16>(a, cut.waves, ctx->device, st) : launch_decode<BF16>(a, cut.waves, ctx->device, st);
    return ok ? launched() : NGEMM_ERR_DEVICE;
}

size_t ngemm_attention_prompt_workspace_bytes(int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                                              int64_t q_tokens, int64_t k_tokens)
{
    if (batch < 1 || q_heads < 1 || q_heads > 65536 || kv_heads < 1 || q_heads % kv_heads || !head_dim_ok(head_dim) || q_tokens < 1 || k_tokens < 0 ||
        batch > kMaxCount || q_tokens > kMaxCount || k_tokens > kMaxCount || (q_tokens + 128 * batch) * q_heads > kMaxCount)
        return 0;
    size_t bytes = 0;
    with_prompt_form(head_dim, [&](auto form) {
        bytes = prompt_cut<decltype(form)>(batch, q_heads, kv_heads, q_tokens, k_tokens).bytes;
    });
    return bytes;
}

ngemm_status ngemm_attention_prompt(ngemm_ctx *ctx, ngemm_type type, int64_t batch, int64_t q_heads, int64_t kv_heads, int64_t head_dim,
                                    int64_t q_tokens, const void *Q_dev, int64_t q_token_stride, int64_t q_head_stride,
                                    int64_t k_tokens, const void *K_dev, int64_t k_token_stride, int64_t k_head_stride,
                                    const void *V_dev, int64_t v_token_stride, int64_t v_head_stride,
                                    const int32_t *q_offsets_dev, const int32_t *k_offsets_dev, int causal, float scale,
                                    void *O_dev, int64_t o_token_stride, int64_t o_head_stride,
                                    void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!ctx_ok(ctx)) return NGEMM_ERR_INVALID_ARG;
    if ((type != NGEMM_F16 && type != NGEMM_BF16) || !std::isfinite(scale)) return NGEMM_ERR_INVALID_ARG;
    if (batch < 0 || batch > kMaxCount || q_heads < 1 || q_heads > 65536 || kv_heads < 1 || q_heads % kv_heads || !head_dim_ok(head_dim) || q_tokens < 0 ||
        k_tokens < 0 || q_tokens > kMaxCount || k_tokens > kMaxCount || (q_tokens + 128 * batch) * q_heads > kMaxCount)
        return NGEMM_ERR_BAD_SHAPE;
    if (q_tokens == 0) return NGEMM_OK;
    if (batch == 0 || (!k_offsets_dev && k_tokens != q_tokens)) return NGEMM_ERR_BAD_SHAPE;
    if ((q_tokens * (q_heads / kv_heads) / kPromptRows + batch) * kv_heads > kMaxGroups) return NGEMM_ERR_BAD_SHAPE;
    if (!q_offsets_dev) return NGEMM_ERR_INVALID_ARG;
    const Rows q{const_cast<void *>(Q_dev), q_token_stride, q_head_stride}, k{const_cast<void *>(K_dev), k_token_stride, k_head_stride},
        v{const_cast<void *>(V_dev), v_token_stride, v_head_stride}, o{O_dev, o_token_stride, o_head_stride};
    if (const ngemm_status s = check_rows(q, type, q_tokens, q_heads, head_dim, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_rows(k, type, k_tokens, kv_heads, head_dim, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_rows(v, type, k_tokens, kv_heads, head_dim, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_rows(o, type, q_tokens, q_heads, head_dim, true); s != NGEMM_OK) return s;
    const size_t need = ngemm_attention_prompt_workspace_bytes(batch, q_heads, kv_heads, head_dim, q_tokens, k_tokens);
    if (need > 0 && !workspace_dev) return NGEMM_ERR_INVALID_ARG;
    if (workspace_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    if (need > 0 && ((uintptr_t)workspace_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    // the kernel's scale is not negative (the sign goes to Q), and not 0 (hidden scores are minus infinity)
    const float scale2 = std::fmax(std::fabs(scale) * 1.44269504f, 1.17549435e-38f);
    const PromptArgs a{q, k, v, o, q_offsets_dev, k_offsets_dev ? k_offsets_dev : q_offsets_dev, (int32_t)batch, (int32_t)q_heads, (int32_t)kv_heads,
                       (int32_t)head_dim, (int32_t)q_tokens, (int32_t)k_tokens, causal != 0, scale2, std::signbit(scale) ? 0x80008000u : 0u, 0, 0, nullptr};
    const bool vec = rows_in_pieces(q) && rows_in_pieces(k) && rows_in_pieces(v) && rows_in_pieces(o);
    hipStream_t st = (hipStream_t)hip_stream;
    const bool ok = type == NGEMM_F16 ? launch_prompt<F16>(a, vec, workspace_dev, ctx->device, st) : launch_prompt<BF16>(a, vec, workspace_dev, ctx->device, st);
    return ok ? launched() : NGEMM_ERR_DEVICE;
}

}  // extern "C"
