// What the host sides of the cache, of attention and of the rotations share: checks of rows, the cache's descriptor, launches' helpers.
#pragma once
#include "ngemm.h"
#include "ngemm_host.h"
#include "attention_common.h"

#include <algorithm>
#include <atomic>

struct ngemm_kv_cache {
    uint32_t magic;
    int device;
    int64_t num_pages, page_tokens, kv_heads, head_dim;
    uint8_t *data;           // device, caller-owned
};

namespace ngemm {

constexpr uint32_t kCacheMagic = 0x4e474b56u;   // "NGKV"
constexpr int64_t kMaxCount = 0x7fffffff - 4096;
constexpr int64_t kMaxLength = 1 << 30;         // tokens of a sequence in the cache
constexpr int64_t kMaxGroups = (1 << 23) - 1;   // workgroups of a launch: with 512 threads each, a launch counts threads in 32 bits
constexpr int64_t kMaxStride = 1ll << 40;       // elements
constexpr int64_t kMaxReach = 1ll << 60;        // elements from the first row's first to the last row's last: in bytes within 63 bits

inline bool cache_ok(const ngemm_kv_cache *c) { return c && c->magic == kCacheMagic; }

inline bool head_dim_ok(int64_t d) { return d >= 16 && d <= 256 && d % 16 == 0; }

inline int64_t elem_bytes(int type) { return type == NGEMM_F32 ? 4 : 2; }

// Rows that a call reads may overlap (a stride of 0 gives every token or head the same row).
inline ngemm_status check_rows(const Rows &r, int type, int64_t tokens, int64_t heads, int64_t head_dim, bool written)
{
    if (tokens == 0) return NGEMM_OK;
    if (!r.data || ((uintptr_t)r.data & (elem_bytes(type) - 1)) != 0) return NGEMM_ERR_INVALID_ARG;
    const __int128 t = r.token_stride, h = r.head_stride;
    if (t < 0 || h < 0 || t > kMaxStride || h > kMaxStride) return NGEMM_ERR_BAD_SHAPE;
    if ((tokens - 1) * t + (heads - 1) * h + head_dim > kMaxReach) return NGEMM_ERR_BAD_SHAPE;
    if (written) {                                       // no two elements at one place: heads inside tokens or tokens inside heads
        const bool heads_inside = (heads == 1 || h >= head_dim) && (tokens == 1 || t >= (heads - 1) * h + head_dim);
        const bool tokens_inside = (tokens == 1 || t >= head_dim) && (heads == 1 || h >= (tokens - 1) * t + head_dim);
        if (!heads_inside && !tokens_inside) return NGEMM_ERR_BAD_SHAPE;
    }
    return NGEMM_OK;
}

inline CacheView view_of(const ngemm_kv_cache *c, const int32_t *pages, int64_t pages_stride)
{
    return CacheView{c->data, pages, pages_stride, (int32_t)c->num_pages, (int32_t)c->kv_heads, (int32_t)c->head_dim,
                     (int32_t)(c->page_tokens / kBlockTokens)};
}

inline ngemm_status launched() { return hipGetLastError() == hipSuccess ? NGEMM_OK : NGEMM_ERR_DEVICE; }

// Whether 16-byte pieces of rows lie at 16-byte multiples.
inline bool in_pieces(const Rows &r, int type)
{
    const int64_t pieces = 16 / elem_bytes(type);
    return ((uintptr_t)r.data & 15u) == 0 && r.token_stride % pieces == 0 && r.head_stride % pieces == 0;
}

// What a call that moves rows of K and V to or from the cache launches: heads of a workgroup, workgroups (0: nothing to do).
struct MovePlan {
    int32_t heads = 0;
    int64_t groups = 0, slots = 0;                       // slots: workgroups of a head
};
inline ngemm_status plan_move(MovePlan &plan, const ngemm_ctx *ctx, const ngemm_kv_cache *cache, int type, int64_t batch, int64_t tokens, const Rows &k,
                              const Rows &v, const int32_t *offsets, const int32_t *pages, int64_t pages_stride, bool written)
{
    if (!ctx_ok(ctx) || !cache_ok(cache) || cache->device != ctx->device) return NGEMM_ERR_INVALID_ARG;
    if (type != NGEMM_F32 && type != NGEMM_F16 && type != NGEMM_BF16) return NGEMM_ERR_INVALID_ARG;
    if (batch < 0 || tokens < 0 || batch > kMaxCount || tokens > kMaxCount || pages_stride < 0 || pages_stride > kMaxCount) return NGEMM_ERR_BAD_SHAPE;
    if (tokens == 0) return NGEMM_OK;
    if (batch == 0) return NGEMM_ERR_BAD_SHAPE;
    if (!offsets || !pages) return NGEMM_ERR_INVALID_ARG;
    for (const Rows &r : {k, v})
        if (const ngemm_status s = check_rows(r, type, tokens, cache->kv_heads, cache->head_dim, written); s != NGEMM_OK) return s;
    // heads of a workgroup: two of them share finding the place where that leaves some thousands of workgroups (40000 tokens of 8 heads
    // read: 53 us with two, 58 with one, 55 with four; 1700 workgroups of one head or 850 of two the same, fewer are slower)
    const int64_t slots = move_slots(tokens, batch);
    if (slots * cache->kv_heads > kMaxCount || slots * 16 > kMaxCount) return NGEMM_ERR_BAD_SHAPE;
    const int64_t heads = std::min<int64_t>(cache->kv_heads, std::max<int64_t>(slots * cache->kv_heads >= 4096 ? 2 : 1, slots * cache->kv_heads / kMaxGroups + 1));
    const int64_t groups = slots * ((cache->kv_heads + heads - 1) / heads);
    if (groups > kMaxGroups) return NGEMM_ERR_BAD_SHAPE;
    plan = MovePlan{(int32_t)heads, groups, slots};
    return NGEMM_OK;
}

// LDS beyond 64 KiB is asked for once per kernel and device, before its first launch: programs that only multiply pay nothing for it.
template <class KERNEL, int BYTES, class F>
bool allow_lds(int device, F kernel)
{
    if constexpr (BYTES <= 65536) return true;
    static std::atomic<uint64_t> allowed{0};             // devices; others ask each time
    const uint64_t mine = device < 64 ? 1ull << device : 0;
    if (allowed.load(std::memory_order_acquire) & mine) return true;
    if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, BYTES) != hipSuccess) return false;
    allowed.fetch_or(mine, std::memory_order_release);
    return true;
}

// f(Index<head_dim>{})
template <int D = 256, class F>
void with_head_dim(int64_t head_dim, F &&f)
{
    if (head_dim == D) f(Index<D>{});
    else if constexpr (D > 16) with_head_dim<D - 16>(head_dim, f);
}

}  // namespace ngemm
