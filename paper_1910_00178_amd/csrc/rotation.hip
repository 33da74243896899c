// Host side of the norms and rotations of include/ngemm.h: argument validation and launches.
#include "attention_host.h"
#include "rotation.h"

#include <algorithm>
#include <cmath>
#include <new>

using namespace ngemm;

struct ngemm_rotation {
    uint32_t magic;
    int device, pairs;
    int64_t positions, dim;
    const float *table;      // device, caller-owned
};

namespace {

constexpr uint32_t kRotationMagic = 0x4e47524fu;   // "NGRO"

bool rotation_ok(const ngemm_rotation *r) { return r && r->magic == kRotationMagic; }

RotationView view_of(const ngemm_rotation *r)
{
    return r ? RotationView{r->table, (int32_t)r->positions, (int32_t)r->dim} : RotationView{nullptr, 0, 0};
}

// Weights, eps and rotation of a call on heads of head_dim.
ngemm_status check_turn(const ngemm_ctx *ctx, const ngemm_rotation *r, int64_t head_dim, float eps, const void *w0, const void *w1)
{
    if (r && (!rotation_ok(r) || r->device != ctx->device)) return NGEMM_ERR_INVALID_ARG;
    if (r && r->dim > head_dim) return NGEMM_ERR_BAD_SHAPE;
    if (!(eps >= 0.0f) || !std::isfinite(eps) || ((uintptr_t)w0 & 3u) != 0 || ((uintptr_t)w1 & 3u) != 0) return NGEMM_ERR_INVALID_ARG;
    return NGEMM_OK;
}

// f(Index<LANES>{}, Index<PAIRS>{})
template <class F>
void with_turn_form(int64_t head_dim, const ngemm_rotation *r, F &&f)
{
    auto with_pairs = [&](auto lanes) {
        if (!r) f(lanes, Index<kNoPairs>{});
        else if (r->pairs == NGEMM_PAIRS_HALVES) f(lanes, Index<kHalves>{});
        else f(lanes, Index<kNeighbours>{});
    };
    if (head_dim <= 64) with_pairs(Index<4>{});
    else if (head_dim <= 128) with_pairs(Index<8>{});
    else with_pairs(Index<16>{});
}

// f(E{}) for an element type
template <class F>
void with_type(int type, F &&f)
{
    if (type == NGEMM_F32) f(F32{});
    else if (type == NGEMM_F16) f(F16{});
    else f(BF16{});
}

bool type_ok(int type) { return type == NGEMM_F32 || type == NGEMM_F16 || type == NGEMM_BF16; }

}  // namespace

extern "C" {

size_t ngemm_rotation_bytes(int64_t positions, int64_t dim)
{
    if (positions < 1 || positions > kMaxLength || dim < 16 || dim > 256 || dim % 16) return 0;
    return (size_t)positions * (size_t)dim * 4;
}

ngemm_status ngemm_rotation_create(ngemm_ctx *ctx, int64_t positions, int64_t dim, ngemm_pairs pairs, const float *table_dev, size_t table_bytes,
                                   ngemm_rotation **out)
{
    if (!out) return NGEMM_ERR_INVALID_ARG;
    *out = nullptr;
    if (!ctx_ok(ctx) || (pairs != NGEMM_PAIRS_HALVES && pairs != NGEMM_PAIRS_NEIGHBOURS)) return NGEMM_ERR_INVALID_ARG;
    const size_t need = ngemm_rotation_bytes(positions, dim);
    if (need == 0) return NGEMM_ERR_BAD_SHAPE;
    if (!table_dev || ((uintptr_t)table_dev & 15u) != 0) return NGEMM_ERR_INVALID_ARG;
    if (table_bytes < need) return NGEMM_ERR_BUFFER_TOO_SMALL;
    ngemm_rotation *r = new (std::nothrow) ngemm_rotation{kRotationMagic, ctx->device, (int)pairs, positions, dim, table_dev};
    if (!r) return NGEMM_ERR_DEVICE;
    *out = r;
    return NGEMM_OK;
}

ngemm_status ngemm_rotation_free(ngemm_rotation *rotation)
{
    if (!rotation) return NGEMM_OK;
    if (!rotation_ok(rotation)) return NGEMM_ERR_INVALID_ARG;
    rotation->magic = 0;
    delete rotation;
    return NGEMM_OK;
}

ngemm_status ngemm_qk_norm_rotate(ngemm_ctx *ctx, ngemm_type type, int64_t head_dim, int64_t tokens,
                                  int64_t q_heads, const void *Q_dev, int64_t q_token_stride, int64_t q_head_stride, const float *q_weight_dev,
                                  int64_t k_heads, const void *K_dev, int64_t k_token_stride, int64_t k_head_stride, const float *k_weight_dev,
                                  float eps, const ngemm_rotation *rotation, const int32_t *positions_dev,
                                  void *QO_dev, int64_t qo_token_stride, int64_t qo_head_stride,
                                  void *KO_dev, int64_t ko_token_stride, int64_t ko_head_stride, void *hip_stream)
{
    if (!ctx_ok(ctx) || !type_ok(type)) return NGEMM_ERR_INVALID_ARG;
    if (!head_dim_ok(head_dim) || tokens < 0 || tokens > kMaxCount || q_heads < 0 || k_heads < 0 || q_heads > 65536 || k_heads > 65536)
        return NGEMM_ERR_BAD_SHAPE;
    if (const ngemm_status s = check_turn(ctx, rotation, head_dim, eps, q_heads ? q_weight_dev : nullptr, k_heads ? k_weight_dev : nullptr); s != NGEMM_OK) return s;
    if (tokens == 0 || q_heads + k_heads == 0) return NGEMM_OK;
    if (rotation && !positions_dev) return NGEMM_ERR_INVALID_ARG;
    const Rows from[2] = {{const_cast<void *>(Q_dev), q_token_stride, q_head_stride}, {const_cast<void *>(K_dev), k_token_stride, k_head_stride}};
    const Rows to[2] = {{QO_dev, qo_token_stride, qo_head_stride}, {KO_dev, ko_token_stride, ko_head_stride}};
    const int64_t heads[2] = {q_heads, k_heads};
    bool vec = true;
    for (int i = 0; i < 2; ++i) {
        if (heads[i] == 0) continue;
        if (const ngemm_status s = check_rows(from[i], type, tokens, heads[i], head_dim, false); s != NGEMM_OK) return s;
        if (const ngemm_status s = check_rows(to[i], type, tokens, heads[i], head_dim, true); s != NGEMM_OK) return s;
        vec = vec && in_pieces(from[i], type) && in_pieces(to[i], type);
    }
    const int64_t lanes = head_dim <= 64 ? 4 : head_dim <= 128 ? 8 : 16, rows = tokens * (q_heads + k_heads);
    // Four heads an item where that leaves some wavefronts for each SIMD: tokens of 32 + 8 heads of 128, bf16, with four and with one: 64 tokens 5.8 and 4.0 us, 512 6.2 and 6.3,
    // 800 6.8 and 7.8, 1600 10.2 and 13.9, 10000 45 and 62
    const int64_t U = rows * lanes >= (int64_t)3 * 64 * 1024 ? 4 : 1;
    const int64_t chunks_q = (q_heads + U - 1) / U, chunks = chunks_q + (k_heads + U - 1) / U, items = tokens * chunks;
    const int64_t groups = (items + 256 / lanes - 1) / (256 / lanes);
    if (groups > kMaxGroups) return NGEMM_ERR_BAD_SHAPE;
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const TurnArgs a{{{from[0], to[0], q_weight_dev, (int32_t)q_heads}, {from[1], to[1], k_weight_dev, (int32_t)k_heads}}, view_of(rotation), positions_dev,
                     eps, (int32_t)head_dim, (int32_t)items, (int32_t)chunks, (int32_t)chunks_q};
    hipStream_t st = (hipStream_t)hip_stream;
    with_type(type, [&](auto e) {
        with_turn_form(head_dim, rotation, [&](auto l, auto p) {
            typedef decltype(e) E;
            constexpr int LANES = decltype(l)::value, PAIRS = decltype(p)::value;
            const dim3 grid((unsigned)groups), block(256);
            if (U == 4 && vec) hipLaunchKernelGGL((qk_norm_rotate_kernel<E, LANES, PAIRS, 4, true>), grid, block, 0, st, a);
            else if (U == 4) hipLaunchKernelGGL((qk_norm_rotate_kernel<E, LANES, PAIRS, 4, false>), grid, block, 0, st, a);
            else if (vec) hipLaunchKernelGGL((qk_norm_rotate_kernel<E, LANES, PAIRS, 1, true>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((qk_norm_rotate_kernel<E, LANES, PAIRS, 1, false>), grid, block, 0, st, a);
        });
    });
    return launched();
}

ngemm_status ngemm_kv_write_rotated(ngemm_ctx *ctx, const ngemm_kv_cache *cache, ngemm_type type, int64_t batch, int64_t tokens,
                                    const void *K_dev, int64_t k_token_stride, int64_t k_head_stride,
                                    const void *V_dev, int64_t v_token_stride, int64_t v_head_stride,
                                    const float *k_weight_dev, float eps, const ngemm_rotation *rotation,
                                    const int32_t *offsets_dev, const int32_t *starts_dev,
                                    const int32_t *pages_dev, int64_t pages_stride, void *hip_stream)
{
    const Rows k{const_cast<void *>(K_dev), k_token_stride, k_head_stride}, v{const_cast<void *>(V_dev), v_token_stride, v_head_stride};
    MovePlan plan;
    if (const ngemm_status s = plan_move(plan, ctx, cache, type, batch, tokens, k, v, offsets_dev, pages_dev, pages_stride, false); s != NGEMM_OK) return s;
    if (const ngemm_status s = check_turn(ctx, rotation, cache->head_dim, eps, k_weight_dev, nullptr); s != NGEMM_OK) return s;
    if (plan.groups == 0) return NGEMM_OK;
    // four heads of a workgroup share a token's angles and weights where that leaves some thousands of workgroups (17200 tokens of 8 heads, written and read
    // back: 53.5 us with four, 55.5 with two, 59 with one; 64 sequences of a token 14.5 with four, 9.5 with one)
    if (plan.slots * cache->kv_heads >= 8192 && plan.heads < 4) {
        plan.heads = (int32_t)std::min<int64_t>(cache->kv_heads, 4);
        plan.groups = plan.slots * ((cache->kv_heads + plan.heads - 1) / plan.heads);
    }
    DeviceGuard g(ctx->device);
    if (!g.ok) return NGEMM_ERR_DEVICE;
    const TurnedMoveArgs a{{view_of(cache, pages_dev, pages_stride), k, v, offsets_dev, starts_dev, (int32_t)batch, (int32_t)tokens, plan.heads},
                           view_of(rotation), k_weight_dev, eps};
    const bool vec = in_pieces(k, type) && in_pieces(v, type);
    hipStream_t st = (hipStream_t)hip_stream;
    with_type(type, [&](auto e) {
        with_turn_form(cache->head_dim, rotation, [&](auto l, auto p) {
            typedef decltype(e) E;
            constexpr int LANES = decltype(l)::value, PAIRS = decltype(p)::value;
            const dim3 grid((unsigned)plan.groups), block(16 * LANES);
            if (vec) hipLaunchKernelGGL((kv_write_rotated_kernel<E, LANES, PAIRS, true>), grid, block, 0, st, a);
            else hipLaunchKernelGGL((kv_write_rotated_kernel<E, LANES, PAIRS, false>), grid, block, 0, st, a);
        });
    });
    return launched();
}

}  // extern "C"
