// Host side of the calls with several query rows and of eviction: argument checks and launches.
// As everywhere, a call is checked on the host before anything is enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kvqp_checks.h"

using namespace kvqp;

extern "C" {

// Alignment that the kernels of the calls below take for granted: whole pieces of 16 bytes of codes and rows, and
// dwords of the scales and zeros that belong to tokens.
static bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
static bool cache_aligned(const kvqp_cfg* c, const kvqp_cache* cache) {
    const uintptr_t keys = c->key_axis == KVQP_KEY_PER_CHANNEL ? 16 : 4;
    return aligned(cache->k_codes, 16) && aligned(cache->v_codes, 16) && aligned(cache->k_scale, keys) && aligned(cache->k_zero, keys) &&
           aligned(cache->v_scale, 4) && aligned(cache->v_zero, 4) && aligned(cache->tail_k, 16) && aligned(cache->tail_v, 16) &&
           aligned(cache->head_n_kept, 4);
}
// (token numbers, and the words of a head's value codes, at most 64 a token, are 32 bits in the kernels)
constexpr int kMostTokens = 1 << 26;
// Checks of a cache that several query rows or an eviction read.
static int check_read_cache(const kvqp_cfg* cfg, const kvqp_cache* cache) {
    int rc = check_common(cfg);
    if (rc) return rc;
    if (!cache) return KVQP_ERR_INVALID_ARG;
    if (outliers_on(*cfg)) return KVQP_ERR_UNSUPPORTED;
    if (cache->n_kept < 0 || cache->tail_len < 0 || cache->tail_len > cache->tail_cap) return KVQP_ERR_INVALID_ARG;
    if (cache->n_kept > kMostTokens || cache->n_cap > kMostTokens || cache->tail_cap > kMostTokens) return KVQP_ERR_UNSUPPORTED;
    if ((rc = check_cache_ptrs(cfg, cache, cache->n_kept, cache->tail_len > 0))) return rc;
    return cache_aligned(cfg, cache) ? KVQP_OK : KVQP_ERR_INVALID_ARG;
}

int kvqp_tree_workspace_bytes(const kvqp_cfg* cfg, int32_t n_rows, size_t* bytes) {
    const int rc = check_common(cfg);
    if (rc) return rc;
    if (!bytes || n_rows < 1) return KVQP_ERR_INVALID_ARG;
    if (n_rows > KVQP_MOST_ROWS) return KVQP_ERR_UNSUPPORTED;
    // (not the most for the most rows: fewer row blocks get more splits.  What fills its row block needs as much as any with the same blocks.)
    const int gq = cfg->n_q_heads / cfg->n_kv_heads;
    *bytes = plan_tree(*cfg, n_rows, 0, 0).ws_bound;
    for (int rows = 16; rows < gq * n_rows; rows += rows < 64 ? rows : 64) *bytes = std::max(*bytes, plan_tree(*cfg, rows / gq, 0, 0).ws_bound);
    return KVQP_OK;
}

int kvqp_tree_workspace_init(void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!workspace || workspace_bytes < kTreeCounterBytes) return KVQP_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return KVQP_ERR_INVALID_ARG;
    return launch_tree_init(workspace, (hipStream_t)hip_stream) == hipSuccess ? KVQP_OK : KVQP_ERR_HIP;
}

int kvqp_tree_attn(const kvqp_cfg* cfg, const void* q, const void* k_new, const void* v_new, const uint32_t* mask, int32_t mask_per_batch,
                   int32_t n_rows, const kvqp_cache* cache, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = check_read_cache(cfg, cache);
    if (rc) return rc;
    if (!q || !k_new || !v_new || !out || n_rows < 1) return KVQP_ERR_INVALID_ARG;
    if (n_rows > KVQP_MOST_ROWS) return KVQP_ERR_UNSUPPORTED;
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(out, 16) || !aligned(mask, 4) || !aligned(lse, 4)) return KVQP_ERR_INVALID_ARG;
    const TreePlan plan = plan_tree(*cfg, n_rows, cache->n_kept, cache->tail_len);
    if (plan.ws_bytes > 0 && (!workspace || workspace_bytes < plan.ws_bytes)) return KVQP_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return KVQP_ERR_INVALID_ARG;
    if (launch_tree(*cfg, q, k_new, v_new, mask, mask_per_batch != 0, n_rows, *cache, out, lse, workspace, plan, (hipStream_t)hip_stream) != hipSuccess)
        return KVQP_ERR_HIP;
    return KVQP_OK;
}

int kvqp_accumulate_weights(const kvqp_cfg* cfg, const void* q, const float* lse, int32_t n_rows, const kvqp_cache* cache, float* weights,
                            int32_t w_cap, float decay, void* hip_stream) {
    const int rc = check_read_cache(cfg, cache);
    if (rc) return rc;
    if (!q || !lse || !weights || n_rows < 1) return KVQP_ERR_INVALID_ARG;
    if (n_rows > KVQP_MOST_ROWS) return KVQP_ERR_UNSUPPORTED;
    if (!aligned(q, 16) || !aligned(lse, 4) || !aligned(weights, 4)) return KVQP_ERR_INVALID_ARG;
    if ((long long)w_cap < (long long)cache->n_kept + cache->tail_len) return KVQP_ERR_INVALID_ARG;
    if (!(decay >= 0.0f) || decay > 3.0e38f) return KVQP_ERR_INVALID_ARG;
    if (cache->n_kept + cache->tail_len == 0) return KVQP_OK;      // no token to weigh
    if (launch_weights(*cfg, q, lse, n_rows, *cache, weights, w_cap, decay, (hipStream_t)hip_stream) != hipSuccess) return KVQP_ERR_HIP;
    return KVQP_OK;
}

int kvqp_evict_workspace_bytes(const kvqp_cfg* cfg, int32_t n_kept, size_t* bytes) {
    const int rc = check_common(cfg);
    if (rc) return rc;
    if (!bytes || n_kept < 0) return KVQP_ERR_INVALID_ARG;
    *bytes = ((size_t)cfg->batch * cfg->n_kv_heads * n_kept * sizeof(int32_t) + 15) / 16 * 16;
    return KVQP_OK;
}

int kvqp_evict(const kvqp_cfg* cfg, const kvqp_cache* src, const float* weights, int32_t w_cap, int32_t n_keep, int32_t unit, kvqp_cache* dst,
               float* weights_out, int32_t w_cap_out, int32_t* idx_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_read_cache(cfg, src);
    if (rc) return rc;
    if (!dst || !weights || n_keep < 1) return KVQP_ERR_INVALID_ARG;
    if (!(unit == 1 || unit == 32 || unit == 64 || unit == 128) || unit > n_keep) return KVQP_ERR_INVALID_ARG;
    if ((long long)w_cap < (long long)src->n_kept + src->tail_len) return KVQP_ERR_INVALID_ARG;
    if ((src->head_n_kept != nullptr) != (dst->head_n_kept != nullptr)) return KVQP_ERR_INVALID_ARG;
    const int bound = src->head_n_kept ? (n_keep < src->n_kept ? n_keep : src->n_kept) : evict_kept(src->n_kept, n_keep, unit);
    if (dst->n_cap > kMostTokens || dst->tail_cap > kMostTokens) return KVQP_ERR_UNSUPPORTED;
    if (dst->tail_cap < src->tail_len) return KVQP_ERR_INVALID_ARG;
    if ((rc = check_cache_ptrs(cfg, dst, bound, src->tail_len > 0))) return rc;
    if (!cache_aligned(cfg, dst) || !aligned(weights, 4) || !aligned(weights_out, 4) || !aligned(idx_out, 4)) return KVQP_ERR_INVALID_ARG;
    const size_t heads = (size_t)cfg->batch * cfg->n_kv_heads;
    // What is read and what is written must not share memory: workgroups do both at the same time.
    const void* in[] = {src->k_codes, src->v_codes, src->k_scale, src->k_zero, src->v_scale, src->v_zero, src->tail_k, src->tail_v, src->head_n_kept, weights};
    void* const outs[] = {dst->k_codes, dst->v_codes, dst->k_scale, dst->k_zero, dst->v_scale, dst->v_zero, dst->tail_k, dst->tail_v, dst->head_n_kept,
                          weights_out, idx_out, workspace};
    size_t in_bytes[10], out_bytes[12];
    fill_sizes(cfg, layout_tokens(*src, src->n_kept), src->tail_cap, in_bytes);
    fill_sizes(cfg, layout_tokens(*dst, bound), dst->tail_cap, out_bytes);
    in_bytes[8] = out_bytes[8] = heads * sizeof(int32_t);
    in_bytes[9] = heads * (size_t)w_cap * sizeof(float);
    if (weights_out && (long long)w_cap_out < (long long)bound + src->tail_len) return KVQP_ERR_INVALID_ARG;
    out_bytes[9] = weights_out ? heads * (size_t)w_cap_out * sizeof(float) : 0;
    out_bytes[10] = heads * (size_t)bound * sizeof(int32_t);
    out_bytes[11] = (out_bytes[10] + 15) / 16 * 16;
    if (bound > 0 && (!workspace || workspace_bytes < out_bytes[11])) return KVQP_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return KVQP_ERR_INVALID_ARG;
    auto meet = [](const void* p, size_t np, const void* r, size_t nr) {
        return p && r && np && nr && (uintptr_t)p < (uintptr_t)r + nr && (uintptr_t)r < (uintptr_t)p + np;
    };
    for (int o = 0; o < 12; ++o) {
        for (int i = 0; i < 10; ++i)
            if (meet(in[i], in_bytes[i], outs[o], out_bytes[o])) return KVQP_ERR_INVALID_ARG;
        for (int p = 0; p < o; ++p)
            if (meet(outs[p], out_bytes[p], outs[o], out_bytes[o])) return KVQP_ERR_INVALID_ARG;
    }
    if (launch_evict(*cfg, *src, weights, w_cap, n_keep, unit, bound, *dst, weights_out, weights_out ? w_cap_out : 0, idx_out, (int32_t*)workspace,
                     (hipStream_t)hip_stream) != hipSuccess)
        return KVQP_ERR_HIP;
    dst->n_kept = bound;
    dst->tail_len = src->tail_len;
    return KVQP_OK;
}

}  // extern "C"
