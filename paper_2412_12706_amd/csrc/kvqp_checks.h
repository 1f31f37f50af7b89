// Argument checks that the entry points share (host only).
#pragma once
#include "kvqp_internal.h"

namespace kvqp {

inline bool is_pow2_group(int g) { return g == 32 || g == 64 || g == 128; }

// Checks of the fields every entry point reads.
inline int check_common(const kvqp_cfg* c) {
    if (!c) return KVQP_ERR_INVALID_ARG;
    if (c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return KVQP_ERR_INVALID_ARG;
    if (c->n_q_heads % c->n_kv_heads) return KVQP_ERR_INVALID_ARG;
    if (!(c->bits == 2 || c->bits == 4 || c->bits == 8 || c->bits == 16)) return KVQP_ERR_INVALID_ARG;
    if (c->key_axis != KVQP_KEY_PER_CHANNEL && c->key_axis != KVQP_KEY_PER_TOKEN) return KVQP_ERR_INVALID_ARG;
    if (c->decode_splits < 0) return KVQP_ERR_INVALID_ARG;
    if (c->bits != 16) {
        if (c->group_size < 1 || c->head_dim % c->group_size) return KVQP_ERR_INVALID_ARG;
    }
    if (!(c->sm_scale > 0.0f) || c->sm_scale > 3.0e38f) return KVQP_ERR_INVALID_ARG;   /* positive and finite */
    if (!(c->outlier_threshold >= 0.0f) || c->outlier_threshold > 3.0e38f) return KVQP_ERR_INVALID_ARG;
    if (c->outlier_threshold > 0.0f && c->bits == 16) return KVQP_ERR_INVALID_ARG;   /* nothing is quantized at 16 bits */
    if (c->decode_cache_hint < KVQP_CACHE_AUTO || c->decode_cache_hint > KVQP_CACHE_KEEP) return KVQP_ERR_INVALID_ARG;
    if (c->outlier_overflow_cap < 0 || c->outlier_overflow_cap > (1 << 28)) return KVQP_ERR_INVALID_ARG;
    const int gq = c->n_q_heads / c->n_kv_heads;
    if (c->head_dim != kHeadDim) return KVQP_ERR_UNSUPPORTED;
    if (!(gq == 1 || gq == 2 || gq == 4 || gq == 8)) return KVQP_ERR_UNSUPPORTED;
    if (c->bits != 16 && !is_pow2_group(c->group_size)) return KVQP_ERR_UNSUPPORTED;
    if ((long long)c->batch * c->n_kv_heads > 65535) return KVQP_ERR_UNSUPPORTED;   // (batch, kv head) is the y index of every launch but decode's, which has a counter for each
    return KVQP_OK;
}

// Checks of the prompt-side fields (compress, quantize_selected, sizes).
inline int check_prompt(const kvqp_cfg* c) {
    if (c->seq_len < 1 || c->window < 1 || c->window > c->seq_len) return KVQP_ERR_INVALID_ARG;
    if (c->pool_kernel < 1 || c->pool_kernel % 2 == 0) return KVQP_ERR_INVALID_ARG;
    if (c->budget < 0) return KVQP_ERR_INVALID_ARG;
    const int gq = c->n_q_heads / c->n_kv_heads;
    if (c->window * gq > 256 || c->pool_kernel > 63) return KVQP_ERR_UNSUPPORTED;
    if (c->seq_len - c->window > 131072) return KVQP_ERR_UNSUPPORTED;   // selection sweeps at most 128 rows of 1024 candidates
    return KVQP_OK;
}

inline int n_kept_of(const kvqp_cfg* c) {
    const int P = c->seq_len - c->window;
    return c->budget < P ? c->budget : P;
}

// Any count is fine: a partly filled last block and a short last key group are part of the format.
inline int check_n_kept(const kvqp_cfg* c, int n_kept) {
    (void)c;
    return n_kept < 0 ? KVQP_ERR_INVALID_ARG : KVQP_OK;
}

// A non-zero capacity must hold the tokens and keep every head's buffers aligned.
inline int check_cap(const kvqp_cfg* c, int n_cap, int n_kept) {
    if (n_cap == 0) return KVQP_OK;
    if (n_cap < n_kept || n_cap % 64) return KVQP_ERR_INVALID_ARG;
    if (c->bits != 16 && n_cap % c->group_size) return KVQP_ERR_INVALID_ARG;
    return KVQP_OK;
}

inline int fill_sizes(const kvqp_cfg* cfg, int n_tok, int32_t tail_cap, size_t sizes_out[8]) {
    const size_t heads = (size_t)cfg->batch * cfg->n_kv_heads;
    const size_t km = k_meta_elems(n_tok, cfg->bits, cfg->group_size, cfg->key_axis) * 2 * heads;
    const size_t vm = v_meta_elems(n_tok, cfg->bits, cfg->group_size) * 2 * heads;
    const size_t tail = heads * (size_t)tail_cap * kHeadDim * 2;
    sizes_out[0] = k_code_words(n_tok, cfg->bits) * 4 * heads;
    sizes_out[1] = v_code_words(n_tok, cfg->bits) * 4 * heads;
    sizes_out[2] = km; sizes_out[3] = km;
    sizes_out[4] = vm; sizes_out[5] = vm;
    sizes_out[6] = tail; sizes_out[7] = tail;
    return KVQP_OK;
}

inline int check_cache_ptrs(const kvqp_cfg* c, const kvqp_cache* cache, int n_kept, bool need_tail) {
    if (!cache) return KVQP_ERR_INVALID_ARG;
    if (check_cap(c, cache->n_cap, n_kept)) return KVQP_ERR_INVALID_ARG;
    if (n_kept > 0) {
        if (!cache->k_codes || !cache->v_codes) return KVQP_ERR_INVALID_ARG;
        if (c->bits != 16 && (!cache->k_scale || !cache->k_zero || !cache->v_scale || !cache->v_zero))
            return KVQP_ERR_INVALID_ARG;
        if (outliers_on(*c) && (!cache->k_out || !cache->v_out || !cache->k_ovf || !cache->v_ovf)) return KVQP_ERR_INVALID_ARG;
    }
    if (need_tail && (!cache->tail_k || !cache->tail_v)) return KVQP_ERR_INVALID_ARG;
    return KVQP_OK;
}

}  // namespace kvqp
