// Host side of rotary positions and the paged cache: argument checks and launches.
// As everywhere, a call is checked on the host before anything is enqueued.
#include <hip/hip_runtime.h>

#include <math.h>

#include "kvqp_checks.h"

using namespace kvqp;

namespace {

bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
bool good_type(int dtype) { return dtype == KVQP_HALF || dtype == KVQP_BFLOAT16; }
// (numbers of rows and tokens are 32 bits in the kernels, with room for a sum)
constexpr int kMost = 1 << 30;
// What a launch has at most along an axis, of workgroups of 256 threads.
constexpr int64_t kMostWorkgroups = ((int64_t)1 << 24) - 1;

int check_rope(const kvqp_rope* r) {
    if (!r || !r->table || !aligned(r->table, 16) || r->n_positions < 1) return KVQP_ERR_INVALID_ARG;
    if (r->rot_dim < 16 || r->rot_dim > kHeadDim || r->rot_dim % 16) return KVQP_ERR_INVALID_ARG;
    return r->interleaved == 0 || r->interleaved == 1 ? KVQP_OK : KVQP_ERR_INVALID_ARG;
}

int check_pages(const kvqp_cfg* cfg, const kvqp_pages* g) {
    const int rc = check_common(cfg);
    if (rc) return rc;
    if (!g || !good_type(g->dtype) || (g->form != KVQP_E4M3 && g->form != KVQP_INT8)) return KVQP_ERR_INVALID_ARG;
    if (g->page_tokens != 16 && g->page_tokens != 32 && g->page_tokens != 64) return g->page_tokens < 1 ? KVQP_ERR_INVALID_ARG : KVQP_ERR_UNSUPPORTED;
    if (g->n_pages < 1 || g->max_pages < 1 || g->n_open < 1 || (!g->open_slot && g->n_open < cfg->batch)) return KVQP_ERR_INVALID_ARG;
    if ((int64_t)g->max_pages * g->page_tokens > kMost) return KVQP_ERR_UNSUPPORTED;
    const void* buffers[] = {g->k_codes, g->v_codes, g->k_scale, g->v_scale, g->open_k, g->open_v};
    for (const void* p : buffers)
        if (!p || !aligned(p, 16)) return KVQP_ERR_INVALID_ARG;
    if (!g->table || !g->lengths || !aligned(g->table, 4) || !aligned(g->lengths, 4) || !aligned(g->open_slot, 4)) return KVQP_ERR_INVALID_ARG;
    return KVQP_OK;
}

int check_rows(const kvqp_cfg* cfg, int32_t n_rows, const int32_t* row_start) {
    if (n_rows < 0 || !aligned(row_start, 4)) return KVQP_ERR_INVALID_ARG;
    if (!row_start && n_rows != cfg->batch) return KVQP_ERR_INVALID_ARG;
    return n_rows > kMost ? KVQP_ERR_UNSUPPORTED : KVQP_OK;
}
bool good_stride(int64_t stride, int heads) { return stride % 8 == 0 && stride >= (int64_t)heads * kHeadDim && stride <= (int64_t)1 << 31; }

// Memory that a call touches, as one span.
struct Span {
    const void* p;
    int64_t bytes;
};
bool meet(Span a, Span b) {
    return a.p && b.p && a.bytes > 0 && b.bytes > 0 && (uintptr_t)a.p < (uintptr_t)b.p + b.bytes && (uintptr_t)b.p < (uintptr_t)a.p + a.bytes;
}
Span rows_span(const void* p, int64_t n, int64_t stride, int heads) { return {p, n > 0 ? ((n - 1) * stride + (int64_t)heads * kHeadDim) * 2 : 0}; }
constexpr int kPageSpans = 9;
void page_spans(const kvqp_cfg& c, const kvqp_pages& g, Span out[kPageSpans]) {
    const int64_t codes = (int64_t)g.n_pages * c.n_kv_heads * g.page_tokens * kHeadDim, scales = (int64_t)g.n_pages * c.n_kv_heads * 4;
    const int64_t open = (int64_t)g.n_open * c.n_kv_heads * 2 * g.page_tokens * kHeadDim * 2;
    const Span all[kPageSpans] = {{g.k_codes, codes}, {g.v_codes, codes}, {g.k_scale, scales}, {g.v_scale, scales}, {g.open_k, open}, {g.open_v, open},
                                  {g.table, (int64_t)c.batch * g.max_pages * 4}, {g.lengths, (int64_t)c.batch * 4}, {g.open_slot, (int64_t)c.batch * 4}};
    for (int i = 0; i < kPageSpans; ++i) out[i] = all[i];
}
// Whether what is written meets what is read, or what else is written.
bool any_meet(const Span* out, int n_out, const Span* in, int n_in) {
    for (int o = 0; o < n_out; ++o) {
        for (int i = 0; i < n_in; ++i)
            if (meet(out[o], in[i])) return true;
        for (int i = 0; i < o; ++i)
            if (meet(out[o], out[i])) return true;
    }
    return false;
}

}  // namespace

extern "C" {

int kvqp_rope_frequencies(int32_t rot_dim, double base, int32_t scaling, double factor, double context, double low, double high,
                          double* inv_freq) {
    if (!inv_freq || rot_dim < 16 || rot_dim > kHeadDim || rot_dim % 16) return KVQP_ERR_INVALID_ARG;
    if (!(base > 0) || !isfinite(base) || scaling < KVQP_ROPE_PLAIN || scaling > KVQP_ROPE_PARTS) return KVQP_ERR_INVALID_ARG;
    if (scaling != KVQP_ROPE_PLAIN && (!(factor >= 1) || !isfinite(factor))) return KVQP_ERR_INVALID_ARG;
    if (scaling == KVQP_ROPE_PARTS && (!(context > 0) || !isfinite(context) || !(low >= 0) || !(high > low) || !isfinite(high))) return KVQP_ERR_INVALID_ARG;
    if (scaling == KVQP_ROPE_BASE) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int j = 0; j < rot_dim / 2; ++j) {
        double f = pow(base, -2.0 * j / rot_dim);
        if (scaling == KVQP_ROPE_LINEAR) f /= factor;
        if (scaling == KVQP_ROPE_PARTS) {
            const double turns = context * f / 6.283185307179586476925;
            const double g = fmin(fmax((turns - low) / (high - low), 0.0), 1.0);
            f = g * f + (1 - g) * (f / factor);
        }
        inv_freq[j] = f;
    }
    return KVQP_OK;
}

int kvqp_rope_table(const double* inv_freq, int32_t rot_dim, int32_t n_positions, double magnitude, float* table, void* hip_stream) {
    if (!inv_freq || !table || !aligned(table, 8) || rot_dim < 16 || rot_dim > kHeadDim || rot_dim % 16 || n_positions < 1) return KVQP_ERR_INVALID_ARG;
    if (n_positions > kMost || (int64_t)n_positions * (rot_dim / 2) > kMostWorkgroups * 256) return KVQP_ERR_UNSUPPORTED;
    if (!isfinite(magnitude)) return KVQP_ERR_INVALID_ARG;
    for (int j = 0; j < rot_dim / 2; ++j)
        if (!isfinite(inv_freq[j])) return KVQP_ERR_INVALID_ARG;
    return launch_rope_table(inv_freq, rot_dim, n_positions, magnitude, table, (hipStream_t)hip_stream) == hipSuccess ? KVQP_OK : KVQP_ERR_HIP;
}

int kvqp_rotate(const kvqp_rope* rope, int32_t dtype, int32_t batch, int32_t heads, int32_t rows, const kvqp_rows* x, const kvqp_rows* out,
                const int32_t* positions, int32_t positions_per_batch, int32_t first, int32_t inverse, void* hip_stream) {
    const int rc = check_rope(rope);
    if (rc) return rc;
    if (!good_type(dtype) || batch < 1 || heads < 1 || rows < 0 || !x || !out) return KVQP_ERR_INVALID_ARG;
    if (batch > 65535 || heads > 65535 || rows > kMost) return KVQP_ERR_UNSUPPORTED;
    if (rows == 0) return KVQP_OK;
    if (!x->data || !out->data || !aligned(x->data, 16) || !aligned(out->data, 16) || !aligned(positions, 4)) return KVQP_ERR_INVALID_ARG;
    if (!positions && (first < 0 || (int64_t)first + rows > rope->n_positions)) return KVQP_ERR_INVALID_ARG;
    // an axis of one entry has no stride that counts
    const int64_t entries[3] = {batch, heads, rows};
    int64_t xs[3] = {x->batch_stride, x->head_stride, x->row_stride}, os[3] = {out->batch_stride, out->head_stride, out->row_stride};
    int64_t x_span = kHeadDim, o_span = kHeadDim;
    bool same = x->data == out->data;
    for (int i = 0; i < 3; ++i) {
        if (entries[i] == 1) xs[i] = os[i] = 0;
        if (xs[i] % 8 || os[i] % 8 || xs[i] < 0 || os[i] < 0 || xs[i] > (int64_t)1 << 40 || os[i] > (int64_t)1 << 40) return KVQP_ERR_INVALID_ARG;
        if (entries[i] > 1 && os[i] < kHeadDim) return KVQP_ERR_INVALID_ARG;
        if ((double)entries[i] * xs[i] > 1e15 || (double)entries[i] * os[i] > 1e15) return KVQP_ERR_INVALID_ARG;      // (spans are sums of these)
        same = same && xs[i] == os[i];
        x_span += (entries[i] - 1) * xs[i];
        o_span += (entries[i] - 1) * os[i];
    }
    // the rows of out must not meet each other: by falling strides, each axis holds what is inside it
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (os[order[j]] < os[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
    int64_t inside = kHeadDim;
    for (int i = 0; i < 3; ++i) {
        if (entries[order[i]] == 1) continue;
        if (os[order[i]] < inside) return KVQP_ERR_INVALID_ARG;
        inside += (entries[order[i]] - 1) * os[order[i]];
    }
    const Span written = {out->data, o_span * 2};
    if (!same && meet(written, {x->data, x_span * 2})) return KVQP_ERR_INVALID_ARG;
    if (meet(written, {rope->table, (int64_t)rope->n_positions * rope->rot_dim * 4}) ||
        meet(written, {positions, (positions_per_batch ? (int64_t)batch : 1) * rows * 4}))
        return KVQP_ERR_INVALID_ARG;
    if (rows > kMostWorkgroups * 32) return KVQP_ERR_UNSUPPORTED;
    const kvqp_rows from = {x->data, xs[0], xs[1], xs[2]}, to = {out->data, os[0], os[1], os[2]};
    if (launch_rotate(*rope, dtype, batch, heads, rows, from, to, positions, positions_per_batch != 0, first, inverse != 0, (hipStream_t)hip_stream) != hipSuccess)
        return KVQP_ERR_HIP;
    return KVQP_OK;
}

int kvqp_paged_append(const kvqp_cfg* cfg, const kvqp_pages* pages, const kvqp_rope* rope, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, const void* v, int64_t v_stride, int32_t n_rows, const int32_t* row_start, const int32_t* positions,
                      void* q_out, void* hip_stream) {
    int rc = check_pages(cfg, pages);
    if (rc) return rc;
    if ((rc = check_rows(cfg, n_rows, row_start))) return rc;
    if (rope && (rc = check_rope(rope))) return rc;
    if (!k || !v || (q != nullptr) != (q_out != nullptr) || (positions && !rope)) return KVQP_ERR_INVALID_ARG;
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(positions, 4)) return KVQP_ERR_INVALID_ARG;
    const int hq = cfg->n_q_heads, hkv = cfg->n_kv_heads;
    if ((q && !good_stride(q_stride, hq)) || !good_stride(k_stride, hkv) || !good_stride(v_stride, hkv)) return KVQP_ERR_INVALID_ARG;
    if (n_rows == 0) return KVQP_OK;
    if ((int64_t)n_rows / pages->page_tokens + 2 * (int64_t)cfg->batch > kMostWorkgroups) return KVQP_ERR_UNSUPPORTED;
    Span pool[kPageSpans];
    page_spans(*cfg, *pages, pool);
    const bool in_place = q == q_out && q_stride == (int64_t)hq * kHeadDim;
    const Span out[7] = {pool[0], pool[1], pool[2], pool[3], pool[4], pool[5], {q_out, (int64_t)n_rows * hq * kHeadDim * 2}};
    const Span in[9] = {rows_span(k, n_rows, k_stride, hkv), rows_span(v, n_rows, v_stride, hkv), pool[6], pool[7], pool[8],
                        {row_start, ((int64_t)cfg->batch + 1) * 4}, {positions, (int64_t)n_rows * 4},
                        {rope ? rope->table : nullptr, rope ? (int64_t)rope->n_positions * rope->rot_dim * 4 : 0},
                        in_place ? Span{nullptr, 0} : rows_span(q, n_rows, q_stride, hq)};
    if (any_meet(out, 7, in, 9)) return KVQP_ERR_INVALID_ARG;
    for (int i = 0; i < 6; ++i)
        if (in_place && meet(pool[i], rows_span(q, n_rows, q_stride, hq))) return KVQP_ERR_INVALID_ARG;
    if (launch_paged_append(*cfg, *pages, rope, q, q_stride, k, k_stride, v, v_stride, n_rows, row_start, positions, q_out, (hipStream_t)hip_stream) != hipSuccess)
        return KVQP_ERR_HIP;
    return KVQP_OK;
}

int kvqp_paged_workspace_bytes(const kvqp_cfg* cfg, int32_t n_rows, size_t* bytes) {
    const int rc = check_common(cfg);
    if (rc) return rc;
    if (!bytes || n_rows < 0) return KVQP_ERR_INVALID_ARG;
    if (n_rows > kMost) return KVQP_ERR_UNSUPPORTED;
    *bytes = paged_workspace_bound(*cfg, n_rows);
    return KVQP_OK;
}

int kvqp_paged_workspace_init(void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (!workspace || workspace_bytes < KVQP_PAGED_COUNTERS) return KVQP_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return KVQP_ERR_INVALID_ARG;
    return launch_paged_init(workspace, (hipStream_t)hip_stream) == hipSuccess ? KVQP_OK : KVQP_ERR_HIP;
}

int kvqp_paged_attn(const kvqp_cfg* cfg, const kvqp_pages* pages, const void* q, int64_t q_stride, int32_t n_rows, const int32_t* row_start,
                    int32_t window, void* out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    int rc = check_pages(cfg, pages);
    if (rc) return rc;
    if ((rc = check_rows(cfg, n_rows, row_start))) return rc;
    if (!q || !out || window < 0) return KVQP_ERR_INVALID_ARG;
    if (cfg->sm_scale >= 0x1p100f) return KVQP_ERR_UNSUPPORTED;      // (times the scales of queries and keys it is a factor in binary32)
    if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !good_stride(q_stride, cfg->n_q_heads)) return KVQP_ERR_INVALID_ARG;
    if (n_rows == 0) return KVQP_OK;
    if (paged_attn_workgroups(*cfg, *pages, n_rows, row_start != nullptr) > kMostWorkgroups) return KVQP_ERR_UNSUPPORTED;
    const size_t need = paged_workspace_need(*cfg, *pages, n_rows, row_start != nullptr);
    if (need > 0 && (!workspace || workspace_bytes < need)) return KVQP_ERR_WORKSPACE;
    if (!aligned(workspace, 16)) return KVQP_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)n_rows * cfg->n_q_heads;
    Span in[kPageSpans + 2];
    page_spans(*cfg, *pages, in);
    in[kPageSpans] = rows_span(q, n_rows, q_stride, cfg->n_q_heads);
    in[kPageSpans + 1] = {row_start, ((int64_t)cfg->batch + 1) * 4};
    const Span written[3] = {{out, rows * kHeadDim * 2}, {lse, rows * 4}, {workspace, (int64_t)need}};
    if (any_meet(written, 3, in, kPageSpans + 2)) return KVQP_ERR_INVALID_ARG;
    if (launch_paged_attn(*cfg, *pages, q, q_stride, n_rows, row_start, window, out, lse, workspace, (hipStream_t)hip_stream) != hipSuccess) return KVQP_ERR_HIP;
    return KVQP_OK;
}

int kvqp_paged_read(const kvqp_cfg* cfg, const kvqp_pages* pages, int32_t first, int32_t count, void* k_out, void* v_out, void* hip_stream) {
    const int rc = check_pages(cfg, pages);
    if (rc) return rc;
    if (first < 0 || count < 0 || (int64_t)first + count > (int64_t)pages->max_pages * pages->page_tokens) return KVQP_ERR_INVALID_ARG;
    if (count == 0) return KVQP_OK;
    if (count / 64 + 2 > kMostWorkgroups) return KVQP_ERR_UNSUPPORTED;
    if (!k_out || !v_out || !aligned(k_out, 16) || !aligned(v_out, 16)) return KVQP_ERR_INVALID_ARG;
    Span in[kPageSpans];
    page_spans(*cfg, *pages, in);
    const int64_t bytes = (int64_t)cfg->batch * cfg->n_kv_heads * count * kHeadDim * 2;
    const Span written[2] = {{k_out, bytes}, {v_out, bytes}};
    if (any_meet(written, 2, in, kPageSpans)) return KVQP_ERR_INVALID_ARG;
    return launch_paged_read(*cfg, *pages, first, count, k_out, v_out, (hipStream_t)hip_stream) == hipSuccess ? KVQP_OK : KVQP_ERR_HIP;
}

}  // extern "C"
