// Memory- and undefined-behaviour check of the host side of the calls with several query rows and of eviction
// (csrc/rows_api.cpp), linked with that one file under -fsanitize=address,undefined and with stand-ins for the launches: a rejected
// call must reach none of them, an accepted one exactly one.  Every combination of a set of field values goes through.
// Test infrastructure only.
#include <cstdio>
#include <cstdlib>

#include "kvqp_internal.h"

static int g_launches = 0;

namespace kvqp {
TreePlan plan_tree(const kvqp_cfg&, int n_rows, int n_kept, int tail_len) {
    TreePlan p{};
    p.row_tiles = 1; p.row_blocks = 1; p.n_splits = n_kept + tail_len > 64 ? 2 : 1; p.most_splits = 2;
    p.ws_bytes = p.n_splits > 1 ? (size_t)n_rows * 64 : 0; p.ws_bound = (size_t)n_rows * 64;
    return p;
}
hipError_t launch_tree(const kvqp_cfg&, const void*, const void*, const void*, const uint32_t*, bool, int, const kvqp_cache&, void*, float*, void*,
                       const TreePlan&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_tree_init(void*, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_weights(const kvqp_cfg&, const void*, const float*, int, const kvqp_cache&, float*, int, float, hipStream_t) { ++g_launches; return hipSuccess; }
int evict_kept(int n, int n_keep, int unit) { return n <= n_keep ? n : n % unit + (n_keep - n % unit) / unit * unit; }
hipError_t launch_evict(const kvqp_cfg&, const kvqp_cache&, const float*, int, int, int, int, const kvqp_cache&, float*, int, int32_t*, int32_t*, hipStream_t) {
    ++g_launches;
    return hipSuccess;
}
}  // namespace kvqp

static char* at(size_t n) { return (char*)(uintptr_t)(n << 28); }

static kvqp_cache cache_at(size_t place, int n_kept, int tail, int cap) {
    kvqp_cache c{};
    void** p[] = {&c.k_codes, &c.v_codes, &c.k_scale, &c.k_zero, &c.v_scale, &c.v_zero, &c.tail_k, &c.tail_v};
    for (int i = 0; i < 8; ++i) *p[i] = at(place + i);
    c.n_kept = n_kept; c.tail_len = tail; c.tail_cap = tail > 0 ? tail : 1; c.n_cap = cap;
    return c;
}

static void expect(int rc, int launches_before, bool may_skip, const char* what) {
    const int made = g_launches - launches_before;
    if ((rc == KVQP_OK && made != 1 && !may_skip) || (rc != KVQP_OK && made != 0) || rc < KVQP_ERR_HIP || rc > 0) {
        std::printf("%s: rc %d after %d launches\n", what, rc, made);
        std::exit(1);
    }
}

int main() {
    const int bits[] = {2, 3, 4, 8, 16}, groups[] = {0, 32, 64, 128, 100}, kepts[] = {-1, 0, 1, 63, 256, 1 << 28, 0x7fffffff}, tails[] = {-1, 0, 40, 0x7fffffff},
              rows[] = {-1, 0, 1, 256, 257, 0x7fffffff}, units[] = {-1, 0, 1, 32, 128}, caps[] = {0, 64, 256, 0x7fffffc0, -64};
    int calls = 0, taken = 0;
    for (int b : bits) for (int g : groups) for (int axis = 0; axis < 3; ++axis) for (int n : kepts) for (int t : tails) for (int cap : caps) {
        kvqp_cfg c{};
        c.batch = 2; c.n_q_heads = 8; c.n_kv_heads = 4; c.head_dim = 128; c.bits = b; c.group_size = g; c.key_axis = axis; c.sm_scale = 0.1f;
        const kvqp_cache src = cache_at(1, n, t, cap);
        size_t bytes = 0;
        for (int r : rows) {
            int before = g_launches;
            int rc = kvqp_tree_workspace_bytes(&c, r, &bytes);
            expect(rc, before, true, "sizes");
            rc = kvqp_tree_attn(&c, at(20), at(21), at(22), nullptr, 0, r, &src, at(23), nullptr, at(24), 1 << 20, nullptr);
            expect(rc, before, false, "tree"); taken += rc == KVQP_OK;
            before = g_launches;
            rc = kvqp_accumulate_weights(&c, at(20), (float*)at(21), r, &src, (float*)at(22), 0x7fffffff, 0.5f, nullptr);
            expect(rc, before, n == 0 && t == 0, "weights"); taken += rc == KVQP_OK;
            calls += 2;
        }
        for (int u : units) for (int keep : {-1, 0, 1, 32, 200, 0x7fffffff}) {
            kvqp_cache dst = cache_at(40, 0, t > 0 && t < 1000 ? t : 0, cap);
            int before = g_launches;
            int rc = kvqp_evict_workspace_bytes(&c, n, &bytes);
            expect(rc, before, true, "sizes");
            rc = kvqp_evict(&c, &src, (float*)at(100), 1 << 20, keep, u, &dst, nullptr, 0, nullptr, at(200), (size_t)1 << 40, nullptr);
            expect(rc, before, false, "evict"); taken += rc == KVQP_OK;
            ++calls;
        }
    }
    std::printf("rows_driver: clean, %d calls, %d taken\n", calls, taken);
    return taken > 1000 ? 0 : 1;
}
