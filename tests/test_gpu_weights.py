"""kvqp_accumulate_weights: the attention weight that cached tokens receive, against the formula in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev
from tests.rows_util import D, SM, attention, half, logit_error, make

pytestmark = pytest.mark.gpu


def seen_by(n, tail, N):
    """[N, n + tail]: packed tokens, and the tail rows up to the row's own place"""
    return np.arange(n + tail)[None] <= n + tail - N + np.arange(N)[:, None]


def run(cfg, cache, keys, counts, tail, q, decay, lse_of=None, extra=5):
    B, Hq, N, _ = q.shape
    Hkv, gq = cfg.n_kv_heads, Hq // cfg.n_kv_heads
    rng = np.random.default_rng(1)
    cap = cache.n_kept + tail + extra
    w0 = rng.random((B, Hkv, cap)).astype(np.float32) * np.float32(0.01)
    lse = np.zeros((B, Hq, N))
    for h in range(B * Hkv):
        b, g = divmod(h, Hkv)
        for a in range(g * gq, (g + 1) * gq):
            vis = seen_by(counts[h], tail, N)
            vis[:, :counts[h]] = True
            lse[b, a] = attention(q[b, a].astype(np.float64), keys[h], keys[h], vis)[1]
    if lse_of is not None:
        lse = lse_of(lse)
    lse = lse.astype(np.float32)
    w = kvqp.accumulate_weights(cfg, dev(q), dev(lse), cache, dev(w0), decay=decay)
    torch.cuda.synchronize()
    w = w.cpu().numpy().astype(np.float64)
    for h in range(B * Hkv):
        b, g = divmod(h, Hkv)
        n = counts[h]
        add, slack = np.zeros(n + tail), 0.0
        for a in range(g * gq, (g + 1) * gq):
            rows = q[b, a].astype(np.float64)
            vis = seen_by(n, tail, N)
            vis[:, :n] = True
            p = np.where(vis, np.exp((rows @ keys[h].T) * SM - lse[b, a].astype(np.float64)[:, None]), 0.0)
            add += np.where(np.isneginf(lse[b, a])[:, None], 0.0, p).sum(0)
            slack = max(slack, logit_error(rows, keys[h]))
        ref = float(np.float32(decay)) * w0[b, g, :n + tail].astype(np.float64) + add
        # (a weight's relative error is its exponent's absolute one; the sums round at most 2^-24 per row and once more)
        off = np.abs(w[b, g, :n + tail] - ref) - ((slack + 2.0 ** -19 + gq * N * 2.0 ** -24) * add + 2.0 ** -23 * ref + 2.0 ** -120)
        assert off.max(initial=-1) <= 0, (h, off.max(), int(off.argmax()), n)
        assert np.array_equal(w[b, g, n + tail:], w0[b, g, n + tail:])        # entries past the tail are left alone
    return w


CASES = [  # B, Hkv, Gq, n, tail, bits, G, axis, N, decay
    (1, 2, 4, 256, 32, 4, 32, 0, 1, 1.0), (1, 1, 1, 1, 0, 4, 32, 0, 1, 1.0), (2, 2, 8, 333, 40, 4, 64, 0, 5, 0.5), (1, 1, 4, 700, 64, 4, 128, 0, 33, 1.0),
    (1, 2, 2, 99, 1, 2, 32, 0, 1, 0.0), (1, 1, 4, 500, 70, 2, 64, 0, 64, 0.9), (1, 3, 1, 65, 3, 2, 128, 0, 2, 1.0),
    (1, 2, 4, 129, 17, 8, 32, 0, 4, 1.0), (1, 1, 8, 64, 32, 8, 128, 0, 30, 2.0), (2, 1, 2, 100, 9, 16, 32, 0, 3, 1.0), (1, 1, 4, 31, 100, 16, 32, 0, 100, 0.25),
    (1, 2, 4, 256, 32, 4, 32, 1, 1, 1.0), (1, 1, 8, 161, 8, 4, 64, 1, 8, 1.0), (1, 1, 1, 127, 12, 4, 128, 1, 9, 0.0),
    (1, 2, 2, 99, 12, 2, 32, 1, 10, 1.0), (1, 1, 4, 300, 31, 8, 64, 1, 17, 0.75), (1, 1, 4, 0, 40, 4, 32, 0, 7, 1.0), (1, 1, 2, 40, 0, 4, 32, 0, 1, 1.0),
    (1, 1, 2, 40, 3, 4, 32, 0, 6, 1.0), (1, 1, 2, 32, 256, 4, 32, 0, 256, 1.0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_weights_against_the_formula(orc, case):
    B, Hkv, Gq, n, tail, bits, G, axis, N, decay = case
    rng = np.random.default_rng(hash(case) % 2 ** 31)
    cfg, cache, keys, _ = make(orc, rng, B, Hkv, Gq, n, tail, bits, G, axis)
    run(cfg, cache, keys, [n] * (B * Hkv), tail, half(rng, B, Hkv * Gq, N, D), decay)


@pytest.mark.parametrize("bits,G,axis,n_cap", [(4, 32, 0, 0), (2, 64, 1, 0), (8, 128, 1, 640), (16, 32, 0, 576)])
def test_heads_with_their_own_counts(orc, bits, G, axis, n_cap):
    rng = np.random.default_rng(2)
    counts = [513, 0, 1, 100, 257, 64]
    cfg, cache, keys, _ = make(orc, rng, 2, 3, 4, 513, 20, bits, G, axis, counts=counts, n_cap=n_cap)
    run(cfg, cache, keys, counts, 20, half(rng, 2, 12, 6, D), 0.9)


def test_a_row_that_saw_nothing_adds_nothing(orc):
    rng = np.random.default_rng(3)
    cfg, cache, keys, _ = make(orc, rng, 1, 2, 2, 90, 10, 4, 32, 0)

    def without(lse):
        lse[0, 1, 2] = lse[0, 3] = -np.inf
        return lse
    run(cfg, cache, keys, [90, 90], 10, half(rng, 1, 4, 5, D), 1.0, lse_of=without)


def test_weights_without_the_old_ones_do_not_read_them(orc):
    """decay 0: the weights of one call, whatever was there; a row's weights add up to one."""
    rng = np.random.default_rng(4)
    cfg, cache, keys, _ = make(orc, rng, 1, 2, 4, 200, 12, 4, 32, 0)
    q, kn, vn = half(rng, 1, 8, 1, D), half(rng, 1, 2, 1, D), half(rng, 1, 2, 1, D)
    # (the drafted token is the tail row that comes next: see it once as such, then as part of the tail)
    cache.tail_len -= 1
    tk, tv = (cache.buffers[k].view(torch.float16).view(1, 2, -1, D)[:, :, 11:12].contiguous() for k in ("tail_k", "tail_v"))
    lse = torch.empty((1, 8, 1), device="cuda")
    kvqp.tree_attn(cfg, dev(q), tk, tv, None, cache, lse=lse)
    cache.tail_len += 1
    w = torch.full((1, 2, 212), float("nan"), device="cuda")
    kvqp.accumulate_weights(cfg, dev(q), lse, cache, w, decay=0.0)
    total = w.double().sum(-1).cpu().numpy()
    assert np.abs(total - 4.0).max() <= 4 * (2 * logit_error(q[0, 0].astype(np.float64), keys[0]) + 2.0 ** -18)


def test_the_same_bits_again_and_in_a_replayed_graph(orc):
    rng = np.random.default_rng(5)
    cfg, cache, keys, _ = make(orc, rng, 1, 2, 4, 1000, 32, 2, 32, 0)
    q, lse = dev(half(rng, 1, 8, 3, D)), torch.full((1, 8, 3), 6.0, device="cuda")
    ref = torch.zeros((1, 2, 1032), device="cuda")
    w = torch.zeros_like(ref)
    kvqp.accumulate_weights(cfg, q, lse, cache, w)
    w.zero_()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        kvqp.accumulate_weights(cfg, q, lse, cache, w)
    w.zero_()
    for _ in range(4):
        g.replay()
        kvqp.accumulate_weights(cfg, q, lse, cache, ref)
        torch.cuda.synchronize()
        assert torch.equal(w, ref)
