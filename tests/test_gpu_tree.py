"""kvqp_tree_attn: several query rows (a tree of drafted tokens, a chain, one token) over the packed cache, the tail and each other,
against the attention formula (paper Section 3, Eq. (3), on the dequantized survivors) in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev
from tests.rows_util import D, ancestors, attention, half, logit_error, make, mask_words, out_error

pytestmark = pytest.mark.gpu


def check(cfg, cache, keys, values, q, kn, vn, seen, mask, workspace=None, stream=None):
    """Calls the operator and compares outputs and sums of every row; seen [B or 1, N, N] bool."""
    B, Hq, N, _ = q.shape
    Hkv, gq = cfg.n_kv_heads, Hq // cfg.n_kv_heads
    lse = torch.full((B, Hq, N), 7.0, device="cuda")
    out = torch.full((B, Hq, N, D), 7.0, dtype=torch.float16, device="cuda")
    kvqp.tree_attn(cfg, dev(q), dev(kn), dev(vn), mask, cache, out=out, lse=lse, workspace=workspace, stream=stream)
    torch.cuda.synchronize()
    out, lse = out.cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    for h in range(B * Hkv):
        b, g = divmod(h, Hkv)
        k64 = np.concatenate([keys[h], kn[b, g].astype(np.float64)])
        v64 = np.concatenate([values[h], vn[b, g].astype(np.float64)])
        vis = np.concatenate([np.ones((N, len(keys[h])), bool), seen[b % len(seen)]], 1)
        for a in range(gq):
            rows = q[b, g * gq + a].astype(np.float64)
            with np.errstate(invalid="ignore"):
                ref, ref_lse, spread = attention(rows, k64, v64, vis)
            delta = logit_error(rows, np.where(np.isfinite(k64), k64, 0.0))
            got, got_lse = out[b, g * gq + a], lse[b, g * gq + a]
            empty = ~vis.any(1)
            assert (got[empty] == 0).all() and (got_lse[empty] == -np.inf).all()
            off = np.abs(got - ref) - out_error(ref, spread, delta)
            assert off.max() <= 0, (h, a, off.max(), np.unravel_index(off.argmax(), off.shape))
            live = ~empty
            assert np.abs(got_lse[live] - ref_lse[live]).max(initial=0) <= delta + 2.0 ** -18 + 2.0 ** -22 * np.abs(ref_lse[live]).max(initial=0), (h, a)
    return out, lse


def draft(rng, B, Hkv, Gq, N, scale=1.0):
    return half(rng, B, Hkv * Gq, N, D, scale=scale), half(rng, B, Hkv, N, D), half(rng, B, Hkv, N, D)


CASES = [  # B, Hkv, Gq, n, tail, bits, G, axis, N
    (1, 2, 4, 256, 32, 4, 32, 0, 4), (1, 1, 1, 1, 0, 4, 32, 0, 1), (2, 2, 1, 33, 1, 4, 64, 0, 7), (1, 2, 8, 517, 40, 4, 128, 0, 3),
    (1, 2, 4, 256, 32, 2, 32, 0, 8), (1, 3, 2, 97, 5, 2, 64, 0, 16), (1, 1, 4, 1000, 64, 2, 128, 0, 13), (1, 1, 8, 65, 0, 2, 32, 0, 2),
    (2, 2, 4, 300, 17, 8, 32, 0, 5), (1, 1, 1, 64, 3, 8, 64, 0, 64), (1, 1, 2, 129, 31, 8, 128, 0, 9),
    (1, 2, 4, 256, 32, 16, 32, 0, 6), (3, 1, 2, 71, 9, 16, 32, 0, 1), (1, 1, 8, 31, 33, 16, 32, 0, 12),
    (1, 2, 4, 255, 32, 4, 32, 1, 4), (2, 1, 8, 161, 8, 4, 64, 1, 11), (1, 1, 4, 640, 1, 4, 128, 1, 1),
    (1, 2, 2, 99, 12, 2, 32, 1, 10), (1, 1, 1, 515, 65, 2, 64, 1, 33), (1, 1, 4, 64, 32, 2, 128, 1, 5),
    (1, 2, 4, 130, 7, 8, 32, 1, 3), (1, 1, 2, 77, 0, 8, 64, 1, 20), (2, 1, 1, 40, 40, 8, 128, 1, 2),
    (1, 1, 4, 0, 32, 4, 32, 0, 4), (1, 2, 1, 0, 0, 2, 32, 1, 5), (1, 1, 8, 200, 32, 4, 32, 0, 70),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rows_against_the_formula(orc, case):
    B, Hkv, Gq, n, tail, bits, G, axis, N = case
    rng = np.random.default_rng(hash(case) % 2 ** 31)
    cfg, cache, keys, values = make(orc, rng, B, Hkv, Gq, n, tail, bits, G, axis)
    q, kn, vn = draft(rng, B, Hkv, Gq, N)
    parents = [int(rng.integers(max(-1, i - 5), i)) for i in range(N)]
    check(cfg, cache, keys, values, q, kn, vn, ancestors(parents)[None], kvqp.tree_mask(parents))


@pytest.mark.parametrize("N,Gq", [(1, 4), (5, 2), (32, 1), (33, 1), (100, 1), (256, 2)])
def test_without_a_mask_rows_form_a_chain(orc, N, Gq):
    rng = np.random.default_rng(N)
    cfg, cache, keys, values = make(orc, rng, 1, 2, Gq, 100, 10, 4, 32, 0)
    q, kn, vn = draft(rng, 1, 2, Gq, N)
    a = check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, N, N), bool)), None)
    b = check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, N, N), bool)), kvqp.tree_mask(list(range(-1, N - 1))))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


def test_a_mask_for_every_batch_item_and_any_pattern(orc):
    """Masks need not be trees: any bits, other ones per item, rows that see no drafted token, bits past the last token."""
    rng = np.random.default_rng(3)
    B, N = 3, 40
    cfg, cache, keys, values = make(orc, rng, B, 2, 4, 150, 20, 4, 32, 1)
    q, kn, vn = draft(rng, B, 2, 4, N)
    seen = rng.random((B, N, N)) < 0.3
    seen[1, 5] = False
    words = mask_words(seen)
    words[..., 1] |= np.int32(-1 << 8)
    check(cfg, cache, keys, values, q, kn, vn, seen, dev(words))


@pytest.mark.parametrize("bits,axis", [(4, 0), (2, 1), (16, 0)])
def test_rows_that_see_nothing(orc, bits, axis):
    rng = np.random.default_rng(4)
    N = 9
    cfg, cache, keys, values = make(orc, rng, 1, 2, 2, 0, 0, bits, 32, axis)
    q, kn, vn = draft(rng, 1, 2, 2, N)
    seen = np.tril(np.ones((1, N, N), bool))
    seen[0, [0, 4]] = False
    check(cfg, cache, keys, values, q, kn, vn, seen, dev(mask_words(seen[0])))


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf, 65504.0])
@pytest.mark.parametrize("n", [0, 70])
def test_what_a_row_does_not_see_does_not_reach_it(orc, bad, n):
    """A drafted token's key and value of any content leave the rows that do not see it alone."""
    rng = np.random.default_rng(5)
    N = 37
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, n, 3, 4, 32, 0)
    q, kn, vn = draft(rng, 1, 2, 4, N)
    seen = np.tril(np.ones((1, N, N), bool))
    seen[0, :, 6] = seen[0, :, 35] = False         # padding: nobody sees them
    kn[:, :, 6] = bad
    vn[:, :, [6, 35]] = bad
    check(cfg, cache, keys, values, q, kn, vn, seen, dev(mask_words(seen[0])))
    # and one that only its own row sees
    seen[0, 36, 35] = True
    out = kvqp.tree_attn(cfg, dev(q), dev(kn), dev(vn), dev(mask_words(seen[0])), cache).cpu().numpy()
    if not np.isfinite(bad):
        assert not np.isfinite(out[:, :, 36]).any()
    assert np.isfinite(out[:, :, :36]).all()


@pytest.mark.parametrize("bits,G,axis,n_cap", [(4, 32, 0, 0), (2, 64, 1, 0), (8, 128, 1, 640), (16, 32, 0, 576), (2, 32, 0, 704)])
def test_heads_with_their_own_counts(orc, bits, G, axis, n_cap):
    rng = np.random.default_rng(6)
    B, Hkv, Gq, n, N = 2, 3, 4, 513, 6
    counts = [513, 0, 1, 100, 257, 64]
    cfg, cache, keys, values = make(orc, rng, B, Hkv, Gq, n, 15, bits, G, axis, counts=counts, n_cap=n_cap)
    q, kn, vn = draft(rng, B, Hkv, Gq, N)
    parents = [-1, 0, 0, 1, 2, 2]
    check(cfg, cache, keys, values, q, kn, vn, ancestors(parents)[None], kvqp.tree_mask(parents))


@pytest.mark.parametrize("bits,G,axis", [(4, 32, 0), (2, 128, 0), (16, 32, 0), (4, 64, 1)])
def test_long_caches_are_cut_into_splits(orc, bits, G, axis):
    rng = np.random.default_rng(7)
    for Gq, N in ((1, 1), (4, 12), (8, 30)):
        cfg, cache, keys, values = make(orc, rng, 1, 1, Gq, 6001, 50, bits, G, axis)
        q, kn, vn = draft(rng, 1, 1, Gq, N)
        ws = kvqp.alloc_tree_workspace(cfg, N)
        ws.fill_(0xFF)
        kvqp.tree_workspace_init(ws)
        check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, N, N), bool)), None, workspace=ws)


@pytest.mark.parametrize("scale", [2.0 ** -12, 1.0, 30.0])
@pytest.mark.parametrize("axis", [0, 1])
def test_small_and_large_queries(orc, scale, axis):
    """Logits of almost nothing, and a softmax that one token takes: the power of two that queries are scaled by, and references that move."""
    rng = np.random.default_rng(8)
    for bits in (2, 4, 8, 16):
        cfg, cache, keys, values = make(orc, rng, 1, 2, 2, 400, 30, bits, 32, axis if bits < 16 else 0)
        q, kn, vn = draft(rng, 1, 2, 2, 5, scale=scale)
        q[0, 0, 0] = 0
        check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, 5, 5), bool)), None)


def test_one_row_agrees_with_the_decode_step(orc):
    """One drafted token that is also the last tail row: the same softmax as kvqp_decode_attn."""
    rng = np.random.default_rng(9)
    for bits, axis in ((4, 0), (2, 0), (8, 1), (16, 0)):
        cfg, cache, keys, values = make(orc, rng, 2, 2, 4, 333, 20, bits, 32, axis)
        q = half(rng, 2, 8, 1, D)
        ref = kvqp.decode_attn(cfg, dev(q[:, :, 0]), cache)
        tail_k = cache.buffers["tail_k"].view(torch.float16).view(2, 2, -1, D)
        tail_v = cache.buffers["tail_v"].view(torch.float16).view(2, 2, -1, D)
        cache.tail_len -= 1
        out = kvqp.tree_attn(cfg, dev(q), tail_k[:, :, 19:20].contiguous(), tail_v[:, :, 19:20].contiguous(), None, cache)
        assert (out[:, :, 0].float() - ref.float()).abs().max().item() <= 2e-3


def test_the_same_bits_again_and_in_a_replayed_graph(orc):
    """Nothing depends on the order in which workgroups run; a captured call, replayed between eager ones, gives the eager result, and
    two graphs with workspaces of their own do so side by side."""
    rng = np.random.default_rng(10)
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, 3000, 32, 4, 32, 0)
    q, kn, vn = (dev(x) for x in draft(rng, 1, 2, 4, 8))
    q2 = dev(half(rng, 1, 8, 8, D))
    outs = [torch.empty_like(q) for _ in range(2)]
    lses = [torch.empty((1, 8, 8), device="cuda") for _ in range(2)]
    spaces = [kvqp.alloc_tree_workspace(cfg, 8) for _ in range(2)]
    eager = []
    for x in (q, q2):
        lse = torch.empty((1, 8, 8), device="cuda")
        eager.append((kvqp.tree_attn(cfg, x, kn, vn, None, cache, lse=lse), lse))
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for x, o, l, w, s in zip((q, q2), outs, lses, spaces, streams):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            kvqp.tree_attn(cfg, x, kn, vn, None, cache, out=o, lse=l, workspace=w)
        graphs.append(g)
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        again = kvqp.tree_attn(cfg, q, kn, vn, None, cache)
        assert torch.equal(again, eager[0][0])
        for o, l, (eo, el) in zip(outs, lses, eager):
            assert torch.equal(o, eo) and torch.equal(l, el)


def test_another_stream_and_its_own_temporaries(orc):
    rng = np.random.default_rng(11)
    cfg, cache, keys, values = make(orc, rng, 1, 1, 4, 2500, 16, 4, 32, 0)
    q, kn, vn = draft(rng, 1, 1, 4, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, 4, 4), bool)), None, stream=s)
