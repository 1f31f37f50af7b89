"""Several query rows and eviction over the range of calls: the hints about caching, launches that many heads and long heads lead
to, one workspace for unlike calls, rows that hold anything."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev
from tests.rows_util import D, attention, half, logit_error, make, out_error
from tests.test_gpu_evict import check as check_evict
from tests.test_gpu_evict import target
from tests.test_gpu_tree import check as check_tree
from tests.test_gpu_tree import draft
from tests.test_gpu_weights import run as check_weights

pytestmark = pytest.mark.gpu


def chain(N):
    return np.tril(np.ones((1, N, N), bool))


def many(cfg, cache, heads):
    """The one head of a cache, for so many batch items."""
    c = kvqp.Cfg(**{**cfg.__dict__, "batch": heads})
    return c, kvqp.Cache({k: t.repeat(heads) for k, t in cache.buffers.items()}, cache.n_kept, cache.tail_len, cache.tail_cap, cache.n_cap)


@pytest.mark.parametrize("bits,axis", [(2, 0), (4, 0), (8, 0), (16, 0), (2, 1), (4, 1), (8, 1)])
def test_hints_change_no_bit(orc, bits, axis):
    """What the calls compute does not depend on which caches their loads go through."""
    rng = np.random.default_rng(31)
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, 1500, 20, bits, 32, axis)
    for N in (3, 7, 16):           # one, two and four tiles of rows
        q, kn, vn = draft(rng, 1, 2, 4, N)
        got = []
        for hint in (kvqp.CACHE_AUTO, kvqp.CACHE_STREAM, kvqp.CACHE_KEEP):
            c = kvqp.Cfg(**{**cfg.__dict__, "decode_cache_hint": hint})
            out, lse = check_tree(c, cache, keys, values, q, kn, vn, chain(N), None)
            got.append((out, lse, check_weights(c, cache, keys, [1500, 1500], 20, q, 0.5)))
        for other in got[1:]:
            assert all(np.array_equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("bits,axis", [(4, 0), (2, 0), (8, 1), (16, 0)])
def test_one_workspace_for_unlike_calls(orc, bits, axis):
    """Calls of other row counts, token counts and heads, in turn, with the workspace that the largest of them asks for."""
    rng = np.random.default_rng(32)
    made = [make(orc, rng, *shape, bits, 32, axis) + (shape[2], N) for shape, N in
            [((1, 1, 4, 3000, 40), 9), ((1, 2, 8, 900, 3), 20), ((3, 2, 1, 700, 0), 1), ((1, 1, 8, 40, 0), 33)]]
    size = max(kvqp.tree_workspace_bytes(m[0], m[5]) for m in made)
    ws = kvqp.tree_workspace_init(kvqp.alloc_workspace(size))
    for order in ((0, 1, 2, 3), (1, 0, 3, 0, 2, 1)):
        for i in order:
            cfg, cache, keys, values, Gq, N = made[i]
            q, kn, vn = draft(rng, cfg.batch, cfg.n_kv_heads, Gq, N)
            check_tree(cfg, cache, keys, values, q, kn, vn, chain(N), None, workspace=ws)
    assert not ws[:4096].any()          # every launch leaves the counters as it found them


@pytest.mark.parametrize("bits,axis", [(4, 0), (2, 0), (8, 0), (16, 0), (4, 1), (2, 1)])
@pytest.mark.parametrize("Gq,N", [(1, 4), (8, 4), (8, 11)])
def test_every_head_of_many_long_ones(orc, bits, axis, Gq, N):
    """A workgroup to a whole head, more than sixteen blocks to a wave: the result is the same for each of many equal heads, and the formula's."""
    rng = np.random.default_rng(33)
    heads = 160 if N < 11 else 90
    cfg, one, keys, values = make(orc, rng, 1, 1, Gq, 7003, 33, bits, 64, axis)
    c, cache = many(cfg, one, heads)
    q, kn, vn = draft(rng, 1, 1, Gq, N)
    lse = torch.empty((heads, Gq, N), device="cuda")
    out = kvqp.tree_attn(c, *(dev(np.repeat(x, heads, 0)) for x in (q, kn, vn)), None, cache, lse=lse)
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    k64, v64 = (np.concatenate([a[0], b[0, 0].astype(np.float64)]) for a, b in ((keys, kn), (values, vn)))
    seen = np.concatenate([np.ones((N, 7003 + 33), bool), chain(N)[0]], 1)
    for a in range(Gq):
        rows = q[0, a].astype(np.float64)
        ref, ref_lse, spread = attention(rows, k64, v64, seen)
        delta = logit_error(rows, k64)
        assert (np.abs(out[0, a].cpu().numpy() - ref) <= out_error(ref, spread, delta)).all()
        assert (np.abs(lse[0, a].cpu().numpy() - ref_lse) <= delta + 2.0 ** -18 + 2.0 ** -23 * np.abs(ref_lse)).all()


@pytest.mark.parametrize("bits,axis", [(4, 0), (2, 0), (16, 0), (8, 1)])
@pytest.mark.parametrize("N", [2, 5, 70])
def test_weights_of_many_long_heads(orc, bits, axis, N):
    rng = np.random.default_rng(34)
    heads, n = 512, 4500
    cfg, one, keys, _ = make(orc, rng, 1, 1, 4, n, 70, bits, 32, axis)
    q = half(rng, 1, 4, N, D)
    ref = check_weights(cfg, one, keys, [n], 70, q, 0.0)
    c, cache = many(cfg, one, heads)
    _, _, lse = weigh(cfg, one, q)
    w = torch.full((heads, 1, n + 70), 3.0, device="cuda")
    kvqp.accumulate_weights(c, dev(np.repeat(q, heads, 0)), lse.repeat(heads, 1, 1), cache, w, decay=0.0)
    single = torch.full((1, 1, n + 70), 3.0, device="cuda")
    kvqp.accumulate_weights(cfg, dev(q), lse, one, single, decay=0.0)
    assert torch.equal(w, single.expand(heads, 1, n + 70))
    assert np.isfinite(ref).all()


def weigh(cfg, cache, q):
    """Sums of the rows' softmax over the cache alone (each drafted row hidden from all)."""
    N = q.shape[2]
    kn = torch.zeros((1, cfg.n_kv_heads, N, D), dtype=torch.float16, device="cuda")
    lse = torch.empty((1, cfg.n_q_heads, N), device="cuda")
    mask = torch.zeros((N, (N + 31) // 32), dtype=torch.int32, device="cuda")
    return kvqp.tree_attn(cfg, dev(q), kn, kn, mask, cache, lse=lse), mask, lse


@pytest.mark.parametrize("bits,axis", [(4, 0), (8, 1), (16, 0)])
def test_weights_of_heads_with_very_unlike_counts(orc, bits, axis):
    rng = np.random.default_rng(35)
    counts = [4001, 1, 0, 33, 2000, 4000]
    cfg, cache, keys, _ = make(orc, rng, 2, 3, 2, 4001, 35, bits, 32, axis, counts=counts)
    for N in (3, 20, 40):
        check_weights(cfg, cache, keys, counts, 35, half(rng, 2, 6, N, D), 0.9)


def test_rows_that_saw_nothing_may_hold_anything(orc):
    """A padded row (its sum is -inf) adds nothing to the weights, whatever its query holds."""
    rng = np.random.default_rng(36)
    for N, bits, axis in ((3, 4, 0), (6, 2, 1), (18, 16, 0), (40, 8, 0)):
        cfg, cache, keys, _ = make(orc, rng, 1, 2, 4, 300, 50, bits, 32, axis)
        q = half(rng, 1, 8, N, D)
        lse = torch.full((1, 8, N), 6.0, device="cuda")
        lse[0, 3, 1] = lse[0, 5] = -torch.inf
        q0, q1 = q.copy(), q.copy()
        q0[0, 3, 1] = q0[0, 5] = 0
        q1[0, 3, 1] = np.nan
        q1[0, 5] = np.inf
        a, b = (kvqp.accumulate_weights(cfg, dev(x), lse, cache, torch.zeros((1, 2, 350), device="cuda")) for x in (q0, q1))
        assert torch.equal(a, b) and torch.isfinite(a).all()


def test_a_scale_of_almost_nothing(orc):
    """Every visible token has the same weight then, and the others none."""
    rng = np.random.default_rng(37)
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, 45, 3, 4, 32, 0)
    c = kvqp.Cfg(**{**cfg.__dict__, "sm_scale": 1.2e-38})
    q, kn, vn = draft(rng, 1, 2, 4, 6, scale=2.0 ** -12)
    lse = torch.empty((1, 8, 6), device="cuda")
    out = kvqp.tree_attn(c, dev(q), dev(kn), dev(vn), None, cache, lse=lse).cpu().numpy().astype(np.float64)
    for h in range(8):
        for i in range(6):
            v = np.concatenate([values[h // 4], vn[0, h // 4, :i + 1].astype(np.float64)])
            # (the mean: values rounded once, the output once, 60 sums in binary32)
            assert np.abs(out[0, h, i] - v.mean(0)).max() <= 2.0 ** -11 * (np.abs(v).mean(0) + np.abs(v.mean(0))).max() + 2.0 ** -17 * np.abs(v).max()
            assert abs(lse[0, h, i].item() - np.log(len(v))) <= 2.0 ** -18


@pytest.mark.parametrize("n,unit,n_keep,bits,G,axis", [(9000, 1, 5000, 2, 64, 1), (33100, 1, 20001, 2, 128, 1), (40003, 1, 777, 4, 32, 1),
                                                       (33100, 32, 30010, 4, 32, 0), (70000, 64, 2000, 2, 64, 0), (33500, 1, 33499, 16, 32, 0)])
def test_evictions_from_long_heads(orc, n, unit, n_keep, bits, G, axis):
    """More units than a workgroup's keys of one, eight and thirty-two to a thread."""
    rng = np.random.default_rng(38)
    cfg, src, _, _ = make(orc, rng, 1, 1, 1, n, 3, bits, G, axis)
    w = np.exp(rng.standard_normal((1, 1, n + 3))).astype(np.float32)
    w[0, 0, rng.integers(0, n, n // 10)] = 1.0            # (ties at the cut)
    short = n % unit
    kept = short + (n_keep - short) // unit * unit
    check_evict(orc, cfg, src, w, n_keep, unit, [n], target(cfg, kept, 3, 0), 3)


@pytest.mark.parametrize("kind", ["zeros", "two values", "nan", "infinite", "different"])
@pytest.mark.parametrize("n,unit,n_keep", [(1, 1, 1), (63, 1, 20), (130, 1, 65), (256, 1, 255), (257, 1, 100), (300, 64, 65), (8192, 32, 4000), (8250, 32, 8193), (1025, 1, 1024)])
def test_ties_among_few_units(orc, kind, n, unit, n_keep):
    rng = np.random.default_rng(39)
    shape = (1, 2, n + 3)
    cfg, src, _, _ = make(orc, rng, 1, 2, 1, n, 3, 4, 32, 1)
    w = {"zeros": lambda: np.zeros(shape), "two values": lambda: rng.integers(0, 2, shape) * 0.25, "nan": lambda: np.where(rng.random(shape) < 0.02, np.nan, rng.integers(0, 3, shape)),
         "infinite": lambda: np.where(rng.random(shape) < 0.05, np.inf, 1.0), "different": lambda: np.exp(2 * rng.standard_normal(shape))}[kind]().astype(np.float32)
    short = n % unit
    kept = n if n <= n_keep else short + (n_keep - short) // unit * unit
    check_evict(orc, cfg, src, w, n_keep, unit, [n] * 2, target(cfg, kept, 3, 0), 3)


@pytest.mark.parametrize("bits,axis,N", [(4, 0, 3), (2, 1, 6), (16, 0, 15), (8, 0, 30)])
def test_a_row_of_anything_stays_alone(orc, bits, axis, N):
    """A padded row's query may hold NaN or infinities: the other rows' results are the same bits."""
    rng = np.random.default_rng(40)
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, 1200, 20, bits, 32, axis)
    q, kn, vn = draft(rng, 1, 2, 4, N)
    out, lse = check_tree(cfg, cache, keys, values, q, kn, vn, chain(N), None)
    bad = q.copy()
    bad[0, 2, 1] = np.nan
    bad[0, 6, 0, 5] = np.inf
    bad[0, 7, N - 1] = -np.inf
    lse2 = torch.empty((1, 8, N), device="cuda")
    out2 = kvqp.tree_attn(cfg, dev(bad), dev(kn), dev(vn), None, cache, lse=lse2).cpu().numpy().astype(np.float64)
    same = np.ones((8, N), bool)
    same[2, 1] = same[6, 0] = same[7, N - 1] = False
    assert np.array_equal(out2[0][same], out[0][same]) and np.array_equal(lse2.cpu().numpy()[0][same], lse[0][same])
    assert not np.isfinite(out2[0][~same]).any()


def test_captured_calls_that_make_their_own_workspaces(orc):
    rng = np.random.default_rng(41)
    cfg, cache, keys, values = make(orc, rng, 1, 2, 4, 2600, 32, 4, 32, 1)
    q, kn, vn = (dev(x) for x in draft(rng, 1, 2, 4, 8))
    w = dev(np.exp(rng.standard_normal((1, 2, 2640))).astype(np.float32))
    eager, into = kvqp.tree_attn(cfg, q, kn, vn, None, cache), [target(cfg, 2000, 32, 0) for _ in range(2)]
    kvqp.evict(cfg, cache, w, 2000, into[0])
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        kvqp.tree_attn(cfg, q, kn, vn, None, cache, out=out)
        kvqp.evict(cfg, cache, w, 2000, into[1])
        again = kvqp.tree_attn(cfg, q, kn, vn, None, cache)
    for _ in range(4):
        out.zero_()
        for t in into[1].buffers.values():
            t.zero_()
        g.replay()
        assert torch.equal(kvqp.tree_attn(cfg, q, kn, vn, None, cache), eager)
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(again, eager)
        for k, t in into[0].buffers.items():
            assert torch.equal(t, into[1].buffers[k]), k


@pytest.mark.parametrize("bits,G,axis,unit,ragged", [(4, 32, 0, 1, False), (2, 64, 1, 1, True), (8, 128, 0, 128, False), (16, 32, 0, 32, True), (2, 32, 0, 1, True)])
def test_evictions_from_a_layout_with_room(orc, bits, G, axis, unit, ragged):
    """src laid out for more tokens than it has (n_cap), dst for others again."""
    rng = np.random.default_rng(42)
    counts = [450, 449, 0, 300] if ragged else [450] * 4
    cfg, src, _, _ = make(orc, rng, 2, 2, 1, 450, 6, bits, G, axis, counts=counts if ragged else None, n_cap=640)
    w = np.exp(2 * rng.standard_normal((2, 2, 470))).astype(np.float32)
    check_evict(orc, cfg, src, w, 333, unit, counts, target(cfg, 384, 9, 384, ragged=ragged), 6)


def test_caches_of_more_than_four_gigabytes(orc):
    """Heads whose codes begin past 2^32 bytes."""
    rng = np.random.default_rng(43)
    heads, n, N = 600, 30000, 2
    cfg, one, keys, values = make(orc, rng, 1, 1, 2, n, 5, 16, 32, 0)
    c, cache = many(cfg, one, heads)
    assert cache.buffers["k_codes"].numel() > 1 << 32
    q, kn, vn = draft(rng, 1, 1, 2, N)
    k64, v64 = (np.concatenate([a[0], b[0, 0].astype(np.float64)]) for a, b in ((keys, kn), (values, vn)))
    lse = torch.empty((heads, 2, N), device="cuda")
    out = kvqp.tree_attn(c, *(dev(np.repeat(x, heads, 0)) for x in (q, kn, vn)), None, cache, lse=lse)
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    seen = np.concatenate([np.ones((N, n + 5), bool), chain(N)[0]], 1)
    for a in range(2):
        rows = q[0, a].astype(np.float64)
        ref, ref_lse, spread = attention(rows, k64, v64, seen)
        assert (np.abs(out[-1, a].cpu().numpy() - ref) <= out_error(ref, spread, logit_error(rows, k64))).all()
    lse1 = torch.full((1, 2, N), 10.0, device="cuda")
    w1 = kvqp.accumulate_weights(cfg, dev(q), lse1, one, torch.zeros((1, 1, n + 5), device="cuda"))
    w = kvqp.accumulate_weights(c, dev(np.repeat(q, heads, 0)), lse1.repeat(heads, 1, 1), cache, torch.zeros((heads, 1, n + 5), device="cuda"))
    assert torch.equal(w, w1.expand_as(w))
    single, dst = target(cfg, 29000, 5, 0), target(c, 29000, 5, 0)
    kvqp.evict(cfg, one, w1, 29000, single)
    kvqp.evict(c, cache, w, 29000, dst)
    for name in ("k_codes", "v_codes", "tail_k", "tail_v"):
        a = dst.buffers[name].view(heads, -1)
        b = single.buffers[name].view(1, -1)
        if name.startswith("tail"):       # (the rest of the room for tail rows is left alone)
            a, b = a[:, :5 * 256], b[:, :5 * 256]
        assert torch.equal(a, b.expand_as(a)), name


def test_a_cache_without_room_is_refused(orc):
    rng = np.random.default_rng(44)
    cfg, src, _, _ = make(orc, rng, 1, 2, 1, 300, 5, 4, 32, 1)
    w = dev(np.ones((1, 2, 305), np.float32))
    for n_layout, tail_cap in ((128, 5), (200, 4)):
        dst = target(cfg, n_layout, tail_cap, 0)
        dst.tail_cap = 5
        with pytest.raises(ValueError, match="no room"):
            kvqp.evict(cfg, src, w, 200, dst)
    assert kvqp.evict(cfg, src, w, 200, target(cfg, 200, 5, 0)).n_kept == 200
