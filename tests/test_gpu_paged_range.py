"""Attention over pages over the range of calls: batches that are not split, long tables, windows and pieces of prompts in splits, padded batches, shared pages,
strided queries, graphs with workspaces of their own.  The oracle is plain torch in 64 bits on the GPU, batched over heads and rows."""
import dataclasses
import math
import random

import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.paged_util import BF16, D, HALF, Made, attention, near, rows, starts_of
from tests.test_gpu_paged import FORMS, check_attention, config, ints

pytestmark = pytest.mark.gpu


class Pool:
    """Random pages on the GPU (codes and scales as a quantizer leaves them), without the rows they came from."""

    def __init__(self, g, lengths, hkv, page, dtype, form, most=None):
        b = len(lengths)
        self.page, self.hkv, self.dtype = page, hkv, dtype
        most = most or max(1, -(-max(lengths) // page))
        n = b * most
        dev = "cuda"
        if form == "e4m3":      # numbers below the largest, no NaN
            codes = lambda *s: (torch.randint(0, 0x7F, s, generator=g, device=dev, dtype=torch.uint8) + 128 * torch.randint(0, 2, s, generator=g, device=dev, dtype=torch.uint8)).view(
                torch.float8_e4m3fn)
            scale = lambda: torch.exp2(torch.randint(-9, -6, (n, hkv), generator=g, device=dev).float())
        else:
            codes = lambda *s: torch.randint(-127, 128, s, generator=g, device=dev, dtype=torch.int8)
            scale = lambda: torch.exp2(torch.randint(-7, -4, (n, hkv), generator=g, device=dev).float())
        open_ = lambda: torch.randn((b, hkv, 2 * page, D), generator=g, device=dev).to(dtype)
        table = torch.randperm(n, generator=g, device=dev).to(torch.int32).view(b, most)
        self.pages = kvqp.Pages(codes(n, hkv, page, D), codes(n, hkv, D, page), scale(), scale(), open_(), open_(), table, ints(lengths))

    def numbers(self, i, t):
        p, P = self.pages, self.page
        at = p.table[i, :t // P].long()
        k = p.k_codes.view(torch.uint8)[at].view(p.k_codes.dtype).double() * p.k_scale[at].double()[..., None, None]
        v = (p.v_codes.view(torch.uint8)[at].view(p.v_codes.dtype).double() * p.v_scale[at].double()[..., None, None]).transpose(2, 3)
        k, v = (x.transpose(0, 1).reshape(self.hkv, -1, D) for x in (k, v))
        rest = torch.arange(t // P * P, t, device="cuda") % (2 * P)
        return torch.cat([k, p.open_k[i][:, rest].double()], 1), torch.cat([v, p.open_v[i][:, rest].double()], 1)

    def check(self, cfg, q, counts, window=0, starts=True, workspace=None):
        """Tolerances as in tests.paged_util.attention, with each factor replaced by its largest over a row's tokens."""
        lengths = self.pages.lengths.tolist()
        hq, gq, at = q.shape[1], q.shape[1] // self.hkv, 0
        lse = torch.full(q.shape[:2], 55.0, device="cuda")
        got = kvqp.paged_attn(cfg, self.pages, q, ints(starts_of(counts)) if starts else None, window=window, lse=lse, workspace=workspace)
        for i, m in enumerate(counts):
            t = lengths[i]
            if m == 0:
                continue
            k, v = self.numbers(i, t)
            x = q[at:at + m].double().view(m, self.hkv, gq, D).permute(1, 2, 0, 3).reshape(self.hkv, gq * m, D)
            logits = torch.matmul(x, k.transpose(1, 2).contiguous()) * cfg.sm_scale
            pos = torch.arange(t - m, t, device="cuda").repeat(gq).view(-1, 1)
            token = torch.arange(t, device="cuda")
            hidden = (token > pos) | ((token <= pos - window) if window else torch.zeros((1, t), dtype=torch.bool, device="cuda"))
            logits = logits.masked_fill(hidden, -math.inf)
            want_lse = torch.logsumexp(logits, -1)
            w = torch.softmax(logits, -1)
            want, mean = torch.matmul(w, v), torch.matmul(w, v.abs())
            d = cfg.sm_scale * (132 * 2.0 ** -24 * torch.matmul(x.abs(), k.abs().transpose(1, 2).contiguous()).amax(-1, keepdim=True)
                                + 2.0 ** -25 * x.abs().amax(-1, keepdim=True) * k.abs().sum(-1).amax(-1).view(-1, 1, 1))
            steps = (t / 32 + 80) * 2.0 ** -24
            off = (2.0 ** -11 + 2 * d + 2 * steps) * mean + t * 2.0 ** -28 * w.amax(-1, keepdim=True) * v.abs().amax(1, keepdim=True)
            back = lambda y: y.view(self.hkv, gq, m, -1).permute(2, 0, 1, 3).reshape(m, hq, -1)
            near(got[at:at + m], back(want).cpu(), back(off).cpu(), self.dtype)
            far = (lse[at:at + m].double() - back(want_lse.unsqueeze(-1)).squeeze(-1)).abs()
            assert bool((far <= back(d).squeeze(-1) + steps + 2.0 ** -22 * back(want_lse.unsqueeze(-1)).squeeze(-1).abs()).all())
            at += m
        return got


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("b,hkv,gq,page,tokens,count,window", [(1, 8, 4, 16, 9001, 1, 0), (1, 1, 8, 16, 20011, 3, 0), (3, 2, 8, 32, 7013, 5, 0), (2, 4, 4, 64, 5003, 8, 1000), (1, 2, 1, 16, 17000, 40, 0),
                                                               (2, 2, 4, 16, 9500, 700, 0), (1, 8, 8, 64, 3001, 333, 0), (2, 16, 1, 32, 6001, 250, 517), (40, 1, 2, 16, 600, 1, 0)])
def test_long_sequences(dtype, form, b, hkv, gq, page, tokens, count, window):
    g = generator(b + tokens)
    lengths = [max(count, tokens - 1777 * i % tokens) for i in range(b)]
    pool = Pool(g, lengths, hkv, page, dtype, form)
    q = torch.randn((b * count, hkv * gq, D), generator=g, device="cuda").to(dtype)
    pool.check(config(b, hkv * gq, hkv), q, [count] * b, window, starts=count > 1)


def test_more_sequences_than_are_split():
    """600 of them, and 300 of one head (looked at in two turns)."""
    for b, hkv, most in ((600, 2, 300), (300, 1, 500), (512, 1, 330)):
        g = generator(b)
        lengths = [1 + (i * 7919) % most for i in range(b)]
        pool = Pool(g, lengths, hkv, 16, HALF, "e4m3")
        counts = [0 if i % 7 == 3 else min(1 + i % 3, lengths[i]) for i in range(b)]
        q = torch.randn((sum(counts), 2 * hkv, D), generator=g, device="cuda").to(HALF)
        pool.check(config(b, 2 * hkv, hkv), q, counts)
        q = torch.randn((b, 2 * hkv, D), generator=g, device="cuda").to(HALF)
        pool.check(config(b, 2 * hkv, hkv), q, [1] * b, starts=False)


def test_random_calls():
    r, g = random.Random(5), generator(77)
    for _ in range(25):
        hkv, gq, page = r.choice((1, 2, 4)), r.choice((1, 2, 4, 8)), r.choice((16, 32, 64))
        dtype, form = r.choice(FORMS)
        b = r.choice((1, 2, 5, 20))
        lengths = [int(round(math.exp(r.uniform(0, math.log(4000 // b + 64))))) for _ in range(b)]
        counts = [min(t, r.choice((0, 1, 2, 7, 65, t))) for t in lengths]
        window = r.choice((0, 0, r.randint(1, 300)))
        print(f"  b={b} hkv={hkv} gq={gq} page={page} {dtype} {form} lengths={lengths} counts={counts} window={window}", flush=True)
        if not sum(counts):
            continue
        pool = Pool(g, lengths, hkv, page, dtype, form, most=max(1, -(-max(lengths) // page)) + r.choice((0, 40)))
        pool.check(config(b, hkv * gq, hkv), torch.randn((sum(counts), hkv * gq, D), generator=g, device="cuda").to(dtype), counts, window)


def test_padded_batches_and_strided_queries():
    g = generator(3)
    pool = Pool(g, [300, 17, 90], 2, 16, BF16, "e4m3")
    cfg = config(3, 8, 2)
    fused = torch.randn((9, 12 * D), generator=g, device="cuda").to(BF16)
    q = fused[:, 2 * D:10 * D].unflatten(1, (8, D))
    starts = ints([0, 2, 2, 5])                       # rows 5 .. 8 are nobody's
    out, lse = torch.full((9, 8, D), 4.0, dtype=BF16, device="cuda"), torch.full((9, 8), 4.0, device="cuda")
    kvqp.paged_attn(cfg, pool.pages, q, starts, out=out, lse=lse)
    assert bool((out[5:] == 4).all()) and bool((lse[5:] == 4).all())
    want = kvqp.paged_attn(cfg, pool.pages, q[:5].contiguous(), starts)
    assert torch.equal(out[:5], want)


def test_shared_pages():
    """Two sequences that begin alike read the same pages, a third one the same open rows in a place of their own."""
    g = torch.Generator().manual_seed(4)
    made = Made(g, [100, 100], 2, 16)
    made.table[1, :5] = made.table[0, :5]
    for i in (0, 1):
        made.k[1][:, :80], made.v[1][:, :80] = made.k[0][:, :80], made.v[0][:, :80]
        made.put(i, 0, 100)
    check_attention(config(2, 4, 2), made, made.pages(), rows(g, 5, 4, D), [3, 2], 0)


def test_two_graphs_with_workspaces_of_their_own():
    g = generator(6)
    pool = Pool(g, [4000, 2500], 2, 16, HALF, "int8")
    cfg = config(2, 8, 2)
    graphs, outs, qs = [], [], []
    for i in range(2):
        q, ws = torch.zeros((2, 8, D), dtype=HALF, device="cuda"), kvqp.alloc_paged_workspace(cfg, 2)
        out = torch.empty_like(q)
        kvqp.paged_attn(cfg, pool.pages, q, out=out, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            kvqp.paged_attn(cfg, pool.pages, q, out=out, workspace=ws)
        graphs.append((graph, ws)), outs.append(out), qs.append(q)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for step in range(4):
        want = []
        for q in qs:
            q.copy_(torch.randn((2, 8, D), generator=g, device="cuda"))
            want.append(kvqp.paged_attn(cfg, pool.pages, q))      # (eager work between the replays)
        torch.cuda.synchronize()
        for (graph, _), out, s in zip(graphs, outs, streams):
            out.zero_()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_lengths_out_of_range_stay_in_the_buffers():
    """What the device arrays say is cut to what there is: no result is stated, but nothing beside the outputs changes, and the next call is right."""
    g = generator(8)
    pool = Pool(g, [64, 50], 2, 16, HALF, "e4m3")
    cfg, ws = config(2, 4, 2), kvqp.alloc_paged_workspace(config(2, 4, 2), 6)
    q = torch.randn((6, 4, D), generator=g, device="cuda").to(HALF)
    for lengths, starts in (([1 << 30, -5], [0, 3, 6]), ([64, 50], [0, 9, 6]), ([64, 50], [5, 2, 4]), ([2, 50], [0, 5, 6]), ([64, 50], [-3, 1, 100])):
        pool.pages.lengths.copy_(ints(lengths))
        guard = torch.full((3, 6, 4, D), 9.0, dtype=HALF, device="cuda")
        kvqp.paged_attn(cfg, pool.pages, q, ints(starts), out=guard[1], workspace=ws)
        assert bool((guard[[0, 2]] == 9).all())
    pool.pages.lengths.copy_(ints([64, 50]))
    pool.check(cfg, q, [3, 3], workspace=ws)


def test_a_sequence_of_open_tokens_alone_and_empty_calls():
    g = generator(9)
    pool = Pool(g, [13, 0, 5], 2, 64, BF16, "int8")
    cfg = config(3, 8, 2)
    q = torch.randn((18, 8, D), generator=g, device="cuda").to(BF16)
    pool.check(cfg, q, [13, 0, 5])
    assert kvqp.paged_attn(cfg, pool.pages, q[:0], ints([0, 0, 0, 0])).shape == (0, 8, D)
    lse = torch.zeros((3, 8), device="cuda")
    out = kvqp.paged_attn(cfg, pool.pages, q[:3], lse=lse)
    assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all()) and bool(torch.isfinite(lse[[0, 2]]).all())


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page", [16, 32])
def test_pages_before_a_window_may_be_anybodys(dtype, form, page):
    """What the table names before every row's window holds NaN codes and scales of every kind: it reaches nobody.  Few rows, and a piece of a prompt."""
    for count, window in ((1, 100), (5, 70), (200, 130), (300, 40)):
        g = generator(page + count)
        pool = Pool(g, [1000], 2, page, dtype, form, most=80)
        q = torch.randn((count, 8, D), generator=g, device="cuda").to(dtype)
        cfg, p = config(1, 8, 2), pool.pages
        want = pool.check(cfg, q, [count], window)
        gone = p.table[0, :(1000 - count - window + 1) // page].long()
        p.k_codes.view(torch.uint8)[gone], p.v_codes.view(torch.uint8)[gone] = 0x7F, 0x7F
        for i, x in enumerate((math.nan, math.inf, 2.0 ** 100)):
            p.k_scale[gone[i::3]], p.v_scale[gone[i::3]] = x, x
        got = kvqp.paged_attn(cfg, p, q, ints([0, count]), window=window)
        assert torch.equal(got, want)


def test_a_window_beyond_every_token_is_none():
    g = generator(12)
    pool = Pool(g, [700, 90], 2, 16, HALF, "e4m3", most=50)
    cfg, q = config(2, 8, 2), torch.randn((400, 8, D), generator=g, device="cuda").to(HALF)
    want = pool.check(cfg, q, [330, 70])
    for window in (800, 1 << 30, (1 << 31) - 1):
        assert torch.equal(kvqp.paged_attn(cfg, pool.pages, q, ints([0, 330, 400]), window=window), want)


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page", [16, 32, 64])
def test_loads_past_the_memory_side_cache_give_the_same(dtype, form, page):
    """decode_cache_hint is about time alone: a step, drafted rows, holes in the table, a window."""
    g = generator(page)
    pool = Pool(g, [1500, 1, 77, 640], 2, page, dtype, form)
    pool.pages.table[0, 3], pool.pages.table[3, 1] = -1, 1 << 20
    for counts, window in (([1] * 4, 0), ([2, 1, 0, 2], 0), ([1] * 4, 200), ([7, 1, 5, 8], 90)):
        q = torch.randn((sum(counts), 16, D), generator=g, device="cuda").to(dtype)
        got = [kvqp.paged_attn(dataclasses.replace(config(4, 16, 2), decode_cache_hint=hint), pool.pages, q, ints(starts_of(counts)), window=window) for hint in (0, 1, 2)]
        assert torch.equal(got[0], got[1]) and torch.equal(got[1], got[2]) and bool(torch.isfinite(got[0]).all())
    pool = Pool(g, [1500, 1, 77, 640], 2, page, dtype, form)
    pool.check(dataclasses.replace(config(4, 8, 2), decode_cache_hint=1), torch.randn((4, 8, D), generator=g, device="cuda").to(dtype), [1] * 4)


@pytest.mark.parametrize("hkv,gq,lengths,n,starts", [
    (1, 4, [22820, 48308, 37470], 48, [[0, 48, 0, 48], [48, 0, 48, 0], [-5, 48, 20, 100]]),                    # one tile of 16 rows and two
    (8, 4, [3000 + 517 * i for i in range(20)], 64, [[0, 64] * 10 + [0], [64, 0] * 10 + [64], [5 * i % 64 for i in range(21)]]),
    (2, 8, [9000, 4000, 12000, 7000], 700, [[0, 700, 0, 700, 0], [0, 350, 300, 700, 650], [700, 0, 700, 699, 700]]),      # tiles of many rows
    (1, 1, [300 + 37 * i for i in range(300)], 300, [[i % 2 * 300 for i in range(301)], list(range(300, -1, -1))])])      # (looked at in two turns)
def test_starts_that_descend_leave_the_workspace_as_it_was(hkv, gq, lengths, n, starts):
    """No result is stated for them, but the arrival counters are zero afterwards, and calls that share the workspace are right."""
    g, b = generator(hkv + n), len(lengths)
    pool = Pool(g, lengths, hkv, 16, HALF, "e4m3")
    cfg = config(b, hkv * gq, hkv)
    q = torch.randn((n, hkv * gq, D), generator=g, device="cuda").to(HALF)
    ws = kvqp.alloc_paged_workspace(cfg, n)
    counts = [n // b + (i < n % b) for i in range(b)]
    want = kvqp.paged_attn(cfg, pool.pages, q, ints(starts_of(counts)), workspace=ws)
    for bad in starts:
        guard = torch.full((3, n, hkv * gq, D), 9.0, dtype=HALF, device="cuda")
        kvqp.paged_attn(cfg, pool.pages, q, ints(bad), out=guard[1], workspace=ws)
        assert bool((guard[[0, 2]] == 9).all()) and bool((ws[:16384] == 0).all())
        assert torch.equal(kvqp.paged_attn(cfg, pool.pages, q, ints(starts_of(counts)), workspace=ws), want)
    pool.check(cfg, q, counts, workspace=ws)


@pytest.mark.parametrize("hkv,gq", [(400, 1), (385, 2), (513, 1)])
def test_more_heads_than_shares(hkv, gq):
    """Few rows are split by one share a head, or not at all, many rows not at all; one workspace, made for the most rows, serves all."""
    g = generator(hkv)
    pool = Pool(g, [1300], hkv, 16, HALF, "e4m3")
    cfg = config(1, hkv * gq, hkv)
    ws = kvqp.alloc_paged_workspace(cfg, 140)
    for n in (140, 1, 20):
        pool.check(cfg, torch.randn((n, hkv * gq, D), generator=g, device="cuda").to(HALF), [n], workspace=ws)
    assert bool((ws[:16384] == 0).all())


@pytest.mark.parametrize("dtype,form", [(HALF, "int8"), (BF16, "e4m3")])
@pytest.mark.parametrize("hkv,gq,page,lengths,counts,window", [
    (1, 1, 16, [20011], [70], 0), (1, 4, 32, [20011], [130], 0),           # 79 splits of a piece: four sixteens and a fifteen
    (1, 1, 16, [4300], [128], 0), (1, 1, 16, [4300], [5], 0), (1, 8, 64, [8400], [3], 0),      # 17 and 33: one is left over
    (1, 1, 64, [70003], [129], 0), (1, 2, 16, [70003], [3], 0),            # 274
    (1, 2, 16, [30000, 11000], [90, 40], 0), (2, 4, 32, [900, 41000, 5], [40, 70, 3], 0), (1, 4, 64, [50000, 300], [200, 9], 30000)])
def test_joins_of_more_than_sixteen_splits(dtype, form, hkv, gq, page, lengths, counts, window):
    """By sixteens first, and then theirs, for one, two and eight tiles of rows; again with the workspace as that left it."""
    g = generator(sum(lengths) + gq)
    pool = Pool(g, lengths, hkv, page, dtype, form)
    cfg = config(len(lengths), hkv * gq, hkv)
    ws = kvqp.alloc_paged_workspace(cfg, sum(counts))
    q = torch.randn((sum(counts), hkv * gq, D), generator=g, device="cuda").to(dtype)
    first = pool.check(cfg, q, counts, window, workspace=ws)
    assert bool((ws[:16384] == 0).all()) and torch.equal(kvqp.paged_attn(cfg, pool.pages, q, ints(starts_of(counts)), window=window, workspace=ws), first)


@pytest.mark.parametrize("count", [1, 40])
def test_a_captured_call_makes_its_own_workspace(count):
    """Without a workspace a captured call has one of the graph's memory, prepared by every replay; on the current stream, and on the capturing one by name."""
    g = generator(10 + count)
    pool = Pool(g, [9000, 300], 2, 16, BF16, "e4m3")
    cfg, starts = config(2, 8, 2), ints([0, count, 2 * count])
    q = torch.zeros((2 * count, 8, D), dtype=BF16, device="cuda")
    kvqp.paged_attn(cfg, pool.pages, q, starts)
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        first = kvqp.paged_attn(cfg, pool.pages, q, starts)
        second = kvqp.paged_attn(cfg, pool.pages, q, starts, stream=s)
    for _ in range(4):
        q.copy_(torch.randn(q.shape, generator=g, device="cuda"))
        want = kvqp.paged_attn(cfg, pool.pages, q, starts)
        first.zero_(), second.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(first, want) and torch.equal(second, want)
