"""The paged cache of 8-bit codes: appending (bit for bit the definition), attention (against 64 bits), reading back."""
import math

import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.paged_util import BF16, D, HALF, Made, attention, finite, near, quantized, rotated, rows, starts_of

pytestmark = pytest.mark.gpu
FORMS = [(HALF, "e4m3"), (BF16, "int8"), (HALF, "int8"), (BF16, "e4m3")]


def config(b, hq, hkv, scale=D ** -0.5):
    return kvqp.Cfg(batch=b, n_q_heads=hq, n_kv_heads=hkv, sm_scale=scale)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- appending ----

def arrive(made, g, counts, rope, hq, positions=None, special=None):
    """New rows of every sequence: on the CPU by the definition (made then holds them), returned as the call takes them."""
    hkv, dtype = made.hkv, made.dtype
    n = sum(counts)
    q, k, v = rows(g, n, hq, D, dtype=dtype), rows(g, n, hkv, D, dtype=dtype, by=3.0), rows(g, n, hkv, D, dtype=dtype)
    if special:
        special(q, k, v)
    owner = torch.repeat_interleave(torch.arange(len(counts)), torch.tensor(counts))
    at = torch.cat([torch.arange(t, t + m) for t, m in zip(made.lengths, counts)]) if n else torch.zeros(0, dtype=torch.long)
    p = at if positions is None else positions
    kr, qr = k.float(), q.float()
    if rope is not None:
        table = rope.table.cpu()
        kr = rotated(kr, p[:, None].expand(n, hkv), table, rope.rot_dim, rope.interleaved)
        qr = rotated(qr, p[:, None].expand(n, hq), table, rope.rot_dim, rope.interleaved)
    kr, vr, qr = finite(kr, dtype), finite(v.float(), dtype), qr.to(dtype)
    for i, m in enumerate(counts):
        t = made.lengths[i]
        made.k[i] = torch.cat([made.k[i], kr[owner == i].transpose(0, 1)], 1)
        made.v[i] = torch.cat([made.v[i], vr[owner == i].transpose(0, 1)], 1)
        made.put(i, t, t + m)
        made.lengths[i] = t + m
    return q, k, v, qr


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,lengths,counts,hq,hkv", [(16, [0, 15, 16, 31], [1, 1, 1, 1], 4, 2), (16, [5, 0, 100, 47], [3, 40, 0, 17], 8, 1), (32, [0, 31, 70], [64, 1, 90], 2, 2),
                                                        (64, [10, 63, 129], [200, 65, 0], 8, 4), (16, [7], [80], 1, 1), (32, [3, 35], [95, 64], 4, 4)])
def test_append_is_the_definition(dtype, form, page, lengths, counts, hq, hkv):
    g = torch.Generator().manual_seed(page + len(lengths) + sum(counts))
    made = Made(g, lengths, hkv, page, dtype, form, extra_pages=-(-max(counts) // page) + 1)
    rope = kvqp.rope_table(400, kvqp.rope_frequencies(64 if page == 32 else 128), interleaved=page == 16)
    pages = made.pages()
    q, k, v, want_q = arrive(made, g, counts, rope, hq)
    pages.lengths.copy_(ints(made.lengths))
    single = all(n == 1 for n in counts)
    got = kvqp.paged_append(config(len(lengths), hq, hkv), pages, k.cuda(), v.cuda(), None if single else ints(starts_of(counts)), q=q.cuda(), rope=rope)
    assert torch.equal(got.cpu(), want_q)
    made.same(pages)


def test_a_blocks_codes_do_not_depend_on_the_calls():
    g = torch.Generator().manual_seed(3)
    cfg, total = config(1, 2, 2), 75
    k, v = rows(g, total, 2, D).cuda(), rows(g, total, 2, D).cuda()
    rope = kvqp.rope_table(100, kvqp.rope_frequencies())
    results = []
    for cuts in ([75], [1] * 75, [15, 2, 40, 18], [33, 42]):
        pages = kvqp.alloc_pages(cfg, 8, 5)
        pages.table.copy_(ints([[3, 1, 7, 0, 2]]))
        for x in (pages.k_codes, pages.v_codes):
            x.view(torch.uint8).zero_()
        for x in (pages.k_scale, pages.v_scale, pages.open_k, pages.open_v):
            x.zero_()
        at = 0
        for n in cuts:
            pages.lengths.fill_(at + n)
            kvqp.paged_append(cfg, pages, k[at:at + n], v[at:at + n], ints([0, n]), rope=rope)
            at += n
        results.append(pages)
    for name in Made.NAMES:
        for other in results[1:]:
            a, b = (getattr(r, name) for r in (results[0], other))
            if name in ("open_k", "open_v"):          # (the two last blocks: tokens 48 .. 74; what else is there is older)
                at = [t % 32 for t in range(48, 75)]
                assert torch.equal(a[:, :, at], b[:, :, at]), name
            else:
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), name


def test_cut_back_and_append_again():
    """Drafted tokens that were not accepted: a sequence goes back over a block's border and takes other rows."""
    g = torch.Generator().manual_seed(4)
    made = Made(g, [29, 40], 2, 16, extra_pages=4)
    cfg, pages = config(2, 2, 2), made.pages()
    _, k, v, _ = arrive(made, g, [7, 8], None, 2)
    pages.lengths.copy_(ints(made.lengths))
    kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, 7, 15]))
    made.same(pages)
    made.lengths = [30, 42]                                    # 1 and 2 of them are accepted
    made.k, made.v = ([x[i][:, :t] for i, t in enumerate(made.lengths)] for x in (made.k, made.v))
    pages.lengths.copy_(ints(made.lengths))
    q = rows(g, 2, 2, D)
    check_attention(cfg, made, pages, q, [1, 1], 0)
    _, k, v, _ = arrive(made, g, [3, 9], None, 2)
    pages.lengths.copy_(ints(made.lengths))
    kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, 3, 12]))
    for i in range(2):                                         # the blocks that the sequences have now
        for block in range(made.lengths[i] // 16):
            page = int(made.table[i, block])
            for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
                assert torch.equal(getattr(made, name)[page].view(torch.uint8), getattr(pages, name)[page].cpu().view(torch.uint8)), (i, block, name)
    check_attention(cfg, made, pages, rows(g, 4, 2, D), [2, 2], 0)


def test_not_finite_rows_are_stored_finite():
    def special(q, k, v):
        q[0, 0, 0] = math.nan
        k[0, 0, 3], k[1, 1, 64], v[2, 0, 5], v[3, 1, 6], k[4, 0, 1] = math.inf, math.nan, -math.inf, math.nan, 65504.0
        k[4, 0, 65] = 65504.0                                  # turned past the largest number
    g = torch.Generator().manual_seed(5)
    made = Made(g, [12], 2, 16)
    pages, rope = made.pages(), kvqp.rope_table(64, kvqp.rope_frequencies())
    q, k, v, want_q = arrive(made, g, [6], rope, 2, special=special)
    pages.lengths.copy_(ints(made.lengths))
    got = kvqp.paged_append(config(1, 2, 2), pages, k.cuda(), v.cuda(), ints([0, 6]), q=q.cuda(), rope=rope).cpu()
    assert torch.equal(got.isnan(), want_q.isnan()) and torch.equal(got[~got.isnan()], want_q[~want_q.isnan()])
    made.same(pages)
    assert bool(pages.open_k.cpu()[0, :, 12:18].isfinite().all())


@pytest.mark.parametrize("form", ["e4m3", "int8"])
def test_scales_at_their_ends(form):
    """Blocks of zeros, of the smallest and the largest numbers, and largest values around a power of two times M."""
    most = 448.0 if form == "e4m3" else 127.0
    tops = [0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -120, most, most + 2, most * 2.0 ** -10, 1.0, 3.0e38, 255.0, 0.5]
    g = torch.Generator().manual_seed(6)
    n = 16 * len(tops)
    made = Made(g, [0], 1, 16, BF16, form, extra_pages=len(tops) + 1)
    pages, cfg = made.pages(), config(1, 1, 1)

    def special(q, k, v):
        for j, top in enumerate(tops):
            for x in (k, v):
                block = x[16 * j:16 * j + 16, 0]
                block.copy_((torch.rand((16, D), generator=g) * 2 - 1) * top)
                block[3, 17] = -top
    _, k, v, _ = arrive(made, g, [n], None, 1, special=special)
    pages.lengths.copy_(ints(made.lengths))
    kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, n]))
    made.same(pages)


def test_positions_of_their_own_and_slices_of_a_projection():
    g = torch.Generator().manual_seed(7)
    made = Made(g, [3, 20], 2, 16)
    rope, cfg = kvqp.rope_table(64, kvqp.rope_frequencies(64)), config(2, 4, 2)
    pages = made.pages()
    p = torch.tensor([40, 5, -1, 63, 64, 7, 0])
    q, k, v, want_q = arrive(made, g, [4, 3], rope, 4, positions=p)
    pages.lengths.copy_(ints(made.lengths))
    fused = torch.full((9, 8 * D + 8), 9.0, dtype=HALF, device="cuda")      # two rows of padding behind the last sequence's
    fused[:7, :4 * D], fused[:7, 4 * D:6 * D], fused[:7, 6 * D:8 * D] = (x.flatten(1).cuda() for x in (q, k, v))
    part = [fused[:, a * D:b * D].unflatten(1, (b - a, D)) for a, b in ((0, 4), (4, 6), (6, 8))]
    out = torch.full((9, 4, D), 3.0, dtype=HALF, device="cuda")
    kvqp.paged_append(cfg, pages, part[1], part[2], ints([0, 4, 7]), q=part[0], rope=rope, positions=torch.cat([p, torch.tensor([1, 1])]).to(torch.int32).cuda(), q_out=out)
    assert torch.equal(out[:7].cpu().isnan(), want_q.isnan()) and torch.equal(out[:7].cpu()[~want_q.isnan()], want_q[~want_q.isnan()])
    assert bool((out[7:] == 3).all())
    made.same(pages)
    whole = q.cuda()
    assert kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, 4, 7]), q=whole, rope=rope, positions=p.to(torch.int32).cuda(), q_out=whole) is whole
    assert torch.equal(whole.cpu()[~want_q.isnan()], want_q[~want_q.isnan()])
    made.same(pages)


def test_places_of_open_blocks_and_tokens_without_a_page():
    g = torch.Generator().manual_seed(8)
    made = Made(g, [10, 30], 1, 16)
    cfg, pages = config(2, 1, 1), made.pages()
    _, k, v, _ = arrive(made, g, [9, 5], None, 1)
    pages.lengths.copy_(ints(made.lengths))
    # two more places, and the sequences in others than their own; sequence 0's first block has no page
    for name in ("open_k", "open_v"):
        x = getattr(pages, name)
        setattr(pages, name, torch.cat([x, x.new_full((2, *x.shape[1:]), 2.0)])[[2, 1, 3, 0]].contiguous())
    pages.open_slot = ints([3, 1])
    gone = int(pages.table[0, 0])
    pages.table[0, 0] = -1
    kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, 9, 14]))
    fp8 = made.k_codes[gone].view(torch.uint8)
    fp8.fill_(0x7F), made.v_codes[gone].view(torch.uint8).fill_(0x7F)
    made.k_scale[gone] = made.v_scale[gone] = math.nan
    for name in ("open_k", "open_v"):
        x = getattr(pages, name)
        assert bool((x[[0, 2]] == 2).all())
        setattr(pages, name, x[[3, 1]].contiguous())
    made.same(pages)


# ---- attention ----

def check_attention(cfg, made, pages, q, counts, window, skip=None, workspace=None, starts=True):
    """The call against 64 bits; skip: which tokens of a sequence have no page."""
    n, hq = q.shape[:2]
    lse = torch.full((n, hq), 77.0, device="cuda")
    lengths = pages.lengths.cpu().tolist()
    got = kvqp.paged_attn(cfg, pages, q.cuda(), ints(starts_of(counts)) if starts else None, window=window, lse=lse, workspace=workspace).cpu()
    lse, at = lse.cpu().double(), 0
    for i, m in enumerate(counts):
        k, v = made.numbers(i, "k", lengths[i]), made.numbers(i, "v", lengths[i])
        positions = [lengths[i] - m + j for j in range(m)]
        if skip and i in skip:      # (tokens left out: far below all others)
            stay = torch.tensor([t for t in range(lengths[i]) if t not in skip[i]], dtype=torch.long)
            place = {int(t): j for j, t in enumerate(stay)}
            positions = [max([place[t] for t in range(x + 1) if t in place], default=-1) for x in positions]
            k, v = k[:, stay], v[:, stay]
            assert window == 0
        want, want_lse, off, off_lse = attention(q[at:at + m].double(), k, v, positions, window, cfg.sm_scale)
        near(got[at:at + m], want, off, made.dtype)
        empty = want_lse == -math.inf
        assert torch.equal(lse[at:at + m] == -math.inf, empty)
        assert bool(((lse[at:at + m] - want_lse).abs()[~empty] <= off_lse[~empty]).all())
        at += m


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,lengths,counts,hq,hkv,window", [(16, [1, 16, 17, 130], [1, 1, 1, 1], 8, 2, 0), (32, [33, 0, 95, 64], [3, 0, 2, 5], 8, 1, 0), (64, [700, 63], [4, 5], 4, 4, 0),
                                                               (16, [300, 41, 3], [9, 2, 3], 16, 2, 20), (64, [2051], [1], 2, 2, 0), (32, [520, 515], [17, 1], 4, 2, 200)])
def test_attention(dtype, form, page, lengths, counts, hq, hkv, window):
    g = torch.Generator().manual_seed(page + len(lengths) + hq)
    made = Made(g, lengths, hkv, page, dtype, form)
    q = rows(g, sum(counts), hq, D, dtype=dtype)
    check_attention(config(len(lengths), hq, hkv), made, made.pages(), q, counts, window, starts=any(n != 1 for n in counts))


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,length,count,hq,hkv,window", [(16, 200, 200, 2, 1, 0), (64, 333, 333, 4, 4, 0), (32, 401, 150, 8, 1, 0), (16, 300, 130, 2, 2, 37)])
def test_attention_of_a_prompt(dtype, form, page, length, count, hq, hkv, window):
    g = torch.Generator().manual_seed(page + length)
    made = Made(g, [length, 50], hkv, page, dtype, form)
    q = rows(g, count + 50, hq, D, dtype=dtype)
    check_attention(config(2, hq, hkv), made, made.pages(), q, [count, 50], window)


def test_many_splits_and_segments():
    """A long sequence beside short ones: splits that join, more pages than are looked up at a time."""
    g = torch.Generator().manual_seed(12)
    made = Made(g, [12345, 1, 200], 1, 16, HALF, "e4m3")
    cfg = config(3, 2, 1)
    ws = kvqp.alloc_paged_workspace(cfg, 8)
    for counts in ([1, 1, 1], [6, 1, 1], [2, 0, 3]):
        check_attention(cfg, made, made.pages(), rows(g, sum(counts), 2, D), counts, 0, workspace=ws)
    assert bool((ws[:16384] == 0).all())


def test_pages_that_are_not_there_and_odd_places():
    g = torch.Generator().manual_seed(13)
    made = Made(g, [100, 70], 2, 16)
    cfg, pages = config(2, 4, 2), made.pages()
    pages.table[0, 2], pages.table[0, 5], pages.table[1, 0] = -1, 1 << 20, -(1 << 31)
    skip = {0: set(range(32, 48)) | set(range(80, 96)), 1: set(range(16))}
    check_attention(cfg, made, pages, rows(g, 6, 4, D), [4, 2], 0, skip=skip)
    pages.open_slot = ints([0, 2])                             # sequence 1 has no open block
    skip[1] |= set(range(64, 70))
    check_attention(cfg, made, pages, rows(g, 6, 4, D), [4, 2], 0, skip=skip)
    pages.table.fill_(-1)
    pages.open_slot = ints([-1, 2])
    lse = torch.zeros((2, 4), device="cuda")
    out = kvqp.paged_attn(cfg, pages, rows(g, 2, 4, D).cuda(), lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_freed_pages_before_a_window():
    g = torch.Generator().manual_seed(14)
    made = Made(g, [400], 1, 16)
    pages = made.pages()
    pages.table[0, :(400 - 3 - 100 + 1) // 16] = -1            # blocks before every row's window
    check_attention(config(1, 2, 1), made, pages, rows(g, 3, 2, D), [3], 100)


def test_rows_do_not_reach_each_other():
    g = torch.Generator().manual_seed(15)
    made = Made(g, [90], 1, 16)
    cfg, pages = config(1, 8, 1), made.pages()
    q = rows(g, 10, 8, D)
    want = kvqp.paged_attn(cfg, pages, q.cuda(), ints([0, 10]))
    q[3, 2], q[5, 7, 9] = math.nan, math.inf
    got = kvqp.paged_attn(cfg, pages, q.cuda(), ints([0, 10]))
    other = torch.ones((10, 8), dtype=torch.bool)
    other[3, 2] = other[5, 7] = False
    assert torch.equal(got.cpu()[other], want.cpu()[other])


@pytest.mark.parametrize("dtype,form", FORMS)
def test_scales_far_apart(dtype, form):
    """Values of pages that differ by 2^15, keys by as much, and a row that attends the small ones alone."""
    g = torch.Generator().manual_seed(16)
    made = Made(g, [96], 1, 16, dtype, form)
    for block in range(6):
        by = 2.0 ** (15 - 3 * block) if block != 2 else 2.0 ** 15
        made.v[0][:, 16 * block:16 * block + 16] = finite(made.v[0][:, 16 * block:16 * block + 16].float() * by / 2 ** 3, dtype)
    made.k[0][:, :16, 0] = -40.0                               # block 0, with the largest values, is hardly attended
    made.put(0, 0, 96)
    q = rows(g, 1, 1, D, dtype=dtype)
    q[0, 0, 0] = 30.0
    check_attention(config(1, 1, 1), made, made.pages(), q, [1], 0)


def test_heads_are_reproducible_and_batches_independent():
    g = torch.Generator().manual_seed(17)
    made = Made(g, [1500, 700], 2, 32, BF16, "int8")
    cfg, pages = config(2, 8, 2), made.pages()
    q = rows(g, 2, 8, D, dtype=BF16).cuda()
    first = kvqp.paged_attn(cfg, pages, q)
    for _ in range(5):
        assert torch.equal(kvqp.paged_attn(cfg, pages, q), first)


# ---- reading back ----

@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,lengths,first,count", [(16, [1, 40, 0], 0, 40), (32, [200, 131], 0, 200), (64, [300, 64], 37, 150), (16, [90], 33, 1), (32, [64], 0, 96)])
def test_read(dtype, form, page, lengths, first, count):
    g = torch.Generator().manual_seed(page + count)
    made = Made(g, lengths, 2, page, dtype, form)
    pages = made.pages()
    got = kvqp.paged_read(config(len(lengths), 2, 2), pages, count, first)
    for name, x in zip("kv", got):
        want = torch.zeros((len(lengths), 2, count, D), dtype=torch.float64)
        for i, t in enumerate(lengths):
            y = made.numbers(i, name)[:, first:first + count]
            want[i, :, :y.shape[1]] = y
        assert torch.equal(x.cpu(), finite(want, dtype))


def test_read_without_pages():
    g = torch.Generator().manual_seed(18)
    made = Made(g, [50], 1, 16)
    pages = made.pages()
    pages.table[0, 1] = 1 << 30
    k, v = kvqp.paged_read(config(1, 1, 1), pages, 60)
    assert bool((k[0, 0, 16:32] == 0).all()) and bool((v[0, 0, 16:32] == 0).all()) and bool((k[0, 0, 50:] == 0).all()) and bool((v[0, 0, 50:] == 0).all())
    assert torch.equal(k[0, 0, 32:50].cpu().double(), made.numbers(0, "k")[0, 32:50]) and torch.equal(v[0, 0, :16].cpu().double(), made.numbers(0, "v")[0, :16])


def test_codes_at_the_types_end():
    """A code times its scale may lie past the type's largest number: it is cut to that."""
    g = torch.Generator().manual_seed(19)
    made = Made(g, [16], 1, 16, HALF, "e4m3")
    made.k[0][0, 0, :4] = torch.tensor([65504.0, -65504.0, 65000.0, 60000.0])
    made.put(0, 0, 16)
    k, _ = kvqp.paged_read(config(1, 1, 1), made.pages(), 16)
    assert torch.equal(k[0, 0].cpu(), finite(made.numbers(0, "k")[0], HALF)) and float(k[0, 0, 0, 0]) == 65504


# ---- together ----

def test_a_serving_run():
    """Prompts in pieces, single tokens, a captured step, and a prompt that goes to be pruned: append, attend, read, compress, decode."""
    g = torch.Generator().manual_seed(20)
    b, hq, hkv, page = 2, 8, 2, 16
    cfg = config(b, hq, hkv)
    made = Made(g, [0, 0], hkv, page, extra_pages=30)
    pages, rope = made.pages(), kvqp.rope_table(512, kvqp.rope_frequencies())
    ws = kvqp.alloc_paged_workspace(cfg, 300)
    for counts in ([150, 33], [130, 0], [1, 260], [1, 1]):
        q, k, v, want_q = arrive(made, g, counts, rope, hq)
        pages.lengths.copy_(ints(made.lengths))
        qr = kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints(starts_of(counts)), q=q.cuda(), rope=rope)
        assert torch.equal(qr.cpu(), want_q)
        check_attention(cfg, made, pages, want_q, counts, 0, workspace=ws)
    made.same(pages)
    # one step, captured: the lengths are the device's
    buffers = [torch.zeros((b, h, D), dtype=HALF, device="cuda") for h in (hq, hkv, hkv, hq, hq)]
    kvqp.paged_attn(cfg, pages, buffers[3], out=buffers[4], workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages.lengths.add_(1)
        kvqp.paged_append(cfg, pages, buffers[1], buffers[2], q=buffers[0], rope=rope, q_out=buffers[3])
        kvqp.paged_attn(cfg, pages, buffers[3], out=buffers[4], workspace=ws)
    for step in range(18):
        q, k, v, want_q = arrive(made, g, [1, 1], rope, hq)
        for x, y in zip(buffers, (q, k, v)):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        assert pages.lengths.tolist() == made.lengths and torch.equal(buffers[3].cpu(), want_q)
        eager = kvqp.paged_attn(cfg, pages, buffers[3], workspace=ws)
        assert torch.equal(eager, buffers[4])
        if step in (0, 9, 17):
            made.same(pages)
            check_attention(cfg, made, pages, want_q, [1, 1], 0, workspace=ws)
    # the first 256 tokens of both are pruned to 64 at 4 bits
    prune = kvqp.Cfg(batch=b, n_q_heads=hq, n_kv_heads=hkv, seq_len=256, window=32, budget=64, bits=4, group_size=32)
    kk, vv = kvqp.paged_read(cfg, pages, 256)
    q_obs = kvqp.rotate(rope, rows(g, b, hq, 32, D).cuda(), first=224)
    cache = kvqp.compress(prune, q_obs, kk, vv, kvqp.alloc_cache(prune))
    out = kvqp.decode_attn(prune, q_obs[:, :, -1].contiguous(), cache)
    whole = torch.stack([attention(q_obs[i, :, -1:].cpu().double().transpose(0, 1), kk[i].cpu().double(), vv[i].cpu().double(), [255], 0, cfg.sm_scale)[0][0] for i in range(b)])
    assert bool(torch.isfinite(out).all())
    kept = kvqp.quantize_selected(kvqp.Cfg(**{**prune.__dict__, "bits": 16}), kk, vv,
                                  torch.arange(224, dtype=torch.int32, device="cuda").expand(b, hkv, 224).contiguous(),
                                  kvqp.alloc_cache(kvqp.Cfg(**{**prune.__dict__, "bits": 16, "budget": 224})))
    full = kvqp.decode_attn(kvqp.Cfg(**{**prune.__dict__, "bits": 16}), q_obs[:, :, -1].contiguous(), kept)
    assert float((full.double().cpu() - whole).abs().max()) <= 2e-3      # (the decode bar; nothing is pruned here)


def test_two_streams_with_workspaces_of_their_own():
    g = torch.Generator().manual_seed(21)
    made = Made(g, [5000], 2, 32)
    cfg, pages = config(1, 8, 2), made.pages()
    q = [rows(g, 1, 8, D).cuda() for _ in range(2)]
    want = [kvqp.paged_attn(cfg, pages, x) for x in q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [kvqp.alloc_paged_workspace(cfg, 1, stream=s) for s in streams]
    got = [[], []]
    for _ in range(10):
        for i in range(2):
            got[i].append(kvqp.paged_attn(cfg, pages, q[i], workspace=spaces[i], stream=streams[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_offsets_past_32_bits():
    """A pool of more than 4 GB of codes, used at its far end."""
    cfg, n = config(1, 2, 2), (1 << 32) // (2 * 64 * D) + 64
    pages = kvqp.alloc_pages(cfg, n, 4, page_tokens=64)
    g = torch.Generator().manual_seed(22)
    far = [n - 1, n - 3, n - 2, n - 9]
    pages.table.copy_(ints([far]))
    k, v = rows(g, 200, 2, D), rows(g, 200, 2, D)
    pages.lengths.fill_(200)
    kvqp.paged_append(cfg, pages, k.cuda(), v.cuda(), ints([0, 200]))
    made = Made(g, [0], 2, 64, extra_pages=4, spare=0)
    made.k[0], made.v[0] = k.transpose(0, 1), v.transpose(0, 1)
    made.put(0, 0, 200)
    made.lengths = [200]
    for block in range(3):
        mine = int(made.table[0, block])
        assert torch.equal(pages.k_codes[far[block]].cpu().view(torch.uint8), made.k_codes[mine].view(torch.uint8))
        assert torch.equal(pages.v_codes[far[block]].cpu().view(torch.uint8), made.v_codes[mine].view(torch.uint8))
    check_attention(cfg, made, pages, rows(g, 3, 2, D), [3], 0)
    kk, vv = kvqp.paged_read(cfg, pages, 200)
    assert torch.equal(kk[0].cpu(), finite(made.numbers(0, "k"), HALF)) and torch.equal(vv[0].cpu(), finite(made.numbers(0, "v"), HALF))
