"""What the calls of rotary positions and the paged cache refuse, and their sizes and frequencies: all of it on the host, before anything could be launched."""
import ctypes as C
import math

import pytest
import torch

from paper_2412_12706_amd import kvqp

A = 1 << 20         # an address that nothing reads
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(kvqp.LIB_PATH):
        from paper_2412_12706_amd import build
        build.build()
    kvqp.lib()
    return kvqp._fn_rows


def cfg(**kw):
    return kvqp.Cfg(**{"batch": 2, "n_q_heads": 8, "n_kv_heads": 2, **kw})._bytes()


# buffers of their own, 16 MB apart
PAGES = {"dtype": 0, "form": 0, "page_tokens": 16, "n_pages": 8, "max_pages": 4, "n_open": 2, **{n: (i + 1) << 24 for i, n in enumerate(
    ("k_codes", "v_codes", "k_scale", "v_scale", "open_k", "open_v", "table", "lengths"))}, "open_slot": 0}


def pages(**kw):
    return kvqp._pack_pages(*{**PAGES, **kw}.values())


def rope(table=1 << 28, n=64, rot=128, interleaved=0):
    return kvqp._pack_rope(table, n, rot, interleaved)


# ---- rotation ----

ROTATE = {"rope": rope(), "dtype": 0, "batch": 2, "heads": 3, "rows": 5, "x": (A, 5 * 384, 128, 384), "out": (A << 4, 5 * 384, 128, 384), "positions": 0, "per_batch": 0,
          "first": 0, "inverse": 0}


def rotate(lib, **kw):
    c = {**ROTATE, **kw}
    row = [None if c[n] is None else kvqp._pack_rows(*c[n]) for n in ("x", "out")]
    return lib["kvqp_rotate"](c["rope"], c["dtype"], c["batch"], c["heads"], c["rows"], *row, c["positions"], c["per_batch"], c["first"], c["inverse"], 0)


@pytest.mark.parametrize("kw,code", [
    ({"rope": None}, INVALID), ({"rope": rope(table=0)}, INVALID), ({"rope": rope(table=(1 << 28) + 8)}, INVALID), ({"rope": rope(n=0)}, INVALID),
    ({"rope": rope(rot=0)}, INVALID), ({"rope": rope(rot=24)}, INVALID), ({"rope": rope(rot=144)}, INVALID), ({"rope": rope(interleaved=2)}, INVALID),
    ({"dtype": 2}, INVALID), ({"batch": 0}, INVALID), ({"heads": 0}, INVALID), ({"rows": -1}, INVALID), ({"rows": (1 << 30) + 1}, UNSUPPORTED), ({"batch": 65536}, UNSUPPORTED),
    ({"x": None}, INVALID), ({"out": None}, INVALID), ({"x": (0, 1920, 128, 384)}, INVALID), ({"x": (A + 8, 1920, 128, 384)}, INVALID),
    ({"x": (A, 1920, 128, 388)}, INVALID), ({"x": (A, -1920, 128, 384)}, INVALID), ({"out": (A << 4, 1920, 128, 0)}, INVALID), ({"out": (A << 4, 1920, 120, 384)}, INVALID),
    ({"out": (A << 4, 1920, 128, 256)}, INVALID),                  # rows within each other
    ({"out": (A, 1920, 640, 128)}, INVALID),                       # x's memory in another order
    ({"out": (A + 256, 1920, 128, 384)}, INVALID), ({"out": (1 << 28, 1920, 128, 384)}, INVALID),
    ({"first": -1}, INVALID), ({"first": 60}, INVALID), ({"positions": A + 2}, INVALID), ({"positions": (A << 4) + 64}, INVALID),
    ({"x": (A, 1 << 41, 128, 384)}, INVALID), ({"rows": 1 << 30, "x": (A, 0, 0, 1 << 40), "positions": 1 << 40}, INVALID),
])
def test_rotate_refuses(lib, kw, code):
    assert rotate(lib, **kw) == code


def test_rotate_of_nothing(lib):
    assert rotate(lib, rows=0, x=(0, 0, 0, 0)) == 0


def test_frequencies():
    d, base = 64, 10000.0
    plain = kvqp.rope_frequencies(d, base)
    assert plain == pytest.approx([base ** (-2 * j / d) for j in range(d // 2)], rel=1e-15)
    assert kvqp.rope_frequencies(d, base, kvqp.ROPE_LINEAR, 4.0) == pytest.approx([f / 4 for f in plain], rel=1e-15)
    far = kvqp.rope_frequencies(d, base, kvqp.ROPE_BASE, 8.0)
    assert far[0] == plain[0] and far[-1] == pytest.approx(plain[-1] / 8, rel=1e-13)
    parts = kvqp.rope_frequencies(d, base, kvqp.ROPE_PARTS, 8.0, 4096.0, 1.0, 32.0)
    for f, p in zip(plain, parts):
        turns = 4096.0 * f / (2 * math.pi)
        g = min(max((turns - 1) / 31, 0), 1)
        assert p == pytest.approx(g * f + (1 - g) * f / 8, rel=1e-14)
    assert parts[0] == plain[0] and parts[-1] == pytest.approx(plain[-1] / 8, rel=1e-15) and any(f / 8 < p < f for f, p in zip(plain, parts))


@pytest.mark.parametrize("args", [(0,), (24,), (256,), (64, 0.0), (64, -5.0), (64, math.inf), (64, math.nan), (64, 1e4, 4), (64, 1e4, -1), (64, 1e4, 1, 0.5), (64, 1e4, 1, math.nan),
                                  (64, 1e4, 2, math.inf), (64, 1e4, 3, 2.0, 0.0), (64, 1e4, 3, 2.0, 100.0, 4.0, 4.0), (64, 1e4, 3, 2.0, 100.0, -1.0, 4.0),
                                  (64, 1e4, 3, 2.0, 100.0, 1.0, math.nan)])
def test_frequencies_refuse(args):
    with pytest.raises(kvqp.KvqpError) as e:
        kvqp.rope_frequencies(*args)
    assert e.value.code == INVALID


def test_table_refuses(lib):
    f = (C.c_double * 64)(*[1.0] * 64)
    call = kvqp.lib().kvqp_rope_table
    assert call(None, 128, 4, 1.0, A, 0) == INVALID and call(f, 128, 4, 1.0, 0, 0) == INVALID and call(f, 128, 4, 1.0, A + 4, 0) == INVALID
    assert call(f, 20, 4, 1.0, A, 0) == INVALID and call(f, 128, 0, 1.0, A, 0) == INVALID and call(f, 128, 4, math.nan, A, 0) == INVALID
    assert call(f, 128, (1 << 30) + 1, 1.0, A, 0) == UNSUPPORTED
    f[63] = math.inf
    assert call(f, 128, 4, 1.0, A, 0) == INVALID


# ---- the cache ----

BAD_PAGES = [({"dtype": 2}, INVALID), ({"form": 2}, INVALID), ({"page_tokens": 0}, INVALID), ({"page_tokens": 8}, UNSUPPORTED), ({"page_tokens": 128}, UNSUPPORTED),
             ({"n_pages": 0}, INVALID), ({"max_pages": 0}, INVALID), ({"max_pages": (1 << 26) + 1}, UNSUPPORTED), ({"n_open": 0}, INVALID), ({"n_open": 1}, INVALID),
             ({"k_codes": 0}, INVALID), ({"v_codes": (2 << 24) + 8}, INVALID), ({"k_scale": (3 << 24) + 4}, INVALID), ({"v_scale": 0}, INVALID), ({"open_k": 0}, INVALID),
             ({"open_v": (6 << 24) + 2}, INVALID), ({"table": 0}, INVALID), ({"lengths": 0}, INVALID), ({"lengths": (8 << 24) + 2}, INVALID), ({"open_slot": 6}, INVALID)]

APPEND = {"cfg": cfg(), "pages": pages(), "rope": rope(), "q": 16 << 24, "qs": 1024, "k": 17 << 24, "ks": 256, "v": 18 << 24, "vs": 256, "n": 5, "starts": 19 << 24, "positions": 0,
          "q_out": 20 << 24}
ATTN = {"cfg": cfg(), "pages": pages(), "q": 16 << 24, "qs": 1024, "n": 5, "starts": 19 << 24, "window": 0, "out": 20 << 24, "lse": 21 << 24, "ws": 1 << 32, "ws_bytes": 1 << 30}
READ = {"cfg": cfg(), "pages": pages(), "first": 0, "count": 40, "k": 16 << 24, "v": 17 << 24}


def call(lib, name, base, kw):
    return lib[name](*{**base, **kw}.values(), 0)


@pytest.mark.parametrize("kw,code", BAD_PAGES)
def test_a_cache_that_is_not_one(lib, kw, code):
    for name, base in (("kvqp_paged_append", APPEND), ("kvqp_paged_attn", ATTN), ("kvqp_paged_read", READ)):
        assert call(lib, name, base, {"pages": pages(**kw)}) == code, name
        assert call(lib, name, base, {"pages": None}) == INVALID and call(lib, name, base, {"cfg": cfg(head_dim=64)}) == UNSUPPORTED
        assert call(lib, name, base, {"cfg": cfg(n_q_heads=6)}) == UNSUPPORTED and call(lib, name, base, {"cfg": cfg(n_q_heads=7)}) == INVALID


@pytest.mark.parametrize("kw,code", [
    ({"k": 0}, INVALID), ({"v": 0}, INVALID), ({"q": 0}, INVALID), ({"q_out": 0}, INVALID), ({"q": (16 << 24) + 8}, INVALID), ({"k": (17 << 24) + 2}, INVALID), ({"v": (18 << 24) + 4}, INVALID),
    ({"q_out": (20 << 24) + 8}, INVALID), ({"qs": 1020}, INVALID), ({"qs": 896}, INVALID), ({"ks": 128}, INVALID), ({"vs": 260}, INVALID), ({"ks": 1 << 50}, INVALID),
    ({"n": -1}, INVALID), ({"n": (1 << 30) + 1}, UNSUPPORTED), ({"starts": 0}, INVALID), ({"starts": A + 2}, INVALID), ({"positions": A + 1}, INVALID),
    ({"rope": None, "positions": A}, INVALID), ({"rope": rope(rot=40)}, INVALID),
    ({"q_out": 17 << 24}, INVALID), ({"q_out": 1 << 24}, INVALID), ({"q_out": (16 << 24) + 256}, INVALID), ({"q_out": 16 << 24, "qs": 2048}, INVALID),
    ({"k": 5 << 24}, INVALID), ({"v": 2 << 24}, INVALID), ({"positions": (20 << 24) + 64}, INVALID), ({"starts": 3 << 24}, INVALID),
    ({"pages": pages(v_codes=1 << 24)}, INVALID), ({"pages": pages(open_v=(5 << 24) + 1024)}, INVALID), ({"pages": pages(lengths=4 << 24)}, INVALID),
    ({"rope": rope(table=20 << 24)}, INVALID),
])
def test_append_refuses(lib, kw, code):
    assert call(lib, "kvqp_paged_append", APPEND, kw) == code


@pytest.mark.parametrize("kw,code", [
    ({"q": 0}, INVALID), ({"out": 0}, INVALID), ({"q": (16 << 24) + 8}, INVALID), ({"out": (20 << 24) + 8}, INVALID), ({"lse": (21 << 24) + 2}, INVALID), ({"qs": 512}, INVALID),
    ({"qs": 1028}, INVALID), ({"n": -1}, INVALID), ({"starts": 0}, INVALID), ({"window": -1}, INVALID), ({"out": 16 << 24}, INVALID), ({"out": 6 << 24}, INVALID),
    ({"lse": 20 << 24}, INVALID), ({"lse": 7 << 24}, INVALID), ({"ws": 0, "pages": pages(max_pages=4000)}, WORKSPACE),
    ({"ws_bytes": 1000, "pages": pages(max_pages=4000)}, WORKSPACE), ({"ws": (1 << 32) + 8, "pages": pages(max_pages=4000)}, INVALID),
    ({"ws": 16 << 24, "pages": pages(max_pages=4000)}, INVALID),
])
def test_attention_refuses(lib, kw, code):
    assert call(lib, "kvqp_paged_attn", ATTN, kw) == code


@pytest.mark.parametrize("kw,code", [({"k": 0}, INVALID), ({"v": 0}, INVALID), ({"k": (16 << 24) + 8}, INVALID), ({"first": -1}, INVALID), ({"count": -1}, INVALID), ({"first": 30, "count": 35}, INVALID),
                                     ({"count": 65}, INVALID), ({"v": 16 << 24}, INVALID), ({"k": 2 << 24}, INVALID), ({"first": (1 << 31) - 1, "count": (1 << 31) - 1}, INVALID)])
def test_read_refuses(lib, kw, code):
    assert call(lib, "kvqp_paged_read", READ, kw) == code


def test_attention_refuses_a_factor_that_binary32_does_not_hold(lib):
    for scale, code in ((2.0 ** 100, UNSUPPORTED), (3e38, UNSUPPORTED), (2.0 ** 99, 0), (0.0, INVALID)):
        assert call(lib, "kvqp_paged_attn", {**ATTN, "n": 0} if code == 0 else ATTN, {"cfg": cfg(sm_scale=scale)}) == code


def test_more_than_a_launch_can_have(lib):
    """2^24 workgroups of 256 threads are more threads than a launch counts."""
    far = {"k": 1 << 50, "v": 1 << 52, "q": 1 << 54, "q_out": 1 << 56}
    assert call(lib, "kvqp_paged_append", APPEND, {**far, "n": 1 << 28}) == UNSUPPORTED
    assert call(lib, "kvqp_paged_attn", ATTN, {"q": 1 << 54, "out": 1 << 56, "lse": 0, "n": 1 << 29}) == UNSUPPORTED
    assert call(lib, "kvqp_paged_read", READ, {"pages": pages(max_pages=1 << 26), "k": 1 << 54, "v": 1 << 56, "count": 1 << 30}) == UNSUPPORTED
    assert rotate(lib, rope=rope(n=1 << 30), batch=1, heads=1, rows=1 << 29, x=(1 << 50, 128, 128, 128), out=(1 << 52, 128, 128, 128)) == UNSUPPORTED
    assert kvqp.lib().kvqp_rope_table((C.c_double * 64)(*[1.0] * 64), 128, 1 << 26, 1.0, A, 0) == UNSUPPORTED


def test_calls_of_nothing(lib):
    assert call(lib, "kvqp_paged_append", APPEND, {"n": 0}) == 0 and call(lib, "kvqp_paged_attn", ATTN, {"n": 0}) == 0 and call(lib, "kvqp_paged_read", READ, {"count": 0}) == 0


def test_workspace(lib):
    c = kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2)
    sizes = [kvqp.paged_workspace_bytes(c, n) for n in (0, 1, 2, 100, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] >= 16384
    with pytest.raises(kvqp.KvqpError):
        kvqp.paged_workspace_bytes(c, -1)
    init = kvqp.lib().kvqp_paged_workspace_init
    assert init(0, 1 << 20, 0) == WORKSPACE and init(A, 16383, 0) == WORKSPACE and init(A + 8, 1 << 20, 0) == INVALID


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (32, 8), (64, 8), (8, 1), (128, 16)])
def test_every_call_is_content_with_the_stated_workspace(lib, hq, hkv):
    """Over batches, rows and capacities: a call with the stated bytes is not refused for its workspace (one with NULL for its queries, the check behind that, is never launched)."""
    for batch in (1, 2, 7, 48, 200, 3000):
        c = kvqp.Cfg(batch=batch, n_q_heads=hq, n_kv_heads=hkv)
        if batch * hkv > 65535:
            continue
        for n in (1, batch, 3 * batch + 1, 100 * batch, 5000 * batch + 3):
            nbytes = kvqp.paged_workspace_bytes(c, n)
            for most in (1, 30, 500, 100000):
                # (out over q: refused behind the workspace's check)
                g = pages(n_open=batch, max_pages=most)
                args = {**ATTN, "cfg": c._bytes(), "pages": g, "q": 1 << 50, "out": 1 << 50, "qs": hq * 128, "n": n, "ws_bytes": nbytes}
                assert call(lib, "kvqp_paged_attn", args, {}) == INVALID


@pytest.mark.parametrize("hq,hkv", [(1, 1), (32, 8), (8, 1), (256, 32), (384, 384), (385, 385), (400, 400), (1024, 512), (513, 513), (4096, 512), (2048, 2048)])
def test_a_workspace_for_many_rows_serves_fewer(lib, hq, hkv):
    """A stated size does not fall with the rows, and calls of fewer rows are content with it (their queries lie over their results: refused behind the workspace's check)."""
    for batch in (1, 2, 31, 100):
        c = kvqp.Cfg(batch=batch, n_q_heads=hq, n_kv_heads=hkv)
        if batch * hkv > 65535:
            continue
        ns = [n for n in (1, 2, 8, 9, 64, 128, 140, 400, 4000, 40000) if n == 1 or n >= batch]
        sizes = [kvqp.paged_workspace_bytes(c, n) for n in ns]
        assert sizes == sorted(sizes)
        for n, nbytes in zip(ns, sizes):
            for fewer in [m for m in (1, batch, 3 * batch, 16 * batch, n // 2, n) if 1 <= m <= n]:
                args = {**ATTN, "cfg": c._bytes(), "pages": pages(n_open=batch, max_pages=5000), "q": 1 << 50, "out": 1 << 50, "qs": hq * 128, "n": fewer, "ws_bytes": nbytes}
                assert call(lib, "kvqp_paged_attn", args, {}) == INVALID, (batch, n, fewer)


def test_the_binding_refuses_what_is_not_on_a_gpu():
    c = kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2)
    p = kvqp.alloc_pages(c, 8, 4, device="cpu")
    q, kv = torch.zeros((2, 8, 128), dtype=torch.float16), torch.zeros((2, 2, 128), dtype=torch.float16)
    with pytest.raises(ValueError):
        kvqp.paged_attn(c, p, q)
    with pytest.raises(ValueError):
        kvqp.paged_append(c, p, kv, kv)
    with pytest.raises(ValueError):
        kvqp.paged_read(c, p, 4)
    with pytest.raises(ValueError):
        kvqp.rotate(kvqp.Rope(torch.zeros((4, 64, 2))), torch.zeros((1, 1, 2, 128), dtype=torch.float16))
    with pytest.raises(ValueError):
        kvqp.alloc_pages(c, 8, 4, form="fp4", device="cpu")


def test_the_binding_checks_types_and_shapes(monkeypatch):
    """As on a GPU: every buffer of a cache and every row array has its type, shape and order."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    launched = []
    monkeypatch.setattr(kvqp, "_call", lambda name, *a: launched.append(name))
    monkeypatch.setattr(kvqp, "alloc_paged_workspace", lambda *a, **kw: torch.zeros(4))
    c = kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2)
    q, kv = torch.zeros((3, 8, 128), dtype=torch.float16), torch.zeros((3, 2, 128), dtype=torch.float16)
    starts = torch.zeros(3, dtype=torch.int32)

    def fresh(**kw):
        p = kvqp.alloc_pages(c, 8, 4, device="cpu")
        for name, f in kw.items():
            setattr(p, name, f(getattr(p, name)))
        return p
    kvqp.paged_attn(c, fresh(), q, starts)
    kvqp.paged_append(c, fresh(), kv, kv, starts, q=q)
    kvqp.paged_read(c, fresh(), 5)
    assert launched == ["kvqp_paged_attn", "kvqp_paged_append", "kvqp_paged_read"]
    bad = [dict(k_codes=lambda t: t.view(torch.uint8)), dict(v_codes=lambda t: t.view(torch.int8)), dict(v_codes=lambda t: t.transpose(2, 3)), dict(k_scale=lambda t: t.double()),
           dict(v_scale=lambda t: t[:7]), dict(open_k=lambda t: t.float()), dict(open_v=lambda t: t.bfloat16()), dict(open_v=lambda t: t[:, :, :16]), dict(table=lambda t: t.long()),
           dict(table=lambda t: t[:1]), dict(table=lambda t: t.t().contiguous().t()), dict(lengths=lambda t: t[:1]), dict(open_slot=lambda t: torch.zeros(3, dtype=torch.int32))]
    for kw in bad:
        for run in (lambda p: kvqp.paged_attn(c, p, q, starts), lambda p: kvqp.paged_append(c, p, kv, kv, starts), lambda p: kvqp.paged_read(c, p, 5)):
            with pytest.raises(ValueError):
                run(fresh(**kw))
    for args in ((q.float(), starts), (q[:, :4], starts), (q.transpose(0, 1).contiguous().transpose(0, 1), starts), (q, starts[:2]), (q, starts.long()), (q[..., :64], starts)):
        with pytest.raises(ValueError):
            kvqp.paged_attn(c, fresh(), *args)
    for kw in (dict(out=torch.zeros((3, 8, 64))), dict(lse=torch.zeros((3, 4))), dict(lse=torch.zeros((3, 8)).double())):
        with pytest.raises(ValueError):
            kvqp.paged_attn(c, fresh(), q, starts, **kw)
    rope = kvqp.Rope(torch.zeros((8, 64, 2)))
    for kw in (dict(q_out=q), dict(q=q[:2]), dict(q=q, q_out=q[:2]), dict(rope=kvqp.Rope(torch.zeros((8, 32, 2)))), dict(rope=rope, positions=starts[:2]), dict(rope=rope, positions=starts.long())):
        with pytest.raises(ValueError):
            kvqp.paged_append(c, fresh(), kv, kv, starts, **kw)
    for args in ((kv[:2], kv), (kv, kv.bfloat16()), (kv.float(), kv)):
        with pytest.raises(ValueError):
            kvqp.paged_append(c, fresh(), *args, starts)
    x = torch.zeros((2, 3, 4, 128), dtype=torch.float16)
    for kw in (dict(x=x.float()), dict(x=x[0]), dict(x=x[..., ::2]), dict(positions=torch.zeros(3, dtype=torch.int32)), dict(positions=torch.zeros((2, 4))), dict(out=x.bfloat16()), dict(out=x[:1])):
        with pytest.raises(ValueError):
            kvqp.rotate(rope, **{"x": x, **kw})


def test_memory_that_changes_under_a_field_is_seen(monkeypatch):
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    seen = []
    monkeypatch.setattr(kvqp, "_call", lambda name, device, stream, args: seen.append(args))
    c, q = kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2), torch.zeros((2, 8, 128), dtype=torch.float16)
    kv, p, rope = q[:, :2].contiguous(), kvqp.alloc_pages(c, 8, 4, device="cpu"), kvqp.Rope(torch.zeros((8, 64, 2)))
    run = lambda: (kvqp.paged_append(c, p, kv, kv, q=q, rope=rope), seen[-1][1:3])[1]
    first = run()
    assert run() == first
    for name in ("k_codes", "v_codes", "k_scale", "v_scale", "open_k", "open_v", "table", "lengths"):
        t = getattr(p, name)
        was = run()
        t.data = t.data.clone()
        assert run()[0] == kvqp.Pages(p.k_codes, p.v_codes, p.k_scale, p.v_scale, p.open_k, p.open_v, p.table, p.lengths)._bytes(c, 0) != was[0]
    rope.table.data = rope.table.data.clone()
    assert run()[1] == kvqp.Rope(rope.table)._bytes(0) != first[1]


@pytest.mark.parametrize("tiles,compiles", [(2, True), (3, False), (4, True)])
def test_the_join_is_compiled_for_tiles_that_it_covers(tmp_path, tiles, compiles):
    """A pass of it takes two row tiles, so three would end behind the outputs: only even numbers compile (host side alone: nothing is built)."""
    import os
    import shutil
    import subprocess
    from paper_2412_12706_amd import build
    if shutil.which("hipcc") is None:
        pytest.skip("no hipcc")
    with open(os.path.join(build.CSRC, "paged_attn.hip")) as f:
        text = f.read()
    launch = "paged_rows<BF, INT8, 2, false><<<"
    assert launch in text
    (tmp_path / "x.hip").write_text(text.replace(launch, f"paged_rows<BF, INT8, {tiles}, false><<<"))
    r = subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-I" + os.path.join(build.ROOT, "include"), "-I" + build.CSRC,
                        "-DKVQP_PAGED_BITS=1", "-fsyntax-only", str(tmp_path / "x.hip")], capture_output=True, text=True, timeout=200)
    assert (r.returncode == 0) == compiles and ("static assertion" in r.stderr) != compiles, r.stderr[-2000:]


def test_fields_assigned_by_another_thread(monkeypatch):
    """Calls go on while another thread replaces fields: each finds a description, and the next one after an assignment the new one."""
    import sys
    import threading
    import time
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: 0)
    c, p, rope = kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2), kvqp.alloc_pages(kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2), 8, 4, device="cpu"), kvqp.Rope(torch.zeros((8, 64, 2)))
    others, done, interval = [p.lengths.clone() for _ in range(2)], threading.Event(), sys.getswitchinterval()

    def assign():
        i = 0
        while not done.is_set():
            i += 1
            p.lengths, rope.interleaved = others[i % 2], bool(i % 2)
    worker = threading.Thread(target=assign)
    sys.setswitchinterval(1e-6)
    try:
        worker.start()
        until = time.time() + 1.5
        while time.time() < until:
            assert len(p._bytes(c, 0)) == len(rope._bytes(0)) + 72
    finally:
        done.set()
        worker.join()
        sys.setswitchinterval(interval)
    for i in range(4):
        p.lengths, rope.interleaved = others[i % 2], bool(i % 2)
        assert p._bytes(c, 0) == p._checked(c, 0) and rope._bytes(0) == kvqp.Rope(rope.table, interleaved=bool(i % 2))._bytes(0)
