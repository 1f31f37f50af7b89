"""What the calls of several query rows and eviction refuse, and the sizes they state: host only, nothing reaches a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.rows_util import ancestors, mask_words

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3


def cfg(**kw):
    return kvqp.Cfg(**{**dict(batch=1, n_q_heads=8, n_kv_heads=2, bits=4, group_size=32), **kw})


def struct(at=1 << 20, **kw):
    """A cache of addresses that nothing will read, each buffer 1 MB from the next."""
    c = kvqp.CacheStruct()
    for i, n in enumerate(("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero", "tail_k", "tail_v")):
        setattr(c, n, at + (i << 20))
    c.n_kept, c.tail_len, c.tail_cap, c.n_cap = 256, 16, 32, 0
    for n, x in kw.items():
        setattr(c, n, x)
    return c


FAR = 1 << 30


def tree(c=None, cache=None, n=4, q=FAR, kn=FAR, vn=FAR, mask=None, out=FAR, lse=None, ws=FAR, ws_bytes=1 << 30):
    c = cfg() if c is None else c
    cs = struct() if cache is None else cache
    return kvqp.lib().kvqp_tree_attn(C.byref(c.struct()), q, kn, vn, mask, 0, n, C.byref(cs), out, lse, ws, ws_bytes, None)


def weigh(c=None, cache=None, n=4, q=FAR, lse=FAR, w=FAR, w_cap=1000, decay=1.0):
    c = cfg() if c is None else c
    cs = struct() if cache is None else cache
    return kvqp.lib().kvqp_accumulate_weights(C.byref(c.struct()), q, lse, n, C.byref(cs), w, w_cap, decay, None)


def evict(c=None, src=None, dst=None, w=FAR, w_cap=1000, keep=128, unit=1, w_out=None, w_cap_out=0, idx=None, ws=2 * FAR, ws_bytes=1 << 20):
    c = cfg() if c is None else c
    src = struct() if src is None else src
    dst = struct(1 << 28) if dst is None else dst
    return kvqp.lib().kvqp_evict(C.byref(c.struct()), C.byref(src), w, w_cap, keep, unit, C.byref(dst), w_out, w_cap_out, idx, ws, ws_bytes, None)


# A call that is refused launches nothing.  (Here there is no GPU: a call that is not refused fails with KVQP_ERR_HIP, -4, or, with one, is never made.)

@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(n=0)), (UNSUPPORTED, dict(n=257)), (INVALID, dict(q=None)), (INVALID, dict(kn=None)), (INVALID, dict(vn=None)), (INVALID, dict(out=None)),
    (INVALID, dict(q=FAR + 8)), (INVALID, dict(kn=FAR + 2)), (INVALID, dict(vn=FAR + 4)), (INVALID, dict(out=FAR + 8)), (INVALID, dict(mask=FAR + 2)),
    (INVALID, dict(lse=FAR + 1)), (WORKSPACE, dict(ws=None, cache=struct(n_kept=65536))), (WORKSPACE, dict(ws_bytes=4096, cache=struct(n_kept=65536))), (INVALID, dict(ws=FAR + 8)),
    (INVALID, dict(c=cfg(sm_scale=0.0))), (INVALID, dict(c=cfg(bits=3))), (UNSUPPORTED, dict(c=cfg(head_dim=64))), (UNSUPPORTED, dict(c=cfg(n_q_heads=6))),
    (UNSUPPORTED, dict(c=cfg(outlier_threshold=6.0))), (INVALID, dict(cache=struct(n_kept=-1))), (INVALID, dict(cache=struct(tail_len=33))),
    (INVALID, dict(cache=struct(k_codes=0))), (INVALID, dict(cache=struct(v_zero=0))), (INVALID, dict(cache=struct(tail_v=0))),
    (INVALID, dict(cache=struct(k_codes=(1 << 20) + 4))), (INVALID, dict(cache=struct(k_scale=(1 << 22) + 8))), (INVALID, dict(cache=struct(v_scale=(1 << 22) + 2))),
    (INVALID, dict(cache=struct(n_cap=192))), (INVALID, dict(cache=struct(n_cap=290))), (UNSUPPORTED, dict(cache=struct(n_kept=(1 << 28) + 1))),
    (INVALID, dict(cache=struct(head_n_kept=FAR + 2))),
])
def test_tree_refusals(code, kw):
    assert tree(**kw) == code


def test_null_structs_are_refused():
    lib = kvqp.lib()
    assert lib.kvqp_tree_attn(None, FAR, FAR, FAR, None, 0, 4, C.byref(struct()), FAR, None, FAR, 1 << 30, None) == INVALID
    assert lib.kvqp_tree_attn(C.byref(cfg().struct()), FAR, FAR, FAR, None, 0, 4, None, FAR, None, FAR, 1 << 30, None) == INVALID
    assert lib.kvqp_accumulate_weights(None, FAR, FAR, 1, C.byref(struct()), FAR, 1000, 1.0, None) == INVALID
    assert lib.kvqp_accumulate_weights(C.byref(cfg().struct()), FAR, FAR, 1, None, FAR, 1000, 1.0, None) == INVALID
    assert lib.kvqp_evict(None, C.byref(struct()), FAR, 1000, 10, 1, C.byref(struct(1 << 28)), None, 0, None, 2 * FAR, 1 << 20, None) == INVALID
    assert lib.kvqp_evict(C.byref(cfg().struct()), None, FAR, 1000, 10, 1, C.byref(struct(1 << 28)), None, 0, None, 2 * FAR, 1 << 20, None) == INVALID
    assert lib.kvqp_evict(C.byref(cfg().struct()), C.byref(struct()), FAR, 1000, 10, 1, None, None, 0, None, 2 * FAR, 1 << 20, None) == INVALID


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(n=0)), (UNSUPPORTED, dict(n=257)), (INVALID, dict(q=None)), (INVALID, dict(lse=None)), (INVALID, dict(w=None)), (INVALID, dict(q=FAR + 8)),
    (INVALID, dict(w=FAR + 2)), (INVALID, dict(lse=FAR + 2)), (INVALID, dict(w_cap=271)), (INVALID, dict(w_cap=-1)), (INVALID, dict(decay=-0.5)),
    (INVALID, dict(decay=float("nan"))), (INVALID, dict(decay=float("inf"))), (UNSUPPORTED, dict(c=cfg(outlier_threshold=6.0))),
    (INVALID, dict(cache=struct(tail_k=(7 << 20) + 2))),
])
def test_weights_refusals(code, kw):
    assert weigh(**kw) == code


def test_weights_of_an_empty_cache_are_nothing_to_do():
    assert weigh(cache=struct(n_kept=0, tail_len=0), w_cap=0) == OK


@pytest.mark.parametrize("code,kw", [
    (INVALID, dict(keep=0)), (INVALID, dict(unit=0)), (INVALID, dict(unit=2)), (INVALID, dict(unit=256)), (INVALID, dict(keep=20, unit=32)), (INVALID, dict(w=None)),
    (INVALID, dict(w_cap=271)), (INVALID, dict(w_out=3 * FAR, w_cap_out=143)), (INVALID, dict(w_out=FAR, w_cap_out=1000)), (INVALID, dict(w_out=FAR - 400, w_cap_out=500)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=1000)), (INVALID, dict(ws=2 * FAR + 4)), (INVALID, dict(ws=FAR)), (INVALID, dict(idx=2 * FAR)),
    (INVALID, dict(idx=FAR)), (INVALID, dict(idx=3 * FAR + 1)), (INVALID, dict(dst=struct())), (INVALID, dict(dst=struct(tail_cap=15, at=1 << 28))),
    (INVALID, dict(dst=struct(1 << 28, n_cap=64))), (INVALID, dict(dst=struct(1 << 28, n_cap=200))), (INVALID, dict(dst=struct(1 << 28, v_codes=1 << 20))),
    (INVALID, dict(dst=struct(1 << 28, tail_k=(7 << 20) + 1024))), (INVALID, dict(dst=struct(1 << 28, k_zero=0))), (INVALID, dict(dst=struct(1 << 28, k_zero=(1 << 28) + 4))),
    (INVALID, dict(dst=struct(1 << 28, head_n_kept=3 * FAR))), (INVALID, dict(src=struct(head_n_kept=3 * FAR))), (INVALID, dict(src=struct(n_kept=-1))),
    (INVALID, dict(src=struct(head_n_kept=3 * FAR), dst=struct(1 << 28, head_n_kept=3 * FAR))), (UNSUPPORTED, dict(c=cfg(outlier_threshold=2.0))),
])
def test_evict_refusals(code, kw):
    assert evict(**kw) == code


@pytest.mark.parametrize("kw", [dict(batch=1), dict(batch=32), dict(n_q_heads=2), dict(n_q_heads=16, bits=2), dict(batch=300)])
def test_workspace_sizes(kw):
    c = cfg(**kw)
    for n in (1, 4, 16, 17, 64, 256):
        have = kvqp.tree_workspace_bytes(c, n)
        rows = c.n_q_heads // c.n_kv_heads * n
        tiles = 1 if rows <= 16 else 2 if rows <= 32 else 4
        blocks = -(-rows // (16 * tiles))
        base = c.batch * c.n_kv_heads * blocks
        splits = max(1, min(64, 256 // base))
        assert have >= (4096 + base * splits * 16 * tiles * 130 * 4 if splits > 1 else 0)
    assert kvqp.evict_workspace_bytes(c, 1000) >= c.batch * c.n_kv_heads * 4000
    assert kvqp.lib().kvqp_tree_workspace_init(None, 4096, None) == WORKSPACE
    assert kvqp.lib().kvqp_tree_workspace_init(FAR, 4095, None) == WORKSPACE
    assert kvqp.lib().kvqp_tree_workspace_init(FAR + 8, 4096, None) == INVALID
    for bad in (0, -1, 257):
        with pytest.raises(kvqp.KvqpError):
            kvqp.tree_workspace_bytes(c, bad)


def test_tree_mask_is_ancestors():
    rng = np.random.default_rng(0)
    for n in (1, 5, 31, 32, 33, 64, 100, 256):
        parents = [int(rng.integers(max(-1, i - 6), i)) for i in range(n)]
        assert np.array_equal(kvqp.tree_mask(parents, device="cpu").numpy(), mask_words(ancestors(parents)))
    two = kvqp.tree_mask([[-1, 0, 1], [-1, -1, 0]], device="cpu").numpy()
    assert two.tolist() == [[[1], [3], [7]], [[1], [2], [5]]]
    for bad in ([0], [-2], [-1, 1], [-1, 5, 0]):
        with pytest.raises(ValueError):
            kvqp.tree_mask(bad, device="cpu")


def test_the_binding_wants_contiguous_tensors_of_its_types_on_the_gpu():
    c = cfg()
    q, kn = torch.zeros((1, 8, 4, 128), dtype=torch.float16), torch.zeros((1, 2, 4, 128), dtype=torch.float16)
    cache = kvqp.Cache({n: torch.zeros(16, dtype=torch.uint8) for n in ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero", "tail_k", "tail_v")}, 0, 0, 0)
    w = torch.zeros((1, 2, 300))
    for call in (lambda: kvqp.tree_attn(c, q, kn, kn, None, cache), lambda: kvqp.accumulate_weights(c, q, torch.zeros((1, 8, 4)), cache, w),
                 lambda: kvqp.evict(c, cache, w, 10, cache), lambda: kvqp.tree_attn(c, q.float(), kn, kn, None, cache),
                 lambda: kvqp.tree_attn(c, q[:, :, 0], kn, kn, None, cache), lambda: kvqp.tree_attn(c, q.transpose(1, 2), kn, kn, None, cache)):
        with pytest.raises(ValueError):
            call()


def test_product_names_no_other_path():
    """(the new sources stay free of anything but HIP and the header)"""
    import os
    root = os.path.join(os.path.dirname(kvqp.__file__), "csrc")
    for name in ("tree_attn.hip", "evict.hip"):
        text = open(os.path.join(root, name)).read().lower()
        for word in ("cuda", "nccl", "triton", "hipmalloc", "hipfree", "synchronize()"):
            assert word not in text, (name, word)


def test_host_side_is_clean_under_asan_and_ubsan(tmp_path):
    import os
    import shutil
    from tests.test_sanitize_host import ENV, ROOT, SAN, run
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if shutil.which("hipcc") is None or not os.path.exists(clang):
        pytest.skip("no hipcc")
    flags = ["-x", "hip", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-Xarch_host",
             "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-I" + os.path.join(ROOT, "include"),
             "-I" + os.path.join(ROOT, "paper_2412_12706_amd", "csrc")]
    objs = []
    for src in (os.path.join(ROOT, "paper_2412_12706_amd", "csrc", "rows_api.cpp"), os.path.join(SAN, "rows_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        run(["hipcc"] + flags + ["-c", src, "-o", objs[-1]])
    exe = str(tmp_path / "rows_driver")
    run([clang, "-fsanitize=address", "-fsanitize=undefined"] + objs + ["-o", exe])
    assert "rows_driver: clean" in run([exe], env=ENV)


def test_token_counts_that_indexes_cannot_hold_are_refused():
    """Words of a head's value codes have 32-bit numbers in the kernels: 2^26 tokens of 16 bits are the most."""
    most = 1 << 26
    assert tree(cache=struct(n_kept=most + 1)) == UNSUPPORTED and tree(cache=struct(n_cap=most + 32)) == UNSUPPORTED
    assert weigh(cache=struct(n_kept=most + 1)) == UNSUPPORTED
    assert evict(src=struct(n_kept=most + 1)) == UNSUPPORTED and evict(dst=struct(1 << 28, n_cap=most + 32)) == UNSUPPORTED
