"""Memory that the binding allocates for a call on a stream of its own is that stream's: what is free on the current stream may still have
work pending there."""
import contextlib
import types

import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.rows_util import D


class Recorder:
    """Which stream was current when memory was allocated."""

    def __init__(self, monkeypatch):
        self.current, self.seen = ["current"], []

        @contextlib.contextmanager
        def on(stream):
            self.current.append(stream)
            yield
            self.current.pop()
        monkeypatch.setattr(torch.cuda, "stream", on)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
        for name in ("empty", "empty_like"):
            real = getattr(torch, name)

            def recorded(*a, real=real, **kw):
                self.seen.append(self.current[-1])
                return real(*a, **kw)
            monkeypatch.setattr(torch, name, recorded)


@pytest.fixture
def calls(monkeypatch):
    """Calls on tensors in host memory, with everything that needs a GPU left out."""
    for name in ("_want", "_same_device", "_call"):
        monkeypatch.setattr(kvqp, name, lambda *a, **kw: None)
    monkeypatch.setattr(kvqp, "tree_workspace_init", lambda workspace, stream=None: workspace)
    cfg = kvqp.Cfg(batch=1, n_q_heads=8, n_kv_heads=2, seq_len=288, window=32, budget=256)
    cache = kvqp.alloc_cache(cfg, device="cpu")
    dst = kvqp.alloc_cache(cfg, device="cpu")
    cache.n_kept = 256
    q, kv = torch.zeros((1, 8, 3, D), dtype=torch.float16), torch.zeros((1, 2, 3, D), dtype=torch.float16)
    w = torch.zeros((1, 2, 300))
    return {"tree_attn": lambda s: kvqp.tree_attn(cfg, q, kv, kv, None, cache, stream=s),
            "evict": lambda s: kvqp.evict(cfg, cache, w, 128, dst, stream=s),
            "alloc_tree_workspace": lambda s: kvqp.alloc_tree_workspace(cfg, 3, "cpu", s)}


@pytest.mark.parametrize("name", ["tree_attn", "evict", "alloc_tree_workspace"])
def test_a_call_on_another_stream_takes_that_streams_memory(calls, monkeypatch, name):
    recorder = Recorder(monkeypatch)
    calls[name](None)
    assert recorder.seen and set(recorder.seen) == {"current"}
    recorder.seen.clear()
    calls[name](types.SimpleNamespace(cuda_stream=0x9009))
    assert recorder.seen and set(recorder.seen) == {0x9009}


@pytest.mark.gpu
def test_memory_just_freed_on_the_current_stream_is_not_taken(orc, monkeypatch):
    """Blocks of the sizes that the call needs are free on the current stream: it takes others."""
    import numpy as np
    from tests.rows_util import half, make
    rng = np.random.default_rng(52)
    cfg, cache, _, _ = make(orc, rng, 1, 2, 4, 3000, 20, 4, 32, 0)
    q, kn, vn = (torch.from_numpy(half(rng, *s)).cuda() for s in ((1, 8, 5, D), (1, 2, 5, D), (1, 2, 5, D)))
    w = torch.rand((1, 2, 3020), device="cuda")
    dst = kvqp.alloc_cache(kvqp.Cfg(**{**cfg.__dict__, "budget": 2000}), tail_cap=cache.tail_cap)
    want = kvqp.tree_attn(cfg, q, kn, vn, None, cache)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    real, taken = kvqp._call, []
    monkeypatch.setattr(kvqp, "_call", lambda name, device, stream, args: (taken.append(args), real(name, device, stream, args))[1])
    sizes = [q.numel() * 2, kvqp.tree_workspace_bytes(cfg, 5), kvqp.evict_workspace_bytes(cfg, 3000)]
    blocks = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
    spans = [(b.data_ptr(), b.data_ptr() + b.numel()) for b in blocks]
    del blocks
    out = kvqp.tree_attn(cfg, q, kn, vn, None, cache, stream=s)
    kvqp.evict(cfg, cache, w, 2000, dst, stream=s)
    torch.cuda.synchronize()
    places = [out.data_ptr(), taken[0][10], taken[1][10]]
    assert not any(a <= p < b for p in places for a, b in spans)
    assert torch.equal(out, want)


@pytest.mark.parametrize("name", ["compress", "compress_ragged", "decode_attn", "alloc_decode_workspace"])
def test_compress_and_decode_on_another_stream_take_that_streams_memory(monkeypatch, name):
    monkeypatch.setattr(kvqp, "decode_workspace_init", lambda cfg, workspace, stream=None: workspace)
    monkeypatch.setattr(kvqp, "_entry", lambda entry: lambda *a: 0)
    kvqp.lib()
    monkeypatch.setattr(kvqp, "_stream_handle", lambda stream: 0)
    cfg = kvqp.Cfg(batch=1, n_q_heads=8, n_kv_heads=2, seq_len=288, window=32, budget=256)
    cache = kvqp.alloc_cache(cfg, device="cpu", ragged=name == "compress_ragged")
    q, k = torch.zeros((1, 8, 32, D), dtype=torch.float16), torch.zeros((1, 2, 288, D), dtype=torch.float16)
    # (compress_ragged calls the library itself: without a workspace's address it launches nothing)
    monkeypatch.setattr(kvqp, "_ptr", lambda t: None)
    call = {"compress": lambda s: kvqp.compress(cfg, q, k, k, cache, stream=s),
            "compress_ragged": lambda s: kvqp.compress_ragged(cfg, q, k, k, [256, 100], cache, stream=s),
            "decode_attn": lambda s: kvqp.decode_attn(cfg, q[:, :, 0], cache, stream=s),
            "alloc_decode_workspace": lambda s: kvqp.alloc_decode_workspace(cfg, "cpu", s)}[name]
    recorder = Recorder(monkeypatch)
    for stream, where in ((None, "current"), (types.SimpleNamespace(cuda_stream=0x9009), 0x9009)):
        recorder.seen.clear()
        if name == "compress_ragged":
            with pytest.raises(kvqp.KvqpError):
                call(stream)
        else:
            call(stream)
        assert recorder.seen and set(recorder.seen) == {where}


@pytest.mark.gpu
def test_a_captured_call_on_the_capturing_stream_makes_its_own_memory(orc):
    import numpy as np
    from tests.rows_util import half, make
    rng = np.random.default_rng(54)
    cfg, cache, _, _ = make(orc, rng, 1, 2, 4, 2600, 20, 4, 32, 0)
    q, kn, vn = (torch.from_numpy(half(rng, *s)).cuda() for s in ((1, 8, 5, D), (1, 2, 5, D), (1, 2, 5, D)))
    want, step = kvqp.tree_attn(cfg, q, kn, vn, None, cache), kvqp.decode_attn(cfg, q[:, :, 0].contiguous(), cache)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    one = q[:, :, 0].contiguous()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        out = kvqp.tree_attn(cfg, q, kn, vn, None, cache, stream=s)
        out1 = kvqp.decode_attn(cfg, one, cache, stream=s)
    for _ in range(4):
        out.zero_(), out1.zero_()
        g.replay()
        again = kvqp.tree_attn(cfg, q, kn, vn, None, cache)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(out1, step) and torch.equal(again, want)
