"""A target of an eviction whose buffers are too small for what would be written is refused before anything is launched (on tensors in host
memory: nothing here reaches a GPU)."""
import pytest
import torch

from paper_2412_12706_amd import kvqp


@pytest.fixture
def made(monkeypatch):
    """Calls that reached the library."""
    calls = []

    def want(what, t, dtype, shape, device):
        if t.dtype is not dtype or tuple(t.shape) != tuple(shape):
            raise ValueError(what)
    monkeypatch.setattr(kvqp, "_want", want)
    monkeypatch.setattr(kvqp, "_call", lambda *a: calls.append(a))
    return calls


def config(bits, G, axis, n):
    return kvqp.Cfg(batch=2, n_q_heads=8, n_kv_heads=2, seq_len=n + 32, window=32, budget=n, bits=bits, group_size=G, key_axis=axis)


def cache(bits, G, axis, n, ragged=False, n_cap=0):
    c = kvqp.alloc_cache(config(bits, G, axis, n), device="cpu", ragged=ragged, n_cap=n_cap)
    c.n_kept, c.tail_len = n, 7
    return c


SHAPES = [(2, 32, 0), (2, 64, 1), (4, 32, 0), (4, 128, 1), (8, 64, 0), (16, 32, 0)]


@pytest.mark.parametrize("bits,G,axis", SHAPES)
@pytest.mark.parametrize("keep,n_cap", [(300, 0), (160, 0), (33, 0), (300, 384)])
def test_every_buffer_is_looked_at(made, bits, G, axis, keep, n_cap):
    cfg, src, w = config(bits, G, axis, 500), cache(bits, G, axis, 500), torch.zeros((2, 2, 507))
    kvqp.evict(cfg, src, w, keep, cache(bits, G, axis, keep, n_cap=n_cap))
    assert len(made) == 1
    for name in kvqp._NAMES:
        dst = cache(bits, G, axis, keep, n_cap=n_cap)
        if dst.buffers[name].numel() == 0:
            continue
        dst.buffers[name] = dst.buffers[name][:-2]
        with pytest.raises(ValueError, match="no room.*" + name):
            kvqp.evict(cfg, src, w, keep, dst)
    assert len(made) == 1


def test_a_target_made_for_larger_groups_is_refused(made):
    for axis in (0, 1):
        with pytest.raises(ValueError, match="no room"):
            kvqp.evict(config(4, 32, axis, 500), cache(4, 32, axis, 500), torch.zeros((2, 2, 507)), 300, cache(4, 128, axis, 300))
    assert not made


def test_counts_of_another_type_or_number_are_refused(made):
    cfg, src, w = config(4, 32, 0, 500), cache(4, 32, 0, 500, ragged=True), torch.zeros((2, 2, 507))
    for counts in (torch.zeros(4, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)):
        dst = cache(4, 32, 0, 300, ragged=True)
        dst.head_n_kept = counts
        with pytest.raises(ValueError, match="head_n_kept"):
            kvqp.evict(cfg, src, w, 300, dst)
    assert not made
    for counts in (torch.zeros(4, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)):
        dst = cache(4, 32, 0, 300, ragged=True)
        dst.head_n_kept = counts
        kvqp.evict(cfg, src, w, 300, dst)
    assert len(made) == 2
