"""What the binding makes of a caller's numbers before a call (nothing here reaches a GPU)."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp


@pytest.mark.parametrize("parents", [[-1, 0, 0, 1, 2], [[-1, 0, 1], [-1, -1, 0]]])
def test_parents_may_be_lists_arrays_or_tensors(parents):
    want = kvqp.tree_mask(parents, device="cpu")
    for given in (tuple(parents), np.array(parents), torch.tensor(parents), torch.tensor(parents, dtype=torch.int32)):
        assert torch.equal(kvqp.tree_mask(given, device="cpu"), want)


def test_a_budget_past_32_bits_keeps_everything(monkeypatch):
    """(a C integer would be what is left of it: 2^32 + 5 would keep five tokens)"""
    calls = []
    monkeypatch.setattr(kvqp, "_want", lambda *a: None)
    monkeypatch.setattr(kvqp, "_call", lambda name, device, stream, args: calls.append(args))
    cfg = kvqp.Cfg(batch=1, n_q_heads=8, n_kv_heads=2, seq_len=532, window=32, budget=500)
    src, dst = kvqp.alloc_cache(cfg, device="cpu"), kvqp.alloc_cache(cfg, device="cpu")
    src.n_kept = 500
    for keep in (500, (1 << 31) - 1, 1 << 31, (1 << 32) + 5):
        kvqp.evict(cfg, src, torch.zeros((1, 2, 500)), keep, dst)
    assert all(500 <= args[4] < 1 << 31 for args in calls) and len(calls) == 4
    kvqp.evict(cfg, src, torch.zeros((1, 2, 500)), -1 - (1 << 32), dst)
    assert calls[-1][4] < 1            # (and is refused)
