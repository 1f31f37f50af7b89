"""A workspace of kvqp_tree_attn made for so many drafted tokens serves every call of fewer."""
import numpy as np
import pytest

from paper_2412_12706_amd import kvqp


def needed(c, n, splits=None):
    """What one call of n rows may use: partial results of as many splits as a long cache gets, behind the counters."""
    rows = c.n_q_heads // c.n_kv_heads * n
    tiles = 1 if rows <= 16 else 2 if rows <= 32 else 4
    base = c.batch * c.n_kv_heads * -(-rows // (16 * tiles))
    splits = max(1, min(64, 256 // base))
    return 4096 + base * splits * 16 * tiles * 130 * 4 if splits > 1 else 0


@pytest.mark.parametrize("batch,hq,hkv", [(1, 32, 8), (8, 32, 8), (32, 32, 8), (1, 2, 2), (3, 24, 3), (1, 8, 1), (100, 4, 2), (5, 40, 5), (300, 2, 2)])
def test_a_workspace_for_more_rows_serves_fewer(batch, hq, hkv):
    c = kvqp.Cfg(batch=batch, n_q_heads=hq, n_kv_heads=hkv)
    most = 0
    for n in range(1, kvqp.MOST_ROWS + 1):
        most = max(most, needed(c, n))
        assert kvqp.tree_workspace_bytes(c, n) == most, n


@pytest.mark.gpu
def test_the_largest_drafts_workspace_serves_a_small_one(orc):
    from tests.rows_util import make
    from tests.test_gpu_tree import check, draft
    rng = np.random.default_rng(53)
    cfg, cache, keys, values = make(orc, rng, 1, 8, 4, 4500, 20, 4, 32, 0)
    ws = kvqp.alloc_tree_workspace(cfg, 40)
    for N in (16, 8, 1, 40):
        q, kn, vn = draft(rng, 1, 8, 4, N)
        check(cfg, cache, keys, values, q, kn, vn, np.tril(np.ones((1, N, N), bool)), None, workspace=ws)
