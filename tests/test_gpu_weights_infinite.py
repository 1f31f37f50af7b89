"""kvqp_accumulate_weights over keys with infinite elements: rows that add nothing (their sum is -inf, or there is no such row) add nothing to those
tokens either."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev
from tests.rows_util import D, SM, half, logit_error, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,axis", [(16, 0), (4, 0), (8, 1)])
@pytest.mark.parametrize("Gq,N", [(1, 1), (2, 5), (4, 5), (8, 7)])
def test_infinite_keys(orc, bits, axis, Gq, N):
    """Tail keys (at 16 bits packed ones, too) with an element of +-inf: the logit is infinite, and the weight 0 or infinite, by the query's sign."""
    rng = np.random.default_rng(51)
    n, tail = 75, 40
    cfg, cache, keys, _ = make(orc, rng, 1, 2, Gq, n, tail, bits, 32, axis)
    places = [n + 3, n + 33] + ([5, 40, 74] if bits == 16 else [])
    for i, t in enumerate(places):
        for h in range(2):
            buf, row = (cache.buffers["tail_k"].view(torch.float16).view(2, -1, D), t - n) if t >= n else (cache.buffers["k_codes"].view(torch.float16).view(2, -1, D), t)
            keys[h][t, 11] = -np.inf if i % 2 else np.inf
            buf[h, row, 11] = float(keys[h][t, 11])
    q = half(rng, 1, 2 * Gq, N, D)
    q[..., 11] = np.abs(q[..., 11]) + np.float16(0.5)
    if N > 1:
        q[0, 0, 1, 11] = -1.0             # (this row gives the others of the tokens everything)
    lse = (6.0 + rng.random((1, 2 * Gq, N))).astype(np.float32)
    if N > 2:
        lse[0, Gq - 1, 2] = -np.inf
    w = kvqp.accumulate_weights(cfg, dev(q), dev(lse), cache, torch.zeros((1, 2, n + tail), device="cuda")).cpu().numpy().astype(np.float64)
    for h in range(2):
        ref, slack = np.zeros(n + tail), 0.0
        for a in range(h * Gq, (h + 1) * Gq):
            seen = np.arange(n + tail)[None] <= n + tail - N + np.arange(N)[:, None]
            live = seen & ~np.isneginf(lse[0, a])[:, None]
            with np.errstate(invalid="ignore"):
                x = np.where(live, (q[0, a].astype(np.float64) @ keys[h].T) * SM - lse[0, a].astype(np.float64)[:, None], -np.inf)
            with np.errstate(over="ignore"):
                ref += np.exp(x).sum(0)
            slack = max(slack, logit_error(q[0, a].astype(np.float64), np.where(np.isfinite(keys[h]), keys[h], 0.0)))
        assert not np.isnan(w[0, h]).any(), np.flatnonzero(np.isnan(w[0, h]))
        big = np.isinf(ref)
        assert np.array_equal(np.isinf(w[0, h]), big) and (w[0, h][big] > 0).all() and big.any()
        # (a weight's relative error is its exponent's absolute one; the sums round at most 2^-24 per row and once more)
        off = np.abs(w[0, h][~big] - ref[~big]) - ((slack + 2.0 ** -19 + Gq * N * 2.0 ** -24 + 2.0 ** -23) * ref[~big] + 2.0 ** -120)
        assert off.max() <= 0, off.max()
