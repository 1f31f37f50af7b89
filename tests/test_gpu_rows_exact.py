"""How near outputs of several query rows come to the formula in 64 bits: nothing before their last rounding may be felt."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev
from tests.rows_util import D, attention, make
from tests.test_gpu_tree import draft

pytestmark = pytest.mark.gpu


def errors(cfg, cache, keys, values, q, kn, vn):
    """Outputs of a chain: how far they are from the formula's, and how far the formula's rounded once to binary16 are (rms)."""
    B, Hq, N, _ = q.shape
    gq = Hq // cfg.n_kv_heads
    out = kvqp.tree_attn(cfg, dev(q), dev(kn), dev(vn), None, cache).cpu().numpy().astype(np.float64)
    ref = np.zeros_like(out)
    for b in range(B):
        for a in range(Hq):
            h = b * cfg.n_kv_heads + a // gq
            k64, v64 = (np.concatenate([x[h], y[b, a // gq].astype(np.float64)]) for x, y in ((keys, kn), (values, vn)))
            seen = np.concatenate([np.ones((N, len(keys[h])), bool), np.tril(np.ones((N, N), bool))], 1)
            ref[b, a] = attention(q[b, a].astype(np.float64), k64, v64, seen)[0]
    rms = lambda x: float(np.sqrt((x * x).mean()))
    return rms(out - ref), rms(ref.astype(np.float16).astype(np.float64) - ref)


# What is left before the last rounding, all of it rms and relative to an output of 0.05 and more of values of 1 (these caches'): a weight's and a value's
# two parts 2^-21 each, logits 2^-19 (20 roundings of 2^-25 of sums eight times as large as a logit of 2), sums over a wave's blocks 40 roundings of
# 2^-25 of 20 times the output: together under 2^-16.  The last rounding is a quarter of a step, 2^-12.8 on average, so the ratio is under
# 1.01.  Values rounded to binary16 before the product (independent errors as large as the last rounding's) make it 1.3 and more.
@pytest.mark.parametrize("bits,G,axis", [(4, 32, 0), (4, 64, 1), (4, 128, 0), (2, 32, 1), (2, 64, 0), (2, 128, 1), (8, 32, 0), (8, 64, 0), (8, 128, 1), (16, 32, 0)])
@pytest.mark.parametrize("Gq,N", [(1, 3), (4, 6), (8, 9)])
def test_outputs_are_rounded_once(orc, bits, G, axis, Gq, N):
    rng = np.random.default_rng(1000 * bits + G + axis + N)
    for n, tail, counts in ((900, 21, None), (300, 0, [300, 77])):
        cfg, cache, keys, values = make(orc, rng, 1, 2, Gq, n, tail, bits, G, axis, counts=counts)
        mine, once = errors(cfg, cache, keys, values, *draft(rng, 1, 2, Gq, N))
        assert mine <= 1.05 * once, (n, mine / once)
