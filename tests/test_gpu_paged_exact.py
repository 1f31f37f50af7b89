"""How near attention over pages comes to the formula in 64 bits: nothing before the last rounding of binary16 outputs may be felt."""
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.paged_util import BF16, D, HALF, starts_of
from tests.test_gpu_paged import FORMS, config, ints
from tests.test_gpu_paged_range import Pool, generator

pytestmark = pytest.mark.gpu


def errors(pool, cfg, q, counts, window):
    """How far outputs are from the formula's, and how far the formula's rounded once are (rms)."""
    gq, at, lengths = cfg.n_q_heads // cfg.n_kv_heads, 0, pool.pages.lengths.tolist()
    out = kvqp.paged_attn(cfg, pool.pages, q, ints(starts_of(counts)), window=window).double()
    ref = torch.zeros_like(out)
    for i, n in enumerate(counts):
        t = lengths[i]
        k, v = pool.numbers(i, t)
        pos, token = torch.arange(t - n, t, device="cuda").view(-1, 1), torch.arange(t, device="cuda")
        hidden = (token > pos) | ((token <= pos - window) if window else (token < 0))
        for a in range(cfg.n_q_heads):
            logits = torch.matmul(q[at:at + n, a].double(), k[a // gq].t().contiguous()) * cfg.sm_scale
            ref[at:at + n, a] = torch.matmul(torch.softmax(logits.masked_fill(hidden, -torch.inf), 1), v[a // gq])
        at += n
    rms = lambda x: float(x.square().mean().sqrt())
    return rms(out - ref), rms(ref.to(pool.dtype).double() - ref)


# What is left before the last rounding, rms and relative to a typical output: logits of a few units with 20 roundings of 2^-25 of sums some eight times as large,
# 2^-18 of a weight; a weight's two parts 2^-22; sums over a wave's tokens and the joins 60 roundings of 2^-25 at random, 2^-22.  Errors of single tokens' weights are independent, so
# outputs, which are averages, have no more than that of their size.  The last rounding of binary16 is a quarter of a step, 2^-12.8 on average: the ratio is under 1.01.  (One rounding
# of the weights to binary16 is as large as the last rounding: 1.3 and more.)  Of bfloat16 it is 2^-9.8, and one part of 2^-12.8 makes 1 + 2^-7.
@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("hkv,gq,page,lengths,counts,window", [(2, 4, 16, [1000], [1], 0), (2, 4, 32, [700, 2600], [2, 1], 0), (1, 8, 64, [5000, 900], [4, 3], 0), (2, 2, 16, [600, 900], [13, 16], 300),
                                                               (2, 4, 16, [900], [70], 0), (1, 1, 64, [3000, 500], [200, 300], 0), (2, 8, 32, [1900], [60], 700)])
def test_outputs_are_rounded_once(dtype, form, hkv, gq, page, lengths, counts, window):
    g = generator(hkv + gq + page)
    pool = Pool(g, lengths, hkv, page, dtype, form)
    q = torch.randn((sum(counts), hkv * gq, D), generator=g, device="cuda").to(dtype)
    mine, once = errors(pool, config(len(lengths), hkv * gq, hkv), q, counts, window)
    print(f"  {mine / once:.4f}", flush=True)
    assert mine <= 1.05 * once, mine / once


@pytest.mark.parametrize("dtype", [HALF, BF16])
def test_outputs_of_open_rows_are_rounded_once(dtype):
    """Sequences without a whole block: the rows' own type is multiplied."""
    g = generator(5)
    pool = Pool(g, [63, 40, 55], 2, 64, dtype, "int8")
    for counts in ([1, 1, 1], [9, 9, 9], [40, 40, 40]):
        q = torch.randn((sum(counts), 8, D), generator=g, device="cuda").to(dtype)
        mine, once = errors(pool, config(3, 8, 2), q, counts, 0)
        assert mine <= 1.05 * once, mine / once
