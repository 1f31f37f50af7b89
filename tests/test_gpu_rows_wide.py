"""Key and value groups of any span that binary16 has: scales on both sides of 256, from where a product in binary16 would overflow, up to groups
from the type's lowest to its highest number."""
import numpy as np
import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev, upload_cache
from tests.rows_util import D, SM, attention, half, out_error
from tests.test_gpu_rows_exact import errors

pytestmark = pytest.mark.gpu
LOUD = [7, 36, 65, 94]


def wide(orc, rng, n, tail, bits, G, axis, k_scale, v_scale, Gq, N, full=False):
    """A cache whose keys have four channels, and whose values have all, of such a standard deviation; queries that are as much smaller there.
    Besides: what the keys' codes times scales and their zeros come to, by magnitude, which is what their products are rounded by."""
    k, v = half(rng, 1, 2, n + tail, D).astype(np.float64), half(rng, 1, 2, n + tail, D).astype(np.float64) * v_scale
    k[..., LOUD] *= k_scale
    if full:          # (groups from one end of binary16 to the other)
        for x, channels in ((k, LOUD), (v, [20])):
            x[:, :, ::7, channels] = 65504.0
            x[:, :, 3::7, channels] = -65504.0
    k, v = (np.clip(x, -65504, 65504).astype(np.float16) for x in (k, v))
    idx = np.broadcast_to(np.arange(n, dtype=np.int32), (1, 2, n)).copy()
    oc = orc.quantize_selected(k, v, idx, W=tail, bits=bits, G=G, key_axis=axis)
    cache = upload_cache(oc)
    cache.tail_len = tail
    keys, values = zip(*(orc.dequantize_head(oc, 0, g) for g in range(2)))
    oc.k_codes = np.zeros_like(oc.k_codes)
    zeros = [orc.dequantize_head(oc, 0, g)[0] for g in range(2)]
    parts = [np.concatenate([np.abs(keys[g] - zeros[g]) + np.abs(zeros[g]), np.abs(k[0, g, n:].astype(np.float64))]) for g in range(2)]
    keys, values = ([np.concatenate([x[g][:n], y[0, g, n:].astype(np.float64)]) for g in range(2)] for x, y in ((keys, k), (values, v)))
    cfg = kvqp.Cfg(batch=1, n_q_heads=2 * Gq, n_kv_heads=2, seq_len=n + tail, window=tail, budget=n, bits=bits, group_size=G, key_axis=axis, sm_scale=SM)
    q = half(rng, 1, 2 * Gq, N, D)
    small = slice(None) if axis == 1 else LOUD           # (keys per token: every channel shares its group with a loud one)
    q[..., small] = (q[..., small].astype(np.float64) / (65504.0 if full else max(k_scale, 1.0))).astype(np.float16)
    return cfg, cache, keys, values, parts, q, half(rng, 1, 2, N, D), half(rng, 1, 2, N, D)


def logit_error(q, parts):
    """Operands are exact to 2^-21 of what is multiplied, and a chain of at most 40 matrix instructions rounds its sum in binary32, three half-steps
    each: 2^-21 + 120 * 2^-24 < 2^-17 of the sum of magnitudes."""
    return 2.0 ** -17 * SM * float((np.abs(q) @ parts.T).max())


def check(cfg, cache, keys, values, parts, q, kn, vn):
    """Outputs, sums and weights of a chain against the formula."""
    _, Hq, N, _ = q.shape
    gq, n, tail = Hq // 2, cache.n_kept, cache.tail_len
    lse = torch.empty((1, Hq, N), device="cuda")
    out = kvqp.tree_attn(cfg, dev(q), dev(kn), dev(vn), None, cache, lse=lse).cpu().numpy().astype(np.float64)
    lse, lse_in = lse.cpu().numpy().astype(np.float64), (6.0 + np.random.default_rng(1).random((1, Hq, N))).astype(np.float32)
    tight = 0
    for a in range(Hq):
        g, rows = a // gq, q[0, a].astype(np.float64)
        k64, v64 = (np.concatenate([x[g], y[0, g].astype(np.float64)]) for x, y in ((keys, kn), (values, vn)))
        seen = np.concatenate([np.ones((N, n + tail), bool), np.tril(np.ones((N, N), bool))], 1)
        ref, ref_lse, spread = attention(rows, k64, v64, seen)
        delta = logit_error(rows, np.concatenate([parts[g], np.abs(kn[0, g].astype(np.float64))]))
        assert np.isfinite(out[0, a]).all() and (np.abs(lse[0, a] - ref_lse) <= delta + 2.0 ** -18 + 2.0 ** -22 * np.abs(ref_lse)).all(), a
        assert (np.abs(out[0, a]) <= np.abs(v64).max() * (1 + 2.0 ** -10)).all()
        if delta <= 0.1:        # (a weight is off by e^delta - 1 <= 1.06 delta in numerator and denominator; larger ones say little)
            tight += 1
            assert (np.abs(out[0, a] - ref) <= out_error(ref, spread, 1.1 * delta)).all(), (a, np.abs(out[0, a] - ref).max())
    w = kvqp.accumulate_weights(cfg, dev(q), dev(lse_in), cache, torch.zeros((1, 2, n + tail), device="cuda")).cpu().numpy().astype(np.float64)
    for g in range(2):
        add, slack = np.zeros(n + tail), 0.0
        for a in range(g * gq, (g + 1) * gq):
            rows = q[0, a].astype(np.float64)
            seen = np.arange(n + tail)[None] <= n + tail - N + np.arange(N)[:, None]
            seen[:, :n] = True
            x = np.where(seen, (rows @ keys[g].T) * SM - lse_in[0, a].astype(np.float64)[:, None], -np.inf)
            assert x.max() < 80.0
            add += np.exp(x).sum(0)
            slack = max(slack, logit_error(rows, parts[g]))
        # (a weight's relative error is its exponent's absolute one; the sums round at most 2^-24 per row and once more)
        assert (np.abs(w[0, g] - add) <= (np.expm1(slack) + 2.0 ** -19 + gq * N * 2.0 ** -24) * add + 2.0 ** -23 * add + 2.0 ** -120).all(), g
    return tight


# (k_scale: a group of 32 normal numbers spans about four of them, so 2-bit scales are 1.4, 4-bit ones 0.28 and 8-bit ones 0.017 of it)
@pytest.mark.parametrize("bits,G,axis,k_scale", [(2, 32, 0, 160.0), (2, 32, 0, 400.0), (2, 64, 0, 9000.0), (4, 32, 0, 850.0), (4, 32, 0, 2000.0), (4, 128, 0, 9000.0),
                                                 (8, 32, 0, 13000.0), (8, 128, 0, 16000.0), (2, 32, 1, 300.0), (4, 64, 1, 3000.0), (8, 32, 1, 16000.0)])
@pytest.mark.parametrize("Gq,N", [(1, 3), (4, 6), (8, 9)])
def test_wide_key_groups(orc, bits, G, axis, k_scale, Gq, N):
    rng = np.random.default_rng(int(k_scale) + bits + G + N)
    cfg, cache, *rest = wide(orc, rng, 300, 12, bits, G, axis, k_scale, 1.0, Gq, N)
    scales = cache.buffers["k_scale"].view(torch.float16).float()
    assert scales.max().item() > 200.0
    assert check(cfg, cache, *rest) == 2 * Gq


@pytest.mark.parametrize("bits,G,axis", [(2, 32, 0), (4, 32, 0), (8, 64, 0), (2, 64, 1), (4, 128, 1), (8, 32, 1)])
@pytest.mark.parametrize("Gq,N", [(1, 3), (4, 6), (8, 9)])
def test_wide_value_groups(orc, bits, G, axis, Gq, N):
    """(as test_outputs_are_rounded_once, with values up to the end of binary16)"""
    for v_scale in (60.0, 9000.0):
        rng = np.random.default_rng(int(v_scale) + bits + G + N)
        cfg, cache, keys, values, _, q, kn, vn = wide(orc, rng, 400, 12, bits, G, axis, 1.0, v_scale, Gq, N)
        mine, once = errors(cfg, cache, keys, values, q, kn, (vn * np.float16(v_scale)).astype(np.float16))
        assert mine <= 1.05 * once, (v_scale, mine / once)


@pytest.mark.parametrize("bits,G,axis", [(2, 32, 0), (4, 64, 0), (8, 128, 0), (2, 64, 1), (4, 32, 1), (8, 32, 1)])
@pytest.mark.parametrize("Gq,N", [(1, 3), (4, 6), (8, 9)])
def test_groups_from_the_lowest_number_to_the_highest(orc, bits, G, axis, Gq, N):
    rng = np.random.default_rng(bits + G + N)
    cfg, cache, *rest = wide(orc, rng, 200, 12, bits, G, axis, 1.0, 1.0, Gq, N, full=True)
    assert check(cfg, cache, *rest) == 2 * Gq


def test_one_row_agrees_with_the_decode_step_on_wide_keys(orc):
    for bits, k_scale in ((2, 1000.0), (4, 4000.0)):
        rng = np.random.default_rng(bits)
        cfg, cache, _, _, _, q, _, _ = wide(orc, rng, 333, 20, bits, 32, 0, k_scale, 1.0, 4, 1)
        ref = kvqp.decode_attn(cfg, dev(q[:, :, 0]), cache)
        tail_k, tail_v = (cache.buffers[x].view(torch.float16).view(1, 2, -1, D) for x in ("tail_k", "tail_v"))
        cache.tail_len -= 1
        out = kvqp.tree_attn(cfg, dev(q), tail_k[:, :, 19:20].contiguous(), tail_v[:, :, 19:20].contiguous(), None, cache)
        assert (out[:, :, 0].float() - ref.float()).abs().max().item() <= 2e-3
