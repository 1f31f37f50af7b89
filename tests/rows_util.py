"""What the tests of drafted tokens, accumulated weights and eviction share: small caches made by the CPU checker, and the
formulas in 64 bits on what the checker reads back from them."""
import numpy as np
import torch

from paper_2412_12706_amd import kvqp
from tests.gpu_util import dev, upload_cache

D = 128
SM = float(np.float32(128 ** -0.5))


def half(rng, *shape, scale=1.0):
    return (rng.standard_normal(shape, dtype=np.float32) * scale).astype(np.float16)


def make(orc, rng, B, Hkv, Gq, n, tail, bits, G, axis, counts=None, n_cap=0, loud=10.0):
    """A cache of n packed and `tail` plain tokens per head -> (cfg, device cache, keys, values): the last two are lists, per head,
    of 64-bit [count + tail, D] arrays.  counts: every head's own number of packed tokens (under n)."""
    heads = B * Hkv
    k, v = half(rng, B, Hkv, n + max(tail, 1), D), half(rng, B, Hkv, n + max(tail, 1), D)
    k[..., [7, 36, 65, 94]] *= np.float16(loud)
    W = max(tail, 1)
    idx = np.broadcast_to(np.arange(n, dtype=np.int32), (B, Hkv, n)).copy()
    cfg = kvqp.Cfg(batch=B, n_q_heads=Hkv * Gq, n_kv_heads=Hkv, seq_len=n + W, window=W, budget=n, bits=bits, group_size=G, key_axis=axis, sm_scale=SM)
    keys, values = [], []
    if counts is None and not n_cap:
        oc = orc.quantize_selected(k, v, idx, W=W, bits=bits, G=G, key_axis=axis)
        cache = upload_cache(oc)
        counts = [n] * heads
    else:
        cache = kvqp.alloc_cache(cfg, n_cap=n_cap, ragged=counts is not None)
        for t in cache.buffers.values():
            t.fill_(0x5A)                       # (what a head does not fill must not matter)
        if counts is None:
            kvqp.quantize_selected(cfg, dev(k), dev(v), dev(idx), cache)
            counts = [n] * heads
        else:
            kvqp.quantize_selected_ragged(cfg, dev(k), dev(v), dev(idx), counts, cache)
    for h in range(heads):
        b, g = divmod(h, Hkv)
        c = counts[h]
        one = orc.quantize_selected(np.concatenate([k[b:b + 1, g:g + 1, :c], k[b:b + 1, g:g + 1, n:]], 2),
                                    np.concatenate([v[b:b + 1, g:g + 1, :c], v[b:b + 1, g:g + 1, n:]], 2),
                                    idx[:1, :1, :c].copy(), W=W, bits=bits, G=G, key_axis=axis)
        kd, vd = orc.dequantize_head(one, 0, 0) if c else (np.zeros((0, D)), np.zeros((0, D)))
        keys.append(np.concatenate([kd, k[b, g, n:n + tail].astype(np.float64)]))
        values.append(np.concatenate([vd, v[b, g, n:n + tail].astype(np.float64)]))
    cache.tail_len = tail
    torch.cuda.synchronize()
    return cfg, cache, keys, values


def attention(q, keys, values, seen):
    """q [R, D], keys / values [T, D], seen [R, T] -> out [R, D], lse [R], sum of weight * |value| [R, D]"""
    with np.errstate(divide="ignore", invalid="ignore"):
        logits = np.where(seen, (q @ keys.T) * SM, -np.inf)
        top = logits.max(1, keepdims=True, initial=-np.inf)
        p = np.where(seen, np.exp(logits - np.where(np.isfinite(top), top, 0.0)), 0.0)
        total = p.sum(1, keepdims=True)
        lse = np.where(total > 0, top + np.log(total), -np.inf)[:, 0]
        w = np.where(total > 0, p / np.where(total > 0, total, 1.0), 0.0)
    v = np.where(np.isfinite(values), values, 0.0)
    return w @ v, lse, w @ np.abs(v)


def logit_error(q, keys):
    """How far a logit may be off: operands are exact to 2^-22 of what is multiplied, and a chain of at most 20 matrix
    instructions rounds its sum in binary32, three half-steps each: 2^-22 + 60 * 2^-24 < 2^-18 of the sum of magnitudes.  A code times its
    scale and the zero it is added to are at most the span of their group, together eight times the key's own size here."""
    return 2.0 ** -18 * 8.0 * SM * float((np.abs(q) @ np.abs(keys).T).max(initial=0.0))


def out_error(ref, spread, delta):
    """How far an output may be off: its own rounding and that of the values to binary16 (half a step each: 2^-11), a weight's
    share of the logits' error in numerator and denominator, and what lies below binary16's smallest step."""
    return 2.0 ** -11 * np.abs(ref) + (2.0 ** -11 + 2.0 * delta + 2.0 ** -18) * spread + 2.0 ** -24


def ancestors(parents):
    n = len(parents)
    seen = np.zeros((n, n), bool)
    for i, p in enumerate(parents):
        if p >= 0:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def mask_words(seen):
    """bool [..., n, n] -> int32 [..., n, ceil(n / 32)]"""
    n = seen.shape[-1]
    bits = np.zeros(seen.shape[:-1] + (-(-n // 32) * 32,), np.uint8)
    bits[..., :n] = seen
    return np.packbits(bits, axis=-1, bitorder="little").view(np.int32)
