"""Performance cases of drafted tokens and eviction over the quantized-pruned KV cache.

A serving program that decodes speculatively keeps asking three things of a compressed cache.  At
every step it verifies drafted tokens: `tree_attn` attends, for a tree (or a chain, or a single
token) of them, over the packed tokens, the full-precision tail and every row's own ancestors.  For
the accepted rows it adds up how much attention each cached token received (`accumulate_weights`).
And when a cache has grown past its budget, `evict` keeps the tokens that received most.  The listed
cases walk the sizes at which this is done -- one layer of one sequence up to the layers of a model
in one call -- over bit widths, key axes, query-head groups, token counts and draft sizes; `draw`
gives others of the same ranges.

A cache here is made from standard normal keys and values (four key channels per head scaled up, as
in the repository's tests) by the quantizer's definition in plain torch, in the layout that the
library's header states.  The plain forms read that layout back with shifts and masks, work in 32
bits and round once; `exact` redoes everything in 64 bits from the definitions.
"""
import math

import torch

own = False
D = 128
DEV = "cuda"
SCALE = 128 ** -0.5
PER_CHANNEL, PER_TOKEN = 0, 1


# ------------------------------------------------------------------------------------------- cases

def _case(name, do, batch, hq, hkv, tokens, bits, group, axis=PER_CHANNEL, tail=32, rows=1, counts="equal", trees="shared",
          decay=1.0, keep=0, unit=1):
    """batch: independent caches of one call; tokens: packed tokens of a head (the largest count where heads have their own); rows:
    drafted tokens, or query rows that are added up; keep, unit: an eviction's budget and how many neighbours stay together."""
    c = {"do": do, "batch": batch, "hq": hq, "hkv": hkv, "tokens": tokens, "tail": tail, "rows": rows, "bits": bits, "group": group,
         "axis": axis, "counts": counts, "trees": trees, "decay": decay, "keep": keep, "unit": unit}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # Verification.  One layer of a short prompt and a small tree: latency counts.
        _case("tree-8-short", "tree", 1, 32, 8, 1024, 4, 32, rows=8),
        # A single new token (nothing drafted this step) over an odd count of 2-bit tokens with a short tail.
        _case("tree-1-2bit-odd", "tree", 1, 32, 8, 10007, 2, 64, tail=19, rows=1),
        # A wide tree over one layer of a long cache: many query rows for every byte.
        _case("tree-64-long", "tree", 1, 32, 8, 16384, 4, 32, rows=64),
        # The layers of a model in one call, a chain of usual length: the largest amount of cache.
        _case("tree-8-layers", "tree", 32, 32, 8, 8192, 4, 32, rows=8),
        # Heads that kept different numbers of tokens, keys per token at 8 bits, eight query heads per KV head, a tree per sequence.
        _case("tree-13-heads-own", "tree", 4, 64, 8, 5003, 8, 128, axis=PER_TOKEN, tail=41, rows=13, counts="own", trees="own"),
        # Pruned but not quantized, one query head per KV head.
        _case("tree-5-16bit", "tree", 2, 16, 16, 4100, 16, 32, tail=33, rows=5),
        # Weights of one decoded token, one layer.
        _case("weights-1-short", "weights", 1, 32, 8, 1024, 4, 32, rows=1),
        # Weights of an accepted chain in all layers.
        _case("weights-4-layers", "weights", 32, 32, 8, 8192, 4, 32, rows=4),
        # Weights of a whole window of rows, as after a prompt, with heads of their own counts and old weights fading.
        _case("weights-32-heads-own", "weights", 4, 32, 8, 12011, 2, 32, axis=PER_TOKEN, tail=64, rows=32, counts="own", decay=0.9),
        # One appended block leaves again: whole key groups move, nothing is rounded anew.
        _case("evict-group-short", "evict", 1, 32, 8, 1056, 4, 32, keep=1024, unit=32),
        # The layers of a model, single tokens, keys per token.
        _case("evict-token-layers", "evict", 32, 32, 8, 8192, 4, 32, axis=PER_TOKEN, keep=6144),
        # Single tokens out of per-channel groups: keys are quantized in the groups that the survivors form.
        _case("evict-regroup-odd", "evict", 2, 32, 8, 12003, 2, 32, tail=17, keep=8001),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    do = rng.choice(("tree", "tree", "weights", "evict"))
    hkv = rng.choice((1, 2, 4, 8, 16))
    gq = rng.choice((1, 2, 4, 8))
    batch = _between(rng, 1, 32)
    bits = rng.choice((2, 4, 8, 16))
    group = rng.choice((32, 64, 128))
    axis = rng.choice((PER_CHANNEL, PER_TOKEN))
    # (at most 2^21 packed tokens over all heads, as in the largest listed case)
    tokens = _between(rng, 16, min(32768, (1 << 21) // (batch * hkv)))
    tail = rng.randint(1, 96)
    counts, trees = "equal", "shared"
    rows, decay, keep, unit = 1, 1.0, 0, 1
    if do == "evict":
        tokens = max(tokens, 256)
        unit = rng.choice((1, 1, group))
        keep = max(unit, int(tokens * rng.uniform(0.3, 0.97)))
    else:
        # (and no more multiplications than the largest listed ones have)
        most = (1 << 30) // (tokens * batch * hkv * gq)
        rows = _between(rng, 1, max(1, min(64, most))) if do == "tree" else _between(rng, 1, max(1, min(32, most)))
        tail = max(tail, rows)
        counts = rng.choice(("equal", "equal", "own"))
        trees = rng.choice(("shared", "own"))
        decay = rng.choice((1.0, 0.95)) if do == "weights" else 1.0
    return _case(None, do, batch, hkv * gq, hkv, tokens, bits, group, axis, tail, rows, counts, trees, decay, keep, unit)


def _heads(c):
    return c["batch"] * c["hkv"]


def _counts(c):
    """Packed tokens of every head: all alike, or between a quarter and all of the largest."""
    n = c["tokens"]
    if c["counts"] == "equal":
        return [n] * _heads(c)
    return [n if h == 0 else n // 4 + (h * 7919 % 101) * (n - n // 4) // 101 for h in range(_heads(c))]


def _key_bytes(c):
    """Bytes of one packed key: codes, and its share of scales and zeros."""
    if c["bits"] == 16:
        return 2 * D
    return D * c["bits"] / 8 + (4 * D / c["group"])


def work(c):
    n, r, t = sum(_counts(c)), c["rows"] * c["hq"] // c["hkv"], c["tail"]
    h, key = _heads(c), _key_bytes(c)
    if c["do"] == "tree":
        return {"bytes": n * 2 * key + h * ((t + c["rows"]) * 4 * D + r * (4 * D + 4)),
                "flops": 4 * D * r * (n + h * (t + c["rows"]))}
    if c["do"] == "weights":
        return {"bytes": n * (key + 8) + h * (t * (2 * D + 8) + r * (2 * D + 4)), "flops": 2 * D * r * (n + h * t)}
    kept = h * _kept(c)
    return {"bytes": 4 * n + kept * (4 * key + 8) + h * t * (8 * D + 8), "flops": n + kept * D}


def _kept(c):
    """Tokens of a head after an eviction: the newest, incomplete unit stays, and whole units fill what is left."""
    if c["keep"] >= c["tokens"]:
        return c["tokens"]
    short = c["tokens"] % c["unit"]
    return short + (c["keep"] - short) // c["unit"] * c["unit"]


# ------------------------------------------------------------------------------------------ inputs

def _up(n, m):
    return -(-n // m) * m


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _quantize(x, bits):
    """Codes, scale and zero of groups along axis -2 (x: [..., members, 1 or channels])."""
    z, m = x.amin(-2, keepdim=True), x.amax(-2, keepdim=True)
    s = ((m.float() - z.float()) / (2 ** bits - 1)).half()
    inv = torch.where(s == 0, torch.zeros_like(s).float(), 1.0 / s.float())
    code = torch.round((x.float() - z.float()) * inv).clamp_(0, 2 ** bits - 1)
    return code.to(torch.int32), s.squeeze(-2), z.squeeze(-2)


def _per_channel(x, c):
    """x: [heads, n, D] half -> codes [heads, n, D], scale, zero [heads, groups, D]; the last group may be short."""
    heads, n, g = x.shape[0], x.shape[1], c["group"]
    full = torch.cat([x, x[:, -1:].expand(heads, _up(n, g) - n, D)], 1)
    code, s, z = _quantize(full.view(heads, -1, g, D), c["bits"])
    return code.view(heads, -1, D)[:, :n], s, z


def _per_token(x, c):
    """... -> codes, scale, zero [heads, n, D / group]"""
    heads, n, g = x.shape[0], x.shape[1], c["group"]
    code, s, z = _quantize(x.reshape(heads, n, D // g, g, 1), c["bits"])
    return code.view(heads, n, D), s.squeeze(-1), z.squeeze(-1)


def _rows_of_zeros(x, n):
    """x: [heads, rows, ...] with zeros up to n rows"""
    return torch.cat([x, x.new_zeros(x.shape[0], n - x.shape[1], *x.shape[2:])], 1) if n > x.shape[1] else x


def _words(x):
    """The fields of a word, in the last axis, put together (their places do not overlap)."""
    w = x.to(torch.int64).sum(-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _key_shifts(bits):
    e = 32 // bits
    return torch.tensor([bits * (r // 2) + 16 * (r % 2) for r in range(e)], device=DEV)


def _pack_keys(code, c):
    """codes [heads, n, D] -> words [heads, rows of 32, D * bits / 32]: two neighbouring channels in a word's halves"""
    code = _rows_of_zeros(code, _up(code.shape[1], 32))
    e = 32 // c["bits"]
    return _words(code.to(torch.int64).view(*code.shape[:2], D // e, e) << _key_shifts(c["bits"]))


def _value_geometry(bits):
    """tokens of a superblock, words of a tile, fields of a half-word"""
    return (64 if bits == 2 else 32), (4 if bits == 16 else 2 if bits == 8 else 1), 16 // bits


def _pack_values(code, c):
    """codes [heads, n, D] -> words [heads, superblocks, words]: tile-transposed"""
    bits, heads = c["bits"], code.shape[0]
    sb, wpt, f = _value_geometry(bits)
    code = _rows_of_zeros(code, _up(code.shape[1], sb))
    # token = sb, blk, H, kb, i; channel = tile, n; run = (blk, i) = (word of the tile, field)
    x = code.view(heads, -1, sb // 32, 2, 4, 4, 8, 16).permute(0, 1, 4, 7, 6, 2, 5, 3)      # heads, s, kb, n, tile, blk, i, H
    x = x.reshape(heads, x.shape[1], 4, 16, 8 * wpt, f, 2)
    shift = torch.tensor([[bits * p + 16 * h for h in range(2)] for p in range(f)], device=DEV)
    w = _words((x.to(torch.int64) << shift).flatten(-2))                                    # heads, s, kb, n, y
    return w.view(heads, w.shape[1], 4, 16, 2 * wpt, 4).permute(0, 1, 4, 2, 3, 5).reshape(heads, w.shape[1], -1)


def _made(c, seed):
    """The tensors of a case."""
    g = _generator(seed)
    heads, n, t, rows, gq = _heads(c), c["tokens"], c["tail"], c["rows"], c["hq"] // c["hkv"]
    counts = _counts(c)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    def keys(count):
        k = normal(heads, count, D)
        k.view(-1, c["hkv"], count, D).mul_(loud)
        return k.half()

    loud = torch.ones((c["hkv"], 1, D), device=DEV)
    at = torch.arange(c["hkv"], device=DEV).view(-1, 1) * 29 + 7 + torch.arange(4, device=DEV) * 37
    loud.view(c["hkv"], D).scatter_(1, at % D, 10.0)

    s = {"case": c}
    k, v = keys(n), normal(heads, n, D).half()
    live = None
    if c["counts"] != "equal":
        s["head_n"] = torch.tensor(counts, dtype=torch.int32, device=DEV)
        live = torch.arange(n, device=DEV) < s["head_n"].view(-1, 1)
    if c["bits"] == 16:
        kc, vc = (x.view(torch.int16).to(torch.int32) & 0xFFFF for x in (k, v))
        names = ()
    else:
        if c["axis"] == PER_CHANNEL:
            kc, s["k_scale"], s["k_zero"] = _per_channel(k, c)
            names = ("v_scale", "v_zero")
        else:
            kc, s["k_scale"], s["k_zero"] = _per_token(k, c)
            names = ("k_scale", "k_zero", "v_scale", "v_zero")
        vc, s["v_scale"], s["v_zero"] = _per_token(v, c)
    if live is not None:
        kc, vc = kc * live.unsqueeze(-1), vc * live.unsqueeze(-1)
    for name in names:
        x = s[name] if live is None else s[name] * live.unsqueeze(-1)
        s[name] = _rows_of_zeros(x, _up(n, 32)).contiguous()
    s["k_codes"], s["v_codes"] = _pack_keys(kc, c), _pack_values(vc, c)
    s["tail_k"], s["tail_v"] = keys(t), normal(heads, t, D).half()

    if c["do"] == "tree":
        s["q"] = normal(c["batch"], c["hq"], rows, D).half()
        s["k_new"], s["v_new"] = (x.view(c["batch"], c["hkv"], rows, D) for x in (keys(rows), normal(heads, rows, D).half()))
        # drafted tokens: each one continues one of the four before it, or the sequence itself
        up = torch.randint(1, 5, (c["batch"] if c["trees"] == "own" else 1, rows), generator=g, device=DEV).cpu().tolist()
        s["sees"] = torch.tensor([_ancestors([i - u[i] for i in range(rows)]) for u in up], device=DEV)
        s["mask"] = _words(_padded_bits(s["sees"]).to(torch.int64) << torch.arange(32, device=DEV))
        s["lse"] = torch.empty((c["batch"], c["hq"], rows), dtype=torch.float32, device=DEV)
    elif c["do"] == "weights":
        s["q"] = normal(c["batch"], c["hq"], rows, D).half()
        # (as after a few such calls: a row's weights add up to one)
        s["weights"] = (normal(heads, n + t + 32).exp_() * (gq * rows / n)).view(c["batch"], c["hkv"], -1)
        logits = _masked_logits(s, gq)
        s["lse"] = torch.logsumexp(logits, -1).view(c["batch"], c["hq"], rows)
    else:
        s["weights"] = normal(heads, n + t).mul_(2.0).exp_().view(c["batch"], c["hkv"], -1)
    return s


def _ancestors(parents):
    sees = []
    for i, p in enumerate(parents):
        row = list(sees[p]) if p >= 0 else [False] * len(parents)
        row[i] = True
        sees.append(row)
    return sees


def _padded_bits(sees):
    n = sees.shape[-1]
    full = sees.new_zeros(*sees.shape[:-1], _up(n, 32))
    full[..., :n] = sees
    return full.view(*sees.shape[:-1], -1, 32)


def _handle(s):
    """What a program that uses the library holds: the configuration, the cache, and buffers for results."""
    from paper_2412_12706_amd import kvqp
    c = s["case"]
    cfg = kvqp.Cfg(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"], bits=c["bits"], group_size=c["group"], key_axis=c["axis"],
                   sm_scale=SCALE)
    none = torch.empty(0, dtype=torch.float16, device=DEV)
    names = ("k_codes", "v_codes", "k_scale", "k_zero", "v_scale", "v_zero", "tail_k", "tail_v")
    cache = kvqp.Cache({k: s.get(k, none) for k in names}, c["tokens"], c["tail"], c["tail"], 0, s.get("head_n"))
    s["kvqp"], s["cfg"], s["cache"] = kvqp, cfg, cache
    if c["do"] == "tree":
        s["workspace"] = kvqp.alloc_tree_workspace(cfg, c["rows"])
        s["trees"] = s["mask"] if c["trees"] == "own" else s["mask"][0]
    elif c["do"] == "evict":
        kept = _kept(c)
        rows, groups = _up(kept, 32), _up(kept, c["group"]) // c["group"]
        sb = _value_geometry(c["bits"])[0]
        like = {"k_codes": rows, "v_codes": _up(kept, sb) // sb, "v_scale": rows, "v_zero": rows, "tail_k": c["tail"], "tail_v": c["tail"],
                "k_scale": groups if c["axis"] == PER_CHANNEL else rows, "k_zero": groups if c["axis"] == PER_CHANNEL else rows}
        new = {k: torch.empty((s[k].shape[0], like[k]) + s[k].shape[2:], dtype=s[k].dtype, device=DEV) if k in s else none for k in names}
        s["dst"] = kvqp.Cache(new, 0, 0, c["tail"], 0)
        s["weights_out"] = torch.empty((c["batch"], c["hkv"], kept + c["tail"]), dtype=torch.float32, device=DEV)
        s["idx"] = torch.empty((c["batch"], c["hkv"], kept), dtype=torch.int32, device=DEV)
        s["workspace"] = kvqp.alloc_evict_workspace(cfg, cache)


def prepare(case, seed):
    s = _made(case, seed)
    if own:
        _handle(s)
    return s


# ------------------------------------------------------------------------------------- plain forms

def _key_codes(w, bits):
    """words [heads, rows, D / e] -> codes [heads, rows, D]"""
    return ((w.unsqueeze(-1) >> _key_shifts(bits)) & (2 ** bits - 1)).flatten(2)


def _value_codes(w, bits):
    """words [heads, superblocks, words] -> codes [heads, tokens, D]"""
    sb, wpt, f = _value_geometry(bits)
    heads = w.shape[0]
    w = w.view(heads, -1, 2 * wpt, 4, 16, 4).permute(0, 1, 3, 4, 2, 5).reshape(heads, -1, 4, 16, 8, wpt)     # heads, s, kb, n, tile, word
    field = torch.arange(f, device=DEV).view(-1, 1) * bits + torch.arange(2, device=DEV) * 16
    x = ((w.unsqueeze(-1).unsqueeze(-1) >> field) & (2 ** bits - 1)).view(heads, -1, 4, 16, 8, sb // 32, 4, 2)
    return x.permute(0, 1, 5, 7, 2, 6, 4, 3).reshape(heads, -1, D)                                         # ... blk, H, kb, i, tile, n


def _bits_to_half(code):
    return code.to(torch.int16).view(torch.float16)


def _keys(s, of=torch.float32):
    """The packed keys as numbers, [heads, tokens, D]"""
    c = s["case"]
    code = _key_codes(s["k_codes"], c["bits"])[:, :c["tokens"]]
    if c["bits"] == 16:
        return _bits_to_half(code).to(of)
    return _read(code, s["k_scale"], s["k_zero"], c, c["axis"] == PER_CHANNEL, of)


def _values(s, of=torch.float32):
    c = s["case"]
    code = _value_codes(s["v_codes"], c["bits"])[:, :c["tokens"]]
    if c["bits"] == 16:
        return _bits_to_half(code).to(of)
    return _read(code, s["v_scale"], s["v_zero"], c, False, of)


def _read(code, scale, zero, c, per_channel, of):
    n, g = code.shape[1], c["group"]
    if per_channel:
        at = torch.arange(n, device=DEV) // g
        return code.to(of) * scale.to(of)[:, at] + zero.to(of)[:, at]
    x = code.to(of).view(code.shape[0], n, D // g, g)
    return (x * scale.to(of)[:, :n].unsqueeze(-1) + zero.to(of)[:, :n].unsqueeze(-1)).view(code.shape)


def _valid(s):
    """Which of the packed tokens a head has, [heads, 1, tokens], or None for all"""
    if "head_n" not in s:
        return None
    return (torch.arange(s["case"]["tokens"], device=DEV) < s["head_n"].view(-1, 1)).unsqueeze(1)


def _masked_logits(s, gq, of=torch.float32):
    """Rows over packed tokens and tail, [heads, gq * rows, tokens + tail]: row i of the last `rows` tail rows sees those up to itself."""
    c = s["case"]
    q = s["q"].view(_heads(c), -1, D).to(of)
    logits = torch.matmul(q, torch.cat([_keys(s, of), s["tail_k"].to(of)], 1).transpose(1, 2)) * SCALE
    if "head_n" in s:
        logits[..., :c["tokens"]].masked_fill_(~_valid(s), -math.inf)
    i = torch.arange(c["rows"], device=DEV).repeat(gq).view(-1, 1)
    later = torch.arange(c["tail"], device=DEV) > c["tail"] - c["rows"] + i
    logits[..., c["tokens"]:].masked_fill_(later, -math.inf)
    return logits


def _tree_plain(s, of=torch.float32):
    c = s["case"]
    heads, gq, rows = _heads(c), c["hq"] // c["hkv"], c["rows"]
    new = [s[k].view(heads, rows, D).to(of) for k in ("k_new", "v_new")]
    k = torch.cat([_keys(s, of), s["tail_k"].to(of), new[0]], 1)
    v = torch.cat([_values(s, of), s["tail_v"].to(of), new[1]], 1)
    logits = torch.matmul(s["q"].view(heads, gq * rows, D).to(of), k.transpose(1, 2)) * SCALE
    if "head_n" in s:
        logits[..., :c["tokens"]].masked_fill_(~_valid(s), -math.inf)
    hidden = ~s["sees"].expand(c["batch"], rows, rows)
    hidden = hidden.view(c["batch"], 1, 1, rows, rows).expand(c["batch"], c["hkv"], gq, rows, rows).reshape(heads, gq * rows, rows)
    logits[..., -rows:].masked_fill_(hidden, -math.inf)
    m = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - m)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total
    lse = m + torch.log(total)
    shape = (c["batch"], c["hq"], rows)
    return out.view(*shape, D), lse.view(shape)


def _weights_plain(s, of=torch.float32):
    """The new running sums, in place of the old ones"""
    c = s["case"]
    heads, n, gq = _heads(c), c["tokens"], c["hq"] // c["hkv"]
    got = torch.exp(_masked_logits(s, gq, of) - s["lse"].view(heads, -1, 1).to(of)).sum(1)
    w = s["weights"].view(heads, -1).to(of)
    if "head_n" not in s:
        w[:, :n + c["tail"]] = c["decay"] * w[:, :n + c["tail"]] + got
    else:
        tail = s["head_n"].view(-1, 1).long() + torch.arange(c["tail"], device=DEV)
        later = c["decay"] * w.gather(1, tail) + got[:, n:]
        w[:, :n] = torch.where(_valid(s).squeeze(1), c["decay"] * w[:, :n] + got[:, :n], w[:, :n])
        w.scatter_(1, tail, later)
    return w.view(s["weights"].shape)


def _survivors(w, c):
    """w: [heads, tokens] -> the kept positions, ascending; equal weights: the lower position"""
    heads, n, u = w.shape[0], c["tokens"], c["unit"]
    kept, short = _kept(c), n % u
    if kept == n:
        return torch.arange(n, device=DEV).expand(heads, n)
    score = w[:, :n - short].double().view(heads, -1, u).sum(-1).float()
    order = torch.sort(score, dim=1, descending=True, stable=True)[1][:, :(kept - short) // u]
    at = torch.sort(order, dim=1)[0]
    at = (at.unsqueeze(-1) * u + torch.arange(u, device=DEV)).flatten(1)
    return torch.cat([at, torch.arange(n - short, n, device=DEV).expand(heads, short)], 1)


def _rows_at(x, idx):
    return torch.gather(x, 1, idx.view(*idx.shape, *([1] * (x.dim() - 2))).expand(*idx.shape, *x.shape[2:]))


def _regroups(c):
    """Per-channel key groups that do not stay whole."""
    return c["bits"] != 16 and c["axis"] == PER_CHANNEL and c["unit"] % c["group"] != 0


def _whole_groups(idx, c):
    """Which of the survivors' groups were one group before, and the groups' first tokens, [heads, groups]"""
    kept, g = idx.shape[1], c["group"]
    start = torch.arange(0, kept, g, device=DEV)
    end = (start + g).clamp(max=kept)
    first, last = idx[:, start], idx[:, end - 1]
    return (first % g == 0) & (last - first == end - start - 1) & (end - start == (c["tokens"] - first).clamp(max=g)), first


def _evict_plain(s):
    c = s["case"]
    heads = _heads(c)
    w = s["weights"].view(heads, -1)
    idx = _survivors(w, c)
    rows = _up(idx.shape[1], 32)
    out = {"idx": idx.to(torch.int32).view(c["batch"], c["hkv"], -1), "tail_k": s["tail_k"].clone(), "tail_v": s["tail_v"].clone(),
           "weights": torch.cat([w.gather(1, idx), w[:, c["tokens"]:]], 1).view(c["batch"], c["hkv"], -1)}
    vc = _rows_at(_value_codes(s["v_codes"], c["bits"]), idx)
    if _regroups(c):
        x = _read(_key_codes(s["k_codes"], c["bits"])[:, :c["tokens"]], s["k_scale"], s["k_zero"], c, True, torch.float64)
        x = _rows_at(x.float().clamp(-65504, 65504).half(), idx)      # (one rounding to 32 bits, one to 16)
        kc, out["k_scale"], out["k_zero"] = _per_channel(x, c)
        # a group whose tokens were one group before stays as it was
        whole, first = _whole_groups(idx, c)
        kc = torch.where(whole.repeat_interleave(c["group"], 1)[:, :idx.shape[1]].unsqueeze(-1), _rows_at(_key_codes(s["k_codes"], c["bits"]), idx), kc)
        for k in ("k_scale", "k_zero"):
            out[k] = torch.where(whole.unsqueeze(-1), _rows_at(s[k], first // c["group"]), out[k])
    else:
        kc = _rows_at(_key_codes(s["k_codes"], c["bits"]), idx)
        if c["bits"] != 16 and c["axis"] == PER_CHANNEL:
            out["k_scale"], out["k_zero"] = (_rows_at(s[k], idx[:, ::c["group"]] // c["group"]) for k in ("k_scale", "k_zero"))
        elif c["bits"] != 16:
            out["k_scale"], out["k_zero"] = (_rows_of_zeros(_rows_at(s[k], idx), rows) for k in ("k_scale", "k_zero"))
    if c["bits"] != 16:
        out["v_scale"], out["v_zero"] = (_rows_of_zeros(_rows_at(s[k], idx), rows) for k in ("v_scale", "v_zero"))
    out["k_codes"], out["v_codes"] = _pack_keys(kc, c), _pack_values(vc, c)
    return out


def run(s):
    c = s["case"]
    if own:
        kvqp = s["kvqp"]
        if c["do"] == "tree":
            out = kvqp.tree_attn(s["cfg"], s["q"], s["k_new"], s["v_new"], s["trees"], s["cache"], lse=s["lse"], workspace=s["workspace"])
            return out, s["lse"]
        if c["do"] == "weights":
            return kvqp.accumulate_weights(s["cfg"], s["q"], s["lse"], s["cache"], s["weights"], decay=c["decay"])
        kvqp.evict(s["cfg"], s["cache"], s["weights"], c["keep"], s["dst"], weights_out=s["weights_out"], unit=c["unit"], idx_out=s["idx"],
                   workspace=s["workspace"])
        # (the packed words are returned as they are stored: equal words are equal codes, each of them)
        kept = {k: x for k, x in s["dst"].buffers.items() if x.numel()}
        return dict(kept, idx=s["idx"], weights=s["weights_out"])
    if c["do"] == "tree":
        out, s["lse"] = _tree_plain(s)
        return out.half(), s["lse"]
    if c["do"] == "weights":
        s["weights"] = _weights_plain(s)
        return s["weights"]
    return _evict_plain(s)


# ------------------------------------------------------------------------------------------- exact

def _exact_head(s, h):
    """One head's packed keys and values as 64-bit numbers, read from the header's statement of the layout."""
    c = s["case"]
    bits, n, g = c["bits"], _counts(c)[h], c["group"]
    t = torch.arange(n, device=DEV).view(-1, 1)
    d = torch.arange(D, device=DEV).view(1, -1)
    e, field = 32 // bits, 2 ** bits - 1
    r = d % e
    kc = (s["k_codes"][h].reshape(-1)[t * (D // e) + d // e] >> (bits * (r // 2) + 16 * (r % 2))) & field
    sb = 64 if bits == 2 else 32
    wpt = {16: 4, 8: 2}.get(bits, 1)
    low = t % sb
    blk, half, kb, i = low // 32, low // 16 % 2, low // 4 % 4, low % 4
    run_ = 4 * blk + i
    y = d // 16 * wpt + run_ // (e // 2)
    at = t // sb * (64 * 8 * wpt) + ((y // 4) * 64 + kb * 16 + d % 16) * 4 + y % 4
    vc = (s["v_codes"][h].reshape(-1)[at] >> (bits * (run_ % (e // 2)) + 16 * half)) & field
    if bits == 16:
        return tuple(x.to(torch.int16).view(torch.float16).double() for x in (kc, vc))
    gk = s["k_scale"][h].double(), s["k_zero"][h].double()
    k = kc.double() * (gk[0][t // g, d] if c["axis"] == PER_CHANNEL else gk[0][t, d // g])
    k = k + (gk[1][t // g, d] if c["axis"] == PER_CHANNEL else gk[1][t, d // g])
    v = vc.double() * s["v_scale"][h].double()[t, d // g] + s["v_zero"][h].double()[t, d // g]
    return k, v


def exact(case, seed):
    c = case
    s = _made(c, seed)
    gq, rows, t = c["hq"] // c["hkv"], c["rows"], c["tail"]
    if c["do"] == "tree":
        out = torch.empty((c["batch"], c["hq"], rows, D), dtype=torch.float64, device=DEV)
        lse = torch.empty((c["batch"], c["hq"], rows), dtype=torch.float64, device=DEV)
        for h in range(_heads(c)):
            b, g = divmod(h, c["hkv"])
            k, v = _exact_head(s, h)
            k = torch.cat([k, s["tail_k"][h].double(), s["k_new"][b, g].double()])
            v = torch.cat([v, s["tail_v"][h].double(), s["v_new"][b, g].double()])
            sees = s["sees"][b if c["trees"] == "own" else 0]
            sees = torch.cat([sees.new_ones(rows, k.shape[0] - rows), sees], 1)
            for a in range(g * gq, (g + 1) * gq):
                logits = (s["q"][b, a].double() @ k.t().contiguous()) * SCALE
                logits = torch.where(sees, logits, torch.full_like(logits, -math.inf))
                lse[b, a] = torch.logsumexp(logits, 1)
                out[b, a] = torch.softmax(logits, 1) @ v
        return out, lse
    if c["do"] == "weights":
        w = s["weights"].double()
        i = torch.arange(rows, device=DEV).view(-1, 1)
        for h in range(_heads(c)):
            b, g = divmod(h, c["hkv"])
            k = torch.cat([_exact_head(s, h)[0], s["tail_k"][h].double()])
            n = k.shape[0] - t
            seen = torch.arange(n + t, device=DEV) <= n + t - rows + i
            total = torch.zeros(n + t, dtype=torch.float64, device=DEV)
            for a in range(g * gq, (g + 1) * gq):
                p = torch.exp((s["q"][b, a].double() @ k.t().contiguous()) * SCALE - s["lse"][b, a].double().view(-1, 1))
                total += torch.where(seen, p, torch.zeros_like(p)).sum(0)
            w[b, g, :n + t] = c["decay"] * w[b, g, :n + t] + total
        return w
    # an eviction: moved numbers are what they were; only groups that are formed anew have scales that are computed
    res = {k: None for k in ("k_codes", "v_codes", "idx", "tail_k", "tail_v")}
    weights, ks, kz, vs, vz = [], [], [], [], []
    for h in range(_heads(c)):
        w = s["weights"].view(_heads(c), -1)[h].double().cpu()
        n, u, kept = c["tokens"], c["unit"], _kept(c)
        short = n % u
        score = w[:n - short].view(-1, u).sum(1).to(torch.float32 if u > 1 else torch.float64).tolist()
        best = sorted(range(len(score)), key=lambda j: (-score[j], j))[:(kept - short) // u] if kept < n else range(len(score))
        idx = [j * u + a for j in sorted(best) for a in range(u)] + list(range(n - short, n))
        weights.append(torch.cat([w[idx], w[n:]]))
        if c["bits"] == 16:
            continue
        rest = _up(kept, 32) - kept
        at = torch.tensor(idx, device=DEV)
        for into, name in ((vs, "v_scale"), (vz, "v_zero")):
            into.append(torch.cat([s[name][h][at].double(), torch.zeros(rest, D // c["group"], dtype=torch.float64, device=DEV)]))
        for into, name in ((ks, "k_scale"), (kz, "k_zero")):
            if c["axis"] == PER_TOKEN:
                into.append(torch.cat([s[name][h][at].double(), torch.zeros(rest, D // c["group"], dtype=torch.float64, device=DEV)]))
            elif not _regroups(c):
                into.append(s[name][h][at[::c["group"]] // c["group"]].double())
        if _regroups(c):
            x = _exact_head(s, h)[0][at].float().clamp(-65504, 65504).half().double()
            parts = x.split(c["group"])
            sets, g = [idx[j:j + c["group"]] for j in range(0, kept, c["group"])], c["group"]
            old = [p[0] // g if list(p) == list(range(p[0] // g * g, min(n, p[0] // g * g + g))) else None for p in sets]
            kz.append(torch.stack([p.amin(0) if o is None else s["k_zero"][h][o].double() for p, o in zip(parts, old)]))
            ks.append(torch.stack([(p.amax(0) - p.amin(0)) / (2 ** c["bits"] - 1) if o is None else s["k_scale"][h][o].double()
                                   for p, o in zip(parts, old)]))
    res["weights"] = torch.stack(weights).view(c["batch"], c["hkv"], -1)
    if c["bits"] != 16:
        res.update(k_scale=torch.stack(ks), k_zero=torch.stack(kz), v_scale=torch.stack(vs), v_zero=torch.stack(vz))
    return res
