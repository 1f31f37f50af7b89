"""Performance cases of rotary positions and the paged 8-bit cache.

A serving program holds the prompts and sequences that are not pruned yet in pages: blocks of a few
tokens, 8 bits an element, one power-of-two scale for each block and KV head, keys and values apart.
Four things are asked of it.  Rows are rotated to their positions (`rotate`); new rows are rotated and
appended, blocks that became full are quantized (`paged_append`); queries -- one row of each sequence,
a few drafted ones, or a piece of a prompt -- attend over the pages (`paged_attn`); and a prompt is
taken out again as plain rows, to be pruned by `compress` (`paged_read`).  The listed cases walk the
sizes at which this is done, from one row of one sequence up; `draw` gives others of the same ranges.

The cache here is made from standard normal keys and values (four key channels per head scaled up, as
in the repository's tests) by the quantizer's definition in plain torch.  The plain forms read pages
with index operations, work in 32 bits and round once; `exact` redoes everything in 64 bits.
"""
import math

import torch

own = False
D = 128
DEV = "cuda"
SCALE = 128 ** -0.5


# ------------------------------------------------------------------------------------------- cases

def _case(name, do, batch, hq, hkv, rows, tokens, page=16, dtype="half", form="e4m3", ragged=False, rot=128, interleaved=False,
          inverse=False, window=0):
    """rows: new rows of a sequence (the most, where they differ), tokens: its length with them (the longest); ragged: every sequence
    has its own number of both; rot: rotated channels."""
    c = {"do": do, "batch": batch, "hq": hq, "hkv": hkv, "rows": rows, "tokens": tokens, "page": page, "dtype": dtype, "form": form,
         "ragged": ragged, "rot": rot, "interleaved": interleaved, "inverse": inverse, "window": window}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # The queries of a decode step of 32 sequences, each at a position of its own: latency counts.
        _case("rotate-step", "rotate", 32, 32, 8, 1, 8192, ragged=True),
        # A prompt's queries as a slice of a fused projection, neighbouring channels in pairs, half of the head; the way back (a gradient).
        _case("rotate-prompt-part", "rotate", 2, 32, 8, 16381, 16381, dtype="bfloat16", rot=64, interleaved=True, inverse=True),
        # One new token of one sequence.
        _case("append-1", "append", 1, 32, 8, 1, 1024),
        # A decode step of many sequences of their own lengths; every sixteenth of them completes a block.
        _case("append-step", "append", 96, 32, 8, 1, 4096, form="int8", dtype="bfloat16", ragged=True),
        # Prompts of odd lengths together.
        _case("append-prompts", "append", 4, 32, 8, 8191, 8191, page=32, ragged=True),
        # Attention of one new token over a short cache.
        _case("attn-1-short", "attn", 1, 32, 8, 1, 1024),
        # A decode step of 32 long sequences.
        _case("attn-step", "attn", 32, 32, 8, 1, 8192),
        # Drafted chains of 5 tokens, sequences of their own lengths, eight query heads per KV head.
        _case("attn-drafted", "attn", 48, 64, 8, 5, 16001, page=32, dtype="bfloat16", form="int8", ragged=True),
        # A whole prompt: the largest amount of products.
        _case("attn-prompt", "attn", 1, 32, 8, 8192, 8192, page=64),
        # A piece of a prompt over what went before, within a sliding window, one query head per KV head.
        _case("attn-piece", "attn", 2, 16, 16, 509, 12345, page=16, dtype="bfloat16", window=4096, ragged=True),
        # A short prompt goes to be pruned.
        _case("read-short", "read", 1, 32, 8, 0, 999),
        # Long prompts go to be pruned.
        _case("read-long", "read", 2, 32, 8, 0, 32768, page=32, form="int8"),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    do = rng.choice(("rotate", "append", "attn", "attn", "attn", "read"))
    hkv = rng.choice((1, 2, 4, 8, 16))
    hq = hkv * rng.choice((1, 2, 4, 8))
    page = rng.choice((16, 32, 64))
    dtype, form = rng.choice(("half", "bfloat16")), rng.choice(("e4m3", "int8"))
    ragged, window = rng.choice((True, False)), 0
    rot, interleaved = rng.choice((32, 64, 96, 128, 128, 128)), rng.choice((True, False))
    batch = _between(rng, 1, 128)
    if do == "rotate":
        tokens = _between(rng, 1, max(1, min(32768, (1 << 20) // (batch * hq))))
        rows = rng.choice((1, tokens))
    elif do == "append":
        tokens = _between(rng, 1, max(1, min(16384, (1 << 17) // batch)))
        rows = rng.choice((1, 1, min(tokens, rng.randint(2, 9)), max(1, min(tokens, (1 << 20) // (batch * hq)))))
    elif do == "attn":
        # (at most 2^21 tokens over all heads, and no more products than the whole prompt's)
        tokens = _between(rng, 1, min(65536, (1 << 21) // (batch * hkv)))
        most = max(1, min(tokens, (1 << 30) // (tokens * batch * hq)))
        rows = rng.choice((1, min(most, rng.randint(2, 9)), _between(rng, 1, most)))
        window = rng.choice((0, 0, 0, _between(rng, 1, tokens)))
    else:
        tokens, rows = _between(rng, 1, max(1, min(65536, (1 << 19) // (batch * hkv)))), 0
    return _case(None, do, batch, hq, hkv, rows, tokens, page, dtype, form, ragged, rot, interleaved, rng.choice((True, False)) and do == "rotate", window)


def _lengths(c):
    """Every sequence's length with its new rows, and the number of those: all alike, or their own."""
    b, n, t = c["batch"], c["rows"], c["tokens"]
    own_n, own_t = [n] * b, [t] * b
    if c["ragged"] and c["do"] == "append" and n == t:      # prompts that are appended whole
        own_n = own_t = [max(1, t - (i * 7919 % 61) * t // 100) for i in range(b)]
    elif c["ragged"]:
        own_n = [max(min(n, 1), n - (i * 5 % 7) * n // 13) for i in range(b)]
        own_t = [max(m, t if i == 0 else 1 + (i * 7919 % 101) * (t - 1) // 101) for i, m in enumerate(own_n)]
    if c["do"] == "append" and n >= c["page"]:
        # (a pass that fills whole blocks starts at one, so that it can be repeated)
        own_t = [m + (x - m) // c["page"] * c["page"] for m, x in zip(own_n, own_t)]
    return own_t, own_n


def _seen(c):
    """How many (row, token) pairs attention has, over all sequences."""
    total = 0
    for t, n in zip(*_lengths(c)):
        w = c["window"] or t
        first = t - n + 1       # tokens that the first row sees, without a window
        full = min(n, max(0, w - first))
        total += full * first + full * (full - 1) // 2 + (n - full) * w
    return total


def work(c):
    lengths, rows = _lengths(c)
    n, row = sum(rows), 2 * D
    if c["do"] == "rotate":
        vectors = c["batch"] * c["rows"] * c["hq"]
        return {"bytes": vectors * 2 * row + (c["batch"] if c["rows"] == 1 else 1) * c["rows"] * c["rot"] * 4, "flops": 3 * vectors * c["rot"]}
    if c["do"] == "append":
        closed = sum(t // c["page"] - (t - m) // c["page"] for t, m in zip(lengths, rows)) * c["page"]
        kept = sum(min(m, 2 * c["page"]) for m in rows)
        return {"bytes": n * (2 * c["hq"] + 2 * c["hkv"]) * row + closed * c["hkv"] * 2 * D + kept * c["hkv"] * 2 * row + n * c["rot"] * 4,
                "flops": 3 * n * (c["hq"] + c["hkv"]) * c["rot"] + 4 * closed * c["hkv"] * D}
    if c["do"] == "attn":
        read = sum(min(t, (c["window"] or t) + m - 1) for t, m in zip(lengths, rows))
        return {"bytes": read * c["hkv"] * 2 * (D + 4 / c["page"]) + n * c["hq"] * (2 * row + 4), "flops": 4 * D * c["hq"] * _seen(c)}
    return {"bytes": sum(lengths) * c["hkv"] * 2 * D + c["batch"] * c["tokens"] * c["hkv"] * 2 * row, "flops": sum(lengths) * c["hkv"] * 2 * D}


# ------------------------------------------------------------------------------------------ inputs

def _type(c):
    return torch.float16 if c["dtype"] == "half" else torch.bfloat16


def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _table(n, rot, base=500000.0):
    """cos and sin of every position and pair, [n, rot / 2, 2]: 64-bit angles, rounded once"""
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)
    a = torch.arange(n, dtype=torch.float64, device=DEV).unsqueeze(1) * f
    return torch.stack([torch.cos(a), torch.sin(a)], -1).float()


def _two_to(e):
    """2 ** e as float32, exactly, for -126 <= e <= 127"""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _quantize(x, form):
    """Blocks [..., tokens, channels] of 16-bit values -> codes, scales [...]: the least power of two that holds the largest."""
    m, e = torch.frexp(x.abs().amax((-2, -1)).float())
    e = torch.where(m <= 0.875, e - 9, e - 8) if form == "e4m3" else torch.where(m <= 127 / 128, e - 7, e - 6)
    e = torch.where(m == 0, -126, e).clamp(min=-126)
    y = x.float() * _two_to(-e)[..., None, None]
    return (y.to(torch.float8_e4m3fn) if form == "e4m3" else torch.round(y).to(torch.int8)), _two_to(e)


def _made(c, seed):
    """The tensors of a case."""
    g, dtype = _generator(seed), _type(c)
    lengths, rows = _lengths(c)
    b, hq, hkv, p = c["batch"], c["hq"], c["hkv"], c["page"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)

    s = {"case": c, "lengths": lengths, "rows": rows}
    if c["do"] in ("rotate", "append"):
        s["table"] = _table(max(lengths), c["rot"])
    if c["do"] == "rotate":
        n = c["rows"]
        fused = normal(b, n, (hq + 2 * hkv) * D).to(dtype)
        s["x"] = fused[..., :hq * D].view(b, n, hq, D).transpose(1, 2)          # [batch, heads, rows, D], as the projection left it
        s["positions"] = torch.tensor([[t - m] for t, m in zip(lengths, rows)], dtype=torch.int32, device=DEV) if n == 1 else None
        return s

    # pages in any order, and the 16-bit rows of the last two blocks of each sequence
    most = max(1, -(-max(lengths) // p))
    s["table_of_pages"] = torch.randperm(b * most, generator=g, device=DEV).to(torch.int32).view(b, most)
    s["device_lengths"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    starts = [0]
    for m in rows:
        starts.append(starts[-1] + m)
    s["row_start"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    loud = torch.ones((hkv, D), device=DEV)
    at = torch.arange(hkv, device=DEV).view(-1, 1) * 29 + 7 + torch.arange(4, device=DEV) * 37
    loud.scatter_(1, at % D, 10.0)
    fp8 = torch.float8_e4m3fn if c["form"] == "e4m3" else torch.int8
    for name, by in (("k", loud.view(1, hkv, 1, D)), ("v", 1.0)):
        codes = torch.empty((b * most, hkv, p, D) if name == "k" else (b * most, hkv, D, p), dtype=fp8, device=DEV)
        scale = torch.empty((b * most, hkv), device=DEV)
        ring = torch.zeros((b, hkv, 2 * p, D), dtype=dtype, device=DEV)
        for i in range(b):
            page = s["table_of_pages"][i].long()
            x = (normal(most, hkv, p, D) * by).to(dtype)
            q, f = _quantize(x, c["form"])
            codes.view(torch.uint8)[page] = (q if name == "k" else q.view(torch.uint8).transpose(2, 3)).view(torch.uint8)
            scale[page] = f
            last = max(0, (lengths[i] - 1) // p)
            for block in (max(0, last - 1), last):
                ring[i, :, block % 2 * p:(block % 2 + 1) * p] = x[block]
        s[name + "_codes"], s[name + "_scale"], s["open_" + name] = codes, scale, ring
    if c["do"] == "append":
        n = starts[-1]
        s["q"], s["v"] = normal(n, hq, D).to(dtype), normal(n, hkv, D).to(dtype)
        s["k"] = (normal(n, hkv, D) * loud).to(dtype)
    elif c["do"] == "attn":
        s["q"] = normal(starts[-1], hq, D).to(dtype)
    return s


def _handle(s):
    """What a program that uses the library holds: the configuration, the pages, and buffers for results."""
    from paper_2412_12706_amd import kvqp
    c = s["case"]
    s["kvqp"] = kvqp
    s["cfg"] = kvqp.Cfg(batch=c["batch"], n_q_heads=c["hq"], n_kv_heads=c["hkv"], sm_scale=SCALE)
    if "table" in s:
        s["rope"] = kvqp.Rope(s["table"], c["rot"], c["interleaved"])
    if c["do"] == "rotate":
        s["out"] = torch.empty((c["batch"], c["hq"], c["rows"], D), dtype=_type(c), device=DEV)
        return
    s["pages"] = kvqp.Pages(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["open_k"], s["open_v"], s["table_of_pages"], s["device_lengths"])
    if c["do"] == "append":
        s["q_out"] = torch.empty_like(s["q"])
    elif c["do"] == "attn":
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        s["workspace"] = kvqp.alloc_paged_workspace(s["cfg"], s["q"].shape[0])
    else:
        s["k_out"], s["v_out"] = (torch.empty((c["batch"], c["hkv"], c["tokens"], D), dtype=_type(c), device=DEV) for _ in range(2))


def prepare(case, seed):
    s = _made(case, seed)
    if own:
        _handle(s)
    return s


# ------------------------------------------------------------------------------------- plain forms

def _rotated(x, cs, c):
    """x: [..., D] in 32 or 64 bits, cs: [..., rot / 2, 2] to match"""
    r = c["rot"]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    cos, sin = cs[..., 0], -cs[..., 1] if c["inverse"] else cs[..., 1]
    y = [a * cos - b * sin, b * cos + a * sin]
    y = torch.stack(y, -1).flatten(-2) if c["interleaved"] else torch.cat(y, -1)
    return torch.cat([y, x[..., r:]], -1)


def _rotate_plain(s):
    c = s["case"]
    cs = s["table"][s["positions"].long()].unsqueeze(1) if s["positions"] is not None else s["table"][:c["rows"]]
    return _rotated(s["x"].float(), cs, c).to(_type(c))


def _row_owners(s):
    """Of every new row: its sequence and its position"""
    n = s["row_start"][1:] - s["row_start"][:-1]
    total = s["q"].shape[0]
    seq = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), n, output_size=total)
    first = s["device_lengths"] - n - s["row_start"][:-1]
    return seq, torch.arange(total, device=DEV) + first[seq]


def _finite(x, dtype):
    most = torch.finfo(dtype).max
    return torch.nan_to_num(x, nan=0.0, posinf=most, neginf=-most).clamp(-most, most).to(dtype)


def _append_plain(s):
    c, dtype, p = s["case"], _type(s["case"]), s["case"]["page"]
    seq, pos = _row_owners(s)
    cs = s["table"][pos].unsqueeze(1)
    q = _rotated(s["q"].float(), cs, c).to(dtype)
    new = {"k": _finite(_rotated(s["k"].float(), cs, c), dtype), "v": _finite(s["v"].float(), dtype)}
    # the blocks that are full now: tokens from the new rows, or from the open block's
    n = s["row_start"][1:] - s["row_start"][:-1]
    before = s["device_lengths"] - n
    full = s["device_lengths"] // p - before // p
    total = sum(t // p - (t - m) // p for t, m in zip(s["lengths"], s["rows"]))
    if total:
        owner = torch.repeat_interleave(torch.arange(n.numel(), device=DEV), full, output_size=total)
        block = torch.arange(total, device=DEV) - (torch.cumsum(full, 0) - full)[owner] + before[owner] // p
        token = block.unsqueeze(1) * p + torch.arange(p, device=DEV)
        row = token - before[owner].unsqueeze(1)
        source = (row + s["row_start"][owner].unsqueeze(1)).clamp(min=0)
        page = s["table_of_pages"][owner, block].long()
        for name in ("k", "v"):
            old = s["open_" + name][owner.unsqueeze(1), :, token % (2 * p)]
            x = torch.where((row >= 0)[..., None, None], new[name][source], old).transpose(1, 2)
            codes, s[name + "_scale"][page] = _quantize(x, c["form"])
            bytes_ = codes.view(torch.uint8)
            s[name + "_codes"].view(torch.uint8)[page] = bytes_ if name == "k" else bytes_.transpose(2, 3)
    # the open block and the one before it stay in 16 bits
    last = (s["device_lengths"].clamp(min=1) - 1) // p
    stays = pos >= (last[seq] - 1) * p
    slot = torch.where(stays, pos % (2 * p), 0)
    for name in ("k", "v"):
        ring = s["open_" + name]
        # (rows that do not stay go to a place behind the last)
        at = torch.where(stays, seq * (2 * p) + slot, ring.shape[0] * 2 * p)
        flat = torch.cat([ring.transpose(1, 2).flatten(0, 1), ring.new_empty(1, *ring.shape[1:2], D)])
        flat[at] = new[name]
        ring.copy_(flat[:-1].view(ring.shape[0], 2 * p, *ring.shape[1:2], D).transpose(1, 2))
    return q


def _tokens(s, name, count, of=torch.float32):
    """The first `count` tokens of every sequence as numbers, [batch, heads, count, D]: pages, and the open block in 16 bits"""
    c, p = s["case"], s["case"]["page"]
    pages = -(-count // p)
    at = s["table_of_pages"][:, :pages].long()
    x = s[name + "_codes"].view(torch.uint8)[at].view(s[name + "_codes"].dtype)
    if name == "v":
        x = x.transpose(-1, -2)
    x = (x.to(of) * s[name + "_scale"][at].to(of)[..., None, None]).transpose(1, 2).flatten(2, 3)[:, :, :count]
    token = torch.arange(count, device=DEV)
    begin = s["device_lengths"].view(-1, 1) // p * p
    ring = s["open_" + name][:, :, token % (2 * p)].to(of)
    return torch.where((token >= begin)[:, None, :, None], ring, x)


def _attn_plain(s):
    c = s["case"]
    b, hq, hkv = c["batch"], c["hq"], c["hkv"]
    gq, most, count = hq // hkv, max(s["rows"]), max(s["lengths"])
    seq, pos = _row_owners(s)
    place = torch.arange(pos.numel(), device=DEV) - s["row_start"][seq]
    q = torch.zeros((b, most, hq, D), device=DEV)
    q[seq, place] = s["q"].float()
    q = q.view(b, most, hkv, gq, D).permute(0, 2, 3, 1, 4).reshape(b * hkv, gq * most, D)
    k, v = (_tokens(s, name, count).reshape(b * hkv, count, D) for name in ("k", "v"))
    logits = torch.matmul(q, k.transpose(1, 2).contiguous()).view(b, hkv, gq, most, count) * SCALE
    n = s["row_start"][1:] - s["row_start"][:-1]
    at = ((s["device_lengths"] - n).view(-1, 1) + torch.arange(most, device=DEV)).unsqueeze(-1)
    token = torch.arange(count, device=DEV)
    hidden = token > at
    if c["window"]:
        hidden = hidden | (token <= at - c["window"])
    logits.masked_fill_(hidden[:, None, None], -math.inf)
    m = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    w = torch.exp(logits.sub_(m))
    total = w.sum(-1, keepdim=True)
    out = torch.matmul(w.view(b * hkv, gq * most, count), v).view(b, hkv, gq, most, D) / total
    lse = m + torch.log(total)
    out, lse = (x.permute(0, 3, 1, 2, 4).reshape(b, most, hq, -1)[seq, place] for x in (out, lse))
    return out.to(_type(c)), lse.squeeze(-1)


def _read_plain(s):
    c = s["case"]
    live = (torch.arange(c["tokens"], device=DEV) < s["device_lengths"].view(-1, 1))[:, None, :, None]
    most = torch.finfo(_type(c)).max
    return tuple(torch.where(live, _tokens(s, name, c["tokens"]), 0.0).clamp(-most, most).to(_type(c)) for name in ("k", "v"))


def run(s):
    c = s["case"]
    if own:
        kvqp = s["kvqp"]
        if c["do"] == "rotate":
            return kvqp.rotate(s["rope"], s["x"], s["positions"], out=s["out"], inverse=c["inverse"])
        if c["do"] == "attn":
            kvqp.paged_attn(s["cfg"], s["pages"], s["q"], s["row_start"], window=c["window"], out=s["out"], lse=s["lse"], workspace=s["workspace"])
            return s["out"], s["lse"]
        if c["do"] == "read":
            return kvqp.paged_read(s["cfg"], s["pages"], c["tokens"], k_out=s["k_out"], v_out=s["v_out"])
        q = kvqp.paged_append(s["cfg"], s["pages"], s["k"], s["v"], s["row_start"], q=s["q"], q_out=s["q_out"], rope=s["rope"])
    else:
        if c["do"] == "rotate":
            return _rotate_plain(s)
        if c["do"] == "attn":
            return _attn_plain(s)
        if c["do"] == "read":
            return _read_plain(s)
        q = _append_plain(s)
    return {"q": q, **{name: s[name] for name in ("k_codes", "v_codes", "k_scale", "v_scale", "open_k", "open_v")}}


# ------------------------------------------------------------------------------------------- exact

def _exact_rotated(x, pos, c, base=500000.0):
    """x: [rows, heads, D] in 64 bits at 64-bit positions, pair by pair (the sines and cosines are inputs of 32 bits)"""
    y = x.clone()
    half = c["rot"] // 2
    for j in range(half):
        i, k = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
        a = pos.double() * base ** (-2.0 * j / c["rot"])
        cos, sin = (f(a).float().double().unsqueeze(-1) for f in (torch.cos, torch.sin))
        if c["inverse"]:
            sin = -sin
        y[..., i] = x[..., i] * cos - x[..., k] * sin
        y[..., k] = x[..., i] * sin + x[..., k] * cos
    return y


def _exact_tokens(s, name, i, h):
    """One sequence's keys or values of one head in 64 bits, block by block"""
    c, p, n = s["case"], s["case"]["page"], s["lengths"][i]
    page = s["table_of_pages"][i][:n // p].long()
    x = s[name + "_codes"].view(torch.uint8)[page, h].view(s[name + "_codes"].dtype).double()
    x = (x if name == "k" else x.transpose(1, 2)) * s[name + "_scale"][page, h].double().view(-1, 1, 1)
    begin = n // p * p
    rest = [t % (2 * p) for t in range(begin, n)]
    return torch.cat([x.reshape(-1, D), s["open_" + name][i, h][rest].double()])


def exact(case, seed):
    c = case
    s = _made(c, seed)
    if c["do"] == "rotate":
        n = c["rows"]
        pos = s["positions"].view(-1, 1).expand(-1, n) if n == 1 else torch.arange(n, device=DEV).expand(c["batch"], n)
        x = s["x"].transpose(1, 2).double()
        return _exact_rotated(x.reshape(-1, c["hq"], D), pos.reshape(-1), c).view(x.shape).transpose(1, 2).contiguous()
    if c["do"] == "append":
        pos = torch.cat([torch.arange(t - m, t, device=DEV) for t, m in zip(s["lengths"], s["rows"])])
        k, v = _exact_rotated(s["k"].double(), pos, c), s["v"].double()
        got = {"q": _exact_rotated(s["q"].double(), pos, c)}
        for name, x in (("k", k), ("v", v)):
            ring, at, p = s["open_" + name].double(), 0, c["page"]
            for i, (t, m) in enumerate(zip(s["lengths"], s["rows"])):
                begin = max(t - m, max(0, (t - 1) // p - 1) * p)
                for j in range(begin, t):
                    ring[i, :, j % (2 * p)] = x[at + j - (t - m)]
                at += m
            got["open_" + name] = ring
            # (codes and scales are whole numbers and powers of two of rounded rows: nothing that 64 bits would have otherwise)
            got[name + "_codes"] = got[name + "_scale"] = None
        return got
    if c["do"] == "read":
        got = []
        for name in ("k", "v"):
            x = torch.zeros((c["batch"], c["hkv"], c["tokens"], D), dtype=torch.float64, device=DEV)
            for i in range(c["batch"]):
                for h in range(c["hkv"]):
                    x[i, h, :s["lengths"][i]] = _exact_tokens(s, name, i, h)
            got.append(x)
        return tuple(got)
    gq, at = c["hq"] // c["hkv"], 0
    out = torch.empty((s["q"].shape[0], c["hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.empty((s["q"].shape[0], c["hq"]), dtype=torch.float64, device=DEV)
    for i, (t, m) in enumerate(zip(s["lengths"], s["rows"])):
        pos = torch.arange(t - m, t, device=DEV).view(-1, 1)
        token = torch.arange(t, device=DEV)
        sees = (token <= pos) & (token > pos - (c["window"] or t + 1))
        for h in range(c["hkv"]):
            k, v = (_exact_tokens(s, name, i, h) for name in ("k", "v"))
            for a in range(h * gq, (h + 1) * gq):
                logits = (s["q"][at:at + m, a].double() @ k.t().contiguous()) * SCALE
                logits = torch.where(sees, logits, torch.full_like(logits, -math.inf))
                lse[at:at + m, a] = torch.logsumexp(logits, 1)
                out[at:at + m, a] = torch.softmax(logits, 1) @ v
        at += m
    return out, lse
