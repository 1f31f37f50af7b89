"""Attention over pages with logits of any size that binary32 holds: rows far below zero and far above it, where a logit's own rounding is many powers of two."""
import math

import pytest
import torch

from paper_2412_12706_amd import kvqp
from tests.paged_util import BF16, D, HALF, Made, near, rows, starts_of
from tests.test_gpu_paged import FORMS, config, ints

pytestmark = pytest.mark.gpu


def call(cfg, made, q, counts):
    lse = torch.full(q.shape[:2], 77.0, device="cuda")
    out = kvqp.paged_attn(cfg, made.pages(), q.cuda(), ints(starts_of(counts)), lse=lse)
    return out.cpu(), lse.cpu().double()


def steps(t):      # roundings of the sums over t tokens, relative (tests.paged_util.attention)
    return (t / 32 + 80) * 2.0 ** -24


def made_with(g, length, page, dtype, form, key):
    """A sequence of one head whose keys are what `key` gives for their tokens in channel 3, and 0 elsewhere"""
    made = Made(g, [length], 1, page, dtype, form)
    made.k[0].zero_()
    made.k[0][0, :, 3] = key(torch.arange(length)).to(dtype)
    made.put(0, 0, length)
    assert torch.equal(made.numbers(0, "k")[0, :, 3], made.k[0][0, :, 3].double())      # (powers of two, and three times one: codes hold them)
    return made


# Few rows in one and in two tiles, and many; a few groups of tokens, and splits.
SHAPES = [(16, 300, 1), (32, 2900, 5), (64, 700, 9), (16, 2900, 40)]


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,length,count", SHAPES)
@pytest.mark.parametrize("log2", [20, 23, 28, 37, 99, 104, 126])
def test_rows_whose_logits_are_all_alike(dtype, form, page, length, count, log2):
    """Every weight is the same, so an output is the mean, whatever the logit; heads of one call have it positive, negative and small."""
    g = torch.Generator().manual_seed(log2)
    a = (14 if log2 > 50 else 10) if dtype is HALF else 50 if log2 > 50 else 5
    made = made_with(g, length, page, dtype, form, lambda t: torch.full(t.shape, 2.0 ** a))
    q = torch.zeros((count, 4, D), dtype=dtype)
    q[:, 0, 3], q[:, 1, 3], q[:, 2, 3], q[:, 3, 3] = 2.0 ** a, -(2.0 ** a), 2.0 ** -12, -1.5 * 2.0 ** (a - 1)
    scale = 0.7 * 2.0 ** (log2 - 2 * a)
    got, lse = call(config(1, 4, 1, scale), made, q, [count])
    v = made.numbers(0, "v")[0]
    scale = float(torch.tensor(scale, dtype=torch.float32))
    for i in range(count):
        seen = v[:length - count + 1 + i]
        n = len(seen)
        want = seen.mean(0).expand(4, D)
        off = (2.0 ** -11 + 2 * steps(n)) * seen.abs().mean(0).expand(4, D)
        near(got[i], want, off, dtype)
        want_lse = q[i, :, 3].double() * 2.0 ** a * scale + math.log(n)
        assert bool(((lse[i] - want_lse).abs() <= steps(n) + 2.0 ** -21 * want_lse.abs()).all())


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,length,count", SHAPES)
@pytest.mark.parametrize("log2", [12, 40, 101, 124])
def test_a_token_above_all_others(dtype, form, page, length, count, log2):
    """One token's logit is a third of the others', far below zero, or three times as large, above it: its value is the output."""
    g = torch.Generator().manual_seed(log2 + 1)
    a = (14 if log2 > 50 else 10) if dtype is HALF else 50 if log2 > 50 else 5
    for winner in (0, 77, length // 2, length - count - (length - count) % page - 1, length - count):
        for sign in (-1, 1):
            made = made_with(g, length, page, dtype, form, lambda t: torch.where((t == winner) == (sign > 0), 3.0, 1.0) * 2.0 ** a)
            q = torch.zeros((count, 1, D), dtype=dtype)
            q[:, 0, 3] = sign * 2.0 ** a
            got, lse = call(config(1, 1, 1, 2.0 ** (log2 - 2 * a)), made, q, [count])
            want = made.numbers(0, "v")[0, winner].expand(count, 1, D)
            near(got, want, 2.0 ** -11 * want.abs(), dtype)
            want_lse = sign * 2.0 ** log2 * (1 if sign < 0 else 3)
            assert bool(((lse - want_lse).abs() <= 2.0 ** -21 * abs(want_lse)).all())


@pytest.mark.parametrize("count", [1, 9, 40])
def test_queries_that_are_no_numbers_give_none(count):
    """An infinite query, or NaN, makes its own row NaN, beside rows that are far below zero."""
    g = torch.Generator().manual_seed(3)
    made = made_with(g, 400, 16, BF16, "e4m3", lambda t: torch.full(t.shape, 2.0 ** 50))
    q = torch.zeros((count, 4, D), dtype=BF16)
    q[:, 0, 3], q[:, 1, 3], q[:, 2, 3], q[:, 3, 3] = math.inf, -(2.0 ** 55), math.nan, 1.0
    got, _ = call(config(1, 4, 1, 1.0), made, q, [count])
    assert bool(got[:, [0, 2]].isnan().all())
    v = made.numbers(0, "v")[0]
    for i in range(count):
        seen = v[:400 - count + 1 + i]
        want = seen.mean(0).expand(2, D)
        near(got[i, [1, 3]], want, (2.0 ** -11 + 2 * steps(400)) * seen.abs().mean(0).expand(2, D), BF16)


@pytest.mark.parametrize("form", ["e4m3", "int8"])
@pytest.mark.parametrize("page,length,count", SHAPES)
@pytest.mark.parametrize("small", [-16, -20, -27])
def test_small_elements_of_a_query_that_meet_large_keys(form, page, length, count, small):
    """A bfloat16 query's largest element meets keys of 0, and one that is 2^16 .. 2^27 times smaller makes the logits."""
    g = torch.Generator().manual_seed(-small)
    made = Made(g, [length], 1, page, BF16, form)
    made.k[0].zero_()
    made.k[0][0, :, 9] = (torch.randint(-8, 9, (length,), generator=g) * 2.0 ** (-small - 3)).to(BF16)      # (whole numbers of up to 4 bits: codes hold them)
    made.put(0, 0, length)
    k, v = made.numbers(0, "k")[0], made.numbers(0, "v")[0]
    assert torch.equal(k, made.k[0][0].double())
    q = torch.zeros((count, 2, D), dtype=BF16)
    q[:, :, 40] = 1.75
    q[:, 0, 9], q[:, 1, 9] = 6.0 * (1 + 2.0 ** -7) * 2.0 ** small, -3.0 * (1 + 2.0 ** -6) * 2.0 ** small
    assert torch.equal(q[0, 1, 9].double(), torch.tensor(-3.0 * (1 + 2.0 ** -6) * 2.0 ** small, dtype=torch.float64))
    got, lse = call(config(1, 2, 1, 1.0), made, q, [count])
    for i in range(count):
        seen = slice(0, length - count + 1 + i)
        x = q[i].double() @ k[seen].t()
        w = torch.softmax(x, 1)
        # (logits of up to 6.1 are one product, and a multiplication by a factor that is rounded: 4 roundings)
        d = 4 * 2.0 ** -24 * 6.1
        off = (2.0 ** -11 + 2 * d + 2 * steps(length)) * (w @ v[seen].abs()) + length * 2.0 ** -28 * w.amax(1, keepdim=True) * v[seen].abs().amax(0)
        near(got[i], w @ v[seen], off, BF16)
        assert bool(((lse[i] - torch.logsumexp(x, 1)).abs() <= d + steps(length) + 2.0 ** -22 * 20).all())


@pytest.mark.parametrize("dtype,form", FORMS)
@pytest.mark.parametrize("page,length,count", SHAPES)
def test_small_values_beside_a_page_of_large_ones(dtype, form, page, length, count):
    """Rows that do not attend the page of the largest values see the others as they are, whose scales are 2^22 (binary16) and 2^26 times smaller."""
    g = torch.Generator().manual_seed(length)
    made = Made(g, [length], 1, page, dtype, form)
    apart = 22 if dtype is HALF else 26
    high, low = (2.0 ** 13, 2.0 ** (13 - apart)) if dtype is HALF else (2.0 ** 40, 2.0 ** (40 - apart))
    v = torch.randn((1, length, D), generator=g).clamp(-4, 4) * low
    v[:, page:2 * page] *= high / low
    made.v[0] = v.to(dtype)
    made.k[0].zero_()
    made.k[0][0, page:2 * page, 3] = -128.0
    made.put(0, 0, length)
    q = torch.zeros((count, 1, D), dtype=dtype)
    q[:, 0, 3] = 2.0
    got, _ = call(config(1, 1, 1, 1.0), made, q, [count])
    v = made.numbers(0, "v")[0]
    for i in range(count):
        n = length - count + 1 + i
        seen = torch.cat([v[:page], v[2 * page:n]])
        # the large ones' weights are e^-256; a value of this type is as near as 2^-24 of the number that a code of 1 stands for in the largest scale times what lies
        # between that and a half's largest: 2^7 for e4m3, 2^5 for integers
        scale = high * 8 / (448 if form == "e4m3" else 127)
        off = (2.0 ** -11 + 2 * steps(n)) * seen.abs().mean(0) + 2.0 ** -25 * scale / (128 if form == "e4m3" else 32)
        near(got[i, 0], seen.mean(0), off, dtype)
