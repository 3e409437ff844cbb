"""Attention over a cache on the GPU where keys, values or scales are at the ends of their types' ranges."""
import math

import pytest

from test_gpu_attention_forms import Case, no_wait_gave_up, tdt  # noqa: F401 (a fixture of every test)

pytestmark = pytest.mark.gpu

# new tokens, before: in one piece and shared out, single tokens and several, and prompts
SIZES = [([1], [70]), ([1], [3000]), ([5], [300]), ([90], [200])]


def at(c, b, i):
    """(page, place) of position i of sequence b."""
    return int(c.table[b, i // c.page]), i % c.page


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
def test_keys_of_minus_infinity(dt, new, before):
    """A score of -inf counts nothing, and where there is no other the result is zero."""
    import torch
    c = Case(dt, "plain", new, before, 4, 1, 64, 16, seed=1)
    c.t[0].zero_()
    c.t[0][:, :, :, 0] = -math.inf
    c.q[..., 0] = 1.0
    assert not c.run().any()
    n, i = at(c, 0, 5)
    c.t[0][n, 0, i, 0] = 2.0  # the one key that counts
    assert torch.equal(c.run(), c.t[1][n, 0, i].expand_as(c.q))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
def test_values_that_are_infinite(dt, new, before):
    """A weight times infinity is infinity, of both signs NaN; the head's other values do not change."""
    import torch
    c = Case(dt, "plain", new, before, 4, 2, 64, 16, seed=2)
    c.q.mul_(0.1)  # (every weight is above the smallest that fp16 holds next to the largest)
    want = c.run()
    n, i = at(c, 0, 33)
    c.t[1][n, 0, i, 7], c.t[1][n, 0, i, 60] = math.inf, -math.inf
    c.t[1][n, 1, i, 0] = math.inf
    n, i = at(c, 0, 50)
    c.t[1][n, 1, i, 0] = -math.inf
    y = c.run()
    keep = torch.ones_like(y, dtype=torch.bool)
    keep[:, :2, 7] = keep[:, :2, 60] = keep[:, 2:, 0] = False
    c.t[1][~c.t[1].isfinite()] = 0
    assert y[keep].isfinite().all()
    assert (y[:, :2, 7] == math.inf).all() and (y[:, :2, 60] == -math.inf).all() and y[:, 2:, 0].isnan().all()
    # (computed again or not: off by what the two may be off)
    close = 4 * 2.0 ** {"f32": -18, "f16": -10, "bf16": -7}[dt]
    assert ((y[keep].double() - want[keep].double()).abs() <= close * c.t[1].abs().max().double()).all()


@pytest.mark.parametrize("new, before", SIZES)
def test_fp32_keys_that_round_to_infinity_in_fewer_bits(new, before):
    """The largest fp32 values are beyond tf32's range when rounded to it; equal scores average the values."""
    import torch
    c = Case("f32", "plain", new, before, 2, 1, 32, 16, seed=3)
    c.t[0].zero_()
    c.t[0][..., 4], c.q[..., 4] = torch.finfo(torch.float32).max, 2.0 ** -126  # (a product of 4)
    y = c.run()
    v = torch.cat([c.t[1][n, 0] for n in c.table[0] if n >= 0]).double()
    mean = v.cumsum(0)[before[0]:before[0] + new[0]] / (before[0] + 1 + torch.arange(new[0], device="cuda")[:, None])
    # a weight is off by its exponential's argument and 2 ulp, twice; a sum of n keys by n roundings
    assert ((y.double() - mean[:, None]).abs() <= (before[0] + 100) * 2.0 ** -22 * v.abs().max()).all()


def test_fp32_value_that_rounds_to_infinity_in_fewer_bits():
    import torch
    c = Case("f32", "plain", [1], [0], 2, 1, 32, 16, seed=4)
    c.t[1][..., 3], c.t[1][..., 5] = torch.finfo(torch.float32).max, -torch.finfo(torch.float32).max
    n, i = at(c, 0, 0)
    y, v = c.run(), c.t[1][n, 0, i].expand_as(c.q)
    assert torch.equal(y[..., 3], v[..., 3]) and torch.equal(y[..., 5], v[..., 5])
    # The weight is 1.  A value goes in as its nearest tf32 (11 bits; the rest is at most 2^-11 of it) and that rest, of which the
    # tensor cores take 11 bits: what they drop is below 2^-10 of the rest, 2^-21 of the value; the sum and its scaling are 3 roundings
    # of 2^-24, one of them truncated: below 2^-21 too.
    assert ((y - v).abs() <= 2.0 ** -20 * v.abs()).all()


@pytest.mark.parametrize("new, before", SIZES + [([1, 3, 1], [2500, 40, 900])])
@pytest.mark.parametrize("dt, far", [(dt, f) for dt in ("f32", "f16", "bf16") for f in (2.0 ** -100, 1e-36, 2.0 ** -149, 2.0 ** 40, 2.0 ** 100)
                                     if dt != "f16" or f < 1])
@pytest.mark.parametrize("where", ["first", "some", "all"])
def test_codes_with_far_scales_of_values(dt, new, before, far, where):
    """Values next to zero, or huge, beside others or alone, weigh what their scores say."""
    import torch
    c = Case(dt, "q8", new, before, 4, 2, 64, 16, seed=5)
    scale = c.t[3]
    if where == "first":
        for b in range(len(new)):
            scale[at(c, b, 0)[0], 0, :9] = far
    elif where == "some":
        scale[torch.rand(scale.shape, generator=c.g, device="cuda") < 0.3] = far
    else:
        scale.fill_(far)
    # a weight over codes is one fp16 part for bf16, two for the others
    c.check(c.run(), 2.0 ** (-11 if dt == "bf16" else -21))


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
def test_codes_behind_what_is_seen_do_not_matter(dt, new, before):
    """Scales of every kind in the places behind a sequence."""
    import torch
    c = Case(dt, "q8", new, before, 4, 2, 64, 256, seed=6)
    want = c.run()
    n, i = at(c, 0, new[0] + before[0] - 1)
    for j, far in enumerate([0.0, 2.0 ** -149, 2.0 ** 127, math.inf, -math.inf, math.nan, -math.nan]):
        if i + 1 + j < c.page:
            c.t[2][n, :, i + 1 + j], c.t[3][n, :, i + 1 + j] = far, far
    assert torch.equal(c.run(), want)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
def test_the_largest_values(dt, new, before):
    """An average of largest values is one, although their sum is beyond the range."""
    import torch
    top = torch.finfo(tdt(dt)).max
    c = Case(dt, "plain", new, before, 4, 2, 64, 16, seed=7)
    c.t[1][..., 3], c.t[1][..., 9] = top, -top
    y = c.run()
    # (weights, their sum and the division are off by some 2^-20 in all; in fp16 and bf16 a result next to the top rounds to it)
    for at_, want in ((3, top), (9, -top)):
        assert ((y[..., at_].double() - want).abs() <= top * (2.0 ** -18 if dt == "f32" else 0)).all()
    assert y.isfinite().all()


FORMS = [([90], [200], 4, 2, 64, 16), ([200], [0], 4, 2, 128, 128), ([90], [0], 2, 1, 256, 64), ([100, 70], [3000, 10], 4, 2, 256, 32),
         ([130, 1, 90], [2500, 900, 300], 4, 1, 128, 64), ([6, 1], [2000, 90], 4, 2, 64, 16)]


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("f16", "plain"), ("bf16", "plain"), ("f16", "q8"), ("bf16", "q8"), ("f32", "q8")])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", FORMS)
@pytest.mark.parametrize("what", ["key", "value", "late value"])
def test_nan_reaches_those_that_see_it(dt, kind, new, before, q_heads, heads, dim, page, what):
    """One NaN in a key or value of the first sequence: rows before it and other sequences and heads stay, those behind it are NaN (of a value:
    in its place)."""
    import torch
    c = Case(dt, kind, new, before, q_heads, heads, dim, page, seed=8)
    want = c.run()
    j = before[0] + new[0] - 3 if what == "late value" else before[0] // 2 + 1
    n, i = at(c, 0, j)
    if kind == "q8":
        c.t[2 if what == "key" else 3][n, 0, i] = math.nan
    else:
        c.t[0 if what == "key" else 1][n, 0, i, 5] = math.nan
    y = c.run()
    nan = torch.zeros_like(y, dtype=torch.bool)
    rows = slice(max(0, j - before[0]), new[0])
    nan[rows, :q_heads // heads, :] = True
    if kind == "plain" and what != "key":
        nan[rows, :q_heads // heads, :5] = nan[rows, :q_heads // heads, 6:] = False
    assert torch.equal(y.isnan(), nan)
    if kind == "plain":
        c.t[0][n, 0, i, 5] = c.t[1][n, 0, i, 5] = 0  # (what the others do not see)
    else:
        c.t[2][n, 0, i] = c.t[3][n, 0, i] = 1
    # (what was computed again is off by fp32's roundings, what was not by those that it had)
    tol = 4 * 2.0 ** {"f32": -18, "f16": -10, "bf16": -7}[dt] * c.values()[1].abs().max()
    assert ((y.double() - want.double()).abs()[~nan] <= tol).all()
    assert torch.equal(y[new[0]:], want[new[0]:]) and torch.equal(y[:, q_heads // heads:], want[:, q_heads // heads:])


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
def test_a_value_of_infinity_or_nan_that_nothing_weighs(dt, new, before):
    """Every score is -inf: zeros, whatever the values are."""
    c = Case(dt, "plain", new, before, 4, 1, 64, 16, seed=9)
    c.t[0].zero_()
    c.t[0][:, :, :, 0] = -math.inf
    c.q[..., 0] = 1.0
    c.t[1][..., 2], c.t[1][..., 3] = math.nan, math.inf
    assert not c.run().any()


@pytest.mark.parametrize("dt, new", [("f32", 1), ("f16", 1), ("bf16", 1), ("bf16", 5), ("f16", 70), ("bf16", 70)])
def test_positions_up_to_the_last(dt, new):
    """A sequence that ends at position 2^31 - 2, of whose pages the first, one in the middle and the last two exist."""
    import torch
    import paper_2110_06037_gb300 as sn
    width, page, dim = 1 << 23, 256, 64
    g = torch.Generator(device="cuda").manual_seed(10)
    k, v = (torch.randn(4, 1, page, dim, generator=g, device="cuda").to(tdt(dt)) for _ in range(2))
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    there = [0, 5000001, width - 2, width - 1]
    for n, i in enumerate(there):
        table[0, i] = n
    pos = 2 ** 31 - 1 - new
    q = torch.randn(new, 1, dim, generator=g, device="cuda").to(tdt(dt))
    y = sn.KVCache(k, v).attend(q, table, offsets=torch.tensor([0, new], dtype=torch.int32, device="cuda"), max_len=new,
                                pos=torch.tensor([pos], dtype=torch.int32, device="cuda"))
    at_ = torch.cat([i * page + torch.arange(page, device="cuda") for i in there])
    s = q[:, 0].double() @ k[:, 0].flatten(0, 1).double().T / 8
    s = s.masked_fill(at_[None] > pos + torch.arange(new, device="cuda")[:, None], -math.inf)
    want = torch.softmax(s, dim=1) @ v[:, 0].flatten(0, 1).double()
    # scores of some 5 in magnitudes, off by 2 (dim + 8) 2^-24 of these; weights and results rounded once (prompts: both)
    assert ((y[:, 0].double() - want).abs() <= {"f32": 2.0 ** -14, "f16": 2.0 ** -9, "bf16": 2.0 ** -6}[dt] * v.abs().max()).all()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("new, before", SIZES)
@pytest.mark.parametrize("power", [-121, -115, -100, 60, 110, 121])
def test_codes_with_far_queries(dt, new, before, power):
    """Queries near the ends of the range, and keys' scales that bring the scores back."""
    c = Case(dt, "q8", new, before, 4, 2, 64, 16, seed=11)
    c.q.mul_(2.0 ** power)
    c.t[2].mul_(2.0 ** -power)
    c.check(c.run(), 2.0 ** (-11 if dt == "bf16" else -21))
