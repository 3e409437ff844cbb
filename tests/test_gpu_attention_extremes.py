"""Attention over a cache on the GPU where keys, values or scales are at the ends of their types' ranges."""
import math

import pytest

from test_gpu_attention_forms import Case

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
    assert torch.equal(c.run(), c.t[1][n, 0, i].expand_as(c.q))


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
