"""The example model: the block operators together, as they are used."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("dt, tol", [("f32", 1e-3), ("bf16", 0.15)])
def test_prompt_then_tokens_is_one_longer_prompt(dt, tol):
    """Logits of 20 tokens at once against 12 at once and 8 one by one.  fp32: three layers of sums of a
    few hundred terms, 1e-3 of the largest logit is thousands of roundings.  bf16: every layer rounds its
    rows about ten times to 2^-9 in ways that differ between the two (10 x 3 x 2^-9 = 0.06 of a logit)."""
    import torch
    import state_space_lm as lm
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    m = lm.Model(layers=3, dim=256, dtype=dtype)
    toks = torch.randint(0, 1000, (2, 20), device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    off = torch.tensor([0, 20, 40], dtype=torch.int32, device="cuda")
    whole = m.prompt(toks.reshape(-1), m.caches(2), off, 20).float().view(2, 20, -1)
    caches = m.caches(2)
    off = torch.tensor([0, 12, 24], dtype=torch.int32, device="cuda")
    part = m.prompt(toks[:, :12].reshape(-1), caches, off, 12).float().view(2, 12, -1)
    scale = whole.abs().max()
    assert (part - whole[:, :12]).abs().max() <= tol * scale
    for t in range(12, 20):
        pos = torch.full((2,), t, dtype=torch.int32, device="cuda")
        assert (m.token(toks[:, t], caches, pos).float() - whole[:, t]).abs().max() <= tol * scale


def test_generation_from_a_graph_is_generation_call_by_call():
    import torch
    import state_space_lm as lm
    m = lm.Model(layers=2, dim=128)
    gen = torch.Generator("cuda").manual_seed(2)
    prompts = [torch.randint(0, 1000, (n,), device="cuda", generator=gen) for n in (1, 5, 90)]
    out = lm.generate(m, prompts, 6)
    off = torch.tensor([0, 1, 6, 96], dtype=torch.int32, device="cuda")
    caches = m.caches(3)
    now = m.prompt(torch.cat(prompts), caches, off, 90)[off[1:].long() - 1].argmax(1)
    pos = torch.tensor([1, 5, 90], dtype=torch.int32, device="cuda")
    for t in range(6):
        assert torch.equal(out[:, t], now)
        now = m.token(now, caches, pos).argmax(1)
        pos += 1
