"""Tensors that the block operators' front end refuses before anything is launched."""
import pytest

pytestmark = pytest.mark.gpu


def calls(what, t):
    """The call that takes `t` (rows of 64 on three axes, or as an output) in the place that `what` names."""
    import torch
    import paper_2110_06037_gb300 as sn

    def new(*shape):
        return torch.zeros(shape, device="cuda")

    n, m = t.shape[0], t.shape[1]
    if what in ("x", "out"):
        w = sn.Q4Weights(torch.zeros(64, 32, dtype=torch.uint8, device="cuda"), torch.ones(64, 1, dtype=torch.float16, device="cuda"), 64, 64)
        return lambda: sn.dense_q4(t, w) if what == "x" else sn.dense_q4(new(n, m, 64), w, out=t)
    if what in ("y", "gate", "residual", "total", "normed"):
        norm = sn.BlockNorm(64, post=new(64), pre=new(64), gate="silu")
        a = {"y": new(n, m, 64), "gate": new(n, m, 64), "residual": new(n, m, 64), "total": None, "normed": None}
        a[what] = t
        return lambda: norm(a["y"], residual=a["residual"], gate=a["gate"], out=a["total"], out_normed=a["normed"])
    if what == "conv":
        return lambda: sn.causal_conv(t, new(64, 4))
    ssm = sn.StateSpace(1, 32, 1, 16, new(1))
    if what == "xbc":
        return lambda: ssm.scan(t, new(n, m, 1))
    return lambda: ssm.scan(new(n, m, 64), t[:, :, :1])


@pytest.mark.parametrize("what", ["x", "out", "y", "gate", "residual", "total", "normed", "conv", "xbc", "dt"])
@pytest.mark.parametrize("axis", [0, 1])
def test_rows_that_lie_on_one_another_are_refused(what, axis):
    """An expanded axis, the inner one too: its rows are not as many as its shape says."""
    import torch
    import paper_2110_06037_gb300 as sn
    t = torch.zeros(4, 64, device="cuda").unsqueeze(axis)
    t = t.expand(3, 4, 64) if axis == 0 else t.expand(4, 3, 64)
    with pytest.raises(sn.SnError):
        calls(what, t)()
    calls(what, t.contiguous())()  # the same values in rows of their own
