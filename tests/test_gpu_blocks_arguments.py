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


def test_a_handle_of_another_device_is_refused():
    import torch
    import paper_2110_06037_gb300 as sn
    x = torch.zeros(2, 64, device="cuda")
    w = sn.Q4Weights(*sn.quantize_q4(torch.randn(64, 64, device="cuda")), 64, 64)
    norm = sn.BlockNorm(64, post=torch.ones(64, device="cuda"))
    c = 32 + 2 * 16
    ssm = sn.StateSpace(1, 32, 1, 16, torch.zeros(1, device="cuda"), conv_weight=torch.zeros(c, 4, device="cuda"))
    kept, state = torch.zeros(2, 4, c, device="cuda"), torch.zeros(2, 1, 32, 16, device="cuda")
    uses = [(w, lambda: sn.dense_q4(x, w)), (norm, lambda: norm(x)), (ssm, lambda: ssm.scan(x[None], x[None, :, :1])),
            (ssm, lambda: ssm.step(x, x[:, :1], kept, state, None))]
    for handle, use in uses:
        assert handle.device == x.get_device()
        use()
        handle.device += 1
        with pytest.raises(sn.SnError, match="device"):
            use()
        handle.device -= 1


def test_handles_are_set_up_on_the_device_of_their_tensors(monkeypatch):
    import contextlib
    import torch
    import paper_2110_06037_gb300 as sn
    entered = []

    def device(d):
        entered.append(d)
        return contextlib.nullcontext()

    t = torch.randn(8, 64, device="cuda")
    monkeypatch.setattr(torch.cuda, "device", device)
    codes, scales = sn.quantize_q4(t)
    sn.Q4Weights(codes, scales, 64, 64)
    assert entered == [t.device, t.device]


def test_tensors_of_the_host_are_refused():
    import torch
    import paper_2110_06037_gb300 as sn
    norm = sn.BlockNorm(64, post=torch.ones(64, device="cuda"), pre=torch.ones(64, device="cuda"), gate="silu")
    x, h = torch.zeros(2, 64, device="cuda"), torch.zeros(2, 64)
    for kw in ({"residual": h, "gate": x}, {"gate": h}, {"gate": x, "out": h}, {"gate": x, "out_normed": h}):
        with pytest.raises(sn.SnError):
            norm(x, **kw)
    with pytest.raises(sn.SnError):
        norm(h, gate=x)
    with pytest.raises(sn.SnError):
        sn.quantize_q4(h)
    with pytest.raises(sn.SnError):
        sn.causal_conv(x[None], torch.zeros(64, 4))


def test_buffers_without_an_axis_of_entries_are_refused():
    import torch
    import paper_2110_06037_gb300 as sn
    one, x = torch.zeros((), device="cuda"), torch.zeros(1, 4, 64, device="cuda")
    ssm = sn.StateSpace(1, 32, 1, 16, torch.zeros(1, device="cuda"), conv_weight=torch.zeros(64, 4, device="cuda"))
    for use in (lambda: sn.causal_conv(x, torch.zeros(64, 4, device="cuda"), kept=one), lambda: ssm.scan(x, x[:, :, :1], state_in=one),
                lambda: ssm.scan(x, x[:, :, :1], state_out=one), lambda: ssm.step(x[0], x[0, :, :1], one, one, None),
                lambda: sn.StateSpace(1, 32, 1, 16, torch.zeros(1, device="cuda"), conv_weight=one),
                lambda: sn.Q4Weights(one.to(torch.uint8), one.half(), 64, 64)):
        with pytest.raises(sn.SnError):
            use()


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_a_scan_of_empty_sequences_hands_their_states_on(dt):
    import torch
    import paper_2110_06037_gb300 as sn
    dtype = {"f32": torch.float32, "bf16": torch.bfloat16}[dt]
    ssm = sn.StateSpace(2, 32, 1, 16, torch.zeros(2, device="cuda"))
    x, step = torch.zeros(0, 96, dtype=dtype, device="cuda"), torch.zeros(0, 2, dtype=dtype, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    state, out = torch.randn(3, 2, 32, 16, device="cuda"), torch.full((3, 2, 32, 16), 5.0, device="cuda")
    assert ssm.scan(x, step, offsets=off, max_len=0, state_in=state, state_out=out).shape == (0, 64)
    assert torch.equal(out, state)
    ssm.scan(x, step, offsets=off, max_len=0, state_out=out)
    assert bool((out == 0).all())
