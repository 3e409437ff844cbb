"""How exact the block operators are, by bounds that leave room for fp32 sums and the output's rounding alone.

The bounds follow from the arithmetic and were fixed before their first run; E32 is half a unit of fp32."""
import numpy as np
import pytest

from oracle import blocks as ob
from test_gpu_blocks import E32, U, close, dev, host, q4, tdt

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------ 4-bit dense
def sums_bound(mag, k, group):
    """A group's sum of up to 128 exact products, truncated at each; a multiplication and an addition a
    group in fp32; up to 80 further additions (warps, blocks, bias).  Nothing else is rounded."""
    return (128 + 2 * -(-k // group) + 80) * E32 * mag


DENSE = [(9, 640, 130, 32, "bf16"), (20, 1100, 96, 64, "f16"), (32, 2050, 64, 128, "bf16"), (33, 1027, 130, 128, "bf16"),
         (64, 256, 128, 128, "f16"), (127, 640, 640, 64, "bf16"), (129, 72, 384, 32, "f16"), (257, 1100, 513, 128, "bf16"),
         (300, 4096, 96, 32, "bf16"), (700, 192, 1500, 64, "f16"), (90, 65, 33, 32, "bf16"), (2050, 320, 160, 32, "f16")]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, k, n, group, sdt", DENSE)
def test_dense_rounds_no_weight(dt, rows, k, n, group, sdt):
    """A weight q * scale has up to 15 bits: a product with it rounded to 8 or 11 would not hold the bound
    where an output is a small difference of large terms."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(rows + k)
    w, codes, scales, b = q4(rng, n, k, group, sdt)
    x = dev(rng.normal(size=(rows, k)), dt)
    pre, mag = ob.dense(host(x), codes, scales, k, group, b)
    y = sn.dense_q4(x, w)
    close(y, pre, sums_bound(mag, k, group), dt)
    sn.check_device()
    assert sn.dense_q4(x, w).equal(y)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_dense_of_a_row_does_not_depend_on_the_rows_beside_it(dt):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(3)
    k, n, group = 700, 200, 64
    w, codes, scales, b = q4(rng, n, k, group, "bf16")
    x = dev(rng.normal(size=(100, k)), dt)
    pre, mag = ob.dense(host(x), codes, scales, k, group, b)
    alone = torch.cat([sn.dense_q4(x[i:i + 1], w) for i in range(100)])
    close(sn.dense_q4(x, w), host(alone), 2 * sums_bound(mag, k, group) + U[dt] * np.abs(pre), dt)


@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("sdt", ["f16", "bf16"])
def test_dense_fp16_with_groups_of_far_apart_scales(rows, sdt):
    """The largest products come from the group of the smallest scale."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(9)
    n, k = 48, 192
    codes = rng.integers(0, 256, (n, k // 2)).astype(np.uint8)
    small = 2.0 ** -20 if sdt == "f16" else 2.0 ** -34
    scales = dev(rng.uniform(1, 1.9, (n, 3)) * np.array([2.0 ** 8, small, 2.0 ** -2]), sdt)
    x = rng.normal(size=(rows, k))
    x[:, :64] *= 2.0 ** -24 / 2.0 ** -8  # (fp16's smallest values)
    x[:, 64:128] = np.clip(x[:, 64:128] * 2.0 ** 14, -60000, 60000)
    x[:, 128:] = 0
    x = dev(x, "f16")
    if sdt == "bf16":
        x[:, :64] = 0  # nothing beside them then
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, k, 64)
    pre, mag = ob.dense(host(x), codes, host(scales), k, 64)
    close(sn.dense_q4(x, w), pre, sums_bound(mag, k, 64), "f16")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -118, 2.0 ** 100])
def test_dense_with_scales_at_the_ends_of_bf16(dt, rows, size):
    """No factor on the way leaves fp32's range: codes of 0 and inputs of 0 give 0, never NaN."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(10)
    codes = rng.integers(0, 256, (40, 64)).astype(np.uint8)
    codes[:, ::3] = 0
    scales = dev(rng.uniform(1, 1.5, (40, 2)), "bf16") * size
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, 128, 64)
    x = rng.normal(size=(rows, 128)) * (2.0 ** -14 if size > 1 else 2.0 ** 10)
    if size > 1 and dt == "f16":
        x[:] = 0  # (the outputs would be beyond fp16)
    x[0] = 0
    x = dev(x, dt)
    pre, mag = ob.dense(host(x), codes, host(scales), 128, 64)
    y = sn.dense_q4(x, w)
    close(y, pre, sums_bound(mag, 128, 64) + 2.0 ** -126, dt)
    assert bool((y[0] == 0).all())


# -------------------------------------------------------------------- scan
def half_spacing(ref, dt):
    """Half the distance of a type's values around ref: what one rounding may be off."""
    bits = {"f16": 11, "bf16": 8}[dt]
    _, e = np.frexp(ref)  # |ref| in [2^(e - 1), 2^e)
    return np.maximum(np.ldexp(1.0, e - bits - 1), 2.0 ** -25 if dt == "f16" else 1e-37)


def ramps(rng, kind, t, h):
    if kind == "erase":  # one step far beyond the others, then small ones, again and again
        raw = rng.normal(size=(t, h)) - 3
        raw[5::37] = 3000.0
        raw[20::53] = 1e4
        return raw
    return float(kind) * rng.uniform(0.9, 1.1, (t, h))


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["0.1", "1", "5", "20", "60", "erase"])
@pytest.mark.parametrize("lens, sizes", [([300], (2, 64, 1, 16)), ([127, 64, 130], (3, 32, 1, 8)), ([1100], (1, 64, 1, 64))])
def test_scan_keeps_its_precision_whatever_the_steps(dt, kind, lens, sizes):
    """y is rounded once; what it is made of is good to 2^-14 of the terms' sizes (two 16-bit parts of each
    factor, exponents that matter, up to 32, to 2^-21 of themselves), also where every step times a is
    large, or one step before them was.  A decay taken as the difference of two running sums is off by
    2^-24 of those sums."""
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(sum(lens))
    a = -rng.uniform(12, 16, h).astype(np.float32)
    xbc = dev(rng.normal(size=(sum(lens), h * p + 2 * g * n)), dt)
    step = dev(ramps(rng, kind, sum(lens), h), dt)
    if dt == "f16":
        step = step.clamp(max=1e4)
    ssm = sn.StateSpace(h, p, g, n, dev(a))
    out = torch.empty(len(lens), h, p, n, device="cuda")
    at = np.concatenate(([0], np.cumsum(lens)))
    y = ssm.scan(xbc, step, offsets=torch.tensor(at, dtype=torch.int32, device="cuda"), max_len=max(lens), state_out=out)
    sn.check_device()
    for i, (s, e) in enumerate(zip(at, at[1:])):
        ref, my, sref, ms = ob.scan(host(xbc)[s:e], host(step)[s:e], sizes, a, None, None, np.zeros((h, p, n)))
        got = host(y)[s:e]
        # a value that rounds to none of fp16's is infinite
        beyond = (np.abs(ref) + 2.0 ** -14 * my >= 65520) & (got == np.copysign(np.inf, ref)) if dt == "f16" else np.zeros(ref.shape, bool)
        err = np.where(beyond, 0, np.abs(np.where(beyond, ref, got) - ref))
        # (a state is the last few steps' where steps are large: 64 roundings and exponents to 2^-19)
        assert (np.abs(host(out)[i] - sref) <= 2.0 ** -18 * ms + 1e-37).all()
        assert (err <= half_spacing(ref, dt) + 2.0 ** -14 * my).all(), float((err / (half_spacing(ref, dt) + 2.0 ** -14 * my)).max())


# ------------------------------------------------------------------- norms
def norm_bound(v, ev, kind, eps, w, b):
    """(norm of v, what it may be off) per element, v [rows, d] off by ev each.

    To first order: the centred value is off by ev and by the mean's error (its own roundings, and the mean
    of ev); 1 / sqrt(mean square + eps) relatively by half the mean square's error, at most the root mean
    square of the centred values' errors over sqrt(mean square + eps).  Sums of a row are trees of at
    most 64 roundings, rsqrtf and the products a few more."""
    m = v.mean(1, keepdims=True) if kind == "layer" else 0.0
    c = v - m
    ec = ev + ((ev.mean(1, keepdims=True) + 64 * E32 * np.abs(v).mean(1, keepdims=True)) if kind == "layer" else 0.0) + E32 * np.abs(c)
    r = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    er = np.sqrt((ec * ec).mean(1, keepdims=True)) * r + 40 * E32  # relative
    out = c * r * w
    bound = np.abs(w) * r * ec + np.abs(out) * (er + 4 * E32)
    return (out, bound) if b is None else (out + b, bound + E32 * np.abs(out + b))


def block_norm_bound(y, res, g, per, kind, eps, use, gate, at):
    """(total, bound, normed or None, bound) of fp64 inputs."""
    zero = np.zeros(y.shape)
    gv = np.ones(y.shape) if g is None else ob.act(g, gate)[np.arange(len(y)) // per]
    # __expf is good to 2 + 1.173 |g| ulp, __fdividef to 2 (an ulp is at most 2 E32), and the sum and product
    eg = zero if g is None else np.abs(gv) * (12 + 3 * np.abs(g[np.arange(len(y)) // per])) * E32
    t, e = (y * gv, np.abs(y) * eg + E32 * np.abs(y * gv)) if at == "before" else (y, zero)
    if "post" in use:
        t, e = norm_bound(t, e, kind, eps, use["post"].astype(np.float64), use["post_bias"] if "post_bias" in use else None)
    if at == "after":
        t, e = t * gv, e * np.abs(gv) + np.abs(t) * eg + E32 * np.abs(t * gv)
    if "scale" in use:  # (which may be multiplied into the weight, and into the bias)
        t, e = t * use["scale"], e * np.abs(use["scale"]) + 4 * E32 * np.abs(t * use["scale"])
        if "post_bias" in use:
            e = e + 4 * E32 * np.abs(use["scale"] * use["post_bias"] * (gv if at == "after" else 1.0))
    if res is not None:
        e = e + E32 * np.abs(res + t) + E32 * np.abs(t)
        t = res + t
    if "pre" not in use:
        return t, e, None, None
    n, en = norm_bound(t, e, kind, eps, use["pre"].astype(np.float64), use["pre_bias"] if "pre_bias" in use else None)
    return t, e, n, en


@pytest.mark.parametrize("dt, rdt", [("f32", "f32"), ("f16", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("rows, d", [(5, 31), (4, 512), (3, 1024), (2, 4104), (2, 20001), (1301, 4096), (700, 512), (650, 1096)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("eps", [1e-5, 0.5])
def test_norms_are_off_by_their_roundings(dt, rdt, rows, d, kind, eps):
    """A norm with another eps, without its bias, or with sums in 16 bits would be far outside."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(rows + d)
    w = {k: (1 + 0.2 * rng.normal(size=d)).astype(np.float32) for k in ("post", "pre", "scale")}
    w |= {k: (0.1 * rng.normal(size=d)).astype(np.float32) for k in ("post_bias", "pre_bias")}
    y, r = dev(rng.normal(size=(rows, d)) + 0.5, dt), dev(2 * rng.normal(size=(rows, d)), rdt)
    for gate, at, per, names, with_res in (
            ("none", "after", 1, w, True), ("sigmoid", "before", 3, w, True), ("silu", "after", 1, w, True),
            ("silu", "before", 1, ("post", "pre"), True), ("linear", "after", 1, ("post", "post_bias", "scale"), False)):
        g = None if gate == "none" else dev(2 * rng.normal(size=(-(-rows // per), d)), dt)
        use = {k: w[k] for k in names}
        norm = sn.BlockNorm(d, kind, eps, gate=gate, gate_at=at, **{k: dev(v) for k, v in use.items()})
        total, normed = norm(y, residual=r if with_res else None, gate=g, rows_per_gate=per)
        t, e, n, en = block_norm_bound(host(y), host(r) if with_res else None, None if g is None else host(g), per, kind, eps, use, gate, at)
        close(total, t, e, rdt if with_res else dt)
        if n is not None:
            close(normed, n, en, dt)


def test_the_norms_bound_sees_another_eps_and_a_missing_bias():
    """Planted in the reference: what the bound is for."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(1)
    rows, d = 1301, 4096
    use = {k: (1 + 0.2 * rng.normal(size=d)).astype(np.float32) for k in ("post", "pre")}
    use["pre_bias"] = (0.01 * rng.normal(size=d)).astype(np.float32)
    y, r = dev(rng.normal(size=(rows, d))), dev(rng.normal(size=(rows, d)))
    _, normed = sn.BlockNorm(d, "layer", 1e-3, **{k: dev(v) for k, v in use.items()})(y, residual=r)
    for eps, names in ((1.1e-3, ("post", "pre", "pre_bias")), (1e-3, ("post", "pre"))):
        _, _, n, en = block_norm_bound(host(y), host(r), None, 1, "layer", eps, {k: use[k] for k in names}, "none", "after")
        with pytest.raises(AssertionError):
            close(normed, n, en, "f32")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("act", ["none", "relu", "relu6", "hswish", "hsigmoid"])
def test_dense_activations_pass_nan_on(dt, rows, act):
    import paper_2110_06037_gb300 as sn
    w, _, _, _ = q4(np.random.default_rng(2), 40, 130, 64, "bf16", act=act)
    x = dev(np.random.default_rng(3).normal(size=(rows, 130)), dt)
    ref = host(sn.dense_q4(x, w))
    x[1, 77] = float("nan")
    got = host(sn.dense_q4(x, w))
    assert np.isnan(got[1]).all()
    assert np.array_equal(np.delete(got, 1, 0), np.delete(ref, 1, 0)) and not np.isnan(ref).any()
