"""The state-space block's operators on the GPU against their fp64 oracle.

Error bounds: a result of m roundings of 2^-24 on terms of magnitudes that sum to M is off by at most
m 2^-24 M to first order; the kernels may add in any order and use CUDA's expf and log1pf (2 ulp).
U is the output type's rounding.  Every bound was fixed before its first run.
"""
import numpy as np
import pytest

from oracle import blocks as ob

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
U = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}  # half the spacing of the smallest values


def tdt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def dev(a, name="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(tdt(name))


def ints(a):
    import torch
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound, dt):
    got = host(got)
    assert got.shape == ref.shape
    err = np.abs(got - ref) - (U[dt] * np.abs(ref) + bound + TINY[dt])
    assert not np.isnan(got).any()
    assert err.max(initial=-1.0) <= 0, (float(err.max()), np.unravel_index(err.argmax(), err.shape))


# ------------------------------------------------------------ 4-bit dense
def q4(rng, n, k, group, sdt, bias=True, act="none"):
    """(Q4Weights, codes, scales as fp64, bias) of random codes over the whole range."""
    import torch
    import paper_2110_06037_gb300 as sn
    codes = rng.integers(0, 256, (n, (k + 1) // 2)).astype(np.uint8)
    scales = dev(rng.uniform(0.5, 1.5, (n, -(-k // group))) / np.sqrt(k) * np.where(rng.random((n, 1)) < 0.1, 30.0, 1.0), sdt)
    b = rng.normal(size=n).astype(np.float32) if bias else None
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, k, group, bias=dev(b) if bias else None, act=act)
    return w, codes, host(scales), b


def dense_bound(mag, k, group, dt, rows):
    """Tensor-core sums of up to 128 exact products, then a rounding a group, a warp and a block; for many
    rows of 16-bit x also the rounding of the scaled weight."""
    m = (128 + k / group + 80) * E32 * mag
    return m + (U[dt] * mag if rows > 8 else 0.0)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, k, n, group, sdt, act", [
    (1, 64, 16, 64, "bf16", "none"), (1, 1, 1, 32, "f16", "none"), (1, 63, 15, 128, "f16", "relu"),
    (2, 65, 17, 32, "bf16", "hswish"), (5, 130, 33, 128, "bf16", "none"), (8, 1280, 1000, 32, "f16", "none"),
    (9, 100, 40, 32, "f16", "hsigmoid"), (10, 2050, 111, 128, "f16", "none"), (11, 320, 129, 64, "bf16", "relu6"),
    (16, 4096, 64, 64, "bf16", "none"), (17, 513, 257, 32, "f16", "none"), (31, 96, 300, 64, "bf16", "none"),
    (33, 1027, 130, 128, "bf16", "relu"), (64, 256, 128, 128, "f16", "none"), (127, 640, 640, 64, "bf16", "none"),
    (129, 72, 384, 32, "f16", "none"), (257, 1100, 513, 128, "bf16", "hswish"), (3, 25088, 40, 64, "bf16", "none"),
    (16, 9000, 24, 128, "f16", "none")])
def test_dense(dt, rows, k, n, group, sdt, act):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(rows * 1000 + k)
    w, codes, scales, b = q4(rng, n, k, group, sdt, act=act)
    x = dev(rng.normal(size=(rows, k)), dt)
    pre, mag = ob.dense(host(x), codes, scales, k, group, b)
    y = sn.dense_q4(x, w)
    assert y.dtype == x.dtype
    slope = 1.5 if act in ("hswish",) else 1.0  # the activations' steepest slope (and 8 roundings of their own)
    bound = slope * dense_bound(mag, k, group, dt, rows) + (8 * E32 * (np.abs(pre) + 3) if act.startswith("h") else 0)
    close(y, ob.act(pre, act), bound, dt)
    assert sn.dense_q4(x, w).equal(y)  # the same again, to the bit


@pytest.mark.parametrize("rows, k, n", [(5, 8192, 96), (40, 2050, 512), (300, 8192, 96), (200, 513, 1700), (600, 3001, 2600)])
def test_dense_fp32_does_not_lose_precision_with_length(rows, k, n):
    """The tensor cores' own sums are truncated to some 24 bits at each of at most 40 products, half a unit
    each on average (40 * 2^-25), and fp32 additions of those sums round at random; the sum of all of them
    would be off by 5 k / 16 of such steps, all one way."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(k)
    w, codes, scales, b = q4(rng, n, k, 64, "f16")
    x = dev(rng.normal(size=(rows, k)))
    pre, _ = ob.dense(host(x), codes, scales, k, 64, b)
    d = host(sn.dense_q4(x, w)) - pre
    assert np.sqrt((d * d).sum() / (pre * pre).sum()) < 40 * 2.0 ** -25


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [1, 7, 40, 200])
@pytest.mark.parametrize("off", [0, 1, 8])
def test_dense_rows_apart_and_in_place_of_a_slice(dt, rows, off):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(off)
    k, n = 192, 72
    w, codes, scales, _ = q4(rng, n, k, 64, "bf16", bias=False)
    wide = dev(rng.normal(size=(rows, k + 24)), dt)
    out = torch.full((rows, n + 9), 7.0, dtype=tdt(dt), device="cuda")
    x = wide[:, off:off + k]
    sn.dense_q4(x, w, out=out[:, off:off + n])
    pre, mag = ob.dense(host(x), codes, scales, k, 64)
    close(out[:, off:off + n], pre, dense_bound(mag, k, 64, dt, rows), dt)
    rest = torch.cat((out[:, :off], out[:, off + n:]), dim=1)
    assert bool((rest == 7.0).all())
    lead = sn.dense_q4(x.unflatten(0, (1, rows)), w)
    assert lead.shape == (1, rows, n)


def test_dense_no_rows_no_bias_and_another_stream():
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(5)
    w, codes, scales, _ = q4(rng, 100, 300, 64, "f16", bias=False)
    assert sn.dense_q4(torch.empty(0, 300, device="cuda"), w).shape == (0, 100)
    x = dev(rng.normal(size=(50, 300)), "f32")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    y = sn.dense_q4(x, w, stream=s)
    s.synchronize()
    pre, mag = ob.dense(host(x), codes, scales, 300, 64)
    close(y, pre, dense_bound(mag, 300, 64, "f32", 50), "f32")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [3, 70])
def test_dense_what_is_not_finite_stays_in_its_row(dt, rows):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(6)
    w, codes, scales, _ = q4(rng, 48, 130, 32, "bf16", bias=False)
    x = dev(rng.normal(size=(rows, 130)), dt)
    ref = host(sn.dense_q4(x, w))
    x[1, 129] = float("inf")
    got = host(sn.dense_q4(x, w))
    q = ob.unpack(codes, 130)[:, 129]
    assert np.array_equal(got[1] == np.inf, q > 0) and np.array_equal(got[1] == -np.inf, q < 0)
    assert np.isnan(got[1][q == 0]).all()
    assert np.array_equal(np.delete(got, 1, 0), np.delete(ref, 1, 0))
    x[1, 129] = float("nan")
    got = host(sn.dense_q4(x, w))
    assert np.isnan(got[1]).all() and np.array_equal(np.delete(got, 1, 0), np.delete(ref, 1, 0))


@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("size", [1e-30, 1e30])
def test_dense_fp32_range(rows, size):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(7)
    w, codes, scales, _ = q4(rng, 33, 200, 64, "f16", bias=False)
    x = dev(rng.normal(size=(rows, 200)) * size)
    pre, mag = ob.dense(host(x), codes, scales, 200, 64)
    close(sn.dense_q4(x, w), pre, dense_bound(mag, 200, 64, "f32", rows), "f32")


@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("size", [2.0 ** -30, 2.0 ** 20])
def test_dense_fp16_with_scales_beyond_fp16(rows, size):
    """bf16 scales that are no fp16 values: x carries the other half of the product."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(8)
    codes = rng.integers(0, 256, (40, 64)).astype(np.uint8)
    scales = dev(rng.uniform(0.5, 1.5, (40, 2)) * size, "bf16")
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, 128, 64)
    x = dev(rng.normal(size=(rows, 128)) * min(1 / size, 2.0 ** 9) * 2.0 ** -4, "f16")
    pre, mag = ob.dense(host(x), codes, host(scales), 128, 64)
    close(sn.dense_q4(x, w), pre, dense_bound(mag, 128, 64, "f16", rows), "f16")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n, k, group", [(1, 1, 32), (5, 31, 32), (7, 64, 64), (33, 129, 128), (16, 1000, 64)])
def test_quantize(dt, n, k, group):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(k)
    w = dev(rng.normal(size=(n, k)) * 10.0 ** rng.integers(-3, 3, (n, 1)), dt)
    w[0, : min(k, group)] = 0
    for sdt in ("f16", "bf16"):
        codes, scales = sn.quantize_q4(w, group, tdt(sdt))
        v = w.float().cpu().numpy()
        pad = np.pad(v, ((0, 0), (0, -k % group))).reshape(n, -1, group)
        s = torch.from_numpy(np.abs(pad).max(2) / np.float32(7)).to(tdt(sdt))
        s = torch.where(s > 0, s, torch.ones_like(s))
        assert torch.equal(scales.cpu(), s)
        q = np.clip(np.rint(pad / s.float().numpy()[:, :, None]), -8, 7).reshape(n, -1)[:, :k]
        assert np.array_equal(ob.unpack(codes.cpu().numpy(), k), q.astype(np.int64))
        if k % 2:
            assert bool((codes[:, -1] >> 4 == 0).all())


# ------------------------------------------------------------------- norms
@pytest.mark.parametrize("dt, rdt", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows, d", [(1, 1), (3, 8), (5, 31), (2, 256), (9, 257), (4, 512), (3, 520), (2, 1000), (3, 1024),
                                     (2, 2048), (3, 2051), (2, 4096), (2, 4104), (1, 8192), (2, 8193), (1, 20001)])
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_norm(dt, rdt, rows, d, kind):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(rows * 7 + d)
    w = {k: (1 + 0.2 * rng.normal(size=d)).astype(np.float32) for k in ("post", "post_bias", "pre", "pre_bias", "scale")}
    y, r = dev(rng.normal(size=(rows, d)) + 0.5, dt), dev(2 * rng.normal(size=(rows, d)), rdt)
    for gate, at, per, some in (("none", "after", 1, True), ("linear", "before", 1, True), ("sigmoid", "after", 2, True),
                                ("silu", "before", rows, False), ("silu", "after", 1, False)):
        g = None if gate == "none" else dev(2 * rng.normal(size=(-(-rows // per), d)), dt)
        use = w if some else {"post": w["post"], "pre": w["pre"]}
        norm = sn.BlockNorm(d, kind, 1e-3, gate=gate, gate_at=at, **{k: dev(v) for k, v in use.items()})
        total, normed = norm(y, residual=r, gate=g, rows_per_gate=per)
        assert total.dtype == r.dtype and normed.dtype == y.dtype
        ref, refn = ob.block_norm(host(y), host(r), None if g is None else host(g), per, kind, 1e-3, gate_act=gate, at=at, **use)
        # of a row: sums of up to d values in a tree (20 roundings) and some 20 more, on values up to its largest;
        # the mean's error of that size is up to 1/sqrt(eps) = 32 times as large behind the division
        size = 1 + np.abs(ref).max(1, keepdims=True) + np.abs(host(y)).max(1, keepdims=True)
        if g is not None:
            size = size * (1 + np.abs(host(g)).max())
        close(total, ref, 64 * E32 * size * 32, rdt)
        close(normed, refn, 64 * E32 * size * 32 * 32, dt)


@pytest.mark.parametrize("dt, rdt", [("f32", "f32"), ("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("d", [512, 1000, 2056, 4096])
@pytest.mark.parametrize("kind, gate, at, per, parts", [
    ("rms", "silu", "after", 1, "all"), ("layer", "sigmoid", "before", 3, "all"), ("rms", "none", "after", 1, "pre"),
    ("rms", "silu", "before", 1, "post"), ("layer", "linear", "after", 1000, "plain")])
def test_norm_of_many_rows(dt, rdt, d, kind, gate, at, per, parts):
    """More rows than a wave of blocks; every row against the rows one by one, in place too."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(d)
    rows = 1301
    w = {k: (1 + 0.2 * rng.normal(size=d)).astype(np.float32) for k in ("post", "post_bias", "pre", "pre_bias", "scale")}
    names = {"all": w, "pre": ("pre",), "post": ("post",), "plain": ("scale",)}[parts]
    use = {k: w[k] for k in names}
    wide = dev(rng.normal(size=(rows, 2 * d + 16)) + 0.5, dt)
    y, g = (None if parts == "pre" else wide[:, 8:d + 8]), wide[:: per if per > 1 else 1, d + 8:2 * d + 8]
    g = None if gate == "none" else g[: -(-rows // per)]
    if g is not None and g.shape[0] * per < rows:
        g = wide[: -(-rows // per), d + 8:2 * d + 8]
    r = None if parts == "post" else dev(2 * rng.normal(size=(rows, d)), rdt)
    norm = sn.BlockNorm(d, kind, 1e-3, gate=gate, gate_at=at, **{k: dev(v) for k, v in use.items()})
    total, normed = norm(y, residual=r, gate=g, rows_per_gate=per, dtype=tdt(dt))
    ref, refn = ob.block_norm(None if y is None else host(y), None if r is None else host(r), None if g is None else host(g),
                              per, kind, 1e-3, gate_act=gate, at=at, **use)
    size = 1 + np.abs(ref).max(1, keepdims=True) + np.abs(host(wide)).max()
    if g is not None:
        size = size * (1 + np.abs(host(g)).max())
    if total is not r:
        close(total, ref, 64 * E32 * size * 32, rdt if r is not None else dt)
    if normed is not None:
        close(normed, refn, 64 * E32 * size * 32 * 32, dt)
    if y is not None and r is not None and normed is not None:
        r2, y2 = r.clone(), y.clone()
        a, b = norm(y2, residual=r2, gate=g, rows_per_gate=per, out=r2, out_normed=y2)
        assert torch.equal(a, total) and torch.equal(b, normed)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("d", [40, 1000, 9000])
def test_norm_parts_alone_strides_and_in_place(dt, d):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(d)
    rows = 6
    wide = dev(rng.normal(size=(rows, 3 * d + 5)), dt)
    y, g = wide[:, 1:d + 1], wide[:, d + 1:2 * d + 1]
    w = (1 + 0.1 * rng.normal(size=d)).astype(np.float32)
    gated = sn.BlockNorm(d, post=dev(w), gate="silu", gate_at="before")
    total, none = gated(y, gate=g)
    assert none is None
    ref, _ = ob.block_norm(host(y), gate=host(g), post=w, gate_act="silu", at="before")
    size = 64 * E32 * 32 * (1 + np.abs(ref).max(1, keepdims=True))
    close(total, ref, size, dt)
    first = sn.BlockNorm(d, pre=dev(w))  # the first norm of a stack: the residual alone
    same, n = first(None, residual=y)
    assert same is y
    close(n, ob.block_norm(None, host(y), pre=w)[1], size, dt)
    r = dev(rng.normal(size=(rows, d)), "f32")
    both = sn.BlockNorm(d, pre=dev(w))
    a, b = both(total, residual=r)
    keep, t2 = r.clone(), total.clone()
    c, e = both(t2, residual=keep, out=keep, out_normed=t2)
    assert torch.equal(a, c) and torch.equal(b, e) and c.data_ptr() == keep.data_ptr() and e.data_ptr() == t2.data_ptr()
    assert first(None, residual=r[:0])[1].shape == (0, d)


@pytest.mark.parametrize("d", [40, 4096, 9000])
def test_norm_keeps_nan_and_inf_in_their_row_and_takes_a_zero_row(d):
    import torch
    import paper_2110_06037_gb300 as sn
    norm = sn.BlockNorm(d, post=torch.ones(d, device="cuda"), pre=torch.ones(d, device="cuda"))
    y, r = torch.randn(5, d, device="cuda"), torch.zeros(5, d, device="cuda")
    y[0] = 0
    y[1, 3] = float("nan")
    y[2, d - 1] = float("inf")
    total, n = norm(y, residual=r)
    assert bool((total[0] == 0).all()) and bool((n[0] == 0).all())
    assert bool(total[1].isnan().all()) and bool(n[1].isnan().all()) and bool(n[2].isnan().any())
    assert bool(total[3:].isfinite().all()) and bool(n[3:].isfinite().all())


# ------------------------------------------------------------- convolution
def run_conv(x, lens, w, b, act, kept=None, pos=None, slots=None):
    at = np.concatenate(([0], np.cumsum(lens)))
    y, mag, k = np.zeros(x.shape), np.zeros(x.shape), None if kept is None else kept.copy()
    for i, (s, e) in enumerate(zip(at, at[1:])):
        slot = i if slots is None else slots[i]
        mine = None if kept is None or slot < 0 else kept[slot]
        y[s:e], mag[s:e], mine = ob.conv(x[s:e], w, b, act == "silu", mine, 0 if pos is None else pos[i])
        if mine is not None:
            k[slot] = mine
    return y, mag, k


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens, c, width, act", [
    ([1], 1, 1, "none"), ([0, 1, 2, 3, 0], 24, 4, "silu"), ([33, 31, 32], 40, 4, "silu"), ([70], 333, 3, "silu"),
    ([5, 100], 1026, 2, "none"), ([40, 9], 64, 8, "silu"), ([65], 17, 5, "silu"), ([7], 8, 6, "none"), ([40], 16, 7, "silu")])
def test_conv(dt, lens, c, width, act):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(c + width)
    w, b = rng.normal(size=(c, width)).astype(np.float32), rng.normal(size=c).astype(np.float32)
    x = dev(rng.normal(size=(sum(lens), c)), dt)
    slots = list(rng.permutation(len(lens) + 2)[: len(lens)])
    slots[-1] = -1 if len(lens) > 1 else slots[-1]
    pos = [int(v) for v in rng.integers(0, 9, len(lens))]
    pos[0] = 2 ** 31 - 1 - lens[0]
    kept = dev(rng.normal(size=(len(lens) + 2, width, c)), dt)
    off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
    ref, mag, kref = run_conv(host(x), lens, w, b, act, host(kept), pos, slots)
    y = sn.causal_conv(x, dev(w), dev(b), act=act, offsets=off, max_len=max(lens), kept=kept, slots=ints(slots), pos=ints(pos))
    close(y, ref, 32 * E32 * mag, dt)
    assert np.array_equal(host(kept), kref)
    # from nothing, without bias, kept or offsets, rows apart
    wide = dev(rng.normal(size=(3, 37, c + 3)), dt)
    v = wide[:, :, 1:c + 1]
    ref, mag, _ = run_conv(host(v).reshape(-1, c), [37] * 3, w, None, act)
    close(sn.causal_conv(v, dev(w), act=act), ref.reshape(3, 37, c), (32 * E32 * mag).reshape(3, 37, c), dt)


def test_conv_many_tokens():
    """More runs of tokens than fit one grid axis of 65535, and neighbours that differ."""
    import torch
    import paper_2110_06037_gb300 as sn
    t = 2_200_000
    x = (torch.arange(t, device="cuda") % 251).to(torch.float16)[None, :, None].contiguous()
    w = torch.tensor([[1.0, 4.0]], device="cuda")
    y = sn.causal_conv(x, w, act="none")
    ref = 4 * x.float()
    ref[:, 1:] += x[:, :-1].float()
    assert torch.equal(y, ref.half())


# -------------------------------------------------------------------- scan
def ssm_weights(rng, h, fast=False):
    a = -rng.uniform(0.2, 16 if fast else 2, h).astype(np.float32)
    return a, rng.normal(size=h).astype(np.float32), rng.uniform(-4, 0, h).astype(np.float32)


def run_scan(xbc, dt, lens, sizes, a, d, b, state, slots):
    h, p, _, n = sizes
    at = np.concatenate(([0], np.cumsum(lens)))
    y, my = np.zeros((len(xbc), h * p)), np.zeros((len(xbc), h * p))
    out, mag = state.copy(), np.abs(state)
    for i, (s, e) in enumerate(zip(at, at[1:])):
        start = state[slots[i]] if slots[i] >= 0 else np.zeros((h, p, n))
        y[s:e], my[s:e], so, mo = ob.scan(xbc[s:e], dt[s:e], sizes, a, d, b, start)
        if slots[i] >= 0:
            out[slots[i]], mag[slots[i]] = so, mo
    return y, my, out, mag


def scan_bound(mag, n):
    """n steps of three roundings on what is carried along, a few on each term, and expf's and softplus'."""
    return (64 + 8 * n) * E32 * mag


@pytest.mark.parametrize("lens", [[2000], [100, 300, 900]])
def test_scan_state_keeps_fp32s_precision(lens):
    """The state of bf16 tokens is an fp32 sum.  Its products are exact to 2^-25; the tensor cores truncate
    its sums at 16 products a chunk (16 * 2^-25); the weights' exponentials are good to 2^-22."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(31)
    h, p, g, n = 4, 64, 1, 128
    a = -rng.uniform(1, 16, h).astype(np.float32)
    x, dt = dev(rng.normal(size=(sum(lens), h * p + 2 * g * n)), "bf16"), dev(rng.normal(size=(sum(lens), h)) - 3, "bf16")
    out = torch.empty(len(lens), h, p, n, device="cuda")
    offs = np.concatenate(([0], np.cumsum(lens)))
    sn.StateSpace(h, p, g, n, dev(a)).scan(x, dt, offsets=ints(offs), max_len=max(lens), state_out=out)
    for b in range(len(lens)):
        rows = slice(offs[b], offs[b + 1])
        _, _, ref, _ = ob.scan(host(x[rows]), host(dt[rows]), (h, p, g, n), a, None, None, np.zeros((h, p, n)))
        d = host(out[b]) - ref
        assert np.sqrt((d * d).sum() / (ref * ref).sum()) < 1e-6


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens, sizes", [
    ([1], (1, 1, 1, 1)), ([0, 5, 1], (2, 8, 1, 16)), ([17, 64, 0, 33], (4, 64, 2, 128)), ([65], (6, 48, 2, 40)),
    ([100, 128], (3, 33, 3, 31)), ([300], (2, 64, 1, 64)), ([63, 129], (2, 32, 1, 128)), ([40], (1, 130, 1, 200)),
    ([200, 3], (4, 16, 4, 16)), ([90], (2, 80, 1, 256)), ([64, 640], (2, 64, 2, 128)), ([150], (8, 64, 1, 96)),
    ([70], (2, 64, 1, 112))])
def test_scan(dt, lens, sizes):
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(sum(lens) + p)
    a, d, b = ssm_weights(rng, h, fast=p == 64)
    rows, c = sum(lens), h * p + 2 * g * n
    wide = dev(rng.normal(size=(rows, c + 8 + h)), dt)
    xbc, step = wide[:, 8:8 + c], wide[:, 8 + c:]
    slots = [int(v) for v in rng.permutation(len(lens) + 1)[: len(lens)]]
    if len(lens) > 2:
        slots[-1] = -1
    state = dev(rng.normal(size=(len(lens) + 1, h, p, n)))
    off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
    ref, my, sref, ms = run_scan(host(xbc), host(step), lens, sizes, a, d, b, host(state), slots)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    out = torch.full_like(state, 5.0)
    y = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out, slots=ints(slots))
    # 16-bit types may carry the factors of y's products in two 16-bit parts
    close(y, ref, scan_bound(my, max(lens)) + (2.0 ** -14 * my if dt != "f32" else 0), dt)
    used = [s for s in slots if s >= 0]
    close(out[used], sref[used], scan_bound(ms, max(lens))[used], "f32")
    rest = [s for s in range(len(lens) + 1) if s not in used]
    assert bool((out[rest] == 5.0).all())
    again = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=state, slots=ints(slots))
    assert torch.equal(again, y) and torch.equal(state[used], out[used])  # in place, and the same to the bit


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens, sizes", [([1500, 3, 1100], (3, 64, 1, 128)), ([2300], (2, 40, 2, 24)), ([1025], (1, 80, 1, 72))])
def test_scan_of_long_prompts_with_few_heads(dt, lens, sizes):
    """Sequences that are cut into segments, short ones beside them; states from and to the same buffer."""
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(sum(lens))
    a, d, b = ssm_weights(rng, h)
    rows, c = sum(lens), h * p + 2 * g * n
    xbc, step = dev(rng.normal(size=(rows, c)), dt), dev(rng.normal(size=(rows, h)) - 2, dt)
    state = dev(rng.normal(size=(len(lens), h, p, n)))
    slots = list(range(len(lens)))[::-1]
    off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
    ref, my, sref, ms = run_scan(host(xbc), host(step), lens, sizes, a, d, b, host(state), slots)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    out = torch.empty_like(state)
    y = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out, slots=ints(slots))
    close(y, ref, scan_bound(my, max(lens)) + (2.0 ** -14 * my if dt != "f32" else 0), dt)
    close(out, sref, scan_bound(ms, max(lens)), "f32")
    again = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=state, slots=ints(slots))
    assert torch.equal(again, y) and torch.equal(state, out)


@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("lens, apart", [([5, 0, 70] * 12 + [900, 1, 300], True), ([700, 700], False)])
def test_scan_cuts_each_sequence_by_its_own_length(dt, lens, apart):
    """More sequences than a warp looks over at once, few of them long; and a batch of equal ones."""
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes = 1, 32, 1, 16
    rng = np.random.default_rng(len(lens))
    a, d, b = ssm_weights(rng, h)
    rows, c = sum(lens), h * p + 2 * g * n
    xbc, step = dev(rng.normal(size=(rows, c)), dt), dev(rng.normal(size=(rows, h)) - 2, dt)
    state = dev(rng.normal(size=(len(lens), h, p, n)))
    slots = list(range(len(lens)))
    ref, my, sref, ms = run_scan(host(xbc), host(step), lens, sizes, a, d, b, host(state), slots)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    out = torch.empty_like(state)
    if apart:
        off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
        y = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out)
    else:
        y = ssm.scan(xbc.unflatten(0, (len(lens), -1)), step.unflatten(0, (len(lens), -1)), state_in=state, state_out=out).flatten(0, 1)
    close(y, ref, scan_bound(my, max(lens)) + (2.0 ** -14 * my if dt != "f32" else 0), dt)
    close(out, sref, scan_bound(ms, max(lens)), "f32")


@pytest.mark.parametrize("lens, sizes", [
    ([16], (1, 64, 1, 128)), ([127, 0, 1, 130, 64], (3, 64, 3, 64)), ([129], (8, 64, 2, 128)), ([385, 5], (2, 32, 1, 96)),
    ([256, 256], (2, 40, 2, 24)), ([300], (2, 8, 1, 8)), ([40, 500], (2, 136, 1, 104)), ([128] * 9, (4, 64, 1, 16)),
    ([700], (40, 64, 1, 128)), ([513, 2], (4, 72, 2, 120))])
def test_scan_of_bf16_rows_that_lie_aligned(lens, sizes):
    """Rows that the copies of the tensor-core form take: head and state sizes that fill its tiles or not."""
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(sum(lens) + n)
    a, d, b = ssm_weights(rng, h, fast=n == 64)
    rows, c = sum(lens), h * p + 2 * g * n
    xbc, step = dev(rng.normal(size=(rows, c)), "bf16"), dev(rng.normal(size=(rows, h)) - 1, "bf16")
    state = dev(rng.normal(size=(len(lens), h, p, n)))
    off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
    ref, my, sref, ms = run_scan(host(xbc), host(step), lens, sizes, a, d, b, host(state), list(range(len(lens))))
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    out = torch.empty_like(state)
    y = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out)
    close(y, ref, scan_bound(my, max(lens)) + 2.0 ** -14 * my, "bf16")
    close(out, sref, scan_bound(ms, max(lens)), "f32")
    for _ in range(3):
        assert torch.equal(ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out), y)
    sn.check_device()


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scan_of_infinite_and_nan_channels(dt):
    """One channel's x is not finite at one token: every other channel, and that one before it, as without."""
    import torch
    import paper_2110_06037_gb300 as sn
    torch.manual_seed(4)
    h, p, g, n = 3, 64, 1, 128
    xbc = torch.randn(1, 400, h * p + 2 * g * n, device="cuda").to(tdt(dt))
    step = torch.randn(1, 400, h, device="cuda").to(tdt(dt))
    ssm = sn.StateSpace(h, p, g, n, -torch.rand(h, device="cuda"))
    ref = ssm.scan(xbc, step)
    for value in (float("nan"), float("inf"), -float("inf")):
        x = xbc.clone()
        x[0, 200, 70], x[0, 37, 191] = value, value
        y = ssm.scan(x, step)
        keep = torch.ones_like(y, dtype=torch.bool)
        keep[0, 200:, 70], keep[0, 37:, 191] = False, False
        assert torch.equal(y[keep], ref[keep])
        assert not bool(y[0, 200:, 70].isfinite().any()) and not bool(y[0, 37:, 191].isfinite().any())


@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_scan_equal_lengths_from_zero_without_skip_or_bias(dt):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(11)
    sizes = h, p, g, n = 4, 64, 1, 64
    a, _, _ = ssm_weights(rng, h)
    xbc, step = dev(rng.normal(size=(3, 77, h * p + 2 * g * n)), dt), dev(rng.normal(size=(3, 77, h)) - 2, dt)
    ssm = sn.StateSpace(h, p, g, n, dev(a))
    ref, my, _, _ = run_scan(host(xbc).reshape(231, -1), host(step).reshape(231, -1), [77] * 3, sizes, a, None, None,
                             np.zeros((3, h, p, n)), [0, 1, 2])
    y = ssm.scan(xbc, step)
    close(y.view(231, -1), ref, scan_bound(my, 77) + (2.0 ** -14 * my if dt != "f32" else 0), dt)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scan_of_time_steps_at_the_ends_of_their_range(dt):
    """Steps that erase the state (d a far below 0), that leave it alone (d = 0), and large ones with no decay."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(12)
    sizes = h, p, g, n = 3, 64, 1, 128
    a = np.array([-16.0, -1.0, 0.0], np.float32)
    xbc = dev(rng.normal(size=(1, 200, h * p + 2 * g * n)), dt)
    raw = rng.normal(size=(1, 200, h))
    raw[:, ::7] = 60.0
    raw[:, 3::5] = -200.0
    raw[0, 70:75] = -np.inf
    step = dev(raw, dt)
    ssm = sn.StateSpace(h, p, g, n, dev(a))
    out = torch.empty(1, h, p, n, device="cuda")
    y = ssm.scan(xbc, step, state_out=out)
    ref, my, sref, ms = run_scan(host(xbc)[0], host(step)[0], [200], sizes, a, None, None, np.zeros((1, h, p, n)), [0])
    close(y[0], ref, scan_bound(my, 200) + (2.0 ** -14 * my if dt != "f32" else 0), dt)
    close(out, sref, scan_bound(ms, 200), "f32")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scan_keeps_nan_in_its_sequence_and_behind_its_token(dt):
    import torch
    import paper_2110_06037_gb300 as sn
    torch.manual_seed(0)
    h, p, g, n = 2, 64, 1, 128
    xbc = torch.randn(2, 200, h * p + 2 * g * n, device="cuda").to(tdt(dt))
    step = torch.randn(2, 200, h, device="cuda").to(tdt(dt))
    ssm = sn.StateSpace(h, p, g, n, -torch.rand(h, device="cuda"))
    ref = ssm.scan(xbc, step)
    xbc[0, 90, 5] = float("nan")  # one channel of one head
    y = ssm.scan(xbc, step)
    assert torch.equal(y[1], ref[1]) and torch.equal(y[0, :64], ref[0, :64])
    assert bool(y[0, 90:, 5].isnan().all())
    assert torch.equal(y[0, :, 64:], ref[0, :, 64:])


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_scan_in_two_parts_is_scan_in_one(dt):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(13)
    sizes = h, p, g, n = 4, 64, 2, 128
    a, d, b = ssm_weights(rng, h)
    xbc, step = dev(rng.normal(size=(2, 300, h * p + 2 * g * n)), dt), dev(rng.normal(size=(2, 300, h)), dt)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    s1 = torch.zeros(2, h, p, n, device="cuda")
    whole = ssm.scan(xbc, step, state_out=s1)
    s2 = torch.zeros_like(s1)
    one = ssm.scan(xbc[:, :130].contiguous(), step[:, :130].contiguous(), state_out=s2)
    two = ssm.scan(xbc[:, 130:].contiguous(), step[:, 130:].contiguous(), state_in=s2, state_out=s2)
    _, my, _, ms = run_scan(host(xbc).reshape(600, -1), host(step).reshape(600, -1), [300, 300], sizes, a, d, b,
                            np.zeros((2, h, p, n)), [0, 1])
    tol = (2 * scan_bound(my, 300) + (2.0 ** -13 * my if dt != "f32" else 0)).reshape(2, 300, -1)
    close(torch.cat((one, two), 1), host(whole), tol + U[dt] * np.abs(host(whole)), dt)
    close(s2, host(s1), 2 * scan_bound(ms, 300), "f32")


# -------------------------------------------------------------------- step
@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("batch, sizes, width", [
    (1, (1, 1, 1, 1), 1), (3, (2, 8, 1, 16), 4), (5, (4, 64, 2, 128), 4), (2, (6, 48, 2, 40), 3), (4, (3, 33, 3, 31), 2),
    (1, (32, 64, 1, 128), 4), (40, (8, 64, 1, 64), 4), (2, (1, 130, 1, 200), 5), (3, (2, 256, 1, 256), 8), (2, (2, 20, 1, 255), 4)])
def test_step(dt, batch, sizes, width):
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(batch + p)
    a, d, b = ssm_weights(rng, h)
    c = h * p + 2 * g * n
    cw, cb = rng.normal(size=(c, width)).astype(np.float32), rng.normal(size=c).astype(np.float32)
    wide = dev(rng.normal(size=(batch, c + 3 + h)), dt)
    xbc, step = wide[:, 3:3 + c], wide[:, 3 + c:]
    slots = [int(v) for v in rng.permutation(batch + 2)[:batch]]
    if batch > 2:
        slots[1] = -1
        slots[2] = batch + 9  # beyond the entries: none
    pos = [int(v) for v in rng.integers(0, 2 * width, batch)]
    pos[-1] = 2 ** 31 - 1
    kept, state = dev(rng.normal(size=(batch + 2, width, c)), dt), dev(rng.normal(size=(batch + 2, h, p, n)))
    k0, s0 = host(kept), host(state)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b), dev(cw), dev(cb))
    out = torch.full_like(state, 5.0)
    kept2 = kept.clone()
    y = ssm.step(xbc, step, kept, state, ints(pos), state_out=out, slots=ints(slots))
    yr, bound = np.zeros((batch, h * p)), np.zeros((batch, h * p))
    sref, sb, kref = np.full(s0.shape, 5.0), np.zeros(s0.shape), k0.copy()
    for i in range(batch):
        if not 0 <= slots[i] < batch + 2:
            continue
        v, vm, kref[slots[i]] = ob.conv(host(xbc)[i:i + 1], cw, cb, True, k0[slots[i]], pos[i])
        ve = 32 * E32 * vm + 8 * E32 * np.abs(v)  # what the convolution may be off
        yy, my, s, ms = ob.scan(v, host(step)[i:i + 1], sizes, a, d, b, s0[slots[i]])
        _, me, _, mse = ob.scan(np.abs(v) + ve, host(step)[i:i + 1], sizes, a, np.abs(d), b, np.abs(s0[slots[i]]))
        _, m0, _, ms0 = ob.scan(np.abs(v), host(step)[i:i + 1], sizes, a, np.abs(d), b, np.abs(s0[slots[i]]))
        yr[i], bound[i] = yy[0], (me - m0 + 320 * E32 * me)[0]
        sref[slots[i]], sb[slots[i]] = s, mse - ms0 + 64 * E32 * mse
    close(y, yr, bound, dt)
    close(out, sref, sb, "f32")
    assert np.array_equal(host(kept), kref)
    again = ssm.step(xbc, step, kept2, state, ints(pos), slots=ints(slots))
    used = [s for s in slots if 0 <= s < batch + 2]
    assert torch.equal(again, y) and torch.equal(state[used], out[used]) and torch.equal(kept, kept2)


def test_step_of_a_far_entry():
    """An entry whose first value lies beyond 2^31 elements."""
    import torch
    import paper_2110_06037_gb300 as sn
    torch.manual_seed(3)
    h, p, g, n, w = 16, 64, 1, 128, 4
    c, entries = h * p + 2 * n, 17000
    state = torch.empty(entries, h, p, n, device="cuda")
    kept = torch.zeros(entries, w, c, device="cuda")
    far = entries - 1
    assert far * h * p * n > 2 ** 31
    ssm = sn.StateSpace(h, p, g, n, -torch.rand(h, device="cuda"), conv_weight=torch.randn(c, w, device="cuda"))
    x, dt = torch.randn(2, c, device="cuda"), torch.randn(2, h, device="cuda")
    x[1], dt[1] = x[0], dt[0]
    state[0] = torch.randn(h, p, n, device="cuda")
    state[far] = state[0]
    y = ssm.step(x, dt, kept, state, ints([0, 0]), slots=ints([0, far]))
    assert torch.equal(y[0], y[1]) and torch.equal(state[0], state[far]) and torch.equal(kept[0], kept[far])
    xs = x[:, None].expand(2, 70, c).contiguous()
    ds = dt[:, None].expand(2, 70, h).contiguous()
    y = ssm.scan(xs, ds, state_in=state, state_out=state, slots=ints([0, far]))
    assert torch.equal(y[0], y[1]) and torch.equal(state[0], state[far])


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_a_prompt_and_its_next_tokens_are_one_sequence(dt):
    """causal_conv and scan over 40 tokens, then six steps, against the oracle over all 46."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(21)
    sizes = h, p, g, n = 4, 64, 1, 128
    a, d, b = ssm_weights(rng, h)
    c, w = h * p + 2 * g * n, 4
    cw, cb = rng.normal(size=(c, w)).astype(np.float32) / 2, rng.normal(size=c).astype(np.float32)
    x, step = dev(rng.normal(size=(1, 46, c)), dt), dev(rng.normal(size=(1, 46, h)), dt)
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b), dev(cw), dev(cb))
    kept, state = torch.zeros(1, w, c, dtype=tdt(dt), device="cuda"), torch.zeros(1, h, p, n, device="cuda")
    v = sn.causal_conv(x[:, :40].contiguous(), dev(cw), dev(cb), kept=kept)
    ys = [ssm.scan(v, step[:, :40].contiguous(), state_out=state)[0]]
    for t in range(40, 46):
        ys.append(ssm.step(x[:, t], step[:, t], kept, state, ints([t])))
    vr, vm, _ = ob.conv(host(x)[0], cw, cb, True)
    ref, my, _, _ = ob.scan(vr, host(step)[0], sizes, a, d, b, np.zeros((h, p, n)))
    # the prompt's convolved values are rounded to the type: each of x, B and C off by its rounding
    _, me, _, _ = ob.scan(np.abs(vr) * (1 + U[dt]) + 48 * E32 * vm, host(step)[0], sizes, a, np.abs(d), b, np.zeros((h, p, n)))
    _, m0, _, _ = ob.scan(np.abs(vr), host(step)[0], sizes, a, np.abs(d), b, np.zeros((h, p, n)))
    close(torch.cat(ys), ref, me - m0 + scan_bound(me, 46) + (2.0 ** -14 * me if dt != "f32" else 0), dt)
