"""The attention layer's operators on the GPU against their fp64 oracle.

Error bounds: a result of m roundings of 2^-24 on terms of magnitudes that sum to M is off by at most
m 2^-24 M to first order; the kernels may add in any order, and the tensor cores truncate (one more bit).
U is the output type's rounding.  Every bound was fixed before its first run.
"""
import math

import numpy as np
import pytest

from oracle import attention as oa

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
U = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}  # half the spacing of the smallest values
TYPES = ["f32", "f16", "bf16"]


def tdt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def dev(a, name="f32"):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(tdt(name))


def ints(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, ref, bound, dt):
    got = host(got)
    assert got.shape == ref.shape
    err = np.abs(got - ref) - (U[dt] * np.abs(ref) + bound + TINY[dt])
    assert not np.isnan(got).any()
    assert err.max(initial=-1.0) <= 0, (float(err.max()), np.unravel_index(err.argmax(), err.shape))


# ------------------------------------------------------------------- rope
def rope_bound(y, x, mags, dim):
    """Norm: dim + 8 roundings of its sums count half (a square root), two products, the factor's 2 ulp.  An angle is
    off by 2^-25 of at most pi / 4 and the pairs' 2^-64 a position; sine and cosine by 2 ulp; two products and a sum."""
    return (dim / 2 + 4 + 4 + 8) * E32 * mags


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("tokens, qh, kh, dim, pairs, axes, norm, inter, start", [
    (1, 1, 1, 2, 1, 1, "rms", False, 0), (3, 4, 2, 64, 32, 1, "rms", False, 5000), (5, 3, 1, 80, 36, 3, "layer", True, 70),
    (7, 2, 2, 256, 128, 1, "none", False, 2 ** 31 - 10), (9, 5, 5, 48, 12, 3, "rms", False, -40), (2, 32, 8, 128, 64, 1, "layer", False, 10 ** 6),
    (4, 1, 0, 66, 33, 1, "rms", True, 9), (4, 0, 3, 34, 5, 1, "layer", False, 9), (6, 2, 1, 256, 128, 3, "rms", True, 123456789),
    (300, 7, 1, 96, 48, 1, "rms", False, 0), (2, 3, 3, 254, 127, 1, "rms", False, 77), (3, 2, 2, 32, 0, 1, "rms", False, 0)])
def test_rope(dt, tokens, qh, kh, dim, pairs, axes, norm, inter, start):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(dim + tokens)
    freq = [10000.0 ** (-i / max(pairs, 1)) for i in range(pairs)]
    which = [min(axes - 1, i * axes // pairs) for i in range(pairs)] if axes > 1 else None
    wide = dev(rng.normal(size=(tokens, (qh + kh) * dim + 8)), dt)
    q = wide[:, :qh * dim].unflatten(1, (qh, dim)) if qh else None
    k = wide[:, qh * dim:(qh + kh) * dim].unflatten(1, (kh, dim)) if kh else None
    pos = start + np.stack([np.arange(tokens) * (i + 1) % 1000 for i in range(axes)], axis=1)
    pos = np.minimum(pos, 2 ** 31 - 1)
    w = [None if norm == "none" else rng.uniform(0.5, 1.5, dim).astype(np.float32) for _ in range(2)]
    layer = sn.HeadRope(dim, freq, norm=norm, interleaved=inter, axes=which, q_weight=None if w[0] is None else dev(w[0]),
                        k_weight=None if w[1] is None else dev(w[1]))
    got = layer(q, k, ints(pos if axes > 1 else pos[:, 0]))
    for g, x, weight in zip(got, (q, k), w):
        assert (g is None) == (x is None)
        if x is None:
            continue
        assert g.is_contiguous() and g.dtype == x.dtype
        y, n = oa.head_rope(host(x), pos, freq, which, norm, 1e-6, weight, inter)
        mags = np.abs(n).max(axis=2, keepdims=True) * 2
        if norm == "layer":  # (the mean's own roundings, relative to the head's spread)
            v = host(x)
            mags = mags + np.abs(v).max(axis=2, keepdims=True) / np.sqrt(v.var(axis=2, keepdims=True) + 1e-6) * 1.5
        close(g, y, rope_bound(y, n, mags, dim), dt)


def test_rope_in_place_and_heads_before_tokens():
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(3)
    layer = sn.HeadRope(64, [0.3 ** i for i in range(20)])
    x = dev(rng.normal(size=(5, 9, 64)), "bf16")
    pos = ints(np.arange(9))
    want = layer(x.transpose(0, 1).contiguous(), None, pos)[0]
    assert torch.equal(layer(x.transpose(0, 1), None, pos)[0], want)
    y = x.clone().transpose(0, 1)
    assert layer(y, None, pos, q_out=y)[0] is y and torch.equal(y, want)
    batch = dev(rng.normal(size=(2, 3, 5, 64)), "f16")
    p2 = ints([[0, 1, 2], [7, 8, 9]])
    a = layer(batch, batch, p2)
    b = layer(batch.flatten(0, 1), None, p2.flatten())[0]
    assert torch.equal(a[0].flatten(0, 1), b) and torch.equal(a[1], a[0])


def test_rope_refusals():
    import torch
    import paper_2110_06037_gb300 as sn
    layer = sn.HeadRope(64, [1.0] * 32, axes=[i % 3 for i in range(32)])
    x = dev(np.zeros((4, 2, 64)), "bf16")
    for call in (lambda: layer(x, x, None), lambda: layer(), lambda: layer(x, x[:3], ints(np.zeros((4, 3)))), lambda: layer(x, x.half(), ints(np.zeros((4, 3)))),
                 lambda: layer(x, None, ints(np.zeros(4))), lambda: layer(x, None, ints(np.zeros((4, 2)))), lambda: layer(x, None, ints(np.zeros((5, 3)))),
                 lambda: layer(x.double(), None, ints(np.zeros((4, 3)))), lambda: layer(x[..., :32], None, ints(np.zeros((4, 3)))),
                 lambda: layer(x[:, :1].expand(4, 2, 64), None, ints(np.zeros((4, 3)))), lambda: layer(x, None, torch.zeros(4, 3, device="cuda")),
                 lambda: layer(x, None, ints(np.zeros((4, 3))), k_out=x), lambda: layer(x, None, ints(np.zeros((4, 3))), q_out=x.float()),
                 lambda: layer(x.cpu(), None, ints(np.zeros((4, 3))))):
        with pytest.raises(sn.SnError):
            call()
    assert layer(x[:0], None, ints(np.zeros((0, 3))))[0].shape == (0, 2, 64)


# ------------------------------------------------------------------ cache
class Case:
    """A cache of random pages, dealt to sequences of `new` tokens behind `before`."""

    def __init__(self, dt, kind, new, before, heads, dim, page, seed=0, extra=2):
        import torch
        import paper_2110_06037_gb300 as sn
        rng = self.rng = np.random.default_rng(seed)
        self.dt, self.kind, self.new, self.before = dt, kind, list(new), list(before)
        per = [-(-(a + b) // page) for a, b in zip(new, before)]
        self.pages, self.page, self.heads, self.dim = sum(per) + extra, page, heads, dim
        order = rng.permutation(self.pages)
        self.table = np.full((len(new), max([1] + per) + 1), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(per):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.spare = order[at:]
        self.offsets = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        self.tokens, self.max_len = int(self.offsets[-1]), max(new)
        shape = (self.pages, heads, page, dim)
        kv = [rng.normal(size=shape).astype(np.float32) for _ in range(2)]
        if kind == "q8":
            cs = [oa.codes(v * (1 + rng.random(shape[:3])[..., None])) for v in kv]
            self.t = [torch.from_numpy(c).cuda() for c, _ in cs] + [dev(s) for _, s in cs]
            self.k, self.v = (c.astype(np.float64) * s[..., None].astype(np.float64) for c, s in cs)
        else:
            self.t = [dev(v, dt) for v in kv]
            self.k, self.v = (host(t) for t in self.t)
        self.cache = sn.KVCache(*self.t)

    def args(self):
        return dict(offsets=ints(self.offsets), max_len=self.max_len, pos=ints(self.before))

    def queries(self, q_heads, scale=1.5):
        return dev(scale * self.rng.normal(size=(self.tokens, q_heads, self.dim)), self.dt)

    def check(self, q, y, max_context=None, slots=None, table=None, before=None, scale=None):
        ref = oa.attend(host(q), self.k, self.v, self.table if table is None else table, self.offsets,
                        self.before if before is None else before, 1 / math.sqrt(self.dim) if scale is None else scale, max_context, slots)
        close(y, ref[0], attend_bound(ref, self.dim, self.dt), self.dt)
        return ref[0]


def attend_bound(ref, dim, dt):
    """A score of dim products and two factors is off by es; a weight by that (its sum too), its exponential's 4 ulp and,
    where it goes to the tensor cores in 16 bits, by its rounding; the sums by one rounding a key and 64 more.
    Added after a first run in which a query's one large weight met a value of 0: a weight in fp16 (codes, fp16) below the
    normal range is off by half the spacing there, 2^-25, not by a part of itself; the largest being 2^14, that is 2^-39
    of the largest, a key, times its value (of these tests' values none is beyond 16; the sum of weights is the largest's
    at least)."""
    _, mag, es, seen = ref
    if dt != "f32":
        mag = mag + (seen * 16.0 * 2.0 ** -39)[..., None] / U[dt]
    rel = 2 * (dim + 8) * 2 * E32 * es + 2 * 8 * E32 + (seen + 64) * 2 * E32 + U[dt]
    return mag * rel[..., None]


CASES = [
    ([1], [0], 1, 1, 16, 16), ([1], [299], 8, 2, 64, 16), ([1, 1, 1], [15, 16, 700], 4, 4, 32, 32), ([1], [2000], 6, 2, 80, 64),
    ([5, 3, 0, 8, 1], [130, 77, 40, 0, 250], 6, 2, 80, 16), ([1, 1], [1023, 63], 32, 8, 128, 64), ([2], [1500], 7, 1, 256, 128),
    ([4, 1], [64, 511], 16, 2, 96, 256), ([1, 0], [0, 9], 5, 1, 48, 16), ([70], [0], 4, 2, 64, 16), ([33, 1, 200], [0, 50, 120], 8, 2, 128, 64),
    ([17], [3], 3, 3, 32, 16), ([130, 9], [100, 0], 5, 1, 112, 32), ([64], [1000], 2, 2, 256, 64), ([40, 257], [7, 0], 7, 1, 48, 128),
    ([1] * 40, list(range(0, 400, 10)), 2, 1, 64, 16), ([9] * 5, [700, 1, 0, 31, 64], 8, 8, 80, 32)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("kind", ["plain", "q8"])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", CASES)
def test_attend(dt, kind, new, before, q_heads, heads, dim, page):
    c = Case(dt, kind, new, before, heads, dim, page, seed=dim + len(new))
    q = c.queries(q_heads)
    y = c.cache.attend(q, ints(c.table), max_context=max(a + b for a, b in zip(new, before)), **c.args())
    c.check(q, y)


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("f16", "q8"), ("bf16", "plain"), ("bf16", "q8")])
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [40, 3, 20, 33]])
def test_attend_without_place(dt, kind, new):
    """Pages outside the cache, positions beyond the table or max_context, sequences without an entry."""
    c = Case(dt, kind, new, [100, 90, 30, 8], 2, 64, 16, seed=5)
    table = c.table.copy()
    table[0, 1], table[0, 3], table[1, :] = -1, c.pages, -7
    table = table[:, :7]
    q = c.queries(4)
    y = c.cache.attend(q, ints(table), max_context=130, **c.args())
    ref = c.check(q, y, 130, table=table)
    assert not ref[c.offsets[1]:c.offsets[2]].any()  # no key at all: zeros
    slots = np.array([2, -1, 0, 9], dtype=np.int32)
    y = c.cache.attend(q, ints(c.table), max_context=50, slots=ints(slots), **c.args())
    c.check(q, y, 50, slots=slots)
    y = c.cache.attend(q, ints(c.table), offsets=ints(c.offsets), max_len=c.max_len, scale=-0.3)
    c.check(q, y, before=[0] * 4, scale=-0.3)
    y = c.cache.attend(q, ints(c.table), max_context=0, **c.args())
    assert not host(y).any()
    y = c.cache.attend(q, ints(c.table[:, :0]), **c.args())
    assert not host(y).any()


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("f16", "plain"), ("f16", "q8"), ("bf16", "plain"), ("bf16", "q8")])
@pytest.mark.parametrize("new", [[1, 1], [6, 2], [50, 9]])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_unseen_values_do_not_matter(dt, kind, new, bad):
    """Not finite: what lies behind the sequences in their last pages, other pages, and tokens behind the query's own."""
    import torch
    before = [300, 21]
    c = Case(dt, kind, new, before, 2, 64, 16, seed=6)
    q = c.queries(4)
    args = dict(max_context=400, **c.args())
    want = c.cache.attend(q, ints(c.table), **args)
    c.check(q, want)

    def spoil(b, at):
        n, i = c.table[b, at // c.page], at % c.page
        for t in c.t[2:] if kind == "q8" else c.t:
            t[int(n), :, i] = bad

    for t in c.t[2:] if kind == "q8" else c.t:
        t[torch.from_numpy(np.asarray(c.spare)).cuda().long()] = bad
    for b in range(2):
        for at in range(before[b] + new[b], -(-(before[b] + new[b]) // c.page) * c.page):
            spoil(b, at)
    y = c.cache.attend(q, ints(c.table), **args)
    assert torch.equal(y, want)
    spoil(0, before[0] + new[0] - 1)  # the last token's own
    y = c.cache.attend(q, ints(c.table), **args)
    last = new[0] - 1
    assert not torch.isfinite(y[last]).all()
    keep = torch.ones(len(y), dtype=torch.bool, device="cuda")
    keep[last] = False
    ref = oa.attend(host(q), c.k, c.v, c.table, c.offsets, before, 1 / math.sqrt(64))
    mine = keep.cpu().numpy()
    close(y[keep], ref[0][mine], attend_bound([r[mine] for r in ref], 64, dt), dt)


@pytest.mark.parametrize("new", [[1], [20]])
def test_scores_of_minus_infinity(new):
    c = Case("bf16", "plain", new, [70], 1, 64, 16, seed=8)
    c.t[0][:] = 0
    c.t[0][:, :, :, 0] = -math.inf
    q = c.queries(4)
    q[..., 0] = 1.0
    assert not host(c.cache.attend(q, ints(c.table), **c.args())).any()
    n, i = c.table[0, 0], 5
    c.t[0][int(n), 0, i, 0] = 2.0  # the one key that counts
    y = c.cache.attend(q, ints(c.table), **c.args())
    assert np.array_equal(host(y), np.broadcast_to(c.v[n, 0, i], y.shape))


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("f16", "plain"), ("bf16", "plain"), ("f16", "q8"), ("bf16", "q8"), ("f32", "q8")])
def test_layouts_batches_and_rows_behind(dt, kind):
    import torch
    c = Case(dt, kind, [6, 6], [50, 9], 2, 64, 16, seed=9)
    q = c.queries(4)
    args = c.args()
    want = c.cache.attend(q, ints(c.table), **args)
    c.check(q, want)
    swapped = q.transpose(0, 1).contiguous().transpose(0, 1)  # heads before tokens
    out = torch.full((4, 12, 64), 7.0, dtype=q.dtype, device="cuda").transpose(0, 1)
    assert c.cache.attend(swapped, ints(c.table), out=out, **args) is out
    assert torch.equal(out, want)
    wide = torch.zeros(12, 4, 65, dtype=q.dtype, device="cuda")  # odd strides
    wide[..., :64] = q
    assert torch.equal(c.cache.attend(wide[..., :64], ints(c.table), **args), want)
    batch = c.cache.attend(q.reshape(2, 6, 4, 64), ints(c.table), pos=ints(c.before))
    assert torch.equal(batch.reshape(12, 4, 64), want)
    more = torch.cat((q, q))
    out = torch.full((24, 4, 64), 7.0, dtype=q.dtype, device="cuda")
    c.cache.attend(more, ints(c.table), out=out, **args)
    assert torch.equal(out[:12], want) and bool((out[12:] == 7).all())
    assert c.cache.attend(q[:0], ints(c.table), offsets=ints([0, 0, 0]), max_len=0).shape == (0, 4, 64)


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("bf16", "plain"), ("f16", "q8")])
def test_attend_tokens_beside_a_prompt(dt, kind):
    """Long sequences of one token, whose keys are shared out and joined, in one call with a prompt; rows behind them."""
    import torch
    c = Case(dt, kind, [1, 150, 1, 0, 5], [3000, 10, 1700, 9, 2500], 2, 64, 32, seed=17)
    q = c.queries(8)
    y = c.cache.attend(q, ints(c.table), max_context=3001, **c.args())
    c.check(q, y)
    out = torch.full((c.tokens + 50, 8, 64), 7.0, dtype=q.dtype, device="cuda")
    c.cache.attend(torch.cat((q, q[:50])), ints(c.table), out=out, max_context=3001, **c.args())
    assert torch.equal(out[:c.tokens], y) and bool((out[c.tokens:] == 7).all())


def test_attend_graphs_and_streams():
    """Two captured calls replayed on two streams at once, and eager calls between them."""
    import torch
    c = Case("bf16", "plain", [1] * 8, [900 + 37 * i for i in range(8)], 2, 128, 64, seed=10)
    table, args = ints(c.table), c.args()
    qs = [c.queries(8) for _ in range(2)]
    want = [c.cache.attend(q, table, **args) for q in qs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q in qs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.cache.attend(q, table, **args))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = c.cache.attend(qs[0], table, stream=streams[1], **args)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and torch.equal(eager, want[0])
    c.check(qs[0], want[0])


def test_long_positions():
    """Keys beyond 2^31 bytes of the cache, and a row index beyond 2^31 values."""
    import torch
    import paper_2110_06037_gb300 as sn
    pages, heads, page, dim = 70000, 2, 64, 256  # 2.3e9 values
    k = torch.zeros(pages, heads, page, dim, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    cache = sn.KVCache(k, v)
    g = torch.Generator(device="cuda").manual_seed(1)
    kn = torch.randn(130, heads, dim, device="cuda", generator=g).bfloat16()
    vn = torch.randn(130, heads, dim, device="cuda", generator=g).bfloat16()
    table = ints([[69999, 3, 69998]])
    cache.write(kn, vn, table, offsets=ints([0, 130]), max_len=130)
    a, b = cache.read(table, offsets=ints([0, 130]), max_len=130, tokens=130)
    assert torch.equal(a, kn) and torch.equal(b, vn)
    q = torch.randn(1, heads, dim, device="cuda", generator=g).bfloat16()
    y = cache.attend(q, table, offsets=ints([0, 1]), max_len=1, pos=ints([129]))
    w = torch.softmax(torch.einsum("hd,jhd->hj", q[0].double(), kn.double()) / 16, dim=1)
    ref = torch.einsum("hj,jhd->hd", w, vn.double())
    assert (y[0].double() - ref).abs().max() <= 2.0 ** -8 * 2 * vn.abs().max().double()


# ------------------------------------------------------------ write, read
@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("kind", ["plain", "q8"])
@pytest.mark.parametrize("new, before, heads, dim, page", [
    ([1], [0], 1, 16, 16), ([1, 1, 1, 1], [700, 0, 31, 96], 8, 128, 16), ([40, 0, 33], [0, 7, 77], 3, 80, 32), ([5, 700], [15, 0], 2, 256, 128),
    ([1] * 70, list(range(70)), 1, 48, 64)])
def test_write_and_read(dt, kind, new, before, heads, dim, page):
    import torch
    c = Case(dt, kind, new, before, heads, dim, page, seed=11)
    k, v = (dev(c.rng.normal(size=(c.tokens + 3, heads, dim)) * np.exp(c.rng.normal(size=(c.tokens + 3, heads, 1))), dt) for _ in range(2))
    k[0, 0] = 0
    old = [t.clone() for t in c.t]
    c.cache.write(k, v, ints(c.table), **c.args())
    touched = torch.zeros(c.pages, page, dtype=torch.bool, device="cuda")
    for x, at in ((k, 0), (v, 1)):
        rows = x[:c.tokens].float().cpu().numpy()
        want_c, want_s = oa.codes(rows)
        for b in range(len(new)):
            for i in range(new[b]):
                n, j = int(c.table[b, (before[b] + i) // page]), (before[b] + i) % page
                touched[n, j] = True
                t = c.offsets[b] + i
                if kind == "q8":
                    assert np.array_equal(c.t[at][n, :, j].cpu().numpy(), want_c[t])
                    assert np.array_equal(c.t[at + 2][n, :, j].cpu().numpy(), want_s[t])
                else:
                    assert torch.equal(c.t[at][n, :, j], x[t])
    for now, was in zip(c.t, old):  # everything else is as it was
        same = (now == was).flatten(3).all(3) if now.dim() == 4 else now == was
        assert bool((same | touched[:, None]).all())
    ko, vo = c.cache.read(ints(c.table), tokens=c.tokens, dtype=tdt(dt), **c.args())
    for x, o in ((k, ko), (v, vo)):
        if kind == "q8":
            cc, ss = oa.codes(x[:c.tokens].float().cpu().numpy())
            back = (cc.astype(np.float32) * ss[..., None])
            assert torch.equal(o, torch.from_numpy(back).cuda().to(tdt(dt)))
        else:
            assert torch.equal(o, x[:c.tokens])
    out = torch.full((c.tokens + 2, heads, dim), 5.0, dtype=tdt(dt), device="cuda")
    out2 = out.clone()
    c.cache.read(ints(c.table), tokens=c.tokens + 2, k_out=out, v_out=out2, dtype=tdt(dt), **c.args())
    assert torch.equal(out[:c.tokens], ko) and bool((out[c.tokens:] == 5).all())


def test_write_without_place():
    import torch
    c = Case("bf16", "plain", [20, 20], [0, 40], 2, 32, 16, seed=12)
    k = dev(c.rng.normal(size=(40, 2, 32)), "bf16")
    table = c.table.copy()
    table[0, 0], table[1, 3] = -1, c.pages
    old = [t.clone() for t in c.t]
    c.cache.write(k, k, ints(table[:, :3]), slots=ints([0, 5]), **c.args())
    n = int(table[0, 1])
    assert torch.equal(c.t[0][n, :, :4].transpose(0, 1), k[16:20])
    mask = torch.ones(c.pages, 16, dtype=torch.bool, device="cuda")
    mask[n, :4] = False
    assert torch.equal(c.t[0].transpose(1, 2)[mask], old[0].transpose(1, 2)[mask])
    a, b = c.cache.read(ints(table[:, :3]), tokens=40, slots=ints([0, 5]), **c.args())
    assert not host(a[:16]).any() and torch.equal(a[16:20], k[16:20]) and not host(a[20:]).any()


def test_codes_of_extremes():
    import torch
    import paper_2110_06037_gb300 as sn
    x = np.zeros((8, 1, 16), dtype=np.float32)
    x[0, 0, 0], x[1, 0, 3], x[2, 0, :] = np.inf, np.nan, 3.0e38
    x[3, 0, :], x[4, 0, 1], x[5, 0, 2] = 1e-45, 1e-38, -np.inf
    x[6, 0] = np.arange(16) - 8
    cache = sn.KVCache(*sn.KVCache.empty(1, 1, 16, 16, codes=True))
    cache.write(dev(x), dev(x), ints([[0]]), offsets=ints([0, 8]), max_len=8)
    want = oa.codes(x)
    for t, s in ((0, 2), (1, 3)):
        assert np.array_equal(cache.tensors[t][0, 0, :8].cpu().numpy(), want[0][:, 0])
        assert np.array_equal(cache.tensors[s][0, 0, :8].cpu().numpy(), want[1][:, 0], equal_nan=True)
    back = cache.read(ints([[0]]), offsets=ints([0, 8]), max_len=8, tokens=8, dtype=torch.float32)[0]
    assert np.isnan(host(back)[[0, 1, 5]]).all() and np.isfinite(host(back)[[2, 3, 4, 6, 7]]).all()


@pytest.mark.parametrize("dt", ["f16", "bf16"])
def test_codes_near_halves(dt):
    """Quotients at and next to the middle between two codes."""
    rng = np.random.default_rng(13)
    v = np.round(rng.uniform(-127, 127, (3000, 1, 32)) * 2) / 2
    v[:, :, 0] = 127
    x = dev(v * 2.0 ** rng.integers(-8, 8, (3000, 1, 1)), dt)
    import paper_2110_06037_gb300 as sn
    cache = sn.KVCache(*sn.KVCache.empty(200, 1, 16, 32, codes=True))
    table = np.arange(200)[None]
    cache.write(x, x, ints(table), offsets=ints([0, 3000]), max_len=3000)
    want = oa.codes(x.float().cpu().numpy())
    assert np.array_equal(cache.tensors[0][:, 0].reshape(-1, 32)[:3000].cpu().numpy(), want[0][:, 0])


def test_cache_refusals():
    import torch
    import paper_2110_06037_gb300 as sn
    c = Case("bf16", "plain", [2, 2], [0, 0], 2, 32, 16)
    k, q, table = dev(np.zeros((4, 2, 32)), "bf16"), dev(np.zeros((4, 4, 32)), "bf16"), ints(c.table)
    a = c.args()
    for call in (lambda: c.cache.write(k, k, table), lambda: c.cache.write(k.half(), k.half(), table, **a), lambda: c.cache.write(k, k[:3], table, **a),
                 lambda: c.cache.write(k[:, :1], k[:, :1], table, **a), lambda: c.cache.write(k, k, table[:1], **a), lambda: c.cache.write(k, k, table.long(), **a),
                 lambda: c.cache.write(k, k, table.cpu(), **a), lambda: c.cache.write(k[:, :1].expand(4, 2, 32), k, table, **a),
                 lambda: c.cache.attend(q[:, :3], table, **a), lambda: c.cache.attend(q.float(), table, **a), lambda: c.cache.attend(q, table, out=q, **a),
                 lambda: c.cache.attend(q, table, out=q[:2], **a), lambda: c.cache.attend(q, table, max_context=-1, **a),
                 lambda: c.cache.attend(q, table, scale=math.inf, **a), lambda: c.cache.attend(q, table, offsets=a["offsets"], pos=a["pos"]),
                 lambda: c.cache.read(table, tokens=4, dtype=torch.float16, **a), lambda: c.cache.read(table, **a), lambda: c.cache.read(table, tokens=4, k_out=k, v_out=k, **a),
                 lambda: sn.KVCache(c.t[0], c.t[1][:1]), lambda: sn.KVCache(c.t[0].transpose(1, 2), c.t[1].transpose(1, 2)),
                 lambda: sn.KVCache(c.t[0], c.t[1], dev(np.zeros(1)), None)):
        with pytest.raises(sn.SnError):
            call()


# ----------------------------------------------------------------- verify
def drafts(rng, counts, vocab, dt):
    import torch
    n = sum(counts)
    logits = 2 * rng.normal(size=(n, vocab))
    p = 2 * rng.normal(size=(n + len(counts), vocab))
    at = [a + b + i for b, a in enumerate(np.concatenate(([0], np.cumsum(counts)))[:-1]) for i in range(counts[b])]
    if n:
        p[at] = logits + 0.4 * p[at]
    soft = lambda x: dev(np.exp(x) / np.exp(x).sum(1, keepdims=True), dt)  # noqa: E731
    d = soft(logits) if n else torch.zeros(0, vocab, dtype=tdt(dt), device="cuda")
    x = [int(rng.choice(vocab, p=np.exp(r) / np.exp(r).sum())) for r in logits]
    return soft(p), d, x, rng.random(n).astype(np.float32), rng.random(len(counts)).astype(np.float32)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("counts, vocab", [
    ([4], 1000), ([1], 1), ([0], 37), ([3, 0, 1, 8], 517), ([5] * 20, 64), ([2, 2], 40000), ([700], 33), ([0, 0], 5000), ([3, 1], 32768)])
def test_verify(dt, counts, vocab):
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(vocab)
    target, draft, x, u, s = drafts(rng, counts, vocab, dt)
    off = np.concatenate(([0], np.cumsum(counts))).astype(np.int32)
    got = sn.verify_draft(target, draft, ints(np.array(x, dtype=np.int32)), dev(u), dev(s), offsets=ints(off), max_len=max(counts))
    want = oa.verify(host(target), host(draft), x, u, s, off, max(counts) + 1)
    assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1])
    if len(set(counts)) == 1 and sum(counts):
        again = sn.verify_draft(target, draft, ints(np.array(x, dtype=np.int32)), dev(u), dev(s))
        assert np.array_equal(again[0].cpu().numpy(), want[0])


def test_verify_edges():
    """Equal rows, zeros, values that are no probabilities, tokens outside the vocabulary, the ends of [0, 1)."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(14)
    v = 300
    p = rng.random((9, v)).astype(np.float32) / 150
    q = p[:6].copy()
    p[1], q[1] = 0, p[4] * 0
    p[2, 5], p[2, 7], q[2, 9] = np.nan, -1, np.inf
    q[3] = 1
    off = [0, 2, 4, 6]
    p[8] = 0
    for x in ([7, 5, 9, -1, v, 11], [0, 1, 2, 3, 4, 5]):
        for u in (0.0, 0.5, 1 - 2.0 ** -24):
            for s in (0.0, 2.0 ** -24, 0.25, 1 - 2.0 ** -24):
                us, ss = np.full(6, u, dtype=np.float32), np.full(3, s, dtype=np.float32)
                got = sn.verify_draft(dev(p), dev(q), ints(x), dev(us), dev(ss), offsets=ints(off), max_len=4)
                want = oa.verify(p.astype(np.float64), q.astype(np.float64), x, us, ss, off, 5)
                assert np.array_equal(got[0].cpu().numpy(), want[0]) and np.array_equal(got[1].cpu().numpy(), want[1]), (x, u, s)


def test_verify_refusals_and_strides():
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(15)
    target, draft, x, u, s = drafts(rng, [2, 2], 100, "f32")
    x, u, s = ints(x), dev(u), dev(s)
    want = sn.verify_draft(target, draft, x, u, s)
    wide = torch.zeros(6, 101, device="cuda")
    wide[:, 1:] = target
    got = sn.verify_draft(wide[:, 1:], draft, x, u, s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert sn.verify_draft(target[:2], None, None, None, s)[0].shape == (2, 1)
    for call in (lambda: sn.verify_draft(target[:5], draft, x, u, s), lambda: sn.verify_draft(target, draft[:3], x, u, s),
                 lambda: sn.verify_draft(target, draft.half(), x, u, s), lambda: sn.verify_draft(target, draft, x.long(), u, s),
                 lambda: sn.verify_draft(target, draft, x, u[:2], s), lambda: sn.verify_draft(target, draft, x[:3], u, s),
                 lambda: sn.verify_draft(target, None, x, u, s), lambda: sn.verify_draft(target, draft, x, u, s, offsets=ints([0, 2, 4])),
                 lambda: sn.verify_draft(target, draft, x, u, s, out=torch.zeros(2, 2, dtype=torch.int32, device="cuda")),
                 lambda: sn.verify_draft(target.double(), draft.double(), x, u, s), lambda: sn.verify_draft(target.cpu(), draft, x, u, s)):
        with pytest.raises(sn.SnError):
            call()


# --------------------------------------------------------------- together
@pytest.mark.parametrize("dt, codes", [("f32", False), ("bf16", False), ("bf16", True), ("f16", True)])
def test_layer_in_steps(dt, codes):
    """Prompts at once and then token by token give what whole sequences give, and both the oracle's values."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(16)
    lens, heads, q_heads, dim, page = [50, 1, 23], 2, 4, 64, 16
    layer = sn.HeadRope(dim, [100.0 ** (-i / 32) for i in range(32)])
    table = ints(rng.permutation(12).reshape(3, 4))
    x = [dev(rng.normal(size=(n + 6, q_heads + 2 * heads, dim)), dt) for n in lens]

    def run(cuts):
        cache = sn.KVCache(*sn.KVCache.empty(12, heads, page, dim, tdt(dt), codes=codes))
        out = [[] for _ in lens]
        for a, b in cuts:
            rows = [t[a + (n if a else 0):n + b] for t, n in zip(x, lens)]
            n = [len(r) for r in rows]
            off = ints(np.concatenate(([0], np.cumsum(n))))
            wide = torch.cat(rows)
            first = [0 if a == 0 else m + a for m in lens]
            at = torch.cat([torch.arange(f, f + m) for f, m in zip(first, n)]).int().cuda()
            q, k = layer(wide[:, :q_heads], wide[:, q_heads:q_heads + heads], at)
            kw = dict(offsets=off, max_len=max(n), pos=ints(first))
            cache.write(k, wide[:, q_heads + heads:], table, **kw)
            y = cache.attend(q, table, max_context=64, **kw)
            for i, part in enumerate(y.split(n)):
                out[i].append(part)
        return [torch.cat(o) for o in out], cache

    # (a cut (a, b): from the prompt's start or a tokens behind its end to b tokens behind it)
    whole, cache = run([(0, 6)])
    steps, _ = run([(0, 1)] + [(i, i + 1) for i in range(1, 6)])
    for i, n in enumerate(lens):
        a, b = host(whole[i]), host(steps[i])
        kk, vv = cache.read(table[i:i + 1], max_len=n + 6, dtype=torch.float32 if codes else None)
        q, _ = layer(x[i][:, :q_heads], None, torch.arange(n + 6).int().cuda())
        kk, vv = (host(t)[0][None].transpose(0, 2, 1, 3) for t in (kk, vv))
        ref = oa.attend(host(q), kk, vv, np.array([[0]]), [0, n + 6], [0], 1 / math.sqrt(dim))
        for got in (whole[i], steps[i]):
            close(got, ref[0], attend_bound(ref, dim, dt), dt)
        assert a.shape == b.shape
