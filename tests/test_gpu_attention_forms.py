"""Attention over a cache on the GPU, each of its kernels' instances by its sizes, against the definition in 64 bits.

Error bounds, for terms of magnitudes that sum to M (the weights' values here): a score of dim products and eight
factors and roundings is off by (dim + 8) 2^-24 of the magnitude of its products, and by as much again where the tensor
cores truncate; a weight by that, and so is their sum; the exponential's argument and 2 ulp count 8 roundings, twice; the sums
one a key and 64 more, twice for truncation.  What goes to the tensor cores in 16 bits is off by PART of itself (one part: half
a step of its type; two parts: the square of that), in fp16 also by half the spacing of the smallest values, 2^-25, where the
largest weight is 2^14.  The result is rounded once, by U of itself.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

E32 = 2.0 ** -24
U = {"f32": 0.0, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 1e-37, "f16": 2.0 ** -24, "bf16": 1e-37}  # half the spacing of the smallest values


@pytest.fixture(autouse=True)
def no_wait_gave_up():
    import paper_2110_06037_gb300 as sn
    sn.check_device()
    yield
    sn.check_device()


def tdt(name):
    import torch
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def ints(a):
    import torch
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


class Case:
    """A cache of random pages, dealt to sequences of `new` tokens behind `before`, and their queries."""

    def __init__(self, dt, kind, new, before, q_heads, heads, dim, page, seed=0):
        import torch
        import paper_2110_06037_gb300 as sn
        self.g = g = torch.Generator(device="cuda").manual_seed(seed)
        self.dt, self.new, self.before, self.dim, self.heads, self.page = dt, list(new), list(before), dim, heads, page
        per = [-(-(a + b) // page) for a, b in zip(new, before)]
        pages = sum(per) + 2
        order = np.random.default_rng(seed).permutation(pages)
        self.table = np.full((len(new), max([1] + per) + 1), -1, dtype=np.int32)
        for i, n in enumerate(per):
            self.table[i, :n] = order[sum(per[:i]):sum(per[:i + 1])]
        self.offsets = np.concatenate(([0], np.cumsum(new))).astype(np.int32)
        shape = (pages, heads, page, dim)
        if kind == "q8":
            kv = [torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) for _ in range(2)]
            scales = [(0.5 + torch.rand(shape[:3], generator=g, device="cuda")) / 64 for _ in range(2)]
            self.t = kv + scales
        else:
            self.t = [torch.randn(shape, generator=g, device="cuda").to(tdt(dt)) for _ in range(2)]
        self.cache = sn.KVCache(*self.t)
        self.q = (1.5 * torch.randn(int(self.offsets[-1]), q_heads, dim, generator=g, device="cuda")).to(tdt(dt))
        self.args = dict(offsets=ints(self.offsets), max_len=max(new), pos=ints(before), max_context=max(a + b for a, b in zip(new, before)))

    def run(self, **kw):
        return self.cache.attend(self.q, ints(self.table), **{**self.args, **kw})

    def values(self):
        """(keys, values) as fp64 [pages, heads, page, dim]."""
        k, v = (t.double() for t in self.t[:2])
        return (k, v) if len(self.t) == 2 else (k * self.t[2].double()[..., None], v * self.t[3].double()[..., None])

    def reference(self):
        """(y, magnitude of what is averaged, magnitude of a score's products, keys seen, largest value)."""
        import torch
        k, v = self.values()
        scale, group = 1 / math.sqrt(self.dim), self.q.shape[1] // self.heads
        y = torch.zeros(self.q.shape, dtype=torch.float64, device="cuda")
        mag, es = torch.zeros_like(y), torch.zeros(y.shape[:2], dtype=torch.float64, device="cuda")
        seen, top = torch.zeros_like(es), torch.zeros_like(es)
        for b, (n, at) in enumerate(zip(self.new, self.before)):
            if n == 0:
                continue
            ids = torch.from_numpy(self.table[b, :-(-(n + at) // self.page)]).long().cuda()
            rows = slice(int(self.offsets[b]), int(self.offsets[b + 1]))
            last = at + torch.arange(n, device="cuda")
            unseen = torch.arange(n + at, device="cuda")[None, :] > last[:, None]
            for h in range(self.q.shape[1]):
                kk, vv = (t[ids, h // group].flatten(0, 1)[:n + at] for t in (k, v))
                q = self.q[rows, h].double()
                s = (q @ kk.T * scale).masked_fill(unseen, -math.inf)
                w = torch.softmax(s, dim=1)
                y[rows, h], mag[rows, h] = w @ vv, w @ vv.abs()
                es[rows, h] = (q.abs() @ kk.abs().T * scale).masked_fill(unseen, 0).amax(dim=1)
                seen[rows, h], top[rows, h] = (last + 1).double(), vv.abs().max()
        return y, mag, es, seen, top

    def check(self, got, part):
        y, mag, es, seen, top = self.reference()
        rel = 2 * (self.dim + 8) * 2 * E32 * es + 16 * E32 + (seen + 64) * 2 * E32 + part
        bound = mag * rel[..., None]
        if self.dt == "f16" or len(self.t) > 2:
            bound = bound + (seen * top * 2.0 ** -39)[..., None]
        err = (got.double() - y).abs() - (U[self.dt] * (y.abs() + bound) + bound + TINY[self.dt])
        assert not got.isnan().any()
        assert float(err.max()) <= 0, (float(err.max()), np.unravel_index(int(err.argmax()), tuple(err.shape)))


# new, before, query heads, heads, dim, page: more than 64 rows a sequence, 16-bit values.  Heads beyond 128 values go by one tile
# of 128 rows and 64 keys at a time; up to eight of these are one block's, and so are more where blocks are many
PROMPTS = [
    ([40], [0], 4, 2, 192, 16), ([65], [0], 1, 1, 256, 128), ([70], [0], 1, 1, 144, 16), ([130], [0], 2, 2, 256, 256), ([90], [60], 3, 1, 176, 32),
    ([100, 1, 66], [100, 300, 60], 7, 1, 192, 32), ([80], [432], 4, 4, 256, 64), ([640], [560], 32, 8, 256, 128),
    ([90, 70], [2000, 777], 4, 2, 256, 16), ([200], [3000], 8, 2, 144, 256), ([66, 65], [1000, 999], 2, 2, 240, 128),
    # and where few rows have many keys, whose units are shared out and joined, heads of up to 128
    ([90], [1100], 4, 2, 128, 16), ([130, 1, 70], [5000, 40, 2000], 8, 2, 96, 64), ([100], [2500], 2, 1, 80, 256), ([70], [3000], 3, 1, 64, 32),
    ([66], [1500], 2, 2, 16, 128), ([300], [1000], 1, 1, 128, 256), ([129, 65], [1200, 4000], 5, 1, 48, 128),
    # two tiles of rows a block
    ([300, 17], [0, 5], 8, 2, 128, 256), ([260], [700], 4, 2, 64, 256), ([128, 257], [3, 0], 2, 2, 112, 128)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", PROMPTS)
def test_prompts(dt, new, before, q_heads, heads, dim, page):
    import torch
    c = Case(dt, "plain", new, before, q_heads, heads, dim, page, seed=dim + len(new))
    y = c.run()
    c.check(y, U[dt])
    for _ in range(3):
        assert torch.equal(c.run(), y)


# What weights (and fp32 values) are off by: two parts of 16 bits; in tf32 each of two factors by 2^-21 (what is dropped of its
# second part) and the product of the second parts, 2^-22, left out; codes: two parts of fp16, one for bf16.
FEW = {("f32", "plain"): 2.0 ** -19, ("f16", "plain"): 2.0 ** -22, ("bf16", "plain"): 2.0 ** -16, ("f32", "q8"): 2.0 ** -21, ("f16", "q8"): 2.0 ** -21,
       ("bf16", "q8"): 2.0 ** -11}
# Enough to do that items have more than 8 rows (tokens times the heads that share): up to 12 rows go by 16, up to 48 by 32.
# 450 keys: a block takes whole items; 740: units are shared out
ROWS = {12: [3, 3, 2, 1] * 12, 48: [12, 7, 9, 0, 5] * 4}


@pytest.mark.parametrize("dt, kind", FEW)
@pytest.mark.parametrize("dim, rows, context, heads", [
    (48, 12, 450, 7), (64, 12, 740, 5), (64, 48, 450, 7), (16, 48, 740, 5), (112, 12, 740, 5), (128, 12, 450, 7), (128, 48, 740, 5), (80, 48, 450, 7),
    (208, 12, 450, 7), (256, 12, 740, 5), (256, 48, 450, 7), (144, 48, 740, 5)])
def test_few_rows(dt, kind, dim, rows, context, heads):
    import torch
    new = ROWS[rows]
    c = Case(dt, kind, new, [max(0, context - n - 7 * i) for i, n in enumerate(new)], 4 * heads, heads, dim, 64, seed=dim + rows)
    y = c.run()
    c.check(y, FEW[dt, kind])
    assert torch.equal(c.run(), y)


@pytest.mark.parametrize("dt, kind", [k for k in FEW if k[0] == "f32" or k[1] == "q8"])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", [
    ([100] * 14, list(range(14)), 16, 4, 128, 32), ([900, 300], [0, 77], 8, 2, 128, 64), ([700, 0, 133], [5, 9, 600], 12, 3, 64, 16),
    ([333, 401], [100, 0], 8, 2, 256, 256), ([1100], [40], 5, 1, 96, 128)])
def test_prompts_by_few_rows(dt, kind, new, before, q_heads, heads, dim, page):
    """Prompts in fp32 and over codes."""
    c = Case(dt, kind, new, before, q_heads, heads, dim, page, seed=dim + len(new))
    c.check(c.run(), FEW[dt, kind])


@pytest.mark.parametrize("dt, kind", FEW)
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", [
    # single tokens and drafts in items of 8 rows, short and shared out, alone and beside prompts; groups that do not divide 8
    ([1, 1, 1], [0, 15, 700], 8, 8, 128, 16), ([1], [5000], 3, 1, 96, 64), ([2, 0, 3], [1000, 0, 70], 7, 1, 64, 256), ([1, 1], [2000, 30], 20, 1, 240, 32),
    ([1, 200, 1, 9], [4000, 0, 63, 1500], 8, 2, 128, 128), ([1] * 33, list(range(33)), 4, 4, 32, 16), ([1], [3000], 200, 2, 128, 64)])
def test_tokens(dt, kind, new, before, q_heads, heads, dim, page):
    c = Case(dt, kind, new, before, q_heads, heads, dim, page, seed=dim + len(new))
    y = c.run()
    part = U[dt] if kind == "plain" and dt != "f32" and max(new) > 64 else FEW[dt, kind]  # (a prompt's weights are one part)
    c.check(y, part)


@pytest.mark.parametrize("dt, kind", [("f32", "plain"), ("bf16", "plain"), ("f16", "q8")])
@pytest.mark.parametrize("context", [64, 4096])
def test_rows_behind_empty_sequences_are_left(dt, kind, context):
    import torch
    c = Case(dt, kind, [9], [0], 4, 2, 64, 16)
    out = torch.full_like(c.q, 7.0)
    c.cache.attend(c.q, ints(np.zeros((3, 300))), offsets=ints([0, 0, 0, 0]), max_len=0, pos=ints([5, 0, 9]), max_context=context, out=out)
    assert bool((out == 7).all())


PROMPT_FORMS = [([200, 9, 70], [0, 30, 5], 8, 2, 128, 64), ([90, 1], [200, 0], 4, 2, 48, 16), ([70, 66], [0, 100], 4, 2, 256, 128),
                ([80, 5], [2500, 3000], 4, 2, 128, 32)]


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", PROMPT_FORMS)
def test_prompt_layouts_and_rows_behind(dt, new, before, q_heads, heads, dim, page):
    """Heads before tokens, strides that no vector load fits, rows behind the last sequence; scales of both signs and zero."""
    import torch
    c = Case(dt, "plain", new, before, q_heads, heads, dim, page, seed=21)
    want, n = c.run(), len(c.q)
    kw = dict(**c.args)
    swapped = c.q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full((q_heads, n, dim), 7.0, dtype=c.q.dtype, device="cuda").transpose(0, 1)
    assert c.cache.attend(swapped, ints(c.table), out=out, **kw) is out and torch.equal(out, want)
    for shift in (0, 1):
        wide = torch.full((n + 3, q_heads, dim + 3), 7.0, dtype=c.q.dtype, device="cuda")
        result = wide.clone()
        wide[:n, :, shift:shift + dim] = c.q
        c.cache.attend(wide[..., shift:shift + dim], ints(c.table), out=result[..., shift:shift + dim], **kw)
        assert torch.equal(result[:n, :, shift:shift + dim], want)
        result[:n, :, shift:shift + dim] = 7
        assert bool((result == 7).all())
    minus = c.cache.attend(-c.q, ints(c.table), scale=-1 / math.sqrt(dim), **kw)
    assert torch.equal(minus, want)
    c.q.zero_()
    assert torch.equal(c.run(scale=0.0), c.run())


@pytest.mark.parametrize("dt", ["f16", "bf16"])
@pytest.mark.parametrize("new, before, q_heads, heads, dim, page", PROMPT_FORMS)
def test_prompts_at_once_and_replayed(dt, new, before, q_heads, heads, dim, page):
    """Two captured calls replayed on two streams, eager ones between them."""
    import torch
    cs = [Case(dt, "plain", new, before, q_heads, heads, dim, page, seed=s) for s in (22, 23)]
    tables = [ints(c.table) for c in cs]
    want = [c.run() for c in cs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for c, t in zip(cs, tables):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(c.cache.attend(c.q, t, **c.args))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        eager = cs[0].cache.attend(cs[0].q, tables[0], stream=streams[1], **cs[0].args)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1]) and torch.equal(eager, want[0])
