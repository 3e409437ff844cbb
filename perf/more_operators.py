"""Operators of attention layers in their serving form, as they stand between state-space blocks.

Such a layer normalises and rotates its queries and keys, writes keys and values into a paged cache,
and reads the cache back for every new token: one token a sequence, a few drafted ones, or a prompt.
Drafted tokens are then verified against the probabilities of the model that drafted nothing.

  rope    v' = norm(v) * w over each head (rms, layer or none), then pairs (a, b) of its first
          2 F values turn by theta_i = pos[axis_i] * f_i: (a cos - b sin, a sin + b cos); the pairs
          are (i, i + F), or (2 i, 2 i + 1) interleaved
  kv      keys and values of new tokens into pages, [pages, heads, page, dim] each, as they are or
          as codes c = rint(v / s), s = max |v| / 127 a token and head (1 for zeros); and back
  attend  y_i = sum_j softmax_j(q_i k_j / sqrt(D)) v_j over the keys at positions j <= before + i of
          the query's own sequence; query heads share key heads by group
  verify  token x_i stays while u_i q_i(x_i) < p_i(x_i); at the first that does not, the next token is
          drawn from max(p - q, 0) (or p, where that is zero everywhere) of its row, without one from
          the last row of p: the first index whose cumulative sum exceeds u times the total

`own` chooses between the plain form (elementary torch operations in 32 bits, in 64 for angles and
cumulative sums, rounded once at the end) and the calls of this package.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-6


def _uneven(seed, n, lo, hi):
    r = random.Random(seed)
    return ",".join(str(r.randint(lo, hi)) for _ in range(n))


def listed():
    return [
        # one token of one sequence: the smallest call
        {"name": "rope_token", "op": "rope", "dtype": "f16", "tokens": 1, "q_heads": 32, "k_heads": 8, "dim": 128,
         "pairs": 64, "axes": 1, "norm": "rms", "interleaved": False, "start": 5000},
        # a long prompt
        {"name": "rope_prompt", "op": "rope", "dtype": "bf16", "tokens": 8192, "q_heads": 32, "k_heads": 8, "dim": 128,
         "pairs": 64, "axes": 1, "norm": "rms", "interleaved": False, "start": 0},
        # frames of a video in fp32: positions in time, height and width, a part of each head turned
        {"name": "rope_frames", "op": "rope", "dtype": "f32", "tokens": 1111, "q_heads": 6, "k_heads": 2, "dim": 80,
         "pairs": 36, "axes": 3, "norm": "layer", "interleaved": True, "start": 70},
        # one token of each of a few sequences, kept as codes
        {"name": "kv_tokens", "op": "kv", "dtype": "f16", "kind": "q8", "new": "1,1,1,1", "before": "700,0,31,4096",
         "heads": 8, "dim": 128, "page": 16},
        # a long prompt beside a short one, kept as codes
        {"name": "kv_prompt", "op": "kv", "dtype": "bf16", "kind": "q8", "new": "8000,333", "before": "0,77",
         "heads": 8, "dim": 128, "page": 64},
        # one token of a short conversation: latency
        {"name": "attend_token", "op": "attend", "dtype": "f16", "kind": "plain", "new": "1", "before": "299",
         "q_heads": 8, "heads": 2, "dim": 64, "page": 16},
        # one token behind a very long context: one row, all the work along the cache
        {"name": "attend_long", "op": "attend", "dtype": "bf16", "kind": "plain", "new": "1", "before": "131071",
         "q_heads": 32, "heads": 8, "dim": 128, "page": 64},
        # one token of every sequence of a batch of uneven lengths, over codes
        {"name": "attend_batch_q8", "op": "attend", "dtype": "bf16", "kind": "q8", "new": ",".join(["1"] * 64),
         "before": _uneven(1, 64, 500, 9000), "q_heads": 32, "heads": 8, "dim": 128, "page": 32},
        # drafted tokens, fp32, odd sizes, a sequence that has none and one without a past
        {"name": "attend_drafts", "op": "attend", "dtype": "f32", "kind": "plain", "new": "5,3,0,8,1",
         "before": "1030,77,40,0,2500", "q_heads": 6, "heads": 2, "dim": 80, "page": 16},
        # prompts: the tensor cores count
        {"name": "attend_prompt", "op": "attend", "dtype": "bf16", "kind": "plain", "new": "4096,1,777",
         "before": "0,50,1200", "q_heads": 32, "heads": 8, "dim": 128, "page": 64},
        # four drafted tokens of one sequence over a small vocabulary
        {"name": "verify_1", "op": "verify", "dtype": "f32", "drafts": "4", "vocab": 1000},
        # a batch over a large one, some sequences with fewer drafts or none
        {"name": "verify_batch", "op": "verify", "dtype": "f32",
         "drafts": ",".join(["5"] * 50 + ["3", "0", "1", "8"] * 3 + ["2", "4"]), "vocab": 128000},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "kv", "attend", "attend", "attend", "verify"])
    dt = rng.choice(["f32", "f16", "bf16", "bf16"])
    dim = rng.choice([32, 48, 64, 64, 80, 96, 128, 128, 128, 256])
    page = rng.choice([16, 32, 64, 128])
    if op == "rope":
        hk = rng.choice([1, 2, 3, 4, 8])
        hq = hk * rng.choice([1, 2, 4, 7, 8])
        axes = rng.choice([1, 1, 3])
        top = 8192 * 40 * 128 * 2 // ((hq + hk) * dim * SIZE[dt])
        return {"op": op, "dtype": dt, "tokens": _log_int(rng, 1, min(8192, top)), "q_heads": hq, "k_heads": hk,
                "dim": dim, "pairs": rng.choice([dim // 2, dim // 2, dim // 4]), "axes": axes,
                "norm": rng.choice(["rms", "rms", "layer", "none"]), "interleaved": rng.random() < 0.3,
                "start": rng.choice([0, _log_int(rng, 1, 1000000)])}
    if op == "verify":
        batch = _log_int(rng, 1, 64)
        n = rng.choice([1, 3, 5, 5, 8])
        return {"op": op, "dtype": rng.choice(["f32", "f32", "bf16", "f16"]),
                "drafts": ",".join(str(rng.choice([n, n, n, rng.randint(0, n)])) for _ in range(batch)),
                "vocab": _log_int(rng, 32, min(128000, 50000000 // (batch * (n + 1))))}
    heads = rng.choice([1, 2, 3, 8, 8])
    kind = rng.choice(["plain", "q8"])
    if op == "kv":
        n = rng.choice([1, 2, 5, 16])
        top = max(2, 8192 * 8 * 128 * 2 // (heads * dim * SIZE[dt] * n))
        new = [rng.choice([1, _log_int(rng, 1, min(8192, top))]) for _ in range(n)]
        return {"op": op, "dtype": dt, "kind": kind, "new": ",".join(map(str, new)),
                "before": ",".join(str(rng.choice([0, _log_int(rng, 1, 5000)])) for _ in new), "heads": heads,
                "dim": dim, "page": page}
    group = rng.choice([1, 2, 4, 4, 5, 7, 8])
    form = rng.choice(["token", "token", "draft", "prompt"])
    if form == "prompt":
        n = rng.choice([1, 1, 2, 4])
        pairs = 4096 * 4096 * 32 * 128 // (2 * heads * group * dim) // n // (4 if dt == "f32" else 1)
        new = [_log_int(rng, 9, max(10, min(4096, int(math.sqrt(pairs))))) for _ in range(n)]
        before = [rng.choice([0, 0, _log_int(rng, 1, 1000)]) for _ in new]
    else:
        n = _log_int(rng, 1, 64)
        size = 1 if kind == "q8" else SIZE[dt]
        top = max(2, 131072 * 8 * 128 * 2 // (heads * dim * size * n))
        longest = _log_int(rng, 1, min(131000, top))
        new = [1 if form == "token" else rng.randint(0 if i else 1, 8) for i in range(n)]
        before = [rng.randint(longest // 10, longest) for _ in new]
    return {"op": op, "dtype": dt, "kind": kind, "new": ",".join(map(str, new)), "before": ",".join(map(str, before)),
            "q_heads": heads * group, "heads": heads, "dim": dim, "page": page}


# ------------------------------------------------------------------ inputs
def _numbers(text):
    return [int(v) for v in text.split(",")]


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _frequencies(case):
    """Angle a position of each pair, and the position axis that it turns by (sections one behind the other)."""
    n, axes = case["pairs"], case["axes"]
    return [10000.0 ** (-i / n) for i in range(n)], [min(axes - 1, i * axes // n) for i in range(n)]


def _codes(v):
    """Codes and scales a row of the last axis."""
    top = v.float().abs().amax(dim=-1)
    s = torch.where(top > 0, top / 127.0, 1.0)
    return torch.round(v.float() / s[..., None]).clamp(-127, 127).to(torch.int8), s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rnd(*shape, dt=torch.float32):
        return torch.randn(shape, device="cuda", generator=g).to(dt)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if own:
        import paper_2110_06037_gb300 as sn
    if case["op"] == "rope":
        t, d = case["tokens"], case["dim"]
        wide = rnd(t, (case["q_heads"] + case["k_heads"]) * d, dt=dt)  # one projection makes both
        cut = case["q_heads"] * d
        s["q"], s["k"] = wide[:, :cut].unflatten(1, (-1, d)), wide[:, cut:].unflatten(1, (-1, d))
        at = case["start"] + torch.arange(t, device="cuda")
        if case["axes"] == 3:  # frames of 20 rows of 30
            at = torch.stack((at // 600, at // 30 % 20, at % 30), dim=1)
        s["pos"] = at.to(torch.int32)
        s["qw"], s["kw"] = 1.0 + 0.1 * rnd(d), 1.0 + 0.1 * rnd(d)
        if case["norm"] == "none":
            s["qw"] = s["kw"] = None
        f, axis = _frequencies(case)
        s["f"], s["axis"] = torch.tensor(f, dtype=torch.float64, device="cuda"), torch.tensor(axis, device="cuda")
        if own:  # the layer's handle: weights and frequencies
            s["rope"] = sn.HeadRope(d, f, norm=case["norm"], eps=EPS, q_weight=s["qw"], k_weight=s["kw"],
                                    interleaved=case["interleaved"], axes=axis)
        return s
    if case["op"] == "verify":
        n, vocab = _numbers(case["drafts"]), case["vocab"]
        at, rows = _starts(n), sum(n)
        s["offsets"], s["max_len"] = ints(at), max(n)
        logits = 2.0 * rnd(rows, vocab)
        s["draft"] = torch.softmax(logits, dim=1).to(dt)
        noise = -torch.log(-torch.log(torch.rand((rows, vocab), device="cuda", generator=g).clamp(1e-7, 1 - 1e-7)))
        s["tokens"] = (logits + noise).argmax(dim=1).to(torch.int32) if rows else ints([])
        where = torch.tensor([a + i + j for i, a in enumerate(at[:-1]) for j in range(n[i])], dtype=torch.long,
                             device="cuda")
        target = 2.0 * rnd(rows + len(n), vocab)
        target[where] = logits + 0.4 * target[where]
        s["target"] = torch.softmax(target, dim=1).to(dt)
        s["accept"] = torch.rand(rows, device="cuda", generator=g)
        s["sample"] = torch.rand(len(n), device="cuda", generator=g)
        return s
    # a cache whose pages are dealt to the sequences in no order
    new, before, h, d, page = _numbers(case["new"]), _numbers(case["before"]), case["heads"], case["dim"], case["page"]
    per = [-(-(a + b) // page) for a, b in zip(new, before)]
    pages, width = sum(per) + 3, max(1, max(per))
    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(new), width), -1, dtype=torch.int32, device="cuda")
    for i, (a, b) in enumerate(zip(_starts(per), per)):
        table[i, :b] = order[a:a + b]
    at = _starts(new)
    s.update(table=table, pos=ints(before), offsets=ints(at), max_len=max(new))
    codes = case["kind"] == "q8"
    if case["op"] == "kv":
        s["k"], s["v"] = rnd(at[-1], h, d, dt=dt), rnd(at[-1], h, d, dt=dt)
        kept = [torch.zeros(pages, h, page, d, dtype=torch.int8 if codes else dt, device="cuda") for _ in range(2)]
        scales = [torch.zeros(pages, h, page, device="cuda") for _ in range(2)] if codes else [None, None]
    else:
        s["q"] = 1.5 * rnd(at[-1], case["q_heads"], d)
        s["q"] = s["q"].to(dt)
        kept, scales = [], []
        for _ in range(2):
            v = rnd(pages, h, page, d, dt=dt)
            c, f = _codes(v) if codes else (v, None)
            kept.append(c)
            scales.append(f)
        s["context"] = max(a + b for a, b in zip(new, before))
    s.update(kc=kept[0], vc=kept[1], ks=scales[0], vs=scales[1])
    if own:  # the layer's handle: the cache's buffers
        s["cache"] = sn.KVCache(s["kc"], s["vc"], s["ks"], s["vs"])
    return s


# ------------------------------------------------------------- plain forms
def _plain_head_norm(v, kind, weight):
    v = v.float()
    if kind == "none":
        return v
    if kind == "layer":
        v = v - v.mean(dim=-1, keepdim=True)
    return v * torch.rsqrt((v * v).mean(dim=-1, keepdim=True) + EPS) * weight


def _plain_rope(s):
    c = s["case"]
    n = c["pairs"]
    pos = s["pos"] if s["pos"].dim() == 2 else s["pos"][:, None]
    angle = pos[:, s["axis"]].double() * s["f"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = []
    for v, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x = _plain_head_norm(v, c["norm"], w)
        y = x.clone()
        if c["interleaved"]:
            a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
            y[..., 0:2 * n:2], y[..., 1:2 * n:2] = a * cos - b * sin, a * sin + b * cos
        else:
            a, b = x[..., :n], x[..., n:2 * n]
            y[..., :n], y[..., n:2 * n] = a * cos - b * sin, a * sin + b * cos
        out.append(y.to(v.dtype))
    return out


def _spots(s):
    """Page and place in it of every new token."""
    page = s["kc"].shape[2]
    t = torch.arange(s["k"].shape[0], device="cuda")
    seq = (t[:, None] >= s["offsets"][None, 1:]).sum(dim=1)
    at = s["pos"][seq].long() + t - s["offsets"][seq].long()
    return s["table"][seq, at // page].long(), at % page


def _plain_kv(s):
    page, place = _spots(s)
    out = []
    for v, kept, scale in ((s["k"], s["kc"], s["ks"]), (s["v"], s["vc"], s["vs"])):
        if scale is None:
            kept[page, :, place] = v
            out.append(kept[page, :, place])
        else:
            c, f = _codes(v)
            kept[page, :, place], scale[page, :, place] = c, f
            out.append((kept[page, :, place].float() * scale[page, :, place][..., None]).to(v.dtype))
    return out


def _plain_attend(s):
    c = s["case"]
    h, d, page = c["heads"], c["dim"], c["page"]
    group = c["q_heads"] // h
    y = torch.empty_like(s["q"])
    at = 0
    for i, (n, before) in enumerate(zip(_numbers(c["new"]), _numbers(c["before"]))):
        if n == 0:
            continue
        total = n + before
        ids = s["table"][i, :-(-total // page)].long()
        kv = []
        for kept, scale in ((s["kc"], s["ks"]), (s["vc"], s["vs"])):
            x = kept[ids].float()
            x = x if scale is None else x * scale[ids][..., None]
            kv.append(x.transpose(0, 1).reshape(h, -1, d)[:, :total])
        q = s["q"][at:at + n].float().reshape(n, h, group, d).permute(1, 2, 0, 3).reshape(h, group * n, d)
        w = (q @ kv[0].transpose(1, 2)).reshape(h, group, n, total) * (1.0 / math.sqrt(d))
        if n > 1:
            seen = torch.arange(total, device="cuda")[None] <= before + torch.arange(n, device="cuda")[:, None]
            w = torch.where(seen, w, -math.inf)
        w = torch.exp(w - w.amax(dim=-1, keepdim=True))
        w = (w / w.sum(dim=-1, keepdim=True)).reshape(h, group * n, total)
        o = (w @ kv[1]).reshape(h, group, n, d).permute(2, 0, 1, 3)
        y[at:at + n] = o.reshape(n, h * group, d).to(y.dtype)
        at += n
    return y


def _plain_verify(s):
    off = s["offsets"].long()
    n, batch = off[1:] - off[:-1], off.numel() - 1
    step = torch.arange(s["max_len"], device="cuda")
    real = step[None] < n[:, None]
    row = torch.where(real, off[:-1, None] + step, 0)                   # of the draft
    trow = off[:-1, None] + torch.arange(batch, device="cuda")[:, None] + torch.arange(s["max_len"] + 1, device="cuda")
    if s["tokens"].numel():
        tok = s["tokens"].long()[row]
        ok = real & (s["accept"].double()[row] * s["draft"][row, tok].double()
                     < s["target"][torch.where(real, trow[:, :-1], 0), tok].double())
        count = ok.long().cumprod(dim=1).sum(dim=1)
    else:
        tok, count = row, torch.zeros_like(n)
    seq = torch.arange(batch, device="cuda")
    p = s["target"][trow[seq, count]].double()
    w = p
    if s["tokens"].numel():
        last = torch.where(count < n, off[:-1] + count, 0)
        w = torch.where((count < n)[:, None], (p - s["draft"][last].double()).clamp_min(0.0), p)
        w = torch.where((w.sum(dim=1) > 0)[:, None], w, p)
    cumulative = w.cumsum(dim=1)
    bar = s["sample"].double() * cumulative[:, -1]
    drawn = (cumulative <= bar[:, None]).sum(dim=1).clamp_max(w.shape[1] - 1)
    out = torch.full((batch, s["max_len"] + 1), -1, dtype=torch.int32, device="cuda")
    out[:, :-1] = torch.where(step[None] < count[:, None], tok, -1).to(torch.int32)
    out[seq, count] = drawn.to(torch.int32)
    return [out, count.to(torch.int32)]


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"rope": _plain_rope, "kv": _plain_kv, "attend": _plain_attend, "verify": _plain_verify}[op](state)
    import paper_2110_06037_gb300 as sn
    if op == "rope":
        return list(state["rope"](state["q"], state["k"], state["pos"]))
    if op == "kv":
        cache = state["cache"]
        cache.write(state["k"], state["v"], state["table"], offsets=state["offsets"], max_len=state["max_len"],
                    pos=state["pos"])
        return list(cache.read(state["table"], offsets=state["offsets"], max_len=state["max_len"], pos=state["pos"],
                               tokens=state["k"].shape[0], dtype=state["k"].dtype))
    if op == "attend":
        return state["cache"].attend(state["q"], state["table"], offsets=state["offsets"], max_len=state["max_len"],
                                     pos=state["pos"], max_context=state["context"])
    return list(sn.verify_draft(state["target"], state["draft"], state["tokens"], state["accept"], state["sample"],
                                offsets=state["offsets"], max_len=state["max_len"]))


# ------------------------------------------------------------------- work
def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "rope":
        n = case["tokens"] * (case["q_heads"] + case["k_heads"])
        return {"bytes": 2 * e * n * case["dim"] + 4 * case["tokens"] * case["axes"],
                "flops": n * (5 * case["dim"] + 6 * case["pairs"])}
    if case["op"] == "verify":
        # the tokens' own probabilities, and a row of p (and of q, where there are drafts) a sequence
        n = _numbers(case["drafts"])
        rows = len(n) + sum(1 for v in n if v)
        return {"bytes": rows * case["vocab"] * e + sum(n) * (8 + 2 * e) + len(n) * 8,
                "flops": 2 * rows * case["vocab"]}
    new, before, h, d = _numbers(case["new"]), _numbers(case["before"]), case["heads"], case["dim"]
    kept = d + 4 if case["kind"] == "q8" else d * e  # bytes of a key
    if case["op"] == "kv":
        return {"bytes": sum(new) * h * (4 * d * e + 4 * kept), "flops": 6 * sum(new) * h * d}
    pairs = sum(n * b + n * (n + 1) // 2 for n, b in zip(new, before))
    return {"bytes": 2 * e * sum(new) * case["q_heads"] * d + sum(2 * kept * h * (n + b) for n, b in zip(new, before) if n),
            "flops": 4 * case["q_heads"] * d * pairs}


# ------------------------------------------- the definitions in 64 bits
def _exact_rope(case, s):
    f, axis = _frequencies(case)
    pos = s["pos"].reshape(case["tokens"], -1).double()
    out = []
    for v, w in ((s["q"].double(), s["qw"]), (s["k"].double(), s["kw"])):
        if case["norm"] != "none":
            m = v.sum(-1, keepdim=True) / v.shape[-1] if case["norm"] == "layer" else 0.0
            v = v - m
            v = v / torch.sqrt((v ** 2).sum(-1, keepdim=True) / v.shape[-1] + EPS) * w.double()
        y = v.clone()
        for i in range(case["pairs"]):
            a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + case["pairs"])
            turn = torch.polar(torch.ones_like(pos[:, 0]), pos[:, axis[i]] * f[i])[:, None]
            z = torch.complex(v[..., a], v[..., b]) * turn
            y[..., a], y[..., b] = z.real, z.imag
        out.append(y)
    return out


def _exact_kv(case, s):
    if case["kind"] == "plain":
        return [s["k"].double(), s["v"].double()]
    out = []
    for v in (s["k"].double(), s["v"].double()):
        top = v.abs().max(dim=-1, keepdim=True).values
        # scales are kept in 32 bits, and a code is the nearest to the quotient in 32 bits
        scale = torch.where(top == 0, torch.ones_like(top), top / 127).float().double()
        out.append((v / scale).float().double().round() * scale)
    return out


def _exact_attend(case, s):
    h, page = case["heads"], case["page"]
    group = case["q_heads"] // h
    if sum(n * (n + b) for n, b in zip(_numbers(case["new"]), _numbers(case["before"]))) * case["q_heads"] * case["dim"] > 4e11:
        return None
    y = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for i, (first, n, before) in enumerate(zip(_starts(_numbers(case["new"])), _numbers(case["new"]), _numbers(case["before"]))):
        if n == 0:
            continue
        j = torch.arange(n + before, device="cuda")
        id, place = s["table"][i].long()[j // page], j % page
        late = j[None, :] > (before + torch.arange(n, device="cuda"))[:, None]
        for head in range(h):
            k, v = s["kc"][id, head, place].double(), s["vc"][id, head, place].double()
            if s["ks"] is not None:
                k, v = k * s["ks"][id, head, place, None].double(), v * s["vs"][id, head, place, None].double()
            for one in range(head * group, (head + 1) * group):
                e = torch.mm(s["q"][first:first + n, one].double(), k.t()) / math.sqrt(case["dim"])
                e.masked_fill_(late, -math.inf)
                y[first:first + n, one] = torch.mm(torch.softmax(e, dim=1), v)
    return y


def _exact_verify(case, s):
    n = _numbers(case["drafts"])
    out = torch.full((len(n), max(n) + 1), -1, dtype=torch.int32)
    count = torch.zeros(len(n), dtype=torch.int32)
    tokens = s["tokens"].tolist()
    for b, first in enumerate(_starts(n)[:-1]):
        for i in range(n[b] + 1):
            p, w = s["target"][first + b + i].double(), None
            if i < n[b]:
                q, x = s["draft"][first + i].double(), tokens[first + i]
                if bool(s["accept"][first + i].double() * q[x] < p[x]):
                    out[b, i] = x
                    continue
                w = torch.where(p > q, p - q, torch.zeros_like(p))
            if w is None or not bool(w.any()):
                w = p
            c = w.cumsum(0)
            at = torch.searchsorted(c, (s["sample"][b].double() * c[-1]).reshape(1), right=True)
            out[b, i], count[b] = int(at.clamp_max(len(c) - 1)), i
            break
    return [out.cuda(), count.cuda()]


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "kv": _exact_kv, "attend": _exact_attend, "verify": _exact_verify}[case["op"]](case, s)
