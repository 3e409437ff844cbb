"""Operators of a state-space language model in its serving form.

A block of such a model is: norm, a dense layer with 4-bit weights that makes gate, channels and
time steps, a short causal convolution over the channels, the selective scan, the gated norm, a
second 4-bit dense layer, and the sum into the residual stream with its norms.  A prompt goes
through all of it at once (thousands of rows), then one token a sequence at a time.

  dense   y[m, j] = act(bias[j] + sum_k x[m, k] * q[j, k] * s[j, k // group]),
          q in -8..7, two codes a byte (low half first, two's complement), s fp16 or bf16
  norm    t = post(y * g) or g * post(y), r' = r + scale * t, n = pre(r'), g = gate, sigmoid(gate)
          or silu(gate), post and pre norms over a row (rms or layer) with fp32 weights
  conv    c[t, ch] = act(b[ch] + sum_w cw[ch, w] * x[t - W + 1 + w, ch]) inside each sequence; the
          last W inputs are kept at their position modulo W for the tokens that follow
  scan    d_t = softplus(dt_t + dt_bias), h_t = exp(d_t a) h_{t-1} + d_t x_t B_t^T,
          y_t = h_t C_t + D x_t, for each head (P x N state; heads share B and C by group)
  step    conv and scan for one token of every sequence, from the kept inputs and state

`own` chooses between the plain form (elementary torch operations in 32 bits, rounded once at
the end) and the calls of this package.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
EPS = 1e-5


def listed():
    return [
        # the smallest call: the 1000-class head of a small net for one image, where launches count
        {"name": "dense_head_1", "op": "dense", "dtype": "f16", "rows": 1, "k": 1280, "n": 1000, "group": 32,
         "scale": "f16", "act": "none"},
        # a large classifier's first dense layer for one image: nothing but reading weights
        {"name": "dense_wide_1", "op": "dense", "dtype": "bf16", "rows": 1, "k": 25088, "n": 4096, "group": 64,
         "scale": "bf16", "act": "relu"},
        # a few tokens at once in fp32, with sizes that fit no tile and a last group that is cut off
        {"name": "dense_odd_7", "op": "dense", "dtype": "f32", "rows": 7, "k": 2050, "n": 1111, "group": 128,
         "scale": "f16", "act": "none"},
        # the input projection of a block for a prompt: the tensor cores count, not the weights
        {"name": "dense_prompt_2048", "op": "dense", "dtype": "bf16", "rows": 2048, "k": 4096, "n": 8448,
         "group": 128, "scale": "bf16", "act": "none"},
        # one token between two blocks: gated, scaled, summed, normed again
        {"name": "norm_token", "op": "norm", "dtype": "f16", "res": "f16", "rows": 1, "dim": 4096, "kind": "rms",
         "gate": "sigmoid", "at": "after", "residual": True, "pre": True, "scale": True, "per_gate": 1},
        # a prompt's rows between two blocks, residual stream in fp32
        {"name": "norm_prompt", "op": "norm", "dtype": "bf16", "res": "f32", "rows": 8190, "dim": 4096,
         "kind": "rms", "gate": "silu", "at": "after", "residual": True, "pre": True, "scale": True,
         "per_gate": 1},
        # the convolution over a long prompt
        {"name": "conv_prompt", "op": "conv", "dtype": "bf16", "lengths": "8192", "channels": 4352, "width": 4,
         "act": "silu"},
        # prompts of uneven length in one batch, an empty one and a single token among them
        {"name": "conv_ragged", "op": "conv", "dtype": "f32", "lengths": "1,0,77,1030,3,200", "channels": 333,
         "width": 3, "act": "silu"},
        # the scan over a long prompt
        {"name": "scan_prompt", "op": "scan", "dtype": "bf16", "lengths": "8192", "heads": 64, "head_dim": 64,
         "groups": 1, "state": 128},
        # prompts of uneven length, odd head and state sizes, two groups
        {"name": "scan_ragged", "op": "scan", "dtype": "f32", "lengths": "1,0,77,1030,3,200", "heads": 6,
         "head_dim": 48, "groups": 2, "state": 40},
        # one token of one sequence
        {"name": "step_1", "op": "step", "dtype": "f16", "batch": 1, "heads": 32, "head_dim": 64, "groups": 1,
         "state": 128, "width": 4},
        # one token of every sequence of a large batch: reading and writing the states
        {"name": "step_128", "op": "step", "dtype": "bf16", "batch": 128, "heads": 64, "head_dim": 64,
         "groups": 1, "state": 128, "width": 4},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _lengths(rng, total):
    n = rng.choice([1, 1, 2, 3, 5, 8])
    return ",".join(str(0 if i and rng.random() < 0.1 else _log_int(rng, 1, max(1, total // n))) for i in range(n))


def draw(rng):
    op = rng.choice(["dense", "dense", "norm", "conv", "scan", "scan", "step"])
    dt = rng.choice(["f32", "f16", "bf16", "bf16"])
    if op == "dense":
        rows = _log_int(rng, 1, 2048)
        k, n = _log_int(rng, 64, 8192), _log_int(rng, 32, 8192)
        return {"op": op, "dtype": dt, "rows": rows, "k": k, "n": n, "group": rng.choice([32, 64, 128]),
                "scale": rng.choice(["f16", "bf16"]), "act": rng.choice(["none", "relu", "hswish"])}
    if op == "norm":
        residual = rng.random() < 0.7
        return {"op": op, "dtype": dt, "res": rng.choice([dt, "f32"]), "rows": _log_int(rng, 1, 8190),
                "dim": _log_int(rng, 32, 4096), "kind": rng.choice(["rms", "layer"]),
                "gate": rng.choice(["none", "linear", "sigmoid", "silu"]), "at": rng.choice(["before", "after"]),
                "residual": residual, "pre": residual, "scale": residual and rng.random() < 0.7,
                "per_gate": rng.choice([1, 1, 7])}
    if op == "conv":
        return {"op": op, "dtype": dt, "lengths": _lengths(rng, 8192 if dt != "f32" else 4096),
                "channels": _log_int(rng, 32, 4352), "width": rng.choice([2, 3, 4, 4]),
                "act": rng.choice(["silu", "none"])}
    groups = rng.choice([1, 1, 2, 4])
    heads = groups * _log_int(rng, 1, 64 // groups)
    p, n = rng.choice([32, 48, 64, 64, 80]), rng.choice([16, 40, 64, 128, 128])
    if op == "scan":
        return {"op": op, "dtype": dt, "lengths": _lengths(rng, 8192 if dt == "bf16" else 2048), "heads": heads,
                "head_dim": min(p, 64), "groups": groups, "state": n}
    return {"op": op, "dtype": dt, "batch": _log_int(rng, 1, 100), "heads": heads, "head_dim": p, "groups": groups,
            "state": n, "width": rng.choice([2, 4, 4])}


# ------------------------------------------------------------------ inputs
def _offsets(case):
    at = [0]
    for n in case["lengths"].split(","):
        at.append(at[-1] + int(n))
    return at


def _ssm_weights(case, rnd):
    """a in -16..-1, time steps of about 1e-3 to 1e-1 and D about 1, as such models are initialised."""
    h, c = case["heads"], case["heads"] * case["head_dim"] + 2 * case["groups"] * case["state"]
    step = torch.exp(rnd(h, uniform=True) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    return {"a": -(1.0 + 15.0 * rnd(h, uniform=True)), "d": 1.0 + 0.1 * rnd(h),
            "dt_bias": step + torch.log(-torch.expm1(-step))}, c


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def rnd(*shape, dt=torch.float32, uniform=False):
        make = torch.rand if uniform else torch.randn
        return make(shape, device="cuda", generator=g).to(dt)

    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "dense":
        n, k, group = case["n"], case["k"], case["group"]
        s["x"] = rnd(case["rows"], k, dt=dt)
        s["codes"] = torch.randint(0, 256, (n, (k + 1) // 2), device="cuda", generator=g, dtype=torch.uint8)
        s["scales"] = ((0.5 + rnd(n, -(-k // group), uniform=True)) * (0.25 / math.sqrt(k))).to(DTYPES[case["scale"]])
        s["bias"] = 0.1 * rnd(n)
        if own:  # the layer's handle: the weights laid out once, when a program loads them
            import paper_2110_06037_gb300 as sn
            s["w"] = sn.Q4Weights(s["codes"], s["scales"], k, group, bias=s["bias"], act=case["act"])
    elif case["op"] == "norm":
        m, d = case["rows"], case["dim"]
        s["y"] = rnd(m, d, dt=dt)
        s["gate"] = rnd(-(-m // case["per_gate"]), d, dt=dt) if case["gate"] != "none" else None
        s["r"] = (3.0 * rnd(m, d)).to(DTYPES[case["res"]]) if case["residual"] else None
        s["post"], s["post_b"] = 1.0 + 0.1 * rnd(d), 0.1 * rnd(d) if case["kind"] == "layer" else None
        s["pre"] = 1.0 + 0.1 * rnd(d) if case["pre"] else None
        s["pre_b"] = 0.1 * rnd(d) if case["pre"] and case["kind"] == "layer" else None
        s["scale"] = 0.1 + 0.02 * rnd(d) if case["scale"] else None
        if own:  # the layer's handle: weights and options
            import paper_2110_06037_gb300 as sn
            s["norm"] = sn.BlockNorm(d, kind=case["kind"], eps=EPS, post=s["post"], post_bias=s["post_b"],
                                     pre=s["pre"], pre_bias=s["pre_b"], scale=s["scale"], gate=case["gate"],
                                     gate_at=case["at"])
    elif case["op"] == "conv":
        at, c, w = _offsets(case), case["channels"], case["width"]
        s["x"] = rnd(at[-1], c, dt=dt)
        s["offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
        s["max_len"] = max(b - a for a, b in zip(at, at[1:]))
        s["conv_w"], s["conv_b"] = rnd(c, w) / math.sqrt(w), 0.1 * rnd(c)
        s["kept"] = torch.zeros(len(at) - 1, w, c, dtype=dt, device="cuda")
    elif case["op"] == "scan":
        at = _offsets(case)
        weights, c = _ssm_weights(case, rnd)
        s.update(weights)
        s["xbc"] = _act(rnd(at[-1], c), "silu").to(dt)  # what the convolution leaves
        s["dt"] = rnd(at[-1], case["heads"], dt=dt)
        s["offsets"] = torch.tensor(at, dtype=torch.int32, device="cuda")
        s["max_len"] = max(b - a for a, b in zip(at, at[1:]))
        s["h1"] = torch.zeros(len(at) - 1, case["heads"], case["head_dim"], case["state"], device="cuda")
        if own:  # the layer's handle: weights and sizes
            import paper_2110_06037_gb300 as sn
            s["ssm"] = sn.StateSpace(case["heads"], case["head_dim"], case["groups"], case["state"], s["a"], s["d"],
                                     s["dt_bias"])
    else:
        weights, c = _ssm_weights(case, rnd)
        s.update(weights)
        b, w = case["batch"], case["width"]
        s["xbc"], s["dt"] = rnd(b, c, dt=dt), rnd(b, case["heads"], dt=dt)
        s["conv_w"], s["conv_b"] = rnd(c, w) / math.sqrt(w), 0.1 * rnd(c)
        s["kept"] = rnd(b, w, c, dt=dt)
        s["pos"] = torch.randint(0, 5000, (b,), device="cuda", generator=g, dtype=torch.int32)
        s["h0"] = 0.3 * rnd(b, case["heads"], case["head_dim"], case["state"])
        s["h1"] = torch.zeros_like(s["h0"])
        if own:  # the layer's handle: weights and sizes
            import paper_2110_06037_gb300 as sn
            s["ssm"] = sn.StateSpace(case["heads"], case["head_dim"], case["groups"], case["state"], s["a"], s["d"],
                                     s["dt_bias"], conv_weight=s["conv_w"], conv_bias=s["conv_b"])
    return s


# ------------------------------------------------------------- plain forms
def _act(v, act):
    if act == "relu":
        return v.clamp_min(0.0)
    if act == "hswish":
        return v * ((v + 3.0).clamp(0.0, 6.0) / 6.0)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "sigmoid":
        return torch.sigmoid(v)
    return v


def _plain_dense(s):
    c = s["case"]
    n, k = c["n"], c["k"]
    low, high = (s["codes"] & 15).to(torch.int32), (s["codes"] >> 4).to(torch.int32)
    q = torch.stack((low, high), dim=2).reshape(n, -1)[:, :k]
    q = (q - 16 * (q > 7)).float()
    w = q * s["scales"].float().repeat_interleave(c["group"], dim=1)[:, :k]
    y = s["x"].float() @ w.t() + s["bias"]
    return _act(y, c["act"]).to(s["x"].dtype)


def _plain_row_norm(v, kind, weight, bias):
    if kind == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    v = v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * weight
    return v if bias is None else v + bias


def _plain_norm(s):
    c = s["case"]
    t = s["y"].float()
    g = None
    if s["gate"] is not None:
        g = _act(s["gate"].float(), c["gate"]).repeat_interleave(c["per_gate"], dim=0)[: c["rows"]]
    if g is not None and c["at"] == "before":
        t = t * g
    t = _plain_row_norm(t, c["kind"], s["post"], s["post_b"])
    if g is not None and c["at"] == "after":
        t = t * g
    if s["scale"] is not None:
        t = t * s["scale"]
    if s["r"] is None:
        return [t.to(s["y"].dtype)]
    r = s["r"].float() + t
    return [r.to(s["r"].dtype), _plain_row_norm(r, c["kind"], s["pre"], s["pre_b"]).to(s["y"].dtype)]


def _padded(v, offsets, max_len):
    """Rows of [tokens, ...] as [sequences, max_len, ...] in 32 bits, zeros behind each end, and which are real."""
    t = torch.arange(max_len, device=v.device)
    real = t[None, :] < (offsets[1:] - offsets[:-1])[:, None]
    at = torch.where(real, offsets[:-1, None].long() + t[None, :], 0)
    return v[at].float() * real.view(*real.shape, *([1] * (v.dim() - 1))), real


def _plain_conv(s):
    c = s["case"]
    w, x = c["width"], s["x"]
    xp, real = _padded(x, s["offsets"], s["max_len"])
    taps = torch.nn.functional.pad(xp, (0, 0, w - 1, 0)).unfold(1, w, 1)
    y = _act((taps * s["conv_w"]).sum(dim=3) + s["conv_b"], c["act"])
    # the last w inputs of every sequence, each at its position modulo w
    n = (s["offsets"][1:] - s["offsets"][:-1]).long()
    last = n[:, None] - 1 - torch.remainder(n[:, None] - 1 - torch.arange(w, device=x.device), w)
    kept = torch.where((last >= 0)[:, :, None],
                       x[(s["offsets"][:-1, None].long() + last).clamp(0, max(0, x.shape[0] - 1))], s["kept"])
    return [y[real].to(x.dtype), kept]


def _decays(a):
    """exp of the sums of a over (s, t] for every t >= s of the last axis, 0 above: [..., t, s]."""
    n = a.shape[-1]
    below = torch.ones(n, n, dtype=torch.bool, device=a.device).tril(-1)
    sums = torch.where(below, a[..., :, None].expand(*a.shape, n), 0.0).cumsum(dim=-2)
    return torch.where(below | torch.eye(n, dtype=torch.bool, device=a.device), torch.exp(sums), 0.0)


def _plain_scan(s, piece=64):
    """In pieces: inside a piece every pair of tokens, between pieces the states."""
    c = s["case"]
    h, p, g, n = c["heads"], c["head_dim"], c["groups"], c["state"]
    v, real = _padded(s["xbc"], s["offsets"], s["max_len"])
    raw, _ = _padded(s["dt"], s["offsets"], s["max_len"])
    d = torch.nn.functional.softplus(raw + s["dt_bias"], threshold=40.0) * real[:, :, None]
    b, tokens = v.shape[:2]
    short = -tokens % piece
    v, d = torch.nn.functional.pad(v, (0, 0, 0, short)), torch.nn.functional.pad(d, (0, 0, 0, short))
    m = v.shape[1] // piece
    x = v[..., : h * p].reshape(b, m, piece, h, p).permute(0, 3, 1, 2, 4)
    bs = v[..., h * p: h * p + g * n].reshape(b, m, piece, g, n).permute(0, 3, 1, 2, 4)
    cs = v[..., h * p + g * n:].reshape(b, m, piece, g, n).permute(0, 3, 1, 2, 4)
    d = d.reshape(b, m, piece, h).permute(0, 3, 1, 2)
    a = d * s["a"][:, None, None]
    pairs = (cs @ bs.transpose(-1, -2)).repeat_interleave(h // g, dim=1)
    bs, cs = bs.repeat_interleave(h // g, dim=1), cs.repeat_interleave(h // g, dim=1)
    xd = x * d[..., None]
    inside = _decays(a)
    y = (pairs * inside) @ xd
    made = (xd * inside[..., -1, :, None]).transpose(-1, -2) @ bs            # what each piece adds to the state
    total = a.sum(dim=-1)
    between = _decays(torch.nn.functional.pad(total, (1, 0)))[..., 1:]       # state before piece i, piece j
    states = (between @ made.reshape(b, h, m, p * n)).reshape(b, h, m + 1, p, n)
    y = y + torch.exp(a.cumsum(dim=-1))[..., None] * (cs @ states[:, :, :m].transpose(-1, -2))
    y = y + s["d"][:, None, None, None] * x
    y = y.permute(0, 2, 3, 1, 4).reshape(b, m * piece, h * p)[:, :tokens]
    return [y[real].to(s["xbc"].dtype), states[:, :, m]]


def _plain_step(s):
    c = s["case"]
    h, p, g, n, w = c["heads"], c["head_dim"], c["groups"], c["state"], c["width"]
    x, b, pos = s["xbc"], c["batch"], s["pos"].long()
    back = torch.arange(w - 1, -1, -1, device=x.device)                       # tokens back of each tap
    at = torch.remainder(pos[:, None] - back, w)
    taps = s["kept"].float().gather(1, at[:, :, None].expand(b, w, x.shape[1]))
    taps = torch.where((back == 0)[None, :, None], x.float()[:, None], taps)
    taps = taps * (pos[:, None] >= back)[:, :, None]
    v = _act((taps * s["conv_w"].t()).sum(dim=1) + s["conv_b"], "silu")
    d = torch.nn.functional.softplus(s["dt"].float() + s["dt_bias"], threshold=40.0)
    xs = v[:, : h * p].reshape(b, h, p)
    bs = v[:, h * p: h * p + g * n].reshape(b, g, n).repeat_interleave(h // g, dim=1)
    cs = v[:, h * p + g * n:].reshape(b, g, n).repeat_interleave(h // g, dim=1)
    h1 = torch.exp(d * s["a"])[:, :, None, None] * s["h0"] + (d[:, :, None] * xs)[..., None] * bs[:, :, None, :]
    y = (h1 * cs[:, :, None, :]).sum(dim=3) + s["d"][:, None] * xs
    kept = torch.where((torch.arange(w, device=x.device)[None] == pos[:, None] % w)[:, :, None], x[:, None], s["kept"])
    return [y.reshape(b, h * p).to(x.dtype), h1, kept]


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"dense": _plain_dense, "norm": _plain_norm, "conv": _plain_conv, "scan": _plain_scan,
                "step": _plain_step}[op](state)
    import paper_2110_06037_gb300 as sn
    if op == "dense":
        return sn.dense_q4(state["x"], state["w"])
    if op == "norm":
        r, n = state["norm"](state["y"], residual=state["r"], gate=state["gate"],
                             rows_per_gate=state["case"]["per_gate"])
        return [r] if n is None else [r, n]
    if op == "conv":
        y = sn.causal_conv(state["x"], state["conv_w"], state["conv_b"], act=state["case"]["act"],
                           offsets=state["offsets"], max_len=state["max_len"], kept=state["kept"])
        return [y, state["kept"]]
    if op == "scan":
        y = state["ssm"].scan(state["xbc"], state["dt"], offsets=state["offsets"], max_len=state["max_len"],
                              state_out=state["h1"])
        return [y, state["h1"]]
    y = state["ssm"].step(state["xbc"], state["dt"], state["kept"], state["h0"], state["pos"], state_out=state["h1"])
    return [y, state["h1"], state["kept"]]


# ------------------------------------------------------------------- work
def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "dense":
        m, n, k = case["rows"], case["n"], case["k"]
        weights = n * (-(-k // 2) + 2 * -(-k // case["group"]) + 4)
        return {"bytes": weights + e * m * (k + n), "flops": 2 * m * n * k}
    if case["op"] == "norm":
        m, d = case["rows"], case["dim"]
        per = e  # y
        per += 2 * SIZE[case["res"]] + e if case["residual"] else e
        gate = -(-m // case["per_gate"]) * d * e if case["gate"] != "none" else 0
        return {"bytes": m * d * per + gate + 4 * d * (1 + case["pre"] + case["scale"]),
                "flops": m * d * (8 + 8 * case["pre"] + 4 * (case["gate"] != "none"))}
    if case["op"] == "conv":
        at, c, w = _offsets(case), case["channels"], case["width"]
        return {"bytes": 2 * e * at[-1] * c + 4 * c * (w + 1) + (len(at) - 1) * w * c * e,
                "flops": at[-1] * c * (2 * w + 5)}
    h, p, g, n = case["heads"], case["head_dim"], case["groups"], case["state"]
    c = h * p + 2 * g * n
    if case["op"] == "scan":
        at = _offsets(case)
        return {"bytes": e * at[-1] * (c + h + h * p) + 4 * (len(at) - 1) * h * p * n + 12 * h,
                "flops": 5 * at[-1] * h * p * n}
    b, w = case["batch"], case["width"]
    return {"bytes": b * (8 * h * p * n + e * (c * (w + 1) + h + h * p)) + 4 * c * (w + 1) + 12 * h,
            "flops": b * (5 * h * p * n + c * (2 * w + 5))}


# ------------------------------------------- the definitions in 64 bits
def _exact_gate(v, act):
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    if act == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-v))
    return v


def _exact_norm(v, kind, weight, bias):
    if kind == "layer":
        v = v - v.sum(1, keepdim=True) / v.shape[1]
    v = v / torch.sqrt((v ** 2).sum(1, keepdim=True) / v.shape[1] + EPS) * weight.double()
    return v + bias.double() if bias is not None else v


def exact(case, seed):
    s = prepare(case, seed)
    x = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    if case["op"] == "dense":
        k = torch.arange(case["k"], device="cuda")
        code = (s["codes"].long()[:, k // 2] >> (4 * (k % 2))) & 15
        table = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, -8, -7, -6, -5, -4, -3, -2, -1], dtype=torch.float64, device="cuda")
        y = torch.mm(x["x"], (table[code] * x["scales"][:, k // case["group"]]).t()) + x["bias"][None]
        if case["act"] == "relu":
            y = torch.where(y > 0, y, torch.zeros_like(y))
        if case["act"] == "hswish":
            y = torch.where(y <= -3, torch.zeros_like(y), torch.where(y >= 3, y, y * (y + 3) / 6))
        return y
    if case["op"] == "norm":
        row = torch.arange(case["rows"], device="cuda") // case["per_gate"]
        g = _exact_gate(x["gate"][row], case["gate"]) if case["gate"] != "none" else 1.0
        before, after = (g, 1.0) if case["at"] == "before" else (1.0, g)
        t = _exact_norm(x["y"] * before, case["kind"], s["post"], s["post_b"]) * after
        t = t * x["scale"] if case["scale"] else t
        if not case["residual"]:
            return [t]
        return [x["r"] + t, _exact_norm(x["r"] + t, case["kind"], s["pre"], s["pre_b"])]
    if case["op"] == "conv":
        at, w = _offsets(case), case["width"]
        y, kept = x["x"] * 0, x["kept"].clone()
        for i, (a, b) in enumerate(zip(at, at[1:])):
            v = x["x"][a:b]
            acc = x["conv_b"] + torch.zeros_like(v)
            for back in range(min(w, b - a)):
                acc[back:] += x["conv_w"][:, w - 1 - back] * v[: b - a - back]
            y[a:b] = _exact_gate(acc, case["act"])
            for t in range(max(0, b - a - w), b - a):
                kept[i, t % w] = v[t]
        return [y, kept]
    h, p, g, n = case["heads"], case["head_dim"], case["groups"], case["state"]
    head = torch.arange(h, device="cuda") // (h // g)

    def parts(v):
        return (v[..., : h * p].reshape(-1, h, p), v[..., h * p: h * p + g * n].reshape(-1, g, n)[:, head],
                v[..., h * p + g * n:].reshape(-1, g, n)[:, head])

    def soft(v):
        return torch.clamp_min(v, 0.0) + torch.log1p(torch.exp(-v.abs()))

    if case["op"] == "scan":
        at = _offsets(case)
        length = [b - a for a, b in zip(at, at[1:])]
        xs, bs, cs = parts(x["xbc"])
        d = soft(x["dt"] + x["dt_bias"])
        y = torch.zeros_like(xs)
        state = torch.zeros(len(length), h, p, n, dtype=torch.float64, device="cuda")
        for t in range(max(length)):  # the t-th token of every sequence that has one
            who = torch.tensor([i for i, m in enumerate(length) if m > t], device="cuda")
            row = torch.tensor([at[i] + t for i, m in enumerate(length) if m > t], device="cuda")
            dx = d[row][:, :, None] * xs[row]
            now = state[who] * torch.exp(d[row] * x["a"])[:, :, None, None] + dx[..., None] * bs[row][:, :, None, :]
            y[row] = torch.einsum("bhpn,bhn->bhp", now, cs[row]) + x["d"][None, :, None] * xs[row]
            state[who] = now
        return [y.reshape(at[-1], h * p), state]
    b, w = case["batch"], case["width"]
    pos = s["pos"].long()
    v, kept = x["conv_b"] + x["conv_w"][:, w - 1] * x["xbc"], x["kept"].clone()
    seq = torch.arange(b, device="cuda")
    for back in range(1, w):
        old = x["kept"][seq, (pos - back) % w] * (pos >= back)[:, None]
        v = v + x["conv_w"][:, w - 1 - back] * old
    kept[seq, pos % w] = x["xbc"]
    xs, bs, cs = parts(_exact_gate(v, "silu"))
    d = soft(x["dt"] + x["dt_bias"])
    h1 = x["h0"] * torch.exp(d * x["a"])[..., None, None] + torch.einsum("bh,bhp,bhn->bhpn", d, xs, bs)
    y = torch.einsum("bhpn,bhn->bhp", h1, cs) + x["d"][None, :, None] * xs
    return [y.reshape(b, h * p), h1, kept]
