"""Operators of a state-space language model's block: Python front end over the C ABI.

    w = Q4Weights(codes, scales, k, group)       # 4-bit weights, laid out once
    y = dense_q4(x, w)                           # one row to a prompt's rows
    norm = BlockNorm(dim, post=..., pre=..., scale=..., gate="silu")
    r, n = norm(y, residual=r, gate=z)
    c = causal_conv(xbc, weight, bias, kept=kept)
    ssm = StateSpace(heads, head_dim, groups, state, a, d, dt_bias, conv_weight, conv_bias)
    y = ssm.scan(c, dt, state_out=state)         # a prompt
    y = ssm.step(xbc, dt, kept, state, pos)      # the tokens that follow, one at a time

Tensors are CUDA tensors of fp32, fp16 or bf16; rows may lie apart (a slice of a
wider projection), the values of a row are contiguous.  Weights of norms,
convolutions and scans and all states are fp32.  Calls run on `stream` (default:
PyTorch's current one) and return without waiting; what they allocate is allocated
for that stream.  Bad arguments raise SnError with the library's status.

Handles (Q4Weights, BlockNorm, StateSpace) keep their weight tensors alive and hold
nothing else between calls.
"""
from __future__ import annotations

import ctypes as C

from . import _sn
from ._sn import SnError, check, lib
from .api import _stream_ptr, _torch

NORM_KINDS = {"rms": 0, "layer": 1}
GATES = {"none": 0, None: 0, "linear": 1, "sigmoid": 2, "silu": 3}
_dtypes = {}  # torch dtype -> sn_dtype, filled on first use (the import of torch is not this module's)
_torch_mod = None

# A call's own work on the GPU can be a few microseconds, as much as marshalling it on
# the host: the usual case (rows in two axes, the current stream) goes straight through.


def _setup():
    global _torch_mod
    _torch_mod = _torch()
    _dtypes.update({_torch_mod.float32: _sn.SN_F32, _torch_mod.float16: _sn.SN_F16, _torch_mod.bfloat16: _sn.SN_BF16})
    return _torch_mod


def _dtype_map():
    if not _dtypes:
        _setup()
    return _dtypes


def _stream(stream, device):
    """Handle of the stream, or of the device's current one."""
    if stream is not None:
        return stream.cuda_stream
    raw = getattr(_torch_mod._C, "_cuda_getCurrentRawStream", None)
    return raw(device) if raw is not None else _stream_ptr(None)


def _refuse(msg):
    raise SnError(_sn.SN_EINVAL, msg)


def _dt(t, what):
    code = (_dtypes or _dtype_map()).get(t.dtype)
    if code is None:
        _refuse(f"{what} must be fp32, fp16 or bf16, not {t.dtype}")
    return code


def _rows(t, width, what, like=None):
    """(data pointer, row stride, rows) of a tensor [..., width] whose leading axes collapse to rows."""
    shape = t.shape
    if len(shape) == 2 and shape[1] == width and t.is_cuda and (like is None or t.dtype is like):
        s0, s1 = t.stride()
        if s1 == 1:
            rows = shape[0]
            return t.data_ptr(), (s0 if rows > 1 or s0 > width else width), rows
    return _any_rows(t, width, what, like)


def _any_rows(t, width, what, like):
    if not t.is_cuda:
        _refuse(f"{what} must be a CUDA tensor")
    if like is not None and t.dtype != like:
        _refuse(f"{what} must be {like}, not {t.dtype}")
    shape = t.shape
    if len(shape) == 0 or shape[-1] != width:
        _refuse(f"{what} must have rows of {width}, not shape {tuple(shape)}")
    if len(shape) != 2:
        if len(shape) == 1:
            t = t[None]
        elif len(shape) > 2:
            try:
                t = t.view(-1, width) if t.numel() else t.reshape(0, width)
            except RuntimeError:
                _refuse(f"the leading axes of {what} do not collapse to evenly spaced rows (strides {t.stride()})")
        shape = t.shape
    s0, s1 = t.stride()
    rows = shape[0]
    if s1 != 1 and width > 1:
        _refuse(f"the values of a row of {what} must be contiguous")
    if rows <= 1:
        s0 = max(s0, width)
    return t.data_ptr(), s0, rows


def _whole(t, shape, dtype, what):
    """Data pointer of a contiguous CUDA tensor of exactly this shape and type; 0 for None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    _refuse(f"{what} must be a contiguous CUDA {dtype} tensor of shape {tuple(shape)}, not {t.dtype} {tuple(t.shape)} "
            f"on {t.device}")


def _index(t, n, what):
    return None if t is None else _whole(t, (n,), _torch_mod.int32, what)


def _new(shape, dtype, device, stream):
    if stream is None:
        return _torch_mod.empty(shape, dtype=dtype, device=device)
    with _torch_mod.cuda.stream(stream):
        return _torch_mod.empty(shape, dtype=dtype, device=device)


def _out(out, shape, width, dtype, like, stream, what):
    """(tensor, data pointer, row stride) of an output, allocated where none is given."""
    if out is None:
        out = _new(shape, dtype, like.device, stream)
        return out, out.data_ptr(), width
    if tuple(out.shape) != tuple(shape) or out.dtype != dtype:
        _refuse(f"{what} must be {dtype} of shape {tuple(shape)}")
    return out, *_rows(out, width, what)[:2]


def _scratch(call, device, stream):
    """A buffer of the bytes that `call` names (through its last argument), or None."""
    n = C.c_int64()
    check(call(n))
    return _new((n.value,), _torch_mod.uint8, device, stream) if n.value else None


def check_device(stream=None):
    """Wait for the stream; raises SnError (SN_ETIMEOUT) if a kernel's bounded wait gave up."""
    check(lib().sn_check_device(_stream_ptr(stream)))


# ------------------------------------------------------------ 4-bit weights
def quantize_q4(w, group=64, scale_dtype=None, stream=None):
    """Symmetric 4-bit codes and scales of a float weight matrix [n, k] by groups of `group`
    neighbours in a row: (codes uint8 [n, (k + 1) // 2], scales [n, ceil(k / group)]).

    scale = max |w| / 7 in scale_dtype (torch.bfloat16 by default, or torch.float16), code = w / scale
    rounded, in -8..7; two codes a byte in two's complement, the lower k in the low half."""
    torch = _setup()
    scale_dtype = scale_dtype or torch.bfloat16
    if w.dim() != 2:
        _refuse("w must be a matrix")
    n, k = w.shape
    if group not in (32, 64, 128):
        _refuse("group must be 32, 64 or 128")
    if scale_dtype not in (torch.float16, torch.bfloat16):
        _refuse("scale_dtype must be torch.float16 or torch.bfloat16")
    dt, ptr = _dt(w, "w"), _whole(w, (n, k), w.dtype, "w")
    codes = _new((n, (k + 1) // 2), torch.uint8, w.device, stream)
    scales = _new((n, -(-k // group)), scale_dtype, w.device, stream)
    check(lib().sn_q4_quantize(ptr, dt, n, k, group, _dtype_map()[scale_dtype], codes.data_ptr(), scales.data_ptr(),
                               _stream(stream, w.get_device())))
    return codes, scales


class Q4Weights:
    """4-bit weights [n, k] in the kernels' layout: codes and scales as quantize_q4 gives them (of any
    origin), bias fp32 [n] or None, act one of the layer activations ("none", "relu", "relu6", "hswish",
    "hsigmoid").  Building it waits for `stream`; after that it serves any stream."""

    def __init__(self, codes, scales, k, group, bias=None, act="none", stream=None):
        torch = _setup()
        n, k, group = int(codes.shape[0]), int(k), int(group)
        if act not in _sn.SN_ACT:
            _refuse(f"unknown act {act!r}")
        if scales.dtype not in (torch.float16, torch.bfloat16):
            _refuse(f"scales must be fp16 or bf16, not {scales.dtype}")
        nbytes = C.c_int64()
        check(lib().sn_q4_bytes(n, k, group, C.byref(nbytes)))
        cp = _whole(codes, (n, (k + 1) // 2), torch.uint8, "codes")
        sp = _whole(scales, (n, -(-k // group)), scales.dtype, "scales")
        bp = _whole(bias, (n,), torch.float32, "bias")
        self.packed = _new((nbytes.value,), torch.uint8, codes.device, stream)
        self.bias, self.n, self.k, self.group, self.act = bias, n, k, group, act
        self._c = _sn.sn_q4_weights(n, k, group, _dtype_map()[scales.dtype], _sn.SN_ACT[act], self.packed.data_ptr(), bp)
        self._ref = C.byref(self._c)
        check(lib().sn_q4_pack(cp, sp, self._ref, _stream(stream, codes.get_device())))
        self._call, self._want = lib().sn_q4_dense, lib().sn_q4_workspace


def dense_q4(x, w, out=None, stream=None):
    """y = act(x W^T + bias) with 4-bit weights: x [..., k] -> [..., n] of x's type, for any number of rows."""
    dt = _dt(x, "x")
    ptr, ld, rows = _rows(x, w.k, "x")
    shape = x.shape
    out, optr, old = _out(out, (rows, w.n) if len(shape) == 2 else (*shape[:-1], w.n), w.n, x.dtype, x, stream, "out")
    work = None
    if rows > 8:  # (fewer never need scratch)
        work = _scratch(lambda n: w._want(w._ref, dt, rows, ptr, ld, C.byref(n)), x.device, stream)
    rc = w._call(w._ref, dt, rows, ptr, ld, optr, old, None if work is None else work.data_ptr(),
                 0 if work is None else work.numel(), _stream(stream, x.get_device()))
    if rc:
        check(rc)
    return out


# ------------------------------------------------------------------- norms
class BlockNorm:
    """The norms behind and before a block, with the block's gate, residual scale and sum:

        t = post(y * g) (gate_at "before") or g * post(y) ("after")
        total = residual + scale * t,   normed = pre(total)

    kind "rms" or "layer"; post, pre: fp32 weights [dim] or None (no such norm); scale: fp32 [dim] or
    None; gate "none", "linear", "sigmoid" or "silu" says what is done to the gate tensor."""

    def __init__(self, dim, kind="rms", eps=1e-5, post=None, post_bias=None, pre=None, pre_bias=None, scale=None,
                 gate="none", gate_at="after"):
        if kind not in NORM_KINDS or gate not in GATES or gate_at not in ("before", "after"):
            _refuse(f"unknown kind {kind!r}, gate {gate!r} or gate_at {gate_at!r}")
        self.dim, self.has_pre = int(dim), pre is not None
        self.weights = (post, post_bias, pre, pre_bias, scale)
        f32 = _setup().float32
        ptrs = [_whole(t, (self.dim,), f32, what)
                for t, what in zip(self.weights, ("post", "post_bias", "pre", "pre_bias", "scale"))]
        self._c = _sn.sn_norm_params(self.dim, NORM_KINDS[kind], GATES[gate], int(gate_at == "after"), eps, *ptrs)
        self._ref, self._call = C.byref(self._c), lib().sn_block_norm

    def __call__(self, y=None, residual=None, gate=None, rows_per_gate=1, out=None, out_normed=None, dtype=None, stream=None):
        """(total, normed): total in the residual's type (y's without one), normed in y's type, or None
        without pre weights.  y None: total is the residual itself (a block's first norm), and normed has
        the type `dtype` (default: the residual's).  out may be residual or y, out_normed may be y."""
        first = y if y is not None else residual
        if first is None:
            _refuse("neither y nor residual")
        dtype = first.dtype if y is not None or dtype is None else dtype
        dt, d = (_dtypes or _dtype_map()).get(dtype), self.dim
        if dt is None:
            _refuse(f"rows must be fp32, fp16 or bf16, not {dtype}")
        yp = rp = gp = total = sp = normed = np_ = None
        ldy = ldr = ldg = lds = ldn = 0
        sdt, rdt = dtype, dt
        if y is not None:
            yp, ldy, rows = _rows(y, d, "y")
        if residual is not None:
            sdt = residual.dtype
            rdt = _dt(residual, "residual")
            rp, ldr, n = _rows(residual, d, "residual")
            if y is not None and n != rows:
                _refuse("residual and y have different rows")
            rows = n
        if gate is not None:
            gp, ldg, n = _rows(gate, d, "gate", dtype)
            if rows_per_gate < 1 or n * rows_per_gate < rows:
                _refuse("too few gate rows")
        if y is not None or out is not None:
            total, sp, lds = _out(out, first.shape, d, sdt, first, stream, "out")
        if self.has_pre:
            normed, np_, ldn = _out(out_normed, first.shape, d, dtype, first, stream, "out_normed")
        rc = self._call(self._ref, dt, rows, yp, ldy, gp, ldg, rows_per_gate, rdt, rp, ldr, sp, lds, np_, ldn,
                        _stream(stream, first.get_device()))
        if rc:
            check(rc)
        return (residual if total is None else total), normed


# --------------------------------------------------- convolution and scan
def _sequences(t, offsets, max_len):
    """(tokens, batch, max_len, offsets pointer) of [batch, len, c], or of [tokens, c] with offsets."""
    if offsets is None:
        if t.dim() != 3:
            _refuse("without offsets the input is [batch, tokens, channels]")
        return t.shape[0] * t.shape[1], t.shape[0], t.shape[1], None
    if t.dim() != 2 or max_len is None:
        _refuse("with offsets the input is [tokens, channels], and max_len is needed")
    n = offsets.numel() - 1
    if n < 0:
        _refuse("offsets are empty")
    return t.shape[0], n, min(int(max_len), t.shape[0]), _index(offsets, n + 1, "offsets")


def causal_conv(x, weight, bias=None, act="silu", offsets=None, max_len=None, kept=None, slots=None, pos=None, out=None,
                stream=None):
    """Causal convolution of every channel along its sequence's tokens.

    x [batch, tokens, c], or [tokens, c] with offsets (int32 [batch + 1] on the device) and max_len (at
    least the longest sequence); weight fp32 [c, width], width up to 8; act "silu" or "none".  kept
    [entries, width, c] holds a sequence's last inputs (position i at i % width): with pos (int32
    [batch], the position of each sequence's first token here) the convolution goes on from it, and it
    is brought up to date in place.  slots (int32 [batch]): the entry of each sequence (default: its
    index; -1: none)."""
    if act not in ("silu", "none", None):
        _refuse(f"unknown act {act!r}")
    f32 = (_torch_mod or _setup()).float32
    if weight.dim() != 2:
        _refuse("weight must be [channels, width]")
    c, width = weight.shape
    dt = _dt(x, "x")
    tokens, batch, max_len, op = _sequences(x, offsets, max_len)
    xp, ldx, _ = _rows(x, c, "x")
    out, yp, ldy = _out(out, x.shape, c, x.dtype, x, stream, "out")
    kp, n = None, batch
    if kept is not None:
        n = kept.shape[0]
        kp = _whole(kept, (n, width, c), x.dtype, "kept")
    if kept is not None and slots is None and n < batch:
        _refuse("kept has fewer entries than there are sequences")
    rc = lib().sn_causal_conv(dt, c, width, int(act == "silu"), _whole(weight, (c, width), f32, "weight"),
                              _whole(bias, (c,), f32, "bias"), tokens, batch, max_len, op, xp, ldx, yp, ldy, kp, n,
                              _index(slots, batch, "slots"), _index(pos, batch, "pos"), _stream(stream, x.get_device()))
    if rc:
        check(rc)
    return out


class StateSpace:
    """The selective scan of one layer: heads x head_dim channels, B and C of `state` values in `groups`
    groups of heads; a, d, dt_bias fp32 [heads] (d, dt_bias may be None).  conv_weight [channels, width]
    and conv_bias [channels] are those of the layer's convolution, for step."""

    def __init__(self, heads, head_dim, groups, state, a, d=None, dt_bias=None, conv_weight=None, conv_bias=None):
        self.heads, self.head_dim, self.groups, self.state = int(heads), int(head_dim), int(groups), int(state)
        self.inner, self.channels = self.heads * self.head_dim, self.heads * self.head_dim + 2 * self.groups * self.state
        f32 = _setup().float32
        self.width = int(conv_weight.shape[1]) if conv_weight is not None else 0
        self.weights = (a, d, dt_bias, conv_weight, conv_bias)
        if a is None:
            _refuse("a is needed")
        self._c = _sn.sn_ssm_params(
            self.heads, self.head_dim, self.groups, self.state, self.width, _whole(a, (self.heads,), f32, "a"),
            _whole(d, (self.heads,), f32, "d"), _whole(dt_bias, (self.heads,), f32, "dt_bias"),
            _whole(conv_weight, (self.channels, self.width), f32, "conv_weight"),
            _whole(conv_bias, (self.channels,), f32, "conv_bias"))
        self._ref, self._scan, self._step = C.byref(self._c), lib().sn_ssm_scan, lib().sn_ssm_step

    def _states(self, state_in, state_out, batch, slots):
        n, ptrs = batch, []
        for t, what in ((state_in, "state_in"), (state_out, "state_out")):
            if t is not None:
                n = t.shape[0]
            ptrs.append(_whole(t, (n, self.heads, self.head_dim, self.state), _torch_mod.float32, what))
        if state_in is not None and state_out is not None and state_in.shape[0] != state_out.shape[0]:
            _refuse("state_in and state_out have different entries")
        if slots is None and n < batch:
            _refuse("fewer states than sequences")
        return n, ptrs[0], ptrs[1]

    def scan(self, xbc, dt, offsets=None, max_len=None, state_in=None, state_out=None, slots=None, out=None,
             stream=None):
        """y of every token of every sequence: xbc (the convolution's output) [batch, tokens, channels] or
        [tokens, channels] with offsets and max_len, dt [..., heads] of the same type.  States are fp32
        [entries, heads, head_dim, state]; state_in None: from zero; state_out (which may be state_in)
        receives the last ones."""
        code = _dt(xbc, "xbc")
        tokens, batch, max_len, op = _sequences(xbc, offsets, max_len)
        xp, ldx, _ = _rows(xbc, self.channels, "xbc")
        dp, ldd, n = _rows(dt, self.heads, "dt", like=xbc.dtype)
        if n != tokens:
            _refuse("dt and xbc have different tokens")
        n, si, so = self._states(state_in, state_out, batch, slots)
        out, yp, ldy = _out(out, (*xbc.shape[:-1], self.inner), self.inner, xbc.dtype, xbc, stream, "out")
        work = _scratch(lambda b: lib().sn_ssm_workspace(self._ref, code, tokens, batch, max_len, C.byref(b)), xbc.device,
                        stream)
        rc = self._scan(self._ref, code, tokens, batch, max_len, op, xp, ldx, dp, ldd, si, so, n,
                        _index(slots, batch, "slots"), yp, ldy, None if work is None else work.data_ptr(),
                        0 if work is None else work.numel(), _stream(stream, xbc.get_device()))
        if rc:
            check(rc)
        return out

    def step(self, xbc, dt, kept, state, pos, state_out=None, slots=None, out=None, stream=None):
        """One token of every sequence: xbc [batch, channels] before the convolution, dt [batch, heads],
        pos int32 [batch] (tokens that each sequence has had).  kept (as in causal_conv) is brought up to
        date in place, and so is state unless state_out is given."""
        code = _dt(xbc, "xbc")
        xp, ldx, batch = _rows(xbc, self.channels, "xbc")
        dp, ldd, n = _rows(dt, self.heads, "dt", like=xbc.dtype)
        if n != batch:
            _refuse("dt and xbc have different rows")
        if state_out is None:
            state_out = state
        n, si, so = self._states(state, state_out, batch, slots)
        if kept.shape[0] != n:
            _refuse("kept and the states have different entries")
        kp = _whole(kept, (n, self.width, self.channels), xbc.dtype, "kept")
        shape = xbc.shape
        out, yp, ldy = _out(out, (batch, self.inner) if len(shape) == 2 else (*shape[:-1], self.inner), self.inner,
                            xbc.dtype, xbc, stream, "out")
        rc = self._step(self._ref, code, batch, xp, ldx, dp, ldd, kp, si, so, n, _index(slots, batch, "slots"),
                        _index(pos, batch, "pos"), yp, ldy, _stream(stream, xbc.get_device()))
        if rc:
            check(rc)
        return out
