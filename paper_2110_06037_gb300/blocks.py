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
for that stream.  They run on the device of their tensors, which is one for all of a
call's tensors and its handle's.  Bad arguments raise SnError with the library's status.

Handles (Q4Weights, BlockNorm, StateSpace) keep their weight tensors alive and hold
nothing else between calls.  The calls themselves go through the native module
_blocks (bind/blocks.cpp), which checks tensors and calls include/sn.h; setting
handles up goes through ctypes.
"""
from __future__ import annotations

import contextlib
import ctypes as C

from . import _sn
from ._sn import SnError, check, lib
from .api import _stream_ptr, _torch

NORM_KINDS = {"rms": 0, "layer": 1}
GATES = {"none": 0, None: 0, "linear": 1, "sigmoid": 2, "silu": 3}
_native = None


def _load():
    """The native module (it needs libsn.so and PyTorch loaded); raises if it was not built."""
    global _native
    if _native is None:
        _torch()
        lib()
        from . import _blocks
        _native = _blocks
    return _native


def _refuse(msg):
    raise SnError(_sn.SN_EINVAL, msg)


def _on(stream):
    """Context in which PyTorch's current stream, whose allocations and launches these are, is `stream`."""
    return contextlib.nullcontext() if stream is None else _torch().cuda.stream(stream)


@contextlib.contextmanager
def _beside(t, stream):
    """The same for a handle's setting up, on the device of `t`."""
    with _torch().cuda.device(t.device if t.is_cuda else None), _on(stream):
        yield


def _device_of(*tensors):
    """Index of the one device that the tensors (None: no tensor) are on, -1 without any."""
    found = sorted({t.get_device() for t in tensors if t is not None})
    if len(found) > 1:
        _refuse(f"a handle's weights are on several devices: {found}")
    return found[0] if found else -1


def _dtype_code(dtype, what):
    torch = _torch()
    code = {torch.float32: _sn.SN_F32, torch.float16: _sn.SN_F16, torch.bfloat16: _sn.SN_BF16}.get(dtype)
    if code is None:
        _refuse(f"{what} must be fp32, fp16 or bf16, not {dtype}")
    return code


def _whole(t, shape, dtype, what):
    """Data pointer of a contiguous CUDA tensor of exactly this shape and type; None for None."""
    if t is None:
        return None
    if t.dtype == dtype and tuple(t.shape) == shape and t.is_cuda and t.is_contiguous():
        return t.data_ptr()
    _refuse(f"{what} must be a contiguous CUDA {dtype} tensor of shape {shape}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def check_device(stream=None):
    """Wait for the stream; raises SnError (SN_ETIMEOUT) if a kernel's bounded wait gave up."""
    check(lib().sn_check_device(_stream_ptr(stream)))


# ------------------------------------------------------------ 4-bit weights
def quantize_q4(w, group=64, scale_dtype=None, stream=None):
    """Symmetric 4-bit codes and scales of a float weight matrix [n, k] by groups of `group`
    neighbours in a row: (codes uint8 [n, (k + 1) // 2], scales [n, ceil(k / group)]).

    scale = max |w| / 7 in scale_dtype (torch.bfloat16 by default, or torch.float16), code = w / scale
    rounded, in -8..7; two codes a byte in two's complement, the lower k in the low half."""
    torch = _torch()
    scale_dtype = scale_dtype or torch.bfloat16
    if w.dim() != 2:
        _refuse("w must be a matrix")
    n, k = w.shape
    if group not in (32, 64, 128):
        _refuse("group must be 32, 64 or 128")
    if scale_dtype not in (torch.float16, torch.bfloat16):
        _refuse("scale_dtype must be torch.float16 or torch.bfloat16")
    dt, ptr = _dtype_code(w.dtype, "w"), _whole(w, (n, k), w.dtype, "w")
    with _beside(w, stream):
        codes = torch.empty((n, (k + 1) // 2), dtype=torch.uint8, device=w.device)
        scales = torch.empty((n, -(-k // group)), dtype=scale_dtype, device=w.device)
        check(lib().sn_q4_quantize(ptr, dt, n, k, group, _dtype_code(scale_dtype, "scales"), codes.data_ptr(), scales.data_ptr(),
                                   _stream_ptr(stream)))
    return codes, scales


class Q4Weights:
    """4-bit weights [n, k] in the kernels' layout: codes and scales as quantize_q4 gives them (of any
    origin), bias fp32 [n] or None, act one of the layer activations ("none", "relu", "relu6", "hswish",
    "hsigmoid").  Building it waits for `stream`; after that it serves any stream."""

    def __init__(self, codes, scales, k, group, bias=None, act="none", stream=None):
        torch = _torch()
        if codes.dim() != 2:
            _refuse("codes must be [n, (k + 1) // 2]")
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
        self.device = _device_of(codes, scales, bias)
        with _beside(codes, stream):
            self.packed = torch.empty((nbytes.value,), dtype=torch.uint8, device=codes.device)
            self.bias, self.n, self.k, self.group, self.act = bias, n, k, group, act
            self._c = _sn.sn_q4_weights(n, k, group, _dtype_code(scales.dtype, "scales"), _sn.SN_ACT[act], self.packed.data_ptr(), bp)
            self._at = C.addressof(self._c)
            check(lib().sn_q4_pack(cp, sp, C.byref(self._c), _stream_ptr(stream)))
        self._dense = _load().dense_q4


def dense_q4(x, w, out=None, stream=None):
    """y = act(x W^T + bias) with 4-bit weights: x [..., k] -> [..., n] of x's type, for any number of rows."""
    if stream is None:
        return w._dense(w._at, w.device, x, out)
    with _on(stream):
        return w._dense(w._at, w.device, x, out)


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
        self.dim = int(dim)
        self.weights = (post, post_bias, pre, pre_bias, scale)
        f32 = _torch().float32
        ptrs = [_whole(t, (self.dim,), f32, what)
                for t, what in zip(self.weights, ("post", "post_bias", "pre", "pre_bias", "scale"))]
        self.device = _device_of(*self.weights)
        self._c = _sn.sn_norm_params(self.dim, NORM_KINDS[kind], GATES[gate], int(gate_at == "after"), eps, *ptrs)
        self._at = C.addressof(self._c)
        self._norm = _load().block_norm

    def __call__(self, y=None, residual=None, gate=None, rows_per_gate=1, out=None, out_normed=None, dtype=None, stream=None):
        """(total, normed): total in the residual's type (y's without one), normed in y's type, or None
        without pre weights.  y None: total is the residual itself (a block's first norm), and normed has
        the type `dtype` (default: the residual's).  out may be residual or y, out_normed may be y."""
        if stream is None:
            return self._norm(self._at, self.device, y, residual, gate, rows_per_gate, out, out_normed, dtype)
        with _on(stream):
            return self._norm(self._at, self.device, y, residual, gate, rows_per_gate, out, out_normed, dtype)


# --------------------------------------------------- convolution and scan
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
    conv = (_native or _load()).causal_conv
    if stream is None:
        return conv(x, weight, bias, act == "silu", offsets, max_len, kept, slots, pos, out)
    with _on(stream):
        return conv(x, weight, bias, act == "silu", offsets, max_len, kept, slots, pos, out)


class StateSpace:
    """The selective scan of one layer: heads x head_dim channels, B and C of `state` values in `groups`
    groups of heads; a, d, dt_bias fp32 [heads] (d, dt_bias may be None).  conv_weight [channels, width]
    and conv_bias [channels] are those of the layer's convolution, for step."""

    def __init__(self, heads, head_dim, groups, state, a, d=None, dt_bias=None, conv_weight=None, conv_bias=None):
        self.heads, self.head_dim, self.groups, self.state = int(heads), int(head_dim), int(groups), int(state)
        self.inner, self.channels = self.heads * self.head_dim, self.heads * self.head_dim + 2 * self.groups * self.state
        f32 = _torch().float32
        if conv_weight is not None and conv_weight.dim() != 2:
            _refuse("conv_weight must be [channels, width]")
        self.width = int(conv_weight.shape[1]) if conv_weight is not None else 0
        self.weights = (a, d, dt_bias, conv_weight, conv_bias)
        if a is None:
            _refuse("a is needed")
        self._c = _sn.sn_ssm_params(
            self.heads, self.head_dim, self.groups, self.state, self.width, _whole(a, (self.heads,), f32, "a"),
            _whole(d, (self.heads,), f32, "d"), _whole(dt_bias, (self.heads,), f32, "dt_bias"),
            _whole(conv_weight, (self.channels, self.width), f32, "conv_weight"),
            _whole(conv_bias, (self.channels,), f32, "conv_bias"))
        self.device = _device_of(*self.weights)
        self._at = C.addressof(self._c)
        self._scan, self._step = _load().scan, _load().step

    def scan(self, xbc, dt, offsets=None, max_len=None, state_in=None, state_out=None, slots=None, out=None,
             stream=None):
        """y of every token of every sequence: xbc (the convolution's output) [batch, tokens, channels] or
        [tokens, channels] with offsets and max_len, dt [..., heads] of the same type.  States are fp32
        [entries, heads, head_dim, state]; state_in None: from zero; state_out (which may be state_in)
        receives the last ones."""
        if stream is None:
            return self._scan(self._at, self.device, xbc, dt, offsets, max_len, state_in, state_out, slots, out)
        with _on(stream):
            return self._scan(self._at, self.device, xbc, dt, offsets, max_len, state_in, state_out, slots, out)

    def step(self, xbc, dt, kept, state, pos, state_out=None, slots=None, out=None, stream=None):
        """One token of every sequence: xbc [batch, channels] before the convolution, dt [batch, heads],
        pos int32 [batch] (tokens that each sequence has had).  kept (as in causal_conv) is brought up to
        date in place, and so is state unless state_out is given."""
        if stream is None:
            return self._step(self._at, self.device, xbc, dt, kept, state, pos, state_out, slots, out)
        with _on(stream):
            return self._step(self._at, self.device, xbc, dt, kept, state, pos, state_out, slots, out)
