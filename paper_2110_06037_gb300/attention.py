"""Operators of an attention layer in its serving form, as such layers stand between state-space blocks:
Python front end over the C ABI.

    rope = HeadRope(dim, frequencies, norm="rms", q_weight=qw, k_weight=kw)
    q, k = rope(q, k, pos)                        # norms of the heads and rotation, one pass
    cache = KVCache(*KVCache.empty(pages, heads, page, dim, torch.bfloat16, codes=True))
    cache.write(k, v, table, offsets=offsets, max_len=n, pos=pos)
    y = cache.attend(q, table, offsets=offsets, max_len=n, pos=pos, max_context=longest)
    tokens, accepted = verify_draft(target, draft, drafted, accept, sample)

Tensors, streams, devices and errors are as in blocks.py.  Heads of a token and tokens may lie apart
(slices of a wider projection, or heads before tokens); the values of a head are contiguous.
"""
from __future__ import annotations

import ctypes as C

from . import _sn, blocks
from ._sn import check, lib
from .api import _torch
from .blocks import _device_of, _dtype_code, _load, _on, _refuse, _whole

HEAD_NORMS = {"rms": 0, "layer": 1, "none": 2, None: 2}


class HeadRope:
    """Norm of every head of queries and keys, and the rotation of pairs of its values by its position.

    dim: values of a head (even, up to 256).  frequencies: radians a position of each pair, up to dim / 2
    of them (fewer leave the last values as they are).  norm "rms", "layer" or "none", with fp32 weights [dim]
    or None.  Pairs are values i and i + len(frequencies), or 2 i and 2 i + 1 (interleaved).  axes: the
    position axis of each pair (default: axis 0 for all).  Setting it up waits for `stream`; after that it
    serves any stream."""

    def __init__(self, dim, frequencies, norm="rms", eps=1e-6, q_weight=None, k_weight=None, interleaved=False, axes=None,
                 device=None, stream=None):
        torch = _torch()
        self.dim = int(dim)
        f = [float(v) for v in frequencies]
        if norm not in HEAD_NORMS:
            _refuse(f"unknown norm {norm!r}")
        a = None if axes is None else [int(v) for v in axes]
        if a is not None and (len(a) != len(f) or any(v < 0 or v > 65535 for v in a)):
            _refuse("axes must name an axis of each pair")
        if self.dim < 2 or self.dim % 2 or len(f) > self.dim // 2:
            _refuse("dim must be even and have at least two values a frequency")
        if HEAD_NORMS[norm] == 2 and (q_weight is not None or k_weight is not None):
            _refuse("weights without a norm")
        n = len(f)
        host = (C.c_double * n)(*f)
        turns = (C.c_uint64 * n)()
        check(lib().sn_rope_turns(host, n, turns))
        qp, kp = (_whole(t, (self.dim,), torch.float32, what) for t, what in ((q_weight, "q_weight"), (k_weight, "k_weight")))
        self.weights = (q_weight, k_weight)
        self.device = _device_of(*self.weights)
        if device is None:
            device = torch.device("cuda", self.device if self.device >= 0 else torch.cuda.current_device())
        device = torch.device(device)
        if device.type != "cuda":
            _refuse(f"device must be a CUDA device, not {device}")
        at = device.index if device.index is not None else torch.cuda.current_device()
        if self.device not in (-1, at):
            _refuse(f"the weights are on device {self.device}, not {at}")
        self.device = at
        signed = [t - (1 << 64) if t >> 63 else t for t in turns]
        with torch.cuda.device(at), _on(stream):
            self.turns = torch.tensor(signed, dtype=torch.int64, device="cuda")
            self.axis = None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")
            torch.cuda.current_stream().synchronize()
        self.axes = max(a) + 1 if a else 1
        self._c = _sn.sn_rope_params(self.dim, n, self.axes, HEAD_NORMS[norm], int(bool(interleaved)), eps,
                                     self.turns.data_ptr() if n else None, self.axis.data_ptr() if a else None, qp, kp)
        self._at = C.addressof(self._c)
        self._rope = _load().head_rope

    def __call__(self, q=None, k=None, pos=None, q_out=None, k_out=None, stream=None):
        """(q, k) normalised and rotated: q [..., q_heads, dim], k [..., k_heads, dim] of the same tokens and
        type, either None; pos int32, a position of each token, or [..., axes].  q_out may be q, k_out may be k."""
        if stream is None:
            return self._rope(self._at, self.device, q, k, pos, q_out, k_out)
        with _on(stream):
            return self._rope(self._at, self.device, q, k, pos, q_out, k_out)


class KVCache:
    """Paged cache of one layer's keys and values.

    k, v: [pages, heads, page, dim], contiguous, fp32, fp16 or bf16, or int8 codes with fp32 scales
    [pages, heads, page]; page 16, 32, 64, 128 or 256, dim a multiple of 16 up to 256.  The handle keeps the tensors
    and nothing else.  Its calls take the pages of each sequence, table int32 [entries, pages a sequence] (position p is in
    page table[entry, p // page]; a page outside the cache is none), pos int32 [batch] (the position of each sequence's
    first token here; None: 0), and slots int32 [batch] (the entry of each sequence; default: its index, -1: none).
    Tokens are [batch, tokens, heads, dim], or [tokens, heads, dim] with offsets (int32 [batch + 1]) and max_len
    (at least the longest sequence)."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        torch = _torch()
        if k.dim() != 4:
            _refuse("k must be [pages, heads, page, dim]")
        self.pages, self.heads, self.page, self.dim = (int(n) for n in k.shape)
        if any(n > 0x7fffffff for n in k.shape):
            _refuse("k is too large")
        self.codes = k.dtype == torch.int8
        dtype = _sn.SN_QI8 if self.codes else _dtype_code(k.dtype, "k and v")
        shape = tuple(k.shape)
        if self.codes and (k_scale is None or v_scale is None):
            _refuse("codes need k_scale and v_scale")
        if not self.codes and (k_scale is not None or v_scale is not None):
            _refuse("scales go with int8 codes")
        self.tensors = (k, v, k_scale, v_scale)
        ptrs = [_whole(k, shape, k.dtype, "k"), _whole(v, shape, k.dtype, "v")]
        ptrs += [_whole(t, shape[:3], torch.float32, what) for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale"))]
        self.device = _device_of(*self.tensors)
        self._c = _sn.sn_kv_cache(dtype, self.pages, self.heads, self.page, self.dim, *ptrs)
        self._at = C.addressof(self._c)
        nbytes = C.c_int64()  # (every check of the cache itself)
        check(lib().sn_attend_workspace(self._at, _sn.SN_F32 if self.codes else dtype, self.heads, 0, 0, 0, 0, C.byref(nbytes)))
        native = _load()
        self._write, self._read, self._attend = native.kv_write, native.kv_read, native.attend

    @staticmethod
    def empty(pages, heads, page, dim, dtype=None, codes=False, device="cuda"):
        """(k, v, k_scale, v_scale) of an empty cache: of `dtype` (scales None), or of codes."""
        torch = _torch()
        kv = [torch.zeros(pages, heads, page, dim, dtype=torch.int8 if codes else dtype, device=device) for _ in range(2)]
        return (*kv, *([torch.ones(pages, heads, page, device=device) for _ in range(2)] if codes else (None, None)))

    def write(self, k, v, table, offsets=None, max_len=None, pos=None, slots=None, stream=None):
        """Store the tokens' keys and values (of the cache's type, or of any type as codes)."""
        if stream is None:
            return self._write(self._at, self.device, k, v, table, offsets, max_len, pos, slots)
        with _on(stream):
            return self._write(self._at, self.device, k, v, table, offsets, max_len, pos, slots)

    def read(self, table, offsets=None, max_len=None, pos=None, tokens=None, dtype=None, slots=None, k_out=None, v_out=None,
             stream=None):
        """(k, v) of the sequences' positions from pos on: max_len of each, or with offsets those of `tokens`
        token rows.  dtype: that of the result, for codes.  Positions without a page read as zeros."""
        if stream is None:
            return self._read(self._at, self.device, table, offsets, max_len, pos, tokens, dtype, slots, k_out, v_out)
        with _on(stream):
            return self._read(self._at, self.device, table, offsets, max_len, pos, tokens, dtype, slots, k_out, v_out)

    def attend(self, q, table, offsets=None, max_len=None, pos=None, max_context=None, scale=None, slots=None, out=None,
               stream=None):
        """Attention of the tokens' queries [..., q_heads, dim] over the keys of their sequences up to their own
        position (written before).  q_heads is a multiple of the cache's heads, in that order.  max_context: at least every
        sequence's pos + length (default: all that the table has room for).  scale: default 1 / sqrt(dim).  A result that is
        not finite is computed again in fp32, which is slow."""
        if stream is None:
            return self._attend(self._at, self.device, q, table, offsets, max_len, pos, max_context, scale, slots, out)
        with _on(stream):
            return self._attend(self._at, self.device, q, table, offsets, max_len, pos, max_context, scale, slots, out)


def verify_draft(target, draft, tokens, accept, sample, offsets=None, max_len=None, out=None, count=None, stream=None):
    """(tokens int32 [batch, max_len + 1], accepted int32 [batch]) of drafted tokens.

    target [drafts + batch, vocab] and draft [drafts, vocab]: probabilities, one type; a sequence's target rows are its
    tokens' and one more.  tokens int32 and accept fp32 [drafts], sample fp32 [batch]: numbers in [0, 1).  Without
    offsets (int32 [batch + 1], with max_len) every sequence has drafts / batch tokens.  Token i stays while
    accept q(x) < p(x); the next one is drawn by `sample` from max(p - q, 0) of the first that does not, or from the last
    row of p.  A row of the result: the accepted tokens, the next one, -1 behind it."""
    verify = (blocks._native or _load()).verify_draft
    if stream is None:
        return verify(target, draft, tokens, accept, sample, offsets, max_len, out, count)
    with _on(stream):
        return verify(target, draft, tokens, accept, sample, offsets, max_len, out, count)
