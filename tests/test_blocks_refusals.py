"""What the block operators refuse, and what they do with nothing to do.  Every check is made on the
host before anything is launched, so this runs without a GPU: the addresses are never read."""
import ctypes as C

import pytest

from paper_2110_06037_gb300 import _sn

P = 1 << 20  # an aligned address that nothing reads
OK, EINVAL, EUNSUPPORTED = _sn.SN_OK, _sn.SN_EINVAL, _sn.SN_EUNSUPPORTED


def weights(**kw):
    a = dict(n=64, k=128, group=64, scale_dtype=_sn.SN_BF16, act=0, packed=P, bias=P)
    a.update(kw)
    return _sn.sn_q4_weights(*[a[f] for f, _ in _sn.sn_q4_weights._fields_])


def dense(w=None, dtype=_sn.SN_BF16, rows=1, x=P, ldx=128, y=2 * P, ldy=64, work=None, nbytes=0):
    return _sn.lib().sn_q4_dense(C.byref(w or weights()), dtype, rows, x, ldx, y, ldy, work, nbytes, None)


@pytest.mark.parametrize("kw, status", [
    (dict(n=0), EINVAL), (dict(k=0), EINVAL), (dict(k=-1), EINVAL), (dict(group=16), EINVAL), (dict(group=0), EINVAL),
    (dict(scale_dtype=_sn.SN_F32), EINVAL), (dict(scale_dtype=9), EINVAL), (dict(act=5), EINVAL), (dict(act=-1), EINVAL),
    (dict(packed=None), EINVAL), (dict(packed=P + 16), EINVAL), (dict(bias=P + 2), EINVAL),
    (dict(k=(1 << 24) + 1), EUNSUPPORTED), (dict(n=(1 << 26) + 1), EUNSUPPORTED)])
def test_q4_weights(kw, status):
    assert dense(weights(**kw)) == status
    assert _sn.lib().sn_q4_pack(P, P, C.byref(weights(**kw)), None) == status
    assert _sn.lib().sn_last_error()


@pytest.mark.parametrize("kw", [dict(dtype=_sn.SN_QI8), dict(dtype=-1), dict(rows=-1), dict(x=None), dict(y=None),
                                dict(ldx=127), dict(ldy=63), dict(x=P + 1), dict(y=P + 1)])
def test_q4_dense_arguments(kw):
    assert dense(**kw) == EINVAL


def test_q4_other_entries():
    lib, n = _sn.lib(), C.c_int64()
    assert lib.sn_q4_bytes(1, 1, 32, None) == EINVAL and lib.sn_q4_bytes(1, 1, 48, C.byref(n)) == EINVAL
    assert lib.sn_q4_bytes(17, 65, 64, C.byref(n)) == OK and n.value >= 2 * 2 * 512 + 2 * 2 * 32 + 32 * 4
    assert lib.sn_q4_quantize(None, 0, 1, 1, 32, 1, P, P, None) == EINVAL
    assert lib.sn_q4_quantize(P, 3, 1, 1, 32, 1, P, P, None) == EINVAL
    assert lib.sn_q4_quantize(P, 0, 1, 1, 32, 0, P, P, None) == EINVAL
    assert lib.sn_q4_pack(None, P, C.byref(weights()), None) == EINVAL
    assert lib.sn_q4_workspace(C.byref(weights()), 0, -1, P, 128, C.byref(n)) == EINVAL
    assert lib.sn_q4_dense(None, 0, 1, P, 128, P, 64, None, 0, None) == EINVAL
    assert dense(rows=0, x=None, y=None) == OK


def norm(rows=4, dtype=_sn.SN_F16, y=P, ldy=32, gate=None, ldg=32, per=1, rdt=_sn.SN_F32, res=2 * P, ldr=32, s=3 * P,
         lds=32, n=4 * P, ldn=32, **kw):
    a = dict(dim=32, kind=0, gate=0, gate_after=1, eps=1e-5, post=P, post_bias=None, pre=P, pre_bias=None, scale=None)
    a.update(kw)
    p = _sn.sn_norm_params(*[a[f] for f, _ in _sn.sn_norm_params._fields_])
    if "gate_kind" in kw:
        p.gate = kw["gate_kind"]
    return _sn.lib().sn_block_norm(C.byref(p), dtype, rows, y, ldy, gate, ldg, per, rdt, res, ldr, s, lds, n, ldn, None)


@pytest.mark.parametrize("kw", [
    dict(dim=0), dict(kind=2), dict(gate_after=2), dict(eps=-1.0), dict(eps=float("nan")), dict(post=P + 1),
    dict(post=None, post_bias=P), dict(pre=None, pre_bias=P, n=None), dict(dtype=3), dict(rows=-1), dict(rdt=_sn.SN_BF16),
    dict(gate=P), dict(y=None, res=None), dict(s=None, n=None, pre=None), dict(ldy=31), dict(ldr=31), dict(lds=31),
    dict(ldn=31), dict(y=P + 1), dict(res=P + 2), dict(s=4 * P), dict(s=P), dict(s=2 * P, ldr=64), dict(n=P, ldy=40),
    dict(n=2 * P), dict(pre=None), dict(n=None)])
def test_block_norm(kw):
    assert norm(**kw) == EINVAL


def test_block_norm_nothing_and_limits():
    assert norm(rows=0, y=None, res=None, s=None, n=None) == OK
    assert norm(dim=(1 << 28) + 1) == EUNSUPPORTED and norm(rows=1 << 31) == EUNSUPPORTED


def conv(dtype=_sn.SN_F16, c=16, w=4, silu=1, wp=P, bp=None, tokens=8, batch=2, max_len=4, off=None, x=P, ldx=16, y=2 * P,
         ldy=16, kept=3 * P, n=2, slots=None, pos=None):
    return _sn.lib().sn_causal_conv(dtype, c, w, silu, wp, bp, tokens, batch, max_len, off, x, ldx, y, ldy, kept, n, slots, pos, None)


@pytest.mark.parametrize("kw, status", [
    (dict(dtype=3), EINVAL), (dict(c=0), EINVAL), (dict(w=0), EINVAL), (dict(w=9), EUNSUPPORTED), (dict(silu=2), EINVAL),
    (dict(wp=None), EINVAL), (dict(wp=P + 2), EINVAL), (dict(tokens=-1), EINVAL), (dict(tokens=9), EINVAL),
    (dict(batch=-1), EINVAL), (dict(off=P, max_len=9), EINVAL), (dict(off=P + 2), EINVAL), (dict(x=None), EINVAL),
    (dict(y=None), EINVAL), (dict(ldx=15), EINVAL), (dict(y=P), EINVAL), (dict(n=0), EINVAL), (dict(kept=3 * P + 1), EINVAL),
    (dict(batch=65536, max_len=1, tokens=65536), EUNSUPPORTED), (dict(batch=1, max_len=1 << 31, tokens=1 << 31), EUNSUPPORTED)])
def test_causal_conv(kw, status):
    assert conv(**kw) == status


def test_causal_conv_nothing():
    assert conv(tokens=0, batch=0, max_len=0, x=None, y=None) == OK
    assert conv(tokens=0, batch=2, max_len=0, x=None, y=None) == OK


def ssm(**kw):
    a = dict(heads=4, head_dim=8, groups=2, state=16, width=4, a=P, d=P, dt_bias=P, conv_w=P, conv_b=None)
    a.update(kw)
    return _sn.sn_ssm_params(*[a[f] for f, _ in _sn.sn_ssm_params._fields_])


def scan(p=None, dtype=_sn.SN_F16, tokens=8, batch=2, max_len=4, off=None, x=P, ldx=96, dt=2 * P, ldd=4, si=3 * P, so=4 * P,
         n=2, slots=None, y=5 * P, ldy=32, work=None, nbytes=0):
    return _sn.lib().sn_ssm_scan(C.byref(p or ssm()), dtype, tokens, batch, max_len, off, x, ldx, dt, ldd, si, so, n, slots, y,
                                 ldy, work, nbytes, None)


def step(p=None, dtype=_sn.SN_F16, batch=2, x=P, ldx=96, dt=2 * P, ldd=4, kept=6 * P, si=3 * P, so=4 * P, n=2, slots=None,
         pos=P, y=5 * P, ldy=32):
    return _sn.lib().sn_ssm_step(C.byref(p or ssm()), dtype, batch, x, ldx, dt, ldd, kept, si, so, n, slots, pos, y, ldy, None)


@pytest.mark.parametrize("kw, status", [
    (dict(heads=0), EINVAL), (dict(head_dim=0), EINVAL), (dict(groups=0), EINVAL), (dict(groups=3), EINVAL),
    (dict(state=0), EINVAL), (dict(a=None), EINVAL), (dict(a=P + 2), EINVAL), (dict(head_dim=257), EUNSUPPORTED),
    (dict(state=257), EUNSUPPORTED)])
def test_ssm_sizes(kw, status):
    assert scan(ssm(**kw)) == status and step(ssm(**kw)) == status
    assert _sn.lib().sn_ssm_workspace(C.byref(ssm(**kw)), 0, 8, 2, 4, C.byref(C.c_int64())) == status


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(tokens=9), dict(batch=-1), dict(x=None), dict(dt=None), dict(y=None), dict(ldx=95), dict(ldd=3),
    dict(ldy=31), dict(y=P), dict(y=2 * P), dict(si=3 * P + 2), dict(n=0), dict(slots=P + 1), dict(x=P + 1)])
def test_ssm_scan(kw):
    assert scan(**kw) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(batch=-1), dict(x=None), dict(dt=None), dict(y=None), dict(kept=None), dict(so=None), dict(ldx=95),
    dict(ldy=31), dict(y=P), dict(n=0), dict(pos=P + 1), dict(p=ssm(conv_w=None)), dict(p=ssm(width=0))])
def test_ssm_step(kw):
    assert step(**kw) == EINVAL


def test_ssm_nothing_and_limits():
    assert scan(tokens=0, batch=0, max_len=0, x=None, dt=None, y=None) == OK
    assert step(batch=0, x=None, dt=None, y=None, kept=None) == OK
    assert step(ssm(width=9)) == EUNSUPPORTED
    assert step(batch=65536) == EUNSUPPORTED
