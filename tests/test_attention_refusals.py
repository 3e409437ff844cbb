"""What the attention layer's operators refuse, and what they do with nothing to do.  Every check is made
on the host before anything is launched, so this runs without a GPU: the addresses are never read."""
import ctypes as C
import math
from fractions import Fraction

import numpy as np
import pytest

from oracle import attention as oa
from paper_2110_06037_gb300 import _sn

P = 1 << 20  # an aligned address that nothing reads
OK, EINVAL, EUNSUPPORTED = _sn.SN_OK, _sn.SN_EINVAL, _sn.SN_EUNSUPPORTED
BF16, QI8 = _sn.SN_BF16, _sn.SN_QI8


def rope(dtype=BF16, tokens=4, qh=8, q=P, lq=512, hq=64, yq=2 * P, lyq=512, hyq=64, kh=2, k=3 * P, lk=128, hk=64, yk=4 * P,
         lyk=128, hyk=64, pos=P, **kw):
    a = dict(head_dim=64, pairs=32, axes=1, norm=0, interleaved=0, eps=1e-6, turns=P, axis=None, q_weight=P, k_weight=P)
    a.update(kw)
    p = _sn.sn_rope_params(*[a[f] for f, _ in _sn.sn_rope_params._fields_])
    return _sn.lib().sn_head_rope(C.byref(p), dtype, tokens, qh, q, lq, hq, yq, lyq, hyq, kh, k, lk, hk, yk, lyk, hyk, pos, None)


@pytest.mark.parametrize("kw", [
    dict(head_dim=0), dict(head_dim=63), dict(pairs=33), dict(pairs=-1), dict(axes=0), dict(norm=3), dict(norm=-1),
    dict(interleaved=2), dict(eps=-1.0), dict(eps=math.nan), dict(turns=None), dict(turns=P + 4), dict(axis=P + 2),
    dict(q_weight=P + 1), dict(norm=2), dict(dtype=QI8), dict(tokens=-1), dict(qh=-1), dict(pos=None), dict(pos=P + 2),
    dict(q=None), dict(yq=None), dict(k=None), dict(yk=None), dict(lq=511), dict(hq=63), dict(lq=-512), dict(q=P + 1), dict(hyk=0),
    dict(yk=2 * P), dict(yq=P, lyq=1024), dict(yq=3 * P), dict(yk=P), dict(lq=64, hq=64)])
def test_rope_arguments(kw):
    assert rope(**kw) == EINVAL
    assert _sn.lib().sn_last_error()


def test_rope_limits_and_nothing():
    assert rope(head_dim=258, pairs=1) == EUNSUPPORTED and rope(tokens=1 << 31) == EUNSUPPORTED and rope(qh=65536) == EUNSUPPORTED
    assert rope(tokens=0, q=None, k=None, pos=P) == OK and rope(qh=0, kh=0, q=None, k=None) == OK


def turns(values):
    n = len(values)
    out = (C.c_uint64 * max(n, 1))()
    return _sn.lib().sn_rope_turns((C.c_double * max(n, 1))(*values), n, out), list(out)[:n]


def test_rope_turns():
    """A fraction of a turn is off by at most two units of 2^-64 for angles of up to a turn (one rounding down, and
    1 / 2 pi in two doubles: 2^-106 of the angle); of 2^20 radians by 2^20 / 2 pi 2^-106 more, none of it a unit."""
    rng = np.random.default_rng(0)
    values = [0.0, 1.0, -1.0, 1e-300, -1e-18, 2 * math.pi, -2 * math.pi, 2.0 ** 20, -2.0 ** 20, math.pi, 0.5]
    values += [10000.0 ** (-i / 64) for i in range(64)] + list(rng.normal(size=200)) + list(rng.uniform(-2 ** 20, 2 ** 20, 200))
    rc, got = turns(values)
    assert rc == OK
    for v, g in zip(values, got):
        exact = (Fraction(v) / oa.TWO_PI) % 1 * (1 << 64)
        gap = (g - exact) % (1 << 64)
        assert min(gap, (1 << 64) - gap) <= 2, v
    assert turns([math.nan])[0] == EINVAL and turns([math.inf])[0] == EINVAL and turns([2.0 ** 20 + 1])[0] == EINVAL
    assert _sn.lib().sn_rope_turns(None, 1, None) == EINVAL and _sn.lib().sn_rope_turns(None, -1, None) == EINVAL
    assert _sn.lib().sn_rope_turns(None, 0, None) == OK


def cache(**kw):
    a = dict(dtype=BF16, pages=8, heads=2, page=16, head_dim=64, k=P, v=2 * P, k_scale=None, v_scale=None)
    a.update(kw)
    return _sn.sn_kv_cache(*[a[f] for f, _ in _sn.sn_kv_cache._fields_])


def kv(name, c=None, dtype=BF16, tokens=8, batch=2, max_len=4, off=None, pos=None, table=P, n=2, width=4, slots=None, k=3 * P,
       lk=128, hk=64, v=4 * P, lv=128, hv=64):
    return getattr(_sn.lib(), name)(C.byref(c or cache()), dtype, tokens, batch, max_len, off, pos, table, n, width, slots, k, lk, hk,
                                    v, lv, hv, None)


def attend(c=None, dtype=BF16, qh=8, scale=0.125, tokens=8, batch=2, max_len=4, ctx=64, off=None, pos=None, table=P, n=2, width=4,
           slots=None, q=3 * P, lq=512, hq=64, y=4 * P, ly=512, hy=64, work=None, nbytes=0):
    return _sn.lib().sn_attend(C.byref(c or cache()), dtype, qh, scale, tokens, batch, max_len, ctx, off, pos, table, n, width, slots,
                               q, lq, hq, y, ly, hy, work, nbytes, None)


BAD_CACHE = [(dict(dtype=4), EINVAL), (dict(dtype=-1), EINVAL), (dict(pages=0), EINVAL), (dict(heads=0), EINVAL),
             (dict(page=8), EINVAL), (dict(page=48), EINVAL), (dict(page=512), EINVAL), (dict(head_dim=0), EINVAL),
             (dict(head_dim=24), EUNSUPPORTED), (dict(head_dim=272), EUNSUPPORTED), (dict(k=None), EINVAL), (dict(v=P + 8), EINVAL),
             (dict(k_scale=P), EINVAL), (dict(dtype=QI8), EINVAL), (dict(dtype=QI8, k_scale=P, v_scale=P + 4), EINVAL),
             (dict(heads=65536), EUNSUPPORTED)]


@pytest.mark.parametrize("kw, status", BAD_CACHE)
def test_caches(kw, status):
    assert kv("sn_kv_write", cache(**kw)) == status and kv("sn_kv_read", cache(**kw)) == status
    assert attend(cache(**kw)) == status
    assert _sn.lib().sn_attend_workspace(C.byref(cache(**kw)), BF16, 8, 1, 1, 1, 1, C.byref(C.c_int64())) == status


BAD_SEQUENCES = [dict(tokens=9), dict(tokens=-1), dict(batch=-1), dict(max_len=9, off=P), dict(off=P + 2), dict(pos=P + 1),
                 dict(slots=P + 2), dict(table=None), dict(table=P + 2), dict(n=-1), dict(n=1), dict(width=-1), dict(dtype=QI8),
                 dict(dtype=_sn.SN_F16), dict(dtype=7)]


@pytest.mark.parametrize("kw", BAD_SEQUENCES + [
    dict(k=None), dict(v=None), dict(k=3 * P + 1), dict(lk=127), dict(hk=63), dict(lv=64, hv=64), dict(lk=-128)])
def test_kv_arguments(kw):
    assert kv("sn_kv_write", **kw) == EINVAL and kv("sn_kv_read", **kw) == EINVAL


@pytest.mark.parametrize("kw", BAD_SEQUENCES + [
    dict(qh=0), dict(qh=3), dict(scale=math.nan), dict(scale=math.inf), dict(ctx=-1), dict(q=None), dict(y=None), dict(y=3 * P),
    dict(lq=511), dict(hq=0), dict(ly=64), dict(q=3 * P + 1)])
def test_attend_arguments(kw):
    assert attend(**kw) == EINVAL


def test_attention_limits_and_nothing():
    lib, n = _sn.lib(), C.c_int64()
    assert kv("sn_kv_read", v=3 * P) == EINVAL
    many = dict(batch=65536, max_len=1, tokens=65536, n=65536)
    assert kv("sn_kv_write", **many) == EUNSUPPORTED and kv("sn_kv_read", **many) == EUNSUPPORTED and attend(**many) == EUNSUPPORTED
    assert attend(cache(heads=32768), qh=65536) == EUNSUPPORTED
    for nothing in (dict(tokens=0, max_len=0), dict(tokens=0, batch=0, max_len=0)):
        assert kv("sn_kv_write", k=None, v=None, **nothing) == OK and kv("sn_kv_read", k=None, v=None, **nothing) == OK
        assert attend(q=None, y=None, **nothing) == OK
    assert lib.sn_attend_workspace(C.byref(cache()), BF16, 8, 1, 1, 1, 1, None) == EINVAL
    assert lib.sn_attend_workspace(C.byref(cache()), BF16, 8, -1, 1, 1, 1, C.byref(n)) == EINVAL
    assert lib.sn_attend_workspace(C.byref(cache()), BF16, 8, 1, 1, 1, 1 << 40, C.byref(n)) == OK and n.value >= 0
    if n.value:
        assert attend(ctx=1 << 40, tokens=1, batch=1, max_len=1) == EINVAL  # without its scratch


def verify(dtype=_sn.SN_F32, vocab=100, tokens=4, batch=2, max_len=2, off=None, target=P, lt=100, draft=2 * P, ld=100, x=P, u=P, s=P,
           out=3 * P, count=4 * P):
    return _sn.lib().sn_verify_draft(dtype, vocab, tokens, batch, max_len, off, target, lt, draft, ld, x, u, s, out, count, None)


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(vocab=0), dict(tokens=-1), dict(batch=-1), dict(max_len=-1), dict(tokens=5), dict(off=P + 2), dict(target=None),
    dict(target=P + 2), dict(lt=99), dict(draft=None), dict(ld=99), dict(x=None), dict(u=None), dict(s=None), dict(out=None),
    dict(count=None), dict(out=3 * P + 2), dict(count=3 * P), dict(out=P)])
def test_verify_arguments(kw):
    assert verify(**kw) == EINVAL


def test_verify_limits_and_nothing():
    assert verify(vocab=(1 << 24) + 1, lt=1 << 25, ld=1 << 25) == EUNSUPPORTED
    assert verify(batch=65536, tokens=0, max_len=0) == EUNSUPPORTED
    assert verify(batch=0, tokens=0, max_len=0, target=None, draft=None, out=None) == OK


def test_handles():
    torch = pytest.importorskip("torch")
    import paper_2110_06037_gb300 as sn
    for call in (lambda: sn.HeadRope(64, [1.0] * 33, device="cuda:0"), lambda: sn.HeadRope(63, [1.0], device="cuda:0"),
                 lambda: sn.HeadRope(64, [1.0], norm="max", device="cuda:0"), lambda: sn.HeadRope(64, [1.0], axes=[0, 1], device="cuda:0"),
                 lambda: sn.HeadRope(64, [1.0], axes=[-1], device="cuda:0"), lambda: sn.HeadRope(64, [math.inf], device="cuda:0"),
                 lambda: sn.HeadRope(64, [1.0], device="cpu"), lambda: sn.HeadRope(64, [1.0], q_weight=torch.ones(64), device="cuda:0"),
                 lambda: sn.HeadRope(64, [1.0], norm="none", q_weight=torch.ones(64), device="cuda:0"),
                 lambda: sn.KVCache(torch.zeros(2, 2, 16), torch.zeros(2, 2, 16)),
                 lambda: sn.KVCache(*sn.KVCache.empty(2, 2, 16, 16, torch.float32, device="cpu")),
                 lambda: sn.KVCache(torch.zeros(2, 2, 16, 16, dtype=torch.int8), torch.zeros(2, 2, 16, 16, dtype=torch.int8)),
                 lambda: sn.KVCache(torch.zeros(2, 2, 16, 16, dtype=torch.float64), torch.zeros(2, 2, 16, 16, dtype=torch.float64))):
        with pytest.raises(sn.SnError):
            call()
