"""Attention over batches whose sequences are all empty, with token rows behind them: nothing is launched, so that this
runs without a GPU and the addresses are never read."""
import ctypes as C

import pytest

from paper_2110_06037_gb300 import _sn

P = 1 << 20
TYPES = {"f32": _sn.SN_F32, "f16": _sn.SN_F16, "bf16": _sn.SN_BF16}


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("context", [0, 64, 4096, 1 << 20])
@pytest.mark.parametrize("heads, q_heads", [(2, 2), (2, 16), (1, 128)])
def test_all_sequences_empty(dt, codes, context, heads, q_heads):
    lib, n, t = _sn.lib(), C.c_int64(-1), TYPES[dt]
    c = _sn.sn_kv_cache(_sn.SN_QI8 if codes else t, 64, heads, 64, 64, P, 2 * P, *((3 * P, 4 * P) if codes else (None, None)))
    assert lib.sn_attend_workspace(C.byref(c), t, q_heads, 5, 3, 0, context, C.byref(n)) == _sn.SN_OK
    assert n.value == 0
    ld = q_heads * 64
    assert lib.sn_attend(C.byref(c), t, q_heads, 1.0, 5, 3, 0, context, P, P, P, 3, 64, None, 5 * P, ld, 64, 6 * P, ld, 64, None, 0,
                         None) == _sn.SN_OK, lib.sn_last_error()
