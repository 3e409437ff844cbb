"""Further refusals of the block operators' C entries, made on the host: the addresses are never read."""
import ctypes as C

import pytest

from paper_2110_06037_gb300 import _sn

P = 1 << 20


@pytest.mark.parametrize("dtype", [_sn.SN_F32, _sn.SN_F16, _sn.SN_BF16])
@pytest.mark.parametrize("rows", [1, 64])
def test_dense_over_its_own_input(dtype, rows):
    """A block's outputs would be inputs of blocks that have not run."""
    w = _sn.sn_q4_weights(64, 64, 64, _sn.SN_BF16, 0, 8 * P, None)
    assert _sn.lib().sn_q4_dense(C.byref(w), dtype, rows, P, 64, P, 64, 4 * P, 1 << 30, None) == _sn.SN_EINVAL
    assert b"y over x" in _sn.lib().sn_last_error()
