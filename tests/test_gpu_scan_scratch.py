"""The scan's scratch and grids follow the tokens there are, not sequences times the longest one's segments."""
import ctypes as C

import numpy as np
import pytest

from oracle import blocks as ob
from test_gpu_blocks import close, dev, host, ints, run_scan, scan_bound, ssm_weights

pytestmark = pytest.mark.gpu


def workspace(dtype, tokens, batch, max_len, heads, head_dim, state):
    from paper_2110_06037_gb300 import _sn
    p, n = _sn.sn_ssm_params(heads, head_dim, 1, state, 0, 1 << 20), C.c_int64()
    _sn.check(_sn.lib().sn_ssm_workspace(C.byref(p), dtype, tokens, batch, max_len, C.byref(n)))
    return n.value


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("batch, long, short, heads", [(256, 8192, 10, 8), (1024, 4096, 20, 24), (4000, 30000, 1, 4)])
def test_scratch_of_many_short_sequences_beside_a_long_one(dtype, batch, long, short, heads):
    """States at the cuts of what is long enough to be cut, and for bf16 a table of 3 KB for a chunk and
    head: less than the states of the sequences themselves, and than 64 of the long one's."""
    tokens, state = long + (batch - 1) * short, heads * 64 * 128 * 4
    tables = 3200 * heads * (tokens // 128 + batch + 2)
    n = workspace(dtype, tokens, batch, long, heads, 64, 128)
    assert n <= batch * state and n <= 64 * 2 * state + tables


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens, sizes", [
    ([3, 900] * 3 + [5] * 70 + [2100, 0, 640, 127, 1, 1300], (2, 32, 1, 16)), ([64, 63, 65, 128] * 9 + [1025], (1, 64, 1, 128)),
    ([511, 512, 513, 1023, 1024, 1025], (1, 72, 1, 24)), ([700] * 5, (1, 8, 1, 8))])
def test_scan_of_sequences_that_are_cut_beside_some_that_are_not(dt, lens, sizes):
    import torch
    import paper_2110_06037_gb300 as sn
    h, p, g, n = sizes
    rng = np.random.default_rng(len(lens))
    a, d, b = ssm_weights(rng, h)
    rows, c = sum(lens), h * p + 2 * g * n
    xbc, step = dev(rng.normal(size=(rows, c)), dt), dev(rng.normal(size=(rows, h)) - 2, dt)
    state = dev(rng.normal(size=(len(lens), h, p, n)))
    ref, my, sref, ms = run_scan(host(xbc), host(step), lens, sizes, a, d, b, host(state), list(range(len(lens))))
    ssm = sn.StateSpace(h, p, g, n, dev(a), dev(d), dev(b))
    off = ints(np.concatenate(([0], np.cumsum(lens))).tolist())
    out = torch.full_like(state, 5.0)
    for _ in range(2):
        y = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=out)
        close(y, ref, scan_bound(my, max(lens)) + (2.0 ** -14 * my if dt != "f32" else 0), dt)
        close(out, sref, scan_bound(ms, max(lens)), "f32")
    again = ssm.scan(xbc, step, offsets=off, max_len=max(lens), state_in=state, state_out=state)
    assert torch.equal(again, y) and torch.equal(state, out)
    sn.check_device()
