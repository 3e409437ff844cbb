"""The block operators' oracle against closed forms and a second formulation."""
import numpy as np

from oracle import blocks as ob


def test_unpack_order_and_sign():
    assert ob.unpack(np.array([[0x2F, 0x87]], np.uint8), 4).tolist() == [[-1, 2, 7, -8]]
    assert ob.unpack(np.array([[0x2F, 0x87]], np.uint8), 3).tolist() == [[-1, 2, 7]]


def test_dense_scales_by_group():
    codes = np.full((1, 48), 0x11, np.uint8)  # 96 ones
    y, mag = ob.dense(np.ones((1, 96)), codes, np.array([[2.0, 3.0, -5.0]]), 96, 32)
    assert y.tolist() == [[0.0]] and mag.tolist() == [[320.0]]


def test_norms_of_known_rows():
    v = np.array([[3.0, -3.0, 3.0, -3.0]])
    assert np.allclose(ob.row_norm(v, "rms", 0.0, 1.0, None), [[1, -1, 1, -1]])
    assert np.allclose(ob.row_norm(v + 7, "layer", 0.0, 2.0, 1.0), [[3, -1, 3, -1]])
    total, n = ob.block_norm(v, residual=np.ones((1, 4)), gate=np.zeros((1, 4)), post=np.ones(4), pre=np.ones(4),
                             gate_act="sigmoid", eps=0.0)
    assert np.allclose(total, [[1.5, 0.5, 1.5, 0.5]])
    assert np.allclose(n, total / np.sqrt((1.5 ** 2 + 0.5 ** 2) / 2))


def test_conv_in_two_parts_is_conv_in_one():
    rng = np.random.default_rng(0)
    x, w = rng.normal(size=(9, 5)), rng.normal(size=(5, 4))
    whole, _, k1 = ob.conv(x, w, None, True, np.zeros((4, 5)))
    a, _, k = ob.conv(x[:2], w, None, True, np.zeros((4, 5)))
    b, _, k2 = ob.conv(x[2:], w, None, True, k, 2)
    assert np.allclose(np.concatenate((a, b)), whole) and np.array_equal(k1, k2)
    assert np.allclose(ob.conv(np.eye(6)[:, :1], w[:1], None, False)[0][:4, 0], w[0, ::-1])  # an impulse


def test_scan_is_the_sum_over_pairs():
    rng = np.random.default_rng(1)
    sizes = h, p, g, n = 4, 3, 2, 5
    xbc, dt, a = rng.normal(size=(7, h * p + 2 * g * n)), rng.normal(size=(7, h)), -rng.uniform(0.1, 2, h)
    s0 = rng.normal(size=(h, p, n))
    y, _, s, _ = ob.scan(xbc, dt, sizes, a, None, None, s0)
    d = np.log1p(np.exp(dt))
    for i in range(h):
        grp = i // 2
        x, b = xbc[:, i * p:(i + 1) * p], xbc[:, h * p + grp * n:h * p + (grp + 1) * n]
        c = xbc[:, h * p + (g + grp) * n:h * p + (g + grp + 1) * n]
        at = np.concatenate(([0], np.cumsum(d[:, i] * a[i])))
        for t in range(7):
            ref = np.exp(at[t + 1]) * s0[i] @ c[t]
            for u in range(t + 1):
                ref = ref + np.exp(at[t + 1] - at[u + 1]) * d[u, i] * (c[t] @ b[u]) * x[u]
            assert np.allclose(ref, y[t, i * p:(i + 1) * p])
        ref = np.exp(at[-1]) * s0[i] + sum(np.exp(at[-1] - at[u + 1]) * d[u, i] * np.outer(x[u], b[u]) for u in range(7))
        assert np.allclose(ref, s[i])
