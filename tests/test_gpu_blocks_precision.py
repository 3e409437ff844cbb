"""How exact the block operators are, by bounds that leave room for fp32 sums and the output's rounding alone.

The bounds follow from the arithmetic and were fixed before their first run; E32 is half a unit of fp32."""
import numpy as np
import pytest

from oracle import blocks as ob
from test_gpu_blocks import E32, U, close, dev, host, q4, tdt

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------ 4-bit dense
def sums_bound(mag, k, group):
    """A group's sum of up to 128 exact products, truncated at each; a multiplication and an addition a
    group in fp32; up to 80 further additions (warps, blocks, bias).  Nothing else is rounded."""
    return (128 + 2 * -(-k // group) + 80) * E32 * mag


DENSE = [(9, 640, 130, 32, "bf16"), (20, 1100, 96, 64, "f16"), (32, 2050, 64, 128, "bf16"), (33, 1027, 130, 128, "bf16"),
         (64, 256, 128, 128, "f16"), (127, 640, 640, 64, "bf16"), (129, 72, 384, 32, "f16"), (257, 1100, 513, 128, "bf16"),
         (300, 4096, 96, 32, "bf16"), (700, 192, 1500, 64, "f16"), (90, 65, 33, 32, "bf16"), (2050, 320, 160, 32, "f16")]


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows, k, n, group, sdt", DENSE)
def test_dense_rounds_no_weight(dt, rows, k, n, group, sdt):
    """A weight q * scale has up to 15 bits: a product with it rounded to 8 or 11 would not hold the bound
    where an output is a small difference of large terms."""
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(rows + k)
    w, codes, scales, b = q4(rng, n, k, group, sdt)
    x = dev(rng.normal(size=(rows, k)), dt)
    pre, mag = ob.dense(host(x), codes, scales, k, group, b)
    y = sn.dense_q4(x, w)
    close(y, pre, sums_bound(mag, k, group), dt)
    sn.check_device()
    assert sn.dense_q4(x, w).equal(y)


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
def test_dense_of_a_row_does_not_depend_on_the_rows_beside_it(dt):
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(3)
    k, n, group = 700, 200, 64
    w, codes, scales, b = q4(rng, n, k, group, "bf16")
    x = dev(rng.normal(size=(100, k)), dt)
    pre, mag = ob.dense(host(x), codes, scales, k, group, b)
    alone = torch.cat([sn.dense_q4(x[i:i + 1], w) for i in range(100)])
    close(sn.dense_q4(x, w), host(alone), 2 * sums_bound(mag, k, group) + U[dt] * np.abs(pre), dt)


@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("sdt", ["f16", "bf16"])
def test_dense_fp16_with_groups_of_far_apart_scales(rows, sdt):
    """The largest products come from the group of the smallest scale."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(9)
    n, k = 48, 192
    codes = rng.integers(0, 256, (n, k // 2)).astype(np.uint8)
    small = 2.0 ** -20 if sdt == "f16" else 2.0 ** -34
    scales = dev(rng.uniform(1, 1.9, (n, 3)) * np.array([2.0 ** 8, small, 2.0 ** -2]), sdt)
    x = rng.normal(size=(rows, k))
    x[:, :64] *= 2.0 ** -24 / 2.0 ** -8  # (fp16's smallest values)
    x[:, 64:128] = np.clip(x[:, 64:128] * 2.0 ** 14, -60000, 60000)
    x[:, 128:] = 0
    x = dev(x, "f16")
    if sdt == "bf16":
        x[:, :64] = 0  # nothing beside them then
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, k, 64)
    pre, mag = ob.dense(host(x), codes, host(scales), k, 64)
    close(sn.dense_q4(x, w), pre, sums_bound(mag, k, 64), "f16")


@pytest.mark.parametrize("dt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows", [2, 64])
@pytest.mark.parametrize("size", [2.0 ** -126, 2.0 ** -118, 2.0 ** 100])
def test_dense_with_scales_at_the_ends_of_bf16(dt, rows, size):
    """No factor on the way leaves fp32's range: codes of 0 and inputs of 0 give 0, never NaN."""
    import torch
    import paper_2110_06037_gb300 as sn
    rng = np.random.default_rng(10)
    codes = rng.integers(0, 256, (40, 64)).astype(np.uint8)
    codes[:, ::3] = 0
    scales = dev(rng.uniform(1, 1.5, (40, 2)), "bf16") * size
    w = sn.Q4Weights(torch.from_numpy(codes).cuda(), scales, 128, 64)
    x = rng.normal(size=(rows, 128)) * (2.0 ** -14 if size > 1 else 2.0 ** 10)
    if size > 1 and dt == "f16":
        x[:] = 0  # (the outputs would be beyond fp16)
    x[0] = 0
    x = dev(x, dt)
    pre, mag = ob.dense(host(x), codes, host(scales), 128, 64)
    y = sn.dense_q4(x, w)
    close(y, pre, sums_bound(mag, 128, 64) + 2.0 ** -126, dt)
    assert bool((y[0] == 0).all())
