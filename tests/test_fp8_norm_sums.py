"""Sums of the norm: how exact they are, and squares that leave fp32's range at the low end."""
import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import dequantise, e4m3_round, scale_exponent, unpack

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1.0, 2.0 ** -20, 2.0 ** 30])
def test_many_small_squares_beside_large_ones(size, dtype):
    """A row of 16384 whose squares are 1 (columns 0, 8, .. 248) or 2^-24: added to a sum of 1 one by one, each of the small ones
    is lost, half a unit in the last place, to even.  A sum whose additions depend on one another no more than 16 deep (4 of a
    lane's, 3 that join its parts, 5 across a warp, 4 across 16 warps) is off by at most 16 * 2^-24 of itself, the root by half
    that; mean and eps add nothing (powers of two, eps = 0), rsqrt 2 units (2^-22), the two products and the weight's own rounding
    1.5 * 2^-23: y is good to (8 + 4 + 3) * 2^-24.  What the large columns show of it: their weights place y at 17 times a scale,
    halfway between the format's 16 and 18, and that far above or below."""
    D, big = 16384, 248
    h = torch.zeros(2, D, dtype=torch.float64)
    h[:, :1024] = 2.0 ** -12
    h[:, 1024::8 * 4] = 2.0 ** -12
    h[:, 0:big + 1:8] = 1.0
    x = h.numpy()
    rms = np.sqrt((x * x).mean(1, keepdims=True))
    tolerance = 15 * 2.0 ** -24
    w = np.zeros(D)
    w[0:big + 1:16] = 17.0 * (1.0 + tolerance) * rms[0, 0]
    w[8:big + 1:16] = 17.0 * (1.0 - tolerance) * rms[0, 0]
    weight = torch.tensor(w).float().to(DEV)
    q, s = sc.new_fp8(2, D)
    sc.svdcache_residual_rmsnorm_fp8((h * size).to(dtype).to(DEV), None, None, weight, 0.0, q, s)
    got = dequantise(q, s, 2, D)
    assert (got[:, 0:big + 1:16] == 18.0).all(), got[:, 0:big + 1:16]
    assert (got[:, 8:big + 1:16] == 16.0).all(), got[:, 8:big + 1:16]


@pytest.mark.parametrize("eps", [1e-6, 1e-30])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_squares_below_the_smallest_number(dtype, eps):
    """Elements of about 1e-30: their mean square is nothing beside eps, so y = h / sqrt(eps), small but of full precision."""
    g = torch.Generator().manual_seed(3)
    h = (torch.randn(5, 392, generator=g, dtype=torch.float64) * 1e-30).to(dtype).to(DEV)
    q, s = sc.new_fp8(5, 392)
    sc.svdcache_residual_rmsnorm_fp8(h, None, None, None, eps, q, s)
    y = h.double().cpu().numpy() / np.sqrt(np.float64(np.float32(eps)))
    v, e = unpack(q, s, 5, 392)
    top = np.stack([np.abs(y[:, i:i + 128]).max(1) for i in range(0, 392, 128)], 1)
    # y is good to 2^-18 of itself: no maximum here is that near a scale's step
    assert (scale_exponent(top * (1 - 2.0 ** -18)) == scale_exponent(top * (1 + 2.0 ** -18))).all()
    np.testing.assert_array_equal(e, scale_exponent(top))
    z = y / np.repeat(np.exp2(e), 128, axis=1)[:, :392]
    near = e4m3_round(z * (1 - 2.0 ** -18)) != e4m3_round(z * (1 + 2.0 ** -18))
    np.testing.assert_array_equal(v[~near], e4m3_round(z)[~near])
    assert near.mean() < 0.01
