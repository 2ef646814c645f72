"""The example that runs the 8-bit operators and the cache together: its full step against a plain 64-bit block on the same
8-bit weights, and its cached steps against computing every step."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import dequantise, gelu64, np64

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mlp_stream_fp8", os.path.join(ROOT, "examples", "mlp_stream_fp8.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_block_matches_a_plain_block(example):
    rows, width = 200, 384
    s = example.Stream(1, rows, width, 32, seed=3)
    out = s.step(0.0, full=True, cache=False)
    b = s.blocks[0]
    h = np64(s.start.bfloat16())
    y = h / np.sqrt((h * h).mean(1, keepdims=True) + 1e-6) * np64(b.norm)
    up, down = dequantise(*b.up, b.hidden, width), dequantise(*b.down, width, b.hidden)
    f = gelu64(y @ up.T + np64(b.up_bias)) @ down.T + np64(b.down_bias)
    # y and the hidden layer are rounded to e4m3 (relative error up to 2^-4, rms below 2^-5 each); over the products' many
    # terms the errors are independent, so F is off by about sqrt(2) * 2^-5 = 4.4 % of what its terms add up to; bound 8 %
    assert np.linalg.norm(np64(b.feature) - f) <= 0.08 * np.linalg.norm(f)
    np.testing.assert_allclose(np64(out), h + np64(b.feature), atol=2.0 ** -8 * 16)
    assert sc.gemm_status() == 0


def test_cached_stream_stays_near_the_full_one(example):
    r = example.run(blocks=3, rows=512, width=512, rank=64, steps=6, interval=3)
    assert r["status"] == 0 and r["states"] == [(2, 0)] * 3
    # the input drifts by 5 % a step: features of steps at most two apart differ by a fraction of that times their share of h
    assert 0.0 < r["worst"] < 0.3
