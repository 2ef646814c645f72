"""The README's calls, run as they stand and checked against their formula in 64 bits (bounds as in test_rotary.py and test_fp8_linear.py)."""
import os
import re

import numpy as np
import pytest
import torch

from tests.fp8_util import dequantise, np64
from tests.test_rotary import U, check, rotate64

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_from_a_block_s_input_to_queries_and_keys():
    code = re.search(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), re.S).group(1)
    n = {}
    exec(code, n)
    tokens, heads, dim, width = n["tokens"], n["heads"], n["dim"], n["width"]
    A, B = dequantise(n["x"], n["x_scales"], tokens, width), dequantise(n["w"], n["w_scales"], 3 * heads * dim, width)
    y, size = A @ B.T, np.abs(A) @ np.abs(B).T
    off = np.abs(np64(n["packed"].view(tokens, -1)) - y)
    assert (off <= 2.0 ** -22 * (width / 32 + 10) * size + 2.0 ** -8 * np.abs(y) * 1.01).all()
    # the angles: three axes of 8, 14 and 14 pairs
    speeds = [10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) * 2 / d) for d in (16, 28, 28)]
    angle = torch.cat([n["positions"].cpu().double()[:, i:i + 1] * s for i, s in enumerate(speeds)], 1)
    table = torch.stack([angle.cos(), angle.sin()], -1)
    assert float((n["table"].cpu().double() - table).abs().max()) <= 2 * U
    for got, heads_in in ((n["q_out"], n["q"]), (n["k_out"], n["k"])):
        x = heads_in.double()[None]
        normed = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)
        want, magnitude = rotate64(normed, n["table"][None], 0, dim, False)
        check(got[None], want, 16 * U * magnitude)
