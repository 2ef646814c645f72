"""Arguments of the 8-bit calls that would be read as something else, written where they should not, or cut on their way to
the C ABI: each is refused, in words, before anything is launched."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import random_fp8

gpu = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def small():
    """Operands of a 4 x 32 product over K = 128, and rows that were quantised into the first of them."""
    a, sa = sc.new_fp8(4, 128)
    x = torch.linspace(-3.0, 3.0, 512, device=DEV).view(4, 128)
    sc.svdcache_quantize_fp8(x, a, sa)
    b, sb = random_fp8(32, 128, 1)
    return x, a, sa, b, sb


OTHER_BYTES = [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.int8, torch.bool]


@gpu
@pytest.mark.parametrize("dtype", OTHER_BYTES + [torch.float8_e8m0fnu])
def test_bytes_of_another_type_are_not_read_as_e4m3(small, dtype):
    x, a, sa, b, sb = small
    C = torch.zeros(4, 32, device=DEV)
    before = sc.svdcache_kernel_launches()
    for call in (lambda: sc.svdcache_quantize_fp8(x, a.view(dtype), sa),
                 lambda: sc.svdcache_residual_rmsnorm_fp8(x, None, None, None, 1e-6, a.view(dtype), sa),
                 lambda: sc.svdcache_gemm_fp8(a.view(dtype), sa, b, sb, 128, C),
                 lambda: sc.svdcache_gemm_fp8(a, sa, b.view(dtype), sb, 128, C),
                 lambda: sc.svdcache_gemm_fp8(a, sa, b, sb, 128, torch.zeros(4, 32, dtype=torch.uint8, device=DEV).view(dtype), S_out=sa)):
        with pytest.raises(ValueError):
            call()
    assert sc.svdcache_kernel_launches() == before


@gpu
@pytest.mark.parametrize("dtype", OTHER_BYTES + [torch.float8_e4m3fn])
def test_bytes_of_another_type_are_not_scales(small, dtype):
    x, a, sa, b, sb = small
    C = torch.zeros(4, 32, device=DEV)
    before = sc.svdcache_kernel_launches()
    for call in (lambda: sc.svdcache_quantize_fp8(x, a, sa.view(dtype)),
                 lambda: sc.svdcache_residual_rmsnorm_fp8(x, None, None, None, 1e-6, a, sa.view(dtype)),
                 lambda: sc.svdcache_gemm_fp8(a, sa.view(dtype), b, sb, 128, C),
                 lambda: sc.svdcache_gemm_fp8(a, sa, b, sb.view(dtype), 128, C)):
        with pytest.raises(ValueError):
            call()
    assert sc.svdcache_kernel_launches() == before


@gpu
def test_the_format_s_own_types_are_taken(small):
    x, a, sa, b, sb = small
    C, D = torch.zeros(4, 32, device=DEV), torch.ones(4, 32, device=DEV)
    sc.svdcache_gemm_fp8(a, sa, b, sb, 128, C)
    v, e = torch.float8_e4m3fn, torch.float8_e8m0fnu
    q, s = sc.new_fp8(4, 128)
    sc.svdcache_quantize_fp8(x, q.view(v), s.view(e))
    assert torch.equal(q, a) and torch.equal(s, sa)
    sc.svdcache_gemm_fp8(q.view(v), s.view(e), b.view(v), sb.view(e), 128, D)
    assert torch.equal(C, D)
