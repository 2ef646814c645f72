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


FIRST_IN_A_CAPTURE = """
import torch
from paper_2601_07396_b200 import binding as sc
x, w = torch.ones(40, 2048, device="cuda"), torch.ones(64, 2048, device="cuda")
(a, sa), (b, sb) = sc.new_fp8(40, 2048), sc.new_fp8(64, 2048)
C = torch.zeros(40, 64, device="cuda")
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    sc.svdcache_quantize_fp8(w, b, sb, tile_rows=128)
    sc.svdcache_residual_rmsnorm_fp8(x, None, None, None, 0.0, a, sa)
    sc.svdcache_gemm_fp8(a, sa, b, sb, 2048, C)
assert float(C.abs().max()) == 0.0              # captured, not run
graph.replay()
torch.cuda.synchronize()
assert bool((C == 2048.0).all()), C
assert sc.gemm_status() == 0
print("first calls captured")
"""


@gpu
def test_a_process_may_begin_with_captured_calls():
    r = subprocess.run([sys.executable, "-c", FIRST_IN_A_CAPTURE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "first calls captured" in r.stdout, r.stdout + r.stderr


@gpu
def test_the_default_status_word_is_the_library_s_own():
    word = sc.svdcache_gemm_fp8_status_word()
    assert word and word % 4 == 0 and word == sc.svdcache_gemm_fp8_status_word()
    assert sc.gemm_status() == sc.gemm_status("cuda:0") == sc.gemm_status(torch.device("cuda", 0)) == 0


def test_status_entries_refuse():
    assert sc.lib().svdcache_gemm_fp8_status_word(None) == -1
    assert sc.lib().svdcache_gemm_fp8_status_query(None) == -1


@gpu
def test_status_words_that_are_none(small):
    """A word on the host or of another type would be written by the kernel when a wait runs out."""
    x, a, sa, b, sb = small
    C = torch.zeros(4, 32, device=DEV)
    before = sc.svdcache_kernel_launches()
    for bad in (torch.zeros(1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32).pin_memory(), torch.zeros(1, dtype=torch.int64, device=DEV),
                torch.zeros(1, device=DEV), torch.zeros(0, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int16, device=DEV)):
        with pytest.raises(ValueError):
            sc.svdcache_gemm_fp8(a, sa, b, sb, 128, C, status=bad)
    with pytest.raises(TypeError):
        sc.svdcache_gemm_fp8(a, sa, b, sb, 128, C, status=a.data_ptr())
    assert sc.svdcache_kernel_launches() == before
    word = torch.zeros(3, dtype=torch.int32, device=DEV)
    sc.svdcache_gemm_fp8(a, sa, b, sb, 128, C, status=word[1:])
    torch.cuda.synchronize()
    assert word.tolist() == [0, 0, 0] and bool(C.isfinite().all())


@gpu
def test_whole_numbers_are_not_cut(small):
    """Arguments that would be in order modulo 2^32."""
    x, a, sa, b, sb = small
    C = torch.zeros(4, 32, device=DEV)
    before = sc.svdcache_kernel_launches()
    for wrap in (1 << 32, -(1 << 32)):
        with pytest.raises(sc.SvdCacheError):
            sc.svdcache_quantize_fp8(x, a, sa, tile_rows=1 + wrap)
        with pytest.raises(sc.SvdCacheError):
            sc.svdcache_gemm_fp8(a, sa, b, sb, 128, C, act=sc.ACT_GELU + wrap)
        with pytest.raises(ValueError):
            sc.svdcache_gemm_fp8(a, sa, b, sb, 128 + wrap, C)
    assert sc.svdcache_kernel_launches() == before


@pytest.mark.parametrize("rows,cols", [(1, (1 << 32) + 8), ((1 << 64) + 1, 8), (-(1 << 64) + 1, 8), (1, -(1 << 32) + 8)])
def test_sizes_are_not_cut(rows, cols):
    with pytest.raises(sc.SvdCacheError):
        sc.svdcache_fp8_scale_bytes(rows, cols)
