"""The time-out exits of the product's kernels: every wait runs out (about a millisecond; nothing is loaded, so nothing is in
flight), the kernel returns with its status in the given word and nowhere else, and the next product is right.  Nothing here
faults or hangs."""
import ctypes
import time

import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import random_fp8
from tests.test_fp8_linear import T
from tests.test_fp8_plans import run_plan

gpu = pytest.mark.gpu
DEV = "cuda"
LIMIT = 2_000_000      # cycles: about 1 ms


@gpu
@pytest.mark.parametrize("M,N,K,out,plan", [
    (5, 300, 4100, "bf16", (0, 16, 1)), (5, 300, 4100, "bf16", (0, 16, 8)), (30, 130, 1540, "f32", (0, 32, 6)), (190, 400, 4100, "fp8", (0, 64, 3)),
    (128, 900, 3000, "f32", (0, 128, 2)), (3000, 900, 300, "bf16", (0, 64, 1)), (5, 70, 300, "f32", (1, 128, 2)), (700, 520, 2100, "bf16", (1, 192, 2)),
    (700, 520, 2100, "fp8", (1, 256, 2)), (20000, 300, 200, "fp8", (1, 128, 2)), (9000, 1093, 40, "f32", (1, 192, 2))])
def test_waits_that_run_out_are_reported_and_the_device_stays_usable(M, N, K, out, plan):
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    status = torch.zeros(3, dtype=torch.int32, device=DEV)
    if out == "fp8":
        C, S = sc.new_fp8(M, N)
    else:
        C, S = torch.zeros(M, -(-N // 8) * 8, dtype=T[out], device=DEV), None
    torch.cuda.synchronize()
    t0 = time.monotonic()
    sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, C[:, :N], plan, S_out=S, status=status[1:2], limit_cycles=LIMIT)
    torch.cuda.synchronize()
    assert time.monotonic() - t0 < 5.0
    assert status.tolist() == [0, -6, 0] and sc.gemm_status(DEV) == 0
    run_plan(M, N, K, out, plan, sc.ACT_NONE, True)
    # sticky: an ordinary product with the same word leaves it
    sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, C[:, :N], plan, S_out=S, status=status[1:2])
    assert status.tolist() == [0, -6, 0]


def test_limits_that_are_refused():
    P, plan = 1 << 20, (ctypes.c_int32 * 3)(0, 16, 1)      # nothing reads the address
    args = [P, 112, P, P, 112, P, None, 0, P, 64, 1, None, 4, 64, 100, P, plan]
    for limit in (-1, 200_000_001, 10 ** 12):
        assert sc.lib().svdcache_selftest_gemm_fp8(*args, limit, None) == -1
