"""The product with adapters where its room, its types and its requests end, against its formula in 64 bits (bounds as in
test_adapters.py)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import check_near, np64, random_fp8
from tests.test_adapters import NONE, POOL, Pool, P, T, adapted64, cut, ints, random_pool
from tests.test_fp8_linear import check_padding, half_ulp, junk_fp8

gpu = pytest.mark.gpu
DEV = "cuda"


def least_workspace(M, rank, requests):
    """What the header names as always enough for two values."""
    return (-(-M // 256) + requests) * (-(-rank // 32) * 32768 + 1024)


def close(y, err, got, dtype):
    off = np.abs(np64(got) - y)
    bad = ~(off <= err + half_ulp(np.abs(y) + err, dtype))
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[:4].tolist()}: {off[bad][:4]} > {err[bad][:4]}"


# ------------------------------------------------------------------------------------------ workspaces ---

def test_workspaces_that_are_too_small():
    L, pool = sc.lib(), Pool(**(POOL | dict(rank=64, up_ld=64, up_stride=64 * 64, down_stride=64 * 128)))
    for M in (1, 300, 5000):
        for out in (sc.F32, sc.BF16):
            for size in (0, 256, least_workspace(M, 64, 3) // 2):
                assert L.svdcache_gemm_fp8_adapters(P, 128, P, P, 128, P, None, 0, P, 64, out, None, M, 64, 128, ctypes.byref(pool), P, P, 3, P, size, P, None) == -5


@gpu
@pytest.mark.parametrize("out", ["f32", "fp8", "bf16"])
@pytest.mark.parametrize("M,N,K,rank,requests", [(777, 1000, 1160, 24, 7), (40, 260, 700, 128, 3), (300, 700, 640, 72, 2), (4600, 1500, 328, 32, 2), (9, 130, 300, 8, 9)])
def test_the_least_workspace_holds_two_values(M, N, K, rank, requests, out):
    """Every type of output in the room that bf16 output needs: then t is within 2^-16, as it is for that."""
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    which = [i % 3 - 1 if i else 0 for i in range(requests)]
    pool = random_pool(2, rank, N, K, 3, set(which))
    starts = cut(M, requests, M)
    y, err = adapted64(a, sa, b, sb, M, N, K, None, NONE, pool, starts, which, "bf16")
    n = least_workspace(M, rank, requests)
    hold = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device=DEV)
    args = (pool, ints(starts), ints(which), hold[256:256 + n])
    if out == "fp8":
        q, s = junk_fp8(M, N)
        sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, q[:, :N], *args, S_out=s)
        check_near(q, s, y, err)
        check_padding(q, s, M, N)
    else:
        C = torch.full((M, -(-N // 8) * 8), 7.0, dtype=T[out], device=DEV)
        sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C[:, :N], *args)
        close(y, err, C[:, :N], T[out])
    assert sc.gemm_status() == 0
    assert bool((hold[:256] == 0xFF).all()) and bool((hold[-256:] == 0xFF).all())
