"""Products whose tiles are shared by the CTAs of a cluster, in company: a CTA's sums travel to the others' shared memory,
and its own may be taken by another kernel's CTA as soon as it leaves.  Results have to be, bit for bit, those of the same
product alone, whatever follows on the same stream (kernels that start early) or runs on others."""
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import check_near, random_fp8
from tests.test_fp8_linear import product64

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("M,N,K,plan", [(1, 128, 9216, (0, 16, 8)), (11, 130, 1540, (0, 16, 6)), (31, 300, 4100, (0, 32, 4)), (64, 130, 6000, (0, 64, 8)),
                                        (64, 400, 6000, (0, 64, 2)), (100, 2100, 6000, (0, 128, 6)), (128, 900, 3000, (0, 128, 2)), (250, 400, 9000, (0, 64, 3))])
def test_shared_tiles_in_company(M, N, K, plan):
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    pitch = -(-N // 16) * 16

    def product(C, S, stream=None):
        sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, C[:, :N], plan, S_out=S, stream=stream)

    want, want_s = sc.new_fp8(M, N)
    product(want, want_s)
    torch.cuda.synchronize()
    y, err = product64(a, sa, b, sb, M, N, K, None, sc.ACT_NONE)
    check_near(want, want_s, y, err)

    # what the others do: rows through shared memory, and products whose own rings and sums are all NaN
    x = torch.full((4096, 1024), float("nan"), dtype=torch.bfloat16, device=DEV)
    nan, nan_s = sc.new_fp8(4096, 1024)
    sc.svdcache_quantize_fp8(x, nan, nan_s)
    assert bool((nan & 0x7F == 0x7F).all())
    few, few_s = nan[:40], nan_s
    junk = [torch.empty(40, 4096, dtype=torch.float32, device=DEV) for _ in range(3)]
    runs, streams = 60, [torch.cuda.Stream() for _ in range(3)]
    out = torch.zeros(3, runs, M, pitch, dtype=torch.uint8, device=DEV)
    out_s = torch.zeros(3, runs, want_s.numel(), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for i in range(runs):
        for j, s in enumerate(streams):
            product(out[j, i], out_s[j, i], s)
            sc.svdcache_gemm_fp8(few, few_s, nan, nan_s, 1024, junk[j], stream=s)
    torch.cuda.synchronize()
    assert bool((out == want).all()) and bool((out_s == want_s).all())
    assert all(bool(t.isnan().all()) for t in junk)
    assert sc.gemm_status(DEV) == 0
