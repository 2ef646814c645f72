"""Every kernel and tile that a product may be taken by, whichever the model of their times prefers today: tiles of 16 to 128
rows with K shared by 1 to 8 CTAs, pairs of CTAs at each width and type, in one round of tiles and in several, at sizes that
end inside tiles, groups and pieces of scales.  Bounds as in test_fp8_linear.py (product64)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import check_near, np64, random_fp8
from tests.test_fp8_linear import T, check_padding, half_ulp, junk_fp8, product64

gpu = pytest.mark.gpu
DEV = "cuda"
OUT = {"f32": sc.F32, "bf16": sc.BF16, "fp8": sc.FP8}


def run_plan(M, N, K, out, plan, act, has_bias, tile_rows=128):
    a, sa = random_fp8(M, K, M + 1)
    b, sb = random_fp8(N, K, N + 2, tile_rows)
    bias = (20.0 * torch.randn(N, generator=torch.Generator().manual_seed(K))).to(DEV) if has_bias else None
    y, err = product64(a, sa, b, sb, M, N, K, bias, act)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    if out == "fp8":
        q, s = junk_fp8(M, N)
        sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, q[:, :N], plan, S_out=s, bias=bias, act=act, status=status)
        check_near(q, s, y, err)
        check_padding(q, s, M, N)
    else:
        buf = torch.full((M, -(-N // 8) * 8 + 8), 7.0, dtype=T[out], device=DEV)
        sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, buf[:, :N], plan, bias=bias, act=act, status=status)
        off = np.abs(np64(buf[:, :N]) - y)
        bad = off > err + half_ulp(np.abs(y) + err, T[out])
        assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[:4].tolist()}"
        assert bool((buf[:, N:] == 7.0).all()), "columns beyond N were written"
    assert int(status.item()) == 0


ROWS = {16: [1, 7, 16], 32: [17, 32], 64: [33, 64, 193], 128: [65, 128, 300]}


@gpu
@pytest.mark.parametrize("splits", [1, 2, 3, 4, 6, 8])
@pytest.mark.parametrize("tile_m", [16, 32, 64, 128])
def test_tiles_of_every_height_shared_by_every_number_of_ctas(tile_m, splits):
    for M in ROWS[tile_m]:
        run_plan(M, 261, 2100, "f32", (0, tile_m, splits), sc.ACT_NONE, False)      # 17 groups: no two CTAs' shares need be alike
        run_plan(M, 130, 2048, "fp8", (0, tile_m, splits), sc.ACT_GELU, True)
        run_plan(M, 20, 128 * 2 * splits - 100, "bf16", (0, tile_m, splits), sc.ACT_NONE, True, tile_rows=1)   # the fewest groups


@gpu
@pytest.mark.parametrize("M,N,K", [(9, 40000, 70), (31, 25000, 140), (3000, 900, 300), (2900, 1700, 129)])
def test_more_tiles_than_the_device_runs_at_once(M, N, K):
    tile_m = 16 if M <= 16 else 32 if M <= 32 else 64
    for size in {tile_m, 128 if M > 64 else tile_m}:
        run_plan(M, N, K, "bf16", (0, size, 1), sc.ACT_NONE, True)
        run_plan(M, N, K, "fp8", (0, size, 1), sc.ACT_GELU, False)


PAIR_SIZES = [("f32", 128), ("f32", 192), ("bf16", 128), ("bf16", 192), ("fp8", 128), ("fp8", 256)]


@gpu
@pytest.mark.parametrize("out,bn", PAIR_SIZES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (5, 70, 300), (257, 513, 130), (700, 520, 2100)])
def test_pairs_in_one_round(M, N, K, out, bn):
    run_plan(M, N, K, out, (1, bn, 2), sc.ACT_NONE, True)
    run_plan(M, N, K, out, (1, bn, 2), sc.ACT_GELU, False, tile_rows=1)


@gpu
@pytest.mark.parametrize("out,bn", PAIR_SIZES)
@pytest.mark.parametrize("M,N,K", [(4600, 1500, 328), (20000, 300, 200), (9000, 1093, 40)])
def test_pairs_in_several_rounds(M, N, K, out, bn):
    clusters = torch.cuda.get_device_properties(0).multi_processor_count // 2
    assert -(-M // 256) * -(-N // bn) > clusters
    run_plan(M, N, K, out, (1, bn, 2), sc.ACT_GELU, True)


@gpu
@pytest.mark.parametrize("act", [sc.ACT_NONE, sc.ACT_GELU])
@pytest.mark.parametrize("M,N,K,plan", [(3, 300, 1540, (0, 16, 1)), (40, 300, 1540, (0, 64, 3)), (200, 300, 2100, (0, 128, 8)), (300, 300, 200, (1, 128, 2)),
                                        (300, 300, 200, (1, 256, 2))])
def test_infinities_in_an_8_bit_output(M, N, K, plan, act):
    """Inf and NaN become the NaN code and stay with their element; their group's scale is that of its finite values."""
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    bias = torch.randn(N, generator=torch.Generator().manual_seed(1))
    bias[5], bias[130], bias[131], bias[299] = float("inf"), float("-inf"), float("nan"), float("inf")
    bias = bias.to(DEV)
    with np.errstate(invalid="ignore"):
        y, err = product64(a, sa, b, sb, M, N, K, bias, act)
    q, s = junk_fp8(M, N)
    sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, q[:, :N], plan, S_out=s, bias=bias, act=act)
    check_near(q, s, y, err)
    check_padding(q, s, M, N)


@gpu
@pytest.mark.parametrize("M,N,K,out", [(1, 640, 4096, "bf16"), (24, 6724, 9381, "bf16"), (100, 2100, 6000, "fp8"), (959, 7366, 3318, "f32"),
                                       (2048, 1152, 1152, "fp8"), (40, 512, 100, "bf16")])
def test_a_product_is_taken_by_the_plan_that_is_told(M, N, K, out):
    plan = sc.svdcache_gemm_fp8_plan(M, N, K, OUT[out])
    pairs, size, ctas, rounds = plan
    assert rounds >= 1 and ((pairs, ctas) == (1, 2) or pairs == 0)
    a, sa = random_fp8(M, K, 0)      # seeds that are multiples of 3: rows as far apart as the plan takes them to be
    b, sb = random_fp8(N, K, 3, 128)
    got = []
    for by in (lambda C, S: sc.svdcache_gemm_fp8(a, sa, b, sb, K, C, S_out=S), lambda C, S: sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, C, plan, S_out=S)):
        if out == "fp8":
            q, s = junk_fp8(M, N)
            by(q[:, :N], s)
            got.append((q, s))
        else:
            C = torch.full((M, -(-N // 8) * 8), 7.0, dtype=T[out], device=DEV)
            by(C[:, :N], None)
            got.append((C,))
    assert all(torch.equal(x, y) for x, y in zip(*got))


@gpu
@pytest.mark.parametrize("M,N,K,out,plan", [
    (17, 128, 1024, "bf16", (0, 16, 1)), (16, 128, 1024, "bf16", (0, 32, 1)), (65, 128, 1024, "bf16", (0, 32, 1)), (64, 128, 1024, "bf16", (0, 128, 1)),
    (64, 128, 1024, "bf16", (0, 48, 1)), (64, 128, 1024, "bf16", (0, 64, 5)), (64, 128, 1024, "bf16", (0, 64, 0)), (64, 128, 1024, "bf16", (0, 64, 8)),
    (64, 128, 384, "bf16", (0, 64, 2)), (64, 30000, 2048, "bf16", (0, 64, 2)), (300, 128, 1024, "bf16", (1, 256, 2)), (300, 128, 1024, "fp8", (1, 192, 2)),
    (300, 128, 1024, "f32", (1, 64, 2)), (300, 128, 1024, "f32", (1, 128, 1))])
def test_plans_that_no_product_of_the_size_may_be_taken_by(M, N, K, out, plan):
    a, sa = random_fp8(M, K, 0)
    b, sb = random_fp8(N, K, 3)
    C = torch.zeros(M, N, dtype=T.get(out, torch.uint8), device=DEV)
    before = sc.svdcache_kernel_launches()
    with pytest.raises(sc.SvdCacheError) as e:
        sc.svdcache_selftest_gemm_fp8(a, sa, b, sb, K, C, plan, S_out=sc.new_fp8(M, N)[1])
    assert e.value.code == -1 and sc.svdcache_kernel_launches() == before


def test_plan_entries_refuse():
    L, plan = sc.lib(), (ctypes.c_int32 * 4)()
    ask = lambda M=4, N=64, K=100, lda=112, ldb=112, out=1, p=plan: L.svdcache_gemm_fp8_plan(M, N, K, lda, ldb, out, p)  # noqa: E731
    assert ask(p=None) == -1 and ask(out=3) == -1
    assert ask(M=0) == -2 and ask(M=-1) == -2 and ask(N=0) == -2 and ask(K=131073) == -2 and ask(lda=99) == -2 and ask(ldb=99) == -2
    P = 1 << 20      # nothing reads it
    args = [P, 112, P, P, 112, P, None, 0, P, 64, 1, None, 4, 64, 100, P]
    assert L.svdcache_selftest_gemm_fp8(*args, None, 0, None) == -1
    assert L.svdcache_selftest_gemm_fp8(*args[:1], 104, *args[2:], plan, 0, None) == -3
