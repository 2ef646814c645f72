"""The 8-bit linear path around a cached block (quantiser, residual addition with RMS norm, matrix product) through the
C ABI against plain 64-bit forms, with bounds that follow from the arithmetic:

  quantiser   the input is exact in fp32, the scale a power of two: bit for bit the definition's result.
  norm        fp32: h = H + X is rounded once (2^-24); the sum of D squares is formed by fewer than 64 dependent
              additions, so it is good to 64 * 2^-24, its root to half that; mean, eps, rsqrt (2 ulp), two products
              add less than 8 * 2^-24: y is good to 2^-18 of itself.
  product     products of e4m3 values are exact; an MMA of 32 columns adds to the fp32 sum with an error of at most
              2^-22 of the sum of the magnitudes so far (the tensor core truncates): 2^-22 (K / 32 + 2 + splits) of
              sum |a b| in all.  The slope of gelu is below 1.13; its own arithmetic is good to 2^-17.
"""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import (check_exact, check_near, dequantise, gelu64, np64, random_fp8, scale_exponent, unpack)

gpu = pytest.mark.gpu
DEV = "cuda"
T = {"f32": torch.float32, "bf16": torch.bfloat16}


def features(rows, cols, dtype, seed, pad=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * torch.exp(0.7 * torch.randn(cols, generator=g))
    buf = torch.full((rows, cols + pad), float("nan")).to(T[dtype])
    buf[:, :cols] = x.to(T[dtype])
    return buf.to(DEV)[:, :cols]


def half_ulp(y, dtype):
    """Half the spacing of the type's values at |y|: 8 significant bits in bf16, 24 in fp32."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -120))) - (8.0 if dtype == torch.bfloat16 else 24.0))


def junk_fp8(rows, cols):
    """An output whose bytes, pitch and scale padding can be recognised afterwards."""
    q = torch.full((rows, -(-cols // 16) * 16 + 16), 0xA5, dtype=torch.uint8, device=DEV)
    s = torch.full((sc.svdcache_fp8_scale_bytes(rows, cols),), 0xA5, dtype=torch.uint8, device=DEV)
    return q, s


def check_padding(q, s, rows, cols):
    assert bool((q[:, cols:] == 0xA5).all()), "bytes beyond the row's end were written"
    i, j, g = -(-rows // 128), -(-cols // 512), -(-cols // 128)
    e = s.view(i, j, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(128 * i, 4 * j).clone()
    e[:rows, :g] = 0xA5
    assert bool((e == 0xA5).all()), "scales of rows or groups that do not exist were written"


# ----------------------------------------------------------------------------------------- quantiser ---

@gpu
@pytest.mark.parametrize("tile_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 15), (1, 128, 0), (3, 7, 9), (127, 130, 14), (128, 512, 0), (129, 1000, 24),
                                           (300, 641, 7), (5, 8200, 0), (1000, 64, 0), (2, 131072, 0)])
def test_quantiser_is_the_definition(rows, cols, pad, dtype, tile_rows):
    x = features(rows, cols, dtype, rows + cols, pad)
    q, s = junk_fp8(rows, cols)
    sc.svdcache_quantize_fp8(x, q, s, tile_rows=tile_rows)
    check_exact(q, s, np64(x), tile_rows)
    check_padding(q, s, rows, cols)


@gpu
@pytest.mark.parametrize("tile_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantiser_at_the_ends_of_the_range(dtype, tile_rows):
    """Zeros, powers of two around the scale's steps, the largest and smallest numbers, halves between e4m3 values,
    Inf and NaN."""
    x = torch.zeros(260, 700, dtype=torch.float32)
    for i, top in enumerate([448.0, 449.0, 447.0, 1.75, 1.7578125, 2.0 ** -126, 2.0 ** -133, 3.38e38, 1e-30, 480.0, 464.0, 1.0]):
        x[i, 0] = top
        x[i, 1:128] = top * torch.linspace(-1, 1, 127)
        x[i, 300] = -top
    x[20, 5], x[20, 6], x[20, 7] = float("inf"), float("-inf"), 3.0
    x[21, 130:258] = float("nan")
    x[22, 690:] = torch.tensor([float("nan"), 1.0, float("inf"), -2.0, 0.0, 5.0, 6.0, 7.0, 8.0, float("-inf")])
    x[23, :128] = torch.arange(128) / 8.0 + 1.0 / 16.0
    x[200, :] = torch.finfo(torch.float32).min
    if dtype == "bf16":
        x[200, :] = torch.finfo(torch.bfloat16).min
    x = x.to(T[dtype]).to(DEV)
    xp = torch.zeros(260, 704, dtype=T[dtype], device=DEV)
    xp[:, :700] = x
    q, s = junk_fp8(260, 700)
    sc.svdcache_quantize_fp8(xp[:, :700], q, s, tile_rows=tile_rows)
    check_exact(q, s, np64(x), tile_rows)


# -------------------------------------------------------------------------------------------- norm ---

def run_norm(h, x, weight, eps, keep="new"):
    rows, D = h.shape
    q, s = junk_fp8(rows, D)
    h64 = np64(h) + (np64(x) if x is not None else 0.0)
    out = None if keep is None else h if keep == "in place" else torch.full((rows, D + 8), 7.0, dtype=h.dtype, device=DEV)[:, :D]
    sc.svdcache_residual_rmsnorm_fp8(h, x, out, weight, eps, q, s)
    rms = np.sqrt((h64 * h64).mean(1, keepdims=True) + eps)
    w = np64(weight) if weight is not None else 1.0
    y = h64 / rms * w
    check_near(q, s, y, 2.0 ** -18 * np.abs(y))
    check_padding(q, s, rows, D)
    if out is not None:
        got = np64(out)
        assert (np.abs(got - h64) <= half_ulp(h64, h.dtype) * (1 + 2.0 ** -12)).all()
    return q, s


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,D,pad", [(1, 8, 0), (1, 1152, 0), (2, 120, 8), (7, 128, 0), (127, 136, 40), (128, 256, 0), (129, 1000, 24),
                                        (65, 1024, 0), (33, 2056, 8), (17, 3072, 0), (9, 4096, 0), (5, 8192, 0), (3, 12296, 8),
                                        (3, 16384, 0), (1, 16384, 0), (700, 64, 0)])
def test_norm_matches_the_formula(rows, D, pad, dtype):
    h, x = features(rows, D, dtype, 3 * D + rows, pad), features(rows, D, dtype, D, pad)
    w = (1.0 + 0.2 * torch.randn(D, generator=torch.Generator().manual_seed(D))).to(DEV)
    run_norm(h, x, w, 1e-6)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("has_x,has_w,keep", [(False, True, "new"), (True, False, "in place"), (False, False, None), (True, True, None)])
def test_norm_without_its_options(has_x, has_w, keep, dtype):
    rows, D = 37, 392
    h, x = features(rows, D, dtype, 5), features(rows, D, dtype, 6) if has_x else None
    w = torch.linspace(-2.0, 2.0, D, device=DEV) if has_w else None
    run_norm(h, x, w, 1e-5, keep)


@gpu
def test_norm_of_zero_and_of_rows_that_are_not_finite():
    rows, D = 40, 328
    h, x = features(rows, D, "f32", 1), torch.zeros(rows, D, device=DEV)
    h[3] = 0.0                                   # rms = sqrt(eps): y = 0
    h[5, 17] = float("nan")
    h[7, 300] = float("inf")                     # the mean is Inf: every finite element becomes 0, the Inf itself NaN
    x[9, 1] = float("-inf")
    h[11] = 1e-30
    q, s = junk_fp8(rows, D)
    out = torch.empty_like(h)
    sc.svdcache_residual_rmsnorm_fp8(h, x, out, None, 1e-6, q, s)
    v, e = unpack(q, s, rows, D)
    assert (v[3] == 0).all() and (e[3] == 0).all()
    assert np.isnan(v[5]).all() and (e[5] == 0).all()
    for r, c in ((7, 300), (9, 1)):
        assert np.isnan(v[r, c]) and (np.delete(v[r], c) == 0).all() and (e[r] == 0).all()
    assert bool(torch.isinf(out[9, 1])) and bool(torch.isnan(out[5, 17]))
    good = [r for r in range(rows) if r not in (3, 5, 7, 9, 11)]
    h64 = np64(h)[good]
    y = h64 / np.sqrt((h64 ** 2).mean(1, keepdims=True) + 1e-6)
    got = dequantise(q, s, rows, D)[good]
    assert (np.abs(got - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -9 * np.abs(y).max(1, keepdims=True)).all()


# ----------------------------------------------------------------------------------------- product ---

def product64(a, sa, b, sb, M, N, K, bias, act):
    """(result, bound on the kernel's error before its output is rounded), in 64 bits."""
    A, B = dequantise(a, sa, M, K), dequantise(b, sb, N, K)
    y = A @ B.T
    err = 2.0 ** -22 * (K / 32 + 2 + 8) * (np.abs(A) @ np.abs(B).T)
    if bias is not None:
        y = y + np64(bias)
        err = err + 2.0 ** -23 * (np.abs(y) + np.abs(np64(bias)))
    if act == sc.ACT_GELU:
        x = y
        y = gelu64(x)
        err = 1.13 * err + 2.0 ** -17 * np.abs(y) + 1e-30
    return y, err


def run_product(M, N, K, out, act=sc.ACT_NONE, has_bias=False, seed=0, tile_rows=128):
    a, sa = random_fp8(M, K, seed + 1)
    b, sb = random_fp8(N, K, seed + 2, tile_rows)
    bias = (20.0 * torch.randn(N, generator=torch.Generator().manual_seed(seed))).to(DEV) if has_bias else None
    y, err = product64(a, sa, b, sb, M, N, K, bias, act)
    if out == "fp8":
        q, s = junk_fp8(M, N)
        sc.svdcache_gemm_fp8(a, sa, b, sb, K, q[:, :N], S_out=s, bias=bias, act=act)
        check_near(q, s, y, err)
        check_padding(q, s, M, N)
        result = (q.clone(), s.clone())
    else:
        buf = torch.full((M, -(-N // 8) * 8 + 8), 7.0, dtype=T[out], device=DEV)
        sc.svdcache_gemm_fp8(a, sa, b, sb, K, buf[:, :N], bias=bias, act=act)
        got = np64(buf[:, :N])
        off = np.abs(got - y)
        bad = off > err + half_ulp(np.abs(y) + err, T[out])
        assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[:4].tolist()}: {got[bad][:4]} for {y[bad][:4]}"
        assert bool((buf[:, N:] == 7.0).all()), "columns beyond N were written"
        result = (buf.clone(),)
    assert sc.gemm_status(DEV) == 0
    return result


SHAPES = [(1, 1, 1), (1, 16, 32), (1, 128, 4096), (2, 1000, 96), (3, 130, 129), (8, 6912, 1152), (15, 300, 200), (16, 128, 128), (17, 100, 520),
          (32, 256, 640), (33, 257, 384), (48, 520, 1000), (64, 128, 2048), (65, 129, 513), (100, 384, 300), (128, 128, 512),
          (129, 300, 1160), (200, 1152, 777), (256, 256, 1024), (257, 513, 130), (384, 640, 256), (511, 260, 1152), (640, 2000, 384),
          (777, 1000, 1160), (1024, 768, 1152), (1500, 136, 48)]


@gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product_matches_the_formula(M, N, K):
    run_product(M, N, K, "bf16", seed=M + N)
    run_product(M, N, K, "fp8", sc.ACT_GELU, True, seed=M)


@gpu
@pytest.mark.parametrize("M,N,K", [(1, 260, 4097), (5, 64, 300), (40, 200, 1000), (130, 390, 1300), (600, 520, 640)])
@pytest.mark.parametrize("out", ["f32", "bf16", "fp8"])
@pytest.mark.parametrize("act", [sc.ACT_NONE, sc.ACT_GELU])
@pytest.mark.parametrize("has_bias", [False, True])
def test_product_with_every_epilogue(M, N, K, out, act, has_bias):
    run_product(M, N, K, out, act, has_bias, seed=K, tile_rows=1)


# few tiles and a long sum, so that 3, 4, 6 or 8 CTAs share a tile of 16, 32, 64 or 128 rows, evenly or not
@gpu
@pytest.mark.parametrize("M,N,K", [(3, 130, 1100), (11, 130, 1540), (16, 260, 2000), (20, 130, 800), (31, 130, 1540), (32, 400, 2100), (50, 130, 800),
                                   (64, 130, 1540), (100, 2100, 1100), (100, 2100, 6000), (200, 1500, 4100), (193, 2500, 2600), (260, 130, 2000)])
def test_product_of_tiles_that_ctas_share(M, N, K):
    run_product(M, N, K, "f32", seed=N + K)
    run_product(M, N, K, "fp8", sc.ACT_GELU, True, seed=N)


@gpu
@pytest.mark.parametrize("out", ["bf16", "fp8"])
def test_product_at_the_widths_of_the_streams(out):
    run_product(2048, 1152, 4608, out, sc.ACT_NONE, True)
    run_product(1024, 3072, 3072, out, sc.ACT_GELU, True)


@gpu
@pytest.mark.parametrize("M,N,K", [(9200, 1400, 200), (4600, 1500, 328), (5000, 2300, 129), (20000, 300, 640)])
def test_product_of_many_tiles_per_cluster(M, N, K):
    """Every width of tile over several rounds, with a last column tile that ends in each part of it."""
    run_product(M, N, K, "bf16", sc.ACT_NONE, True, seed=1)
    run_product(M, N, K, "fp8", sc.ACT_GELU, True, seed=2)


@gpu
@pytest.mark.parametrize("M", [4, 700])
def test_nan_codes_stay_in_their_row_and_column(M):
    N, K = 300, 700
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    a[2, 699] = 0x7F
    b[150, 0] = 0xFF
    C = torch.empty(M, 304, dtype=torch.float32, device=DEV)[:, :N]
    sc.svdcache_gemm_fp8(a, sa, b, sb, K, C)
    want = np.zeros((M, N), bool)
    want[2], want[:, 150] = True, True
    np.testing.assert_array_equal(np.isnan(np64(C)), want)
    q, s = junk_fp8(M, N)
    sc.svdcache_gemm_fp8(a, sa, b, sb, K, q[:, :N], S_out=s)
    v, _ = unpack(q, s, M, N)
    np.testing.assert_array_equal(np.isnan(v), want)


@gpu
@pytest.mark.parametrize("M,N,K", [(1, 640, 4096), (96, 512, 1024), (700, 1000, 1160)])
def test_results_do_not_change_from_run_to_run(M, N, K):
    for out in ("f32", "fp8"):
        first = run_product(M, N, K, out, seed=3)
        for _ in range(3):
            assert all(torch.equal(x, y) for x, y in zip(first, run_product(M, N, K, out, seed=3)))


@gpu
def test_no_rows_launch_nothing():
    n = sc.svdcache_kernel_launches()
    q, s = torch.empty(0, 256, dtype=torch.uint8, device=DEV), torch.empty(0, dtype=torch.uint8, device=DEV)
    h = torch.empty(0, 256, dtype=torch.bfloat16, device=DEV)
    sc.svdcache_quantize_fp8(h, q, s)
    sc.svdcache_residual_rmsnorm_fp8(h, h, h, None, 1e-6, q, s)
    b, sb = random_fp8(64, 256, 1)
    sc.svdcache_gemm_fp8(q, s, b, sb, 256, torch.empty(0, 64, dtype=torch.bfloat16, device=DEV))
    assert sc.svdcache_kernel_launches() == n


@gpu
def test_chain_on_another_stream_and_in_a_graph():
    """norm -> product with gelu and 8-bit output -> product, on a side stream, then replayed from a CUDA graph on new
    inputs: both equal the same calls made one by one on the default stream."""
    M, D, F = 200, 384, 1024
    w1, s1 = random_fp8(F, D, 3, 128, spread=0.0)
    w2, s2 = random_fp8(D, F, 4, 128, spread=0.0)
    bias = torch.randn(F, device=DEV)
    h, x = features(M, D, "bf16", 1), features(M, D, "bf16", 2)
    q, qs = sc.new_fp8(M, D)
    u, us = sc.new_fp8(M, F)
    y, h2 = torch.empty(M, D, dtype=torch.bfloat16, device=DEV), torch.empty_like(h)

    def chain():
        sc.svdcache_residual_rmsnorm_fp8(h, x, h2, None, 1e-6, q, qs)
        sc.svdcache_gemm_fp8(q, qs, w1, s1, D, u, S_out=us, bias=bias, act=sc.ACT_GELU)
        sc.svdcache_gemm_fp8(u, us, w2, s2, F, y)

    chain()
    torch.cuda.synchronize()
    ref = y.clone()
    assert bool(ref.isfinite().all()) and float(ref.float().abs().max()) > 0
    y.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain()
    side.synchronize()
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    x.copy_(features(M, D, "bf16", 9))
    graph.replay()
    torch.cuda.synchronize()
    got = y.clone()
    chain()
    torch.cuda.synchronize()
    assert torch.equal(got, y) and not torch.equal(got, ref)
    assert sc.gemm_status(DEV) == 0


@gpu
def test_graph_with_two_branches():
    """Two products on two streams, joined by a norm, a memset before and a copy after, captured and replayed."""
    M, D = 300, 512
    a, sa = random_fp8(M, D, 1, spread=0.0)
    w = [random_fp8(D, D, 2 + i, 128, spread=0.0) for i in range(2)]
    y = [torch.zeros(M, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q, qs = sc.new_fp8(M, D)
    h, last = torch.empty_like(y[0]), torch.empty_like(y[0])
    side = torch.cuda.Stream()

    def work():
        y[0].zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            sc.svdcache_gemm_fp8(a, sa, *w[1], D, y[1])
        sc.svdcache_gemm_fp8(a, sa, *w[0], D, y[0])
        torch.cuda.current_stream().wait_stream(side)
        sc.svdcache_residual_rmsnorm_fp8(y[0], y[1], h, None, 1e-6, q, qs)
        last.copy_(h)

    work()
    torch.cuda.synchronize()
    want = [t.clone() for t in (*y, h, q, qs, last)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for t in (*y, h, q, qs, last):
            t.fill_(1)
        qs.zero_(), q.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, u) for t, u in zip((*y, h, q, qs, last), want))


@gpu
def test_offsets_beyond_32_bits():
    """4.5 GB of rows: the norm in place, the quantiser, and a product with 4.5 GB of output, at rows on either side of
    the places where a 32-bit byte or element offset would wrap, and the last ones."""
    M, D, N = 280000, 8192, 8192
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    h = torch.randn(M, D, generator=g, device=DEV, dtype=torch.bfloat16)
    rows = torch.tensor([0, 1, 131071, 131072, 131073, 262143, 262144, 262145, M - 2, M - 1], device=DEV)
    before = np64(h[rows])
    q, s = sc.new_fp8(M, D)
    sc.svdcache_residual_rmsnorm_fp8(h, None, h, None, 1e-6, q, s)
    np.testing.assert_array_equal(np64(h[rows]), before)
    y = before / np.sqrt((before ** 2).mean(1, keepdims=True) + 1e-6)
    v = unpack_rows(q, s, M, D, rows)
    assert (np.abs(v - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -8).all()
    sc.svdcache_quantize_fp8(h, q, s)
    a = unpack_rows(q, s, M, D, rows)
    assert (np.abs(a - before) <= 2.0 ** -4 * np.abs(before) + 2.0 ** -8).all()
    del h
    b, sb = random_fp8(N, D, 3, 128, spread=0.0)
    C = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    sc.svdcache_gemm_fp8(q, s, b, sb, D, C)
    B = dequantise(b, sb, N, D)
    want = a @ B.T
    err = 2.0 ** -22 * (D / 32 + 10) * (np.abs(a) @ np.abs(B).T)
    assert (np.abs(np64(C[rows]) - want) <= err + half_ulp(np.abs(want) + err, torch.bfloat16)).all()
    assert sc.gemm_status(DEV) == 0


def unpack_rows(q, s, M, D, rows):
    """What the given rows of an 8-bit matrix stand for."""
    v = q[rows, :D].view(torch.float8_e4m3fn).double()
    e = sc.fp8_scale_exponents(s, M, D)[rows].double() - 127.0
    return (v * torch.exp2(e).repeat_interleave(128, 1)[:, :D]).cpu().numpy()


# ----------------------------------------------------------------------------- refusals (host only) ---

INVALID, SHAPE, ALIGN = -1, -2, -3
P = 1 << 20      # a 16-byte aligned address that nothing reads: every call below is refused before a launch


def _raw(name, base, **change):
    args = dict(base, **change)
    return getattr(sc.lib(), name)(*args.values())


def test_scale_buffer_size():
    assert sc.svdcache_fp8_scale_bytes(1, 1) == 512
    assert sc.svdcache_fp8_scale_bytes(128, 512) == 512
    assert sc.svdcache_fp8_scale_bytes(129, 513) == 4 * 512
    assert sc.svdcache_fp8_scale_bytes(0, 8) == 0
    assert sc.svdcache_fp8_scale_bytes(118800, 3072) == 929 * 6 * 512
    out = ctypes.c_size_t(0)
    L = sc.lib()
    assert L.svdcache_fp8_scale_bytes(-1, 8, ctypes.byref(out)) == SHAPE
    assert L.svdcache_fp8_scale_bytes(1, 0, ctypes.byref(out)) == SHAPE
    assert L.svdcache_fp8_scale_bytes(1, 131073, ctypes.byref(out)) == SHAPE
    assert L.svdcache_fp8_scale_bytes(1 << 31, 8, ctypes.byref(out)) == SHAPE
    assert L.svdcache_fp8_scale_bytes(1, 8, None) == INVALID


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), INVALID), (dict(tile_rows=64), INVALID), (dict(rows=-1), SHAPE), (dict(cols=0), SHAPE), (dict(cols=200000), SHAPE),
    (dict(X=None), INVALID), (dict(Q=None), INVALID), (dict(S=None), INVALID), (dict(ld=99), SHAPE), (dict(ldq=99), SHAPE),
    (dict(ld=101), ALIGN), (dict(ldq=120), ALIGN), (dict(X=P + 8), ALIGN), (dict(Q=P + 1), ALIGN), (dict(S=P + 4), ALIGN), (dict(rows=0), 0)])
def test_quantiser_refuses(change, code):
    base = dict(X=P, rows=4, cols=100, ld=104, dtype=1, tile_rows=1, Q=P, ldq=112, S=P, stream=None)
    assert _raw("svdcache_quantize_fp8", base, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(dtype=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(rows=-1), SHAPE), (dict(D=100), SHAPE),
    (dict(D=16392, ldh=16392, ldx=16392, ldo=16392, ldq=16400), SHAPE), (dict(D=0), SHAPE), (dict(H=None), INVALID), (dict(Q=None), INVALID),
    (dict(S=None), INVALID), (dict(ldh=96), SHAPE), (dict(ldx=96), SHAPE), (dict(ldo=96), SHAPE), (dict(ldq=96), SHAPE), (dict(ldh=105), ALIGN),
    (dict(ldx=106), ALIGN), (dict(ldo=108), ALIGN), (dict(ldq=104), ALIGN), (dict(H=P + 2), ALIGN), (dict(X=P + 8), ALIGN), (dict(H_out=P + 4), ALIGN),
    (dict(weight=P + 4), ALIGN), (dict(Q=P + 8), ALIGN), (dict(S=P + 8), ALIGN), (dict(rows=0), 0)])
def test_norm_refuses(change, code):
    base = dict(H=P, ldh=104, X=P, ldx=104, H_out=P, ldo=104, weight=P, eps=1e-6, Q=P, ldq=112, S=P, rows=4, D=104, dtype=1, stream=None)
    assert _raw("svdcache_residual_rmsnorm_fp8", base, **change) == code


@pytest.mark.parametrize("change,code", [
    (dict(act=2), INVALID), (dict(act=-1), INVALID), (dict(out=3), INVALID), (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE),
    (dict(N=131073), SHAPE), (dict(K=131073), SHAPE), (dict(M=(1 << 31) - 256), SHAPE), (dict(status=None), INVALID), (dict(status=P + 2), ALIGN),
    (dict(bias=P + 1), ALIGN), (dict(A=None), INVALID), (dict(B=None), INVALID), (dict(C=None), INVALID), (dict(SA=None), INVALID),
    (dict(SB=None), INVALID), (dict(out=2, SC=None, ldc=80), INVALID), (dict(lda=99), SHAPE), (dict(ldb=99), SHAPE), (dict(ldc=63), SHAPE),
    (dict(lda=104), ALIGN), (dict(ldb=104), ALIGN), (dict(ldc=68), ALIGN), (dict(out=2, ldc=72, SC=P), ALIGN), (dict(A=P + 8), ALIGN), (dict(B=P + 8), ALIGN),
    (dict(C=P + 8), ALIGN), (dict(SA=P + 8), ALIGN), (dict(SB=P + 8), ALIGN), (dict(out=2, ldc=64, SC=P + 8), ALIGN), (dict(M=0, status=None), 0)])
def test_product_refuses(change, code):
    base = dict(A=P, lda=112, SA=P, B=P, ldb=112, SB=P, bias=None, act=0, C=P, ldc=64, out=1, SC=None, M=4, N=64, K=100, status=P, stream=None)
    assert _raw("svdcache_gemm_fp8", base, **change) == code


def test_binding_refuses_what_the_library_cannot_see():
    x = torch.zeros(4, 128)
    q, s = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(ValueError):
        sc.svdcache_quantize_fp8(x, q, s)                       # not on the device
    if not torch.cuda.is_available():
        return
    x, q, s = x.to(DEV), q.to(DEV), s.to(DEV)
    for args in ((x, q[:3], s), (x, q[:, :100], s), (x, q.float(), s), (x, q, s[:511]), (x.t(), q, s), (x, q, s.float())):
        with pytest.raises(ValueError):
            sc.svdcache_quantize_fp8(*args)
    h = x.bfloat16()
    for args in ((h, x, None, None), (h, h[:, :64], None, None), (h, None, x, None), (h, None, None, x[0].bfloat16()), (h, None, None, x[0, :64])):
        with pytest.raises(ValueError):
            sc.svdcache_residual_rmsnorm_fp8(*args, 1e-6, q, s)
    C = torch.zeros(4, 4, device=DEV)
    for kw in (dict(bias=torch.zeros(3, device=DEV)), dict(bias=torch.zeros(4, device=DEV).half())):
        with pytest.raises(ValueError):
            sc.svdcache_gemm_fp8(q, s, q, s, 128, C, **kw)
    for args in ((q, s, q, s, 200, C), (q, s, q, s, 128, C[:2]), (q, s, q[:2], s, 128, C), (q, s, q, s, 128, torch.zeros(4, 16, device=DEV).byte())):
        with pytest.raises(ValueError):
            sc.svdcache_gemm_fp8(*args)


def test_reference_rounding_of_the_tests():
    """The 64-bit form itself: hand-picked values."""
    assert scale_exponent(np.array([448.0, 448.1, 224.0, 1.75, 0.0])).tolist() == [0.0, 1.0, -1.0, -8.0, 0.0]
    from tests.fp8_util import e4m3_round, e4m3_values
    assert e4m3_round(np.array([17.0, 19.0, 0.001, 2.0 ** -10, 3 * 2.0 ** -10, 447.0])).tolist() == [16.0, 20.0, 2.0 ** -9, 0.0, 2.0 ** -8, 448.0]
    b = np.arange(256, dtype=np.uint8)
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(e4m3_values(b), want)
