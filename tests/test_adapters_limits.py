"""The product with adapters where its room, its types and its requests end, against its formula in 64 bits (bounds as in
test_adapters.py)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2601_07396_b200 import binding as sc
from tests.fp8_util import check_near, dequantise, np64, random_fp8
from tests.test_adapters import NONE, POOL, Pool, P, T, adapted64, cut, ints, random_pool, run
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
@pytest.mark.parametrize("M,N,K,rank,requests", [(777, 1000, 1160, 24, 7), (40, 260, 700, 128, 3), (300, 700, 640, 72, 2), (4600, 1500, 328, 32, 2), (9, 130, 300, 8, 9),
                                                    (9200, 260, 330, 32, 3), (9200, 260, 330, 120, 60), (1025, 700, 530, 64, 4), (257, 1000, 2100, 48, 1), (1500, 300, 200, 64, 700)])
def test_the_least_workspace_holds_two_values(M, N, K, rank, requests, out):
    """Every type of output in the room that bf16 output needs: t is within 2^-16 for 8-bit output, as it is for that, and for fp32 output
    within 2^-24 all the same."""
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    which = [i % 3 - 1 if i else 0 for i in range(requests)]
    pool = random_pool(2, rank, N, K, 3, set(which))
    starts = cut(M, requests, M)
    y, err = adapted64(a, sa, b, sb, M, N, K, None, NONE, pool, starts, which, "f32" if out == "f32" else "bf16")
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


@gpu
def test_bands_of_rows_in_a_graph():
    """fp32 output in the least workspace by several launches, captured once and replayed for other requests, twice on two streams at once."""
    M, N, K, rank, requests = 9200, 264, 520, 32, 2
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    pool = random_pool(3, rank, N, K, 3, {0, 1, 2})
    plans = [([0, 4000, M], [0, 1]), ([0, 3071, 3073], [2, 0]), ([9000, 9100, 9199], [1, 2]), ([4607, 4608, 4609], [0, 2])]
    lanes = []
    for _ in range(2):
        C, ws = torch.zeros(M, N, device=DEV), torch.full((least_workspace(M, rank, requests),), 0xFF, dtype=torch.uint8, device=DEV)
        start, which, stream = ints(plans[0][0]), ints(plans[0][1]), torch.cuda.Stream()
        torch.cuda.synchronize()
        before = sc.svdcache_kernel_launches()
        sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C, pool, start, which, ws, stream=stream)
        assert sc.svdcache_kernel_launches() - before >= 4          # two of each band
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C, pool, start, which, ws)
        lanes.append((C, start, which, stream, graph))
    for i in range(len(plans)):
        now = [plans[(i + j) % len(plans)] for j in range(2)]
        for (C, start, which, stream, graph), (s, w) in zip(lanes, now):
            C.zero_()
            start.copy_(ints(s))
            which.copy_(ints(w))
        torch.cuda.synchronize()
        for C, start, which, stream, graph in lanes:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for (C, *_), (s, w) in zip(lanes, now):
            y, err = adapted64(a, sa, b, sb, M, N, K, None, NONE, pool, s, w, "f32")
            close(y, err, C, torch.float32)
    assert sc.gemm_status() == 0


# ---------------------------------------------------------------------- tensor memory and shared memory ---

SM_BYTES, SM_COLUMNS = 228 * 1024, 512
PLANS = [(0, t, s) for t in (16, 32, 64, 128) for s in (1, 2, 3, 4, 6, 8)] + [(1, n, 2) for n in (128, 192, 256)]


def launches(shapes):
    """((CTAs, of a cluster, columns, bytes) of each kernel) of every rank and plan."""
    for M, N, K, requests in shapes:
        for rank in range(8, 129, 8):
            for plan in PLANS:
                if not plan[0] and -(-K // 128) < 2 * plan[2] > 2:            # a shared tile gives each CTA two groups of K
                    continue
                for out in (sc.F32, sc.BF16):
                    for brief in (False, True):
                        yield (M, N, K, requests, rank, plan), sc.svdcache_selftest_adapters_sizes(M, N, K, rank, requests, out, plan, brief)


def test_no_set_of_ctas_that_fit_an_sm_asks_for_more_tensor_memory_than_it_has():
    """An SM starts CTAs by their shared memory; tcgen05.alloc waits without a limit where columns are short, and CTAs of clusters wait for one
    another while they hold theirs.  So no CTAs of any of these kernels, on any streams, may fit together with more than 512."""
    least = {}                                            # columns -> the least bytes that a CTA asks for with them
    clusters = set()
    shapes = [(M, 512, K, requests) for M in (1, 16, 40, 64, 100, 512, 5000) for K in (1, 128, 129, 300, 520, 1100, 2048, 6300, 40000) for requests in (1, 3, 64, 300)]
    for which, sizes in launches(shapes):
        for ctas, cluster, columns, shared in sizes:
            assert columns in (64, 128, 256, 512) and 0 < shared <= 227 * 1024 and ctas % cluster == 0, which
            least[columns] = min(least.get(columns, shared), shared)
        clusters.add(sizes[0][1])
    assert clusters == {1, 2, 4, 8} and set(least) == {64, 128, 256, 512}
    # the fewest bytes that hold more columns than an SM has, of any mixture
    need = {0: 0}
    for n in range(1, SM_COLUMNS // 64 + 2):
        need[n] = min(least[c] + need[max(n - c // 64, 0)] for c in least)
    assert need[SM_COLUMNS // 64 + 1] > SM_BYTES, least


def test_shared_tasks_of_the_narrow_product_are_no_more_than_sms():
    for (M, N, K, requests, rank, plan), (narrow, _) in launches([(64, 512, 2048, 64), (512, 256, 2048, 128), (40, 512, 9000, 1), (5000, 512, 40000, 3)]):
        rows = 256 if plan[0] else plan[1]
        tasks = -(-M // rows) * (2 if plan[0] else 1) + requests - 1
        assert narrow[1] == 1 or tasks * narrow[1] <= 148, (M, N, K, requests, rank, plan)


def test_ctas_of_the_narrow_product_fit_beside_the_projection_s():
    """Small tiles that no CTAs share begin beside it; 2 KB are what the system takes, 2 KB the kernels' own."""
    for which, (narrow, projection) in launches([(1, 512, 3000, 1), (64, 512, 20000, 64), (100, 512, 700, 8)]):
        if which[-1][0] == 0 and which[-1][2] == 1:
            assert narrow[3] + projection[3] + 4096 <= SM_BYTES, which


MANY = [(64, 512, 2048, 128, 64, "f32"), (512, 256, 2048, 64, 128, "bf16"), (130, 300, 1100, 104, 130, "fp8"), (16, 260, 4100, 128, 16, "bf16"), (600, 520, 1300, 128, 100, "f32")]


@gpu
@pytest.mark.parametrize("M,N,K,rank,requests,out", MANY)
def test_wide_adapters_of_many_requests(M, N, K, rank, requests, out):
    run(M, N, K, rank, cut(M, requests, rank), [i * 5 % 9 - 1 for i in range(requests)], 8, out, NONE, True, seed=M)


@gpu
def test_wide_adapters_of_many_requests_on_several_streams():
    """Each call is bit for bit what it is alone, among others whose CTAs hold as much tensor memory."""
    jobs = []
    for i, (M, N, K, rank, requests, out) in enumerate(MANY):
        a, sa = random_fp8(M, K, i)
        b, sb = random_fp8(N, K, i + 10, 128)
        pool = random_pool(8, rank, N, K, i, set(range(8)))
        jobs.append((a, sa, b, sb, K, pool, ints(cut(M, requests, rank)), ints([j % 9 - 1 for j in range(requests)])))
    x, plain, side = random_fp8(64, 2048, 5), random_fp8(300, 2048, 6, 128), torch.zeros(64, 304, device=DEV)

    def make():
        rooms = []
        for M, N, K, rank, requests, out in MANY:
            C = sc.new_fp8(M, N) if out == "fp8" else (torch.zeros(M, -(-N // 8) * 8, dtype=T[out], device=DEV), None)
            rooms.append((C, sc.new_adapters_workspace(M, rank, requests)))
        return rooms

    def go(i, room, stream=None):
        (C, s), ws = room
        a, sa, b, sb, K, pool, start, which = jobs[i]
        sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C[:, :MANY[i][1]], pool, start, which, ws, S_out=s, stream=stream)

    want = make()
    for i, room in enumerate(want):
        go(i, room)
    torch.cuda.synchronize()
    lanes = [(torch.cuda.Stream(), make()) for _ in range(4)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for turn in range(10):
        for n, (stream, rooms) in enumerate(lanes):
            for i in range(len(jobs)):
                k = (i + n + turn) % len(jobs)
                go(k, rooms[k], stream)
        sc.svdcache_gemm_fp8(*x, *plain, 2048, side[:, :300], stream=other)
    torch.cuda.synchronize()
    for _, rooms in lanes:
        for ((C, _s), _w), ((V, _t), _v) in zip(rooms, want):
            assert torch.equal(C, V)
    assert sc.gemm_status() == 0


# ------------------------------------------------------------------------------------ neighbouring requests ---

@gpu
@pytest.mark.parametrize("M,N,K", [(9, 300, 2100), (60, 300, 700), (64, 18432, 520), (130, 260, 2100), (700, 1300, 600)])
def test_a_request_among_others(M, N, K):
    """Rows of one request, by tiles that CTAs share, by tiles of their own and by pairs: with and without adapters beside it, and as one
    of 1, 3, 5 and more requests, some of which hold NaN, they are what the formula says within the bound of any order of rounding."""
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    pool = random_pool(4, 40, N, K, 3, {0, 1, 2, 3})
    pool.factor[3] = float("nan")
    lo, hi = M // 3, M // 3 + max(M // 3, 2)
    y, err = adapted64(a, sa, b, sb, M, N, K, None, NONE, pool, [lo, hi], [1], "f32")
    y, err = y[lo:hi], err[lo:hi]
    each = list(range(lo + 1, hi))                       # a request for each of its rows
    variants = [([lo, hi], [1]), ([0, lo, hi, M], [-1, 1, -1]), ([0, lo, hi, M], [0, 1, 2]), ([0, lo, hi, M], [3, 1, 3]), ([0, lo // 2, lo, lo, hi, M], [0, 2, 3, 1, 0]),
                ([0, lo] + each + [hi, M], [3] + [1] * (hi - lo) + [0])]
    for starts, which in variants:
        C = torch.zeros(M, N if N % 4 == 0 else -(-N // 4) * 4, device=DEV)[:, :N]
        twice = torch.zeros_like(C)
        for out in (C, twice):
            sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, out, pool, ints(starts), ints(which), sc.new_adapters_workspace(M, 40, len(which)))
        close(y, err, C[lo:hi], torch.float32)
        assert torch.equal(C[lo:hi], twice[lo:hi])
    assert sc.gemm_status() == 0


# ----------------------------------------------------------------------------------------------- slots ---

def random_requests(rng, M, first, tile_rows, ordered):
    n = int(rng.integers(1, 12) if rng.random() < 0.7 else rng.integers(30, 100))
    start = np.sort(rng.integers(0, first + M + 40, n + 1)) if ordered else rng.integers(-20, first + M + 40, n + 1)
    if rng.random() < 0.4:
        start = first + (start - first) // tile_rows * tile_rows
    if not ordered and rng.random() < 0.3:
        start[rng.integers(0, n + 1)] = rng.choice([-(1 << 31), (1 << 31) - 1])
    return start, rng.integers(-1, 5, n)


@pytest.mark.parametrize("tile_rows", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("ordered", [True, False])
def test_what_the_kernels_find_out_about_requests(tile_rows, ordered):
    """Their own code: each pair of a tile and a request with rows in common has one slot, which knows it, and no two tiles' lists meet.
    Whatever the rows say, nothing outside the tables is written (the guards around them) and no index leads out of them."""
    rng = np.random.default_rng(tile_rows)
    count = 3
    L = sc.lib()
    for _ in range(150):
        M, first = int(rng.integers(1, 900)), int(rng.integers(0, 3)) * 256
        start, which = random_requests(rng, M, first, tile_rows, ordered)
        n, tiles = len(which), -(-M // tile_rows)
        s32, w32 = torch.tensor(start, dtype=torch.int32), torch.tensor(which, dtype=torch.int32)
        room = [np.full((k + 2, 2 + m), -9, dtype=np.int32).reshape(-1) for k, m in ((tiles + n, 4), (tiles, 4), (tiles + n, 2), (tiles, 1 + 2 * tile_rows))]
        sizes = [(tiles + n) * 4, tiles * 4, (tiles + n) * 2, tiles * (1 + 2 * tile_rows)]
        assert L.svdcache_selftest_adapters_slots(s32.data_ptr(), w32.data_ptr(), n, first, M, count, tile_rows, *[r.ctypes.data + 16 for r in room]) == 0
        for r, size in zip(room, sizes):
            assert (r[:4] == -9).all() and (r[4 + size:] == -9).all()
        tasks, entries, listed, own = (r[4:4 + size].reshape(-1, k) for r, size, k in zip(room, sizes, (4, 4, 2, 1 + 2 * tile_rows)))
        for got, want in zip(sc.svdcache_selftest_adapters_slots(s32, w32, M, count, tile_rows, first), (tasks, entries, listed, own)):
            assert (got.numpy() == want).all()
        rows = np.clip(start - first, 0, M)
        taken = set()
        assert ((tasks[:, 3] < 0) | ((tasks[:, 0] >= 0) & (tasks[:, 0] < tiles) & (tasks[:, 1] >= 0) & (tasks[:, 1] < tasks[:, 2]) & (tasks[:, 2] <= M) & (tasks[:, 3] < count))).all()
        for tile in range(tiles):
            place, many, number, adapter = entries[tile]
            got = listed[place:place + many]
            assert 0 <= place and 0 <= many and place + many <= tiles + n
            assert 0 <= own[tile, 0] <= tile_rows
            mine = own[tile, 1:1 + 2 * own[tile, 0]].reshape(-1, 2)
            for part in (got, mine):
                assert ((part[:, 0] >= 0) & (part[:, 0] < tiles + n) & (part[:, 1] >= 0) & (part[:, 1] < count)).all()
            assert many == 0 or (0 <= number < tiles + n and 0 <= adapter < count)
            if ordered:
                want = [(tile, max(a, tile * tile_rows), min(b, (tile + 1) * tile_rows), w) for a, b, w in zip(rows, rows[1:], which)
                        if min(b, (tile + 1) * tile_rows) > max(a, tile * tile_rows) and 0 <= w < count]
                assert [tuple(tasks[j]) for j, _ in got] == want and (got == mine).all() and (many == 0 or tuple(got[0]) == (number, adapter))
                places = set(range(place, place + many))
                assert not taken & places
                taken |= places


ANY_ROWS = [[40, 10, 70, 20, 5], [-5, 1 << 30, -(1 << 31), 3, (1 << 31) - 1], [30, 30, 0, 64, 0], [63, 62, 61, 60, 59], [1000, 900, 800, 0, 2000]]


@gpu
@pytest.mark.parametrize("M,N,plan,out", [(64, 260, (0, 64, 1), "f32"), (64, 260, (0, 64, 4), "f32"), (300, 130, (0, 128, 2), "bf16"), (600, 700, (1, 128, 2), "bf16"), (600, 700, (1, 256, 2), "fp8")])
def test_rows_in_no_order(M, N, plan, out):
    """Rows that decrease or lie outside: the call ends, with nothing outside its buffers touched, and the next one is in order.  (More
    requests than a small tile has rows among them.)"""
    K, rank = 1200, 24
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    pool = random_pool(3, rank, N, K, 3, {0, 1, 2})
    rng = np.random.default_rng(M)
    cases = [(s, [0, 1, 2, 0]) for s in ANY_ROWS] + [([int(x) for x in rng.integers(-20, M + 20, 201)], [int(x) for x in rng.integers(-1, 4, 200)]) for _ in range(3)]
    for i, (starts, which) in enumerate(cases + [([0, 20, M - 5, M], [2, -1, 1])]):
        n = sc.svdcache_adapters_workspace_bytes(M, rank, len(which))
        hold = torch.full((n + 512,), 0xFF, dtype=torch.uint8, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        args = (pool, ints(starts), ints(which), hold[256:256 + n], plan)
        if out == "fp8":
            q, s = junk_fp8(M, N)
            sc.svdcache_selftest_gemm_fp8_adapters(a, sa, b, sb, K, q[:, :N], *args, S_out=s, status=status)
            check_padding(q, s, M, N)
        else:
            C = torch.full((M + 2, -(-N // 8) * 8 + 8), 7.0, dtype=T[out], device=DEV)
            sc.svdcache_selftest_gemm_fp8_adapters(a, sa, b, sb, K, C[1:-1, :N], *args, status=status)
            assert bool((C[1:-1, N:] == 7.0).all()) and bool((C[0] == 7.0).all()) and bool((C[-1] == 7.0).all())
        assert int(status) == 0 and bool((hold[:256] == 0xFF).all()) and bool((hold[-256:] == 0xFF).all())
    y, err = adapted64(a, sa, b, sb, M, N, K, None, NONE, pool, starts, which, out)
    if out == "fp8":
        check_near(q, s, y, err)
    else:
        close(y, err, C[1:-1, :N], T[out])


# ----------------------------------------------------------------------------------------- named plans ---

@gpu
@pytest.mark.parametrize("M,N,K", [(4096, 8192, 2048), (2048, 4096, 8192), (3000, 2000, 700), (600, 700, 2100), (8, 2304, 1152)])
def test_the_plan_that_is_reported_gives_what_the_call_gives(M, N, K):
    """Bit for bit, the narrow product among it: above and below the 25 us from which fewer CTAs share it, with long and shorter K."""
    a, sa = random_fp8(M, K, 1)
    b, sb = random_fp8(N, K, 2, 128)
    pool = random_pool(3, 64, N, K, 3, {0, 1, 2})
    args = (pool, ints([0, M // 3, M // 2, M]), ints([2, 0, 1]), sc.new_adapters_workspace(M, 64, 3))
    one, two = (torch.zeros(M, N, device=DEV) for _ in range(2))
    sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, one, *args)
    sc.svdcache_selftest_gemm_fp8_adapters(a, sa, b, sb, K, two, *args, sc.svdcache_gemm_fp8_plan(M, N, K, sc.F32, a.stride(0), b.stride(0)))
    assert torch.equal(one, two) and bool(one.any()) and sc.gemm_status() == 0


# ------------------------------------------------------------------------------- sums beyond bf16's range ---

@gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M", [5, 100, 700])
def test_narrow_sums_beyond_bf16(M, out):
    """A row of ones by a `down` of ones is exactly 16, times the factor: infinite, or finite above the largest bf16 (3.3895e38)."""
    N, K = 40, 16
    a, sa = sc.new_fp8(M, K)
    b, sb = sc.new_fp8(N, K)
    sc.svdcache_quantize_fp8(torch.ones(M, K, device=DEV), a, sa)
    sc.svdcache_quantize_fp8(torch.zeros(N, K, device=DEV), b, sb, tile_rows=128)
    sign = torch.where(torch.arange(N, device=DEV) % 2 == 0, 1.0, -1.0)
    pool = sc.new_adapters(4, 8, N, K)
    for i, (factor, up) in enumerate([(1e38, 1.0), (-1e38, 1.0), (2.125e37, 2.0 ** -100), (-2.125e37, 2.0 ** -100)]):
        sc.svdcache_adapter_load(pool, i, torch.ones(1, K, device=DEV), (up * sign)[:, None].contiguous(), factor)
    C = torch.zeros(M, N, dtype=T[out], device=DEV)
    starts = [0, 1, 2, M - 2, M - 1, M]
    sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C, pool, ints(starts), ints([0, 1, -1, 2, 3]), sc.new_adapters_workspace(M, 8, 5))
    inf = float("inf") * sign
    assert torch.equal(C[0].float(), inf) and torch.equal(C[1].float(), -inf) and bool((C[2:M - 2] == 0).all())
    # t = 16 fl(2.125e37), within 2^-16 (bf16) or 2^-24 of itself, then the product's and the output's rounding
    want = 16.0 * float(np.float32(2.125e37)) * 2.0 ** -100
    bound = want * ((2.0 ** -16 + 2.0 ** -8) if out == "bf16" else (2.0 ** -24 + 2.0 ** -22))
    for row, way in ((M - 2, 1.0), (M - 1, -1.0)):
        assert np.abs(np64(C[row]) - way * want * np64(sign)).max() <= 1.001 * bound
    assert sc.gemm_status() == 0


# ------------------------------------------------------------------------------- an adapter as its user has it ---

@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("K", [1152, 12288])
def test_the_adapter_s_term_against_the_adapter_before_it_is_rounded(K, dtype):
    """A value of `down` in e4m3 is off by at most 2^-4 of the power of two below it, evenly spread: 2^-4 / sqrt(3) of itself in the mean square, and so
    is a sum of many; 4096 outputs of 16 sums are within a tenth of that."""
    M, N, r = 64, 64, 16
    g = torch.Generator().manual_seed(K)
    x, down, up = torch.randn(M, K, generator=g), torch.randn(r, K, generator=g) / K ** 0.5, torch.randn(N, r, generator=g).bfloat16()
    (a, sa), (b, sb) = sc.new_fp8(M, K), sc.new_fp8(N, K)
    sc.svdcache_quantize_fp8(x.to(DEV), a, sa)
    sc.svdcache_quantize_fp8(torch.zeros(N, K, device=DEV), b, sb, tile_rows=128)
    pool, C = sc.new_adapters(1, r, N, K), torch.zeros(M, N, device=DEV)
    down = down.to(dtype).to(DEV)
    sc.svdcache_adapter_load(pool, 0, down, up.to(dtype).to(DEV), 2.0)
    sc.svdcache_gemm_fp8_adapters(a, sa, b, sb, K, C, pool, ints([0, M]), ints([0]), sc.new_adapters_workspace(M, r, 1))
    want = 2.0 * (dequantise(a, sa, M, K) @ np64(down).T) @ np64(up).T
    assert np.linalg.norm(np64(C) - want) <= 1.1 * 2.0 ** -4 / 3 ** 0.5 * np.linalg.norm(want)
    assert sc.gemm_status() == 0
