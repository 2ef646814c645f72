"""Plain 64-bit forms of the 8-bit operators and the checks that compare the library with them.  Everything here
follows from the definition of the format (a power-of-two scale per group, e4m3 by round to nearest even), in numpy."""
from __future__ import annotations

import numpy as np
import torch

from paper_2601_07396_b200 import binding as sc

GROUP = 128


def np64(t: torch.Tensor) -> np.ndarray:
    return t.detach().double().cpu().numpy()


def e4m3_values(b: np.ndarray) -> np.ndarray:
    """The values of e4m3 bytes: sign, 4 exponent bits (bias 7), 3 fraction bits; S.1111.111 is NaN, no Inf."""
    b = b.astype(np.int64)
    e, f = (b >> 3) & 15, b & 7
    v = np.where(e > 0, (1.0 + f / 8.0) * np.exp2(e - 7.0), f / 8.0 * 2.0 ** -6)
    return np.where((b & 127) == 127, np.nan, np.where(b >> 7 == 1, -v, v))


def e4m3_step(v: np.ndarray) -> np.ndarray:
    """Spacing of e4m3 values at |v|."""
    k = np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -6)))
    return np.exp2(k - 3.0)


def e4m3_round(v: np.ndarray) -> np.ndarray:
    step = e4m3_step(v)
    return np.round(v / step) * step      # numpy rounds halves to even


def scale_exponent(top: np.ndarray) -> np.ndarray:
    """Least e >= -127 with 448 * 2^e >= top; 0 where top is 0."""
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(np.maximum(top, 1e-300) / 448.0)) - 1.0
    for _ in range(3):
        e = np.where(448.0 * np.exp2(e) < top, e + 1.0, e)
    return np.where(top > 0, np.maximum(e, -127.0), 0.0)


def group_tops(y: np.ndarray, tile_rows: int = 1) -> np.ndarray:
    """Largest finite magnitude per group [rows, groups] (per 128 x 128 tile, repeated, for tile_rows = 128)."""
    rows, cols = y.shape
    groups = -(-cols // GROUP)
    a = np.zeros((rows, groups * GROUP))
    a[:, :cols] = np.where(np.isfinite(y), np.abs(y), 0.0)
    top = a.reshape(rows, groups, GROUP).max(2)
    if tile_rows == 128:
        for i in range(0, rows, 128):
            top[i:i + 128] = top[i:i + 128].max(0)
    return top


def unpack(q: torch.Tensor, s: torch.Tensor, rows: int, cols: int):
    """(values of the bytes [rows, cols], scale exponents [rows, groups]) of an 8-bit matrix, in 64 bits."""
    b = q.view(torch.uint8)[:, :cols].cpu().numpy()
    e = sc.fp8_scale_exponents(s, rows, cols).cpu().numpy().astype(np.float64) - 127.0
    return e4m3_values(b), e


def dequantise(q, s, rows, cols):
    v, e = unpack(q, s, rows, cols)
    return v * np.repeat(np.exp2(e), GROUP, axis=1)[:, :cols]


def check_exact(q, s, y: np.ndarray, tile_rows: int = 1):
    """q, s are the 8-bit form of exactly y, bit for bit."""
    rows, cols = y.shape
    v, e = unpack(q, s, rows, cols)
    want_e = scale_exponent(group_tops(y, tile_rows))
    np.testing.assert_array_equal(e, want_e)
    z = np.where(np.isfinite(y), y, np.nan) / np.repeat(np.exp2(want_e), GROUP, axis=1)[:, :cols]
    np.testing.assert_array_equal(v, e4m3_round(z))


def check_near(q, s, y: np.ndarray, err: np.ndarray):
    """q, s are the 8-bit form of values that lie within `err` of y (elementwise; where y is not finite: NaN).
    A group's scale is that of some maximum within the error, and each value lies within half a step of the format,
    at that scale, of some value within the error."""
    rows, cols = y.shape
    v, e = unpack(q, s, rows, cols)
    fin = np.isfinite(y)
    ym, err = np.where(fin, y, 0.0), np.where(fin, err, 0.0)
    least = group_tops(np.maximum(np.abs(ym) - err, 0.0))
    lo = np.where(least > 0, scale_exponent(least), -127.0)
    hi = scale_exponent(group_tops(np.abs(ym) + err))
    ok = ((e >= lo) & (e <= hi)) | (least == 0) & (e == 0)      # a group that may be all zero may have the scale of zeros
    assert ok.all(), f"{(~ok).sum()} scales are not those of their groups: {np.argwhere(~ok)[:4].tolist()}"
    scale = np.repeat(np.exp2(e), GROUP, axis=1)[:, :cols]
    np.testing.assert_array_equal(np.isnan(v), ~fin)
    off = np.abs(np.where(fin, v, 0.0) * scale - ym)
    half = 0.5 * e4m3_step((np.abs(ym) + err) / scale) * scale
    bad = off > half * (1 + 1e-12) + err
    assert not bad.any(), f"{bad.sum()} values are off: {np.argwhere(bad)[:4].tolist()}, by {off[bad][:4]} > {(half + err)[bad][:4]}"


def gelu64(x: np.ndarray) -> np.ndarray:
    u = np.sqrt(2.0 / np.pi) * (x + 0.044715 * x ** 3)
    return 0.5 * x * (1.0 + np.tanh(u))


def random_fp8(rows, cols, seed, tile_rows=1, dev="cuda", spread=3.0):
    """An 8-bit matrix with random values, groups of very different scale, and junk where no result may come from:
    NaN codes between the rows' ends and the pitch, NaN bytes for scales of rows and groups that do not exist."""
    g = torch.Generator().manual_seed(seed)
    groups, ntile = -(-cols // GROUP), -(-rows // 128)
    q = torch.full((rows, -(-cols // 16) * 16 + 16 * (seed % 3)), 0x7F, dtype=torch.uint8)
    vals = torch.randn(rows, cols, generator=g) * 100.0
    q[:, :cols] = vals.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    e = torch.round(torch.randn(rows, groups, generator=g) * spread).int().clamp(-20, 20) - 6 + 127
    if tile_rows == 128:
        e = e[:: 128].repeat_interleave(128, 0)[:rows]
    i, j = ntile, -(-groups // 4)
    full = torch.full((128 * i, 4 * j), 255, dtype=torch.uint8)
    full[:rows, :groups] = e.to(torch.uint8)
    s = full.view(i, 4, 32, j, 4).permute(0, 3, 2, 1, 4).contiguous().reshape(-1)
    return q.to(dev), s.to(dev)
