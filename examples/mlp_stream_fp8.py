"""A stream of MLP blocks in 8 bits with their features cached.

Every block adds F = down(gelu(up(norm(h)))) to the residual stream h.  At a full step the linear layers run in 8 bits:
``svdcache_residual_rmsnorm_fp8`` adds the previous block's feature to h and hands the norm's output, quantised, to
``svdcache_gemm_fp8``, whose epilogue applies bias and gelu and quantises again for the second product; its output F is
the block's feature, which ``svdcache_full_step`` projects and stores.  At a cached step no layer runs:
``svdcache_cached_step`` returns Fhat, and the next block adds that.  The basis of each block is calibrated on the
features of a few full steps first.

    python examples/mlp_stream_fp8.py [--blocks 4 --rows 4608 --width 3072 --rank 64 --steps 12 --interval 6]

Inputs and weights are synthetic (seeded); printed are the times of both kinds of step and how far the cached stream is
from the one that computes every step.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2601_07396_b200 import binding as sc  # noqa: E402


class Block:
    """An MLP block: weights in 8 bits with a scale per 128 x 128 tile, and its cache."""

    def __init__(self, rows: int, width: int, hidden: int, rank: int, seed: int):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.rows, self.width, self.hidden, self.rank = rows, width, hidden, rank
        self.norm = 1.0 + 0.1 * rand(width)
        self.up, self.down = self._weight(rand(hidden, width) / width ** 0.5), self._weight(rand(width, hidden) / hidden ** 0.5)
        self.up_bias, self.down_bias = 0.1 * rand(hidden), 0.1 * rand(width)
        self.feature = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
        self.state = sc.new_state(rows, width, rank, sc.BF16)
        self.basis = None

    @staticmethod
    def _weight(w: torch.Tensor):
        q, s = sc.new_fp8(*w.shape)
        sc.svdcache_quantize_fp8(w, q, s, tile_rows=128)
        return q, s

    def compute(self, y, u) -> None:
        """feature = down(gelu(up(y))): y the norm's output, u room for the hidden layer, both 8-bit matrices."""
        sc.svdcache_gemm_fp8(*y, *self.up, self.width, u[0][:, :self.hidden], S_out=u[1], bias=self.up_bias, act=sc.ACT_GELU)
        sc.svdcache_gemm_fp8(*u, *self.down, self.hidden, self.feature, bias=self.down_bias)


class Stream:
    def __init__(self, blocks: int, rows: int, width: int, rank: int, seed: int = 0):
        hidden = 4 * width
        self.rows, self.width = rows, width
        self.blocks = [Block(rows, width, hidden, rank, seed + 1 + b) for b in range(blocks)]
        self.h = torch.empty(rows, width, dtype=torch.bfloat16, device="cuda")
        self.y, self.u = sc.new_fp8(rows, width), sc.new_fp8(rows, hidden)
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.start, self.drift = (torch.randn(rows, width, generator=g, device="cuda") for _ in range(2))

    def step(self, t: float, full: bool, cache: bool = True) -> torch.Tensor:
        """One step of the denoising loop at time t (its input drifts slowly): h after the last block."""
        self.h.copy_(self.start + 0.05 * t * self.drift)
        previous = None
        for b in self.blocks:
            if full:
                sc.svdcache_residual_rmsnorm_fp8(self.h, previous, self.h, b.norm, 1e-6, *self.y)
                b.compute(self.y, self.u)
                if cache:
                    sc.svdcache_full_step(b.feature, b.basis, b.state, b.rank, 0.9)
            else:
                if previous is not None:
                    self.h += previous
                sc.svdcache_cached_step(b.state, b.basis, b.feature, b.rank)
            previous = b.feature
        return self.h + previous

    def calibrate(self, times) -> None:
        """Each block's basis from the stack of its features at the given times."""
        stacks = [[] for _ in self.blocks]
        for t in times:
            self.step(t, full=True, cache=False)
            for stack, b in zip(stacks, self.blocks):
                stack.append(b.feature.clone())
        for stack, b in zip(stacks, self.blocks):
            V, _, _, _ = sc.svdcache_calibrate(torch.cat(stack), b.rank)
            b.basis = sc.svdcache_basis_prepare(V, sc.BF16)


def run(blocks: int, rows: int, width: int, rank: int, steps: int, interval: int, seed: int = 0) -> dict:
    s = Stream(blocks, rows, width, rank, seed)
    s.calibrate([-2.0, -1.0])
    exact = [s.step(float(t), full=True, cache=False).float() for t in range(steps)]
    marks, worst = {True: [], False: []}, 0.0
    for t in range(steps):
        full = t % interval == 0
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        out = s.step(float(t), full)
        b.record()
        marks[full].append((a, b))
        worst = max(worst, float((out.float() - exact[t]).norm() / exact[t].norm()))
    torch.cuda.synchronize()
    ms = {full: min(a.elapsed_time(b) for a, b in pairs) if pairs else None for full, pairs in marks.items()}
    return {"full_ms": ms[True], "cached_ms": ms[False], "worst": worst, "status": sc.gemm_status(),
            "states": [sc.svdcache_state_query(b.state) for b in s.blocks]}


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("blocks", 4), ("rows", 4608), ("width", 3072), ("rank", 64), ("steps", 12), ("interval", 6), ("seed", 0)):
        ap.add_argument("--" + name, type=int, default=value)
    r = run(**vars(ap.parse_args()))
    cached = "-" if r["cached_ms"] is None else f"{r['cached_ms']:.3f} ms"
    print(f"full step {r['full_ms']:.3f} ms, cached step {cached}, worst relative distance from computing every step {r['worst']:.4f}, "
          f"status {r['status']}, full steps and status per block {r['states']}")


if __name__ == "__main__":
    main()
