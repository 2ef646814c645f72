"""What the 8-bit operators around a cached block are measured on: the residual addition with the
root-mean-square norm and an 8-bit output, the quantiser, and the matrix product of 8-bit operands with a
power-of-two scale per group of 128.  ``run`` computes them in plain torch (``own`` false) or through the
library (``own`` true); ``exact`` computes them in 64 bits.

8-bit matrices are e4m3 values with one scale per 1 x 128 group of a row (for weights, per 128 x 128 tile,
repeated for each of its rows).  A scale is a power of two held as its biased exponent in one byte.  The
scales of a matrix lie in 512-byte pieces, one per 128 rows and 4 groups: [rows / 128][groups / 4][32][4][4],
where the byte at (i, j, r, w, b) belongs to row 128 i + 32 w + r and group 4 j + b.
"""
import torch

own = False

GROUP = 128
E4M3_MAX = 448.0
DEV = "cuda"


# ------------------------------------------------------------------------------------------ the cases ---

def listed():
    return [
        # one conditioning vector: launch latency is all there is
        {"name": "norm one row", "op": "norm", "rows": 1, "cols": 3072, "dtype": "bf16", "pad": 0},
        # 8 images of 256 tokens through a 1152-wide block
        {"name": "norm 2048 x 1152", "op": "norm", "rows": 2048, "cols": 1152, "dtype": "bf16", "pad": 0},
        # fp32 stream, width not a multiple of the group, rows padded in memory
        {"name": "norm ragged fp32", "op": "norm", "rows": 777, "cols": 1000, "dtype": "f32", "pad": 24},
        # the video-shaped stream: 33 latent frames of 3600 tokens
        {"name": "norm video", "op": "norm", "rows": 118800, "cols": 3072, "dtype": "bf16", "pad": 0},
        # activations that no norm precedes (the attention's output of the image-shaped stream)
        {"name": "quantise rows", "op": "quant", "rows": 4608, "cols": 3072, "dtype": "bf16", "pad": 0, "tiles": False},
        # a weight matrix of the MLP, brought into 8 bits when a model is loaded
        {"name": "quantise weight tiles", "op": "quant", "rows": 12288, "cols": 3072, "dtype": "bf16", "pad": 0, "tiles": True},
        # modulation: one conditioning vector to 6 vectors of the model's width, bound by the weights' bytes
        {"name": "product one row", "op": "gemm", "rows": 1, "outs": 18432, "cols": 3072, "out": "bf16", "act": "none", "bias": True},
        # one image of a 1152-wide block into its MLP
        {"name": "product 256 x 4608 x 1152", "op": "gemm", "rows": 256, "outs": 4608, "cols": 1152, "out": "fp8", "act": "gelu", "bias": True},
        # nothing is a multiple of a tile
        {"name": "product ragged", "op": "gemm", "rows": 777, "outs": 1000, "cols": 1160, "out": "bf16", "act": "none", "bias": False},
        # image-shaped stream, MLP up: bias, gelu and the next product's 8-bit operand in the epilogue
        {"name": "product MLP up", "op": "gemm", "rows": 4608, "outs": 12288, "cols": 3072, "out": "fp8", "act": "gelu", "bias": True},
        # image-shaped stream, MLP down: long reduction, few output columns
        {"name": "product MLP down", "op": "gemm", "rows": 4608, "outs": 3072, "cols": 12288, "out": "bf16", "act": "none", "bias": True},
        # video-shaped stream, the attention's output projection
        {"name": "product video", "op": "gemm", "rows": 118800, "outs": 3072, "cols": 3072, "out": "bf16", "act": "none", "bias": True},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    op = rng.choice(["norm", "quant", "gemm", "gemm"])
    if op == "gemm":
        while True:
            rows, outs, cols = spread(1, 118800), spread(16, 18432), spread(32, 12288)
            if rng.random() < 0.5:   # model widths are round more often than not
                outs, cols = -(-outs // 128) * 128, -(-cols // 128) * 128
            if rows * outs * cols <= 118800 * 3072 * 3072 and rows * outs <= 118800 * 3072 and rows * cols <= 118800 * 3072:
                break
        return {"op": op, "rows": rows, "outs": outs, "cols": cols, "out": rng.choice(["bf16", "bf16", "fp8"]),
                "act": rng.choice(["none", "gelu"]), "bias": rng.random() < 0.7}
    while True:
        rows, cols = spread(1, 118800), 8 * spread(8, 2048)
        if rows * cols <= 118800 * 3072 // 2:
            break
    case = {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "f32"]), "pad": rng.choice([0, 0, 8, 40])}
    if op == "quant":
        case["tiles"] = rng.random() < 0.3
    return case


def work(case):
    rows, cols = case["rows"], case["cols"]
    groups = -(-cols // GROUP)
    if case["op"] == "gemm":
        outs = case["outs"]
        out = 2 * rows * outs if case["out"] == "bf16" else rows * outs + rows * -(-outs // GROUP)
        return {"bytes": (rows + outs) * (cols + groups) + out + (4 * outs if case["bias"] else 0), "flops": 2 * rows * outs * cols}
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":
        return {"bytes": rows * cols * (3 * e + 1) + rows * groups + 4 * cols, "flops": 8 * rows * cols}
    return {"bytes": rows * cols * (e + 1) + rows * groups, "flops": 3 * rows * cols}


# ----------------------------------------------------------------------------------------- the inputs ---

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _features(g, rows, cols, dtype, pad):
    """Hidden features: channels of unequal size, a few of them large; rows `pad` elements apart."""
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    size = torch.exp(0.5 * _randn(g, cols))
    size[torch.randperm(cols, generator=g, device=DEV)[: max(1, cols // 256)]] *= 20.0
    x = torch.empty(rows, cols + pad, dtype=t, device=DEV)[:, :cols]
    x.copy_(_randn(g, rows, cols).mul_(size))
    return x


def _eight_bits(rows, cols):
    """An 8-bit matrix (rows 16 bytes or a multiple of that apart) and its scales, all zero."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=DEV)
    s = torch.zeros(-(-rows // 128), -(-cols // 512), 32, 4, 4, dtype=torch.uint8, device=DEV)
    return q, s


def prepare(case, seed):
    g = _gen(seed)
    rows, cols = case["rows"], case["cols"]
    if case["op"] == "gemm":
        outs = case["outs"]
        a = _quantise(_features(g, rows, cols, "bf16", 0).float(), False)
        w = _quantise(_randn(g, outs, cols) / cols ** 0.5, True)
        s = {"case": dict(case), "a": _stored(*a), "w": _stored(*w), "bias": 0.5 * _randn(g, outs) if case["bias"] else None}
        s["out"] = _eight_bits(rows, outs) if case["out"] == "fp8" else torch.zeros(rows, -(-outs // 8) * 8, dtype=torch.bfloat16, device=DEV)[:, :outs]
        return s
    s = {"case": dict(case), "x": _features(g, rows, cols, case["dtype"], case["pad"]), "q": _eight_bits(rows, cols)}
    if case["op"] == "norm":
        s["h"] = _features(g, rows, cols, case["dtype"], case["pad"]).mul_(3.0)   # the residual stream outgrows what is added to it
        s["h_out"] = torch.zeros_like(s["h"])
        s["weight"] = 1.0 + 0.1 * _randn(g, cols)
        s["eps"] = 1e-6
    return s


# ------------------------------------------------------------------------------------ the plain forms ---

def _quantise(y, tiles):
    """(values in e4m3, biased exponents [rows, groups]) of y, in 32 bits."""
    rows, cols = y.shape
    groups = -(-cols // GROUP)
    part = torch.nn.functional.pad(y, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    top = torch.where(part.isfinite(), part.abs(), 0.0).amax(2)
    if tiles:
        n = -(-rows // 128)
        top = torch.nn.functional.pad(top, (0, 0, 0, n * 128 - rows)).view(n, 128, groups).amax(1).repeat_interleave(128, 0)[:rows]
    m, e = torch.frexp(top / E4M3_MAX)   # top / 448 = m 2^e, 1/2 <= m < 1: the next power of two is 2^e, or 2^(e-1) for m = 1/2
    e = torch.where(top > 0, (e - (m == 0.5).int()).clamp(min=-127), 0)
    q = torch.where(part.isfinite(), part * torch.exp2(-e.float())[:, :, None], torch.nan).reshape(rows, -1)[:, :cols]
    return q.to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _packed(e):
    """Biased exponents [rows, groups] in the order that scales are stored in; zero where there is no row or group."""
    rows, groups = e.shape
    i, j = -(-rows // 128), -(-groups // 4)
    full = torch.nn.functional.pad(e, (0, 4 * j - groups, 0, 128 * i - rows))
    return full.view(i, 4, 32, j, 4).permute(0, 3, 2, 1, 4).contiguous()


def _stored(q, e):
    rows, cols = q.shape
    held, s = _eight_bits(rows, cols)
    held[:, :cols] = q.view(torch.uint8)
    s.copy_(_packed(e))
    return held, s


def _exponents(s, rows, cols):
    i, j = s.shape[:2]
    return s.permute(0, 3, 2, 1, 4).reshape(128 * i, 4 * j)[:rows, : -(-cols // GROUP)]


def _values(held, rows, cols, t):
    """What an 8-bit matrix stands for, in the type t."""
    q, s = held
    scale = torch.exp2(_exponents(s, rows, cols).to(t) - 127.0)
    return q[:, :cols].view(torch.float8_e4m3fn).to(t) * scale.repeat_interleave(GROUP, 1)[:, :cols]


def _answer(q, s, cols):
    """An 8-bit result as torch's own 8-bit types: values, and scales in the order they are stored in."""
    return {"q": q[:, :cols].view(torch.float8_e4m3fn) if q.dtype == torch.uint8 else q, "s": s.view(torch.float8_e8m0fnu)}


def run(state):
    case = state["case"]
    cols = case["cols"]
    if own:
        return _run_own(state)
    if case["op"] == "quant":
        q, e = _quantise(state["x"].float(), case["tiles"])
        return _answer(q, _packed(e), cols)
    if case["op"] == "norm":
        h = state["h"].float() + state["x"].float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + state["eps"]) * state["weight"]
        q, e = _quantise(y, False)
        return {"h": h.to(state["h"].dtype)} | _answer(q, _packed(e), cols)
    y = _values(state["a"], case["rows"], cols, torch.float32) @ _values(state["w"], case["outs"], cols, torch.float32).t()
    if state["bias"] is not None:
        y = y + state["bias"]
    if case["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(0.7978845608028654 * (y + 0.044715 * y * y * y)))
    if case["out"] == "bf16":
        return y.to(torch.bfloat16)
    q, e = _quantise(y, False)
    return _answer(q, _packed(e), case["outs"])


def _run_own(state):
    from paper_2601_07396_b200 import binding as sc
    case = state["case"]
    if case["op"] == "quant":
        q, s = state["q"]
        sc.svdcache_quantize_fp8(state["x"], q, s, tile_rows=128 if case["tiles"] else 1)
        return _answer(q, s, case["cols"])
    if case["op"] == "norm":
        q, s = state["q"]
        sc.svdcache_residual_rmsnorm_fp8(state["h"], state["x"], state["h_out"], state["weight"], state["eps"], q, s)
        return {"h": state["h_out"]} | _answer(q, s, case["cols"])
    act = sc.ACT_GELU if case["act"] == "gelu" else sc.ACT_NONE
    if case["out"] == "bf16":
        sc.svdcache_gemm_fp8(*state["a"], *state["w"], case["cols"], state["out"], bias=state["bias"], act=act)
        return state["out"]
    q, s = state["out"]
    sc.svdcache_gemm_fp8(*state["a"], *state["w"], case["cols"], q[:, : case["outs"]], S_out=s, bias=state["bias"], act=act)
    return _answer(q, s, case["outs"])


# --------------------------------------------------------------------------------------- in 64 bits ---

def _e4m3_64(v):
    """v rounded to the nearest e4m3 value, ties to even: steps of 2^(k-3) in [2^k, 2^(k+1)), 2^-9 below 2^-6."""
    k = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(k - 3.0)
    return torch.round(v / step) * step


def _quantised_64(y, tiles=False):
    """The definition, group by group of columns: s the least power of two with 448 s >= the largest |y|."""
    rows, cols = y.shape
    q, s = torch.empty_like(y), torch.zeros(-(-rows // 128), -(-cols // 512), 32, 4, 4, dtype=torch.float64, device=y.device)
    s += 2.0 ** -127
    at = torch.arange(rows, device=y.device)
    for g in range(-(-cols // GROUP)):
        part = y[:, g * GROUP:(g + 1) * GROUP]
        top = part.abs().amax(1)
        if tiles:
            for i in range(0, rows, 128):
                top[i:i + 128] = top[i:i + 128].max().clone()
        guess = torch.floor(torch.log2(top.clamp(min=1e-300) / E4M3_MAX)) - 1.0
        for _ in range(3):   # from below, so that no rounding of the logarithm decides
            guess = torch.where(E4M3_MAX * torch.exp2(guess) < top, guess + 1.0, guess)
        scale = torch.where(top > 0, torch.exp2(guess.clamp(min=-127.0)), 1.0)
        q[:, g * GROUP:(g + 1) * GROUP] = _e4m3_64(part / scale[:, None])
        s[at // 128, g // 4, at % 32, at % 128 // 32, g % 4] = scale
    return {"q": q, "s": s}


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "quant":
        return _quantised_64(state["x"].double(), case["tiles"])
    if case["op"] == "norm":
        h = state["h"].double().add_(state["x"].double())
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["cols"] + state["eps"]) * state["weight"].double()
        return {"h": h} | _quantised_64(y)
    rows, outs, cols = case["rows"], case["outs"], case["cols"]
    y = torch.zeros(rows, outs, dtype=torch.float64, device=DEV)
    (qa, sa), (qw, sw) = state["a"], state["w"]
    rest = -(-cols // GROUP)
    for g in range(rest):   # sum over the groups: s_a s_w (q_a q_w^T)
        lo, hi = g * GROUP, min(cols, (g + 1) * GROUP)
        ea, ew = (s[:, g // 4, :, :, g % 4].transpose(1, 2).reshape(-1).double() for s in (sa, sw))
        pa, pw = (q[:, lo:hi].contiguous().view(torch.float8_e4m3fn).double() for q in (qa, qw))
        y.addmm_(pa * torch.pow(2.0, ea[:rows] - 127)[:, None], (pw * torch.pow(2.0, ew[:outs] - 127)[:, None]).t())
    if state["bias"] is not None:
        y += state["bias"].double()
    if case["act"] == "gelu":   # 0.5 (1 + tanh u) = 1 / (1 + exp(-2u))
        y /= 1.0 + torch.exp(-2.0 * (2.0 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3))
    return y if case["out"] == "bf16" else _quantised_64(y)
