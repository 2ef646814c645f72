"""What the operators between the 8-bit product and attention, and beside the product, are measured on: rotary positions of
several axes (their table, and its application), the norm of queries and keys per head with that rotation, and the product of
8-bit operands with low-rank adapters of many requests.  ``run`` computes them in plain torch (``own`` false) or through the
library (``own`` true); ``exact`` computes them in 64 bits.

Heads: [batch, tokens, heads, dim] with any strides but the last.  A table holds (cos, sin) for each token and pair: of
neighbours (2i, 2i + 1) or of halves (i, i + r / 2), among the first r elements of a head; tokens outside its range are not
rotated.

Adapters of rank R on a projection of `cols` to `outs`: down [count, R, cols] in 8 bits (e4m3, a power-of-two scale per
1 x 128 group, each adapter's scales in the order of a matrix of its own), up [count, outs, R] bf16, and a factor for each.
A request is a run of rows with one adapter, or with none (-1).
"""
import random

import torch

own = False

GROUP = 128
E4M3_MAX = 448.0
DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}


# ------------------------------------------------------------------------------------------ the cases ---

def listed():
    return [
        # image-shaped stream: 512 text tokens at the origin and 64 x 64 patches, angles made when a generation begins
        {"name": "table image", "op": "table", "text": 512, "grid": "1,64,64", "dims": "16,56,56", "base": 10000.0, "type": "i32"},
        # video-shaped stream: 33 latent frames of 45 x 80 patches, frames at fractional times
        {"name": "table video", "op": "table", "text": 0, "grid": "33,45,80", "dims": "16,56,56", "base": 256.0, "type": "f32"},
        # one token: launch latency is all there is
        {"name": "rotate one token", "op": "rotate", "batch": 1, "tokens": 1, "heads": 24, "kv": 0, "dim": 128, "r": 128, "lead": 0, "tail": 0,
         "halves": False, "inverse": False, "dtype": "bf16", "packed": False, "heads_first": False},
        # nothing round: fp32, a head of 72 of which 48 are rotated, halves, tokens before and behind the table's
        {"name": "rotate ragged fp32", "op": "rotate", "batch": 3, "tokens": 777, "heads": 5, "kv": 0, "dim": 72, "r": 48, "lead": 13, "tail": 64,
         "halves": True, "inverse": False, "dtype": "f32", "packed": True, "heads_first": False},
        # keys of the video-shaped stream back to where they were before the rotation
        {"name": "rotate back video", "op": "rotate", "batch": 1, "tokens": 118800, "heads": 24, "kv": 0, "dim": 128, "r": 128, "lead": 0, "tail": 0,
         "halves": False, "inverse": True, "dtype": "bf16", "packed": False, "heads_first": False},
        # image-shaped stream: queries and keys out of the packed projection into attention's order
        {"name": "norm and rotate image", "op": "qk", "batch": 1, "tokens": 4608, "heads": 24, "kv": 24, "dim": 128, "r": 128, "lead": 0, "tail": 0,
         "halves": False, "inverse": False, "dtype": "bf16", "packed": True, "heads_first": True},
        # eight images of 256 tokens through a 1152-wide block of 16 heads, in fp32, keys shared by pairs of heads
        {"name": "norm and rotate shared keys", "op": "qk", "batch": 8, "tokens": 256, "heads": 16, "kv": 8, "dim": 72, "r": 72, "lead": 0, "tail": 0,
         "halves": True, "inverse": False, "dtype": "f32", "packed": True, "heads_first": False},
        # video-shaped stream with 256 tokens of text behind it, which have no position
        {"name": "norm and rotate video", "op": "qk", "batch": 1, "tokens": 119056, "heads": 24, "kv": 24, "dim": 128, "r": 128, "lead": 0, "tail": 256,
         "halves": False, "inverse": False, "dtype": "bf16", "packed": True, "heads_first": False},
        # modulation of eight requests, one row each with an adapter of its own: the weights' bytes
        {"name": "adapters one row each", "op": "adapt", "rows": 8, "outs": 18432, "cols": 3072, "rank": 16, "pool": 8, "requests": 8, "even": True,
         "bare": False, "out": "bf16", "act": "none", "bias": True, "cut": 1},
        # nothing is a multiple of a tile; some requests have no adapter, some no rows
        {"name": "adapters ragged", "op": "adapt", "rows": 777, "outs": 1000, "cols": 1160, "rank": 24, "pool": 3, "requests": 7, "even": False,
         "bare": True, "out": "f32", "act": "none", "bias": False, "cut": 2},
        # two image-shaped requests with different adapters, MLP up: gelu and the next product's 8-bit operand
        {"name": "adapters MLP up", "op": "adapt", "rows": 9216, "outs": 12288, "cols": 3072, "rank": 32, "pool": 4, "requests": 2, "even": True,
         "bare": False, "out": "fp8", "act": "gelu", "bias": True, "cut": 3},
        # one image-shaped request, MLP down, a wide adapter
        {"name": "adapters MLP down", "op": "adapt", "rows": 4608, "outs": 3072, "cols": 12288, "rank": 128, "pool": 2, "requests": 1, "even": True,
         "bare": False, "out": "bf16", "act": "none", "bias": True, "cut": 4},
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    def axes_of(r, most):
        """r as a sum of even sizes, one for each axis."""
        n = rng.randint(1, min(most, r // 2))
        cuts = sorted(rng.sample(range(1, r // 2), n - 1))
        return [2 * (b - a) for a, b in zip([0] + cuts, cuts + [r // 2])]

    op = rng.choice(["table", "rotate", "qk", "qk", "adapt", "adapt"])
    if op == "table":
        while True:
            dims = axes_of(8 * spread(1, 32), 4)
            sides = [spread(1, 400) for _ in dims]
            tokens = 1
            for s in sides:
                tokens *= s
            text = rng.choice([0, 0, spread(1, 1024)])
            if (tokens + text) * sum(dims) <= 118800 * 128:
                break
        return {"op": op, "text": text, "grid": ",".join(map(str, sides)), "dims": ",".join(map(str, dims)),
                "base": rng.choice([100.0, 256.0, 10000.0, 1000000.0]), "type": rng.choice(["i32", "i64", "f32"])}
    if op in ("rotate", "qk"):
        while True:
            dtype = rng.choice(["bf16", "bf16", "f32"])
            batch, tokens, heads, dim = rng.choice([1, 1, 2, 3, 8]), spread(1, 118800), spread(1, 48), rng.choice([64, 128, 128, 8 * spread(1, 32)])
            kv = 0 if op == "rotate" else rng.choice([heads, heads, max(1, heads // 2), 1])
            if batch * tokens * (heads + kv) * dim * (2 if dtype == "bf16" else 4) <= 118800 * 48 * 128 * 2:
                break
        lead, tail = (rng.randint(0, tokens // 3) if rng.random() < 0.3 else 0 for _ in range(2))
        return {"op": op, "batch": batch, "tokens": tokens, "heads": heads, "kv": kv, "dim": dim, "r": dim if rng.random() < 0.6 else 8 * rng.randint(1, dim // 8),
                "lead": lead, "tail": tail, "halves": rng.random() < 0.4, "inverse": op == "rotate" and rng.random() < 0.4, "dtype": dtype,
                "packed": rng.random() < 0.6, "heads_first": rng.random() < 0.4}
    while True:
        rows, outs, cols, rank = spread(1, 32768), spread(16, 18432), spread(32, 12288), 8 * spread(1, 16)
        if rng.random() < 0.5:   # model widths are round more often than not
            outs, cols = -(-outs // 128) * 128, -(-cols // 128) * 128
        if rows * outs * cols <= 9216 * 3072 * 12288 and rows * outs <= 9216 * 12288 and rows * cols <= 9216 * 12288:
            break
    requests = min(rows, spread(1, 32))
    return {"op": op, "rows": rows, "outs": outs, "cols": cols, "rank": rank, "pool": spread(1, 16), "requests": requests, "even": rng.random() < 0.4,
            "bare": rng.random() < 0.4, "out": rng.choice(["bf16", "bf16", "fp8", "f32"]), "act": rng.choice(["none", "gelu"]), "bias": rng.random() < 0.7,
            "cut": rng.randint(0, 1 << 20)}


def _requests(case):
    """(first rows of the requests and the end, their adapters)."""
    rng = random.Random(case["cut"])
    rows, n = case["rows"], case["requests"]
    starts = [rows * i // n for i in range(n + 1)] if case["even"] else [0] + sorted(rng.randint(0, rows) for _ in range(n - 1)) + [rows]
    which = rng.sample(range(case["pool"]), n) if n <= case["pool"] else [rng.randrange(case["pool"]) for _ in range(n)]
    if case["bare"]:
        which = [-1 if rng.random() < 0.3 else a for a in which]
    return starts, which


def _numbers(text):
    return [int(x) for x in text.split(",")]


def work(case):
    if case["op"] == "table":
        dims, tokens = _numbers(case["dims"]), 1
        for s in _numbers(case["grid"]):
            tokens *= s
        tokens += case["text"]
        size = 8 if case["type"] == "i64" else 4
        return {"bytes": tokens * (size * len(dims) + 4 * sum(dims)), "flops": 20 * tokens * sum(dims)}
    if case["op"] in ("rotate", "qk"):
        e = 2 if case["dtype"] == "bf16" else 4
        n = case["batch"] * case["tokens"] * (case["heads"] + case["kv"]) * case["dim"]
        table = 4 * case["r"] * (case["tokens"] - case["lead"] - case["tail"])
        return {"bytes": 2 * e * n + table + (8 * case["dim"] if case["op"] == "qk" else 0), "flops": (3 if case["op"] == "rotate" else 8) * n}
    rows, outs, cols, rank = case["rows"], case["outs"], case["cols"], case["rank"]
    groups = -(-cols // GROUP)
    starts, which = _requests(case)
    runs = [(b - a, w) for a, b, w in zip(starts, starts[1:], which) if b > a and w >= 0]
    used, adapted = len({w for _, w in runs}), sum(n for n, _ in runs)
    out = rows * outs + rows * -(-outs // GROUP) if case["out"] == "fp8" else rows * outs * (2 if case["out"] == "bf16" else 4)
    return {"bytes": (rows + outs + used * rank) * (cols + groups) + 2 * used * rank * outs + out + (4 * outs if case["bias"] else 0),
            "flops": 2 * rows * outs * cols + 2 * adapted * rank * (cols + outs)}


# ----------------------------------------------------------------------------------------- the inputs ---

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _positions(g, text, sides, kind):
    """Text at the origin, then a grid that begins anywhere in the first 64 places of each axis; in fp32 the first axis
    counts time in steps that are no whole number."""
    places = torch.stack(torch.meshgrid(*[torch.arange(s, device=DEV, dtype=torch.float64) for s in sides], indexing="ij"), -1).reshape(-1, len(sides))
    places = places + torch.randint(0, 64, (len(sides),), generator=g, device=DEV)
    if kind == "f32":
        places[:, 0] *= 0.25 + torch.rand((), generator=g, device=DEV, dtype=torch.float64)
    return torch.cat([torch.zeros(text, len(sides), device=DEV, dtype=torch.float64), places]).to(TYPES[kind]).contiguous()


def _features(g, rows, cols):
    """Hidden features: channels of unequal size, a few of them large."""
    size = torch.exp(0.5 * _randn(g, cols))
    size[torch.randperm(cols, generator=g, device=DEV)[: max(1, cols // 256)]] *= 20.0
    return _randn(g, rows, cols).mul_(size)


def _eight_bits(rows, cols):
    """An 8-bit matrix (rows 16 bytes or a multiple of that apart) and its scales, all zero."""
    q = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=DEV)
    return q, torch.zeros(-(-rows // 128), -(-cols // 512), 32, 4, 4, dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": dict(case)}
    if case["op"] == "table":
        dims = _numbers(case["dims"])
        s["positions"] = _positions(g, case["text"], _numbers(case["grid"]), case["type"])
        s["dims"], s["bases"] = dims, [case["base"]] * len(dims)
        s["table"] = torch.zeros(s["positions"].shape[0], sum(dims) // 2, 2, device=DEV)
        return s
    if case["op"] in ("rotate", "qk"):
        t, b, n, h, kv, d, r = TYPES[case["dtype"]], case["batch"], case["tokens"], case["heads"], case["kv"], case["dim"], case["r"]
        every = h + 2 * kv if kv else 2 * h                      # packed: queries, keys and values (or what else the projection gives) of a token
        size = torch.exp(0.5 * _randn(g, d))
        if case["packed"]:
            all_heads = torch.empty(b, n, every, d, dtype=t, device=DEV)
            for i in range(b):
                all_heads[i].copy_(_randn(g, n, every, d).mul_(size))
            s["q"], s["k"] = all_heads[:, :, :h], all_heads[:, :, h:h + kv]
        else:
            s["q"], s["k"] = ((_randn(g, b, n, m, d).mul_(size)).to(t) for m in (h, kv))
        for x in ("q", "k"):
            shape = s[x].shape
            s[x + "_out"] = (torch.zeros(b, shape[2], n, d, dtype=t, device=DEV).transpose(1, 2) if case["heads_first"]
                             else torch.zeros(shape, dtype=t, device=DEV))
        places = torch.arange(n - case["lead"] - case["tail"], device=DEV, dtype=torch.float64) + torch.randint(0, 64, (), generator=g, device=DEV)
        angle = places[:, None] * 10000.0 ** (-torch.arange(r // 2, device=DEV, dtype=torch.float64) / (r // 2))
        s["table"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        s["q_weight"], s["k_weight"], s["eps"] = 1.0 + 0.1 * _randn(g, d), 1.0 + 0.1 * _randn(g, d), 1e-6
        return s
    rows, outs, cols, rank, pool = case["rows"], case["outs"], case["cols"], case["rank"], case["pool"]
    s["a"] = _stored(*_quantise(_features(g, rows, cols).to(torch.bfloat16).float(), 1))
    s["w"] = _stored(*_quantise(_randn(g, outs, cols) / cols ** 0.5, 128))
    s["bias"] = 0.5 * _randn(g, outs) if case["bias"] else None
    down = [_stored(*_quantise(_randn(g, rank, cols) / cols ** 0.5, 1)) for _ in range(pool)]
    s["down"], s["down_scales"] = torch.stack([q for q, _ in down]), torch.stack([e.reshape(-1) for _, e in down])
    s["up"] = (0.5 * _randn(g, pool, outs, rank) / rank ** 0.5).to(torch.bfloat16)
    s["factor"] = 0.5 + torch.rand(pool, generator=g, device=DEV)
    s["starts"], s["which"] = _requests(case)
    s["row_start"], s["adapter"] = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (s["starts"], s["which"]))
    room = -(-rows // 256) + case["requests"]                      # where the narrow products pass from one kernel to the next
    s["workspace"] = torch.zeros(room * 256 * -(-rank // 32) * 128 + 1024 * room, dtype=torch.uint8, device=DEV)
    if case["out"] == "fp8":
        s["out"] = _eight_bits(rows, outs)
    else:
        s["out"] = torch.zeros(rows, -(-outs // 8) * 8, dtype=TYPES[case["out"]], device=DEV)[:, :outs]
    return s


# ------------------------------------------------------------------------------------ the plain forms ---

def _quantise(y, tile_rows):
    """(values in e4m3, biased exponents [rows, groups]) of y, in 32 bits."""
    rows, cols = y.shape
    groups = -(-cols // GROUP)
    part = torch.nn.functional.pad(y, (0, groups * GROUP - cols)).view(rows, groups, GROUP)
    top = torch.where(part.isfinite(), part.abs(), 0.0).amax(2)
    if tile_rows > 1:
        n = -(-rows // tile_rows)
        top = torch.nn.functional.pad(top, (0, 0, 0, n * tile_rows - rows)).view(n, tile_rows, groups).amax(1).repeat_interleave(tile_rows, 0)[:rows]
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


def _values(q, s, rows, cols, t):
    """What an 8-bit matrix stands for, in the type t."""
    i, j = -(-rows // 128), -(-cols // 512)
    e = s.view(i, j, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(128 * i, 4 * j)[:rows, : -(-cols // GROUP)]
    scale = torch.exp2(e.to(t) - 127.0)
    return q[:, :cols].view(torch.float8_e4m3fn).to(t) * scale.repeat_interleave(GROUP, 1)[:, :cols]


def _answer(q, s, cols):
    """An 8-bit result as torch's own 8-bit types: values, and scales in the order they are stored in."""
    return {"q": q[:, :cols].view(torch.float8_e4m3fn) if q.dtype == torch.uint8 else q, "s": s.view(torch.float8_e8m0fnu)}


def _rotated(x, state):
    """x [batch, tokens, heads, dim] in 32 bits, its tokens of the table's range rotated."""
    case, table = state["case"], state["table"]
    r, lead = case["r"], case["lead"]
    part = x[:, lead:lead + table.shape[0], :, :r]
    c, s = table[None, :, None, :, 0], table[None, :, None, :, 1]
    if case["inverse"]:
        s = -s
    if case["halves"]:
        a, b = part[..., : r // 2], part[..., r // 2:]
        turned = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    x[:, lead:lead + table.shape[0], :, :r] = turned
    return x


def run(state):
    case = state["case"]
    if own:
        return _run_own(state)
    if case["op"] == "table":
        # far positions lose their angle in 32 bits
        angles = [state["positions"][:, a].double()[:, None] * base ** (-torch.arange(0, d, 2, device=DEV, dtype=torch.float64) / d)
                  for a, (d, base) in enumerate(zip(state["dims"], state["bases"]))]
        angle = torch.cat(angles, 1)
        return torch.stack([angle.cos(), angle.sin()], -1).float()
    if case["op"] == "rotate":
        return _rotated(state["q"].float().clone(), state).to(state["q"].dtype)
    if case["op"] == "qk":
        answer = {}
        for x in ("q", "k"):
            y = state[x].float()
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + state["eps"]) * state[x + "_weight"]
            answer[x] = _rotated(y, state).to(state[x].dtype)
        return answer
    rows, outs, cols, rank = case["rows"], case["outs"], case["cols"], case["rank"]
    x = _values(*state["a"], rows, cols, torch.float32)
    y = x @ _values(*state["w"], outs, cols, torch.float32).t()
    for lo, hi, a in zip(state["starts"], state["starts"][1:], state["which"]):
        if hi > lo and a >= 0:
            narrow = x[lo:hi] @ _values(state["down"][a], state["down_scales"][a], rank, cols, torch.float32).t()
            y[lo:hi] += (narrow * state["factor"][a]) @ state["up"][a].float().t()
    if state["bias"] is not None:
        y = y + state["bias"]
    if case["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh(0.7978845608028654 * (y + 0.044715 * y * y * y)))
    if case["out"] != "fp8":
        return y.to(TYPES[case["out"]])
    q, e = _quantise(y, 1)
    return _answer(q, _packed(e), outs)


def _run_own(state):
    from paper_2601_07396_b200 import binding as sc
    case = state["case"]
    if case["op"] == "table":
        sc.svdcache_rotary_table(state["positions"], state["dims"], state["bases"], state["table"])
        return state["table"]
    if case["op"] == "rotate":
        sc.svdcache_rotary(state["q"], state["table"], state["q_out"], first=case["lead"], halves=case["halves"], inverse=case["inverse"])
        return state["q_out"]
    if case["op"] == "qk":
        sc.svdcache_qk_rmsnorm_rotary(state["q"], state["k"], state["q_weight"], state["k_weight"], state["eps"], state["table"], state["q_out"],
                                      state["k_out"], first=case["lead"], halves=case["halves"])
        return {"q": state["q_out"], "k": state["k_out"]}
    adapters = sc.Adapters(state["down"], state["down_scales"], state["up"], state["factor"])
    more = {"bias": state["bias"], "act": sc.ACT_GELU if case["act"] == "gelu" else sc.ACT_NONE}
    if case["out"] != "fp8":
        sc.svdcache_gemm_fp8_adapters(*state["a"], *state["w"], case["cols"], state["out"], adapters, state["row_start"], state["adapter"],
                                      state["workspace"], **more)
        return state["out"]
    q, s = state["out"]
    sc.svdcache_gemm_fp8_adapters(*state["a"], *state["w"], case["cols"], q[:, : case["outs"]], adapters, state["row_start"], state["adapter"],
                                  state["workspace"], S_out=s, **more)
    return _answer(q, s, case["outs"])


# --------------------------------------------------------------------------------------- in 64 bits ---

def _e4m3_64(v):
    """v rounded to the nearest e4m3 value, ties to even: steps of 2^(k-3) in [2^k, 2^(k+1)), 2^-9 below 2^-6."""
    k = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(k - 3.0)
    return torch.round(v / step) * step


def _quantised_64(y):
    """The definition, group by group of columns: s the least power of two with 448 s >= the largest |y|."""
    rows, cols = y.shape
    q, s = torch.empty_like(y), torch.zeros(-(-rows // 128), -(-cols // 512), 32, 4, 4, dtype=torch.float64, device=y.device)
    s += 2.0 ** -127
    at = torch.arange(rows, device=y.device)
    for g in range(-(-cols // GROUP)):
        part = y[:, g * GROUP:(g + 1) * GROUP]
        top = part.abs().amax(1)
        guess = torch.floor(torch.log2(top.clamp(min=1e-300) / E4M3_MAX)) - 1.0
        for _ in range(3):   # from below, so that no rounding of the logarithm decides
            guess = torch.where(E4M3_MAX * torch.exp2(guess) < top, guess + 1.0, guess)
        scale = torch.where(top > 0, torch.exp2(guess.clamp(min=-127.0)), 1.0)
        q[:, g * GROUP:(g + 1) * GROUP] = _e4m3_64(part / scale[:, None])
        s[at // 128, g // 4, at % 32, at % 128 // 32, g % 4] = scale
    return {"q": q, "s": s}


def _turned_64(y, table, lead, r, halves, inverse):
    """The rotation as a complex product."""
    z = torch.view_as_complex(table.double().contiguous())
    z = (z.conj() if inverse else z)[None, :, None, :]
    part = y[:, lead:lead + table.shape[0], :, :r]
    if halves:
        w = torch.complex(part[..., : r // 2].contiguous(), part[..., r // 2:].contiguous()) * z
        part[..., : r // 2], part[..., r // 2:] = w.real, w.imag
    else:
        w = torch.complex(part[..., 0::2].contiguous(), part[..., 1::2].contiguous()) * z
        part[..., 0::2], part[..., 1::2] = w.real, w.imag
    return y


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "table":
        out, at = torch.empty_like(state["table"], dtype=torch.float64), 0
        for a, (d, base) in enumerate(zip(state["dims"], state["bases"])):
            for i in range(d // 2):
                turn = state["positions"][:, a].double() / base ** (2 * i / d)
                out[:, at, 0], out[:, at, 1] = torch.cos(turn), torch.sin(turn)
                at += 1
        return out
    if case["op"] == "rotate":
        return _turned_64(state["q"].double().clone(), state["table"], case["lead"], case["r"], case["halves"], case["inverse"])
    if case["op"] == "qk":
        answer = {}
        for x in ("q", "k"):
            y = state[x].double().clone()
            y /= torch.sqrt((y * y).sum(-1, keepdim=True) / case["dim"] + state["eps"])
            answer[x] = _turned_64(y * state[x + "_weight"].double(), state["table"], case["lead"], case["r"], case["halves"], False)
        return answer
    rows, outs, cols, rank = case["rows"], case["outs"], case["cols"], case["rank"]

    def part_of(q, s, n, g):
        """Group g of a matrix's columns, as values."""
        e = s.view(-(-n // 128), -(-cols // 512), 32, 4, 4)[:, g // 4, :, :, g % 4].transpose(1, 2).reshape(-1).double()
        return q[:, g * GROUP:min(cols, (g + 1) * GROUP)].contiguous().view(torch.float8_e4m3fn).double() * torch.pow(2.0, e[:n] - 127)[:, None]

    runs = [(lo, hi, a) for lo, hi, a in zip(state["starts"], state["starts"][1:], state["which"]) if hi > lo and a >= 0]
    y = torch.zeros(rows, outs, dtype=torch.float64, device=DEV)
    narrow = torch.zeros(rows, rank, dtype=torch.float64, device=DEV)
    for g in range(-(-cols // GROUP)):
        xa = part_of(*state["a"], rows, g)
        y.addmm_(xa, part_of(*state["w"], outs, g).t())
        for lo, hi, a in runs:
            narrow[lo:hi].addmm_(xa[lo:hi], part_of(state["down"][a], state["down_scales"][a], rank, g).t())
    for lo, hi, a in runs:
        y[lo:hi].addmm_(narrow[lo:hi], state["up"][a].double().t(), alpha=float(state["factor"][a]))
    if state["bias"] is not None:
        y += state["bias"].double()
    if case["act"] == "gelu":   # 0.5 (1 + tanh u) = 1 / (1 + exp(-2u))
        y /= 1.0 + torch.exp(-2.0 * (2.0 / torch.pi) ** 0.5 * (y + 0.044715 * y ** 3))
    return y if case["out"] != "fp8" else _quantised_64(y)
