"""Performance cases of the 8-bit transformer layer operators.

Each case is one call of an operator as a program using this package makes it,
on buffers that such a program keeps:

  norm   h = x + resid; y = h / rms(h) * weight; y rounded to the type of x, or
         in 8 bits (e4m3) with a scale for every 128 columns of a row.
  quant  a tensor that another kernel wrote, in 8 bits: a scale for every 128
         columns of a row (activations) or every 128 x 128 block (weights).
  gemm   an 8-bit product with a scale for each block of 128, then bias, GELU,
         gate and residual; the result rounded, or in 8 bits again.
  rope   rotary positions with several axes on q and k, with or without the
         root-mean-square norm of each head in front of it.

Scales of activations lie block by block ([blocks, rows]), those of weights as
[row blocks, column blocks].  8-bit outputs are returned as float8 values with
their scales beside them.

``listed()`` holds sizes of the package's own workloads (a video model of width
2048 with 14310 image and 256 text tokens, DiT-XL/2 with its width of 1152) and
ragged ones, ``draw()`` gives others of the same ranges, ``exact()`` restates
each call in float64.
"""

import math

import torch

own = False

DEV = "cuda"
TD = {"f32": torch.float32, "bf16": torch.bfloat16}
F8 = torch.float8_e4m3fn
Q_MAX = 448.0           # largest e4m3 value
S_MIN = 2.0 ** -100     # smallest scale
EPS = 1e-6
THETA = 10000.0


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------

def listed():
    return [
        # qkv of one new token of the video model's text stream: the smallest
        # product, where latency and the reading of the weights count.
        dict(name="gemm 1x6144x2048 bf16", kind="gemm", m=1, n=6144, k=2048, dtype="bf16", epilogue="bias"),
        # fc2 of the video model's text stream: few rows, a long reduction.
        dict(name="gemm 256x2048x8192 gated", kind="gemm", m=256, n=2048, k=8192, dtype="bf16", epilogue="gated"),
        # A small ragged layer with an fp32 result, as a check against fp32 runs it.
        dict(name="gemm 1077x1000x712 f32", kind="gemm", m=1077, n=1000, k=712, dtype="f32", epilogue="bias"),
        # fc2 of a DiT-XL/2 step (16 samples of 256 tokens): gate and residual.
        dict(name="gemm 4096x1152x4608 gated", kind="gemm", m=4096, n=1152, k=4608, dtype="bf16", epilogue="gated"),
        # fc1 of the video model's image stream: GELU, and 8 bits for fc2.
        dict(name="gemm 14310x8192x2048 gelu8", kind="gemm", m=14310, n=8192, k=2048, dtype="bf16", epilogue="gelu8"),
        # The norm in front of one token's qkv.
        dict(name="norm 1x2048 q8", kind="norm", rows=1, width=2048, dtype="bf16", resid=True, q8=True),
        # The norm of all of the video model's tokens, with the addition.
        dict(name="norm 14566x2048 q8", kind="norm", rows=14566, width=2048, dtype="bf16", resid=True, q8=True),
        # An fp32 norm of a width that no vector divides.
        dict(name="norm 1333x1001 f32", kind="norm", rows=1333, width=1001, dtype="f32", resid=True, q8=False),
        # Attention output of the video model, for its out-projection.
        dict(name="quant 14566x2048", kind="quant", rows=14566, width=2048, dtype="bf16", tile=1),
        # Weights of fc1 when a model is loaded.
        dict(name="quant 8192x2048 weights", kind="quant", rows=8192, width=2048, dtype="f32", tile=128),
        # q and k of one token, four query heads to a key head, one ladder of
        # frequencies over time, height and width.
        dict(name="rope 1 token 16+4 heads", kind="rope", rows=1, hq=16, hk=4, dim=128, dtype="bf16", axes="16,24,24",
             halves=True, ladder=True, norm=False, inverse=False),
        # q and k of the video model, normalised and rotated over time, height
        # and width.
        dict(name="rope 14566 rows 3 axes norm", kind="rope", rows=14566, hq=16, hk=16, dim=128, dtype="bf16",
             axes="16,56,56", halves=False, ladder=False, norm=True, inverse=False),
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer spread over the logarithm of [lo, hi], a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def _axes(rng, dim):
    """Even widths of one to three axes that fill dim, or leave some of it alone."""
    rot = dim if rng.random() < 0.7 else 2 * rng.randint(3, dim // 2)
    n = rng.randint(1, 3)
    cuts = sorted(rng.sample(range(1, rot // 2), n - 1))
    return ",".join(str(2 * (b - a)) for a, b in zip([0] + cuts, cuts + [rot // 2]))


def draw(rng):
    kind = rng.choice(["gemm", "gemm", "gemm", "norm", "norm", "quant", "rope", "rope"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "gemm":
        n, k = _log_int(rng, 48, 12288), _log_int(rng, 48, 8192)
        most = 14310 * 8192 * 2048 // (n * k)
        m = _log_int(rng, 1, max(1, min(14566, most)))
        return dict(kind=kind, m=m, n=n, k=k, dtype=dtype, epilogue=rng.choice(["bias", "gated", "gelu", "gelu8"]))
    rows = _log_int(rng, 1, 14566)
    if kind == "norm":
        return dict(kind=kind, rows=rows, width=_log_int(rng, 48, 8192, rng.choice([1, 8, 128])) if rows < 5000 else
                    _log_int(rng, 48, 2048, rng.choice([1, 8, 128])), dtype=dtype, resid=rng.random() < 0.6,
                    q8=rng.random() < 0.6)
    if kind == "quant":
        return dict(kind=kind, rows=rows, width=_log_int(rng, 48, 2048, rng.choice([1, 8, 128])), dtype=dtype,
                    tile=rng.choice([1, 1, 128]))
    dim = rng.choice([32, 64, 72, 80, 96, 128, 128, 256])
    hk = rng.choice([1, 2, 4, 8])
    hq = hk * rng.choice([1, 2, 4])
    # at most the bytes of the video model's q and k
    rows = max(1, min(rows, 14566 * 32 * 128 // (dim * (hq + hk))))
    norm = rng.random() < 0.5
    return dict(kind=kind, rows=rows, hq=hq, hk=hk, dim=dim, dtype=dtype, axes=_axes(rng, dim), halves=rng.random() < 0.5,
                ladder=rng.random() < 0.5, norm=norm, inverse=not norm and rng.random() < 0.3)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

class _Rand:
    """Seeded normal tensors made on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(1000003 * (seed % (1 << 40)) + 29)

    def __call__(self, *dims, scale=1.0):
        return torch.randn(dims, generator=self.g, device=DEV, dtype=torch.float32).mul_(scale)

    def hidden(self, rows, width):
        """A residual stream: a spread of channel magnitudes with a few large ones."""
        x = self(rows, width)
        return x.mul_(torch.exp(self(width, scale=0.7)))


def _blocks(n):
    return (n + 127) // 128


def _pad16(n):
    return (n + 15) // 16 * 16


def _held8(rows, width):
    """An 8-bit buffer of whole 16-byte rows, and its part that holds values."""
    return torch.zeros((rows, _pad16(width)), dtype=torch.uint8, device=DEV).view(F8)[:, :width]


def _inputs(case, seed):
    """Everything the call reads, as tensors on the GPU."""
    r = _Rand(seed)
    kind, td = case["kind"], TD[case["dtype"]]
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        d = {"bias": r(n, scale=0.05).to(td)}
        for name, x, tile in (("a", r.hidden(m, k), 1), ("w", r(n, k, scale=0.02), 128)):
            q, s = _plain_quant(x, tile)
            d[name] = _held8(*x.shape)
            d[name].copy_(q)
            d[name + "_scale"] = s
        if case["epilogue"] == "gated":
            d["rpb"] = max(1, -(-m // 16))
            # the gate is the third of the six modulation chunks of a block
            d["gate"] = r(-(-m // d["rpb"]), 6 * n, scale=0.5)[:, 2 * n:3 * n]
            d["resid"] = r.hidden(m, n).to(td)
        return d
    if kind == "rope":
        rows, dim = case["rows"], case["dim"]
        n_axes = len(case["axes"].split(","))
        pos = torch.randint(0, 128, (n_axes, rows), generator=r.g, device=DEV, dtype=torch.int32)
        pos[0] = torch.arange(rows, device=DEV, dtype=torch.int32) + int(torch.randint(
            0, 20000, (1,), generator=torch.Generator().manual_seed(seed % (1 << 40))))
        # q and k lie in the rows of one packed qkv tensor
        qkv = r(rows, (case["hq"] + 2 * case["hk"]) * dim).to(td)
        d = {"pos": pos, "q": qkv[:, :case["hq"] * dim], "k": qkv[:, case["hq"] * dim:(case["hq"] + case["hk"]) * dim]}
        if case["norm"]:
            d["wq"], d["wk"] = (1 + r(dim, scale=0.2)).to(td), (1 + r(dim, scale=0.2)).to(td)
        return d
    d = {"x": r.hidden(case["rows"], case["width"]).to(td)}
    if kind == "norm":
        d["weight"] = (1 + r(case["width"], scale=0.2)).to(td)
        if case["resid"]:
            d["resid"] = r.hidden(case["rows"], case["width"]).to(td)
    return d


def _ladder(axes, one_ladder):
    """The axis of every pair of a head and its radians per position."""
    axis = [a for a, width in enumerate(axes) for _ in range(width // 2)]
    if one_ladder:
        freq = [THETA ** (-2.0 * p / sum(axes)) for p in range(len(axis))]
    else:
        freq = [THETA ** (-2.0 * i / width) for width in axes for i in range(width // 2)]
    return torch.tensor(axis, device=DEV), torch.tensor(freq, dtype=torch.float64, device=DEV)


def prepare(case, seed):
    s = {"case": dict(case), **_inputs(case, seed)}
    kind, td = case["kind"], TD[case["dtype"]]
    if kind == "rope":
        s["axes"] = tuple(int(a) for a in case["axes"].split(","))
        s["axis"], s["freq"] = _ladder(s["axes"], case["ladder"])
        s["q_out"], s["k_out"] = (torch.empty(s[n].shape, dtype=td, device=DEV) for n in "qk")
        return s
    rows, width = (case["m"], case["n"]) if kind == "gemm" else (case["rows"], case["width"])
    if kind == "norm" and case["resid"]:
        s["sum"] = torch.empty((rows, width), dtype=td, device=DEV)
    if kind == "quant" or case.get("q8") or case.get("epilogue") == "gelu8":
        s["q8"] = _held8(rows, width)
        dims = (_blocks(rows), _blocks(width)) if case.get("tile") == 128 else (_blocks(width), rows)
        s["scale"] = torch.empty(dims, dtype=torch.float32, device=DEV)
    else:
        s["out"] = torch.empty((rows, width), dtype=td, device=DEV)
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    from paper_2607_27842_gb300 import featfix as ff
    c = s["case"]
    kind, dt = c["kind"], c["dtype"]
    if kind == "gemm":
        ff.featfix_op_gemm8(dt, s["a"], s["a_scale"], s["w"], s["w_scale"], out=s.get("out"), bias=s["bias"],
                            act=1 if c["epilogue"].startswith("gelu") else 0, gate=s.get("gate"),
                            rows_per_batch=s.get("rpb", 0), resid=s.get("resid"), q=s.get("q8"), q_scale=s.get("scale"))
        return {"q": s["q8"], "scale": s["scale"]} if "q8" in s else {"out": s["out"]}
    if kind == "norm":
        ff.featfix_op_rms_norm(dt, s["x"], s["weight"], EPS, resid=s.get("resid"), sum_out=s.get("sum"),
                               out=s.get("out"), q=s.get("q8"), q_scale=s.get("scale"))
        d = {"q": s["q8"], "scale": s["scale"]} if c["q8"] else {"out": s["out"]}
        if c["resid"]:
            d["sum"] = s["sum"]
        return d
    if kind == "quant":
        ff.featfix_op_quant8(dt, s["x"], s["q8"], s["scale"], c["tile"])
        return {"q": s["q8"], "scale": s["scale"]}
    ff.featfix_op_rope(dt, s["pos"], s["axes"], c["dim"], q=s["q"], q_out=s["q_out"], k=s["k"], k_out=s["k_out"],
                       theta=THETA, halves=c["halves"], one_ladder=c["ladder"], inverse=c["inverse"],
                       q_weight=s.get("wq"), k_weight=s.get("wk"), eps=EPS)
    return {"q": s["q_out"], "k": s["k_out"]}


def _plain_quant(x, tile):
    """x (fp32) in e4m3, and its scales: tile 1 per row and 128 columns, 128 per
    128 x 128 block."""
    rows, width = x.shape
    pad = torch.nn.functional.pad(x, (0, -width % 128, 0, -rows % tile))
    v = pad.view(pad.shape[0] // tile, tile, pad.shape[1] // 128, 128)
    scale = (v.abs().amax(dim=(1, 3)) / Q_MAX).clamp(min=S_MIN)
    q = (v / scale[:, None, :, None]).clamp(-Q_MAX, Q_MAX).to(F8).view(pad.shape)[:rows, :width]
    return q, scale if tile == 128 else scale.t().contiguous()


def _plain_values(q, scale, tile):
    """The values that an 8-bit tensor stands for."""
    per = scale.t() if tile == 1 else scale.repeat_interleave(128, 0)[:q.shape[0]]
    return q.float() * per.repeat_interleave(128, 1)[:, :q.shape[1]]


def _plain_rms(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _plain_rope(x, s, weight):
    c = s["case"]
    rot = sum(s["axes"])
    # an angle of up to 35000 radians in 32 bits alone would be 2e-3 off
    ang = s["pos"].double()[s["axis"]].t() * s["freq"]
    ang = torch.remainder(ang, 2 * math.pi).float()[:, None, :]
    cos, sin = ang.cos(), ang.sin()
    if c["inverse"]:
        sin = -sin
    v = x.float().reshape(x.shape[0], -1, c["dim"])
    if weight is not None:
        v = _plain_rms(v) * weight.float()
    if c["halves"]:
        u, w = v[..., :rot // 2], v[..., rot // 2:rot]
        turned = torch.cat([u * cos - w * sin, u * sin + w * cos], -1)
    else:
        u, w = v[..., 0:rot:2], v[..., 1:rot:2]
        turned = torch.stack([u * cos - w * sin, u * sin + w * cos], -1).flatten(-2)
    return torch.cat([turned, v[..., rot:]], -1).reshape(x.shape).to(x.dtype)


def _run_plain(s):
    c = s["case"]
    kind, td = c["kind"], TD[c["dtype"]]
    if kind == "quant":
        q, scale = _plain_quant(s["x"].float(), c["tile"])
        return {"q": q, "scale": scale}
    if kind == "rope":
        return {"q": _plain_rope(s["q"], s, s.get("wq")), "k": _plain_rope(s["k"], s, s.get("wk"))}
    if kind == "norm":
        h = s["x"].float()
        if c["resid"]:
            h = h + s["resid"].float()
        y = _plain_rms(h) * s["weight"].float()
        if c["q8"]:
            q, scale = _plain_quant(y, 1)
            d = {"q": q, "scale": scale}
        else:
            d = {"out": y.to(td)}
        if c["resid"]:
            d["sum"] = h.to(td)
        return d
    y = _plain_values(s["a"], s["a_scale"], 1) @ _plain_values(s["w"], s["w_scale"], 128).t() + s["bias"].float()
    if c["epilogue"].startswith("gelu"):
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if c["epilogue"] == "gelu8":
        q, scale = _plain_quant(y, 1)
        return {"q": q, "scale": scale}
    if c["epilogue"] == "gated":
        y = s["resid"].float() + s["gate"].repeat_interleave(s["rpb"], 0)[:c["m"]] * y
    return {"out": y.to(td)}


# ----------------------------------------------------------------------------
# the same in float64, from the definitions
# ----------------------------------------------------------------------------

def _exact_quant(x):
    """(x / scale, scale) per row and 128 columns, the former without its rounding."""
    parts, scales = [], []
    for b in range(0, x.shape[1], 128):
        part = x[:, b:b + 128]
        scale = torch.clamp(part.abs().max(dim=1).values / Q_MAX, min=S_MIN)
        parts.append(part / scale.unsqueeze(1))
        scales.append(scale)
    return torch.cat(parts, 1), torch.stack(scales)


def exact(case, seed):
    d = _inputs(case, seed)
    kind = case["kind"]
    if kind == "gemm":
        acc = torch.zeros((case["m"], case["n"]), dtype=torch.float64, device=DEV)
        of_row = torch.arange(case["n"], device=DEV) // 128
        for b in range(_blocks(case["k"])):
            at = slice(128 * b, min(case["k"], 128 * b + 128))
            part = d["a"][:, at].to(torch.float64) @ d["w"][:, at].to(torch.float64).T
            acc += part * d["a_scale"][b].double()[:, None] * d["w_scale"][of_row, b].double()[None, :]
        acc += d["bias"].double()
        if case["epilogue"].startswith("gelu"):
            # x (1 + tanh u) / 2 = x / (1 + exp(-2u))
            acc = acc * torch.sigmoid(2 * math.sqrt(2 / math.pi) * acc * (1 + 0.044715 * acc ** 2))
        if case["epilogue"] == "gelu8":
            q, scale = _exact_quant(acc)
            return {"q": q, "scale": scale}
        if case["epilogue"] == "gated":
            of_sample = torch.arange(case["m"], device=DEV) // d["rpb"]
            acc = d["resid"].double() + d["gate"].double()[of_sample] * acc
        return {"out": acc}
    if kind == "quant":
        x = d["x"].double()
        if case["tile"] == 1:
            q, scale = _exact_quant(x)
            return {"q": q, "scale": scale}
        rows, cols = x.shape
        scale = torch.empty((_blocks(rows), _blocks(cols)), dtype=torch.float64, device=DEV)
        for i in range(scale.shape[0]):
            for j in range(scale.shape[1]):
                block = x[128 * i:128 * i + 128, 128 * j:128 * j + 128]
                scale[i, j] = torch.clamp(block.abs().max() / Q_MAX, min=S_MIN)
                block /= scale[i, j]
        return {"q": x, "scale": scale}
    if kind == "norm":
        h = d["x"].double()
        if case["resid"]:
            h = h + d["resid"].double()
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["width"] + EPS) * d["weight"].double()
        q, scale = _exact_quant(y) if case["q8"] else (None, None)
        got = {"q": q, "scale": scale} if case["q8"] else {"out": y}
        if case["resid"]:
            got["sum"] = h
        return got
    axes = [int(a) for a in case["axes"].split(",")]
    rot, sign = sum(axes), -1.0 if case["inverse"] else 1.0
    got = {}
    for name, heads in (("q", case["hq"]), ("k", case["hk"])):
        v = d[name].double().reshape(case["rows"], heads, case["dim"])
        if case["norm"]:
            v = v / torch.sqrt((v * v).sum(-1, keepdim=True) / case["dim"] + EPS) * d["w" + name].double()
        y, p = v.clone(), 0
        for a, width in enumerate(axes):
            for i in range(width // 2):
                f = THETA ** (-2 * p / rot) if case["ladder"] else THETA ** (-2 * i / width)
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), sign * f * d["pos"][a].double())
                j, k = (p, p + rot // 2) if case["halves"] else (2 * p, 2 * p + 1)
                z = torch.complex(v[..., j], v[..., k]) * turn[:, None]
                y[..., j], y[..., k] = z.real, z.imag
                p += 1
        got[name] = y.reshape(case["rows"], heads * case["dim"])
    return got


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    kind, b = case["kind"], 4 if case["dtype"] == "f32" else 2
    if kind == "gemm":
        m, n, k = case["m"], case["n"], case["k"]
        out = m * n + 4 * m * _blocks(n) if case["epilogue"] == "gelu8" else m * n * b
        more = m * n * b + 4 * min(m, 16) * n if case["epilogue"] == "gated" else 0
        return {"bytes": m * k + n * k + 4 * _blocks(k) * (m + _blocks(n)) + n * b + more + out, "flops": 2 * m * n * k}
    if kind == "rope":
        n = case["rows"] * (case["hq"] + case["hk"]) * case["dim"]
        return {"bytes": 2 * n * b + 4 * case["rows"] * len(case["axes"].split(",")), "flops": 4 * n}
    n, rows = case["rows"] * case["width"], _blocks(case["rows"]) if case.get("tile") == 128 else case["rows"]
    in8 = n + 4 * rows * _blocks(case["width"])
    if kind == "quant":
        return {"bytes": n * b + in8, "flops": 2 * n}
    resid = 2 * n * b if case["resid"] else 0
    return {"bytes": n * b + resid + case["width"] * b + (in8 if case["q8"] else n * b), "flops": 4 * n}
