"""Performance cases of the 8-bit key-value cache's operators and of the norms
before and after a block.

Each case is one call of an operator as a program using this package makes it,
on buffers that such a program keeps:

  write      new tokens' keys and values into a paged cache: e4m3 values with a
             scale for every token and head.
  read       the last tokens of each sequence back out of the cache, in the
             model's type and in adjacent rows.
  attention  one new token of each sequence over its cached tokens, several
             query heads to a key head, optionally over a window's last tokens
             only, with the logarithm of the softmax sum where asked for.
  norms      h = resid_scale * x + gate * (norm(y) * weight_after), the end of a
             block; norm(h) * weight * (1 + scale) + shift, the beginning of the
             next one, rounded or in 8 bits with a scale for every 128 columns.

A cache is k8, v8 [pages, page size, heads, dim] with k_scale, v_scale [pages,
page size, heads]; row b of the page table holds the pages of sequence b, lens[b]
its tokens, of which the last row_start[b + 1] - row_start[b] are the rows of a
write or read.  Values in 8 bits are returned as float8 with their scales beside
them.

``listed()`` holds sizes of the package's own workloads (a video model of width
2048, 16 heads of 128, 14310 image and 256 text tokens; DiT-XL/2 with its heads of
72 over 256 tokens) and generic and ragged ones, ``draw()`` gives others of the same
ranges, ``exact()`` restates each call in float64.
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


# ----------------------------------------------------------------------------
# the cases
# ----------------------------------------------------------------------------

def listed():
    return [
        # One new token of one sequence, four key heads: latency alone.
        dict(name="write 1 token 4 heads", kind="write", seqs=1, new=1, had=300, ragged=False, heads=4, dim=128, page=64,
             layout="token", dtype="bf16"),
        # All of the video model's tokens, as the keys and values of a later call.
        dict(name="write 14566 tokens 16 heads", kind="write", seqs=1, new=14566, had=0, ragged=False, heads=16, dim=128,
             page=64, layout="token", dtype="bf16"),
        # Pieces of different length of 37 sequences behind what they hold, with
        # DiT-XL/2's heads, in fp32, heads outside of the tokens of a page.
        dict(name="write 37 ragged f32 dim 72", kind="write", seqs=37, new=150, had=400, ragged=True, heads=16, dim=72,
             page=24, layout="head", dtype="f32"),
        # The video model's cached tokens back in adjacent rows.
        dict(name="read 14566 tokens 16 heads", kind="read", seqs=1, tokens=14566, ragged=False, heads=16, dim=128, page=64,
             layout="token", dtype="bf16"),
        # Sequences of different length, three heads of 80, pages of 24.
        dict(name="read 19 ragged f32 dim 80", kind="read", seqs=19, tokens=777, ragged=True, heads=3, dim=80, page=24,
             layout="head", dtype="f32"),
        # One sequence just past a prompt of 256 tokens: latency alone.
        dict(name="attention 1x257 16+4 heads", kind="attention", seqs=1, tokens=257, ragged=False, hq=16, hk=4, dim=128,
             page=64, layout="token", dtype="bf16", window=0, lse=False),
        # One long sequence: its length has to be shared out over the whole GPU.
        dict(name="attention 1x131072 16+4 heads", kind="attention", seqs=1, tokens=131072, ragged=False, hq=16, hk=4,
             dim=128, page=64, layout="token", dtype="bf16", window=0, lse=False),
        # A batch in service: 64 sequences of 1 to 8192 tokens, pages of 16.
        dict(name="attention 64 ragged 32+8 heads", kind="attention", seqs=64, tokens=8192, ragged=True, hq=32, hk=8,
             dim=128, page=16, layout="token", dtype="bf16", window=0, lse=False),
        # DiT-XL/2's heads in fp32, a key head to each query head, with the
        # softmax's sums, heads outside of the tokens of a page.
        dict(name="attention 48x700 16+16 f32 dim 72", kind="attention", seqs=48, tokens=700, ragged=True, hq=16, hk=16,
             dim=72, page=32, layout="head", dtype="f32", window=256, lse=True),
        # The norms around one token's MLP.
        dict(name="norms 1x2048 q8", kind="norms", rows=1, width=2048, dtype="bf16", samples=1, after=True, modulated=False,
             q8=True, centered=False),
        # All of the video model's tokens: gate, shift and scale of two samples.
        dict(name="norms 14566x2048 q8", kind="norms", rows=14566, width=2048, dtype="bf16", samples=2, after=True,
             modulated=True, q8=True, centered=False),
        # fp32 rows of a width that no vector divides, norms that subtract the
        # mean, as an adaLN block has them.
        dict(name="norms 1333x1001 f32", kind="norms", rows=1333, width=1001, dtype="f32", samples=3, after=False,
             modulated=True, q8=False, centered=True),
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer spread over the logarithm of [lo, hi], a multiple of step."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(step, int(round(v / step)) * step)


def draw(rng):
    kind = rng.choice(["write", "write", "read", "attention", "attention", "attention", "attention", "norms", "norms"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norms":
        rows = _log_int(rng, 1, 14566)
        width = _log_int(rng, 48, 8192 if rows < 3500 else 2048, rng.choice([1, 8, 128]))
        return dict(kind=kind, rows=rows, width=width, dtype=dtype, samples=rng.randint(1, min(rows, 8)),
                    after=rng.random() < 0.7, modulated=rng.random() < 0.6, q8=rng.random() < 0.5,
                    centered=rng.random() < 0.4)
    dim = rng.choice([32, 64, 72, 80, 96, 128, 128, 128, 256])
    heads = rng.choice([1, 2, 3, 4, 8, 16])
    more = dict(kind=kind, dim=dim, page=rng.choice([8, 16, 16, 24, 32, 64, 64, 128]), dtype=dtype,
                layout=rng.choice(["token", "head"]), ragged=rng.random() < 0.6)
    seqs = _log_int(rng, 1, 256)
    most = 64 * 4096 * 8 * 128 // (heads * dim)      # tokens that the largest attention reads
    if kind == "attention":
        group = rng.choice([1, 2, 4, 5, 8, 16])
        most = most * 4 // max(4, group)             # and the products of its query heads
        tokens = _log_int(rng, 1, max(1, min(131072, most // seqs)))
        return dict(more, seqs=seqs, tokens=tokens, hq=heads * group, hk=heads,
                    window=_log_int(rng, 1, tokens) if rng.random() < 0.3 else 0, lse=rng.random() < 0.3)
    most = 14566 * 16 * 128 // (heads * dim)         # of the largest write
    new = _log_int(rng, 1, max(1, most // seqs))
    if kind == "read":
        return dict(more, seqs=seqs, tokens=new, heads=heads)
    return dict(more, seqs=seqs, new=rng.choice([1, new]), had=rng.choice([0, _log_int(rng, 1, 2000)]), heads=heads)


def _spread(n, most, least):
    """n lengths from `least` to `most`, evenly spread and out of order; the first is `most`."""
    return [most - int((most - least + 0.999) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _counts(case):
    """Rows of each sequence in the call, and its tokens with them."""
    n = case["seqs"]
    if case["kind"] == "attention":
        # of a larger batch, the last place stays free
        lens = _spread(n, case["tokens"], min(1, case["tokens"])) if case["ragged"] else [case["tokens"]] * n
        if case["ragged"] and n > 2 and not case["lse"]:
            lens[-1] = 0
        return [1] * n, lens
    if case["kind"] == "read":
        rows = _spread(n, case["tokens"], 0) if case["ragged"] else [case["tokens"]] * n
        return rows, rows
    rows = _spread(n, case["new"], 0) if case["ragged"] and case["new"] > 1 else [case["new"]] * n
    had = _spread(n, case["had"], 0)[::-1] if case["ragged"] else [case["had"]] * n
    return rows, [a + b for a, b in zip(rows, had)]


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

class _Rand:
    """Seeded normal tensors made on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(1000003 * (seed % (1 << 40)) + 71)

    def __call__(self, *dims, scale=1.0):
        return torch.randn(dims, generator=self.g, device=DEV, dtype=torch.float32).mul_(scale)

    def hidden(self, rows, width):
        """A residual stream: a spread of channel magnitudes with a few large ones."""
        return self(rows, width).mul_(torch.exp(self(width, scale=0.7)))

    def heads(self, rows, heads, dim, channel=0.4):
        """Keys or values: channels and tokens of different magnitude."""
        return self(rows, heads, dim).mul_(torch.exp(self(heads, dim, scale=channel))).mul_(
            torch.exp(self(rows, 1, 1, scale=0.3)))


def _blocks(n):
    return (n + 127) // 128


def _pad16(n):
    return (n + 15) // 16 * 16


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _pool(r, pages, page, heads, dim, layout):
    """A filled pool of pages: 8-bit values and their scales, in the order of the layout."""
    rows = page * heads
    q = torch.zeros((pages, rows, _pad16(dim)), dtype=torch.uint8, device=DEV)
    s = torch.empty((pages, rows), dtype=torch.float32, device=DEV)
    step = max(1, (1 << 27) // (rows * dim))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        codes, scale = _plain_quant_heads(r.heads(n * page, heads, dim))
        q[p:p + n, :, :dim] = codes.view(torch.uint8).view(n, rows, dim)
        s[p:p + n] = scale.view(n, rows)
    dims = (pages, page, heads) if layout == "token" else (pages, heads, page)
    q, s = q.view(*dims, -1)[..., :dim], s.view(dims)
    return (q, s) if layout == "token" else (q.transpose(1, 2), s.transpose(1, 2))


def _inputs(case, seed):
    """Everything the call reads, as tensors on the GPU."""
    r = _Rand(seed)
    td = TD[case["dtype"]]
    if case["kind"] == "norms":
        rows, width = case["rows"], case["width"]
        d = {"x": r.hidden(rows, width).to(td), "y": r.hidden(rows, width).to(td),
             "weight": (1 + r(width, scale=0.2)).to(td), "rpb": -(-rows // case["samples"])}
        if case["after"]:
            d["weight_after"] = (1 + r(width, scale=0.2)).to(td)
        if case["modulated"]:
            # three of the six chunks of a block's modulation
            mod = r(-(-rows // d["rpb"]), 6 * width, scale=0.5)
            d["gate"], d["shift"], d["scale"] = (mod[:, i * width:(i + 1) * width] for i in (2, 3, 4))
        return d
    counts, lens = _counts(case)
    page, dim = case["page"], case["dim"]
    heads = case["hk"] if case["kind"] == "attention" else case["heads"]
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 3, generator=r.g, device=DEV).to(torch.int32)
    # places of the table behind a sequence's end are never looked at
    table = torch.full((case["seqs"], max(1, max(need))), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    d = {"table": table, "lens": _int32(lens)}
    for name in "kv":
        d[name + "8"], d[name + "_scale"] = _pool(r, sum(need) + 3, page, heads, dim, case["layout"])
    if case["kind"] == "attention":
        q = r.heads(case["seqs"], case["hq"], dim)
        d["q"] = q.view(case["seqs"], -1).to(td)
        return d
    rows = sum(counts)
    if case["kind"] == "read" or case["new"] > 1:
        d["row_start"] = _int32([sum(counts[:i]) for i in range(len(counts) + 1)])
    if case["kind"] == "write":
        # the keys and values lie in the rows of one packed qkv tensor
        qkv = torch.cat([r.heads(rows, heads, dim).view(rows, -1) for _ in range(3)], 1).to(td)
        d["k"], d["v"] = qkv[:, heads * dim:2 * heads * dim], qkv[:, 2 * heads * dim:]
    return d


def prepare(case, seed):
    s = {"case": dict(case), **_inputs(case, seed)}
    td = TD[case["dtype"]]
    empty = lambda *dims: torch.empty(dims, dtype=td, device=DEV)
    if case["kind"] == "norms":
        rows, width = case["rows"], case["width"]
        s["sum"] = empty(rows, width)
        if case["q8"]:
            s["q8"] = torch.zeros((rows, _pad16(width)), dtype=torch.uint8, device=DEV).view(F8)[:, :width]
            s["q8_scale"] = torch.empty((_blocks(width), rows), dtype=torch.float32, device=DEV)
        else:
            s["out"] = empty(rows, width)
        return s
    if case["kind"] == "read":
        rows = sum(_counts(case)[0])
        s["k"], s["v"] = (empty(rows, case["heads"] * case["dim"]) for _ in range(2))
    if case["kind"] == "attention":
        s["out"] = empty(*s["q"].shape)
        if case["lse"]:
            s["lse"] = torch.empty((case["seqs"], case["hq"]), dtype=torch.float32, device=DEV)
        if own:
            from paper_2607_27842_gb300 import featfix as ff
            n = ff.featfix_op_kv_attention_workspace(case["seqs"], case["hq"], case["hk"], case["dim"],
                                                     s["table"].shape[1] * case["page"])
            s["workspace"] = torch.empty(n, dtype=torch.uint8, device=DEV)
    return s


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _cache(s):
    return s["k8"], s["k_scale"], s["v8"], s["v_scale"]


def _written(s):
    return {"k8": s["k8"].view(F8), "k_scale": s["k_scale"], "v8": s["v8"].view(F8), "v_scale": s["v_scale"]}


def _run_own(s):
    from paper_2607_27842_gb300 import featfix as ff
    c = s["case"]
    kind, dt = c["kind"], c["dtype"]
    if kind == "write":
        ff.featfix_op_kv_write(dt, s["k"], s["v"], _cache(s), s["table"], s["lens"], row_start=s.get("row_start"))
        return _written(s)
    if kind == "read":
        ff.featfix_op_kv_read(dt, _cache(s), s["table"], s["lens"], s["k"], s["v"], row_start=s["row_start"])
        return {"k": s["k"], "v": s["v"]}
    if kind == "attention":
        ff.featfix_op_kv_attention(dt, s["q"], _cache(s), s["table"], s["lens"], s["out"], s["workspace"],
                                   scale=c["dim"] ** -0.5, window=c["window"], lse=s.get("lse"))
        return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}
    ff.featfix_op_block_norms(dt, s["y"], s["x"], EPS, weight_after=s.get("weight_after"), norm_after=c["after"],
                              resid_scale=0.9, gate=s.get("gate"), sum_out=s["sum"], weight=s["weight"],
                              shift=s.get("shift"), scale=s.get("scale"), rows_per_batch=s["rpb"],
                              centered=c["centered"], out=s.get("out"), q=s.get("q8"), q_scale=s.get("q8_scale"))
    return {"q": s["q8"], "scale": s["q8_scale"], "sum": s["sum"]} if c["q8"] else {"out": s["out"], "sum": s["sum"]}


def _plain_quant_heads(x):
    """x (fp32) in e4m3, and a scale for each vector of its last dimension."""
    scale = (x.abs().amax(-1) / Q_MAX).clamp(min=S_MIN)
    return (x / scale[..., None]).clamp(-Q_MAX, Q_MAX).to(F8), scale


def _plain_places(s, page):
    """Page and place in it of every row of the call."""
    counts, lens = s["row_start"].diff() if "row_start" in s else torch.ones_like(s["lens"]), s["lens"]
    n = (s["k"] if "k" in s else s["q"]).shape[0]
    start = counts.cumsum(0) - counts
    seq = torch.repeat_interleave(torch.arange(len(counts), device=DEV), counts, output_size=n)
    pos = torch.arange(n, device=DEV) - start[seq] + (lens - counts)[seq]
    return s["table"][seq, pos // page].long(), pos % page


def _plain_attention(s):
    c = s["case"]
    hk, dim, page = c["hk"], c["dim"], c["page"]
    group, width = c["hq"] // hk, s["table"].shape[1] * page
    pos = torch.arange(width, device=DEV)
    step = max(1, (1 << 28) // (width * hk * dim))
    outs, lses = [], []
    for b in range(0, c["seqs"], step):
        table, lens = s["table"][b:b + step], s["lens"][b:b + step, None]
        at = (table[:, pos // page].long().clamp(min=0), (pos % page)[None])
        seen = (pos < lens) & (pos >= lens - (c["window"] or width))
        q = s["q"][b:b + step].float().view(-1, hk, group, dim)
        k = s["k8"][at].view(F8).float() * s["k_scale"][at][..., None]
        x = q @ k.permute(0, 2, 3, 1) * dim ** -0.5
        del k
        x = x.masked_fill(~seen[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        p = torch.exp(x - top.clamp(min=-3e38))
        total = p.sum(-1, keepdim=True)
        v = s["v8"][at].view(F8).float() * s["v_scale"][at][..., None]
        o = p @ v.transpose(1, 2) / total.clamp(min=1e-37)
        outs.append(o.reshape(-1, c["hq"] * dim).to(s["q"].dtype))
        lses.append((top + total.log()).reshape(-1, c["hq"]))
    return {"out": torch.cat(outs), "lse": torch.cat(lses)} if c["lse"] else {"out": torch.cat(outs)}


def _plain_norm(x, centered):
    if centered:
        x = x - x.mean(-1, keepdim=True)
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _run_plain(s):
    c = s["case"]
    kind, td = c["kind"], TD[c["dtype"]]
    if kind == "write":
        at = _plain_places(s, c["page"])
        for name in "kv":
            q, scale = _plain_quant_heads(s[name].float().view(-1, c["heads"], c["dim"]))
            s[name + "8"][at] = q.view(torch.uint8)
            s[name + "_scale"][at] = scale
        return _written(s)
    if kind == "read":
        at = _plain_places(s, c["page"])
        got = {}
        for name in "kv":
            x = s[name + "8"][at].view(F8).float() * s[name + "_scale"][at][..., None]
            got[name] = x.to(td).view(s[name].shape)
        return got
    if kind == "attention":
        return _plain_attention(s)

    def rows(m):
        return m.repeat_interleave(s["rpb"], 0)[:c["rows"]]

    h = s["y"].float()
    if c["after"]:
        h = _plain_norm(h, c["centered"]) * s["weight_after"].float()
    if c["modulated"]:
        h = h * rows(s["gate"])
    h = 0.9 * s["x"].float() + h
    y = _plain_norm(h, c["centered"]) * s["weight"].float()
    if c["modulated"]:
        y = y * (1 + rows(s["scale"])) + rows(s["shift"])
    if not c["q8"]:
        return {"out": y.to(td), "sum": h.to(td)}
    pad = torch.nn.functional.pad(y, (0, -c["width"] % 128))
    q, scale = _plain_quant_heads(pad.view(c["rows"], -1, 128))
    return {"q": q.view(pad.shape)[:, :c["width"]], "scale": scale.t().contiguous(), "sum": h.to(td)}


# ----------------------------------------------------------------------------
# the same in float64, from the definitions
# ----------------------------------------------------------------------------

def _exact_attention(case, d):
    hk, dim = case["hk"], case["dim"]
    out = torch.zeros((case["seqs"], case["hq"], dim), dtype=torch.float64, device=DEV)
    lse = torch.full((case["seqs"], case["hq"]), -math.inf, dtype=torch.float64, device=DEV)
    for b, n in enumerate(_counts(case)[1]):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == first:
            continue
        token = torch.arange(first, n, device=DEV)
        page, slot = d["table"][b].long()[torch.div(token, case["page"], rounding_mode="floor")], token % case["page"]
        for h in range(hk):
            heads = slice(h * case["hq"] // hk, (h + 1) * case["hq"] // hk)
            key = d["k8"][page, slot, h].view(F8).to(torch.float64) * d["k_scale"][page, slot, h].double().unsqueeze(1)
            value = d["v8"][page, slot, h].view(F8).to(torch.float64) * d["v_scale"][page, slot, h].double().unsqueeze(1)
            x = d["q"][b].double().view(-1, dim)[heads] @ key.T / math.sqrt(dim)
            out[b, heads] = torch.softmax(x, 1) @ value
            lse[b, heads] = torch.logsumexp(x, 1)
    got = {"out": out.view(case["seqs"], -1)}
    if case["lse"]:
        got["lse"] = lse
    return got


def _exact_cache(case, d):
    counts, lens = _counts(case)
    page, dim = case["page"], case["dim"]
    token = [t for n, total in zip(counts, lens) for t in range(total - n, total)]
    seq = [b for b, n in enumerate(counts) for _ in range(n)]
    token, seq = torch.tensor(token, device=DEV), torch.tensor(seq, device=DEV)
    pages, slots = d["table"].long()[seq, torch.div(token, page, rounding_mode="floor")], token % page
    got = {}
    for name in "kv":
        q, scale = d[name + "8"].contiguous().view(F8).to(torch.float64), d[name + "_scale"].double()
        if case["kind"] == "read":
            got[name] = (q[pages, slots] * scale[pages, slots].unsqueeze(2)).flatten(1)
            continue
        x = d[name].double().reshape(len(seq), case["heads"], dim)
        s = torch.clamp(x.abs().max(dim=2).values / Q_MAX, min=S_MIN)
        scale[pages, slots] = s
        q[pages, slots] = x / s.unsqueeze(2)
        got[name + "8"], got[name + "_scale"] = q, scale
    return got


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "attention":
        return _exact_attention(case, d)
    if case["kind"] != "norms":
        return _exact_cache(case, d)

    def norm(x, weight):
        if case["centered"]:
            x = x - x.sum(1, keepdim=True) / case["width"]
        return x / torch.sqrt((x * x).sum(1, keepdim=True) / case["width"] + EPS) * weight.double()

    of_sample = torch.arange(case["rows"], device=DEV) // d["rpb"]
    y = d["y"].double()
    if case["after"]:
        y = norm(y, d["weight_after"])
    if case["modulated"]:
        y = d["gate"].double()[of_sample] * y
    h = 0.9 * d["x"].double() + y
    y = norm(h, d["weight"])
    if case["modulated"]:
        y = y + y * d["scale"].double()[of_sample] + d["shift"].double()[of_sample]
    if not case["q8"]:
        return {"out": y, "sum": h}
    parts, scales = [], []
    for b in range(0, case["width"], 128):
        s = torch.clamp(y[:, b:b + 128].abs().max(dim=1).values / Q_MAX, min=S_MIN)
        parts.append(y[:, b:b + 128] / s.unsqueeze(1))
        scales.append(s)
    return {"q": torch.cat(parts, 1), "scale": torch.stack(scales), "sum": h}


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------

def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norms":
        n = case["rows"] * case["width"]
        mod = 12 * case["samples"] * case["width"] if case["modulated"] else 0
        out = n + 4 * case["rows"] * _blocks(case["width"]) if case["q8"] else n * b
        return {"bytes": 3 * n * b + out + (2 if case["after"] else 1) * case["width"] * b + mod, "flops": 12 * n}
    counts, lens = _counts(case)
    if case["kind"] == "attention":
        seen = sum(min(n, case["window"] or n) for n in lens)
        lse = 4 * case["hq"] * case["seqs"] if case["lse"] else 0
        return {"bytes": seen * case["hk"] * 2 * (case["dim"] + 4) + 2 * case["seqs"] * case["hq"] * case["dim"] * b + lse,
                "flops": 4 * seen * case["hq"] * case["dim"]}
    n = 2 * sum(counts) * case["heads"]
    return {"bytes": n * (case["dim"] * (b + 1) + 4), "flops": 2 * n * case["dim"]}
