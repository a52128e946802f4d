"""Operators of rankers held in 8 bits and of answers that are drawn, as cases that can be timed.

  quantize  rows (activations) or weights to e4m3 with a scale for each block of 128: `Context.quantize_e4m3`
  matmul    product of two such operands, with bias, ReLU and quantised output where a layer has them:
            `Context.matmul_e4m3`
  sample    draws from the softmax of scores with temperature, top-k, top-p and min-p, from given random numbers:
            `Context.sample`

With `own` the framework is called as a program calls it; without, the operators are written out in torch.
Sizes come from the repository's configurations (1,024 problems x 60,000 candidates, 64 x 2,048, the ranker
64-1024-1024-512-256-1) or are generic powers of two and their neighbours.
"""
import functools
import math

import torch

own = False

DEV = "cuda"
BLOCK = 128
TOP = 448.0  # largest e4m3 value
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
SCALE_BYTES = {"f32": 4, "e8m0": 1}


def listed():
    return [
        # activations of 60,000 candidates in front of a 1,024-wide layer
        dict(name="quantize_rows", kind="quantize", rows=60000, cols=1024, x="bf16", block_rows=1, scale="e8m0"),
        # a weight matrix, once per model
        dict(name="quantize_weights", kind="quantize", rows=8192, cols=8192, x="f32", block_rows=128, scale="f32"),
        # one row through a layer: a single request, latency counts
        dict(name="matmul_one_row", kind="matmul", m=1, n=4096, k=4096, scale="e8m0", d="bf16", bias=False, relu=False),
        # a short batch against large weights, scales of any value
        dict(name="matmul_few_rows", kind="matmul", m=48, n=8192, k=8192, scale="f32", d="bf16", bias=False, relu=False),
        # a hidden layer of the wide ranker over one problem's candidates, quantised for the next layer
        dict(name="matmul_layer", kind="matmul", m=60000, n=1024, k=1024, scale="e8m0", d="e4m3", bias=True, relu=True),
        # sizes that end inside tiles and blocks
        dict(name="matmul_ragged", kind="matmul", m=4001, n=4104, k=4250, scale="f32", d="f32", bias=True, relu=False),
        # the largest square
        dict(name="matmul_large", kind="matmul", m=8192, n=8192, k=8192, scale="e8m0", d="bf16", bias=False, relu=False),
        # one problem's scores: a dispatcher that draws one candidate per call
        dict(name="sample_one", kind="sample", p=1, c=60000, x="f32", draws=1, top_k=50, top_p=0.9, min_p=0.0, t=0.8,
             spread=2.2, masked=0.0, segments=False, per_row=False),
        # a small pool for a short list of problems
        dict(name="sample_tiny", kind="sample", p=64, c=2048, x="f32", draws=5, top_k=40, top_p=0.95, min_p=0.05, t=1.0,
             spread=1.0, masked=0.1, segments=False, per_row=False),
        # 16 candidates to measure for each problem of the tuning table
        dict(name="sample_table", kind="sample", p=1024, c=60000, x="f32", draws=16, top_k=0, top_p=0.95, min_p=0.0, t=1.0,
             spread=2.2, masked=0.0, segments=False, per_row=False),
        # every problem against its own candidates, with settings of its own
        dict(name="sample_segments", kind="sample", p=4096, c=32768, x="f32", draws=4, top_k=100, top_p=0.9, min_p=0.02,
             t=1.0, spread=2.2, masked=0.05, segments=True, per_row=True),
        # 16-bit scores over a large set, a batch of requests
        dict(name="sample_wide", kind="sample", p=64, c=131072, x="bf16", draws=1, top_k=0, top_p=0.92, min_p=0.001, t=0.7,
             spread=3.0, masked=0.0, segments=False, per_row=False),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["quantize", "matmul", "matmul", "sample", "sample"])
    if kind == "quantize":
        cols = _log(rng, 1, 16384)
        rows = _log(rng, 1, max(1, min(200000, (60 << 20) // cols)))
        return dict(kind=kind, rows=rows, cols=cols, x=rng.choice(["f32", "bf16", "f16"]), block_rows=rng.choice([1, 128]),
                    scale=rng.choice(["e8m0", "f32"]))
    if kind == "matmul":
        n, k = _log(rng, 1, 8192), _log(rng, 16, 8192)
        m = rng.choice([1, _log(rng, 1, 128), _log(rng, 128, 60000)])
        m = max(1, min(m, int(4e11 / n / k)))
        return dict(kind=kind, m=m, n=n, k=k, scale=rng.choice(["e8m0", "f32"]), d=rng.choice(["f32", "bf16", "f16", "e4m3"]),
                    bias=rng.random() < 0.5, relu=rng.random() < 0.5)
    c = _log(rng, 1, 534600)
    p = _log(rng, 1, max(1, min(4096, (32 << 20) // c)))
    return dict(kind=kind, p=p, c=c, x=rng.choice(["f32", "bf16", "f16"]), draws=rng.choice([1, 1, 5, 32]),
                top_k=rng.choice([0, 1, _log(rng, 2, 2000)]), top_p=rng.choice([1.0, round(rng.uniform(0.05, 1.0), 3)]),
                min_p=rng.choice([0.0, round(0.5 * rng.random() ** 3, 4)]), t=rng.choice([1.0, round(rng.uniform(0.1, 3.0), 2)]),
                spread=rng.choice([0.05, 1.0, 3.0, 8.0]), masked=rng.choice([0.0, 0.3]), segments=rng.random() < 0.4,
                per_row=rng.random() < 0.4)


# ---- inputs ------------------------------------------------------------------------------------


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _rows(g, rows, cols):
    """Values whose size differs from row to row and from block to block of columns, as activations' does."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    x *= torch.exp2(3 * torch.randn(rows, 1, generator=g, device=DEV))
    at = torch.arange(cols, device=DEV) // BLOCK
    return x.mul_(torch.exp2(2 * torch.randn(int(at[-1]) + 1, generator=g, device=DEV))[at])


def _padded(q):
    """The same values in rows that begin on 16-byte boundaries."""
    cols = q.shape[1]
    wide = torch.zeros(q.shape[0], -(-cols // 16) * 16, dtype=torch.uint8, device=q.device)
    wide[:, :cols] = q.view(torch.uint8)
    return wide.view(torch.float8_e4m3fn)[:, :cols]


@functools.lru_cache(maxsize=None)
def _context():
    from paper_2609_35587_b200 import binding as ks
    from paper_2609_35587_b200 import workloads as wl
    return ks.Context(wl.gpu_desc(), 0)


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case, "kind": case["kind"]}
    if case["kind"] == "quantize":
        s["data"] = _rows(g, case["rows"], case["cols"]).to(TYPES[case["x"]])
    elif case["kind"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        a, s["a_scale"] = _quantize(_rows(g, m, k), 1, case["scale"])
        b, s["b_scale"] = _quantize(torch.randn(n, k, generator=g, device=DEV) / math.sqrt(k), BLOCK, case["scale"])
        s["a"], s["b"] = _padded(a), _padded(b)
        s["bias"] = torch.randn(n, generator=g, device=DEV) if case["bias"] else None
    else:
        p, c = case["p"], case["c"]
        if case["segments"]:  # lengths spread over their logarithm, some empty
            lens = torch.exp(torch.rand(p, generator=g, device=DEV) * math.log(c + 1)).long().clamp_(max=c)
            lens[torch.rand(p, generator=g, device=DEV) < 0.02] = 0
            s["seg_off"] = torch.cat([lens.new_zeros(1), lens.cumsum(0)])
            shape = (int(s["seg_off"][-1]),)
            s["longest"] = int(lens.max())
        else:
            s["seg_off"] = None
            shape = (p, c)
        x = torch.randn(shape, generator=g, device=DEV) * case["spread"]
        if case["masked"]:
            hidden = torch.rand(shape, generator=g, device=DEV) < case["masked"]
            x = torch.where(hidden, torch.full_like(x, -math.inf), x)
        s["scores"] = x.to(TYPES[case["x"]])
        s["u"] = torch.rand(p, case["draws"], generator=g, device=DEV)
        rows = p if case["per_row"] else 1
        f = lambda v: torch.full((rows,), v, device=DEV)  # noqa: E731
        t, k, top_p, min_p = f(float(case["t"])), f(case["top_k"]), f(float(case["top_p"])), f(float(case["min_p"]))
        if case["per_row"]:  # half the rows ask for something of their own
            other = torch.rand(rows, generator=g, device=DEV) < 0.5
            t = torch.where(other, 0.25 + torch.rand(rows, generator=g, device=DEV), t)
            k = torch.where(other, torch.randint(0, 64, (rows,), generator=g, device=DEV), k)
            top_p = torch.where(other, 0.5 + 0.5 * torch.rand(rows, generator=g, device=DEV), top_p)
            min_p = torch.where(other, torch.zeros_like(min_p), min_p)
        s["t"], s["k"], s["tp"], s["mp"] = t, k.int(), top_p, min_p
        # what a serving program keeps beside its requests: their settings as the call takes them
        if case["per_row"]:
            s["params"] = torch.stack([t, k.int().view(torch.float32), top_p, min_p], 1).contiguous().view(torch.uint8)
    return s


# ---- the operators in plain form ----------------------------------------------------------------


def _blocks(x, block_rows):
    """[rows, cols] -> [row blocks, block_rows, column blocks, 128], zeros behind the ends."""
    r, c = -(-x.shape[0] // block_rows) * block_rows, -(-x.shape[1] // BLOCK) * BLOCK
    x = torch.nn.functional.pad(x, (0, c - x.shape[1], 0, r - x.shape[0]))
    return x.view(r // block_rows, block_rows, c // BLOCK, BLOCK)


def _quantize(x, block_rows, scale):
    rows, cols = x.shape
    b = _blocks(x.float(), block_rows)
    amax = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax((1, 3))
    top = torch.full_like(amax, TOP)
    if scale == "e8m0":  # the smallest power of two that brings the block below 448 = 0.875 * 2^9
        part, e = torch.frexp(amax)
        e = (e - 9 + (part > 0.875).int()).clamp(-127, 127)
        e = torch.where(amax > 0, e, torch.full_like(e, -127))
        s = (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)
        inv = torch.exp2(-e.double()).float()
    else:
        amax = amax.clamp(min=2.0 ** -100)
        s, inv = torch.div(amax, top), torch.div(top, amax)
    q = (b * inv[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(-1, b.shape[2] * BLOCK)[:rows, :cols], s


def _values(q, s, block_rows, to=torch.float32):
    b = _blocks(q.to(to), block_rows) * s.to(to)[:, None, :, None]
    return b.view(-1, b.shape[2] * BLOCK)[:q.shape[0], :q.shape[1]]


def _matmul(s):
    d = _values(s["a"], s["a_scale"], 1) @ _values(s["b"], s["b_scale"], BLOCK).t()
    if s["bias"] is not None:
        d = d + s["bias"]
    if s["case"]["relu"]:
        d = torch.where(d > 0, d, torch.zeros_like(d))
    return _quantize(d, 1, s["case"]["scale"]) if s["case"]["d"] == "e4m3" else d.to(TYPES[s["case"]["d"]])


def _sample(s):
    """All rows at once, in 64 bits: sorted by (score descending, index ascending), cut, put back in the order of the indices."""
    x = s["scores"]
    if s["seg_off"] is None:
        x = x.double()
    else:
        at = s["seg_off"][:-1, None] + torch.arange(max(1, s["longest"]), device=DEV)
        inside = at < s["seg_off"][1:, None]
        x = torch.nn.functional.pad(x, (0, 1))[torch.where(inside, at, torch.zeros_like(at))].double()
        x = torch.where(inside, x, torch.full_like(x, -math.inf))
    p, c = x.shape
    t, k, top_p, min_p = (v.expand(p)[:, None].double() for v in (s["t"], s["k"], s["tp"], s["mp"]))
    v, order = torch.sort(torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x), dim=1, descending=True, stable=True)
    best = v[:, :1]
    w = torch.where(v == best, torch.ones_like(v), torch.exp((v - best) / t))
    w = torch.where(v > -math.inf, w, torch.zeros_like(w))
    rank = torch.arange(c, device=DEV)
    w = torch.where((k <= 0) | (rank < k), w, torch.zeros_like(w))
    before = torch.cumsum(w, 1) - w
    w = torch.where((top_p >= 1) | (before < top_p * w.sum(1, keepdim=True)), w, torch.zeros_like(w))
    w = torch.where(w >= min_p, w, torch.zeros_like(w))
    w = torch.zeros_like(w).scatter_(1, order, w)
    cum = torch.cumsum(w, 1)
    total = cum[:, -1:]
    idx = torch.searchsorted(cum, s["u"].double() * total, right=True).clamp_(max=c - 1)
    some = (total > 0).expand_as(idx)
    logp = torch.log(w.gather(1, idx) / total)
    return {"idx": torch.where(some, idx, torch.full_like(idx, -1)).int(),
            "logp": torch.where(some, logp, torch.full_like(logp, -math.inf)).float()}


def run(state):
    s, c = state, state["case"]
    if own:
        ctx = _context()
        if s["kind"] == "quantize":
            return ctx.quantize_e4m3(s["data"], block_rows=c["block_rows"], scale=c["scale"])
        if s["kind"] == "matmul":
            return ctx.matmul_e4m3(s["a"], s["a_scale"], s["b"], s["b_scale"], bias=s["bias"], relu=c["relu"],
                                   out_dtype=TYPES[c["d"]])
        if c["per_row"]:
            idx, logp = ctx.sample(s["scores"], s["u"], params=s["params"], d_seg_off=s["seg_off"])
        else:
            idx, logp = ctx.sample(s["scores"], s["u"], temperature=c["t"], top_k=c["top_k"],
                                   top_p=c["top_p"], min_p=c["min_p"], d_seg_off=s["seg_off"])
        return {"idx": idx, "logp": logp}
    if s["kind"] == "quantize":
        return _quantize(s["data"], c["block_rows"], c["scale"])
    if s["kind"] == "matmul":
        return _matmul(s)
    return _sample(s)


def work(case):
    if case["kind"] == "quantize":
        n, br = case["rows"] * case["cols"], case["block_rows"]
        scales = -(-case["rows"] // br) * -(-case["cols"] // BLOCK)
        return {"bytes": n * (BYTES[case["x"]] + 1) + scales * SCALE_BYTES[case["scale"]], "flops": 2 * n}
    if case["kind"] == "matmul":
        m, n, k, sb = case["m"], case["n"], case["k"], SCALE_BYTES[case["scale"]]
        kb = -(-k // BLOCK)
        read = m * k + n * k + (m + -(-n // BLOCK)) * kb * sb + (4 * n if case["bias"] else 0)
        return {"bytes": read + m * n * BYTES[case["d"]] + (m * -(-n // BLOCK) * sb if case["d"] == "e4m3" else 0),
                "flops": 2 * m * n * k}
    p, c = case["p"], case["c"]
    # a segment's length is spread over its logarithm: (c / log c) on average
    scores = p * c if not case["segments"] else int(p * max(1.0, c / math.log(c + 1)))
    return {"bytes": scores * BYTES[case["x"]] + p * case["draws"] * 12, "flops": 4 * scores}


# ---- the operators from their definitions, in 64 bits -------------------------------------------


def _exact_quantize(x, block_rows, scale):
    """Block by block of columns; scales as numbers, values rounded to the three mantissa bits and the range of e4m3."""
    rows, cols = x.shape
    x = x.double()
    qs, ss = [], []
    for c0 in range(0, cols, BLOCK):
        part = x[:, c0:c0 + BLOCK]
        amax = part.abs().amax(1)
        if block_rows > 1:
            pad = -rows % block_rows
            amax = torch.cat([amax, amax.new_zeros(pad)]).view(-1, block_rows).amax(1)
        if scale == "e8m0":
            half, e = torch.frexp(amax / TOP)  # (a logarithm may miss an exact power of two)
            s = torch.exp2(torch.where(half == 0.5, e - 1, e).clamp(-127, 127).double())
            s = torch.where(amax > 0, s, torch.full_like(s, 2.0 ** -127))
        else:
            s = amax.clamp(min=2.0 ** -100) / TOP
        v = part / s.repeat_interleave(block_rows)[:rows, None]
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        qs.append(torch.round(v / step) * step)
        ss.append(s)
    return torch.cat(qs, 1), torch.stack(ss, 1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "quantize":
        return _exact_quantize(s["data"], case["block_rows"], case["scale"])
    if case["kind"] == "matmul":
        d = torch.zeros(case["m"], case["n"], dtype=torch.float64, device=DEV)
        for i in range(s["a_scale"].shape[1]):
            at = slice(i * BLOCK, (i + 1) * BLOCK)
            part = s["a"][:, at].double() @ s["b"][:, at].double().t()
            part *= s["a_scale"][:, i].double()[:, None]
            part *= s["b_scale"][:, i].double().repeat_interleave(BLOCK)[None, :case["n"]]
            d += part
        if case["bias"]:
            d += s["bias"].double()
        if case["relu"]:
            d.clamp_(min=0)
        return _exact_quantize(d, 1, case["scale"]) if case["d"] == "e4m3" else d
    off = s["seg_off"].tolist() if case["segments"] else None
    x = s["scores"].double()
    rows, draws = case["p"], case["draws"]
    settings = [v.expand(rows).tolist() for v in (s["t"], s["k"], s["tp"], s["mp"])]
    idx = torch.full((rows, draws), -1, dtype=torch.int32, device=DEV)
    logp = torch.full((rows, draws), -math.inf, dtype=torch.float64, device=DEV)
    for i, (t, k, top_p, min_p) in enumerate(zip(*settings)):
        v = x[i] if off is None else x[off[i]:off[i + 1]]
        live = torch.nonzero(v > -math.inf)[:, 0]
        if not live.numel():
            continue
        v = v[live]
        w = torch.softmax(v / t, 0)
        by, at = torch.sort(w, descending=True, stable=True)
        if k > 0:
            by, at = by[:k], at[:k]
        if top_p < 1:
            cum = torch.cumsum(by, 0)
            n = int((cum < top_p * cum[-1]).sum()) + 1
            by, at = by[:n], at[:n]
        at = at[by >= min_p * by[0]]
        at, _ = torch.sort(at)
        cum = torch.cumsum(w[at], 0)
        j = torch.searchsorted(cum, s["u"][i].double() * cum[-1], right=True).clamp(max=len(at) - 1)
        idx[i] = live[at[j]].int()
        logp[i] = torch.log(w[at[j]] / cum[-1])
    return {"idx": idx, "logp": logp}
