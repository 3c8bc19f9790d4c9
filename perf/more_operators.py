"""Workloads of the 8-bit layers and of the experts made of them, each in a plain form and as a call of the library.

The operators: the root-mean-square norm with the residual's addition (and the weighted sum of the experts' rows) whose
output are 8-bit codes with a scale per token; the matrix product of such codes with 8-bit weights that have a scale per
channel; the choice of the experts of each token, with the lists of rows that it makes; and the matrix products of the rows
of each expert with that expert's weights.  `run` computes them from elementary torch operations, or through the library
where `own` is set.

A code c of a row with scale s stands for s * c, c in -127..127 and s = max |row| / 127.
"""
import math

import torch

own = False

DEV = "cuda"
SHORT = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.bfloat16}   # what the values of 8-bit codes are returned in
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6


# ---- the cases ---------------------------------------------------------------------------------
def listed():
    return [
        # one new token between two layers (d = 4096)
        dict(name="norm one token", op="norm", type="fp16", tokens=1, width=4096, join=0),
        # the tokens of a prompt, odd count
        dict(name="norm prompt", op="norm", type="bf16", tokens=8191, width=4096, join=0),
        # behind a layer of experts: four rows a token are weighed, summed and added to the residual (d = 2048)
        dict(name="norm behind experts", op="norm", type="bf16", tokens=3001, width=2048, join=4),
        # one new token through a wide layer
        dict(name="matmul one token", op="matmul", type="fp16", rows=1, inner=4096, outer=16384, bias=False, relu=False, add=False),
        # the output layer for a few sequences: 32-bit scores, an odd count of them
        dict(name="matmul scores", op="matmul", type="fp32", rows=37, inner=2048, outer=32001, bias=True, relu=False, add=False),
        # a short prompt through the first layer of a feed-forward block
        dict(name="matmul short prompt", op="matmul", type="fp16", rows=509, inner=2048, outer=8192, bias=True, relu=True, add=False),
        # the tokens of a batch of prompts, with the residual
        dict(name="matmul prompts", op="matmul", type="bf16", rows=8192, inner=4096, outer=4096, bias=False, relu=False, add=True),
        # the experts of one decode step
        dict(name="route decode step", op="route", type="fp32", tokens=18, experts=64, top=8, whole=False),
        # the experts of a prompt
        dict(name="route prompt", op="route", type="bf16", tokens=8191, experts=128, top=8, whole=True),
        # the first products of the experts of one decode step: few rows each, some experts without any
        dict(name="grouped decode step", op="grouped", type="i8", out="bf16", tokens=18, top=8, experts=64, inner=2048, outer=2048,
             skew=True, relu=True),
        # the same of a batch of prompts, unevenly spread
        dict(name="grouped prompts", op="grouped", type="i8", out="bf16", tokens=4096, top=2, experts=16, inner=2048, outer=8192,
             skew=True, relu=True),
        # experts that were not quantised, a short prompt, odd sizes
        dict(name="grouped short prompt", op="grouped", type="bf16", out="bf16", tokens=301, top=4, experts=11, inner=1040, outer=2050,
             skew=False, relu=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm", "matmul", "matmul", "route", "grouped", "grouped"))
    t = rng.choice(("fp16", "bf16", "bf16", "fp32"))
    if op == "norm":
        join = rng.choice((0, 0, 1, 2, 4, 8))
        width = 8 * _log(rng, 16, 2048)
        return dict(op=op, type=t, tokens=_log(rng, 1, min(8191, 30_000_000 // (width * (1 + join)))), width=width, join=join)
    if op == "matmul":
        inner, outer = 16 * _log(rng, 8, 512), _log(rng, 64, 32001)
        return dict(op=op, type=t, rows=_log(rng, 1, min(8192, 100_000_000_000 // (inner * outer))), inner=inner, outer=outer,
                    bias=rng.random() < 0.5, relu=rng.random() < 0.3, add=rng.random() < 0.3)
    if op == "route":
        experts = _log(rng, 2, 256)
        return dict(op=op, type=t, tokens=_log(rng, 1, 8191), experts=experts, top=rng.randint(1, min(8, experts)),
                    whole=rng.random() < 0.5)
    kind = rng.choice(("i8", "i8", "bf16", "fp16"))
    experts, inner, outer = _log(rng, 1, 64), 16 * _log(rng, 8, 256), _log(rng, 64, 8192)
    experts = max(1, min(experts, 130_000_000 // (inner * outer)))
    top = rng.randint(1, min(8, experts))
    rows = _log(rng, 1, min(8192, 50_000_000_000 // (inner * outer)))
    return dict(op=op, type=kind, out=rng.choice(("fp16", "bf16", "fp32")) if kind == "i8" else kind, tokens=max(1, rows // top), top=top,
                experts=experts, inner=inner, outer=outer, skew=rng.random() < 0.5, relu=rng.random() < 0.3)


def _offsets(c):
    """First rows of the experts: evenly spread, or some with ten times the rows of others and some with none where rows are few."""
    n, rows = c["experts"], c["tokens"] * c["top"]
    share = [math.exp(-2.5 * ((7 * e + 3) % n) / n) if c["skew"] else 1.0 for e in range(n)]
    total, at, seen = sum(share), [0], 0.0
    for x in share:
        seen += x
        at.append(int(round(rows * seen / total)))
    at[-1] = rows
    return at


# ---- inputs --------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)


def _codes(x):
    """8-bit codes and scales of the rows of x."""
    scale = x.abs().amax(-1) / 127
    return torch.round(x / scale[..., None]).clamp(-127, 127).to(torch.int8), scale


def _loud(g, rows, width):
    """Activations: normal values, with a few channels that stand out."""
    x = _randn(g, rows, width)
    x[:, torch.randperm(width, generator=g, device=DEV)[:max(1, width // 512)]] *= 8
    return x


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 29)
    c, s = case, dict(case)
    if c["op"] == "norm":
        t, T, n = TYPES[c["type"]], c["tokens"], c["width"]
        s["residual"] = (4 * _loud(g, T, n)).to(t)
        s["weight"] = (1 + 0.2 * _randn(g, n)).to(t)
        s["value"] = torch.empty((T, n), device=DEV, dtype=SHORT[c["type"]])
        if c["join"]:
            s["x"] = _randn(g, T * c["join"], n).to(t)
            s["places"] = torch.randperm(T * c["join"], generator=g, device=DEV).view(T, c["join"]).int()
            s["shares"] = torch.softmax(_randn(g, T, c["join"]), -1)
        else:
            s["x"] = _randn(g, T, n).to(t)
    elif c["op"] == "matmul":
        s["x"], s["x_scale"] = _codes(_loud(g, c["rows"], c["inner"]))
        s["w"], s["w_scale"] = _codes(0.02 * _randn(g, c["outer"], c["inner"]))
        s["b"] = _randn(g, c["outer"]).to(TYPES[c["type"]]) if c["bias"] else None
        s["residual"] = (4 * _randn(g, c["rows"], c["outer"])).to(TYPES[c["type"]]) if c["add"] else None
    elif c["op"] == "route":
        s["logits"] = (2 * _randn(g, c["tokens"], c["experts"])).to(TYPES[c["type"]])
    else:
        T, E, n, k = c["tokens"], c["experts"], c["outer"], c["inner"]
        x = _loud(g, T, k)
        w = _randn(g, E * n, k)
        if c["type"] == "i8":
            s["x"], s["x_scale"] = _codes(x)
            s["w"], s["w_scale"] = _codes(w.mul_(0.02))
            s["w_scale"] = s["w_scale"].view(E, n)
        else:
            s["x"], s["w"] = x.to(TYPES[c["type"]]), w.mul_(0.02).to(TYPES[c["type"]])
            s["x_scale"] = s["w_scale"] = None
        s["w"] = s["w"].view(E, n, k)
        at = _offsets(c)
        s["offsets"] = torch.tensor(at, device=DEV, dtype=torch.int32)
        s["most"] = max(b - a for a, b in zip(at, at[1:]))
        order = torch.randperm(T * c["top"], generator=g, device=DEV)
        s["rows"] = (order // c["top"]).int()
    return s


# ---- plain forms ---------------------------------------------------------------------------------
def _plain_norm(s):
    x = s["x"].float()
    if s["join"]:
        x = (x[s["places"].long()] * s["shares"][..., None]).sum(1)
    h = x + s["residual"].float()
    y = (h * torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS) * s["weight"].float()).double()   # 64 bits: values next to a border of two codes
    scale = y.abs().amax(-1, keepdim=True) / 127
    codes = torch.round(y / scale).clamp(-127, 127)
    return h.to(s["x"].dtype), (codes * scale).float().to(SHORT[s["type"]])


def _plain_matmul(s):
    y = (s["x"].float() @ s["w"].float().t()) * s["x_scale"][:, None] * s["w_scale"]
    if s["bias"]:
        y = y + s["b"].float()
    if s["relu"]:
        y = y.clamp(min=0)
    if s["add"]:
        y = y + s["residual"].float()
    return y.to(TYPES[s["type"]])


def _plain_route(s):
    z, k, E = s["logits"].float(), s["top"], s["experts"]
    top, experts = torch.sort(z, dim=-1, descending=True, stable=True)          # of equals the lowest index first
    top, experts = top[:, :k], experts[:, :k]
    p = torch.exp(top - top[:, :1])
    weights = p / (torch.exp(z - top[:, :1]) if s["whole"] else p).sum(-1, keepdim=True)
    by, order = torch.sort(experts.reshape(-1), stable=True)
    offsets = torch.searchsorted(by, torch.arange(E + 1, device=DEV))
    places = torch.empty_like(order)
    places[order] = torch.arange(order.numel(), device=DEV)
    return experts.int(), weights, offsets.int(), (order // k).int(), places.view(-1, k).int()


def _plain_grouped(s):
    at, n = s["offsets"].long(), s["rows"].numel()
    i = torch.arange(s["most"], device=DEV)
    source = s["rows"].long()[(at[:-1, None] + i).clamp(max=n - 1)]           # [experts, most], each list padded
    y = torch.bmm(s["x"][source].float(), s["w"].float().transpose(1, 2))
    if s["x_scale"] is not None:
        y = y * s["x_scale"][source][..., None] * s["w_scale"][:, None]
    if s["relu"]:
        y = y.clamp(min=0)
    r = torch.arange(n, device=DEV)
    e = torch.searchsorted(at, r, right=True) - 1
    return y[e, r - at[e]].to(TYPES[s["out"]])


def run(state):
    s = state
    op = s["op"]
    if own:
        from paper_2310_11453_b200 import binding as B
        if op == "norm":
            codes, scale, h, _ = B.rms_norm_quant(s["x"], s["weight"], EPS, residual=s["residual"], rows=s["places"] if s["join"] else None,
                                                  row_weights=s["shares"] if s["join"] else None, h=True)
            return h, torch.mul(codes, scale[:, None], out=s["value"])
        if op == "matmul":
            return B.matmul_i8(s["x"], s["x_scale"], s["w"], s["w_scale"], out_dtype=TYPES[s["type"]], bias=s["b"], relu=s["relu"],
                               residual=s["residual"])
        if op == "route":
            return B.route_topk(s["logits"], s["top"], normalise=not s["whole"])
        return B.matmul_grouped(s["x"], s["w"], s["offsets"], rows=s["rows"], x_scale=s["x_scale"], w_scale=s["w_scale"], relu=s["relu"],
                                out_dtype=TYPES[s["out"]])
    return {"norm": _plain_norm, "matmul": _plain_matmul, "route": _plain_route, "grouped": _plain_grouped}[op](s)


# ---- what a pass cannot do without ---------------------------------------------------------------
def _size(t):
    return {"i8": 1, "fp16": 2, "bf16": 2, "fp32": 4}[t]


def work(case):
    c = case
    if c["op"] == "norm":
        T, n, z, j = c["tokens"], c["width"], _size(c["type"]), c["join"]
        return {"bytes": T * n * ((j or 1) * z + 2 * z + 1) + n * z + T * (4 + 8 * j), "flops": T * n * (2 * j + 8)}
    if c["op"] == "matmul":
        m, k, n, z = c["rows"], c["inner"], c["outer"], _size(c["type"])
        return {"bytes": m * k + n * k + 4 * m + 4 * n + z * (m * n * (2 if c["add"] else 1) + (n if c["bias"] else 0)),
                "flops": 2 * m * n * k}
    if c["op"] == "route":
        T, E, k = c["tokens"], c["experts"], c["top"]
        return {"bytes": T * E * _size(c["type"]) + 16 * T * k + 4 * (E + 1), "flops": T * E * (k + 2)}
    at, z = _offsets(c), _size(c["type"])
    k, n, R = c["inner"], c["outer"], at[-1]
    met = sum(b > a for a, b in zip(at, at[1:]))
    scales = 4 * (c["tokens"] + met * n) if c["type"] == "i8" else 0
    return {"bytes": z * (c["tokens"] * k + met * n * k) + scales + 4 * (R + c["experts"] + 1) + R * n * _size(c["out"]),
            "flops": 2 * R * n * k}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_norm(s):
    h = s["residual"].double()
    if s["join"]:
        for j in range(s["join"]):
            h = h + s["x"].double().index_select(0, s["places"][:, j].long()) * s["shares"][:, j].double().unsqueeze(1)
    else:
        h = h + s["x"].double()
    y = h / (h.pow(2).sum(1, keepdim=True) / h.shape[1] + EPS).sqrt() * s["weight"].double()
    step = y.abs().max(1, keepdim=True).values / 127
    return h, (y / step).round() * step


def _exact_product(x, w, relu, xs=None, ws=None, bias=None, add=None):
    y = torch.mm(x.double(), w.double().t())                    # whole numbers up to 2^31: exact
    if xs is not None:
        y *= torch.outer(xs.double(), ws.double())
    if bias is not None:
        y += bias.double()
    if relu:
        y = torch.where(y > 0, y, torch.zeros_like(y))
    return y if add is None else y.add_(add.double())


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "norm":
        return _exact_norm(s)
    if s["op"] == "matmul":
        return _exact_product(s["x"], s["w"], s["relu"], s["x_scale"], s["w_scale"], s["b"], s["residual"])
    if s["op"] == "route":
        z = s["logits"].double()
        left, picked = z.clone(), []
        for _ in range(s["top"]):
            m = left.max(1, keepdim=True).values
            first = (left == m).double().argmax(1)
            picked.append(first)
            left.scatter_(1, first.unsqueeze(1), -math.inf)
        experts = torch.stack(picked, 1)
        weights = (torch.softmax(z, 1) if s["whole"] else torch.softmax(z.gather(1, experts), 1)).double()
        if s["whole"]:
            weights = weights.gather(1, experts)
        hits = (experts.view(-1, 1) == torch.arange(s["experts"], device=DEV)).long()
        count = hits.sum(0)
        offsets = torch.cat((count.new_zeros(1), count.cumsum(0)))
        places = offsets[experts.view(-1)] + (hits.cumsum(0) - hits).gather(1, experts.view(-1, 1)).view(-1)
        rows = torch.zeros_like(places).scatter_(0, places, torch.arange(places.numel(), device=DEV) // s["top"])
        return experts.int(), weights, offsets.int(), rows.int(), places.view(-1, s["top"]).int()
    at = s["offsets"].tolist()
    out = torch.zeros((at[-1], s["outer"]), device=DEV, dtype=torch.float64)
    for e, (a, b) in enumerate(zip(at, at[1:])):
        if b > a:
            r = s["rows"][a:b].long()
            scaled = s["x_scale"] is not None
            out[a:b] = _exact_product(s["x"][r], s["w"][e], s["relu"], s["x_scale"][r] if scaled else None, s["w_scale"][e] if scaled else None)
    return out
