"""Workloads of the operators around attention at inference, each in a plain form and as a call of the library.

The operators: norm and rotation of query and key heads in one pass, attention of prompts with a sliding
window and sinks, the key/value cache held in 4 bits (append, read back, attention over it) and the copying
of its pages.  `run` computes them from elementary torch operations, or through the library where `own` is set.

A page of the cache holds `page` tokens of every key/value head: per head the key codes, the value codes, then
(step, eta) pairs of the keys and of the values, all contiguous.  A stored value is eta + step * code, code in
0..15, step = (max - min) / 15 and eta = min over the head's row, both rounded to the cache's type.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


# ---- the cases ---------------------------------------------------------------------------------
def listed():
    return [
        # one new token of one sequence: 32 heads of 128 (d = 4096)
        dict(name="norm_rope one token", op="norm_rope", type="fp16", tokens=1, heads=32, kv_heads=32, dim=128, rot=128,
             inter=False, far=30000),
        # the tokens of a prompt, odd count, grouped key/value heads, positions far out
        dict(name="norm_rope prompt", op="norm_rope", type="bf16", tokens=8191, heads=32, kv_heads=8, dim=128, rot=128,
             inter=False, far=1000000),
        # short prompts of different lengths, packed; the 125M shape (12 heads of 64)
        dict(name="window short prompts", op="window", type="fp16", batch=5, seq=509, ragged=True, heads=12, kv_heads=12,
             dim=64, window=128, sinks=4),
        # a batch of prompts in the shape of the decoder block (16 heads of 128, 4 x 2048)
        dict(name="window prompts", op="window", type="fp16", batch=4, seq=2048, ragged=False, heads=16, kv_heads=16,
             dim=128, window=1024, sinks=4),
        # one long prompt, grouped heads
        dict(name="window long prompt", op="window", type="bf16", batch=1, seq=8192, ragged=False, heads=32, kv_heads=8,
             dim=128, window=4096, sinks=16),
        # one decode step of a batch: a token per sequence, two rows of padding
        dict(name="append decode step", op="append", type="fp16", tokens=18, pad=2, kv_heads=8, dim=128, page=64),
        # a prompt enters the cache
        dict(name="append prompt", op="append", type="bf16", tokens=8190, pad=3, kv_heads=16, dim=128, page=16),
        # one sequence, one token, a short context: the smallest call
        dict(name="cache one sequence", op="cache", type="fp16", batch=1, nq=1, length=1000, heads=16, kv_heads=16, dim=128,
             page=16, window=0, sinks=0),
        # a batch in flight, contexts of different lengths, grouped heads
        dict(name="cache batch", op="cache", type="fp16", batch=32, nq=1, length=8192, heads=32, kv_heads=8, dim=128, page=64,
             window=0, sinks=0),
        # few long sequences, four new tokens each (drafted ones being checked), window and sinks
        dict(name="cache long, drafted tokens", op="cache", type="bf16", batch=2, nq=4, length=150001, heads=32, kv_heads=8,
             dim=128, page=32, window=100000, sinks=64),
        # a sequence is forked: its last page is copied in every layer
        dict(name="pages fork", op="pages", layers=24, pages=64, pairs=1, kv_heads=8, dim=128, page=64),
        # a fragmented cache is compacted
        dict(name="pages compact", op="pages", layers=4, pages=4096, pairs=1500, kv_heads=8, dim=128, page=64),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("norm_rope", "window", "window", "append", "cache", "cache", "pages"))
    t = rng.choice(("fp16", "bf16"))
    dim = rng.choice((64, 128))
    kv = rng.choice((1, 2, 4, 5, 8, 12, 16))
    group = rng.choice((1, 1, 2, 3, 4, 8))
    if kv * group > 32:
        group = 1
    page = rng.choice((16, 32, 64))
    if op == "norm_rope":
        return dict(op=op, type=t, tokens=_log(rng, 1, 8191), heads=kv * group, kv_heads=kv, dim=dim,
                    rot=rng.choice((dim, dim, dim // 2)), inter=rng.random() < 0.5, far=_log(rng, 100, 1000000))
    if op == "window":
        batch = _log(rng, 1, 8)
        seq = _log(rng, 1, min(4096, 8192 // batch))
        return dict(op=op, type=t, batch=batch, seq=seq, ragged=rng.random() < 0.5, heads=kv * group, kv_heads=kv, dim=dim,
                    window=rng.choice((0, _log(rng, 1, 4096))), sinks=rng.choice((0, 1, 4, _log(rng, 1, 200))))
    if op == "append":
        return dict(op=op, type=t, tokens=_log(rng, 2, 8190), pad=rng.choice((0, 0, 1)), kv_heads=kv, dim=dim, page=page)
    if op == "cache":
        batch, nq = _log(rng, 1, 32), rng.choice((1, 1, 1, 2, 3, 5))
        return dict(op=op, type=t, batch=batch, nq=nq, length=_log(rng, 1, 200000 // batch), heads=kv * group, kv_heads=kv,
                    dim=dim, page=page, window=rng.choice((0, 0, _log(rng, 1, 8192))), sinks=rng.choice((0, 4, _log(rng, 1, 100))))
    pages = _log(rng, 8, 4096)
    return dict(op=op, layers=rng.choice((1, 2, 4)), pages=pages, pairs=rng.randint(1, pages // 3), kv_heads=min(kv, 8), dim=dim,
                page=page)


def _lengths(n, top, ragged):
    """Lengths of n sequences: all `top`, or falling from it to about a quarter (odd ones among them)."""
    return [max(1, top - (b * top * 3) // (4 * n) - (b % 3)) if ragged else top for b in range(n)]


# ---- the cache's layout --------------------------------------------------------------------------
def _fields(pages, kv_heads, page, dim):
    """Views of a cache u8 [..., pages, page_bytes]: key codes [.., H, page, dim/2], value codes
    [.., H, page/8, 8, 4, dim/32, 2, 2] (octets of tokens, eighths of the row, pairs of tokens, words, the token
    of the pair, bytes) and the (step, eta) bytes [.., H, page, 4] of each."""
    half = page * dim // 2
    blocks = pages.unflatten(-1, (kv_heads, page * (dim + 8)))
    k = blocks[..., :half].unflatten(-1, (page, dim // 2))
    v = blocks[..., half:2 * half].unflatten(-1, (page // 8, 8, 4, dim // 32, 2, 2))
    ks = blocks[..., 2 * half:2 * half + 4 * page].unflatten(-1, (page, 4))
    vs = blocks[..., 2 * half + 4 * page:].unflatten(-1, (page, 4))
    return k, v, ks, vs


def _nibbles(b):
    return torch.stack((b & 15, b >> 4), -1).flatten(-2)


def _bytes(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _quantise(x):
    """Codes u8 and (step, eta) of rows x [..., dim]; values next to a border of two codes need 64 bits."""
    w = x.double()
    lo, hi = w.amin(-1, keepdim=True), w.amax(-1, keepdim=True)
    step = ((hi - lo) / 15).to(x.dtype)
    s = step.double()
    code = torch.where(s > 0, torch.round((w - lo) / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(w))
    return code.clamp(0, 15).to(torch.uint8), torch.cat((step, lo.to(x.dtype)), -1)


def _store(pages, at, k, v, kv_heads, page, dim):
    """Writes rows k, v [n, H, dim] at the slots `at` [n]."""
    fk, fv, fks, fvs = _fields(pages, kv_heads, page, dim)
    p, j = at // page, at % page
    kc, kse = _quantise(k)
    vc, vse = _quantise(v)
    fk[p, :, j] = _bytes(kc)
    fks[p, :, j] = kse.view(torch.uint8)
    fv[p, :, j // 8, :, (j % 8) // 2, :, j % 2] = _bytes(vc).unflatten(-1, (8, dim // 32, 2))
    fvs[p, :, j] = vse.view(torch.uint8)


def _load(pages, at, kv_heads, page, dim, dtype):
    """The rows at the slots `at` [n], as 32-bit values [n, H, dim]."""
    fk, fv, fks, fvs = _fields(pages, kv_heads, page, dim)
    p, j = at // page, at % page
    kse, vse = fks[p, :, j].view(dtype).float(), fvs[p, :, j].view(dtype).float()
    k = _nibbles(fk[p, :, j]).float() * kse[..., :1] + kse[..., 1:]
    v = _nibbles(fv[p, :, j // 8, :, (j % 8) // 2, :, j % 2].flatten(-3)).float() * vse[..., :1] + vse[..., 1:]
    return k, v


# ---- inputs --------------------------------------------------------------------------------------
def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _page_bytes(c):
    return c["kv_heads"] * c["page"] * (c["dim"] + 8)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 17)
    s = dict(c)
    if c["op"] == "pages":
        s["pages"] = torch.randint(0, 256, (c["layers"], c["pages"], _page_bytes(c)), generator=g, device=DEV, dtype=torch.uint8)
        perm = torch.randperm(c["pages"], generator=g, device=DEV)[:2 * c["pairs"]]
        s["pairs"] = perm.view(2, -1).t().contiguous().int()        # (source, destination)
        return s
    dt = TYPES[c["type"]]
    dim, hk = c["dim"], c["kv_heads"]
    # keys have a few channels that stand out, as keys do
    loud = torch.ones(dim, device=DEV)
    loud[torch.randperm(dim, generator=g, device=DEV)[:3]] = 4.0
    if c["op"] == "norm_rope":
        T, h = c["tokens"], c["heads"]
        s["qkv"] = _randn(g, T, (h + 2 * hk) * dim, dtype=dt)        # as one fused projection leaves them
        s["wq"] = (1 + 0.2 * _randn(g, dim)).to(dt)
        s["wk"] = (loud + 0.2 * _randn(g, dim)).to(dt)
        first = torch.randint(0, c["far"], (1,), generator=g, device=DEV)
        s["positions"] = (first + torch.arange(T, device=DEV)).int()
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, c["rot"], 2, device=DEV, dtype=torch.float64) / c["rot"])).float()
    elif c["op"] == "window":
        lens = _lengths(c["batch"], c["seq"], c["ragged"])
        T, h = sum(lens), c["heads"]
        s["qkv"] = torch.cat((_randn(g, T, h * dim, dtype=dt), (_randn(g, T, hk, dim) * loud / 2).to(dt).flatten(1),
                              _randn(g, T, hk * dim, dtype=dt)), 1)
        at = [0]
        for n in lens:
            at.append(at[-1] + n)
        s["cu"] = torch.tensor(at, device=DEV, dtype=torch.int32)
        s["top"] = max(lens)
    elif c["op"] == "append":
        T, page = c["tokens"], c["page"]
        n = T // page + 4
        s["k"] = (_randn(g, T, hk, dim) * loud).to(dt).flatten(1)
        s["v"] = _randn(g, T, hk * dim, dtype=dt)
        s["pages"] = torch.zeros((n, _page_bytes(c)), device=DEV, dtype=torch.uint8)
        slots = torch.randperm(n * page, generator=g, device=DEV)[:T].sort().values
        s["rows"] = torch.arange(T - c["pad"], device=DEV)           # the tokens that are no padding
        slots[T - c["pad"]:] = -1
        s["slots"] = slots
        s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
        s["type_"] = dt
    else:
        page, b = c["page"], c["batch"]
        lens = _lengths(b, c["length"], True)
        per = -(-max(lens) // page)
        n = b * per + 3
        s["pages"] = torch.zeros((n, _page_bytes(c)), device=DEV, dtype=torch.uint8)
        s["table"] = torch.randperm(n, generator=g, device=DEV)[:b * per].view(b, per).int()
        every = torch.arange(n * page, device=DEV)
        for i in range(0, n * page, 65536):
            at = every[i:i + 65536]
            _store(s["pages"], at, (_randn(g, at.numel(), hk, dim) * loud / 2).to(dt), _randn(g, at.numel(), hk, dim, dtype=dt),
                   hk, page, dim)
        s["lens"] = torch.tensor(lens, device=DEV, dtype=torch.int32)
        s["q"] = _randn(g, b * c["nq"], c["heads"] * dim, dtype=dt)
        s["top"] = max(lens)
        s["type_"] = dt
    return s


# ---- plain forms ---------------------------------------------------------------------------------
def _norm_rope(s, x, w):
    T, dim, rot = x.shape[0], s["dim"], s["rot"]
    x = x.reshape(T, -1, dim).float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w.float()
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()   # far positions: 64 bits
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if s["inter"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, x[..., rot:]), -1).reshape(T, -1)


def _visible(i, j, window, sinks):
    """Whether position i sees position j."""
    seen = (j <= i) & (i >= 0)
    return seen & ((i - j < window) | (j < sinks)) if window > 0 else seen


def _softmax(x, seen):
    """Rows of probabilities over the last axis; a row that sees nothing is zero."""
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, torch.ones_like(total))


def _plain_window(s):
    dim, h, hk, cu, top = s["dim"], s["heads"], s["kv_heads"], s["cu"].long(), s["top"]
    qkv = s["qkv"]
    T, b = qkv.shape[0], cu.numel() - 1
    i = torch.arange(top, device=DEV)
    rows = (cu[:-1, None] + i).clamp(max=T - 1)                       # padded [batch, top]
    x = qkv[rows].float()
    q = x[..., :h * dim].reshape(b, top, hk, h // hk, dim).permute(0, 2, 3, 1, 4).reshape(b, hk, -1, dim)
    k = x[..., h * dim:(h + hk) * dim].reshape(b, top, hk, dim).permute(0, 2, 3, 1)
    v = x[..., (h + hk) * dim:].reshape(b, top, hk, dim).transpose(1, 2)
    seen = _visible(i[:, None], i, s["window"], s["sinks"]) & (i < (cu[1:] - cu[:-1])[:, None])[:, None]
    p = (q @ k).mul_(1 / math.sqrt(dim)).view(b, hk, h // hk, top, top)
    p = _softmax(p, seen[:, None, None]).view(b, hk, -1, top)
    o = (p @ v).view(b, hk, h // hk, top, dim).permute(0, 3, 1, 2, 4).reshape(b, top, h * dim).to(qkv.dtype)
    r = torch.arange(T, device=DEV)
    at = torch.searchsorted(cu, r, right=True) - 1
    return o[at, r - cu[at]]


def _plain_append(s):
    dim, hk, page = s["dim"], s["kv_heads"], s["page"]
    rows = s["rows"]
    at = s["slots"][rows]
    k, v = s["k"].unflatten(-1, (hk, dim))[rows], s["v"].unflatten(-1, (hk, dim))[rows]
    _store(s["pages"], at, k, v, hk, page, dim)
    ko, vo = _load(s["pages"], at, hk, page, dim, s["type_"])
    s["k_out"][rows] = ko.flatten(1).to(s["type_"])
    s["v_out"][rows] = vo.flatten(1).to(s["type_"])
    return s["k_out"], s["v_out"]


def _plain_cache(s):
    dim, h, hk, page, b, nq, top = s["dim"], s["heads"], s["kv_heads"], s["page"], s["batch"], s["nq"], s["top"]
    j = torch.arange(top, device=DEV)
    at = s["table"].long()[:, j // page] * page + j % page
    k, v = _load(s["pages"], at.view(-1), hk, page, dim, s["type_"])
    k, v = k.view(b, top, hk, dim).permute(0, 2, 3, 1), v.view(b, top, hk, dim).transpose(1, 2)
    q = s["q"].float().view(b, nq, hk, h // hk, dim).transpose(1, 2).reshape(b, hk, -1, dim)
    lens = s["lens"].long()
    i = lens[:, None] - nq + torch.arange(nq, device=DEV)
    seen = _visible(i[:, :, None], j, s["window"], s["sinks"])
    p = (q @ k).mul_(1 / math.sqrt(dim)).view(b, hk, nq, h // hk, top)
    p = _softmax(p, seen[:, None, :, None]).view(b, hk, -1, top)
    o = (p @ v).view(b, hk, nq, h // hk, dim).transpose(1, 2)
    return o.reshape(b * nq, h * dim).to(s["type_"])


def run(state):
    s = state
    op = s["op"]
    if own:
        from paper_2310_11453_b200 import binding as B
        if op == "norm_rope":
            n, m = s["heads"] * s["dim"], s["kv_heads"] * s["dim"]
            return B.qk_norm_rope(s["qkv"][:, :n], s["qkv"][:, n:n + m], s["positions"], s["inv_freq"], s["heads"], s["kv_heads"],
                                  s["dim"], wq=s["wq"], wk=s["wk"], eps=1e-6, interleaved=s["inter"])
        if op == "window":
            n, m = s["heads"] * s["dim"], s["kv_heads"] * s["dim"]
            x = s["qkv"]
            return B.attention_window(x[:, :n], x[:, n:n + m], x[:, n + m:], s["batch"], s["top"], s["heads"], s["kv_heads"], s["dim"],
                                      window=s["window"], sinks=s["sinks"], cu_q=s["cu"])
        if op == "pages":
            return B.kv4_copy_pages(s["pages"], s["pairs"])
        cache = B.Kv4Cache(s["pages"], s["page"], s["kv_heads"], s["dim"], s["type_"])
        if op == "append":
            B.kv4_append(cache, s["k"], s["v"], s["slots"])
            return B.kv4_read(cache, s["slots"], k=s["k_out"], v=s["v_out"])
        return B.attention_kv4(s["q"], cache, s["table"], s["lens"], s["batch"], s["nq"], s["heads"], window=s["window"],
                               sinks=s["sinks"])
    if op == "norm_rope":
        n, m = s["heads"] * s["dim"], s["kv_heads"] * s["dim"]
        x = s["qkv"]
        return _norm_rope(s, x[:, :n], s["wq"]).to(x.dtype), _norm_rope(s, x[:, n:n + m], s["wk"]).to(x.dtype)
    if op == "window":
        return _plain_window(s)
    if op == "append":
        return _plain_append(s)
    if op == "cache":
        return _plain_cache(s)
    s["pages"][:, s["pairs"][:, 1].long()] = s["pages"][:, s["pairs"][:, 0].long()]
    return s["pages"]


# ---- what a pass cannot do without ---------------------------------------------------------------
def _seen_by_any(n, nq, window, sinks):
    """Cached tokens that one of the last nq positions of n sees."""
    if window <= 0:
        return n
    lo = max(0, max(0, n - nq) - window + 1)
    return n - lo + min(sinks, lo)


def _pairs_seen(n, window, sinks):
    """Pairs (i, j) of a prompt of n tokens with j visible from i."""
    total = 0
    for i in range(n):
        lo = max(0, i - window + 1) if window > 0 else 0
        total += i + 1 - lo + min(sinks, lo)
    return total


def work(case):
    c = case
    if c["op"] == "pages":
        return {"bytes": 2 * c["layers"] * c["pairs"] * _page_bytes(c) + 8 * c["pairs"], "flops": 0}
    dim, hk = c["dim"], c["kv_heads"]
    if c["op"] == "norm_rope":
        n = c["tokens"] * (c["heads"] + hk) * dim
        return {"bytes": 4 * n + 4 * c["tokens"] + 4 * dim + 2 * c["rot"], "flops": 8 * n}
    if c["op"] == "append":
        n = (c["tokens"] - c["pad"]) * hk
        return {"bytes": 2 * n * (4 * dim + dim + 8) + 8 * c["tokens"], "flops": 8 * n * dim}
    if c["op"] == "window":
        lens = _lengths(c["batch"], c["seq"], c["ragged"])
        pairs = sum(_pairs_seen(n, c["window"], c["sinks"]) for n in lens)
        return {"bytes": sum(lens) * 4 * (c["heads"] + hk) * dim, "flops": 4 * dim * c["heads"] * pairs}
    lens = _lengths(c["batch"], c["length"], True)
    tokens = sum(_seen_by_any(n, c["nq"], c["window"], c["sinks"]) for n in lens)
    return {"bytes": tokens * hk * (dim + 8) + 4 * c["batch"] * c["nq"] * c["heads"] * dim + 4 * (tokens // c["page"] + c["batch"]),
            "flops": 4 * dim * c["heads"] * c["nq"] * tokens}


# ---- the definitions in 64 bits --------------------------------------------------------------------
def _exact_turn(x, w, pos, freq, inter):
    x = x.double()
    x = x / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt() * w.double()
    r = freq.numel()
    unit = torch.polar(torch.ones_like(freq), freq * pos[:, None])[:, None]           # e^(i angle), [T, 1, r]
    first = torch.arange(r, device=x.device) * (2 if inter else 1)
    second = first + (1 if inter else r)
    z = torch.complex(x[..., first], x[..., second]) * unit
    x[..., first], x[..., second] = z.real, z.imag
    return x


def _exact_rows(q, k, v, seen, dim):
    """softmax(q k^T / sqrt(dim)) v over the places that are seen, 64 bits."""
    z = (q @ k.t() / math.sqrt(dim)).masked_fill(~seen, -math.inf)
    none = ~seen.any(-1, keepdim=True)
    return torch.softmax(z.masked_fill(none, 0.0), -1).masked_fill(none, 0.0) @ v


def _exact_seen(i, n, window, sinks):
    j = torch.arange(n, device=i.device)[None]
    i = i[:, None]
    near = (i - j < window) if window > 0 else torch.ones_like(i - j, dtype=torch.bool)
    return (j <= i) & (near | (j < sinks))


def _exact_value(x):
    """What 4 bits, a step and an eta keep of the rows x [..., dim]."""
    w = x.double()
    eta = w.min(-1, keepdim=True).values
    step = ((w.max(-1, keepdim=True).values - eta) / 15).to(x.dtype).double()
    codes = torch.nan_to_num((w - eta) / step, nan=0.0, posinf=0.0).round().clamp(0, 15)
    return eta + step * codes


def _exact_cached(s, b, n):
    """Keys and values [n, H, dim] of sequence b, decoded byte by byte."""
    dim, hk, page = s["dim"], s["kv_heads"], s["page"]
    block = page * (dim + 8)
    t = torch.arange(n, device=DEV)[:, None, None]
    h = torch.arange(hk, device=DEV)[None, :, None]
    d = torch.arange(dim, device=DEV)[None, None, :]
    pid = s["table"][b].long()[t // page]
    j = t % page
    base = (pid * hk + h) * block
    flat = s["pages"].view(-1)
    kc = (flat[base + j * (dim // 2) + d // 2].long() >> (4 * (d % 2))) & 15
    e = d % (dim // 8)
    off = (j // 8) * 4 * dim + ((d // (dim // 8)) * 4 + (j % 8) // 2) * (dim // 8) + (e // 4) * 4 + (j % 2) * 2 + (e % 4) // 2
    vc = (flat[base + page * dim // 2 + off].long() >> (4 * (e % 2))) & 15

    def number(at):
        return torch.stack((flat[at], flat[at + 1]), -1).view(s["type_"]).squeeze(-1).double()

    ks, vs = base + page * dim + 4 * j, base + page * dim + 4 * page + 4 * j
    return number(ks + 2) + number(ks) * kc, number(vs + 2) + number(vs) * vc


def exact(case, seed):
    if case["op"] == "pages":
        return None                                                # bytes are moved, nothing is computed
    s = prepare(case, seed)
    op = s["op"]
    dim, hk = s["dim"], s["kv_heads"]
    if op == "append":
        out = []
        for x in (s["k"], s["v"]):
            y = _exact_value(x.view(x.shape[0], hk, dim)).reshape(x.shape)
            out.append(torch.where(s["slots"][:, None] >= 0, y, torch.zeros_like(y)))
        return tuple(out)
    if op == "norm_rope":
        T, n = s["tokens"], s["heads"] * dim
        pos, freq = s["positions"].double(), s["inv_freq"].double()
        q = _exact_turn(s["qkv"][:, :n].reshape(T, -1, dim), s["wq"], pos, freq, s["inter"])
        k = _exact_turn(s["qkv"][:, n:n + hk * dim].reshape(T, -1, dim), s["wk"], pos, freq, s["inter"])
        return q.reshape(T, -1), k.reshape(T, -1)
    g = s["heads"] // hk
    if op == "window":
        x, cu = s["qkv"], s["cu"].tolist()
        o = torch.zeros((x.shape[0], s["heads"], dim), device=DEV, dtype=torch.float64)
        for a, b in zip(cu, cu[1:]):
            seen = _exact_seen(torch.arange(b - a, device=DEV), b - a, s["window"], s["sinks"])
            for h in range(s["heads"]):
                kh = s["heads"] + h // g
                q, k, v = (x[a:b, n * dim:(n + 1) * dim].double() for n in (h, kh, kh + hk))
                o[a:b, h] = _exact_rows(q, k, v, seen, dim)
        return o.flatten(1)
    o = torch.zeros((s["batch"], s["nq"], s["heads"], dim), device=DEV, dtype=torch.float64)
    for b, n in enumerate(s["lens"].tolist()):
        k, v = _exact_cached(s, b, n)
        seen = _exact_seen(torch.arange(n - s["nq"], n, device=DEV), n, s["window"], s["sinks"])
        for h in range(s["heads"]):
            q = s["q"].view(s["batch"], s["nq"], s["heads"], dim)[b, :, h].double()
            o[b, :, h] = _exact_rows(q, k[:, h // g], v[:, h // g], seen, dim)
    return o.view(s["batch"] * s["nq"], -1)
