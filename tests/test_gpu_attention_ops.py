"""The attention operators on the GPU against their definitions in 64 bits.

Tolerances.  u(T) = eps(T) / 2 is one rounding to T; e = 2^-24 one of fp32.  Outputs are rounded once: u |o|.
Attention: probabilities (for the cache: probability times step) are rounded to 16 bits for the product with the
values, which moves o by at most u(P) sum_j p_j |v_j| (P: the type of v, fp16 for the cache), and a score that is off
by d moves its probability by a factor e^d, its row's sum too: (2 d) sum_j p_j |v_j|.  A score is a sum of D products
in fp32: d <= 4 D e scale max |q| . |k| (the 4 covers the order of the tensor core's sums, the scaling and the exponent's
argument).  The sums over j in fp32 add at most n e, far below, which is counted as 64 e per thousand keys."""
import math

import pytest
import torch

from paper_2310_11453_b200 import binding as B
from tests import attention_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def randn(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def check(got, want, tol, what=""):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, worst {float(((got - want).abs() / tol.clamp(min=1e-300)).max()):.3g} x the tolerance"


# ---- norm and rotation ---------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("T,heads,kv,dim,rot,inter", [
    (1, 32, 32, 128, 128, False), (1, 1, 1, 16, 16, True), (5, 12, 4, 64, 64, False), (7, 5, 3, 80, 32, False), (3, 3, 1, 256, 256, True),
    (130, 40, 8, 128, 64, True), (700, 9, 9, 64, 64, True), (33, 2, 2, 96, 96, False), (2, 4, 2, 128, 0, False), (601, 33, 11, 128, 128, False)])
def test_norm_rope(dt, T, heads, kv, dim, rot, inter):
    qkv = randn(T + dim, T, (heads + 2 * kv) * dim + 16, dtype=dt, scale=2.0)
    q, k = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv) * dim]
    wq, wk = (1 + randn(3, dim, scale=0.3)).to(dt), (1 + randn(4, dim, scale=0.3)).to(dt)
    pos = torch.randint(0, 1 << 20, (T,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(T)).int()
    pos[0] = 2 ** 31 - 1
    freq = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))).float()
    for eps, w in ((1e-5, (wq, wk)), (1e-6, (None, None)), (-1.0, (None, None))):
        outs = B.qk_norm_rope(q, k, pos, freq, heads, kv, dim, wq=w[0], wk=w[1], eps=eps, interleaved=inter)
        for got, x, g in zip(outs, (q, k), w):
            want, size, turns = R.norm_rope(x, g, pos, freq, dim, eps, inter)
            # norm: a sum of dim squares and a handful of roundings; angle: a fraction of a turn in fp32, its fp64 product
            tol = (dim + 32) * E * size + 2 * math.pi * (2.0 ** -25 + turns * 2.0 ** -51) * size + R.half_step(dt) * want.abs() + 1e-7 * (dt != F32) + 1e-30
            check(got, want, tol, f"eps {eps}")


def test_norm_rope_padding_in_place_and_other_streams():
    T, heads, kv, dim = 37, 6, 2, 128
    pos = torch.arange(T, device=DEV).int() * 1000
    pos[[3, 36]] = -1
    freq = (10000.0 ** (-torch.arange(0, dim, 2, device=DEV).double() / dim)).float()
    qkv = randn(1, T, (heads + 2 * kv) * dim, dtype=F16)
    q, k = qkv[:, :heads * dim], qkv[:, heads * dim:(heads + kv) * dim]
    want = B.qk_norm_rope(q, k, pos.clamp(min=0), freq, heads, kv, dim)
    before = qkv.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.qk_norm_rope(q, k, pos, freq, heads, kv, dim, q_out=q, k_out=k)
    torch.cuda.current_stream().wait_stream(s)
    keep = pos >= 0
    for g, w, b in zip(got, want, (before[:, :heads * dim], before[:, heads * dim:(heads + kv) * dim])):
        assert torch.equal(g[keep], w[keep]) and torch.equal(g[~keep], b[~keep])
    assert torch.equal(qkv[:, (heads + kv) * dim:], before[:, (heads + kv) * dim:])
    e = torch.empty((0, heads * dim), device=DEV, dtype=F16)
    B.qk_norm_rope(e, torch.empty((0, kv * dim), device=DEV, dtype=F16), pos[:0], freq, heads, kv, dim)


# ---- the cache -----------------------------------------------------------------------------------
def rows_for(kind, T, heads, dim, dt, seed):
    x = randn(seed, T, heads, dim)
    if kind == "ties":                           # steps and values on a coarse grid: quotients fall on borders exactly
        x = torch.randint(-20, 21, (T, heads, dim), device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).float() / 8
        x[..., 0], x[..., 1] = -2.5, 5.0         # range 7.5: a step of 0.5
        x = x.clamp(-2.5, 5.0)
    elif kind == "constant":
        x = x[..., :1].expand(T, heads, dim).clone()
    elif kind == "wide":                         # from the smallest numbers of the type to the largest
        x = x * torch.exp2(torch.randint(-24, 15, (T, heads, 1), device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).float())
        x = x.clamp(-60000, 60000)
        x[0, 0] = torch.linspace(-60000, 60000, dim, device=DEV)
        x[-1, -1] = torch.arange(dim, device=DEV) % 3 * 2.0 ** -24
    elif kind == "nonfinite":
        x[::2, 0, 5], x[1::3, -1, 7], x[2::5, 0, 0] = math.nan, math.inf, -math.inf
    elif kind == "huge":
        x = x * (1e4 if dt == F16 else 1e38)
    return x.clamp(-65504, 65504).to(dt) if dt == F16 and kind != "nonfinite" else x.to(dt)


@pytest.mark.parametrize("kind", ["normal", "ties", "constant", "wide", "nonfinite", "huge"])
@pytest.mark.parametrize("dt,T,heads,dim,page", [(F16, 50, 3, 128, 16), (BF16, 33, 2, 64, 64), (F16, 1, 1, 64, 32), (BF16, 200, 5, 128, 32)])
def test_append_stores_the_codes_of_exact_arithmetic(kind, dt, T, heads, dim, page):
    n = T // page + 3
    cache = B.Kv4Cache(torch.randint(0, 256, (n, B.kv4_page_bytes(page, heads, dim)), device=DEV, dtype=torch.uint8,
                                     generator=torch.Generator(device=DEV).manual_seed(9)), page, heads, dim, dt)
    kv = torch.cat([rows_for(kind, T, heads, dim, dt, s).flatten(1) for s in (1, 2)], 1)
    k, v = kv[:, :heads * dim], kv[:, heads * dim:]
    slots = torch.randperm(n * page, device=DEV, generator=torch.Generator(device=DEV).manual_seed(T))[:T]
    slots[T // 2:][::7] = torch.tensor([-1, n * page, -(1 << 40), 1 << 40], device=DEV).repeat(T)[:slots[T // 2:][::7].numel()]
    before = [x.clone() for x in R.decode_pages(cache.pages, page, heads, dim, torch.int16)]
    B.kv4_append(cache, k, v, slots)
    after = R.decode_pages(cache.pages, page, heads, dim, torch.int16)
    ok = ((slots >= 0) & (slots < n * page)).cpu()
    at = slots.cpu()[ok]
    for x, c0, s0, c1, s1 in ((k, before[0], before[2], after[0], after[2]), (v, before[1], before[3], after[1], after[3])):
        codes, step, eta = R.quantise(x.cpu().reshape(T, heads, dim)[ok])
        fine = ~torch.isnan(step)
        assert torch.equal(c1.reshape(n * page, heads, dim)[at][fine.expand_as(codes)], codes[fine.expand_as(codes)])
        se = s1.reshape(n * page, heads, 2)[at].view(dt)
        assert torch.equal(torch.isnan(se), (~fine).expand_as(se))
        assert torch.equal(torch.nan_to_num(se), torch.nan_to_num(torch.cat((step, eta), -1)))
        rest = torch.ones(n * page, dtype=torch.bool)
        rest[at] = False                          # every other slot is as it was
        assert torch.equal(c1.reshape(n * page, heads, dim)[rest], c0.reshape(n * page, heads, dim)[rest])
        assert torch.equal(s1.reshape(n * page, heads, 2)[rest], s0.reshape(n * page, heads, 2)[rest])
    # and back: eta + step * code, rounded once; rows without a slot stay
    ko, vo = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    B.kv4_read(cache, slots, k=ko, v=vo)
    for x, got in ((k, ko), (v, vo)):
        codes, step, eta = R.quantise(x.reshape(T, heads, dim))
        want = (eta.double() + step.double() * codes).flatten(1)
        okd = ok.to(DEV)
        check(got[okd], want[okd], R.half_step(dt) * want[okd].abs() + 2 * E * want[okd].abs() + torch.finfo(dt).smallest_normal * torch.finfo(dt).eps
              + 2 * E * eta.double().abs().expand(T, heads, dim).flatten(1)[okd])
        assert (got[~okd] == 7.0).all()


def test_read_in_any_order_and_repeated():
    page, heads, dim, dt = 32, 2, 64, BF16
    cache = B.Kv4Cache.empty(4, page, heads, dim, dt, DEV)
    k, v = randn(1, 128, heads * dim, dtype=dt), randn(2, 128, heads * dim, dtype=dt)
    B.kv4_append(cache, k, v, torch.arange(128, device=DEV))
    a = B.kv4_read(cache, torch.arange(128, device=DEV))
    order = torch.randint(0, 128, (300,), device=DEV)
    b = B.kv4_read(cache, order)
    assert torch.equal(b[0], a[0][order]) and torch.equal(b[1], a[1][order])
    z = B.kv4_read(cache, torch.tensor([-1, 128], device=DEV))
    assert not z[0].any() and not z[1].any()


# ---- attention over the cache ----------------------------------------------------------------------
def fill(batch, lens, page, heads, dim, dt, seed, spare=2, k_scale=1.0):
    """A cache with sequences of the given lengths in shuffled pages; returns (cache, table)."""
    per = max(1, max((n + page - 1) // page for n in lens))
    total = batch * per + spare
    cache = B.Kv4Cache.empty(total, page, heads, dim, dt, DEV)
    table = torch.randperm(total, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))[:batch * per].view(batch, per).int()
    T = total * page
    loud = torch.ones(dim, device=DEV)
    loud[3] = 5.0
    for i in range(0, T, 16384):
        m = min(16384, T - i)
        k = (randn(seed + i, m, heads, dim, scale=k_scale) * loud).to(dt).flatten(1)
        B.kv4_append(cache, k, (randn(seed + i + 1, m, heads * dim) + 0.5).to(dt), torch.arange(i, i + m, device=DEV))
    return cache, table


def cached(cache, table_row, n, h):
    """Values of head h of a sequence's first n tokens, 64 bits: k, v [n, D], and the steps and etas [n, 4]."""
    page, dim = cache.page_size, cache.head_dim
    ids = table_row[:(n + page - 1) // page].long()
    valid = (ids >= 0) & (ids < cache.pages.shape[0])
    blocks = cache.pages[ids.clamp(0, cache.pages.shape[0] - 1)]
    kc, vc, ks, vs = R.decode_pages(blocks.view(ids.numel(), cache.kv_heads, -1)[:, h].contiguous(), page, 1, dim, cache.dtype)
    ks, vs = ks.reshape(-1, 2)[:n].double(), vs.reshape(-1, 2)[:n].double()
    k = ks[:, 1:] + ks[:, :1] * kc.reshape(-1, dim)[:n]
    v = vs[:, 1:] + vs[:, :1] * vc.reshape(-1, dim)[:n]
    return k.to(DEV), v.to(DEV), ks.to(DEV), vs.to(DEV), valid.repeat_interleave(page)[:n]


def check_kv4(q, cache, table, lens, batch, n_q, heads, window, sinks, scale, o, some=None):
    dim, hk = cache.head_dim, cache.kv_heads
    sc = scale or 1 / math.sqrt(dim)
    for b in range(batch):
        n = min(max(int(lens[b]), 0), table.shape[1] * cache.page_size)
        pos = torch.arange(n_q, device=DEV) + n - n_q
        for h in range(heads) if some is None else some:
            rows = slice(b * n_q, (b + 1) * n_q)
            got = o[rows, h * dim:(h + 1) * dim]
            if n == 0:
                assert not got.any()
                continue
            k, v, ks, vs, valid = cached(cache, table[b], n, h // (heads // hk))
            seen = R.visible(pos, torch.arange(n, device=DEV), window, sinks) & valid[None]
            qh = q[rows, h * dim:(h + 1) * dim].double()
            want, p = R.attend(qh, k, v, seen, sc)
            use = seen.any(0)
            k, v, ks, vs, p = (x[use] if x.shape[0] == n else x[:, use] for x in (k, v, ks, vs, p))
            # sizes: a score is step * (q . code) + eta * sum q
            size_k = 15 * ks[:, 0] + ks[:, 1].abs()
            d = 4 * dim * E * sc * qh.abs().amax(-1, keepdim=True) * math.sqrt(dim) * (size_k.max() if size_k.numel() else 0.0)
            mass = p @ (v.abs() + 8 * vs[:, :1] if v.numel() else v)
            tol = (R.half_step(F16) + 2 * d + 64 * E * (1 + n / 1000)) * mass + R.half_step(cache.dtype) * want.abs() + 1e-7
            check(got, want, tol, f"sequence {b} head {h}")


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens,n_q,hk,g,dim,page,window,sinks", [
    ([1], 1, 1, 1, 128, 16, 0, 0), ([1000], 1, 16, 1, 128, 16, 0, 0), ([0, 1, 63, 64, 65], 1, 2, 4, 128, 64, 0, 0),
    ([700, 5, 0, 2], 4, 2, 4, 64, 32, 0, 0), ([300, 17, 129], 3, 3, 3, 128, 16, 50, 4), ([515, 64], 2, 1, 8, 64, 64, 64, 0),
    ([200, 90], 1, 4, 2, 128, 32, 1, 0), ([200, 90], 1, 4, 2, 128, 32, 1, 3), ([130], 9, 2, 5, 64, 16, 16, 1), ([333, 40], 21, 1, 1, 128, 16, 0, 0),
    ([5000, 777], 1, 2, 16, 128, 64, 0, 0), ([4097], 5, 5, 2, 64, 64, 100, 200), ([2500] * 9 + [1] * 8, 1, 8, 4, 128, 16, 1000, 17),
    ([40000], 2, 1, 4, 128, 64, 30000, 5), ([i * 37 % 301 for i in range(70)], 1, 2, 2, 64, 16, 0, 0), ([0] * 33 + [900, 0, 65], 2, 1, 1, 64, 64, 0, 0)])
def test_attention_kv4(dt, lens, n_q, hk, g, dim, page, window, sinks):
    batch, heads = len(lens), hk * g
    cache, table = fill(batch, lens, page, hk, dim, dt, seed=len(lens) + n_q)
    q = randn(5, batch * n_q, heads * dim + 64, dtype=dt)[:, :heads * dim]
    o = torch.full((batch * n_q, heads * dim + 8), 3.0, device=DEV, dtype=dt)
    lt = torch.tensor(lens, device=DEV, dtype=torch.int32)
    B.attention_kv4(q, cache, table, lt, batch, n_q, heads, window=window, sinks=sinks, o=o[:, :heads * dim])
    assert (o[:, heads * dim:] == 3.0).all()
    check_kv4(q, cache, table, lens, batch, n_q, heads, window, sinks, 0.0, o[:, :heads * dim])
    again = B.attention_kv4(q, cache, table, lt, batch, n_q, heads, window=window, sinks=sinks)
    assert torch.equal(again, o[:, :heads * dim])                     # same bits
    sc = 0.3
    check_kv4(q, cache, table, lens, batch, n_q, heads, window, sinks, sc,
              B.attention_kv4(q, cache, table, lt, batch, n_q, heads, window=window, sinks=sinks, scale=sc), some=[0, heads - 1])


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens,n_q,hk,g,dim,page,window,sinks", [
    ([i * 37 % 301 for i in range(110)], 1, 2, 3, 64, 16, 0, 0),                   # more lists than the GPU holds CTAs, short
    ([3, 700] + [i * 29 % 90 for i in range(38)], 1, 8, 1, 128, 64, 0, 0),         # the same with a long bound of the lengths
    ([i * 31 % 200 for i in range(80)], 3, 2, 4, 64, 32, 60, 2),                   # with more than 8 query rows
    ([4500] + [0] * 50 + [1, 130] * 75, 1, 1, 4, 64, 64, 0, 0),                    # one long list among many
    ([20000], 4, 1, 4, 128, 64, 0, 0), ([20000, 9], 1, 2, 4, 64, 32, 0, 0),        # lists too long for a cluster
    ([16384], 1, 1, 2, 64, 64, 0, 0), ([8191, 70, 0, 1], 1, 4, 2, 128, 64, 0, 0),  # clusters with four chunks per warp, and ragged
    ([64 * 8, 64 * 8 + 1], 6, 2, 2, 128, 16, 0, 0)])                               # one chunk per warp of a CTA, and one more
def test_attention_kv4_ways_of_cutting_the_lists(dt, lens, n_q, hk, g, dim, page, window, sinks):
    batch, heads = len(lens), hk * g
    cache, table = fill(batch, lens, page, hk, dim, dt, seed=len(lens) + n_q)
    q = randn(5, batch * n_q, heads * dim, dtype=dt)
    lt = torch.tensor(lens, device=DEV, dtype=torch.int32)
    o = B.attention_kv4(q, cache, table, lt, batch, n_q, heads, window=window, sinks=sinks)
    check_kv4(q, cache, table, lens, batch, n_q, heads, window, sinks, 0.0, o, some=[0, heads - 1])
    assert torch.equal(B.attention_kv4(q, cache, table, lt, batch, n_q, heads, window=window, sinks=sinks), o)


@pytest.mark.parametrize("dt", [F16, BF16])
def test_attention_kv4_sizes_of_the_values(dt):
    """Tiny and huge queries, keys and values: peaked and flat rows."""
    hk, dim, page, n = 2, 128, 32, 900
    for qs, ks, vs in ((1e-4, 1.0, 1.0), (30.0, 1.0, 1.0), (1.0, 1e-3, 1e-3), (1.0, 1.0, 3000.0), (1.0, 8.0, 1e-4), (0.0, 1.0, 1.0)):
        cache = B.Kv4Cache.empty(30, page, hk, dim, dt, DEV)
        B.kv4_append(cache, randn(1, 960, hk * dim, dtype=dt, scale=ks), randn(2, 960, hk * dim, dtype=dt, scale=vs), torch.arange(960, device=DEV))
        table = torch.arange(30, device=DEV).int().view(1, 30)
        q = randn(3, 2, 2 * hk * dim, dtype=dt, scale=qs)
        lens = torch.tensor([n], device=DEV).int()
        o = B.attention_kv4(q, cache, table, lens, 1, 2, 2 * hk)
        check_kv4(q, cache, table, [n], 1, 2, 2 * hk, 0, 0, 0.0, o)


def test_attention_kv4_of_what_it_must_not_see():
    """Pages that no query sees may be numbered anything, tokens behind the end or outside the window may hold NaN, a page
    number outside the cache hides its tokens, and lens beyond the table are clamped."""
    hk, g, dim, page, dt = 2, 2, 64, 16, F16
    heads, n = hk * g, 500
    cache, table = fill(1, [n], page, hk, dim, dt, seed=4, spare=3)
    nan = torch.full((page, hk * dim), math.nan, device=DEV, dtype=dt)
    q = randn(6, 2, heads * dim, dtype=dt)
    lens = torch.tensor([n], device=DEV).int()
    want = B.attention_kv4(q, cache, table, lens, 1, 2, heads, window=100, sinks=4)
    hidden = table.clone()
    hidden[0, 1:24] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31], device=DEV).int().repeat(8)[:23]   # tokens 16..383: outside
    slots = table[0, -1].long() * page + torch.arange(page, device=DEV)
    B.kv4_append(cache, nan, nan, torch.where(torch.arange(page, device=DEV) >= n % page, slots, -torch.ones_like(slots)))
    edge = table[0, 24].long() * page + torch.arange(page, device=DEV)
    B.kv4_append(cache, nan, nan, torch.where(torch.arange(384, 400, device=DEV) < n - 2 - 99, edge, -torch.ones_like(edge)))
    first = table[0, 0].long() * page + torch.arange(page, device=DEV)
    B.kv4_append(cache, nan, nan, torch.where(torch.arange(page, device=DEV) >= 4, first, -torch.ones_like(first)))
    got = B.attention_kv4(q, cache, hidden, lens, 1, 2, heads, window=100, sinks=4)
    assert torch.equal(got, want)
    lost = hidden.clone()
    lost[0, 28] = cache.pages.shape[0]                                # visible tokens 448..463
    lost[0, 0] = -5                                                   # and the sinks
    check_kv4(q, cache, lost, [n], 1, 2, heads, 100, 4, 0.0, B.attention_kv4(q, cache, lost, lens, 1, 2, heads, window=100, sinks=4))
    none = torch.full_like(table, -1)
    assert not B.attention_kv4(q, cache, none, lens, 1, 2, heads).any()
    cache2, table2 = fill(1, [64], page, hk, dim, dt, seed=5)
    big = torch.tensor([10 ** 9], device=DEV).int()
    check_kv4(q, cache2, table2, [64], 1, 2, heads, 0, 0, 0.0, B.attention_kv4(q, cache2, table2, big, 1, 2, heads))
    assert not B.attention_kv4(q, cache2, table2, -big, 1, 2, heads).any()
    # a visible NaN shows, in its own head's rows only
    B.kv4_append(cache2, nan, nan, torch.where(torch.arange(page, device=DEV) == 3, table2[0, 1].long() * page + 3, -1))
    assert torch.isnan(B.attention_kv4(q, cache2, table2, torch.tensor([64], device=DEV).int(), 1, 2, heads)).all()
    assert torch.isfinite(B.attention_kv4(q, cache2, table2, torch.tensor([18], device=DEV).int(), 1, 2, heads)).all()


@pytest.mark.parametrize("dt,big", [(F16, 60000.0), (BF16, 1e30)])
def test_attention_kv4_huge_values_of_a_later_token(dt, big):
    """The last drafted token's values are huge: the queries before it are as if it were not there."""
    hk, g, dim, page, n, n_q = 1, 2, 128, 32, 200, 3
    cache, table = fill(1, [n], page, hk, dim, dt, seed=11)
    q = randn(2, n_q, g * hk * dim, dtype=dt)
    at = table[0, (n - 1) // page].long().view(1) * page + (n - 1) % page
    B.kv4_append(cache, randn(3, 1, hk * dim, dtype=dt), randn(4, 1, hk * dim, dtype=F32).mul(big / 4).clamp(-big, big).to(dt), at)
    lens = torch.tensor([n], device=DEV).int()
    o = B.attention_kv4(q, cache, table, lens, 1, n_q, g * hk)
    check_kv4(q, cache, table, [n], 1, n_q, g * hk, 0, 0, 0.0, o)
    short = B.attention_kv4(q[:2], cache, table, lens - 1, 1, 2, g * hk)
    check_kv4(q[:2], cache, table, [n - 1], 1, 2, g * hk, 0, 0, 0.0, short)
    assert (o[:2].double() - short.double()).abs().max() <= 4 * R.half_step(dt) * float(short.abs().max())


def test_attention_kv4_in_a_graph_and_on_two_streams():
    hk, g, dim, page, dt, batch = 4, 4, 128, 32, F16, 3
    heads = hk * g
    cache, table = fill(batch, [3000] * batch, page, hk, dim, dt, seed=8)
    lens = torch.tensor([2999, 5, 1], device=DEV).int()
    q = randn(1, batch, heads * dim, dtype=dt)
    o = torch.empty_like(q)
    ws = torch.empty(B.attention_kv4_ws_bytes(batch, 1, heads, hk, dim), dtype=torch.uint8, device=DEV)
    B.attention_kv4(q, cache, table, lens, batch, 1, heads, o=o, ws=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attention_kv4(q, cache, table, lens, batch, 1, heads, o=o, ws=ws)
        lens.add_(1)
    for start in ([2990, 5, 0], [1, 2000, 64]):
        lens.copy_(torch.tensor(start, device=DEV))
        for i in range(3):                                           # the lengths grow inside the graph
            graph.replay()
            want = B.attention_kv4(q, cache, table, torch.tensor([s + i for s in start], device=DEV).int(), batch, 1, heads)
            assert torch.equal(o, want)
    streams = [torch.cuda.Stream() for _ in range(2)]
    qs = [randn(10 + i, batch, heads * dim, dtype=dt) for i in range(2)]
    lens = torch.tensor([2999, 5, 1], device=DEV).int()
    wants = [B.attention_kv4(x, cache, table, lens, batch, 1, heads) for x in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        outs = []
        for s, x in zip(streams, qs):
            with torch.cuda.stream(s):
                outs.append(B.attention_kv4(x, cache, table, lens, batch, 1, heads))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, wants))


def test_attention_kv4_reports_waits_that_run_out():
    hk, dim, page, dt = 2, 128, 32, F16
    cache, table = fill(2, [700, 300], page, hk, dim, dt, seed=3)
    q, lens = randn(1, 2, 2 * hk * dim, dtype=dt), torch.tensor([700, 300], device=DEV).int()
    ws = torch.empty(B.attention_kv4_ws_bytes(2, 1, 2 * hk, hk, dim), dtype=torch.uint8, device=DEV)
    want = B.attention_kv4(q, cache, table, lens, 2, 1, 2 * hk, ws=ws)
    assert B.ws_status(ws) == B.OK
    B.debug_wait_limit(0)
    try:
        B.attention_kv4(q, cache, table, lens, 2, 1, 2 * hk, ws=ws)
        assert B.ws_status(ws) == B.ERR_TIMEOUT
    finally:
        B.debug_wait_limit(-1)
    assert torch.equal(B.attention_kv4(q, cache, table, lens, 2, 1, 2 * hk, ws=ws), want)
    assert B.ws_status(ws) == B.OK


@pytest.mark.parametrize("batch,longest", [(2, 16500), (80, 200)])       # lists cut over the GPU: too long for clusters, too many
def test_attention_kv4_cut_lists_in_a_graph_on_two_streams_and_when_waits_run_out(batch, longest):
    hk, heads, dim, page, dt = 2, 8, 64, 64, BF16
    first = [longest] + [(i * 53 + 1) % longest for i in range(1, batch)]
    cache, table = fill(batch, first, page, hk, dim, dt, seed=9)
    lens = torch.tensor(first, device=DEV).int() - 3
    qs = [randn(20 + i, batch, heads * dim, dtype=dt) for i in range(2)]
    ws = [torch.empty(B.attention_kv4_ws_bytes(batch, 1, heads, hk, dim), dtype=torch.uint8, device=DEV) for _ in range(2)]
    wants = [[B.attention_kv4(x, cache, table, lens + i, batch, 1, heads) for i in range(3)] for x in qs]
    check_kv4(qs[0], cache, table, [max(n - 3, 0) for n in first], batch, 1, heads, 0, 0, 0.0, wants[0][0], some=[1])
    o, graph = torch.empty_like(qs[0]), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.attention_kv4(qs[0], cache, table, lens, batch, 1, heads, o=o, ws=ws[0])
        lens.add_(1)
    for i in range(3):
        graph.replay()
        assert torch.equal(o, wants[0][i])
    lens.sub_(3)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        outs = []
        for s, x, w in zip(streams, qs, ws):
            with torch.cuda.stream(s):
                outs.append(B.attention_kv4(x, cache, table, lens, batch, 1, heads, ws=w))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b[0]) for a, b in zip(outs, wants))
    B.debug_wait_limit(0)
    try:
        B.attention_kv4(qs[0], cache, table, lens, batch, 1, heads, ws=ws[0])
        assert B.ws_status(ws[0]) == B.ERR_TIMEOUT
    finally:
        B.debug_wait_limit(-1)
    assert torch.equal(B.attention_kv4(qs[0], cache, table, lens, batch, 1, heads, ws=ws[0]), wants[0][0])
    assert B.ws_status(ws[0]) == B.OK


def test_cache_beyond_32_bit_offsets():
    """A cache of 5 GB: the last pages lie beyond 2^32 bytes."""
    page, hk, dim, dt = 64, 8, 128, F16
    nbytes = B.kv4_page_bytes(page, hk, dim)
    total = (5 << 30) // nbytes
    pages = torch.zeros((total, nbytes), dtype=torch.uint8, device=DEV)
    cache = B.Kv4Cache(pages, page, hk, dim, dt)
    ids = torch.tensor([total - 1, 0, total - 2, total // 2], device=DEV).int()
    at = (ids.long()[:, None] * page + torch.arange(page, device=DEV)).view(-1)
    k, v = randn(1, 256, hk * dim, dtype=dt), randn(2, 256, hk * dim, dtype=dt)
    B.kv4_append(cache, k, v, at)
    small = B.Kv4Cache.empty(4, page, hk, dim, dt, DEV)
    B.kv4_append(small, k, v, torch.arange(256, device=DEV))
    q = randn(3, 1, 4 * hk * dim, dtype=dt)
    lens = torch.tensor([250], device=DEV).int()
    a = B.attention_kv4(q, cache, ids.view(1, 4), lens, 1, 1, 4 * hk)
    assert torch.equal(a, B.attention_kv4(q, small, torch.arange(4, device=DEV).int().view(1, 4), lens, 1, 1, 4 * hk))
    assert all(torch.equal(x, y) for x, y in zip(B.kv4_read(cache, at), B.kv4_read(small, torch.arange(256, device=DEV))))
    B.kv4_copy_pages(pages, torch.tensor([[total - 1, total - 3], [0, 7]], device=DEV).int())
    assert torch.equal(pages[total - 3], small.pages[0]) and torch.equal(pages[7], small.pages[1])


# ---- pages ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape,n", [((1, 3, 1152), 1), ((9, 16 * 4), 3), ((5, 40, 69632), 13), ((2, 30, 16), 7), ((3, 12, 33 * 1024 + 16), 4)])
def test_copy_pages(shape, n):
    g = torch.Generator(device=DEV).manual_seed(n)
    pages = torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8)
    num = shape[-2]
    perm = torch.randperm(num, generator=g, device=DEV)
    src, dst = perm[:n].clone(), perm[num - n:]
    src[-1] = src[0]                                                  # one source feeds two pages
    pairs = torch.stack((src, dst), 1).int()
    bad = torch.tensor([[-1, 0], [0, -1], [num, 0], [0, num], [2 ** 31 - 1, -2 ** 31], [5 % num, 5 % num]], device=DEV).int()
    want = pages.clone()
    want[..., dst, :] = want[..., src, :]
    got = B.kv4_copy_pages(pages, torch.cat((bad, pairs)))
    assert got is pages and torch.equal(pages, want)
    B.kv4_copy_pages(pages, pairs[:0])
    assert torch.equal(pages, want)


# ---- prompts with a window -------------------------------------------------------------------------
def check_window(q, k, v, o, seqs, heads, hk, dim, window, sinks, scale=0.0, some=None):
    sc = scale or 1 / math.sqrt(dim)
    dt = q.dtype
    for q0, nq, k0, nk in seqs:
        if nq == 0:
            continue
        pos = torch.arange(nq, device=DEV) + nk - nq
        seen = R.visible(pos, torch.arange(nk, device=DEV), window, sinks)
        for h in range(heads) if some is None else some:
            j = h // (heads // hk)
            qh, kh, vh = (x[a:a + n, c * dim:(c + 1) * dim].double() for x, a, n, c in ((q, q0, nq, h), (k, k0, nk, j), (v, k0, nk, j)))
            want, p = R.attend(qh, kh, vh, seen, sc)
            size = (qh.norm(dim=-1, keepdim=True) * torch.nan_to_num(kh, nan=0.0, posinf=0.0, neginf=0.0).norm(dim=-1).max()) if nk else 0.0
            mass = p @ torch.nan_to_num(vh, nan=0.0, posinf=0.0, neginf=0.0).abs()
            tol = (R.half_step(dt) + 8 * dim * E * sc * size + 64 * E * (1 + nk / 1000)) * mass + R.half_step(dt) * want.abs() + 1e-7
            check(o[q0:q0 + nq, h * dim:(h + 1) * dim], want, tol, f"rows {q0}.. head {h}")


def packed(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return torch.tensor(cu, device=DEV, dtype=torch.int32), cu


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("lens,heads,hk,dim,window,sinks", [
    ([1], 1, 1, 64, 0, 0), ([64, 64], 2, 2, 128, 0, 0), ([127, 1, 0, 129, 128], 4, 2, 64, 0, 0), ([300, 17], 3, 1, 128, 50, 4),
    ([513], 2, 1, 128, 128, 0), ([700, 33], 4, 4, 64, 1, 0), ([640], 2, 2, 64, 1, 300), ([1000, 500], 8, 2, 128, 200, 16),
    ([2049], 2, 1, 128, 0, 0), ([1500], 1, 1, 64, 129, 65), ([400], 6, 3, 128, 5000, 7), ([260, 3, 385], 2, 2, 128, 256, 1)])
def test_attention_window(dt, lens, heads, hk, dim, window, sinks):
    cu, at = packed(lens)
    T = at[-1]
    x = randn(T, T, (heads + 2 * hk) * dim, dtype=dt, scale=1.3)
    q, k, v = x[:, :heads * dim], x[:, heads * dim:(heads + hk) * dim], x[:, (heads + hk) * dim:]
    o = torch.full((T + 2, heads * dim + 8), 3.0, device=DEV, dtype=dt)
    B.attention_window(q, k, v, len(lens), max(lens), heads, hk, dim, window=window, sinks=sinks, cu_q=cu, o=o[:T, :heads * dim])
    assert (o[T:] == 3.0).all() and (o[:, heads * dim:] == 3.0).all()
    seqs = [(a, n, a, n) for a, n in zip(at, lens)]
    check_window(q, k, v, o[:T, :heads * dim], seqs, heads, hk, dim, window, sinks)
    again = B.attention_window(q, k, v, len(lens), max(lens) + 200, heads, hk, dim, window=window, sinks=sinks, cu_q=cu)
    assert torch.equal(again, o[:T, :heads * dim])                    # an upper bound beyond the lengths changes nothing
    sc = 0.2
    got = B.attention_window(q, k, v, len(lens), max(lens), heads, hk, dim, window=window, sinks=sinks, cu_q=cu, scale=sc)
    check_window(q, k, v, got, seqs, heads, hk, dim, window, sinks, sc, some=[heads - 1])


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("batch,seq_q,seq_k,window,sinks", [(2, 256, 256, 0, 0), (3, 100, 100, 64, 4), (2, 70, 333, 0, 0), (1, 1, 500, 100, 3),
                                                            (2, 130, 1000, 257, 70), (2, 200, 90, 0, 0), (1, 129, 0, 0, 0), (2, 300, 140, 64, 2)])
def test_attention_window_unpacked_and_behind_known_tokens(dt, batch, seq_q, seq_k, window, sinks):
    heads, hk, dim = 4, 2, 128
    q = randn(1, batch * seq_q, heads * dim, dtype=dt)
    kv = randn(2, batch * seq_k, 2 * hk * dim, dtype=dt)
    k, v = kv[:, :hk * dim], kv[:, hk * dim:]
    o = B.attention_window(q, k, v, batch, seq_q, heads, hk, dim, window=window, sinks=sinks, seq_k=seq_k)
    check_window(q, k, v, o, [(b * seq_q, seq_q, b * seq_k, seq_k) for b in range(batch)], heads, hk, dim, window, sinks)


@pytest.mark.parametrize("batch", [70, 33])
def test_attention_window_many_ragged_prompts(batch):
    """One long prompt among many short and empty ones: each block of rows is found in a batch of more than a warp's lanes."""
    heads, hk, dim, dt = 2, 1, 64, F16
    lens = [(i * 53) % 200 if i % 5 else 0 for i in range(batch)]
    lens[batch - 2] = 1500
    cu, at = packed(lens)
    q, k, v = (randn(i, at[-1], w * dim, dtype=dt) for i, w in ((1, heads), (2, hk), (3, hk)))
    o = B.attention_window(q, k, v, batch, 1500, heads, hk, dim, window=100, sinks=1, cu_q=cu)
    check_window(q, k, v, o, [(a, n, a, n) for a, n in zip(at, lens)], heads, hk, dim, 100, 1)
    big = B.attention_window(q, k, v, batch, 1 << 20, heads, hk, dim, window=100, sinks=1, cu_q=cu)
    assert torch.equal(big, o)


def test_attention_window_lengths_apart_and_rows_outside():
    """Queries and keys packed apart, bounds below the lengths, offsets that are no offsets."""
    heads, hk, dim, dt = 2, 1, 64, F16
    lq, lk = [5, 200, 0, 64], [300, 200, 40, 10]
    cq, aq = packed(lq)
    ck, ak = packed(lk)
    q, k, v = randn(1, aq[-1] + 9, heads * dim, dtype=dt), randn(2, ak[-1] + 5, hk * dim, dtype=dt), randn(3, ak[-1] + 5, hk * dim, dtype=dt)
    o = torch.full_like(q, 3.0)
    B.attention_window(q, k, v, 4, 200, heads, hk, dim, window=90, sinks=2, cu_q=cq, cu_k=ck, seq_k=300, o=o)
    check_window(q, k, v, o, list(zip(aq, lq, ak, lk)), heads, hk, dim, 90, 2)
    assert (o[aq[-1]:] == 3.0).all()
    o = torch.full_like(q, 3.0)
    B.attention_window(q, k, v, 4, 130, heads, hk, dim, cu_q=cq, cu_k=ck, seq_k=250, o=o)   # rows past the bounds are left out
    lq2, lk2 = [min(n, 130) for n in lq], [min(n, 250) for n in lk]
    check_window(q, k, v, o, list(zip(aq, lq2, ak, lk2)), heads, hk, dim, 0, 0)
    assert (o[aq[1] + 130:aq[2]] == 3.0).all()
    wild = torch.tensor([-7, 20, 10 ** 9, 5, 2 ** 31 - 1], device=DEV).int()
    rows = q.shape[0]
    o = B.attention_window(q, q[:, :dim], q[:, :dim], 4, rows, heads, hk, dim, cu_q=wild, o=torch.full_like(q, 3.0))
    # clamped: rows 0..19, 20..end, none (the end before the start), 5..end; rows from 5 on belong to two sequences
    check_window(q, q[:, :dim], q[:, :dim], o, [(0, 5, 0, 5)], heads, hk, dim, 0, 0)
    assert torch.isfinite(o).all()


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_window_of_what_it_must_not_see(dt, dim):
    """Infinities and NaN at keys that come later, lie outside the window or belong to the next sequence."""
    heads, hk, lens, window, sinks = 2, 1, [400, 150], 100, 3
    cu, at = packed(lens)
    T = at[-1]
    q, k, v = randn(1, T, heads * dim, dtype=dt), randn(2, T, hk * dim, dtype=dt), randn(3, T, hk * dim, dtype=dt)
    clean = B.attention_window(q, k, v, 2, 400, heads, hk, dim, window=window, sinks=sinks, cu_q=cu)
    for bad in (math.nan, math.inf, -math.inf):
        for row in (30, 399, 400, 549):
            k2, v2 = k.clone(), v.clone()
            k2[row], v2[row, ::3] = bad, bad
            got = B.attention_window(q, k2, v2, 2, 400, heads, hk, dim, window=window, sinks=sinks, cu_q=cu)
            seen = torch.zeros(T, dtype=torch.bool, device=DEV)       # rows that see it
            a, n = (0, 400) if row < 400 else (400, 150)
            seen[a:a + n] = R.visible(torch.arange(n, device=DEV), torch.arange(n, device=DEV), window, sinks)[:, row - a]
            assert torch.isfinite(got[~seen]).all()
            err = (got[~seen].double() - clean[~seen].double()).abs()
            assert (err <= 4 * R.half_step(dt) * v.abs().max().double()).all()
            if math.isnan(bad):
                assert torch.isnan(got[seen]).all()


@pytest.mark.parametrize("dt", [F16, BF16])
def test_attention_window_rows_of_padding_hold_anything(dt):
    """Rows between and behind the sequences are never initialised: NaN and infinities there change nothing."""
    heads, hk, dim = 4, 2, 128
    q0, lens = [0, 150, 400], [130, 193, 57]
    rows = 600
    q, k, v = (randn(i, rows, w * dim, dtype=dt) for i, w in ((1, heads), (2, hk), (3, hk)))
    inside = torch.zeros(rows, dtype=torch.bool, device=DEV)
    for a, n in zip(q0, lens):
        inside[a:a + n] = True
    for x, bad in ((q, math.nan), (k, math.inf), (v, math.nan)):
        x[~inside] = bad
    for a, n in zip(q0, lens):                                        # one sequence at a time: cu need not be contiguous
        cu = torch.tensor([a, a + n], device=DEV, dtype=torch.int32)
        o = B.attention_window(q, k, v, 1, n, heads, hk, dim, window=70, sinks=2, cu_q=cu, o=torch.full_like(q, 3.0))
        check_window(q, k, v, o, [(a, n, a, n)], heads, hk, dim, 70, 2)
        keep = torch.ones(rows, dtype=torch.bool, device=DEV)
        keep[a:a + n] = False
        assert (o[keep] == 3.0).all()


def test_attention_window_agrees_with_the_causal_core():
    """No window, equal heads: bitlinear_attention_causal's operation."""
    batch, seq, heads = 2, 320, 3
    x = randn(5, batch * seq, 3 * heads * 128, dtype=F16)
    q, k, v = (x[:, i * heads * 128:(i + 1) * heads * 128] for i in range(3))
    a = B.attention_causal(q, k, v, batch, seq, heads)
    b = B.attention_window(q, k, v, batch, seq, heads)
    assert (a.double() - b.double()).abs().max() <= 8 * R.half_step(F16) * float(v.abs().max())
    g = torch.cuda.CUDAGraph()
    o = torch.empty_like(b)
    with torch.cuda.graph(g):
        B.attention_window(q, k, v, batch, seq, heads, o=o)
    x.copy_(randn(6, *x.shape, dtype=F16))
    g.replay()
    assert torch.equal(o, B.attention_window(q, k, v, batch, seq, heads))


def test_attention_window_when_its_waits_run_out():
    """With no polls allowed every wait runs out: the rows are computed the slow way, and counted."""
    heads, hk, dim, lens = 4, 2, 128, [300, 0, 140]
    cu, at = packed(lens)
    q, kv = randn(1, at[-1], heads * dim, dtype=F16), randn(2, at[-1], 2 * hk * dim, dtype=F16)
    k, v = kv[:, :hk * dim], kv[:, hk * dim:]
    B.debug_window_fallbacks()
    want = B.attention_window(q, k, v, 3, 300, heads, hk, dim, window=100, sinks=2, cu_q=cu)
    assert B.debug_window_fallbacks() == 0
    B.debug_wait_limit(0)
    try:
        got = B.attention_window(q, k, v, 3, 300, heads, hk, dim, window=100, sinks=2, cu_q=cu)
        assert B.debug_window_fallbacks() > 0
    finally:
        B.debug_wait_limit(-1)
    check_window(q, k, v, got, [(a, n, a, n) for a, n in zip(at, lens)], heads, hk, dim, 100, 2)
    assert (got.double() - want.double()).abs().max() <= 8 * R.half_step(F16) * float(v.abs().max())
    assert B.debug_window_fallbacks() == 0


def test_calls_with_nothing_to_do():
    dt, hk, dim, page = F16, 2, 64, 16
    cache = B.Kv4Cache.empty(2, page, hk, dim, dt, DEV)
    none = torch.empty((0, hk * dim), device=DEV, dtype=dt)
    at = torch.empty(0, device=DEV, dtype=torch.int64)
    B.kv4_append(cache, none, none, at)
    assert B.kv4_read(cache, at)[0].shape == (0, hk * dim)
    lens = torch.zeros(3, device=DEV, dtype=torch.int32)
    q = randn(1, 3, 2 * hk * dim, dtype=dt)
    assert not B.attention_kv4(q, cache, torch.empty((3, 0), device=DEV, dtype=torch.int32), lens + 5, 3, 1, 2 * hk).any()
    assert not B.attention_kv4(q, cache, torch.zeros((3, 2), device=DEV, dtype=torch.int32), lens, 3, 1, 2 * hk).any()
    assert B.attention_kv4(q[:0], cache, torch.empty((0, 2), device=DEV, dtype=torch.int32), lens[:0], 0, 1, 2 * hk).shape == (0, 2 * hk * dim)
    assert B.attention_window(q[:0], none, none, 0, 0, 2 * hk, hk, dim).shape == (0, 2 * hk * dim)
    assert not B.attention_window(q, none, none, 3, 1, 2 * hk, hk, dim, seq_k=0).any()          # queries, and not a key
    empty = B.Kv4Cache.empty(0, page, hk, dim, dt, DEV)
    B.kv4_append(empty, q[:, :hk * dim], q[:, :hk * dim], torch.zeros(3, device=DEV, dtype=torch.int64))
    assert not B.attention_kv4(q, empty, torch.zeros((3, 1), device=DEV, dtype=torch.int32), lens + 1, 3, 1, 2 * hk).any()
    B.kv4_copy_pages(empty.pages, torch.zeros((1, 2), device=DEV, dtype=torch.int32))


def test_arguments_that_do_not_fit_each_other_are_refused():
    dt, hk, dim, page = F16, 2, 64, 16
    cache = B.Kv4Cache.empty(4, page, hk, dim, dt, DEV)
    k, at = randn(1, 3, hk * dim, dtype=dt), torch.arange(3, device=DEV)
    table, lens, q = torch.zeros((3, 2), device=DEV, dtype=torch.int32), torch.ones(3, device=DEV, dtype=torch.int32), randn(2, 3, 2 * hk * dim, dtype=dt)
    pos, freq = torch.zeros(3, device=DEV, dtype=torch.int32), torch.ones(32, device=DEV)
    for bad in (lambda: B.kv4_append(cache, k, k[:2], at), lambda: B.kv4_append(cache, k, k, at[:2]), lambda: B.kv4_append(cache, k, k, at.cpu()),
                lambda: B.kv4_append(cache, k.t().contiguous().t(), k, at), lambda: B.kv4_read(cache, at, k=k[:, :64]),
                lambda: B.attention_kv4(q[:2], cache, table, lens, 3, 1, 2 * hk), lambda: B.attention_kv4(q, cache, table[:2], lens, 3, 1, 2 * hk),
                lambda: B.attention_kv4(q, cache, table.t(), lens, 3, 1, 2 * hk), lambda: B.attention_kv4(q, cache, table, lens[:2], 3, 1, 2 * hk),
                lambda: B.attention_window(q, k, k[:2], 1, 3, 2 * hk, hk, dim), lambda: B.attention_window(q, k, k, 1, 3, 2 * hk, hk, dim, cu_q=pos),
                lambda: B.qk_norm_rope(q, k, pos[:2], freq, 2 * hk, hk, dim), lambda: B.qk_norm_rope(q, k, pos, freq, 2 * hk, hk, 2 * dim),
                lambda: B.kv4_copy_pages(cache.pages, table[:, :1]), lambda: B.kv4_copy_pages(cache.pages[:, :16], table)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.kv4_append(cache, k.float(), k, at), lambda: B.kv4_append(cache, k, k, at.int()), lambda: B.kv4_append(cache, None, k, at),
                lambda: B.attention_kv4(q.bfloat16(), cache, table, lens, 3, 1, 2 * hk), lambda: B.attention_kv4(q, cache, table.long(), lens, 3, 1, 2 * hk),
                lambda: B.attention_window(q, k.float(), k, 1, 3, 2 * hk, hk, dim), lambda: B.qk_norm_rope(q, k, pos.long(), freq, 2 * hk, hk, dim),
                lambda: B.qk_norm_rope(q, k, pos, freq, 2 * hk, hk, dim, wq=torch.ones(dim, device=DEV)), lambda: B.attention_window(q, k, k, "1", 3, 4, 2, dim)):
        with pytest.raises(TypeError):
            bad()
    small = torch.empty(256, device=DEV, dtype=torch.uint8)
    for bad, code in ((lambda: B.attention_kv4(q, cache, table, lens, 3, 1, 2 * hk, ws=small), B.ERR_WORKSPACE),
                      (lambda: B.attention_window(q.float(), k.float(), k.float(), 1, 3, 2 * hk, hk, dim), B.ERR_UNSUPPORTED),
                      (lambda: B.attention_kv4(q, cache, table, lens, 3, 1, 2 * hk, scale=-1.0), B.ERR_SHAPE)):
        with pytest.raises(B.BitLinearError) as err:
            bad()
        assert err.value.code == code


def test_a_captured_decode_step_replayed():
    """Norm and rotation in place, append, attention and a copy of pages in one graph; positions and lengths advance inside it."""
    heads, hk, dim, page, dt, batch = 8, 2, 128, 16, BF16, 3
    freq = (10000.0 ** (-torch.arange(0, dim, 2, device=DEV).double() / dim)).float()
    pages = torch.zeros((2, 40, B.kv4_page_bytes(page, hk, dim)), dtype=torch.uint8, device=DEV)
    cache = B.Kv4Cache(pages[0], page, hk, dim, dt)
    table = torch.randperm(36, device=DEV)[:batch * 10].view(batch, 10).int()
    start = torch.tensor([0, 15, 70], device=DEV).int()
    lens = start.clone()
    x = randn(1, 12, batch, (heads + 2 * hk) * dim, dtype=dt)
    step = torch.zeros(1, device=DEV, dtype=torch.int64)
    o = torch.empty((batch, heads * dim), device=DEV, dtype=dt)
    pairs = torch.tensor([[0, 38], [1, 39]], device=DEV).int()

    def decode(out):
        y = x[step][0].clone()
        q, k, v = y[:, :heads * dim], y[:, heads * dim:(heads + hk) * dim], y[:, (heads + hk) * dim:]
        B.qk_norm_rope(q, k, lens, freq, heads, hk, dim, q_out=q, k_out=k)
        at = lens.long()
        B.kv4_append(cache, k, v, table.long().gather(1, (at // page)[:, None])[:, 0] * page + at % page)
        lens.add_(1)
        B.attention_kv4(q, cache, table, lens, batch, 1, heads, window=40, sinks=3, o=out)
        B.kv4_copy_pages(pages, pairs)
        step.add_(1)
    wants = []
    for _ in range(12):
        decode(o)
        wants.append(o.clone())
    final = pages.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        decode(o)
    for _ in range(2):
        pages.zero_(); lens.copy_(start); step.zero_()
        for want in wants:
            graph.replay()
            assert torch.equal(o, want)
        assert torch.equal(pages, final) and torch.equal(pages[:, 38], pages[:, 0])


# ---- together ------------------------------------------------------------------------------------
def test_a_prompt_and_decode_steps_through_bitlinear_layers():
    """A prompt enters the cache, a sequence is forked, and both decode tokens: BitLinear projections by the decode
    GEMVs, norm and rotation, append, attention over the cache.  Every step is checked against its definition on what the
    step before it left."""
    heads, hk, dim, page, dt, n0 = 8, 4, 128, 32, F16, 75
    d, width, freq = heads * dim, (heads + 2 * hk) * dim, (10000.0 ** (-torch.arange(0, dim, 2, device=DEV).double() / dim)).float()
    W = B.binarize_pack(randn(1, width, d), layout=B.DECODE)
    torch.cuda.synchronize()
    pages = torch.zeros((2, 16, B.kv4_page_bytes(page, hk, dim)), dtype=torch.uint8, device=DEV)   # two layers, the second is used
    cache = B.Kv4Cache(pages[1], page, hk, dim, dt)
    split = lambda x: (x[:, :d], x[:, d:d + hk * dim], x[:, d + hk * dim:])  # noqa: E731
    x = randn(2, n0, d, dtype=dt)
    q, k, v = split(B.gemv_decode_batch_ws(x, W["W_packed"], W["beta"], width))
    pos = torch.arange(n0, device=DEV).int()
    q, k = B.qk_norm_rope(q, k, pos, freq, heads, hk, dim)
    o = B.attention_window(q, k, v, 1, n0, heads, hk, dim, window=48, sinks=2)
    check_window(q, k, v, o, [(0, n0, 0, n0)], heads, hk, dim, 48, 2)
    table = torch.tensor([[3, 9, 1, 14], [3, 9, 6, 11]], device=DEV).int()     # the second shares the first's full pages
    B.kv4_append(cache, k, v, table[0].long().repeat_interleave(page)[:n0] * page + torch.arange(n0, device=DEV) % page)
    B.kv4_copy_pages(pages, torch.tensor([[1, 6]], device=DEV).int())          # the fork's own copy of the last page
    lens = torch.full((2,), n0, device=DEV, dtype=torch.int32)
    h = torch.cat((o[-1:], o[-2:-1]))
    for step in range(30):
        q, k, v = split(B.gemv_decode_batch_ws(h, W["W_packed"], W["beta"], width))
        q2, k2 = B.qk_norm_rope(q, k, lens, freq, heads, hk, dim)
        at = lens.long()
        B.kv4_append(cache, k2, v, table[torch.arange(2, device=DEV), at // page].long() * page + at % page)
        lens = lens + 1
        o = B.attention_kv4(q2, cache, table, lens, 2, 1, heads, window=48, sinks=2)
        check_kv4(q2, cache, table, lens.tolist(), 2, 1, heads, 48, 2, 0.0, o)
        h = o
    assert not torch.equal(o[0], o[1]) and not pages[0].any()
    shared = B.kv4_read(cache, torch.arange(3 * page, 4 * page, device=DEV))
    want = R.quantise(B.qk_norm_rope(*split(B.gemv_decode_batch_ws(x, W["W_packed"], W["beta"], width))[:2], pos, freq, heads, hk, dim)[1][:page].view(page, hk, dim))
    assert torch.equal(shared[0], (want[1].float() * want[0] + want[2].float()).to(dt).flatten(1))
