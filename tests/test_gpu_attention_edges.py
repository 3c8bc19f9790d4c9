"""The attention operators at inputs where a wrong answer hides."""
import math

import pytest
import torch

from paper_2310_11453_b200 import binding as B
from tests import attention_ref as R
from tests.test_gpu_attention_ops import BF16, DEV, F16, F32, check_kv4, check_window, fill, packed, randn

pytestmark = pytest.mark.gpu


# ---- attention over the cache: what is not finite shows, however the work was cut ------------------
# lengths, n_q, key/value heads, group, head_dim, page: each way of cutting the lists
CUTS = [
    ([129], 1, 2, 2, 64, 16), ([65, 641, 1], 1, 2, 4, 128, 32), ([321, 64 * 6 + 1], 3, 2, 4, 64, 64),          # clusters
    ([64 * 320 + 1], 1, 1, 4, 128, 64), ([64 * 313 + 1, 9], 2, 2, 8, 64, 32),                                  # a CTA of 32 warps joins a row
    ([64 * 266 + 1, 9, 321, 65], 1, 8, 8, 64, 64),                                                             # a CTA of 8 warps
    ([64 * (i % 5) + 1 for i in range(110)], 1, 2, 3, 64, 16), ([65 + 64 * (i % 3) for i in range(80)], 3, 2, 4, 64, 32),   # a warp, and lists
    ([64 * 70 + 1] + [0] * 50 + [1, 129] * 75, 1, 1, 4, 64, 64),                                               # that one warp holds as a whole
]


def laid_out(dt, cut, positive=False):
    lens, n_q, hk, g, dim, page = cut
    cache, table = fill(len(lens), lens, page, hk, dim, dt, seed=len(lens) + n_q)
    if positive:                                                       # every key value lies between 1 and 2
        T = cache.pages.shape[0] * page
        rows = torch.rand((T, hk * dim), device=DEV, generator=torch.Generator(device=DEV).manual_seed(3)) + 1
        B.kv4_append(cache, rows.to(dt), randn(4, T, hk * dim, dtype=dt), torch.arange(T, device=DEV))
    q = randn(5, len(lens) * n_q, hk * g * dim, dtype=dt)
    return cache, table, torch.tensor(lens, device=DEV, dtype=torch.int32), q


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("dt,bad,positive", [(F16, math.nan, False), (BF16, math.inf, False), (F16, -math.inf, False), (BF16, -math.inf, True)])
def test_attention_kv4_query_that_is_not_finite(dt, bad, positive, cut):
    """One row of one head holds a value that is not finite: no softmax of its scores exists, so the row is NaN (its scores are
    NaN, or some are +infinity, or, where all keys are positive, all are -infinity).  All other rows keep their bits."""
    cache, table, lens, q = laid_out(dt, cut, positive)
    batch, n_q, heads, dim = len(cut[0]), cut[1], cut[2] * cut[3], cut[4]
    want = B.attention_kv4(q, cache, table, lens, batch, n_q, heads)
    assert torch.isfinite(want).all()
    for b in {0, batch - 1, batch // 2}:
        for h in {0, heads - 1}:
            q2 = q.clone()
            q2[b * n_q + n_q - 1, h * dim + dim // 3] = bad
            got = B.attention_kv4(q2, cache, table, lens, batch, n_q, heads)
            expect = want.clone()
            if cut[0][b] > 0:
                expect[b * n_q + n_q - 1, h * dim:(h + 1) * dim] = math.nan
            assert torch.equal(torch.isnan(got), torch.isnan(expect)), (b, h)
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(expect)), (b, h)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("cut", CUTS)
def test_attention_kv4_newest_token_that_is_not_finite(dt, cut):
    """The newest token's key or value of one key/value head is stored as NaN, alone in its chunk where the length is 64 k + 1:
    the newest query of that head's group is NaN.  Queries before it, other heads and other sequences keep their bits."""
    lens, n_q, hk, g, dim, page = cut
    batch, heads = len(lens), hk * g
    for what in ("key", "value"):
        cache, table, lt, q = laid_out(dt, cut)
        want = B.attention_kv4(q, cache, table, lt, batch, n_q, heads)
        for b in {0, batch - 1}:
            if lens[b] == 0:
                continue
            at = table[b, (lens[b] - 1) // page].long().view(1) * page + (lens[b] - 1) % page
            pages = cache.pages.clone()
            k, v = B.kv4_read(cache, at)
            (k if what == "key" else v)[0, (hk - 1) * dim + 5] = math.nan
            hit = B.Kv4Cache(pages, page, hk, dim, dt)
            B.kv4_append(hit, k, v, at)
            kept = cache.pages.clone().view(cache.pages.shape[0], hk, -1)
            kept[:, hk - 1] = pages.view(cache.pages.shape[0], hk, -1)[:, hk - 1]       # the other heads as they were, to the bit
            got = B.attention_kv4(q, B.Kv4Cache(kept.view_as(pages), page, hk, dim, dt), table, lt, batch, n_q, heads)
            expect = want.clone()
            expect[b * n_q + n_q - 1, (hk - 1) * g * dim:] = math.nan
            assert torch.equal(torch.isnan(got), torch.isnan(expect)), (what, b)
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(expect)), (what, b)


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("given", [False, True])
def test_attention_kv4_rows_are_nan_where_waits_run_out(given, cut):
    """With no polls allowed no chunk arrives: rows that miss tokens are NaN, whether or not the caller can ask for the status, and
    whatever the workspace held.  A sequence without tokens waits for nothing."""
    lens, n_q, hk, g, dim, page = cut
    batch, heads = len(lens), hk * g
    cache, table, lt, q = laid_out(BF16, cut)
    want = B.attention_kv4(q, cache, table, lt, batch, n_q, heads)
    size = B.attention_kv4_ws_bytes(batch, n_q, heads, hk, dim)
    ws = torch.randint(0, 256, (size,), device=DEV, dtype=torch.uint8) if given else None
    o = torch.full_like(want, 3.0)
    B.debug_wait_limit(0)
    try:
        B.attention_kv4(q, cache, table, lt, batch, n_q, heads, o=o, ws=ws)
        if given:
            assert B.ws_status(ws) == B.ERR_TIMEOUT
        torch.cuda.synchronize()
    finally:
        B.debug_wait_limit(-1)
    some = (lt > 0).repeat_interleave(n_q)
    assert torch.isnan(o[some]).all() and not o[~some].any()
    assert torch.equal(B.attention_kv4(q, cache, table, lt, batch, n_q, heads, o=o, ws=ws), want)
    assert not given or B.ws_status(ws) == B.OK


@pytest.mark.parametrize("lens", [[0, 300], [0, 64 * 270], [0] * 90 + [1]])
def test_attention_kv4_a_report_stays(lens):
    """Warps report waits that ran out each in a word of its own: the first CTA, which has nothing to do here, clears nobody else's.
    Every such word counts, and a call that ends well clears them all."""
    hk, heads, dim, page = 2, 4, 64, 64
    cut = (lens, 1, hk, heads // hk, dim, page)
    batch = len(lens)
    cache, table, lt, q = laid_out(F16, cut)
    ws = torch.randint(0, 256, (B.attention_kv4_ws_bytes(batch, 1, heads, hk, dim),), device=DEV, dtype=torch.uint8)
    B.debug_wait_limit(0)
    try:
        for _ in range(100):
            B.attention_kv4(q, cache, table, lt, batch, 1, heads, ws=ws)
            assert B.ws_status(ws) == B.ERR_TIMEOUT
    finally:
        B.debug_wait_limit(-1)
    B.attention_kv4(q, cache, table, lt, batch, 1, heads, ws=ws)
    assert B.ws_status(ws) == B.OK
    words = ws.view(torch.int32)
    n = int(words[0]) & 0x7FF
    assert n % 8 == 0 and not words[1:1 + n].any()
    for i in (1, 2, n // 2, n - 1, n):
        words[i] = B.ERR_TIMEOUT
        assert B.ws_status(ws) == B.ERR_TIMEOUT
        words[i] = 0
    assert B.ws_status(ws) == B.OK
    words[1:1 + n] = B.ERR_TIMEOUT
    B.attention_kv4(q, cache, table, lt, batch, 1, heads, ws=ws)
    assert B.ws_status(ws) == B.OK


@pytest.mark.parametrize("size,step", [(2.0 ** 117, 1e-35), (2.0 ** 110, 1e-33), (2.0 ** -100, 2.0 ** 100)])
def test_attention_kv4_sizes_of_the_query_at_the_ends_of_bf16(size, step):
    hk, g, dim, page, n = 1, 2, 128, 32, 300
    cache = B.Kv4Cache.empty(10, page, hk, dim, BF16, DEV)
    B.kv4_append(cache, (randn(1, 320, hk * dim) * step).to(BF16), randn(2, 320, hk * dim, dtype=BF16), torch.arange(320, device=DEV))
    q = (randn(3, 1, g * hk * dim) * size).to(BF16)
    table, lens = torch.arange(10, device=DEV).int().view(1, 10), torch.tensor([n], device=DEV).int()
    check_kv4(q, cache, table, [n], 1, 1, g * hk, 0, 0, 0.0, B.attention_kv4(q, cache, table, lens, 1, 1, g * hk))


# ---- prompts with a window -------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_attention_window_query_that_is_not_finite(dt, dim, bad):
    """Every key is positive where the query is not finite, so -infinity makes every score -infinity: no softmax exists."""
    heads, hk, lens = 2, 1, [1, 300, 70]
    cu, at = packed(lens)
    q, v = randn(1, at[-1], heads * dim, dtype=dt), randn(3, at[-1], hk * dim, dtype=dt)
    k = randn(2, at[-1], hk * dim, dtype=dt)
    k[:, 7] = k[:, 7].abs() + 0.5
    want = B.attention_window(q, k, v, 3, 300, heads, hk, dim, window=100, sinks=2, cu_q=cu)
    for row in (0, 1, 200, at[-1] - 1):
        q2 = q.clone()
        q2[row, dim + 7] = bad
        got = B.attention_window(q2, k, v, 3, 300, heads, hk, dim, window=100, sinks=2, cu_q=cu)
        expect = want.clone()
        expect[row, dim:] = math.nan
        assert torch.equal(torch.isnan(got), torch.isnan(expect)), row
        assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(expect)), row


def test_attention_window_packed_chunks_behind_known_tokens_need_no_bound_of_the_keys():
    heads, hk, dim, dt = 4, 2, 128, F16
    lq, lk = [16, 1, 40, 16], [100, 700, 41, 16]
    cq, aq = packed(lq)
    ck, ak = packed(lk)
    q, k, v = randn(1, aq[-1], heads * dim, dtype=dt), randn(2, ak[-1], hk * dim, dtype=dt), randn(3, ak[-1], hk * dim, dtype=dt)
    o = B.attention_window(q, k, v, 4, 40, heads, hk, dim, window=64, sinks=3, cu_q=cq, cu_k=ck)
    check_window(q, k, v, o, list(zip(aq, lq, ak, lk)), heads, hk, dim, 64, 3)
    assert torch.equal(o, B.attention_window(q, k, v, 4, 40, heads, hk, dim, window=64, sinks=3, cu_q=cq, cu_k=ck, seq_k=700))


# ---- norm and rotation -----------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("dim,rot", [(128, 64), (80, 32), (256, 16), (64, 0)])
@pytest.mark.parametrize("inter", [False, True])
def test_norm_rope_values_that_do_not_turn_stay_apart(dt, dim, rot, inter):
    """An infinity or NaN behind rot_dim says nothing about other values (without the norm; with it, the mean is infinite)."""
    T, heads, kv = 9, 3, 2
    q, k = randn(1, T, heads * dim, dtype=dt), randn(2, T, kv * dim, dtype=dt)
    for x, n in ((q, heads), (k, kv)):
        x.view(T, n, dim)[1, 0, rot] = math.inf
        x.view(T, n, dim)[2, n - 1, dim - 1] = -math.inf
        x.view(T, n, dim)[3, 1, rot + (dim - rot) // 2] = math.nan
        x.view(T, n, dim)[4, 0, rot + 8] = math.inf
    pos = torch.arange(T, device=DEV).int() * 77
    freq = (10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=torch.float64) / max(rot, 1))).float()
    for x, y in zip((q, k), B.qk_norm_rope(q, k, pos, freq, heads, kv, dim, eps=-1.0, interleaved=inter)):
        x, y = x.view(T, -1, dim)[..., rot:], y.view(T, -1, dim)[..., rot:]
        assert torch.equal(torch.isnan(y), torch.isnan(x)) and torch.equal(torch.nan_to_num(y, nan=1.5), torch.nan_to_num(x, nan=1.5))
    for x, y in zip((q, k), B.qk_norm_rope(q, k, pos, freq, heads, kv, dim, eps=1e-6, interleaved=inter)):
        want = R.norm_rope(x, None, pos, freq, dim, 1e-6, inter)[0]
        assert torch.equal(torch.isnan(y), torch.isnan(want))


# ---- the binding -----------------------------------------------------------------------------------
def test_a_single_row_may_have_any_stride():
    heads, hk, dim, page, dt = 4, 2, 64, 16, F16

    def odd(seed, width):                                              # one row out of rows of an odd length
        x = torch.empty((1, width + 5), device=DEV, dtype=dt)
        x[:, :width] = randn(seed, 1, width, dtype=dt)
        return x[:, :width]
    q, k, v = odd(1, heads * dim), odd(2, hk * dim), odd(3, hk * dim)
    dense = [x.clone(memory_format=torch.contiguous_format) for x in (q, k, v)]
    pos, freq = torch.tensor([7], device=DEV).int(), torch.ones(dim // 2, device=DEV)
    for a, b in zip(B.qk_norm_rope(q, k, pos, freq, heads, hk, dim), B.qk_norm_rope(*dense[:2], pos, freq, heads, hk, dim)):
        assert torch.equal(a, b)
    assert torch.equal(B.attention_window(q, k, v, 1, 1, heads, hk, dim), B.attention_window(*dense, 1, 1, heads, hk, dim))
    cache = B.Kv4Cache.empty(2, page, hk, dim, dt, DEV)
    B.kv4_append(cache, k, v, torch.tensor([5], device=DEV))
    outs = [odd(4, hk * dim), odd(5, hk * dim)]
    for a, b in zip(B.kv4_read(cache, torch.tensor([5], device=DEV), k=outs[0], v=outs[1]), B.kv4_read(cache, torch.tensor([5], device=DEV))):
        assert torch.equal(a, b)
    table, lens = torch.zeros((1, 1), device=DEV, dtype=torch.int32), torch.tensor([6], device=DEV).int()
    assert torch.equal(B.attention_kv4(q, cache, table, lens, 1, 1, heads, o=odd(6, heads * dim)), B.attention_kv4(dense[0], cache, table, lens, 1, 1, heads))
