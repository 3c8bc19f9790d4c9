"""The 8-bit layers and the expert operators on the GPU against their definitions in 64 bits.

Tolerances.  u(T) = eps(T) / 2 is one rounding to T, e = 2^-24 one of fp32.  Outputs are rounded once: u |y|; a 16-bit output
under the smallest normal number, half a unit there (fp16: 2^-25).
Norm: h is a sum of n terms, (n + 1) e of their sizes.  The mean is a sum of at most 32 squares per thread and 11 joins, and its square
root halves that: with the products 40 e.  A code is the rounding of v = 127 h w / max |h w|: five roundings of at most 127 e beside
the terms' own, below 2^-13, so it may differ by one where the exact v is that near to a border, and nowhere else.
Matrix product of codes: exact, then its conversion, two scales, bias, residual: 5 e of the sizes of the terms.
Of fp16 and bf16: K products in fp32 in any order, truncating or not: 2 K e sum |x| |w|; none at all for small whole numbers.
Weights of experts: exp of a difference d (rounded: e |d| relative, |d| < 64 here), 2 e for exp, E terms in the sum: (72 + E) e."""
import math

import pytest
import torch

from paper_2310_11453_b200 import binding as B
from tests import layers8_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
F16, BF16, F32, I8 = torch.float16, torch.bfloat16, torch.float32, torch.int8
TINY = {F16: 2.0 ** -25, BF16: 1e-40, F32: 1e-40}


def randn(seed, *shape, dtype=F32, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def whole(seed, lo, hi, *shape, dtype=I8):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).to(dtype)


def check(got, want, tol, what=""):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    same = (got == want) | torch.isnan(want)                       # infinities among them
    bad = ~same & ~((got - want).abs() <= tol)
    assert not bad.any(), f"{what}: {int(bad.sum())} values off, worst {float(((got - want).abs() / tol.clamp(min=1e-300))[bad].max()):.3g} x the tolerance"


# ---- norm ------------------------------------------------------------------------------------------
def check_norm(x, weight=None, eps=1e-6, residual=None, rows=None, row_weights=None, **kw):
    dt, n = x.dtype, 2 + (rows.shape[1] if rows is not None else 0)
    codes, scale, h, y = B.rms_norm_quant(x, weight, eps, residual, rows, row_weights, h=kw.pop("h", True), y=True, **kw)
    wh, size = R.summed(x, residual, rows, row_weights)            # before the call wrote in place: callers pass copies
    return codes, scale, h, y, wh, size, n, dt


def verify_norm(codes, scale, h, y, wh, size, n, dt, weight, eps):
    K = wh.shape[1]
    check(h, wh, n * E * size + R.half_step(dt) * wh.abs() + TINY[dt], "h")
    want = R.normed(wh, weight, eps)
    w = weight.double().abs() if weight is not None and eps >= 0 else torch.ones(K, dtype=torch.float64, device=DEV)
    r = want.abs() / (wh.abs() * w).clamp(min=1e-300)              # the norm's factor, wherever h is not 0
    r = r.amax(-1, keepdim=True)
    off = n * E * size * w * r                                     # of y, from the terms of h
    rel = off.pow(2).mean(-1, keepdim=True).sqrt() / want.pow(2).mean(-1, keepdim=True).sqrt().clamp(min=1e-300)
    near = 40 * E + rel
    check(y, want, off + near * want.abs() + R.half_step(dt) * want.abs() + TINY[dt], "y")
    top = want.abs().amax(-1, keepdim=True)
    check(scale[:, None], top / 127, (near + 4 * E) * top / 127 + off.amax(-1, keepdim=True) / 127 + 1e-40, "scale")
    v = torch.where(top > 0, want / top.clamp(min=1e-300) * 127, torch.zeros_like(want))
    slack = 2.0 ** -13 + 127 * (off + off.amax(-1, keepdim=True)) / top.clamp(min=1e-300)
    d = (codes.double() - v).abs()
    assert bool((d <= 0.5 + slack).all()), f"codes: worst {float((d - slack).max())}"


@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("T,K,pad", [(1, 8, 0), (3, 128, 8), (5, 264, 0), (130, 768, 16), (1, 4096, 0), (37, 2056, 8), (301, 5120, 0), (2, 16392, 0), (3, 32768, 8),
                                     (150, 8192, 0)])
def test_norm(dt, T, K, pad):
    buf = randn(T + K, T, 2 * K + 2 * pad, dtype=dt, scale=3.0)
    x, res = buf[:, :K], buf[:, K + pad:2 * K + pad]
    weight = (1 + randn(5, K, scale=0.3)).to(dt)
    for w, eps, r in ((weight, 1e-6, res), (None, 1e-2, None), (weight, 0.0, res), (weight, -1.0, None)):
        verify_norm(*check_norm(x, w, eps, r), w, eps)


@pytest.mark.parametrize("dt", [F16, BF16, F32])
@pytest.mark.parametrize("T,K,k,x_rows", [(1, 64, 1, 1), (9, 768, 2, 5), (33, 2048, 8, 264), (5, 4104, 64, 40), (4, 16384, 3, 12)])
def test_norm_of_summed_rows(dt, T, K, k, x_rows):
    x, res = randn(K + k, x_rows, K, dtype=dt), randn(7, T, K, dtype=dt)
    rows = whole(3, 0, x_rows - 1, T, k, dtype=torch.int32)
    if T > 1:                                                      # rows that are not there: nothing is added
        rows[0, 0], rows[1] = -1, -1
        rows[2 % T, k - 1] = x_rows
    p = torch.softmax(randn(8, T, k), -1)
    weight = (1 + randn(5, K, scale=0.3)).to(dt)
    verify_norm(*check_norm(x, weight, 1e-5, res, rows, p), weight, 1e-5)
    verify_norm(*check_norm(x, None, 1e-5, None, rows, None), None, 1e-5)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_norm_of_values_at_the_ends_of_the_range(dt):
    K = 1024
    x = randn(1, 8, K)
    x[0] *= 1e37
    x[1] *= 1e-37
    x[2] = 0
    x[3] = 1e-30
    x[4, 1:] = 0                                                   # a single value
    x[5] *= 1e25
    x[6] *= 1e-22
    x = x.to(dt)
    for eps in (1e-6, 0.0, 1e-38, -1.0):
        codes, scale, h, y = B.rms_norm_quant(x, None, eps, h=True, y=True)
        want = R.normed(x.double(), None, eps)
        tol = (64 * E + R.half_step(dt)) * want.abs() + 1e-38 * 2.0 ** -7
        check(y, want, tol, f"y at eps {eps}")
        top = want.abs().amax(-1)
        check(scale, top / 127, 64 * E * top + 1e-44, f"scale at eps {eps}")
        v = torch.where(top[:, None] > 0, want / top[:, None].clamp(min=1e-300) * 127, torch.zeros_like(want))
        assert bool(((codes.double() - v).abs() <= 0.5 + 2.0 ** -13).all()), eps
        assert torch.equal(h, x)


@pytest.mark.parametrize("dt", [F16, BF16, F32])
def test_norm_of_rows_that_are_not_finite(dt):
    x = randn(1, 6, 512, dtype=dt)
    x[1, 5], x[2, 0], x[3, 511], x[4, 7] = math.nan, math.inf, -math.inf, math.inf
    x[4, 8] = -math.inf
    for eps in (1e-6, -1.0):
        codes, scale, h, y = B.rms_norm_quant(x, None, eps, h=True, y=True)
        assert torch.equal(torch.isnan(scale).cpu(), torch.tensor([False, True, True, True, True, False]))
        assert not codes[1:5].any() and codes[0].abs().max() == 127
        assert torch.equal(torch.isnan(y[1]).all().cpu(), torch.tensor(eps > 0)) or eps < 0
        if eps > 0:
            assert bool(torch.isnan(y[2, 0])) and not bool(y[2, 1:].any())          # finite / infinite = 0
        check(h, x.double(), 0 * x.double().abs().nan_to_num(), "h")


def test_norm_in_place_on_other_streams_and_with_nothing_to_do():
    T, K = 45, 1536
    x, res, weight = randn(1, T, K, dtype=BF16), randn(2, T, K, dtype=BF16), randn(3, K, dtype=BF16)
    want = B.rms_norm_quant(x, weight, residual=res, h=True, y=True)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        r2, x2 = res.clone(), x.clone()
        codes = torch.full((T, K + 16), 99, dtype=I8, device=DEV)
        got = B.rms_norm_quant(x2, weight, residual=r2, h=r2, y=x2, x_q=codes[:, :K], scale=torch.empty(T, device=DEV))
    s.synchronize()
    assert got[2] is r2 and got[3] is x2
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    assert bool((codes[:, K:] == 99).all())
    q, sc, h, y = B.rms_norm_quant(x, weight, x_q=None, y=True)
    assert q is None and sc is None and h is None and y.shape == x.shape
    assert B.rms_norm_quant(x[:0], weight)[0].shape == (0, K)
    with pytest.raises(ValueError):
        B.rms_norm_quant(x, weight[:-8])
    with pytest.raises(TypeError):
        B.rms_norm_quant(x, weight.float())
    with pytest.raises(ValueError):
        B.rms_norm_quant(x, weight, row_weights=torch.ones(T, 1, device=DEV))
    with pytest.raises(B.BitLinearError):
        B.rms_norm_quant(x, weight, x_q=None)


@pytest.mark.parametrize("T,K", [(3, 512), (40, 8192), (200, 3000)])
def test_norm_of_which_one_output_is_wanted(T, K):
    x, res, weight = randn(1, T, K, dtype=F16), randn(2, T, K, dtype=F16), randn(3, K, dtype=F16)
    codes, scale, h, y = B.rms_norm_quant(x, weight, residual=res, h=True, y=True)
    only = B.rms_norm_quant(x, weight, residual=res, h=True, x_q=None)
    assert torch.equal(only[2], h) and only[0] is None and only[1] is None and only[3] is None
    assert torch.equal(B.rms_norm_quant(x, weight, residual=res, x_q=None, y=True)[3], y)
    q, s, none, none2 = B.rms_norm_quant(x, weight, residual=res)
    assert torch.equal(q, codes) and torch.equal(s, scale) and none is None and none2 is None


# ---- matrix product of codes -------------------------------------------------------------------------
def check_product(got, x, w, yt, xs=None, ws=None, bias=None, relu=False, residual=None, exact=True):
    want, size = R.product(x, w, xs, ws, bias, relu, residual)
    tol = 5 * E * size + R.half_step(yt) * want.abs() + TINY[yt]
    if not exact:
        tol = tol + 2 * x.shape[1] * E * (x.double().abs() @ w.double().abs().t())
    if want.numel():
        check(got, want, tol)


SIZES = [(1, 16, 1), (1, 4096, 1000), (2, 48, 5), (15, 144, 129), (16, 128, 128), (17, 2048, 513), (31, 272, 255), (33, 1040, 130), (64, 4096, 256), (65, 768, 384),
         (100, 4112, 77), (128, 512, 256), (129, 256, 257), (255, 1168, 300), (257, 2064, 511), (300, 1024, 1024), (513, 4096, 640), (1000, 784, 2050)]


@pytest.mark.parametrize("yt", [F16, BF16, F32])
@pytest.mark.parametrize("M,K,N", SIZES)
def test_matmul(yt, M, K, N):
    x, w = whole(M + K, -128, 127, M, K), whole(N, -128, 127, N, K)
    xs, ws = randn(1, M).abs() * 0.01, randn(2, N).abs() * 0.003
    bias, res = randn(3, N, dtype=yt), randn(4, M, N, dtype=yt)
    check_product(B.matmul_i8(x, xs, w, ws, out_dtype=yt), x, w, yt, xs, ws)
    got = B.matmul_i8(x, xs, w, ws, out_dtype=yt, bias=bias, relu=True, residual=res)
    check_product(got, x, w, yt, xs, ws, bias, True, res)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_matmul_of_the_longest_rows(M):
    K, N = 131056, 130
    x, w = whole(1, -128, 127, M, K), whole(2, -128, 127, N, K)
    x[0], w[0] = -128, -128                                        # the largest sum there is
    got = B.matmul_i8(x, None, w, None, out_dtype=F32)
    assert float(got[0, 0]) == 128.0 * 128 * K
    check_product(got, x, w, F32)


@pytest.mark.parametrize("M,N", [(3, 200), (70, 130), (300, 260)])
def test_matmul_strides_and_what_lies_around(M, N):
    K = 320
    xb, wb = whole(1, -127, 127, M, K + 48), whole(2, -127, 127, N, K + 16)
    x, w = xb[:, 16:16 + K], wb[:, :K]
    xs, ws = randn(1, M).abs(), randn(2, N).abs()
    buf = torch.full((M + 2, N + 7), 7.0, dtype=BF16, device=DEV)
    res = randn(9, M, N + 3, dtype=BF16)[:, 1:N + 1]
    got = B.matmul_i8(x, xs, w, ws, residual=res, y=buf[1:-1, 3:3 + N])
    check_product(got, x, w, BF16, xs, ws, residual=res)
    buf[1:-1, 3:3 + N] = 7.0
    assert bool((buf == 7.0).all())
    h = res.clone()
    assert B.matmul_i8(x, xs, w, ws, residual=h, y=h) is h         # in place
    check_product(h, x, w, BF16, xs, ws, residual=res)


def test_matmul_shows_what_is_not_finite():
    x, w = whole(1, -127, 127, 5, 256), whole(2, -127, 127, 200, 256)
    xs, ws = torch.ones(5, device=DEV), torch.ones(200, device=DEV)
    xs[1], ws[3] = math.nan, math.nan
    got = B.matmul_i8(x, xs, w, ws, relu=True)
    assert bool(torch.isnan(got[1]).all()) and bool(torch.isnan(got[:, 3]).all())
    assert not bool(torch.isnan(got[[0, 2, 3, 4]][:, [0, 1, 2] + list(range(4, 200))]).any())


def test_matmul_refusals():
    x, w, s = whole(1, -9, 9, 4, 64), whole(2, -9, 9, 8, 64), torch.ones(4, device=DEV)
    with pytest.raises(ValueError):
        B.matmul_i8(x, s[:3], w, None)
    with pytest.raises(TypeError):
        B.matmul_i8(x.float(), s, w, None)
    with pytest.raises(ValueError):
        B.matmul_i8(x, s, w[:, :32], None)
    with pytest.raises(TypeError):
        B.matmul_i8(x, s, w, None, out_dtype=torch.int32)
    with pytest.raises(B.BitLinearError):
        B.matmul_i8(x[:, :24], s, w[:, :24], None)                 # K not a multiple of 16
    assert B.matmul_i8(x[:0], s[:0], w, None).shape == (0, 8)


# ---- the choice of experts ---------------------------------------------------------------------------
def check_route(z, k, normalise, positions=None):
    chosen, weights, offsets, rows, places = B.route_topk(z, k, normalise, positions)
    c, w, o, r, p = R.route(z, k, normalise, positions)
    assert chosen.tolist() == c and offsets.tolist() == o and places.tolist() == p
    assert rows[:len(r)].tolist() == r
    got = weights.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(w))
    assert bool(((got - w).abs() <= (72 + z.shape[1]) * E * w + 1e-37)[~torch.isnan(w)].all())


@pytest.mark.parametrize("dt", [F32, F16, BF16])
@pytest.mark.parametrize("T,E_,k", [(1, 1, 1), (1, 8, 2), (18, 64, 8), (33, 33, 32), (64, 100, 3), (65, 16, 1), (200, 128, 8), (1000, 257, 4), (67, 512, 32), (3000, 7, 2)])
def test_route(dt, T, E_, k):
    z = randn(T + E_, T, E_ + 3, dtype=dt, scale=2.0)[:, 1:E_ + 1]
    check_route(z, k, True)
    check_route(z, k, False)


def test_route_of_many_tokens():
    T, E_, k = 40001, 8, 2                                         # more runs of tokens than the placing kernel sums up itself
    z = randn(1, T, E_, dtype=BF16)
    check_route(z, k, True)
    check_route(z, k, True, whole(2, -1, 3, T, dtype=torch.int32))


@pytest.mark.parametrize("T", [5, 64, 130])
def test_route_ties_padding_and_scores_that_are_not_finite(T):
    z = whole(T, -1, 1, T, 40, dtype=F32)                          # many equal scores, zeros of both signs
    z[0] = 0.0
    z[0, 1::2] = -0.0
    z[1] = -math.inf
    z[2, 7] = math.nan
    z[3, 11] = math.inf
    z[4] = -math.inf
    z[4, [3, 9]] = 1.0
    check_route(z, 3, True)
    check_route(z, 3, False)
    z[2, 8:] = math.nan
    z[2, :7] = -math.inf
    check_route(z, 9, True)
    pos = torch.arange(T, device=DEV).int()
    pos[[0, T - 1]] = -1
    check_route(z, 3, True, pos)
    pos[:] = -5                                                    # nothing but padding
    rows = torch.full((T * 3,), 77, dtype=torch.int32, device=DEV)
    out = B.route_topk(z, 3, True, pos, rows=rows)
    assert not out[2].any() and bool((out[0] == -1).all()) and bool((out[4] == -1).all()) and not out[1].any() and bool((rows == 77).all())


def test_route_of_no_tokens_and_refusals():
    z = randn(1, 4, 8)
    out = B.route_topk(z[:0], 2)
    assert out[2].tolist() == [0] * 9 and out[3].numel() == 0
    with pytest.raises(ValueError):
        B.route_topk(z, 9)
    with pytest.raises(TypeError):
        B.route_topk(z.double(), 2)
    with pytest.raises(ValueError):
        B.route_topk(z, 2, positions=torch.zeros(3, dtype=torch.int32, device=DEV))


# ---- products grouped by expert ------------------------------------------------------------------------
def lists(counts):
    return torch.tensor([0] + [sum(counts[:i + 1]) for i in range(len(counts))], dtype=torch.int32, device=DEV)


def check_grouped(got, x, w, counts, rows, yt, first=0, **kw):
    exact = kw.pop("whole", False) or x.dtype == I8
    at = first
    for e, n in enumerate(counts):
        r = rows[at:at + n].long() if rows is not None else torch.arange(at, at + n, device=DEV)
        one = {k: (v[r] if k == "xs" else v[e]) for k, v in kw.items() if k != "relu" and v is not None}
        check_product(got[at:at + n], x[r], w[e], yt, relu=kw.get("relu", False), exact=exact, **one)
        at += n


GROUPS = [([1], 1, 64, 40), ([0, 3, 0, 1], 4, 144, 130), ([5, 16, 17, 0, 33, 1], 30, 512, 300), ([64, 0, 65, 200], 100, 784, 257), ([0, 0, 300], 300, 1040, 513),
          ([700, 0, 5], 256, 256, 256), ([1] * 40, 7, 2048, 128), ([129, 257, 1, 130], 517, 2064, 520)]


@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("yt", [F16, BF16, F32])
@pytest.mark.parametrize("counts,T,K,N", GROUPS)
def test_grouped_codes(counts, T, K, N, yt, listed):
    n, e = sum(counts), len(counts)
    x_rows = T if listed else n
    x, w = whole(K, -128, 127, x_rows, K), whole(N, -128, 127, e, N, K)
    rows = whole(4, 0, x_rows - 1, n, dtype=torch.int32) if listed else None
    xs, ws, bias = randn(1, x_rows).abs() * 0.01, randn(2, e, N).abs() * 0.01, randn(3, e, N, dtype=yt)
    got = B.matmul_grouped(x, w, lists(counts), rows, xs, ws, out_dtype=yt)
    check_grouped(got, x, w, counts, rows, yt, xs=xs, ws=ws)
    got = B.matmul_grouped(x, w, lists(counts), rows, xs, ws, bias=bias, relu=True, out_dtype=yt)
    check_grouped(got, x, w, counts, rows, yt, xs=xs, ws=ws, bias=bias, relu=True)


@pytest.mark.parametrize("dt", [F16, BF16])
@pytest.mark.parametrize("counts,T,K,N", GROUPS)
def test_grouped_values(counts, T, K, N, dt):
    n, e = sum(counts), len(counts)
    rows = whole(4, 0, T - 1, n, dtype=torch.int32)
    x, w, bias = randn(1, T, K, dtype=dt), randn(2, e, N, K, dtype=dt, scale=0.05), randn(3, e, N, dtype=F32)
    check_grouped(B.matmul_grouped(x, w, lists(counts), rows), x, w, counts, rows, dt)
    check_grouped(B.matmul_grouped(x, w, lists(counts), rows, bias=bias, out_dtype=F32), x, w, counts, rows, F32, bias=bias)
    x, w = whole(5, -8, 8, T, K, dtype=dt), whole(6, -8, 8, e, N, K, dtype=dt)       # whole numbers: every sum is exact
    check_grouped(B.matmul_grouped(x, w, lists(counts), rows, out_dtype=F32), x, w, counts, rows, F32, whole=True)


@pytest.mark.parametrize("dt", [I8, BF16])
@pytest.mark.parametrize("scale", [1, 12])
def test_grouped_rows_outside_the_lists_and_bad_indices(dt, scale):
    K, N, e, T = 192, 140, 4, 50 * scale
    x, w = whole(1, -8, 8, T, K, dtype=dt), whole(2, -8, 8, e, N + 3, K + 32, dtype=dt)[:, :N, :K]
    R_ = 60 * scale
    rows = whole(3, 0, T - 1, R_, dtype=torch.int32)
    counts = [7 * scale, 0, 20 * scale, 13]
    first = 5
    offsets = lists(counts) + first
    y = torch.full((R_ + 1, N + 5), 9.0, device=DEV)
    got = B.matmul_grouped(x, w, offsets, rows, y=y[:R_, :N])
    check_grouped(got, x, w, counts, rows, F32, first=first, whole=True)
    last = first + sum(counts)
    y[first:last, :N] = 9.0
    assert bool((y == 9.0).all())
    # offsets beyond the list are cut to it, rows beyond x to its ends
    rows[first], rows[first + 1] = -7, T + 1000
    offsets[-1] = R_ + 12345
    got = B.matmul_grouped(x, w, offsets, rows, out_dtype=F32)
    counts[-1] = R_ - first - sum(counts[:-1])
    check_grouped(got, x, w, counts, rows.clamp(0, T - 1), F32, first=first, whole=True)
    offsets[:] = torch.tensor([-3, 10, -2 ** 31, 2 ** 31 - 1, 4], device=DEV)          # nothing sensible: nothing out of range is touched
    y = torch.full((R_ + 2, N), 9.0, device=DEV)
    B.matmul_grouped(x, w, offsets, rows, y=y[1:-1])
    assert bool((y[0] == 9.0).all()) and bool((y[-1] == 9.0).all())


def test_grouped_many_experts_and_refusals():
    e, K, N = 1024, 64, 20
    counts = [(i * 7) % 5 for i in range(e)]
    n = sum(counts)
    x, w = whole(1, -9, 9, n, K), whole(2, -9, 9, e, N, K)
    check_grouped(B.matmul_grouped(x, w, lists(counts), out_dtype=F32), x, w, counts, None, F32)
    with pytest.raises(ValueError):
        B.matmul_grouped(x, w, lists(counts)[:-1])
    with pytest.raises(TypeError):
        B.matmul_grouped(x, w.half(), lists(counts))
    with pytest.raises(TypeError):
        B.matmul_grouped(x.float(), w.float(), lists(counts))
    with pytest.raises(B.BitLinearError):
        B.matmul_grouped(x.half(), w.half(), lists(counts), x_scale=torch.ones(n, device=DEV))
    assert B.matmul_grouped(x[:0], w, lists([0] * e)).shape == (0, N)


@pytest.mark.parametrize("dt", [I8, F16])
@pytest.mark.parametrize("counts", [[2, 0, 3], [90, 0, 333]])
def test_grouped_strides(counts, dt):
    K, N, T, n = 336, 150, 50, sum(counts)
    xb, wb = whole(1, -8, 8, max(T, n), K + 64, dtype=dt), whole(2, -8, 8, len(counts), N + 2, K + 16, dtype=dt)
    x, w = xb[:, 32:32 + K], wb[:, :N, :K]
    rows = whole(3, 0, T - 1, n, dtype=torch.int32)
    check_grouped(B.matmul_grouped(x[:T], w, lists(counts), rows, out_dtype=F32), x, w, counts, rows, F32, whole=True)
    check_grouped(B.matmul_grouped(x[:n], w, lists(counts), out_dtype=F32), x, w, counts, None, F32, whole=True)


def test_grouped_many_long_lists_and_the_longest_rows():
    e, K, N = 1024, 64, 260
    counts = [17 + (i * 11) % 23 for i in range(e)]
    n = sum(counts)
    x, w = whole(1, -9, 9, 500, K), whole(2, -9, 9, e, N, K)
    rows = whole(3, 0, 499, n, dtype=torch.int32)
    got = B.matmul_grouped(x, w, lists(counts), rows, out_dtype=F32)
    expert = torch.repeat_interleave(torch.arange(e, device=DEV), torch.tensor(counts, device=DEV))
    want = torch.cat([torch.einsum("rk,rnk->rn", x[rows[a:a + 4000].long()].double(), w[expert[a:a + 4000]].double()) for a in range(0, n, 4000)])
    assert torch.equal(got.double(), want)
    K = 1 << 20
    for counts in ([3, 0, 2], [130, 5]):
        x, w = whole(4, -2, 2, 20, K, dtype=BF16), whole(5, -2, 2, len(counts), 140, K, dtype=BF16)      # sums up to 2^22: exact
        rows = whole(6, 0, 19, sum(counts), dtype=torch.int32)
        got, at = B.matmul_grouped(x, w, lists(counts), rows, out_dtype=F32), 0
        for i, c in enumerate(counts):
            assert torch.equal(got[at:at + c].double(), (x.double() @ w[i].double().t())[rows[at:at + c].long()])
            at += c


@pytest.mark.parametrize("polls", [0, 1, 3])
@pytest.mark.parametrize("counts", [[3, 0, 9], [300, 77]])
def test_grouped_waits_that_run_out(counts, polls):
    x, w = whole(1, -9, 9, 64, 2048), whole(2, -9, 9, len(counts), 600, 2048)
    rows = whole(3, 0, 63, sum(counts), dtype=torch.int32)
    want = B.matmul_grouped(x, w, lists(counts), rows, out_dtype=F32)
    offsets = lists(counts)
    torch.cuda.synchronize()
    B.debug_wait_limit(polls)
    try:
        got = B.matmul_grouped(x, w, offsets, rows, out_dtype=F32)
        torch.cuda.synchronize()
    finally:
        B.debug_wait_limit(-1)
    bad = torch.isnan(got)
    assert torch.equal(got[~bad], want[~bad]) and (polls > 0 or bool(bad.all()))
    assert torch.equal(B.matmul_grouped(x, w, offsets, rows, out_dtype=F32), want)


@pytest.mark.parametrize("values", [[0, 300, 5, 700, 2, 900, 900, 20], [900, 0, 900, 0, 900, 0, 900, 0], [5, 4, 3, 2, 1, 0, -1, -2]])
def test_grouped_offsets_that_decrease_touch_nothing_twice_and_nothing_else(values):
    e, K, N, R_ = 7, 64, 300, 900
    x, w = whole(1, -9, 9, R_, K), whole(2, -9, 9, e, N, K)
    y = torch.full((R_ + 2, N), 9.25, device=DEV)
    B.matmul_grouped(x, w, torch.tensor(values, dtype=torch.int32, device=DEV), y=y[1:-1])
    assert bool((y[0] == 9.25).all()) and bool((y[-1] == 9.25).all())
    every = torch.einsum("rk,enk->ern", x.double(), w.double())
    known = (y[1:-1].double() == every).all(-1).any(0) | (y[1:-1] == 9.25).all(-1)
    assert bool(known.all())                                       # a row is some expert's product, or untouched


def test_results_beyond_32_bits():
    M, K, N = 140001, 32, 32768                                    # 4.6e9 outputs
    x, w = whole(1, -9, 9, M, K), whole(2, -9, 9, N, K)
    got = B.matmul_i8(x, None, w, None)
    for rows in (slice(0, 3), slice(65534, 65540), slice(131070, 131075), slice(M - 300, M)):
        check_product(got[rows], x[rows], w, BF16)
    off = torch.tensor([0, 70000, M], dtype=torch.int32, device=DEV)
    got = B.matmul_grouped(x, torch.stack((w, -w)), off, y=got)
    check_product(got[65530:65545], x[65530:65545], w, BF16)
    check_product(got[M - 300:], x[M - 300:], -w, BF16)
    del got
    T, K = 530001, 4096                                            # 2.2e9 values
    x = torch.zeros((T, K), dtype=F16, device=DEV)
    x[-5:] = randn(3, 5, K, dtype=F16)
    codes, scale, _, _ = B.rms_norm_quant(x)
    want = B.rms_norm_quant(x[-5:].clone())
    assert torch.equal(codes[-5:], want[0]) and torch.equal(scale[-5:], want[1]) and not codes[:-5].any()


def test_weights_quantised_just_before_they_are_used():
    """Weights are read ahead of the stream's order, but not ahead of the kernel that quantises them."""
    x, xs = whole(1, -127, 127, 3, 2048), torch.ones(3, device=DEV)
    latent = [randn(i, 4096, 2048, dtype=BF16) for i in range(6)]
    want = []
    for w in latent:
        q, s, _, _ = B.rms_norm_quant(w, eps=-1.0)
        torch.cuda.synchronize()
        want.append(B.matmul_i8(x, xs, q, s, out_dtype=F32))
    q, s = torch.empty((4096, 2048), dtype=I8, device=DEV), torch.empty(4096, device=DEV)
    for _ in range(3):
        got = []
        for w in latent:                                           # the same buffer again and again
            B.rms_norm_quant(w, eps=-1.0, x_q=q, scale=s)
            got.append(B.matmul_i8(x, xs, q, s, out_dtype=F32))
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_norm_of_nothing_but_rows_that_are_not_there():
    x, res = randn(1, 0, 256, dtype=BF16), randn(2, 5, 256, dtype=BF16)
    rows = torch.tensor([[-1, 0], [7, -1], [-1, -1], [1 << 30, 3], [0, 0]], dtype=torch.int32, device=DEV)
    q, s, h, _ = B.rms_norm_quant(x, None, 1e-6, res, rows, torch.full((5, 2), math.nan, device=DEV), h=True)
    want = B.rms_norm_quant(res, None, 1e-6)
    assert torch.equal(h, res) and torch.equal(q, want[0]) and torch.equal(s, want[1])


@pytest.mark.parametrize("T,E_", [(7, 8), (200, 24)])
def test_captured_without_a_call_before(T, E_):
    z = randn(3, T, E_)
    x, w = whole(1, -9, 9, T, 208), whole(2, -9, 9, E_, 104, 208)
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            chosen, weights, offsets, rows, places = B.route_topk(z, 2)
            up = B.matmul_grouped(x, w, offsets, rows, out_dtype=F32)
            q, sc, _, _ = B.rms_norm_quant(up, rows=places, row_weights=weights)
    for _ in range(2):
        z.copy_(randn(9, T, E_))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
    check_route(z, 2, True)
    c = R.route(z, 2, True)
    assert chosen.tolist() == c[0]
    counts = [b - a for a, b in zip(c[2], c[2][1:])]
    check_grouped(up, x, w, counts, rows, F32)
    want = B.rms_norm_quant(up, rows=places, row_weights=weights)
    assert torch.equal(q, want[0]) and torch.equal(sc, want[1])


# ---- together --------------------------------------------------------------------------------------------
def block(x, res, p):
    """A feed-forward block of experts in 8 bits between two norms, as a decoder of such layers runs it."""
    codes, scale, h, y = B.rms_norm_quant(x, p["norm"], residual=res, h=True, y=True)
    logits = B.matmul_i8(codes, scale, p["gate"], p["gate_scale"], out_dtype=F32)
    chosen, weights, offsets, rows, places = B.route_topk(logits, p["k"])
    up = B.matmul_grouped(codes, p["up"], offsets, rows, scale, p["up_scale"], relu=True)
    mid, mid_scale, _, _ = B.rms_norm_quant(up, eps=-1.0)
    down = B.matmul_grouped(mid, p["down"], offsets, None, mid_scale, p["down_scale"])
    codes, scale, out, _ = B.rms_norm_quant(down, p["norm2"], residual=h, rows=places, row_weights=weights, h=True)
    return dict(h=h, y=y, logits=logits, chosen=chosen, weights=weights, offsets=offsets, rows=rows, places=places, up=up, down=down, out=out, codes=codes,
                scale=scale)


def parameters(d, ffn, e, k):
    def quantised(*shape):
        w = randn(sum(shape), *shape, scale=0.05).to(BF16)
        q, s, _, _ = B.rms_norm_quant(w.view(-1, shape[-1]), eps=-1.0)
        return q.view(shape), s.view(shape[:-1])
    p = dict(norm=(1 + randn(1, d, scale=0.2)).to(BF16), norm2=(1 + randn(2, d, scale=0.2)).to(BF16), k=k)
    p["gate"], p["gate_scale"] = quantised(e, d)
    p["up"], p["up_scale"] = quantised(e, ffn, d)
    p["down"], p["down_scale"] = quantised(e, d, ffn)
    return p


@pytest.mark.parametrize("T,d,ffn,e,k", [(1, 512, 768, 8, 2), (19, 768, 1040, 16, 4), (333, 512, 512, 5, 2)])
def test_block_of_experts(T, d, ffn, e, k):
    p = parameters(d, ffn, e, k)
    x, res = randn(11, T, d, dtype=BF16), randn(12, T, d, dtype=BF16, scale=3.0)
    r = block(x, res, p)
    # each stage against the definition, fed what the stage before it left
    verify_norm(*B.rms_norm_quant(x, p["norm"], residual=res, h=True, y=True), *R.summed(x, res), 2, BF16, p["norm"], 1e-6)
    codes, scale, _, _ = B.rms_norm_quant(x, p["norm"], residual=res)
    check_product(r["logits"], codes, p["gate"], F32, scale, p["gate_scale"])
    assert r["chosen"].tolist() == R.route(r["logits"], k, True)[0]
    counts = (r["offsets"][1:] - r["offsets"][:-1]).tolist()
    check_grouped(r["up"], codes, p["up"], counts, r["rows"], BF16, xs=scale, ws=p["up_scale"], relu=True)
    mid, ms, _, _ = B.rms_norm_quant(r["up"], eps=-1.0)
    check_grouped(r["down"], mid, p["down"], counts, None, BF16, xs=ms, ws=p["down_scale"])
    wh, size = R.summed(r["down"], r["h"], r["places"], r["weights"])
    check(r["out"], wh, (k + 2) * E * size + R.half_step(BF16) * wh.abs() + 1e-40)


@pytest.mark.parametrize("T", [13, 150])
def test_block_of_a_padded_batch(T):
    """Rows of padding visit no expert and change nobody's result."""
    p = parameters(512, 768, 8, 2)
    x, res = randn(41, T, 512, dtype=BF16), randn(42, T, 512, dtype=BF16)
    real = torch.arange(T, device=DEV) % 3 != 1
    pos = torch.where(real, torch.arange(T, device=DEV), -1).int()

    def run(x, res, pos):
        codes, scale, h, _ = B.rms_norm_quant(x, p["norm"], residual=res, h=True)
        logits = B.matmul_i8(codes, scale, p["gate"], p["gate_scale"], out_dtype=F32)
        _, weights, offsets, rows, places = B.route_topk(logits, 2, positions=pos)
        up = B.matmul_grouped(codes, p["up"], offsets, rows, scale, p["up_scale"], relu=True)
        mid, mid_scale, _, _ = B.rms_norm_quant(up, eps=-1.0)
        down = B.matmul_grouped(mid, p["down"], offsets, None, mid_scale, p["down_scale"])
        return B.rms_norm_quant(down, p["norm2"], residual=h, rows=places, row_weights=weights, h=True), h

    (q, s, h, _), first = run(x, res, pos)
    (wq, ws, wh, _), _ = run(x[real], res[real], None)
    assert torch.equal(q[real], wq) and torch.equal(s[real], ws) and torch.equal(h[real], wh)
    assert torch.equal(h[~real], first[~real])                     # padding: the residual alone


def test_block_in_graphs_that_run_at_once():
    p = parameters(512, 768, 8, 2)
    xs, rs = [randn(20 + i, 77, 512, dtype=BF16) for i in range(2)], [randn(30 + i, 77, 512, dtype=BF16) for i in range(2)]
    want = [block(x, r, p) for x, r in zip(xs, rs)]
    torch.cuda.synchronize()
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], []
    for s, x, r in zip(streams, xs, rs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            with torch.cuda.graph(g, stream=s):
                outs.append(block(x, r, p))
        graphs.append(g)
    for _ in range(3):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for a, b in zip(outs, want):
        for name in b:
            assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("polls", [0, 1])
def test_waits_that_run_out(polls):
    x, w = whole(1, -9, 9, 300, 4096), whole(2, -9, 9, 600, 4096)
    want = {m: B.matmul_i8(x[:m], None, w, None, out_dtype=F32) for m in (2, 50, 300)}
    torch.cuda.synchronize()
    for m in want:
        B.debug_wait_limit(polls)
        try:
            got = B.matmul_i8(x[:m], None, w, None, out_dtype=F32)
            torch.cuda.synchronize()
        finally:
            B.debug_wait_limit(-1)
        bad = torch.isnan(got)
        assert torch.equal(got[~bad], want[m][~bad])               # a value is right or it is NaN
        assert polls > 0 or bool(bad.all())
        assert torch.equal(B.matmul_i8(x[:m], None, w, None, out_dtype=F32), want[m])
