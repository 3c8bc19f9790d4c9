"""Calls of the 8-bit layers that the ordinary ranges do not reach.

Tolerances as in test_gpu_layers8: e = 2^-24 is one rounding of fp32, u(T) = eps(T) / 2 one to T.  Scaling by powers of two is exact, so
rows that leave the range have those of the others: the sum h 2 e of its terms, the norm's factor 40 e with the products, one rounding on
output.  Where an output is below the smallest normal number of its type the rounding is half of the smallest denormal one (bf16:
2^-134, under 1e-40; fp32: 2^-150, with one more for the factor, under 1e-44)."""

import pytest
import torch

from paper_2310_11453_b200 import binding as B
from tests import layers8_ref as R
from tests.test_gpu_layers8 import BF16, DEV, E, F32, check, lists, randn, whole

pytestmark = pytest.mark.gpu
LEAST = {BF16: 1e-40, F32: 1e-44}


# ---- norm: weights and values at the ends of the range -------------------------------------------------
def check_range(x, weight, eps, rows=None, row_weights=None):
    """y, scale and codes of rows without cancellation (one term, or terms of one sign)."""
    dt = x.dtype
    codes, scale, h, y = B.rms_norm_quant(x, weight, eps, rows=rows, row_weights=row_weights, h=True, y=True)
    wh, _ = R.summed(x, None, rows, row_weights)
    n = 2 + (rows.shape[1] if rows is not None else 0)
    want = R.normed(wh, weight, eps)
    near = (40 + 2 * n) * E
    check(y, want, (near + R.half_step(dt)) * want.abs() + LEAST[dt], "y")
    top = want.abs().amax(-1)
    check(scale, top / 127, (near + 4 * E) * top / 127 + 1e-44, "scale")
    v = torch.where(top[:, None] > 0, want / top[:, None].clamp(min=1e-300) * 127, torch.zeros_like(want))
    slack = 2.0 ** -13 + 127 * 2 * n * E
    worst = float(((codes.double() - v).abs() - 0.5 - slack).max())
    assert worst <= 0, f"codes: {worst} beyond half a step"


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("T,K", [(5, 1024), (200, 1024), (3, 16392)])
@pytest.mark.parametrize("weight", [1e-32, 1e-35, 1e-37, 1e30])
@pytest.mark.parametrize("size", [1.0, 1e-10, 1e-25, 3e5, 1e25])
def test_norm_of_weights_at_the_ends_of_the_range(dt, T, K, weight, size):
    x = randn(K, T, K, scale=size).to(dt)
    w = ((1 + 0.2 * randn(3, K)) * weight).to(dt)
    for eps in (0.0, 1e-6):
        check_range(x, w, eps)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_norm_of_a_value_that_dwarfs_the_others(dt):
    """A weight of 0 hides the largest value from the codes, which are those of the others whatever it takes to hold its square."""
    K = 1024
    x = randn(1, 6, K)
    x[:, 17] = torch.tensor([1e38, -3e38, 1e30, 1e20, 3e19, 2.0], device=DEV)
    x, w = x.to(dt), (1 + 0.2 * randn(2, K)).to(dt)
    w[17] = 0
    check_range(x, w, 0.0)
    check_range(x, w, 1e-6)
    w2 = w.clone()                                                 # and weights that bring the others back
    w2[torch.arange(K, device=DEV) != 17] *= 1e30
    check_range(x, w2, 1e-6)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_norm_of_summed_rows_at_the_ends_of_the_range(dt):
    K, T = 1024, 7
    rows = whole(1, 0, 11, T, 2, dtype=torch.int32)
    p = torch.softmax(randn(2, T, 2), -1)
    for size, weight in ((1.0, 1e-33), (1e-20, 1e-30), (1e-30, 1.0), (1e25, 1.0), (1e30, 1e-20), (1e30, 1e20)):
        x = (randn(3, 12, K).abs() * size).to(dt)
        check_range(x, ((1 + 0.2 * randn(4, K)) * weight).to(dt), 1e-6, rows, p)
        check_range(x, ((1 + 0.2 * randn(4, K)) * weight).to(dt), 0.0, rows, p)


# ---- weights written just before they are used --------------------------------------------------------------
@pytest.mark.parametrize("M", [1, 40, 300])
@pytest.mark.parametrize("eps", [-1.0, 1e-6])
def test_weights_written_by_the_kernel_before(M, eps):
    """Whatever writes the weights on the stream, a norm that lets its successor start early included, the product sees what it wrote."""
    N, K = 4096, 2048
    x, xs = whole(1, -127, 127, M, K), torch.ones(M, device=DEV)
    latent = [randn(i, N, K, dtype=BF16) for i in range(6)]
    want = []
    for w in latent:
        q, s, _, _ = B.rms_norm_quant(w, eps=eps)
        torch.cuda.synchronize()
        want.append(B.matmul_i8(x, xs, q, s, out_dtype=F32))
    q, s = torch.empty((N, K), dtype=torch.int8, device=DEV), torch.empty(N, device=DEV)

    def run():
        got = []
        for w in latent:                                           # the same buffer again and again
            B.rms_norm_quant(w, eps=eps, x_q=q, scale=s)
            got.append(B.matmul_i8(x, xs, q, s, out_dtype=F32))
        for w in latent:                                           # the product before is still running when this one's weights are written
            B.matmul_i8(x, xs, q, s, out_dtype=F32)
            B.rms_norm_quant(w, eps=eps, x_q=q, scale=s)
            got.append(B.matmul_i8(x, xs, q, s, out_dtype=F32))
        return got
    for _ in range(3):
        for a, b in zip(run(), want + want):
            assert torch.equal(a, b)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = run()
    for _ in range(3):
        q.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want + want):
            assert torch.equal(a, b)


# ---- waits that run out ---------------------------------------------------------------------------------------
def limited(polls, call):
    B.debug_wait_limit(polls)
    try:
        return call()
    finally:
        B.debug_wait_limit(-1)


def right_or_nan(got, want):
    bad = torch.isnan(got)
    return torch.equal(got[~bad], want[~bad])


@pytest.mark.parametrize("polls", [1, 2, 5, 30])
@pytest.mark.parametrize("M,K,N,listed", [(2, 4096, 600, False), (50, 2048, 600, False), (50, 8192, 128, False), (300, 1024, 512, False), (300, 4096, 2048, False),
                                          (9, 1024, 600, True), (300, 2048, 1024, True)])
def test_copies_of_a_call_that_gave_up_do_not_reach_the_next(polls, M, K, N, listed):
    """A call whose waits run out leaves nothing on its way: calls right behind it, on the same SMs and the same shared memory, are right."""
    x, w = whole(1, -9, 9, M, K), whole(2, -9, 9, N, K)
    rows, offsets = whole(3, 0, M - 1, M, dtype=torch.int32), lists([M])
    y = torch.empty((M, N), device=DEV)

    def call(y):
        return B.matmul_grouped(x, w[None], offsets, rows, y=y) if listed else B.matmul_i8(x, None, w, None, y=y)
    want = call(torch.empty((M, N), device=DEV))
    z = randn(5, 100, 64)
    chosen = B.route_topk(z, 4)[0].clone()
    codes = B.rms_norm_quant(z)[0].clone()
    torch.cuda.synchronize()
    for _ in range(12):
        got = limited(polls, lambda: call(y))
        after = call(torch.empty((M, N), device=DEV))
        route, q = B.route_topk(z, 4)[0], B.rms_norm_quant(z)[0]
        assert torch.equal(after, want) and torch.equal(route, chosen) and torch.equal(q, codes)
        assert right_or_nan(got, want)


@pytest.mark.parametrize("polls", [1, 2, 4, 10, 30, 100])
@pytest.mark.parametrize("M,K,N,listed", [(4096, 256, 8192, False), (2500, 512, 4096, True), (64, 128, 120000, False), (40, 512, 100000, True)])
def test_waits_that_run_out_with_many_tiles_to_come(polls, M, K, N, listed):
    """Some warps give up while others still read their sums: every value is right or NaN, whichever tile it is of."""
    x, w = whole(1, -9, 9, M, K), whole(2, -9, 9, N, K)
    rows, offsets = whole(3, 0, M - 1, M, dtype=torch.int32), lists([M])

    def call():
        return B.matmul_grouped(x, w[None], offsets, rows, out_dtype=F32) if listed else B.matmul_i8(x, None, w, None, out_dtype=F32)
    want = call()
    torch.cuda.synchronize()
    for _ in range(4):
        assert right_or_nan(limited(polls, call), want)
        assert torch.equal(call(), want)


# ---- offsets that decrease ------------------------------------------------------------------------------------
@pytest.mark.parametrize("values", [[0, 300, 5, 700, 2, 900, 900, 20], [900, 0, 900, 0, 900, 0, 900, 0], [5, 4, 3, 2, 1, 0, -1, -2], [-9, 40, 30, 41, 2000, 50, 60, 70],
                                    [100, 130, 120, 135, 10, 139, 140, 139]])
@pytest.mark.parametrize("R_", [900, 140])
@pytest.mark.parametrize("listed", [True, False])
def test_offsets_that_decrease_give_each_row_to_its_owner(values, R_, listed):
    """An offset is cut to 0..R, and one below an offset before it counts as that one: so each row has at most one owner."""
    e, K, N = 7, 64, 300
    x, w = whole(1, -9, 9, R_, K), whole(2, -9, 9, e, N, K)
    rows = whole(3, 0, R_ - 1, R_, dtype=torch.int32) if listed else None
    y = torch.full((R_ + 2, N), 9.25, device=DEV)
    B.matmul_grouped(x, w, torch.tensor(values, dtype=torch.int32, device=DEV), rows, y=y[1:-1])
    want, reached = torch.full((R_ + 2, N), 9.25, device=DEV, dtype=torch.float64), 0
    source = x.double() if rows is None else x.double()[rows.long()]
    for i in range(e):
        first = max(reached, min(max(values[i], 0), R_))
        reached = max(first, min(max(values[i + 1], 0), R_))
        want[1 + first:1 + reached] = source[first:reached] @ w[i].double().t()
    assert torch.equal(y.double(), want)


# ---- what outputs keep alive ----------------------------------------------------------------------------------
def test_outputs_keep_little_more_than_themselves_alive():
    """New outputs may share a storage, of 1 MiB at most: a scale kept does not keep a matrix of codes."""
    def bytes_of(t):
        return t.untyped_storage().nbytes()
    for T, K in ((4096, 2048), (64, 16384), (3, 64)):
        q, s, _, _ = B.rms_norm_quant(randn(1, T, K, dtype=BF16), eps=-1.0)
        assert bytes_of(q) <= max(1 << 20, q.numel()) and bytes_of(s) <= max(1 << 20, 4 * T)
    for T, e, k in ((40000, 64, 8), (20, 8, 2)):
        out = B.route_topk(randn(1, T, e), k)
        assert all(bytes_of(t) <= max(1 << 20, 4 * t.numel()) for t in out)
