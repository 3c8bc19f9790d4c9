"""What the 8-bit layers and the expert operators refuse, on the host and before any launch, and their sizes."""
import pytest
import torch

from paper_2310_11453_b200 import binding as B
from paper_2310_11453_b200 import build as bl_build

P = 1 << 20                                     # an aligned address that is never read: every call here is refused or empty


@pytest.fixture(scope="module", autouse=True)
def built():
    bl_build.build()


def norm(**kw):
    f = dict(x=P, dt=B.BF16, x_rows=4, T=4, K=64, ld_x=64, rows=None, row_weights=None, top_k=0, residual=P + 4096, ld_res=64, weight=P,
             eps=1e-6, h=P + 8192, ld_h=64, y=None, ld_y=0, x_q=P, ld_q=64, scale=P)
    f.update(kw)
    return B.lib().bitlinear_rms_norm_quant(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=B.I8), B.ERR_UNSUPPORTED), (dict(dt=9), B.ERR_UNSUPPORTED), (dict(T=-1), B.ERR_SHAPE), (dict(T=5), B.ERR_SHAPE),
    (dict(T=1 << 40, x_rows=1 << 40), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE), (dict(K=60), B.ERR_SHAPE),
    (dict(K=32776, ld_x=32776), B.ERR_SHAPE), (dict(eps=float("nan")), B.ERR_SHAPE), (dict(ld_x=56), B.ERR_SHAPE),
    (dict(ld_x=68), B.ERR_SHAPE), (dict(ld_res=60), B.ERR_SHAPE), (dict(ld_h=68), B.ERR_SHAPE), (dict(y=P, ld_y=56), B.ERR_SHAPE),
    (dict(ld_q=68), B.ERR_SHAPE), (dict(ld_x=1 << 60), B.ERR_SHAPE), (dict(rows=P, top_k=0), B.ERR_SHAPE), (dict(rows=P, top_k=65), B.ERR_SHAPE),
    (dict(row_weights=P), B.ERR_NULL), (dict(x=None), B.ERR_NULL), (dict(h=None, x_q=None), B.ERR_NULL), (dict(scale=None), B.ERR_NULL),
    (dict(x=P + 8), B.ERR_ALIGN), (dict(residual=P + 2), B.ERR_ALIGN), (dict(weight=P + 8), B.ERR_ALIGN), (dict(h=P + 8), B.ERR_ALIGN),
    (dict(x_q=P + 4), B.ERR_ALIGN), (dict(scale=P + 2), B.ERR_ALIGN), (dict(rows=P + 2, top_k=2), B.ERR_ALIGN),
    (dict(h=P + 4096, ld_h=72), B.ERR_SHAPE), (dict(h=P, ld_h=72), B.ERR_SHAPE), (dict(h=P, rows=P, top_k=2), B.ERR_SHAPE),
    (dict(T=0, x=None), B.OK)])
def test_norm_refusals(kw, code):
    assert norm(**kw) == code


def matmul(**kw):
    f = dict(x=P, M=4, K=64, N=10, ld_x=64, xs=P, w=P, ld_w=64, ws=P, bias=None, relu=0, residual=None, ld_res=0, y=P, yt=B.BF16, ld_y=10)
    f.update(kw)
    return B.lib().bitlinear_matmul_i8(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(yt=B.I8), B.ERR_UNSUPPORTED), (dict(M=-1), B.ERR_SHAPE), (dict(M=1 << 40), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE), (dict(K=56), B.ERR_SHAPE),
    (dict(K=131072, ld_x=131072, ld_w=131072), B.ERR_SHAPE), (dict(N=0), B.ERR_SHAPE), (dict(N=1 << 25, ld_y=1 << 25), B.ERR_SHAPE),
    (dict(ld_x=48), B.ERR_SHAPE), (dict(ld_x=72), B.ERR_SHAPE), (dict(ld_w=72), B.ERR_SHAPE), (dict(ld_w=1 << 60), B.ERR_SHAPE),
    (dict(ld_y=9), B.ERR_SHAPE), (dict(residual=P, ld_res=9), B.ERR_SHAPE), (dict(residual=P, ld_res=12), B.ERR_SHAPE),
    (dict(x=None), B.ERR_NULL), (dict(w=None), B.ERR_NULL), (dict(y=None), B.ERR_NULL), (dict(x=P + 8), B.ERR_ALIGN), (dict(w=P + 8), B.ERR_ALIGN),
    (dict(y=P + 1), B.ERR_ALIGN), (dict(yt=B.F32, y=P + 2), B.ERR_ALIGN), (dict(bias=P + 1), B.ERR_ALIGN), (dict(xs=P + 2), B.ERR_ALIGN),
    (dict(M=0, x=None), B.OK)])
def test_matmul_refusals(kw, code):
    assert matmul(**kw) == code


def route(**kw):
    f = dict(z=P, dt=B.F32, T=4, E=8, ld=8, k=2, normalise=1, positions=None, chosen=P, weights=P, offsets=P, rows=P, places=P, ws=None, ws_bytes=0)
    f.update(kw)
    return B.lib().bitlinear_route_topk(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=B.I8), B.ERR_UNSUPPORTED), (dict(T=-1), B.ERR_SHAPE), (dict(T=1 << 30), B.ERR_SHAPE), (dict(E=0), B.ERR_SHAPE),
    (dict(E=513, ld=513), B.ERR_SHAPE), (dict(k=0), B.ERR_SHAPE), (dict(k=9), B.ERR_SHAPE), (dict(k=33, E=64, ld=64), B.ERR_SHAPE),
    (dict(ld=7), B.ERR_SHAPE), (dict(z=None), B.ERR_NULL), (dict(chosen=None), B.ERR_NULL), (dict(weights=None), B.ERR_NULL),
    (dict(offsets=None), B.ERR_NULL), (dict(rows=None), B.ERR_NULL), (dict(places=None), B.ERR_NULL), (dict(z=P + 2), B.ERR_ALIGN),
    (dict(dt=B.F16, z=P + 1), B.ERR_ALIGN), (dict(offsets=P + 2), B.ERR_ALIGN), (dict(T=65), B.ERR_WORKSPACE),
    (dict(T=65, ws=P, ws_bytes=64), B.ERR_WORKSPACE), (dict(T=65, ws=P + 8, ws_bytes=1 << 20), B.ERR_ALIGN)])
def test_route_refusals(kw, code):
    assert route(**kw) == code


def test_route_workspace():
    assert B.route_topk_ws_bytes(64, 512) == 0 and B.route_topk_ws_bytes(0, 8) == 0
    assert B.route_topk_ws_bytes(-1, 8) == 0 and B.route_topk_ws_bytes(100, 0) == 0 and B.route_topk_ws_bytes(100, 513) == 0
    for T, E in [(65, 1), (8191, 128), (1 << 20, 511)]:
        runs = -(-T // 64)
        need = B.route_topk_ws_bytes(T, E)
        assert need % 256 == 0 and need >= runs * E * 9 + (4 * (runs + 1) * E if runs > 512 else 0)


def grouped(**kw):
    f = dict(x=P, operand=B.I8, x_rows=8, K=64, N=10, ld_x=64, xs=P, w=P, ld_w=64, stride=640, ws=P, E=3, offsets=P, rows=P, R=8, bias=None,
             relu=0, y=P, yt=B.BF16, ld_y=10)
    f.update(kw)
    return B.lib().bitlinear_matmul_grouped(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(operand=B.F32), B.ERR_UNSUPPORTED), (dict(operand=B.BF16), B.ERR_UNSUPPORTED), (dict(yt=B.I8), B.ERR_UNSUPPORTED),
    (dict(R=-1), B.ERR_SHAPE), (dict(E=0), B.ERR_SHAPE), (dict(E=1025), B.ERR_SHAPE), (dict(x_rows=0), B.ERR_SHAPE),
    (dict(x_rows=7, rows=None), B.ERR_SHAPE), (dict(K=56), B.ERR_SHAPE), (dict(stride=632), B.ERR_SHAPE), (dict(stride=576), B.ERR_SHAPE),
    (dict(stride=656), B.ERR_SHAPE), (dict(stride=1 << 60), B.ERR_SHAPE), (dict(ld_w=56), B.ERR_SHAPE), (dict(ld_y=8), B.ERR_SHAPE),
    (dict(x=None), B.ERR_NULL), (dict(w=None), B.ERR_NULL), (dict(offsets=None), B.ERR_NULL), (dict(y=None), B.ERR_NULL),
    (dict(x=P + 8), B.ERR_ALIGN), (dict(offsets=P + 2), B.ERR_ALIGN), (dict(rows=P + 2), B.ERR_ALIGN), (dict(ws=P + 2), B.ERR_ALIGN),
    (dict(R=0, rows=None, x=None), B.OK)])
def test_grouped_refusals(kw, code):
    assert grouped(**kw) == code


def test_binding_refuses_what_is_not_on_a_gpu():
    x, s = torch.zeros((4, 64), dtype=torch.int8), torch.ones(4)
    with pytest.raises(ValueError):
        B.rms_norm_quant(torch.zeros(4, 64))
    with pytest.raises(ValueError):
        B.matmul_i8(x, s, x, s)
    with pytest.raises(ValueError):
        B.route_topk(torch.zeros(4, 8), 2)
    with pytest.raises(ValueError):
        B.matmul_grouped(x, x.view(1, 4, 64), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        B.matmul_i8(None, s, x, s)
