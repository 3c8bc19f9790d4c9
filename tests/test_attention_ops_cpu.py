"""What the attention operators refuse, on the host and before any launch, and their sizes."""
import ctypes as C
import subprocess
import sys

import pytest
import torch

from paper_2310_11453_b200 import binding as B
from paper_2310_11453_b200 import build as bl_build

P = 1 << 20                                     # an aligned address that is never read: every call here is refused or empty


@pytest.fixture(scope="module", autouse=True)
def built():
    bl_build.build()


def cache(**kw):
    f = dict(pages=P, num_pages=8, page_size=16, kv_heads=2, head_dim=64, dtype=B.F16)
    f.update(kw)
    return C.byref(B._Kv4CacheStruct(f["pages"], f["num_pages"], f["page_size"], f["kv_heads"], f["head_dim"], f["dtype"]))


def norm_rope(**kw):
    f = dict(q=P, k=P, dt=B.F16, T=4, heads=4, kv_heads=2, head_dim=64, ld_q=256, ld_k=128, wq=None, wk=None, eps=1e-6,
             rot=64, inter=0, inv_freq=P, positions=P, q_out=P, k_out=P, ld_qo=256, ld_ko=128)
    f.update(kw)
    return B.lib().bitlinear_qk_norm_rope(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=7), B.ERR_UNSUPPORTED), (dict(T=-1), B.ERR_SHAPE), (dict(T=1 << 40), B.ERR_SHAPE), (dict(heads=0), B.ERR_SHAPE),
    (dict(kv_heads=0), B.ERR_SHAPE), (dict(head_dim=24), B.ERR_SHAPE), (dict(head_dim=272), B.ERR_SHAPE),
    (dict(rot=24), B.ERR_SHAPE), (dict(rot=80), B.ERR_SHAPE), (dict(rot=-16), B.ERR_SHAPE), (dict(ld_q=248), B.ERR_SHAPE),
    (dict(ld_q=260), B.ERR_SHAPE), (dict(ld_k=120), B.ERR_SHAPE), (dict(ld_qo=260), B.ERR_SHAPE), (dict(ld_ko=64), B.ERR_SHAPE),
    (dict(q=None), B.ERR_NULL), (dict(k=None), B.ERR_NULL), (dict(positions=None), B.ERR_NULL), (dict(inv_freq=None), B.ERR_NULL),
    (dict(q_out=None), B.ERR_NULL), (dict(q=P + 8), B.ERR_ALIGN), (dict(wq=P + 2), B.ERR_ALIGN), (dict(positions=P + 2), B.ERR_ALIGN),
    (dict(q_out=P, ld_qo=264), B.ERR_SHAPE), (dict(T=0, q=None), B.OK)])
def test_norm_rope_refusals(kw, code):
    assert norm_rope(**kw) == code


def window(**kw):
    f = dict(q=P, k=P, v=P, o=P, dt=B.F16, batch=2, cu_q=None, cu_k=None, seq_q=16, seq_k=16, rows_q=32, rows_k=32, heads=4,
             kv_heads=2, head_dim=64, ld_q=256, ld_k=128, ld_v=128, ld_o=256, window=0, sinks=0, scale=0.0)
    f.update(kw)
    return B.lib().bitlinear_attention_window(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(dt=B.F32), B.ERR_UNSUPPORTED), (dict(head_dim=96), B.ERR_UNSUPPORTED), (dict(batch=-1), B.ERR_SHAPE),
    (dict(seq_q=-1), B.ERR_SHAPE), (dict(seq_q=1 << 31, rows_q=1 << 33), B.ERR_SHAPE), (dict(kv_heads=3), B.ERR_SHAPE),
    (dict(sinks=-1), B.ERR_SHAPE), (dict(scale=-1.0), B.ERR_SHAPE), (dict(scale=float("nan")), B.ERR_SHAPE),
    (dict(scale=float("inf")), B.ERR_SHAPE), (dict(cu_k=P), B.ERR_NULL), (dict(rows_q=31), B.ERR_SHAPE), (dict(rows_k=31), B.ERR_SHAPE),
    (dict(ld_q=252), B.ERR_SHAPE), (dict(ld_v=132), B.ERR_SHAPE), (dict(q=None), B.ERR_NULL), (dict(v=None), B.ERR_NULL),
    (dict(o=P + 8), B.ERR_ALIGN), (dict(cu_q=P + 2), B.ERR_ALIGN), (dict(batch=0, q=None), B.OK), (dict(seq_q=0, q=None), B.OK)])
def test_window_refusals(kw, code):
    assert window(**kw) == code


BAD_CACHES = [(dict(dtype=B.F32), B.ERR_UNSUPPORTED), (dict(head_dim=80), B.ERR_UNSUPPORTED), (dict(page_size=24), B.ERR_SHAPE),
              (dict(page_size=128), B.ERR_SHAPE), (dict(kv_heads=0), B.ERR_SHAPE), (dict(num_pages=-1), B.ERR_SHAPE),
              (dict(pages=None), B.ERR_NULL), (dict(pages=P + 8), B.ERR_ALIGN)]


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches_that_are_refused(kw, code):
    L = B.lib()
    assert L.bitlinear_kv4_append(cache(**kw), P, P, 4, 256, 256, P, None) == code
    assert L.bitlinear_kv4_read(cache(**kw), P, P, 4, 256, 256, P, None) == code
    assert L.bitlinear_attention_kv4(P, 2, 1, 4, 320, cache(**kw), P, 4, P, 0, 0, 0.0, P, 320, P, 1 << 30, None) == code


@pytest.mark.parametrize("name", ["append", "read"])
@pytest.mark.parametrize("args,code", [
    ((P, P, -1, 128, 128, P), B.ERR_SHAPE), ((P, P, 1 << 40, 128, 128, P), B.ERR_SHAPE), ((P, P, 4, 120, 128, P), B.ERR_SHAPE),
    ((P, P, 4, 128, 132, P), B.ERR_SHAPE), ((None, P, 4, 128, 128, P), B.ERR_NULL), ((P, None, 4, 128, 128, P), B.ERR_NULL),
    ((P, P, 4, 128, 128, None), B.ERR_NULL), ((P + 8, P, 4, 128, 128, P), B.ERR_ALIGN), ((P, P, 4, 128, 128, P + 4), B.ERR_ALIGN),
    ((None, None, 0, 128, 128, None), B.OK)])
def test_append_and_read_refusals(name, args, code):
    L = B.lib()
    fn = L.bitlinear_kv4_append if name == "append" else L.bitlinear_kv4_read
    assert fn(cache(), *args, None) == code
    assert fn(None, *args, None) == B.ERR_NULL


def kv4(**kw):
    f = dict(q=P, batch=2, n_q=1, heads=4, ld_q=256, cache=cache(), table=P, max_pages=4, lens=P, window=0, sinks=0, scale=0.0, o=P,
             ld_o=256, ws=P, ws_bytes=1 << 40)
    f.update(kw)
    return B.lib().bitlinear_attention_kv4(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(cache=None), B.ERR_NULL), (dict(batch=-1), B.ERR_SHAPE), (dict(n_q=0), B.ERR_SHAPE), (dict(heads=3), B.ERR_SHAPE),
    (dict(heads=0), B.ERR_SHAPE), (dict(sinks=-1), B.ERR_SHAPE), (dict(max_pages=-1), B.ERR_SHAPE), (dict(max_pages=1 << 62), B.ERR_SHAPE),
    (dict(scale=-0.5), B.ERR_SHAPE), (dict(ld_q=128), B.ERR_SHAPE), (dict(ld_o=260), B.ERR_SHAPE), (dict(q=None), B.ERR_NULL),
    (dict(lens=None), B.ERR_NULL), (dict(table=None), B.ERR_NULL), (dict(o=P + 4), B.ERR_ALIGN), (dict(table=P + 2), B.ERR_ALIGN),
    (dict(ws=None), B.ERR_WORKSPACE), (dict(ws_bytes=16), B.ERR_WORKSPACE), (dict(ws=P + 4), B.ERR_ALIGN), (dict(batch=0, q=None), B.OK)])
def test_attention_kv4_refusals(kw, code):
    assert kv4(**kw) == code


@pytest.mark.parametrize("args,code", [
    ((P, 0, 8, 1, 0, P, 1), B.ERR_SHAPE), ((P, 24, 8, 1, 0, P, 1), B.ERR_SHAPE), ((P, 64, -1, 1, 0, P, 1), B.ERR_SHAPE),
    ((P, 64, 8, -1, 512, P, 1), B.ERR_SHAPE), ((P, 64, 8, 2, 256, P, 1), B.ERR_SHAPE), ((P, 64, 8, 2, 520, P, 1), B.ERR_SHAPE),
    ((P, 64, 8, 1, 0, P, -1), B.ERR_SHAPE), ((P, 1 << 30, 8, 1, 0, P, 1 << 30), B.ERR_SHAPE), ((None, 64, 8, 1, 0, P, 1), B.ERR_NULL),
    ((P, 64, 8, 1, 0, None, 1), B.ERR_NULL), ((P + 8, 64, 8, 1, 0, P, 1), B.ERR_ALIGN), ((P, 64, 8, 1, 0, P + 4, 1), B.ERR_ALIGN),
    ((None, 64, 8, 1, 0, None, 0), B.OK)])
def test_copy_pages_refusals(args, code):
    assert B.lib().bitlinear_kv4_copy_pages(*args, None) == code


def test_sizes():
    assert B.kv4_page_bytes(64, 8, 128) == 64 * 8 * 136
    assert B.kv4_page_bytes(16, 1, 64) == 16 * 72
    for bad in ((8, 1, 64), (128, 1, 64), (48, 1, 64), (16, 0, 64), (16, 1, 96)):
        assert B.kv4_page_bytes(*bad) == 0
    assert B.attention_kv4_ws_bytes(4, 1, 32, 8, 128) > 0
    for bad in ((-1, 1, 8, 8, 128), (1, 0, 8, 8, 128), (1, 1, 8, 3, 128), (1, 1, 8, 8, 96)):
        assert B.attention_kv4_ws_bytes(*bad) == 0


def test_the_binding_refuses_host_tensors_and_wrong_types():
    x = torch.zeros((2, 64), dtype=torch.float16)
    pos = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        B.qk_norm_rope(x, x, pos, torch.zeros(8), 1, 1, 64)
    with pytest.raises(ValueError):
        B.attention_window(x, x, x, 1, 2, 1, head_dim=64)
    with pytest.raises(ValueError):
        B.kv4_copy_pages(torch.zeros((2, 64), dtype=torch.uint8), torch.zeros((1, 2), dtype=torch.int32))
    with pytest.raises(ValueError):
        B.Kv4Cache(torch.zeros((2, 16 * 72), dtype=torch.uint8), 16, 1, 64, torch.float16)
    with pytest.raises(TypeError):
        B.Kv4Cache(torch.zeros((2, 16 * 72), dtype=torch.uint8), 16, 1, 64, torch.float32)
    with pytest.raises(ValueError):
        B.Kv4Cache(torch.zeros((2, 16 * 72), dtype=torch.uint8), 20, 1, 64, torch.float16)


def test_layout_reference_is_a_bijection():
    from tests.attention_ref import value_place
    for dim in (64, 128):
        seen = {value_place(t, d, dim) for t in range(32) for d in range(dim)}
        assert len(seen) == 32 * dim and max(b for b, _ in seen) == 32 * dim // 2 - 1


def test_parts_named_by_any_bits_stay_within_the_workspace(tmp_path):
    """part_count of csrc/kv4.cuh, compiled for the host: what it lets pass lies within the warps' parts, whatever it is given."""
    from paper_2310_11453_b200.build import CSRC, NVCC
    src, exe = tmp_path / "parts.cu", tmp_path / "parts"
    src.write_text('#include <stdio.h>\n#include <stdlib.h>\n#include "kv4.cuh"\nint main(int n, char** v) {\n'
                   '  for (int i = 1; i + 2 < n; i += 3) printf("%d\\n", bl::kv4::part_count(atoi(v[i]), atoi(v[i + 1]), atoi(v[i + 2])));\n}\n')
    subprocess.run([NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    ends = (-2 ** 31, -2 ** 31 + 1, -10 ** 9, -1, 0, 1, 2, 3, 50, 1775, 1776, 3551, 3552, 10 ** 9, 2 ** 31 - 2, 2 ** 31 - 1)
    args = [(a, b, w) for a in ends for b in ends for w in (1, 64, 1776)]
    out = subprocess.run([str(exe)] + [str(x) for t in args for x in t], check=True, capture_output=True, text=True).stdout.split()
    for (first, last, warps), n in zip(args, map(int, out), strict=True):
        w0 = first // 2
        assert n == (last - w0 + 1 if 0 <= w0 <= last < warps else 0), (first, last, warps)


def test_workspace_sizes_that_do_not_fit_are_refused():
    """Sizes that attention_kv4 refuses have no workspace; sums and products of them may pass 32 bits.  In a process of its own: a
    division by a count of rows that wrapped around to 0 ends it."""
    sizes = [(1, 1 << 20, 4096, 1, 128), (0, 1 << 20, 4096, 1, 128), (1, 1 << 30, 4, 1, 64), (1, 2 ** 31 - 1, 1, 1, 128), (1, 1, 8192, 1, 128),
             (2 ** 31 - 1, 1, 4096, 4096, 128), (1 << 20, 1 << 11, 1, 1, 64), (1, 1, 2 ** 31 - 1, 1, 64), (1, 5, 2 ** 30, 2, 64)]
    code = f"from paper_2310_11453_b200 import binding as B\nprint([B.attention_kv4_ws_bytes(*s) for s in {sizes}])"
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert done.returncode == 0, done
    assert done.stdout.strip() == str([0] * len(sizes))
    assert B.attention_kv4_ws_bytes(1, 1 << 18, 4096, 1, 128) > 0 and B.attention_kv4_ws_bytes(1 << 18, 1, 4096, 4096, 128) > 0


@pytest.mark.parametrize("scale", [2.5e38, 3.0e38, -0.0])
def test_scales_that_pass_fp32_in_the_exponent_are_refused(scale):
    """Scores are taken times log2(e): 2.4e38 and more would be an infinite factor, and NaN of a score of 0."""
    assert window(scale=scale, batch=0) == (B.ERR_SHAPE if scale > 0 else B.OK)
    assert kv4(scale=scale, batch=0) == (B.ERR_SHAPE if scale > 0 else B.OK)
    assert window(scale=2e38, batch=0) == B.OK and kv4(scale=2e38, batch=0) == B.OK


def test_norm_rope_refuses_an_eps_that_is_no_number():
    """A negative eps means no norm; NaN compares like one, and would leave the norm out in silence."""
    assert norm_rope(eps=float("nan"), T=0) == B.ERR_SHAPE
    for eps in (-1.0, 0.0, 1e-6, float("-inf")):
        assert norm_rope(eps=eps, T=0) == B.OK


def test_a_cache_object_cannot_be_pointed_elsewhere():
    """The calls use what the constructor checked: an assignment afterwards would be ignored by them, so it is refused."""
    cache = object.__new__(B.Kv4Cache)
    for name in ("pages", "page_size", "kv_heads", "head_dim", "dtype"):
        with pytest.raises(AttributeError):
            setattr(cache, name, 1)
