"""64-bit definitions of the attention operators, for the tests (bitlinear.h, "attention at inference")."""
import math

import torch


def visible(i, j, window, sinks):
    """[len(i), len(j)] truth values: position i sees position j."""
    i, j = i[:, None], j[None, :]
    near = (i - j < window) if window > 0 else torch.ones_like(i - j, dtype=torch.bool)
    return (j <= i) & (i >= 0) & (near | (j < sinks))


def attend(q, k, v, seen, scale):
    """q [n, D], k, v [m, D], all of one head, 64 bits.  Returns (o [n, D], probabilities [n, m]); a query that sees
    nothing gets zeros, and values at places that are not seen do not enter."""
    z = torch.where(seen, q @ torch.nan_to_num(k, nan=0.0, posinf=0.0, neginf=0.0).t() * scale, torch.full_like(seen, -math.inf, dtype=q.dtype))
    top = z.amax(-1, keepdim=True) if z.shape[1] else torch.zeros((z.shape[0], 1), dtype=q.dtype, device=q.device)
    p = torch.exp(z - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-300)
    return p @ torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0), p


def half_step(dtype):
    """Largest relative error of one rounding."""
    return torch.finfo(dtype).eps / 2


def norm_rope(x, w, pos, inv_freq, head_dim, eps, interleaved):
    """x [T, heads * head_dim].  Returns (y, size of the values a rotation mixes, |turns|), 64 bits, x's shape."""
    T = x.shape[0]
    v = x.double().reshape(T, -1, head_dim)
    if eps >= 0:
        v = v / (v.pow(2).mean(-1, keepdim=True) + eps).sqrt()
        if w is not None:
            v = v * w.double()
    half = inv_freq.numel()
    t = (pos.double()[:, None] * inv_freq.double())[:, None]
    a = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    b = a + (1 if interleaved else half)
    y, size, turns = v.clone(), v.abs(), torch.zeros_like(v)
    y[..., a] = v[..., a] * t.cos() - v[..., b] * t.sin()
    y[..., b] = v[..., b] * t.cos() + v[..., a] * t.sin()
    size[..., a] = size[..., b] = v[..., a].abs() + v[..., b].abs()
    turns[..., a] = turns[..., b] = (t / (2 * math.pi)).abs().expand(T, v.shape[1], half)
    return y.reshape(T, -1), size.reshape(T, -1), turns.reshape(T, -1)


def quantise(x):
    """Rows x [..., D].  Returns codes (int64), step and eta [..., 1] of x's dtype (NaN where a row is not finite)."""
    w = x.double()
    fine = torch.isfinite(w).all(-1, keepdim=True)
    w = torch.where(fine, w, torch.zeros_like(w))
    lo, hi = w.amin(-1, keepdim=True), w.amax(-1, keepdim=True)
    step = ((hi - lo) / 15).to(x.dtype)
    s = step.double()
    codes = torch.where(s > 0, torch.round((w - lo) / torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(w))
    nan = torch.full_like(step, math.nan)
    return codes.clamp(0, 15).long(), torch.where(fine, step, nan), torch.where(fine, lo.to(x.dtype), nan)


def value_place(t, d, head_dim):
    """(byte, shift) of value code d of token t within a head's value codes, from the header's index formula."""
    eighth, e = d // (head_dim // 8), d % (head_dim // 8)
    word, half = e // 4, t % 2
    sizes = (8, 4, head_dim // 32, 2, 2)
    at = t // 8
    for n, i in zip(sizes, (eighth, t % 8 // 2, word, half, e % 4 // 2)):
        at = at * n + i
    return at, 4 * (e % 2)


def decode_pages(pages, page_size, kv_heads, head_dim, dtype):
    """Every token of the cache: (key codes, value codes [pages, page_size, heads, D] int64, and their (step, eta)
    [pages, page_size, heads, 2] of dtype), following the header."""
    P = pages.shape[0]
    blocks = pages.reshape(P, kv_heads, page_size * (head_dim + 8)).cpu()
    n = page_size * head_dim // 2
    kb = blocks[:, :, :n].reshape(P, kv_heads, page_size, head_dim // 2).long()
    k = torch.stack((kb & 15, kb >> 4), -1).flatten(-2)
    vb = blocks[:, :, n:2 * n].long()
    place = torch.tensor([[value_place(t, d, head_dim) for d in range(head_dim)] for t in range(page_size)])
    v = (vb[:, :, place[..., 0]] >> place[..., 1]) & 15
    ks = blocks[:, :, 2 * n:2 * n + 4 * page_size].contiguous().view(dtype).reshape(P, kv_heads, page_size, 2)
    vs = blocks[:, :, 2 * n + 4 * page_size:].contiguous().view(dtype).reshape(P, kv_heads, page_size, 2)
    return tuple(x.transpose(1, 2) for x in (k, v, ks, vs))
