"""Definitions of the 8-bit layers and of the choice of experts, in 64 bits and row by row where order matters."""
import torch


def half_step(t):
    """A rounding to t, relative to the value."""
    return torch.finfo(t).eps / 2


def summed(x, residual=None, rows=None, row_weights=None):
    """(h, sum of the sizes of its terms) of rms_norm_quant."""
    if rows is None:
        h, size = x.double(), x.double().abs()
    else:
        r = rows.long()
        there = (r >= 0) & (r < x.shape[0])
        p = row_weights.double() if row_weights is not None else torch.ones(r.shape, dtype=torch.float64, device=x.device)
        h = torch.zeros((r.shape[0], x.shape[1]), dtype=torch.float64, device=x.device)
        size = torch.zeros_like(h)
        for j in range(r.shape[1]):
            if x.shape[0] == 0:
                break
            term = p[:, j, None] * x.double()[r[:, j].clamp(0, x.shape[0] - 1)]
            term = torch.where(there[:, j, None], term, torch.zeros_like(term))
            h, size = h + term, size + term.abs()
    if residual is not None:
        h, size = h + residual.double(), size + residual.double().abs()
    return h, size


def normed(h, weight, eps):
    if eps < 0:
        return h
    y = h / (h.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    return torch.nan_to_num(y, nan=0.0) * (weight.double() if weight is not None else 1.0) if eps == 0 and bool((h == 0).all(-1).any()) \
        else y * (weight.double() if weight is not None else 1.0)


def product(x, w, x_scale=None, w_scale=None, bias=None, relu=False, residual=None):
    """(y, sum of the sizes of the terms after the scales) of one matrix product."""
    p = x.double() @ w.double().t()
    if x_scale is not None:
        p = p * x_scale.double()[:, None]
    if w_scale is not None:
        p = p * w_scale.double()
    size = p.abs()
    if bias is not None:
        p, size = p + bias.double(), size + bias.double().abs()
    if relu:
        p = torch.where(p < 0, torch.zeros_like(p), p)
    if residual is not None:
        p, size = p + residual.double(), size + residual.double().abs()
    return p, size


def route(logits, top_k, normalise, positions=None):
    """(chosen, weights, offsets, rows, places) as lists and a 64-bit tensor, token by token."""
    z = logits.double().cpu()
    T, E = z.shape
    pad = [False] * T if positions is None else [int(p) < 0 for p in positions.tolist()]
    chosen, weights = [], torch.zeros((T, top_k), dtype=torch.float64)
    for t in range(T):
        v = z[t].tolist()
        order = sorted(range(E), key=lambda e: (v[e] != v[e], -v[e] if v[e] == v[e] else 0.0, e))[:top_k]
        chosen.append([-1] * top_k if pad[t] else order)
        if not pad[t]:
            picked = z[t, order]
            m = picked[0]
            weights[t] = torch.exp(picked - m) / (torch.exp(picked - m) if normalise else torch.exp(z[t] - m)).sum()
            if bool(z[t].isnan().any()):
                weights[t] = float("nan")
    lists = [[(t, j) for t in range(T) for j in range(top_k) if chosen[t][j] == e] for e in range(E)]
    offsets, rows, places = [0], [], [[-1] * top_k for _ in range(T)]
    for pairs in lists:
        for t, j in pairs:
            places[t][j] = len(rows)
            rows.append(t)
        offsets.append(len(rows))
    return chosen, weights, offsets, rows, places
