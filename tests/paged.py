"""A paged cache for the tests, and the paged entry points' definitions in 64 bits (plain formulas, a sequence and a head at a time)."""
import math

import numpy as np
import torch


def pool(keys, values, page, d, kv_heads, seed=0, device="cpu", spare=3, table_extra=2, fill=float("nan"), layout="tokens"):
    """Pages for sequences with the given keys and values ([len, kv_heads, d] each): pool tensors, block table.

    Slots nobody writes hold `fill`; table entries behind a sequence's pages point nowhere.  layout: "tokens" [pages, page, heads, d],
    "heads" [pages, heads, page, d] seen through a transpose, "fused" K and V side by side in one pool."""
    rng = np.random.default_rng(seed)
    need = [-(-k.shape[0] // page) for k in keys]
    n = sum(need) + spare
    order = rng.permutation(n)
    if layout == "fused":
        both = torch.full((n, 2, page, kv_heads, d), fill, dtype=torch.bfloat16)
        kc, vc = both[:, 0], both[:, 1]
    elif layout == "heads":
        kc, vc = (torch.full((n, kv_heads, page, d), fill, dtype=torch.bfloat16).transpose(1, 2) for _ in range(2))
    else:
        kc, vc = (torch.full((n, page, kv_heads, d), fill, dtype=torch.bfloat16) for _ in range(2))
    table = torch.full((len(keys), max(need) + table_extra), 2 ** 31 - 1, dtype=torch.int32)
    at = 0
    for b, (k, v) in enumerate(zip(keys, values)):
        pages = torch.from_numpy(order[at:at + need[b]].copy())
        at += need[b]
        table[b, :need[b]] = pages.to(torch.int32)
        for i, pg in enumerate(pages.tolist()):
            m = min(page, k.shape[0] - i * page)
            kc[pg, :m] = k[i * page:i * page + m]
            vc[pg, :m] = v[i * page:i * page + m]
    if layout == "fused":
        both = both.to(device)
        return both[:, 0], both[:, 1], table.to(device)
    if layout == "heads":
        return kc.transpose(1, 2).contiguous().to(device).transpose(1, 2), vc.transpose(1, 2).contiguous().to(device).transpose(1, 2), table.to(device)
    return kc.to(device), vc.to(device), table.to(device)


def threshold(y, e):
    """tau of sum [y - tau]_+^e = 1 along the last dimension, by halving the bracket [y_max - 1, y_max]."""
    hi = y.amax(-1, keepdim=True)
    lo = hi - 1.0
    for _ in range(80):
        mid = (lo + hi) / 2
        more = (y - mid).clamp_min(0).pow(e).sum(-1, keepdim=True) >= 1.0
        lo, hi = torch.where(more, mid, lo), torch.where(more, hi, mid)
    return lo


def attend(q, k, v, first_pos, alpha, scale=None, slope=0.0, sm_scale=None):
    """Rows of one head: q [n, d] at positions first_pos .., k, v [len, d] (bf16 values).  Returns o, tau and what a float32
    evaluation may be off by: (o, tau, tol_o, tol_tau, support_low, support_high).

    y = (alpha-1) c (sm_scale <q,k> - slope dist).  In float32 (u = 2^-24): <q,k> is off by at most d u sum|q k| (any order of d
    additions of exact bf16 products), the products with the scale by 4 u of y, c (a logarithm, a power, a product and a sum, a few
    ulp each) by 16 u of y, the bias by 4 u of itself: dy.  tau as a function of y moves by at most max dy (it is monotone and moves
    with y); the iteration stops within 1e-7 max(1, |tau|) or at a mass within 32 sums' rounding (2e-6 covers 16 u sqrt(n) and the 1.6e-6 of the
    bracketed form) of 1, and |d mass / d tau| >= e for terms of at most 1.  So y - tau is off by at most D = dy + tol_tau, p by what it changes over
    [-D, D], o by sum dp |v| plus its own rounding (2^-8) and the rounding of the sum in float32 (n u sum p |v|)."""
    u = 2.0 ** -24
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    L = k.shape[0]
    e = 1.0 / (alpha - 1.0)
    sm = 1.0 / math.sqrt(d) if sm_scale is None else sm_scale
    pos = torch.arange(first_pos, first_pos + n, dtype=torch.float64)[:, None]
    j = torch.arange(L, dtype=torch.float64)
    c = torch.ones_like(pos)
    if scale is not None:
        beta, gamma, delta = (float(x) for x in scale)
        c = delta + torch.where(pos > 0, beta * torch.log((pos + 1).clamp_min(2.0)) ** gamma, torch.zeros_like(pos))
    a = (alpha - 1.0) * c
    y = a * (sm * (q @ k.T) - slope * (pos - j))
    y = torch.where(j <= pos, y, torch.full_like(y, -math.inf))
    seen = (j <= pos).double()
    dy = u * a.abs() * (sm * d * (q.abs() @ k.abs().T) + 4 * slope * (pos - j).abs()) * seen + 20 * u * torch.where(seen > 0, y.abs(), 0 * seen)
    dy = dy.amax(-1, keepdim=True)
    tau = threshold(y, e)
    tol_tau = dy + 2e-7 * tau.abs().clamp_min(1.0) + 2e-6 / min(e, 1.0)
    D = dy + tol_tau
    w = y - tau
    p = w.clamp_min(0).pow(e)
    dp = (w + D).clamp_min(0).pow(e) - (w - D).clamp_min(0).pow(e)
    o = p @ v
    tol_o = dp @ v.abs() + 2.0 ** -8 * o.abs() + L * u * (p @ v.abs()) + 1e-30
    return o, tau[:, 0], tol_o, tol_tau[:, 0], (w > D).sum(-1), (w > -D).sum(-1)


def rotate(x, rotation, pos, interleaved):
    """x [n, heads, d] at the given positions, in 64 bits."""
    r = rotation.shape[1]
    x = x.double().clone()
    cos, sin = rotation[pos].double()[:, None, :r // 2], rotation[pos].double()[:, None, r // 2:]
    lo = x[..., 0:r:2] if interleaved else x[..., :r // 2]
    hi = x[..., 1:r:2] if interleaved else x[..., r // 2:r]
    a, b = lo * cos - hi * sin, hi * cos + lo * sin
    if interleaved:
        x[..., 0:r:2], x[..., 1:r:2] = a, b
    else:
        x[..., :r // 2], x[..., r // 2:r] = a, b
    return x
