"""Softmax attention's definition in 64 bits, forward and backward, one head at a time, and what the kernels may be off by.

Roundings counted (u = 2^-24, the half step of float32; h the half step of what enters a tensor-core product: 2^-8 of bfloat16, 0 where everything
stays float32; r the half step of an output, 2^-8 or u):
  scores     a dot product of d exact products in any order d u sum|q k|; the cap's tanh an absolute 8 u (one exp2 and one reciprocal of 2 u each,
             a sum, around values below 1), so cap 8 u, and the products around it 4 u of the value; the slope 4 u of itself; c (a logarithm, a
             power, a product and a sum, the power's exponent below 2) 32 u of the score; the base-2 exponent, its difference from the maximum 4 u
             of both: together ds, the error of an exponent
  p          relative ds + 8 u (exp2 2 u, or a polynomial of 2^-22 at most; the division by the mass), the mass itself by its terms' and N u
  lse        the largest ds of the row + (N + 8) u + 4 u |lse|
  O          sum p |v| (h + dp) + r |O|, in float32 sums N u more
  D = <p,dP> the bfloat16 kernels take it from the rounded O they are given: sum |dO| dO_err, the float32 ones from float32 sums
  dS         p dP's and D's errors, and h of its own on the way into a product
Bounds are worst cases added up: they hold for every element."""
import math

import torch

U = 2.0 ** -24


def ranges(N, causal, given=None):
    """begin, end of the keys each row sees, as the call's arguments say."""
    i = torch.arange(N)
    lo, hi = torch.zeros(N, dtype=torch.long), (i + 1 if causal else torch.full((N,), N))
    if given is not None:
        lo, hi = given[:, 0].long().clamp_min(0), torch.minimum(given[:, 1].long(), hi)
    return lo, hi


def head(q, k, v, lo, hi, c=None, sm=None, cap=0.0, slope=0.0, d_o=None, bf16=True, pos=None):
    """One head: q [n, d], k, v [m, d]; rows see the keys lo .. hi - 1; c [n] the rows' scales; pos: the rows' positions (0 .. n - 1).
    Returns a dict of values and, under name + "_tol", of bounds; with d_o the gradients too (dk, dv of this query head alone)."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    m = k.shape[0]
    h, r = (2.0 ** -8, 2.0 ** -8) if bf16 else (0.0, U)
    sm = 1.0 / math.sqrt(d) if sm is None else sm
    c = torch.ones(n, dtype=torch.float64) if c is None else c.double()
    j = torch.arange(m)
    pos = torch.arange(n) if pos is None else pos
    sees = (j >= lo[:, None]) & (j < hi[:, None])
    some = sees.any(1)
    z = sm * (q @ k.T)
    dz = sm * (d + 4) * U * (q.abs() @ k.abs().T)
    grow = torch.ones_like(z)
    x = z
    if cap:
        t = torch.tanh(z / cap)
        x, grow = cap * t, 1 - t * t
        dz = dz + 8 * U * cap + 4 * U * x.abs()
    dist = (pos[:, None] - j).abs().double()
    x = x - slope * dist
    s = torch.where(sees, c[:, None] * x, -math.inf)
    lse = torch.logsumexp(s, 1)
    safe = torch.where(some, lse, 0.0)[:, None]
    p = torch.where(sees, torch.exp(s - safe), 0.0)
    score = torch.where(sees, s, 0.0).abs()
    top = score.amax(1, keepdim=True)
    ds = c.abs()[:, None] * (dz + 4 * U * slope * dist + 4 * U * x.abs()) + 36 * U * score + 4 * U * (top + safe.abs())
    ds = torch.where(sees, ds, 0.0)
    worst = ds.amax(1, keepdim=True)
    dp = (ds + worst + (m + 16) * U) * 1.01
    out = dict(o=p @ v, lse=lse, lse_tol=worst[:, 0] + (m + 8) * U + 4 * U * safe[:, 0].abs())
    out["o_tol"] = (p * (h + dp)) @ v.abs() + m * U * (p @ v.abs()) + r * out["o"].abs() + 1e-30
    if d_o is None:
        return out
    g = d_o.double()
    dP = g @ v.T
    dP_err = (d + 4) * U * (g.abs() @ v.abs().T)
    dot = (p * dP).sum(1, keepdim=True)
    flow = p * (dP - dot)
    # D from the O given (rounded, and off by what its products were rounded by), or from the float32 probabilities
    dot_err = (g.abs() * out["o_tol"]).sum(1, keepdim=True) + (p * (dP_err + dP.abs() * (dp + m * U))).sum(1, keepdim=True) + d * U * (g.abs() * out["o"].abs()).sum(1, keepdim=True)
    flow_err = p * (dp * (dP - dot).abs() + dP_err + dot_err + 4 * U * (dP.abs() + dot.abs()))
    w = c[:, None] * grow * flow
    # (1 - tanh^2 in float32: 8 u absolute from the tanh's error twice)
    w_err = c.abs()[:, None] * (grow.abs() * flow_err + 20 * U * flow.abs()) + 4 * U * w.abs()
    out["dq"], out["dk"], out["dv"] = sm * (w @ k), sm * (w.T @ q), p.T @ g
    out["dq_tol"] = sm * ((h * w.abs() + w_err) @ k.abs()) * 1.01 + m * U * sm * (w.abs() @ k.abs()) + r * out["dq"].abs() + 1e-30
    out["dk_tol"] = sm * ((h * w.abs() + w_err).T @ q.abs()) * 1.01 + n * U * sm * (w.abs().T @ q.abs())
    out["dv_tol"] = (p * (h + dp)).T @ g.abs() + n * U * (p.T @ g.abs())
    out["dc"] = (flow * x).sum(1)
    # either sum dS x in float32, or sum p dP x - sum p dP sum p x: errors of the float32 probabilities and sums, not of the rounded O
    big = lambda t: (p * t).sum(1)  # noqa: E731
    eps = dp.amax(1) + (2 * m + 40) * U
    out["dc_tol"] = eps * (big(dP.abs() * x.abs()) + big(dP.abs()) * big(x.abs())) + big(dP_err * x.abs()) + big(dP_err) * big(x.abs()) + \
        big((dP - dot).abs() * (dz + 4 * U * slope * dist)) + 1e-30
    return out


def scale(beta, gamma, delta, n):
    """c of rows that see n keys."""
    n = n.double()
    return delta + torch.where(n > 1, beta * torch.log(torch.clamp(n, min=2.0)) ** gamma, 0.0)


def scale_grads(dc, beta, gamma, n):
    n = n.double()
    log_n = torch.log(torch.clamp(n, min=2.0))
    w = torch.where(n > 1, log_n ** gamma, 0.0)
    return (dc * w).sum(), (dc * w * beta * torch.log(log_n)).sum(), dc.sum()


def problem(q, k, v, causal, given=None, beta=None, gamma=None, delta=None, c_rows=None, slopes=None, cap=0.0, sm=None, d_o=None):
    """A whole call on the CPU: [B, H, N, d] and [B, G, N, d]; values and bounds of every output, dk and dv summed over shared heads."""
    bf16 = q.dtype == torch.bfloat16
    r = 2.0 ** -8 if bf16 else U
    B, H, N, d = q.shape
    G = k.shape[1]
    got = {}
    put = lambda name, shape: got.setdefault(name, torch.zeros(shape, dtype=torch.float64))  # noqa: E731
    for b in range(B):
        lo, hi = ranges(N, causal, None if given is None else given[b])
        n = (hi - lo).clamp_min(0)
        for hh in range(H):
            kh = hh * G // H
            c = None
            if c_rows is not None:
                c = c_rows[b, hh]
            elif beta is not None:
                c = scale(beta[hh].double(), gamma[hh].double(), delta[hh].double(), n)
            one = head(q[b, hh], k[b, kh], v[b, kh], lo, hi, c, sm, cap, 0.0 if slopes is None else float(slopes[hh]),
                       None if d_o is None else d_o[b, hh], bf16)
            for name in ("o", "o_tol", "dq", "dq_tol"):
                if name in one:
                    put(name, (B, H, N, d))[b, hh] = one[name]
            for name in ("lse", "lse_tol", "dc", "dc_tol"):
                if name in one:
                    put(name, (B, H, N))[b, hh] = one[name]
            for name in ("dk", "dk_tol", "dv", "dv_tol"):
                if name in one:
                    put(name, (B, G, N, d))[b, kh] += one[name]
            if beta is not None and d_o is not None:
                log_n = torch.log(torch.clamp(n.double(), min=2.0))
                w = torch.where(n > 1, log_n ** gamma[hh].double(), 0.0)
                gr = scale_grads(one["dc"], beta[hh].double(), gamma[hh].double(), n)
                for name, x, weight in (("dbeta", gr[0], w), ("dgamma", gr[1], (w * beta[hh].double() * torch.log(log_n)).abs()),
                                        ("ddelta", gr[2], torch.ones_like(w))):
                    put(name, (H,))[hh] += x
                    # (the weights are float32 powers and logarithms, 32 u; ln ln n is off by 4 u of 1 where ln n is near 1)
                    put(name + "_tol", (H,))[hh] += (one["dc_tol"] * weight + one["dc"].abs() * (32 * U * weight + 8 * U * w * beta[hh].abs())).sum() + U * x.abs()
    for name in ("dk", "dv"):
        if name in got:
            got[name + "_tol"] += r * got[name].abs() + 1e-30
    return got


def check(name, value, want, context=""):
    """Every element within its bound; rows that see nothing exactly."""
    x, y, tol = value.detach().cpu().double(), want[name], want[name + "_tol"]
    assert x.shape == y.shape, (name, x.shape, y.shape)
    same = (x == y) | (torch.isinf(y) & (x == y))
    off = torch.where(same, torch.zeros_like(y), (x - y).abs() - tol)
    assert not torch.isnan(x).any(), "%s %s: NaN" % (name, context)
    worst = off.flatten().argmax() if off.numel() else 0
    if off.numel():
        assert (off <= 0).all(), "%s %s: %d of %d off, worst %g against %g within %g" % (
            name, context, int((off > 0).sum()), off.numel(), float(x.flatten()[worst]), float(y.flatten()[worst]), float(tol.flatten()[worst]))
