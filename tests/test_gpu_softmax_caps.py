"""Softmax attention with caps far above the scores, forward and backward: a score is off by a part of itself, not by a part of the cap.

x = cap tanh(z / cap) = z (1 - (z / cap)^2 / 3 + ..).  A tanh that is off by a few u = 2^-24 of its value keeps x within the 36 u |score| that
tests/softmax.py grants every score anyway, so the bounds are those of the call without a cap."""
import pytest
import torch

import paged
import softmax
from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


def _inputs(B, H, G, N, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((B, n, N, d), generator=g).to(dtype).cuda() for n in (H, G, G, H)]


def _bounds_without_a_cap(want, plain):
    """The capped call's values with the uncapped call's bounds (scores differ by less than 1 % of themselves: 1.05)."""
    return {n: (1.05 * plain[n] if n.endswith("_tol") else x) for n, x in want.items()}


def _problem(q, k, v, d_o, cap, slopes=None, c_rows=None):
    cpu = lambda x: None if x is None else x.cpu()  # noqa: E731
    args = (cpu(q), cpu(k), cpu(v), True, None, None, None, None, cpu(c_rows), cpu(slopes))
    return _bounds_without_a_cap(softmax.problem(*args, cap, None, cpu(d_o)), softmax.problem(*args, 0.0, None, cpu(d_o)))


def _run(q, k, v, d_o, cap, **t):
    o, lse = binding.entmax_attn_softmax_fwd(q, k, v, True, softcap=cap, **t)
    dq, dk, dv, dc, _ = binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, True, softcap=cap, want_scale_rows=True, **t)
    return dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv, dc=dc)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("cap", [100.0, 1e3, 1e6, 1e12])
@pytest.mark.parametrize("kind", ["plain", "slopes+rows"])
def test_scores_far_below_the_cap(cap, kind, dtype):
    B, H, G, N, d = 1, 2, 1, 200, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype, seed=3)
    t = {}
    if kind != "plain":
        t = dict(alibi_slopes=torch.tensor([0.5, 0.0], device="cuda"), c_rows=0.5 + torch.rand((B, H, N), generator=torch.Generator().manual_seed(1)).cuda())
    want = _problem(q, k, v, d_o, cap, t.get("alibi_slopes"), t.get("c_rows"))
    for name, x in _run(q, k, v, d_o, cap, **t).items():
        softmax.check(name, x, want, "cap %g" % cap)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("cap", [1e3, 1e5])
def test_scores_far_below_the_cap_next_to_rows_beyond_it(cap, dtype):
    # every sixteenth row has scores far beyond the cap, the others have theirs as without them (those rows' d_o is 0: no gradient of theirs
    # in dk and dv, and D = 0)
    B, H, G, N, d = 1, 2, 1, 200, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype, seed=4)
    far = torch.arange(N, device="cuda") % 16 == 5
    q[:, :, far] *= 4 * cap
    d_o[:, :, far] = 0.0
    near = ~far.cpu()
    got, want = _run(q, k, v, d_o, cap), _problem(q, k, v, d_o, cap)
    for name in ("o", "lse", "dq", "dc"):
        softmax.check(name, got[name][:, :, near], {n: want[n][:, :, near] for n in (name, name + "_tol")}, "cap %g" % cap)
    for name in ("dk", "dv"):
        softmax.check(name, got[name], want, "cap %g" % cap)


@pytest.mark.parametrize("cap", [1e3, 1e5])
@pytest.mark.parametrize("n", [1, 4, 130])
def test_paged_scores_far_below_the_cap_next_to_rows_beyond_it(n, cap):
    # rows of a warp: two query heads of the same tokens, one of them with scores far beyond the cap
    H, KH, d, page = 4, 2, 64, 16
    g = torch.Generator().manual_seed(5)
    lens = [n + 70, n + 400]
    keys, values = ([torch.randn((m, KH, d), generator=g).to(bf16) for m in lens] for _ in range(2))
    q = torch.randn((2 * n, H, d), generator=g).to(bf16)
    q[:, 0::2] *= 4 * cap
    kc, vc, table = paged.pool(keys, values, page, d, KH, 5, "cuda")
    o, lse = binding.entmax_attn_softmax_paged_fwd(q.cuda(), kc, vc, table, torch.tensor(lens, dtype=torch.int32, device="cuda"),
                                                   torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), softcap=cap)
    for b in range(2):
        pos = torch.arange(lens[b] - n, lens[b])
        rows = slice(b * n, (b + 1) * n)
        for h in range(1, H, 2):
            args = (q[rows, h], keys[b][:, h // 2], values[b][:, h // 2], torch.zeros_like(pos), pos + 1, None, None)
            want = _bounds_without_a_cap(softmax.head(*args, cap, pos=pos), softmax.head(*args, 0.0, pos=pos))
            softmax.check("o", o[rows, h], want)
            softmax.check("lse", lse[rows, h], want)


@pytest.mark.parametrize("dtype", [f32, bf16])
@pytest.mark.parametrize("name", ["sm_scale", "softcap"])
@pytest.mark.parametrize("value", [2.0 ** -100, 2.0 ** 100])
def test_the_least_and_the_largest_scales_and_caps(name, value, dtype):
    # with slopes, and with scales of 0 among others: what is left are the slopes' terms, the uncapped scores, or the largest score alone
    B, H, G, N, d = 1, 2, 1, 200, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype, seed=6)
    c = 0.5 + torch.rand((B, H, N), generator=torch.Generator().manual_seed(1))
    c[:, :, ::7] = 0.0
    t = dict(alibi_slopes=torch.tensor([0.5, 0.03], device="cuda"), c_rows=c.cuda())
    if name == "sm_scale" and value > 1:
        k *= 2.0 ** -100                                          # (scores of order 8)
    o, lse = binding.entmax_attn_softmax_fwd(q, k, v, True, **{name: value}, **t)
    dq, dk, dv, dc, _ = binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, True, want_scale_rows=True, **{name: value}, **t)
    cap, sm = (0.0, value) if name == "sm_scale" else (value, None)
    args = (q.cpu(), k.cpu(), v.cpu(), True, None, None, None, None, c, t["alibi_slopes"].cpu())
    want = softmax.problem(*args, cap, sm, d_o.cpu())
    if cap > 1:
        want = _bounds_without_a_cap(want, softmax.problem(*args, 0.0, None, d_o.cpu()))
    for n, x in dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv, dc=dc).items():
        softmax.check(n, x, want, "%s %g" % (name, value))
