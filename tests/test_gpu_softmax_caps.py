"""Softmax attention with caps far above the scores, forward and backward: a score is off by a part of itself, not by a part of the cap.

x = cap tanh(z / cap) = z (1 - (z / cap)^2 / 3 + ..).  A tanh that is off by a few u = 2^-24 of its value keeps x within the 36 u |score| that
tests/softmax.py grants every score anyway, so the bounds are those of the call without a cap."""
import pytest
import torch

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
