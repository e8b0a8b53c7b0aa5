"""The backward kernels a call without a gradient of its scale takes, and masks over many tiles, against the definition in 64 bits.

The dQ kernel is compiled apart for calls that want dL/dc, for calls with scales or slopes that do not, and for calls with neither (most training steps): the last two
take D and the rounding of dS otherwise.  Tolerances: tests/softmax.py."""
import pytest
import torch

import softmax
from paper_2506_16640_b200 import autograd, binding

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


def _inputs(B, H, G, N, d, dtype=bf16, seed=0, sigma=1.0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((B, N, (H + 2 * G) * d), generator=g) * sigma).to(dtype).cuda()
    q, k, v = (x.view(B, N, -1, d).transpose(1, 2) for x in qkv.split([H * d, G * d, G * d], 2))
    return q, k, v, torch.randn((B, N, H, d), generator=g).to(dtype).cuda().transpose(1, 2)


def _terms(kind, B, H, N):
    g = torch.Generator().manual_seed(91)
    t = {}
    for word in kind.split("+"):
        if word == "cap":
            t["softcap"] = 20.0
        elif word == "lowcap":
            t["softcap"] = 1.5
        elif word == "slopes":
            t["alibi_slopes"] = torch.where(torch.arange(H) % 2 == 0, 2.0 ** -(torch.arange(H) + 1.0), torch.zeros(H)).cuda()
        elif word == "length":
            t["beta"], t["gamma"], t["delta"] = (0.2 + 0.6 * torch.rand(H, generator=g).cuda() for _ in range(3))
        elif word == "rows":
            t["c_rows"] = (torch.randn((B, H, N), generator=g) * 1.5).cuda()
        elif word == "ranges":
            a = torch.randint(-3, N + 3, (B, N), generator=g)
            n = (torch.rand((B, N), generator=g) ** 2 * (N + 6)).long()
            n = torch.where(torch.rand((B, N), generator=g) < 0.15, torch.randint(-2, 2, (B, N), generator=g), n)
            t["row_ranges"] = torch.stack([a, a + n], -1).to(torch.int32).cuda()
    return t


def _check(q, k, v, d_o, causal, t, context=""):
    cpu = lambda x: None if x is None else x.detach().cpu()  # noqa: E731
    o, lse = binding.entmax_attn_softmax_fwd(q, k, v, causal, **t)
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    got = binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, causal, status=status, **t)
    assert int(status[0]) == 0 and got[3] is None and got[4] is None
    want = softmax.problem(cpu(q), cpu(k), cpu(v), causal, cpu(t.get("row_ranges")), cpu(t.get("beta")), cpu(t.get("gamma")), cpu(t.get("delta")),
                           cpu(t.get("c_rows")), cpu(t.get("alibi_slopes")), t.get("softcap", 0.0), None, cpu(d_o))
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + got[:3]):
        softmax.check(name, x, want, context)
    return (o, lse) + got[:3]


SIZES = [(1, 1, 1, 1, 64), (2, 3, 1, 2, 128), (1, 2, 2, 63, 64), (1, 4, 2, 128, 128), (1, 2, 1, 129, 64), (2, 2, 2, 257, 128), (1, 6, 2, 300, 64),
         (1, 3, 3, 520, 128), (3, 8, 1, 150, 64)]


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("B,H,G,N,d", SIZES)
@pytest.mark.parametrize("causal", [True, False])
def test_sizes(B, H, G, N, d, causal, dtype):
    _check(*_inputs(B, H, G, N, d, dtype, seed=N), causal, {})


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("kind", ["cap", "lowcap", "slopes", "ranges", "ranges+cap", "ranges+slopes", "length", "rows", "cap+slopes", "cap+rows", "ranges+cap+slopes+length"])
@pytest.mark.parametrize("B,H,G,N,d", [(2, 2, 1, 200, 64), (1, 4, 4, 390, 128)])
def test_terms(B, H, G, N, d, kind, dtype):
    _check(*_inputs(B, H, G, N, d, dtype, seed=len(kind)), "ranges" not in kind, _terms(kind, B, H, N))


@pytest.mark.parametrize("kind", ["plain", "slopes"])
@pytest.mark.parametrize("d", [64, 128])
def test_large_and_small_scores(d, kind):
    for sigma in (0.01, 6.0, 30.0):
        _check(*_inputs(1, 2, 1, 260, d, seed=9, sigma=sigma), True, _terms(kind, 1, 2, 260), "sigma %g" % sigma)


@pytest.mark.parametrize("kind", ["plain", "slopes"])
def test_long_rows(kind):
    _check(*_inputs(1, 2, 1, 2003, 128, seed=30), True, _terms(kind, 1, 2, 2003))


def test_autograd_of_plain_calls():
    q, k, v, d_o = _inputs(2, 4, 2, 260, 64, seed=12)
    leaves = [x.detach().requires_grad_(True) for x in (q, k, v)]
    o, lse = autograd.softmax_attention(*leaves, return_lse=True)
    want = softmax.problem(*(x.cpu() for x in (q, k, v)), True, d_o=d_o.cpu())
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + torch.autograd.grad(o, leaves, d_o)):
        softmax.check(name, x, want)


@pytest.mark.parametrize("mask,kind", [("documents", "plain"), ("documents", "cap"), ("prefix", "plain"), ("window", "length"), ("both ways", "plain")])
def test_ranges_over_many_tiles(mask, kind):
    # 66 tiles: a K/V tile's Q tiles are looked for 32 at a time, three times; between the documents a hole of 40 tiles, where none is found
    B, H, G, N, d, hole, behind = 1, 2, 1, 8400, 64, 1500, 6700
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=41)
    cu = torch.tensor([[0, 100, hole, hole]], dtype=torch.int32, device="cuda")
    first = binding.entmax_attn_row_ranges(cu, N, mask != "both ways")
    cu = torch.tensor([[behind, 8000, 8390]], dtype=torch.int32, device="cuda")
    pre = torch.tensor([[1200, 30]], dtype=torch.int32, device="cuda") if mask == "prefix" else None
    last = binding.entmax_attn_row_ranges(cu, N, mask != "both ways", prefix_len=pre, window=700 if mask == "window" else 0)
    ranges = torch.where((first[..., 1:] > first[..., :1]), first, last)
    # a row far behind sees keys of the first documents, one of those sees keys far ahead
    ranges[0, 8395] = torch.tensor([40, 130], device="cuda")
    ranges[0, 70] = torch.tensor([6800, 6900], device="cuda")
    t = dict(_terms(kind, B, H, N), row_ranges=ranges)
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    runs = []
    for _ in range(4):
        o, lse = binding.entmax_attn_softmax_fwd(q, k, v, False, **t)
        runs.append((o, lse) + binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, False, status=status, **t)[:3])
    assert int(status[0]) == 0
    for other in runs[1:]:
        for x, y in zip(runs[0], other):
            assert torch.equal(x, y)
    # the definition, without the hole: nothing there is seen by or sees anyone, and distances do not matter
    keep = torch.cat([torch.arange(hole), torch.arange(behind, N)])
    cpu = lambda x: None if x is None else x.cpu()  # noqa: E731
    closed = ranges.cpu()[:, keep]
    closed = torch.where(closed >= behind, closed - (behind - hole), closed)
    want = softmax.problem(*(x.cpu()[:, :, keep] for x in (q, k, v)), False, closed, cpu(t.get("beta")), cpu(t.get("gamma")), cpu(t.get("delta")),
                           None, None, t.get("softcap", 0.0), None, d_o.cpu()[:, :, keep])
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), runs[0]):
        softmax.check(name, x.cpu()[:, :, keep], want, mask)
        assert (x[:, :, hole:behind] == (-float("inf") if name == "lse" else 0.0)).all()
