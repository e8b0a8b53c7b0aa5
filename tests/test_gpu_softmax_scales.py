"""Softmax attention with scales that are not finite: in rows that see nothing they have no say, elsewhere they are reported and what they make of the
row is not taken for an empty one."""
import pytest
import torch

import paged
import softmax
from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def _inputs(B, H, G, N, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn((B, n, N, d), generator=g).to(dtype).cuda() for n in (H, G, G, H)]


def _status():
    return torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
@pytest.mark.parametrize("rows_grad", [True, False])
def test_scales_of_rows_that_see_nothing(dtype, bad, rows_grad):
    # padding behind the documents and a hole between them, with whatever a model projects from it as its scale
    B, H, G, N, d = 1, 2, 1, 200, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype)
    cu = torch.tensor([[3, 90, 150]], dtype=torch.int32, device="cuda")
    ranges = binding.entmax_attn_row_ranges(cu, N, True)
    empty = (ranges[..., 0] >= ranges[..., 1])[:, None].expand(B, H, N)
    assert int(empty.sum()) == H * 53
    c = 0.5 + torch.rand((B, H, N), generator=torch.Generator().manual_seed(1)).cuda()
    want = softmax.problem(*(x.cpu() for x in (q, k, v)), False, ranges.cpu(), None, None, None, c.cpu(), None, 0.0, None, d_o.cpu())
    c[empty] = bad
    o, lse = binding.entmax_attn_softmax_fwd(q, k, v, False, c_rows=c, row_ranges=ranges)
    dq, dk, dv, dc, _ = binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, False, c_rows=c, row_ranges=ranges, want_scale_rows=rows_grad)
    for name, x in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)) + ((("dc", dc),) if rows_grad else ()):
        softmax.check(name, x, want)
    assert (o[empty] == 0).all() and (dq[empty] == 0).all() and (lse[empty] == -INF).all()


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("kind", ["rows", "length"])
def test_a_scale_that_is_not_finite_is_reported(dtype, bad, kind):
    B, H, G, N, d = 1, 2, 1, 150, 64
    q, k, v, _ = _inputs(B, H, G, N, d, dtype, seed=1)
    t = {"c_rows": torch.ones((B, H, N), device="cuda")}
    if kind == "rows":
        t["c_rows"][0, 1, 77] = bad
    else:
        t = dict(beta=torch.tensor([1.0, bad], device="cuda"), gamma=torch.ones(2, device="cuda"), delta=torch.ones(2, device="cuda"))
    status = _status()
    binding.entmax_attn_softmax_fwd(q, k, v, True, **t, status=status)
    assert int(status[0]) == binding.FLAG_BAD_SCALE
    binding.entmax_attn_softmax_fwd(q, k, v, True, status=status)
    assert int(status[0]) == 0


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_rows_of_a_scale_that_is_not_finite_are_no_empty_rows(dtype, bad, cap):
    B, H, G, N, d = 1, 2, 1, 300, 64
    q, k, v, _ = _inputs(B, H, G, N, d, dtype, seed=2)
    c = torch.ones((B, H, N), device="cuda")
    ref, ref_lse = binding.entmax_attn_softmax_fwd(q, k, v, True, c_rows=c, softcap=cap)
    c[0, 1, 277] = bad
    o, lse = binding.entmax_attn_softmax_fwd(q, k, v, True, c_rows=c, softcap=cap)
    assert torch.isnan(lse[0, 1, 277]) and torch.isnan(o[0, 1, 277]).all()
    # the other rows have what they had
    o[0, 1, 277], lse[0, 1, 277] = ref[0, 1, 277], ref_lse[0, 1, 277]
    assert torch.equal(o, ref) and torch.equal(lse, ref_lse)


@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("new,lens", [([1, 1], [20, 40]), ([1, 1], [6000, 30000]), ([4], [9000]), ([140, 1], [200, 30]), ([140], [30000])])
def test_paged_rows_of_a_scale_that_is_not_finite_whether_cut_or_not(new, lens, bad):
    # sequences of one CTA, sequences cut over many and joined, chunks whose keys are shared out and joined
    H, KH, d, page = 4, 2, 64, 64
    g = torch.Generator().manual_seed(3)
    keys, values = ([torch.randn((m, KH, d), generator=g).to(bf16) for m in lens] for _ in range(2))
    q = torch.randn((sum(new), H, d), generator=g).to(bf16).cuda()
    kc, vc, table = paged.pool(keys, values, page, d, KH, 3, "cuda")
    cu = torch.tensor([0] + [sum(new[:i + 1]) for i in range(len(new))], dtype=torch.int32, device="cuda")
    kv = torch.tensor(lens, dtype=torch.int32, device="cuda")
    one = torch.ones(H, device="cuda")
    delta = torch.tensor([1.0, 1.0, bad, 1.0], device="cuda")
    ref, ref_lse = binding.entmax_attn_softmax_paged_fwd(q, kc, vc, table, kv, cu, 0 * one, one, one)
    status = _status()
    o, lse = binding.entmax_attn_softmax_paged_fwd(q, kc, vc, table, kv, cu, 0 * one, one, delta, status=status)
    assert int(status[0]) == binding.FLAG_BAD_SCALE
    assert torch.isnan(o[:, 2]).all() and torch.isnan(lse[:, 2]).all()
    for h in (0, 1, 3):                          # (the other heads have what they had)
        assert torch.equal(o[:, h], ref[:, h]) and torch.equal(lse[:, h], ref_lse[:, h])
