"""What softmax_attention sees when row ranges are given without a word about `causal`."""
import pytest
import torch

import softmax
from paper_2506_16640_b200 import autograd, binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal,prefix", [(True, True), (True, False), (False, False)])
def test_ranges_say_all_that_is_visible(causal, prefix):
    # documents with prefixes that all of the document sees; documents that see themselves both ways
    B, H, G, N, d = 2, 2, 1, 150, 64
    g = torch.Generator().manual_seed(7)
    q, k, v, d_o = (torch.randn((B, n, N, d), generator=g).to(torch.bfloat16).cuda() for n in (H, G, G, H))
    cu = torch.tensor([[0, 60, 140], [0, 20, 150]], dtype=torch.int32, device="cuda")
    pre = torch.tensor([[25, 40], [0, 100]], dtype=torch.int32, device="cuda") if prefix else None
    ranges = binding.entmax_attn_row_ranges(cu, N, causal, prefix_len=pre)
    leaves = [x.requires_grad_(True) for x in (q, k, v)]
    o, lse = autograd.softmax_attention(*leaves, row_ranges=ranges, return_lse=True)
    got = torch.autograd.grad(o, leaves, d_o)
    want = softmax.problem(*(x.detach().cpu() for x in leaves), False, ranges.cpu(), d_o=d_o.cpu())
    for name, x in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + got):
        softmax.check(name, x, want)
    # the same said, and the other said: j <= i of the ranges
    assert torch.equal(autograd.softmax_attention(*leaves, row_ranges=ranges, causal=False), o)
    cut = softmax.problem(*(x.detach().cpu() for x in leaves), True, ranges.cpu())
    softmax.check("o", autograd.softmax_attention(*leaves, row_ranges=ranges, causal=True), cut)


def test_without_ranges_the_mask_is_causal():
    g = torch.Generator().manual_seed(8)
    q, k, v = (torch.randn((1, 2, 90, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    assert torch.equal(autograd.softmax_attention(q, k, v), autograd.softmax_attention(q, k, v, causal=True))
    want = softmax.problem(*(x.cpu() for x in (q, k, v)), False)
    softmax.check("o", autograd.softmax_attention(q, k, v, causal=False), want)
