"""Softmax attention over a paged cache in batches whose sequences are shared between the two kernels in every way."""
import pytest
import torch

import paged
import softmax
from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu

bf16 = torch.bfloat16


@pytest.mark.parametrize("bound", [0, 20])
def test_a_batch_whose_sequences_take_either_kernel(bound):
    # the cutoff between the kernels goes by the average chunk where the longest fills more than 64 rows: here 16 rows, so that
    # chunks of five tokens of four query heads take the tensor-core kernel next to the single tokens and the chunk of 20
    new = [1] * 120 + [5] * 10 + [20] + [2, 4, 3]
    g = torch.Generator().manual_seed(4)
    order = torch.randperm(len(new), generator=g).tolist()
    new = [new[i] for i in order]
    lens = [n + int(x) for n, x in zip(new, torch.randint(0, 400, (len(new),), generator=g))]
    H, KH, d, page = 8, 2, 64, 16
    keys, values = ([torch.randn((m, KH, d), generator=g).to(bf16) for m in lens] for _ in range(2))
    q = torch.randn((sum(new), H, d), generator=g).to(bf16)
    kc, vc, table = paged.pool(keys, values, page, d, KH, 4, "cuda")
    cu = [0] + torch.tensor(new).cumsum(0).tolist()
    kv, cu_q = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (lens, cu))
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    o, lse = binding.entmax_attn_softmax_paged_fwd(q.cuda(), kc, vc, table, kv, cu_q, max_q_len=bound, status=status)
    assert int(status[0]) == 0
    for b, n in enumerate(new):
        pos, rows = torch.arange(lens[b] - n, lens[b]), slice(cu[b], cu[b + 1])
        for h in (0, 7):
            want = softmax.head(q[rows, h], keys[b][:, h // 4], values[b][:, h // 4], torch.zeros_like(pos), pos + 1, pos=pos)
            softmax.check("o", o[rows, h], want, "%d of %d" % (n, lens[b]))
            softmax.check("lse", lse[rows, h], want)
