"""Tables of a serving step whose caller expected no new tokens."""
import pytest
import torch

from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("total,flags", [(0, binding.FLAG_BAD_LENGTH), (2, binding.FLAG_BAD_LENGTH), (3, 0), (5, 0)])
def test_more_new_tokens_than_rows_are_reported(total, flags):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    kv, cu, pos, slots, left = binding.entmax_attn_paged_tables(dev([4, 0]), dev([1, 2]), dev([[1, 0], [0, 0]]), dev([3, 2]), dev([2]), 16, 6, total,
                                                               status=status)
    assert int(status[0]) == flags
    assert kv.tolist() == [5, 2] and cu.tolist() == [0, 1, 3] and left.tolist() == [1]
    assert pos.tolist()[:3] == [4, 0, 1][:total] and slots.tolist()[:3] == [20, 32, 33][:total]


def test_no_new_tokens_and_no_rows():
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    kv, cu, pos, slots, left = binding.entmax_attn_paged_tables(dev([4, 20]), dev([0, -1]), dev([[1, 0], [0, 5]]), dev([3, 2, 7, 7]), dev([2]), 16, 6, 0,
                                                               status=status)
    assert int(status[0]) == 0
    assert kv.tolist() == [4, 0] and cu.tolist() == [0, 0, 0] and left.tolist() == [4] and pos.numel() == slots.numel() == 0
