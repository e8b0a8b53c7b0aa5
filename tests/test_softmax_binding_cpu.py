"""Refusals of the softmax attention binding that come before any device work."""
import pytest
import torch

from paper_2506_16640_b200 import binding
from paper_2506_16640_b200 import build as lib_build


@pytest.fixture(scope="module", autouse=True)
def lib():
    lib_build.build()


@pytest.mark.parametrize("given", [(), ("beta",), ("beta", "gamma"), ("gamma", "delta")])
def test_parameter_gradients_need_all_three_parameters(given):
    q, k, v, o, d_o = (torch.zeros((1, 2, 5, 64), dtype=torch.bfloat16) for _ in range(5))
    with pytest.raises(binding.EntmaxAttnError, match="scale parameters"):
        binding.entmax_attn_softmax_bwd(q, k, v, o, torch.zeros((1, 2, 5)), d_o, True, want_param_grads=True, **{n: torch.ones(2) for n in given})
