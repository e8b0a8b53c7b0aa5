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


@pytest.mark.parametrize("name", ["sm_scale", "softcap"])
def test_scales_and_caps_beyond_float32_s_room(name):
    # with a cap of 1e37 c times the cap overflows, with one of 1e-33 what a slope is in its units times the least factor is no longer small
    import ctypes
    lib = binding.load()
    strides = [binding.Strides(0, 0, 0)] * 4
    for value, fits in ((2.0 ** 100, True), (1.3e30, False), (3e38, False), (float("inf"), False), (float("nan"), False), (2.0 ** -100, True), (7e-31, False),
                        (1e-38, False), (-1.0, False), (0.0, True), (50.0, True)):
        both = dict(sm_scale=0.0, softcap=0.0)
        both[name] = value
        dense = binding.SoftmaxParams(1, 2, 2, 5, 64, 0, 1, both["sm_scale"], both["softcap"], *strides)
        assert (lib.entmax_attn_softmax_workspace_bytes(ctypes.byref(dense)) > 0) == fits, value
        cache = binding.PagedCache(batch=1, kv_heads=2, head_dim=64, page_size=16, num_pages=4, max_pages=4, table_stride=4, stride_page=2048, stride_token=128,
                                   stride_head=64)
        paged = binding.SoftmaxPagedParams(1, 2, 0, 0, 0, both["softcap"], both["sm_scale"], 128, 64)
        assert (lib.entmax_attn_softmax_paged_workspace_bytes(ctypes.byref(cache), ctypes.byref(paged), 0) > 0) == fits, value
