"""Softmax attention, its paged form and the serving tables without a GPU: refusals before any device work, and the 64-bit reference's own pins."""
import ctypes
import math

import pytest
import torch

import softmax
from paper_2506_16640_b200 import build as lib_build


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    from paper_2506_16640_b200 import binding
    return binding.load()


X = ctypes.c_void_p(1 << 20)                  # never dereferenced: every call here is refused
SHAPE, ALPHA, DTYPE, ALIGN, WORKSPACE, NULL = -1, -2, -3, -4, -5, -6


def _params(**kw):
    from paper_2506_16640_b200.binding import SoftmaxParams, Strides
    base = dict(batch=2, heads=4, kv_heads=2, seq=33, head_dim=64, dtype=0, causal=1, sm_scale=0.0, softcap=0.0)
    strides = {n: Strides(*kw.pop(n, (0, 0, 0))) for n in "qkvo"}
    base.update(kw)
    return SoftmaxParams(**base, **strides)


BAD = [(dict(batch=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(seq=0), SHAPE),
       (dict(head_dim=96), SHAPE), (dict(seq=1 << 30), SHAPE), (dict(dtype=2), DTYPE), (dict(sm_scale=-1.0), ALPHA), (dict(sm_scale=math.nan), ALPHA),
       (dict(softcap=-1.0), ALPHA), (dict(softcap=math.inf), ALPHA), (dict(softcap=1e-38, sm_scale=1e38), ALPHA), (dict(q=(8448, 2112, 60)), SHAPE),
       (dict(k=(4224, 2112, 68)), SHAPE), (dict(v=(4224, 0, 64)), SHAPE), (dict(o=(0, 2112, 64)), SHAPE)]


def _fwd(lib, p, terms=None, q=X, lse=X):
    return lib.entmax_attn_softmax_fwd(ctypes.byref(p), q, X, X, None if terms is None else ctypes.byref(terms), X, lse, None, None)


def test_forward_refusals(lib):
    from paper_2506_16640_b200.binding import SoftmaxTerms
    for kw, rc in BAD:
        assert _fwd(lib, _params(**kw)) == rc, kw
        assert lib.entmax_attn_softmax_workspace_bytes(ctypes.byref(_params(**kw))) == 0, kw
    assert _fwd(lib, _params(), q=None) == NULL
    assert _fwd(lib, _params(), q=ctypes.c_void_p((1 << 20) + 8)) == ALIGN
    assert _fwd(lib, _params(), lse=ctypes.c_void_p((1 << 20) + 2)) == ALIGN
    assert _fwd(lib, _params(), SoftmaxTerms(beta=1 << 20)) == NULL
    assert _fwd(lib, _params(), SoftmaxTerms(beta=1 << 20, gamma=1 << 20, delta=1 << 20, c_rows=1 << 20)) == NULL
    assert _fwd(lib, _params(), SoftmaxTerms(row_ranges=(1 << 20) + 4)) == ALIGN
    assert _fwd(lib, _params(), SoftmaxTerms(alibi_slopes=(1 << 20) + 1)) == ALIGN
    assert lib.entmax_attn_softmax_fwd(None, X, X, X, None, X, X, None, None) == NULL


def test_sizes_beyond_the_launches_are_refused(lib):
    assert _fwd(lib, _params(heads=1 << 28, kv_heads=1, batch=1, seq=1)) == SHAPE
    assert _fwd(lib, _params(heads=1 << 10, kv_heads=1, batch=1 << 10, seq=1 << 10)) == SHAPE


def test_backward_refusals(lib):
    from paper_2506_16640_b200.binding import SoftmaxGrads, SoftmaxTerms, Strides
    p = _params()
    size = lib.entmax_attn_softmax_workspace_bytes(ctypes.byref(p))
    assert size > 0 and size % 256 == 0

    def bwd(grads, terms=None, ws=X, nbytes=size, d_o=X):
        return lib.entmax_attn_softmax_bwd(ctypes.byref(p), X, X, X, None if terms is None else ctypes.byref(terms), X, X, d_o,
                                           None if grads is None else ctypes.byref(grads), X, X, X, ws, nbytes, None, None)

    assert bwd(None) == NULL
    assert bwd(SoftmaxGrads(), d_o=None) == NULL
    assert bwd(SoftmaxGrads(dbeta=1 << 20)) == NULL
    assert bwd(SoftmaxGrads(dbeta=1 << 20, dgamma=1 << 20, ddelta=1 << 20)) == NULL         # no scale to differentiate
    assert bwd(SoftmaxGrads(dq=Strides(0, 2112, 64))) == SHAPE
    assert bwd(SoftmaxGrads(d_o=Strides(8448, 2112, 63))) == SHAPE
    assert bwd(SoftmaxGrads(), ws=None) == WORKSPACE
    assert bwd(SoftmaxGrads(), ws=ctypes.c_void_p((1 << 20) + 128)) == WORKSPACE
    assert bwd(SoftmaxGrads(), nbytes=size - 1) == WORKSPACE
    assert bwd(SoftmaxGrads(), SoftmaxTerms(gamma=1 << 20)) == NULL


def test_row_ranges_refusals(lib):
    call = lambda B=1, N=8, docs=2, causal=1, window=0, cu=X, pre=None, out=X: lib.entmax_attn_row_ranges(B, N, docs, causal, window, cu, pre, out, None)  # noqa: E731
    assert call(B=0) == SHAPE and call(N=0) == SHAPE and call(docs=0) == SHAPE and call(window=-1) == SHAPE and call(B=1 << 15, N=1 << 15) == SHAPE
    assert call(causal=0, pre=X) == SHAPE
    assert call(cu=None) == NULL and call(out=None) == NULL
    assert call(out=ctypes.c_void_p((1 << 20) + 4)) == ALIGN and call(cu=ctypes.c_void_p((1 << 20) + 2)) == ALIGN


def _cache(**kw):
    from paper_2506_16640_b200.binding import PagedCache
    base = dict(batch=3, kv_heads=2, head_dim=64, page_size=16, num_pages=100, max_pages=20, table_stride=20, stride_page=16 * 128,
                stride_token=128, stride_head=64)
    base.update(kw)
    return PagedCache(**base)


def _paged(**kw):
    from paper_2506_16640_b200.binding import SoftmaxPagedParams
    base = dict(total_q=3, q_heads=4, max_q_len=0, max_kv_len=0, window=0, softcap=0.0, sm_scale=0.0, q_stride_t=256, q_stride_h=64)
    base.update(kw)
    return SoftmaxPagedParams(**base)


BAD_CACHES = [dict(batch=0), dict(kv_heads=0), dict(head_dim=96), dict(page_size=8), dict(page_size=48), dict(num_pages=0), dict(max_pages=0),
              dict(table_stride=19), dict(stride_page=1028), dict(stride_token=4), dict(stride_head=0)]
BAD_PAGED = [dict(total_q=0), dict(q_heads=0), dict(q_heads=3), dict(q_heads=2 * 129), dict(sm_scale=-1.0), dict(softcap=-1.0), dict(softcap=math.nan),
             dict(window=-1), dict(max_q_len=-1), dict(max_kv_len=-1), dict(q_stride_t=252), dict(q_stride_h=8), dict(total_q=1 << 30)]


def test_paged_refusals(lib):
    size = lambda c, p, uniform=0: lib.entmax_attn_softmax_paged_workspace_bytes(ctypes.byref(c), ctypes.byref(p), uniform)  # noqa: E731

    def fwd(c, p, q=X, cu=X, beta=None, ws=X, nbytes=1 << 40):
        return lib.entmax_attn_softmax_paged_fwd(ctypes.byref(c), ctypes.byref(p), q, X, X, cu, X, X, beta, None, None, None, X, X, ws, nbytes, None, None)

    assert size(_cache(), _paged()) > 0 and size(_cache(), _paged(), 1) > 0
    assert size(_cache(), _paged(total_q=4), 1) == 0          # four tokens over three sequences
    for kw in BAD_CACHES:
        assert size(_cache(**kw), _paged()) == 0 and fwd(_cache(**kw), _paged()) == SHAPE, kw
    for kw in BAD_PAGED:
        assert size(_cache(), _paged(**kw)) == 0 and fwd(_cache(), _paged(**kw)) in (SHAPE, ALPHA), kw
    assert fwd(_cache(), _paged(), q=None) == NULL
    assert fwd(_cache(), _paged(), beta=X) == NULL
    assert fwd(_cache(), _paged(), q=ctypes.c_void_p((1 << 20) + 8)) == ALIGN
    assert fwd(_cache(), _paged(), cu=ctypes.c_void_p((1 << 20) + 1)) == ALIGN
    assert fwd(_cache(), _paged(), ws=None) == WORKSPACE
    assert fwd(_cache(), _paged(), nbytes=size(_cache(), _paged()) - 1) == WORKSPACE
    assert fwd(_cache(), _paged(total_q=4), cu=None) == SHAPE


def test_tables_refusals(lib):
    from paper_2506_16640_b200.binding import PagedTablesParams

    def call(kv=X, slots=X, free=X, count=X, **kw):
        base = dict(batch=3, total_q=5, page_size=16, num_pages=10, max_pages=4, free_capacity=10, table_stride=4)
        base.update(kw)
        return lib.entmax_attn_paged_tables(ctypes.byref(PagedTablesParams(**base)), kv, X, X, free, count, X, X, X, slots, X, None, None)

    for kw in (dict(batch=0), dict(total_q=-1), dict(page_size=8), dict(page_size=24), dict(num_pages=0), dict(max_pages=0), dict(free_capacity=-1),
               dict(table_stride=3), dict(max_pages=1 << 21, table_stride=1 << 21)):
        assert call(**kw) == SHAPE, kw
    assert call(kv=None) == NULL and call(count=None) == NULL and call(free=None) == NULL
    assert call(kv=ctypes.c_void_p((1 << 20) + 2)) == ALIGN and call(slots=ctypes.c_void_p((1 << 20) + 4)) == ALIGN


@pytest.mark.parametrize("cap,slope,scaled", [(0.0, 0.0, False), (3.0, 0.0, True), (0.0, 0.3, True), (2.0, 0.1, False)])
def test_reference_gradients_are_autograds(cap, slope, scaled):
    g = torch.Generator().manual_seed(0)
    n, d = 23, 16
    q, k, v, do = (torch.randn((n, d), generator=g, dtype=torch.float64) for _ in range(4))
    c = torch.randn(n, generator=g, dtype=torch.float64) if scaled else torch.ones(n, dtype=torch.float64)
    lo = torch.randint(0, n, (n,), generator=g)
    hi = torch.minimum(lo + torch.randint(0, n, (n,), generator=g), torch.tensor(n))
    leaves = [x.clone().requires_grad_(True) for x in (q, k, v, c)]
    z = leaves[0] @ leaves[1].T / math.sqrt(d)
    if cap:
        z = cap * torch.tanh(z / cap)
    j = torch.arange(n)
    s = (z - slope * (j[:, None] - j).abs().double()) * leaves[3][:, None]
    sees = (j >= lo[:, None]) & (j < hi[:, None])
    w = torch.where(sees, torch.exp(s), 0.0)
    o = (w @ leaves[2]) / w.sum(1, keepdim=True).clamp_min(1e-300)
    want = torch.autograd.grad(o, leaves, do)
    got = softmax.head(q, k, v, lo, hi, c, None, cap, slope, do, bf16=False)
    assert torch.allclose(got["o"], o.detach(), atol=1e-12)
    for name, x in zip(("dq", "dk", "dv", "dc"), want):
        assert torch.allclose(got[name], x, atol=1e-11), name
    assert (got["lse"][lo >= hi] == -math.inf).all() and (got["o"][lo >= hi] == 0).all()


def test_reference_scale_gradients_are_autograds():
    g = torch.Generator().manual_seed(1)
    n = torch.arange(0, 40)
    leaf = [torch.tensor(x, dtype=torch.float64, requires_grad=True) for x in (0.7, 0.6, 0.9)]
    dc = torch.randn(40, generator=g, dtype=torch.float64)
    want = torch.autograd.grad((softmax.scale(*leaf, n) * dc).sum(), leaf)
    got = softmax.scale_grads(dc, leaf[0].detach(), leaf[1].detach(), n)
    for x, y in zip(got, want):
        assert torch.allclose(x, y)


def test_reference_two_keys_in_closed_form():
    q = torch.tensor([[1.0, 0.0]])
    k, v = torch.tensor([[2.0, 0.0], [0.0, 5.0]]), torch.tensor([[1.0, 0.0], [0.0, 1.0]])
    got = softmax.head(q, k, v, torch.tensor([0]), torch.tensor([2]), sm=0.5, bf16=False)
    p = 1 / (1 + math.exp(-1.0))
    assert torch.allclose(got["o"], torch.tensor([[p, 1 - p]], dtype=torch.float64))
    assert abs(float(got["lse"]) - math.log(math.e + 1)) < 1e-12
