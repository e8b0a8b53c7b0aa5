"""Softmax attention in training: entmax_attn_softmax_fwd / _bwd, entmax_attn_row_ranges and softmax_attention against the definition in 64 bits.

Tolerances: tests/softmax.py derives them element by element from the roundings the kernels make."""
import pytest
import torch

import softmax
from paper_2506_16640_b200 import autograd, binding

pytestmark = pytest.mark.gpu

bf16, f32 = torch.bfloat16, torch.float32


def _inputs(B, H, G, N, d, dtype=bf16, seed=0, sigma=1.0, layout="fused"):
    """q, k, v, d_o on the GPU; layout "fused": views of one projection [B, N, (H + 2 G) d]; "heads": contiguous [B, heads, N, d]."""
    g = torch.Generator().manual_seed(seed)
    if layout == "fused":
        qkv = (torch.randn((B, N, (H + 2 * G) * d), generator=g) * sigma).to(dtype).cuda()
        q, k, v = (x.view(B, N, -1, d).transpose(1, 2) for x in qkv.split([H * d, G * d, G * d], 2))
        d_o = torch.randn((B, N, H, d), generator=g).to(dtype).cuda().transpose(1, 2)
    else:
        q, k, v = ((torch.randn((B, n, N, d), generator=g) * sigma).to(dtype).cuda() for n in (H, G, G))
        d_o = torch.randn((B, H, N, d), generator=g).to(dtype).cuda()
    return q, k, v, d_o


def _terms(kind, B, H, N, seed=0):
    g = torch.Generator().manual_seed(77 + seed)
    t = {}
    for word in kind.split("+"):
        if word == "cap":
            t["softcap"] = 20.0
        elif word == "lowcap":
            t["softcap"] = 1.5                                # most scores in the flat part
        elif word == "slopes":
            t["alibi_slopes"] = torch.where(torch.arange(H) % 2 == 0, 2.0 ** -(torch.arange(H) + 1.0), torch.zeros(H)).cuda()
        elif word == "length":
            t["beta"], t["gamma"], t["delta"] = (0.2 + 0.6 * torch.rand(H, generator=g).cuda() for _ in range(3))
        elif word == "rows":
            # scales of either sign, some 0
            c = torch.randn((B, H, N), generator=g) * 1.5
            t["c_rows"] = torch.where(torch.rand((B, H, N), generator=g) < 0.1, torch.zeros(()), c).cuda()
        elif word == "ranges":
            # anything: empty rows, single keys, beyond both ends, whole rows
            a = torch.randint(-3, N + 3, (B, N), generator=g)
            n = (torch.rand((B, N), generator=g) ** 2 * (N + 6)).long()
            n = torch.where(torch.rand((B, N), generator=g) < 0.15, torch.randint(-2, 2, (B, N), generator=g), n)
            t["row_ranges"] = torch.stack([a, a + n], -1).to(torch.int32).cuda()
    return t


def _want(q, k, v, causal, t, d_o=None, sm=None):
    cpu = lambda x: None if x is None else x.detach().cpu()  # noqa: E731
    return softmax.problem(cpu(q), cpu(k), cpu(v), causal, cpu(t.get("row_ranges")), cpu(t.get("beta")), cpu(t.get("gamma")), cpu(t.get("delta")),
                           cpu(t.get("c_rows")), cpu(t.get("alibi_slopes")), t.get("softcap", 0.0), sm, cpu(d_o))


def _forward(q, k, v, causal, t, **kw):
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    out = binding.entmax_attn_softmax_fwd(q, k, v, causal, status=status, **t, **kw)
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    return out


def _backward(q, k, v, o, lse, d_o, causal, t, **kw):
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    out = binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, causal, status=status, want_scale_rows=True, want_param_grads="beta" in t, **t, **kw)
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    return out


def _both_ways(q, k, v, d_o, causal, t, sm=None, context=""):
    kw = {} if sm is None else {"sm_scale": sm}
    o, lse = _forward(q, k, v, causal, t, **kw)
    dq, dk, dv, dc, params = _backward(q, k, v, o, lse, d_o, causal, t, **kw)
    want = _want(q, k, v, causal, t, d_o, sm)
    for name, x in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv), ("dc", dc)):
        softmax.check(name, x, want, context)
    if params is not None:
        for name, x in zip(("dbeta", "dgamma", "ddelta"), params):
            softmax.check(name, x, want, context)
    return o, lse, dq, dk, dv, dc


SIZES = [(1, 1, 1, 1, 64), (2, 3, 1, 2, 128), (1, 2, 2, 63, 64), (1, 4, 2, 128, 128), (1, 2, 1, 129, 64), (2, 2, 2, 257, 128), (1, 6, 2, 300, 64),
         (1, 3, 3, 520, 128), (3, 8, 1, 150, 64)]


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("B,H,G,N,d", SIZES)
@pytest.mark.parametrize("causal", [True, False])
def test_sizes(B, H, G, N, d, causal, dtype):
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype, seed=N)
    _both_ways(q, k, v, d_o, causal, {})


@pytest.mark.parametrize("B,H,G,N,d", [(500, 4, 2, 1, 64), (260, 3, 3, 3, 128)])
def test_many_short_sequences(B, H, G, N, d):
    q, k, v, d_o = _inputs(B, H, G, N, d, bf16, seed=B)
    _both_ways(q, k, v, d_o, True, {})


KINDS = ["cap", "lowcap", "slopes", "length", "rows", "ranges", "cap+slopes+length", "ranges+rows+cap", "ranges+slopes+length", "rows+slopes"]


@pytest.mark.parametrize("dtype", [bf16, f32])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("B,H,G,N,d", [(2, 2, 1, 200, 64), (1, 4, 4, 390, 128)])
def test_terms(B, H, G, N, d, kind, dtype):
    q, k, v, d_o = _inputs(B, H, G, N, d, dtype, seed=len(kind))
    _both_ways(q, k, v, d_o, "ranges" not in kind, _terms(kind, B, H, N))


@pytest.mark.parametrize("kind", ["ranges", "ranges+cap+slopes+length"])
def test_ranges_under_the_causal_mask(kind):
    q, k, v, d_o = _inputs(2, 2, 2, 333, 64, seed=5)
    _both_ways(q, k, v, d_o, True, _terms(kind, 2, 2, 333))


@pytest.mark.parametrize("d", [64, 128])
def test_large_and_small_scores(d):
    # scores in the thousands: one-hot rows and exact ties; scores near 0: uniform rows
    for sigma in (0.01, 6.0, 30.0):
        q, k, v, d_o = _inputs(1, 2, 1, 260, d, seed=9, sigma=sigma)
        _both_ways(q, k, v, d_o, True, {}, context="sigma %g" % sigma)


@pytest.mark.parametrize("sm", [1.0, 0.013])
def test_given_scale(sm):
    q, k, v, d_o = _inputs(1, 2, 1, 140, 64, seed=3)
    _both_ways(q, k, v, d_o, True, _terms("cap+slopes+rows", 1, 2, 140), sm=sm)


def test_rows_that_rise_late():
    # the largest scores come last (and first): every tile raises a row's maximum
    B, H, N, d = 1, 2, 700, 64
    for order in (1, -1):
        q, k, v, d_o = _inputs(B, H, H, N, d, seed=4, layout="heads")
        ramp = torch.linspace(0.02, 6.0, N).cuda()[::order] if order == 1 else torch.linspace(6.0, 0.02, N).cuda()
        k = (q[:, :, :1].float() * ramp[None, None, :, None]).to(bf16)
        q = q[:, :, :1].expand(-1, -1, N, -1).contiguous()
        _both_ways(q, k, v, d_o, False, {}, context=str(order))


@pytest.mark.parametrize("dtype", [bf16, f32])
def test_every_row_empty(dtype):
    q, k, v, d_o = _inputs(2, 2, 1, 150, 64, dtype)
    t = {"row_ranges": torch.zeros((2, 150, 2), dtype=torch.int32, device="cuda"), **_terms("length", 2, 2, 150)}
    o, lse = _forward(q, k, v, False, t)
    assert (o == 0).all() and (lse == -float("inf")).all()
    for x in _backward(q, k, v, o, lse, d_o, False, t)[:4]:
        assert (x == 0).all()


@pytest.mark.parametrize("N,docs", [(1, [0, 1]), (200, [0, 7, 7, 130, 190, 190]), (300, [10, 140, 300]), (260, [0, 260])])
@pytest.mark.parametrize("causal,prefix,window", [(True, False, 0), (True, True, 0), (True, True, 20), (True, False, 5), (False, False, 0),
                                                  (False, False, 9)])
def test_row_ranges(N, docs, causal, prefix, window):
    cu = torch.tensor([docs, [min(x, N // 2) for x in docs]], dtype=torch.int32)
    pre = torch.tensor([[3, 0, 50, 1000, 2][:len(docs) - 1]] * 2, dtype=torch.int32) if prefix else None
    got = binding.entmax_attn_row_ranges(cu.cuda(), N, causal, prefix_len=None if pre is None else pre.cuda(), window=window).cpu()
    for b in range(2):
        want = [(0, 0)] * N
        for e in range(len(docs) - 1):
            first, last = int(cu[b, e]), int(cu[b, e + 1])
            for i in range(first, last):
                w = window or N
                lo = max(first, i - w + 1)
                hi = max(i + 1, min(last, first + int(pre[b, e])) if prefix else 0) if causal else min(last, i + w)
                want[i] = (lo, hi)
        assert got[b].tolist() == [list(x) for x in want]


def test_documents_equal_the_documents_alone():
    # packed documents give each what it gets by itself
    lengths, d, H, G = [40, 1, 200, 129], 64, 4, 2
    N = sum(lengths) + 17
    q, k, v, d_o = _inputs(1, H, G, N, d, seed=8)
    cu = torch.tensor([[0, 40, 41, 241, 370]], dtype=torch.int32, device="cuda")
    t = {"row_ranges": binding.entmax_attn_row_ranges(cu, N, True), **_terms("length+cap", 1, H, N)}
    o, lse = _forward(q, k, v, False, t)
    got = _backward(q, k, v, o, lse, d_o, False, t)
    del t["row_ranges"]
    at = 0
    for n in lengths:
        s = slice(at, at + n)
        one = softmax.problem(*(x[:, :, s].cpu() for x in (q, k, v)), True, None, t["beta"].cpu(), t["gamma"].cpu(), t["delta"].cpu(), None, None,
                              t["softcap"], None, d_o[:, :, s].cpu())
        for name, x in (("o", o), ("lse", lse), ("dq", got[0]), ("dk", got[1]), ("dv", got[2])):
            softmax.check(name, x[:, :, s], one, "document of %d" % n)
        at += n
    for x in (o, *got[:4]):
        assert (x[:, :, at:] == 0).all()


def test_outputs_with_strides_between_canaries():
    B, H, G, N, d = 2, 3, 1, 131, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=2)
    t = _terms("cap+length", B, H, N)
    o, lse = _forward(q, k, v, True, t)
    ref = _backward(q, k, v, o, lse, d_o, True, t)

    def room(heads):
        pool = torch.full((B, N + 2, heads + 2, d + 8), 7.0, dtype=bf16, device="cuda")
        return pool, pool[:, 1:-1, 1:-1, :d].transpose(1, 2)

    def untouched(pool, view):
        view.fill_(7.0)
        return bool((pool == 7.0).all())

    po, vo = room(H)
    o2, _ = _forward(q, k, v, True, t, o=vo)
    assert torch.equal(o2, o)
    (pq, vq), (pk, vk), (pv, vv) = room(H), room(G), room(G)
    nbytes = 1 << 22
    ws = torch.full((nbytes,), 0xff, dtype=torch.uint8, device="cuda")      # NaN everywhere
    got = _backward(q, k, v, o2, lse, d_o, True, t, dq=vq, dk=vk, dv=vv, workspace=ws)
    for x, y in zip(got[:4], ref[:4]):
        assert torch.equal(x, y)
    for p_, v_ in ((po, vo), (pq, vq), (pk, vk), (pv, vv)):
        assert untouched(p_, v_)


@pytest.mark.parametrize("B,H,G,N,d", [(1, 4, 2, 900, 128), (2, 4, 1, 513, 64)])
def test_repeats_are_bit_equal(B, H, G, N, d):
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=6)
    t = _terms("length+cap", B, H, N)
    o, lse = _forward(q, k, v, True, t)
    first = (o, lse, *_backward(q, k, v, o, lse, d_o, True, t)[:4])
    for _ in range(3):
        o2, lse2 = _forward(q, k, v, True, t)
        for x, y in zip(first, (o2, lse2, *_backward(q, k, v, o2, lse2, d_o, True, t)[:4])):
            assert torch.equal(x, y)


def test_autograd():
    B, H, G, N, d = 2, 4, 2, 130, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=12)
    t = _terms("length+cap+slopes", B, H, N)
    leaves = [x.detach().requires_grad_(True) for x in (q, k, v, t["beta"], t["gamma"], t["delta"])]
    o, lse = autograd.softmax_attention(*leaves, alibi_slopes=t["alibi_slopes"], softcap=t["softcap"], return_lse=True)
    got = torch.autograd.grad(o, leaves, d_o)
    want = _want(q, k, v, True, t, d_o)
    for name, x in zip(("dq", "dk", "dv", "dbeta", "dgamma", "ddelta"), got):
        softmax.check(name, x, want)
    # a gradient that is broadcast, and one with respect to the table of scales
    c = (0.5 + torch.rand((B, H, N), device="cuda")).requires_grad_(True)
    o = autograd.softmax_attention(leaves[0], leaves[1], leaves[2], c_rows=c)
    got = torch.autograd.grad(o.float().sum(), leaves[:3] + [c])
    want = _want(q, k, v, True, {"c_rows": c}, torch.ones_like(o))
    for name, x in zip(("dq", "dk", "dv", "dc"), got):
        softmax.check(name, x, want)


def test_no_second_derivatives_and_no_broadcast_inputs():
    q, k, v, _ = _inputs(1, 2, 2, 40, 64, seed=14)
    leaves = [x.detach().requires_grad_(True) for x in (q, k, v)]
    (dq,) = torch.autograd.grad(autograd.softmax_attention(*leaves).float().square().sum(), leaves[:1], create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dq.float().sum(), leaves)
    with pytest.raises(binding.EntmaxAttnError):
        autograd.softmax_attention(q, k[:, :1].expand(1, 2, 40, 64), v)


def test_autograd_against_differences():
    # the directional derivative of a smooth loss in float32 against central differences in 64 bits of the definition
    B, H, G, N, d = 1, 2, 1, 70, 64
    q, k, v, d_o = _inputs(B, H, G, N, d, f32, seed=13)
    t = _terms("cap+length+slopes", B, H, N)
    leaves = [x.detach().contiguous().requires_grad_(True) for x in (q, k, v, t["beta"], t["gamma"], t["delta"])]
    o = autograd.softmax_attention(*leaves, alibi_slopes=t["alibi_slopes"], softcap=t["softcap"])
    got = torch.autograd.grad(o, leaves, d_o)
    g = torch.Generator().manual_seed(1)
    names = ("q", "k", "v", "beta", "gamma", "delta")
    base = {n: x.detach().cpu().double() for n, x in zip(names, leaves)}
    for which, name in enumerate(names):
        way = torch.randn(base[name].shape, generator=g, dtype=torch.float64)

        def loss(step):
            at = dict(base)
            at[name] = base[name] + step * way
            w = softmax.problem(at["q"], at["k"], at["v"], True, None, at["beta"], at["gamma"], at["delta"], None, t["alibi_slopes"].cpu(), t["softcap"])
            return (w["o"] * d_o.cpu().double()).sum()

        # steps of 1e-4: the third derivative's share is 1e-8 of it, the difference's rounding 1e-12 / 1e-4
        want = float((loss(1e-4) - loss(-1e-4)) / 2e-4)
        have = float((got[which].cpu().double() * way).sum())
        size = float((got[which].cpu().double().abs() * way.abs()).sum())
        assert abs(have - want) <= 1e-4 * size + 1e-6, (name, have, want)


def test_graph_replay_and_second_stream():
    B, H, G, N, d = 1, 4, 2, 400, 128
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=20)
    t = _terms("length+cap", B, H, N)
    o, lse = _forward(q, k, v, True, t)
    ref = (o, lse, *_backward(q, k, v, o, lse, d_o, True, t)[:4])
    out = [torch.empty_like(x) for x in ref]
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        binding.entmax_attn_softmax_fwd(q, k, v, True, **t, o=out[0], lse=out[1])
        binding.entmax_attn_softmax_bwd(q, k, v, out[0], out[1], d_o, True, **t, want_param_grads=True, dq=out[2], dk=out[3], dv=out[4],
                                        d_scale_rows=out[5], workspace=ws)
    for _ in range(2):
        for x in out:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(out, ref):
            assert torch.equal(x, y)
    # the stream argument alone, with the calls' own memory
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    o2, lse2 = binding.entmax_attn_softmax_fwd(q, k, v, True, **t, stream=other)
    got = binding.entmax_attn_softmax_bwd(q, k, v, o2, lse2, d_o, True, **t, want_scale_rows=True, stream=other)
    other.synchronize()
    for x, y in zip((o2, lse2, *got[:4]), ref):
        assert torch.equal(x, y)


def test_training_step_captured():
    # (the captured step has leaves of its own: where an eager graph of the same leaves lives, PyTorch adds up their gradients on that
    # graph's stream and ends the capture)
    q, k, v, d_o = _inputs(1, 2, 2, 200, 64, seed=21)
    eager = [x.detach().requires_grad_(True) for x in (q, k, v)]
    alive = autograd.softmax_attention(*eager)
    want = torch.autograd.grad(autograd.softmax_attention(*eager), eager, d_o)
    torch.cuda.synchronize()
    leaves = [x.detach().requires_grad_(True) for x in (q, k, v)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = autograd.softmax_attention(*leaves)
        got = torch.autograd.grad(o, leaves, d_o)
    for x in got:
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert torch.equal(alive, o)


def test_long_rows_by_sample():
    # 5000 tokens: a few rows and keys of the whole against the definition
    B, H, G, N, d = 1, 2, 1, 5003, 128
    q, k, v, d_o = _inputs(B, H, G, N, d, seed=30)
    o, lse = _forward(q, k, v, True, {})
    dq, dk, dv, dc, _ = _backward(q, k, v, o, lse, d_o, True, {})
    want = _want(q[:, :, :], k, v, True, {}, d_o)
    for name, x in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv), ("dc", dc)):
        softmax.check(name, x, want)


def test_refusals():
    q, k, v, d_o = _inputs(1, 4, 2, 40, 64)
    E = binding.EntmaxAttnError
    fwd = binding.entmax_attn_softmax_fwd
    with pytest.raises(E):
        fwd(q.half(), k.half(), v.half(), True)
    with pytest.raises(E):
        fwd(q, k.float(), v, True)
    with pytest.raises(E):
        fwd(q, k[:, :, :30], v, True)
    with pytest.raises(E):
        fwd(q[:, :3], k, v, True)
    with pytest.raises(E):
        fwd(q[..., :32], k[..., :32], v[..., :32], True)
    with pytest.raises(E):
        fwd(q.cpu(), k.cpu(), v.cpu(), True)
    with pytest.raises(E):
        fwd(q, k[:, :1].expand(-1, 2, -1, -1), v, True)          # a head stride of 0
    with pytest.raises(E):
        fwd(q, k, v, True, beta=torch.ones(4, device="cuda"))
    with pytest.raises(E):
        fwd(q, k, v, True, softcap=-1.0)
    with pytest.raises(E):
        fwd(q, k, v, True, softcap=float("nan"))
    with pytest.raises(E):
        fwd(q, k, v, True, sm_scale=float("inf"))
    with pytest.raises(E):
        fwd(q, k, v, True, c_rows=torch.ones((1, 4, 41), device="cuda"))
    with pytest.raises(E):
        fwd(q, k, v, False, row_ranges=torch.zeros((1, 40, 2), dtype=torch.int64, device="cuda"))
    ones = torch.ones(4, device="cuda")
    with pytest.raises(E):
        fwd(q, k, v, True, ones, ones, ones, c_rows=torch.ones((1, 4, 40), device="cuda"))
    o, lse = fwd(q, k, v, True)
    with pytest.raises(E):
        binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, True, want_param_grads=True)
    with pytest.raises(E):
        binding.entmax_attn_softmax_bwd(q, k, v, o, lse, d_o, True, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(E):
        binding.entmax_attn_softmax_bwd(q, k, v, o, lse[:, :2], d_o, True)
    cu = torch.tensor([[0, 40]], dtype=torch.int32, device="cuda")
    with pytest.raises(E):
        binding.entmax_attn_row_ranges(cu, 40, False, prefix_len=torch.ones((1, 1), dtype=torch.int32, device="cuda"))
    with pytest.raises(E):
        binding.entmax_attn_row_ranges(cu, 40, True, window=-1)
    with pytest.raises(E):
        binding.entmax_attn_row_ranges(cu.long(), 40, True)
