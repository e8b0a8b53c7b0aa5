"""Softmax attention (the alpha = 1 member of the family) in training and in serving, and the tables serving needs, as timed cases.

    op "train"   softmax_attention through torch autograd: a training step's forward and backward pass of one layer
    op "eval"    entmax_attn_softmax_fwd: the forward pass alone
    op "attend"  entmax_attn_softmax_paged_fwd: new tokens attend to everything a paged cache holds of their sequences
    op "tables"  entmax_attn_paged_tables: lengths, block table, positions and slots of a serving step from the requests' lengths

Attention cases: z = <q,k> / sqrt(d), x = cap tanh(z / cap) - m |i - j| (cap = 0: not capped; slopes m with `alibi`), scores c x with
    scale  "none"    c = 1
           "length"  c = delta + beta (ln n)^gamma, n the number of keys a row sees, beta, gamma, delta ~ U per head
           "rows"    a table c[b, h, i] that the model projects from the layer input (training only)
    mask   "causal"  j <= i;  "docs"  several documents packed into a row, padding behind them;  "prefix"  documents whose first tokens are seen by
           all of the document;  `window` > 0: only the last `window` keys
Paged cases: `batch` sequences of up to `kv` tokens, `chunks` of them bring up to `new` tokens, the others one; `page` tokens to a page.
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _attn(name, op, B, N, heads, kv_heads, d, *, scale="none", mask="causal", cap=0.0, alibi=False, window=0):
    c = dict(op=op, B=B, N=N, heads=heads, kv_heads=kv_heads, d=d, scale=scale, mask=mask, cap=cap, alibi=alibi, window=window)
    return dict(c, name=name) if name else c


def _paged(name, batch, chunks, new, kv, heads, kv_heads, d, page, *, ragged=True, scale="none", cap=0.0, alibi=False, window=0):
    c = dict(op="attend", batch=batch, chunks=chunks, new=new, kv=kv, heads=heads, kv_heads=kv_heads, d=d, page=page, ragged=ragged, scale=scale,
             cap=cap, alibi=alibi, window=window)
    return dict(c, name=name) if name else c


def _tables(name, batch, chunks, new, kv, page, *, room=1.0):
    c = dict(op="tables", batch=batch, chunks=chunks, new=new, kv=kv, page=page, room=room)
    return dict(c, name=name) if name else c


def listed():
    return [
        # a training step of a 12-head, 1024-token study with a learned length-dependent scale
        _attn("train_8x12x1024_d64_length", "train", 8, 1024, 12, 12, 64, scale="length"),
        # packed documents with padding, grouped heads, capped scores: a language model's layer
        _attn("train_docs_2x16x8192_d128_cap", "train", 2, 8192, 16, 4, 128, mask="docs", cap=50.0),
        # a long-context training step
        _attn("train_1x16x16384_d128", "train", 1, 16384, 16, 8, 128),
        # documents with a prefix that all of the document sees (instructions), slopes, an odd length
        _attn("train_prefix_3x12x1501_d64_alibi", "train", 3, 1501, 12, 4, 64, mask="prefix", alibi=True),
        # evaluation of a sliding-window layer on a long text
        _attn("eval_1x16x20011_d128_window", "eval", 1, 20011, 16, 8, 128, scale="rows", cap=30.0, window=4096),
        # one token of one conversation with a small model: nothing but latency
        _paged("decode_1x777_h12_d64", 1, 0, 1, 777, 12, 12, 64, 16),
        # a full decode batch of a grouped-head model, short contexts, learned scale
        _paged("decode_64x4096_h32_d128", 64, 0, 1, 4096, 32, 8, 128, 16, scale="length"),
        # long contexts, many query heads per K/V head, capped scores
        _paged("decode_8x65536_h32_d128_cap", 8, 0, 1, 65536, 32, 4, 128, 128, cap=50.0),
        # five proposed tokens of each sequence checked at once, half of the heads with slopes
        _paged("verify_32x5_kv8192_h32_d128", 32, 32, 5, 8192, 32, 8, 128, 32, ragged=False, alibi=True),
        # continuous batching: two prompts' chunks among single tokens, sliding window
        _paged("mixed_24_new500_kv9001_h16_d64", 24, 2, 500, 9001, 16, 4, 64, 16, window=4096),
        # tables of a step of a full decode batch
        _tables("tables_256x1", 256, 0, 1, 2048, 16),
        # tables of a step that starts many prompts among single tokens
        _tables("tables_1000_new900", 1000, 64, 900, 6000, 32),
    ]


_HEADS = [(12, 12), (12, 4), (16, 8), (16, 2), (16, 16), (32, 8), (32, 4), (8, 1), (6, 2), (10, 2)]
_PAIRS = 1 << 32          # padded (row, key) pairs of a drawn training case, at most; the largest listed one has as many
_PAGED_PAIRS = 1 << 30
_CACHE = 1 << 30          # elements of K of a drawn paged case, at most


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["train", "train", "eval", "decode", "few", "mixed", "chunk", "tables"])
    if kind == "tables":
        batch, kv = _log_int(rng, 1, 1024), _log_int(rng, 1, 16384)
        return _tables(None, batch, rng.randint(0, min(batch, 64)), _log_int(rng, 1, 1024), kv, rng.choice([16, 32, 64, 128]),
                       room=rng.choice([1.0, 1.0, 1.0, 0.6]))
    heads, kv_heads = rng.choice(_HEADS)
    d = rng.choice([64, 128])
    scale, cap, alibi = rng.choice(["none", "length", "rows"]), rng.choice([0.0, 0.0, 30.0, 50.0]), rng.random() < 0.25
    if kind in ("train", "eval"):
        N = _log_int(rng, 1, 24000)
        B = _log_int(rng, 1, 16)
        while B > 1 and B * heads * N * N > _PAIRS:
            B -= 1
        while heads * N * N > _PAIRS:
            N = N * 3 // 4
        return _attn(None, kind, B, N, heads, kv_heads, d, scale=scale, mask=rng.choice(["causal", "causal", "docs", "prefix"]), cap=cap,
                     alibi=alibi, window=_log_int(rng, 16, 8192) if rng.random() < 0.25 else 0)
    page = rng.choice([16, 16, 32, 64, 128, 256])
    batch = _log_int(rng, 1, 128)
    new = {"decode": 1, "few": rng.randint(2, 12)}.get(kind) or _log_int(rng, 13, 2048)
    kv = new + _log_int(rng, 1, 65536) - 1
    if kind == "chunk":
        batch = min(batch, 6)
    while batch > 1 and (batch * new * heads * kv > _PAGED_PAIRS or batch * kv * kv_heads * d > _CACHE):
        batch //= 2
    while batch * new * heads * kv > _PAGED_PAIRS:
        new = (new + 1) // 2
        kv = max(new, kv * 3 // 4)
    chunks = 0 if kind == "decode" else min(batch, 2) if kind == "mixed" else batch
    return _paged(None, batch, chunks, new, kv, heads, kv_heads, d, page, ragged=rng.random() < 0.8, scale="none" if scale == "rows" else scale,
                  cap=cap, alibi=alibi, window=_log_int(rng, 16, 8192) if rng.random() < 0.25 else 0)


# ------------------------------------------------------------------------------------------------------------ inputs
def _documents(case):
    """Boundaries of the documents of every batch row and their prefix lengths, part of the case: as many for every row, the last ones
    empty where a row has fewer; behind the last one padding."""
    rng = random.Random(case["B"] * 1000003 + case["N"])
    B, N = case["B"], case["N"]
    cu, prefix = [], []
    for _ in range(B):
        ends = [0]
        real = max(1, int(N * rng.uniform(0.85, 1.0)))
        while ends[-1] < real and len(ends) < 33:
            ends.append(min(real, ends[-1] + max(1, int(N * rng.betavariate(1.0, 4.0)))))
        cu.append(ends)
        prefix.append([int((b - a) * rng.uniform(0.0, 0.6)) for a, b in zip(ends, ends[1:])])
    most = max(len(c) for c in cu)
    cu = [c + [c[-1]] * (most - len(c)) for c in cu]
    prefix = [p + [0] * (most - 1 - len(p)) for p in prefix]
    return cu, prefix if case["mask"] == "prefix" else None


def _lengths(case):
    """New tokens and lengths (new ones included) of every sequence: part of the case, the same for every seed."""
    rng = random.Random(case["batch"] * 1000003 + case["kv"])
    ragged = case.get("ragged", True)
    new, kv = [], []
    for b in range(case["batch"]):
        n = case["new"] if b < case["chunks"] else 1
        total = max(case["kv"], n) if case["op"] == "tables" else case["kv"]
        if ragged and b > 0:
            total = max(1, int(total * rng.uniform(0.1, 1.0)))
            n = max(1, min(n, int(n * rng.uniform(0.3, 1.0)) + 1))
        new.append(min(n, total))
        kv.append(total)
    return new, kv


def _slopes(H):
    """Slopes on half of the heads, none on the others."""
    m = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H)
    return torch.where(torch.arange(H, device="cuda") % 2 == 0, m, torch.zeros_like(m))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    rand = lambda *s: torch.rand(s, generator=gen, device="cuda")  # noqa: E731
    s = dict(case)
    if case["op"] in ("train", "eval"):
        B, N, H, G, d = case["B"], case["N"], case["heads"], case["kv_heads"], case["d"]
        # views of a fused projection's output, as a layer has them: [B, N, heads, d] seen as [B, heads, N, d]
        qkv = randn(B, N, (H + 2 * G) * d)
        s["q"], s["k"], s["v"] = (x.view(B, N, -1, d).transpose(1, 2) for x in qkv.split([H * d, G * d, G * d], 2))
        s["leaves"] = [s["q"], s["k"], s["v"]]
        s["beta"] = s["gamma"] = s["delta"] = s["c_rows"] = None
        if case["scale"] == "length":
            s["beta"], s["gamma"], s["delta"] = 0.2 + 0.4 * rand(H), 0.3 + 0.4 * rand(H), 0.5 + 0.5 * rand(H)
            s["leaves"] += [s["beta"], s["gamma"], s["delta"]]
        elif case["scale"] == "rows":
            s["c_rows"] = 0.5 + rand(B, H, N)
            s["leaves"] += [s["c_rows"]]
        if case["op"] == "train":
            for x in s["leaves"]:
                x.requires_grad_(True)
            s["d_o"] = randn(B, N, H, d).transpose(1, 2)
        s["slopes"] = _slopes(H) if case["alibi"] else None
        s["cu"] = s["prefix"] = None
        if case["mask"] != "causal":
            cu, prefix = _documents(case)
            s["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
            s["prefix"] = torch.tensor(prefix, dtype=torch.int32, device="cuda") if prefix else None
        elif case["window"]:
            s["cu"] = torch.tensor([[0, N]] * B, dtype=torch.int32, device="cuda")
        return s
    new, kv = _lengths(case)
    B, ps = case["batch"], case["page"]
    need = [-(-n // ps) for n in kv]
    if case["op"] == "tables":
        old = [t - n for n, t in zip(new, kv)]
        have = [-(-n // ps) for n in old]
        n_pages = sum(need) + 3
        order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
        s["table"] = torch.zeros((B, max(need) + 1), dtype=torch.int32, device="cuda")
        at = 0
        for b, n in enumerate(have):
            s["table"][b, :n] = order[at:at + n]
            at += n
        s["free"] = order[at:].contiguous()
        s["free_count"] = torch.tensor([int((n_pages - at) * case["room"])], dtype=torch.int32, device="cuda")
        s["old"] = torch.tensor(old, dtype=torch.int32, device="cuda")
        s["new_len"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        return dict(s, T=sum(new), n_pages=n_pages)
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    T = sum(new)
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cu = torch.tensor([0] + [sum(new[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
    s.update(T=T, max_new=max(new), max_kv=max(kv), table=table, cu=cu, lens=torch.tensor(kv, dtype=torch.int32, device="cuda"))
    s["k_cache"], s["v_cache"] = randn(n_pages, ps, G, d), randn(n_pages, ps, G, d)
    s["q"] = randn(T, H, d)
    s["beta"] = s["gamma"] = s["delta"] = None
    if case["scale"] == "length":
        s["beta"], s["gamma"], s["delta"] = 0.2 + 0.4 * rand(H), 0.3 + 0.4 * rand(H), 0.5 + 0.5 * rand(H)
    s["slopes"] = _slopes(H) if case["alibi"] else None
    return s


# ------------------------------------------------------------------------------------------------- the plain forms
def _visible(s):
    """begin, end [B, N] of the keys every row sees."""
    N, i = s["N"], torch.arange(s["N"], device="cuda")
    if s["cu"] is None:
        return torch.zeros_like(i)[None], (i + 1)[None]
    cu = s["cu"].long()
    doc = torch.searchsorted(cu[:, 1:].contiguous(), i.expand(len(cu), N).contiguous(), right=True)
    real = doc < cu.shape[1] - 1
    doc = doc.clamp_max(cu.shape[1] - 2)
    first, last = cu.gather(1, doc), cu.gather(1, doc + 1)
    end = (i + 1).expand(len(cu), N)
    if s["prefix"] is not None:
        end = torch.maximum(end, torch.minimum(first + s["prefix"].long().gather(1, doc), last))
    begin = torch.maximum(first, i - s["window"] + 1) if s["window"] else first
    return torch.where(real, begin, 0), torch.where(real, end, 0)


def _length_scale(s, n, shape):
    """c of rows that see n keys (a float tensor), per head."""
    at = lambda x: x.detach().view(shape)  # noqa: E731
    grown = torch.where(n > 1, at(s["beta"]) * torch.log(n).clamp_min(1e-30).pow(at(s["gamma"])), 0.0)
    return at(s["delta"]) + grown


def _attention(s):
    B, N, H, G, d, cap = s["B"], s["N"], s["heads"], s["kv_heads"], s["d"], s["cap"]
    R, sm = H // G, 1.0 / math.sqrt(s["d"])
    q = s["q"].detach().float().reshape(B, G, R * N, d)
    k, v = s["k"].detach().float(), s["v"].detach().float()
    x = (q @ k.transpose(2, 3)).mul_(sm)                     # [B, G, R N, N]
    if cap:
        x.div_(cap).tanh_().mul_(cap)
    capped = x
    x = x.view(B, G, R, N, N)
    j = torch.arange(N, device="cuda")
    if s["slopes"] is not None:
        x = x - s["slopes"].view(G, R, 1, 1) * (j[:, None] - j).abs()
    begin, end = _visible(s)
    n = (end - begin).clamp_min(0).float()[:, None, None, :, None]
    c = None
    if s["beta"] is not None:
        c = _length_scale(s, n, (G, R, 1, 1))
    elif s["c_rows"] is not None:
        c = s["c_rows"].detach().view(B, G, R, N, 1)
    p = x * c if c is not None else x.clone()
    p.masked_fill_(((j < begin[..., None]) | (j >= end[..., None]))[:, None, None], float("-inf"))
    top = p.amax(-1, keepdim=True)
    top = torch.where(top > float("-inf"), top, 0.0)
    mass = p.sub_(top).exp_().sum(-1, keepdim=True)
    lse = (top + mass.log()).view(B, H, N)
    p.div_(torch.where(mass > 0, mass, 1.0))
    p2 = p.view(B, G, R * N, N)
    heads = lambda t: t.view(B, H, N, d).to(torch.bfloat16)  # noqa: E731
    o = heads(p2 @ v)
    if s["op"] == "eval":
        return o, lse
    g = s["d_o"].float().reshape(B, G, R * N, d)
    dv = p2.transpose(2, 3) @ g
    ds = (g @ v.transpose(2, 3)).view_as(p)
    ds.sub_(torch.einsum("bgrij,bgrij->bgri", p, ds)[..., None]).mul_(p)
    more = ()
    if c is not None:
        dc = torch.einsum("bgrij,bgrij->bgri", ds, x).view(B, H, N)
        ds.mul_(c)
        more = (dc,)
    if s["beta"] is not None:
        n = n.view(-1, 1, N)
        log_n = torch.log(n).clamp_min(1e-30)
        w = torch.where(n > 1, log_n.pow(s["gamma"].detach().view(H, 1)), 0.0)
        total = lambda t: t.double().sum((0, 2)).float()  # noqa: E731
        more = (total(dc * w), total(dc * w * s["beta"].detach().view(H, 1) * log_n.log()), total(dc))
    ds = ds.view(B, G, R * N, N)
    if cap:
        ds.mul_(capped.div_(cap).square_().neg_().add_(1.0))
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    return (o, lse, heads(dq.mul_(sm)), dk.mul_(sm).to(torch.bfloat16), dv.to(torch.bfloat16)) + more


def _tokens(s):
    """Sequence, position and number within the chunk of every new token."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    n = t - s["cu"][b]
    return b, s["lens"][b] - (s["cu"][b + 1] - s["cu"][b]) + n, n


def _attend(s):
    B, H, G, d, N, L = s["batch"], s["heads"], s["kv_heads"], s["d"], s["max_new"], s["max_kv"]
    R = H // G
    table = s["table"][:, :-(-L // s["page"])].long()
    k = s["k_cache"][table].view(B, -1, G, d)[:, :L].float().permute(0, 2, 3, 1)          # [B, G, d, L]
    v = s["v_cache"][table].view(B, -1, G, d)[:, :L].float().transpose(1, 2)              # [B, G, L, d]
    n = torch.arange(N, device="cuda")
    new = s["cu"][1:] - s["cu"][:-1]
    rows = (s["cu"][:-1, None] + n).clamp_max(s["T"] - 1)
    q = s["q"][rows].float().view(B, N, G, R, d).permute(0, 2, 3, 1, 4)                   # [B, G, R, N, d]
    pos = ((s["lens"] - new)[:, None] + n).clamp_max(L - 1)[:, None, None, :, None].float()   # [B, 1, 1, N, 1]
    x = (q.reshape(B, G, R * N, d) @ k).view(B, G, R, N, L).mul_(1.0 / math.sqrt(d))
    if s["cap"]:
        x.div_(s["cap"]).tanh_().mul_(s["cap"])
    j = torch.arange(L, device="cuda").float()
    if s["slopes"] is not None:
        x -= s["slopes"].view(G, R, 1, 1) * (pos - j)
    if s["beta"] is not None:
        sees = (pos + 1).clamp_max(s["window"]) if s["window"] else pos + 1
        x *= _length_scale(s, sees, (G, R, 1, 1))
    x.masked_fill_((j > pos) | (j <= pos - s["window"]) if s["window"] else j > pos, float("-inf"))
    top = x.amax(-1, keepdim=True)
    mass = x.sub_(top).exp_().sum(-1, keepdim=True)
    o = ((x.view(B, G, R * N, L) @ v).view(B, G, R, N, d) / mass).permute(0, 3, 1, 2, 4).reshape(B, N, H, d)
    lse = (top + mass.log()).view(B, H, N).transpose(1, 2)
    b, _, at = _tokens(s)
    return o[b, at].to(torch.bfloat16), lse[b, at]


def _build_tables(s):
    ps, old, new = s["page"], s["old"].long(), s["new_len"].long()
    have = (old + ps - 1) // ps
    need = (old + new + ps - 1) // ps - have
    taken = need.cumsum(0)
    ok = (need == 0) | (taken <= s["free_count"])
    kv_len = torch.where(ok, old + new, -1 - old).int()
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    col = torch.arange(s["table"].shape[1], device="cuda")
    nth = (taken - need)[:, None] + col - have[:, None]
    fresh = ok[:, None] & (col >= have[:, None]) & (col < (have + need)[:, None])
    page = s["free"][(s["free_count"] - 1 - nth).clamp(0, len(s["free"]) - 1)]
    table = torch.where(fresh, page, s["table"])
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(cu, t, right=True) - 1
    pos = torch.where(ok[b], old[b] + t - cu[b], -1)
    slot = torch.where(ok[b], table[b, pos.clamp_min(0) // ps].long() * ps + pos % ps, -1)
    left = s["free_count"] - torch.where(ok, taken, 0).amax()
    return table, kv_len, cu.int(), pos.int(), slot, left.int()


# --------------------------------------------------------------------------------------------------------- the pass
def run(s):
    if own:
        from paper_2506_16640_b200 import autograd, binding
        if s["op"] == "tables":
            kv_len, cu, pos, slot, left = binding.entmax_attn_paged_tables(s["old"], s["new_len"], s["table"], s["free"], s["free_count"], s["page"],
                                                                           s["n_pages"], s["T"])
            return s["table"], kv_len, cu, pos, slot, left
        if s["op"] == "attend":
            return binding.entmax_attn_softmax_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["cu"], s["beta"], s["gamma"],
                                                         s["delta"], alibi_slopes=s["slopes"], softcap=s["cap"], window=s["window"],
                                                         max_q_len=s["max_new"], max_kv_len=s["max_kv"])
        ranges = None
        if s["cu"] is not None:
            ranges = binding.entmax_attn_row_ranges(s["cu"], s["N"], True, prefix_len=s["prefix"], window=s["window"])
        causal = ranges is None
        if s["op"] == "eval":
            return binding.entmax_attn_softmax_fwd(s["q"], s["k"], s["v"], causal, s["beta"], s["gamma"], s["delta"], c_rows=s["c_rows"],
                                                   alibi_slopes=s["slopes"], row_ranges=ranges, softcap=s["cap"])
        o, lse = autograd.softmax_attention(s["q"], s["k"], s["v"], s["beta"], s["gamma"], s["delta"], c_rows=s["c_rows"], alibi_slopes=s["slopes"],
                                            row_ranges=ranges, causal=causal, softcap=s["cap"], return_lse=True)
        return (o.detach(), lse) + torch.autograd.grad(o, s["leaves"], s["d_o"])
    if s["op"] == "tables":
        return _build_tables(s)
    return _attend(s) if s["op"] == "attend" else _attention(s)


def _pairs(case):
    """Visible (row, key) pairs of one head, over the batch."""
    B, N = case["B"], case["N"]
    w = case["window"] or N
    causal = lambda n: n * (n + 1) // 2 - max(0, n - w) * (max(0, n - w) + 1) // 2  # noqa: E731
    if case["mask"] == "causal":
        return B * causal(N)
    total = 0
    cu, prefix = _documents(case)
    for b in range(B):
        for e, (lo, hi) in enumerate(zip(cu[b], cu[b][1:])):
            total += causal(hi - lo)
            for i in range(min(prefix[b][e], hi - lo) if prefix else 0):
                total += prefix[b][e] - 1 - i                # the keys of the prefix ahead of row i
    return total


def work(case):
    if case["op"] == "tables":
        new, kv = _lengths(case)
        ps = case["page"]
        fresh = sum(-(-t // ps) - -(-(t - n) // ps) for n, t in zip(new, kv))
        return {"bytes": 16 * case["batch"] + 8 * fresh + 12 * sum(new), "flops": 0}
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "attend":
        new, kv = _lengths(case)
        w = case["window"] or 1 << 30
        pairs = keys = 0
        for n, t in zip(new, kv):
            pairs += sum(min(w, p + 1) for p in range(t - n, t)) * H
            keys += min(t, w + n - 1)
        return {"bytes": 2 * keys * G * d * 2 + sum(new) * H * (d * 2 * 2 + 4), "flops": 4 * d * pairs}
    rows, pairs = case["B"] * case["N"], _pairs(case) * H
    size = rows * (2 * H + 2 * G) * d * 2 + rows * H * 4                     # q, k, v, o and lse
    if case["op"] == "eval":
        return {"bytes": size, "flops": 4 * d * pairs}
    # the forward's, and q, k, v, d_o in, dq, dk, dv out; two products forward, five backward
    return {"bytes": size + rows * (3 * H + 4 * G) * d * 2, "flops": 14 * d * pairs}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_rows(q, k, v, i, sees, cap, slope, c):
    """O and lse of the query rows i of one head, all in 64 bits; sees [rows, keys]."""
    z = q @ k.T / math.sqrt(q.shape[1])
    if cap:
        z = cap * torch.tanh(z / cap)
    if slope is not None:
        z = z - slope.double() * (i[:, None] - torch.arange(len(k), device="cuda")).abs()
    z = torch.where(sees, z * c, -math.inf)
    lse = torch.logsumexp(z, 1)
    weight = torch.exp(z - torch.where(lse > -math.inf, lse, 0.0)[:, None])
    return weight @ v, lse


def _exact_c(beta, gamma, delta, n):
    return delta + torch.where(n > 1, beta * torch.exp(gamma * torch.log(torch.log(n.clamp_min(2.0)))), 0.0)


def _exact_attention(s):
    B, N, H, G, d, train = s["B"], s["N"], s["heads"], s["kv_heads"], s["d"], s["op"] == "train"
    cu, prefix = _documents(s) if s["mask"] != "causal" else ([[0, N]] * B, None)
    lo, hi = torch.zeros((B, N), dtype=torch.int64), torch.zeros((B, N), dtype=torch.int64)
    for b in range(B):
        for e, (first, last) in enumerate(zip(cu[b], cu[b][1:])):
            for i in range(first, last):
                lo[b, i] = max(first, i - s["window"] + 1) if s["window"] else first
                hi[b, i] = max(i + 1, min(last, first + prefix[b][e])) if prefix else i + 1
    lo, hi = lo.cuda(), hi.cuda()
    leaf = {n: s[n].detach().double().requires_grad_(train) for n in ("q", "k", "v", "beta", "gamma", "delta", "c_rows") if s[n] is not None}
    grads = {n: torch.zeros_like(x) for n, x in leaf.items()}
    o = torch.zeros((B, H, N, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, H, N), dtype=torch.float64, device="cuda")
    j = torch.arange(N, device="cuda")
    for b in range(B):
        for h in range(H):
            for n0 in range(0, N, 4096):
                i = torch.arange(n0, min(N, n0 + 4096), device="cuda")
                sees = (j >= lo[b, i][:, None]) & (j < hi[b, i][:, None])
                n = sees.sum(1).double()
                at = {"q": (b, h, i), "k": (b, h * G // H), "v": (b, h * G // H), "beta": (h,), "gamma": (h,), "delta": (h,), "c_rows": (b, h, i)}
                part = {m: leaf[m].detach()[at[m]].requires_grad_(train) for m in leaf}
                c = part["c_rows"] if "c_rows" in part else _exact_c(part["beta"], part["gamma"], part["delta"], n) if "beta" in part else torch.ones_like(n)
                out, norm = _exact_rows(part["q"], part["k"], part["v"], i, sees, s["cap"], None if s["slopes"] is None else s["slopes"][h], c[:, None])
                o[b, h, i], lse[b, h, i] = out.detach(), norm.detach()
                if train:
                    got = torch.autograd.grad(out, list(part.values()), s["d_o"][b, h, i].double(), allow_unused=True)
                    for m, g in zip(part, got):
                        if g is not None:
                            grads[m][at[m]] += g
    return (o, lse) + tuple(grads[m] for m in leaf) if train else (o, lse)


def _exact_attend(s):
    H, G, d = s["heads"], s["kv_heads"], s["d"]
    new, kv = _lengths(s)
    o = torch.empty((s["T"], H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["T"], H), dtype=torch.float64, device="cuda")
    t = 0
    for b, (n, total) in enumerate(zip(new, kv)):
        page = s["table"][b].long()[: -(-total // s["page"])]
        keys, values = (c[page].flatten(0, 1)[:total].double() for c in (s["k_cache"], s["v_cache"]))
        j = torch.arange(total, device="cuda")
        for h in range(H):
            for n0 in range(0, n, 1024):
                i = torch.arange(total - n + n0, total - n + min(n, n0 + 1024), device="cuda")
                sees = j <= i[:, None]
                if s["window"]:
                    sees = sees & (i[:, None] - j < s["window"])
                m = sees.sum(1, keepdim=True).double()
                c = torch.ones_like(m) if s["beta"] is None else _exact_c(s["beta"][h].double(), s["gamma"][h].double(), s["delta"][h].double(), m)
                at = slice(t + n0, t + min(n, n0 + 1024))
                o[at, h], lse[at, h] = _exact_rows(s["q"][at, h].double(), keys[:, h * G // H], values[:, h * G // H], i, sees, s["cap"],
                                                   None if s["slopes"] is None else s["slopes"][h], c)
        t += n
    return o, lse


def exact(case, seed):
    if case["op"] == "tables":
        return None                                          # whole numbers
    if case["op"] == "attend":
        new, kv = _lengths(case)
        if sum(n * t for n, t in zip(new, kv)) * case["heads"] > 1 << 31:
            return None
        return _exact_attend(prepare(case, seed))
    if case["B"] * case["heads"] * case["N"] ** 2 * (3 if case["op"] == "train" else 1) > 1 << 34:
        return None
    return _exact_attention(prepare(case, seed))
