"""Serving from a paged key/value cache, as timed cases: what a server of an entmax model calls for every layer of every step.

    op "append"   entmax_attn_paged_append: the new tokens' rows of the fused QKV projection are rotated to their positions, the keys and
                  values go to their slots of the cache's pages
    op "attend"   entmax_attn_paged_fwd: the new tokens attend to everything the cache holds of their sequences

A case names its sizes: `batch` sequences of up to `kv` tokens (new ones included; with `ragged` their lengths differ), `chunks` of them
bring up to `new` tokens each, the others one.  `page` tokens to a page, the pages of a sequence anywhere in the pool.
    scale  "none"    c = 1: supports of dozens to hundreds of keys
           "length"  ASEntmax, c = delta + beta (ln n)^gamma with beta, gamma, delta ~ U[0.5, 1.5] per head: short supports
    keys   "gauss"   N(0, 1);  "planted": four keys that match the query for some of the new tokens (associative recall)
"""
from __future__ import annotations

import math
import random

import torch

own = False


def _case(name, op, batch, chunks, new, kv, heads, kv_heads, d, page, *, ragged=True, alpha=1.5, scale="length", alibi=False,
          keys="gauss", rot=0, interleaved=False):
    c = dict(op=op, batch=batch, chunks=chunks, new=new, kv=kv, heads=heads, kv_heads=kv_heads, d=d, page=page, ragged=ragged,
             alpha=alpha, scale=scale, alibi=alibi, keys=keys, rot=rot, interleaved=interleaved)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of one conversation with a small model: nothing but latency
        _case("append_1x1_h12_d64", "append", 1, 0, 1, 777, 12, 12, 64, 16, rot=64),
        # a step of a full decode batch
        _case("append_256x1_h32_d128", "append", 256, 0, 1, 2048, 32, 8, 128, 16, rot=128),
        # six prompts prefilled together, half of each head rotated, pairs side by side
        _case("append_6x8192_h32_d128", "append", 6, 6, 8192, 8192, 32, 8, 128, 64, rot=64, interleaved=True),
        # one token of one conversation with a small model
        _case("decode_1x777_h12_d64", "attend", 1, 0, 1, 777, 12, 12, 64, 16),
        # a full decode batch of a grouped-head model, short contexts
        _case("decode_64x4096_h32_d128", "attend", 64, 0, 1, 4096, 32, 8, 128, 16, keys="planted"),
        # long contexts, many query heads per K/V head
        _case("decode_8x65536_h32_d128", "attend", 8, 0, 1, 65536, 32, 4, 128, 128),
        # flat maps: c = 1 and alpha = 1.25, supports in the hundreds
        _case("decode_16x8192_h16_d64_flat", "attend", 16, 0, 1, 8192, 16, 8, 64, 16, alpha=1.25, scale="none"),
        # five proposed tokens of each sequence checked at once, NAPE (slopes on half of the heads), sparsemax
        _case("verify_32x5_kv8192_h32_d128", "attend", 32, 32, 5, 8192, 32, 8, 128, 32, ragged=False, alpha=2.0, alibi=True),
        # continuous batching: two prompts' chunks among single tokens
        _case("mixed_24_new500_kv9001_h16_d64", "attend", 24, 2, 500, 9001, 16, 4, 64, 16, keys="planted"),
        # a chunk of a long prompt
        _case("chunk_2048_kv32768_h16_d128", "attend", 1, 1, 2048, 32768, 16, 8, 128, 64, keys="planted"),
        # a batch of whole prompts
        _case("prompts_4x4096_h16_d64", "attend", 4, 4, 4096, 4096, 16, 2, 64, 32),
        # whole prompts with c = 1: long supports
        _case("prompts_3x2500_h12_d64_flat", "attend", 3, 3, 2500, 2500, 12, 4, 64, 16, scale="none"),
    ]


_HEADS = [(12, 12), (12, 4), (16, 8), (16, 2), (16, 16), (32, 8), (32, 4), (8, 1), (6, 2), (10, 2)]
_PAIRS = 1 << 30          # padded (row, key) pairs of a drawn case, at most; the largest listed one has as many
_CACHE = 1 << 30          # elements of K of a drawn case, at most


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, kv_heads = rng.choice(_HEADS)
    d = rng.choice([64, 128])
    page = rng.choice([16, 16, 32, 64, 128, 256])
    batch = _log_int(rng, 1, 128)
    if rng.random() < 0.3:
        new = _log_int(rng, 1, 8192)
        kv = new + _log_int(rng, 1, 32768) - 1
        while batch > 1 and (batch * new > 65536 or batch * kv * kv_heads * d > _CACHE):
            batch //= 2
        return _case(None, "append", batch, rng.randint(0, batch), new, kv, heads, kv_heads, d, page, ragged=rng.random() < 0.7,
                     rot=rng.choice([0, d // 2, d]), interleaved=rng.random() < 0.3)
    kind = rng.choice(["decode", "decode", "few", "mixed", "chunk", "prompt"])
    new = {"decode": 1, "few": rng.randint(2, 12)}.get(kind) or _log_int(rng, 13, 4096)
    kv = new if kind == "prompt" else new + _log_int(rng, 1, 65536) - 1
    if kind in ("chunk", "prompt"):
        batch = min(batch, 6)
    while batch > 1 and (batch * new * heads * kv > _PAIRS or batch * kv * kv_heads * d > _CACHE):
        batch //= 2
    while batch * new * heads * kv > _PAIRS:
        new = (new + 1) // 2
        kv = new if kind == "prompt" else max(new, kv * 3 // 4)
    chunks = 0 if kind == "decode" else min(batch, 2) if kind == "mixed" else batch
    return _case(None, "attend", batch, chunks, new, kv, heads, kv_heads, d, page, ragged=rng.random() < 0.8,
                 alpha=rng.choice([1.25, 1.5, 1.5, 1.5, 1.7, 2.0]), scale=rng.choice(["none", "length", "length"]),
                 alibi=rng.random() < 0.25, keys=rng.choice(["gauss", "planted"]))


# ------------------------------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """New tokens and lengths (new ones included) of every sequence: part of the case, the same for every seed."""
    rng = random.Random(case["batch"] * 1000003 + case["kv"])
    new, kv = [], []
    for b in range(case["batch"]):
        n = case["new"] if b < case["chunks"] else 1
        total = case["kv"]
        if case["ragged"] and b > 0:
            total = max(1, int(total * rng.uniform(0.1, 1.0)))
            n = max(1, min(n, int(n * rng.uniform(0.3, 1.0)) + 1))
            if case["new"] == case["kv"] and b < case["chunks"]:
                n = total                                    # a whole prompt
        new.append(min(n, total))
        kv.append(total)
    return new, kv


def _rotation(n_pos, rot):
    angle = torch.arange(n_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)
    return torch.cat([angle.cos(), angle.sin()], 1).to(torch.float32).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    new, kv = _lengths(case)
    B, H, G, d, ps = case["batch"], case["heads"], case["kv_heads"], case["d"], case["page"]
    T = sum(new)
    need = [-(-n // ps) for n in kv]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((B, max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    cu = torch.tensor([0] + [sum(new[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
    s = dict(case, T=T, max_new=max(new), max_kv=max(kv), table=table, cu=cu, lens=torch.tensor(kv, dtype=torch.int32, device="cuda"))
    s["k_cache"], s["v_cache"] = randn(n_pages, ps, G, d), randn(n_pages, ps, G, d)
    if case["op"] == "append":
        s["qkv"] = randn(T, (H + 2 * G) * d)                 # the fused projection's output
        s["rotation"] = _rotation(max(kv), case["rot"]) if case["rot"] else None
        return s
    s["q"] = randn(T, H, d)
    s["beta"] = s["gamma"] = s["delta"] = s["slopes"] = None
    if case["scale"] == "length":
        s["beta"], s["gamma"], s["delta"] = (0.5 + torch.rand(H, generator=gen, device="cuda") for _ in range(3))
    if case["alibi"]:
        m = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H)
        s["slopes"] = torch.where(torch.arange(H, device="cuda") % 2 == 0, m, torch.zeros_like(m))
    if case["keys"] == "planted":
        # four slots anywhere in the past of every 8th new token match the query of one of its heads
        b_of, pos, _ = _tokens(s)
        pick = torch.arange(0, T, 8, device="cuda")
        j = (torch.rand((len(pick), 4, G), generator=gen, device="cuda") * (pos[pick] + 1)[:, None, None]).long().clamp_max(max(kv) - 1)
        g = torch.arange(G, device="cuda").expand_as(j)
        qv = s["q"][pick][:, :: H // G].float()[:, None].expand(-1, 4, -1, -1)
        key = 3 * math.sqrt(d) * qv / qv.norm(dim=-1, keepdim=True) + 0.1 * torch.randn(qv.shape, generator=gen, device="cuda")
        page = table[b_of[pick][:, None, None], j // ps].long()
        # (one writer to a slot: the last in the order of the list)
        flat = ((page * ps + j % ps) * G + g).reshape(-1)
        flat, idx = flat.sort(stable=True)
        last = torch.ones_like(flat, dtype=torch.bool)
        last[:-1] = flat[1:] != flat[:-1]
        s["k_cache"].view(-1, d)[flat[last]] = key.reshape(-1, d)[idx[last]].to(torch.bfloat16)
    return s


def _tokens(s):
    """Sequence, position and number within the chunk of every new token."""
    t = torch.arange(s["T"], device="cuda", dtype=torch.int32)
    b = torch.searchsorted(s["cu"], t, right=True) - 1
    n = t - s["cu"][b]
    return b, s["lens"][b] - (s["cu"][b + 1] - s["cu"][b]) + n, n


# --------------------------------------------------------------------------------------------------------- the pass
def _rotate(x, cos, sin, rot, interleaved):
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    if interleaved:
        u, w = r[..., 0::2], r[..., 1::2]
        r = torch.stack([u * cos - w * sin, w * cos + u * sin], -1).flatten(-2)
    else:
        u, w = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([u * cos - w * sin, w * cos + u * sin], -1)
    return torch.cat([r, rest], -1).to(torch.bfloat16)


def _split(s):
    H, G, d = s["heads"], s["kv_heads"], s["d"]
    return (x.view(s["T"], -1, d) for x in s["qkv"].split([H * d, G * d, G * d], 1))


def _append(s):
    q, k, v = _split(s)
    b, pos, _ = _tokens(s)
    page, slot = s["table"][b, pos // s["page"]].long(), (pos % s["page"]).long()
    rot = s["rot"]
    if rot:
        at = s["rotation"][pos]
        cos, sin = at[:, None, :rot // 2], at[:, None, rot // 2:]
        q, k = _rotate(q, cos, sin, rot, s["interleaved"]), _rotate(k, cos, sin, rot, s["interleaved"])
    else:
        q = q.contiguous()
    s["k_cache"][page, slot] = k
    s["v_cache"][page, slot] = v
    return q, s["k_cache"], s["v_cache"]


def _threshold(y, alpha):
    """tau of sum [y - tau]_+^e = 1 over the last dimension, e = 1 / (alpha - 1) >= 1: Newton steps on the e-norm of [y - tau]_+, which is convex and
    decreasing, from y_max - 1 upwards."""
    e = 1.0 / (alpha - 1.0)
    tau = y.amax(-1, keepdim=True) - 1.0
    for _ in range(20):
        u = (y - tau).clamp_min_(0)
        if alpha == 2.0:
            s1, s0 = (u > 0).sum(-1, keepdim=True), u.sum(-1, keepdim=True)
        elif alpha == 1.5:
            s1, s0 = u.sum(-1, keepdim=True), u.square_().sum(-1, keepdim=True)
        else:
            s1 = u.pow(e - 1.0).sum(-1, keepdim=True)
            s0 = u.pow_(e).sum(-1, keepdim=True)
        tau = tau + ((s0 - s0.pow(1.0 - 1.0 / e)) / s1).clamp_min_(0)
    return tau


def _attend(s):
    B, H, G, d, N, L = s["batch"], s["heads"], s["kv_heads"], s["d"], s["max_new"], s["max_kv"]
    R, alpha = H // G, s["alpha"]
    pages = -(-L // s["page"])
    table = s["table"][:, :pages].long()
    k = s["k_cache"][table].view(B, -1, G, d)[:, :L].float().permute(0, 2, 3, 1)          # [B, G, d, L]
    v = s["v_cache"][table].view(B, -1, G, d)[:, :L].float().transpose(1, 2)              # [B, G, L, d]
    n = torch.arange(N, device="cuda")
    new = s["cu"][1:] - s["cu"][:-1]
    rows = (s["cu"][:-1, None] + n).clamp_max(s["T"] - 1)
    q = s["q"][rows].float().view(B, N, G, R, d).permute(0, 2, 3, 1, 4)                   # [B, G, R, N, d]
    pos = ((s["lens"] - new)[:, None] + n).clamp_max(L - 1)[:, None, None, :, None].float()   # [B, 1, 1, N, 1]
    per_head = lambda x: x.view(1, G, R, 1, 1)  # noqa: E731
    y = (q.reshape(B, G, R * N, d) @ k).view(B, G, R, N, L).mul_(1.0 / math.sqrt(d))
    j = torch.arange(L, device="cuda").float()
    if s["slopes"] is not None:
        y -= per_head(s["slopes"]) * (pos - j)
    if s["beta"] is not None:
        c = per_head(s["delta"]) + torch.where(pos > 0, per_head(s["beta"]) * torch.log(pos + 1).clamp_min(1e-30).pow(per_head(s["gamma"])), 0.0)
        y *= c
    y.mul_(alpha - 1.0).masked_fill_(j > pos, float("-inf"))
    tau = _threshold(y, alpha)
    p = y.sub_(tau).clamp_min_(0)
    p = p if alpha == 2.0 else p.square_() if alpha == 1.5 else p.pow_(1.0 / (alpha - 1.0))
    o = (p.view(B, G, R * N, L) @ v).view(B, G, R, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, H, d)
    tau = tau.view(B, H, N).transpose(1, 2)
    b, _, at = _tokens(s)
    return o[b, at].to(torch.bfloat16), tau[b, at]


def run(s):
    if own:
        from paper_2506_16640_b200 import binding
        if s["op"] == "append":
            q, k, v = _split(s)
            q = binding.entmax_attn_paged_append(q, k, v, s["k_cache"], s["v_cache"], s["table"], s["lens"], s["cu"],
                                                 rotation=s["rotation"], interleaved=s["interleaved"])
            return q, s["k_cache"], s["v_cache"]
        o, tau, _ = binding.entmax_attn_paged_fwd(s["q"], s["k_cache"], s["v_cache"], s["alpha"], s["table"], s["lens"], s["cu"],
                                                  s["beta"], s["gamma"], s["delta"], alibi_slopes=s["slopes"],
                                                  max_q_len=s["max_new"], max_kv_len=s["max_kv"])
        return o, tau
    return _append(s) if s["op"] == "append" else _attend(s)


def work(case):
    new, kv = _lengths(case)
    H, G, d = case["heads"], case["kv_heads"], case["d"]
    if case["op"] == "append":
        T = sum(new)
        return {"bytes": T * ((H + 2 * G) * d * 2 * 2 + case["rot"] * 4), "flops": T * (H + G) * case["rot"] * 3}
    pairs = sum(n * (t - n) + n * (n + 1) // 2 for n, t in zip(new, kv)) * H
    # K of every visible key; of V the rows of the supports alone, which are few and not counted
    return {"bytes": sum(kv) * G * d * 2 + sum(new) * H * (d * 2 * 2 + 4), "flops": 2 * d * pairs}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def _exact_append(s):
    H, G, d, rot = s["heads"], s["kv_heads"], s["d"], s["rot"]
    x = s["qkv"].double().view(s["T"], H + 2 * G, d)
    new, kv = _lengths(s)
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    out, t = x[:, :H + G].clone(), 0
    for b, (n, total) in enumerate(zip(new, kv)):
        where = torch.arange(total - n, total, device="cuda")
        if rot:
            turn = torch.complex(*(s["rotation"][where].double().unflatten(1, (2, rot // 2)).unbind(1)))[:, None]
            a = x[t:t + n, :H + G, :rot]
            a = a.unflatten(2, (rot // 2, 2)) if s["interleaved"] else a.unflatten(2, (2, rot // 2)).transpose(2, 3)
            z = torch.view_as_real(torch.complex(a[..., 0], a[..., 1]) * turn)
            out[t:t + n, :, :rot] = (z if s["interleaved"] else z.transpose(2, 3)).flatten(2)
        page = s["table"][b].long()[where // s["page"]]
        k_cache[page, where % s["page"]] = out[t:t + n, H:]
        v_cache[page, where % s["page"]] = x[t:t + n, H + G:]
        t += n
    return out[:, :H], k_cache, v_cache


def _exact_attend(s):
    H, G, d, alpha = s["heads"], s["kv_heads"], s["d"], s["alpha"]
    R = H // G
    new, kv = _lengths(s)
    o = torch.empty((s["T"], H, d), dtype=torch.float64, device="cuda")
    tau = torch.empty((s["T"], H), dtype=torch.float64, device="cuda")
    t = 0
    for b, (n, total) in enumerate(zip(new, kv)):
        page = s["table"][b].long()[: -(-total // s["page"])]
        keys, values = (c[page].flatten(0, 1)[:total].double() for c in (s["k_cache"], s["v_cache"]))
        j = torch.arange(total, device="cuda", dtype=torch.float64)
        for h in range(H):
            for n0 in range(0, n, 1024):
                i = torch.arange(total - n + n0, total - n + min(n, n0 + 1024), device="cuda", dtype=torch.float64)[:, None]
                at = slice(t + n0, t + min(n, n0 + 1024))
                z = s["q"][at, h].double() @ keys[:, h // R].T / math.sqrt(d)
                if s["slopes"] is not None:
                    z -= s["slopes"][h].double() * (i - j)
                if s["beta"] is not None:
                    length = torch.where(i > 0, torch.log(i + 1.0).clamp_min(1e-300) ** s["gamma"][h].double(), 0.0)
                    z *= s["delta"][h].double() + s["beta"][h].double() * length
                z = torch.where(j <= i, z * (alpha - 1.0), -math.inf)
                hi = z.amax(1, keepdim=True)
                lo = hi - 1.0
                for _ in range(46):                          # the mass falls with the threshold: halve the bracket
                    mid = (lo + hi) / 2
                    more = (z - mid).clamp_min(0).pow(1.0 / (alpha - 1.0)).sum(1, keepdim=True) >= 1.0
                    lo, hi = torch.where(more, mid, lo), torch.where(more, hi, mid)
                p = (z - lo).clamp_min(0).pow(1.0 / (alpha - 1.0))
                o[at, h] = p @ values[:, h // R]
                tau[at, h] = lo[:, 0]
        t += n
    return o, tau


def exact(case, seed):
    new, kv = _lengths(case)
    if case["op"] == "attend" and sum(n * t for n, t in zip(new, kv)) * case["heads"] > 1 << 31:
        return None
    s = prepare(case, seed)
    return _exact_append(s) if case["op"] == "append" else _exact_attend(s)
