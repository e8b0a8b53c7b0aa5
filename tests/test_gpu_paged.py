"""Serving from a paged cache: entmax_attn_paged_append and entmax_attn_paged_fwd against their definitions in 64 bits.

Tolerances: tests/paged.py derives them row by row from the roundings a float32 evaluation makes."""
import numpy as np
import pytest
import torch

import paged
from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu


def _problem(new, lens, H, KH, d, page, seed=0, sigma=1.0, layout="tokens", rows_behind=0, plant=True):
    """Packed queries and a filled pool; some keys match a query, so that supports of one and of many keys occur."""
    g = torch.Generator().manual_seed(seed)
    T = sum(new)
    q = (torch.randn((T + rows_behind, H, d), generator=g) * sigma).to(torch.bfloat16)
    keys = [(torch.randn((n, KH, d), generator=g) * sigma).to(torch.bfloat16) for n in lens]
    values = [torch.randn((n, KH, d), generator=g).to(torch.bfloat16) for n in lens]
    t = 0
    for b, n in enumerate(new):
        for i in range(0, n if plant else 0, 3):
            x = q[t + i, (i // 3) % H].float()
            at = int(torch.randint(0, lens[b] - n + i + 1, (1,), generator=g))
            keys[b][at, ((i // 3) % H) // (H // KH)] = (2.5 * d ** 0.5 * x / x.norm()).to(torch.bfloat16)
        t += n
    kc, vc, table = paged.pool(keys, values, page, d, KH, seed, "cuda", layout=layout)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    return dict(q=q.cuda(), keys=keys, values=values, kc=kc, vc=vc, table=table, cu=cu,
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), new=list(new), kv=list(lens), H=H, KH=KH, d=d)


def _scales(H, seed, kind):
    g = torch.Generator().manual_seed(1000 + seed)
    if kind is None:
        return None
    if kind == "cool":                        # low temperatures: supports of one or two keys
        return [torch.full((H,), x) for x in (1.5, 1.2, 2.0)]
    return [0.5 + torch.rand(H, generator=g) for _ in range(3)]


def _run(pr, alpha, scale=None, slopes=None, **kw):
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    sc = [t.cuda() for t in scale] if scale is not None else [None] * 3
    al = torch.tensor(slopes, dtype=torch.float32, device="cuda") if slopes is not None else None
    kw.setdefault("support_size", torch.full(pr["q"].shape[:2], -1, dtype=torch.int32, device="cuda"))
    out = binding.entmax_attn_paged_fwd(pr["q"], pr["kc"], pr["vc"], alpha, pr["table"], pr["lens"], kw.pop("cu", pr["cu"]), *sc,
                                        alibi_slopes=al, status=status, **kw)
    torch.cuda.synchronize()
    return (*out, int(status[0]))


def _check(pr, alpha, got, scale=None, slopes=None, skip=(), sm_scale=None, heads=None, rows=None):
    o, tau, supp, flags = got
    assert flags == 0
    o, tau, supp = o.cpu().double(), tau.cpu().double(), supp.cpu()
    R = pr["H"] // pr["KH"]
    q = pr["q"].cpu()
    t = 0
    for b, (n, L) in enumerate(zip(pr["new"], pr["kv"])):
        for h in (heads or range(pr["H"])) if n and b not in skip else ():
            sc = None if scale is None else [s[h] for s in scale]
            m = 0.0 if slopes is None else slopes[h]
            for i in ([slice(0, n)] if rows is None else [slice(r, r + 1) for r in rows if r < n]):
                at = slice(t + i.start, t + i.stop)
                ro, rt, to, tt, lo, hi = paged.attend(q[at, h], pr["keys"][b][:, h // R], pr["values"][b][:, h // R], L - n + i.start, alpha, sc,
                                                      m, sm_scale)
                et, eo = (tau[at, h] - rt).abs() / tt, (o[at, h] - ro).abs() / to
                assert float(et.max()) <= 1.0, ("tau", b, h, i, int(et.argmax()), float(et.max()))
                assert float(eo.max()) <= 1.0, ("o", b, h, i, int(eo.max(1)[0].argmax()), float(eo.max()))
                s = supp[at, h]
                assert bool(((s >= lo) & (s <= hi)).all()), ("support", b, h, i)
        t += n


LENGTHS = [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 700, 1500]


@pytest.mark.parametrize("H,KH,d,page", [(4, 4, 64, 16), (6, 2, 128, 32), (8, 1, 64, 64), (16, 1, 128, 128), (4, 2, 128, 256), (20, 1, 64, 16)])
def test_single_tokens(H, KH, d, page):
    pr = _problem([1] * len(LENGTHS), LENGTHS, H, KH, d, page, seed=H)
    sc = _scales(H, 1, "length")
    got = _run(pr, 1.5, sc)
    _check(pr, 1.5, got, sc)
    # (the bounds choose the kernels, so the last bits may differ)
    _check(pr, 1.5, _run(pr, 1.5, sc, cu=None, max_q_len=1, max_kv_len=max(LENGTHS)), sc)


@pytest.mark.parametrize("alpha", [1.25, 1.5, 1.7, 2.0, 3.0])
@pytest.mark.parametrize("kind", [None, "length", "cool"])
def test_alphas_and_temperatures(alpha, kind):
    pr = _problem([1, 3, 40], [900, 333, 640], 4, 2, 64, 16, seed=3)
    sc = _scales(4, 2, kind)
    _check(pr, alpha, _run(pr, alpha, sc), sc)


@pytest.mark.parametrize("new,lens,H,KH,d,page", [
    ([5, 1, 0, 3, 8], [700, 1, 90, 3, 8], 8, 2, 128, 32),            # a few tokens each, an idle sequence, nothing but new tokens
    ([9, 17, 33], [33, 17, 400], 3, 1, 64, 16),                      # on both sides of the 32 rows where the kernels change over
    ([200, 1, 64, 33], [200, 513, 300, 1025], 4, 4, 64, 64),         # whole prompts among single tokens
    ([130, 259], [1000, 259], 6, 2, 128, 16),                        # groups of three: 126 rows to a tile
    ([300], [300], 8, 1, 64, 128),
    ([77, 500], [1111, 1536], 2, 1, 128, 256),
    ([3, 70], [200, 71], 40, 1, 64, 16),                             # more query heads to a K/V head than the few-row kernel takes
    ([2, 5], [300, 6], 128, 1, 64, 32),
])
def test_chunks(new, lens, H, KH, d, page):
    pr = _problem(new, lens, H, KH, d, page, seed=len(new) + H)
    sc = _scales(H, 4, "length")
    got = _run(pr, 1.5, sc)
    _check(pr, 1.5, got, sc)
    hinted = _run(pr, 1.5, sc, max_q_len=max(new), max_kv_len=max(lens))
    _check(pr, 1.5, hinted, sc)


@pytest.mark.parametrize("new,lens", [([1, 1], [600, 40]), ([4, 120], [64, 500])])
def test_alibi(new, lens):
    pr = _problem(new, lens, 4, 2, 64, 16, seed=7)
    slopes = [0.5, 0.0, 0.0625, 0.0]
    sc = _scales(4, 5, "length")
    for alpha in (1.5, 2.0):
        _check(pr, alpha, _run(pr, alpha, sc, slopes), sc, slopes)


@pytest.mark.parametrize("new", [1, 150])
def test_equal_logits_see_every_key(new):
    # q = 0: every visible key weighs 1/n, far more of them than any list holds
    pr = _problem([new, 1], [2600, 700], 2, 1, 64, 16, plant=False)
    pr["q"].zero_()
    o, tau, supp, flags = got = _run(pr, 1.5)
    _check(pr, 1.5, got)
    n = torch.arange(2600 - new + 1, 2601, dtype=torch.float64)
    # sums of up to 2600/32 equal terms by a lane are off by 82 * 2^-24 = 5e-6 of themselves at most, tau by that over e sum u = 2 sqrt(n): 5e-8,
    # of 0.0196 in the longest row 2.5e-6
    assert torch.allclose(tau[:new, 0].cpu().double(), -n.pow(-0.5), rtol=1e-5)
    assert torch.equal(supp[:new, 0].cpu().long(), n.long())


@pytest.mark.parametrize("sigma", [0.02, 0.3])
def test_flat_rows(sigma):
    pr = _problem([1, 90], [2000, 1300], 4, 2, 64, 32, sigma=sigma, plant=False)
    for alpha in (1.25, 1.5, 2.0):
        _check(pr, alpha, _run(pr, alpha))


@pytest.mark.parametrize("layout", ["tokens", "heads", "fused"])
@pytest.mark.parametrize("new,lens", [([1, 1, 1], [100, 31, 257]), ([100, 2], [257, 40])])
def test_layouts_and_strided_queries(layout, new, lens):
    pr = _problem(new, lens, 4, 2, 64, 32, layout=layout)
    T = sum(new)
    wide = torch.full((T, 4 + 3, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 2:6] = pr["q"]
    want = _run(pr, 1.5)
    pr["q"] = wide[:, 2:6]
    got = _run(pr, 1.5)
    _check(pr, 1.5, got)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_rows_behind_the_last_sequence_stay():
    for new, lens in (([1, 2], [50, 70]), ([60, 1], [300, 9])):
        pr = _problem(new, lens, 4, 2, 64, 16, rows_behind=9)
        T = sum(new)
        o = torch.full((T + 9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
        tau = torch.full((T + 9, 4), 7.0, device="cuda")
        supp = torch.full((T + 9, 4), 7, dtype=torch.int32, device="cuda")
        got = _run(pr, 1.5, o=o, tau=tau, support_size=supp)
        _check(pr, 1.5, got)
        assert bool((o[T:] == 7).all() and (tau[T:] == 7).all() and (supp[T:] == 7).all())


def test_workspace_in_slices():
    # a table with room for 2^20 tokens and no bound on the lengths given: the rows' share of the workspace covers a few blocks at a time
    new, lens = [40, 1, 700, 1], [300, 90, 700, 33]
    pr = _problem(new, lens, 4, 2, 64, 16)
    wide = torch.full((len(new), (1 << 20) // 16), -1, dtype=torch.int32, device="cuda")
    wide[:, :pr["table"].shape[1]] = pr["table"]
    pr["table"] = wide
    _check(pr, 1.5, _run(pr, 1.5))


@pytest.mark.parametrize("new,lens,bad", [([1, 1, 1], [5, 0, 40], 1), ([1, 1, 1], [5, 49, 40], 1), ([3, 60, 1], [40, 30, 9], 1),
                                          ([3, 60, 1], [40, 65, 9], 1)])
def test_lengths_that_do_not_fit(new, lens, bad):
    # the sequence is left out and reported, the others are served (48 tokens of room, or 64 with the chunk)
    room = 48 if max(new) == 1 else 64
    ok = [min(max(n, L), room) for n, L in zip(new, lens)]
    pr = _problem(new, ok, 4, 2, 64, 16)
    pr["table"] = pr["table"][:, :room // 16].contiguous()
    pr["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    o, tau, supp, flags = _run(pr, 1.5)
    assert flags == binding.FLAG_BAD_LENGTH
    a, e = sum(new[:bad]), sum(new[:bad + 1])
    assert bool((o[a:e] == 0).all() and torch.isneginf(tau[a:e]).all() and (supp[a:e] == 0).all())
    pr["kv"] = lens
    _check(pr, 1.5, (o, tau, supp, 0), skip=(bad,))


@pytest.mark.parametrize("new", [[1, 1], [50, 1]])
def test_pages_outside_the_pool(new):
    lens = [200, 100]
    pr = _problem(new, lens, 4, 2, 64, 16)
    good = _run(pr, 1.5)
    for bad in (-1, pr["kc"].shape[0], 2 ** 31 - 1):
        pr["table"][0, 3] = bad
        o, tau, supp, flags = _run(pr, 1.5)
        assert flags == binding.FLAG_BAD_PAGE
        assert bool(torch.isfinite(o).all() and torch.isfinite(tau).all())
        assert torch.equal(o[new[0]:], good[0][new[0]:]) and torch.equal(tau[new[0]:], good[1][new[0]:])


@pytest.mark.parametrize("new,max_q,max_kv,bad", [([2, 7, 1], 4, 0, 1), ([1, 1, 1], 0, 60, 0), ([70, 20, 90], 80, 0, 2)])
def test_bounds_that_are_too_small(new, max_q, max_kv, bad):
    lens = [100, 50, 95]
    pr = _problem(new, lens, 4, 2, 64, 16)
    o, tau, supp, flags = _run(pr, 1.5, max_q_len=max_q, max_kv_len=max_kv)
    assert flags == binding.FLAG_BAD_LENGTH
    left_out = [bad] if max_q else [b for b in range(3) if lens[b] > max_kv]
    for b in left_out:
        a, e = sum(new[:b]), sum(new[:b + 1])
        assert bool((o[a:e] == 0).all() and torch.isneginf(tau[a:e]).all() and (supp[a:e] == 0).all())
    _check(pr, 1.5, (o, tau, supp, 0), skip=left_out)


def test_large_batches():
    # more sequences than a launch for few rows takes, some idle, some with a few tokens; then enough blocks that none is cut
    g = np.random.default_rng(0)
    lens = [int(n) for n in g.integers(1, 90, 600)]
    new = [min(n, int(m)) for n, m in zip(lens, g.integers(0, 4, 600))]
    pr = _problem(new, lens, 4, 2, 64, 16)
    sc = _scales(4, 2, "length")
    _check(pr, 1.5, _run(pr, 1.5, sc, max_q_len=3, max_kv_len=90), sc, skip=range(0, 600, 3))
    _check(pr, 1.5, _run(pr, 1.5, sc), sc, skip=[b for b in range(600) if b % 7])
    lens = [int(n) for n in g.integers(40, 700, 60)]
    new = [min(n, int(m)) for n, m in zip(lens, g.integers(33, 60, 60))]
    pr = _problem(new, lens, 8, 8, 64, 16)
    sc = _scales(8, 2, "length")
    _check(pr, 1.5, _run(pr, 1.5, sc), sc, heads=[0, 3, 7], skip=range(1, 60, 4))


@pytest.mark.parametrize("new,lens,H,KH,d,page,slopes,columns", [
    ([70, 33, 40], [9000, 300, 5000], 4, 2, 64, 16, None, 0),
    ([70, 33, 40], [9000, 300, 5000], 4, 2, 128, 64, [0.0, 0.01, 0.3, 2.0], 0),
    ([70, 33, 40], [9000, 300, 5000], 2, 1, 64, 256, None, 1100),           # a table for 281600 keys: rows of several lengths share a class
    ([35] * 80 + [300], list(range(35, 115)) + [9000], 4, 4, 64, 16, None, 0),      # one long chunk among short prompts
    ([257] * 24, [257] * 12 + [900] * 12, 16, 8, 64, 32, [0.1] * 16, 0),
])
def test_uneven_and_even_units(new, lens, H, KH, d, page, slopes, columns):
    # chunks whose keys are shared among work items, and such that whole units are dealt evenly
    pr = _problem(new, lens, H, KH, d, page)
    if columns:
        wide = torch.full((len(new), columns), 2 ** 31 - 1, dtype=torch.int32, device="cuda")
        wide[:, :pr["table"].shape[1]] = pr["table"]
        pr["table"] = wide
    sc = _scales(H, 3, "length")
    got = _run(pr, 1.5, sc, slopes)
    again = _run(pr, 1.5, sc, slopes)
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    _check(pr, 1.5, got, sc, slopes, heads=[0, H - 1], skip=[b for b in range(len(new)) if len(new) > 3 and b % 9 not in (0, 8)])


def test_units_that_are_cut_only_after_they_were_dealt():
    # 152 equal units of 13 tiles for 148 SMs: no unit is too long by itself, but four CTAs would take two of them; the plan kernel's warps have
    # to agree on that way, call for call
    pr = _problem([256] * 19, [3328] * 19, 8, 8, 64, 16)
    sc = _scales(8, 3, "length")
    got = _run(pr, 1.5, sc, max_q_len=256, max_kv_len=3328)
    _check(pr, 1.5, got, sc, heads=[0, 7], skip=range(1, 18), rows=[0, 100, 255])
    for _ in range(30):
        again = _run(pr, 1.5, sc, max_q_len=256, max_kv_len=3328)
        assert all(torch.equal(x, y) for x, y in zip(got[:3], again[:3]))


@pytest.mark.parametrize("n", [1, 5, 40])
def test_uniform_chunks_without_offsets(n):
    lens = [41, 300, 64]
    pr = _problem([n] * 3, lens, 4, 2, 64, 16)
    _check(pr, 1.5, _run(pr, 1.5, cu=None))


@pytest.mark.parametrize("new,H,KH,sigma", [(1, 16, 2, 1.0), (40, 1, 1, 1.0), (1, 4, 1, 0.05), (20, 2, 1, 0.05)])
def test_long_contexts(new, H, KH, sigma):
    # rows of 2200 groups; a unit cut into more work items than a row's lanes
    pr = _problem([new], [70001], H, KH, 64, 64, sigma=sigma, plant=sigma == 1.0)
    sc = _scales(H, 5, "length") if sigma == 1.0 else None
    _check(pr, 1.5, _run(pr, 1.5, sc), sc, heads=[0, H - 1], rows=[0, new // 2, new - 1])


@pytest.mark.parametrize("new,lens,H,KH,alpha", [([400, 390], [2600, 400], 8, 2, 1.5), ([1] * 50, [2000 - 7 * b for b in range(50)], 32, 4, 1.25)])
def test_more_rows_with_long_supports_than_lists_hold(new, lens, H, KH, alpha):
    # enough rows for the kernels with many rows to a CTA, each with hundreds of keys or all of them in its support
    pr = _problem(new, lens, H, KH, 64, 32, sigma=0.3, plant=False)
    pr["q"][::2] = 0
    _check(pr, alpha, _run(pr, alpha), heads=[0, H - 1], skip=range(3, len(new), 5), rows=[0, 1, 170, 389])


def test_two_calls_at_once():
    a = _problem([1] * 40, [600 + b for b in range(40)], 8, 2, 64, 16, seed=1)
    b = _problem([300, 1], [900, 77], 8, 2, 64, 16, seed=2)
    want = [binding.entmax_attn_paged_fwd(p["q"], p["kc"], p["vc"], 1.5, p["table"], p["lens"], p["cu"])[:2] for p in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = []
        for p, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                got.append(binding.entmax_attn_paged_fwd(p["q"], p["kc"], p["vc"], 1.5, p["table"], p["lens"], p["cu"])[:2])
        torch.cuda.synchronize()
        for w, x in zip(want, got):
            assert torch.equal(w[0], x[0]) and torch.equal(w[1], x[1])


@pytest.mark.parametrize("kind", ["zero", "negative", "nan"])
def test_scales_without_an_order(kind):
    # c = 0: every key alike; c < 0: the smallest products win; c not finite: reported, rows finite or not but the call ends
    for new, lens in (([1, 3], [200, 50]), ([90, 1], [200, 50])):
        pr = _problem(new, lens, 4, 2, 64, 16)
        sc = [torch.full((4,), x) for x in {"zero": (0.0, 1.0, 0.0), "negative": (-0.5, 1.0, -1.0), "nan": (1.0, 1.0, float("nan"))}[kind]]
        got = _run(pr, 1.5, sc)
        if kind == "nan":
            assert got[3] == binding.FLAG_BAD_SCALE
        else:
            _check(pr, 1.5, got, sc)


@pytest.mark.parametrize("new,lens,H,KH", [([64], [32768], 16, 4), ([64] + [200] * 11, [20000] + [200] * 11, 4, 2)])
def test_heads_of_scale_zero_in_units_of_many_work_items(new, lens, H, KH):
    # delta = beta = 0: the mean of V; more items to a unit than a row has lanes, 32 of them and eight
    pr = _problem(new, lens, H, KH, 64, 16)
    sc = _scales(H, 6, "length")
    for t in (sc[0], sc[2]):
        t[::3] = 0.0
    got = _run(pr, 1.5, sc, max_q_len=max(new), max_kv_len=max(lens))
    _check(pr, 1.5, got, sc, heads=[0, 1, 3, H - 1], skip=range(2, len(new)), rows=[0, 1, 40, 63])
    # (every key; sums of up to 1024 equal terms by a lane are off by 6e-5 of themselves at most, tau by half of that, and by 1e-7 of 0.0055 for the step
    # it ends at)
    n = torch.arange(lens[0] - 63, lens[0] + 1)
    assert torch.equal(got[2][:64, 0].cpu().long(), n) and torch.allclose(got[1][:64, 0].cpu().double(), -n.double().pow(-0.5), rtol=1e-4)


@pytest.mark.parametrize("alpha", [1.5, 2.0, 3.0])
@pytest.mark.parametrize("new,lens,H,KH", [
    ([1, 3, 1], [257, 300, 1], 4, 2), ([1] * 80, [40 + b for b in range(80)], 8, 4),     # rows of few tokens: a CTA each, 32 lanes,
    ([1] * 256, [5 + b % 40 for b in range(256)], 40, 8),                                # and eight
    ([100], [600], 2, 1), ([300, 100], [300, 900], 4, 2), ([256] * 40, [256 + b for b in range(40)], 1, 1),       # the same of longer chunks
])
def test_scores_without_room_for_a_bracket(new, lens, H, KH, alpha):
    # scores beyond 2^24, where y_max - 1 is no float of its own: exact products of powers of two, so the result is the mean of V over the keys
    # that share the largest score; queries of either sign, so that largest scores are negative too
    d, page = 64, 16
    g = torch.Generator().manual_seed(H + len(new))
    T = sum(new)
    unit = 2.0 ** 25                                          # of the scores y = (alpha - 1) <q,k>
    q = torch.zeros((T, H, d))
    q[..., 0] = 2.0 ** 13 / (alpha - 1.0) * torch.where(torch.rand((T, H), generator=g) < 0.5, -1.0, 1.0)
    keys, marks, values = [], [], []
    for n in lens:
        k = torch.zeros((n, KH, d))
        m = 128 + torch.randint(0, 128, (n, KH), generator=g)
        m[torch.rand((n, KH), generator=g) < 4.0 / n] = 254
        m[torch.rand((n, KH), generator=g) < 4.0 / n] = 129
        k[..., 0] = m * 2.0 ** 12
        keys.append(k.to(torch.bfloat16))
        marks.append(m.double())
        values.append(torch.randn((n, KH, d), generator=g).to(torch.bfloat16))
    kc, vc, table = paged.pool(keys, values, page, d, KH, 3, "cuda")
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    pr = dict(q=q.to(torch.bfloat16).cuda(), kc=kc, vc=vc, table=table, cu=cu, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    o, tau, supp, flags = _run(pr, alpha, sm_scale=1.0, max_q_len=max(new), max_kv_len=max(lens))
    assert flags == 0
    o, tau, supp, t, several = o.cpu().double(), tau.cpu().double(), supp.cpu(), 0, 0
    sign = q[..., 0].sign().double()
    for b, (n, L) in enumerate(zip(new, lens)):
        j, i = torch.arange(L), torch.arange(L - n, L)[:, None]
        for h in range(H) if b % 16 == 0 or len(new) < 60 else (b % H,):
            y = sign[t:t + n, h, None] * unit * marks[b][:, h // (H // KH)]
            y = torch.where(j <= i, y, -torch.inf)
            top = y.amax(1, keepdim=True)
            ties = (y == top).double()
            count, v = ties.sum(1, keepdim=True), values[b][:, h // (H // KH)].double()
            several += int((count > 1).sum())
            # p = 1 / count within e / |t| times the 1e-7 at which the iteration stops (t = -count^(1 - alpha), count <= 40: 1e-5 of p for alpha = 3),
            # or a mass within 1.6e-6 of 1; one rounding of O
            assert bool(((o[t:t + n, h] - ties @ v / count).abs() <= 2.0 ** -8 * (ties @ v / count).abs() + 2e-5 * (ties @ v.abs()) / count).all()), (b, h)
            assert torch.equal(supp[t:t + n, h].long(), count[:, 0].long()), (b, h)
            want = top - count.pow(1.0 - alpha)
            assert bool(((tau[t:t + n, h, None] - want).abs() <= 2.0 ** -23 * want.abs()).all()), (b, h)
        t += n
    assert several > 0


def test_offsets_beyond_32_bits():
    # a pool of more than 2^32 bytes, the sequence's pages at its end
    d, KH, page = 128, 2, 256
    n = (1 << 32) // (page * KH * d * 2) + 40
    pr = _problem([1, 70], [300, 500], 4, KH, d, page)
    kc = torch.zeros((n, page, KH, d), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    m = pr["kc"].shape[0]
    kc[n - m:], vc[n - m:] = pr["kc"], pr["vc"]
    pr["table"] = torch.where(pr["table"] < m, pr["table"] + (n - m), pr["table"])
    pr["kc"], pr["vc"] = kc, vc
    _check(pr, 1.5, _run(pr, 1.5))


def test_repeats_are_bit_equal():
    pr = _problem([1, 5, 300], [900, 128, 900], 8, 2, 128, 16)
    a = _run(pr, 1.5)
    for _ in range(3):
        b = _run(pr, 1.5)
        assert all(torch.equal(x, y) for x, y in zip(a[:3], b[:3]))


@pytest.mark.parametrize("new,lens,H,KH,d,alpha,sigma", [
    ([188, 7, 106], [3962, 228, 444], 33, 1, 64, 1.1, 0.02), ([300, 250, 90], [300, 250, 90], 40, 2, 128, 1.5, 1.0),
    ([482, 334], [482, 334], 33, 1, 128, 1.7, 1.0), ([41] * 20, [125 + 9 * b for b in range(20)], 20, 1, 64, 1.5, 0.3),
    ([130, 259, 401], [1000, 259, 401], 6, 2, 128, 2.0, 0.3), ([3, 1, 8, 7], [96, 191, 196, 1219], 33, 1, 128, 1.5, 1.0),
])
def test_repeats_are_bit_equal_whatever_ran_before(new, lens, H, KH, d, alpha, sigma):
    # groups that leave rows of a 128-row tile empty: nothing of an earlier kernel's shared memory may show
    pr = _problem(new, lens, H, KH, d, 16, sigma=sigma)
    others = [_problem([200, 60], [700, 60], 8, 2, x, 16, sigma=s) for x, s in ((64, 1.0), (128, 0.02), (128, 30.0))]
    want = _run(pr, alpha)
    _check(pr, alpha, want, heads=[0, H - 1], rows=[0, 1, 40, 187], skip=range(3, len(new)))
    for i in range(12):
        _run(others[i % 3], 1.5)
        got = _run(pr, alpha)
        assert all(torch.equal(x, y) for x, y in zip(want[:3], got[:3])), i


@pytest.mark.parametrize("H,KH,n", [(6, 2, 150), (33, 1, 100), (4, 2, 190), (20, 1, 61)])
def test_a_sequence_does_not_depend_on_the_queries_packed_behind_it(H, KH, n):
    # the last tile of its chunk holds rows of the next sequence (or rows behind the last one)
    pr = _problem([n, 150], [900, 400], H, KH, 64, 16, rows_behind=70)
    want = _run(pr, 1.5)
    for fill in (0.0, 0.01, -3.0, 1e4, float("inf"), float("nan")):
        pr["q"][n:] = fill
        got = _run(pr, 1.5)
        assert all(torch.equal(x[:n], y[:n]) for x, y in zip(want[:3], got[:3])), fill


def test_graph_replay_and_second_stream():
    pr = _problem([1, 1, 90], [64, 200, 300], 4, 2, 64, 16)
    sc = [t.cuda() for t in _scales(4, 1, "length")]
    o = torch.empty((92, 4, 64), dtype=torch.bfloat16, device="cuda")
    tau = torch.empty((92, 4), device="cuda")
    side = torch.cuda.Stream()

    def call():
        binding.entmax_attn_paged_fwd(pr["q"], pr["kc"], pr["vc"], 1.5, pr["table"], pr["lens"], pr["cu"], *sc, o=o, tau=tau)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    eager = o.clone(), tau.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    o.zero_()
    tau.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, eager[0]) and torch.equal(tau, eager[1])
    # other lengths through the same graph: one token less of the first sequences' past
    pr["lens"][:2] -= 1
    g.replay()
    torch.cuda.synchronize()
    again = o.clone()
    call()
    torch.cuda.synchronize()
    assert torch.equal(again, o) and not torch.equal(o[:2], eager[0][:2])


def test_memory_of_a_call_on_another_stream():
    # what the call allocates is given away in the order of its own stream, not of the current one that never waits for it
    pr = _problem([1] * 9 + [100], [300] * 9 + [400], 4, 2, 64, 16)
    want = _run(pr, 1.5, max_q_len=100, max_kv_len=400)
    side = torch.cuda.Stream()
    args = (pr["q"], pr["kc"], pr["vc"], 1.5, pr["table"], pr["lens"], pr["cu"])
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                   # some ms: the call's work starts after what follows here
        o, tau, _ = binding.entmax_attn_paged_fwd(*args, max_q_len=100, max_kv_len=400, stream=side)
        mine = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 12, 1 << 16, 1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24)]
        torch.cuda.synchronize()
        assert all(bool((m == 7).all()) for m in mine)
        assert torch.equal(o, want[0]) and torch.equal(tau, want[1])
        del mine
    with pytest.raises(binding.EntmaxAttnError, match="workspace"):
        binding.entmax_attn_paged_fwd(*args, workspace=torch.empty(1 << 26, dtype=torch.uint8))


def test_short_and_long_chunks_side_by_side():
    # both kinds of sequences in one call: against the definition, captured in a thread that never made such a call, and replayed among eager ones
    import threading
    new, lens = [1] * 9 + [100, 2, 60], [300, 20, 1, 77, 256, 40, 129, 9, 500, 700, 64, 60]
    pr = _problem(new, lens, 4, 2, 64, 16)
    sc = _scales(4, 1, "length")
    cuda = [t.cuda() for t in sc]
    out = dict(o=torch.zeros((sum(new), 4, 64), dtype=torch.bfloat16, device="cuda"), tau=torch.zeros((sum(new), 4), device="cuda"),
               support_size=torch.zeros((sum(new), 4), dtype=torch.int32, device="cuda"))
    call = lambda **kw: binding.entmax_attn_paged_fwd(pr["q"], pr["kc"], pr["vc"], 1.5, pr["table"], pr["lens"], pr["cu"], *cuda, **kw)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    failed = []

    def capture():
        try:
            with torch.cuda.graph(graph):
                call(**out)
        except Exception as e:  # noqa: BLE001
            failed.append(e)

    torch.cuda.synchronize()
    t = threading.Thread(target=capture)
    t.start()
    t.join()
    assert not failed, failed
    got = _run(pr, 1.5, sc)
    _check(pr, 1.5, got, sc)
    for _ in range(3):
        for x in out.values():
            x.zero_()
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert torch.equal(out["o"], got[0]) and torch.equal(out["tau"], got[1]) and torch.equal(out["support_size"], got[2])
        assert torch.equal(eager[0], got[0]) and torch.equal(eager[1], got[1])
    again = torch.cuda.CUDAGraph()
    with torch.cuda.graph(again):
        call(**out)
    out["o"].zero_()
    again.replay()
    torch.cuda.synchronize()
    assert torch.equal(out["o"], got[0])


def test_eager_call_while_another_stream_of_the_thread_is_captured():
    # the library's second stream is part of the first graph's capture until that ends: the other call does without it
    new, lens = [1] * 9 + [100, 2, 60], [300, 20, 1, 77, 256, 40, 129, 9, 500, 700, 64, 60]
    pr = _problem(new, lens, 4, 2, 64, 16)
    args = (pr["q"], pr["kc"], pr["vc"], 1.5, pr["table"], pr["lens"], pr["cu"])

    def buffers():
        return dict(o=torch.zeros((sum(new), 4, 64), dtype=torch.bfloat16, device="cuda"), tau=torch.zeros((sum(new), 4), device="cuda"),
                    workspace=torch.empty(1 << 26, dtype=torch.uint8, device="cuda"))

    want, captured, eager = buffers(), buffers(), buffers()
    binding.entmax_attn_paged_fwd(*args, **want)             # (the second stream is there from now on)
    torch.cuda.synchronize()
    graph, other = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):
        binding.entmax_attn_paged_fwd(*args, **captured)
        binding.entmax_attn_paged_fwd(*args, stream=other, **eager)
        binding.entmax_attn_paged_fwd(*args, **captured)
    other.synchronize()
    assert torch.equal(eager["o"], want["o"]) and torch.equal(eager["tau"], want["tau"])
    assert bool((captured["o"] == 0).all())
    for _ in range(2):
        captured["o"].zero_()
        graph.replay()
        binding.entmax_attn_paged_fwd(*args, **eager)
        torch.cuda.synchronize()
        assert torch.equal(captured["o"], want["o"]) and torch.equal(captured["tau"], want["tau"]) and torch.equal(eager["o"], want["o"])


@pytest.mark.parametrize("new", [1, 150])
def test_equal_logits_of_128(new):
    # every visible key in the support, and every one of its V rows gathered, four rows of 128 in flight
    pr = _problem([new, 1], [2600, 700], 2, 1, 128, 16, plant=False)
    pr["q"].zero_()
    got = _run(pr, 1.5)
    _check(pr, 1.5, got)
    assert torch.equal(got[2][:new, 0].cpu().long(), torch.arange(2600 - new + 1, 2601))


@pytest.mark.parametrize("sigma", [0.02, 0.3])
@pytest.mark.parametrize("alpha", [1.25, 1.5, 1.9, 2.0])
def test_flat_rows_of_128(sigma, alpha):
    pr = _problem([1, 90], [2000, 1300], 4, 2, 128, 32, sigma=sigma, plant=False)
    _check(pr, alpha, _run(pr, alpha))


@pytest.mark.parametrize("new,lens,H,KH,alpha", [([400, 390], [2600, 400], 8, 2, 1.5), ([1] * 50, [2000 - 7 * b for b in range(50)], 32, 4, 1.25),
                                                 ([1] * 3 + [700], [9001, 30, 5000, 700], 4, 4, 2.0)])
def test_more_rows_of_128_with_long_supports_than_lists_hold(new, lens, H, KH, alpha):
    # as for head_dim 64; rows whose lists overflow are walked by a CTA
    pr = _problem(new, lens, H, KH, 128, 32, sigma=0.3, plant=False)
    pr["q"][::2] = 0
    _check(pr, alpha, _run(pr, alpha), heads=[0, H - 1], skip=range(3, len(new), 5) if len(new) > 4 else (), rows=[0, 1, 170, 389, 699])


@pytest.mark.parametrize("new,H,KH,sigma", [(1, 16, 2, 1.0), (40, 1, 1, 1.0), (1, 4, 1, 0.05), (20, 2, 1, 0.05)])
def test_long_contexts_of_128(new, H, KH, sigma):
    pr = _problem([new], [40001], H, KH, 128, 64, sigma=sigma, plant=sigma == 1.0)
    sc = _scales(H, 5, "length") if sigma == 1.0 else None
    _check(pr, 1.5, _run(pr, 1.5, sc), sc, heads=[0, H - 1], rows=[0, new // 2, new - 1])


@pytest.mark.parametrize("alpha", [1.1, 2.5, 3.0, 8.0])
@pytest.mark.parametrize("new,lens", [([1, 1], [9000, 4097]), ([80, 3], [6000, 2500]), ([1] * 90, [1500 + b for b in range(90)])])
def test_far_alphas_over_long_contexts(alpha, new, lens):
    pr = _problem(new, lens, 4, 2, 64, 16, seed=9)
    sc = _scales(4, 7, "length")
    _check(pr, alpha, _run(pr, alpha, sc), sc, skip=range(2, len(new), 3), rows=[0, 40, 79])


MIXES = [([1] * 7, [1, 16, 17, 300, 33, 64, 129], 4, 2, 64, 16), ([5, 1, 0, 3, 8], [700, 1, 90, 3, 8], 8, 2, 128, 32),
         ([1] * 9 + [100, 2, 60], [300, 20, 1, 77, 256, 40, 129, 9, 500, 700, 64, 60], 4, 2, 64, 16), ([130, 259], [1000, 259], 6, 2, 128, 16),
         ([300], [300], 8, 1, 64, 128), ([64], [9000], 4, 2, 64, 16), ([2, 5], [300, 6], 128, 1, 64, 32), ([1] * 300, [5] * 300, 40, 8, 64, 16)]


def _paged_workspace(pr, hints):
    T = sum(pr["new"])
    cache = binding._paged_cache("workspace", pr["kc"], pr["vc"], pr["table"], pr["lens"], pr["cu"], None, T, pr["kc"].device)
    params = binding.PagedParams(T, pr["H"], *hints, 1.5, 0.0, pr["H"] * pr["d"], pr["d"])
    return binding.entmax_attn_paged_workspace_bytes(cache, params, False)


@pytest.mark.parametrize("hinted", [False, True])
@pytest.mark.parametrize("new,lens,H,KH,d,page", MIXES)
def test_attention_writes_nothing_outside_its_outputs(new, lens, H, KH, d, page, hinted):
    from test_gpu_robustness import Guarded
    pr = _problem(new, lens, H, KH, d, page, seed=H)
    hints = (max(new), max(lens)) if hinted else (0, 0)
    T = sum(new)
    sc = [t.cuda() for t in _scales(H, 4, "length")]
    slopes = torch.linspace(0.0, 0.5, H, device="cuda")
    inputs = {}
    for n in ("q", "kc", "vc", "table", "cu", "lens"):
        inputs[n] = Guarded(tuple(pr[n].shape), pr[n].dtype)
        inputs[n].t.copy_(pr[n])
    o, tau, supp = Guarded((T, H, d), torch.bfloat16), Guarded((T, H), torch.float32), Guarded((T, H), torch.int32)
    status, ws = Guarded((binding.STATUS_WORDS,), torch.int32), Guarded((_paged_workspace(pr, hints),), torch.uint8)
    i = {n: g.t for n, g in inputs.items()}
    for al in (None, slopes):
        binding.entmax_attn_paged_fwd(i["q"], i["kc"], i["vc"], 1.5, i["table"], i["lens"], i["cu"], *sc, alibi_slopes=al, max_q_len=hints[0],
                                      max_kv_len=hints[1], o=o.t, tau=tau.t, support_size=supp.t, workspace=ws.t, status=status.t)
        torch.cuda.synchronize()
        for name, g in [*inputs.items(), ("O", o), ("tau", tau), ("support", supp), ("status", status), ("workspace", ws)]:
            g.check(name)
        for n, g in inputs.items():
            assert torch.equal(g.t.contiguous().view(torch.uint8), pr[n].contiguous().view(torch.uint8)), n
        _check(pr, 1.5, (o.t, tau.t, supp.t, int(status.t[0])), _scales(H, 4, "length"), None if al is None else slopes.tolist(),
               heads=[0, H - 1], skip=range(5, len(new), 7), rows=[0, 1, 100, 299])


@pytest.mark.parametrize("new,lens,H,KH,d,page", MIXES)
def test_results_do_not_depend_on_what_the_workspace_held(new, lens, H, KH, d, page):
    pr = _problem(new, lens, H, KH, d, page, seed=H)
    sc = _scales(H, 4, "length")
    hints = dict(max_q_len=max(new), max_kv_len=max(lens))
    ws = torch.empty(_paged_workspace(pr, tuple(hints.values())), dtype=torch.uint8, device="cuda")
    want = None
    for fill in (0, 0xFF, 0x7F, 0x5A, 0x80):             # zeros, NaN, large numbers of either sign
        ws.fill_(fill)
        got = _run(pr, 1.5, sc, workspace=ws, **hints)
        want = want or got
        assert all(torch.equal(x, y) for x, y in zip(want[:3], got[:3])) and got[3] == 0


@pytest.mark.parametrize("rot,interleaved", [(0, False), (64, False), (32, True)])
@pytest.mark.parametrize("new,lens,H,KH,d,page", [m for m in MIXES if m[2] < 100])
def test_append_writes_nothing_outside_its_slots(new, lens, H, KH, d, page, rot, interleaved):
    from test_gpu_robustness import Guarded
    qkv, kc, vc, table, cu, kv_len = _append_problem(new, lens, H, KH, d, page)
    rotation = binding.rotation_table(max(lens), rot) if rot else None
    guarded = {}
    for n, t in dict(qkv=qkv, kc=kc, vc=vc, table=table, cu=cu, kv_len=kv_len, rotation=rotation).items():
        if t is not None:
            guarded[n] = Guarded(tuple(t.shape), t.dtype)
            guarded[n].t.copy_(t)
    guarded["q_out"], guarded["status"] = Guarded((sum(new), H, d), torch.bfloat16), Guarded((binding.STATUS_WORDS,), torch.int32)
    i = {n: g.t for n, g in guarded.items()}
    binding.entmax_attn_paged_append(i["qkv"][:, :H], i["qkv"][:, H:H + KH], i["qkv"][:, H + KH:], i["kc"], i["vc"], i["table"], i["kv_len"],
                                     i["cu"], rotation=i.get("rotation"), interleaved=interleaved, q_out=i["q_out"], status=i["status"])
    torch.cuda.synchronize()
    assert int(i["status"][0]) == 0
    for n, g in guarded.items():
        g.check(n)
    _check_append(qkv, H, KH, new, lens, page, rotation, interleaved, (kc, vc), (i["kc"], i["vc"]), table, i["q_out"])
    for n, t in (("qkv", qkv), ("table", table), ("cu", cu), ("kv_len", kv_len)):
        assert torch.equal(i[n].view(torch.uint8), t.contiguous().view(torch.uint8)), n


# ------------------------------------------------------------------------------------------------ append
def _append_problem(new, lens, H, KH, d, page, seed=0, layout="tokens"):
    g = torch.Generator().manual_seed(seed)
    T = sum(new)
    qkv = torch.randn((T, H + 2 * KH, d), generator=g).to(torch.bfloat16)
    past = [torch.randn((n, KH, d), generator=g).to(torch.bfloat16) for n in lens]
    kc, vc, table = paged.pool(past, [-x for x in past], page, d, KH, seed, "cuda", fill=5.0, layout=layout)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    return qkv.cuda(), kc, vc, table, cu, torch.tensor(lens, dtype=torch.int32, device="cuda")


def _check_append(qkv, H, KH, new, lens, page, rotation, interleaved, before, after, table, q_out):
    x = qkv.cpu()
    want_k, want_v = before[0].cpu().clone(), before[1].cpu().clone()
    tol_k = torch.zeros(want_k.shape, dtype=torch.float64)
    exact_k = want_k.double()
    t = 0
    for b, (n, L) in enumerate(zip(new, lens)):
        pos = torch.arange(L - n, L)
        rows = x[t:t + n]
        turned = rows[:, :H + KH].double() if rotation is None else paged.rotate(rows[:, :H + KH], rotation.cpu(), pos, interleaved)
        # two products and a sum in float32 (or fused), one rounding to bf16
        tol = 2.0 ** -8 * turned.abs() + 4 * 2.0 ** -24 * 2 * rows[:, :H + KH].double().abs().amax(-1, keepdim=True)
        if rotation is None:
            tol = torch.zeros_like(tol)
        if q_out is not None:
            assert bool(((q_out[t:t + n].cpu().double() - turned[:, :H]).abs() <= tol[:, :H]).all())
        pg, slot = table[b].cpu().long()[pos // page], pos % page
        exact_k[pg, slot], tol_k[pg, slot] = turned[:, H:], tol[:, H:]
        want_v[pg, slot] = rows[:, H + KH:]
        t += n
    assert bool(((after[0].cpu().double() - exact_k).abs() <= tol_k).all())
    assert torch.equal(after[1].cpu(), want_v)


@pytest.mark.parametrize("rot,interleaved", [(0, False), (16, False), (64, False), (64, True), (32, True)])
@pytest.mark.parametrize("new,lens,H,KH,d,page,layout", [
    ([1, 1, 1], [1, 16, 300], 4, 4, 64, 16, "tokens"),
    ([1, 0, 37, 5], [17, 40, 37, 129], 6, 2, 128, 32, "heads"),
    ([130, 1], [200, 256], 32, 8, 128, 64, "fused"),
    ([3], [3], 1, 1, 64, 16, "tokens"),
    ([b % 3 for b in range(700)], [b % 3 + 5 * (b % 50) + 1 for b in range(700)], 2, 1, 64, 16, "tokens"),
])
def test_append(rot, interleaved, new, lens, H, KH, d, page, layout):
    qkv, kc, vc, table, cu, kv_len = _append_problem(new, lens, H, KH, d, page, layout=layout)
    rotation = binding.rotation_table(max(lens), rot) if rot else None
    before = kc.clone(), vc.clone()
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    q = binding.entmax_attn_paged_append(qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:], kc, vc, table, kv_len, cu, rotation=rotation,
                                         interleaved=interleaved, status=status)
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    _check_append(qkv, H, KH, new, lens, page, rotation, interleaved, before, (kc, vc), table, q)


def test_append_in_place_without_queries_and_uniform():
    new, lens, H, KH, d, page = [2, 2, 2], [30, 2, 65], 4, 2, 64, 16
    qkv, kc, vc, table, cu, kv_len = _append_problem(new, lens, H, KH, d, page)
    rotation = binding.rotation_table(80, 64)
    before = kc.clone(), vc.clone()
    src = qkv.clone()
    q = src[:, :H]
    out = binding.entmax_attn_paged_append(q, src[:, H:H + KH], src[:, H + KH:], kc, vc, table, kv_len, None, rotation=rotation, q_out=q)
    torch.cuda.synchronize()
    assert out.data_ptr() == q.data_ptr()
    _check_append(qkv, H, KH, new, lens, page, rotation, False, before, (kc, vc), table, out)
    assert torch.equal(src[:, H:], qkv[:, H:])
    k2, v2 = before[0].clone(), before[1].clone()
    assert binding.entmax_attn_paged_append(None, qkv[:, H:H + KH], qkv[:, H + KH:], k2, v2, table, kv_len, cu, rotation=rotation) is None
    torch.cuda.synchronize()
    assert torch.equal(k2, kc) and torch.equal(v2, vc)


def test_append_at_far_positions():
    # 64-bit angles: at position 10^6 a float32 angle is off by 0.03
    L, page = 1_000_003, 4096
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn((3, 3, 64), generator=g).to(torch.bfloat16).cuda()
    table = torch.full((1, -(-L // page)), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0                                        # only the last page is there: the others are not touched
    kc = torch.zeros((1, page, 1, 64), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    rotation = binding.rotation_table(L, 64)
    kv_len = torch.tensor([L], dtype=torch.int32, device="cuda")
    q = binding.entmax_attn_paged_append(qkv[:, :1], qkv[:, 1:2], qkv[:, 2:], kc, vc, table, kv_len, rotation=rotation)
    pos = torch.arange(L - 3, L)
    i = torch.arange(32, dtype=torch.float64)
    angle = pos.double()[:, None] * 10000.0 ** (-2 * i / 64)
    x = qkv[:, :2].cpu().double()
    turned = torch.cat([x[..., :32] * angle.cos()[:, None] - x[..., 32:] * angle.sin()[:, None],
                        x[..., 32:] * angle.cos()[:, None] + x[..., :32] * angle.sin()[:, None]], -1)
    # the table's own rounding (2^-24 of each cosine and sine) beside the arithmetic's
    tol = 2.0 ** -8 * turned.abs() + 8 * 2.0 ** -24 * 2 * x.abs().amax(-1, keepdim=True)
    assert bool(((q.cpu().double() - turned[:, :1]).abs() <= tol[:, :1]).all())
    assert bool(((kc[0, pos % page].cpu().double() - turned[:, 1:]).abs() <= tol[:, 1:]).all())
    assert torch.equal(vc[0, pos % page], qkv[:, 2:])


def test_append_leaves_out_what_does_not_fit():
    new, lens, H, KH, d, page = [2, 3, 1, 1], [30, 33, 20, 10], 4, 2, 64, 16
    qkv, kc, vc, table, cu, kv_len = _append_problem(new, lens, H, KH, d, page)
    before = kc.clone(), vc.clone()
    table = table[:, :2].contiguous()                       # room for 32 tokens: the second sequence does not fit
    bad = table.clone()
    bad[2, 1] = kc.shape[0]                                 # the third one's page is not in the pool
    q = torch.full((7, H, d), 9.0, dtype=torch.bfloat16, device="cuda")
    status = torch.zeros(binding.STATUS_WORDS, dtype=torch.int32, device="cuda")
    binding.entmax_attn_paged_append(qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:], kc, vc, bad, kv_len, cu, q_out=q, status=status)
    torch.cuda.synchronize()
    assert int(status[0]) == binding.FLAG_BAD_LENGTH | binding.FLAG_BAD_PAGE
    assert bool((q[2:5] == 9).all()) and torch.equal(q[:2], qkv[:2, :H]) and torch.equal(q[5:], qkv[5:, :H])
    want = before[0].clone(), before[1].clone()
    for b, t0, n, L in ((0, 0, 2, 30), (3, 6, 1, 10)):
        for i in range(n):
            p = L - n + i
            want[0][table[b, p // page].long(), p % page] = qkv[t0 + i, H:H + KH]
            want[1][table[b, p // page].long(), p % page] = qkv[t0 + i, H + KH:]
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("H,KH,d,page", [(4, 2, 64, 16), (6, 6, 128, 32)])
def test_prompt_chunks_then_single_tokens_equal_the_whole_sequence(H, KH, d, page):
    """A prompt in two chunks, then tokens one by one, two sequences at different points: every output equals the full causal problem's row
    (entmax_attn_fwd on the rotated tokens), within the two paths' tolerances for the same inputs."""
    N, B = 150, 2
    g = torch.Generator().manual_seed(11)
    qkv = torch.randn((B, N, H + 2 * KH, d), generator=g).to(torch.bfloat16).cuda()
    rotation = binding.rotation_table(N, d)
    sc = [t.cuda() for t in _scales(H, 3, "length")]
    pages = -(-N // page)
    kc = torch.full((B * pages + 1, page, KH, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    vc = torch.full_like(kc, float("nan"))
    table = torch.randperm(B * pages, generator=g).to(torch.int32).view(B, pages).cuda()
    steps = [(64, 40), (50, 1), (1, 60), (1, 1)] + [(1, 1)] * 30
    at = [0, 0]
    rotated_q = torch.zeros((B, N, H, d), dtype=torch.bfloat16, device="cuda")
    outs = torch.zeros((B, N, H, d), dtype=torch.bfloat16, device="cuda")
    taus = torch.zeros((B, N, H), device="cuda")
    for new in steps:
        rows = torch.cat([qkv[b, at[b]:at[b] + new[b]] for b in range(B)])
        cu = torch.tensor([0, new[0], sum(new)], dtype=torch.int32, device="cuda")
        at = [at[b] + new[b] for b in range(B)]
        kv_len = torch.tensor(at, dtype=torch.int32, device="cuda")
        q = binding.entmax_attn_paged_append(rows[:, :H], rows[:, H:H + KH], rows[:, H + KH:], kc, vc, table, kv_len, cu, rotation=rotation)
        o, tau, _ = binding.entmax_attn_paged_fwd(q, kc, vc, 1.5, table, kv_len, cu, *sc, max_q_len=max(new), max_kv_len=max(at))
        for b, t0 in ((0, 0), (1, new[0])):
            where = slice(at[b] - new[b], at[b])
            rotated_q[b, where], outs[b, where], taus[b, where] = q[t0:t0 + new[b]], o[t0:t0 + new[b]], tau[t0:t0 + new[b]]
    for b in range(B):
        n = at[b]
        flat = table[b].long()
        k = kc[flat].flatten(0, 1)[:n].transpose(0, 1).repeat_interleave(H // KH, 0)[None].contiguous()
        v = vc[flat].flatten(0, 1)[:n].transpose(0, 1).repeat_interleave(H // KH, 0)[None].contiguous()
        q = rotated_q[b, :n].transpose(0, 1)[None].contiguous()
        o, tau = binding.entmax_attn_fwd(q, k, v, 1.5, True, *sc)
        for h in range(H):
            ro, rt, to, tt, _, _ = paged.attend(q[0, h].cpu(), k[0, h].cpu(), v[0, h].cpu(), 0, 1.5, [s[h].cpu() for s in sc])
            assert bool(((taus[b, :n, h].cpu().double() - rt).abs() <= tt).all())
            assert bool(((outs[b, :n, h].cpu().double() - ro).abs() <= to).all())
            assert bool(((tau[0, h].cpu().double() - taus[b, :n, h].cpu().double()).abs() <= 2 * tt).all())
            assert bool(((o[0, h].cpu().double() - outs[b, :n, h].cpu().double()).abs() <= 2 * to).all())
