"""Softmax attention over a paged cache (entmax_attn_softmax_paged_fwd) and the tables of a serving step (entmax_attn_paged_tables): against the
definition in 64 bits (tests/softmax.py derives the tolerances) and a plain walk over the requests."""
import numpy as np
import pytest
import torch

import paged
import softmax
from paper_2506_16640_b200 import binding

pytestmark = pytest.mark.gpu


def _problem(new, lens, H, KH, d, page, seed=0, sigma=1.0, layout="tokens", rows_behind=0):
    g = torch.Generator().manual_seed(seed)
    T = sum(new)
    q = (torch.randn((T + rows_behind, H, d), generator=g) * sigma).to(torch.bfloat16)
    keys = [(torch.randn((max(n, 0), KH, d), generator=g) * sigma).to(torch.bfloat16) for n in lens]
    values = [torch.randn((max(n, 0), KH, d), generator=g).to(torch.bfloat16) for n in lens]
    kc, vc, table = paged.pool(keys, values, page, d, KH, seed, "cuda", layout=layout)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    return dict(q=q.cuda(), keys=keys, values=values, kc=kc, vc=vc, table=table, cu=cu,
                lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), new=list(new), kv=list(lens), H=H, KH=KH, d=d)


def _terms(kind, H, seed=0):
    g = torch.Generator().manual_seed(50 + seed)
    t = {}
    for word in kind.split("+"):
        if word == "cap":
            t["softcap"] = 15.0
        elif word == "slopes":
            t["alibi_slopes"] = torch.where(torch.arange(H) % 2 == 0, 2.0 ** -(torch.arange(H) % 8 + 1.0), torch.zeros(H)).cuda()
        elif word == "length":
            t["beta"], t["gamma"], t["delta"] = (0.2 + 0.6 * torch.rand(H, generator=g).cuda() for _ in range(3))
        elif word == "negative":
            t["beta"], t["gamma"] = torch.zeros(H).cuda(), torch.ones(H).cuda()
            t["delta"] = torch.tensor([-1.0, 0.0, 0.7])[torch.arange(H) % 3].cuda()
        elif word.startswith("window"):
            t["window"] = int(word[6:])
    return t


def _run(pr, t=None, **kw):
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    o, lse = binding.entmax_attn_softmax_paged_fwd(pr["q"], pr["kc"], pr["vc"], pr["table"], pr["lens"], kw.pop("cu", pr["cu"]), status=status,
                                                   **(t or {}), **kw)
    torch.cuda.synchronize()
    return o, lse, int(status[0])


def _check(pr, got, t=None, skip=(), heads=None, flags=0, sm=None):
    t = t or {}
    o, lse, have = got
    assert have == flags
    o, lse, q = o.cpu(), lse.cpu(), pr["q"].cpu()
    at = 0
    for b, n in enumerate(pr["new"]):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        if b in skip:
            assert (o[rows] == 0).all() and (lse[rows] == -float("inf")).all()
            continue
        pos = torch.arange(pr["kv"][b] - n, pr["kv"][b])
        lo = (pos + 1 - t["window"]).clamp_min(0) if t.get("window") else torch.zeros_like(pos)
        for h in heads or range(pr["H"]):
            kh = h * pr["KH"] // pr["H"]
            c = None if "beta" not in t else softmax.scale(*(t[x][h].cpu().double() for x in ("beta", "gamma", "delta")), pos + 1 - lo)
            slope = float(t["alibi_slopes"][h]) if "alibi_slopes" in t else 0.0
            want = softmax.head(q[rows, h], pr["keys"][b][:, kh], pr["values"][b][:, kh], lo, pos + 1, c, sm, t.get("softcap", 0.0), slope, pos=pos)
            where = "sequence %d of %d new tokens over %d, head %d" % (b, n, pr["kv"][b], h)
            softmax.check("o", o[rows, h], want, where)
            softmax.check("lse", lse[rows, h], want, where)


@pytest.mark.parametrize("H,KH,d,page", [(1, 1, 64, 16), (12, 12, 64, 16), (16, 2, 64, 32), (32, 8, 128, 16), (8, 1, 128, 64), (10, 2, 128, 256),
                                         (6, 2, 64, 128), (40, 1, 64, 16)])
def test_single_tokens(H, KH, d, page):
    pr = _problem([1] * 7, [1, 2, 15, 16, 17, 300, 1025], H, KH, d, page, seed=H)
    _check(pr, _run(pr))


@pytest.mark.parametrize("new,lens,H,KH,d,page", [
    ([2, 5, 8], [2, 77, 500], 8, 2, 64, 16), ([3, 1, 9, 12], [900, 1, 9, 64], 12, 4, 128, 32), ([17, 0, 33], [40, 5, 700], 4, 4, 64, 16),
    ([130, 1, 64], [130, 400, 1000], 8, 2, 128, 64), ([257], [1300], 6, 2, 64, 128), ([1, 300, 2, 129, 1], [50, 300, 3, 700, 900], 4, 1, 128, 16),
    ([128, 127, 256], [128, 127, 256], 2, 2, 64, 256), ([20, 21], [600, 33], 16, 2, 128, 16)])
def test_chunks(new, lens, H, KH, d, page):
    pr = _problem(new, lens, H, KH, d, page, seed=sum(new))
    _check(pr, _run(pr))


@pytest.mark.parametrize("H,d,page", [(71, 64, 16), (128, 128, 32), (64, 64, 4096), (65, 128, 64)])
def test_one_kv_head_for_many_query_heads(H, d, page):
    pr = _problem([1, 1, 2, 1], [1, 700, 90, 129], H, 1, d, page, seed=H)
    _check(pr, _run(pr))


@pytest.mark.parametrize("kind", ["cap", "slopes", "length", "negative", "window1", "window40", "cap+slopes+length+window100", "slopes+negative"])
@pytest.mark.parametrize("new,lens", [([1, 1, 1], [1, 200, 1030]), ([3, 2, 5], [600, 2, 70]), ([150, 1, 40], [700, 90, 40])])
def test_terms(kind, new, lens):
    for H, KH, d, page in [(6, 2, 64, 16), (8, 4, 128, 32)]:
        pr = _problem(new, lens, H, KH, d, page, seed=len(kind))
        t = _terms(kind, H)
        _check(pr, _run(pr, t), t)


@pytest.mark.parametrize("sigma", [0.02, 5.0])
@pytest.mark.parametrize("new,lens", [([1, 1], [900, 33]), ([140, 6], [500, 300])])
def test_flat_and_sharp_rows(sigma, new, lens):
    pr = _problem(new, lens, 4, 2, 128, 16, seed=1, sigma=sigma)
    _check(pr, _run(pr))


@pytest.mark.parametrize("layout", ["heads", "fused"])
@pytest.mark.parametrize("new,lens", [([1, 1], [100, 513]), ([131, 4], [200, 90])])
def test_layouts_and_strided_queries(layout, new, lens):
    pr = _problem(new, lens, 6, 2, 64, 16, seed=3, layout=layout)
    wide = torch.zeros((sum(new), 9, 64 + 8), dtype=torch.bfloat16, device="cuda")
    wide[:, :6, :64] = pr["q"]
    pr["q"] = wide[:, :6, :64]
    _check(pr, _run(pr))


@pytest.mark.parametrize("new,lens", [([1, 1], [100, 513]), ([131, 4], [200, 90])])
def test_rows_behind_the_last_sequence_stay(new, lens):
    pr = _problem(new, lens, 4, 2, 64, 16, rows_behind=5)
    T = sum(new)
    o = torch.full((T + 5, 4, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 5, 4), 3.0, device="cuda")
    got = _run(pr, o=o, lse=lse)
    assert (o[T:] == 3.0).all() and (lse[T:] == 3.0).all()
    _check(pr, got)


@pytest.mark.parametrize("new,lens,bad", [([1, 2, 1], [100, 1, 50], [1]), ([1, 1, 1], [-5, 40, -1], [0, 2]), ([200, 1], [100, 30], [0])])
def test_lengths_that_do_not_fit(new, lens, bad):
    pr = _problem(new, lens, 4, 2, 64, 16)
    _check(pr, _run(pr), skip=bad, flags=binding.FLAG_BAD_LENGTH)


@pytest.mark.parametrize("new,max_q,max_kv,bad", [([1, 1, 1], 1, 60, [2]), ([1, 5, 1], 4, 0, [1]), ([130, 140, 1], 130, 0, [1])])
def test_bounds_that_are_too_small(new, max_q, max_kv, bad):
    lens = [50, 200 if not max_kv else 60, 61]
    pr = _problem(new, [max(n, x) for n, x in zip(new, lens)], 4, 2, 64, 16)
    _check(pr, _run(pr, max_q_len=max_q, max_kv_len=max_kv), skip=bad, flags=binding.FLAG_BAD_LENGTH)


@pytest.mark.parametrize("new", [1, 3, 140])
def test_pages_outside_the_pool(new):
    pr = _problem([new] * 3, [300] * 3, 4, 2, 64, 16)
    pr["table"][1, 3] = pr["kc"].shape[0]
    o, lse, flags = _run(pr)
    assert flags == binding.FLAG_BAD_PAGE
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    # the other sequences are as they were
    for b in (0, 2):
        pr2 = dict(pr, new=[new], kv=[300], keys=[pr["keys"][b]], values=[pr["values"][b]], q=pr["q"][b * new:(b + 1) * new])
        _check(pr2, (o[b * new:(b + 1) * new], lse[b * new:(b + 1) * new], 0))


def test_large_batches():
    lens = [1 + (i * 37) % 90 for i in range(700)]
    pr = _problem([1] * 700, lens, 4, 2, 64, 16, seed=2)
    _check(pr, _run(pr), heads=[1])
    new = [1 + (i % 40 == 7) * 150 for i in range(300)]
    lens = [n + (i * 53) % 200 for i, n in enumerate(new)]
    pr = _problem(new, lens, 4, 2, 64, 32, seed=3)
    _check(pr, _run(pr), heads=[2])


def test_uniform_chunks_without_offsets():
    for n in (1, 4, 150):
        pr = _problem([n] * 3, [n, n + 200, n + 7], 4, 2, 64, 16)
        _check(pr, _run(pr, cu=None))


@pytest.mark.parametrize("new,H,KH,d", [(1, 8, 1, 128), (4, 8, 8, 64), (200, 4, 1, 128)])
def test_long_contexts(new, H, KH, d):
    # few rows over a long cache: shared among many CTAs and joined
    pr = _problem([new, new], [20000, 7777], H, KH, d, 64, seed=5)
    _check(pr, _run(pr), heads=[0, H - 1])
    t = _terms("window9000+cap", H)
    _check(pr, _run(pr, t), t, heads=[1 % H])


def test_offsets_beyond_32_bits():
    # a pool whose slots lie more than 2^31 elements apart
    page, KH, d, pages = 16, 1, 64, 5
    stride = (1 << 29) + 64
    big = torch.zeros(4 * stride + page * KH * d, dtype=torch.bfloat16, device="cuda")
    pr = _problem([1, 2, 130], [64, 70, 140], 2, KH, d, page, seed=6)
    small_k, small_v = pr["kc"], pr["vc"]
    for new, lens in (([1], [80]), ([40], [75])):
        pr = _problem(new, lens, 4, KH, d, page, seed=6)
        order = torch.tensor([4, 1, 3, 0, 2])
        kc = big.as_strided((pages, page, KH, d), (stride, KH * d, d, 1))
        vbig = torch.zeros_like(big)
        vc = vbig.as_strided((pages, page, KH, d), (stride, KH * d, d, 1))
        for i in range(-(-lens[0] // page)):
            kc[order[i]] = pr["kc"][pr["table"][0, i].long()]
            vc[order[i]] = pr["vc"][pr["table"][0, i].long()]
            pr["table"][0, i] = order[i]
        pr["kc"], pr["vc"] = kc, vc
        _check(pr, _run(pr))
        del vbig, vc
    assert small_k.shape == small_v.shape


@pytest.mark.parametrize("new,lens,H,KH,d", [([1, 1, 1], [4000, 100, 900], 8, 2, 128), ([130, 1, 5], [300, 2000, 90], 4, 4, 64)])
def test_repeats_are_bit_equal_whatever_the_workspace_held(new, lens, H, KH, d):
    pr = _problem(new, lens, H, KH, d, 16, seed=7)
    ref = _run(pr)
    need = 1 << 27
    for fill in (0, 0xff, 0x7f):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        got = _run(pr, workspace=ws)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("new,lens,H,KH,d,page,kind", [
    ([3, 2, 5], [600, 2, 70], 8, 4, 128, 32, "window100"), ([1] * 5, [700, 33, 64, 1000, 17], 8, 2, 128, 16, "window300"),
    ([300, 1, 140], [700, 90, 400], 8, 4, 64, 16, "window90+cap"), ([300, 260], [333, 1400], 4, 2, 128, 256, "cap")])
def test_many_repeats_over_slots_that_hold_anything(new, lens, H, KH, d, page, kind):
    # tiles with slots that no row sees (NaN here), cleared in time in every one of many runs
    pr = _problem(new, lens, H, KH, d, page, seed=27)
    t = _terms(kind, H)
    ref = _run(pr, t)
    _check(pr, ref, t)
    for _ in range(500):
        got = _run(pr, t)
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


@pytest.mark.parametrize("n", [1, 4, 140])
def test_a_sequence_does_not_depend_on_what_is_packed_around_it(n):
    # the same sequence alone, and with a neighbour of huge queries: bit for bit
    t = _terms("cap+slopes", 4)
    pr = _problem([n, 130], [n + 300, 200], 4, 2, 128, 16, seed=41)
    pr["q"][n:] *= 100.0
    both = _run(pr, t)
    alone = dict(pr, q=pr["q"][:n].contiguous(), cu=pr["cu"][:2].contiguous(), lens=pr["lens"][:1].contiguous(), table=pr["table"][:1].contiguous())
    # (the bounds of the larger call, which the launches go by)
    one = _run(alone, t, max_q_len=n, max_kv_len=0)
    two = _run(pr, t, max_q_len=max(n, 130), max_kv_len=0)
    assert torch.equal(both[0], two[0])
    assert (one[0].float() - two[0][:n].float()).abs().max() <= 2.0 ** -7 * two[0][:n].float().abs().max()
    small = dict(pr, q=pr["q"].clone())
    small["q"][n:] *= 0.001
    three = _run(small, t)
    assert torch.equal(three[0][:n], both[0][:n]) and torch.equal(three[1][:n], both[1][:n])


def test_writes_nothing_outside_its_outputs():
    for new, lens in (([1, 1], [700, 64]), ([140, 3], [400, 50])):
        pr = _problem(new, lens, 6, 2, 64, 16, seed=8)
        T = sum(new)
        po = torch.full((T + 2, 6, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        pl = torch.full((T + 2, 6), 5.0, device="cuda")
        kc, vc = pr["kc"].clone(), pr["vc"].clone()
        _check(pr, _run(pr, o=po[1:-1], lse=pl[1:-1]))
        assert (po[0] == 5.0).all() and (po[-1] == 5.0).all() and (pl[0] == 5.0).all() and (pl[-1] == 5.0).all()
        assert torch.equal(kc.view(torch.int16), pr["kc"].view(torch.int16)) and torch.equal(vc.view(torch.int16), pr["vc"].view(torch.int16))


def test_graph_replay_and_two_calls_at_once():
    prs = [_problem([1, 1], [900, 4000], 8, 2, 128, 16, seed=9), _problem([150, 2], [600, 80], 4, 2, 64, 32, seed=10)]
    refs = [_run(pr) for pr in prs]
    outs = [(torch.empty_like(r[0]), torch.empty_like(r[1])) for r in refs]
    spaces = [torch.empty(1 << 26, dtype=torch.uint8, device="cuda") for _ in prs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for pr, out, ws in zip(prs, outs, spaces):
            binding.entmax_attn_softmax_paged_fwd(pr["q"], pr["kc"], pr["vc"], pr["table"], pr["lens"], pr["cu"], o=out[0], lse=out[1], workspace=ws)
    for _ in range(2):
        for out in outs:
            out[0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for out, ref in zip(outs, refs):
            assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
    streams = [torch.cuda.Stream() for _ in prs]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [binding.entmax_attn_softmax_paged_fwd(pr["q"], pr["kc"], pr["vc"], pr["table"], pr["lens"], pr["cu"], stream=s)
               for pr, s in zip(prs, streams)]
        torch.cuda.synchronize()
        for x, ref in zip(got, refs):
            assert torch.equal(x[0], ref[0]) and torch.equal(x[1], ref[1])


# ------------------------------------------------------------------------------------------------------------ tables
def _walk(kv, new, table, free, count, page, max_pages, n_pages, total):
    """The tables of a step, request by request, on lists."""
    table, free = [list(r) for r in table], list(free)
    stack, rest = list(free[:count]), count
    kv_out, cu, pos, slot, back, flags = [], [0], [-7] * total, [-7] * total, [], 0
    short = False
    for b, (have, m) in enumerate(zip(kv, new)):
        have = -1 - have if have < 0 else have
        at = cu[-1]
        cu.append(at + max(m, 0))
        if have > max_pages * page or m < -1 or (m > 0 and have + m > max_pages * page):
            kv_out.append(-1 - have)
            flags |= binding.FLAG_BAD_LENGTH
            fine = False
        elif m == -1:
            kv_out.append(0)
            back += table[b][:-(-have // page)]
            continue
        else:
            need = -(-(have + m) // page) - -(-have // page)
            short = short or need > rest
            fine = need == 0 or not short
            if fine:
                for i in range(need):
                    table[b][-(-have // page) + i] = stack.pop()
                rest -= need
                kv_out.append(have + m)
            else:
                kv_out.append(-1 - have)
                flags |= binding.FLAG_NO_PAGES
        for i in range(max(m, 0)):
            if at + i < total:
                pos[at + i] = have + i if fine else -1
                pg = table[b][(have + i) // page] if fine else -1
                slot[at + i] = pg * page + (have + i) % page if 0 <= pg < n_pages else -1
    if cu[-1] > total:
        flags |= binding.FLAG_BAD_LENGTH
    stack += back
    return kv_out, cu, pos, slot, table, stack, flags


def _step(kv, new, table, free, count, page, n_pages, total=None, in_place=False):
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    total = sum(max(m, 0) for m in new) if total is None else total
    t_kv, t_new, t_table, t_free, t_count = dev(kv), dev(new), dev(table), dev(free), dev([count])
    pos = torch.full((total,), -7, dtype=torch.int32, device="cuda")
    slot = torch.full((total,), -7, dtype=torch.int64, device="cuda")
    status = torch.full((binding.STATUS_WORDS,), -1, dtype=torch.int32, device="cuda")
    kw = dict(kv_len_out=t_kv, free_count_out=t_count) if in_place else {}
    kv_out, cu, pos, slot, left = binding.entmax_attn_paged_tables(t_kv, t_new, t_table, t_free, t_count, page, n_pages, total, positions=pos,
                                                                   slots=slot, status=status, **kw)
    torch.cuda.synchronize()
    return kv_out.tolist(), cu.tolist(), pos.tolist(), slot.tolist(), t_table.tolist(), t_free.tolist()[:int(left)], int(status[0])


def _requests(B, page, seed, most_new=40, ended=0.1, bad=0.0, again=0.1):
    rng = np.random.default_rng(seed)
    max_pages = 12
    kv = rng.integers(0, max_pages * page // 2, B)
    new = np.where(rng.random(B) < 0.3, rng.integers(0, most_new, B), 1)
    new = np.where(rng.random(B) < ended, -1, new)
    wrong = rng.random(B) < bad
    new = np.where(wrong, rng.choice([max_pages * page + 1, -3, 2 ** 31 - 1 if bad > 0.3 else -2], B), new)
    have = -(-kv // page)
    order = rng.permutation(int(have.sum()) + B * 4)
    table, at = [[-9] * max_pages for _ in range(B)], 0
    for b in range(B):
        table[b][:have[b]] = order[at:at + have[b]].tolist()
        at += int(have[b])
    kv = np.where(rng.random(B) < again, -1 - kv, kv)
    return kv.tolist(), new.tolist(), table, order[at:].tolist(), len(order)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,page,room,bad", [(1, 16, 1.0, 0.0), (3, 32, 1.0, 0.2), (70, 16, 0.1, 0.0), (1000, 16, 1.0, 0.02), (1024, 64, 0.05, 0.1),
                                             (1025, 16, 1.0, 0.0), (3500, 16, 0.15, 0.05)])
def test_tables(B, page, room, bad, in_place):
    kv, new, table, free, n_pages = _requests(B, page, B + page, bad=bad)
    count = int(len(free) * room)
    free = free + [-5] * (n_pages - len(free))                   # room for what comes back
    total = min(sum(max(m, 0) for m in new), 200000)
    want = _walk(kv, new, table, free, count, page, 12, n_pages, total)
    got = _step(kv, new, table, free, count, page, n_pages, total, in_place)
    for name, x, y in zip(("kv_len", "cu_q", "positions", "slots", "table", "stack", "flags"), got, want):
        assert x == y, name


def test_tables_edges():
    # no tokens at all; exactly the last page; one page too few; a token more than fits; more tokens than rows; pages from outside the pool
    assert _step([0], [0], [[1, 2]], [4, 5], 2, 16, 6)[0] == [0]
    assert _step([16], [16], [[3, -1]], [4, 5], 1, 16, 6) == ([32], [0, 16], list(range(16, 32)), list(range(64, 80)), [[3, 4]], [], 0)
    assert _step([16], [1], [[3, -1]], [4, 5], 0, 16, 6) == ([-17], [0, 1], [-1], [-1], [[3, -1]], [], binding.FLAG_NO_PAGES)
    assert _step([31], [2], [[3, 4]], [5], 1, 16, 6) == ([-32], [0, 2], [-1, -1], [-1, -1], [[3, 4]], [5], binding.FLAG_BAD_LENGTH)
    assert _step([3, 4], [2, 2], [[0], [1]], [5], 1, 16, 6, total=3)[:4] == ([5, 6], [0, 2, 4], [3, 4, 4], [3, 4, 20])
    got = _step([16, 3], [1, 1], [[3, -1], [77, -1]], [9], 1, 16, 6)
    assert got[3] == [-1, -1] and got[4] == [[3, 9], [77, -1]] and got[6] == binding.FLAG_BAD_PAGE
    # back onto a stack without room
    assert _step([33], [-1], [[3, 4, 5]], [1, 0], 1, 16, 6) [5:] == ([1, 3], binding.FLAG_BAD_PAGE)
    # a wrong count is held to the stack
    assert _step([0], [1], [[7]], [4], 9, 16, 6) == ([1], [0, 1], [0], [64], [[4]], [], binding.FLAG_BAD_LENGTH)


def test_tables_of_long_prompts():
    # many tokens: several CTAs
    page, B = 16, 37
    new = [1 + (i * 977) % 3000 for i in range(B)]
    kv = [(i * 31) % 500 for i in range(B)]
    have = [-(-x // page) for x in kv]
    most = max(-(-(x + m) // page) for x, m in zip(kv, new))
    order = np.random.default_rng(0).permutation(sum(have) + 37 * 200).tolist()
    table, at = [], 0
    for b in range(B):
        table.append(order[at:at + have[b]] + [-9] * (most - have[b]))
        at += have[b]
    free, count = order[at:], len(order) - at
    want = _walk(kv, new, table, free, count, page, most, len(order), sum(new))
    assert _step(kv, new, table, free, count, page, len(order)) == want


def test_a_serving_run():
    """Prompts, then single tokens, sequences that end and others that take their pages: tables, append, attention of both kinds, against the
    whole sequences; the steps captured as a graph give the same."""
    H, KH, d, page, n_pages, B = 4, 2, 64, 16, 40, 4
    g = torch.Generator().manual_seed(3)
    kc, vc = (torch.full((n_pages, page, KH, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((B, 10), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(n_pages, generator=g).to(torch.int32).cuda()
    count = torch.tensor([n_pages], dtype=torch.int32, device="cuda")
    kv = torch.zeros(B, dtype=torch.int32, device="cuda")
    history = [([], []) for _ in range(B)]
    steps = [[20, 1, 37, 0], [1, 1, 1, 50], [1, 1, 1, 1], [1, -1, 1, 1], [1, 140, -1, 1], [5, 1, 40, 1], [1, 1, 1, 1]]
    for new in steps:
        T = sum(max(m, 0) for m in new)
        qkv = torch.randn((T, H + 2 * KH, d), generator=g).to(torch.bfloat16).cuda()
        q, k, v = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
        status = torch.zeros(binding.STATUS_WORDS, dtype=torch.int32, device="cuda")
        kv, cu, pos, slots, count = binding.entmax_attn_paged_tables(kv, torch.tensor(new, dtype=torch.int32, device="cuda"), table, free, count, page,
                                                                     n_pages, T, kv_len_out=kv, free_count_out=count, status=status)
        assert int(status[0]) == 0
        binding.entmax_attn_paged_append(None, k, v, kc, vc, table, kv, cu)
        # the slot map says the same as the append
        assert torch.equal(kc.view(-1, KH, d)[slots], k) and torch.equal(vc.view(-1, KH, d)[slots], v)
        o, lse = binding.entmax_attn_softmax_paged_fwd(q, kc, vc, table, kv, cu, softcap=15.0, status=status)
        assert int(status[0]) == 0
        oe, _, _ = binding.entmax_attn_paged_fwd(q, kc, vc, 1.5, table, kv, cu, status=status)
        assert int(status[0]) == 0 and torch.isfinite(oe).all()
        at = 0
        for b, m in enumerate(new):
            if m == -1:
                history[b] = ([], [])
                continue
            history[b][0].append(k[at:at + m].cpu())
            history[b][1].append(v[at:at + m].cpu())
            if m:
                keys, values = torch.cat(history[b][0]), torch.cat(history[b][1])
                n = keys.shape[0]
                assert pos[at:at + m].tolist() == list(range(n - m, n))
                where = torch.arange(n - m, n)
                for h in range(H):
                    want = softmax.head(q[at:at + m, h].cpu(), keys[:, h // 2], values[:, h // 2], torch.zeros_like(where), where + 1, None, None, 15.0,
                                        pos=where)
                    softmax.check("o", o[at:at + m, h], want)
                    softmax.check("lse", lse[at:at + m, h], want)
                    one, tau, tol_o, _, _, _ = paged.attend(q[at:at + m, h].cpu(), keys[:, h // 2], values[:, h // 2], n - m, 1.5)
                    assert ((oe[at:at + m, h].cpu().double() - one).abs() <= tol_o).all()
            at += m
    held = [int(x) for b in range(B) for x in table[b][:-(-int(kv[b]) // page)]]
    assert sorted(held + free[:int(count)].tolist()) == list(range(n_pages))


def test_decoding_steps_replayed_from_a_graph():
    """One captured step of tables, append and attention, lengths and stack in place, replayed: every replay is the next step."""
    H, KH, d, page, n_pages, B, steps = 4, 2, 64, 16, 30, 3, 20
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn((B, H + 2 * KH, d), generator=g).to(torch.bfloat16).cuda()
    q, k, v = qkv[:, :H], qkv[:, H:H + KH], qkv[:, H + KH:]
    kc, vc = (torch.zeros((n_pages, page, KH, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.full((B, 8), -1, dtype=torch.int32, device="cuda")
    free = torch.arange(n_pages, dtype=torch.int32, device="cuda")
    count = torch.tensor([n_pages], dtype=torch.int32, device="cuda")
    kv, one = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")

    def step():
        _, cu, _, _, _ = binding.entmax_attn_paged_tables(kv, one, table, free, count, page, n_pages, B, kv_len_out=kv, free_count_out=count)
        binding.entmax_attn_paged_append(None, k, v, kc, vc, table, kv, cu)
        return binding.entmax_attn_softmax_paged_fwd(q, kc, vc, table, kv, cu)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = step()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    assert kv.tolist() == [steps + 1] * B and int(count) == n_pages - B * 2
    # every key of a sequence is the same one: the mean of equal values, and ln n on top of the score
    z = (q.float() * k.float().repeat_interleave(H // KH, 1)).sum(-1) / d ** 0.5
    assert torch.allclose(lse, z + float(np.log(steps + 1)), atol=1e-4, rtol=0)
    assert torch.equal(o, v.repeat_interleave(H // KH, 1))
