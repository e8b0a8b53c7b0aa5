"""Paged-cache entry points without a GPU: sizes, refusals before any device work, and the 64-bit reference's own pins."""
import ctypes
import math

import pytest
import torch

import paged
from paper_2506_16640_b200 import build as lib_build


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    from paper_2506_16640_b200 import binding
    return binding.load()


def _cache(**kw):
    from paper_2506_16640_b200.binding import PagedCache
    base = dict(batch=3, kv_heads=2, head_dim=64, page_size=16, num_pages=100, max_pages=20, table_stride=20, stride_page=16 * 128,
                stride_token=128, stride_head=64)
    base.update(kw)
    return PagedCache(**base)


def _params(**kw):
    from paper_2506_16640_b200.binding import PagedParams
    base = dict(total_q=3, q_heads=4, max_q_len=0, max_kv_len=0, alpha=1.5, sm_scale=0.0, q_stride_t=256, q_stride_h=64)
    base.update(kw)
    return PagedParams(**base)


def _append(**kw):
    from paper_2506_16640_b200.binding import PagedAppendParams
    base = dict(total_q=3, q_heads=4, rot_dim=64, rot_positions=400, interleaved=0, q_stride_t=256, q_stride_h=64, k_stride_t=128,
                k_stride_h=64, v_stride_t=128, v_stride_h=64, out_stride_t=256, out_stride_h=64)
    base.update(kw)
    return PagedAppendParams(**base)


BAD_CACHES = [dict(batch=0), dict(kv_heads=0), dict(head_dim=96), dict(page_size=8), dict(page_size=48), dict(page_size=1 << 17),
              dict(num_pages=0), dict(max_pages=0), dict(table_stride=19), dict(max_pages=1 << 21, table_stride=1 << 21),
              dict(stride_page=1028), dict(stride_token=4), dict(stride_head=32), dict(stride_head=0)]
BAD_PARAMS = [dict(total_q=0), dict(q_heads=0), dict(q_heads=3), dict(q_heads=2 * 129), dict(alpha=1.0), dict(alpha=65.0), dict(alpha=math.nan),
              dict(sm_scale=-1.0), dict(sm_scale=math.inf), dict(max_q_len=-1), dict(max_kv_len=-1), dict(q_stride_t=252), dict(q_stride_h=8),
              dict(total_q=1 << 30)]


def _size(lib, c, p, uniform=0):
    return lib.entmax_attn_paged_workspace_bytes(ctypes.byref(c), ctypes.byref(p), uniform)


def test_workspace_sizes(lib):
    one = _size(lib, _cache(), _params(), 1)
    # three sequences of one token, four heads: a score row of 20 * 16 keys rounded up to 512 each, and its maxima
    assert 3 * 4 * 512 * 4 <= one <= 3 * 4 * 512 * 4 * 2 + 4096
    assert _size(lib, _cache(), _params(max_kv_len=100), 1) < one
    # unknown chunk lengths: room for longer chunks too
    assert _size(lib, _cache(), _params(), 0) > one
    # the scores held at a time are bounded, however many rows there are
    big = _cache(batch=64, max_pages=1 << 15, table_stride=1 << 15)
    assert _size(lib, big, _params(total_q=65536)) < 5 << 30
    for kw in BAD_CACHES:
        assert _size(lib, _cache(**kw), _params()) == 0, kw
    for kw in BAD_PARAMS:
        assert _size(lib, _cache(), _params(**kw)) == 0, kw
    assert _size(lib, _cache(), _params(total_q=4), 1) == 0          # four tokens over three sequences


def test_attention_refusals(lib):
    fake, odd, nul = ctypes.c_void_p(4096), ctypes.c_void_p(4100), ctypes.c_void_p(0)

    def call(c=None, p=None, q=fake, kc=fake, lens=fake, cu=fake, beta=None, o=fake, ws=fake, nbytes=1 << 40, tau=fake):
        c, p = c or _cache(), p or _params()
        return lib.entmax_attn_paged_fwd(ctypes.byref(c), ctypes.byref(p), q, kc, fake, cu, lens, fake, beta, None, None, None, o, tau, None, ws,
                                         nbytes, None, None)

    for kw in BAD_CACHES:
        assert call(c=_cache(**kw)) == -1, kw
    for kw in BAD_PARAMS:
        assert call(p=_params(**kw)) == (-2 if "alpha" in kw or "sm_scale" in kw else -1), kw
    assert call(p=_params(total_q=4), cu=None) == -1
    assert call(q=nul) == call(kc=nul) == call(lens=nul) == call(o=nul) == call(tau=nul) == -6
    assert call(beta=fake) == -6                                      # beta without gamma and delta
    assert call(q=odd) == call(kc=odd) == call(o=odd) == -4
    assert call(lens=ctypes.c_void_p(4097)) == -4
    assert call(ws=nul) == call(ws=ctypes.c_void_p(4096 + 16)) == call(nbytes=1000) == -5


def test_append_refusals(lib):
    fake, odd, nul = ctypes.c_void_p(4096), ctypes.c_void_p(4104), ctypes.c_void_p(0)

    def call(c=None, p=None, q=fake, k=fake, rot=fake, cu=fake, lens=fake, out=fake, kc=fake):
        c, p = c or _cache(), p or _append()
        return lib.entmax_attn_paged_append(ctypes.byref(c), ctypes.byref(p), q, k, fake, rot, cu, lens, fake, out, kc, fake, None, None)

    for kw in BAD_CACHES:
        assert call(c=_cache(**kw)) == -1, kw
    for kw in [dict(total_q=0), dict(rot_dim=80), dict(rot_dim=24), dict(rot_dim=-16), dict(rot_positions=0), dict(k_stride_t=4),
               dict(v_stride_h=60), dict(q_stride_t=8), dict(out_stride_h=68)]:
        assert call(p=_append(**kw)) == -1, kw
    assert call(p=_append(total_q=4), cu=None) == -1
    assert call(q=nul) == call(out=nul) == call(k=nul) == call(kc=nul) == call(lens=nul) == -6
    assert call(rot=nul) == -6 and call(p=_append(rot_dim=0)) == -6   # a table and rot_dim go together
    assert call(q=odd) == call(k=odd) == call(kc=odd) == call(rot=odd) == -4
    assert call(p=_append(out_stride_t=512)) == -1                    # in place with other strides (q and q_out are the same address)


def test_binding_refusals():
    from paper_2506_16640_b200 import binding
    E = binding.EntmaxAttnError
    bf = torch.bfloat16
    kc = torch.zeros((10, 16, 2, 64), dtype=bf)
    table, lens = torch.zeros((3, 4), dtype=torch.int32), torch.ones(3, dtype=torch.int32)
    cu = torch.tensor([0, 1, 2, 3], dtype=torch.int32)
    q, k = torch.zeros((3, 4, 64), dtype=bf), torch.zeros((3, 2, 64), dtype=bf)

    def fwd(match, q=q, kc=kc, vc=None, table=table, lens=lens, cu=cu, **kw):
        with pytest.raises(E, match=match):
            binding.entmax_attn_paged_fwd(q, kc, kc if vc is None else vc, 1.5, table, lens, cu, **kw)

    fwd("bfloat16", q=q.float())
    fwd("bfloat16", q=q[0])
    fwd("bfloat16", kc=kc.float())
    fwd("share", vc=kc[:, :8])
    fwd("head_dim", q=torch.zeros((3, 4, 128), dtype=bf))
    fwd("block_table", table=table.long())
    fwd("block_table", table=table.t())
    fwd("kv_len", lens=lens.long())
    fwd("kv_len", lens=lens[:2])
    fwd("cu_q", cu=cu[:3])
    fwd("multiple", q=torch.zeros((4, 4, 64), dtype=bf), cu=None)
    fwd("beta", beta=torch.ones(3), gamma=torch.ones(4), delta=torch.ones(4))
    fwd("alibi", alibi_slopes=torch.ones(4, dtype=torch.float64))
    fwd("tau", tau=torch.zeros(3, 2))
    fwd("support_size", support_size=torch.zeros((3, 4)))
    fwd("status", status=torch.zeros(2, dtype=torch.int32))
    fwd("CUDA")

    def app(match, q=q, k=k, v=k, kc=kc, **kw):
        with pytest.raises(E, match=match):
            binding.entmax_attn_paged_append(q, k, v, kc, kc, table, lens, cu, **kw)

    app("bfloat16", k=k.float())
    app("bfloat16", v=k[:, :1])
    app("disagree", k=torch.zeros((3, 1, 64), dtype=bf), v=torch.zeros((3, 1, 64), dtype=bf))
    app("disagree", q=q[:2])
    app("rotation", rotation=torch.zeros((9, 64), dtype=torch.float64))
    app("q_out without q", q=None, q_out=q)
    app("CUDA")


def test_reference_pins():
    # equal logits: p = 1/n, tau = -n^(1-alpha); one key: tau = y - 1; sparsemax of two keys by hand; a rotation by 90 degrees
    v = torch.arange(12, dtype=torch.float64).view(6, 2)
    z = torch.zeros((6, 2), dtype=torch.float64)
    for alpha in (1.25, 1.5, 2.0):
        o, tau, *_ , lo, hi = paged.attend(z[:1], z, v, 5, alpha)
        assert torch.allclose(o[0], v.mean(0)) and abs(float(tau) + 6.0 ** (1 - alpha)) < 1e-12 and int(lo) == int(hi) == 6
    o, tau, *_ = paged.attend(z[:1] + 1, z[:1] + 1, v[:1], 0, 2.0)
    assert torch.equal(o[0], v[0]) and abs(float(tau) - (2 / math.sqrt(2) - 1)) < 1e-12
    k = torch.tensor([[0.0, 0.0], [0.5, 0.0]])
    o, tau, *_ = paged.attend(torch.tensor([[1.0, 0.0]]), k, torch.eye(2), 1, 2.0, sm_scale=1.0)
    assert torch.allclose(o, torch.tensor([[0.25, 0.75]], dtype=torch.float64)) and abs(float(tau) + 0.25) < 1e-12
    turn = torch.tensor([[0.0, 1.0]])                                  # cos 0, sin 1
    x = torch.tensor([[[1.0, 2.0, 3.0, 4.0]]])
    assert paged.rotate(x, turn, torch.tensor([0]), False).tolist() == [[[-2.0, 1.0, 3.0, 4.0]]]
    turn = torch.tensor([[0.0, 0.0, 1.0, 1.0]])
    assert paged.rotate(x, turn, torch.tensor([0]), False).tolist() == [[[-3.0, -4.0, 1.0, 2.0]]]
    assert paged.rotate(x, turn, torch.tensor([0]), True).tolist() == [[[-2.0, 1.0, -4.0, 3.0]]]


def test_calls_without_new_tokens_clear_the_status():
    # nothing is launched, and what an earlier call reported does not stay behind
    from paper_2506_16640_b200 import binding
    kc = torch.zeros((10, 16, 2, 64), dtype=torch.bfloat16)
    table, lens, cu = torch.zeros((3, 4), dtype=torch.int32), torch.ones(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    q, k = torch.zeros((0, 4, 64), dtype=torch.bfloat16), torch.zeros((0, 2, 64), dtype=torch.bfloat16)
    status = torch.full((binding.STATUS_WORDS,), 5, dtype=torch.int32)
    assert binding.entmax_attn_paged_append(q, k, k, kc, kc, table, lens, cu, status=status).shape == q.shape
    assert int(status.abs().sum()) == 0
    status.fill_(5)
    o, tau, _ = binding.entmax_attn_paged_fwd(q, kc, kc, 1.5, table, lens, cu, status=status)
    assert o.shape == q.shape and tau.shape == (0, 4) and int(status.abs().sum()) == 0


_BOUNDS = r"""
#include <cstdio>
#include <random>
#include "paged.cuh"
using namespace entmax;
// Keys as a solve finds them whose score kernel has not ended: any of the row's groups.  The table's entry is the key's own where the row sees it,
// and one of the sequence's entries in any case.
int main() {
  std::mt19937 g(7);
  auto upto = [&](int n) { return (int)(g() % (unsigned)n); };
  int behind = 0;
  for (int trial = 0; trial < 200000; ++trial) {
    const int shift = 4 + upto(13), pages = 1 + upto(trial % 3 ? 5 : (1 << 24) >> shift), pos = upto(pages << shift);
    const int key = pos / kGroupKeys * kGroupKeys + upto(kGroupKeys), entry = page_entry(key, shift, pages), seen = upto(pos + 1);
    if (entry < 0 || entry >= pages) return printf("key %d in entry %d of %d\n", key, entry, pages), 1;
    if (page_entry(seen, shift, pages) != seen >> shift) return printf("entry of key %d changed\n", seen), 1;
    behind += key >> shift >= pages;
  }
  return behind > 0 ? 0 : 2;
}
"""


def test_keys_of_unwritten_scores_stay_in_the_block_table(tmp_path):
    import subprocess
    src, exe = tmp_path / "bounds.cu", tmp_path / "bounds"
    src.write_text(_BOUNDS)
    subprocess.run([lib_build._nvcc(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", lib_build.CSRC, "-I", lib_build.INCLUDE,
                    "-o", str(exe), str(src)], check=True, capture_output=True, text=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout
