"""Softmax attention on a device that is not sm_100: the bf16 calls are refused before anything is launched, the float32 ones go on.

The entry points are compiled with a device check that says no and with launches that only count, and called without a device in sight."""
import os
import subprocess
import sys

from paper_2506_16640_b200 import build as lib_build

STUBS = r"""
#include <cuda.h>

#include "softmax_paged.cuh"
#include "sm100_ptx.cuh"
static int launches = 0;
extern "C" int launches_so_far() { return launches; }
namespace entmax {
int check_device_for_bf16() { return ENTMAX_ATTN_EUNSUPPORTED; }
int fail_cuda(cudaError_t) { return ENTMAX_ATTN_ECUDA; }
int check_paged_cache(const entmax_attn_paged_cache* c, int total_q, PagedCache* out) {
  *out = PagedCache{c->batch, c->kv_heads, c->head_dim, 4, c->num_pages, c->max_pages, c->table_stride, c->stride_page, c->stride_token, c->stride_head,
                    nullptr, nullptr, nullptr, total_q};
  return ENTMAX_ATTN_OK;
}
namespace sm100 {
cudaError_t make_box_map(CUtensorMap*, const void*, int, int, int, int, int64_t, int64_t, int64_t, int, int) { ++launches; return cudaSuccess; }
}
cudaError_t launch_softmax_rows_fwd(const SoftmaxArgs&, const void*, const void*, const void*, void*, float*, int32_t*, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t launch_softmax_rows_bwd(const SoftmaxArgs&, const SoftmaxGrads&, const void*, const void*, const void*, const void*, void*, void*, void*, cudaStream_t) {
  ++launches; return cudaSuccess;
}
cudaError_t launch_softmax_fwd(const SoftmaxArgs&, const void*, const void*, const void*, void*, float*, int32_t*, cudaStream_t) { ++launches; return cudaSuccess; }
size_t softmax_bwd_rows_bytes(const SoftmaxArgs&) { return 256; }
size_t softmax_bwd_spans_bytes(const SoftmaxArgs&) { return 256; }
cudaError_t launch_softmax_bwd(const SoftmaxArgs&, const SoftmaxGrads&, const void*, const void*, const void*, const void*, const void*, void*, void*, void*, float*,
                               void*, int32_t*, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t launch_softmax_chunks(const SoftmaxPagedArgs&, const CUtensorMap&, const CUtensorMap&, cudaStream_t) { ++launches; return cudaSuccess; }
}
"""

CALLS = r"""
import ctypes, sys
from paper_2506_16640_b200.binding import PagedCache, SoftmaxGrads, SoftmaxPagedParams, SoftmaxParams
lib = ctypes.CDLL(sys.argv[1])
X, P = ctypes.c_void_p(1 << 20), ctypes.byref                 # (never dereferenced)
def dense(dtype):
    return SoftmaxParams(batch=1, heads=2, kv_heads=2, seq=33, head_dim=64, dtype=dtype, causal=1)
def fwd(dtype):
    return lib.entmax_attn_softmax_fwd(P(dense(dtype)), X, X, X, None, X, X, None, None)
def bwd(dtype):
    return lib.entmax_attn_softmax_bwd(P(dense(dtype)), X, X, X, None, X, X, X, P(SoftmaxGrads()), X, X, X, X, ctypes.c_size_t(1 << 30), None, None)
def paged():
    cache = PagedCache(batch=3, kv_heads=2, head_dim=64, page_size=16, num_pages=100, max_pages=20, table_stride=20, stride_page=2048, stride_token=128,
                       stride_head=64)
    params = SoftmaxPagedParams(total_q=3, q_heads=4, q_stride_t=256, q_stride_h=64)
    return lib.entmax_attn_softmax_paged_fwd(P(cache), P(params), X, X, X, X, X, X, None, None, None, None, X, X, X, ctypes.c_size_t(1 << 30), None, None)
print(fwd(0), bwd(0), paged(), lib.launches_so_far(), fwd(1), bwd(1), lib.launches_so_far())
"""


def test_bf16_calls_are_refused_on_other_devices(tmp_path):
    stubs, lib, calls = tmp_path / "stubs.cu", tmp_path / "libstubs.so", tmp_path / "calls.py"
    stubs.write_text(STUBS)
    calls.write_text(CALLS)
    subprocess.run([lib_build._nvcc(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-O0", "-Xcicc", "-O0", "-Xptxas", "-O0", "--threads", "3",
                    "-Xcompiler", "-fPIC", "-shared", "-I", lib_build.CSRC, "-I", lib_build.INCLUDE, "-o", str(lib), str(stubs),
                    os.path.join(lib_build.CSRC, "softmax_api.cu"), os.path.join(lib_build.CSRC, "softmax_paged.cu")], check=True)
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="-1", PYTHONPATH=lib_build._ROOT)
    out = subprocess.run([sys.executable, str(calls), str(lib)], env=env, check=True, capture_output=True, text=True).stdout
    unsupported = -8
    assert [int(x) for x in out.split()] == [unsupported, unsupported, unsupported, 0, 0, 0, 2]
