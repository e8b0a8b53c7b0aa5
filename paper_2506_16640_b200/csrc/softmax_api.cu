// Entry points of softmax attention over whole sequences (entmax_attn_softmax_fwd / _bwd), the ranges of keys that packed documents leave visible
// (entmax_attn_row_ranges), and the gradients of the per-head scale parameters.
#include <cmath>

#include "softmax.cuh"

namespace entmax {

namespace {

// One thread per row; a binary search among its batch row's boundaries.  Writes 8 bytes per row: a launch's time at any size a batch has (16384 rows: 2 us).
__global__ void __launch_bounds__(256) row_ranges_kernel(int B, int N, int docs, int causal, int window, const int32_t* cu_docs,
                                                         const int32_t* prefix_len, int2* out) {
  pdl_begin();
  const long long at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (at >= (long long)B * N) return;
  const int b = (int)(at / N), i = (int)(at - (long long)b * N);
  const int32_t* cu = cu_docs + (long long)b * (docs + 1);
  int lo = 0, hi = docs;                     // documents that end at or before i: the first `lo` do, those from `hi` on do not
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (cu[mid + 1] <= i) lo = mid + 1; else hi = mid;
  }
  int2 r = make_int2(0, 0);
  if (lo < docs) {
    const int first = max(cu[lo], 0), last = min(cu[lo + 1], N);
    if (i >= first && i < last) {
      r.x = max(first, i - window + 1);
      if (causal) {
        const int prefix = prefix_len ? min(max(prefix_len[(long long)b * docs + lo], 0), last - first) : 0;
        r.y = max(i + 1, first + prefix);
      } else {
        r.y = (int)min((long long)last, (long long)i + window);
      }
    }
  }
  out[at] = r;
}

// dbeta = sum dc (ln n)^gamma, dgamma = sum dc beta (ln n)^gamma ln ln n, ddelta = sum dc over the rows of a head (the first two over n > 1).
// A cluster of CTAs per head; partial sums meet in the shared memory of its first CTA and are added in rank order.  Bound by the latency of its loads: 12 heads x 8192
// rows 8 us, a call with 2 x 16 heads x 4096 rows 8 us longer for it.
constexpr int kScaleCtas = 8, kScaleThreads = 256;
__global__ void __cluster_dims__(kScaleCtas, 1, 1) __launch_bounds__(kScaleThreads)
    softmax_scale_grad_kernel(const SoftmaxArgs a, const float* __restrict__ dc_rows, float* dbeta, float* dgamma, float* ddelta) {
  pdl_begin();
  __shared__ double parts[kScaleThreads / 32][3];
  __shared__ double mine[3];
  const int h = blockIdx.x / kScaleCtas;
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const float beta = a.beta[h], gamma = a.gamma[h];
  double sum[3] = {0.0, 0.0, 0.0};
  const long long rows = (long long)a.B * a.N;
  constexpr int kBatch = 4;                    // rows whose loads are under way together
  for (long long r0 = (long long)rank * kScaleThreads + threadIdx.x; r0 < rows; r0 += kBatch * kScaleCtas * kScaleThreads) {
    float dc[kBatch];
    int n[kBatch];
#pragma unroll
    for (int t = 0; t < kBatch; ++t) {
      const long long r = min(r0 + t * kScaleCtas * kScaleThreads, rows - 1);
      const int b = (int)(r / a.N), i = (int)(r - (long long)b * a.N);
      const int2 sees = visible_keys(a, b, i);
      n[t] = r0 + t * kScaleCtas * kScaleThreads < rows ? sees.y - sees.x : 0;
      dc[t] = dc_rows[((size_t)b * a.H + h) * a.N + i];
    }
#pragma unroll
    for (int t = 0; t < kBatch; ++t) {
      if (n[t] < 1) continue;
      sum[2] += dc[t];
      if (n[t] > 1) {
        const float log_n = logf((float)n[t]), grown = powf(log_n, gamma);
        sum[0] += (double)dc[t] * grown;
        sum[1] += (double)dc[t] * ((double)beta * grown * logf(log_n));
      }
    }
  }
#pragma unroll
  for (int w = 0; w < 3; ++w)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum[w] += __shfl_xor_sync(0xffffffffu, sum[w], o);
  if ((threadIdx.x & 31) == 0)
    for (int w = 0; w < 3; ++w) parts[threadIdx.x >> 5][w] = sum[w];
  __syncthreads();
  if (threadIdx.x < 3) {
    double t = 0.0;
    for (int w = 0; w < kScaleThreads / 32; ++w) t += parts[w][threadIdx.x];
    mine[threadIdx.x] = t;
  }
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank == 0 && threadIdx.x < 3) {
    double t = 0.0;
    for (int c = 0; c < kScaleCtas; ++c) {
      const uint32_t local = (uint32_t)__cvta_generic_to_shared(&mine[threadIdx.x]);
      uint32_t remote;
      double x;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(local), "r"(c));
      asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(x) : "r"(remote) : "memory");
      t += x;
    }
    (threadIdx.x == 0 ? dbeta : threadIdx.x == 1 ? dgamma : ddelta)[h] = (float)t;
  }
  // (no CTA leaves while its shared memory is read)
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Strides of a [batch, heads, seq, head_dim] tensor: all 0 is contiguous; a dimension of one entry has no stride of its own
bool take_strides(const entmax_attn_strides& given, int B, int H, int N, int D, int multiple, entmax_attn_strides* out) {
  entmax_attn_strides s = given;
  if (s.b == 0 && s.h == 0 && s.n == 0) s = entmax_attn_strides{(int64_t)H * N * D, (int64_t)N * D, D};
  if (N == 1) s.n = D;
  if (H == 1) s.h = (int64_t)D * N;
  if (B == 1) s.b = (int64_t)D * N * H;
  if ((N > 1 && (s.n < D || s.n % multiple)) || (H > 1 && (s.h < D || s.h % multiple)) || (B > 1 && (s.b < D || s.b % multiple))) return false;
  *out = s;
  return true;
}

struct BwdWorkspace {
  size_t dc_rows, rows, spans, bytes;   // rows: of the tensor-core kernels, or sum_j p_ij dP_ij of the float32 ones
};
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
BwdWorkspace bwd_workspace(const SoftmaxArgs& a, bool bf16) {
  BwdWorkspace w;
  const size_t per_row = up256((size_t)a.B * a.H * a.N * 4);
  w.dc_rows = 0;
  w.rows = per_row;
  w.spans = w.rows + (bf16 ? up256(softmax_bwd_rows_bytes(a)) : per_row);
  w.bytes = w.spans + (bf16 ? up256(softmax_bwd_spans_bytes(a)) : 0);
  return w;
}

int clear_status(int32_t* status, cudaStream_t stream) {
  if (!status) return ENTMAX_ATTN_OK;
  const cudaError_t err = cudaMemsetAsync(status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}

}  // namespace

int softmax_unit(float given_scale, float softcap, int D, float* sm_scale, float* cap_inv, float* unit) {
  const float least = std::ldexp(1.0f, -100), most = std::ldexp(1.0f, 100);
  for (const float x : {given_scale, softcap})
    if (x != 0.f && !(x >= least && x <= most)) return ENTMAX_ATTN_EINVAL_ALPHA;      // (a NaN too)
  *sm_scale = *unit = given_scale > 0.f ? given_scale : 1.0f / std::sqrt((float)D);
  *cap_inv = 0.f;
  if (softcap > 0.f) {
    *unit = softcap;
    *cap_inv = *sm_scale / softcap;
    if (!std::isnormal(*cap_inv)) return ENTMAX_ATTN_EINVAL_ALPHA;
  }
  return ENTMAX_ATTN_OK;
}

int check_softmax(const entmax_attn_softmax_params* p, const entmax_attn_softmax_terms* terms, SoftmaxArgs* out) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  SoftmaxArgs a = {};
  a.B = p->batch; a.H = p->heads; a.KH = p->kv_heads; a.N = p->seq; a.D = p->head_dim;
  if (a.B < 1 || a.H < 1 || a.KH < 1 || a.N < 1 || a.H % a.KH) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (a.D != 64 && a.D != 128) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (a.H >= 1 << 28 || (long long)a.B * a.H > 0x7fffffffLL / 2 || (long long)a.B * a.H * a.N > 0x7fffffffLL / 2) return ENTMAX_ATTN_EINVAL_SHAPE;
  a.G = a.H / a.KH;
  if (p->dtype != ENTMAX_ATTN_DTYPE_BF16 && p->dtype != ENTMAX_ATTN_DTYPE_FP32) return ENTMAX_ATTN_EINVAL_DTYPE;
  const int rc = softmax_unit(p->sm_scale, p->softcap, a.D, &a.sm_scale, &a.cap_inv, &a.unit);
  if (rc != ENTMAX_ATTN_OK) return rc;
  a.causal = p->causal ? 1 : 0;
  if (!take_strides(p->q, a.B, a.H, a.N, a.D, 8, &a.q) || !take_strides(p->k, a.B, a.KH, a.N, a.D, 8, &a.k) ||
      !take_strides(p->v, a.B, a.KH, a.N, a.D, 8, &a.v) || !take_strides(p->o, a.B, a.H, a.N, a.D, 8, &a.o))
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (terms) {
    a.ranges = reinterpret_cast<const int2*>(terms->row_ranges);
    if (reinterpret_cast<uintptr_t>(terms->row_ranges) & 7u) return ENTMAX_ATTN_EINVAL_ALIGN;
    const int given = (terms->beta != nullptr) + (terms->gamma != nullptr) + (terms->delta != nullptr);
    if ((given != 0 && given != 3) || (given == 3 && terms->c_rows)) return ENTMAX_ATTN_EINVAL_NULL;
    a.beta = terms->beta; a.gamma = terms->gamma; a.delta = terms->delta;
    a.c_rows = terms->c_rows;
    a.alibi = terms->alibi_slopes;
    const uintptr_t all = reinterpret_cast<uintptr_t>(a.beta) | reinterpret_cast<uintptr_t>(a.gamma) | reinterpret_cast<uintptr_t>(a.delta) |
                          reinterpret_cast<uintptr_t>(a.c_rows) | reinterpret_cast<uintptr_t>(a.alibi);
    if (all & 3u) return ENTMAX_ATTN_EINVAL_ALIGN;
  }
  *out = a;
  return ENTMAX_ATTN_OK;
}

cudaError_t launch_softmax_scale_grad(const SoftmaxArgs& a, const float* dc_rows, float* dbeta, float* dgamma, float* ddelta, cudaStream_t stream) {
  return launch_kernel(softmax_scale_grad_kernel, (unsigned)a.H * kScaleCtas, kScaleThreads, 0, stream, a, dc_rows, dbeta, dgamma, ddelta);
}

}  // namespace entmax

using namespace entmax;

extern "C" int entmax_attn_softmax_fwd(const entmax_attn_softmax_params* params, const void* q, const void* k, const void* v,
                                       const entmax_attn_softmax_terms* terms, void* o, float* lse, int32_t* device_status, void* cuda_stream) {
  SoftmaxArgs a;
  int rc = check_softmax(params, terms, &a);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!q || !k || !v || !o || !lse) return ENTMAX_ATTN_EINVAL_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || (reinterpret_cast<uintptr_t>(lse) & 3u)) return ENTMAX_ATTN_EINVAL_ALIGN;
  if (params->dtype == ENTMAX_ATTN_DTYPE_BF16 && (rc = check_device_for_bf16()) != ENTMAX_ATTN_OK) return rc;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  rc = clear_status(device_status, stream);
  if (rc != ENTMAX_ATTN_OK) return rc;
  const cudaError_t err = params->dtype == ENTMAX_ATTN_DTYPE_FP32 ? launch_softmax_rows_fwd(a, q, k, v, o, lse, device_status, stream)
                                                                  : launch_softmax_fwd(a, q, k, v, o, lse, device_status, stream);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}

extern "C" size_t entmax_attn_softmax_workspace_bytes(const entmax_attn_softmax_params* params) {
  SoftmaxArgs a;
  return check_softmax(params, nullptr, &a) == ENTMAX_ATTN_OK ? bwd_workspace(a, params->dtype == ENTMAX_ATTN_DTYPE_BF16).bytes : 0;
}

extern "C" int entmax_attn_softmax_bwd(const entmax_attn_softmax_params* params, const void* q, const void* k, const void* v,
                                       const entmax_attn_softmax_terms* terms, const void* o, const float* lse, const void* d_o,
                                       const entmax_attn_softmax_grads* grads, void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                                       int32_t* device_status, void* cuda_stream) {
  SoftmaxArgs a;
  int rc = check_softmax(params, terms, &a);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!q || !k || !v || !o || !lse || !d_o || !grads || !dq || !dk || !dv) return ENTMAX_ATTN_EINVAL_NULL;
  const int given = (grads->dbeta != nullptr) + (grads->dgamma != nullptr) + (grads->ddelta != nullptr);
  if ((given != 0 && given != 3) || (given == 3 && !a.beta)) return ENTMAX_ATTN_EINVAL_NULL;
  SoftmaxGrads g = {};
  if (!take_strides(grads->d_o, a.B, a.H, a.N, a.D, 8, &g.d_o) || !take_strides(grads->dq, a.B, a.H, a.N, a.D, 8, &g.dq) ||
      !take_strides(grads->dk, a.B, a.KH, a.N, a.D, 8, &g.dk) || !take_strides(grads->dv, a.B, a.KH, a.N, a.D, 8, &g.dv))
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(d_o) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return ENTMAX_ATTN_EINVAL_ALIGN;
  const bool bf16 = params->dtype == ENTMAX_ATTN_DTYPE_BF16;
  const BwdWorkspace w = bwd_workspace(a, bf16);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < w.bytes) return ENTMAX_ATTN_EINVAL_WORKSPACE;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  g.lse = lse;
  g.row_dot = reinterpret_cast<float*>(ws + w.rows);
  g.dc_rows = grads->d_scale_rows ? grads->d_scale_rows : given ? reinterpret_cast<float*>(ws + w.dc_rows) : nullptr;
  if (bf16 && (rc = check_device_for_bf16()) != ENTMAX_ATTN_OK) return rc;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  rc = clear_status(device_status, stream);
  if (rc != ENTMAX_ATTN_OK) return rc;
  cudaError_t err = bf16 ? launch_softmax_bwd(a, g, q, k, v, o, d_o, dq, dk, dv, reinterpret_cast<float*>(ws + w.rows), ws + w.spans, device_status, stream)
                         : launch_softmax_rows_bwd(a, g, q, k, v, d_o, dq, dk, dv, stream);
  if (err == cudaSuccess && given) err = launch_softmax_scale_grad(a, g.dc_rows, grads->dbeta, grads->dgamma, grads->ddelta, stream);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}

extern "C" int entmax_attn_row_ranges(int32_t batch, int32_t seq, int32_t docs, int32_t causal, int32_t window, const int32_t* cu_docs,
                                      const int32_t* prefix_len, int32_t* row_ranges, void* cuda_stream) {
  if (batch < 1 || seq < 1 || docs < 1 || window < 0 || (long long)batch * seq > 0x7fffffffLL / 2) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (prefix_len && !causal) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!cu_docs || !row_ranges) return ENTMAX_ATTN_EINVAL_NULL;
  if (((reinterpret_cast<uintptr_t>(cu_docs) | reinterpret_cast<uintptr_t>(prefix_len)) & 3u) || (reinterpret_cast<uintptr_t>(row_ranges) & 7u))
    return ENTMAX_ATTN_EINVAL_ALIGN;
  const long long rows = (long long)batch * seq;
  const cudaError_t err =
      launch_kernel(row_ranges_kernel, (unsigned)((rows + 255) / 256), 256, 0, static_cast<cudaStream_t>(cuda_stream), batch, seq, docs,
                    causal ? 1 : 0, window > 0 && window < seq ? window : seq, cu_docs, prefix_len, reinterpret_cast<int2*>(row_ranges));
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
