// Softmax attention of new tokens over a paged cache (entmax_attn_softmax_paged_fwd).
#include <cmath>

#include "paged.cuh"
#include "softmax.cuh"

namespace entmax {

namespace {

struct SoftmaxPagedArgs {
  PagedCache c;
  int H, G, window;
  int max_q, max_kv;
  float sm_scale, cap_acc, cap_inv;
  const float *beta, *gamma, *delta, *alibi;
  long long q_st, q_sh;
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  float* lse;
  int32_t* status;
};

// A CTA per new token and query head, a warp per key at a time: right for everything, slow.
template <int D>
__global__ void __launch_bounds__(128) softmax_paged_simple_kernel(const SoftmaxPagedArgs a) {
  pdl_begin();
  __shared__ float tops[4], masses[4], outs[4][D];
  const int t = (int)(blockIdx.x / a.H), h = (int)(blockIdx.x % a.H), kh = h / a.G;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int b = a.c.cu_q ? find_seq(a.c, t) : t / (a.c.T / a.c.B);
  const PagedSeq s = paged_seq(a.c, b);
  if (t < s.q0 || t >= s.q0 + s.n) return;
  const size_t at = (size_t)t * a.H + h;
  constexpr int E = D / 32;
  if (s.len < s.n || s.len > a.max_kv || s.n > a.max_q) {
    if (threadIdx.x == 0) {
      if (a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
      a.lse[at] = -INFINITY;
    }
    for (int d = threadIdx.x; d < D; d += 128) a.o[at * D + d] = __float2bfloat16(0.f);
    return;
  }
  const int pos = s.len - s.n + (t - s.q0);
  const int begin = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  const float c = (a.beta ? length_scale(a.beta[h], a.gamma[h], a.delta[h], pos + 1 - begin) : 1.0f) * a.sm_scale * kLog2e;
  const float slope = a.alibi ? a.alibi[h] / a.sm_scale : 0.f;
  float qv[E], out[E] = {}, top = -INFINITY, mass = 0.f;
  for (int e = 0; e < E; ++e) qv[e] = __bfloat162float(a.q[t * a.q_st + h * a.q_sh + lane * E + e]);
  for (int j = begin + warp; j <= pos; j += 4) {
    const int page = a.c.table[(long long)b * a.c.table_stride + (j >> a.c.ps_shift)];
    const bool ok = (unsigned)page < (unsigned)a.c.n_pages;
    if (!ok && lane == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_PAGE);
    const long long slot = ok ? page * a.c.s_page + (j & ((1 << a.c.ps_shift) - 1)) * a.c.s_tok + kh * a.c.s_head : 0;
    float acc = 0.f, vv[E];
    for (int e = 0; e < E; ++e) {
      acc = fmaf(qv[e], ok ? __bfloat162float(a.k[slot + lane * E + e]) : 0.f, acc);
      vv[e] = ok ? __bfloat162float(a.v[slot + lane * E + e]) : 0.f;
    }
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if (a.cap_acc > 0.f) acc = a.cap_acc * tanh_full(acc * a.cap_inv);
    const float y = c * (acc - slope * (float)(pos - j));
    const float now = fmaxf(top, y), old = exp2f(top - now), p = exp2f(y - now);
    top = now;
    mass = mass * old + p;
    for (int e = 0; e < E; ++e) out[e] = out[e] * old + p * vv[e];
  }
  if (lane == 0) { tops[warp] = top; masses[warp] = mass; }
  for (int e = 0; e < E; ++e) outs[warp][lane * E + e] = out[e];
  __syncthreads();
  const float most = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float total = 0.f;
  for (int w = 0; w < 4; ++w) total += masses[w] * exp2f(tops[w] - most);
  for (int d = threadIdx.x; d < D; d += 128) {
    float x = 0.f;
    for (int w = 0; w < 4; ++w) x += outs[w][d] * exp2f(tops[w] - most);
    a.o[at * D + d] = __float2bfloat16(x / total);
  }
  if (threadIdx.x == 0) a.lse[at] = most * kLn2 + logf(total);
}

int softmax_paged_args(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* p, int uniform, SoftmaxPagedArgs* out) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  SoftmaxPagedArgs a = {};
  const int rc = check_paged_cache(cache, p->total_q, &a.c);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->q_heads < 1 || p->q_heads % a.c.KH || p->q_heads / a.c.KH > 128 || (long long)p->total_q * p->q_heads > 0x7fffffffLL / 2)
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->max_q_len < 0 || p->max_kv_len < 0 || p->window < 0) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (uniform && p->total_q % a.c.B) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!std::isfinite(p->sm_scale) || p->sm_scale < 0.f || !std::isfinite(p->softcap) || p->softcap < 0.f) return ENTMAX_ATTN_EINVAL_ALPHA;
  if (p->q_stride_t < a.c.D || p->q_stride_h < a.c.D || p->q_stride_t % 8 || p->q_stride_h % 8) return ENTMAX_ATTN_EINVAL_SHAPE;
  a.H = p->q_heads;
  a.G = a.H / a.c.KH;
  a.window = p->window;
  a.sm_scale = p->sm_scale > 0.f ? p->sm_scale : 1.0f / std::sqrt((float)a.c.D);
  if (p->softcap > 0.f) {
    a.cap_acc = p->softcap / a.sm_scale;
    a.cap_inv = a.sm_scale / p->softcap;
    if (!std::isfinite(a.cap_acc) || !std::isfinite(a.cap_inv) || a.cap_acc == 0.f) return ENTMAX_ATTN_EINVAL_ALPHA;
  }
  const int most_kv = a.c.max_pages << a.c.ps_shift;
  a.max_kv = p->max_kv_len > 0 && p->max_kv_len < most_kv ? p->max_kv_len : most_kv;
  const int most_q = uniform ? p->total_q / a.c.B : p->total_q;
  a.max_q = p->max_q_len > 0 && p->max_q_len < most_q ? p->max_q_len : most_q;
  a.q_st = p->q_stride_t; a.q_sh = p->q_stride_h;
  *out = a;
  return ENTMAX_ATTN_OK;
}

}  // namespace

}  // namespace entmax

using namespace entmax;

extern "C" size_t entmax_attn_softmax_paged_workspace_bytes(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* params,
                                                            int uniform) {
  SoftmaxPagedArgs a;
  return softmax_paged_args(cache, params, uniform, &a) == ENTMAX_ATTN_OK ? 256 : 0;
}

extern "C" int entmax_attn_softmax_paged_fwd(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* params, const void* q,
                                             const void* k_cache, const void* v_cache, const int32_t* cu_q, const int32_t* kv_len,
                                             const int32_t* block_table, const float* beta, const float* gamma, const float* delta,
                                             const float* alibi_slopes, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                             int32_t* device_status, void* cuda_stream) {
  SoftmaxPagedArgs a;
  const int rc = softmax_paged_args(cache, params, cu_q == nullptr, &a);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!q || !k_cache || !v_cache || !kv_len || !block_table || !o || !lse) return ENTMAX_ATTN_EINVAL_NULL;
  const int given = (beta != nullptr) + (gamma != nullptr) + (delta != nullptr);
  if (given != 0 && given != 3) return ENTMAX_ATTN_EINVAL_NULL;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return ENTMAX_ATTN_EINVAL_ALIGN;
  const uintptr_t words = reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(block_table) |
                          reinterpret_cast<uintptr_t>(beta) | reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(delta) |
                          reinterpret_cast<uintptr_t>(alibi_slopes) | reinterpret_cast<uintptr_t>(lse);
  if (words & 3u) return ENTMAX_ATTN_EINVAL_ALIGN;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) ||
      workspace_bytes < entmax_attn_softmax_paged_workspace_bytes(cache, params, cu_q == nullptr))
    return ENTMAX_ATTN_EINVAL_WORKSPACE;
  a.c.table = block_table; a.c.kv_len = kv_len; a.c.cu_q = cu_q;
  a.beta = beta; a.gamma = gamma; a.delta = delta; a.alibi = alibi_slopes;
  a.q = static_cast<const __nv_bfloat16*>(q); a.k = static_cast<const __nv_bfloat16*>(k_cache); a.v = static_cast<const __nv_bfloat16*>(v_cache);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.status = device_status;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t err;
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  const unsigned grid = (unsigned)((long long)a.c.T * a.H);
  err = a.c.D == 64 ? launch_kernel(softmax_paged_simple_kernel<64>, grid, 128, 0, stream, a)
                    : launch_kernel(softmax_paged_simple_kernel<128>, grid, 128, 0, stream, a);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
