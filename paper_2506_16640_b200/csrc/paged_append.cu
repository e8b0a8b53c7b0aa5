// Rotation of new queries and keys to their positions and append of keys and values to a paged cache, one pass.
//
// Per token and head, x is a row of D elements of which the first r = rot_dim are rotated in pairs by the angle of the token's position,
// whose cosine and sine come from a float32 table [positions][r] (cosines, then sines):
//   halves       pair (i, i + r/2)        interleaved   pair (2i, 2i + 1)
//   x'_lo = x_lo cos - x_hi sin,   x'_hi = x_hi cos + x_lo sin        (float32, rounded to bf16 once)
// The work is moving rows: a lane takes the two 16-byte pieces that hold eight pairs ("unit" p of D / 16), so one set of cosines and sines in
// registers serves every head of the token it meets; four rows are in flight per lane.  A warp takes kSlots rows of one token (query heads,
// key heads, value heads in this order).  Bound by HBM: six prompts of up to 8192 tokens, 32 + 2 * 8 heads of 128, 642 MB in 104 us (6.2 TB/s);
// 256 single tokens take a launch.
#include <cmath>

#include "paged.cuh"

namespace entmax {

namespace {

constexpr int kAppendWarps = 8;
constexpr int kInFlight = 4;

struct AppendArgs {
  PagedCache c;
  int H;                             // query heads (0: none given)
  int rot, n_pos, interleaved;
  long long q_st, q_sh, k_st, k_sh, v_st, v_sh, o_st, o_sh;
  const __nv_bfloat16 *q, *k, *v;
  const float* rotation;
  __nv_bfloat16 *q_out, *k_cache, *v_cache;
  int32_t* status;
  int parts;                         // warps per token
};

__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack(float x, float y) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&t);
}

template <int D>
__global__ void __launch_bounds__(kAppendWarps * 32) paged_append_kernel(const __grid_constant__ AppendArgs a) {
  pdl_begin();
  constexpr int kUnits = D / 16;                 // lanes of a row
  constexpr int kRows = 32 / kUnits;             // rows a warp takes side by side
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
  const long long t_long = w / a.parts;
  if (t_long >= a.c.T) return;
  const int t = (int)t_long, part = (int)(w - t_long * a.parts);
  const int b = a.c.cu_q ? find_seq(a.c, t) : t / (a.c.T / a.c.B);
  const PagedSeq s = paged_seq(a.c, b);
  if (t < s.q0 || t >= s.q0 + s.n) return;       // a row behind the last sequence
  const int pos = s.len - s.n + (t - s.q0);
  const int limit = a.c.max_pages << a.c.ps_shift;
  if (s.len < s.n || s.len > limit || (a.rot > 0 && s.len > a.n_pos)) {
    if (a.status && lane == 0) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
    return;
  }
  const int page = a.c.table[(long long)b * a.c.table_stride + (pos >> a.c.ps_shift)];
  const bool page_ok = (unsigned)page < (unsigned)a.c.n_pages;
  if (!page_ok && a.status && lane == 0) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_PAGE);
  const long long slot = (long long)page * a.c.s_page + (long long)(pos & ((1 << a.c.ps_shift) - 1)) * a.c.s_tok;

  const int p = lane % kUnits;
  const bool turned = p < a.rot / 16;
  // the two 8-element pieces of unit p
  const bool apart = turned && !a.interleaved;
  const int e0 = apart ? 8 * p : 16 * p, e1 = apart ? 8 * p + a.rot / 2 : 16 * p + 8;
  float cs[8], sn[8];
  if (turned) {
    const float4* at = reinterpret_cast<const float4*>(a.rotation + (long long)pos * a.rot + 8 * p);
    const float4* as = reinterpret_cast<const float4*>(a.rotation + (long long)pos * a.rot + a.rot / 2 + 8 * p);
    const float4 c0 = at[0], c1 = at[1], s0 = as[0], s1 = as[1];
    cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
    sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
  }
  const int rows = a.H + 2 * a.c.KH;
  const int r0 = part * (kRows * kInFlight) + lane / kUnits;
  uint4 x0[kInFlight], x1[kInFlight];
#pragma unroll
  for (int u = 0; u < kInFlight; ++u) {
    const int r = r0 + u * kRows;
    if (r < rows) {
      const __nv_bfloat16* src = r < a.H ? a.q + t * a.q_st + r * a.q_sh
                                 : r < a.H + a.c.KH ? a.k + t * a.k_st + (r - a.H) * a.k_sh
                                                    : a.v + t * a.v_st + (r - a.H - a.c.KH) * a.v_sh;
      x0[u] = *reinterpret_cast<const uint4*>(src + e0);
      x1[u] = *reinterpret_cast<const uint4*>(src + e1);
    }
  }
#pragma unroll
  for (int u = 0; u < kInFlight; ++u) {
    const int r = r0 + u * kRows;
    if (r >= rows) continue;
    uint32_t w0[4] = {x0[u].x, x0[u].y, x0[u].z, x0[u].w}, w1[4] = {x1[u].x, x1[u].y, x1[u].z, x1[u].w};
    if (turned && r < a.H + a.c.KH) {
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l0 = bf_lo(w0[e]), h0 = bf_hi(w0[e]), l1 = bf_lo(w1[e]), h1 = bf_hi(w1[e]);
          w0[e] = pack(l0 * cs[e] - h0 * sn[e], h0 * cs[e] + l0 * sn[e]);
          w1[e] = pack(l1 * cs[e + 4] - h1 * sn[e + 4], h1 * cs[e + 4] + l1 * sn[e + 4]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float l0 = bf_lo(w0[e]), l1 = bf_hi(w0[e]), h0 = bf_lo(w1[e]), h1 = bf_hi(w1[e]);
          w0[e] = pack(l0 * cs[2 * e] - h0 * sn[2 * e], l1 * cs[2 * e + 1] - h1 * sn[2 * e + 1]);
          w1[e] = pack(h0 * cs[2 * e] + l0 * sn[2 * e], h1 * cs[2 * e + 1] + l1 * sn[2 * e + 1]);
        }
      }
    }
    __nv_bfloat16* dst;
    if (r < a.H) {
      dst = a.q_out + t * a.o_st + r * a.o_sh;
    } else {
      if (!page_ok) continue;
      const bool key = r < a.H + a.c.KH;
      dst = (key ? a.k_cache : a.v_cache) + slot + (long long)(r - a.H - (key ? 0 : a.c.KH)) * a.c.s_head;
    }
    *reinterpret_cast<uint4*>(dst + e0) = make_uint4(w0[0], w0[1], w0[2], w0[3]);
    *reinterpret_cast<uint4*>(dst + e1) = make_uint4(w1[0], w1[1], w1[2], w1[3]);
  }
}

bool row_strides_ok(int64_t st, int64_t sh, int D) { return st >= D && sh >= D && st % 8 == 0 && sh % 8 == 0; }

}  // namespace

int check_paged_cache(const entmax_attn_paged_cache* p, int total_q, PagedCache* c) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  if (p->batch < 1 || p->kv_heads < 1 || total_q < 1) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->head_dim != 64 && p->head_dim != 128) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->page_size < 16 || p->page_size > 65536 || (p->page_size & (p->page_size - 1)) != 0) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->num_pages < 1 || p->max_pages < 1 || p->table_stride < p->max_pages) return ENTMAX_ATTN_EINVAL_SHAPE;
  if ((long long)p->max_pages * p->page_size > ENTMAX_ATTN_PAGED_MAX_KV) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->stride_page < p->head_dim || p->stride_token < p->head_dim || p->stride_head < p->head_dim) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->stride_page % 8 || p->stride_token % 8 || p->stride_head % 8) return ENTMAX_ATTN_EINVAL_SHAPE;
  c->B = p->batch; c->KH = p->kv_heads; c->D = p->head_dim;
  c->ps_shift = 31 - __builtin_clz((unsigned)p->page_size);
  c->n_pages = p->num_pages; c->max_pages = p->max_pages; c->table_stride = p->table_stride;
  c->s_page = p->stride_page; c->s_tok = p->stride_token; c->s_head = p->stride_head;
  c->T = total_q;
  return ENTMAX_ATTN_OK;
}

}  // namespace entmax

using namespace entmax;

extern "C" int entmax_attn_paged_append(const entmax_attn_paged_cache* cache, const entmax_attn_paged_append_params* params,
                                        const void* q, const void* k, const void* v, const float* rotation,
                                        const int32_t* cu_q, const int32_t* kv_len, const int32_t* block_table, void* q_out,
                                        void* k_cache, void* v_cache, int32_t* device_status, void* cuda_stream) {
  if (!params) return ENTMAX_ATTN_EINVAL_NULL;
  AppendArgs a;
  const int rc = check_paged_cache(cache, params->total_q, &a.c);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (params->q_heads < 0 || (params->q_heads > 0) != (q != nullptr) || (q != nullptr) != (q_out != nullptr)) return ENTMAX_ATTN_EINVAL_NULL;
  if (!k || !v || !k_cache || !v_cache || !kv_len || !block_table) return ENTMAX_ATTN_EINVAL_NULL;
  if (params->rot_dim < 0 || params->rot_dim > a.c.D || params->rot_dim % 16) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (params->rot_dim > 0 && params->rot_positions < 1) return ENTMAX_ATTN_EINVAL_SHAPE;
  if ((params->rot_dim > 0) != (rotation != nullptr)) return ENTMAX_ATTN_EINVAL_NULL;
  if (!cu_q && params->total_q % a.c.B) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!row_strides_ok(params->k_stride_t, params->k_stride_h, a.c.D) || !row_strides_ok(params->v_stride_t, params->v_stride_h, a.c.D) ||
      (q && (!row_strides_ok(params->q_stride_t, params->q_stride_h, a.c.D) ||
             !row_strides_ok(params->out_stride_t, params->out_stride_h, a.c.D))))
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache) ||
      !aligned16(rotation))
    return ENTMAX_ATTN_EINVAL_ALIGN;
  if (((reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(block_table)) & 3u) != 0)
    return ENTMAX_ATTN_EINVAL_ALIGN;
  // in place: the very same rows, or none of them
  if (q && q == q_out && (params->q_stride_t != params->out_stride_t || params->q_stride_h != params->out_stride_h))
    return ENTMAX_ATTN_EINVAL_SHAPE;
  a.c.table = block_table; a.c.kv_len = kv_len; a.c.cu_q = cu_q;
  a.H = params->q_heads;
  a.rot = params->rot_dim; a.n_pos = params->rot_positions; a.interleaved = params->interleaved ? 1 : 0;
  a.q_st = params->q_stride_t; a.q_sh = params->q_stride_h;
  a.k_st = params->k_stride_t; a.k_sh = params->k_stride_h;
  a.v_st = params->v_stride_t; a.v_sh = params->v_stride_h;
  a.o_st = params->out_stride_t; a.o_sh = params->out_stride_h;
  a.q = static_cast<const __nv_bfloat16*>(q); a.k = static_cast<const __nv_bfloat16*>(k); a.v = static_cast<const __nv_bfloat16*>(v);
  a.rotation = rotation;
  a.q_out = static_cast<__nv_bfloat16*>(q_out);
  a.k_cache = static_cast<__nv_bfloat16*>(k_cache); a.v_cache = static_cast<__nv_bfloat16*>(v_cache);
  a.status = device_status;
  const long long rows = (long long)a.H + 2LL * a.c.KH;
  if (rows > 65536) return ENTMAX_ATTN_EINVAL_SHAPE;
  const int per_warp = 32 / (a.c.D / 16) * kInFlight;
  a.parts = (int)((rows + per_warp - 1) / per_warp);
  const long long ctas = ((long long)a.c.T * a.parts + kAppendWarps - 1) / kAppendWarps;
  if (ctas > 0x7fffffffLL) return ENTMAX_ATTN_EINVAL_SHAPE;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t err;
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  err = a.c.D == 64 ? launch_kernel(paged_append_kernel<64>, (unsigned)ctas, kAppendWarps * 32, 0, stream, a)
                    : launch_kernel(paged_append_kernel<128>, (unsigned)ctas, kAppendWarps * 32, 0, stream, a);
  if (err == cudaSuccess) err = cudaGetLastError();
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
