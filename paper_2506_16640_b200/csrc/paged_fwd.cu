// Attention of new tokens over a paged key/value cache: the row solve behind the score kernels (paged_scores_sm100.cu), and the entry
// points.
//
// A row of the workspace holds the maxima of its groups of 32 keys and the scores of the groups that can matter.  W warps take a
// row: y_max from the maxima; the keys above y_max - 1 (App. A: tau >= y_max - 1) out of the groups whose maximum is above it, into shared
// memory; Newton from the left on them; p = [y - tau]_+^e; O = sum_j p_j v_j as a gather of V rows through the block table.  A row with more
// candidates than the list holds walks its groups in the workspace instead.  All sums are taken in a fixed order.
#include <cmath>

#include "paged.cuh"

namespace entmax {

namespace {

constexpr int kMaxNewtonP = 64;

template <int PER>
__device__ __forceinline__ void load_packed_row(const __nv_bfloat16* p, uint32_t (&w)[PER / 2]) {
  if constexpr (PER == 4) {
    const uint2 raw = *reinterpret_cast<const uint2*>(p);
    w[0] = raw.x;
    w[1] = raw.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}
__device__ __forceinline__ float packed_at(const uint32_t* w, int e) {
  return __uint_as_float((e & 1) ? (w[e >> 1] & 0xffff0000u) : (w[e >> 1] << 16));
}

template <int W>
struct SolveShape {
  static constexpr int kRowsPerCta = W == 1 ? 4 : 1;
  static constexpr int kThreads = 32 * W * kRowsPerCta;
  static constexpr int kSeg = W == 1 ? 512 : 256;          // list entries of a warp
};

// The new token and head of row slot r of a unit
struct RowOf {
  PagedSeq s;
  int b, kvh, tok, g;
  bool served;
};
template <bool kMany>
__device__ __forceinline__ RowOf row_of(const PagedArgs& a, int first, int unit, int r) {
  RowOf w;
  w.kvh = unit % a.c.KH;
  const int at = first + unit / a.c.KH;
  int t0 = 0;
  if constexpr (kMany) {
    const int block_tokens = kManyTiles * a.tile_tokens;
    if (a.c.cu_q) {
      w.b = find_seq(a.c, at, block_tokens, 1);
      t0 = (at - (clamped_cu(a.c, w.b) / block_tokens + w.b)) * block_tokens;
    } else {
      const int per = (a.c.T / a.c.B + block_tokens - 1) / block_tokens;
      w.b = at / per;
      t0 = (at - w.b * per) * block_tokens;
    }
  } else {
    w.b = at;
  }
  w.served = w.b < a.c.B && t0 >= 0;
  if (!w.served) return w;
  w.s = paged_seq(a.c, w.b);
  w.tok = t0 + r / a.G;
  w.g = r % a.G;
  w.served = w.tok < w.s.n && paged_ok(a, w.s) && paged_few(a, w.s) != kMany;
  return w;
}

template <int D, int W, bool kMany>
__global__ void __launch_bounds__(SolveShape<W>::kThreads) paged_solve_kernel(const __grid_constant__ PagedArgs a,
                                                                            const __nv_bfloat16* __restrict__ v, int first,
                                                                            long long n_rows) {
  pdl_begin();
  using S = SolveShape<W>;
  constexpr int PER = D / 32;
  __shared__ float list_y[S::kRowsPerCta * W * S::kSeg];
  __shared__ int list_j[S::kRowsPerCta * W * S::kSeg];
  __shared__ float2 red[2][W];
  __shared__ float opart[W == 1 ? 1 : W][D];
  const int lane = threadIdx.x & 31;
  const int warp = W == 1 ? 0 : threadIdx.x >> 5;          // of the row
  const long long row = W == 1 ? (long long)blockIdx.x * S::kRowsPerCta + (threadIdx.x >> 5) : blockIdx.x;
  if (row >= n_rows) return;
  const int slots = kMany ? a.many_slots : a.few_slots;
  const int unit = (int)(row / slots), r = (int)(row - (long long)unit * slots);
  const RowOf w = row_of<kMany>(a, first, unit, r);
  if (!w.served) return;
  const int pos = w.s.len - w.s.n + w.tok;
  const int groups = pos / kGroupKeys + 1;
  const float* max_row = a.group_max + (size_t)row * a.group_stride;
  const float* y_row = a.scores + (size_t)row * a.score_stride;

  int red_slot = 0;
  // sums over the row's warps in a fixed order; every thread gets them
  auto row_sum2 = [&](float x, float y) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      x += __shfl_xor_sync(0xffffffffu, x, o);
      y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    if constexpr (W > 1) {
      if (lane == 0) red[red_slot][warp] = make_float2(x, y);
      __syncthreads();
      x = 0.f; y = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) {
        x += red[red_slot][i].x;
        y += red[red_slot][i].y;
      }
      red_slot ^= 1;
    }
    return make_float2(x, y);
  };

  // ---- y_max; a warp looks at 32 groups together
  float ymax = -INFINITY;
  for (int g0 = warp * 32; g0 < groups; g0 += 32 * W * 4) {
    float m[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int g = g0 + u * 32 * W + lane;
      m[u] = g < groups ? max_row[g] : -INFINITY;
    }
    ymax = fmaxf(ymax, fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ymax = fmaxf(ymax, __shfl_xor_sync(0xffffffffu, ymax, o));
  if constexpr (W > 1) {
    if (lane == 0) red[1][warp].x = ymax;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) ymax = fmaxf(ymax, red[1][i].x);
  }
  const float floor_y = ymax - 1.0f;

  // f(y of 32 keys, first key) for every group of this warp that can hold a key of the support, four in flight
  auto for_groups = [&](auto&& f) {
    for (int g0 = warp * 32; g0 < groups; g0 += 32 * W) {
      const int g = g0 + lane;
      unsigned todo = __ballot_sync(0xffffffffu, g < groups && max_row[g] > floor_y);
      while (todo) {
        int at[4];
        float y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          at[u] = -1;
          y[u] = -INFINITY;
          if (todo) {
            at[u] = (g0 + __ffs(todo) - 1) * kGroupKeys;
            todo &= todo - 1;
            y[u] = y_row[at[u] + lane];
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (at[u] >= 0) f(y[u], at[u]);
      }
    }
  };

  // ---- candidates
  const int seg = (W == 1 ? (int)(threadIdx.x >> 5) : warp) * S::kSeg;
  int cnt = 0;
  for_groups([&](float y, int key0) {
    const unsigned m = __ballot_sync(0xffffffffu, y > floor_y);
    const int at = cnt + __popc(m & ((1u << lane) - 1u));
    if (y > floor_y && at < S::kSeg) {
      list_y[seg + at] = y;
      list_j[seg + at] = key0 + lane;
    }
    cnt += __popc(m);
  });
  bool spilled = cnt > S::kSeg;
  if constexpr (W > 1) spilled = __syncthreads_or(spilled);
  __syncwarp();

  // ---- threshold: Newton from the left on f(tau) = sum [y - tau]_+^e - 1 (bracketed for e < 1)
  TauIter st;
  st.tau = st.lo = floor_y;
  st.hi = ymax;
  for (int it = 0; it < kMaxNewtonP; ++it) {
    float s0 = 0.f, s1 = 0.f;
    auto add = [&](float y) {
      const float d = y - st.tau;
      if (d > 0.f) {
        float ye, ye1;
        pow_pair(d, a.expo_class, a.expo, ye, ye1);
        s0 += ye;
        s1 += ye1;
      }
    };
    if (!spilled) {
      for (int e = lane; e < cnt; e += 32) add(list_y[seg + e]);
    } else {
      for_groups([&](float y, int) { add(y); });
    }
    const float2 s = row_sum2(s0, s1);
    if (!tau_iter_update(st, s.x, s.y, a.expo_class, a.expo, 1e-7f)) break;
  }
  const float tau = st.tau;

  // ---- O = sum_j p_j v_j, four V rows in flight
  float acc[PER];
#pragma unroll
  for (int e = 0; e < PER; ++e) acc[e] = 0.f;
  int support = 0;
  const __nv_bfloat16* v_head = v + (long long)w.kvh * a.c.s_head + lane * PER;
  const int32_t* pages = a.c.table + (long long)w.b * a.c.table_stride;
  auto gather = [&](float y, int j) {                       // a key per lane (y = -inf: none)
    const float d = y - tau;
    float p = 0.f, p1;
    long long off = -1;
    if (d > 0.f) {
      pow_pair(d, a.expo_class, a.expo, p, p1);
      const int page = pages[j >> a.c.ps_shift];
      if ((unsigned)page < (unsigned)a.c.n_pages)
        off = (long long)page * a.c.s_page + (long long)(j & ((1 << a.c.ps_shift) - 1)) * a.c.s_tok;
    }
    unsigned m = __ballot_sync(0xffffffffu, d > 0.f);
    support += __popc(m);
    while (m) {
      float pj[4];
      uint32_t vw[4][PER / 2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int src = m ? __ffs(m) - 1 : 0;
        pj[u] = __shfl_sync(0xffffffffu, p, src);
        const long long at = __shfl_sync(0xffffffffu, off, src);
#pragma unroll
        for (int e = 0; e < PER / 2; ++e) vw[u][e] = 0u;
        if (m && at >= 0) load_packed_row<PER>(v_head + at, vw[u]);
        m &= m - 1;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[e] = fmaf(pj[u], packed_at(vw[u], e), acc[e]);
    }
  };
  if (!spilled) {
    for (int e0 = 0; e0 < cnt; e0 += 32) {
      const int e = e0 + lane;
      gather(e < cnt ? list_y[seg + e] : -INFINITY, e < cnt ? list_j[seg + e] : 0);
    }
  } else {
    for_groups([&](float y, int key0) { gather(y, key0 + lane); });
  }

  const size_t out = (size_t)(w.s.q0 + w.tok) * a.H + w.kvh * a.G + w.g;
  if constexpr (W == 1) {
    store_slice<PER>(a.o + out * D + lane * PER, acc);
    if (lane == 0) {
      a.tau[out] = tau;
      if (a.support) a.support[out] = support;
    }
  } else {
#pragma unroll
    for (int e = 0; e < PER; ++e) opart[warp][lane * PER + e] = acc[e];
    const float2 n = row_sum2(lane == 0 ? (float)support : 0.f, 0.f);     // (a barrier; counts stay below 2^24)
    if ((int)threadIdx.x < D) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) s += opart[i][threadIdx.x];
      a.o[out * D + threadIdx.x] = __float2bfloat16(s);
    }
    if (threadIdx.x == 0) {
      a.tau[out] = tau;
      if (a.support) a.support[out] = (int)n.x;
    }
  }
}

template <bool kMany>
cudaError_t launch_solve(const PagedArgs& a, const void* v, int first, long long units, cudaStream_t stream) {
  const long long rows = units * (kMany ? a.many_slots : a.few_slots);
  const __nv_bfloat16* vb = static_cast<const __nv_bfloat16*>(v);
  const bool one = a.max_kv <= 1024 || (rows >= 4096 && a.max_kv <= 65536);
#define ENTMAX_PAGED_SOLVE(D, W)                                                                                               \
  launch_kernel(paged_solve_kernel<D, W, kMany>, (unsigned)((rows + SolveShape<W>::kRowsPerCta - 1) / SolveShape<W>::kRowsPerCta), \
                SolveShape<W>::kThreads, 0, stream, a, vb, first, rows)
  if (a.c.D == 64) return one ? ENTMAX_PAGED_SOLVE(64, 1) : ENTMAX_PAGED_SOLVE(64, 8);
  return one ? ENTMAX_PAGED_SOLVE(128, 1) : ENTMAX_PAGED_SOLVE(128, 8);
#undef ENTMAX_PAGED_SOLVE
}

// ------------------------------------------------------------------------------------------------ host
constexpr size_t kSliceBytes = (size_t)4 << 30;     // scores held at a time (at least one sequence's or block's)
constexpr int kFewRows = 32;

struct PagedPlan {
  size_t scores, group_max, total;
  int few_seqs;          // sequences to a slice of the "few" kernel
  int many_blocks;       // blocks to a slice of the "many" kernel
  bool few, many;
};

int plan_paged(const entmax_attn_paged_cache* cache, const entmax_attn_paged_params* p, bool uniform, PagedArgs* a, PagedPlan* l) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  const int rc = check_paged_cache(cache, p->total_q, &a->c);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->q_heads < 1 || p->q_heads % a->c.KH) return ENTMAX_ATTN_EINVAL_SHAPE;
  a->H = p->q_heads;
  a->G = a->H / a->c.KH;
  if (a->G > 128) return ENTMAX_ATTN_EINVAL_SHAPE;
  if ((long long)a->c.T * a->H > 0x7fffffffLL / 2 || (long long)a->c.B * a->H > 0x7fffffffLL / 2048) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->max_q_len < 0 || p->max_kv_len < 0) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!(p->alpha > 1.0f) || !(p->alpha <= kAlphaMax)) return ENTMAX_ATTN_EINVAL_ALPHA;
  if (!(p->sm_scale >= 0.f) || !(p->sm_scale < INFINITY)) return ENTMAX_ATTN_EINVAL_ALPHA;
  if (p->q_stride_t < a->c.D || p->q_stride_h < a->c.D || p->q_stride_t % 8 || p->q_stride_h % 8) return ENTMAX_ATTN_EINVAL_SHAPE;
  a->alpha_m1 = p->alpha - 1.0f;
  a->sm_scale = p->sm_scale == 0.f ? 1.0f / sqrtf((float)a->c.D) : p->sm_scale;
  a->expo = 1.0f / (p->alpha - 1.0f);
  a->expo_class = p->alpha == 2.0f ? kExpo1 : p->alpha == 1.5f ? kExpo2 : p->alpha == 1.25f ? kExpo4 : kExpoGeneral;
  const int capacity = a->c.max_pages << a->c.ps_shift;
  a->max_kv = p->max_kv_len > 0 && p->max_kv_len < capacity ? p->max_kv_len : capacity;
  a->max_q = uniform ? a->c.T / a->c.B : a->c.T;
  if (p->max_q_len > 0 && p->max_q_len < a->max_q) a->max_q = p->max_q_len;
  if (a->max_q > a->max_kv) a->max_q = a->max_kv;
  a->score_stride = ((size_t)a->max_kv + 255) / 256 * 256;
  a->group_stride = (int)(a->score_stride / kGroupKeys);

  // few: rows of a sequence's unit; many: the rest
  a->few_rows = (long long)a->max_q * a->G <= 16 ? 16 : a->G <= kFewRows ? kFewRows : 0;
  if (uniform && (long long)(a->c.T / a->c.B) * a->G > a->few_rows) a->few_rows = 0;
  l->few = a->few_rows > 0;
  const int few_tokens = l->few ? (a->max_q < a->few_rows / a->G ? a->max_q : a->few_rows / a->G) : 0;
  a->few_slots = few_tokens * a->G;
  l->many = a->max_q > few_tokens;
  a->tile_tokens = 128 / a->G;
  a->many_slots = kManyTiles * a->tile_tokens * a->G;
  const int block_tokens = kManyTiles * a->tile_tokens;
  a->many_blocks = uniform ? a->c.B * ((a->c.T / a->c.B + block_tokens - 1) / block_tokens) : a->c.T / block_tokens + a->c.B;

  const size_t row_bytes = a->score_stride * sizeof(float);
  size_t rows = 0;
  l->few_seqs = l->many_blocks = 0;
  if (l->few) {
    const size_t per = (size_t)a->c.KH * a->few_slots, fit = kSliceBytes / row_bytes / per;
    l->few_seqs = fit < 1 ? 1 : fit < (size_t)a->c.B ? (int)fit : a->c.B;
    rows = per * l->few_seqs;
  }
  if (l->many) {
    const size_t per = (size_t)a->c.KH * a->many_slots, fit = kSliceBytes / row_bytes / per;
    l->many_blocks = fit < 1 ? 1 : fit < (size_t)a->many_blocks ? (int)fit : a->many_blocks;
    if (per * l->many_blocks > rows) rows = per * l->many_blocks;
  }
  // work items: CTAs enough for a few waves, shares of the keys no shorter than two tiles
  const long long few_units = (long long)l->few_seqs * a->c.KH;
  long long chunks = few_units > 0 ? 4 * 296 / few_units : 1;
  const long long most = ((a->max_kv + 127) / 128 + 1) / 2;
  a->few_chunks = (int)(chunks < 1 ? 1 : chunks > most ? most : chunks);
  const long long many_units = (long long)l->many_blocks * a->c.KH;
  long long splits = many_units > 0 ? (2 * 148 + many_units - 1) / many_units : 1;
  const long long most_splits = ((a->max_kv + 255) / 256 + 3) / 4;
  a->many_splits = (int)(splits < 1 ? 1 : splits > most_splits ? most_splits : splits);

  size_t off = 256;
  l->group_max = off;
  off += (rows * a->group_stride * sizeof(float) + 255) / 256 * 256;
  l->scores = off;
  off += (rows * row_bytes + 255) / 256 * 256;
  l->total = off;
  return ENTMAX_ATTN_OK;
}

}  // namespace

}  // namespace entmax

using namespace entmax;

extern "C" size_t entmax_attn_paged_workspace_bytes(const entmax_attn_paged_cache* cache, const entmax_attn_paged_params* params,
                                                    int uniform) {
  PagedArgs a;
  PagedPlan l;
  if (plan_paged(cache, params, uniform != 0, &a, &l) != ENTMAX_ATTN_OK) return 0;
  if (uniform && params->total_q % cache->batch) return 0;
  return l.total;
}

extern "C" int entmax_attn_paged_fwd(const entmax_attn_paged_cache* cache, const entmax_attn_paged_params* params, const void* q,
                                     const void* k_cache, const void* v_cache, const int32_t* cu_q, const int32_t* kv_len,
                                     const int32_t* block_table, const float* beta, const float* gamma, const float* delta,
                                     const float* alibi_slopes, void* o, float* tau, int32_t* support_size, void* workspace,
                                     size_t workspace_bytes, int32_t* device_status, void* cuda_stream) {
  PagedArgs a;
  PagedPlan l;
  const int rc = plan_paged(cache, params, cu_q == nullptr, &a, &l);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!cu_q && params->total_q % cache->batch) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!q || !k_cache || !v_cache || !kv_len || !block_table || !o || !tau) return ENTMAX_ATTN_EINVAL_NULL;
  const int given = (beta != nullptr) + (gamma != nullptr) + (delta != nullptr);
  if (given != 0 && given != 3) return ENTMAX_ATTN_EINVAL_NULL;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return ENTMAX_ATTN_EINVAL_ALIGN;
  auto aligned4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; };
  if (!aligned4(cu_q) || !aligned4(kv_len) || !aligned4(block_table) || !aligned4(tau) || !aligned4(support_size) || !aligned4(beta) ||
      !aligned4(gamma) || !aligned4(delta) || !aligned4(alibi_slopes))
    return ENTMAX_ATTN_EINVAL_ALIGN;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0 || workspace_bytes < l.total) return ENTMAX_ATTN_EINVAL_WORKSPACE;
  int dev = 0, major = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
  if (err != cudaSuccess) return fail_cuda(err);
  if (major != 10) return ENTMAX_ATTN_EUNSUPPORTED;          // the score kernels need tcgen05 / TMA
  a.c.table = block_table; a.c.kv_len = kv_len; a.c.cu_q = cu_q;
  a.beta = beta; a.gamma = gamma; a.delta = delta; a.alibi = alibi_slopes;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.counter = reinterpret_cast<int32_t*>(ws);
  a.group_max = reinterpret_cast<float*>(ws + l.group_max);
  a.scores = reinterpret_cast<float*>(ws + l.scores);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.tau = tau;
  a.support = support_size;
  a.status = device_status;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  for (int b = 0; l.few && b < a.c.B && err == cudaSuccess; b += l.few_seqs) {
    const int n = a.c.B - b < l.few_seqs ? a.c.B - b : l.few_seqs;
    err = launch_paged_few(a, q, k_cache, params->q_stride_t, params->q_stride_h, b, n, stream);
    if (err == cudaSuccess) err = launch_solve<false>(a, v_cache, b, (long long)n * a.c.KH, stream);
  }
  for (int blk = 0; l.many && blk < a.many_blocks && err == cudaSuccess; blk += l.many_blocks) {
    const int n = a.many_blocks - blk < l.many_blocks ? a.many_blocks - blk : l.many_blocks;
    err = launch_paged_many(a, q, k_cache, params->q_stride_t, params->q_stride_h, blk, n, stream);
    if (err == cudaSuccess) err = launch_solve<true>(a, v_cache, blk, (long long)n * a.c.KH, stream);
  }
  if (err == cudaSuccess) err = cudaGetLastError();
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
