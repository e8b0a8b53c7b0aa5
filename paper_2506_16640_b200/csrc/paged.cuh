// Declarations shared by the kernels that work on a paged key/value cache (paged_append.cu, paged_scores_sm100.cu,
// paged_fwd.cu).
//
// New tokens come packed: the rows cu_q[b] .. cu_q[b+1] - 1 of q belong to sequence b and are its last tokens, so token t
// of them sits at position kv_len[b] - n_b + t.  Position p of sequence b lives in slot p % page_size of page
// block_table[b][p / page_size].  Everything a kernel reads from these device arrays is clamped before it is used as an
// address: lengths that do not fit are reported (FLAG_BAD_LENGTH) and their sequence left out, pages outside the pool are
// reported (FLAG_BAD_PAGE) and read as zeros or left unwritten.
#pragma once

#include "common.cuh"

namespace entmax {

struct PagedCache {
  int B, KH, D;
  int ps_shift, n_pages, max_pages;
  long long table_stride;
  long long s_page, s_tok, s_head;        // element strides
  const int32_t* table;
  const int32_t* kv_len;
  const int32_t* cu_q;                    // nullptr: T / B new tokens each
  int T;                                  // rows of q
};

struct PagedSeq {
  int q0, n, len;                         // first row of q, new tokens, length (new tokens included)
};

__device__ __forceinline__ int clamped_cu(const PagedCache& c, int b) {
  return min(max(c.cu_q[b], 0), c.T);
}
__device__ __forceinline__ PagedSeq paged_seq(const PagedCache& c, int b) {
  PagedSeq s;
  if (c.cu_q) {
    s.q0 = clamped_cu(c, b);
    s.n = max(clamped_cu(c, b + 1) - s.q0, 0);
  } else {
    s.n = c.T / c.B;
    s.q0 = b * s.n;
  }
  s.len = c.kv_len[b];
  return s;
}

// Largest b with cu_q[b] / div + b * add <= x, by the whole warp (every lane returns it): 32 candidates a step.
__device__ __forceinline__ int find_seq(const PagedCache& c, int x, int div, int add) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = c.B;                    // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int b = lo + lane * step;
    const bool le = lane * step < n && (lane == 0 || clamped_cu(c, b) / div + b * add <= x);
    const unsigned m = __ballot_sync(0xffffffffu, le);
    const int k = 31 - __clz(m);          // (a prefix of the lanes; lane 0 is always in it)
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

// Host: checks of the cache description shared by the entry points (defined in paged_append.cu).
int check_paged_cache(const entmax_attn_paged_cache* cache, int total_q, PagedCache* out);

// ------------------------------------------------------------------------------------------- attention
// Rows are handled in units of (block of new tokens, K/V head): block token t and query head kv_head * G + g form row
// t * G + g of the unit, which the score kernels leave in the workspace as
//   group_max[row][group]    maximum over the 32 keys of a group (Eq. 1's units, -inf where none is visible)
//   scores[row][key]         y = (alpha-1) s of every key of the groups whose maximum is above some lower bound of
//                            y_max - 1 (and possibly of others); the other groups are not written
// Two kernels fill it.  "few": one block per sequence with at most few_rows rows, keys as the M side of the MMA.  "many":
// blocks of kManyTiles * tile_tokens tokens of the longer chunks, query rows as the M side.
constexpr int kGroupKeys = 32;
constexpr int kManyTiles = 2;

struct PagedArgs {
  PagedCache c;
  int H, G;
  int expo_class;
  float expo, alpha_m1, sm_scale;
  const float *beta, *gamma, *delta, *alibi;
  int max_q, max_kv;          // longest chunk and sequence that are served (longer: FLAG_BAD_LENGTH)
  int few_rows;               // a sequence with n * G <= few_rows is the "few" kernel's (0: none is)
  int few_slots;              // row slots of a unit there
  int tile_tokens;            // "many": new tokens per 128-row tile, 128 / G
  int many_slots;             // row slots of a unit there
  int many_blocks;            // bound on the number of blocks: T / block_tokens + B
  int few_chunks;             // CTAs per unit of the "few" kernel
  int many_splits;            // work items per unit of the "many" kernel, each a share of the keys
  size_t score_stride;        // floats per row of scores
  int group_stride;           // floats per row of group_max
  float* scores;
  float* group_max;
  int32_t* counter;
  __nv_bfloat16* o;
  float* tau;
  int32_t* support;
  int32_t* status;
};

// Whether the sequence can be served at all, and by which kernel
__device__ __forceinline__ bool paged_ok(const PagedArgs& a, const PagedSeq& s) {
  return s.len >= s.n && s.len <= a.max_kv && s.n <= a.max_q;
}
__device__ __forceinline__ bool paged_few(const PagedArgs& a, const PagedSeq& s) { return (long long)s.n * a.G <= a.few_rows; }

// (alpha-1) c sm_scale of a query at position pos, c = delta + beta (ln n)^gamma with n = pos + 1 (delta for n = 1; 1 without
// scale parameters)
__device__ __forceinline__ float paged_scale(const PagedArgs& a, int head, int pos) {
  float c = 1.0f;
  if (a.beta) {
    c = a.delta[head];
    if (pos > 0) c += a.beta[head] * powf(logf((float)(pos + 1)), a.gamma[head]);
    if (!isfinite(c) && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_SCALE);
  }
  return a.alpha_m1 * (c * a.sm_scale);
}

// The rows of a sequence that cannot be served: zeros, threshold -inf, support 0 (by `threads` threads, this one is `t`)
__device__ __forceinline__ void write_unserved(const PagedArgs& a, const PagedSeq& s, int kv_head, int t, int threads) {
  const int rows = s.n * a.G;
  for (int r = t; r < rows; r += threads) {
    const size_t at = (size_t)(s.q0 + r / a.G) * a.H + kv_head * a.G + r % a.G;
    uint4* o = reinterpret_cast<uint4*>(a.o + at * a.c.D);
    for (int e = 0; e < a.c.D / 8; ++e) o[e] = make_uint4(0u, 0u, 0u, 0u);
    a.tau[at] = -INFINITY;
    if (a.support) a.support[at] = 0;
  }
}

cudaError_t launch_paged_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int unit0, int units,
                             cudaStream_t stream);
cudaError_t launch_paged_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int block0, int blocks,
                              cudaStream_t stream);

}  // namespace entmax
