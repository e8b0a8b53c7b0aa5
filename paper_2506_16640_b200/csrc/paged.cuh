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

// Largest b with cu_q[b] <= x, the sequence of row x, by the whole warp (every lane returns it): 32 candidates a step.
__device__ __forceinline__ int find_seq(const PagedCache& c, int x) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = c.B;                    // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int b = lo + lane * step;
    const bool le = lane * step < n && (lane == 0 || clamped_cu(c, b) <= x);
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
// Rows are handled in units of (new tokens, K/V head): token t of the unit and query head kv_head * G + g form row t * G + g of it.  Of its
// scores y = (alpha-1) s (Eq. 1's units) the score kernels leave in the workspace what can matter: every key above some lower bound of the
// row's threshold is there.  Two kernels, two forms:
//   "few": a unit is a sequence with at most few_rows rows.
//       group_max[row][group]         the maximum over each group of 32 keys (-inf: none visible)
//       scores[row][key]              the scores of the groups whose maximum is above a bound of y_max - 1; other groups are not written
//                                     (some may be)
//   "many": a unit is a block of kManyTiles * tile_tokens tokens of a longer chunk; where units are few or uneven, their K tiles are shared among
//       several work items (ManyCut).  The item whose first K tile is lo keeps records of eight neighbouring keys, those with a value above
//       the bound it had then, in key order:
//       scores[row][256 lo + 8 i ..]  the values, before the scaling by |a|      record_key[row][32 lo + i]  the first key
//       row_info[unit][item][row]     {number of records, the bound the item ended with, |a|, the largest value} (bound and value before the scaling, too)
//       (room for every key: a row of flat logits keeps them all)
constexpr int kGroupKeys = 32;
constexpr int kManyKeys = 256;
constexpr int kManyTiles = 2;
constexpr int kMostSms = 160;       // (sizes the workspace, which is the same on every device)
constexpr int kFewSeqs = 256;   // sequences a launch of the "few" kernel takes

struct PagedArgs {
  PagedCache c;
  int H, G;
  unsigned inv_g;             // ceil(2^16 / G)
  int expo_class;
  float expo, alpha_m1, sm_scale;
  const float *beta, *gamma, *delta, *alibi;
  int sms;
  int max_q, max_kv;          // longest chunk and sequence that are served (longer: FLAG_BAD_LENGTH)
  int few_rows;               // a sequence with n * G <= few_rows is the "few" kernel's (0: none is)
  int few_slots;              // row slots of a unit there
  int tile_tokens;            // "many": new tokens per 128-row tile, 128 / G
  int many_slots;             // row slots of a unit there
  int many_blocks;            // bound on the number of blocks.  Block ids run over the sequences with one to spare each: sequence b has
                              // the ids from cu_q[b] / block_tokens + b on, at least as many as it has blocks
  int many_items;             // most work items of a unit of the "many" kernel
  size_t score_stride;        // floats per row of scores
  int groups, tiles;          // groups of 32 and tiles of 256 keys that a row has room for
  float* scores;
  float* group_max;
  int32_t* record_key;
  float4* row_info;
  float* row_scale;           // "many": [T][H] (alpha-1) c sm_scale
  uint2 record_bytes;         // {32, 4}: what a record takes in scores and in record_key (see the "many" kernel)
  struct PagedBlock* blocks;  // "many": what is known of each block of the slice
  int32_t* order;             // its blocks that have work, those with the longest rows first
  int32_t* counters;          // see Counter
  int32_t* spilled;           // rows whose candidates did not fit their list in the kernel that takes eight or 32 lanes per row
  __nv_bfloat16* o;
  float* tau;
  int32_t* support;
  int32_t* status;
  // r / G of a row slot: exact for r < 512, G <= 128 (r (G - 1) < 2^16)
  __device__ __forceinline__ int by_g(int r) const { return (int)(((unsigned)r * inv_g) >> 16); }
};

enum Counter : int {
  kSpilledRows = 0,           // rows in spilled
  kBlocks,                    // blocks in order
  kCut,                       // K tiles per CTA where the units are cut (see ManyCut), 0 where they are not
  kTiles,                     // K tiles of all blocks together (of one K/V head)
  kCounters
};
struct __align__(16) PagedBlock {
  int b, t0, q0, n;           // sequence (-1: nothing to do here), first token within its chunk, the chunk's first row of q, new tokens
  int len, tiles, start, pad; // length; tiles of 256 keys that the block's last row sees; those of the blocks before it
};

// How a unit's K tiles are shared among work items.  Where the units can be dealt to the CTAs evenly, each is one item (cut = 0).  Otherwise the
// tiles of all units, head by head and block by block, are dealt to the CTAs in runs of `cut`, and a unit's items are its shares in the runs
// it lies in (each starts without a bound).  The rule is the plan kernel's.
struct ManyCut {
  int start, tiles, cut;      // start: the unit's first tile in that order
  __device__ __forceinline__ int items() const { return cut ? (start + tiles - 1) / cut - start / cut + 1 : 1; }
  __device__ __forceinline__ int begin(int item) const {   // first tile of an item; items(): the number of tiles
    return item == 0 ? 0 : cut ? min((start / cut + item) * cut - start, tiles) : tiles;
  }
};
// A kernel whose bounded wait has run out returns before it has written all it should.  Such a call's results are invalid (and flagged), but its
// solve must not read outside the row's room.  "many": the CTA that gives up clears every row's record counts (clear_records).  "few": a group's unwritten
// scores may name a key of the last group that the row does not see, and so a page behind its last one; the look-up stays among the table's entries.
// (Counts and keys held to their room where the solve reads them cost it 2 %.)
__host__ __device__ __forceinline__ int page_entry(int key, int ps_shift, int max_pages) {
  return (int)min((unsigned)key >> ps_shift, (unsigned)max_pages - 1u);
}
// Uncut units: the item, in the order of length, that a CTA takes in a round (every other round backwards)
__device__ __forceinline__ int many_dealt(int round, int cta, int ctas) { return round * ctas + ((round & 1) ? ctas - 1 - cta : cta); }
__device__ __forceinline__ ManyCut many_cut(const int32_t* counters, const PagedBlock& pb, int kv_head) {
  return ManyCut{kv_head * counters[kTiles] + pb.start, pb.tiles, counters[kCut]};
}

// No records for any row of the units of `blocks` blocks, whatever has been written by whom
__device__ __forceinline__ void clear_records(const PagedArgs& a, int blocks, int t, int threads) {
  const size_t n = (size_t)blocks * a.c.KH * a.many_items * a.many_slots;
  for (size_t i = t; i < n; i += threads) a.row_info[i] = make_float4(0.f, -INFINITY, 0.f, -INFINITY);
}

// Whether the sequence can be served at all, and by which kernel
__device__ __forceinline__ bool paged_ok(const PagedArgs& a, const PagedSeq& s) {
  return s.len >= s.n && s.len <= a.max_kv && s.n <= a.max_q;
}
__device__ __forceinline__ bool paged_few(const PagedArgs& a, const PagedSeq& s) { return (long long)s.n * a.G <= a.few_rows; }

// y^e and y^(e-1) of y >= 0, the exponent class known at compile time (kExpoGeneral: any)
template <int EC>
__device__ __forceinline__ void powers(float y, float expo, float& ye, float& ye1) {
  pow_pair_c<EC>(y, y > 0.f, expo, ye, ye1);
}
// A lower bound of a threshold from an iterate that came from the left: a hair below it for the rounding
__device__ __forceinline__ float bound_below(float tau) { return tau - 1e-5f * fmaxf(1.0f, fabsf(tau)); }

// The bound y_max - 1 of a threshold, below y_max in any case: from |y_max| = 2^24 on, where 1 is less than a float's distance from the next, the float
// before it, so that the largest keys are above the bound
__device__ __forceinline__ float one_below(float ymax) {
  const float y = ymax - 1.0f;
  if (y < ymax || !(ymax > -INFINITY)) return y;
  return __int_as_float(__float_as_int(ymax) + (ymax > 0.f ? -1 : 1));
}

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

cudaError_t launch_paged_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int seq0, int seqs,
                             cudaStream_t stream);
// (behind the plan kernel for the same blocks)
cudaError_t launch_paged_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int blocks,
                              cudaStream_t stream);

}  // namespace entmax
