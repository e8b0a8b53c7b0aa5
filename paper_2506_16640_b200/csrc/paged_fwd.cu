// Attention of new tokens over a paged key/value cache: the row solves behind the score kernels (paged_scores_sm100.cu), and the entry
// points.
//
// A row's largest score and a lower bound of its threshold come first: tau >= y_max - 1 (App. A), and the threshold of any subset of the keys is
// a bound too.  The keys above the bound are collected from what the score kernels left, into shared memory; Newton from the left on them;
// p = [y - tau]_+^e; O = sum_j p_j v_j as a gather of V rows through the block table (asked for from memory as soon as a key is a
// candidate).  All sums are taken in a fixed order.
//   rows    eight lanes per row where there are many rows: a record or a group's 32 scores and a V row are a coalesced access of eight
//           lanes, sums take three shuffles, and a warp has four rows' chains of dependent loads under way.  A warp per row where there are
//           fewer.  Rows with more candidates than their list holds are listed for
//   row     a CTA per row, for those and for calls of few or long rows.
// Bound by instructions where the machine is full (182000 rows of prompts 70 us, 71 % of the issue slots), else by the chain maxima - candidates -
// pages - threshold - V rows: 2048 decode rows 13 us with a warp each, 256 rows of 65536 keys 15 us and 256 flat ones of 8192 (supports of
// hundreds) 25 us with a CTA each.
#include <atomic>
#include <cmath>

#include "paged.cuh"

namespace entmax {

namespace {


// Eight lanes' share of a V or O row: 16-byte pieces sl, sl + 8 (head_dim 128)
template <int D>
struct Share {
  uint4 w[D / 64];
};
template <int D>
__device__ __forceinline__ void add_share(float (&acc)[D / 8], float p, const Share<D>& x) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    const uint32_t w[4] = {x.w[c].x, x.w[c].y, x.w[c].z, x.w[c].w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[8 * c + 2 * e] = fmaf(p, __uint_as_float(w[e] << 16), acc[8 * c + 2 * e]);
      acc[8 * c + 2 * e + 1] = fmaf(p, __uint_as_float(w[e] & 0xffff0000u), acc[8 * c + 2 * e + 1]);
    }
  }
}
template <int D>
__device__ __forceinline__ void store_share(__nv_bfloat16* row, int sl, const float (&acc)[D / 8]) {
#pragma unroll
  for (int c = 0; c < D / 64; ++c) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(acc[8 * c + 2 * e], acc[8 * c + 2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&t);
    }
    *reinterpret_cast<uint4*>(row + 64 * c + 8 * sl) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Where V row j of a sequence is, in elements from the K/V head's first (-1: its page is not in the pool)
struct Pages {
  const int32_t* table;
  int shift, n_pages, max_pages;
  long long s_page, s_tok;
  __device__ __forceinline__ long long at(int j) const {
    const int page = table[page_entry(j, shift, max_pages)];
    if ((unsigned)page >= (unsigned)n_pages) return -1;
    return (long long)page * s_page + (long long)(j & ((1 << shift) - 1)) * s_tok;
  }
};
__device__ __forceinline__ Pages pages_of(const PagedCache& c, int b) {
  return Pages{c.table + (long long)b * c.table_stride, c.ps_shift, c.n_pages, c.max_pages, c.s_page, c.s_tok};
}
// (a V row is one or two 128-byte lines)
template <int D>
__device__ __forceinline__ void prefetch_row(const __nv_bfloat16* p) {
  asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
  if (D == 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + 64));
}

// One step of the threshold iteration on the candidates from their sums.  Returns false when st.tau is final.  e >= 1: Newton on the e-norm,
// from the left; the rounding of a long step over many keys can pass the root, and a step back from there lands at or before it.
__device__ __forceinline__ bool solve_step(TauIter& st, float s0, float s1, int expo_class, float expo, float tolerance) {
  if (expo < 1.0f) return tau_iter_update(st, s0, s1, expo_class, expo, 1e-7f);
  if (!(s1 > 0.f)) return false;
  const float step = threshold_step(s0, s1, expo_class, expo);
  st.tau += step;
  return fabsf(step) > tolerance;
}
// (the largest value's size sets how far tau, a float of that size, need be known; where scores are large differences among them are what counts)
__device__ __forceinline__ float step_tolerance(float ymax) { return 1e-7f * fminf(fmaxf(1.0f, fabsf(ymax)), 16.0f); }
constexpr int kMaxSteps = 64;
constexpr int kBoundSteps = 5;       // steps towards the threshold of the cells' maxima
constexpr int kFewCandidates = 8;   // groups above y_max - 1 up to which that bound is not looked for

// What the "many" kernel kept of a row: a list of records per work item of its unit
struct Records {
  const float* values;                  // [256 lo + 8 i]
  const int32_t* keys;                  // [32 lo + i]
  const float4* info;                   // [item][slot]
  int slots, items;                     // items: those that had keys of the row
  ManyCut cut;
};
__device__ __forceinline__ Records records_of(const PagedArgs& a, const ManyCut& cut, int unit, int r, size_t row, int pos) {
  Records rec = {a.scores + row * a.score_stride, a.record_key + row * (size_t)(a.tiles * 32),
                 a.row_info + (size_t)unit * a.many_items * a.many_slots + r, a.many_slots, 0, cut};
  const int all = cut.items();
  while (rec.items < all && cut.begin(rec.items) <= pos / kManyKeys) ++rec.items;
  return rec;
}
// The new tokens that a unit's rows belong to: a block of a sequence's chunk ("many"), or all of a sequence ("few")
struct UnitOf {
  PagedSeq s;
  int b, t0;                            // (b = -1: nothing to do)
  ManyCut cut;
};
template <bool kMany>
__device__ __forceinline__ UnitOf unit_of(const PagedArgs& a, int first, int unit) {
  const int at = unit / a.c.KH;
  UnitOf u;
  u.cut = ManyCut{0, 0, 0};
  if constexpr (kMany) {
    const PagedBlock pb = a.blocks[at];
    u.b = pb.b; u.t0 = pb.t0;
    u.cut = many_cut(a.counters, pb, unit - at * a.c.KH);
    u.s = PagedSeq{pb.q0, pb.n, pb.len};
  } else {
    u.b = first + at;
    u.t0 = 0;
    u.s = paged_seq(a.c, u.b);
    if (!paged_ok(a, u.s) || !paged_few(a, u.s)) u.b = -1;
  }
  return u;
}

// =================================================================================================== plan
// What the "many" kernels need to know of the blocks block0 .. block0 + blocks - 1 of new tokens, and the order their work is handed out in:
// longest rows first (by 1024 classes of length), so that the CTAs end together; clears the counters.  The first CTA does this, the others
// fill in the scales of the rows.  Latency: 5.5 us for one chunk of 2048, 7.5 for 357 blocks of prompts.
constexpr int kPlanThreads = 1024;
__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(const __grid_constant__ PagedArgs a, int block0, int blocks) {
  pdl_begin();
  __shared__ int bin[kPlanThreads];               // blocks of a class, then the next place of the class
  __shared__ int warp_sum[kPlanThreads / 32];
  __shared__ int n_blocks, longest, walk;         // longest block; longest walk of a CTA that takes whole units (both in tiles)
  __shared__ int load[256];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tokens = kManyTiles * a.tile_tokens;
  if (blockIdx.x > 0) {
    // warps take tokens in turn, lanes heads
    for (int t = (blockIdx.x - 1) * (kPlanThreads / 32) + warp; t < a.c.T; t += (gridDim.x - 1) * (kPlanThreads / 32)) {
      const int b = a.c.cu_q ? find_seq(a.c, t) : t / (a.c.T / a.c.B);
      const PagedSeq s = paged_seq(a.c, b);
      if (t < s.q0 || t >= s.q0 + s.n || !paged_ok(a, s) || paged_few(a, s)) continue;
      for (int h = lane; h < a.H; h += 32) a.row_scale[(size_t)t * a.H + h] = paged_scale(a, h, s.len - s.n + t - s.q0);
    }
    return;
  }
  bin[tid] = 0;
  if (tid < 256) load[tid] = 0;
  if (tid == 0) longest = walk = 0;
  if (tid <= kSpilledRows) a.counters[tid] = 0;
  __syncthreads();
  auto class_of = [&](int tiles) { return kPlanThreads - 1 - (int)((long long)(tiles - 1) * kPlanThreads / a.tiles); };
  for (int i = warp * 32; i < blocks; i += kPlanThreads) {
    // (a lane per block; the sequence of each found by a plain search, the loads of the lanes overlap)
    const int blk = block0 + i + lane;
    PagedBlock pb = {-1, 0, 0, 0, 0, 0, 0, 0};
    if (i + lane < blocks) {
      int b, t0;
      if (a.c.cu_q) {
        int lo = 0, hi = a.c.B;
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (clamped_cu(a.c, mid) / tokens + mid <= blk) lo = mid; else hi = mid;
        }
        b = lo;
        t0 = (blk - (clamped_cu(a.c, b) / tokens + b)) * tokens;
      } else {
        const int per = (a.c.T / a.c.B + tokens - 1) / tokens;
        b = blk / per;
        t0 = (blk - b * per) * tokens;
      }
      if (b < a.c.B && t0 >= 0) {
        const PagedSeq s = paged_seq(a.c, b);
        if (t0 < s.n) {
          if (!paged_ok(a, s)) {
            if (a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
            const PagedSeq part = {s.q0 + t0, min(tokens, s.n - t0), s.len};
            for (int kvh = 0; kvh < a.c.KH; ++kvh) write_unserved(a, part, kvh, 0, 1);
          } else if (!paged_few(a, s)) {
            pb.b = b;
            pb.t0 = t0;
            pb.q0 = s.q0;
            pb.n = s.n;
            pb.len = s.len;
            pb.tiles = (s.len - s.n + min(t0 + tokens, s.n) - 1) / kManyKeys + 1;
            atomicAdd(&bin[class_of(pb.tiles)], 1);
          }
        }
      }
      a.blocks[i + lane] = pb;
    }
  }
  __syncthreads();
  const int mine = bin[tid];
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sum[warp] = incl;
  __syncthreads();
  int before = 0;
  for (int i = 0; i < warp; ++i) before += warp_sum[i];
  bin[tid] = before + incl - mine;
  // (a class of several lengths counts as its longest)
  auto class_tiles = [&](int cls) { return (int)(((long long)(kPlanThreads - cls) * a.tiles + kPlanThreads - 1) / kPlanThreads); };
  if (mine > 0 && bin[tid] == 0) longest = class_tiles(tid);
  if (tid == kPlanThreads - 1) {
    n_blocks = before + incl;
    a.counters[kBlocks] = n_blocks;
  }
  // tiles before each block
  int carry = 0;
  for (int i0 = 0; i0 < blocks; i0 += kPlanThreads) {
    const int i = i0 + tid, tiles = i < blocks ? a.blocks[i].tiles : 0;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += up;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    int at = carry;
    for (int k = 0; k < kPlanThreads / 32; ++k) {
      if (k < warp) at += warp_sum[k];
      carry += warp_sum[k];
    }
    if (i < blocks) a.blocks[i].start = at + upto - tiles;
  }
  // Units are cut where the longest walk of a CTA that deals them whole passes the mean by 12 tiles: that is about what the new starts cost.
  // (scores and solves, uncut against cut: two prompts of up to 4096 tokens, 3 tiles: 103 against 118 us; 16 sequences, four with chunks of
  // up to 1000 tokens, 9: 118 against 134; a chunk of 1024 over 30000 keys, 32 heads, 16: 279 against 268; of 2048 over 32768, 16 heads, 20:
  // 266 against 246; three sequences, one with a chunk of 500 over 9001 keys, 27: 104 against 75)
  const int all = carry * a.c.KH;                           // (scores are held for all of them at once, so it fits)
  auto even = [&](int tiles) { return (tiles - 12) * a.sms <= all; };
  // (longest stays as it is from the barriers above on, so that all threads take the same way here)
  if (even(longest)) {
    // nor does the longest unit by itself: each CTA's walk, in the order that the many kernel deals units (item k's class is the last one with
    // no more than k / KH blocks before it)
    // (few instructions and no divisions: they come from memory each time.  The first version of this loop cost 4 us.)
    const int items = n_blocks * a.c.KH, cta = tid & 255;
    int sum = 0;
#pragma unroll 1
    for (int round = tid >> 8; round * a.sms < items; round += kPlanThreads / 256) {
      const int k = many_dealt(round, cta, a.sms);
      if (cta >= a.sms || k >= items) continue;
      int cls = 0;
#pragma unroll 1
      for (int half = kPlanThreads / 2; half > 0; half /= 2)
        if (bin[cls + half] * a.c.KH <= k) cls += half;
      sum += class_tiles(cls);
    }
    sum = atomicAdd(&load[cta], sum) + sum;                 // (the last of a CTA's threads sees the whole)
    atomicMax(&walk, sum);
  }
  __syncthreads();
  if (tid == 0) {
    a.counters[kTiles] = carry;
    a.counters[kCut] = even(max(longest, walk)) ? 0 : (all + a.sms - 1) / a.sms;
  }
  for (int i = tid; i < blocks; i += kPlanThreads) {
    const PagedBlock pb = a.blocks[i];
    if (pb.b >= 0) a.order[atomicAdd(&bin[class_of(pb.tiles)], 1)] = i;
  }
}

// ================================================================================================= rows
// L lanes to a row, 8 or 32.  (CTAs of eight warps: 72 us against 70 on 182000 rows of prompts, 16.8 against 15.6 on 3600 of two chunks)
constexpr int kRowsWarps = 4;
template <int L>
struct RowsShape {
  static constexpr int kRows = 32 * kRowsWarps / L;      // rows of a CTA
  static constexpr int kList = L == 8 ? 96 : 256;        // candidates of a row
  static constexpr unsigned kMask = L == 32 ? 0xffffffffu : (1u << (L & 31)) - 1u;
};

template <int L>
__device__ __forceinline__ float sum_lanes(float x) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
template <int L>
__device__ __forceinline__ float max_lanes(float x) {
#pragma unroll
  for (int o = 1; o < L; o <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float max4(const float4& x) { return fmaxf(fmaxf(x.x, x.y), fmaxf(x.z, x.w)); }

// (Loops are kept rolled: unrolled, this code no longer stayed in the instruction cache, 140 us against 86 on 11402 prompt tokens of 16 heads,
// and 72 against 21 on 64 x 32 decode rows.)
template <int D, int EC, bool kMany, int L>
__global__ void __launch_bounds__(32 * kRowsWarps, L == 8 ? 8 : 6) paged_rows_kernel(const __grid_constant__ PagedArgs a,
                                                                                    const __nv_bfloat16* __restrict__ v, int first,
                                                                                    int units) {
  pdl_begin();
  using S = RowsShape<L>;
  constexpr int kOctets = L / 8;
  __shared__ float list_y[S::kRows][S::kList];
  __shared__ long long list_at[S::kRows][S::kList];      // key, then where its V row is
  const int lane = threadIdx.x & 31, sl = lane & (L - 1), s8 = lane & 7, octet = sl >> 3, row_bit = lane & (32 - L);
  const int slots = kMany ? a.many_slots : a.few_slots;
  const int cta_row = threadIdx.x / L;
  int unit, r;
  if constexpr (kMany) {
    const int per = (slots + S::kRows - 1) / S::kRows;     // CTAs of a unit
    unit = blockIdx.x / per;
    r = (blockIdx.x - unit * per) * S::kRows + cta_row;
  } else {
    const long long row = (long long)blockIdx.x * S::kRows + cta_row;
    unit = (int)(row / slots);
    r = (int)(row - (long long)unit * slots);
  }
  // ---- which row this is
  const int kvh = unit % a.c.KH;
  bool live = unit < units && r < slots;
  UnitOf w;
  w.b = -1;
  if (live) w = unit_of<kMany>(a, first, unit);
  const int r_tok = a.by_g(r), g_head = r - r_tok * a.G;
  const int tok = w.t0 + r_tok;
  live = live && w.b >= 0 && tok < w.s.n;
  if (!__any_sync(0xffffffffu, live)) return;
  const int pos = live ? w.s.len - w.s.n + tok : -1;
  const size_t row = (size_t)unit * slots + r;
  const float* y_row = a.scores + row * a.score_stride;
  float* my_y = list_y[cta_row];
  long long* my_at = list_at[cta_row];
  const float4 none = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);

  // ---- The keys above floor_y go to the list; loops run for the longest of the warp's rows.  A row whose candidates do not fit gets a
  // second try with a higher bound: the threshold of maxima of different keys alone, by a few steps from the left (any iterate is a bound;
  // a hair below it for the rounding).  c = 1, alpha = 1.5, 32768 keys N(0, 1): 585 keys above y_max - 1, about 50 above that.
  int cnt = 0;
  // Candidates are told by the values as they were kept (many: before the scaling by mag), floor_y among them.  What goes to the list, and the
  // threshold, is relative to the largest value: in [-1, 0] whatever the size of the scores.
  float top = -INFINITY, floor_y = -INFINITY, mag = 0.f;
  const Records rec = kMany && live ? records_of(a, w.cut, unit, r, row, pos) : Records{};
  const int groups = live ? pos / kGroupKeys + 1 : 0;
  const float4* max_row = reinterpret_cast<const float4*>(a.group_max + row * a.groups);
  const int chunks = kMany ? 0 : (__reduce_max_sync(0xffffffffu, groups) + 4 * L - 1) / (4 * L);
  const int most_items = kMany ? __reduce_max_sync(0xffffffffu, rec.items) : 0;

  // what the row's items left, a lane each (those past L are read when their turn comes)
  float4 info = make_float4(0.f, -INFINITY, 0.f, -INFINITY);
  if (kMany && sl < rec.items) info = rec.info[(size_t)sl * rec.slots];
  auto row_bits = [&](bool x) { return (__ballot_sync(0xffffffffu, x) >> row_bit) & S::kMask; };
  auto append = [&](const float4& y4, int key) {            // this lane's four keys from `key` on
    // (hardly ever more than one or two of them: a lane's first, then its second, ...)
    unsigned left = (y4.x > floor_y ? 1u : 0u) | (y4.y > floor_y ? 2u : 0u) | (y4.z > floor_y ? 4u : 0u) | (y4.w > floor_y ? 8u : 0u);
    for (;;) {
      const unsigned all = __ballot_sync(0xffffffffu, left != 0u);
      if (all == 0u) break;
      const unsigned bits = (all >> row_bit) & S::kMask;
      const int at = cnt + __popc(bits & ((1u << sl) - 1u));
      if (left && at < S::kList) {
        const int e = __ffs(left) - 1;
        const float y = e < 2 ? (e == 0 ? y4.x : y4.y) : (e == 2 ? y4.z : y4.w);
        my_y[at] = kMany ? mag * (y - top) : y - top;
        my_at[at] = key + e;
      }
      left &= left - 1;
      cnt += __popc(bits);
    }
  };
  // many: f(this lane's four values, their first key) for every L / 2 records, two lanes to a record
  auto for_records = [&](auto&& f) {
#pragma unroll 1
    for (int i = 0; i < most_items; ++i) {
      int n = __float_as_int(__shfl_sync(0xffffffffu, info.x, i & (L - 1), L)), lo = 0;
      if (i < rec.items) {
        if (i >= L) n = __float_as_int(rec.info[(size_t)i * rec.slots].x);
        lo = rec.cut.begin(i);
      } else {
        n = 0;
      }
      const int most = __reduce_max_sync(0xffffffffu, n);
#pragma unroll 1
      for (int s0 = 0; s0 < most; s0 += 2 * L) {
        float4 y[4];
        int key[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int at = s0 + L / 2 * u + (sl >> 1);
          y[u] = none;
          key[u] = 0;
          if (at < n) {
            y[u] = *reinterpret_cast<const float4*>(rec.values + (size_t)lo * kManyKeys + 8 * at + 4 * (sl & 1));
            key[u] = rec.keys[lo * 32 + at] + 4 * (sl & 1);
          }
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (s0 + L / 2 * u >= most) break;
          f(y[u], key[u]);
        }
      }
    }
  };
  // few: this lane's maxima of groups 4 L i + 4 sl ..
  auto maxima = [&](int i) {
    float4 m = none;
    const int g = 4 * (L * i + sl);
    if (g < groups) {
      m = max_row[g >> 2];
      if (g + 1 >= groups) m.y = -INFINITY;
      if (g + 2 >= groups) m.z = -INFINITY;
      if (g + 3 >= groups) m.w = -INFINITY;
    }
    return m;
  };
  if constexpr (kMany) {
    mag = __shfl_sync(0xffffffffu, info.z, 0, L);
    floor_y = info.y;
    top = info.w;
    for (int i = sl + L; i < rec.items; i += L) {
      const float4 other = rec.info[(size_t)i * rec.slots];
      floor_y = fmaxf(floor_y, other.y);
      top = fmaxf(top, other.w);
    }
    floor_y = max_lanes<L>(floor_y);
    top = max_lanes<L>(top);
  } else {
#pragma unroll 4
    for (int i = 0; i < chunks; ++i) top = fmaxf(top, max4(maxima(i)));
    top = max_lanes<L>(top);
    floor_y = one_below(top);
  }
  // (-1 too where a = 0 and nothing bounds the row)
  auto floor_of_list = [&]() { return fmaxf(kMany ? mag * (floor_y - top) : floor_y - top, -1.0f); };
  // over: rows to raise the bound of.  Where groups are looked at, their number tells before anything is collected.
  bool over = false;
  if constexpr (!kMany) {
    int n = 0;
#pragma unroll 1
    for (int i = 0; i < chunks; ++i) {
      const float4 m = maxima(i);
      n += (m.x > floor_y ? 1 : 0) + (m.y > floor_y ? 1 : 0) + (m.z > floor_y ? 1 : 0) + (m.w > floor_y ? 1 : 0);
    }
    over = sum_lanes<L>((float)n) > (float)(S::kList / 4);
  }
#pragma unroll 1
  for (int attempt = 0; attempt < 3; ++attempt) {
    if (a.expo >= 1.0f && __any_sync(0xffffffffu, over)) {
      float tau = floor_of_list();
#pragma unroll 1
      for (int it = 0; it < kBoundSteps; ++it) {
        float s0 = 0.f, s1 = 0.f;
        auto add = [&](float m) {
          float ye, ye1;
          powers<EC>(fmaxf((kMany ? mag * (m - top) : m - top) - tau, 0.f), a.expo, ye, ye1);
          s0 += ye;
          s1 += ye1;
        };
        if constexpr (kMany) {
          for_records([&](const float4& y, int) { add(max4(y)); });
        } else {
#pragma unroll 1
          for (int i = 0; i < chunks; ++i) {
            const float4 m = maxima(i);
            add(m.x);
            add(m.y);
            add(m.z);
            add(m.w);
          }
        }
        s0 = sum_lanes<L>(s0);
        s1 = sum_lanes<L>(s1);
        const bool go = s0 > 1.01f && s1 > 0.f;
        if (go) tau += threshold_step(s0, s1, EC, a.expo);
        if (!__any_sync(0xffffffffu, go && over)) break;
      }
      // (back among the values as they were kept: a hair more for the rounding there)
      if (over) floor_y = fmaxf(floor_y, top + (kMany ? bound_below(tau) / mag : bound_below(tau)) - 0x1p-21f * fabsf(top));
    }
    cnt = 0;
    if constexpr (kMany) {
      for_records(append);
    } else {
#pragma unroll 1
      for (int i = 0; i < chunks; ++i) {
        const float4 m = maxima(i);
        const unsigned mine = (m.x > floor_y ? 1u : 0u) | (m.y > floor_y ? 2u : 0u) | (m.z > floor_y ? 4u : 0u) | (m.w > floor_y ? 8u : 0u);
        if (!__any_sync(0xffffffffu, mine != 0u)) continue;
#pragma unroll 1
        for (int e = 0; e < 4; ++e) {
          unsigned bits = row_bits((mine >> e) & 1u);        // groups 4 (L i + bit) + e
          while (__any_sync(0xffffffffu, bits != 0u)) {
            // four steps in flight, of as many groups as the row has octets of lanes, an octet the next bit each
            float4 y[4];
            int key[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              unsigned my = bits;
#pragma unroll
              for (int o = 0; o < kOctets; ++o) {
                if (o < octet) my &= my - 1;
                bits &= bits - 1;
              }
              y[u] = none;
              key[u] = (4 * (L * i + __ffs(my) - 1) + e) * kGroupKeys + 4 * s8;
              if (my) y[u] = *reinterpret_cast<const float4*>(y_row + key[u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) append(y[u], key[u]);
          }
        }
      }
    }
    // (once more, if that was without a raised bound)
    const bool tried = over;
    over = cnt > S::kList;
    if (a.expo < 1.0f || !__any_sync(0xffffffffu, over && !tried)) break;
  }
  if (live && cnt > S::kList) {
    if (sl == 0) a.spilled[atomicAdd(a.counters + kSpilledRows, 1)] = (int)row;
    live = false;
  }
  if (!live) cnt = 0;
  __syncwarp();
  // ---- where the candidates' V rows are; they are asked for now and come while the threshold is found
  const __nv_bfloat16* v_head = v + (long long)kvh * a.c.s_head;
  const Pages pages = pages_of(a.c, live ? w.b : 0);
  for (int e = sl; e < cnt; e += L) {
    const long long off = pages.at((int)my_at[e]);
    if (off >= 0) prefetch_row<D>(v_head + off);
    my_at[e] = off;
  }

  // ---- threshold
  const int longest = __reduce_max_sync(0xffffffffu, cnt);
  TauIter st;
  st.tau = st.lo = floor_of_list();
  st.hi = 0.f;
  bool done = !live;
  const float tolerance = step_tolerance(kMany ? mag * top : top);
#pragma unroll 1
  for (int it = 0; it < kMaxSteps; ++it) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll 1
    for (int e = sl; e < longest; e += L) {
      float ye, ye1;
      powers<EC>(e < cnt ? fmaxf(my_y[e] - st.tau, 0.f) : 0.f, a.expo, ye, ye1);
      s0 += ye;
      s1 += ye1;
    }
    s0 = sum_lanes<L>(s0);
    s1 = sum_lanes<L>(s1);
    if (!done) done = !solve_step(st, s0, s1, EC, a.expo, tolerance);
    if (__all_sync(0xffffffffu, done)) break;
  }
  const float tau = st.tau;
  // (the list closes up to the support: half and more of the candidates have p = 0.  A page that is not there counts as zeros.)
  int support = 0, kept = 0;
#pragma unroll 1
  for (int e0 = 0; e0 < longest; e0 += L) {
    const int e = e0 + sl;
    float d = 0.f, p, p1;
    long long at = -1;
    if (e < cnt) {
      d = fmaxf(my_y[e] - tau, 0.f);
      at = my_at[e];
    }
    powers<EC>(d, a.expo, p, p1);
    support += __popc(row_bits(d > 0.f));
    const unsigned bits = row_bits(p > 0.f && at >= 0);
    __syncwarp();
    if ((bits >> sl) & 1u) {
      const int to = kept + __popc(bits & ((1u << sl) - 1u));
      my_y[to] = p;
      my_at[to] = at;
    }
    kept += __popc(bits);
  }
  cnt = kept;
  __syncwarp();

  // ---- O = sum_j p_j v_j: an octet of lanes to a V row, four of each octet in flight
  float acc[D / 8];
#pragma unroll
  for (int e = 0; e < D / 8; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int e0 = octet; e0 < cnt; e0 += 4 * kOctets) {
    float p[4];
    Share<D> x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int e = e0 + kOctets * u;
      p[u] = e < cnt ? my_y[e] : 0.f;
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        x[u].w[c] = make_uint4(0u, 0u, 0u, 0u);
        if (p[u] > 0.f) x[u].w[c] = *reinterpret_cast<const uint4*>(v_head + my_at[e] + 64 * c + 8 * s8);
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) add_share<D>(acc, p[u], x[u]);
  }
  if constexpr (L == 32) {
    __syncwarp();
#pragma unroll
    for (int e = 0; e < D / 8; ++e) {
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 8);
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 16);
    }
  }
  if (live && octet == 0) {
    const size_t out = (size_t)(w.s.q0 + tok) * a.H + kvh * a.G + g_head;
    store_share<D>(a.o + out * D, s8, acc);
    if (sl == 0) {
      a.tau[out] = (kMany ? mag * top : top) + tau;
      if (a.support) a.support[out] = support;
    }
  }
}

// ================================================================================================== row
constexpr int kCtaWarps = 8;
constexpr int kSeg = 256;            // list entries of a warp
constexpr int kLongRow = 4096, kRows8Warps = 64;     // (see solve_lanes)
constexpr int kChunks = 8;           // chunks of 32 groups of a warp whose maxima stay in shared memory

// kSpilled: the rows listed by the rows kernel, by CTAs that stay; otherwise a CTA for each of the n_slots row slots
template <int D, bool kMany, bool kSpilled>
__global__ void __launch_bounds__(32 * kCtaWarps, 2) paged_row_kernel(const __grid_constant__ PagedArgs a,
                                                                     const __nv_bfloat16* __restrict__ v, int first, int n_slots) {
  pdl_begin();
  constexpr int W = kCtaWarps;
  __shared__ float list_y[kCtaWarps][kSeg];
  __shared__ long long list_at[kCtaWarps][kSeg];          // key, then where its V row is
  __shared__ float maxima[kCtaWarps][kChunks * 32];
  __shared__ float2 red[2][W];
  __shared__ float opart[W][D];
  const int lane = threadIdx.x & 31, sl = lane & 7, warp = threadIdx.x >> 5;
  const int slots = kMany ? a.many_slots : a.few_slots;
  const int n_rows = kSpilled ? a.counters[kSpilledRows] : n_slots;
  float* my_max = maxima[warp];
  float* my_y = list_y[warp];
  long long* my_at = list_at[warp];
  int red_slot = 0;
  // sums over the row's warps in a fixed order; every thread gets them
  auto row_sum2 = [&](float x, float y) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      x += __shfl_xor_sync(0xffffffffu, x, o);
      y += __shfl_xor_sync(0xffffffffu, y, o);
    }
    if (lane == 0) red[red_slot][warp] = make_float2(x, y);
    __syncthreads();
    x = 0.f; y = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      x += red[red_slot][i].x;
      y += red[red_slot][i].y;
    }
    red_slot ^= 1;
    return make_float2(x, y);
  };

  for (int n = blockIdx.x; n < n_rows; n += gridDim.x) {
    const int row = kSpilled ? a.spilled[n] : n;
    const int unit = row / slots, r = row - unit * slots;
    // ---- which row this is
    const int kvh = unit % a.c.KH;
    const UnitOf w = unit_of<kMany>(a, first, unit);
    const PagedSeq s = w.s;
    const int tok = w.t0 + r / a.G;
    if (w.b < 0 || tok >= s.n) continue;                   // (no row)
    const int pos = s.len - s.n + tok;
    const Pages pages = pages_of(a.c, w.b);
    const __nv_bfloat16* v_head = v + (long long)kvh * a.c.s_head;
    const float* y_row = a.scores + (size_t)row * a.score_stride;
    float ymax = -INFINITY, floor_y = -INFINITY, zmax = -INFINITY;

    // for_keys(f): f(value relative to the largest, key) with a key per lane (-inf: none) for all keys of this warp that are kept and can be in the
    // support, eight (four records) in flight
    const int groups = pos / kGroupKeys + 1;
    const float* max_row = a.group_max + (size_t)row * a.groups;
    // few: group g is warp g mod W's, 32 of a warp's groups are a chunk (so that short rows and runs of neighbouring candidates are
    // spread over the warps)
    const int chunks = (groups + 32 * W - 1) / (32 * W);
    auto max_at = [&](int i) -> float {                    // this lane's group of the warp's chunk i
      if (i < kChunks) return my_max[i * 32 + lane];
      const int g = (i * 32 + lane) * W + warp;
      return g < groups ? max_row[g] : -INFINITY;
    };
    Records rec;
    if constexpr (kMany) rec = records_of(a, w.cut, unit, r, row, pos);
    auto for_keys = [&](auto&& f) {
      if constexpr (!kMany) {
        for (int i = 0; i < chunks; ++i) {
          unsigned todo = __ballot_sync(0xffffffffu, max_at(i) > floor_y);
          while (todo) {
            int at[8];
            float y[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              at[u] = -1;
              y[u] = -INFINITY;
              if (todo) {
                at[u] = ((i * 32 + __ffs(todo) - 1) * W + warp) * kGroupKeys + lane;
                todo &= todo - 1;
                y[u] = y_row[at[u]];
              }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
              if (at[u] >= 0) f(y[u] - ymax, at[u]);
          }
        }
      } else {
        // four records of a work item are a warp's step
        for (int i = 0; i < rec.items; ++i) {
          const int lo = rec.cut.begin(i);
          const float4 info = rec.info[(size_t)i * rec.slots];
          const int n = __float_as_int(info.x);
          for (int st = 4 * warp; st < n; st += 16 * W) {
            float y[4];
            int key[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              const int at = st + 4 * W * u + (lane >> 3);
              y[u] = -INFINITY;
              key[u] = 0;
              if (at < n) {
                y[u] = info.z * (y_row[(size_t)lo * kManyKeys + 8 * at + sl] - zmax);
                key[u] = rec.keys[lo * 32 + at] + sl;
              }
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
              if (st + 4 * W * u < n) f(y[u], key[u]);
          }
        }
      }
    };

    // ---- y_max
    if constexpr (!kMany) {
      float m[kChunks];
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int g = (i * 32 + lane) * W + warp;
        m[i] = g < groups ? max_row[g] : -INFINITY;
      }
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        my_max[i * 32 + lane] = m[i];
        ymax = fmaxf(ymax, m[i]);
      }
      for (int i = kChunks; i < chunks; ++i) ymax = fmaxf(ymax, max_at(i));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) ymax = fmaxf(ymax, __shfl_xor_sync(0xffffffffu, ymax, o));
      if (lane == 0) red[red_slot][warp].x = ymax;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) ymax = fmaxf(ymax, red[red_slot][i].x);
      red_slot ^= 1;
      floor_y = one_below(ymax);
    } else {
      float mag = 0.f, thr = -INFINITY;
      for (int i = 0; i < rec.items; ++i) {
        const float4 info = rec.info[(size_t)i * rec.slots];
        mag = info.z;
        thr = fmaxf(thr, info.y);
        zmax = fmaxf(zmax, info.w);
      }
      ymax = mag * zmax;
      floor_y = fmaxf(mag * (thr - zmax), -1.0f);
    }

    // ---- the threshold of the groups' largest keys as a bound (see the rows kernel)
    if (!kMany && a.expo >= 1.0f) {
      int cand = 0;
      for (int i = 0; i < chunks; ++i) cand += __popc(__ballot_sync(0xffffffffu, max_at(i) > floor_y));
      cand = (int)row_sum2(lane == 0 ? (float)cand : 0.f, 0.f).x;
      float tau = floor_y;
      for (int it = 0; it < kBoundSteps && cand > kFewCandidates; ++it) {
        float s0 = 0.f, s1 = 0.f;
        for (int i = 0; i < chunks; ++i) {
          const float d = max_at(i) - tau;
          if (d > 0.f) {
            float ye, ye1;
            pow_pair(d, a.expo_class, a.expo, ye, ye1);
            s0 += ye;
            s1 += ye1;
          }
        }
        const float2 sum = row_sum2(s0, s1);
        if (!(sum.x > 1.01f) || !(sum.y > 0.f)) break;
        tau += threshold_step(sum.x, sum.y, a.expo_class, a.expo);
      }
      floor_y = fmaxf(floor_y, bound_below(tau));
    }

    // ---- candidates
    int cnt = 0;
    const float floor_rel = kMany ? floor_y : fmaxf(floor_y - ymax, -1.0f);
    for_keys([&](float y, int key) {
      const unsigned m = __ballot_sync(0xffffffffu, y > floor_rel);
      const int at = cnt + __popc(m & ((1u << lane) - 1u));
      if (y > floor_rel && at < kSeg) {
        my_y[at] = y;
        my_at[at] = key;
      }
      cnt += __popc(m);
    });
    // (not while they are collected, where each would wait for the block table by itself)
    __syncwarp();
#pragma unroll 4
    for (int e = lane; e < min(cnt, kSeg); e += 32) {
      const long long off = pages.at((int)my_at[e]);
      if (off >= 0) prefetch_row<D>(v_head + off);
      my_at[e] = off;
    }
    const bool walk = __syncthreads_or(cnt > kSeg);         // more than the lists hold: the kept keys are walked every time

    // ---- threshold
    TauIter st;
    st.tau = st.lo = floor_rel;
    const float tolerance = step_tolerance(ymax);
    st.hi = 0.f;
    for (int it = 0; it < kMaxSteps; ++it) {
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
      if (!walk) {
        for (int e = lane; e < cnt; e += 32) add(my_y[e]);
      } else {
        for_keys([&](float y, int) { add(y); });
      }
      const float2 sum = row_sum2(s0, s1);
      if (!solve_step(st, sum.x, sum.y, a.expo_class, a.expo, tolerance)) break;
    }
    const float tau = st.tau;

    // ---- O = sum_j p_j v_j: a key per eight lanes, 32 (head_dim 128: 16) V rows of a warp in flight
    constexpr int kFlight = D == 64 ? 8 : 4;
    float acc[D / 8];
#pragma unroll
    for (int e = 0; e < D / 8; ++e) acc[e] = 0.f;
    int support = 0;
    auto gather = [&](float y, long long off) {             // a key per lane (y = -inf: none)
      const float d = y - tau;
      float p = 0.f, p1;
      if (d > 0.f) pow_pair(d, a.expo_class, a.expo, p, p1);
      else off = -1;
      const unsigned m = __ballot_sync(0xffffffffu, d > 0.f);
      support += __popc(m);
      // (eight lanes take the keys of their own octet of lanes)
#pragma unroll
      for (int e0 = 0; e0 < 8; e0 += kFlight) {
        if (kFlight < 8 && ((m >> e0) & 0x0f0f0f0fu) == 0u) continue;
        float px[kFlight];
        Share<D> x[kFlight];
#pragma unroll
        for (int u = 0; u < kFlight; ++u) {
          const int src = (lane & 24) + e0 + u;
          px[u] = __shfl_sync(0xffffffffu, p, src);
          const long long at = __shfl_sync(0xffffffffu, off, src);
#pragma unroll
          for (int c = 0; c < D / 64; ++c) {
            x[u].w[c] = make_uint4(0u, 0u, 0u, 0u);
            if (at >= 0) x[u].w[c] = *reinterpret_cast<const uint4*>(v_head + at + 64 * c + 8 * sl);
          }
        }
#pragma unroll
        for (int u = 0; u < kFlight; ++u) add_share<D>(acc, px[u], x[u]);
      }
    };
    if (!walk) {
      for (int e0 = 0; e0 < cnt; e0 += 32) {
        const int e = e0 + lane;
        gather(e < cnt ? my_y[e] : -INFINITY, e < cnt ? my_at[e] : -1);
      }
    } else {
      for_keys([&](float y, int key) { gather(y, y > tau ? pages.at(key) : -1); });
    }
#pragma unroll
    for (int e = 0; e < D / 8; ++e) {
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 8);
      acc[e] += __shfl_xor_sync(0xffffffffu, acc[e], 16);
    }
    const size_t out = (size_t)(s.q0 + tok) * a.H + kvh * a.G + r % a.G;
    if (lane < 8) {
#pragma unroll
      for (int e = 0; e < D / 8; ++e) opart[warp][(e >> 3) * 64 + 8 * sl + (e & 7)] = acc[e];
    }
    const float2 total = row_sum2(lane == 0 ? (float)support : 0.f, 0.f);   // (a barrier; counts stay below 2^24)
    if ((int)threadIdx.x < D) {
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) o += opart[i][threadIdx.x];
      a.o[out * D + threadIdx.x] = __float2bfloat16(o);
    }
    if (threadIdx.x == 0) {
      a.tau[out] = ymax + tau;
      if (a.support) a.support[out] = (int)total.x;
    }
    __syncthreads();                                        // (opart is read before the next row writes it)
  }
}

// Lanes of a row in the solve of a launch; 0: a CTA.  A CTA per row where all fit the machine at once (two to an SM), which takes 8 us for the
// shortest rows, and for two or three rounds of longer ones: 256 rows of 65536 keys 16 us against 27 with a warp each, 320 of 48222 24 against
// 54, 512 of 16384 18 against 23, 384 of 6000 at c = 1 21 against 26; but 576 of 4096 18 against 18, 448 of 2048 16 against 14, 640 of 4096
// 22 against 15, 1120 of 45231 64 against 55.  Eight lanes where there are more rows than the machine holds warps, 64 to an SM (37000 rows of
// chunks 18 us against 39 with a warp each).
int solve_lanes(const PagedArgs& a, long long rows) {
  const int rounds = a.max_kv <= kLongRow ? 1 : a.max_kv <= 4 * kLongRow ? 2 : 3;
  return rows <= rounds * 2 * a.sms ? 0 : rows < kRows8Warps * a.sms ? 32 : 8;
}

template <int D, bool kMany, int L>
cudaError_t launch_rows(const PagedArgs& a, const __nv_bfloat16* v, int first, int units, cudaStream_t stream) {
  constexpr int kRows = RowsShape<L>::kRows;
  const int slots = kMany ? a.many_slots : a.few_slots;
  const unsigned ctas = (unsigned)(kMany ? (long long)units * ((slots + kRows - 1) / kRows) : ((long long)units * slots + kRows - 1) / kRows);
  cudaError_t err;
#define ENTMAX_ROWS(EC) launch_kernel(paged_rows_kernel<D, EC, kMany, L>, ctas, 32 * kRowsWarps, 0, stream, a, v, first, units)
  switch (a.expo_class) {
    case kExpo2: err = ENTMAX_ROWS(kExpo2); break;
    case kExpo1: err = ENTMAX_ROWS(kExpo1); break;
    case kExpo4: err = ENTMAX_ROWS(kExpo4); break;
    default: err = ENTMAX_ROWS(kExpoGeneral); break;
  }
#undef ENTMAX_ROWS
  if (err != cudaSuccess) return err;
  return launch_kernel(paged_row_kernel<D, kMany, true>, 2 * a.sms, 32 * kCtaWarps, 0, stream, a, v, first, 0);
}

template <int D, bool kMany>
cudaError_t launch_solve_d(const PagedArgs& a, const __nv_bfloat16* v, int first, int units, cudaStream_t stream) {
  const int rows = units * (kMany ? a.many_slots : a.few_slots), lanes = solve_lanes(a, rows);
  if (lanes == 0) return launch_kernel(paged_row_kernel<D, kMany, false>, (unsigned)rows, 32 * kCtaWarps, 0, stream, a, v, first, rows);
  return lanes == 8 ? launch_rows<D, kMany, 8>(a, v, first, units, stream) : launch_rows<D, kMany, 32>(a, v, first, units, stream);
}

template <bool kMany>
cudaError_t launch_solve(const PagedArgs& a, const void* v, int first, int units, cudaStream_t stream) {
  const __nv_bfloat16* vb = static_cast<const __nv_bfloat16*>(v);
  return a.c.D == 64 ? launch_solve_d<64, kMany>(a, vb, first, units, stream) : launch_solve_d<128, kMany>(a, vb, first, units, stream);
}

// ------------------------------------------------------------------------------------------------ host
// Scores held at a time (at least one sequence's or block's): launches are milliseconds long there, so that slices cost nothing and a workspace
// stays what a server can spare.
constexpr size_t kSliceBytes = (size_t)4 << 30;
constexpr int kFewRows = 32;         // most rows of the few kernel's MMA
constexpr int kFewWorth = 8;         // (see plan_paged)

// The current device's compute capability (major) and SMs, looked up once per device
cudaError_t device_facts(int* major, int* sms) {
  static std::atomic<int> known[64];               // major << 16 | sms; 0: not looked up yet
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  if (err != cudaSuccess) return err;
  int v = dev >= 0 && dev < 64 ? known[dev].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    int m = 0, n = 0;
    err = cudaDeviceGetAttribute(&m, cudaDevAttrComputeCapabilityMajor, dev);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    if (err != cudaSuccess) return err;
    v = m << 16 | n;
    if (dev >= 0 && dev < 64) known[dev].store(v, std::memory_order_relaxed);
  }
  *major = v >> 16;
  *sms = (v & 0xffff) < kMostSms ? v & 0xffff : kMostSms;
  return cudaSuccess;
}

struct PagedPlan {
  size_t scores, group_max, record_key, row_info, row_scale, blocks, order, spilled, total;
  int few_seqs;          // sequences to a slice of the "few" kernel (at most kFewSeqs)
  int many_blocks;       // blocks to a slice of the "many" kernel
  bool few, many;
  bool both;             // the two side by side, each with buffers of its own
  size_t few_scores, few_spilled;
};

int plan_paged(const entmax_attn_paged_cache* cache, const entmax_attn_paged_params* p, bool uniform, PagedArgs* a, PagedPlan* l) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  const int rc = check_paged_cache(cache, p->total_q, &a->c);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->q_heads < 1 || p->q_heads % a->c.KH) return ENTMAX_ATTN_EINVAL_SHAPE;
  a->H = p->q_heads;
  a->G = a->H / a->c.KH;
  a->inv_g = (65536u + a->G - 1) / a->G;
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
  a->groups = (int)(a->score_stride / kGroupKeys);
  a->tiles = (int)(a->score_stride / kManyKeys);

  // few: rows of a sequence's unit; many: the rest
  a->few_rows = (long long)a->max_q * a->G <= 16 ? 16 : a->G <= kFewRows ? kFewRows : 0;
  if (uniform && (long long)(a->c.T / a->c.B) * a->G > a->few_rows) a->few_rows = 0;
  // Where longer chunks are possible anyway, the single tokens of a handful of sequences are not worth launches of their own.  (taken along by
  // the many kernel against a few kernel beside it, contexts up to 9001: 4 sequences, one of them a chunk of 100, 73 us and 73; 8, two
  // chunks of 500, 79 and 78; 8 with contexts of 30001 124 and 131; 16, four chunks of 1000, 137 and 134; 24, two chunks of 500, 93 and 81)
  if (a->c.B <= kFewWorth && (long long)a->max_q * a->G > a->few_rows) a->few_rows = 0;
  l->few = a->few_rows > 0;
  const int few_tokens = l->few ? (a->max_q < a->few_rows / a->G ? a->max_q : a->few_rows / a->G) : 0;
  a->few_slots = few_tokens * a->G;
  l->many = a->max_q > few_tokens;
  a->tile_tokens = 128 / a->G;
  a->many_slots = kManyTiles * a->tile_tokens * a->G;
  const int block_tokens = kManyTiles * a->tile_tokens;
  a->many_blocks = uniform ? a->c.B * ((a->c.T / a->c.B + block_tokens - 1) / block_tokens) : (a->c.T + block_tokens - 1) / block_tokens + a->c.B - 1;

  const size_t row_bytes = a->score_stride * sizeof(float);
  size_t rows = 0, many_rows = 0;
  l->few_seqs = l->many_blocks = 0;
  if (l->few) {
    const size_t per = (size_t)a->c.KH * a->few_slots, fit = kSliceBytes / row_bytes / per;
    l->few_seqs = a->c.B < kFewSeqs ? a->c.B : kFewSeqs;
    if (fit < (size_t)l->few_seqs) l->few_seqs = fit < 1 ? 1 : (int)fit;
    rows = per * l->few_seqs;
  }
  if (l->many) {
    const size_t per = (size_t)a->c.KH * a->many_slots, fit = kSliceBytes / row_bytes / per;
    l->many_blocks = fit < 1 ? 1 : fit < (size_t)a->many_blocks ? (int)fit : a->many_blocks;
    many_rows = per * l->many_blocks;
  }
  // (one run per SM, of a tile at least)
  a->many_items = a->tiles + 2;
  if (a->many_items > kMostSms + 1) a->many_items = kMostSms + 1;

  size_t off = 256;
  auto take = [&off](size_t floats) { const size_t at = off; off = (off + floats * sizeof(float) + 255) / 256 * 256; return at; };
  l->blocks = take(l->many_blocks * (sizeof(PagedBlock) / sizeof(float)));
  l->order = take(l->many_blocks);
  l->spilled = take(rows > many_rows ? rows : many_rows);
  l->group_max = take(rows * a->groups);
  l->record_key = take(many_rows * a->tiles * 32);
  l->row_info = take(4 * many_rows * a->many_items);
  l->row_scale = take(l->many ? (size_t)a->c.T * a->H : 0);
  // A call with both kinds of sequences and room for all of each runs them side by side (24 sequences, two of them with chunks: 92 us one
  // after the other, 76 now); otherwise they take turns with the same buffers
  l->both = l->few && l->many && l->few_seqs == a->c.B && l->many_blocks == a->many_blocks &&
            (rows + many_rows) * row_bytes <= kSliceBytes;
  l->few_scores = l->scores = take((l->both || rows < many_rows ? many_rows : rows) * a->score_stride);
  l->few_spilled = l->spilled;
  if (l->both) {
    l->few_scores = take(rows * a->score_stride);
    l->few_spilled = take(rows);
  }
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
  int major = 0;
  cudaError_t err = device_facts(&major, &a.sms);
  if (err != cudaSuccess) return fail_cuda(err);
  if (major != 10) return ENTMAX_ATTN_EUNSUPPORTED;          // the score kernels need tcgen05 / TMA
  a.c.table = block_table; a.c.kv_len = kv_len; a.c.cu_q = cu_q;
  a.beta = beta; a.gamma = gamma; a.delta = delta; a.alibi = alibi_slopes;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.counters = reinterpret_cast<int32_t*>(ws);
  a.row_info = reinterpret_cast<float4*>(ws + l.row_info);
  a.row_scale = reinterpret_cast<float*>(ws + l.row_scale);
  a.blocks = reinterpret_cast<PagedBlock*>(ws + l.blocks);
  a.order = reinterpret_cast<int32_t*>(ws + l.order);
  a.spilled = reinterpret_cast<int32_t*>(ws + l.spilled);
  a.group_max = reinterpret_cast<float*>(ws + l.group_max);
  a.record_key = reinterpret_cast<int32_t*>(ws + l.record_key);
  a.scores = reinterpret_cast<float*>(ws + l.scores);
  a.record_bytes = make_uint2(32u, 4u);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.tau = tau;
  a.support = support_size;
  a.status = device_status;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  auto run_few = [&](PagedArgs f, int b, int n, cudaStream_t st) {
    f.scores = reinterpret_cast<float*>(ws + l.few_scores);
    f.spilled = reinterpret_cast<int32_t*>(ws + l.few_spilled);
    f.counters = a.counters + kCounters;
    cudaError_t e = cudaSuccess;
    if (solve_lanes(f, (long long)n * f.c.KH * f.few_slots) != 0) e = cudaMemsetAsync(f.counters, 0, kCounters * sizeof(int32_t), st);
    if (e == cudaSuccess) e = launch_paged_few(f, q, k_cache, params->q_stride_t, params->q_stride_h, b, n, st);
    return e == cudaSuccess ? launch_solve<false>(f, v_cache, b, n * f.c.KH, st) : e;
  };
  auto run_many = [&](int blk, int n) {
    const int scale_ctas = (a.c.T + kPlanThreads / 32 - 1) / (kPlanThreads / 32);
    cudaError_t e = launch_kernel(paged_plan_kernel, 1 + (scale_ctas < a.sms - 1 ? scale_ctas : a.sms - 1), kPlanThreads, 0, stream, a, blk, n);
    if (e == cudaSuccess) e = launch_paged_many(a, q, k_cache, params->q_stride_t, params->q_stride_h, n, stream);
    return e == cudaSuccess ? launch_solve<true>(a, v_cache, 0, n * a.c.KH, stream) : e;
  };
  SideStream* side = nullptr;
  if (l.both) {
    err = side_stream(stream, &side);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  if (side) {
    err = cudaEventRecord(side->fork, stream);
    if (err == cudaSuccess) err = cudaStreamWaitEvent(side->stream, side->fork, 0);
    if (err != cudaSuccess) return fail_cuda(err);
    err = run_few(a, 0, a.c.B, side->stream);
    if (err == cudaSuccess) err = run_many(0, a.many_blocks);
    // (joined whatever happened: a capture must not end with the other stream still forked)
    cudaError_t join = cudaEventRecord(side->join, side->stream);
    if (join == cudaSuccess) join = cudaStreamWaitEvent(stream, side->join, 0);
    if (err == cudaSuccess) err = join;
  } else {
    for (int b = 0; l.few && b < a.c.B && err == cudaSuccess; b += l.few_seqs)
      err = run_few(a, b, a.c.B - b < l.few_seqs ? a.c.B - b : l.few_seqs, stream);
    for (int blk = 0; l.many && blk < a.many_blocks && err == cudaSuccess; blk += l.many_blocks)
      err = run_many(blk, a.many_blocks - blk < l.many_blocks ? a.many_blocks - blk : l.many_blocks);
  }
  if (err == cudaSuccess) err = cudaGetLastError();
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
