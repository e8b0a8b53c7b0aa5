// Scores of new tokens against a paged cache on sm_100a: tcgen05 contractions (bf16 in, fp32 in TMEM), K pages staged by TMA
// straight from the pool (one box per page and 64 columns; no copy of the cache, no gather kernel).
//
// What is kept of S = Q K^T is little: the keys above a lower bound of the row's threshold, a bound that rises while the keys stream by --
// the largest value so far minus 1 (App. A: tau >= y_max - 1), or the threshold of a few of the keys seen (that of a subset never exceeds
// that of the whole row).  So every key of the support is kept, whatever order the tiles come in and however the keys are
// split: a bound taken from fewer keys is lower and keeps more, and what is kept beyond the support has no influence on the result.
// There is room for every key of a row: flat logits cost stores, not another path.
//
// Two shapes of the same product:
//   few   sequences with at most 32 rows (new tokens x query heads of a K/V head): K tile of 128 keys as the M side, rows as N = 16 or
//         32; TMEM lane = key, a warp's 32 keys are a group.  Bound by reading K: 2 CTAs per SM, a ring of TMA tiles each.
//   many  longer chunks: 128 rows as the M side, two such Q tiles against K tiles of 256 keys (N = 256: at N = 128 the operand reads
//         from shared memory bound the MMA).  TMEM lane = row, one thread scans its row's 256 columns: about one instruction
//         per 32 rows and key against 8 with a lane per key.
#include <cuda.h>

#include <atomic>

#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace entmax {

namespace {

using namespace sm100;

// A tile of keys is loaded in boxes of 1 << box_shift = min(page size, 128) of them, lane x of the producer issuing box x.  Boxes past
// the sequence's end are not loaded: whatever the tile holds there, its scores are masked.
__device__ __forceinline__ int boxes_needed(int key0, int tile_keys, int len, int box_shift) {
  const int keys = min(tile_keys, len - key0);
  return (keys + (1 << box_shift) - 1) >> box_shift;
}
// page and first slot of box x of the tile at key0 (page = n_pages, which TMA reads as zeros, where the table is wrong)
__device__ __forceinline__ void page_of_box(const PagedCache& c, int b, int key, int32_t* status, int& page, int& slot) {
  const int at = key >> c.ps_shift;
  slot = key & ((1 << c.ps_shift) - 1);
  page = at < c.max_pages ? c.table[(long long)b * c.table_stride + at] : -1;
  if ((unsigned)page >= (unsigned)c.n_pages) {
    page = c.n_pages;
    if (status) atomicOr(status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_PAGE);
  }
}

// ================================================================================================ few
constexpr int kTile = 128;
constexpr int kFewThreads = 6 * 32;

// NR: rows a thread works on (a multiple of 4); NB: rows of the MMA's B operand
template <int HD, int NR>
struct FewCfg {
  static constexpr int NB = NR <= 16 ? 16 : 32;
  static constexpr int kHalves = HD / 64;
  static constexpr int kKBytes = kTile * HD * 2;
  static constexpr int kQBytes = NB * HD * 2;
  // 96 KB of loads in flight per CTA, two CTAs per SM; 64 KB beside 32 query rows of 128 (three stages and one buffer of query rows instead
  // of two and two: 118 us against 107 on 32 sequences of 8192 keys, five tokens, 32 heads)
  static constexpr int kStages = HD == 64 ? 6 : NR <= 16 ? 3 : 2;
  static constexpr int kQBufs = 2;
  static constexpr int kBarBytes = 256;
  static constexpr int kRowBytes = 4 * NR * 16;            // the rows' parameters, a copy per consumer warp
  static constexpr int kTmem = NB == 16 ? 32 : 64;         // two accumulators
  static constexpr int kFixedBytes = kStages * kKBytes + kQBufs * kQBytes + kRowBytes + kBarBytes + 1024;
};

// A = K tile, B = query rows, both K-major bf16, fp32 accumulate, M = 128, N = NB
__host__ __device__ constexpr uint32_t idesc_few(int nb) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(nb >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}

template <int N>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&acc)[N]) {
  if constexpr (N == 8) tmem_ld8(taddr, acc);
  else if constexpr (N == 16) tmem_ld16(taddr, acc);
  else tmem_ld32(taddr, acc);
}

// The tiles of all sequences and K/V heads, one after another (head by head), are dealt to the CTAs in equal runs: a CTA walks its run as
// segments, each some tiles of one (sequence, K/V head).  So the machine is full and finishes together whatever the lengths are.
// Bound by reading K once: 64 single tokens, contexts up to 4096, 8 K/V heads of 128: 318 MB in 57 us (5.6 TB/s, start-up included; 60 behind a
// flushed L2); five tokens each of 32 sequences over 8192 keys with slopes 94 us (5.7 TB/s).
struct FewSegment {
  int b, kvh;            // sequence (of the slice) and K/V head
  int tile, tiles;       // first tile and number of tiles
};
struct FewWalk {
  long long x, end;      // next tile of the run, end of the run
  int b, kvh;
};

template <int HD, int NR, bool kAlibi>
__global__ void __launch_bounds__(kFewThreads, 2) paged_few_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                 const __grid_constant__ CUtensorMap map_k,
                                                                 const __grid_constant__ PagedArgs a, int seq0, int seqs) {
  pdl_begin();
  using C = FewCfg<HD, NR>;
  constexpr int NB = C::NB;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int warp_sum[kFewThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int box_shift = min(a.c.ps_shift, 7);

  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t k_smem = sbase;                            // [kStages] K tiles
  const uint32_t q_smem = k_smem + C::kStages * C::kKBytes; // [kQBufs] query rows of a segment
  const uint32_t row_par = q_smem + C::kQBufs * C::kQBytes;         // [4 warps][NR]: a, slope, position (float), position (int)
  const uint32_t bars = row_par + C::kRowBytes;
  const uint32_t q_full = bars;                             // [2]
  const uint32_t q_empty = q_full + 16;                     // [2]
  const uint32_t kv_full = q_empty + 16;                    // [kStages]
  const uint32_t kv_empty = kv_full + 8 * C::kStages;       // [kStages]
  const uint32_t s_full = kv_empty + 8 * C::kStages;        // [2]
  const uint32_t s_empty = s_full + 16;                     // [2]
  const uint32_t tmem_slot = s_empty + 16;
  const uint32_t abort_flag = tmem_slot + 4;
  const uint32_t drain_bar = tmem_slot + 8;                 // teardown: every MMA issued so far has finished
  const uint32_t drain_fail = drain_bar + 8;                // uint32: a teardown wait ran out as well
  static_assert(8 * (4 + 2 * C::kStages + 4) + 8 + 16 <= C::kBarBytes, "barrier area");
  // tiles before sequence b, then {first row of q, new tokens, length} of it
  int* before = reinterpret_cast<int*>(smem_raw + (bars + C::kBarBytes - smem_u32(smem_raw)));
  int* info = before + seqs + 1;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full + 8 * t, 1);
      mbar_init(q_empty + 8 * t, 1);
      mbar_init(s_full + 8 * t, 1);
      mbar_init(s_empty + 8 * t, 4);
    }
    for (int t = 0; t < C::kStages; ++t) {
      mbar_init(kv_full + 8 * t, 1);
      mbar_init(kv_empty + 8 * t, 1);
    }
    mbar_init(drain_bar, 1);
    sts_u32(drain_fail, 0u);
    sts_u32(abort_flag, 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, C::kTmem);
    tmem_relinquish();
  }
  // ---- running sum of the sequences' tiles
  const int per = (seqs + kFewThreads - 1) / kFewThreads;   // consecutive sequences of a thread
  int mine = 0;
  for (int i = threadIdx.x * per; i < min(seqs, (int)(threadIdx.x + 1) * per); ++i) {
    const PagedSeq s = paged_seq(a.c, seq0 + i);
    const int tiles = s.n > 0 && paged_ok(a, s) && paged_few(a, s) ? (s.len + kTile - 1) / kTile : 0;
    info[3 * i] = s.q0;
    info[3 * i + 1] = s.n;
    info[3 * i + 2] = s.len;
    before[i + 1] = tiles;
    mine += tiles;
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sum[warp] = incl;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  {
    int at = incl - mine;
    for (int i = 0; i < warp; ++i) at += warp_sum[i];
    if (threadIdx.x == 0) before[0] = 0;
    for (int i = threadIdx.x * per; i < min(seqs, (int)(threadIdx.x + 1) * per); ++i) {
      at += before[i + 1];
      before[i + 1] = at;
    }
  }
  __syncthreads();
  const uint32_t tmem_base = lds_u32(tmem_slot);
  const int head_tiles = before[seqs];                       // of one K/V head
  const long long total = (long long)head_tiles * a.c.KH;
  const long long ctas = min((long long)gridDim.x, max(total / 2, 1ll));   // (runs of two tiles at least)

  FewWalk start;
  start.x = start.end = 0;
  start.b = start.kvh = 0;
  if (blockIdx.x < ctas) {
    start.x = total * blockIdx.x / ctas;
    start.end = total * (blockIdx.x + 1) / ctas;
    if (start.x < start.end) {
      start.kvh = (int)(start.x / head_tiles);
      const int y = (int)(start.x - (long long)start.kvh * head_tiles);
      int lo = 0, hi = seqs;                                 // largest b with before[b] <= y
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (before[mid] <= y) lo = mid; else hi = mid;
      }
      start.b = lo;
    }
  }
  // Slopes: a segment's tiles from the last one backwards, since the nearest keys have the smallest penalty and set the bound (in key order
  // nearly every group of such a head brings a new maximum and is stored)
  auto tile_of = [&](const FewSegment& g, int t) { return kAlibi ? g.tile + g.tiles - 1 - t : g.tile + t; };
  auto next_segment = [&](FewWalk& w, FewSegment& g) -> bool {
    if (w.x >= w.end) return false;
    const int y = (int)(w.x - (long long)w.kvh * head_tiles);
    while (before[w.b + 1] <= y) ++w.b;
    g.b = w.b;
    g.kvh = w.kvh;
    g.tile = y - before[w.b];
    g.tiles = (int)min((long long)(before[w.b + 1] - y), w.end - w.x);
    w.x += g.tiles;
    if (y + g.tiles == head_tiles) {
      w.b = 0;
      ++w.kvh;
    }
    return true;
  };

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer: a lane per page box
    int stage = 0, qb = 0;
    uint32_t phase = 0, qphase = 0;
    bool alive = true;
    auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
    };
    const int boxes = kTile >> box_shift;                    // of a whole tile: a power of two, at most 8
    const int ahead = 32 / boxes;                            // tiles that 32 page numbers, a lane each, cover
    FewWalk w = start;
    FewSegment g;
    while (alive && next_segment(w, g)) {
      const int q0 = info[3 * g.b], len = info[3 * g.b + 2];
      const int b = seq0 + g.b;
      auto look_up = [&](int t, int& page, int& slot) {
        const int at = t + lane / boxes, key = tile_of(g, at) * kTile + ((lane & (boxes - 1)) << box_shift);
        if (at < g.tiles && key < len) page_of_box(a.c, b, key, a.status, page, slot);
      };
      int page = 0, slot = 0, page2 = 0, slot2 = 0;
      look_up(0, page2, slot2);
      alive = wait_all(q_empty + 8 * qb, qphase ^ 1u);
      if (!alive) break;
      if (elect_one()) {
        mbar_expect_tx(q_full + 8 * qb, (uint32_t)(a.few_slots * 128 * C::kHalves));
        for (int hf = 0; hf < C::kHalves; ++hf)
          tma_load_4d(q_smem + qb * C::kQBytes + hf * (NB * 128), &map_q, q_full + 8 * qb, hf * 64, g.kvh * a.G, q0, 0);
      }
      __syncwarp();
      if (++qb == C::kQBufs) { qb = 0; qphase ^= 1u; }
      for (int t = 0; t < g.tiles; ++t) {
        const int key0 = tile_of(g, t) * kTile;
        if (t % ahead == 0) {
          page = page2;
          slot = slot2;
          look_up(t + ahead, page2, slot2);                  // (its latency is covered by the tiles in between)
        }
        const int src = (t % ahead) * boxes + (lane & (boxes - 1));
        const int pg = __shfl_sync(0xffffffffu, page, src), sl = __shfl_sync(0xffffffffu, slot, src);
        alive = wait_all(kv_empty + 8 * stage, phase ^ 1u);
        if (!alive) break;
        const int need = boxes_needed(key0, kTile, len, box_shift);
        const uint32_t box_bytes = 128u << box_shift;
        if (lane == 0) mbar_expect_tx(kv_full + 8 * stage, (uint32_t)need * box_bytes * C::kHalves);
        __syncwarp();
        if (lane < need) {
#pragma unroll
          for (int hf = 0; hf < C::kHalves; ++hf)
            tma_load_4d(k_smem + stage * C::kKBytes + hf * (kTile * 128) + lane * box_bytes, &map_k, kv_full + 8 * stage, hf * 64, sl,
                        g.kvh, pg);
        }
        __syncwarp();
        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!alive && lane == 0) {
      // a wait ran out somewhere in the CTA: the copies this warp armed barriers for must land before shared
      // memory goes away (buffers before the next one to fill: this round of the ring; the others: the previous round)
      bool ok = true;
      for (int t = 0; t < C::kQBufs; ++t) ok &= mbar_drain(q_full + 8 * t, t < qb ? qphase : qphase ^ 1u);
      for (int st = 0; st < C::kStages; ++st) ok &= mbar_drain(kv_full + 8 * st, st < stage ? phase : phase ^ 1u);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_few(NB);
      const uint32_t k_lo = smem_desc_lo(k_smem), q_lo = smem_desc_lo(q_smem);
      int stage = 0, buf = 0, qb = 0;
      uint32_t phase = 0, qphase = 0, sphase[2] = {0, 0};
      bool alive = true;
      FewWalk w = start;
      FewSegment g;
      while (alive && next_segment(w, g)) {
        alive = mbar_wait(q_full + 8 * qb, qphase, abort_flag);
        const uint32_t b_lo = q_lo + qb * (C::kQBytes >> 4);
        for (int t = 0; t < g.tiles && alive; ++t) {
          alive = mbar_wait(kv_full + 8 * stage, phase, abort_flag);
          if (alive) alive = mbar_wait(s_empty + 8 * buf, sphase[buf] ^ 1u, abort_flag);
          if (!alive) break;
          sphase[buf] ^= 1u;
          tc_fence_after();
          const uint32_t a_lo = k_lo + stage * (C::kKBytes >> 4);
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t a_off = (kk >> 2) * ((kTile * 128) >> 4) + (kk & 3) * 2;
            const uint32_t b_off = (kk >> 2) * ((NB * 128) >> 4) + (kk & 3) * 2;
            umma_bf16(tmem_base + buf * NB, a_lo + a_off, b_lo + b_off, kDescHi, idesc, kk > 0 ? 1u : 0u);
          }
          umma_commit(s_full + 8 * buf);
          umma_commit(kv_empty + 8 * stage);
          if (t == g.tiles - 1) umma_commit(q_empty + 8 * qb);
          buf ^= 1;
          if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
        }
        if (++qb == C::kQBufs) { qb = 0; qphase ^= 1u; }
      }
      if (!alive) {
        // the tensor core must be done with shared memory and TMEM before they are released
        umma_commit(drain_bar);
        if (!mbar_drain(drain_bar, 0u)) sts_u32(drain_fail, 1u);
      }
    }
  } else {
    // ------------------------------------------------------------------ a thread per key of the tile, a group per warp
    const int quad = warp & 3;
    const uint32_t taddr = tmem_base + ((uint32_t)(quad * 32) << 16);
    const uint32_t par = row_par + (uint32_t)quad * (NR * 16);
    uint32_t sphase[2] = {0, 0};
    int buf = 0;
    bool alive = true;
    FewWalk w = start;
    FewSegment g;
    while (alive && next_segment(w, g)) {
      const int n = info[3 * g.b + 1], len = info[3 * g.b + 2];
      const int rows = n * a.G;
      const int pos0 = len - n;                              // position of the first new token
      const int unit = g.b * a.c.KH + g.kvh;
      float* score0 = a.scores + (size_t)unit * a.few_slots * a.score_stride;
      float* max0 = a.group_max + ((size_t)unit * a.few_slots + (lane < rows ? lane : 0)) * a.groups;
      __syncwarp();
      if (lane < NR) {
        float ra = 0.f, slope = 0.f;
        int pos = -1;                                        // (rows past the last one see nothing)
        if (lane < rows) {
          const int head = g.kvh * a.G + lane % a.G;
          pos = pos0 + lane / a.G;
          ra = paged_scale(a, head, pos);
          if (kAlibi) slope = a.alibi[head] / a.sm_scale;    // bias in dot-product units
        }
        sts_f4(par + 16 * lane, ra, slope, (float)pos, __int_as_float(pos));
      }
      __syncwarp();
      // (largest value so far) - 1, the same in every lane.  A group at the bound is written too: where the 1 is lost in rounding (see one_below) it
      // holds a value as large as any.
      float bound[NR];
#pragma unroll
      for (int r = 0; r < NR; ++r) bound[r] = r < rows ? -INFINITY : INFINITY;
      for (int t = 0; t < g.tiles; ++t) {
        alive = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * buf, sphase[buf], abort_flag));
        if (!alive) break;
        sphase[buf] ^= 1u;
        tc_fence_after();
        constexpr int kCols = NR <= 8 ? 8 : NR <= 16 ? 16 : 32;
        float acc[kCols];
        load_columns<kCols>(taddr + buf * NB, acc);
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_empty + 8 * buf);
        buf ^= 1;
        const int group = tile_of(g, t) * (kTile / 32) + quad;
        const int j = group * 32 + lane;
        if (group * 32 >= len) continue;                     // (groups nobody looks at)
        const bool edge = group * 32 + 31 > pos0;
        float top = -INFINITY;                               // lane r: the maximum of row r
        // four rows together, so that their reductions overlap
#pragma unroll
        for (int r0 = 0; r0 < NR; r0 += 4) {
          if (r0 > 0 && r0 >= rows) continue;                // (sequences with fewer rows than the longest)
          float y[4], m[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            float ra, slope, posf, posi;
            lds_f4(par + 16 * (r0 + u), ra, slope, posf, posi);
            y[u] = ra * (kAlibi ? fmaf(slope, (float)j - posf, acc[r0 + u]) : acc[r0 + u]);
            if (edge) y[u] = j <= __float_as_int(posi) ? y[u] : -INFINITY;
            m[u] = y[u];
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(m[u]));
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int r = r0 + u;
            if (m[u] >= bound[r]) score0[(size_t)r * a.score_stride + j] = y[u];
            bound[r] = fmaxf(bound[r], m[u] - 1.0f);
            top = lane == r ? m[u] : top;
          }
        }
        if (lane < rows) max0[group] = top;
      }
    }
  }

  // ---------------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (lds_u32(abort_flag)) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_WAIT_EXPIRED);
    // the producer and the MMA issuer have waited for their copies and MMAs in flight; only if one of those waits ran
    // out as well is there nothing left but to give the hardware time
    if (lds_u32(drain_fail)) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 200000ull) { }
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, C::kTmem);
  }
  // sequences that cannot be served
  for (int i = blockIdx.x; i < seqs; i += gridDim.x) {
    PagedSeq s;
    s.q0 = info[3 * i];
    s.n = info[3 * i + 1];
    s.len = info[3 * i + 2];
    if (s.n == 0 || paged_ok(a, s)) continue;
    if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
    for (int kvh = 0; kvh < a.c.KH; ++kvh) write_unserved(a, s, kvh, threadIdx.x, kFewThreads);
  }
}

// =============================================================================================== many
// Two Q tiles share each K tile; a scheduler warp hands out work items, so that producer, MMA issuer and consumers run ahead of one another across
// items.  Bound by the MMA at head_dim 128 (2048 tokens over 32768 keys, 16 heads: 266 GFLOP in 210 us, 1.27 PFLOP/s, tensor pipe 70 % busy) and
// by the consumers' scan at 64, where an accumulator is made in half the time and short rows look at their first tile twice (11402 prompt tokens,
// 16 heads: 86 us; with the scan left out 38).
constexpr int BM = 128;
constexpr int BN = kManyKeys;
constexpr int kManyConsumers = 4 * kManyTiles;
constexpr int kManyThreads = (3 + kManyConsumers) * 32;
constexpr int kSchedWarp = 2 + kManyConsumers;
constexpr int kSchedSlots = 4;
static_assert(kManyTiles * BN == 512, "TMEM budget");
constexpr int kScaleBytes = kSchedSlots * kManyTiles * BM * 4;

template <int HD>
struct ManyCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kQBytes = BM * HD * 2;
  static constexpr int kKBytes = BN * HD * 2;
  static constexpr int kStages = HD == 128 ? 2 : 4;
  static constexpr int kQBufs = HD == 128 ? kManyTiles : 2 * kManyTiles;   // Q tiles: the next item's too where they fit
  static constexpr int kBarBytes = 1024 + 512;
  static constexpr int kSmemBytes = kQBufs * kQBytes + kStages * kKBytes + kBarBytes + kScaleBytes + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory of one CTA");
};

__host__ __device__ constexpr uint32_t idesc_many() {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
}

// A work item: one block of new tokens, one K/V head, one share of the keys.  Published by the scheduler with the pages of its first keys.
struct ManyItem {
  int b, kvh, q0, n, len, t0, lo, hi;      // t0: first token of the block within the chunk; K tiles lo .. hi - 1
  int unit, item;                          // row slots: unit * many_slots; which of the unit's items
};
constexpr int kItemWords = 10 + 64;        // the fields, then page and slot of 32 boxes

// K tiles that Q tile x of the item looks at: lo .. this - 1 (no more than lo: none)
__device__ __forceinline__ int many_tile_end(const PagedArgs& a, const ManyItem& it, int x) {
  const int first = it.t0 + x * a.tile_tokens;
  if (first >= it.n) return it.lo;
  const int last = min(first + a.tile_tokens, it.n) - 1;
  return max(min((it.len - it.n + last) / BN + 1, it.hi), it.lo);
}

// Where x > thr: eight values to record n (one 32-byte store), their first key beside them, and n moved on.  Predicated instructions instead of
// a branch: a lane that has nothing to store costs the warp its issue slots and no divergence.  The scan is bound by the ALU pipe
// (comparisons and integer additions at half rate), so the addresses are products on the other one; the factors come from memory so that they
// stay products.
template <int kFirst>
__device__ __forceinline__ void keep_record_if_greater(float x, float thr, uint32_t& n, const float* rec, const int32_t* key, uint2 bytes,
                                                       int col0, const float* v) {
  asm volatile(
      "{\n"
      " .reg .pred p;\n"
      " .reg .u64 ra, ka;\n"
      " .reg .u32 first;\n"
      " setp.gt.f32 p, %1, %2;\n"
      " mad.wide.u32 ra, %0, %5, %3;\n"
      " mad.wide.u32 ka, %0, %6, %4;\n"
      " add.u32 first, %7, %16;\n"
      " @p st.global.v8.f32 [ra], {%8, %9, %10, %11, %12, %13, %14, %15};\n"
      " @p st.global.u32 [ka], first;\n"
      " @p add.u32 %0, %0, 1;\n"
      "}\n"
      : "+r"(n)
      : "f"(x), "f"(thr), "l"(rec), "l"(key), "r"(bytes.x), "r"(bytes.y), "r"(col0), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
        "f"(v[5]), "f"(v[6]), "f"(v[7]), "n"(kFirst)
      : "memory");
}

// A lower bound of the threshold of a row from eight values of eight of its keys (-inf: none), y = z / margin: the threshold of those alone, by
// three steps from the left, in z's units.  Rows with no more than two of them in the bracket have nothing to gain (-inf
// is returned), nor is it worth the warp's time for less than `enough` rows, a quarter of those it has.  (Eight whatever it has: the warps with the
// last rows of a chunk never had a bound, and their rows came to the solve with hundreds of keys: flat prompts of 2500 tokens 135 us against 117.)
__device__ __forceinline__ float sqrt_fast(float x) { return x * rsqrtf(x); }
template <int EC>
__device__ __forceinline__ float eight_steps(const float (&y)[8], float expo) {
  float tau = -1.0f;                                           // relative to the largest
#pragma unroll 1
  for (int it = 0; it < 3; ++it) {
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      float ye, ye1;
      powers<EC>(fmaxf(y[q] - tau, 0.f), expo, ye, ye1);
      s0 += ye;
      s1 += ye1;
    }
    // threshold_step with the fast square root and quotients: a few ulp, well within the hair below
    const float root = EC == kExpo1 ? s0 : EC == kExpo2 ? s0 * rsqrtf(s0) : EC == kExpo4 ? sqrt_fast(sqrt_fast(s0)) : __powf(s0, __fdividef(1.0f, expo));
    if (s0 > 1.0f && s1 > 0.f) tau += __fdividef(s0 - __fdividef(s0, root), s1);
  }
  return tau;
}
__device__ __forceinline__ float bound_from_eight(const float (&z)[8], float margin, int expo_class, float expo, int enough) {
  const float m = max8(z);
  int n = 0;
#pragma unroll
  for (int q = 0; q < 8; ++q) n += z[q] > m - margin ? 1 : 0;
  if (expo < 1.0f || __popc(__ballot_sync(0xffffffffu, n > 2)) < enough) return -INFINITY;
  float y[8];
  const float r = __fdividef(1.0f, margin);
#pragma unroll
  for (int q = 0; q < 8; ++q) y[q] = (z[q] - m) * r;
  const float tau = expo_class == kExpo2 ? eight_steps<kExpo2>(y, expo)
                    : expo_class == kExpo1 ? eight_steps<kExpo1>(y, expo)
                    : expo_class == kExpo4 ? eight_steps<kExpo4>(y, expo) : eight_steps<kExpoGeneral>(y, expo);
  // a hair below for the rounding of the powers, of tau, and of the sum
  const float bound = m + tau * margin - (1e-5f * margin + 1e-6f * fabsf(m));
  return n > 2 && bound < INFINITY ? bound : -INFINITY;
}

// best - margin (y_max - 1 in z's units), and below the best where the margin is lost in its rounding
__device__ __forceinline__ float margin_below(float best, float margin) { return (best - margin) - fabsf(best) * 0x1p-21f; }

template <int HD, bool kAlibi>
__global__ void __launch_bounds__(kManyThreads, 1) paged_many_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                   const __grid_constant__ CUtensorMap map_k,
                                                                   const __grid_constant__ PagedArgs a, int blocks) {
  pdl_begin();
  using C = ManyCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = sbase;                                   // [kQBufs][kHalves][BM rows x 128 B]
  const uint32_t k_smem = sbase + C::kQBufs * C::kQBytes;          // [kStages][kHalves][BN rows x 128 B]
  const uint32_t scales = k_smem + C::kStages * C::kKBytes;        // float [kSchedSlots][kManyTiles * BM]: a of an item's rows
  const uint32_t bars = scales + kScaleBytes;
  const uint32_t q_full = bars;                                    // [kQBufs]
  const uint32_t q_empty = q_full + 8 * C::kQBufs;                 // [kQBufs]
  const uint32_t s_full = q_empty + 8 * C::kQBufs;                 // [kManyTiles]
  const uint32_t s_empty = s_full + 8 * kManyTiles;                // [kManyTiles]
  const uint32_t k_full = s_empty + 8 * kManyTiles;                // [kStages]
  const uint32_t k_empty = k_full + 8 * C::kStages;                // [kStages]
  const uint32_t w_full = k_empty + 8 * C::kStages;                // [kSchedSlots]
  const uint32_t w_empty = w_full + 8 * kSchedSlots;               // [kSchedSlots]
  const uint32_t w_item = w_empty + 8 * kSchedSlots;               // int32 [kSchedSlots][kItemWords]
  const uint32_t tmem_slot = w_item + 4 * kSchedSlots * kItemWords;
  const uint32_t abort_flag = tmem_slot + 4;
  const uint32_t drain_bar = tmem_slot + 8;                        // teardown: every MMA issued so far has finished
  const uint32_t drain_fail = drain_bar + 8;                       // uint32: a teardown wait ran out as well
  static_assert((2 * kManyTiles + 2 * C::kQBufs + 2 * C::kStages + 2 * kSchedSlots) * 8 + 4 * kSchedSlots * kItemWords + 8 + 16 <= C::kBarBytes,
                "barrier area");
  static_assert((4 * kSchedSlots * kItemWords) % 8 == 0, "drain_bar is 8-byte aligned");

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const int box_shift = min(a.c.ps_shift, 7);

  if (threadIdx.x == 0) {
    for (int t = 0; t < C::kQBufs; ++t) {
      mbar_init(q_full + 8 * t, 1);
      mbar_init(q_empty + 8 * t, 1);
    }
    for (int t = 0; t < kManyTiles; ++t) {
      mbar_init(s_full + 8 * t, 1);
      mbar_init(s_empty + 8 * t, 4);
    }
    for (int t = 0; t < C::kStages; ++t) {
      mbar_init(k_full + 8 * t, 1);
      mbar_init(k_empty + 8 * t, 1);
    }
    for (int t = 0; t < kSchedSlots; ++t) {
      mbar_init(w_full + 8 * t, 1);
      mbar_init(w_empty + 8 * t, 2 + kManyConsumers);              // producer, MMA issuer and consumer warps
    }
    mbar_init(drain_bar, 1);
    sts_u32(abort_flag, 0u);
    sts_u32(drain_fail, 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = lds_u32(tmem_slot);

  // Slopes: an item's tiles from the last one backwards (see paged_few_kernel).  (hi: of the item's Q tile or the item, whose ends meet in the
  // item's last tile.)
  auto tile_of = [&](int lo, int hi, int step) { return kAlibi ? hi - 1 - step : lo + step; };
  auto read_item = [&](int slot) {
    ManyItem it;
    const uint32_t at = w_item + 4u * kItemWords * slot;
    it.b = (int)lds_u32(at);
    it.kvh = (int)lds_u32(at + 4);
    it.q0 = (int)lds_u32(at + 8);
    it.n = (int)lds_u32(at + 12);
    it.len = (int)lds_u32(at + 16);
    it.t0 = (int)lds_u32(at + 20);
    it.lo = (int)lds_u32(at + 24);
    it.hi = (int)lds_u32(at + 28);
    it.unit = (int)lds_u32(at + 32);
    it.item = (int)lds_u32(at + 36);
    return it;
  };

  if (warp == 0) {
    // ------------------------------------------------------------- TMA producer (the whole warp; a lane per page box)
    int stage = 0, slot = 0;
    int qb = 0;
    uint32_t kphase = 0, qphase = 0, wphase = 0;
    bool alive = true;
    auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
    };
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const ManyItem it = read_item(slot);
      const uint32_t boxes_at = w_item + 4u * kItemWords * slot + 40 + 8 * lane;
      int page2 = (int)lds_u32(boxes_at), pslot2 = (int)lds_u32(boxes_at + 4);
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == kSchedSlots) { slot = 0; wphase ^= 1u; }
      if (it.b < 0) break;
      const int boxes = BN >> box_shift;                    // of a whole tile: a power of two, at most 16
      const int ahead = 32 / boxes;
      int end = it.lo;
      for (int x = 0; x < kManyTiles; ++x) end = max(end, many_tile_end(a, it, x));
      auto look_up = [&](int step, int& page, int& pslot) {
        const int at = step + lane / boxes, key = tile_of(it.lo, end, at) * BN + ((lane & (boxes - 1)) << box_shift);
        if (at < end - it.lo && key < it.len) page_of_box(a.c, it.b, key, a.status, page, pslot);
      };
      int page = 0, pslot = 0;
      auto load_q = [&]() -> bool {
        for (int x = 0; x < kManyTiles; ++x) {
          if (many_tile_end(a, it, x) <= it.lo) continue;
          if (!wait_all(q_empty + 8 * qb, qphase ^ 1u)) return false;
          if (elect_one()) {
            mbar_expect_tx(q_full + 8 * qb, (uint32_t)(a.tile_tokens * a.G * 128 * C::kHalves));
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(q_smem + qb * C::kQBytes + hf * (BM * 128), &map_q, q_full + 8 * qb, hf * 64, it.kvh * a.G,
                          it.q0 + it.t0 + x * a.tile_tokens, 0);
          }
          __syncwarp();
          if (++qb == C::kQBufs) { qb = 0; qphase ^= 1u; }
        }
        return true;
      };
      // (with buffers of their own the next item's Q tiles come first, otherwise its K tile does while they wait for theirs)
      if (C::kQBufs > kManyTiles) alive = load_q();
      for (int step = 0; step < end - it.lo && alive; ++step) {
        const int key0 = tile_of(it.lo, end, step) * BN;
        if (step % ahead == 0) {
          page = page2;
          pslot = pslot2;
          look_up(step + ahead, page2, pslot2);             // (its latency is covered by the tiles in between)
        }
        const int src = (step % ahead) * boxes + (lane & (boxes - 1));
        const int pg = __shfl_sync(0xffffffffu, page, src), sl = __shfl_sync(0xffffffffu, pslot, src);
        alive = wait_all(k_empty + 8 * stage, kphase ^ 1u);
        if (!alive) break;
        const int need = boxes_needed(key0, BN, it.len, box_shift);
        const uint32_t box_bytes = 128u << box_shift;
        if (lane == 0) mbar_expect_tx(k_full + 8 * stage, (uint32_t)need * box_bytes * C::kHalves);
        __syncwarp();
        if (lane < need) {
#pragma unroll
          for (int hf = 0; hf < C::kHalves; ++hf)
            tma_load_4d(k_smem + stage * C::kKBytes + hf * (BN * 128) + lane * box_bytes, &map_k, k_full + 8 * stage, hf * 64, sl,
                        it.kvh, pg);
        }
        __syncwarp();
        if (++stage == C::kStages) { stage = 0; kphase ^= 1u; }
        if (C::kQBufs == kManyTiles && step == 0 && alive) alive = load_q();
      }
    }
    if (!alive && lane == 0) {
      // a wait ran out somewhere in the CTA: every copy this warp armed a barrier for must have landed before
      // shared memory goes away.  Stages before `stage` were armed in this round of the ring, the others in the
      // previous one (a barrier that was never armed reports its "previous" phase as complete at once).
      bool ok = true;
      for (int st = 0; st < C::kStages; ++st) ok &= mbar_drain(k_full + 8 * st, st < stage ? kphase : kphase ^ 1u);
      for (int x = 0; x < C::kQBufs; ++x) ok &= mbar_drain(q_full + 8 * x, x < qb ? qphase : qphase ^ 1u);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (warp-wide control flow, one elected lane issues)
    constexpr uint32_t idesc = idesc_many();
    const uint64_t hi = (uint64_t)kDescHi << 32;
    const uint64_t q_desc = hi | smem_desc_lo(q_smem), k_desc = hi | smem_desc_lo(k_smem);
    int stage = 0, slot = 0, qb = 0;
    uint32_t kphase = 0, qphase = 0, wphase = 0, sphase[kManyTiles] = {};
    bool alive = true;
    auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
    };
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      ManyItem it = read_item(slot);
      it.b = __shfl_sync(0xffffffffu, it.b, 0);
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == kSchedSlots) { slot = 0; wphase ^= 1u; }
      if (it.b < 0) break;
      const int lo = __shfl_sync(0xffffffffu, it.lo, 0);
      int tx[kManyTiles], buf[kManyTiles], end = lo;
      uint32_t bphase[kManyTiles];
      for (int x = 0; x < kManyTiles; ++x) {
        tx[x] = __shfl_sync(0xffffffffu, many_tile_end(a, it, x), 0);
        end = max(end, tx[x]);
        buf[x] = qb;
        bphase[x] = qphase;
        if (tx[x] > lo && ++qb == C::kQBufs) { qb = 0; qphase ^= 1u; }
      }
      for (int step = 0; step < end - lo && alive; ++step) {
        const int t = tile_of(lo, end, step);
        alive = wait_all(k_full + 8 * stage, kphase);
        if (!alive) break;
        const uint64_t b_desc = k_desc + (uint64_t)(stage * (C::kKBytes >> 4));
#pragma unroll
        for (int x = 0; x < kManyTiles; ++x) {
          if (t >= tx[x] || !alive) continue;
          if (t == (kAlibi ? tx[x] - 1 : lo)) alive = wait_all(q_full + 8 * buf[x], bphase[x]);
          if (alive) alive = wait_all(s_empty + 8 * x, sphase[x] ^ 1u);
          if (!alive) continue;
          sphase[x] ^= 1u;
          tc_fence_after();
          const uint64_t a_desc = q_desc + (uint64_t)(buf[x] * (C::kQBytes >> 4));
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint32_t a_off = (kk >> 2) * ((BM * 128) >> 4) + (kk & 3) * 2;
              const uint32_t b_off = (kk >> 2) * ((BN * 128) >> 4) + (kk & 3) * 2;
              umma_bf16_desc(tmem_base + x * BN, a_desc + a_off, b_desc + b_off, idesc, kk > 0 ? 1u : 0u);
            }
            umma_commit(s_full + 8 * x);
            if (t == (kAlibi ? lo : tx[x] - 1)) umma_commit(q_empty + 8 * buf[x]);
          }
          __syncwarp();
        }
        if (!alive) break;
        if (elect_one()) umma_commit(k_empty + 8 * stage);
        __syncwarp();
        if (++stage == C::kStages) { stage = 0; kphase ^= 1u; }
      }
    }
    if (!alive && lane == 0) {
      // the tensor core must be done with shared memory and TMEM before they are released
      umma_commit(drain_bar);
      if (!mbar_drain(drain_bar, 0u)) sts_u32(drain_fail, 1u);
    }
  } else if (warp == kSchedWarp) {
    // ------------------------------------------------------------------ scheduler: the next items, ahead of the others
    int slot = 0;
    uint32_t wphase = 0;
    const int n_blocks = a.counters[kBlocks], cut = a.counters[kCut], head_tiles = a.counters[kTiles];
    const int n_items = n_blocks * a.c.KH;
    int x = blockIdx.x * cut;                                // cut: next tile of this CTA's run
    const int x_end = min(x + cut, head_tiles * a.c.KH);
    int round = 0;
    for (bool more = true; more;) {
      ManyItem it;
      it.b = -1;
      it.lo = it.hi = it.len = 0;
      if (cut == 0) {
        // The blocks with the longest rows first, one to a CTA and round, every other round backwards, so that the CTAs end together.
        // (Handed out by an atomic counter the next item came 2 us after it was asked for, half of what one of seven tiles takes.)
        const int k = many_dealt(round, (int)blockIdx.x, (int)gridDim.x);
        more = round * (int)gridDim.x < n_items;
        ++round;
        if (more && k >= n_items) continue;
        if (more) {
          it.kvh = k % a.c.KH;
          const int blk = a.order[k / a.c.KH];
          const PagedBlock pb = a.blocks[blk];
          it.b = pb.b; it.t0 = pb.t0; it.q0 = pb.q0; it.n = pb.n; it.len = pb.len;
          it.hi = pb.tiles;
          it.item = 0;
          it.unit = blk * a.c.KH + it.kvh;
        }
      } else {
        more = x < x_end;
        if (more) {
          it.kvh = x / head_tiles;
          const int y = x - it.kvh * head_tiles;
          int lo = 0, n = blocks;                            // the block with start <= y < start + tiles: 32 candidates a step
          while (n > 1) {
            const int step = (n + 31) / 32;
            const bool le = lane * step < n && (lane == 0 || a.blocks[lo + lane * step].start <= y);
            const int i = 31 - __clz(__ballot_sync(0xffffffffu, le));
            lo += i * step;
            n = min(step, n - i * step);
          }
          const PagedBlock pb = a.blocks[lo];
          const ManyCut c = many_cut(a.counters, pb, it.kvh);
          it.b = pb.b; it.t0 = pb.t0; it.q0 = pb.q0; it.n = pb.n; it.len = pb.len;
          it.lo = y - pb.start;
          it.hi = min(pb.tiles, it.lo + x_end - x);
          it.item = x / cut - c.start / cut;
          it.unit = lo * a.c.KH + it.kvh;
          x += it.hi - it.lo;
        }
      }
      int page = 0, pslot = 0;
      const int boxes = BN >> box_shift, step = lane / boxes;
      const int key = tile_of(it.lo, it.hi, step) * BN + ((lane & (boxes - 1)) << box_shift);
      if (it.b >= 0 && step < it.hi - it.lo && key < it.len) page_of_box(a.c, it.b, key, a.status, page, pslot);
      // a of the item's rows (the consumers would start each item with these loads)
      float ra[kManyTiles * BM / 32];
      const int tile_rows = a.tile_tokens * a.G;
#pragma unroll
      for (int i = 0; i < kManyTiles * BM / 32; ++i) {
        const int in_tile = (32 * i) % BM + lane, tok = it.t0 + 32 * i / BM * a.tile_tokens + in_tile / a.G;
        ra[i] = it.b >= 0 && in_tile < tile_rows && tok < it.n ? a.row_scale[(size_t)(it.q0 + tok) * a.H + it.kvh * a.G + in_tile % a.G] : 0.f;
      }
      if (!__all_sync(0xffffffffu, mbar_wait(w_empty + 8 * slot, wphase ^ 1u, abort_flag))) break;
      if (it.b >= 0) {
        const uint32_t to = scales + 4u * (kManyTiles * BM) * slot;
#pragma unroll
        for (int i = 0; i < kManyTiles * BM / 32; ++i) sts_u32(to + 4 * (32 * i + lane), __float_as_uint(ra[i]));
      }
      const uint32_t at = w_item + 4u * kItemWords * slot;
      sts_u32(at + 40 + 8 * lane, (uint32_t)page);
      sts_u32(at + 44 + 8 * lane, (uint32_t)pslot);
      if (lane == 0) {
        sts_u32(at, (uint32_t)it.b);
        if (it.b >= 0) {
          sts_u32(at + 4, (uint32_t)it.kvh);
          sts_u32(at + 8, (uint32_t)it.q0);
          sts_u32(at + 12, (uint32_t)it.n);
          sts_u32(at + 16, (uint32_t)it.len);
          sts_u32(at + 20, (uint32_t)it.t0);
          sts_u32(at + 24, (uint32_t)it.lo);
          sts_u32(at + 28, (uint32_t)it.hi);
          sts_u32(at + 32, (uint32_t)it.unit);
          sts_u32(at + 36, (uint32_t)it.item);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(w_full + 8 * slot);
      if (++slot == kSchedSlots) { slot = 0; wphase ^= 1u; }
    }
  } else {
    // -------------------------------------------------- consumers: one thread per query row
    const int x = (warp - 2) >> 2;
    const int quad = warp & 3;
    const int row_local = quad * 32 + lane;
    const uint32_t taddr_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(x * BN);
    const uint32_t my_full = s_full + 8 * x, my_empty = s_empty + 8 * x;
    const int tile_rows = a.tile_tokens * a.G;
    const uint2 rec_bytes = a.record_bytes;
    uint32_t fphase = 0, wphase = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = __all_sync(0xffffffffu, mbar_wait(w_full + 8 * slot, wphase, abort_flag));
      if (!alive) break;
      const ManyItem it = read_item(slot);
      const float ra = __uint_as_float(lds_u32(scales + 4u * (uint32_t)((slot * kManyTiles + x) * BM + row_local)));
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == kSchedSlots) { slot = 0; wphase ^= 1u; }
      if (it.b < 0) break;
      const int end = many_tile_end(a, it, x);
      if (end <= it.lo) continue;
      const int tok = it.t0 + x * a.tile_tokens + row_local / a.G;
      const bool valid = row_local < tile_rows && tok < it.n;
      const int head = it.kvh * a.G + row_local % a.G;
      const int pos = it.len - it.n + tok;
      const int lim = valid ? pos : -1;                        // last key the row sees
      const int first_pos = it.len - it.n + it.t0 + x * a.tile_tokens;             // of the tile's rows
      const int last_pos = min(first_pos + a.tile_tokens, it.len) - 1;
      const float slope = kAlibi && valid ? a.alibi[head] / a.sm_scale : 0.f;
      const int slot_row = valid ? x * tile_rows + row_local : 0;
      const size_t row = (size_t)it.unit * a.many_slots + (size_t)slot_row;
      const float* rec = a.scores + row * a.score_stride + (size_t)it.lo * BN;
      const int32_t* rec_key = a.record_key + row * (size_t)(a.tiles * 32) + it.lo * 32;
      uint32_t n_rec = 0;
      // Everything is compared before the scaling, z = <q,k> + slope (j - pos): y = a z, and a negative a turns z around first
      const float sign = ra < 0.f ? -1.f : 1.f;
      const bool turned = __any_sync(0xffffffffu, ra < 0.f);
      // (margin 0 of the tile's other lanes: what the operand holds in their places is not the call's, and none of it counts as near the largest in
      // the votes on bounds, which would let it choose how the warp's rows are rounded)
      const float mag = fabsf(ra), margin = valid ? 1.0f / mag : 0.f;
      const int enough = max(1, (__popc(__ballot_sync(0xffffffffu, valid)) + 3) / 4);
      // Lower bound of the row's threshold: (largest value so far) - margin, or what eight of its keys say, the largest of each of eight
      // classes.  Rows without keys never have a candidate.
      float thr = valid ? -INFINITY : INFINITY, best = -INFINITY;
      float top[8];
#pragma unroll
      for (int g = 0; g < 8; ++g) top[g] = -INFINITY;
      bool flat = false;
      for (int step_no = 0; step_no < end - it.lo && alive; ++step_no) {
        alive = __all_sync(0xffffffffu, mbar_wait(my_full, fphase, abort_flag));
        if (!alive) break;
        fphase ^= 1u;
        tc_fence_after();
        const int col_base = tile_of(it.lo, end, step_no) * BN;
        const int n_steps = min(BN / 64, (last_pos - col_base) / 64 + 1);   // 64-column steps that some row sees
        // 64 columns from column 64 c on, as both looks at them take them
        auto load = [&](float (&v)[64], int c) {
          tmem_ld64(taddr_row + 64 * c, v);
          tmem_ld_wait64(v);
          const int col0 = col_base + 64 * c;
          if (kAlibi) {
            const float t0 = slope * (float)(col0 - pos);
#pragma unroll
            for (int u = 0; u < 64; ++u) v[u] = fmaf(slope, (float)u, v[u]) + t0;
          }
          if (turned) {
#pragma unroll
            for (int u = 0; u < 64; ++u) v[u] *= sign;
          }
          if (col0 + 63 > first_pos) {                         // some row of the tile does not see all of them
            // (as bits: tested several at a time, where a comparison each is one more of the ALU's instructions per column)
            const int seen = lim + 1 - col0;                   // columns that the row sees
            const uint32_t lo = seen >= 32 ? 0xffffffffu : seen > 0 ? (1u << seen) - 1u : 0u;
            const uint32_t hi = seen >= 64 ? 0xffffffffu : seen > 32 ? (1u << (seen - 32)) - 1u : 0u;
#pragma unroll
            for (int u = 0; u < 32; ++u) {
              v[u] = (lo >> u) & 1u ? v[u] : -INFINITY;
              v[32 + u] = (hi >> u) & 1u ? v[32 + u] : -INFINITY;
            }
          }
        };
        // a stream that starts without a bound looks at its first tile twice
        if (step_no == 0) {
#pragma unroll 1
          for (int c = 0; c < n_steps; ++c) {
            float v[64];
            load(v, c);
#pragma unroll
            for (int q = 0; q < 8; ++q) top[q] = fmaxf(top[q], max8(&v[8 * q]));
          }
          best = max8(top);
          const float bound = bound_from_eight(top, margin, a.expo_class, a.expo, enough);
          flat = __any_sync(0xffffffffu, bound > -INFINITY);
          thr = fmaxf(thr, fmaxf(margin_below(best, margin), bound));
        }
        // One straight pass: maxima of eight columns, and eight columns with a candidate go to the row's records as they are, by predicated
        // stores where some row of the warp has one among 32 columns (a vote for 64: chunk of 2048 over 32768 keys 250 -> 243 us here;
        // for eight each: 254)
#pragma unroll 1
        for (int c = 0; c < n_steps; ++c) {
          float v[64];
          load(v, c);
          float g[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) g[q] = max8(&v[8 * q]);
          const float m_lo = fmaxf(fmaxf(g[0], g[1]), fmaxf(g[2], g[3])), m_hi = fmaxf(fmaxf(g[4], g[5]), fmaxf(g[6], g[7]));
          best = max3(best, m_lo, m_hi);
          thr = fmaxf(thr, margin_below(best, margin));
          if (flat) {
#pragma unroll
            for (int q = 0; q < 8; ++q) top[q] = fmaxf(top[q], g[q]);
          }
          const int col0 = col_base + 64 * c;
          if (__any_sync(0xffffffffu, m_lo > thr)) {
            keep_record_if_greater<0>(g[0], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[0]);
            keep_record_if_greater<8>(g[1], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[8]);
            keep_record_if_greater<16>(g[2], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[16]);
            keep_record_if_greater<24>(g[3], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[24]);
          }
          if (__any_sync(0xffffffffu, m_hi > thr)) {
            keep_record_if_greater<32>(g[4], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[32]);
            keep_record_if_greater<40>(g[5], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[40]);
            keep_record_if_greater<48>(g[6], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[48]);
            keep_record_if_greater<56>(g[7], thr, n_rec, rec, rec_key, rec_bytes, col0, &v[56]);
          }
        }
        // the accumulator has been read: hand it back to the MMA issuer
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(my_empty);
        // Where supports are long the bound is taken from the classes again after 2, 4, 8, ... tiles (keys that are a record among all before
        // them come ever more rarely)
        if (flat && step_no > 0 && (step_no & (step_no + 1)) == 0)
          thr = fmaxf(thr, bound_from_eight(top, margin, a.expo_class, a.expo, enough));
      }
      // (bound and best unscaled: a = 0 leaves no bound, and every key is kept)
      if (valid && alive)
        a.row_info[((size_t)it.unit * a.many_items + it.item) * a.many_slots + slot_row] = make_float4(__int_as_float((int)n_rec), thr, mag, best);
    }
  }

  // ---------------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (lds_u32(abort_flag)) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_WAIT_EXPIRED);
    // (see paged_few_kernel)
    if (lds_u32(drain_fail)) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 200000ull) { }
    }
    clear_records(a, blocks, threadIdx.x, kManyThreads);
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

// q [T][H][D] as (D, H, T, 1): a box of G heads by `tokens` tokens is the rows t * G + g of a Q tile
cudaError_t map_queries(CUtensorMap* map, const PagedArgs& a, const void* q, int64_t st, int64_t sh, int tokens) {
  return make_box_map(map, q, a.c.D, a.H, a.c.T, 1, sh, st, a.c.T * st, a.G, tokens);
}
// the pool as (D, slot, K/V head, page): boxes of min(page size, 128) slots
cudaError_t map_pages(CUtensorMap* map, const PagedArgs& a, const void* k) {
  return make_box_map(map, k, a.c.D, 1 << a.c.ps_shift, a.c.KH, a.c.n_pages, a.c.s_tok, a.c.s_head, a.c.s_page,
                      a.c.ps_shift < 7 ? 1 << a.c.ps_shift : 128, 1);
}

// Lets a kernel have its shared memory; once per device
template <auto* kKernel>
cudaError_t allow_smem(int bytes) {
  static std::atomic<unsigned long long> allowed{0};
  int dev = 0;
  cudaError_t err = cudaGetDevice(&dev);
  const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
  if (err != cudaSuccess || (allowed.load(std::memory_order_relaxed) & bit)) return err;
  err = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (err == cudaSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
  return err;
}

template <int HD, int NR, bool kAlibi>
cudaError_t launch_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int seq0, int seqs,
                       cudaStream_t stream) {
  CUtensorMap map_q, map_k;
  const int smem = FewCfg<HD, NR>::kFixedBytes + (4 * kFewSeqs + 4) * 4;
  static_assert(2 * (FewCfg<HD, NR>::kFixedBytes + (4 * kFewSeqs + 4) * 4 + 1024) <= 233472, "two CTAs per SM");
  cudaError_t err = map_queries(&map_q, a, q, q_st, q_sh, a.few_slots / a.G);
  if (err == cudaSuccess) err = map_pages(&map_k, a, k);
  if (err == cudaSuccess) err = allow_smem<&paged_few_kernel<HD, NR, kAlibi>>(smem);
  if (err != cudaSuccess) return err;
  const int sms = a.sms;
  // no more CTAs than the longest lengths could keep busy
  const long long most = (long long)seqs * a.c.KH * ((a.max_kv + kTile - 1) / kTile);
  const long long grid = most / 2 < 1 ? 1 : most / 2 < 2 * sms ? most / 2 : 2 * sms;
  return launch_kernel(paged_few_kernel<HD, NR, kAlibi>, (unsigned)grid, kFewThreads, smem, stream, map_q, map_k, a, seq0, seqs);
}

template <int HD, bool kAlibi>
cudaError_t launch_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int blocks, cudaStream_t stream) {
  CUtensorMap map_q, map_k;
  cudaError_t err = map_queries(&map_q, a, q, q_st, q_sh, a.tile_tokens);
  if (err == cudaSuccess) err = map_pages(&map_k, a, k);
  if (err == cudaSuccess) err = allow_smem<&paged_many_kernel<HD, kAlibi>>(ManyCfg<HD>::kSmemBytes);
  if (err != cudaSuccess) return err;
  return launch_kernel(paged_many_kernel<HD, kAlibi>, (unsigned)a.sms, kManyThreads, ManyCfg<HD>::kSmemBytes, stream, map_q, map_k, a, blocks);
}

}  // namespace

cudaError_t launch_paged_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int seq0, int seqs,
                             cudaStream_t stream) {
#define ENTMAX_FEW(HD, NR)                                                              \
  (a.alibi ? launch_few<HD, NR, true>(a, q, k, q_st, q_sh, seq0, seqs, stream)          \
           : launch_few<HD, NR, false>(a, q, k, q_st, q_sh, seq0, seqs, stream))
#define ENTMAX_FEW_ROWS(HD)                                                             \
  (a.few_slots <= 4 ? ENTMAX_FEW(HD, 4) : a.few_slots <= 8 ? ENTMAX_FEW(HD, 8) : a.few_slots <= 16 ? ENTMAX_FEW(HD, 16) : a.few_slots <= 24 ? ENTMAX_FEW(HD, 24) : ENTMAX_FEW(HD, 32))
  return a.c.D == 64 ? ENTMAX_FEW_ROWS(64) : ENTMAX_FEW_ROWS(128);
#undef ENTMAX_FEW_ROWS
#undef ENTMAX_FEW
}

cudaError_t launch_paged_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int blocks,
                              cudaStream_t stream) {
  if (a.c.D == 64)
    return a.alibi ? launch_many<64, true>(a, q, k, q_st, q_sh, blocks, stream)
                   : launch_many<64, false>(a, q, k, q_st, q_sh, blocks, stream);
  return a.alibi ? launch_many<128, true>(a, q, k, q_st, q_sh, blocks, stream)
                 : launch_many<128, false>(a, q, k, q_st, q_sh, blocks, stream);
}

}  // namespace entmax
