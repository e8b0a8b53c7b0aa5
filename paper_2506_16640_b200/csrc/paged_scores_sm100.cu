// Scores of new tokens against a paged cache on sm_100a: tcgen05 contractions (bf16 in, fp32 in TMEM), K pages staged by TMA
// straight from the pool (one box per page and 64 columns; no copy of the cache, no gather kernel).
//
// What is kept of S = Q K^T is little: the maximum of every 32 keys of a row, and the scores of those groups of 32 whose maximum is
// above (largest value seen so far) - 1.  Eq. 1's threshold is never below y_max - 1 (App. A), so every key of the support is in a
// group that is kept, whatever order the tiles come in and however the keys are split: a bound taken from fewer keys is lower and
// keeps more.  Which further groups are kept has no influence on the result (paged_solve_kernel looks only at the groups above
// the final y_max - 1).
//
// Two shapes of the same product:
//   few   sequences with at most 32 rows (new tokens x query heads of a K/V head): K tile of 128 keys as the M side, rows as N = 16 or
//         32; TMEM lane = key, a warp's 32 keys are a group.  Bound by reading K: 2 CTAs per SM, a ring of TMA tiles each.
//   many  longer chunks: 128 rows as the M side, two such Q tiles against K tiles of 256 keys (N = 256: at N = 128 the operand reads
//         from shared memory bound the MMA).  TMEM lane = row, one thread scans its row's 256 columns: 1.5 instructions
//         per 32 rows and key against 8 with a lane per key.  Bound by the tensor pipe.
#include <cuda.h>

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

template <int HD, int NB>
struct FewCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kKBytes = kTile * HD * 2;
  static constexpr int kQBytes = NB * HD * 2;
  static constexpr int kStages = HD == 128 ? 3 : 6;        // 96 KB of loads in flight per CTA
  static constexpr int kBarBytes = 256;
  static constexpr int kRowBytes = NB * 16;
  static constexpr int kTmem = NB == 16 ? 32 : 64;         // two accumulators
  static constexpr int kSmemBytes = kStages * kKBytes + kQBytes + kRowBytes + kBarBytes + 1024;
};

// A = K tile, B = query rows, both K-major bf16, fp32 accumulate, M = 128, N = NB
__host__ __device__ constexpr uint32_t idesc_few(int nb) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(nb >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
}

template <int NB>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&acc)[NB]) {
  if constexpr (NB == 16) tmem_ld16(taddr, acc);
  else tmem_ld32(taddr, acc);
}

template <int HD, int NB, bool kAlibi>
__global__ void __launch_bounds__(kFewThreads, 2) paged_few_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                 const __grid_constant__ CUtensorMap map_k,
                                                                 const __grid_constant__ PagedArgs a, int unit0) {
  pdl_begin();
  using C = FewCfg<HD, NB>;
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunk = blockIdx.x % a.few_chunks, unit = blockIdx.x / a.few_chunks;
  const int kvh = unit % a.c.KH, b = unit0 + unit / a.c.KH;
  const PagedSeq s = paged_seq(a.c, b);
  if (s.n == 0) return;
  if (!paged_ok(a, s)) {
    if (chunk == 0) {
      if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
      write_unserved(a, s, kvh, threadIdx.x, kFewThreads);
    }
    return;
  }
  if (!paged_few(a, s)) return;
  // the sequence's tiles dealt evenly to as many of the unit's CTAs as get two at least
  const int len_tiles = (s.len + kTile - 1) / kTile;
  const int ctas = min(a.few_chunks, (len_tiles + 1) / 2);
  if (chunk >= ctas) return;
  const int tile0 = (int)((long long)len_tiles * chunk / ctas), tile1 = (int)((long long)len_tiles * (chunk + 1) / ctas);
  const int tiles = tile1 - tile0;
  const int rows = s.n * a.G;
  const int box_shift = min(a.c.ps_shift, 7);

  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t k_smem = sbase;
  const uint32_t q_smem = k_smem + C::kStages * C::kKBytes;
  const uint32_t row_par = q_smem + C::kQBytes;             // per row: a, a * slope, position (float), position (int)
  const uint32_t bars = row_par + C::kRowBytes;
  const uint32_t q_full = bars;
  const uint32_t kv_full = bars + 8;                        // [kStages]
  const uint32_t kv_empty = kv_full + 8 * C::kStages;       // [kStages]
  const uint32_t s_full = kv_empty + 8 * C::kStages;        // [2]
  const uint32_t s_empty = s_full + 16;                     // [2]
  const uint32_t tmem_slot = s_empty + 16;
  const uint32_t abort_flag = tmem_slot + 4;
  const uint32_t drain_bar = tmem_slot + 8;                 // teardown: every MMA issued so far has finished
  const uint32_t drain_fail = drain_bar + 8;                // uint32: a teardown wait ran out as well
  static_assert(8 * (1 + 2 * C::kStages + 4) + 8 + 16 <= C::kBarBytes, "barrier area");

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    for (int t = 0; t < C::kStages; ++t) {
      mbar_init(kv_full + 8 * t, 1);
      mbar_init(kv_empty + 8 * t, 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full + 8 * t, 1);
      mbar_init(s_empty + 8 * t, 4);
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
  if (warp == 2 && lane < NB) {
    float ra = 0.f, slope = 0.f;
    int pos = -1;                                            // (rows past the last one see nothing)
    if (lane < rows) {
      const int head = kvh * a.G + lane % a.G;
      pos = s.len - s.n + lane / a.G;
      ra = paged_scale(a, head, pos);
      if (kAlibi) slope = a.alibi[head] / a.sm_scale;        // bias in dot-product units
    }
    sts_f4(row_par + 16 * lane, ra, slope, (float)pos, __int_as_float(pos));
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = lds_u32(tmem_slot);

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer: a lane per page box
    if (elect_one()) {
      mbar_expect_tx(q_full, (uint32_t)(a.few_slots * 128 * C::kHalves));
      for (int hf = 0; hf < C::kHalves; ++hf)
        tma_load_4d(q_smem + hf * (NB * 128), &map_q, q_full, hf * 64, kvh * a.G, s.q0, 0);
    }
    __syncwarp();
    int stage = 0;
    uint32_t phase = 0;
    bool alive = true;
    const int boxes = kTile >> box_shift;                    // of a whole tile: a power of two, at most 8
    // 32 page numbers ahead, a lane each
    const int ahead = 32 / boxes;                            // tiles they cover
    int page = 0, slot = 0;
    for (int t = 0; t < tiles; ++t) {
      const int key0 = (tile0 + t) * kTile;
      if (t % ahead == 0) {
        const int key = key0 + (lane << box_shift);
        if (key < s.len) page_of_box(a.c, b, key, a.status, page, slot);
      }
      const int src = (t % ahead) * boxes + (lane & (boxes - 1));
      const int pg = __shfl_sync(0xffffffffu, page, src), sl = __shfl_sync(0xffffffffu, slot, src);
      alive = __all_sync(0xffffffffu, mbar_wait(kv_empty + 8 * stage, phase ^ 1u, abort_flag));
      if (!alive) break;
      const int need = boxes_needed(key0, kTile, s.len, box_shift);
      const uint32_t box_bytes = 128u << box_shift;
      if (lane == 0) mbar_expect_tx(kv_full + 8 * stage, (uint32_t)need * box_bytes * C::kHalves);
      __syncwarp();
      if (lane < need) {
#pragma unroll
        for (int hf = 0; hf < C::kHalves; ++hf)
          tma_load_4d(k_smem + stage * C::kKBytes + hf * (kTile * 128) + lane * box_bytes, &map_k, kv_full + 8 * stage, hf * 64, sl,
                      kvh, pg);
      }
      __syncwarp();
      if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
    }
    if (!alive && lane == 0) {
      // a wait ran out somewhere in the CTA: the copies this warp armed barriers for must land before shared
      // memory goes away (stages before `stage`: this round of the ring; the others: the previous round)
      bool ok = mbar_drain(q_full, 0u);
      for (int st = 0; st < C::kStages; ++st) ok &= mbar_drain(kv_full + 8 * st, st < stage ? phase : phase ^ 1u);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint32_t idesc = idesc_few(NB);
      const uint32_t k_lo = smem_desc_lo(k_smem), q_lo = smem_desc_lo(q_smem);
      int stage = 0, buf = 0;
      uint32_t phase = 0, sphase[2] = {0, 0};
      bool alive = mbar_wait(q_full, 0, abort_flag);
      for (int t = 0; t < tiles && alive; ++t) {
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
          umma_bf16(tmem_base + buf * NB, a_lo + a_off, q_lo + b_off, kDescHi, idesc, kk > 0 ? 1u : 0u);
        }
        umma_commit(s_full + 8 * buf);
        umma_commit(kv_empty + 8 * stage);
        buf ^= 1;
        if (++stage == C::kStages) { stage = 0; phase ^= 1u; }
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
    const size_t row0 = (size_t)unit * a.few_slots;
    const int pos0 = s.len - s.n;
    uint32_t sphase[2] = {0, 0};
    int buf = 0;
    bool alive = true;
    float bound[NB];                                         // (largest value so far) - 1, the same in every lane
#pragma unroll
    for (int r = 0; r < NB; ++r) bound[r] = -INFINITY;
    for (int t = 0; t < tiles && alive; ++t) {
      alive = __all_sync(0xffffffffu, mbar_wait(s_full + 8 * buf, sphase[buf], abort_flag));
      if (!alive) break;
      sphase[buf] ^= 1u;
      tc_fence_after();
      float acc[NB];
      load_columns<NB>(taddr + buf * NB, acc);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(s_empty + 8 * buf);
      buf ^= 1;
      const int group = (tile0 + t) * (kTile / 32) + quad;
      const int j = group * 32 + lane;
      if (group * 32 >= s.len) continue;                     // (groups nobody looks at)
      const bool edge = group * 32 + 31 > pos0;
      float mine = -INFINITY;
#pragma unroll
      for (int r = 0; r < NB; ++r) {
        if (r < rows) {
          float ra, slope, posf, posi;
          lds_f4(row_par + 16 * r, ra, slope, posf, posi);
          float y = kAlibi ? ra * fmaf(slope, (float)j - posf, acc[r]) : ra * acc[r];
          if (edge) y = j <= __float_as_int(posi) ? y : -INFINITY;
          float m = y;
          asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(m));
          if (m > bound[r]) a.scores[(row0 + r) * a.score_stride + j] = y;
          bound[r] = fmaxf(bound[r], m - 1.0f);
          if (lane == r) mine = m;
        }
      }
      if (lane < rows) a.group_max[(row0 + lane) * a.group_stride + group] = mine;
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
}

// =============================================================================================== many
constexpr int BM = 128;
constexpr int BN = 256;
constexpr int kManyConsumers = 4 * kManyTiles;
constexpr int kManyThreads = (2 + kManyConsumers) * 32;
constexpr int kSchedSlots = 2;
static_assert(kManyTiles * BN == 512, "TMEM budget");

template <int HD>
struct ManyCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kQBytes = BM * HD * 2;
  static constexpr int kKBytes = BN * HD * 2;
  static constexpr int kStages = HD == 128 ? 2 : 4;
  static constexpr int kBarBytes = 512;
  static constexpr int kSmemBytes = kManyTiles * kQBytes + kStages * kKBytes + kBarBytes + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory of one CTA");
};

__host__ __device__ constexpr uint32_t idesc_many() {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
}

// A work item: one block of new tokens, one K/V head, one share of the keys.  Published by the producer in eight words.
struct ManyItem {
  int b, kvh, q0, n, len, t0, lo, hi;      // t0: first token of the block within the chunk; K tiles lo .. hi - 1
  int unit;                                // row slots: unit * many_slots
};
constexpr int kItemWords = 9;

// K tiles that Q tile x of the item looks at: lo .. this - 1 (no more than lo: none)
__device__ __forceinline__ int many_tile_end(const PagedArgs& a, const ManyItem& it, int x) {
  const int first = it.t0 + x * a.tile_tokens;
  if (first >= it.n) return it.lo;
  const int last = min(first + a.tile_tokens, it.n) - 1;
  return max(min((it.len - it.n + last) / BN + 1, it.hi), it.lo);
}

template <int HD, bool kAlibi>
__global__ void __launch_bounds__(kManyThreads, 1) paged_many_kernel(const __grid_constant__ CUtensorMap map_q,
                                                                   const __grid_constant__ CUtensorMap map_k,
                                                                   const __grid_constant__ PagedArgs a, int block0, int blocks) {
  pdl_begin();
  using C = ManyCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = sbase;                                   // [kManyTiles][kHalves][BM rows x 128 B]
  const uint32_t k_smem = sbase + kManyTiles * C::kQBytes;         // [kStages][kHalves][BN rows x 128 B]
  const uint32_t bars = k_smem + C::kStages * C::kKBytes;
  const uint32_t q_full = bars;                                    // [kManyTiles]
  const uint32_t q_empty = q_full + 8 * kManyTiles;                // [kManyTiles]
  const uint32_t s_full = q_empty + 8 * kManyTiles;                // [kManyTiles]
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
  static_assert((4 * kManyTiles + 2 * C::kStages + 2 * kSchedSlots) * 8 + 4 * kSchedSlots * kItemWords + 8 + 16 <= C::kBarBytes,
                "barrier area");
  static_assert((4 * kSchedSlots * kItemWords) % 8 == 0, "drain_bar is 8-byte aligned");

  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const int box_shift = min(a.c.ps_shift, 7);

  if (threadIdx.x == 0) {
    for (int t = 0; t < kManyTiles; ++t) {
      mbar_init(q_full + 8 * t, 1);
      mbar_init(q_empty + 8 * t, 1);
      mbar_init(s_full + 8 * t, 1);
      mbar_init(s_empty + 8 * t, 4);
    }
    for (int t = 0; t < C::kStages; ++t) {
      mbar_init(k_full + 8 * t, 1);
      mbar_init(k_empty + 8 * t, 1);
    }
    for (int t = 0; t < kSchedSlots; ++t) {
      mbar_init(w_full + 8 * t, 1);
      mbar_init(w_empty + 8 * t, 1 + kManyConsumers);              // MMA issuer + consumer warps
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
    return it;
  };

  if (warp == 0) {
    // ------------------------------------------------------------- scheduler + TMA producer (the whole warp)
    int stage = 0, slot = 0;
    uint32_t kphase = 0, qphase = 0 /* bit x: phase of Q tile slot x */, wphase = 0;
    bool alive = true;
    auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
    };
    const int block_tokens = kManyTiles * a.tile_tokens;
    const int n_items = blocks * a.c.KH * a.many_splits;
    while (alive) {
      int k = 0;
      if (lane == 0) k = atomicAdd(a.counter, 1);
      k = __shfl_sync(0xffffffffu, k, 0);
      ManyItem it;
      it.b = -1;
      if (k < n_items) {
        // a K/V head's blocks one after another, later blocks (longer rows) first: the CTAs that run together stream the same keys
        const int split = k % a.many_splits, u = k / a.many_splits;
        it.kvh = u / blocks;
        const int blk = block0 + blocks - 1 - (u - it.kvh * blocks);
        if (a.c.cu_q) {
          it.b = find_seq(a.c, blk, block_tokens, 1);
          it.t0 = (blk - (clamped_cu(a.c, it.b) / block_tokens + it.b)) * block_tokens;
        } else {
          const int per = (a.c.T / a.c.B + block_tokens - 1) / block_tokens;
          it.b = blk / per;
          it.t0 = (blk - it.b * per) * block_tokens;
        }
        if (it.b >= a.c.B) continue;
        const PagedSeq s = paged_seq(a.c, it.b);
        it.q0 = s.q0; it.n = s.n; it.len = s.len;
        if (it.t0 < 0 || it.t0 >= s.n) continue;
        if (!paged_ok(a, s)) {
          if (split == 0 && it.t0 == 0) {
            if (lane == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
            write_unserved(a, s, it.kvh, lane, 32);
          }
          continue;
        }
        if (paged_few(a, s)) continue;
        it.unit = (blk - block0) * a.c.KH + it.kvh;
        const int last = min(it.t0 + block_tokens, s.n) - 1;
        const int tiles = (s.len - s.n + last) / BN + 1;
        it.lo = (int)((long long)tiles * split / a.many_splits);
        it.hi = (int)((long long)tiles * (split + 1) / a.many_splits);
        if (it.lo >= it.hi) continue;
      }
      alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
      if (!alive) break;
      if (lane == 0) {
        const uint32_t at = w_item + 4u * kItemWords * slot;
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
        }
        mbar_arrive(w_full + 8 * slot);
      }
      __syncwarp();
      if (++slot == kSchedSlots) { slot = 0; wphase ^= 1u; }
      if (it.b < 0) break;
      const int boxes = BN >> box_shift;                    // of a whole tile: a power of two, at most 16
      const int ahead = 32 / boxes;
      int page = 0, pslot = 0;
      int end = it.lo;
      for (int x = 0; x < kManyTiles; ++x) end = max(end, many_tile_end(a, it, x));
      for (int t = it.lo; t < end && alive; ++t) {
        const int key0 = t * BN;
        if ((t - it.lo) % ahead == 0) {
          const int key = key0 + (lane << box_shift);
          if (key < it.len) page_of_box(a.c, it.b, key, a.status, page, pslot);
        }
        const int src = ((t - it.lo) % ahead) * boxes + (lane & (boxes - 1));
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
        if (t == it.lo) {
          for (int x = 0; x < kManyTiles && alive; ++x) {
            if (many_tile_end(a, it, x) <= it.lo) continue;
            alive = wait_all(q_empty + 8 * x, ((qphase >> x) & 1u) ^ 1u);
            if (!alive) break;
            qphase ^= 1u << x;
            if (elect_one()) {
              mbar_expect_tx(q_full + 8 * x, (uint32_t)(a.tile_tokens * a.G * 128 * C::kHalves));
              for (int hf = 0; hf < C::kHalves; ++hf)
                tma_load_4d(q_smem + x * C::kQBytes + hf * (BM * 128), &map_q, q_full + 8 * x, hf * 64, it.kvh * a.G,
                            it.q0 + it.t0 + x * a.tile_tokens, 0);
            }
            __syncwarp();
          }
        }
      }
    }
    if (!alive && lane == 0) {
      // a wait ran out somewhere in the CTA: every copy this warp armed a barrier for must have landed before
      // shared memory goes away.  Stages before `stage` were armed in this round of the ring, the others in the
      // previous one (a barrier that was never armed reports its "previous" phase as complete at once).
      bool ok = true;
      for (int st = 0; st < C::kStages; ++st) ok &= mbar_drain(k_full + 8 * st, st < stage ? kphase : kphase ^ 1u);
      for (int x = 0; x < kManyTiles; ++x) ok &= mbar_drain(q_full + 8 * x, ((qphase >> x) & 1u) ^ 1u);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (warp-wide control flow, one elected lane issues)
    constexpr uint32_t idesc = idesc_many();
    const uint64_t hi = (uint64_t)kDescHi << 32;
    const uint64_t q_desc = hi | smem_desc_lo(q_smem), k_desc = hi | smem_desc_lo(k_smem);
    int stage = 0, slot = 0;
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
      int tx[kManyTiles], end = lo;
      for (int x = 0; x < kManyTiles; ++x) {
        tx[x] = __shfl_sync(0xffffffffu, many_tile_end(a, it, x), 0);
        end = max(end, tx[x]);
      }
      for (int t = lo; t < end && alive; ++t) {
        alive = wait_all(k_full + 8 * stage, kphase);
        if (!alive) break;
        const uint64_t b_desc = k_desc + (uint64_t)(stage * (C::kKBytes >> 4));
#pragma unroll
        for (int x = 0; x < kManyTiles; ++x) {
          if (t >= tx[x] || !alive) continue;
          if (t == lo) {
            alive = wait_all(q_full + 8 * x, (qphase >> x) & 1u);
            qphase ^= 1u << x;
          }
          if (alive) alive = wait_all(s_empty + 8 * x, sphase[x] ^ 1u);
          if (!alive) continue;
          sphase[x] ^= 1u;
          tc_fence_after();
          const uint64_t a_desc = q_desc + (uint64_t)(x * (C::kQBytes >> 4));
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < HD / 16; ++kk) {
              const uint32_t a_off = (kk >> 2) * ((BM * 128) >> 4) + (kk & 3) * 2;
              const uint32_t b_off = (kk >> 2) * ((BN * 128) >> 4) + (kk & 3) * 2;
              umma_bf16_desc(tmem_base + x * BN, a_desc + a_off, b_desc + b_off, idesc, kk > 0 ? 1u : 0u);
            }
            umma_commit(s_full + 8 * x);
            if (t == tx[x] - 1) umma_commit(q_empty + 8 * x);
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
  } else {
    // -------------------------------------------------- consumers: one thread per query row
    const int x = (warp - 2) >> 2;
    const int quad = warp & 3;
    const int row_local = quad * 32 + lane;
    const uint32_t taddr_row = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(x * BN);
    const uint32_t my_full = s_full + 8 * x, my_empty = s_empty + 8 * x;
    const int tile_rows = a.tile_tokens * a.G;
    uint32_t fphase = 0, wphase = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = __all_sync(0xffffffffu, mbar_wait(w_full + 8 * slot, wphase, abort_flag));
      if (!alive) break;
      const ManyItem it = read_item(slot);
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
      const int first_pos = it.len - it.n + it.t0 + x * a.tile_tokens;
      const float ra = valid ? paged_scale(a, head, pos) : 0.f;
      const float slope = kAlibi && valid ? a.alibi[head] / a.sm_scale : 0.f;
      const size_t row = (size_t)it.unit * a.many_slots + (size_t)(valid ? x * tile_rows + row_local : 0);
      float* score_row = a.scores + row * a.score_stride;
      float* max_row = a.group_max + row * a.group_stride;
      float bound = valid ? -INFINITY : INFINITY;              // (largest value so far) - 1
      for (int t = it.lo; t < end && alive; ++t) {
        alive = __all_sync(0xffffffffu, mbar_wait(my_full, fphase, abort_flag));
        if (!alive) break;
        fphase ^= 1u;
        tc_fence_after();
        const int col_base = t * BN;
        const bool edge = col_base + BN - 1 > first_pos;       // some row of the tile does not see all of it
        // y of 32 columns as every use of them computes it
        auto finish = [&](float (&v)[32], int col0) {
          if (kAlibi) {
            const float t0 = (float)(col0 - pos);
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u] = ra * fmaf(slope, t0 + (float)u, v[u]);
          } else {
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u] *= ra;
          }
          if (edge) {
#pragma unroll
            for (int u = 0; u < 32; ++u) v[u] = col0 + u <= lim ? v[u] : -INFINITY;
          }
        };
        float gm[BN / 32], best = -INFINITY;
#pragma unroll
        for (int g = 0; g < BN / 32; ++g) {
          float v[32];
          tmem_ld32(taddr_row + 32 * g, v);
          tmem_ld_wait();
          finish(v, col_base + 32 * g);
          gm[g] = fmaxf(fmaxf(max8(&v[0]), max8(&v[8])), fmaxf(max8(&v[16]), max8(&v[24])));
          best = fmaxf(best, gm[g]);
        }
        bound = fmaxf(bound, best - 1.0f);
        unsigned hit = 0u;
#pragma unroll
        for (int g = 0; g < BN / 32; ++g) hit |= gm[g] > bound ? 1u << g : 0u;
        unsigned any = __reduce_or_sync(0xffffffffu, hit);
        while (any) {
          const int g = __ffs(any) - 1;
          any &= any - 1;
          float v[32];
          tmem_ld32(taddr_row + 32 * g, v);
          tmem_ld_wait();
          finish(v, col_base + 32 * g);
          if ((hit >> g) & 1u) {
            float4* dst = reinterpret_cast<float4*>(score_row + col_base + 32 * g);
#pragma unroll
            for (int u = 0; u < 8; ++u) dst[u] = make_float4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
          }
        }
        // the accumulator has been read: hand it back to the MMA issuer
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(my_empty);
        if (valid) {
          float4* dst = reinterpret_cast<float4*>(max_row + t * (BN / 32));
          dst[0] = make_float4(gm[0], gm[1], gm[2], gm[3]);
          dst[1] = make_float4(gm[4], gm[5], gm[6], gm[7]);
        }
      }
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

template <int HD, int NB, bool kAlibi>
cudaError_t launch_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int unit0, int units,
                       cudaStream_t stream) {
  CUtensorMap map_q, map_k;
  cudaError_t err = map_queries(&map_q, a, q, q_st, q_sh, a.few_slots / a.G);
  if (err == cudaSuccess) err = map_pages(&map_k, a, k);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(paged_few_kernel<HD, NB, kAlibi>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<HD, NB>::kSmemBytes);
  if (err != cudaSuccess) return err;
  return launch_kernel(paged_few_kernel<HD, NB, kAlibi>, (unsigned)((long long)units * a.c.KH * a.few_chunks), kFewThreads, FewCfg<HD, NB>::kSmemBytes,
                       stream, map_q, map_k, a, unit0);
}

template <int HD, bool kAlibi>
cudaError_t launch_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int block0, int blocks,
                        cudaStream_t stream) {
  CUtensorMap map_q, map_k;
  cudaError_t err = map_queries(&map_q, a, q, q_st, q_sh, a.tile_tokens);
  if (err == cudaSuccess) err = map_pages(&map_k, a, k);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(paged_many_kernel<HD, kAlibi>, cudaFuncAttributeMaxDynamicSharedMemorySize, ManyCfg<HD>::kSmemBytes);
  int dev = 0, sms = 0;
  if (err == cudaSuccess) err = cudaGetDevice(&dev);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (err == cudaSuccess) err = cudaMemsetAsync(a.counter, 0, sizeof(int32_t), stream);
  if (err != cudaSuccess) return err;
  const long long items = (long long)blocks * a.c.KH * a.many_splits;
  return launch_kernel(paged_many_kernel<HD, kAlibi>, (unsigned)(items < sms ? items : sms), kManyThreads, ManyCfg<HD>::kSmemBytes, stream, map_q, map_k,
                       a, block0, blocks);
}

}  // namespace

cudaError_t launch_paged_few(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int unit0, int units,
                             cudaStream_t stream) {
#define ENTMAX_FEW(HD, NB)                                                              \
  (a.alibi ? launch_few<HD, NB, true>(a, q, k, q_st, q_sh, unit0, units, stream)        \
           : launch_few<HD, NB, false>(a, q, k, q_st, q_sh, unit0, units, stream))
  if (a.c.D == 64) return a.few_rows <= 16 ? ENTMAX_FEW(64, 16) : ENTMAX_FEW(64, 32);
  return a.few_rows <= 16 ? ENTMAX_FEW(128, 16) : ENTMAX_FEW(128, 32);
#undef ENTMAX_FEW
}

cudaError_t launch_paged_many(const PagedArgs& a, const void* q, const void* k, int64_t q_st, int64_t q_sh, int block0, int blocks,
                              cudaStream_t stream) {
  if (a.c.D == 64)
    return a.alibi ? launch_many<64, true>(a, q, k, q_st, q_sh, block0, blocks, stream)
                   : launch_many<64, false>(a, q, k, q_st, q_sh, block0, blocks, stream);
  return a.alibi ? launch_many<128, true>(a, q, k, q_st, q_sh, block0, blocks, stream)
                 : launch_many<128, false>(a, q, k, q_st, q_sh, block0, blocks, stream);
}

}  // namespace entmax
