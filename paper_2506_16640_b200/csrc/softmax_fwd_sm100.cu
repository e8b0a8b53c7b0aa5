// Softmax attention on sm_100a, forward: whole sequences ([B, H, N, D] tensors) and chunks of new tokens over a paged cache, one kernel.
//
// A work item is two Q tiles of 128 rows that share a K/V head -- two query heads of a group at the same rows where the group is even, two neighbouring
// tiles of one head otherwise -- so that every K/V tile in shared memory is used twice.  K/V tiles come last to first (with slopes the largest
// scores first).  Per Q tile and K/V tile of 128 keys
//   S = Q K^T        both operands in shared memory, S in TMEM;
//   P = exp2(a x - a m)   a thread per row: its 128 scores in registers, running maximum m, running sum l of the float32 probabilities;
//                         P as bf16 over S's own columns (off by 2^-8 of a probability at most: what the product's input type holds);
//   O += P V         P from TMEM, V with the head dim contiguous, O in TMEM.
// O is not rescaled for every rise of the maximum: P may grow up to 2^8 above the m it is measured from before O and l are brought to a new one, exactly, so
// that nothing is lost and the correction is rare.  While one tile's softmax runs the tensor core works on the other's O and next S.
// Bound by the chain of one tile -- S from TMEM, maximum, 128 exponentials a thread (16384 a tile, 1024 cycles of the special-function unit), P to TMEM, then O and
// the next S behind the other tile's -- of which two are under way.  Computing a part of the exponentials on the FMA pipe made it longer.
// 16 heads x 16384 x 128 causal: 850 us, 1.29 PFLOP/s, 80 % of the measured rate of library products; 4 x 16 x 8192 x 64: 800 us; 8 x 12 x 1024 x 64, where starts and
// ends of items count: 34 us (36 with a learned scale).  A cap makes the chain longer: 16 x 8192 x 128 causal 241 us, 376 with one.
// CTA: warps 0..3 and 4..7 the rows of the two tiles, warp 8 MMA issuer, warp 9 TMA producer and scheduler (10, 11: idle, registers go by warpgroups).  Items are handed out by the hardware: a
// running CTA takes over one that has not started (longest rows of a head first).  Every wait is bounded (see sm100_ptx.cuh).
#include <cuda.h>

#include "sm100_ptx.cuh"
#include "softmax_paged.cuh"
#include "softmax_tile.cuh"

namespace entmax {

namespace {

using namespace sm100;

constexpr int kRows = 128, kKeys = 128;
constexpr int kFwdThreads = 384;
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;
static_assert(2 * kSoftmaxRegs + kOtherRegs <= 3 * 168, "no more than the launch's, 168 a thread");
constexpr int kBarArea = 512;

template <int HD>
struct FwdCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kTileBytes = kKeys * HD * 2;
  static constexpr int kStages = HD == 128 ? 4 : 8;                  // K and V tiles in turn
  static constexpr int kSmemBytes = 2 * kTileBytes + kStages * kTileBytes + kBarArea + 1024;
  static_assert(kSmemBytes <= 232448, "shared memory of one CTA");
  static constexpr int kTmemO = 256;
};

// What the scheduler says about an item, in shared memory
struct Work {
  int valid;            // 0: nothing left
  int b, kh;
  int h[2], row0[2];    // head and first row (paged: new token of the sequence) of the two tiles
  int lo[2], hi[2];     // their K/V tiles, lo >= hi: none
  int q0, n, len;       // paged: first row of q, new tokens, length
  int part;             // paged, shared out: where its results go (tile t: part + t), -1: it has all keys
  int first_key;        // paged: no row sees a key before it
};
static_assert(sizeof(Work) == 64, "two of them behind the barriers");

struct FwdArgs {
  SoftmaxArgs a;
  int tiles;            // Q tiles (or pairs of tiles) per head
  int pairs;            // pairs of heads in a group (pair_heads), 1 otherwise
  int pair_heads;
  __nv_bfloat16* o;
  float* lse;
  int32_t* status;
  // paged
  PagedCache c;
  int window, max_q, max_kv, few_rows, shares, box_shift;
  const __nv_bfloat16* v;
  float* part_o;        // [part][128][HD]
  float2* part_ml;      // [part][128] {maximum in base-2 units, sum}
};

__host__ __device__ constexpr uint32_t fwd_idesc_s() {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kKeys >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
}
// A from TMEM, B with N contiguous
template <int HD>
__host__ __device__ constexpr uint32_t fwd_idesc_o() {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
}

// The K/V tiles that the 128 rows from row0 on see, by the whole warp
__device__ __forceinline__ int2 tile_span(const SoftmaxArgs& a, int b, int row0) {
  const int lane = threadIdx.x & 31;
  int lo = 0x7fffffff, hi = 0;
  if (row0 < a.N) {
    if (!a.ranges) {
      lo = 0;
      hi = a.causal ? min(row0 + kRows, a.N) : a.N;
    } else {
      int2 range[kRows / 32];                    // (rows behind the last: the last once more)
#pragma unroll
      for (int t = 0; t < kRows / 32; ++t) range[t] = a.ranges[(size_t)b * a.N + min(row0 + t * 32 + lane, a.N - 1)];
#pragma unroll
      for (int t = 0; t < kRows / 32; ++t) {
        const int2 s = seen_of(a, range[t], min(row0 + t * 32 + lane, a.N - 1));
        if (s.y > s.x) { lo = min(lo, s.x); hi = max(hi, s.y); }
      }
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
    }
  }
  return hi > lo ? make_int2(lo / kKeys, (hi + kKeys - 1) / kKeys) : make_int2(0, 0);
}

// Paged: the sequence of a block id, by the whole warp (see block_start)
__device__ __forceinline__ int find_block(const PagedCache& c, int id, int block) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = c.B;
  while (n > 1) {
    const int step = (n + 31) / 32;
    const bool le = lane * step < n && (lane == 0 || block_start(c, lo + lane * step, block) <= id);
    const int k = 31 - __clz(__ballot_sync(0xffffffffu, le));
    lo += k * step;
    n = min(step, n - k * step);
  }
  return lo;
}

template <int HD, bool PAGED, bool CAP, bool TERMS>
__global__ void __launch_bounds__(kFwdThreads, 1) softmax_fwd_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ FwdArgs f) {
  pdl_begin();
  using C = FwdCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = sbase, kv_smem = sbase + 2 * C::kTileBytes;
  const uint32_t bars = kv_smem + C::kStages * C::kTileBytes;
  const uint32_t work_at = bars;                                     // Work [2]
  const uint32_t answer = bars + 128;                                // 16 bytes
  const uint32_t q_full = bars + 144, q_empty = bars + 160;          // [2] each
  const uint32_t s_full = bars + 176, p_full = bars + 192;
  const uint32_t o_full = bars + 208, o_empty = bars + 224;
  const uint32_t w_full = bars + 240, w_empty = bars + 256;
  const uint32_t next_bar = bars + 272, drain_bar = bars + 280;
  const uint32_t tmem_slot = bars + 288, abort_flag = bars + 292, drain_fail = bars + 296;
  const uint32_t p_half = bars + 304;                                // [2]
  const uint32_t kv_full = bars + 320, kv_empty = bars + 320 + 8 * C::kStages;
  static_assert(320 + 16 * C::kStages <= kBarArea, "barriers");
  const Work* work = reinterpret_cast<const Work*>(smem_raw + (work_at - smem_u32(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full + 8 * t, 1);
      mbar_init(q_empty + 8 * t, 1);
      mbar_init(s_full + 8 * t, 1);
      mbar_init(p_half + 8 * t, 4);
      mbar_init(p_full + 8 * t, 4);
      mbar_init(o_full + 8 * t, 1);
      mbar_init(o_empty + 8 * t, 4);
      mbar_init(w_full + 8 * t, 1);
      mbar_init(w_empty + 8 * t, 9);
    }
    for (int st = 0; st < C::kStages; ++st) {
      mbar_init(kv_full + 8 * st, 1);
      mbar_init(kv_empty + 8 * st, 1);
    }
    mbar_init(next_bar, 1);
    mbar_init(drain_bar, 1);
    sts_u32(abort_flag, 0u);
    sts_u32(drain_fail, 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 8) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(lds_u32(tmem_slot));
  const SoftmaxArgs& a = f.a;
  auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };

  if (warp >= 8) {
  registers_down<kOtherRegs>();
  if (warp == 9) {
    // ------------------------------------------------------------------ scheduler and TMA producer (the whole warp runs the control flow)
    uint32_t next_phase = 0, wphase = 0, qphase[2] = {0, 0}, idx = 0;   // idx: K and V tiles loaded so far
    int slot = 0;
    bool alive = true, asked = false;
    int item = (int)blockIdx.x;
    while (alive) {
      Work w;
      w.valid = item >= 0;
      w.part = -1;
      if (item >= 0) {
        int rest = item;
        if constexpr (!PAGED) {
          // causal: the longest rows of all heads first, with ranges the same order; without a mask a head after the other, whose K/V tiles then stay in L2
          int tile;
          if (a.causal || a.ranges) {
            const int heads = a.B * a.KH * f.pairs;
            tile = f.tiles - 1 - rest / heads;
            rest %= heads;
          }
          const int pair = rest % f.pairs;
          rest /= f.pairs;
          if (!(a.causal || a.ranges)) {
            tile = f.tiles - 1 - rest % f.tiles;
            rest /= f.tiles;
          }
          w.b = rest / a.KH;
          w.kh = rest - w.b * a.KH;
          w.h[0] = w.kh * a.G + (f.pair_heads ? 2 * pair : pair);
          w.h[1] = f.pair_heads ? w.h[0] + 1 : w.h[0];
          w.row0[0] = f.pair_heads ? tile * kRows : tile * 2 * kRows;
          w.row0[1] = f.pair_heads ? w.row0[0] : w.row0[0] + kRows;
          const int2 s0 = tile_span(a, w.b, w.row0[0]);
          const int2 s1 = f.pair_heads ? s0 : tile_span(a, w.b, w.row0[1]);
          w.lo[0] = s0.x; w.hi[0] = s0.y; w.lo[1] = s1.x; w.hi[1] = s1.y;
          w.q0 = 0; w.n = a.N; w.len = a.N; w.first_key = 0;
        } else {
          const int share = rest % f.shares;
          rest /= f.shares;
          const int unit = rest;                                      // (block, K/V head, pair of heads)
          const int pair = rest % f.pairs;
          rest /= f.pairs;
          w.kh = rest % a.KH;
          const int id = rest / a.KH;
          const int block = f.pair_heads ? kRows : 2 * kRows;
          w.b = find_block(f.c, id, block);
          const PagedSeq s = paged_seq(f.c, w.b);
          w.q0 = s.q0; w.n = s.n; w.len = s.len;
          w.h[0] = w.kh * a.G + (f.pair_heads ? 2 * pair : pair);
          w.h[1] = f.pair_heads ? w.h[0] + 1 : w.h[0];
          w.row0[0] = (id - block_start(f.c, w.b, block)) * block;
          w.row0[1] = f.pair_heads ? w.row0[0] : w.row0[0] + kRows;
          w.part = f.shares > 1 ? 2 * (unit * f.shares + share) : -1;
          const bool ok = s.len >= s.n && s.len <= f.max_kv && s.n <= f.max_q && (long long)s.n * a.G > f.few_rows && w.row0[0] < s.n && w.row0[0] >= 0;
          int most = 0, least = 0x7fffffff;
          w.first_key = 0;
          for (int t = 0; t < 2; ++t) {
            w.lo[t] = w.hi[t] = 0;
            if (!ok || w.row0[t] >= s.n) continue;
            const int pos0 = s.len - s.n + w.row0[t];
            const int first = f.window > 0 ? max(0, pos0 - f.window + 1) : 0;
            if (t == 0) w.first_key = first;
            w.lo[t] = first / kKeys;
            w.hi[t] = (min(pos0 + kRows, s.len) + kKeys - 1) / kKeys;
            least = min(least, w.lo[t]);
            most = max(most, w.hi[t]);
          }
          if (f.shares > 1 && most > least) {
            const int all = most - least;
            const int from = least + (int)((long long)all * share / f.shares), to = least + (int)((long long)all * (share + 1) / f.shares);
            for (int t = 0; t < 2; ++t) {
              const bool rows = w.hi[t] > w.lo[t];
              w.lo[t] = max(w.lo[t], from);
              w.hi[t] = rows ? min(w.hi[t], to) : 0;
            }
          }
          if (!ok) w.valid = 2;                                       // nothing of it is this kernel's
        }
      }
      if (w.valid != 2) {
        alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
        if (!alive) break;
        if (lane == 0) {
          *const_cast<Work*>(work + slot) = w;
          mbar_arrive(w_full + 8 * slot);
        }
        __syncwarp();
        if (++slot == 2) { slot = 0; wphase ^= 1u; }
      }
      if (item < 0) break;
      int lo = 0x7fffffff, hi = 0;
      if (w.valid == 1) {
        for (int t = 0; t < 2; ++t)
          if (w.hi[t] > w.lo[t]) { lo = min(lo, w.lo[t]); hi = max(hi, w.hi[t]); }
      }
      if (hi > lo) {
        for (int t = 0; t < 2 && alive; ++t) {
          if (w.hi[t] <= w.lo[t]) continue;
          alive = wait_all(q_empty + 8 * t, qphase[t] ^ 1u);
          if (!alive) break;
          qphase[t] ^= 1u;
          if (elect_one()) {
            mbar_expect_tx(q_full + 8 * t, C::kTileBytes);
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(q_smem + t * C::kTileBytes + hf * (kRows * 128), &map_q, q_full + 8 * t, hf * 64, PAGED ? w.q0 + w.row0[t] : w.row0[t],
                          w.h[t], PAGED ? 0 : w.b);
          }
          __syncwarp();
        }
        // paged: lane x looks after box x of a tile, one tile ahead
        int page = 0, page_next = 0;
        auto look_up = [&](int j) -> int {
          const int key = j * kKeys + (lane << f.box_shift);
          if (j < lo || lane >= (kKeys >> f.box_shift) || key >= w.len || key + (1 << f.box_shift) <= w.first_key) return -2;
          int p = f.c.table[(long long)w.b * f.c.table_stride + (key >> f.c.ps_shift)];
          if ((unsigned)p >= (unsigned)f.c.n_pages) {                 // (read as zeros)
            if (f.status) atomicOr(f.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_PAGE);
            p = f.c.n_pages;
          }
          return p;
        };
        if constexpr (PAGED) page_next = look_up(hi - 1);
        for (int j = hi - 1; j >= lo && alive; --j) {
          if constexpr (PAGED) {
            page = page_next;
            page_next = look_up(j - 1);
          }
          for (int which = 0; which < 2; ++which, ++idx) {
            const int st = idx % C::kStages;
            const uint32_t round = idx / C::kStages;
            alive = wait_all(kv_empty + 8 * st, (round & 1u) ^ 1u);
            if (!alive) break;
            const uint32_t dst = kv_smem + st * C::kTileBytes;
            const CUtensorMap* map = which ? &map_v : &map_k;
            if constexpr (!PAGED) {
              if (elect_one()) {
                mbar_expect_tx(kv_full + 8 * st, C::kTileBytes);
                for (int hf = 0; hf < C::kHalves; ++hf)
                  tma_load_4d(dst + hf * (kKeys * 128), map, kv_full + 8 * st, hf * 64, j * kKeys, w.kh, w.b);
              }
            } else if (which == 1 && (j * kKeys + kKeys > w.len || j * kKeys < w.first_key)) {
              // Slots that no row sees may hold anything, and a NaN times a probability of 0 is one too.  A V tile that has some is put together by this
              // warp, with zeros for them (and not by clearing rows behind a TMA copy: such stores were seen to lose against the copy's own).
              for (int r = lane; r < kKeys; r += 32) {
                const int key = j * kKeys + r;
                const int p = __shfl_sync(0xffffffffu, page, r >> f.box_shift);
                const bool some = p >= 0 && p < f.c.n_pages && key < w.len && key >= w.first_key;
                const uint4* src = reinterpret_cast<const uint4*>(f.v + (some ? (long long)p * f.c.s_page + (long long)(key & ((1 << f.c.ps_shift) - 1)) * f.c.s_tok +
                                                                                      (long long)w.kh * f.c.s_head
                                                                              : 0));
                uint4 x[HD / 8];
#pragma unroll
                for (int e = 0; e < HD / 8; ++e) x[e] = some ? src[e] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int e = 0; e < HD / 8; ++e)
                  asm volatile("st.shared::cta.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (e >> 3) * (kKeys * 128) + r * 128 + (((e & 7) ^ (r & 7)) << 4)),
                               "r"(x[e].x), "r"(x[e].y), "r"(x[e].z), "r"(x[e].w)
                               : "memory");
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(kv_full + 8 * st);
            } else {
              const int boxes = __popc(__ballot_sync(0xffffffffu, page >= 0));
              if (lane == 0) mbar_expect_tx(kv_full + 8 * st, boxes * (C::kHalves * 128) << f.box_shift);
              __syncwarp();
              if (page >= 0) {
                const int slot0 = (j * kKeys + (lane << f.box_shift)) & ((1 << f.c.ps_shift) - 1);
                for (int hf = 0; hf < C::kHalves; ++hf)
                  tma_load_4d(dst + hf * (kKeys * 128) + (lane << (f.box_shift + 7)), map, kv_full + 8 * st, hf * 64, slot0, w.kh, page);
              }
            }
            __syncwarp();
          }
        }
        if (!alive) break;
      }
      // (asked for behind the item's last copy: asked for earlier, an item would wait for a CTA that is busy while others have run out)
      asked = true;
      if (elect_one()) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the last answer has been read
        mbar_expect_tx(next_bar, 16);
        next_cta_request(answer, next_bar);
      }
      __syncwarp();
      alive = wait_all(next_bar, next_phase);
      if (!alive) break;
      next_phase ^= 1u;
      asked = false;
      item = next_cta_answer(answer);
      __syncwarp();
    }
    if (!alive && lane == 0) {
      bool ok = true;
      for (int t = 0; t < 2; ++t) ok &= mbar_drain(q_full + 8 * t, qphase[t] ^ 1u);
      for (int st = 0; st < C::kStages; ++st) {
        const uint32_t armed = idx / C::kStages + ((uint32_t)st < idx % C::kStages ? 1u : 0u);   // times its barrier has been armed
        ok &= mbar_drain(kv_full + 8 * st, (armed & 1u) ^ 1u);
      }
      if (asked) ok &= mbar_drain(next_bar, next_phase);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 8) {
    // ------------------------------------------------------------------ MMA issuer
    constexpr uint32_t id_s = fwd_idesc_s();
    constexpr uint32_t id_o = fwd_idesc_o<HD>();
    const uint64_t dhi = (uint64_t)kDescHi << 32;
    const uint64_t q_d = dhi | smem_desc_lo(q_smem), k_d = dhi | smem_desc_lo(kv_smem), v_d = dhi | mn_desc_lo(kv_smem);
    constexpr uint32_t kStageD = C::kTileBytes >> 4;
    uint32_t wphase = 0, qphase[2] = {0, 0}, pphase[2] = {0, 0}, ophase[2] = {0, 0}, idx = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      Work w;
      w.valid = uniform(work[slot].valid);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        w.lo[t] = uniform(work[slot].lo[t]);
        w.hi[t] = uniform(work[slot].hi[t]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!w.valid) break;
      int lo = 0x7fffffff, hi = 0;
      for (int t = 0; t < 2; ++t)
        if (w.hi[t] > w.lo[t]) { lo = min(lo, w.lo[t]); hi = max(hi, w.hi[t]); }
      if (hi <= lo) continue;
      auto active = [&](int t, int j) { return j >= w.lo[t] && j < w.hi[t]; };
      auto wait_kv = [&](uint32_t i) { return wait_all(kv_full + 8 * (i % C::kStages), (i / C::kStages) & 1u); };
      auto issue_s = [&](int t, int j, uint32_t i) -> bool {
        if (j == w.hi[t] - 1) {
          if (!wait_all(q_full + 8 * t, qphase[t])) return false;
          qphase[t] ^= 1u;
        }
        tc_fence_after();
        if (elect_one()) {
          const uint64_t qt = q_d + t * kStageD, ks = k_d + (i % C::kStages) * kStageD;
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk >> 2) * ((kRows * 128) >> 4) + (kk & 3) * 2;
            umma_bf16_desc(tmem + t * kKeys, qt + off, ks + off, id_s, kk > 0 ? 1u : 0u);
          }
          umma_commit(s_full + 8 * t);
          if (j == w.lo[t]) umma_commit(q_empty + 8 * t);
        }
        __syncwarp();
        return true;
      };
      alive = wait_kv(idx);
      for (int t = 0; t < 2 && alive; ++t)
        if (active(t, hi - 1)) alive = issue_s(t, hi - 1, idx);
      if (!alive) break;
      if (elect_one()) umma_commit(kv_empty + 8 * (idx % C::kStages));
      __syncwarp();
      for (int j = hi - 1; j >= lo && alive; --j, idx += 2) {
        const uint32_t iv = idx + 1, ik = idx + 2;                    // V of this step, K of the next
        alive = wait_kv(iv);
        if (!alive) break;
        if (j > lo) {
          alive = wait_kv(ik);
          if (!alive) break;
        }
        for (int t = 0; t < 2 && alive; ++t) {
          if (active(t, j)) {
            alive = wait_all(p_half + 8 * t, pphase[t]);
            if (!alive) break;
            if (j == w.hi[t] - 1) {
              // the previous item's O has been read
              alive = wait_all(o_empty + 8 * t, ophase[t] ^ 1u);
              if (!alive) break;
              ophase[t] ^= 1u;
            }
            auto add_half = [&](int half) {
              tc_fence_after();
              if (elect_one()) {
                const uint64_t vs = v_d + (iv % C::kStages) * kStageD;
#pragma unroll
                for (int kk = half * (kKeys / 32); kk < (half + 1) * (kKeys / 32); ++kk)
                  umma_bf16_ts(tmem + C::kTmemO + t * HD, tmem + t * kKeys + kk * 8, vs + kk * ((16 * 128) >> 4), id_o,
                               (j < w.hi[t] - 1 || kk > 0) ? 1u : 0u);
                if (half == 1 && j == w.lo[t]) umma_commit(o_full + 8 * t);
              }
              __syncwarp();
            };
            add_half(0);
            alive = wait_all(p_full + 8 * t, pphase[t]);
            if (!alive) break;
            pphase[t] ^= 1u;
            add_half(1);
          }
          if (j > lo && active(t, j - 1)) alive = issue_s(t, j - 1, ik);
        }
        if (!alive) break;
        if (elect_one()) {
          umma_commit(kv_empty + 8 * (iv % C::kStages));
          if (j > lo) umma_commit(kv_empty + 8 * (ik % C::kStages));
        }
        __syncwarp();
      }
    }
    if (!alive && lane == 0) {
      umma_commit(drain_bar);
      if (!mbar_drain(drain_bar, 0u)) sts_u32(drain_fail, 1u);
    }
  }
  } else {
    // ------------------------------------------------------------------ softmax: a thread per row
    registers_up<kSoftmaxRegs>();
    const int t = warp >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
    const uint32_t s_at = lane_base + t * kKeys, o_at = lane_base + C::kTmemO + t * HD;
    uint32_t wphase = 0, sphase = 0, ophase = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const int valid = work[slot].valid, b = work[slot].b, h = work[slot].h[t], i = work[slot].row0[t] + row, lo = work[slot].lo[t],
                hi = work[slot].hi[t], q0 = work[slot].q0, n = work[slot].n, len = work[slot].len, part = work[slot].part;
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!valid) break;
      const bool mine = i < n;
      const int pos = PAGED ? len - n + i : i;                        // among the keys
      int2 sees = make_int2(0, 0x7fffffff);                           // (rows behind the last: whatever comes, nothing is stored)
      float scale = 0.f;
      if (mine) {
        if constexpr (PAGED) {
          sees = make_int2(f.window > 0 ? max(0, pos - f.window + 1) : 0, pos + 1);
          scale = a.beta ? length_scale(a.beta[h], a.gamma[h], a.delta[h], sees.y - sees.x) : 1.0f;
          if (a.beta && f.status && !isfinite(scale)) atomicOr(f.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_SCALE);
        } else {
          sees = visible_keys(a, b, i);
          scale = row_scale(a, b, h, i, sees.y - sees.x);
          if ((a.beta || a.c_rows) && f.status && !isfinite(scale)) atomicOr(f.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_SCALE);
        }
      }
      if (!PAGED && sees.y <= sees.x) scale = 0.f;                    // (it has none, whatever the table holds for it)
      RowSoftmax<CAP, TERMS, PAGED> sm;
      sm.start(mine, scale * a.unit * kLog2e, a.alibi ? a.alibi[h] / a.unit : 0.f, pos);
      for (int j = hi - 1; j >= lo && alive; --j) {
        alive = wait_all(s_full + 8 * t, sphase);
        if (!alive) break;
        sphase ^= 1u;
        tc_fence_after();
        float s[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(s_at + c * 32, s[c]);
        const int k0 = j * kKeys;
        const bool edge = __any_sync(0xffffffffu, sees.x > k0 || sees.y < k0 + kKeys);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_wait32(s[c]);
        const float grown = sm.take(a.cap_inv, s, k0, sees, edge);
        const bool rises = __any_sync(0xffffffffu, grown != 1.0f);    // (asked in every step: the warp's rows may have gone different ways, and the stores are all lanes')
        if (j < hi - 1 && rises) {
#pragma unroll
          for (int c = 0; c < HD / 16; ++c) {
            float v[16];
            uint32_t u[16];
            tmem_ld16(o_at + c * 16, v);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(v[e] * grown);
            tmem_st16(o_at + c * 16, u);
          }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t p[16];
          sm.probabilities(s[c], p);
          tmem_st16(s_at + c * 16, p);
          if (c == 1 || c == 3) {
            // (the first half of P goes ahead)
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive((c == 1 ? p_half : p_full) + 8 * t);
          }
        }
      }
      if (!alive) break;
      float inv = 0.f;
      const float mass = sm.sum();
      if (!PAGED || part < 0) {
        inv = mass != 0.f ? 1.0f / mass : 0.f;                        // (0: it sees nothing; a NaN is none of that)
        if (mine) {
          const float lse = mass != 0.f ? (sm.base() + log2f(mass)) * kLn2 : -INFINITY;
          if constexpr (PAGED) f.lse[(size_t)(q0 + i) * a.H + h] = lse;
          else f.lse[((size_t)b * a.H + h) * a.N + i] = lse;
        }
      } else if (mine) {
        f.part_ml[(size_t)(part + t) * kRows + row] = make_float2(sm.base(), mass);
      }
      __nv_bfloat16* out = PAGED ? f.o + ((long long)(q0 + i) * a.H + h) * HD : f.o + (long long)b * a.o.b + (long long)h * a.o.h + (long long)i * a.o.n;
      const long long stride = PAGED ? (long long)a.H * HD : a.o.n;
      const bool some = hi > lo;
      if (some) {
        alive = wait_all(o_full + 8 * t, ophase);
        if (!alive) break;
        ophase ^= 1u;
        tc_fence_after();
      }
#pragma unroll
      for (int c = 0; c < HD / 32; ++c) {
        float v[32];
        if (some) {
          tmem_ld32(o_at + c * 32, v);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.f;
        }
        if (PAGED && part >= 0) {
          float* to = f.part_o + ((size_t)(part + t) * kRows + row) * HD + c * 32;
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(v[half * 16 + e]);
            store_quad_rows(w, to + half * 16, HD * 4, n - i);
          }
        } else {
          // (a row that sees nothing: its O is 0 times what the tile's other rows left it with, which is 0)
          store_quad_rows(v, inv, out + c * 32, stride, n - i);
        }
      }
      if (some) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(o_empty + 8 * t);
      }
    }
  }

  // ---------------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (lds_u32(abort_flag)) {
    if (threadIdx.x == 0 && f.status) atomicOr(f.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_WAIT_EXPIRED);
    if (lds_u32(drain_fail)) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 200000ull) { }
    }
    __syncthreads();
  }
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int HD, bool PAGED, bool CAP, bool TERMS>
cudaError_t launch_variant(unsigned grid, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const FwdArgs& f,
                           cudaStream_t stream) {
  const cudaError_t err =
      cudaFuncSetAttribute(softmax_fwd_kernel<HD, PAGED, CAP, TERMS>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdCfg<HD>::kSmemBytes);
  if (err != cudaSuccess) return err;
  return launch_kernel(softmax_fwd_kernel<HD, PAGED, CAP, TERMS>, grid, kFwdThreads, FwdCfg<HD>::kSmemBytes, stream, map_q, map_k, map_v, f);
}
template <int HD, bool PAGED>
cudaError_t launch_any(unsigned grid, const CUtensorMap& map_q, const CUtensorMap& map_k, const CUtensorMap& map_v, const FwdArgs& f, cudaStream_t stream) {
  const bool cap = f.a.cap_inv > 0.f, terms = f.a.beta || f.a.c_rows || f.a.alibi;
  if (cap) return terms ? launch_variant<HD, PAGED, true, true>(grid, map_q, map_k, map_v, f, stream)
                        : launch_variant<HD, PAGED, true, false>(grid, map_q, map_k, map_v, f, stream);
  return terms ? launch_variant<HD, PAGED, false, true>(grid, map_q, map_k, map_v, f, stream)
               : launch_variant<HD, PAGED, false, false>(grid, map_q, map_k, map_v, f, stream);
}

template <int HD>
cudaError_t fwd_launch(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status, cudaStream_t stream) {
  CUtensorMap map_q, map_k, map_v;
  cudaError_t err = make_tile_map(&map_q, q, a.D, a.N, a.H, a.B, a.q.n, a.q.h, a.q.b);
  if (err == cudaSuccess) err = make_tile_map(&map_k, k, a.D, a.N, a.KH, a.B, a.k.n, a.k.h, a.k.b);
  if (err == cudaSuccess) err = make_tile_map(&map_v, v, a.D, a.N, a.KH, a.B, a.v.n, a.v.h, a.v.b);
  if (err != cudaSuccess) return err;
  FwdArgs f = {};
  f.a = a;
  f.pair_heads = a.G % 2 == 0;
  f.pairs = f.pair_heads ? a.G / 2 : a.G;
  f.tiles = f.pair_heads ? (a.N + kRows - 1) / kRows : (a.N + 2 * kRows - 1) / (2 * kRows);
  f.o = static_cast<__nv_bfloat16*>(o);
  f.lse = lse;
  f.status = status;
  return launch_any<HD, false>((unsigned)((long long)a.B * a.KH * f.pairs * f.tiles), map_q, map_k, map_v, f, stream);
}

template <int HD>
cudaError_t chunks_launch(const SoftmaxPagedArgs& p, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t stream) {
  CUtensorMap map_q;
  const cudaError_t err = make_tile_map(&map_q, p.q, p.c.D, p.c.T, p.H, 1, p.q_st, p.q_sh, p.c.T * p.q_st);
  if (err != cudaSuccess) return err;
  FwdArgs f = {};
  f.a.B = p.c.B; f.a.H = p.H; f.a.KH = p.c.KH; f.a.G = p.G; f.a.D = p.c.D;
  f.a.sm_scale = p.sm_scale; f.a.cap_inv = p.cap_inv; f.a.unit = p.unit;
  f.a.beta = p.beta; f.a.gamma = p.gamma; f.a.delta = p.delta; f.a.alibi = p.alibi;
  f.pair_heads = p.G % 2 == 0;
  f.pairs = chunk_pairs(p.G);
  f.o = p.o;
  f.lse = p.lse;
  f.status = p.status;
  f.c = p.c;
  f.window = p.window; f.max_q = p.max_q; f.max_kv = p.max_kv; f.few_rows = p.few_rows;
  f.shares = p.shares; f.box_shift = p.box_shift;
  f.part_o = p.chunk_o; f.part_ml = p.chunk_ml;
  f.v = p.v;
  const long long units = ((long long)p.c.T / chunk_block(p.G) + p.c.B) * p.c.KH * f.pairs;
  return launch_any<HD, true>((unsigned)(units * p.shares), map_q, map_k, map_v, f, stream);
}

}  // namespace

cudaError_t launch_softmax_chunks(const SoftmaxPagedArgs& a, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t stream) {
  return a.c.D == 64 ? chunks_launch<64>(a, map_k, map_v, stream) : chunks_launch<128>(a, map_k, map_v, stream);
}

cudaError_t launch_softmax_fwd(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status,
                               cudaStream_t stream) {
  return a.D == 64 ? fwd_launch<64>(a, q, k, v, o, lse, status, stream) : fwd_launch<128>(a, q, k, v, o, lse, status, stream);
}

}  // namespace entmax
