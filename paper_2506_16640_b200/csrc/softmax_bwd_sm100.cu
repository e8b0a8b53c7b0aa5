// Softmax attention on sm_100a, backward: dQ (and dL/dc) query-major, dK and dV key-major.
//
//   P = exp2(a x - lse log2 e),  dP = dO V^T,  D_i = <dO_i, O_i>,  dS = P (dP - D),  dx = dS (1 - tanh^2)
//   dQ_i = c_i sm sum_j dx_ij k_j,   dK_j = sum_i c_i sm dx_ij q_i,   dV_j = sum_i P_ij dO_i
// Two kernels, so that nothing is added up by atomics: the scores and dP are formed twice (seven products instead of five), but no gradient goes
// through memory as a float32 sum and results are the same every time.
//   softmax_dq_kernel   an item is a Q tile of 128 rows: S and dP in TMEM, a row's 128 columns by four threads, dS as bf16 to TMEM and
//                       from there into dQ += dS K.  Leaves -lse log2 e, a and -D of every row, and which keys every tile sees, to the other kernel.
//                       dL/dc_i = sum dS x is formed as (sum p y x - (sum p y)(sum p x) / sum p) / sum p with y = dP - D, all of float32
//                       probabilities and with x measured from the middle of the row's scores: the D above comes from the O that was rounded to bf16,
//                       which is good enough for dS but not for a float32 result.
//   softmax_dkv_kernel  an item is a K/V tile; over all query heads that share it and all Q tiles that see it: S^T = K Q^T and dP^T = V dO^T with the keys
//                       along the lanes, so that P^T and dS^T are, over their own columns, the A operands of dV += P^T dO and dK += dS^T Q; what
//                       depends on the query comes from shared memory.
//
// CTA of both: warp 0 scheduler and TMA producer, warp 1 MMA issuer, warps 2..17 four threads per TMEM lane (32 columns each).  The dQ kernel has a second
// issuer, warp 18, for dQ alone: an issuer is held up by the products it issues, and a wait that is over at once still takes 100 cycles, of which a step has
// five (16 heads x 8192 x 128, no mask: 667 us with one, 580 with two; forward and dK / dV, whose issuers' products depend on one another, lost by a
// second one).  Every wait is bounded.
//
// Bound by a step's chain of barriers, TMEM loads, element code and products: 16 heads x 8192 x 128 causal 294 us for dQ (three products, 1.40 PFLOP/s) and 444 us for
// dK and dV (four, 1.24); without a mask at 64 columns (4 x 16 x 4096) 472 and 695 us.  Short rows: 8 x 12 x 1024 x 64 48 and 60 us, with a learned scale and its
// gradient 73 and 65.  All threads have 96 registers: variants with caps, slopes or scales spill on the element path (dQ with everything 96 bytes stored, 236 read).
#include <cuda.h>

#include <type_traits>

#include "sm100_ptx.cuh"
#include "softmax.cuh"
#include "softmax_tile.cuh"

namespace entmax {

namespace {

using namespace sm100;

constexpr int kT = 128;
constexpr int kWarps = 16;                       // element code
constexpr int kGroups = kWarps / 4;              // threads per TMEM lane, 32 columns each
constexpr int kBwdThreads = (2 + kWarps) * 32;
constexpr int kDqThreads = (3 + kWarps) * 32, kSecond = 2 + kWarps;   // dQ: with a second MMA issuer, that warp
constexpr int kBwdBars = 1536;

template <int HD>
struct BwdCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kTile = kT * HD * 2;
  static constexpr int kKStages = 3, kVStages = 2;
  static constexpr int kSmemQ = (2 + kKStages + kVStages) * kTile + kBwdBars + 1024;
  static constexpr int kRowBytes = 3 * kT * 4;                      // what a step needs to know of its 128 queries
  static constexpr int kSmemKV = 6 * kTile + 2 * kRowBytes + kBwdBars + 1024;
  static_assert(kSmemQ <= 232448 && kSmemKV <= 232448, "shared memory of one CTA");
};

struct BwdWork {
  int valid, b, h, tile, lo, hi;
  int some_short;               // dQ: some row sees keys of the last K/V tile alone
  int pad;
};

struct BwdArgs {
  SoftmaxArgs a;
  SoftmaxGrads g;
  int tiles;                    // of 128 rows, per head
  const __nv_bfloat16 *o, *d_o;
  __nv_bfloat16 *dq, *dk, *dv;
  float* rows;                  // [B H tiles][3][128]: -lse log2 e (-inf: a row that sees nothing), a, -D
  int4* spans;                  // [B tiles] {first key any row sees, one behind the last, largest first, smallest last}, with ranges
  int32_t* status;
};

__host__ __device__ constexpr uint32_t bwd_idesc_kk() {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(kT >> 3) << 17) | ((uint32_t)(kT >> 4) << 24);
}
// A from TMEM, B with N contiguous
template <int HD>
__host__ __device__ constexpr uint32_t bwd_idesc_kn() {
  return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(kT >> 4) << 24);
}
// A bf16 operand written over the columns it came from: every 32 columns hold their 32 entries in the first 16, so K step kk (16 entries) starts here
__device__ __forceinline__ uint32_t a_column(int kk) { return (uint32_t)((kk >> 1) * 32 + (kk & 1) * 8); }

// {first key, one behind the last, largest first, smallest last} over the rows of a tile that see something, by the whole warp
__device__ __forceinline__ int4 span_of(const SoftmaxArgs& a, int b, int row0) {
  const int lane = threadIdx.x & 31;
  int4 s = make_int4(0x7fffffff, 0, 0, 0x7fffffff);
  int2 range[kT / 32];                           // (rows behind the last: the last once more)
#pragma unroll
  for (int t = 0; t < kT / 32; ++t) range[t] = a.ranges[(size_t)b * a.N + min(row0 + t * 32 + lane, a.N - 1)];
#pragma unroll
  for (int t = 0; t < kT / 32; ++t) {
    const int2 v = seen_of(a, range[t], min(row0 + t * 32 + lane, a.N - 1));
    if (v.y <= v.x) continue;
    s.x = min(s.x, v.x); s.y = max(s.y, v.y); s.z = max(s.z, v.x); s.w = min(s.w, v.y);
  }
  s.x = __reduce_min_sync(0xffffffffu, s.x);
  s.y = __reduce_max_sync(0xffffffffu, s.y);
  s.z = __reduce_max_sync(0xffffffffu, s.z);
  s.w = __reduce_min_sync(0xffffffffu, s.w);
  return s;
}

// Item -> (batch row, head) and tile: causal calls hand out the longest tiles of all heads first, and calls with ranges go in the same order (documents end with
// short tiles, and what neighbouring tiles see stays in L2; a head after the other left SMs idle at the end, 35 % of dK and dV's time with four K/V heads); calls
// without a mask a head after the other, whose K/V tiles (Q tiles) then stay in L2
__device__ __forceinline__ void item_of(const SoftmaxArgs& a, int item, int tiles, int heads, int& head, int& tile) {
  if (a.causal || a.ranges) {
    tile = item / heads;
    head = item - tile * heads;
  } else {
    head = item / tiles;
    tile = item - head * tiles;
  }
}

__device__ __forceinline__ void bwd_teardown(uint32_t tmem, uint32_t abort_flag, uint32_t drain_fail, int32_t* status) {
  tc_fence_before();
  __syncthreads();
  if (lds_u32(abort_flag)) {
    if (threadIdx.x == 0 && status) atomicOr(status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_WAIT_EXPIRED);
    if (lds_u32(drain_fail)) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 200000ull) { }
    }
    __syncthreads();
  }
  if ((threadIdx.x >> 5) == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ------------------------------------------------------------------------------------------------ dQ
struct RowTerms {
  float lse2, a, dot, slope, mid;   // mid: about where the row's scores lie (any value will do)
  int2 sees;
  int i;
};

// 32 columns from key j0 on (s: their accumulators, or the tanh of capped ones): dS as bf16 pairs; FINE: what their rounding left
// over as bf16 pairs, and in sums {sum p (dP - D), sum p, and with DC sum p (dP - D) (x - mid), sum p (x - mid)}, the even and the odd columns' apart
template <bool CAP, bool SLOPE, bool FINE, bool DC, bool EDGE>
__device__ __forceinline__ void dq_elements(const RowTerms& r, int j0, const float (&s)[32], const float (&dp)[32], uint32_t (&ds)[16],
                                            uint32_t (&dl)[16], uint64_t (&sums)[4]) {
  const uint64_t a2 = pack2(r.a, r.a), l2 = pack2(-r.lse2, -r.lse2), d2 = pack2(-r.dot, -r.dot);
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const int j = j0 + e;
    const uint64_t t = pack2(s[e], s[e + 1]);
    uint64_t x = t;
    if (SLOPE) x = pack2(fmaf(-r.slope, fabsf((float)(j - r.i)), s[e]), fmaf(-r.slope, fabsf((float)(j + 1 - r.i)), s[e + 1]));
    float p0, p1;
    unpack2(fma2(x, a2, l2), p0, p1);
    p0 = exp2_fast(p0);
    p1 = exp2_fast(p1);
    if (EDGE) {
      p0 = j >= r.sees.x && j < r.sees.y ? p0 : 0.f;
      p1 = j + 1 >= r.sees.x && j + 1 < r.sees.y ? p1 : 0.f;
    }
    const uint64_t p = pack2(p0, p1), v = pack2(dp[e], dp[e + 1]);
    uint64_t d = mul2(p, add2(v, d2));
    if (FINE) {
      sums[0] = add2(d, sums[0]);
      sums[1] = add2(p, sums[1]);
      if (DC) {
        const uint64_t y = add2(x, pack2(-r.mid, -r.mid));
        sums[2] = fma2(d, y, sums[2]);
        sums[3] = fma2(p, y, sums[3]);
      }
    }
    if (CAP) d = mul2(d, fma2(t, pack2(-s[e], -s[e + 1]), pack2(1.0f, 1.0f)));
    float d0, d1;
    unpack2(d, d0, d1);
    ds[e >> 1] = bf16x2(d0, d1);
    if (FINE) dl[e >> 1] = bf16x2(d0 - __uint_as_float(ds[e >> 1] << 16), d1 - __uint_as_float(ds[e >> 1] & 0xffff0000u));
  }
}
// CAP, SLOPE, FINE, DC known at compile time: see RowSoftmax.
// FINE: calls with scales or slopes, whose maps are sharp.  A row of dS sums to zero, so dQ is what remains of a cancellation where its few keys weigh about the
// same, and the rounding, up to 2^-8 of every term, is a part of that: dQ gets what the rounding of dS left over as a second product.  And dK gets D from the float32 probabilities.
// (8 x 12 x 1024 x 64 with a learned scale: dQ 2.5e-3 off in norm without, 1.9e-3 with; the rounding of dQ itself is 1.7e-3.  Plain calls, 2.4e-3, would lose
// 4 to 9 % of the backward pass.)
template <int HD, bool CAP, bool SLOPE, bool FINE, bool DC>
__global__ void __launch_bounds__(kDqThreads, 1) softmax_dq_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                    const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                                                                    const __grid_constant__ BwdArgs f) {
  pdl_begin();
  using C = BwdCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_smem = sbase, do_smem = q_smem + C::kTile, k_smem = do_smem + C::kTile, v_smem = k_smem + C::kKStages * C::kTile;
  const uint32_t bars = v_smem + C::kVStages * C::kTile;
  const uint32_t work_at = bars, answer = bars + 64;
  const uint32_t q_full = bars + 80, q_empty = bars + 88;
  const uint32_t k_full = bars + 96, k_empty = bars + 120;           // [3]
  const uint32_t v_full = bars + 144, v_empty = bars + 160;          // [2]
  const uint32_t s_full = bars + 176, s_empty = bars + 184;
  const uint32_t dp_full = bars + 296, dp_empty = bars + 304;
  const uint32_t ds_full = bars + 192, ds_empty = bars + 200;
  const uint32_t dq_full = bars + 208, dq_empty = bars + 216;
  const uint32_t w_full = bars + 224, w_empty = bars + 240;          // [2]
  const uint32_t next_bar = bars + 256, x_bar = bars + 264, drain_bar = bars + 312;   // drain_bar [2]
  const uint32_t tmem_slot = bars + 280, abort_flag = bars + 284, drain_fail = bars + 288;
  const uint32_t dot_at = bars + 336;                                // float [2][128]: of this item and the one before
  const BwdWork* work = reinterpret_cast<const BwdWork*>(smem_raw + (work_at - smem_u32(smem_raw)));
  constexpr int kS = 0, kDP = kT, kDQ = 2 * kT, kDS = 2 * kT + 128, kDL = kDS + 64;   // (kDL: what the rounding of dS left over)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int st = 0; st < C::kKStages; ++st) { mbar_init(k_full + 8 * st, 1); mbar_init(k_empty + 8 * st, 1); }
    for (int st = 0; st < C::kVStages; ++st) { mbar_init(v_full + 8 * st, 1); mbar_init(v_empty + 8 * st, 1); }
    mbar_init(s_full, 1);
    mbar_init(s_empty, kWarps);
    mbar_init(dp_full, 1);
    mbar_init(dp_empty, kWarps);
    mbar_init(ds_full, kWarps);
    mbar_init(ds_empty, 1);
    mbar_init(dq_full, 1);
    mbar_init(dq_empty, kWarps);
    for (int t = 0; t < 2; ++t) { mbar_init(w_full + 8 * t, 1); mbar_init(w_empty + 8 * t, 2 + kWarps); mbar_init(drain_bar + 8 * t, 1); }
    mbar_init(next_bar, 1);
    mbar_init(x_bar, kWarps);
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
  const uint32_t tmem = uniform(lds_u32(tmem_slot));
  const SoftmaxArgs& a = f.a;
  auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };
  // two barriers at once: the second one's answer comes with the first's
  auto wait_both = [&](uint32_t bar, uint32_t parity, uint32_t bar2, uint32_t parity2) -> bool {
    const bool a1 = mbar_try_wait(bar, parity), a2 = mbar_try_wait(bar2, parity2);
    if (__all_sync(0xffffffffu, a1 && a2)) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag) && mbar_wait(bar2, parity2, abort_flag));
  };

  if (warp == 0) {
    uint32_t next_phase = 0, wphase = 0, qphase = 0, kidx = 0, vidx = 0;
    int slot = 0;
    bool alive = true, asked = false;
    int item = (int)blockIdx.x;
    while (alive) {
      BwdWork w = {};
      w.valid = item >= 0;
      if (item >= 0) {
        int bh;
        item_of(a, item, f.tiles, a.B * a.H, bh, w.tile);
        w.tile = f.tiles - 1 - w.tile;
        w.b = bh / a.H;
        w.h = bh - w.b * a.H;
        const int row0 = w.tile * kT;
        if (a.ranges) {
          const int4 s = span_of(a, w.b, row0);
          if (w.h == 0 && lane == 0) f.spans[w.b * f.tiles + w.tile] = s;
          if (s.y > s.x) {
            w.lo = s.x / kT;
            w.hi = (s.y + kT - 1) / kT;
            w.some_short = s.z >= (w.hi - 1) * kT;
          }
        } else {
          w.hi = ((a.causal ? min(row0 + kT, a.N) : a.N) + kT - 1) / kT;
          w.some_short = w.hi == 1;
        }
      }
      alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
      if (!alive) break;
      if (lane == 0) {
        *const_cast<BwdWork*>(work + slot) = w;
        mbar_arrive(w_full + 8 * slot);
      }
      __syncwarp();
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (item < 0) break;
      if (w.hi > w.lo) {
        alive = wait_all(q_empty, qphase ^ 1u);
        if (!alive) break;
        qphase ^= 1u;
        if (elect_one()) {
          mbar_expect_tx(q_full, 2 * C::kTile);
          for (int hf = 0; hf < C::kHalves; ++hf) {
            tma_load_4d(q_smem + hf * (kT * 128), &map_q, q_full, hf * 64, w.tile * kT, w.h, w.b);
            tma_load_4d(do_smem + hf * (kT * 128), &map_do, q_full, hf * 64, w.tile * kT, w.h, w.b);
          }
        }
        __syncwarp();
        const int kh = w.h / a.G;
        for (int j = w.hi - 1; j >= w.lo && alive; --j) {
          const int ks = kidx % C::kKStages, vs = vidx % C::kVStages;
          alive = wait_all(k_empty + 8 * ks, ((kidx / C::kKStages) & 1u) ^ 1u);
          if (!alive) break;
          ++kidx;
          if (elect_one()) {
            mbar_expect_tx(k_full + 8 * ks, C::kTile);
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(k_smem + ks * C::kTile + hf * (kT * 128), &map_k, k_full + 8 * ks, hf * 64, j * kT, kh, w.b);
          }
          __syncwarp();
          alive = wait_all(v_empty + 8 * vs, ((vidx / C::kVStages) & 1u) ^ 1u);
          if (!alive) break;
          ++vidx;
          if (elect_one()) {
            mbar_expect_tx(v_full + 8 * vs, C::kTile);
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(v_smem + vs * C::kTile + hf * (kT * 128), &map_v, v_full + 8 * vs, hf * 64, j * kT, kh, w.b);
          }
          __syncwarp();
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
      bool ok = mbar_drain(q_full, qphase ^ 1u);
      for (uint32_t st = 0; st < C::kKStages; ++st) ok &= mbar_drain(k_full + 8 * st, ((kidx / C::kKStages + (st < kidx % C::kKStages ? 1u : 0u)) & 1u) ^ 1u);
      for (uint32_t st = 0; st < C::kVStages; ++st) ok &= mbar_drain(v_full + 8 * st, ((vidx / C::kVStages + (st < vidx % C::kVStages ? 1u : 0u)) & 1u) ^ 1u);
      if (asked) ok &= mbar_drain(next_bar, next_phase);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ S and dP.  Each is issued again as soon as the element warps have the last one in
    // registers: while one is on its way between the two sides the tensor core has the other.
    constexpr uint32_t id_kk = bwd_idesc_kk();
    const uint64_t dhi = (uint64_t)kDescHi << 32;
    const uint64_t q_d = dhi | smem_desc_lo(q_smem), do_d = dhi | smem_desc_lo(do_smem), k_d = dhi | smem_desc_lo(k_smem),
                   v_d = dhi | smem_desc_lo(v_smem);
    constexpr uint32_t kStageD = C::kTile >> 4;
    uint32_t wphase = 0, qphase = 0, sphase = 0, dpphase = 0, kidx = 0, vidx = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const int valid = uniform(work[slot].valid), lo = uniform(work[slot].lo), hi = uniform(work[slot].hi);
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!valid) break;
      if (hi <= lo) continue;
      alive = wait_all(q_full, qphase);
      if (!alive) break;
      qphase ^= 1u;
      for (int j = hi - 1; j >= lo && alive; --j) {
        const uint32_t ks = kidx % C::kKStages, vs = vidx % C::kVStages;
        alive = wait_both(k_full + 8 * ks, (kidx / C::kKStages) & 1u, s_empty, sphase ^ 1u);
        if (!alive) break;
        ++kidx;
        sphase ^= 1u;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk >> 2) * ((kT * 128) >> 4) + (kk & 3) * 2;
            umma_bf16_desc(tmem + kS, q_d + off, k_d + ks * kStageD + off, id_kk, kk > 0 ? 1u : 0u);
          }
          umma_commit(s_full);
        }
        __syncwarp();
        alive = wait_both(v_full + 8 * vs, (vidx / C::kVStages) & 1u, dp_empty, dpphase ^ 1u);
        if (!alive) break;
        ++vidx;
        dpphase ^= 1u;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk >> 2) * ((kT * 128) >> 4) + (kk & 3) * 2;
            umma_bf16_desc(tmem + kDP, do_d + off, v_d + vs * kStageD + off, id_kk, kk > 0 ? 1u : 0u);
          }
          umma_commit(dp_full);
          umma_commit(v_empty + 8 * vs);
          if (j == lo) umma_commit(q_empty);
        }
        __syncwarp();
      }
    }
    if (!alive && lane == 0) {
      umma_commit(drain_bar);
      if (!mbar_drain(drain_bar, 0u)) sts_u32(drain_fail, 1u);
    }
  } else if (warp == kSecond) {
    // ------------------------------------------------------------------ dQ
    constexpr uint32_t id_kn = bwd_idesc_kn<HD>();
    const uint64_t kn_d = ((uint64_t)kDescHi << 32) | mn_desc_lo(k_smem);
    constexpr uint32_t kStageD = C::kTile >> 4;
    uint32_t wphase = 0, dsphase = 0, dqphase = 0, kidx = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const int valid = uniform(work[slot].valid), lo = uniform(work[slot].lo), hi = uniform(work[slot].hi);
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!valid) break;
      if (hi <= lo) continue;
      alive = wait_all(dq_empty, dqphase ^ 1u);              // the previous item's dQ has been read
      if (!alive) break;
      dqphase ^= 1u;
      for (int j = hi - 1; j >= lo && alive; --j, ++kidx) {
        const uint32_t ks = kidx % C::kKStages;
        alive = wait_both(k_full + 8 * ks, (kidx / C::kKStages) & 1u, ds_full, dsphase);
        if (!alive) break;
        dsphase ^= 1u;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t kn = kn_d + ks * kStageD;
#pragma unroll
          for (int kk = 0; kk < kT / 16; ++kk)
            umma_bf16_ts(tmem + kDQ, tmem + kDS + kk * 8, kn + kk * ((16 * 128) >> 4), id_kn, (j < hi - 1 || kk > 0) ? 1u : 0u);
#pragma unroll
          for (int kk = 0; FINE && kk < kT / 16; ++kk) umma_bf16_ts(tmem + kDQ, tmem + kDL + kk * 8, kn + kk * ((16 * 128) >> 4), id_kn, 1u);
          umma_commit(k_empty + 8 * ks);                     // (S of this tile came long before)
          umma_commit(ds_empty);
          if (j == lo) umma_commit(dq_full);
        }
        __syncwarp();
      }
    }
    if (!alive && lane == 0) {
      umma_commit(drain_bar + 8);
      if (!mbar_drain(drain_bar + 8, 0u)) sts_u32(drain_fail, 1u);
    }
  } else {
    const int quad = warp & 3, group = (warp - 2) >> 2, row = quad * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
    uint32_t wphase = 0, sphase = 0, dpphase = 0, dsphase = 0, dqphase = 0, xphase = 0, dot_buf = 0;
    int slot = 0;
    bool alive = true;
    // all element warps
    auto meet_all = [&]() -> bool {
      __syncwarp();
      if (lane == 0) mbar_arrive(x_bar);
      const bool ok = wait_all(x_bar, xphase);
      xphase ^= 1u;
      return ok;
    };
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const int valid = work[slot].valid, b = work[slot].b, h = work[slot].h, tile = work[slot].tile, lo = work[slot].lo, hi = work[slot].hi;
      const bool some_short = work[slot].some_short != 0;
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!valid) break;
      RowTerms r;
      r.i = tile * kT + row;
      const bool mine = r.i < a.N;
      r.sees = mine ? visible_keys(a, b, r.i) : make_int2(0, 0);
      const size_t at = ((size_t)b * a.H + h) * a.N + (mine ? r.i : 0);
      const bool some = r.sees.y > r.sees.x;
      // (a row that sees nothing has no scale: what the table holds for it, of padding, may be anything)
      const float held = mine ? row_scale(a, b, h, r.i, r.sees.y - r.sees.x) : 0.f, c = some ? held : 0.f, g = c * a.sm_scale;
      r.a = c * a.unit * kLog2e;
      r.lse2 = some ? f.g.lse[at] * kLog2e : INFINITY;
      r.slope = a.alibi ? a.alibi[h] / a.unit : 0.f;
      // (the logarithm of the scores' mean exponential, which lies between the least and the largest)
      r.mid = DC && fabsf(r.a) > 1e-3f && some ? (r.lse2 - log2f((float)(r.sees.y - r.sees.x))) / r.a : 0.f;
      if (!some) { r.sees = make_int2(0, 0x7fffffff); r.a = 0.f; }   // (probability exp2(-inf) everywhere, without a mask)
      // D of the tile's rows, eight rows a warp: the 32 lanes read D / 32 elements each of O and dO (the loads above are on their way meanwhile)
      {
        constexpr int E = HD / 32;
        static_assert(kT == 8 * kWarps, "eight rows a warp");
        const int first = (warp - 2) * 8;
        float part[8], u[8][E], v[8][E];
        // (all loads first, those of rows behind the last from the last: a condition around each made the eight rows' latencies add up, 5 us of an item)
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const int i = min(tile * kT + first + y, a.N - 1);
          load_slice<E>(f.o + (long long)b * a.o.b + (long long)h * a.o.h + (long long)i * a.o.n + lane * E, u[y]);
          load_slice<E>(f.d_o + (long long)b * f.g.d_o.b + (long long)h * f.g.d_o.h + (long long)i * f.g.d_o.n + lane * E, v[y]);
        }
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          part[y] = 0.f;
#pragma unroll
          for (int e = 0; e < E; ++e) part[y] = fmaf(u[y][e], v[y][e], part[y]);
        }
#pragma unroll
        for (int y = 0; y < 8; ++y) part[y] = warp_sum(part[y]);
        if (lane == 0)
          for (int y = 0; y < 8; ++y) sts_u32(dot_at + dot_buf + 4 * (first + y), __float_as_uint(part[y]));
        alive = meet_all();
        if (!alive) break;
        r.dot = __uint_as_float(lds_u32(dot_at + dot_buf + 4 * row));
        dot_buf ^= 512u;
      }
      if (group == 0) {
        float* out = f.rows + ((size_t)(b * a.H + h) * f.tiles + tile) * (3 * kT) + row;
        out[0] = -r.lse2;
        out[kT] = r.a;
        out[2 * kT] = -r.dot;
      }
      if (some_short) {
        // D of the rows that see keys of the last tile alone, from their float32 probabilities: with few keys the O it came from, rounded to bf16, is what dQ and
        // dK would be least exact by.  (A look at the first step's S and dP, which the loop then takes.)  The four threads of a row meet through the dS
        // columns, which the dQ before has read.
        alive = wait_all(s_full, sphase);
        if (alive) alive = wait_all(dp_full, dpphase);
        if (alive) alive = wait_all(ds_empty, dsphase ^ 1u);
        if (!alive) break;
        tc_fence_after();
        float sum0 = 0.f, sum1 = 0.f;
        const int j0 = (hi - 1) * kT + group * 32;
        float s[32], dp[32];
        tmem_ld32(lane_base + kS + group * 32, s);
        tmem_ld32(lane_base + kDP + group * 32, dp);
        tmem_ld_wait32(s);
        tmem_ld_wait32(dp);
        if (CAP) tanh_scores(a.cap_inv, s);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          float x = s[e];
          if (SLOPE) x = fmaf(-r.slope, fabsf((float)(j0 + e - r.i)), x);
          float p = exp2_fast(fmaf(x, r.a, -r.lse2));
          p = j0 + e >= r.sees.x && j0 + e < r.sees.y ? p : 0.f;
          sum0 = fmaf(p, dp[e], sum0);
          sum1 += p;
        }
        __syncwarp();                            // (with a cap rows may have gone different ways, and the store is all lanes')
        tmem_st2(lane_base + kDS + group * 16, __float_as_uint(sum0), __float_as_uint(sum1));
        tmem_st_wait();
        tc_fence_before();
        alive = meet_all();
        if (!alive) break;
        tc_fence_after();
        float dot = 0.f, mass = 0.f;
#pragma unroll
        for (int other = 0; other < kGroups; ++other) {
          uint32_t x, y;
          tmem_ld2(lane_base + kDS + other * 16, x, y);
          tmem_ld_wait();
          dot += __uint_as_float(x);
          mass += __uint_as_float(y);
        }
        if (some && r.sees.x >= (hi - 1) * kT && mass > 0.f) {
          r.dot = dot / mass;
          if (group == 0) f.rows[((size_t)(b * a.H + h) * f.tiles + tile) * (3 * kT) + 2 * kT + row] = -r.dot;
        }
        tc_fence_before();
        alive = meet_all();                      // (all have read before anyone writes dS there)
        if (!alive) break;
        tc_fence_after();
      }
      uint64_t sums[4] = {0u, 0u, 0u, 0u};       // (pairs of float32 zeros)
      for (int j = hi - 1; j >= lo && alive; --j) {
        alive = wait_all(s_full, sphase);
        if (!alive) break;
        sphase ^= 1u;
        tc_fence_after();
        const int j0 = j * kT + group * 32;
        const bool edge = __any_sync(0xffffffffu, r.sees.x > j0 || r.sees.y < j0 + 32);
        float s[32], dp[32];
        uint32_t ds[16], dl[16];
        tmem_ld32(lane_base + kS + group * 32, s);
        tmem_ld_wait32(s);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(s_empty);
        alive = wait_all(dp_full, dpphase);
        if (!alive) break;
        dpphase ^= 1u;
        tc_fence_after();
        tmem_ld32(lane_base + kDP + group * 32, dp);
        tmem_ld_wait32(dp);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(dp_empty);
        if (CAP) tanh_scores(a.cap_inv, s);
        if (edge) dq_elements<CAP, SLOPE, FINE, DC, true>(r, j0, s, dp, ds, dl, sums);
        else dq_elements<CAP, SLOPE, FINE, DC, false>(r, j0, s, dp, ds, dl, sums);
        // the dS before has been taken
        alive = wait_all(ds_empty, dsphase ^ 1u);
        if (!alive) break;
        dsphase ^= 1u;
        tc_fence_after();
        tmem_st16(lane_base + kDS + group * 16, ds);
        if (FINE) tmem_st16(lane_base + kDL + group * 16, dl);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(ds_full);
      }
      if (!alive) break;
      const bool any = hi > lo;
      if (any) {
        alive = wait_all(dq_full, dqphase);
        if (!alive) break;
        dqphase ^= 1u;
        tc_fence_after();
      }
      for (int c = group; c < HD / 32; c += kGroups) {
        const int col = c * 32;
        float v[32];
        if (any) {
          tmem_ld32(lane_base + kDQ + col, v);
          tmem_ld_wait();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.f;
        }
        store_quad_rows(v, g, f.dq + (long long)b * f.g.dq.b + (long long)h * f.g.dq.h + (long long)r.i * f.g.dq.n + col, f.g.dq.n, a.N - r.i);
      }
      if (FINE) {
        // the four threads of a row meet through the dS columns, which nobody needs until the next item's first dS is written: behind dq_empty of all
        const uint32_t mine_at = lane_base + kDS + group * 16;
        uint32_t u[8] = {};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float x, y;
          unpack2(sums[e], x, y);
          u[e] = __float_as_uint(x + y);
        }
        tmem_st8(mine_at, u);
        tmem_st_wait();
        tc_fence_before();
        alive = meet_all();
        if (!alive) break;
        tc_fence_after();
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int other = 0; other < kGroups; ++other) {
          float v[8];
          tmem_ld8(lane_base + kDS + other * 16, v);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[e] += v[e];
        }
        if (group == 0 && some) {
          const float more = sum[0] / sum[1];    // (sum p is 1 to float32's rounding: dividing by it, in dc as well, takes out what all of the row's probabilities are off by)
          f.rows[((size_t)(b * a.H + h) * f.tiles + tile) * (3 * kT) + 2 * kT + row] = -(r.dot + more);
          if (DC) f.g.dc_rows[at] = (sum[2] - more * sum[3]) / sum[1] * a.unit;
        } else if (DC && group == 0 && mine) {
          f.g.dc_rows[at] = 0.f;
        }
        tc_fence_before();
        alive = meet_all();                      // (all have read before anyone writes the next item's dS there)
        if (!alive) break;
        tc_fence_after();
      }
      if (any) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(dq_empty);
      }
    }
  }
  bwd_teardown(tmem, abort_flag, drain_fail, f.status);
}

// ------------------------------------------------------------------------------------------------ dK, dV
// The Q tiles that see a K/V tile, in order; all roles walk them alike.  Ranges: 32 tiles' spans are looked at together.
struct QTiles {
  int tiles, first, k0, diagonal;
  const int4* spans;
  int base;              // masks: those of the tiles base .. base + 31 that see the keys, and of them those with a row that does not see all
  uint32_t mask, partly;
  bool edge;             // the last tile: whether it has such a row
  __device__ __forceinline__ void start(const BwdArgs& f, int batch, int kt) {
    tiles = f.tiles;
    k0 = kt * kT;
    spans = f.a.ranges ? f.spans + (size_t)batch * f.tiles : nullptr;
    diagonal = f.a.causal && !spans ? kt : -1;
    first = max(diagonal, 0);
    edge = false;
    rewind();
  }
  __device__ __forceinline__ void rewind() {
    base = spans ? -32 : first - 1;
    mask = partly = 0u;
  }
  // the next tile, or -1 (the whole warp)
  __device__ __forceinline__ int next() {
    if (!spans) {
      edge = ++base == diagonal;
      return base < tiles ? base : -1;
    }
    while (mask == 0u) {
      base += 32;
      if (base >= tiles) return -1;
      const int t = base + (threadIdx.x & 31);
      bool sees = false, some = false;
      if (t < tiles) {
        const int4 s = spans[t];
        sees = s.x < k0 + kT && s.y > k0;
        some = s.z > k0 || s.w < k0 + kT;
      }
      mask = __ballot_sync(0xffffffffu, sees);
      partly = __ballot_sync(0xffffffffu, some);
    }
    const int bit = __ffs(mask) - 1;
    mask &= mask - 1u;
    edge = (partly >> bit) & 1u;
    return base + bit;
  }
};

// The transposed scores of 32 queries (columns) and 32 keys (lanes) in the layout of tmem_ld_frag, lanes 0 .. 15 in s[0 .. 15], 16 .. 31 behind them: a thread has four keys
// and eight queries, for which it reads shared memory once (a thread of the plain layout has one key and 32 queries; with four wavefronts to a load that all
// lanes share, those loads took as much of the shared memory's time as the products' operands).
// s: P^T as bf16 pairs goes to u, and in place of s what dP - D is multiplied by, P a (1 - tanh^2).  dist: first query - first key of the thread
template <bool CAP, bool SLOPE, bool SCALED>
__device__ __forceinline__ void dkv_probabilities(float scale, float slope, int dist, uint32_t rows_at, float (&s)[32], uint32_t (&u)[16]) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float l0, l1, m0 = scale, m1 = scale;
    lds_f2(rows_at + 32 * k, l0, l1);
    if (SCALED) lds_f2(rows_at + 4 * kT + 32 * k, m0, m1);
    const uint64_t l2 = pack2(l0, l1), m2 = pack2(m0, m1);
#pragma unroll
    for (int y = 0; y < 4; ++y) {                // keys 0, 8, 16, 24 behind the thread's first
      const int at = (y >> 1) * 16 + 4 * k + (y & 1) * 2;
      float& s0 = s[at];
      float& s1 = s[at + 1];
      const uint64_t t = pack2(s0, s1);
      uint64_t x = t;
      if (SLOPE) x = pack2(fmaf(-slope, fabsf((float)(dist + 8 * k - 8 * y)), s0), fmaf(-slope, fabsf((float)(dist + 8 * k - 8 * y + 1)), s1));
      float p0, p1;
      unpack2(fma2(x, m2, l2), p0, p1);
      p0 = exp2_fast(p0);
      p1 = exp2_fast(p1);
      u[(y >> 1) * 8 + 2 * k + (y & 1)] = bf16x2(p0, p1);
      uint64_t w = mul2(pack2(p0, p1), m2);
      if (CAP) w = mul2(w, fma2(t, pack2(-s0, -s1), pack2(1.0f, 1.0f)));
      unpack2(w, s0, s1);
    }
  }
}

template <int HD, bool CAP, bool SLOPE, bool SCALED>
__global__ void __launch_bounds__(kBwdThreads, 1) softmax_dkv_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                                                                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do,
                                                                     const __grid_constant__ BwdArgs f) {
  pdl_begin();
  using C = BwdCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t k_smem = sbase, v_smem = k_smem + C::kTile, q_smem = v_smem + C::kTile, do_smem = q_smem + 2 * C::kTile;
  const uint32_t rows_smem = do_smem + 2 * C::kTile;                 // [2][3][128] floats
  const uint32_t bars = rows_smem + 2 * C::kRowBytes;
  const uint32_t work_at = bars, answer = bars + 64;
  const uint32_t kv_full = bars + 80, kv_empty = bars + 88;
  const uint32_t q_full = bars + 96, q_empty = bars + 112;           // [2], with the rows' terms
  const uint32_t do_full = bars + 128, do_empty = bars + 144;        // [2]
  const uint32_t s_full = bars + 160, p_full = bars + 168, dp_full = bars + 176, ds_full = bars + 184;
  const uint32_t acc_full = bars + 192, acc_empty = bars + 200;
  const uint32_t w_full = bars + 208, w_empty = bars + 224;          // [2]
  const uint32_t r_empty = bars + 240;                               // [2] the rows' terms have been read
  const uint32_t next_bar = bars + 256, drain_bar = bars + 264;
  const uint32_t tmem_slot = bars + 280, abort_flag = bars + 284, drain_fail = bars + 288;
  const BwdWork* work = reinterpret_cast<const BwdWork*>(smem_raw + (work_at - smem_u32(smem_raw)));
  constexpr int kS = 0, kDP = kT, kDK = 2 * kT, kDV = 2 * kT + HD;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    mbar_init(kv_full, 1);
    mbar_init(kv_empty, 1);
    mbar_init(drain_bar, 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(q_full + 8 * t, 1);
      mbar_init(q_empty + 8 * t, 1);
      mbar_init(do_full + 8 * t, 1);
      mbar_init(do_empty + 8 * t, 1);
      mbar_init(w_full + 8 * t, 1);
      mbar_init(w_empty + 8 * t, 1 + kWarps);
      mbar_init(r_empty + 8 * t, kWarps);
    }
    mbar_init(s_full, 1);
    mbar_init(p_full, kWarps);
    mbar_init(dp_full, 1);
    mbar_init(ds_full, kWarps);
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, kWarps);
    mbar_init(next_bar, 1);
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
  const uint32_t tmem = uniform(lds_u32(tmem_slot));
  const SoftmaxArgs& a = f.a;
  auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };

  if (warp == 0) {
    uint32_t next_phase = 0, wphase = 0, kvphase = 0, idx = 0;       // idx: steps loaded so far
    int slot = 0;
    bool alive = true, asked = false;
    int item = (int)blockIdx.x;
    while (alive) {
      BwdWork w = {};
      w.valid = item >= 0;
      if (item >= 0) {
        int bk;
        item_of(a, item, f.tiles, a.B * a.KH, bk, w.tile);
        w.b = bk / a.KH;
        w.h = bk - w.b * a.KH;
      }
      alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
      if (!alive) break;
      if (lane == 0) {
        *const_cast<BwdWork*>(work + slot) = w;
        mbar_arrive(w_full + 8 * slot);
      }
      __syncwarp();
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (item < 0) break;
      QTiles qt;
      qt.start(f, w.b, w.tile);
      bool first = true;
      for (int g = 0; g < a.G && alive; ++g) {
        const int h = w.h * a.G + g;
        qt.rewind();
        for (int t = qt.next(); t >= 0 && alive; t = qt.next(), ++idx) {
          const int st = idx & 1;
          const uint32_t parity = ((idx >> 1) & 1u) ^ 1u;
          if (first) {
            first = false;
            alive = wait_all(kv_empty, kvphase ^ 1u);
            if (!alive) break;
            kvphase ^= 1u;
            if (elect_one()) {
              mbar_expect_tx(kv_full, 2 * C::kTile);
              for (int hf = 0; hf < C::kHalves; ++hf) {
                tma_load_4d(k_smem + hf * (kT * 128), &map_k, kv_full, hf * 64, w.tile * kT, w.h, w.b);
                tma_load_4d(v_smem + hf * (kT * 128), &map_v, kv_full, hf * 64, w.tile * kT, w.h, w.b);
              }
            }
            __syncwarp();
          }
          alive = wait_all(q_empty + 8 * st, parity);
          if (alive) alive = wait_all(r_empty + 8 * st, parity);
          if (!alive) break;
          if (elect_one()) {
            mbar_expect_tx(q_full + 8 * st, C::kTile + C::kRowBytes);
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(q_smem + st * C::kTile + hf * (kT * 128), &map_q, q_full + 8 * st, hf * 64, t * kT, h, w.b);
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                             rows_smem + st * C::kRowBytes),
                         "l"(reinterpret_cast<uint64_t>(f.rows + ((size_t)(w.b * a.H + h) * f.tiles + t) * (3 * kT))), "r"(C::kRowBytes),
                         "r"(q_full + 8 * st)
                         : "memory");
          }
          __syncwarp();
          alive = wait_all(do_empty + 8 * st, parity);
          if (!alive) {
            ++idx;                               // (Q of this step is on its way)
            break;
          }
          if (elect_one()) {
            mbar_expect_tx(do_full + 8 * st, C::kTile);
            for (int hf = 0; hf < C::kHalves; ++hf)
              tma_load_4d(do_smem + st * C::kTile + hf * (kT * 128), &map_do, do_full + 8 * st, hf * 64, t * kT, h, w.b);
          }
          __syncwarp();
        }
      }
      if (!alive) break;
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
      bool ok = mbar_drain(kv_full, kvphase ^ 1u);
      for (uint32_t st = 0; st < 2; ++st) {
        const uint32_t armed = (idx >> 1) + (st < (idx & 1u) ? 1u : 0u);
        ok &= mbar_drain(q_full + 8 * st, (armed & 1u) ^ 1u);
        ok &= mbar_drain(do_full + 8 * st, (armed & 1u) ^ 1u);       // (one armed less at most: its phase has passed, or this wait ends by its bound)
      }
      if (asked) ok &= mbar_drain(next_bar, next_phase);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else if (warp == 1) {
    constexpr uint32_t id_kk = bwd_idesc_kk(), id_kn = bwd_idesc_kn<HD>();
    const uint64_t dhi = (uint64_t)kDescHi << 32;
    const uint64_t q_d = dhi | smem_desc_lo(q_smem), do_d = dhi | smem_desc_lo(do_smem), k_d = dhi | smem_desc_lo(k_smem),
                   v_d = dhi | smem_desc_lo(v_smem), qn_d = dhi | mn_desc_lo(q_smem), don_d = dhi | mn_desc_lo(do_smem);
    constexpr uint32_t kStageD = C::kTile >> 4;
    uint32_t wphase = 0, kvphase = 0, pphase = 0, dsphase = 0, accphase = 0, idx = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const BwdWork w = work[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (uniform(w.valid) == 0) break;
      QTiles qt;
      qt.start(f, w.b, w.tile);
      int count = 0;
      for (int t = qt.next(); t >= 0; t = qt.next()) ++count;
      const int steps = uniform(count * a.G);
      if (steps == 0) continue;
      alive = wait_all(kv_full, kvphase);
      if (!alive) break;
      kvphase ^= 1u;
      // S^T of step i: over the P^T before, which dV has taken by then (the tensor core works in order)
      auto issue_s = [&](uint32_t i) -> bool {
        const uint32_t st = i & 1u;
        if (!wait_all(q_full + 8 * st, (i >> 1) & 1u)) return false;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk >> 2) * ((kT * 128) >> 4) + (kk & 3) * 2;
            umma_bf16_desc(tmem + kS, k_d + off, q_d + st * kStageD + off, id_kk, kk > 0 ? 1u : 0u);
          }
          umma_commit(s_full);
        }
        __syncwarp();
        return true;
      };
      auto issue_dp = [&](uint32_t i) -> bool {
        const uint32_t st = i & 1u;
        if (!wait_all(do_full + 8 * st, (i >> 1) & 1u)) return false;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < HD / 16; ++kk) {
            const uint32_t off = (kk >> 2) * ((kT * 128) >> 4) + (kk & 3) * 2;
            umma_bf16_desc(tmem + kDP, v_d + off, do_d + st * kStageD + off, id_kk, kk > 0 ? 1u : 0u);
          }
          umma_commit(dp_full);
        }
        __syncwarp();
        return true;
      };
      alive = issue_s(idx);
      if (alive) alive = issue_dp(idx);
      for (int n = 0; n < steps && alive; ++n, ++idx) {
        const uint32_t st = idx & 1u;
        alive = wait_all(p_full, pphase);
        if (!alive) break;
        pphase ^= 1u;
        if (n == 0) {
          alive = wait_all(acc_empty, accphase ^ 1u);
          if (!alive) break;
          accphase ^= 1u;
        }
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kT / 16; ++kk)
            umma_bf16_ts(tmem + kDV, tmem + kS + a_column(kk), don_d + st * kStageD + kk * ((16 * 128) >> 4), id_kn, (n > 0 || kk > 0) ? 1u : 0u);
          umma_commit(do_empty + 8 * st);        // (dP of this step came before)
        }
        __syncwarp();
        if (n + 1 < steps) {
          alive = issue_s(idx + 1);
          if (!alive) break;
        }
        alive = wait_all(ds_full, dsphase);
        if (!alive) break;
        dsphase ^= 1u;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < kT / 16; ++kk)
            umma_bf16_ts(tmem + kDK, tmem + kDP + a_column(kk), qn_d + st * kStageD + kk * ((16 * 128) >> 4), id_kn, (n > 0 || kk > 0) ? 1u : 0u);
          umma_commit(q_empty + 8 * st);
          if (n + 1 == steps) {
            umma_commit(kv_empty);
            umma_commit(acc_full);
          }
        }
        __syncwarp();
        if (n + 1 < steps) alive = issue_dp(idx + 1);
      }
    }
    if (!alive && lane == 0) {
      umma_commit(drain_bar);
      if (!mbar_drain(drain_bar, 0u)) sts_u32(drain_fail, 1u);
    }
  } else {
    const int quad = warp & 3, group = (warp - 2) >> 2, row = quad * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(quad * 32) << 16);
    uint32_t wphase = 0, sphase = 0, dpphase = 0, accphase = 0, idx = 0;
    int slot = 0;
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const int valid = work[slot].valid, b = work[slot].b, kh = work[slot].h, kt = work[slot].tile;
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!valid) break;
      QTiles qt;
      qt.start(f, b, kt);
      const int key = kt * kT + row;
      bool any = false;
      for (int g = 0; g < a.G && alive; ++g) {
        const float slope = a.alibi ? a.alibi[kh * a.G + g] / a.unit : 0.f;
        qt.rewind();
        for (int t = qt.next(); t >= 0 && alive; t = qt.next(), ++idx) {
          any = true;
          const uint32_t st = idx & 1u;
          const int i0 = t * kT + group * 32 + 2 * (lane & 3);        // this thread's first query and first key
          const int key0 = kt * kT + quad * 32 + (lane >> 2);
          const uint32_t rows_at = rows_smem + st * C::kRowBytes + 4 * (group * 32 + 2 * (lane & 3));
          const bool edge = qt.edge;
          int2 sees[8];                          // the eight queries' keys (asked for ahead of the wait; rows behind the last have probabilities of 0 anyway)
          if (edge) {
            if (a.ranges) {
#pragma unroll
              for (int e = 0; e < 8; ++e) sees[e] = a.ranges[(size_t)b * a.N + min(i0 + 8 * (e >> 1) + (e & 1), a.N - 1)];
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e) sees[e] = make_int2(0, a.N);
            }
            if (a.causal) {
#pragma unroll
              for (int e = 0; e < 8; ++e) sees[e].y = min(sees[e].y, i0 + 8 * (e >> 1) + (e & 1) + 1);
            }
          }
          alive = wait_all(s_full, sphase);
          if (alive) alive = wait_all(q_full + 8 * st, (idx >> 1) & 1u);   // (the rows' terms; long there)
          if (!alive) break;
          sphase ^= 1u;
          tc_fence_after();
          const uint32_t s_at = lane_base + kS + group * 32, dp_at = lane_base + kDP + group * 32;
          constexpr uint32_t kLanes16 = 16u << 16;
          float s[32];
          uint32_t u[16];
          tmem_ld_frag(s_at, s);
          tmem_ld_frag(s_at + kLanes16, s + 16);
          tmem_ld_wait32(s);
          if (CAP) tanh_scores_of_rows(a.cap_inv, s);
          dkv_probabilities<CAP, SLOPE, SCALED>(a.unit * kLog2e, slope, i0 - key0, rows_at, s, u);
          if (edge) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const bool on = key0 + 8 * y >= sees[e].x && key0 + 8 * y < sees[e].y;
                float& w = s[(y >> 1) * 16 + 4 * (e >> 1) + (y & 1) * 2 + (e & 1)];
                w = on ? w : 0.f;
                u[(y >> 1) * 8 + 2 * (e >> 1) + (y & 1)] &= on ? 0xffffffffu : (e & 1) ? 0x0000ffffu : 0xffff0000u;
              }
            }
          }
          // (both halves' scores have been read by the warp: the operands go over them, the lanes' 16 columns at the front of their 32)
          tmem_st_frag(s_at, u);
          tmem_st_frag(s_at + kLanes16, u + 8);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(p_full);
          alive = wait_all(dp_full, dpphase);
          if (!alive) break;
          dpphase ^= 1u;
          tc_fence_after();
          float dp[32];
          tmem_ld_frag(dp_at, dp);
          tmem_ld_frag(dp_at + kLanes16, dp + 16);
          float d[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) lds_f2(rows_at + 4 * (2 * kT) + 32 * k, d[2 * k], d[2 * k + 1]);
          tmem_ld_wait32(dp);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint64_t d2 = pack2(d[2 * k], d[2 * k + 1]);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int at = (y >> 1) * 16 + 4 * k + (y & 1) * 2;
              float x0, x1;
              unpack2(mul2(pack2(s[at], s[at + 1]), add2(pack2(dp[at], dp[at + 1]), d2)), x0, x1);
              u[(y >> 1) * 8 + 2 * k + (y & 1)] = bf16x2(x0, x1);
            }
          }
          tmem_st_frag(dp_at, u);
          tmem_st_frag(dp_at + kLanes16, u + 8);
          __syncwarp();
          if (lane == 0) mbar_arrive(r_empty + 8 * st);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(ds_full);
        }
      }
      if (!alive) break;
      if (any) {
        alive = wait_all(acc_full, accphase);
        if (!alive) break;
        accphase ^= 1u;
        tc_fence_after();
      }
#pragma unroll
      for (int which = 0; which < 2; ++which) {
        for (int c = group; c < HD / 32; c += kGroups) {
          const int col = c * 32;
          float v[32];
          if (any) {
            tmem_ld32(lane_base + (which ? kDV : kDK) + col, v);
            tmem_ld_wait();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0.f;
          }
          const entmax_attn_strides& s = which ? f.g.dv : f.g.dk;
          store_quad_rows(v, which ? 1.0f : kLn2 * a.sm_scale / a.unit,   // (the rows' a is c unit log2 e)
                          (which ? f.dv : f.dk) + (long long)b * s.b + (long long)kh * s.h + (long long)key * s.n + col, s.n, a.N - key);
        }
      }
      if (any) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(acc_empty);
      }
    }
  }
  bwd_teardown(tmem, abort_flag, drain_fail, f.status);
}

template <int HD>
cudaError_t bwd_launch(const BwdArgs& f, const void* q, const void* k, const void* v, const void* d_o, cudaStream_t stream) {
  const SoftmaxArgs& a = f.a;
  CUtensorMap map_q, map_k, map_v, map_do;
  cudaError_t err = make_tile_map(&map_q, q, a.D, a.N, a.H, a.B, a.q.n, a.q.h, a.q.b);
  if (err == cudaSuccess) err = make_tile_map(&map_k, k, a.D, a.N, a.KH, a.B, a.k.n, a.k.h, a.k.b);
  if (err == cudaSuccess) err = make_tile_map(&map_v, v, a.D, a.N, a.KH, a.B, a.v.n, a.v.h, a.v.b);
  if (err == cudaSuccess) err = make_tile_map(&map_do, d_o, a.D, a.N, a.H, a.B, f.g.d_o.n, f.g.d_o.h, f.g.d_o.b);
  if (err != cudaSuccess) return err;
  auto dq = [&](auto kernel) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BwdCfg<HD>::kSmemQ);
    return e != cudaSuccess ? e : launch_kernel(kernel, (unsigned)((long long)a.B * a.H * f.tiles), kDqThreads, BwdCfg<HD>::kSmemQ, stream, map_q, map_k, map_v,
                                                map_do, f);
  };
  auto dkv = [&](auto kernel) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, BwdCfg<HD>::kSmemKV);
    return e != cudaSuccess ? e : launch_kernel(kernel, (unsigned)((long long)a.B * a.KH * f.tiles), kBwdThreads, BwdCfg<HD>::kSmemKV, stream, map_q, map_k, map_v,
                                                map_do, f);
  };
  auto both = [&](auto cap, auto slope) {
    constexpr bool kCap = decltype(cap)::value, kSlope = decltype(slope)::value;
    const bool scaled = a.beta || a.c_rows;
    cudaError_t e;
    if (f.g.dc_rows) e = dq(softmax_dq_kernel<HD, kCap, kSlope, true, true>);
    else if (kSlope || scaled) e = dq(softmax_dq_kernel<HD, kCap, kSlope, true, false>);
    else e = dq(softmax_dq_kernel<HD, kCap, kSlope, kSlope, false>);   // (kSlope: not reached, and the same kernel as above)
    if (e != cudaSuccess) return e;
    return scaled ? dkv(softmax_dkv_kernel<HD, kCap, kSlope, true>) : dkv(softmax_dkv_kernel<HD, kCap, kSlope, false>);
  };
  using T = std::true_type;
  using F = std::false_type;
  if (a.cap_inv > 0.f) return a.alibi ? both(T{}, T{}) : both(T{}, F{});
  return a.alibi ? both(F{}, T{}) : both(F{}, F{});
}

}  // namespace

size_t softmax_bwd_rows_bytes(const SoftmaxArgs& a) { return (size_t)a.B * a.H * ((a.N + kT - 1) / kT) * (3 * kT) * 4; }
size_t softmax_bwd_spans_bytes(const SoftmaxArgs& a) { return (size_t)a.B * ((a.N + kT - 1) / kT) * 16; }

cudaError_t launch_softmax_bwd(const SoftmaxArgs& a, const SoftmaxGrads& g, const void* q, const void* k, const void* v, const void* o, const void* d_o,
                               void* dq, void* dk, void* dv, float* rows, void* spans, int32_t* status, cudaStream_t stream) {
  BwdArgs f = {};
  f.a = a;
  f.g = g;
  f.tiles = (a.N + kT - 1) / kT;
  f.o = static_cast<const __nv_bfloat16*>(o);
  f.d_o = static_cast<const __nv_bfloat16*>(d_o);
  f.dq = static_cast<__nv_bfloat16*>(dq);
  f.dk = static_cast<__nv_bfloat16*>(dk);
  f.dv = static_cast<__nv_bfloat16*>(dv);
  f.rows = rows;
  f.spans = static_cast<int4*>(spans);
  f.status = status;
  return a.D == 64 ? bwd_launch<64>(f, q, k, v, d_o, stream) : bwd_launch<128>(f, q, k, v, d_o, stream);
}

}  // namespace entmax
