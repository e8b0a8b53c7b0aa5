// Softmax attention of new tokens over a paged cache (entmax_attn_softmax_paged_fwd): the few rows of a sequence that generates, and the joins.
//
// Few rows (n new tokens x G query heads of a K/V head, 16, 32 or 64 at most): bound by reading K and V once from HBM, so the kernel is built around that
// stream.  The work is tiles of 64 keys of all sequences and K/V heads in a row; every CTA takes an equal run of them, whatever sequences it cuts (short
// sequences that fill the GPU anyway: a CTA for each K/V head of each).  A producer warp
// brings the tiles' pages by TMA (a box per page and 64 columns) three tiles ahead; four warps share the rows (16 each) or the keys of a tile, each with a
// running maximum and sum of its own: S = Q K^T and O += P V by m16n8k16 products with Q, P, O in registers (16 rows do not fill a tcgen05 tile, and
// at 8 flops a byte the stream is six times slower than these products).  The warps meet at the end of a run's sequence.  A sequence that lies in
// one run is finished there; the pieces of one that was cut go to the workspace and a second kernel joins them in order.
// Long chunks take the kernel of softmax_fwd_sm100.cu.
// 64 sequences of up to 4096 keys, 32/8 heads x 128: 115 to 117 us with the join, 5.5 TB/s (84 % of the copy rate); 8 of up to 65536, 32/4 heads: 115 us, 5.7 TB/s; 32 x 5 tokens
// over 8192 keys (20 rows, two groups): 204 us, 5.3 TB/s.
#include <cuda.h>

#include <cmath>
#include <type_traits>

#include "sm100_ptx.cuh"
#include "softmax_paged.cuh"
#include "softmax_tile.cuh"

namespace entmax {

struct FewPiece {          // where a cut sequence's pieces are: CTAs first (its second slot) .. last (their first)
  int b, kh, last, pad;    // b = -1: none begins here
};

namespace {

using namespace sm100;

constexpr int kTileKeys = 64;
constexpr int kFewStages = 3;
constexpr int kFewThreads = 160;                 // four warps of products, one producer
constexpr int kFewBars = 512;
constexpr int kSms = 148;                        // (sizes the workspace too, which is the same on every device)

template <int HD>
struct FewCfg {
  static constexpr int kHalves = HD / 64;
  static constexpr int kTile = kTileKeys * HD * 2;                   // K or V
  static constexpr int kStage = 2 * kTile;
  static constexpr int kMeet = 16 * HD * 4;                          // one warp's O
  static constexpr int kSmem = kFewStages * kStage + kMeet + kFewBars + 1024;
  static_assert(2 * (kSmem + 1024) <= 233472, "two CTAs on an SM");
};

struct FewWork {
  int valid, b, kh, q0, n, len, lo, hi;          // tiles lo .. hi - 1 of the sequence's
  int slot;                                      // -1: it has all of them; 0, 1: this CTA's piece
  int pad[3];
};

__device__ __forceinline__ bool sp_ok(const SoftmaxPagedArgs& a, const PagedSeq& s) { return s.len >= s.n && s.len <= a.max_kv && s.n <= a.max_q; }
// Tiles of 64 keys that the sequence's rows see: first, one behind the last
__device__ __forceinline__ int2 few_tiles(const SoftmaxPagedArgs& a, const PagedSeq& s) {
  if (s.n == 0 || !sp_ok(a, s) || (long long)s.n * a.G > a.few_rows) return make_int2(0, 0);
  const int first = a.window > 0 ? max(0, s.len - s.n - a.window + 1) : 0;
  return make_int2(first / kTileKeys, (s.len + kTileKeys - 1) / kTileKeys);
}

__device__ __forceinline__ void ldsm4(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared::cta.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t at, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared::cta.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(at) : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// RG: groups of 16 rows (1, 2, 4) that sequences have at most; the warps share the rows of one in as few groups as it fills, and the 4 / groups warps of a
// group a tile's keys
template <int HD, int RG>
__global__ void __launch_bounds__(kFewThreads, 2) softmax_few_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                     const __grid_constant__ SoftmaxPagedArgs a) {
  pdl_begin();
  using C = FewCfg<HD>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t sbase = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t meet = sbase + kFewStages * C::kStage;
  const uint32_t bars = meet + C::kMeet;
  const uint32_t full = bars, empty = bars + 8 * kFewStages;
  const uint32_t w_full = bars + 48, w_empty = bars + 64, x_bar = bars + 80, abort_flag = bars + 88, drain_fail = bars + 92;
  const uint32_t work_at = bars + 96;            // FewWork [2]
  const uint32_t stats = bars + 192;             // float2 [4][8]: maximum and sum of a warp's rows (lane / 4), in two rounds
  const FewWork* work = reinterpret_cast<const FewWork*>(smem_raw + (work_at - smem_u32(smem_raw)));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int st = 0; st < kFewStages; ++st) { mbar_init(full + 8 * st, 1); mbar_init(empty + 8 * st, 4); }
    for (int t = 0; t < 2; ++t) { mbar_init(w_full + 8 * t, 1); mbar_init(w_empty + 8 * t, 4); }
    mbar_init(x_bar, 4);
    sts_u32(abort_flag, 0u);
    sts_u32(drain_fail, 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  __syncthreads();
  auto wait_all = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };

  if (warp == 4) {
    // ------------------------------------------------------------------ which tiles are this CTA's, and their way into shared memory
    long long total = 0, ctas = 1, begin = 0, end = 0;
    if (a.whole) {
      const int2 t = few_tiles(a, paged_seq(a.c, blockIdx.x / a.c.KH));
      begin = (long long)(blockIdx.x % a.c.KH) * (t.y - t.x);
      end = begin + (t.y - t.x);
    } else {
      for (int b = lane; b < a.c.B; b += 32) {
        const int2 t = few_tiles(a, paged_seq(a.c, b));
        total += t.y - t.x;
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
      total *= a.c.KH;
      ctas = min((long long)gridDim.x, total);                       // (each of them gets a tile: no gaps between a sequence's pieces)
      begin = blockIdx.x < ctas ? total * blockIdx.x / ctas : 0;
      end = blockIdx.x < ctas ? total * (blockIdx.x + 1) / ctas : 0;
      if (lane == 0) a.pieces[blockIdx.x] = FewPiece{-1, 0, 0, 0};
    }
    uint32_t wphase = 0, idx = 0;
    int slot = 0;
    bool alive = true;
    if (begin < end) {
      // the sequence of the first tile: 32 sequences at a time
      long long before = 0;                      // tiles (of all K/V heads) in front of sequence b
      int b = a.whole ? blockIdx.x / a.c.KH : 0;
      for (int b0 = 0; !a.whole && b0 < a.c.B; b0 += 32) {
        const int2 t = b0 + lane < a.c.B ? few_tiles(a, paged_seq(a.c, b0 + lane)) : make_int2(0, 0);
        const long long mine = (long long)(t.y - t.x) * a.c.KH;
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const long long up = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += up;
        }
        const unsigned past = __ballot_sync(0xffffffffu, before + incl > begin);
        if (past) {
          const int l = __ffs(past) - 1;
          before += __shfl_sync(0xffffffffu, incl - mine, l);
          b = b0 + l;
          break;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
      }
      long long at = begin;
      while (alive && at < end) {
        const PagedSeq s = paged_seq(a.c, b);
        const int2 t = few_tiles(a, s);
        const int tiles = t.y - t.x;
        for (int kh = tiles ? (int)((at - before) / tiles) : a.c.KH; kh < a.c.KH && alive && at < end; ++kh) {
          const long long unit = before + (long long)kh * tiles;
          const int from = (int)(at - unit), to = (int)min((long long)tiles, end - unit);
          FewWork w = {1, b, kh, s.q0, s.n, s.len, t.x + from, t.x + to, -1, {0, 0, 0}};
          if (from > 0) w.slot = 0;
          else if (to < tiles) {
            w.slot = 1;
            // the last CTA that has tiles of it
            if (lane == 0) a.pieces[blockIdx.x] = FewPiece{b, kh, (int)(((unit + tiles) * ctas + total - 1) / total - 1), 0};
          }
          alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
          if (!alive) break;
          if (lane == 0) {
            *const_cast<FewWork*>(work + slot) = w;
            mbar_arrive(w_full + 8 * slot);
          }
          __syncwarp();
          if (++slot == 2) { slot = 0; wphase ^= 1u; }
          const int first_key = a.window > 0 ? max(0, s.len - s.n - a.window + 1) : 0;
          // lane x looks after box x of a tile, one tile ahead (-2: nothing to load)
          auto look_up = [&](int j) -> int {
            const int key = j * kTileKeys + (lane << a.box_shift);
            if (j >= w.hi || lane >= (kTileKeys >> a.box_shift) || key >= s.len || key + (1 << a.box_shift) <= first_key) return -2;
            int p = a.c.table[(long long)b * a.c.table_stride + (key >> a.c.ps_shift)];
            if ((unsigned)p >= (unsigned)a.c.n_pages) {                // (read as zeros)
              if (a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_PAGE);
              p = a.c.n_pages;
            }
            return p;
          };
          int page_next = look_up(w.lo);
          for (int j = w.lo; j < w.hi; ++j, ++idx) {
            const int page = page_next;
            page_next = look_up(j + 1);
            const uint32_t st = idx % kFewStages;
            alive = wait_all(empty + 8 * st, ((idx / kFewStages) & 1u) ^ 1u);
            if (!alive) break;
            const int boxes = __popc(__ballot_sync(0xffffffffu, page >= 0));
            if (lane == 0) mbar_expect_tx(full + 8 * st, (boxes * (2 * C::kHalves * 128)) << a.box_shift);
            __syncwarp();
            if (page >= 0) {
              const int slot0 = (j * kTileKeys + (lane << a.box_shift)) & ((1 << a.c.ps_shift) - 1);
              for (int hf = 0; hf < C::kHalves; ++hf) {
                const uint32_t dst = sbase + st * C::kStage + hf * (kTileKeys * 128) + (lane << (a.box_shift + 7));
                tma_load_4d(dst, &map_k, full + 8 * st, hf * 64, slot0, kh, page);
                tma_load_4d(dst + C::kTile, &map_v, full + 8 * st, hf * 64, slot0, kh, page);
              }
            }
            __syncwarp();
          }
          at = unit + to;
        }
        before += (long long)tiles * a.c.KH;
        ++b;
      }
    }
    if (alive) {
      alive = wait_all(w_empty + 8 * slot, wphase ^ 1u);
      if (alive && lane == 0) {
        const_cast<FewWork*>(work + slot)->valid = 0;
        mbar_arrive(w_full + 8 * slot);
      }
    }
    if (!alive && lane == 0) {
      bool ok = true;
      for (uint32_t st = 0; st < kFewStages; ++st)
        ok &= mbar_drain(full + 8 * st, ((idx / kFewStages + (st < idx % kFewStages ? 1u : 0u)) & 1u) ^ 1u);
      if (!ok) sts_u32(drain_fail, 1u);
    }
  } else {
    // the rows of sequences that cannot be served at all
    for (int b = blockIdx.x; b < a.c.B; b += gridDim.x) {
      const PagedSeq s = paged_seq(a.c, b);
      if (s.n == 0 || sp_ok(a, s)) continue;
      if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_LENGTH);
      const long long rows = (long long)s.n * a.H;
      for (long long r = threadIdx.x; r < rows; r += 128) a.lse[(long long)s.q0 * a.H + r] = -INFINITY;
      uint4* o = reinterpret_cast<uint4*>(a.o + (long long)s.q0 * a.H * HD);
      for (long long e = threadIdx.x; e < rows * (HD / 8); e += 128) o[e] = make_uint4(0u, 0u, 0u, 0u);
    }
    uint32_t wphase = 0, xphase = 0, idx = 0;
    int slot = 0;
    auto serve = [&](const FewWork& w, auto groups) -> bool {
      constexpr int RGS = decltype(groups)::value;
      constexpr int KG = 4 / RGS;                // warps that share the keys
      constexpr int NT = kTileKeys / KG / 8;     // eight-key columns of a warp
      const int rg = warp % RGS, kg = warp / RGS;
      const int r0 = rg * 16 + (lane >> 2);      // this thread's rows: r0, r0 + 8
      bool alive = true;
      const int rows = w.n * a.G;
      uint32_t q[HD / 16][4];
      float scale[2], slope[2], top[2] = {-INFINITY, -INFINITY}, mass[2] = {0.f, 0.f}, out[HD / 8][4];
      int pos[2], begin[2];
      bool flip[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const int r = r0 + 8 * y;
        const bool mine = r < rows;
        const int t = mine ? r / a.G : 0, h = w.kh * a.G + (mine ? r - t * a.G : 0);
        const __nv_bfloat16* src = a.q + (long long)(w.q0 + t) * a.q_st + (long long)h * a.q_sh + 2 * (lane & 3);
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
          q[kk][y] = mine ? *reinterpret_cast<const uint32_t*>(src + 16 * kk) : 0u;
          q[kk][2 + y] = mine ? *reinterpret_cast<const uint32_t*>(src + 16 * kk + 8) : 0u;
        }
        pos[y] = w.len - w.n + t;
        begin[y] = a.window > 0 ? max(0, pos[y] - a.window + 1) : 0;
        const float c = a.beta ? length_scale(a.beta[h], a.gamma[h], a.delta[h], pos[y] + 1 - begin[y]) : 1.0f;
        if (a.beta && a.status && mine && !isfinite(c)) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_SCALE);
        flip[y] = c < 0.f;
        scale[y] = at_least_tiny(fabsf(c * a.unit * kLog2e));    // (see RowSoftmax)
        slope[y] = a.alibi ? a.alibi[h] / a.unit : 0.f;
      }
#pragma unroll
      for (int e = 0; e < HD / 8; ++e)
#pragma unroll
        for (int z = 0; z < 4; ++z) out[e][z] = 0.f;
      const int first_key = a.window > 0 ? max(0, w.len - w.n - a.window + 1) : 0;
      const int all_from = a.window > 0 ? max(0, w.len - a.window) : 0, all_to = w.len - w.n + 1;   // every row sees the keys in between
      for (int j = w.lo; j < w.hi && alive; ++j, ++idx) {
        const uint32_t st = idx % kFewStages;
        alive = wait_all(full + 8 * st, (idx / kFewStages) & 1u);
        if (!alive) break;
        const uint32_t k_at = sbase + st * C::kStage, v_at = k_at + C::kTile;
        const int key0 = kg * (8 * NT);          // this warp's keys of the tile
        const int k0 = j * kTileKeys + key0;
        const bool edge = k0 < all_from || k0 + 8 * NT > all_to;
        float s[NT][4];
#pragma unroll
        for (int e = 0; e < NT; ++e)
#pragma unroll
          for (int z = 0; z < 4; ++z) s[e][z] = 0.f;
        // matrices of a load: keys 0..7 and 8..15 of 16, elements 0..7 and 8..15 of 16; a 16-byte unit u of row r lies at unit u ^ (r % 8)
#pragma unroll
        for (int kk = 0; kk < HD / 16; ++kk) {
#pragma unroll
          for (int e = 0; e < NT; e += 2) {
            const int row = key0 + 8 * e + (lane & 7) + ((lane >> 4) << 3), unit = (kk & 3) * 2 + ((lane >> 3) & 1);
            uint32_t b0, b1, b2, b3;
            ldsm4(k_at + (kk >> 2) * (kTileKeys * 128) + row * 128 + ((unit ^ (row & 7)) << 4), b0, b1, b2, b3);
            mma16816(s[e], q[kk], b0, b1);
            mma16816(s[e + 1], q[kk], b2, b3);
          }
        }
        if (a.cap_inv > 0.f) {
          if (edge) {                            // (what lies in an unseen slot has no say in how the tanh is computed)
#pragma unroll
            for (int e = 0; e < NT; ++e)
#pragma unroll
              for (int z = 0; z < 4; ++z) {
                const int key = k0 + 8 * e + 2 * (lane & 3) + (z & 1);
                s[e][z] = key >= begin[z >> 1] && key <= pos[z >> 1] ? s[e][z] : 0.f;
              }
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {          // a row at a time
            float x[2 * NT];
#pragma unroll
            for (int e = 0; e < NT; ++e) { x[2 * e] = s[e][2 * y]; x[2 * e + 1] = s[e][2 * y + 1]; }
            tanh_scores(a.cap_inv, x);
#pragma unroll
            for (int e = 0; e < NT; ++e) { s[e][2 * y] = x[2 * e]; s[e][2 * y + 1] = x[2 * e + 1]; }
          }
        }
        float most[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < NT; ++e) {
          const int key = k0 + 8 * e + 2 * (lane & 3);
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const int y = z >> 1;
            float x = fmaf(-slope[y], (float)(pos[y] - key - (z & 1)), s[e][z]);
            x = flip[y] ? -x : x;
            if (edge) x = key + (z & 1) >= begin[y] && key + (z & 1) <= pos[y] ? x : -INFINITY;
            s[e][z] = x;
            most[y] = fmaxf(most[y], x);
          }
        }
        float base[2];
        bool rises = false;
        float old[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          most[y] = fmaxf(most[y], __shfl_xor_sync(0xffffffffu, most[y], 1));
          most[y] = fmaxf(most[y], __shfl_xor_sync(0xffffffffu, most[y], 2));
          old[y] = 1.0f;
          if (most[y] > top[y]) {
            old[y] = exp2_fast((top[y] - most[y]) * scale[y]);
            top[y] = most[y];
            mass[y] *= old[y];
            rises = true;
          }
          base[y] = top[y] > -INFINITY ? top[y] * scale[y] : 0.f;
        }
        if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
          for (int e = 0; e < HD / 8; ++e)
#pragma unroll
            for (int z = 0; z < 4; ++z) out[e][z] *= old[z >> 1];
        }
        uint32_t p[NT / 2][4];
#pragma unroll
        for (int e = 0; e < NT; ++e) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float p0 = exp2_fast(fmaf(s[e][2 * y], scale[y], -base[y])), p1 = exp2_fast(fmaf(s[e][2 * y + 1], scale[y], -base[y]));
            mass[y] += p0 + p1;
            p[e >> 1][(e & 1) * 2 + y] = bf16x2(p0, p1);
          }
        }
        // O += P V.  Slots no row sees may hold anything, and a NaN times a probability of 0 is one too: their entries are taken for 0 in the registers.
        auto add_values = [&](auto some_unseen) {
#pragma unroll
          for (int kk = 0; kk < NT / 2; ++kk) {
            const int row = key0 + 16 * kk + (lane & 7) + (((lane >> 3) & 1) << 3);
            uint32_t m0 = 0xffffffffu, m1 = 0xffffffffu;
            if (decltype(some_unseen)::value) {
              auto seen = [&](int key) -> uint32_t {
                return (key >= first_key && key < w.len ? 0x0000ffffu : 0u) | (key + 1 >= first_key && key + 1 < w.len ? 0xffff0000u : 0u);
              };
              m0 = seen(k0 + 16 * kk + 2 * (lane & 3));
              m1 = seen(k0 + 16 * kk + 2 * (lane & 3) + 8);
            }
#pragma unroll
            for (int e = 0; e < HD / 8; e += 2) {
              const int unit = (e & 7) + (lane >> 4);
              uint32_t b0, b1, b2, b3;
              ldsm4_t(v_at + (e >> 3) * (kTileKeys * 128) + row * 128 + ((unit ^ (row & 7)) << 4), b0, b1, b2, b3);
              if (decltype(some_unseen)::value) { b0 &= m0; b1 &= m1; b2 &= m0; b3 &= m1; }
              mma16816(out[e], p[kk], b0, b1);
              mma16816(out[e + 1], p[kk], b2, b3);
            }
          }
        };
        if (k0 < first_key || k0 + 8 * NT > w.len) add_values(std::true_type{});
        else add_values(std::false_type{});
        __syncwarp();
        if (lane == 0) mbar_arrive(empty + 8 * st);
      }
      if (!alive) return false;
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        mass[y] += __shfl_xor_sync(0xffffffffu, mass[y], 1);
        mass[y] += __shfl_xor_sync(0xffffffffu, mass[y], 2);
      }
      // the warps that shared the keys, one after the other into the first of them
      auto meet_all = [&]() -> bool {
        __syncwarp();
        if (lane == 0) mbar_arrive(x_bar);
        const bool ok = wait_all(x_bar, xphase);
        xphase ^= 1u;
        return ok;
      };
#pragma unroll 1
      for (int other = 1; other < KG && alive; ++other) {
        // (RGS > 1: the groups' first warps take turns at the room for one O)
#pragma unroll 1
        for (int turn = 0; turn < RGS && alive; ++turn) {
          if (rg == turn && kg == other) {
#pragma unroll
            for (int e = 0; e < HD / 8; ++e) {
              const uint32_t to = meet + (uint32_t)(e * 32 + lane) * 16;
              sts_f4(to, out[e][0], out[e][1], out[e][2], out[e][3]);
            }
            if ((lane & 3) == 0) sts_f4(stats + (lane >> 2) * 16, top[0], mass[0], top[1], mass[1]);
          }
          alive = meet_all();
          if (!alive) break;
          if (rg == turn && kg == 0) {
            float t[2], m[2];
            lds_f4(stats + (lane >> 2) * 16, t[0], m[0], t[1], m[1]);
            float mine[2], theirs[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const float now = fmaxf(top[y], t[y]), at = now > -INFINITY ? now : 0.f;
              mine[y] = exp2_fast((top[y] - at) * scale[y]);
              theirs[y] = exp2_fast((t[y] - at) * scale[y]);
              top[y] = now;
              mass[y] = mass[y] * mine[y] + m[y] * theirs[y];
            }
#pragma unroll
            for (int e = 0; e < HD / 8; ++e) {
              float x[4];
              lds_f4(meet + (uint32_t)(e * 32 + lane) * 16, x[0], x[1], x[2], x[3]);
#pragma unroll
              for (int z = 0; z < 4; ++z) out[e][z] = out[e][z] * mine[z >> 1] + x[z] * theirs[z >> 1];
            }
          }
          alive = meet_all();
        }
      }
      if (!alive) return false;
      if (kg == 0) {
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int r = r0 + 8 * y;
          if (r >= rows) continue;
          const float base = top[y] > -INFINITY ? top[y] * scale[y] : -INFINITY;   // in base-2 units
          if (w.slot < 0) {
            const int t = r / a.G, h = w.kh * a.G + r - t * a.G;
            const size_t at = (size_t)(w.q0 + t) * a.H + h;
            const float inv = 1.0f / mass[y];
            if ((lane & 3) == 0) a.lse[at] = (base + log2f(mass[y])) * kLn2;
#pragma unroll
            for (int e = 0; e < HD / 8; ++e)
              *reinterpret_cast<uint32_t*>(a.o + at * HD + 8 * e + 2 * (lane & 3)) = bf16x2(out[e][2 * y] * inv, out[e][2 * y + 1] * inv);
          } else {
            const size_t at = ((size_t)blockIdx.x * 2 + w.slot) * (16 * RG) + r;
            if ((lane & 3) == 0) a.part_ml[at] = make_float2(base, mass[y]);
#pragma unroll
            for (int e = 0; e < HD / 8; ++e)
              *reinterpret_cast<float2*>(a.part_o + at * HD + 8 * e + 2 * (lane & 3)) = make_float2(out[e][2 * y], out[e][2 * y + 1]);
          }
        }
      }
      return true;
    };
    bool alive = true;
    while (alive) {
      alive = wait_all(w_full + 8 * slot, wphase);
      if (!alive) break;
      const FewWork w = work[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(w_empty + 8 * slot);
      if (++slot == 2) { slot = 0; wphase ^= 1u; }
      if (!w.valid) break;
      const int rows = w.n * a.G;
      if (rows <= 16) alive = serve(w, std::integral_constant<int, 1>{});
      else if (rows <= 32 || RG < 4) alive = serve(w, std::integral_constant<int, RG < 2 ? RG : 2>{});
      else alive = serve(w, std::integral_constant<int, RG>{});
    }
  }
  __syncthreads();
  if (lds_u32(abort_flag)) {
    if (threadIdx.x == 0 && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_WAIT_EXPIRED);
    if (lds_u32(drain_fail)) {
      const uint64_t t0 = global_ns();
      while (global_ns() - t0 < 200000ull) { }
    }
  }
}

// One row from `count` pieces: sum_p 2^(m_p - M) O_p over the sum of 2^(m_p - M) l_p, by a warp.  at(p): the row's place among the pieces.  Pieces without a key that the row
// sees have l = 0; one whose l is NaN makes the row NaN, as it does where nothing is cut.
template <int HD, typename At>
__device__ __forceinline__ void join_row(const float* part_o, const float2* part_ml, int count, At at, __nv_bfloat16* o, float* lse) {
  const int lane = threadIdx.x & 31;
  float most = -INFINITY;
  for (int p = lane; p < count; p += 32) {
    const float2 ml = part_ml[at(p)];
    if (ml.y != 0.f) most = fmaxf(most, ml.x);
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
  constexpr int E = HD / 32;
  float sum = 0.f, out[E] = {};
  for (int p = 0; p < count; ++p) {
    const size_t x = at(p);
    const float2 ml = part_ml[x];
    const float f = ml.y != 0.f ? exp2_fast(ml.x - most) : 0.f;
    sum = fmaf(ml.y, f, sum);
    float v[E];
    load_slice<E>(part_o + x * HD + lane * E, v);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = ml.y != 0.f ? fmaf(v[e], f, out[e]) : out[e];
  }
  const float inv = sum != 0.f ? 1.0f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) out[e] *= inv;
  store_slice<E>(o + lane * E, out);
  if (lane == 0) *lse = sum != 0.f ? (most + log2f(sum)) * kLn2 : -INFINITY;
}

// The sequences that were cut: CTA x joins the one that begins in CTA x's run without ending there, a warp per row
template <int HD, int RG>
__global__ void __launch_bounds__(128) softmax_few_join_kernel(const __grid_constant__ SoftmaxPagedArgs a) {
  pdl_begin();
  const int first = blockIdx.x;
  const FewPiece piece = a.pieces[first];
  if (piece.b < 0) return;
  const PagedSeq s = paged_seq(a.c, piece.b);
  const int r = blockIdx.y * 4 + (threadIdx.x >> 5);
  if (r >= s.n * a.G) return;
  const int t = r / a.G, h = piece.kh * a.G + r - t * a.G;
  const size_t to = (size_t)(s.q0 + t) * a.H + h;
  join_row<HD>(a.part_o, a.part_ml, piece.last - first + 1,
               [&](int p) { return ((size_t)(first + p) * 2 + (p == 0 ? 1 : 0)) * (16 * RG) + r; }, a.o + to * HD, a.lse + to);
}

// The chunks whose keys were shared out: a warp per row
template <int HD>
__global__ void __launch_bounds__(128) softmax_chunk_join_kernel(const __grid_constant__ SoftmaxPagedArgs a) {
  pdl_begin();
  const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= (long long)a.c.T * a.H) return;
  const int t = (int)(row / a.H), h = (int)(row - (long long)t * a.H);
  const int b = a.c.cu_q ? find_seq(a.c, t) : t / (a.c.T / a.c.B);
  const PagedSeq s = paged_seq(a.c, b);
  if (t < s.q0 || t >= s.q0 + s.n || !sp_ok(a, s) || (long long)s.n * a.G <= a.few_rows) return;
  const ChunkPlace at = chunk_place(a.c, a.G, b, t - s.q0, h);
  const size_t first = ((size_t)at.unit * a.shares * 2 + at.tile) * 128 + at.row;
  join_row<HD>(a.chunk_o, a.chunk_ml, a.shares, [&](int p) { return first + (size_t)p * 256; }, a.o + row * HD, a.lse + row);
}

constexpr size_t kChunkBytes = 256u << 20;       // most scratch for shared-out chunks

struct PagedPlan {
  int rg;                   // row groups of the "few" kernel: 16 rg rows
  int few_ctas;
  bool chunks;              // whether a sequence may have more rows than that
  long long units;          // blocks x K/V heads x pairs
  size_t pieces, part_ml, part_o, chunk_ml, chunk_o, bytes;
};
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

int softmax_paged_args(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* p, int uniform, SoftmaxPagedArgs* out,
                       PagedPlan* plan) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  SoftmaxPagedArgs a = {};
  int rc = check_paged_cache(cache, p->total_q, &a.c);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (p->q_heads < 1 || p->q_heads % a.c.KH || p->q_heads / a.c.KH > 128 || (long long)p->total_q * p->q_heads > 0x7fffffffLL / 2)
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->max_q_len < 0 || p->max_kv_len < 0 || p->window < 0) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (uniform && p->total_q % a.c.B) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->q_stride_t < a.c.D || p->q_stride_h < a.c.D || p->q_stride_t % 8 || p->q_stride_h % 8) return ENTMAX_ATTN_EINVAL_SHAPE;
  a.H = p->q_heads;
  a.G = a.H / a.c.KH;
  a.window = p->window;
  rc = softmax_unit(p->sm_scale, p->softcap, a.c.D, &a.sm_scale, &a.cap_inv, &a.unit);
  if (rc != ENTMAX_ATTN_OK) return rc;
  const int most_kv = a.c.max_pages << a.c.ps_shift;
  a.max_kv = p->max_kv_len > 0 && p->max_kv_len < most_kv ? p->max_kv_len : most_kv;
  const int most_q = uniform ? p->total_q / a.c.B : p->total_q;
  a.max_q = p->max_q_len > 0 && p->max_q_len < most_q ? p->max_q_len : most_q;
  a.q_st = p->q_stride_t; a.q_sh = p->q_stride_h;
  a.box_shift = a.c.ps_shift < 6 ? a.c.ps_shift : 6;

  // Sizes and launches go by the call's bounds alone (the lengths are device data).  Row groups: as many as the longest chunk fills, or, where chunks are longer than
  // 64 rows anyway, as the average one does.
  PagedPlan w = {};
  const long long rows = (long long)a.max_q * a.G;
  const long long typical = rows <= 64 ? rows : ((long long)p->total_q + a.c.B - 1) / a.c.B * a.G;
  w.rg = typical <= 16 ? 1 : typical <= 32 ? 2 : 4;
  a.few_rows = 16 * w.rg;
  w.chunks = rows > a.few_rows;
  // two CTAs per SM, but four tiles for each at least
  const long long keys = a.window > 0 && (long long)a.window + a.max_q < a.max_kv ? (long long)a.window + a.max_q : a.max_kv;
  const long long tiles = (long long)a.c.B * a.c.KH * ((keys + kTileKeys - 1) / kTileKeys);
  const long long ctas = (tiles + 3) / 4;
  w.few_ctas = (int)(ctas < 2 * kSms ? (ctas > 0 ? ctas : 1) : 2 * kSms);
  // A CTA per sequence and K/V head, nothing cut and nothing to join, where it has at most nine tiles more than its equal share: cutting costs a launch, a second
  // meeting of the warps and the join, about as much as they do.  12 heads x 64 over 400 keys (3 more) 9.3 us against 12.2 cut, 777 (9) 13.2 against 12.4 and
  // 2 us less on the host, 1024 (12) 14.9 against 10.6; 256 units x 128 over 1024 keys (2) 26.5 against 33.1, lengths of 1 to 1024 21.7 against 30.3,
  // 64 units (13) 20.2 against 13.9.  32 tiles at most: with one long sequence among short ones the others would wait for it.
  const long long units = (long long)a.c.B * a.c.KH, unit_tiles = (keys + kTileKeys - 1) / kTileKeys, share = units * unit_tiles / (2 * kSms);
  a.whole = units <= 2 * kSms && unit_tiles <= 32 && unit_tiles - (share > 4 ? share : 4) <= 9;
  if (a.whole) w.few_ctas = (int)units;
  const size_t few_slots = a.whole ? 0 : (size_t)w.few_ctas * 2 * a.few_rows;
  w.pieces = 0;
  w.part_ml = w.pieces + up256((size_t)w.few_ctas * sizeof(FewPiece));
  w.part_o = w.part_ml + up256(few_slots * sizeof(float2));
  w.bytes = w.part_o + up256(few_slots * a.c.D * sizeof(float));
  a.shares = 1;
  if (w.chunks) {
    const int block = chunk_block(a.G);
    const long long per_block = (long long)a.c.KH * chunk_pairs(a.G);
    w.units = ((long long)a.c.T / block + a.c.B) * per_block;
    // few blocks over many keys: their keys are shared out, 512 to an item at least
    const long long real = ((long long)a.c.T + block - 1) / block * per_block;
    long long shares = kSms / real;
    const long long by_keys = keys / 512, by_room = (long long)(kChunkBytes / ((size_t)w.units * 256 * (a.c.D * 4 + 8)));
    if (shares > by_keys) shares = by_keys;
    if (shares > by_room) shares = by_room;
    if (w.units * (shares > 1 ? shares : 1) > 0x7fffffffLL) return ENTMAX_ATTN_EINVAL_SHAPE;
    if (shares > 1) {
      a.shares = (int)shares;
      const size_t slots = (size_t)w.units * shares * 256;
      w.chunk_ml = w.bytes;
      w.chunk_o = w.chunk_ml + up256(slots * sizeof(float2));
      w.bytes = w.chunk_o + up256(slots * a.c.D * sizeof(float));
    }
  }
  *out = a;
  *plan = w;
  return ENTMAX_ATTN_OK;
}

// the pool as (D, slot, K/V head, page)
cudaError_t map_pool(CUtensorMap* map, const SoftmaxPagedArgs& a, const void* pool, int box_shift) {
  return make_box_map(map, pool, a.c.D, 1 << a.c.ps_shift, a.c.KH, a.c.n_pages, a.c.s_tok, a.c.s_head, a.c.s_page, 1 << box_shift, 1);
}

template <int HD, int RG>
cudaError_t few_launch(const SoftmaxPagedArgs& a, const PagedPlan& w, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t stream) {
  cudaError_t err = cudaFuncSetAttribute(softmax_few_kernel<HD, RG>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewCfg<HD>::kSmem);
  if (err != cudaSuccess) return err;
  err = launch_kernel(softmax_few_kernel<HD, RG>, (unsigned)w.few_ctas, kFewThreads, FewCfg<HD>::kSmem, stream, map_k, map_v, a);
  if (err != cudaSuccess || a.whole) return err;
  return launch_kernel(softmax_few_join_kernel<HD, RG>, dim3((unsigned)w.few_ctas, 4 * RG), 128, 0, stream, a);
}
template <int HD>
cudaError_t paged_launch(SoftmaxPagedArgs a, const PagedPlan& w, const void* k, const void* v, cudaStream_t stream) {
  CUtensorMap map_k, map_v;
  cudaError_t err = map_pool(&map_k, a, k, a.box_shift);
  if (err == cudaSuccess) err = map_pool(&map_v, a, v, a.box_shift);
  if (err == cudaSuccess)
    err = w.rg == 1 ? few_launch<HD, 1>(a, w, map_k, map_v, stream)
                    : w.rg == 2 ? few_launch<HD, 2>(a, w, map_k, map_v, stream) : few_launch<HD, 4>(a, w, map_k, map_v, stream);
  if (err != cudaSuccess || !w.chunks) return err;
  a.box_shift = a.c.ps_shift < 7 ? a.c.ps_shift : 7;
  err = map_pool(&map_k, a, k, a.box_shift);
  if (err == cudaSuccess) err = map_pool(&map_v, a, v, a.box_shift);
  if (err == cudaSuccess) err = launch_softmax_chunks(a, map_k, map_v, stream);
  if (err != cudaSuccess || a.shares == 1) return err;
  return launch_kernel(softmax_chunk_join_kernel<HD>, (unsigned)(((long long)a.c.T * a.H + 3) / 4), 128, 0, stream, a);
}

}  // namespace

}  // namespace entmax

using namespace entmax;

extern "C" size_t entmax_attn_softmax_paged_workspace_bytes(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* params,
                                                            int uniform) {
  SoftmaxPagedArgs a;
  PagedPlan w;
  return softmax_paged_args(cache, params, uniform, &a, &w) == ENTMAX_ATTN_OK ? w.bytes : 0;
}

extern "C" int entmax_attn_softmax_paged_fwd(const entmax_attn_paged_cache* cache, const entmax_attn_softmax_paged_params* params, const void* q,
                                             const void* k_cache, const void* v_cache, const int32_t* cu_q, const int32_t* kv_len,
                                             const int32_t* block_table, const float* beta, const float* gamma, const float* delta,
                                             const float* alibi_slopes, void* o, float* lse, void* workspace, size_t workspace_bytes,
                                             int32_t* device_status, void* cuda_stream) {
  SoftmaxPagedArgs a;
  PagedPlan w;
  int rc = softmax_paged_args(cache, params, cu_q == nullptr, &a, &w);
  if (rc != ENTMAX_ATTN_OK) return rc;
  if (!q || !k_cache || !v_cache || !kv_len || !block_table || !o || !lse) return ENTMAX_ATTN_EINVAL_NULL;
  const int given = (beta != nullptr) + (gamma != nullptr) + (delta != nullptr);
  if (given != 0 && given != 3) return ENTMAX_ATTN_EINVAL_NULL;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return ENTMAX_ATTN_EINVAL_ALIGN;
  const uintptr_t words = reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(block_table) |
                          reinterpret_cast<uintptr_t>(beta) | reinterpret_cast<uintptr_t>(gamma) | reinterpret_cast<uintptr_t>(delta) |
                          reinterpret_cast<uintptr_t>(alibi_slopes) | reinterpret_cast<uintptr_t>(lse);
  if (words & 3u) return ENTMAX_ATTN_EINVAL_ALIGN;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) || workspace_bytes < w.bytes) return ENTMAX_ATTN_EINVAL_WORKSPACE;
  if ((rc = check_device_for_bf16()) != ENTMAX_ATTN_OK) return rc;
  a.c.table = block_table; a.c.kv_len = kv_len; a.c.cu_q = cu_q;
  a.beta = beta; a.gamma = gamma; a.delta = delta; a.alibi = alibi_slopes;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.v = static_cast<const __nv_bfloat16*>(v_cache);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.status = device_status;
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  a.pieces = reinterpret_cast<FewPiece*>(ws + w.pieces);
  a.part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
  a.part_o = reinterpret_cast<float*>(ws + w.part_o);
  if (a.shares > 1) {
    a.chunk_ml = reinterpret_cast<float2*>(ws + w.chunk_ml);
    a.chunk_o = reinterpret_cast<float*>(ws + w.chunk_o);
  }
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t err;
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  err = a.c.D == 64 ? paged_launch<64>(a, w, k_cache, v_cache, stream) : paged_launch<128>(a, w, k_cache, v_cache, stream);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
