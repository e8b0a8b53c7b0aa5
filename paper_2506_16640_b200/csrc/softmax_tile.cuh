// Element code of the tensor-core kernels of softmax attention: scores of a tile to probabilities.
#pragma once

#include "sm100_ptx.cuh"
#include "softmax.cuh"

namespace entmax {

// Low descriptor word of a tile of 128 rows x 64-element blocks read with its 128-byte rows along K and the row's elements along N (or M), 128-byte
// swizzle: atoms of eight rows repeat every 1024 bytes, 64-element blocks every 128 * 128 bytes.
__device__ __forceinline__ uint32_t mn_desc_lo(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | ((uint32_t)((128 * 128) >> 4) << 16); }

// Rows of a tile that lie one to a lane, 16 32-bit words (64 bytes) of each, to memory: the four lanes of a quad swap 16-byte pieces, so that a store fills
// 64 bytes of eight rows and not 16 of 32, each in a line of its own (32 passes of the load/store unit to an instruction: 2 us of every 128 x 64 tile of two
// gradients).  By the whole warp.  own: where this lane's row has them; pitch: bytes to the next row; left: rows that exist from this lane's on.
__device__ __forceinline__ void store_quad_rows(uint32_t (&w)[16], void* own, long long pitch, int left) {
  const int l = threadIdx.x & 3;
  // a 4 x 4 transpose of pieces: row l's piece k goes to lane k as its row l's
#pragma unroll
  for (int bit = 1; bit < 4; bit *= 2) {
    const bool upper = (l & bit) != 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k & bit) continue;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        uint32_t& lo = w[4 * k + x];
        uint32_t& hi = w[4 * (k + bit) + x];
        const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? lo : hi, bit);
        if (upper) lo = got; else hi = got;
      }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (k - l < left)
      *reinterpret_cast<uint4*>(static_cast<char*>(own) + (k - l) * pitch + l * 16) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
}
// 32 columns as bf16, times mul
__device__ __forceinline__ void store_quad_rows(const float (&v)[32], float mul, __nv_bfloat16* own, long long stride, int left) {
  uint32_t w[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) w[e] = sm100::bf16x2(v[2 * e] * mul, v[2 * e + 1] * mul);
  store_quad_rows(w, own, stride * 2, left);
}

// A value that all lanes have, as one the compiler knows to be the same in all of them: descriptors and loop bounds then stay in uniform registers
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// tanh of N values times inv, in place.  Scores are mostly far below the cap: where a thread has none beyond half of it, the polynomial, two values an instruction; otherwise
// exp2 and a reciprocal, whose absolute error (1.2e-7, times the cap) is a part of the largest of the thread's values.  So the values have to be of one row: what another row's scores are
// must not matter to it.  counts: whether they are anyone's.
template <int N>
__device__ __forceinline__ void tanh_scores(float inv, float (&s)[N], bool counts = true) {
  using namespace sm100;
  float most = fabsf(s[0]);
#pragma unroll
  for (int e = 1; e < N; ++e) most = fmaxf(most, fabsf(s[e]));
  if (!counts || most * inv <= 0.5f) {
    const uint64_t inv2 = pack2(inv, inv);
#pragma unroll
    for (int e = 0; e < N; e += 2) {
      const uint64_t u = mul2(pack2(s[e], s[e + 1]), inv2), w = mul2(u, u);
      uint64_t p = fma2(w, pack2(kTanh8, kTanh8), pack2(kTanh6, kTanh6));
      p = fma2(w, p, pack2(kTanh4, kTanh4));
      p = fma2(w, p, pack2(kTanh2, kTanh2));
      p = fma2(w, p, pack2(kTanh0, kTanh0));
      unpack2(mul2(u, p), s[e], s[e + 1]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = tanh_large(s[e] * inv);
  }
}
// The same for values of several rows (the whole warp): where the warp has one beyond half of the cap, each takes its own way.
template <int N>
__device__ __forceinline__ void tanh_scores_of_rows(float inv, float (&s)[N]) {
  using namespace sm100;
  float most = fabsf(s[0]);
#pragma unroll
  for (int e = 1; e < N; ++e) most = fmaxf(most, fabsf(s[e]));
  if (__all_sync(0xffffffffu, most * inv <= 0.5f)) {
    tanh_scores(inv, s, false);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = tanh_full(s[e] * inv);
    __syncwarp();                                // (the warp goes on together, as the TMEM instructions behind this want it)
  }
}

// What scores are multiplied by, never 0: the least normal number instead, which leaves a score that a slope has made 1e34 units (2^-100 is the least unit) without weight.  A NaN
// stays one.
__device__ __forceinline__ float at_least_tiny(float x) { return x < 1.17549435e-38f ? 1.17549435e-38f : x; }

// the slope's term of N scores from column j0 on
template <int N>
__device__ __forceinline__ void slope_scores(float slope, int pos, int j0, float (&s)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = fmaf(-slope, fabsf((float)(j0 + e - pos)), s[e]);
}

// Running softmax of one row, a tile of 128 scores at a time.  The scores are x = x_ij in units of the accumulator, or of the cap where there is one (CAP: then the
// accumulator's tanh is x), with the sign of c folded in (TERMS: calls with scales or slopes); |a| x are the base-2 exponents.  m is what the probabilities are
// measured from: the maximum, or up to 8 / |a| below it.  CAP and TERMS are known at compile time: branches over code that a call does not need
// would cut the loop's schedule into pieces (plain calls lost a fifth).  UNSEEN: masked keys may be anything, not only data of the call.
template <bool CAP, bool TERMS, bool UNSEEN>
struct RowSoftmax {
  float a, m, slope, sign, minus_am;
  float l0, l1;             // the sum, in two halves
  int pos;
  bool mine;                // a row of the problem
  __device__ __forceinline__ void start(bool is_row, float a_signed, float slope_unit, int position) {
    mine = is_row;
    sign = a_signed < 0.f ? -1.0f : 1.0f;
    a = at_least_tiny(fabsf(a_signed));      // c = 0: every visible key weighs the same, while 0 * -inf would be NaN
    slope = slope_unit;
    pos = position;
    m = -INFINITY;
    minus_am = 0.f;
    l0 = l1 = 0.f;
  }
  // Accumulators to scores (in place), masked ones to -inf; returns the factor that O has to be multiplied by (1 mostly)
  __device__ __forceinline__ float take(float cap_inv, float (&s)[4][32], int k0, int2 sees, bool edge) {
    using namespace sm100;
    const int from = sees.x - k0, to = sees.y - k0;
    if (CAP) {
      if (UNSEEN && edge) {                  // (what a masked score happens to be has no say in how the tanh is computed)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e) s[c][e] = c * 32 + e >= from && c * 32 + e < to ? s[c][e] : 0.f;
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) tanh_scores(cap_inv, s[c], mine);
    }
    if (TERMS) {
      if (slope != 0.f) {
#pragma unroll
        for (int c = 0; c < 4; ++c) slope_scores(slope, pos, k0 + c * 32, s[c]);
      }
      const uint64_t g = pack2(sign, sign);
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 32; e += 2) unpack2(mul2(pack2(s[c][e], s[c][e + 1]), g), s[c][e], s[c][e + 1]);
    }
    if (edge) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 32; ++e) s[c][e] = c * 32 + e >= from && c * 32 + e < to ? s[c][e] : -INFINITY;
    }
    float t[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      t[c] = fmaxf(s[c][0], s[c][1]);
#pragma unroll
      for (int e = 2; e < 32; e += 2) t[c] = max3(t[c], s[c][e], s[c][e + 1]);
    }
    const float most = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
    float grown = 1.0f;
    if ((most - m) * a > 8.0f) {             // (from -inf on: always, unless most is -inf too: NaN)
      grown = exp2_fast((m - most) * a);
      m = most;
      minus_am = -a * m;
      l0 *= grown;
      l1 *= grown;
    }
    return grown;
  }
  // 32 probabilities of the scores, as bf16 pairs; added to the sum as they are in float32
  __device__ __forceinline__ void probabilities(const float (&s)[32], uint32_t (&p)[16]) {
    using namespace sm100;
    const uint64_t a2 = pack2(a, a), b2 = pack2(minus_am, minus_am);
    uint64_t sum = pack2(l0, l1);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      float x, y;
      unpack2(fma2(pack2(s[2 * e], s[2 * e + 1]), a2, b2), x, y);
      x = exp2_fast(x);
      y = exp2_fast(y);
      sum = add2(sum, pack2(x, y));
      p[e] = bf16x2(x, y);
    }
    unpack2(sum, l0, l1);
  }
  __device__ __forceinline__ float sum() const { return l0 + l1; }
  __device__ __forceinline__ float base() const { return -minus_am; }    // in base-2 units
};

}  // namespace entmax
