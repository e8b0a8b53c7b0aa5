// Element code of the tensor-core kernels of softmax attention: scores of a tile to probabilities.
#pragma once

#include "sm100_ptx.cuh"
#include "softmax.cuh"

namespace entmax {

// Low descriptor word of a tile of 128 rows x 64-element blocks read with its 128-byte rows along K and the row's elements along N (or M), 128-byte
// swizzle: atoms of eight rows repeat every 1024 bytes, 64-element blocks every 128 * 128 bytes.
__device__ __forceinline__ uint32_t mn_desc_lo(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | ((uint32_t)((128 * 128) >> 4) << 16); }

// tanh for |u| <= 1 on the FMA pipe: odd polynomial of degree 11, least maximum error (2.4e-7, fitted by iterated weighted least squares)
__device__ __forceinline__ float tanh_small(float u) {
  const float w = u * u;
  float p = fmaf(w, -0.00283948f, 0.01611422f);
  p = fmaf(w, p, -0.0509729f);
  p = fmaf(w, p, 0.13253527f);
  p = fmaf(w, p, -0.33324004f);
  p = fmaf(w, p, 0.99999685f);
  return u * p;
}

// exp2 of two values in [-126, 127] on the FMA pipe: 2^n from the nearest integer, 2^f on [-1/2, 1/2] by a polynomial of degree 5 with the least maximum
// relative error (7.5e-8, fitted the same way).  Smaller values end near 2^-126, far below what a sum of probabilities up to 2^8 notices.
__device__ __forceinline__ void exp2_pair_fma(float& x, float& y) {
  using namespace sm100;
  x = fmaxf(x, -126.0f);
  y = fmaxf(y, -126.0f);
  const uint64_t v = pack2(x, y);
  const uint64_t r = add2(v, pack2(12582912.0f, 12582912.0f));       // 1.5 * 2^23: the sum's low bits are the integer
  const uint64_t n = add2(r, pack2(-12582912.0f, -12582912.0f));
  const uint64_t f = fma2(n, pack2(-1.0f, -1.0f), v);
  uint64_t p = fma2(f, pack2(0.00132765f, 0.00132765f), pack2(0.00967554f, 0.00967554f));
  p = fma2(f, p, pack2(0.05550713f, 0.05550713f));
  p = fma2(f, p, pack2(0.2402212f, 0.2402212f));
  p = fma2(f, p, pack2(0.69314697f, 0.69314697f));
  p = fma2(f, p, pack2(1.00000007f, 1.00000007f));
  float rx, ry, px, py;
  unpack2(r, rx, ry);
  unpack2(p, px, py);
  x = __int_as_float(__float_as_int(px) + (__float_as_int(rx) << 23));
  y = __int_as_float(__float_as_int(py) + (__float_as_int(ry) << 23));
}

// x / sm_scale of N accumulators from column j0 on: capped, with the slope's term, in place (the whole warp)
template <int N>
__device__ __forceinline__ void cap_scores(float cap_acc, float cap_inv, float (&s)[N]) {
  float most = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) most = fmaxf(most, fabsf(s[e]));
  if (__all_sync(0xffffffffu, most * cap_inv <= 1.0f)) {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = cap_acc * tanh_small(s[e] * cap_inv);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) s[e] = cap_acc * tanh_full(s[e] * cap_inv);
  }
}
template <int N>
__device__ __forceinline__ void slope_scores(float slope, int pos, int j0, float (&s)[N]) {
#pragma unroll
  for (int e = 0; e < N; ++e) s[e] = fmaf(-slope, fabsf((float)(j0 + e - pos)), s[e]);
}

// Running softmax of one row, a tile of 128 scores at a time.  The scores are x = x_ij / sm_scale with the sign of c folded in; |a| x are the base-2
// exponents.  m is what the probabilities are measured from: the maximum, or up to 8 / |a| below it.
struct RowSoftmax {
  float a, m, slope, minus_am;
  float l0, l1;             // the sum, in two halves
  int pos;
  bool negative;
  __device__ __forceinline__ void start(float a_signed, float slope_acc, int position) {
    negative = a_signed < 0.f;
    a = fmaxf(fabsf(a_signed), 1e-30f);      // c = 0: every visible key weighs the same, while 0 * -inf would be NaN
    slope = slope_acc;
    pos = position;
    m = -INFINITY;
    minus_am = 0.f;
    l0 = l1 = 0.f;
  }
  // Scores to x (in place), masked ones to -inf; returns the factor that O has to be multiplied by (1 mostly)
  __device__ __forceinline__ float take(const SoftmaxArgs& args, float (&s)[4][32], int k0, int2 sees, bool edge) {
    if (args.cap_acc > 0.f) {
#pragma unroll
      for (int c = 0; c < 4; ++c) cap_scores(args.cap_acc, args.cap_inv, s[c]);
    }
    if (slope != 0.f) {
#pragma unroll
      for (int c = 0; c < 4; ++c) slope_scores(slope, pos, k0 + c * 32, s[c]);
    }
    if (__any_sync(0xffffffffu, negative)) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 32; ++e) s[c][e] = negative ? -s[c][e] : s[c][e];
    }
    if (edge) {
      const int from = sees.x - k0, to = sees.y - k0;
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
      for (int e = 2; e < 32; e += 2) t[c] = sm100::max3(t[c], s[c][e], s[c][e + 1]);
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
  __device__ __forceinline__ void probabilities(float (&s)[32], uint32_t (&p)[16], bool edge) {
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
