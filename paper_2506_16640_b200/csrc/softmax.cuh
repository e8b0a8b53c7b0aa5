// Declarations shared by the kernels of softmax attention, the alpha = 1 member of the family (softmax_*.cu).
//
//   z_ij = sm_scale <q_i, k_j>,  x_ij = cap tanh(z_ij / cap) - m_h |i - j|,  s_ij = c_i x_ij,
//   p_ij = exp(s_ij - lse_i) over the keys j the row sees,  O_i = sum_j p_ij v_j;  a row that sees none: O = 0, lse = -inf.
// Scores are kept in a unit of their own: that of the accumulator <q_i, k_j>, x / unit = acc - (m_h / sm_scale) |i - j| with unit = sm_scale, or of the cap,
// x / unit = tanh(acc * cap_inv) - (m_h / cap) |i - j| with unit = cap; s log2(e) = a_i (x / unit) with a_i = c_i unit log2(e), so that a probability is one
// FMA and one exp2.
#pragma once

#include "common.cuh"

namespace entmax {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct SoftmaxArgs {
  int B, H, KH, G, N, D;              // G = H / KH query heads share a K/V head
  int causal;
  float sm_scale;
  float cap_inv;                      // sm_scale / cap (0: not capped)
  float unit;                         // of the scores: sm_scale, or the cap
  const int2* ranges;                 // [B][N] {first key, one behind the last} or nullptr
  const float *beta, *gamma, *delta;  // [H] or nullptr
  const float* c_rows;                // [B][H][N] or nullptr
  const float* alibi;                 // [H] or nullptr
  entmax_attn_strides q, k, v, o;
};

// The keys [x, y) that row i sees of the ones its range says; y = x where there are none.
__device__ __forceinline__ int2 seen_of(const SoftmaxArgs& a, int2 range, int i) {
  int2 r = make_int2(max(range.x, 0), min(range.y, a.causal ? i + 1 : a.N));
  if (r.y <= r.x) r = make_int2(0, 0);
  return r;
}
// The same from the row's range in memory, or without one
__device__ __forceinline__ int2 visible_keys(const SoftmaxArgs& a, int b, int i) {
  return a.ranges ? seen_of(a, a.ranges[(size_t)b * a.N + i], i) : make_int2(0, a.causal ? i + 1 : a.N);
}

// (ln n)^gamma grown by beta on top of delta; n = 1 (and 0): delta alone
__device__ __forceinline__ float length_scale(float beta, float gamma, float delta, int n) {
  return n > 1 ? delta + beta * powf(logf((float)n), gamma) : delta;
}
// c of row i, which sees n keys
__device__ __forceinline__ float row_scale(const SoftmaxArgs& a, int b, int h, int i, int n) {
  if (a.c_rows) return a.c_rows[((size_t)b * a.H + h) * a.N + i];
  if (a.beta) return length_scale(a.beta[h], a.gamma[h], a.delta[h], n);
  return 1.0f;
}

// tanh on [-1/2, 1/2]: u times a polynomial of degree 4 in u^2 (least maximum error, 3.6e-8, and no more than 2.5 u = 2^-24 of the value itself; fitted by iterated weighted
// least squares), the coefficients from the highest on
constexpr float kTanh8 = 0.016737575f, kTanh6 = -0.052762136f, kTanh4 = 0.13320571f, kTanh2 = -0.33332777f, kTanh0 = 0.99999994f;

// tanh from one exp2 and one reciprocal, within 1.2e-7: a few u of itself where |u| is above 1/2.  Large arguments end at +-1: exp2 overflows to infinity or vanishes.
__device__ __forceinline__ float tanh_large(float u) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(u * (2.0f * kLog2e)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.0f));
  return fmaf(-2.0f, r, 1.0f);
}
// tanh within a few u of itself: what it is off by is multiplied by the cap, which may be far above the score
__device__ __forceinline__ float tanh_full(float u) {
  const float w = u * u, p = fmaf(w, fmaf(w, fmaf(w, fmaf(w, kTanh8, kTanh6), kTanh4), kTanh2), kTanh0);
  return fabsf(u) <= 0.5f ? u * p : tanh_large(u);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Host: the unit of the scores and what goes with it (defined in softmax_api.cu).  Fails for scales and caps beyond 2^+-100: c times the unit, the slope over it and its
// reciprocal have to stay float32 numbers.
int softmax_unit(float given_scale, float softcap, int D, float* sm_scale, float* cap_inv, float* unit);
// Host: checks of the parameters and the terms (defined in softmax_api.cu)
int check_softmax(const entmax_attn_softmax_params* params, const entmax_attn_softmax_terms* terms, SoftmaxArgs* out);

// Gradient outputs and what the backward pass works with
struct SoftmaxGrads {
  const float* lse;
  entmax_attn_strides d_o, dq, dk, dv;
  float* dc_rows;                     // [B][H][N] or nullptr
  float* row_dot;                     // float32 problems: [B][H][N] scratch, sum_j p_ij dP_ij
};

// CUDA-core kernels (float32 problems)
cudaError_t launch_softmax_rows_fwd(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status,
                                    cudaStream_t stream);
cudaError_t launch_softmax_rows_bwd(const SoftmaxArgs& a, const SoftmaxGrads& g, const void* q, const void* k, const void* v, const void* d_o,
                                    void* dq, void* dk, void* dv, cudaStream_t stream);
// Tensor-core kernels (bf16)
cudaError_t launch_softmax_fwd(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status,
                               cudaStream_t stream);
// rows, spans: scratch of so many bytes
size_t softmax_bwd_rows_bytes(const SoftmaxArgs& a);
size_t softmax_bwd_spans_bytes(const SoftmaxArgs& a);
cudaError_t launch_softmax_bwd(const SoftmaxArgs& a, const SoftmaxGrads& g, const void* q, const void* k, const void* v, const void* o, const void* d_o,
                               void* dq, void* dk, void* dv, float* rows, void* spans, int32_t* status, cudaStream_t stream);
// dbeta, dgamma, ddelta [H] from dL/dc of every row
cudaError_t launch_softmax_scale_grad(const SoftmaxArgs& a, const float* dc_rows, float* dbeta, float* dgamma, float* ddelta, cudaStream_t stream);

}  // namespace entmax
