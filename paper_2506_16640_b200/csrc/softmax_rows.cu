// Softmax attention on CUDA cores, forward and backward: float32 problems, whose products the tensor cores' input types cannot hold.
//
// A CTA has 64 query rows (keys in the key-major backward kernel) of one head and walks the 64-key (query) tiles that its rows' masks reach.  Every
// operand tile sits in shared memory as float32 with rows of D + 4, which keeps float4 reads of 8 neighbouring rows free of
// conflicts; 256 threads hold 4 x 4 scores and 4 x D/16 outputs each.  One pass with a running maximum and sum forward (the sum of
// at most 64 terms at a time, then of tiles, all float32); backward one kernel per side, so that nothing is added up by atomics and results
// are the same every time: the query-major one takes its tiles twice, first for sum_j p_ij dP_ij, then for dQ.
// Bound by the FMA pipe and shared memory; meant for checking a model at full precision, not for speed: 8 x 12 x 1024 x 64 causal 0.61 ms forward (21 TFLOP/s) and 2.4 ms
// backward, 16 x 4096 x 128 2.85 (24 TFLOP/s) and 11.7 ms.
#include "softmax.cuh"

namespace entmax {

namespace {

constexpr int kT = 64;                // rows of a tile
constexpr int kRowThreads = 256;

template <int D>
struct RowCfg {
  static constexpr int kLd = D + 4;
  static constexpr int kTile = kT * kLd;            // floats of an operand tile
  static constexpr int kLdS = kT + 4;
  static constexpr int kScores = kT * kLdS;
};

// rows row0 .. of one head into a tile, zeros behind the last
template <int D>
__device__ __forceinline__ void load_rows(float* dst, const float* base, long long stride, int row0, int N) {
  constexpr int kPieces = D / 4;
  for (int t = threadIdx.x; t < kT * kPieces; t += kRowThreads) {
    const int r = t / kPieces, c = (t - r * kPieces) * 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (row0 + r < N) load_slice<4>(base + (long long)(row0 + r) * stride + c, x);
    *reinterpret_cast<float4*>(dst + r * RowCfg<D>::kLd + c) = make_float4(x[0], x[1], x[2], x[3]);
  }
}

// s[y][x] = <A row ty * 4 + y, B row tx + 16 x>
template <int D>
__device__ __forceinline__ void dot_tile(const float* A, const float* B, float (&s)[4][4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int y = 0; y < 4; ++y)
#pragma unroll
    for (int x = 0; x < 4; ++x) s[y][x] = 0.f;
  for (int d = 0; d < D; d += 4) {
    float4 av[4], bv[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) av[y] = *reinterpret_cast<const float4*>(A + (ty * 4 + y) * RowCfg<D>::kLd + d);
#pragma unroll
    for (int x = 0; x < 4; ++x) bv[x] = *reinterpret_cast<const float4*>(B + (tx + 16 * x) * RowCfg<D>::kLd + d);
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        s[y][x] = fmaf(av[y].w, bv[x].w, fmaf(av[y].z, bv[x].z, fmaf(av[y].y, bv[x].y, fmaf(av[y].x, bv[x].x, s[y][x]))));
  }
}

// out[y][..] += sum_j W(ty * 4 + y, j) R[j][cols of tx]; W is S[row][j], or S[j][row] with kTransposed
template <int D, bool kTransposed>
__device__ __forceinline__ void add_product(const float* S, const float* R, float (&out)[4][D / 16]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  for (int j = 0; j < kT; ++j) {
    float w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) w[y] = kTransposed ? S[j * RowCfg<D>::kLdS + ty * 4 + y] : S[(ty * 4 + y) * RowCfg<D>::kLdS + j];
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const float4 r = *reinterpret_cast<const float4*>(R + j * RowCfg<D>::kLd + tx * 4 + 64 * e);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        out[y][4 * e] = fmaf(w[y], r.x, out[y][4 * e]);
        out[y][4 * e + 1] = fmaf(w[y], r.y, out[y][4 * e + 1]);
        out[y][4 * e + 2] = fmaf(w[y], r.z, out[y][4 * e + 2]);
        out[y][4 * e + 3] = fmaf(w[y], r.w, out[y][4 * e + 3]);
      }
    }
  }
}
template <int D>
__device__ __forceinline__ void store_rows(float* base, long long stride, int row0, int N, const float (&out)[4][D / 16], const float (&mul)[4]) {
  const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    const int r = row0 + ty * 4 + y;
    if (r >= N) continue;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const float x[4] = {out[y][4 * e] * mul[y], out[y][4 * e + 1] * mul[y], out[y][4 * e + 2] * mul[y], out[y][4 * e + 3] * mul[y]};
      store_slice<4>(base + (long long)r * stride + tx * 4 + 64 * e, x);
    }
  }
}
// over the 16 threads of a row
__device__ __forceinline__ float row_max(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// The capped score of an accumulator, in the scores' unit, and d z / d (sm_scale acc) at it.  The tanh is exact to a part of itself: an error that does not shrink
// with the score is multiplied by the cap, which may be far above every score.
__device__ __forceinline__ float capped(const SoftmaxArgs& a, float acc, float& slope) {
  slope = 1.0f;
  if (a.cap_inv == 0.f) return acc;
  const float t = tanhf(acc * a.cap_inv);
  slope = 1.0f - t * t;
  return t;
}

// Keys that any row of the tile sees; lo, hi: two words of shared memory
__device__ __forceinline__ int2 tile_range(const int2 (&sees)[4], int* lo_hi) {
  if (threadIdx.x == 0) { lo_hi[0] = 0x7fffffff; lo_hi[1] = 0; }
  __syncthreads();
  if ((threadIdx.x & 15) == 0) {
#pragma unroll
    for (int y = 0; y < 4; ++y)
      if (sees[y].y > sees[y].x) {
        atomicMin(lo_hi, sees[y].x);
        atomicMax(lo_hi + 1, sees[y].y);
      }
  }
  __syncthreads();
  return make_int2(lo_hi[0], lo_hi[1]);
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) softmax_rows_fwd_kernel(const SoftmaxArgs a, const float* q, const float* k, const float* v, float* o, float* lse,
                                                                       int32_t* status) {
  pdl_begin();
  using C = RowCfg<D>;
  extern __shared__ float smem[];
  __shared__ int lo_hi[2];
  float *Q = smem, *K = Q + C::kTile, *V = K + C::kTile, *S = V + C::kTile;
  const int tiles = (a.N + kT - 1) / kT;
  const int tile = tiles - 1 - (int)(blockIdx.x % tiles);
  const int bh = blockIdx.x / tiles, b = bh / a.H, h = bh - b * a.H, kh = h / a.G;
  const int row0 = tile * kT, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  int2 sees[4];
  float scale[4], top[4], mass[4], out[4][D / 16] = {};
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    const int i = row0 + ty * 4 + y;
    sees[y] = i < a.N ? visible_keys(a, b, i) : make_int2(0, 0);
    const float c = i < a.N ? row_scale(a, b, h, i, sees[y].y - sees[y].x) : 0.f;
    if (tx == 0 && status && !isfinite(c)) atomicOr(status + ENTMAX_ATTN_STATUS_FLAGS, ENTMAX_ATTN_FLAG_BAD_SCALE);
    scale[y] = isfinite(c) ? c * a.unit * kLog2e : NAN;      // (infinity times negative scores alone would leave a row as if it saw nothing)
    top[y] = -INFINITY;
    mass[y] = 0.f;
  }
  const float slope = a.alibi ? a.alibi[h] / a.unit : 0.f;
  load_rows<D>(Q, q + b * a.q.b + h * a.q.h, a.q.n, row0, a.N);
  const int2 range = tile_range(sees, lo_hi);
  for (int j0 = range.x / kT * kT; j0 < range.y; j0 += kT) {
    load_rows<D>(K, k + b * a.k.b + kh * a.k.h, a.k.n, j0, a.N);
    load_rows<D>(V, v + b * a.v.b + kh * a.v.h, a.v.n, j0, a.N);
    __syncthreads();
    float s[4][4];
    dot_tile<D>(Q, K, s);
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int i = row0 + ty * 4 + y;
      float most = -INFINITY;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int j = j0 + tx + 16 * x;
        float unused;
        const float xa = capped(a, s[y][x], unused) - slope * fabsf((float)(i - j));
        s[y][x] = j >= sees[y].x && j < sees[y].y ? scale[y] * xa : -INFINITY;
        most = fmaxf(most, s[y][x]);
      }
      const float now = fmaxf(top[y], row_max(most)), base = now > -INFINITY ? now : 0.f;
      const float old = exp2f(top[y] - base);
      float sum = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const float p = exp2f(s[y][x] - base);
        sum += p;
        S[(ty * 4 + y) * C::kLdS + tx + 16 * x] = p;
      }
      mass[y] = mass[y] * old + row_sum(sum);
      top[y] = now;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) out[y][e] *= old;
    }
    __syncthreads();
    add_product<D, false>(S, V, out);
    __syncthreads();
  }
  float inv[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    inv[y] = mass[y] != 0.f ? 1.0f / mass[y] : 0.f;
    const int i = row0 + ty * 4 + y;
    if (tx == 0 && i < a.N) lse[(size_t)bh * a.N + i] = mass[y] != 0.f ? top[y] * kLn2 + logf(mass[y]) : -INFINITY;
  }
  store_rows<D>(o + b * a.o.b + h * a.o.h, a.o.n, row0, a.N, out, inv);
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) softmax_rows_dq_kernel(const SoftmaxArgs a, const SoftmaxGrads g, const float* q, const float* k, const float* v,
                                                                      const float* d_o, float* dq) {
  pdl_begin();
  using C = RowCfg<D>;
  extern __shared__ float smem[];
  __shared__ int lo_hi[2];
  float *Q = smem, *DO = Q + C::kTile, *K = DO + C::kTile, *V = K + C::kTile, *S = V + C::kTile;
  const int tiles = (a.N + kT - 1) / kT;
  const int tile = tiles - 1 - (int)(blockIdx.x % tiles);
  const int bh = blockIdx.x / tiles, b = bh / a.H, h = bh - b * a.H, kh = h / a.G;
  const int row0 = tile * kT, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  int2 sees[4];
  float c[4], lse2[4], dot[4] = {}, dc[4] = {}, out[4][D / 16] = {};
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    const int i = row0 + ty * 4 + y;
    sees[y] = i < a.N ? visible_keys(a, b, i) : make_int2(0, 0);
    const bool some = sees[y].y > sees[y].x;       // (a row that sees nothing has no scale: what the table holds for it, of padding, may be anything)
    c[y] = some ? row_scale(a, b, h, i, sees[y].y - sees[y].x) : 0.f;
    lse2[y] = some ? g.lse[(size_t)bh * a.N + i] * kLog2e : 0.f;
  }
  const float slope = a.alibi ? a.alibi[h] / a.unit : 0.f;
  load_rows<D>(Q, q + b * a.q.b + h * a.q.h, a.q.n, row0, a.N);
  load_rows<D>(DO, d_o + b * g.d_o.b + h * g.d_o.h, g.d_o.n, row0, a.N);
  const int2 range = tile_range(sees, lo_hi);
  for (int pass = 0; pass < 2; ++pass) {
    for (int j0 = range.x / kT * kT; j0 < range.y; j0 += kT) {
      load_rows<D>(K, k + b * a.k.b + kh * a.k.h, a.k.n, j0, a.N);
      load_rows<D>(V, v + b * a.v.b + kh * a.v.h, a.v.n, j0, a.N);
      __syncthreads();
      float s[4][4], dp[4][4];
      dot_tile<D>(Q, K, s);
      dot_tile<D>(DO, V, dp);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int i = row0 + ty * 4 + y;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int j = j0 + tx + 16 * x;
          float grow;
          const float xa = capped(a, s[y][x], grow) - slope * fabsf((float)(i - j));
          const float p = j >= sees[y].x && j < sees[y].y ? exp2f(c[y] * a.unit * kLog2e * xa - lse2[y]) : 0.f;
          if (pass == 0) {
            dot[y] = fmaf(p, dp[y][x], dot[y]);
          } else {
            const float ds = p * (dp[y][x] - dot[y]);
            dc[y] = fmaf(ds, xa, dc[y]);
            S[(ty * 4 + y) * C::kLdS + tx + 16 * x] = ds * grow;
          }
        }
      }
      __syncthreads();
      if (pass == 1) add_product<D, false>(S, K, out);
      __syncthreads();
    }
    if (pass == 0) {
#pragma unroll
      for (int y = 0; y < 4; ++y) dot[y] = row_sum(dot[y]);
    }
  }
  float mul[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    mul[y] = c[y] * a.sm_scale;
    const int i = row0 + ty * 4 + y;
    const float total = row_sum(dc[y]);
    if (tx == 0 && i < a.N) {
      g.row_dot[(size_t)bh * a.N + i] = dot[y];
      if (g.dc_rows) g.dc_rows[(size_t)bh * a.N + i] = total * a.unit;
    }
  }
  store_rows<D>(dq + b * g.dq.b + h * g.dq.h, g.dq.n, row0, a.N, out, mul);
}

template <int D>
__global__ void __launch_bounds__(kRowThreads) softmax_rows_dkv_kernel(const SoftmaxArgs a, const SoftmaxGrads g, const float* q, const float* k, const float* v,
                                                                       const float* d_o, float* dk, float* dv) {
  pdl_begin();
  using C = RowCfg<D>;
  extern __shared__ float smem[];
  __shared__ int lo_hi[2];
  float *K = smem, *V = K + C::kTile, *Q = V + C::kTile, *DO = Q + C::kTile, *P = DO + C::kTile, *S = P + C::kScores;
  const int tiles = (a.N + kT - 1) / kT;
  const int tile = blockIdx.x % tiles;
  const int bk = blockIdx.x / tiles, b = bk / a.KH, kh = bk - b * a.KH;
  const int j0 = tile * kT, ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
  float out_k[4][D / 16] = {}, out_v[4][D / 16] = {};
  load_rows<D>(K, k + b * a.k.b + kh * a.k.h, a.k.n, j0, a.N);
  load_rows<D>(V, v + b * a.v.b + kh * a.v.h, a.v.n, j0, a.N);
  for (int h = kh * a.G; h < (kh + 1) * a.G; ++h) {
    const float slope = a.alibi ? a.alibi[h] / a.unit : 0.f;
    for (int row0 = 0; row0 < a.N; row0 += kT) {
      int2 sees[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int i = row0 + ty * 4 + y;
        sees[y] = i < a.N ? visible_keys(a, b, i) : make_int2(0, 0);
      }
      const int2 range = tile_range(sees, lo_hi);
      __syncthreads();
      if (range.x >= j0 + kT || range.y <= j0) continue;
      load_rows<D>(Q, q + b * a.q.b + h * a.q.h, a.q.n, row0, a.N);
      load_rows<D>(DO, d_o + b * g.d_o.b + h * g.d_o.h, g.d_o.n, row0, a.N);
      __syncthreads();
      float s[4][4], dp[4][4];
      dot_tile<D>(Q, K, s);
      dot_tile<D>(DO, V, dp);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int i = row0 + ty * 4 + y;
        const bool any = sees[y].y > sees[y].x;
        const size_t at = ((size_t)b * a.H + h) * a.N + (any ? i : 0);
        const float c = any ? row_scale(a, b, h, i, sees[y].y - sees[y].x) : 0.f;
        const float lse2 = any ? g.lse[at] * kLog2e : 0.f, dot = any ? g.row_dot[at] : 0.f;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int j = j0 + tx + 16 * x;
          float grow;
          const float xa = capped(a, s[y][x], grow) - slope * fabsf((float)(i - j));
          const float p = j >= sees[y].x && j < sees[y].y ? exp2f(c * a.unit * kLog2e * xa - lse2) : 0.f;
          P[(ty * 4 + y) * C::kLdS + tx + 16 * x] = p;
          S[(ty * 4 + y) * C::kLdS + tx + 16 * x] = p * (dp[y][x] - dot) * grow * (c * a.sm_scale);
        }
      }
      __syncthreads();
      add_product<D, true>(P, DO, out_v);
      add_product<D, true>(S, Q, out_k);
      __syncthreads();
    }
  }
  const float one[4] = {1.f, 1.f, 1.f, 1.f};
  store_rows<D>(dk + b * g.dk.b + kh * g.dk.h, g.dk.n, j0, a.N, out_k, one);
  store_rows<D>(dv + b * g.dv.b + kh * g.dv.h, g.dv.n, j0, a.N, out_v, one);
}

template <int D>
cudaError_t rows_fwd(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status, cudaStream_t stream) {
  using C = RowCfg<D>;
  const int smem = (3 * C::kTile + C::kScores) * 4;
  cudaError_t err = cudaFuncSetAttribute(softmax_rows_fwd_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (err != cudaSuccess) return err;
  const unsigned grid = (unsigned)((long long)a.B * a.H * ((a.N + kT - 1) / kT));
  return launch_kernel(softmax_rows_fwd_kernel<D>, grid, kRowThreads, smem, stream, a, static_cast<const float*>(q), static_cast<const float*>(k),
                       static_cast<const float*>(v), static_cast<float*>(o), lse, status);
}
template <int D>
cudaError_t rows_bwd(const SoftmaxArgs& a, const SoftmaxGrads& g, const void* q, const void* k, const void* v, const void* d_o, void* dq, void* dk,
                     void* dv, cudaStream_t stream) {
  using C = RowCfg<D>;
  const int smem_q = (4 * C::kTile + C::kScores) * 4, smem_kv = (4 * C::kTile + 2 * C::kScores) * 4;
  cudaError_t err = cudaFuncSetAttribute(softmax_rows_dq_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_q);
  if (err == cudaSuccess) err = cudaFuncSetAttribute(softmax_rows_dkv_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_kv);
  if (err != cudaSuccess) return err;
  const long long tiles = (a.N + kT - 1) / kT;
  err = launch_kernel(softmax_rows_dq_kernel<D>, (unsigned)(a.B * a.H * tiles), kRowThreads, smem_q, stream, a, g, static_cast<const float*>(q),
                      static_cast<const float*>(k), static_cast<const float*>(v), static_cast<const float*>(d_o), static_cast<float*>(dq));
  if (err != cudaSuccess) return err;
  return launch_kernel(softmax_rows_dkv_kernel<D>, (unsigned)(a.B * a.KH * tiles), kRowThreads, smem_kv, stream, a, g, static_cast<const float*>(q),
                       static_cast<const float*>(k), static_cast<const float*>(v), static_cast<const float*>(d_o), static_cast<float*>(dk), static_cast<float*>(dv));
}

}  // namespace

cudaError_t launch_softmax_rows_fwd(const SoftmaxArgs& a, const void* q, const void* k, const void* v, void* o, float* lse, int32_t* status,
                                    cudaStream_t stream) {
  return a.D == 64 ? rows_fwd<64>(a, q, k, v, o, lse, status, stream) : rows_fwd<128>(a, q, k, v, o, lse, status, stream);
}
cudaError_t launch_softmax_rows_bwd(const SoftmaxArgs& a, const SoftmaxGrads& g, const void* q, const void* k, const void* v, const void* d_o,
                                    void* dq, void* dk, void* dv, cudaStream_t stream) {
  return a.D == 64 ? rows_bwd<64>(a, g, q, k, v, d_o, dq, dk, dv, stream) : rows_bwd<128>(a, g, q, k, v, d_o, dq, dk, dv, stream);
}

}  // namespace entmax
