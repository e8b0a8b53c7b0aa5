// Softmax attention over a paged cache: what its kernels share (softmax_paged.cu, softmax_fwd_sm100.cu).
#pragma once

#include "paged.cuh"
#include "softmax.cuh"

namespace entmax {

struct FewPiece;

struct SoftmaxPagedArgs {
  PagedCache c;
  int H, G, window;
  int max_q, max_kv;                  // longest chunk and sequence that are served
  int few_rows;                       // sequences with n * G <= few_rows rows are the "few" kernel's
  int whole;                          // "few": a CTA per sequence and K/V head, nothing is cut
  int box_shift;                      // a page's boxes have 1 << box_shift keys
  float sm_scale, cap_inv, unit;
  const float *beta, *gamma, *delta, *alibi;
  long long q_st, q_sh;
  const __nv_bfloat16 *q, *v;
  __nv_bfloat16* o;
  float* lse;
  int32_t* status;
  // "few": the pieces of cut sequences, [CTA][2][row slot] each, and where they are
  float* part_o;
  float2* part_ml;                    // {maximum in base-2 units, sum}
  FewPiece* pieces;
  // chunks: `shares` work items take the keys of a unit between them (1: none is shared); [unit][share][tile][128 rows]
  int shares;
  float* chunk_o;
  float2* chunk_ml;
};

// Chunks are handed out in blocks of new tokens: 128, two heads of a group together, or 256 of one head where the group is odd.  Block id -> sequence and
// first token: sequence b has the ids from cu_q[b] / block + b on, at least as many as it has blocks.
__host__ __device__ __forceinline__ int chunk_block(int G) { return G % 2 == 0 ? 128 : 256; }
__host__ __device__ __forceinline__ int chunk_pairs(int G) { return G % 2 == 0 ? G / 2 : G; }
__device__ __forceinline__ int block_start(const PagedCache& c, int b, int block) {
  const int cu = c.cu_q ? clamped_cu(c, b) : b * (c.T / c.B);
  return cu / block + b;
}
struct ChunkPlace {
  int unit, tile, row;
};
__device__ __forceinline__ ChunkPlace chunk_place(const PagedCache& c, int G, int b, int token, int h) {
  const int block = chunk_block(G), g = h % G, kh = h / G;
  ChunkPlace p;
  const int id = block_start(c, b, block) + token / block;
  p.unit = (id * c.KH + kh) * chunk_pairs(G) + (G % 2 == 0 ? g / 2 : g);
  p.tile = G % 2 == 0 ? g & 1 : (token / 128) & 1;
  p.row = token % 128;
  return p;
}

cudaError_t launch_softmax_chunks(const SoftmaxPagedArgs& a, const CUtensorMap& map_k, const CUtensorMap& map_v, cudaStream_t stream);

}  // namespace entmax
