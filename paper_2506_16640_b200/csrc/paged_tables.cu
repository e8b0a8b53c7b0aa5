// Tables of a serving step from the requests' lengths: kv_len, cu_q, block table, positions, slots, and the stack of free pages.
//
// With n_b tokens in the cache and m_b new ones, sequence b needs ceil((n_b + m_b) / ps) - ceil(n_b / ps) new pages.  Two sums over the sequences, of
// tokens and of pages, say where its rows are and which entries of the stack are its own; a sequence is served if the pages up to and with its own
// suffice.  One cluster of CTAs does all: every CTA sums up all sequences by itself (8 bytes each), 1024 at a time, and writes its share of the
// table entries and tokens as it goes.  What a call may overwrite of its own inputs (lengths, stack, count) is written by one CTA behind the cluster's barrier.
// Bound by latency: the chain of load, block scan, load of a page, store.  256 sequences with a token each: 4.5 us; 1000 with up to 900: 8 us.
#include "paged.cuh"

namespace entmax {

namespace {

constexpr int kTabThreads = 1024;
constexpr int kTabMaxCtas = 8;

struct TablesArgs {
  int B, T, ps_shift, n_pages, max_pages, capacity;
  long long table_stride;
  const int32_t* kv_len;
  const int32_t* new_len;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* free_count;
  int32_t* kv_len_out;
  int32_t* cu_q;
  int32_t* positions;
  long long* slots;
  int32_t* free_count_out;
  int32_t* status;
};

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct Request {
  int have, tokens;        // tokens in the cache, rows of new ones
  int pages, need;         // pages it has, pages it needs
  bool ended, bad;         // its pages go back; its lengths are out of range
};
__device__ __forceinline__ Request read_request(const TablesArgs& a, int b) {
  Request r = {0, 0, 0, 0, false, false};
  if (b >= a.B) return r;
  const int limit = a.max_pages << a.ps_shift;
  int have = a.kv_len[b];
  if (have < 0) have = -1 - have;
  const int m = a.new_len[b];
  r.ended = m == -1;
  r.bad = have > limit || m < -1 || (m > 0 && m > limit - have);
  r.have = have;
  r.tokens = max(m, 0);
  if (have <= limit) r.pages = (int)(((unsigned)have + (1u << a.ps_shift) - 1u) >> a.ps_shift);
  if (!r.bad && m > 0) r.need = (int)(((unsigned)(have + m) + (1u << a.ps_shift) - 1u) >> a.ps_shift) - r.pages;
  return r;
}

// Sums over the threads in front of this one; total: over all.  Two sums at once, saturated well below 2^63.
__device__ __forceinline__ void block_scan(long long& x, long long& y, long long& total_x, long long& total_y, long long (*warp_sums)[2]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long ix = x, iy = y;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long px = __shfl_up_sync(0xffffffffu, ix, o), py = __shfl_up_sync(0xffffffffu, iy, o);
    if (lane >= o) { ix += px; iy += py; }
  }
  __syncthreads();
  if (lane == 31) { warp_sums[warp][0] = ix; warp_sums[warp][1] = iy; }
  __syncthreads();
  long long wx = warp_sums[lane][0], wy = warp_sums[lane][1];       // (32 warps: a lane each)
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long px = __shfl_up_sync(0xffffffffu, wx, o), py = __shfl_up_sync(0xffffffffu, wy, o);
    if (lane >= o) { wx += px; wy += py; }
  }
  total_x = __shfl_sync(0xffffffffu, wx, 31);
  total_y = __shfl_sync(0xffffffffu, wy, 31);
  const long long bx = __shfl_sync(0xffffffffu, wx, (warp + 31) & 31), by = __shfl_sync(0xffffffffu, wy, (warp + 31) & 31);
  x = ix - x + (warp ? bx : 0);
  y = iy - y + (warp ? by : 0);
}

struct __align__(8) Chunk {                  // what is known of 1024 sequences; starts count from the chunk's first
  int tok_start[kTabThreads + 1], page_start[kTabThreads + 1], back_start[kTabThreads + 1];
  int have[kTabThreads], pages[kTabThreads];
  bool ok[kTabThreads];
  long long warp_sums[32][2];
  int taken;                                 // pages taken from the stack by all sequences so far
};
// Largest s with start[s] <= x: the sequence that x belongs to (empty ones in front of it share its start)
__device__ __forceinline__ int owner(const int* start, int x) {
  int lo = 0;
#pragma unroll
  for (int step = kTabThreads / 2; step > 0; step >>= 1)
    if (start[lo + step] <= x) lo += step;
  return lo;
}

// Sums of sequences in front of a chunk
struct Bases {
  long long tokens = 0, pages = 0, back = 0;
};
// One chunk into shared memory; mine: this thread's sequence.  Returns {tokens, pages, pages given back} of the chunk.
__device__ __forceinline__ Bases sum_chunk(const TablesArgs& a, int b, const Bases& base, int count, Chunk& c, Request& mine) {
  mine = read_request(a, b);
  const int back = mine.ended && !mine.bad ? mine.pages : 0;
  long long tokens = mine.tokens, pages = (long long)mine.need | (long long)back << 32, all_tokens, all_pages;   // (2^20 pages of 1024 sequences at most)
  block_scan(tokens, pages, all_tokens, all_pages, c.warp_sums);
  const int page_start = (int)(pages & 0xffffffffLL);
  const long long incl = base.pages + page_start + mine.need;
  const bool ok = b < a.B && !mine.bad && !mine.ended && (mine.need == 0 || incl <= count);
  const int t = threadIdx.x;
  c.tok_start[t] = (int)min(tokens, 0x7fffffffLL);
  c.page_start[t] = page_start;
  c.back_start[t] = (int)(pages >> 32);
  c.have[t] = mine.have;
  c.pages[t] = mine.pages;
  c.ok[t] = ok;
  if (t == kTabThreads - 1) {
    c.tok_start[kTabThreads] = c.page_start[kTabThreads] = c.back_start[kTabThreads] = 0x7fffffff;
  }
  if (ok && mine.need > 0) atomicMax(&c.taken, (int)incl);
  __syncthreads();
  return Bases{all_tokens, all_pages & 0xffffffffLL, all_pages >> 32};
}

__global__ void __launch_bounds__(kTabThreads) paged_tables_kernel(const TablesArgs a, int ctas) {
  pdl_begin();
  __shared__ Chunk c;
  const int rank = blockIdx.x, t = threadIdx.x;
  const int count = min(max(a.free_count[0], 0), a.capacity);
  if (t == 0) c.taken = 0;
  // (the first chunk's scan has a barrier in front of the first use of c.taken)
  int flags = a.free_count[0] != count ? ENTMAX_ATTN_FLAG_BAD_LENGTH : 0;
  Bases base;
  Request mine;
  Bases sums;
  for (int b0 = 0; b0 < a.B; b0 += kTabThreads) {
    const int b = b0 + t;
    if (b0) __syncthreads();                                 // the last chunk has been read
    sums = sum_chunk(a, b, base, count, c, mine);
    if (rank == 0 && b < a.B) {
      a.cu_q[b] = (int)min(base.tokens + c.tok_start[t], 0x7fffffffLL);
      if (mine.bad) flags |= ENTMAX_ATTN_FLAG_BAD_LENGTH;
      else if (!mine.ended && !c.ok[t]) flags |= ENTMAX_ATTN_FLAG_NO_PAGES;
    }
    // entries of new pages (those behind the stack's last are nobody's)
    const int new_pages = (int)min(sums.pages, max(count - base.pages, 0LL));
    for (int k = rank * kTabThreads + t; k < new_pages; k += ctas * kTabThreads) {
      const int s = owner(c.page_start, k);
      if (c.ok[s]) a.table[(long long)(b0 + s) * a.table_stride + c.pages[s] + (k - c.page_start[s])] = a.free_pages[count - 1 - ((int)base.pages + k)];
    }
    // tokens
    const int tokens = (a.positions || a.slots) ? (int)min(sums.tokens, max(a.T - base.tokens, 0LL)) : 0;
    for (int k = rank * kTabThreads + t; k < tokens; k += ctas * kTabThreads) {
      const int s = owner(c.tok_start, k);
      int pos = -1;
      long long slot = -1;
      if (c.ok[s]) {
        pos = c.have[s] + (k - c.tok_start[s]);
        if (a.slots) {
          const int at = pos >> a.ps_shift;
          const int page = at < c.pages[s] ? a.table[(long long)(b0 + s) * a.table_stride + at]
                                           : a.free_pages[count - 1 - ((int)base.pages + c.page_start[s] + (at - c.pages[s]))];
          if ((unsigned)page < (unsigned)a.n_pages) slot = ((long long)page << a.ps_shift) + (pos & ((1 << a.ps_shift) - 1));
          else flags |= ENTMAX_ATTN_FLAG_BAD_PAGE;
        }
      }
      if (a.positions) a.positions[base.tokens + k] = pos;
      if (a.slots) a.slots[base.tokens + k] = slot;
    }
    base.tokens += sums.tokens; base.pages += sums.pages; base.back += sums.back;
  }
  if (ctas > 1) cluster_sync(); else __syncthreads();
  if (rank == 0) {
    // the inputs have been read by all
    if (t == 0) {
      a.cu_q[a.B] = (int)min(base.tokens, 0x7fffffffLL);
      if ((a.positions || a.slots) && base.tokens > a.T) flags |= ENTMAX_ATTN_FLAG_BAD_LENGTH;
    }
    const int left = count - c.taken;
    const bool again = a.B > kTabThreads;                    // the only chunk's values are still there
    Bases at;
    for (int b0 = 0; b0 < a.B; b0 += kTabThreads) {
      const int b = b0 + t;
      if (again) {
        __syncthreads();
        sums = sum_chunk(a, b, at, count, c, mine);
      }
      if (b < a.B) a.kv_len_out[b] = mine.ended && !mine.bad ? 0 : c.ok[t] ? mine.have + mine.tokens : -1 - mine.have;
      const int back = (int)sums.back;
      for (int k = t; k < back; k += kTabThreads) {
        const int s = owner(c.back_start, k);
        const int page = a.table[(long long)(b0 + s) * a.table_stride + (k - c.back_start[s])];
        const long long to = left + at.back + k;
        const bool fits = (unsigned)page < (unsigned)a.n_pages && to < a.capacity;
        if (!fits) flags |= ENTMAX_ATTN_FLAG_BAD_PAGE;
        if (to < a.capacity) a.free_pages[to] = page;
      }
      at.tokens += sums.tokens; at.pages += sums.pages; at.back += sums.back;
    }
    if (t == 0) a.free_count_out[0] = (int)min(left + at.back, (long long)a.capacity);
  }
  if (flags && a.status) atomicOr(a.status + ENTMAX_ATTN_STATUS_FLAGS, flags);
}

}  // namespace

}  // namespace entmax

using namespace entmax;

extern "C" int entmax_attn_paged_tables(const entmax_attn_paged_tables_params* p, const int32_t* kv_len, const int32_t* new_len,
                                        int32_t* block_table, int32_t* free_pages, const int32_t* free_count, int32_t* kv_len_out, int32_t* cu_q,
                                        int32_t* positions, int64_t* slots, int32_t* free_count_out, int32_t* device_status, void* cuda_stream) {
  if (!p) return ENTMAX_ATTN_EINVAL_NULL;
  if (p->batch < 1 || p->total_q < 0 || p->num_pages < 1 || p->max_pages < 1 || p->free_capacity < 0 || p->table_stride < p->max_pages)
    return ENTMAX_ATTN_EINVAL_SHAPE;
  if (p->page_size < 16 || p->page_size > 65536 || (p->page_size & (p->page_size - 1)) != 0) return ENTMAX_ATTN_EINVAL_SHAPE;
  if ((long long)p->max_pages * p->page_size > ENTMAX_ATTN_PAGED_MAX_KV) return ENTMAX_ATTN_EINVAL_SHAPE;
  if (!kv_len || !new_len || !block_table || (!free_pages && p->free_capacity > 0) || !free_count || !kv_len_out || !cu_q || !free_count_out)
    return ENTMAX_ATTN_EINVAL_NULL;
  const uintptr_t all = reinterpret_cast<uintptr_t>(kv_len) | reinterpret_cast<uintptr_t>(new_len) | reinterpret_cast<uintptr_t>(block_table) |
                        reinterpret_cast<uintptr_t>(free_pages) | reinterpret_cast<uintptr_t>(free_count) | reinterpret_cast<uintptr_t>(kv_len_out) |
                        reinterpret_cast<uintptr_t>(cu_q) | reinterpret_cast<uintptr_t>(positions) | reinterpret_cast<uintptr_t>(free_count_out);
  if ((all & 3u) || (reinterpret_cast<uintptr_t>(slots) & 7u)) return ENTMAX_ATTN_EINVAL_ALIGN;
  TablesArgs a;
  a.B = p->batch; a.T = p->total_q;
  a.ps_shift = 31 - __builtin_clz((unsigned)p->page_size);
  a.n_pages = p->num_pages; a.max_pages = p->max_pages; a.capacity = p->free_capacity; a.table_stride = p->table_stride;
  a.kv_len = kv_len; a.new_len = new_len; a.table = block_table; a.free_pages = free_pages; a.free_count = free_count;
  a.kv_len_out = kv_len_out; a.cu_q = cu_q; a.positions = positions; a.slots = reinterpret_cast<long long*>(slots);
  a.free_count_out = free_count_out; a.status = device_status;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t err;
  if (device_status) {
    err = cudaMemsetAsync(device_status, 0, sizeof(int32_t) * ENTMAX_ATTN_STATUS_WORDS, stream);
    if (err != cudaSuccess) return fail_cuda(err);
  }
  // four tokens a thread, as far as a portable cluster goes
  int ctas = 1;
  while (ctas < kTabMaxCtas && (long long)ctas * 4 * kTabThreads < a.T) ctas *= 2;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim = {(unsigned)ctas, 1, 1};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kTabThreads);
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  err = cudaLaunchKernelEx(&cfg, paged_tables_kernel, a, ctas);
  return err == cudaSuccess ? ENTMAX_ATTN_OK : fail_cuda(err);
}
