// The paged cache's bookkeeping on the GPU: pages and slots for new tokens, pages of finished sequences,
// and the copy of accepted keys and values into their slots.
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "launch.cuh"

using namespace stand;

namespace {

constexpr int MAP_THREADS = 256;
constexpr int MAP_SEQS = 8;         // sequences per block when a sequence has few new tokens
constexpr int MAP_TOKENS = 2048;    // new tokens of one sequence per block when it has many

struct MapParams {
  const long long* len;
  const int* n_new;
  int B, width, page, cols, capacity;
  int per_block, split;  // sequences per block; blocks per group of sequences
  const int* free_list;
  const int* n_free;
  int* table;
  long long* slots;
  int* granted;
  long long* len_out;
  int* n_free_out;
};

__device__ __forceinline__ int free_count(const int* n_free, int capacity) {
  const int n = *n_free;
  return n < 0 ? 0 : (n > capacity ? capacity : n);
}

// What sequence b asks for: pages it has, pages it will have; false if the request itself is refused.
__device__ __forceinline__ bool map_request(const MapParams& p, int b, long long& len, int& fresh, long long& have, long long& want) {
  len = p.len[b];
  fresh = p.n_new[b];
  have = want = 0;
  if (len < 0 || fresh < 0 || fresh > p.width || len > (long long)p.cols * p.page) return false;
  have = (len + p.page - 1) / p.page;
  want = (len + fresh + p.page - 1) / p.page;
  return want <= p.cols;
}

// Sum over the block; every thread gets it.  Two barriers.
__device__ __forceinline__ long long block_sum(long long v, long long* s_part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
  if ((threadIdx.x & 31) == 0) s_part[threadIdx.x >> 5] = v;
  __syncthreads();
  long long total = 0;
#pragma unroll
  for (int w = 0; w < MAP_THREADS / 32; ++w) total += s_part[w];
  __syncthreads();
  return total;
}

// need_b = ceil((len_b + new_b) / page) - ceil(len_b / page) pages, taken from the top of the free list at the
// exclusive prefix sum of need.  A few hundred requests are some KB, so a block does not wait for a scan by
// others: it sums the needs before its own sequences itself (from L2), scans its own, and writes.  One launch;
// at these sizes the time is that of a launch and three dependent reads (lengths, free list or table, slots): 3.7 us
// for 256 sequences x 7 tokens, 6.2 us for 96 prompts of up to 8,192 (an empty kernel: 2.6 us).
__global__ void __launch_bounds__(MAP_THREADS) page_map_kernel(const MapParams p) {
  __shared__ long long s_part[MAP_THREADS / 32];
  __shared__ long long s_col[MAP_SEQS], s_have[MAP_SEQS], s_want[MAP_SEQS], s_at[MAP_SEQS];  // s_col, s_off: where the first new token goes
  __shared__ unsigned s_off[MAP_SEQS];
  __shared__ int s_new[MAP_SEQS];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x;
  const int group = blockIdx.x / p.split, part = blockIdx.x % p.split;
  const int first = group * p.per_block;
  const int n_own = p.B - first < p.per_block ? p.B - first : p.per_block;
  const int n_free = free_count(p.n_free, p.capacity);

  long long before = 0;
  for (int b = tid; b < first; b += MAP_THREADS) {
    long long len, have, want;
    int fresh;
    if (map_request(p, b, len, fresh, have, want)) before += want - have;
  }
  before = block_sum(before, s_part);
  if (tid < 32) {
    long long len = 0, have = 0, want = 0;
    int fresh = 0;
    const bool mine = tid < n_own;
    const bool fits = mine && map_request(p, first + tid, len, fresh, have, want);
    const long long need = fits ? want - have : 0;
    long long upto = need;
#pragma unroll
    for (int o = 1; o < MAP_SEQS; o <<= 1) {
      const long long t = __shfl_up_sync(FULL, upto, o);
      if (tid >= o) upto += t;
    }
    upto += before;
    const bool served = fits && (need == 0 || upto <= n_free);
    if (mine) {
      s_col[tid] = len > 0 ? len / p.page : 0;
      s_off[tid] = len > 0 ? (unsigned)(len - s_col[tid] * p.page) : 0u;
      s_have[tid] = have;
      s_want[tid] = served ? want : have;
      s_at[tid] = n_free - 1 - (upto - need);  // index of this sequence's first page in the free list
      s_new[tid] = served ? fresh : 0;
      if (part == 0) {
        if (p.granted) p.granted[first + tid] = served ? fresh : -1;
        if (p.len_out) p.len_out[first + tid] = len + (served ? fresh : 0);
      }
    }
    // the pages taken are the largest prefix sum that the list covers: it lies in the block where the sums pass
    // the list's size, or in the last one
    const long long end = __shfl_sync(FULL, upto, n_own - 1);
    long long taken = mine && upto <= n_free ? upto : before;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const long long t = __shfl_xor_sync(FULL, taken, o);
      taken = t > taken ? t : taken;
    }
    if (tid == 0 && part == 0 && before <= n_free && (end > n_free || first + n_own == p.B)) *p.n_free_out = n_free - (int)taken;
  }
  __syncthreads();

  for (int s = 0; s < n_own; ++s) {
    int* row = p.table + (long long)(first + s) * p.cols;
    for (long long c = s_have[s] + part * MAP_THREADS + tid; c < s_want[s]; c += (long long)p.split * MAP_THREADS)
      row[c] = p.free_list[s_at[s] - (c - s_have[s])];
  }
  // slots: the page of a position is an old table entry or comes from the free list, never from what another
  // thread of this launch writes
  const int items = n_own * p.width;
  for (int i = part * MAP_THREADS + tid; i < items; i += p.split * MAP_THREADS) {
    const int s = p.per_block == 1 ? 0 : i / p.width, j = i - s * p.width;
    long long slot = -1;
    if (j < s_new[s]) {
      // 32-bit arithmetic from the first new token's place on: the long division is done once per sequence
      const unsigned off = s_off[s] + (unsigned)j, c = off / (unsigned)p.page;
      const long long col = s_col[s] + c;
      const int page = col < s_have[s] ? p.table[(long long)(first + s) * p.cols + col] : p.free_list[s_at[s] - (col - s_have[s])];
      if (page >= 0) slot = (long long)page * p.page + (off - c * (unsigned)p.page);
    }
    p.slots[(long long)first * p.width + i] = slot;
  }
}

struct ReleaseParams {
  const long long* len;
  const int* done;
  int B, page, cols, capacity;
  const int* table;
  int* free_list;
  const int* n_free;
  long long* len_out;
  int* n_free_out;
};

// One block per sequence; each sums the pages given back before its own.
__global__ void __launch_bounds__(MAP_THREADS) page_release_kernel(const ReleaseParams p) {
  __shared__ long long s_part[MAP_THREADS / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, own = blockIdx.x;
  const int n_free = free_count(p.n_free, p.capacity);
  auto pages_of = [&](int b) -> long long {
    const long long len = p.len[b];
    if (!p.done[b] || len <= 0) return 0;
    const long long n = (len + p.page - 1) / p.page;
    return n < p.cols ? n : p.cols;
  };
  long long before = 0;
  for (int b = tid; b < own; b += MAP_THREADS) before += pages_of(b);
  before = block_sum(before, s_part);
  const long long mine = pages_of(own);
  for (long long i = tid; i < mine; i += MAP_THREADS) {
    const long long at = n_free + before + i;
    if (at < p.capacity) p.free_list[at] = p.table[(long long)own * p.cols + i];
  }
  if (tid == 0) {
    p.len_out[own] = p.done[own] ? 0 : p.len[own];
    if (own == p.B - 1) {
      const long long n = n_free + before + mine;
      *p.n_free_out = (int)(n < p.capacity ? n : p.capacity);
    }
  }
}

// ---------------------------------------------------------------------------------
// Commit
// ---------------------------------------------------------------------------------
constexpr int COMMIT_THREADS = 256;
constexpr int COMMIT_UNROLL = 4;

struct CommitParams {
  const char* k;
  const char* v;
  char* cache_k;
  char* cache_v;
  const int* path;
  const long long* slots;
  int layers, N, width, heads, page, units;  // units: 16-byte (or element) pieces of one row
  int layers_per_block;
  long long n_slots;
  long long src_k[4], src_v[4], dst[4];  // strides in bytes
};

// A block copies one token's rows of some layers: a piece of W bytes per thread and step, four steps in flight (one layer
// per block: 43 us instead of 14 for 200 accepted paths of 28 layers).  Bound by HBM (each accepted row is read and written once)
// when many tokens are accepted: 279 MB in 47.4 us = 5.9 TB/s, 0.90 of the copy bandwidth; by the chain slot -> row -> store when
// few are: 4.3 us for 16 paths of 28 layers.
template <typename W>
__global__ void __launch_bounds__(COMMIT_THREADS) kv_commit_kernel(const CommitParams p) {
  pdl_trigger();
  pdl_wait();
  const int place = blockIdx.x;
  const long long slot = p.slots[place];
  const int b = place / p.width, j = place - b * p.width;
  const int node = p.path ? p.path[place] : j;
  if (slot < 0 || slot >= p.n_slots || node < 0 || node >= p.N) return;
  const int l0 = blockIdx.y * p.layers_per_block;
  const int nl = p.layers - l0 < p.layers_per_block ? p.layers - l0 : p.layers_per_block;
  const long long page = slot / p.page;
  const long long from_k = b * p.src_k[1] + node * p.src_k[2], from_v = b * p.src_v[1] + node * p.src_v[2];
  const long long to = page * p.dst[1] + (slot - page * p.page) * p.dst[3];
  const int per_layer = 2 * p.heads * p.units, total = nl * per_layer;
  for (int i0 = threadIdx.x; i0 < total; i0 += COMMIT_THREADS * COMMIT_UNROLL) {
    W got[COMMIT_UNROLL];
    char* dst[COMMIT_UNROLL];
#pragma unroll
    for (int e = 0; e < COMMIT_UNROLL; ++e) {
      const int i = i0 + e * COMMIT_THREADS;
      dst[e] = nullptr;
      if (i < total) {
        const int l = i / per_layer, in_layer = i - l * per_layer;
        const int row = in_layer / p.units, unit = in_layer - row * p.units;
        const bool is_v = row >= p.heads;
        const int h = is_v ? row - p.heads : row;
        const char* src = is_v ? p.v + (l0 + l) * p.src_v[0] + from_v + h * p.src_v[3] : p.k + (l0 + l) * p.src_k[0] + from_k + h * p.src_k[3];
        src += unit * (int)sizeof(W);
        dst[e] = (is_v ? p.cache_v : p.cache_k) + (l0 + l) * p.dst[0] + to + h * p.dst[2] + unit * (int)sizeof(W);
        got[e] = __ldg(reinterpret_cast<const W*>(src));
      }
    }
#pragma unroll
    for (int e = 0; e < COMMIT_UNROLL; ++e)
      if (dst[e]) *reinterpret_cast<W*>(dst[e]) = got[e];
  }
}

// Blocks read these inputs while others write those outputs.
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return a && b && x < y + b_bytes && y < x + a_bytes;
}

bool aligned16(const void* p, const long long* strides, int n) {
  bool ok = ((uintptr_t)p & 15) == 0;
  for (int i = 0; i < n; ++i) ok = ok && (strides[i] & 15) == 0;
  return ok;
}

}  // namespace

extern "C" {

int stand_page_map(const int64_t* dev_len, const int32_t* dev_new, int32_t B, int32_t width, int32_t page_size, int32_t max_pages,
                   const int32_t* dev_free, int32_t capacity, const int32_t* dev_n_free, int32_t* dev_table, int64_t* dev_slots,
                   int32_t* dev_granted, int64_t* dev_len_out, int32_t* dev_n_free_out, void* cu_stream) {
  if (B < 1 || width < 1 || width > (1 << 27) || page_size < 1 || page_size > (1 << 27) || max_pages < 0 || capacity < 0) return STAND_E_ARG;
  if (!dev_len || !dev_new || !dev_n_free || !dev_slots || !dev_n_free_out) return STAND_E_ARG;
  if ((max_pages > 0 && !dev_table) || (capacity > 0 && !dev_free)) return STAND_E_ARG;
  if (!aligned(8, dev_len, dev_slots, dev_len_out) || !aligned(4, dev_new, dev_free, dev_n_free, dev_table, dev_granted, dev_n_free_out)) return STAND_E_ARG;
  const size_t longs = (size_t)B * 8, ints = (size_t)B * 4;
  if (overlap(dev_len_out, longs, dev_len, longs) || overlap(dev_granted, ints, dev_new, ints) || overlap(dev_granted, ints, dev_n_free, 4) ||
      overlap(dev_n_free_out, 4, dev_n_free, 4) || overlap(dev_n_free_out, 4, dev_new, ints))
    return STAND_E_ARG;
  MapParams p;
  p.len = (const long long*)dev_len; p.n_new = dev_new; p.B = B; p.width = width; p.page = page_size; p.cols = max_pages;
  p.capacity = capacity; p.free_list = dev_free; p.n_free = dev_n_free; p.table = dev_table; p.slots = (long long*)dev_slots;
  p.granted = dev_granted; p.len_out = (long long*)dev_len_out; p.n_free_out = dev_n_free_out;
  // One sequence per block, unless there are so many that the blocks' sums cost more (eight / one per block: 256 sequences
  // 4.5 / 3.7 us, 1,000 sequences 6.7 / 8.5 us).
  p.per_block = B > 512 && width <= MAP_TOKENS / MAP_SEQS ? MAP_SEQS : 1;
  p.split = (int)(((long long)p.per_block * width + MAP_TOKENS - 1) / MAP_TOKENS);
  const long long blocks = (long long)((B + p.per_block - 1) / p.per_block) * p.split;
  if (blocks > 0x7FFFFFFFll) return STAND_E_ARG;
  return launch_dependent(page_map_kernel, dim3((unsigned)blocks), MAP_THREADS, (cudaStream_t)cu_stream, p);
}

int stand_page_release(const int64_t* dev_len, const int32_t* dev_done, int32_t B, int32_t page_size, int32_t max_pages,
                       const int32_t* dev_table, int32_t capacity, int32_t* dev_free, const int32_t* dev_n_free,
                       int64_t* dev_len_out, int32_t* dev_n_free_out, void* cu_stream) {
  if (B < 1 || page_size < 1 || max_pages < 0 || capacity < 0) return STAND_E_ARG;
  if (!dev_len || !dev_done || !dev_n_free || !dev_len_out || !dev_n_free_out) return STAND_E_ARG;
  if ((max_pages > 0 && !dev_table) || (capacity > 0 && !dev_free)) return STAND_E_ARG;
  if (!aligned(8, dev_len, dev_len_out) || !aligned(4, dev_done, dev_table, dev_free, dev_n_free, dev_n_free_out)) return STAND_E_ARG;
  const size_t longs = (size_t)B * 8;
  if (overlap(dev_len_out, longs, dev_len, longs) || overlap(dev_n_free_out, 4, dev_n_free, 4) || overlap(dev_n_free_out, 4, dev_done, (size_t)B * 4))
    return STAND_E_ARG;
  ReleaseParams p;
  p.len = (const long long*)dev_len; p.done = dev_done; p.B = B; p.page = page_size; p.cols = max_pages; p.capacity = capacity;
  p.table = dev_table; p.free_list = dev_free; p.n_free = dev_n_free; p.len_out = (long long*)dev_len_out;
  p.n_free_out = dev_n_free_out;
  return launch_dependent(page_release_kernel, dim3((unsigned)B), MAP_THREADS, (cudaStream_t)cu_stream, p);
}

int stand_kv_commit(const stand_kv_shape* c, const void* dev_k, const void* dev_v, const int32_t* dev_path, const int64_t* dev_slots,
                    void* dev_cache_k, void* dev_cache_v, void* cu_stream) {
  if (!c || !dev_k || !dev_v || !dev_slots || !dev_cache_k || !dev_cache_v) return STAND_E_ARG;
  if (c->layers < 1 || c->layers > 65535 || c->B < 1 || c->N < 1 || c->heads < 1 || c->dim < 1 || c->width < 1) return STAND_E_ARG;
  if (c->page_size < 1 || c->pages < 0 || c->reserved != 0 || c->dtype < STAND_DTYPE_F32 || c->dtype > STAND_DTYPE_F16) return STAND_E_ARG;
  if ((long long)c->heads * c->dim > (1 << 20) || (long long)c->B * c->width > 0x7FFFFFFFll) return STAND_E_ARG;
  if ((c->own_v_stride != 0 && c->own_v_stride != 1) || c->reserved2 != 0) return STAND_E_ARG;
  const int64_t* v_stride = c->own_v_stride ? c->v_stride : c->src_stride;
  for (int i = 0; i < 4; ++i)
    if (c->src_stride[i] < 0 || c->cache_stride[i] < 0 || v_stride[i] < 0) return STAND_E_ARG;
  const int es = c->dtype == STAND_DTYPE_F32 ? 4 : 2;
  if (!aligned(es, dev_k, dev_v, dev_cache_k, dev_cache_v) || !aligned(8, dev_slots) || !aligned(4, dev_path)) return STAND_E_ARG;
  CommitParams p;
  p.k = (const char*)dev_k; p.v = (const char*)dev_v; p.cache_k = (char*)dev_cache_k; p.cache_v = (char*)dev_cache_v;
  p.path = dev_path; p.slots = (const long long*)dev_slots; p.layers = c->layers; p.N = c->N; p.width = c->width; p.heads = c->heads;
  p.page = c->page_size; p.n_slots = (long long)c->pages * c->page_size;
  for (int i = 0; i < 4; ++i) { p.src_k[i] = c->src_stride[i] * es; p.src_v[i] = v_stride[i] * es; p.dst[i] = c->cache_stride[i] * es; }
  const bool wide = (c->dim * es) % 16 == 0 && aligned16(dev_k, p.src_k, 4) && aligned16(dev_v, p.src_v, 4) &&
                    aligned16(dev_cache_k, p.dst, 4) && aligned16(dev_cache_v, p.dst, 4);
  p.units = wide ? c->dim * es / 16 : c->dim;
  // enough layers per block for its threads to have COMMIT_UNROLL pieces each
  const long long per_layer = 2ll * p.heads * p.units;
  long long lpb = COMMIT_THREADS * COMMIT_UNROLL / per_layer;
  lpb = lpb < 1 ? 1 : (lpb > c->layers ? c->layers : lpb);
  p.layers_per_block = (int)lpb;
  const dim3 grid((unsigned)(c->B * c->width), (unsigned)((c->layers + lpb - 1) / lpb));
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (wide) return launch_dependent(kv_commit_kernel<uint4>, grid, COMMIT_THREADS, st, p);
  if (es == 4) return launch_dependent(kv_commit_kernel<uint32_t>, grid, COMMIT_THREADS, st, p);
  return launch_dependent(kv_commit_kernel<unsigned short>, grid, COMMIT_THREADS, st, p);
}

}  // extern "C"
