// Penalties, biases and grammar masks on the logits of all tree nodes, before verification.
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "launch.cuh"

using namespace stand;

namespace {

constexpr int LG_SMS = 148;        // multiprocessors of a B200
constexpr int LG_THREADS = 256;
constexpr int LG_CHUNK = 4096;     // tokens of the vocabulary per block in a large batch
constexpr int LG_BLOCKS = 5;       // blocks per multiprocessor
constexpr int LG_CHUNK_MAX = 5120; // so many of them still fit its shared memory
constexpr int LG_VECS = 4;         // 16-byte pieces a lane has in flight
constexpr uint32_t PROMPT_BIT = 0x80000000u, DRAFT_BIT = 0x40000000u;  // of a token's count: in the prompt; drafted somewhere

struct LogitsParams {
  const char* in;
  char* out;
  long long in_stride, out_stride;  // bytes between rows
  int B, N, V, chunk, n_chunks, sub, words, masks, biases, text_stride;
  const int* text;
  const long long* n_text;
  const long long* n_prompt;
  const int* tree;
  const float* repetition;
  const float* frequency;
  const float* presence;
  const int* bias_start;
  const int* bias_id;
  const float* bias_value;
  const uint32_t* mask;
  const int* mask_row;
  short parent[NODES_MAX];
};

template <int DT> struct Elem;
template <> struct Elem<0> {
  typedef float T;
  static constexpr int VE = 4;  // elements per 16 bytes
  static constexpr uint32_t NEG_INF = 0xFF800000u;
  __device__ static __forceinline__ float load(const char* p) { return *reinterpret_cast<const float*>(p); }
  __device__ static __forceinline__ void store(char* p, float v) { *reinterpret_cast<float*>(p) = v; }
  // keeps the elements whose bit is set, -inf for the others
  __device__ static __forceinline__ uint4 keep(uint4 d, uint32_t bits) {
    d.x = bits & 1 ? d.x : NEG_INF;
    d.y = bits & 2 ? d.y : NEG_INF;
    d.z = bits & 4 ? d.z : NEG_INF;
    d.w = bits & 8 ? d.w : NEG_INF;
    return d;
  }
};
template <> struct Elem<1> {
  typedef unsigned short T;
  static constexpr int VE = 8;
  __device__ static __forceinline__ float load(const char* p) {
    return __uint_as_float((uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16);
  }
  __device__ static __forceinline__ void store(char* p, float v) {
    unsigned short h;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(h) : "f"(v));
    *reinterpret_cast<unsigned short*>(p) = h;
  }
  // two elements by two bits: b0 lands in bit 7, b1 in bit 15, and prmt spreads those over two bytes each
  __device__ static __forceinline__ uint32_t keep2(uint32_t d, uint32_t bits) {
    uint32_t m;
    asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(m) : "r"((bits & 3u) * 0x4080u));
    return (d & m) | (0xFF80FF80u & ~m);
  }
  __device__ static __forceinline__ uint4 keep(uint4 d, uint32_t bits) {
    d.x = keep2(d.x, bits);
    d.y = keep2(d.y, bits >> 2);
    d.z = keep2(d.z, bits >> 4);
    d.w = keep2(d.w, bits >> 6);
    return d;
  }
};

// 32 mask bits from token t on (those past the mask's end are 0).
__device__ __forceinline__ uint32_t mask_bits(const uint32_t* row, int words, int t) {
  const int w = t >> 5, sh = t & 31;
  uint32_t bits = __ldg(row + w) >> sh;
  if (sh && w + 1 < words) bits |= __ldg(row + w + 1) << (32 - sh);
  return bits;
}

struct Penalty {
  float r, r_inv, f, p;
};

// The penalties' own arithmetic, each operation rounded by itself (no contraction).  x / r is x times 1 / r, rounded
// twice instead of once: an ulp of single precision off at most.  (With a division for each: 256 x 24 rows of 151,936 622 us
// instead of 603, 64 rows of 50,257 17.5 instead of 16.8.)
__device__ __forceinline__ float process(float x, bool met, uint32_t count, const Penalty& q, bool has_bias, float bias) {
  if (met) x = __fmul_rn(x, x > 0.0f ? q.r_inv : q.r);
  if (count) x = __fsub_rn(__fsub_rn(x, __fmul_rn(q.f, (float)count)), q.p);
  if (has_bias) x = __fadd_rn(x, bias);
  return x;
}

// Sends tokens [t0, t1) of a row through: -inf where the mask forbids, `fix` of those whose bit in `touched` (bit 0: token
// c0) is set, the others as they are.  In place only what changes is read or written; a piece that the mask forbids whole
// is not read.
template <int DT, bool MASK, typename F>
__device__ __forceinline__ void stream_row(const char* in, char* out, int t0, int t1, const uint32_t* mask, int words, const uint32_t* touched,
                                           int c0, int lane, F fix) {
  using E = Elem<DT>;
  constexpr int ES = 16 / E::VE;
  constexpr uint32_t ALL = (1u << E::VE) - 1;
  const bool in_place = in == out;
  const uint32_t off = (uint32_t)((uintptr_t)(in + (long long)t0 * ES) & 15);
  int a = t0 + (int)((16 - off) & 15) / ES;  // first token on a 16-byte boundary of the input
  if ((((uintptr_t)in ^ (uintptr_t)out) & 15) != 0 || a > t1) a = t1;
  const int n_vec = (t1 - a) / E::VE;
  const int b = a + n_vec * E::VE;
  // the ends (all of it when input and output lie differently): one element at a time
  const int n_edge = (a - t0) + (t1 - b);
  for (int i = lane; i < n_edge; i += 32) {
    const int t = i < a - t0 ? t0 + i : b + (i - (a - t0));
    if (MASK && !(mask_bits(mask, words, t) & 1)) {
      E::store(out + (long long)t * ES, -INFINITY);
      continue;
    }
    const bool hit = touched[(t - c0) >> 5] >> ((t - c0) & 31) & 1u;
    if (hit) E::store(out + (long long)t * ES, fix(E::load(in + (long long)t * ES), t - c0));
    else if (!in_place) *reinterpret_cast<typename E::T*>(out + (long long)t * ES) = *reinterpret_cast<const typename E::T*>(in + (long long)t * ES);
  }
  const char* src = in + (long long)a * ES;
  char* dst = out + (long long)a * ES;
  const bool even = (a & (E::VE - 1)) == 0;  // a piece's bits lie in one byte (chunks begin at multiples of 512)
#pragma unroll 1
  for (int v0 = lane; v0 < n_vec; v0 += 32 * LG_VECS) {
    uint4 d[LG_VECS];
    uint32_t bits[LG_VECS], hits[LG_VECS];
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32, t = a + v * E::VE;
      bits[e] = ALL;
      hits[e] = 0;
      if (v < n_vec) {
        const int at = t - c0;
        if (even) {
          hits[e] = (uint32_t)reinterpret_cast<const unsigned char*>(touched)[at >> 3] >> (E::VE == 4 ? at & 4 : 0) & ALL;
          if (MASK) bits[e] = (uint32_t)__ldg(reinterpret_cast<const unsigned char*>(mask) + (t >> 3)) >> (E::VE == 4 ? t & 4 : 0) & ALL;
        } else {
          hits[e] = __funnelshift_r(touched[at >> 5], touched[(at >> 5) + 1], at & 31) & ALL;
          if (MASK) bits[e] = mask_bits(mask, words, t) & ALL;
        }
      }
    }
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32;
      d[e] = make_uint4(0, 0, 0, 0);
      hits[e] &= bits[e];
      if (v < n_vec && bits[e] != 0 && !(in_place && bits[e] == ALL && hits[e] == 0)) d[e] = *reinterpret_cast<const uint4*>(src + (size_t)v * 16);
    }
    uint32_t todo = 0;
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32;
      todo |= hits[e] << (e * E::VE);
      if (v < n_vec && !(in_place && bits[e] == ALL && hits[e] == 0)) *reinterpret_cast<uint4*>(dst + (size_t)v * 16) = MASK ? E::keep(d[e], bits[e]) : d[e];
    }
    for (; todo; todo &= todo - 1) {  // over all pieces at once: few rounds for the warp; the lines are at hand
      const int i = __ffs(todo) - 1, t = a + (v0 + i / E::VE * 32) * E::VE + i % E::VE;
      E::store(out + (long long)t * ES, fix(E::load(in + (long long)t * ES), t - c0));
    }
  }
}

// A block takes one chunk of the vocabulary of one sequence, for all its nodes: it counts the text's tokens of that
// chunk once in shared memory and marks them, the biased and the drafted ones in a bit map; then its warps stream the
// nodes' rows through.  Nearly all logits are only copied; those marked are changed as soon as their pieces have
// gone by (after the whole rows it took 936 us instead of 600 for 256 x 24 rows: their lines had left L2).  HBM-bound: every logit is read
// and written once.  Measured: 256 x 24 rows of 151,936 bf16 with biases and masks 603 us = 6.2 TB/s, 0.95 of the copy
// bandwidth (a plain copy of the same bytes 572 - 580); 8 rows of 32,000 4.0 us; 64 rows of 50,257 with texts of 6,000 - 12,000
// 17 us, bound by the chain text - counts - rows.
template <int DT>
__global__ void __launch_bounds__(LG_THREADS, LG_BLOCKS) logits_kernel(const __grid_constant__ LogitsParams p) {
  extern __shared__ uint32_t lg_smem[];
  __shared__ short s_node[NODES_MAX];  // the drafted token of each node, as a place in the chunk; -1: none there
  const int chunk = p.chunk;
  uint32_t* const s_count = lg_smem;                                           // [chunk]
  uint32_t* const s_bits = s_count + chunk;                                    // [chunk / 32 + 1]: marked tokens
  int* const s_bias = reinterpret_cast<int*>(s_bits + chunk / 32 + 1);         // [chunk] with biases: 1 + the entry
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < chunk + chunk / 32 + 1; i += LG_THREADS) s_count[i] = 0;
  if (p.bias_start)
    for (int i = tid; i < chunk; i += LG_THREADS) s_bias[i] = 0;
  const int b = blockIdx.x / p.n_chunks, c0 = (blockIdx.x % p.n_chunks) * chunk;
  const int width = p.V - c0 < chunk ? p.V - c0 : chunk;
  const int n_sub = (width + p.sub - 1) / p.sub;
  const int tasks = p.N * n_sub;
  pdl_wait();
  // all that later steps wait for, asked for at once; and the first piece of each warp's rows on its way to L2
  long long have = 0, first = 0;
  int bias_from = 0, bias_to = 0;
  Penalty q;
  if (p.text) have = p.n_text[b];
  if (p.n_prompt) first = p.n_prompt[b];
  if (p.bias_start) bias_from = max(p.bias_start[b], 0), bias_to = min(p.bias_start[b + 1], p.biases);
  q.r = p.repetition ? p.repetition[b] : 1.0f;
  q.f = p.frequency ? p.frequency[b] : 0.0f;
  q.p = p.presence ? p.presence[b] : 0.0f;
  if (warp < tasks && p.in != p.out) {
    const int u = warp / n_sub, lo = (warp - u * n_sub) * p.sub;
    const long long bytes = (long long)(width - lo < p.sub ? width - lo : p.sub) * (DT == 0 ? 4 : 2);
    const char* row = p.in + ((long long)b * p.N + u) * p.in_stride + (long long)(c0 + lo) * (DT == 0 ? 4 : 2);
    for (long long at = lane * 128; at < bytes; at += 32 * 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + at));
  }
  __syncthreads();
  auto touch = [&](uint32_t i) { atomicOr(&s_bits[i >> 5], 1u << (i & 31)); };
  if (p.tree)
    for (int v = tid; v < p.N; v += LG_THREADS) {
      const int t = p.tree[(long long)b * p.N + v];
      const bool here = v > 0 && t >= c0 && t < c0 + width;
      s_node[v] = here ? (short)(t - c0) : (short)-1;
      if (here) {
        atomicOr(&s_count[t - c0], DRAFT_BIT);
        touch(t - c0);
      }
    }
  if (p.text) {
    const int n = have < 0 ? 0 : (have > p.text_stride ? p.text_stride : (int)have);
    const int* row = p.text + (long long)b * p.text_stride;
    auto count = [&](int t, int i) {
      const uint32_t at = (uint32_t)t - (uint32_t)c0;
      if (at >= (uint32_t)width) return;
      const uint32_t old = i < first ? atomicOr(&s_count[at], PROMPT_BIT) : atomicAdd(&s_count[at], 1u);
      if ((old & ~DRAFT_BIT) == 0) touch(at);
    };
    const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) >> 2);
    const int a = head < n ? head : n;
    const int n4 = (n - a) >> 2;
    if (tid < a) count(row[tid], tid);
    const int4* row4 = reinterpret_cast<const int4*>(row + a);
    for (int i0 = tid; i0 < n4; i0 += LG_THREADS * 4) {
      int4 t[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) t[e] = i0 + e * LG_THREADS < n4 ? row4[i0 + e * LG_THREADS] : make_int4(-1, -1, -1, -1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = a + 4 * (i0 + e * LG_THREADS);
        count(t[e].x, i);
        count(t[e].y, i + 1);
        count(t[e].z, i + 2);
        count(t[e].w, i + 3);
      }
    }
    const int i = a + 4 * n4 + tid;
    if (i < n) count(row[i], i);
  }
  if (p.bias_start) {
    for (int i = bias_from + tid; i < bias_to; i += LG_THREADS) {
      const uint32_t at = (uint32_t)p.bias_id[i] - (uint32_t)c0;
      if (at >= (uint32_t)width) continue;
      atomicMax(&s_bias[at], i + 1);
      touch(at);
    }
  }

  __syncthreads();

  q.r_inv = 1.0f / q.r;
  for (int task = warp; task < tasks; task += LG_THREADS / 32) {
    const int u = task / n_sub, lo = c0 + (task - u * n_sub) * p.sub;
    const int hi = lo + p.sub < c0 + width ? lo + p.sub : c0 + width;
    const long long r = (long long)b * p.N + u;
    const char* in = p.in + r * p.in_stride;
    char* out = p.out + r * p.out_stride;
    const uint32_t* mask = nullptr;
    if (p.mask) {
      const int m = p.mask_row[r];
      if (m >= 0 && m < p.masks) mask = p.mask + (long long)m * p.words;
    }
    auto fix = [&](float x, int at) {  // a marked token of this row
      const uint32_t w = s_count[at];
      uint32_t on_path = 0;
      if (w & DRAFT_BIT)
        for (int v = u; v > 0; v = p.parent[v]) on_path += s_node[v] == at;
      const uint32_t c = (w & ~(PROMPT_BIT | DRAFT_BIT)) + on_path;
      const int e = p.bias_start ? s_bias[at] : 0;
      return process(x, (w & PROMPT_BIT) != 0 || c != 0, c, q, e != 0, e ? p.bias_value[e - 1] : 0.0f);
    };
    if (mask) stream_row<DT, true>(in, out, lo, hi, mask, p.words, s_bits, c0, lane, fix);
    else stream_row<DT, false>(in, out, lo, hi, mask, p.words, s_bits, c0, lane, fix);
  }
}

// Does a row of the output lie over another part of the input?  Rows of `row` bytes, `in_stride` and `out_stride` apart; the
// same rows (in place) do not count, and rows of equal stride may lie between one another.
bool rows_overlap(const void* in, const void* out, long long rows, long long row, long long in_stride, long long out_stride) {
  const uintptr_t x = (uintptr_t)in, y = (uintptr_t)out;
  if (x == y || x + (rows - 1) * in_stride + row <= y || y + (rows - 1) * out_stride + row <= x) return false;
  if (in_stride != out_stride) return true;
  const long long off = (long long)((y > x ? y - x : x - y) % (uintptr_t)in_stride);
  return off < row || in_stride - off < row;
}

}  // namespace

extern "C" int stand_process_logits(const stand_logits* c, const stand_logits_inputs* x, const void* dev_in, void* dev_out,
                                    void* cu_stream) {
  if (!c || !x || !dev_in || !dev_out) return STAND_E_ARG;
  if (c->B < 1 || c->N < 1 || c->N > STAND_MAX_NODES || c->V < 2 || c->V > STAND_MAX_VOCAB) return STAND_E_ARG;
  if (c->dtype != STAND_DTYPE_F32 && c->dtype != STAND_DTYPE_BF16) return STAND_E_ARG;
  if (c->in_stride < c->V || c->out_stride < c->V || c->text_stride < 0 || c->masks < 0 || c->biases < 0 || c->reserved != 0) return STAND_E_ARG;
  if (dev_in == dev_out && c->in_stride != c->out_stride) return STAND_E_ARG;
  const int es = c->dtype == STAND_DTYPE_F32 ? 4 : 2;
  if (rows_overlap(dev_in, dev_out, (long long)c->B * c->N, (long long)c->V * es, c->in_stride * es, c->out_stride * es)) return STAND_E_ARG;
  if (!c->parent && c->N > 1) return STAND_E_ARG;
  if ((x->text != nullptr) != (x->n_text != nullptr) || (x->n_prompt && !x->text)) return STAND_E_ARG;
  if (x->bias_start && c->biases > 0 && (!x->bias_id || !x->bias_value)) return STAND_E_ARG;
  if ((x->mask != nullptr) != (x->mask_row != nullptr)) return STAND_E_ARG;
  if (!aligned(es, dev_in, dev_out) || !aligned(8, x->n_text, x->n_prompt) ||
      !aligned(4, x->text, x->tree_tokens, x->repetition, x->frequency, x->presence, x->bias_start, x->bias_id, x->bias_value, x->mask, x->mask_row))
    return STAND_E_ARG;
  LogitsParams p;
  int depth[STAND_MAX_NODES];
  depth[0] = 0;
  p.parent[0] = -1;
  if (c->parent && c->parent[0] != -1) return STAND_E_ARG;
  for (int u = 1; u < c->N; ++u) {
    const int par = c->parent[u];
    if (par < 0 || par >= u) return STAND_E_ARG;
    depth[u] = depth[par] + 1;
    if (depth[u] > STAND_MAX_DEPTH) return STAND_E_ARG;
    p.parent[u] = (short)par;
  }
  p.in = (const char*)dev_in; p.out = (char*)dev_out; p.in_stride = c->in_stride * es; p.out_stride = c->out_stride * es;
  p.B = c->B; p.N = c->N; p.V = c->V; p.words = (c->V + 31) / 32; p.masks = c->masks; p.biases = c->biases;
  p.text_stride = c->text_stride; p.text = x->text; p.n_text = (const long long*)x->n_text; p.n_prompt = (const long long*)x->n_prompt;
  p.tree = x->tree_tokens; p.repetition = x->repetition; p.frequency = x->frequency; p.presence = x->presence;
  p.bias_start = x->bias_start; p.bias_id = x->bias_id; p.bias_value = x->bias_value; p.mask = x->mask; p.mask_row = x->mask_row;
  // A small batch is cut finer, so that it reaches all multiprocessors (two blocks each) down to 512 tokens (8 rows of 32,000:
  // 4.0 us instead of 9.2); a text is scanned once per chunk, so a large one is not.
  p.chunk = LG_CHUNK;
  while (p.chunk > 512 && (long long)c->B * ((c->V + p.chunk - 1) / p.chunk) < 2 * LG_SMS) p.chunk /= 2;
  // Between one and two rounds of blocks: larger chunks, if that makes it one.  With / without, texts of 6,000: 64 rows of 50,257 12.8 /
  // 16.1 us, 76 of 40,000 12.6 / 14.9, 22 of 151,936 10.0 / 12.7, 93 of 32,000 13.1 / 15.2; just past one round (57 of 50,257) 12.9 / 12.3.
  const long long round = LG_SMS * LG_BLOCKS;
  if (p.chunk == LG_CHUNK && (long long)c->B * ((c->V + LG_CHUNK - 1) / LG_CHUNK) > round)
    for (int ch = LG_CHUNK + 512; ch <= LG_CHUNK_MAX; ch += 512)
      if ((long long)c->B * ((c->V + ch - 1) / ch) <= round) {
        p.chunk = ch;
        break;
      }
  p.n_chunks = (c->V + p.chunk - 1) / p.chunk;
  // few nodes are cut into more pieces: four or so for each warp
  p.sub = p.chunk;
  while (p.sub >= 1024 && c->N * (p.chunk / p.sub) < LG_THREADS / 8) p.sub = (p.sub / 2 + 31) & ~31;
  const long long blocks = (long long)c->B * p.n_chunks;
  if (blocks > 0x7FFFFFFFll) return STAND_E_ARG;
  const size_t smem = (size_t)p.chunk * (sizeof(int) + (x->bias_start ? sizeof(int) : 0)) + p.chunk / 8 + sizeof(int);
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (c->dtype == STAND_DTYPE_BF16) return launch_dependent(logits_kernel<1>, dim3((unsigned)blocks), LG_THREADS, st, p, smem);
  return launch_dependent(logits_kernel<0>, dim3((unsigned)blocks), LG_THREADS, st, p, smem);
}
