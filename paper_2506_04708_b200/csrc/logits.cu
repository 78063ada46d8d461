// Penalties, biases and grammar masks on the logits of all tree nodes, before verification.
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"
#include "launch.cuh"

using namespace stand;

namespace {

constexpr int LG_THREADS = 256;
constexpr int LG_CHUNK = 4096;     // tokens of the vocabulary per block
constexpr int LG_VECS = 8;         // 16-byte pieces a lane has in flight
constexpr uint32_t PROMPT_BIT = 0x80000000u;

struct LogitsParams {
  const char* in;
  char* out;
  long long in_stride, out_stride;  // bytes between rows
  int B, N, V, n_chunks, sub, words, masks, biases, text_stride;
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
  __device__ static __forceinline__ uint32_t keep2(uint32_t d, uint32_t bits) {
    const uint32_t lo = bits & 1 ? d : 0xFF80u, hi = bits & 2 ? d : 0xFF800000u;
    return (lo & 0xFFFFu) | (hi & 0xFFFF0000u);
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

// Copies tokens [t0, t1) of a row, -inf where the mask forbids; in place only what changes is written.  A piece
// that the mask forbids whole is not read.
template <int DT>
__device__ __forceinline__ void stream_row(const char* in, char* out, int t0, int t1, const uint32_t* mask, int words, int lane) {
  using E = Elem<DT>;
  constexpr int ES = 16 / E::VE;
  constexpr uint32_t ALL = (1u << E::VE) - 1;
  const bool in_place = in == out;
  if (in_place && !mask) return;
  const uint32_t off = (uint32_t)((uintptr_t)(in + (long long)t0 * ES) & 15);
  int a = t0 + (int)((16 - off) & 15) / ES;  // first token on a 16-byte boundary of the input
  if ((((uintptr_t)in ^ (uintptr_t)out) & 15) != 0 || a > t1) a = t1;
  const int n_vec = (t1 - a) / E::VE;
  const int b = a + n_vec * E::VE;
  // the ends (all of it when input and output lie differently): one element at a time
  const int n_edge = (a - t0) + (t1 - b);
  for (int i = lane; i < n_edge; i += 32) {
    const int t = i < a - t0 ? t0 + i : b + (i - (a - t0));
    const bool ok = !mask || (mask_bits(mask, words, t) & 1);
    if (ok && in_place) continue;
    if (ok) *reinterpret_cast<typename E::T*>(out + (long long)t * ES) = *reinterpret_cast<const typename E::T*>(in + (long long)t * ES);
    else E::store(out + (long long)t * ES, -INFINITY);
  }
  const char* src = in + (long long)a * ES;
  char* dst = out + (long long)a * ES;
  for (int v0 = 0; v0 < n_vec; v0 += 32 * LG_VECS) {
    uint4 d[LG_VECS];
    uint32_t bits[LG_VECS];
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32 + lane;
      bits[e] = mask && v < n_vec ? mask_bits(mask, words, a + v * E::VE) & ALL : ALL;
    }
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32 + lane;
      d[e] = make_uint4(0, 0, 0, 0);
      if (v < n_vec && bits[e] != 0 && !(in_place && bits[e] == ALL)) d[e] = *reinterpret_cast<const uint4*>(src + (size_t)v * 16);
    }
#pragma unroll
    for (int e = 0; e < LG_VECS; ++e) {
      const int v = v0 + e * 32 + lane;
      if (v < n_vec && !(in_place && bits[e] == ALL))
        *reinterpret_cast<uint4*>(dst + (size_t)v * 16) = bits[e] == ALL ? d[e] : E::keep(d[e], bits[e]);
    }
  }
}

struct Penalty {
  float r, f, p;
};

// The penalties' own arithmetic, each operation rounded by itself (no contraction), so that a row comes out the same
// whichever way its token was found.
__device__ __forceinline__ float process(float x, bool met, uint32_t count, const Penalty& q, bool has_bias, float bias) {
  if (met) x = x > 0.0f ? __fdiv_rn(x, q.r) : __fmul_rn(x, q.r);
  if (count) x = __fsub_rn(__fsub_rn(x, __fmul_rn(q.f, (float)count)), q.p);
  if (has_bias) x = __fadd_rn(x, bias);
  return x;
}

// A block takes one chunk of the vocabulary of one sequence, for all its nodes: it counts the text's tokens of that
// chunk once in shared memory and lists the distinct ones (with the biased ones), then its warps stream the nodes'
// rows through and go over the listed tokens again, 32 at a time.  Nearly all logits are only copied: the list keeps
// the per-token work (a scattered read, the arithmetic, a scattered write, all in L2) out of the stream.  HBM-bound:
// every logit is read and written once.
template <int DT>
__global__ void __launch_bounds__(LG_THREADS) logits_kernel(const __grid_constant__ LogitsParams p) {
  using E = Elem<DT>;
  constexpr int ES = 16 / E::VE;
  __shared__ uint32_t s_count[LG_CHUNK];
  __shared__ uint32_t s_bits[LG_CHUNK / 32];  // tokens that are on the list
  __shared__ unsigned short s_list[LG_CHUNK];
  __shared__ int s_n;
  extern __shared__ int s_bias[];  // [LG_CHUNK] with biases: 1 + the entry of each token
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < LG_CHUNK; i += LG_THREADS) s_count[i] = 0;
  for (int i = tid; i < LG_CHUNK / 32; i += LG_THREADS) s_bits[i] = 0;
  if (p.bias_start)
    for (int i = tid; i < LG_CHUNK; i += LG_THREADS) s_bias[i] = 0;
  if (tid == 0) s_n = 0;
  pdl_wait();
  __syncthreads();
  const int b = blockIdx.x / p.n_chunks, c0 = (blockIdx.x % p.n_chunks) * LG_CHUNK;
  const int width = p.V - c0 < LG_CHUNK ? p.V - c0 : LG_CHUNK;
  auto list = [&](uint32_t i) {
    if (!(atomicOr(&s_bits[i >> 5], 1u << (i & 31)) >> (i & 31) & 1u)) s_list[atomicAdd(&s_n, 1)] = (unsigned short)i;
  };
  if (p.text) {
    const long long have = p.n_text[b];
    const int n = have < 0 ? 0 : (have > p.text_stride ? p.text_stride : (int)have);
    const long long first = p.n_prompt ? p.n_prompt[b] : 0;
    const int* row = p.text + (long long)b * p.text_stride;
    auto count = [&](int t, int i) {
      const uint32_t at = (uint32_t)(t - c0);
      if (t < 0 || at >= (uint32_t)width) return;
      const uint32_t old = i < first ? atomicOr(&s_count[at], PROMPT_BIT) : atomicAdd(&s_count[at], 1u);
      if (old == 0) list(at);
    };
    const int head = (int)(((16 - ((uintptr_t)row & 15)) & 15) >> 2);
    const int a = head < n ? head : n;
    const int n4 = (n - a) >> 2;
    for (int i = tid; i < a; i += LG_THREADS) count(row[i], i);
    const int4* row4 = reinterpret_cast<const int4*>(row + a);
    for (int i = tid; i < n4; i += LG_THREADS) {
      const int4 t = row4[i];
      count(t.x, a + 4 * i);
      count(t.y, a + 4 * i + 1);
      count(t.z, a + 4 * i + 2);
      count(t.w, a + 4 * i + 3);
    }
    for (int i = a + 4 * n4 + tid; i < n; i += LG_THREADS) count(row[i], i);
  }
  if (p.bias_start) {
    const int from = max(p.bias_start[b], 0), to = min(p.bias_start[b + 1], p.biases);
    for (int i = from + tid; i < to; i += LG_THREADS) {
      const int t = p.bias_id[i];
      const uint32_t at = (uint32_t)(t - c0);
      if (t < 0 || at >= (uint32_t)width) continue;
      atomicMax(&s_bias[at], i + 1);
      list(at);
    }
  }
  __syncthreads();

  const int n_list = s_n;
  Penalty q;
  q.r = p.repetition ? p.repetition[b] : 1.0f;
  q.f = p.frequency ? p.frequency[b] : 0.0f;
  q.p = p.presence ? p.presence[b] : 0.0f;
  const int n_sub = (width + p.sub - 1) / p.sub;
  const int tasks = p.N * n_sub;
  for (int task = warp; task < tasks; task += LG_THREADS / 32) {
    const int u = task / n_sub, lo = (task - u * n_sub) * p.sub;
    const int hi = lo + p.sub < width ? lo + p.sub : width;
    const long long r = (long long)b * p.N + u;
    const char* in = p.in + r * p.in_stride;
    char* out = p.out + r * p.out_stride;
    const uint32_t* mask = nullptr;
    if (p.mask) {
      const int m = p.mask_row[r];
      if (m >= 0 && m < p.masks) mask = p.mask + (long long)m * p.words;
    }
    // lane i: the token of the i-th node on the way up from u, the root left out
    int mine = -1, depth = 0;
    if (p.tree) {
      int node = 0;
      for (int v = u; v > 0; v = p.parent[v], ++depth)
        if (lane == depth) node = v;
      if (lane < depth) mine = p.tree[(long long)b * p.N + node];
      if (mine < c0 || mine >= c0 + width) mine = -1;
      else mine -= c0;
      if (__ballot_sync(FULL, mine >= 0) == 0) depth = 0;
    }
    stream_row<DT>(in, out, c0 + lo, c0 + hi, mask, p.words, lane);
    __syncwarp();  // what follows writes over tokens that other lanes have copied
    auto fix = [&](int at, uint32_t on_path) {
      const int t = c0 + at;
      if (mask && !(mask_bits(mask, p.words, t) & 1)) return;
      const uint32_t w = s_count[at], c = (w & ~PROMPT_BIT) + on_path;
      const int e = p.bias_start ? s_bias[at] : 0;
      E::store(out + (long long)t * ES, process(E::load(in + (long long)t * ES), w != 0 || on_path, c, q, e != 0, e ? p.bias_value[e - 1] : 0.0f));
    };
    for (int i0 = 0; i0 < n_list; i0 += 32) {
      const int at = i0 + lane < n_list ? s_list[i0 + lane] : -1;
      uint32_t on_path = 0;
      for (int d = 0; d < depth; ++d) on_path += __shfl_sync(FULL, mine, d) == at;
      if (at >= lo && at < hi) fix(at, on_path);
    }
    if (depth) {  // tokens that only the path holds; of equal ones the first lane goes
      const uint32_t same = __match_any_sync(FULL, mine);
      if (mine >= lo && mine < hi && (__ffs(same) - 1) == lane && !(s_bits[mine >> 5] >> (mine & 31) & 1u)) fix(mine, __popc(same));
    }
    __syncwarp();
  }
}

}  // namespace

extern "C" int stand_process_logits(const stand_logits* c, const stand_logits_inputs* x, const void* dev_in, void* dev_out,
                                    void* cu_stream) {
  if (!c || !x || !dev_in || !dev_out) return STAND_E_ARG;
  if (c->B < 1 || c->N < 1 || c->N > STAND_MAX_NODES || c->V < 2 || c->V > STAND_MAX_VOCAB) return STAND_E_ARG;
  if (c->dtype != STAND_DTYPE_F32 && c->dtype != STAND_DTYPE_BF16) return STAND_E_ARG;
  if (c->in_stride < c->V || c->out_stride < c->V || c->text_stride < 0 || c->masks < 0 || c->biases < 0 || c->reserved != 0) return STAND_E_ARG;
  if (dev_in == dev_out && c->in_stride != c->out_stride) return STAND_E_ARG;
  if (!c->parent && c->N > 1) return STAND_E_ARG;
  if ((x->text != nullptr) != (x->n_text != nullptr) || (x->n_prompt && !x->text)) return STAND_E_ARG;
  if (x->bias_start && c->biases > 0 && (!x->bias_id || !x->bias_value)) return STAND_E_ARG;
  if ((x->mask != nullptr) != (x->mask_row != nullptr)) return STAND_E_ARG;
  const int es = c->dtype == STAND_DTYPE_F32 ? 4 : 2;
  if (((uintptr_t)dev_in | (uintptr_t)dev_out) % es != 0) return STAND_E_ARG;
  LogitsParams p;
  int depth[STAND_MAX_NODES];
  depth[0] = 0;
  p.parent[0] = -1;
  if (c->parent && c->parent[0] != -1) return STAND_E_ARG;
  for (int u = 1; u < c->N; ++u) {
    const int par = c->parent[u];
    if (par < 0 || par >= u) return STAND_E_ARG;
    depth[u] = depth[par] + 1;
    if (depth[u] > STAND_MAX_DEPTH) return STAND_E_ARG;  // a path has a lane per node
    p.parent[u] = (short)par;
  }
  p.in = (const char*)dev_in; p.out = (char*)dev_out; p.in_stride = c->in_stride * es; p.out_stride = c->out_stride * es;
  p.B = c->B; p.N = c->N; p.V = c->V; p.n_chunks = (c->V + LG_CHUNK - 1) / LG_CHUNK; p.words = (c->V + 31) / 32; p.masks = c->masks; p.biases = c->biases;
  p.text_stride = c->text_stride; p.text = x->text; p.n_text = (const long long*)x->n_text; p.n_prompt = (const long long*)x->n_prompt;
  p.tree = x->tree_tokens; p.repetition = x->repetition; p.frequency = x->frequency; p.presence = x->presence;
  p.bias_start = x->bias_start; p.bias_id = x->bias_id; p.bias_value = x->bias_value; p.mask = x->mask; p.mask_row = x->mask_row;
  // every warp gets some of the chunk's rows: few nodes are cut into more pieces
  p.sub = LG_CHUNK / 2;
  while (p.sub > 512 && c->N * (LG_CHUNK / p.sub) < LG_THREADS / 32) p.sub /= 2;
  const long long blocks = (long long)c->B * p.n_chunks;
  if (blocks > 0x7FFFFFFFll) return STAND_E_ARG;
  const size_t smem = x->bias_start ? LG_CHUNK * sizeof(int) : 0;
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (c->dtype == STAND_DTYPE_BF16) return launch_dependent(logits_kernel<1>, dim3((unsigned)blocks), LG_THREADS, st, p, smem);
  return launch_dependent(logits_kernel<0>, dim3((unsigned)blocks), LG_THREADS, st, p, smem);
}
