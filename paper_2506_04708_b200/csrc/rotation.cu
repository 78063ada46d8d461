// Norms of queries and keys per head with the position rotation in the same pass; rows into the paged cache with both on the way,
// in their own type or in 4 bits; rows of the cache back as values.
#include "../../include/stand.h"

#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <initializer_list>
#include <type_traits>

#include "launch.cuh"
#include "overlap.cuh"
#include "packed.cuh"
#include "rotation.cuh"

using namespace stand;

namespace {

constexpr int ROT_THREADS = 256;
constexpr int ROT_E = 16;  // elements of a lane that reads
constexpr int ROW_COUNT = 4096;  // layers, heads: their product counts rows in 32 bits
constexpr int ROT_TOKENS = 16;  // tokens of a block, at most: their cosines and sines lie in shared memory

// The block's table of cosines and sines; the caller's barrier follows.
template <int VE, typename F> __device__ __forceinline__ void turn_tables(const Turn& t, float* cs, int tokens, F position) {
  const int floats = turn_floats<VE>(t.columns), angles = t.columns * VE;
  for (int i = threadIdx.x; i < tokens * angles; i += ROT_THREADS) {
    const int tok = i / angles, k = i - tok * angles;
    float c = 1.0f, s = 0.0f;
    if (k < t.half) turn_angle(position(tok), t.freq[k], c, s);
    float* at = cs + tok * 2 * floats + turn_at<VE>(t.columns, k);
    at[0] = c;
    at[floats] = s;
  }
}

struct RotateParams {
  Turn t;
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  const void* weight_q;
  const void* weight_k;
  int B, N, heads_q, heads;  // heads: of queries and keys together
  int tokens;                // of a block
  int heads_block;           // heads of a block (grid.y blocks share a token's heads)
  bool narrow;               // offsets fit 31 bits, those of a block's steps past the end too
  long long q_in[3], k_in[3], q_to[3], k_to[3];
};

// A block: some tokens' heads.  Its cosines and sines and the weights lie in shared memory; a row belongs to a group of lanes, each with whole pairs
// (two vectors of VE elements that are turned with one another), so that nothing is read or worked out twice and the mean square takes a few shuffles.
// Every element is read and written once, which is the bound for large calls.  16,384 tokens of 32 + 8 heads of 128 in bfloat16, with norm: 74 us = 4.5 TB/s
// (0.69 of the copy bandwidth); the same loop without norm and turn takes 59 us, the rest is issue (61 - 73 % of its slots).  The next row's loads
// ahead of this one's work: 96 us, for the registers.  One token: 2.9 us, a launch.
// I: the type of offsets; 32 bits where they fit, for they are most of the arithmetic.
template <typename T, int VE, typename I> __global__ void __launch_bounds__(ROT_THREADS, 4) rotate_heads_kernel(const __grid_constant__ RotateParams p) {
  extern __shared__ __align__(16) float rot_cs[];
  __shared__ __align__(16) float s_weight[2][ROT_DIM_MAX];  // lanes * units * elements: a power of two, at most 256
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lanes = p.t.lanes, c = tid & (lanes - 1), group = tid / lanes, groups = ROT_THREADS / lanes;
  const int first = blockIdx.x * p.tokens, tokens = p.B * p.N - first < p.tokens ? p.B * p.N - first : p.tokens;
  const int floats = 2 * turn_floats<VE>(p.t.columns);
  const int tok_b = first / p.N, tok_n = first - tok_b * p.N;  // of the block's first token
  if (p.t.freq) {
    turn_tables<VE>(p.t, rot_cs, tokens, [&](int tok) {
      int b = tok_b, n = tok_n + tok;
      while (n >= p.N) n -= p.N, ++b;
      return turn_position(p.t, b, n);
    });
  }
  // Weights in the order of the lanes: element e of lane l's unit k at (k * 2 VE + e) * lanes + l, four elements of a lane together (VE = 1: two apart),
  // so that a row's lanes read without conflict.
  constexpr int K = RowLane<T, VE>::K, Q = VE < 4 ? 1 : 4;
  if (p.weight_q || p.weight_k)
    for (int i = tid; i < lanes * 2 * VE * K; i += ROT_THREADS) {
      const int l = i / Q % lanes, e = i / (Q * lanes) * Q + i % Q, k = e / (2 * VE), in_unit = e % (2 * VE);
      const RowLane<T, VE> at(p.t, l, p.t.freq != nullptr);
      int from = 0;
#pragma unroll
      for (int kk = 0; kk < K; ++kk)
        if (kk == k) from = in_unit < VE ? at.a[kk] + in_unit : at.b[kk] + in_unit - VE;
      if (p.weight_q) s_weight[0][i] = to_float(reinterpret_cast<const T*>(p.weight_q)[from]);
      if (p.weight_k) s_weight[1][i] = to_float(reinterpret_cast<const T*>(p.weight_k)[from]);
    }
  __syncthreads();
  const bool norm = p.t.norm;
  // some heads of all of the block's tokens; queries and keys one after the other, so that strides and weights are the same for all lanes
  auto kind = [&](const void* src, void* dst, const long long (&in_s)[3], const long long (&out_s)[3], const float* weight, int head0, int heads) {
    if (heads <= 0) return;
    RowLane<T, VE> lane(p.t, c, p.t.freq != nullptr);
    const int rows = tokens * heads, step_h = groups % heads, step_t = groups / heads;
    int h = group % heads, tok = group / heads, n = tok_n + tok;
    const I in0 = (I)in_s[0], in1 = (I)in_s[1], in2 = (I)in_s[2], out0 = (I)out_s[0], out1 = (I)out_s[1], out2 = (I)out_s[2];
    const T* const from = reinterpret_cast<const T*>(src) + tok_b * in0 + tok_n * in1 + head0 * in2;
    T* const to = reinterpret_cast<T*>(dst) + tok_b * out0 + tok_n * out1 + head0 * out2;
    I in_at = h * in2 + tok * in1, out_at = h * out2 + tok * out1;
    // a step further, and what is put right where the heads of a token or the tokens of a sequence end
    const I in_step = step_h * in2 + step_t * in1, in_head = in1 - heads * in2, in_seq = in0 - p.N * in1;
    const I out_step = step_h * out2 + step_t * out1, out_head = out1 - heads * out2, out_seq = out0 - p.N * out1;
    auto weights = [&](float (&w)[2 * VE], int k) {
#pragma unroll
      for (int e = 0; e < 2 * VE; e += Q) {
        const float* at = weight + ((k * 2 * VE + e) * lanes + c * Q);
        if constexpr (Q == 4) *reinterpret_cast<float4*>(w + e) = *reinterpret_cast<const float4*>(at);
        else w[e] = *at;
      }
    };
    for (int r = group; r - group < rows; r += groups) {
      while (n >= p.N) n -= p.N, in_at += in_seq, out_at += out_seq;
      const bool in = r < rows;
      T* const out = to + out_at;
      typename RowLane<T, VE>::Raw raw;
      lane.read(from + (in ? in_at : 0), raw);
      lane.row(p.t, raw, weight != nullptr, weights, rot_cs + (in ? tok * floats : 0), in, norm, [&](float (&y)[2 * VE], int a, int b, bool two) {
        store_vec<T, VE>(out + a, y);
        if (two) store_vec<T, VE>(out + b, y + VE);
      });
      h += step_h, tok += step_t, n += step_t, in_at += in_step, out_at += out_step;
      if (h >= heads) h -= heads, ++tok, ++n, in_at += in_head, out_at += out_head;
    }
  };
  const int h0 = blockIdx.y * p.heads_block, h1 = h0 + p.heads_block < p.heads ? h0 + p.heads_block : p.heads;
  kind(p.q, p.q_out, p.q_in, p.q_to, p.weight_q ? s_weight[0] : nullptr, h0, (h1 < p.heads_q ? h1 : p.heads_q) - h0);
  const int k0 = h0 > p.heads_q ? h0 : p.heads_q;
  kind(p.k, p.k_out, p.k_in, p.k_to, p.weight_k ? s_weight[1] : nullptr, k0 - p.heads_q, h1 - k0);
}

struct AppendParams {
  Turn t;
  const void* k;
  const void* v;
  const void* weight;
  const int* path;
  const long long* slots;
  char* cache_k;
  char* cache_v;
  int layers, N, width, heads, page;
  long long places;  // B * width
  int tokens, layers_block;
  int table_floats;  // of all tokens; a block's rows on their way to groups of 16 lie behind them
  long long n_slots;
  long long k_in[4], v_in[4];  // elements
  long long to[4];             // bytes: layer, page, head, token
};

// As above, with a token's place in the cache and angles worked out once for all layers of a block.  1,100 tokens of three prompts in 32 layers, 8 heads of
// 128 in bfloat16, norm and turn, to 4 bits: 54 us (floor 27), to a cache of their own type 54 us (floor 43); layer after layer in blocks of their own
// it took 81 and 65.  In 4 bits the kernel is bound by issue (69 % of its slots, logic unit 48 %): the maximum of 16, a scale, 16 codes and their
// place in two words cost about as much again as norm and turn.
// Packed: a lane takes a group of 16 elements.  Where units are such groups they stay in registers; else (halves that are turned, short units) the
// row goes through shared memory, as what a cache of its type would hold.
template <typename T, int VE, bool PACKED>
__global__ void __launch_bounds__(ROT_THREADS, sizeof(T) == 2 ? 4 : 3) kv_append_kernel(const __grid_constant__ AppendParams p) {
  extern __shared__ __align__(16) float rot_cs[];
  // of a token: where its rows come from (elements) and go to (bytes; -1: nothing is stored) in the first layer and head; its scales
  __shared__ long long s_from[2][ROT_TOKENS], s_to[ROT_TOKENS], s_at[ROT_TOKENS];
  __shared__ int s_scale[ROT_TOKENS];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, lanes = p.t.lanes, c = tid & (lanes - 1), group = tid / lanes, groups = ROT_THREADS / lanes;
  const bool keys = blockIdx.z == 0;
  const long long first = (long long)blockIdx.x * p.tokens;
  const int tokens = p.places - first < p.tokens ? (int)(p.places - first) : p.tokens;
  const int l0 = blockIdx.y * p.layers_block, layers = p.layers - l0 < p.layers_block ? p.layers - l0 : p.layers_block;
  const int floats = 2 * turn_floats<VE>(p.t.columns), dim = p.t.dim;
  if (tid < tokens) {
    const int place = (int)first + tid;  // below 2^31
    const long long slot = p.slots[place];
    const int b = place / p.width, j = place - b * p.width, node = p.path ? p.path[place] : j;
    const long long page = slot >= 0 && slot < p.n_slots && node >= 0 && node < p.N ? slot / p.page : -1;
    const int token = (int)(slot - page * p.page);
    s_from[0][tid] = b * p.k_in[1] + node * p.k_in[2];
    s_from[1][tid] = b * p.v_in[1] + node * p.v_in[2];
    s_to[tid] = page < 0 ? -1 : page * p.to[1] + (PACKED ? token * (dim / 2) : token * p.to[3]);
    s_scale[tid] = p.page * (dim / 2) + token * (dim / 16) - token * (dim / 2);
    s_at[tid] = page < 0 ? 0 : turn_position(p.t, b, node);
  }
  __syncthreads();
  if (keys && p.t.freq) {
    turn_tables<VE>(p.t, rot_cs, tokens, [&](int tok) { return s_at[tok]; });
    __syncthreads();
  }
  T* const mine = reinterpret_cast<T*>(rot_cs + p.table_floats) + group * dim;
  // Keys and values have blocks of their own: strides and what is done are the same for all lanes.  A group of lanes has one token's head in all of the block's layers, the
  // next layer's row on its way while one is worked on.
  auto kind = [&](const void* src, const long long (&in_s)[4], const long long* from, char* cache, auto are_keys) {
    constexpr bool KEYS = decltype(are_keys)::value;
    const bool turn = KEYS && p.t.freq, norm = KEYS && p.t.norm;
    RowLane<T, VE> lane(p.t, c, turn);
    // packed rows that stay as they are go straight to their groups, and so do units that are groups
    const bool same = PACKED && VE == 8 && !turn && !norm, direct = VE == 8 && !(turn && !p.t.pairs);
    const int rows = tokens * p.heads;
    for (int r = group; r - group < rows; r += groups) {
      const int tok = r < rows ? r / p.heads : 0, h = r < rows ? r - tok * p.heads : 0;
      const long long base = s_to[tok];
      const bool in = r < rows && base >= 0;
      if (!__any_sync(FULL, in)) continue;
      const T* row = reinterpret_cast<const T*>(src) + (in ? from[tok] + l0 * in_s[0] + h * in_s[3] : 0);
      const long long to_next_row = in ? in_s[0] : 0;
      char* to = cache + base + l0 * p.to[0] + h * p.to[2];
      const T* weight = reinterpret_cast<const T*>(p.weight) + (long long)l0 * dim;
      const float* cs = rot_cs + tok * floats;
      const int scale_at = s_scale[tok] + c;
      typename RowLane<T, VE>::Raw now, next;
      lane.read(row, now);
      for (int l = 0; l < layers; ++l) {
        row += to_next_row;
        if (l + 1 < layers) lane.read(row, next);
        auto weights = [&](float (&w)[2 * VE], int k) {
          load_vec<T, VE>(weight + lane.a[k], w);
          load_vec<T, VE>(weight + lane.b[k], w + VE);
        };
        if constexpr (!PACKED) {
          T* out = reinterpret_cast<T*>(to);
          lane.row(p.t, now, p.weight != nullptr, weights, cs, in, norm, [&](float (&y)[2 * VE], int a, int b, bool two) {
            store_vec<T, VE>(out + a, y);
            if (two) store_vec<T, VE>(out + b, y + VE);
          });
        } else {
          const bool has = in && c * PK_GROUP < dim;
          PkGroup<T> z;
          if (same) {
#pragma unroll
            for (int i = 0; i < PkGroup<T>::WORDS; ++i) z.w[i] = reinterpret_cast<const uint32_t*>(now.e[0])[VE == 8 ? i : 0];
          } else {
            lane.row(p.t, now, p.weight != nullptr, weights, cs, in, norm, [&](float (&y)[2 * VE], int a, int b, bool two) {
              if (direct) {
                if constexpr (VE == 8) store_vec<T, 16>(reinterpret_cast<T*>(z.w), y);
              } else {
                store_vec<T, VE>(mine + a, y);
                if (two) store_vec<T, VE>(mine + b, y + VE);
              }
            });
            __syncwarp();
            if (!direct && has) copy_vec<T, 16>(reinterpret_cast<T*>(z.w), mine + c * PK_GROUP);
            __syncwarp();  // the row in shared memory has been read
          }
          if (has) {
            uint32_t byte;
            *reinterpret_cast<uint2*>(to + c * 8) = z.codes(byte);
            to[scale_at] = (char)byte;
          }
        }
        to += p.to[0];
        weight += dim;
        now = next;
      }
    }
  };
  if (keys) kind(p.k, p.k_in, s_from[0], p.cache_k, std::true_type{});
  else kind(p.v, p.v_in, s_from[1], p.cache_v, std::false_type{});
}

struct ReadParams {
  const char* cache_k;
  const char* cache_v;
  const long long* slots;
  void* k_out;
  void* v_out;
  int layers, heads, dim, page, lanes;
  long long places, n_slots;
  int layers_block;
  long long from[4];  // bytes: layer, page, head, token
};

// 32 bytes, a sector of memory, in one access; aligned to as many.
__device__ __forceinline__ void store_32(void* to, const uint4& a, const uint4& b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z),
               "r"(b.w)
               : "memory");
}

// A lane: 16 elements of a row, one token's head in all of the block's layers.  Places without a slot give zeros.  Bound by the bytes written: 3 x 509
// places in 32 layers, 8 heads of 128, from 4 bits to bfloat16 (200 MB out, 40 MB in): 45 us = 5.4 TB/s.  Lanes store 32 bytes at a time; in two times
// 16, each of which touches half of a sector, it took 55.
// WIDE: accesses of 16 bytes; 2: results at multiples of 32.
template <typename T, int WIDE, bool PACKED>
__global__ void __launch_bounds__(ROT_THREADS) kv_read_kernel(const __grid_constant__ ReadParams p) {
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, c = tid & (p.lanes - 1), group = tid / p.lanes, groups = ROT_THREADS / p.lanes;
  if (c * ROT_E >= p.dim) return;
  const int l0 = blockIdx.y * p.layers_block, layers = p.layers - l0 < p.layers_block ? p.layers - l0 : p.layers_block;
  const long long r = (long long)blockIdx.x * groups + group, place = r / (2 * p.heads);
  if (place >= p.places) return;
  const bool is_v = r - place * 2 * p.heads >= p.heads;
  const int h = (int)(r - place * 2 * p.heads) - (is_v ? p.heads : 0);
  const long long slot = p.slots[place], page = slot >= 0 && slot < p.n_slots ? slot / p.page : -1;
  const int token = (int)(slot - page * p.page);
  T* out = reinterpret_cast<T*>(is_v ? p.v_out : p.k_out) + ((l0 * p.places + place) * p.heads + h) * p.dim + c * ROT_E;
  const long long out_next = p.places * p.heads * p.dim;
  const char* from = (is_v ? p.cache_v : p.cache_k) + l0 * p.from[0] + (page < 0 ? 0 : page * p.from[1]) + h * p.from[2];
  const int at = PACKED ? token * (p.dim / 2) + c * 8 : 0, scale_at = PACKED ? p.page * (p.dim / 2) + token * (p.dim / 16) + c : 0;
  const long long row_at = PACKED ? 0 : token * p.from[3] + c * ROT_E * (long long)sizeof(T);
#pragma unroll 4
  for (int l = 0; l < layers; ++l, out += out_next, from += p.from[0]) {
    if constexpr (PACKED && WIDE && sizeof(T) == 2) {
      constexpr bool BF16 = std::is_same<T, __nv_bfloat16>::value;
      uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
      if (page >= 0) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(from + at));
        const PkScale<BF16> s(__ldg(reinterpret_cast<const unsigned char*>(from + scale_at)));
        v[0] = pk_word(w.x, s), v[1] = pk_word(w.y, s);
      }
      if constexpr (WIDE == 2) {
        store_32(out, v[0], v[1]);
      } else {
        reinterpret_cast<uint4*>(out)[0] = v[0];
        reinterpret_cast<uint4*>(out)[1] = v[1];
      }
      continue;
    }
    float y[ROT_E] = {};
    if (page >= 0) {
      if constexpr (PACKED) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(from + at));
        const float s = pk_scale(__ldg(reinterpret_cast<const unsigned char*>(from + scale_at)));
        pk_values(w.x, s, y);
        pk_values(w.y, s, y + 8);
      } else {
        const T* row = reinterpret_cast<const T*>(from + row_at);
        if (WIDE) {
          load_vec<T, 16>(row, y);
        } else {
#pragma unroll
          for (int i = 0; i < ROT_E; ++i)
            if (c * ROT_E + i < p.dim) y[i] = to_float(row[i]);
        }
      }
    }
    if (WIDE) {
      store_vec<T, 16>(out, y);
    } else {
#pragma unroll
      for (int i = 0; i < ROT_E; ++i)
        if (c * ROT_E + i < p.dim) out[i] = from_float<T>(y[i]);
    }
  }
}

// ---- host ------------------------------------------------------------------------------------
// The bits of an address and its strides: what accesses have to be aligned to goes by the lowest.
uintptr_t bits_of(const void* p, const long long* strides, int n, int es) {
  uintptr_t bits = (uintptr_t)p;
  for (int i = 0; i < n; ++i) bits |= (uintptr_t)(strides[i] * es);
  return bits;
}
// Elements of a unit's vectors: 8 or 4 where rows allow (accesses of 16 bytes; 8 bytes for 4 short elements), else 1.
int unit_width(const Turn& t, uintptr_t bits, int es) {
  if (turn_fits(t, 8) && (bits & 15) == 0) return 8;
  return turn_fits(t, 4) && (bits & (4 * es - 1)) == 0 ? 4 : 1;
}
int row_lanes(int dim) {  // of 16 elements
  int n = 1;
  while (n * ROT_E < dim) n *= 2;
  return n;
}

int element_size(int dtype) { return dtype == STAND_DTYPE_F32 ? 4 : 2; }
bool type_valid(int dtype) { return dtype >= STAND_DTYPE_F32 && dtype <= STAND_DTYPE_F16; }

// Tokens of a block: as many as make work for its threads (each group of lanes some rows), but no fewer blocks than fill the GPU.
int tokens_per_block(long long places, int rows_of_token, int lanes) {
  const int groups = ROT_THREADS / lanes;
  int tokens = 1;
  while (tokens < ROT_TOKENS && tokens * rows_of_token < 8 * groups && places / (2 * tokens) >= 2 * 148) tokens *= 2;
  return tokens;
}

template <typename T, int VE> int launch_rotate(RotateParams& p, cudaStream_t st) {
  turn_units(p.t, VE);
  const long long places = (long long)p.B * p.N;
  p.tokens = tokens_per_block(places, p.heads, p.t.lanes);
  // few tokens: their heads are shared out over blocks of a row per group of lanes
  p.heads_block = p.heads;
  const int groups = ROT_THREADS / p.t.lanes;
  if (places * ((p.heads + groups - 1) / groups) <= 4 * 148) p.heads_block = groups < p.heads ? groups : p.heads;
  const long long blocks = (places + p.tokens - 1) / p.tokens;
  const dim3 grid((unsigned)blocks, (unsigned)((p.heads + p.heads_block - 1) / p.heads_block));
  const size_t smem = (size_t)p.tokens * 2 * turn_floats<VE>(p.t.columns) * sizeof(float);
  if (p.narrow) return launch_dependent(rotate_heads_kernel<T, VE, int>, grid, ROT_THREADS, st, p, smem);
  return launch_dependent(rotate_heads_kernel<T, VE, long long>, grid, ROT_THREADS, st, p, smem);
}
template <typename T> int launch_rotate(RotateParams& p, int ve, cudaStream_t st) {
  return ve == 8 ? launch_rotate<T, 8>(p, st) : (ve == 4 ? launch_rotate<T, 4>(p, st) : launch_rotate<T, 1>(p, st));
}

template <typename T, int VE> int launch_append(AppendParams& p, bool packed, cudaStream_t st) {
  turn_units(p.t, VE);
  // Tokens enough that each group of lanes has a row (16 at most), and as many layers as leave enough blocks to fill the GPU: a token's angles are
  // worked out once for all layers of a block.  With 2, 4, 8 (times 148 blocks each of keys and values): prompts of 32 layers 72, 55, 58 us, accepted paths of
  // 28 layers 9.2, 9.5, 13.6; keys and values one after the other in one block at best 67 and 10.4.
  const int groups = ROT_THREADS / p.t.lanes;
  p.tokens = groups / p.heads < 1 ? 1 : (groups / p.heads > ROT_TOKENS ? ROT_TOKENS : groups / p.heads);
  while (p.tokens > 1 && p.places <= p.tokens / 2) p.tokens /= 2;
  const long long across = (p.places + p.tokens - 1) / p.tokens;
  int lpb = p.layers;
  while (lpb > 1 && across * ((p.layers + lpb - 1) / lpb) < 4 * 148) lpb = (lpb + 1) / 2;
  p.layers_block = lpb;
  const dim3 grid((unsigned)across, (unsigned)((p.layers + lpb - 1) / lpb), 2);
  p.table_floats = p.tokens * 2 * turn_floats<VE>(p.t.columns);
  const size_t smem = p.table_floats * sizeof(float) + (packed ? (size_t)groups * p.t.dim * sizeof(T) : 0);
  if (packed) return launch_dependent(kv_append_kernel<T, VE, true>, grid, ROT_THREADS, st, p, smem);
  return launch_dependent(kv_append_kernel<T, VE, false>, grid, ROT_THREADS, st, p, smem);
}
template <typename T> int launch_append(AppendParams& p, int ve, bool packed, cudaStream_t st) {
  return ve == 8 ? launch_append<T, 8>(p, packed, st) : (ve == 4 ? launch_append<T, 4>(p, packed, st) : launch_append<T, 1>(p, packed, st));
}
template <typename T> int launch_read(const ReadParams& p, int wide, bool packed, dim3 grid, cudaStream_t st) {
  if (packed) {
    if constexpr (sizeof(T) == 2)
      if (wide == 2) return launch_dependent(kv_read_kernel<T, 2, true>, grid, ROT_THREADS, st, p);
    if (wide) return launch_dependent(kv_read_kernel<T, 1, true>, grid, ROT_THREADS, st, p);
    return launch_dependent(kv_read_kernel<T, 0, true>, grid, ROT_THREADS, st, p);
  }
  if (wide) return launch_dependent(kv_read_kernel<T, 1, false>, grid, ROT_THREADS, st, p);
  return launch_dependent(kv_read_kernel<T, 0, false>, grid, ROT_THREADS, st, p);
}

// What both entry points that turn rows check and derive alike.
bool make_turn(Turn& t, int dim, int rotary, int interleaved, int norm, float eps, const float* freq, const int64_t* base, const int32_t* offset,
               int64_t offset_stride) {
  if (dim < 1 || dim > ROT_DIM_MAX || rotary < 0 || rotary > dim || rotary % 2 != 0 || (rotary > 0) != (freq != nullptr)) return false;
  if ((interleaved != 0 && interleaved != 1) || (norm != 0 && norm != 1) || offset_stride < 0) return false;
  if (norm && !(eps > 0.0f && eps < INFINITY)) return false;
  if (!aligned(4, freq, offset) || !aligned(8, base)) return false;
  t.freq = freq; t.base = (const long long*)base; t.offset = offset; t.offset_stride = offset_stride;
  t.half = rotary / 2; t.pairs = interleaved; t.norm = norm; t.eps = eps; t.inv_dim = 1.0f / (float)dim;
  t.dim = dim;
  return true;
}

RowSet heads_of(const void* p, int B, int N, int heads, const long long (&stride)[3], int dim, int es) {
  return {p, (int64_t)dim * es, 3, {B, N, heads, 1}, {stride[0] * es, stride[1] * es, stride[2] * es, 0}};
}
RowSet rows_of(const void* p, int layers, int B, int N, int heads, const long long (&stride)[4], int dim, int es) {
  return {p, (int64_t)dim * es, 4, {layers, B, N, heads}, {stride[0] * es, stride[1] * es, stride[2] * es, stride[3] * es}};
}
// (strides in bytes; a packed cache's rows are its blocks)
RowSet cache_of(const stand_kv_rows* c, const void* p, const long long (&stride)[4], int es) {
  const int64_t bytes = c->packed ? (int64_t)STAND_PACKED_BLOCK_BYTES(c->page_size, c->dim) : (int64_t)c->dim * es;
  return {p, bytes, 4, {c->layers, c->pages, c->heads, c->packed ? 1 : c->page_size}, {stride[0], stride[1], stride[2], stride[3]}};
}
// Rows to write that lie over one another by a stride of 0 (where there are any rows).
bool stacked(const RowSet& r) {
  bool any = true, zero = false;
  for (int i = 0; i < r.dims; ++i) any = any && r.count[i] > 0, zero = zero || (r.stride[i] == 0 && r.count[i] > 1);
  return any && zero;
}

bool packed_strides(const void* a, const void* b, const int64_t (&stride)[4]) {
  if (stride[3] != 0) return false;
  return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)stride[0] | (uintptr_t)stride[1] | (uintptr_t)stride[2]) & 15) == 0;
}

}  // namespace

extern "C" {

int stand_rotate_heads(const stand_rotation* c, const void* dev_q, const void* dev_k, const void* dev_weight_q, const void* dev_weight_k,
                       const float* dev_freq, const int64_t* dev_base, const int32_t* dev_offset, void* dev_q_out, void* dev_k_out,
                       void* cu_stream) {
  if (!c || !dev_q || !dev_k || !dev_q_out || !dev_k_out || c->B < 1 || c->N < 1 || c->heads_q < 1 || c->heads_kv < 1) return STAND_E_ARG;
  if (!type_valid(c->dtype) || (c->reserved | c->reserved2) != 0 || c->heads_q > (1 << 16) || c->heads_kv > (1 << 16)) return STAND_E_ARG;
  if ((long long)c->B * c->N > 0x7FFFFFFFll) return STAND_E_ARG;
  RotateParams p;
  if (!make_turn(p.t, c->dim, c->rotary_dim, c->interleaved, c->norm, c->eps, dev_freq, dev_base, dev_offset, c->offset_stride)) return STAND_E_ARG;
  if (!c->norm && (dev_weight_q || dev_weight_k)) return STAND_E_ARG;
  const int es = element_size(c->dtype);
  if (!aligned(es, dev_q, dev_k, dev_q_out, dev_k_out, dev_weight_q, dev_weight_k)) return STAND_E_ARG;
  for (int i = 0; i < 3; ++i) {
    p.q_in[i] = c->q_stride[i], p.k_in[i] = c->k_stride[i], p.q_to[i] = c->q_out_stride[i], p.k_to[i] = c->k_out_stride[i];
    if (p.q_in[i] < 0 || p.k_in[i] < 0 || p.q_to[i] < 0 || p.k_to[i] < 0) return STAND_E_ARG;
  }
  const RowSet q = heads_of(dev_q, c->B, c->N, c->heads_q, p.q_in, c->dim, es), k = heads_of(dev_k, c->B, c->N, c->heads_kv, p.k_in, c->dim, es);
  const RowSet qo = heads_of(dev_q_out, c->B, c->N, c->heads_q, p.q_to, c->dim, es), ko = heads_of(dev_k_out, c->B, c->N, c->heads_kv, p.k_to, c->dim, es);
  if (stacked(qo) || stacked(ko) || (rows_meet(qo, q) && !same_rows(qo, q)) || (rows_meet(ko, k) && !same_rows(ko, k)) || rows_meet(qo, k) || rows_meet(ko, q))
    return STAND_E_ARG;
  // the same rows twice, to the same place: each is written twice alike
  if (rows_meet(qo, ko) && !(same_rows(qo, ko) && same_rows(q, k) && dev_weight_q == dev_weight_k)) return STAND_E_ARG;
  p.q = dev_q; p.k = dev_k; p.q_out = dev_q_out; p.k_out = dev_k_out; p.weight_q = dev_weight_q; p.weight_k = dev_weight_k;
  p.B = c->B; p.N = c->N; p.heads_q = c->heads_q; p.heads = c->heads_q + c->heads_kv;
  // (a step past the last row is at most 256 rows, of heads or tokens, further)
  auto reach = [&](const long long (&s3)[3], int heads) { return (long double)(p.B + 1) * s3[0] + (long double)(p.N + 256) * s3[1] + (long double)(heads + 256) * s3[2] + c->dim; };
  p.narrow = reach(p.q_in, c->heads_q) < 2147483647.0L && reach(p.k_in, c->heads_kv) < 2147483647.0L && reach(p.q_to, c->heads_q) < 2147483647.0L &&
             reach(p.k_to, c->heads_kv) < 2147483647.0L;
  const int ve = unit_width(p.t, bits_of(dev_q, p.q_in, 3, es) | bits_of(dev_k, p.k_in, 3, es) | bits_of(dev_q_out, p.q_to, 3, es) | bits_of(dev_k_out, p.k_to, 3, es), es);
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (c->dtype == STAND_DTYPE_F32) return launch_rotate<float>(p, ve, st);
  if (c->dtype == STAND_DTYPE_BF16) return launch_rotate<__nv_bfloat16>(p, ve, st);
  return launch_rotate<__half>(p, ve, st);
}

int stand_kv_append(const stand_kv_rows* c, const void* dev_k, const void* dev_v, const void* dev_weight_k, const float* dev_freq,
                    const int64_t* dev_base, const int32_t* dev_offset, const int32_t* dev_path, const int64_t* dev_slots, void* dev_cache_k,
                    void* dev_cache_v, void* cu_stream) {
  if (!c || !dev_k || !dev_v || !dev_slots || (c->pages != 0 && (!dev_cache_k || !dev_cache_v))) return STAND_E_ARG;
  if (c->layers < 1 || c->layers > ROW_COUNT || c->B < 1 || c->N < 1 || c->heads < 1 || c->heads > ROW_COUNT || c->width < 1) return STAND_E_ARG;
  if (c->page_size < 1 || c->page_size > 4096 || c->pages < 0 || !type_valid(c->dtype) || (c->packed != 0 && c->packed != 1) || (c->reserved | c->reserved2) != 0) return STAND_E_ARG;
  if ((long long)c->B * c->width > 0x7FFFFFFFll) return STAND_E_ARG;
  AppendParams p;
  if (!make_turn(p.t, c->dim, c->rotary_dim, c->interleaved, c->norm, c->eps, dev_freq, dev_base, dev_offset, c->offset_stride)) return STAND_E_ARG;
  if (!c->norm && dev_weight_k) return STAND_E_ARG;
  const int es = element_size(c->dtype);
  if (!aligned(es, dev_k, dev_v, dev_weight_k) || !aligned(8, dev_slots) || !aligned(4, dev_path)) return STAND_E_ARG;
  if (c->packed ? c->dim % PK_GROUP != 0 || c->page_size % 16 != 0 || !packed_strides(dev_cache_k, dev_cache_v, c->cache_stride)
                : !aligned(es, dev_cache_k, dev_cache_v))
    return STAND_E_ARG;
  for (int i = 0; i < 4; ++i) {
    p.k_in[i] = c->k_stride[i], p.v_in[i] = c->v_stride[i], p.to[i] = c->cache_stride[i] * (c->packed ? 1 : es);
    if (p.k_in[i] < 0 || p.v_in[i] < 0 || p.to[i] < 0) return STAND_E_ARG;
  }
  const RowSet ck = cache_of(c, dev_cache_k, p.to, es), cv = cache_of(c, dev_cache_v, p.to, es);
  for (const RowSet& from : {rows_of(dev_k, c->layers, c->B, c->N, c->heads, p.k_in, c->dim, es), rows_of(dev_v, c->layers, c->B, c->N, c->heads, p.v_in, c->dim, es)})
    if (rows_meet(from, ck) || rows_meet(from, cv)) return STAND_E_ARG;
  if (stacked(ck)) return STAND_E_ARG;
  p.k = dev_k; p.v = dev_v; p.weight = dev_weight_k; p.path = dev_path; p.slots = (const long long*)dev_slots;
  p.cache_k = (char*)dev_cache_k; p.cache_v = (char*)dev_cache_v;
  p.layers = c->layers; p.N = c->N; p.width = c->width; p.heads = c->heads; p.page = c->page_size; p.places = (long long)c->B * c->width;
  p.n_slots = (long long)c->pages * c->page_size;
  uintptr_t bits = bits_of(dev_k, p.k_in, 4, es) | bits_of(dev_v, p.v_in, 4, es) | (uintptr_t)dev_weight_k;
  if (!c->packed) bits |= bits_of(dev_cache_k, p.to, 4, 1) | bits_of(dev_cache_v, p.to, 4, 1);
  const int ve = unit_width(p.t, bits, es);
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (c->dtype == STAND_DTYPE_F32) return launch_append<float>(p, ve, c->packed, st);
  if (c->dtype == STAND_DTYPE_BF16) return launch_append<__nv_bfloat16>(p, ve, c->packed, st);
  return launch_append<__half>(p, ve, c->packed, st);
}

int stand_kv_read(const stand_kv_rows* c, const void* dev_cache_k, const void* dev_cache_v, const int64_t* dev_slots, void* dev_k, void* dev_v,
                  void* cu_stream) {
  if (!c || !dev_k || !dev_v || !dev_slots || (c->pages != 0 && (!dev_cache_k || !dev_cache_v))) return STAND_E_ARG;
  if (c->layers < 1 || c->layers > ROW_COUNT || c->B < 1 || c->heads < 1 || c->heads > ROW_COUNT || c->width < 1 || c->dim < 1 || c->dim > ROT_DIM_MAX) return STAND_E_ARG;
  if (c->page_size < 1 || c->page_size > 4096 || c->pages < 0 || !type_valid(c->dtype) || (c->packed != 0 && c->packed != 1) || (c->reserved | c->reserved2) != 0) return STAND_E_ARG;
  if (c->rotary_dim != 0 || c->norm != 0 || (long long)c->B * c->width > 0x7FFFFFFFll) return STAND_E_ARG;
  const int es = element_size(c->dtype);
  if (!aligned(es, dev_k, dev_v) || !aligned(8, dev_slots)) return STAND_E_ARG;
  if (c->packed ? c->dim % PK_GROUP != 0 || c->page_size % 16 != 0 || !packed_strides(dev_cache_k, dev_cache_v, c->cache_stride)
                : !aligned(es, dev_cache_k, dev_cache_v))
    return STAND_E_ARG;
  ReadParams p;
  for (int i = 0; i < 4; ++i) {
    p.from[i] = c->cache_stride[i] * (c->packed ? 1 : es);
    if (p.from[i] < 0) return STAND_E_ARG;
  }
  const RowSet ck = cache_of(c, dev_cache_k, p.from, es), cv = cache_of(c, dev_cache_v, p.from, es);
  const int64_t all = (int64_t)c->layers * c->B * c->width * c->heads * c->dim * es;
  const RowSet k = {dev_k, all, 0, {}, {}}, v = {dev_v, all, 0, {}, {}};
  if (rows_meet(k, ck) || rows_meet(k, cv) || rows_meet(v, ck) || rows_meet(v, cv)) return STAND_E_ARG;
  if (rows_meet(k, v) && !(dev_k == dev_v && same_rows(ck, cv))) return STAND_E_ARG;
  p.cache_k = (const char*)dev_cache_k; p.cache_v = (const char*)dev_cache_v; p.slots = (const long long*)dev_slots; p.k_out = dev_k; p.v_out = dev_v;
  p.layers = c->layers; p.heads = c->heads; p.dim = c->dim; p.page = c->page_size; p.lanes = row_lanes(c->dim);
  p.places = (long long)c->B * c->width; p.n_slots = (long long)c->pages * c->page_size;
  const bool wide = p.dim % ROT_E == 0 && (((uintptr_t)dev_k | (uintptr_t)dev_v) & 15) == 0 &&
                    (c->packed || ((bits_of(dev_cache_k, p.from, 4, 1) | bits_of(dev_cache_v, p.from, 4, 1)) & 15) == 0);
  const int width = !wide ? 0 : ((((uintptr_t)dev_k | (uintptr_t)dev_v) & 31) == 0 ? 2 : 1);
  const int groups = ROT_THREADS / p.lanes;
  const long long across = (p.places * 2 * p.heads + groups - 1) / groups;
  if (across > 0x7FFFFFFFll) return STAND_E_ARG;
  int lpb = p.layers < 4 ? p.layers : 4;  // more in a row are slower: the layers lie far apart (4, 8, 32: 55, 57, 62 us for prompts of 32 layers, before stores of 32 bytes)
  while (lpb > 1 && across * ((p.layers + lpb - 1) / lpb) < 8 * 148) lpb = (lpb + 1) / 2;
  p.layers_block = lpb;
  const dim3 grid((unsigned)across, (unsigned)((p.layers + lpb - 1) / lpb));
  cudaStream_t st = (cudaStream_t)cu_stream;
  if (c->dtype == STAND_DTYPE_F32) return launch_read<float>(p, width, c->packed, grid, st);
  if (c->dtype == STAND_DTYPE_BF16) return launch_read<__nv_bfloat16>(p, width, c->packed, grid, st);
  return launch_read<__half>(p, width, c->packed, grid, st);
}

}  // extern "C"
