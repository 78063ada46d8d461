// Tree attention without matrix instructions: any type (single precision among them), any strides, any head size up to
// ATTN_DIM_MAX.
//
// A block takes up to 32 rows of a pair and walks over its tiles of 64 keys (attention_split.cuh), two tiles of keys and
// values in shared memory (single precision: cp.async; 16-bit types are converted on the way).  A warp has four rows; for the
// scores a lane has two keys, for the sums its share of the head size.  So every value from shared memory is used for four
// rows, and no sum crosses a warp.
// Measured, single precision, 8 x 16 nodes of 16 / 4 heads of 64, texts of 50 - 1,500: 39 us; 32 x 16 nodes, texts of 500 - 4,000:
// 259 us (8 rows a block: the same; 64 rows a block need 230 registers, one block per SM: 65 us where this took 42).
// Where the time goes (8 x 16 nodes, texts of one length): blocks of one piece of two tiles 22 us with launch and joining, of two
// pieces of one tile 27.5, each further tile 7.2 us with two blocks per SM.  So two tiles of an SM take 13,700 cycles; shared
// memory is busy for 6,150 of them, the multiply-add pipe for 4,100.  Neither bounds it: sixteen warps that meet at two
// barriers a tile do not hide the latencies of copy, products, softmax and sums, which follow one another.
#pragma once
#include "async.cuh"
#include "attention_split.cuh"
#include "launch.cuh"
#include "packed.cuh"

namespace stand {

constexpr int ATTN_DIM_MAX = 256;
constexpr int PA_WARPS = 8, PA_THREADS = PA_WARPS * 32, PA_ROWS = 32;  // rows of a block
static_assert(PA_THREADS == 4 * TA_KT, "a thread per row of two tiles");

template <int DP> struct PaShape {
  static constexpr int STAGES = DP == 256 ? 1 : 2;
  static constexpr int KP = DP + 4;                                     // floats between keys: no bank conflicts
  static constexpr int STAGE = TA_KT * KP + TA_KT * DP;                 // floats of a tile of keys and of values
  static constexpr int SMEM = (STAGES * STAGE + PA_ROWS * KP + PA_ROWS * TA_KT) * 4;
};
// Blocks per SM that the split counts on.
inline int plain_ctas(int dim) { return tensor_dim(dim) == 64 ? 2 : 1; }

template <typename T> __device__ __forceinline__ float4 load4(const T* p, bool wide) {
  if constexpr (sizeof(T) == 2) {
    if (wide) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      const T* e = reinterpret_cast<const T*>(&v);
      return make_float4(to_float(e[0]), to_float(e[1]), to_float(e[2]), to_float(e[3]));
    }
  } else if (wide) {
    return *reinterpret_cast<const float4*>(p);
  }
  return make_float4(to_float(p[0]), to_float(p[1]), to_float(p[2]), to_float(p[3]));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// An element that came out as NaN though its row's weights are in order: with the values that are not finite among what the
// row sees, cached tokens k0 .. k1 - 1 and nodes n0 .. n1 - 1.  Rare, so it only has to be right.
template <typename T, bool PACKED>
__device__ __noinline__ float plain_settle(const AttnParams& p, int b, int g, int u, int d, int k0, int k1, int n0, int n1, float o) {
  float sum = attn_odd_cached<T, PACKED>(p, b, g, d, k0, k1);
  const T* tree = reinterpret_cast<const T*>(p.v) + b * p.v_stride[0] + g * p.v_stride[2] + d;
  for (int v = n0; v < n1 && v <= u && !isnan(sum); ++v) {
    const float f = to_float(tree[v * p.v_stride[1]]);
    if (!isfinite(f) && attn_sees(p, b, u, v)) sum += f;
  }
  return sum == 0.0f ? o : sum;
}

// wide: bases and strides allow 4 elements at a time
template <typename T, int DP, bool PACKED>
__global__ void __launch_bounds__(PA_THREADS) plain_attention_kernel(const __grid_constant__ TaSplit p, const bool wide) {
  using Sh = PaShape<DP>;
  constexpr int KT = TA_KT, KP = Sh::KP, STAGES = Sh::STAGES, R = PA_ROWS / PA_WARPS, E = DP / 32;
  constexpr int EV = E < 4 ? E : 4;  // elements of the head size that lie together: lane * EV + 128 * i
  extern __shared__ float pa_smem[];
  __shared__ const T* s_src[3][2][KT];  // where keys and values of a tile lie; null: zeros
  __shared__ const unsigned char* s_scale[PACKED ? 3 : 1][2][KT];  // a packed row's scales (its codes lie at s_src); null: a tree's row
  __shared__ TaRange<PA_THREADS> s_range;
  float* const sq = pa_smem + STAGES * Sh::STAGE;                      // [PA_ROWS][KP]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, D = p.a.dim, D4 = (D + 3) & ~3;
  float* const sp = sq + PA_ROWS * KP + warp * R * KT;                      // [R][KT] of this warp
  pdl_trigger();
  pdl_wait();
  TaWalk walk;
  ta_begin<PA_THREADS>(p, walk, s_range, [] {}, [] {});
  // what a row has beyond the head size counts as zeros
  for (int i = tid; i < STAGES * KT * (D4 - D); i += PA_THREADS) {
    const int row = i / (D4 - D);
    pa_smem[row / KT * Sh::STAGE + row % KT * KP + D + i % (D4 - D)] = 0.0f;
  }

  TaSeg s;
  TaNote note(walk);
  while (walk.next(p, s)) {
    if (tid == 0) note.piece(walk, s, s_range.total, s_range.groups, blockIdx.x / p.group_ctas);
    if (!s.rows) continue;
    const T* kv[2] = {reinterpret_cast<const T*>(p.a.k), reinterpret_cast<const T*>(p.a.v)};
    const T* cache[2] = {reinterpret_cast<const T*>(p.a.cache_k), reinterpret_cast<const T*>(p.a.cache_v)};
    auto find = [&](int tile, int i) {  // where row i of a tile's keys (i < KT) or values is
      if (tile >= s.end) return;
      const int key = i % KT, which = i / KT;
      const T* src = nullptr;
      const unsigned char* scale = nullptr;
      if (tile < s.p_tiles) {
        const int pos = tile * KT + key, c = pos / p.a.page;
        if (pos < s.len) {
          const int page = p.a.table[(long long)s.b * p.a.cols + c];
          if (PACKED) {
            if (page >= 0 && page < p.a.pages) {
              const unsigned char* block = reinterpret_cast<const unsigned char*>(cache[which]) + page * p.a.cache_stride[0] + s.g * p.a.cache_stride[1];
              const int token = pos - c * p.a.page;
              src = reinterpret_cast<const T*>(block + token * (D / 2));
              scale = block + (long long)p.a.page * (D / 2) + token * (D / 16);
            }
          } else if (page >= 0 && page < p.a.pages)
            src = cache[which] + page * p.a.cache_stride[0] + s.g * p.a.cache_stride[1] + (long long)(pos - c * p.a.page) * p.a.cache_stride[2];
        }
      } else {
        const int node = (tile - s.p_tiles) * KT + key;
        const long long* stride = which ? p.a.v_stride : p.a.k_stride;
        if (node < p.a.N) src = kv[which] + s.b * stride[0] + node * stride[1] + s.g * stride[2];
      }
      s_src[tile % 3][which][key] = src;
      if (PACKED) s_scale[tile % 3][which][key] = scale;
    };
    auto fetch = [&](int tile) {
      if (tile < s.end) {
        float* const base = pa_smem + (tile % STAGES) * Sh::STAGE;
        if (PACKED && tile < s.p_tiles) {
          const int groups = D / PK_GROUP;
          for (int i = tid; i < 2 * KT * groups; i += PA_THREADS) {
            const int row = i / groups, c = i - row * groups, key = row % KT;
            const unsigned char* scales = s_scale[tile % 3][row / KT][key];
            float* dst = (row < KT ? base + key * KP : base + KT * KP + key * DP) + c * PK_GROUP;
            float v[PK_GROUP] = {};
            if (scales) {
              const uint2 w = reinterpret_cast<const uint2*>(s_src[tile % 3][row / KT][key])[c];
              const float scale = pk_scale(scales[c]);
              pk_values(w.x, scale, v);
              pk_values(w.y, scale, v + 8);
            }
#pragma unroll
            for (int e = 0; e < PK_GROUP; e += 4) *reinterpret_cast<float4*>(dst + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
          }
        } else if (wide) {
          const int quads = D / 4;
          for (int i = tid; i < 2 * KT * quads; i += PA_THREADS) {
            const int row = i / quads, q = i - row * quads, key = row % KT;
            const T* src = s_src[tile % 3][row / KT][key];
            float* dst = row < KT ? base + key * KP + q * 4 : base + KT * KP + key * DP + q * 4;
            if (!src) *reinterpret_cast<float4*>(dst) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            else if constexpr (sizeof(T) == 4) cp_async16(smem_addr(dst), src + q * 4);
            else *reinterpret_cast<float4*>(dst) = load4(src + q * 4, true);
          }
        } else {
          for (int i = tid; i < 2 * KT * D; i += PA_THREADS) {
            const int row = i / D, d = i - row * D, key = row % KT;
            const T* src = s_src[tile % 3][row / KT][key];
            float* dst = row < KT ? base + key * KP + d : base + KT * KP + key * DP + d;
            if (!src) *dst = 0.0f;
            else if constexpr (sizeof(T) == 4) cp_async4(smem_addr(dst), src + d);
            else *dst = to_float(src[d]);
          }
        }
      }
      cp_commit();
    };

    __syncthreads();  // the piece before has been read
    find(s.begin + tid / (2 * KT), tid % (2 * KT));
    // a warp's rows, by that warp alone
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = warp * R + i, r = s.row0 + row, u = r / p.a.group;
      const bool in = row < p.tile_rows && r < p.rows;
      const T* src = reinterpret_cast<const T*>(p.a.q) + s.b * p.a.q_stride[0] + u * p.a.q_stride[1] + (s.g * p.a.group + r - u * p.a.group) * p.a.q_stride[2];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = lane + 32 * e;
        if (d < D4) sq[row * KP + d] = in && d < D ? to_float(src[d]) : 0.0f;
      }
    }
    int node[R];
    bool live[R];
    float m[R], l[R], o[R][E];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = warp * R + i, r = s.row0 + row;
      node[i] = r / p.a.group;
      live[i] = row < p.tile_rows && r < p.rows && !(p.a.tree && p.a.tree[(long long)s.b * p.a.N + node[i]] < 0);
      m[i] = -INFINITY;
      l[i] = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[i][e] = 0.0f;
    }
    __syncthreads();
    if (STAGES == 2) fetch(s.begin);

    for (int j = s.begin; j < s.end; ++j) {
      if (STAGES == 2) {
        fetch(j + 1);
        if (tid < 2 * KT) find(j + 2, tid);
        cp_wait<1>();
      } else {
        fetch(j);
        if (tid < 2 * KT) find(j + 2, tid);
        cp_wait<0>();
      }
      __syncthreads();
      const float* sk = pa_smem + (j % STAGES) * Sh::STAGE;
      const float* sv = sk + KT * KP;
      // products of neighbours in pairs: half the instructions, two sums that are added at the end
      unsigned long long x2[R][2];
#pragma unroll
      for (int i = 0; i < R; ++i) x2[i][0] = x2[i][1] = pack2(0.0f, 0.0f);
      const float* q0 = sq + warp * R * KP;
#pragma unroll 2
      for (int d = 0; d < D4; d += 4) {
        const ulonglong2 k0 = *reinterpret_cast<const ulonglong2*>(sk + lane * KP + d), k1 = *reinterpret_cast<const ulonglong2*>(sk + (lane + 32) * KP + d);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(q0 + i * KP + d);
          x2[i][0] = fma2(q.y, k0.y, fma2(q.x, k0.x, x2[i][0]));
          x2[i][1] = fma2(q.y, k1.y, fma2(q.x, k1.x, x2[i][1]));
        }
      }
      float x[R][2];
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float lo, hi;
          unpack2(x2[i][c], lo, hi);
          x[i][c] = lo + hi;
        }
      // What no row sees of a text's last tile lies there as zeros.  In the tree, what one row does not see another may:
      // a value that is not finite must then not enter the first one's sum, 0 times it included.
      const bool tree = j >= s.p_tiles, partial = !tree && s.len - j * KT < KT;
      bool odd = false;
      if (tree) {
        const int nodes = p.a.N - (j - s.p_tiles) * KT;
        for (int i = tid; i < (nodes < KT ? nodes : KT) * D; i += PA_THREADS) odd = odd || !isfinite(sv[i / D * DP + i % D]);
        odd = __syncthreads_or(odd);
      }
      uint32_t seen[R][2];  // the tile's keys that a row sees: bits, by halves
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t bits = FULL;
          if (tree) {
            bits = attn_nodes_seen(p.a, s.b, node[i], (j - s.p_tiles) * KT + 32 * c);
          } else if (partial) {
            const int below = s.len - j * KT - 32 * c;
            bits = below >= 32 ? FULL : (below > 0 ? (1u << below) - 1 : 0u);
          }
          seen[i][c] = live[i] ? bits : 0u;
        }
      // row by row in step: the rows' shuffles and exponentials overlap
      float top[R], keep[R], sum[R];
#pragma unroll
      for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int c = 0; c < 2; ++c) x[i][c] = seen[i][c] >> lane & 1u ? x[i][c] * p.a.scale2 : -INFINITY;
        top[i] = fmaxf(x[i][0], x[i][1]);
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1)
#pragma unroll
        for (int i = 0; i < R; ++i) top[i] = fmaxf(top[i], __shfl_xor_sync(FULL, top[i], w));
#pragma unroll
      for (int i = 0; i < R; ++i) {
        top[i] = fmaxf(top[i], m[i]);
        const float base = top[i] == -INFINITY ? 0.0f : top[i];
        keep[i] = exp2f(m[i] - base);
        m[i] = top[i];
        float w[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          w[c] = seen[i][c] >> lane & 1u ? exp2f(x[i][c] - base) : 0.0f;
          sp[i * KT + lane + 32 * c] = w[c];
        }
        sum[i] = w[0] + w[1];
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1)
#pragma unroll
        for (int i = 0; i < R; ++i) sum[i] += __shfl_xor_sync(FULL, sum[i], w);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        l[i] = l[i] * keep[i] + sum[i];
#pragma unroll
        for (int e = 0; e < E; ++e) o[i][e] *= keep[i];
      }
      __syncwarp();
      if (!odd) {
#pragma unroll 1
        for (int k = 0; k < KT; k += 4) {
          float4 w[R];
#pragma unroll
          for (int i = 0; i < R; ++i) w[i] = *reinterpret_cast<const float4*>(sp + i * KT + k);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            unsigned long long v[E / 2];
#pragma unroll
            for (int e = 0; e < E; e += EV) {
              const float* src = sv + (k + kk) * DP + lane * EV + e / EV * 128;
              if constexpr (EV == 4) *reinterpret_cast<ulonglong2*>(v + e / 2) = *reinterpret_cast<const ulonglong2*>(src);
              else v[e / 2] = *reinterpret_cast<const unsigned long long*>(src);
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
              const float wk = kk == 0 ? w[i].x : (kk == 1 ? w[i].y : (kk == 2 ? w[i].z : w[i].w));
              const unsigned long long wk2 = pack2(wk, wk);
#pragma unroll
              for (int e = 0; e < E; e += 2) {
                const unsigned long long r = fma2(wk2, v[e / 2], pack2(o[i][e], o[i][e + 1]));
                unpack2(r, o[i][e], o[i][e + 1]);
              }
            }
          }
        }
      } else {  // row by row, only what it sees
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int c = 0; c < 2; ++c)
            for (uint32_t left = seen[i][c]; left; left &= left - 1) {
              const int k = 32 * c + __ffs(left) - 1;
              const float wk = sp[i * KT + k];
#pragma unroll
              for (int e = 0; e < E; ++e) o[i][e] = fmaf(wk, sv[k * DP + lane * EV + e / EV * 128 + e % EV], o[i][e]);
            }
      }
      __syncthreads();  // the tile has been read
    }

#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int row = warp * R + i, r = s.row0 + row;
      if (row >= p.tile_rows || r >= p.rows) continue;
      const int h = s.g * p.a.group + r - node[i] * p.a.group;
      const long long out = ((long long)s.b * p.a.N + node[i]) * p.a.heads_q + h, at = ta_part_row(p, s, row);
      const bool empty = !live[i] || l[i] == 0.0f;
      float zero = 0.0f;  // NaN if one of them is not finite
#pragma unroll
      for (int e = 0; e < E; ++e) zero = fmaf(o[i][e], 0.0f, zero);
      if (isnan(zero) && live[i] && isfinite(l[i])) {
        const int k1 = s.end * KT, n0 = s.begin > s.p_tiles ? s.begin - s.p_tiles : 0, n1 = s.end > s.p_tiles ? s.end - s.p_tiles : 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int d = lane * EV + e / EV * 128 + e % EV;
          if (isnan(o[i][e]) && d < D)
            o[i][e] = plain_settle<T, PACKED>(p.a, s.b, s.g, node[i], d, s.begin * KT, k1 < s.len ? k1 : s.len, n0 * KT, n1 * KT, o[i][e]);
        }
      }
      if (lane == 0) {
        if (!s.whole) p.part_ml[at] = live[i] ? make_float2(m[i], l[i]) : make_float2(-INFINITY, 0.0f);
        else if (p.a.lse) p.a.lse[out] = empty ? -INFINITY : 0.6931471805599453f * (m[i] + log2f(l[i]));
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int d = lane * EV + e / EV * 128 + e % EV;
        if (!s.whole) p.part_o[at * DP + d] = o[i][e];
        else if (d < D) reinterpret_cast<T*>(p.a.out)[out * D + d] = from_float<T>(empty ? 0.0f : o[i][e] / l[i]);
      }
    }
  }
  if (tid == 0 && blockIdx.x % p.group_ctas == 0) p.records[blockIdx.x / p.group_ctas] = note.r;
}

template <typename T, int DP, bool PACKED> int launch_plain_rows(const AttnParams& a, void* scratch, int sms, cudaStream_t st) {
  TaSplit p;
  // A piece's fixed cost in tiles: with 0, 1, 3, 6 16 x 8 nodes of heads of 128 over 10 - 1,000 take 66, 63, 66, 75 us, 32 x 16 nodes of heads
  // of 64 over 500 - 4,000 261, 259, 268, 285.
  ta_split(p, a, PA_ROWS, DP, sms, plain_ctas(DP), 1, scratch);
  const size_t al = 4 * sizeof(T);
  const bool cached = !PACKED && a.cols > 0;
  uintptr_t bits = (uintptr_t)a.k | (uintptr_t)a.v | (cached ? (uintptr_t)a.cache_k | (uintptr_t)a.cache_v : 0);
  for (int i = 0; i < 3; ++i) bits |= (uintptr_t)((a.k_stride[i] | a.v_stride[i]) * sizeof(T)) | (cached ? (uintptr_t)(a.cache_stride[i] * sizeof(T)) : 0);
  const bool wide = bits % al == 0 && a.dim % 4 == 0;
  static SmemLimit limit;
  const int smem = PaShape<DP>::SMEM;
  int rc = limit.raise(plain_attention_kernel<T, DP, PACKED>, smem);
  if (rc) return rc;
  rc = launch_dependent2(plain_attention_kernel<T, DP, PACKED>, dim3((unsigned)(p.groups * p.group_ctas)), PA_THREADS, st, (size_t)smem, p, wide);
  if (rc) return rc;
  return launch_join<DP, T>(p, st);
}

template <typename T, bool PACKED = false> int launch_plain_attention(const AttnParams& a, void* scratch, int sms, cudaStream_t st) {
  const int dp = tensor_dim(a.dim);
  if (dp == 64) return launch_plain_rows<T, 64, PACKED>(a, scratch, sms, st);
  if (dp == 128) return launch_plain_rows<T, 128, PACKED>(a, scratch, sms, st);
  return launch_plain_rows<T, 256, PACKED>(a, scratch, sms, st);
}

}  // namespace stand
