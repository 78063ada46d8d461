// Tree attention without matrix instructions: any type, any strides, any head size up to ATTN_DIM_MAX.
#pragma once
#include "attention.cuh"
#include "launch.cuh"

namespace stand {

constexpr int ATTN_DIM_MAX = 256;
constexpr int PA_WARPS = 4, PA_ROWS = 4;       // rows per warp
constexpr int PA_BLOCK_ROWS = PA_WARPS * PA_ROWS;
constexpr int PA_KEYS = 32;                    // keys per tile, one per lane
constexpr int PA_OUT = ATTN_DIM_MAX / 32;      // output elements of a row per lane

inline size_t plain_smem_bytes(int dim) { return sizeof(float) * (size_t)(PA_KEYS * (dim + 1) + PA_KEYS * dim + PA_BLOCK_ROWS * dim); }

template <typename T>
__global__ void __launch_bounds__(PA_WARPS * 32) plain_attention_kernel(const AttnParams p) {
  extern __shared__ float pa_smem[];
  __shared__ const T* s_key[PA_KEYS];
  __shared__ const T* s_value[PA_KEYS];
  const int D = p.dim, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float* sk = pa_smem;                       // [PA_KEYS][D + 1]
  float* sv = sk + PA_KEYS * (D + 1);        // [PA_KEYS][D]
  float* sq = sv + PA_KEYS * D;              // [PA_BLOCK_ROWS][D]
  pdl_trigger();
  pdl_wait();
  const int R = p.N * p.group;
  const int b = (int)(blockIdx.x / p.heads_kv), g = (int)(blockIdx.x % p.heads_kv);
  const int r0 = blockIdx.y * PA_BLOCK_ROWS;
  const int n_rows = R - r0 < PA_BLOCK_ROWS ? R - r0 : PA_BLOCK_ROWS;
  const long long len = attn_len(p, b);
  const int last_node = (r0 + n_rows - 1) / p.group;
  const long long n_keys = len + last_node + 1;

  for (int i = tid; i < PA_BLOCK_ROWS * D; i += PA_WARPS * 32) {
    const int r = r0 + i / D, d = i % D;
    float v = 0.0f;
    if (r < R) {
      const int u = r / p.group, h = g * p.group + r % p.group;
      v = to_float(reinterpret_cast<const T*>(p.q)[b * p.q_stride[0] + u * p.q_stride[1] + h * p.q_stride[2] + d]);
    }
    sq[i] = v;
  }
  int node[PA_ROWS];
  bool live[PA_ROWS];
  float m[PA_ROWS], l[PA_ROWS], o[PA_ROWS][PA_OUT];
#pragma unroll
  for (int i = 0; i < PA_ROWS; ++i) {
    const int r = r0 + warp * PA_ROWS + i;
    node[i] = r / p.group;
    live[i] = r < R && !(p.tree && p.tree[(long long)b * p.N + node[i]] < 0);
    m[i] = -INFINITY;
    l[i] = 0.0f;
#pragma unroll
    for (int e = 0; e < PA_OUT; ++e) o[i][e] = 0.0f;
  }

  for (long long k0 = 0; k0 < n_keys; k0 += PA_KEYS) {
    __syncthreads();  // the tile before has been used
    if (tid < PA_KEYS) {
      const long long pos = k0 + tid;
      const T *key = nullptr, *value = nullptr;
      if (pos < len) {
        const long long c = pos / p.page;
        const int page = p.table[(long long)b * p.cols + c];
        if (page >= 0 && page < p.pages) {
          const long long at = page * p.cache_stride[0] + g * p.cache_stride[1] + (pos - c * p.page) * p.cache_stride[2];
          key = reinterpret_cast<const T*>(p.cache_k) + at;
          value = reinterpret_cast<const T*>(p.cache_v) + at;
        }
      } else if (pos < n_keys) {
        const long long at = b * p.kv_stride[0] + (pos - len) * p.kv_stride[1] + g * p.kv_stride[2];
        key = reinterpret_cast<const T*>(p.k) + at;
        value = reinterpret_cast<const T*>(p.v) + at;
      }
      s_key[tid] = key;
      s_value[tid] = value;
    }
    __syncthreads();
    for (int i = tid; i < PA_KEYS * D; i += PA_WARPS * 32) {
      const int j = i / D, d = i % D;
      sk[j * (D + 1) + d] = s_key[j] ? to_float(s_key[j][d]) : 0.0f;
      sv[j * D + d] = s_value[j] ? to_float(s_value[j][d]) : 0.0f;
    }
    __syncthreads();
    float s[PA_ROWS];
#pragma unroll
    for (int i = 0; i < PA_ROWS; ++i) s[i] = 0.0f;
    const float* q0 = sq + warp * PA_ROWS * D;
    for (int d = 0; d < D; ++d) {
      const float kd = sk[lane * (D + 1) + d];
#pragma unroll
      for (int i = 0; i < PA_ROWS; ++i) s[i] = fmaf(q0[i * D + d], kd, s[i]);
    }
    const long long pos = k0 + lane;
#pragma unroll
    for (int i = 0; i < PA_ROWS; ++i) {
      bool sees = live[i] && pos < n_keys;
      if (sees && pos >= len) sees = attn_sees(p, b, node[i], (int)(pos - len));
      const uint32_t seen = __ballot_sync(FULL, sees);
      if (seen == 0) continue;
      const float x = sees ? s[i] * p.scale2 : -INFINITY;
      const float top = fmaxf(m[i], warp_max_f(x));
      const float base = top == -INFINITY ? 0.0f : top;
      const float w = sees ? exp2f(x - base) : 0.0f;
      const float keep = exp2f(m[i] - base);
      m[i] = top;
      l[i] = l[i] * keep + warp_sum_f(w);
#pragma unroll
      for (int e = 0; e < PA_OUT; ++e) o[i][e] *= keep;
      for (int j = 0; j < PA_KEYS; ++j) {
        if (!(seen >> j & 1u)) continue;  // an unseen value may be anything, 0 times it too
        const float wj = __shfl_sync(FULL, w, j);
#pragma unroll
        for (int e = 0; e < PA_OUT; ++e)
          if (e * 32 + lane < D) o[i][e] = fmaf(wj, sv[j * D + e * 32 + lane], o[i][e]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PA_ROWS; ++i) {
    const int r = r0 + warp * PA_ROWS + i;
    if (r >= R) continue;
    const int u = r / p.group, h = g * p.group + r % p.group;
    const long long row = ((long long)b * p.N + u) * p.heads_q + h;
    const bool empty = l[i] == 0.0f;
#pragma unroll
    for (int e = 0; e < PA_OUT; ++e)
      if (e * 32 + lane < D) reinterpret_cast<T*>(p.out)[row * D + e * 32 + lane] = from_float<T>(empty ? 0.0f : o[i][e] / l[i]);
    if (p.lse && lane == 0) p.lse[row] = empty ? -INFINITY : 0.6931471805599453f * (m[i] + log2f(l[i]));
  }
}

template <typename T> int launch_plain_attention(const AttnParams& p, cudaStream_t st) {
  const size_t smem = plain_smem_bytes(p.dim);
  static SmemLimit limit;
  int rc = limit.raise(plain_attention_kernel<T>, plain_smem_bytes(ATTN_DIM_MAX));
  if (rc) return rc;
  const int R = p.N * p.group;
  const dim3 grid((unsigned)(p.B * p.heads_kv), (unsigned)((R + PA_BLOCK_ROWS - 1) / PA_BLOCK_ROWS));
  return launch_dependent(plain_attention_kernel<T>, grid, PA_WARPS * 32, st, p, smem);
}

}  // namespace stand
