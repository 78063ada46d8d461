// Attention of draft trees over a paged cache: what the kernels share.
//
// Row r of a (sequence b, key head g) pair is node u = r / G under query head g * G + r % G, G = heads_q / heads_kv:
// all rows of the pair read the same keys and values, so they are read once for all of them.  The keys in order are
// the len cached positions, then the tree's nodes; node u sees all of the former and, of the latter, those its mask
// names.  With s = scale * log2(e) * q.k the softmax is carried as the running maximum m and the sums l = sum 2^(s-m)
// and o = sum 2^(s-m) v, all in fp32, so that pieces of the keys can be joined: with M = max m_i,
// o = sum 2^(m_i - M) o_i, l likewise; the result is o / l and lse = ln 2 (M + log2 l).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "common.cuh"

namespace stand {

struct AttnParams {
  const char* q;
  const char* k;
  const char* v;
  const char* cache_k;
  const char* cache_v;
  const int* table;
  const long long* len;
  const uint32_t* mask;
  long long mask_stride;
  const int* tree;
  char* out;
  float* lse;
  int B, N, heads_q, heads_kv, group, dim, page, pages, cols, mask_words;
  float scale2;  // scale * log2(e)
  long long q_stride[3], k_stride[3], v_stride[3], cache_stride[3];  // elements (packed cache: bytes)
};

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Cached tokens of sequence b that count.
__device__ __forceinline__ long long attn_len(const AttnParams& p, int b) {
  const long long n = p.len[b], most = (long long)p.cols * p.page;
  return n < 0 ? 0 : (n > most ? most : n);
}

// The nodes first .. first + 31 that node u of sequence b sees, as bits; of the last word of a mask, from bit first % 32
// on.  The last row tile of a pair may have rows beyond the last node: they see nothing, and no mask is read for them.
__host__ __device__ __forceinline__ uint32_t attn_nodes_seen(const AttnParams& p, int b, int u, int first) {
  const int below = u + 1 - first;  // nodes first .. u
  if (u >= p.N || below <= 0) return 0u;
  uint32_t bits = FULL;
  if (p.mask) bits = p.mask[(long long)b * p.mask_stride + (long long)u * p.mask_words + (first >> 5)] >> (first & 31);
  return below >= 32 ? bits : bits & ((1u << below) - 1);
}

// Does node u of sequence b see node v?
__device__ __forceinline__ bool attn_sees(const AttnParams& p, int b, int u, int v) {
  if (v > u) return false;
  return !p.mask || (p.mask[b * p.mask_stride + (long long)u * p.mask_words + (v >> 5)] >> (v & 31) & 1u);
}

// Values that are not finite.  A row's element is the sum of those that it sees, whatever their weights: +inf, -inf or NaN.
// The kernels' sums come out as NaN where such a value met a weight of zero - one that is below its type, or that of a
// key which a lane only carries along - or a row that does not see it.  So an element that is NaN although the row's
// weights are in order is settled by a second look at the values, for all kernels with this: the sum of the values that are
// not finite in element d among the cached tokens k0 .. k1 - 1 of sequence b.  Zero: there are none (such a sum is never zero).
// (A packed group is finite or NaN throughout.)
template <typename T, bool PACKED = false> __device__ __forceinline__ float attn_odd_cached(const AttnParams& p, int b, int g, int d, int k0, int k1) {
  if constexpr (PACKED) {
    bool bad = false;
    const unsigned char* scales = reinterpret_cast<const unsigned char*>(p.cache_v) + g * p.cache_stride[1] + (long long)p.page * (p.dim / 2) + d / 16;
    for (int k = k0; k < k1 && !bad; k += 8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int pos = k + i, col = pos / p.page;
        if (pos >= k1) continue;
        const int page = p.table[(long long)b * p.cols + col];
        if (page >= 0 && page < p.pages) bad = bad || scales[page * p.cache_stride[0] + (pos - col * p.page) * (p.dim / 16)] >= 0xF8;
      }
    }
    return bad ? NAN : 0.0f;
  }
  const T* cache = reinterpret_cast<const T*>(p.cache_v) + g * p.cache_stride[1] + d;
  float sum = 0.0f;
  for (int k = k0; k < k1 && !isnan(sum); k += 8) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int pos = k + i, col = pos / p.page;
      f[i] = 0.0f;
      if (pos >= k1) continue;
      const int page = p.table[(long long)b * p.cols + col];
      if (page >= 0 && page < p.pages) f[i] = to_float(cache[page * p.cache_stride[0] + (long long)(pos - col * p.page) * p.cache_stride[2]]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (!isfinite(f[i])) sum += f[i];
  }
  return sum;
}

}  // namespace stand
