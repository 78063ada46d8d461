// A head's row, normalised and turned by its token's position: what head rotation and cache append share.
//
// y = x * rsqrt(mean(x^2) + eps) * w;  pair i: (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = position * freq[i].
// A lane has a unit of the row: two vectors of VE neighbouring elements that hold VE whole pairs - half a head apart, or next to
// one another - so nothing is read twice and a row in place is safe.  VE is 8, 4 or, where nothing is aligned, 1 (then up to four
// units a lane).  As many lanes as the units need, a power of two, have a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "attention.cuh"
#include "common.cuh"

namespace stand {

constexpr int ROT_DIM_MAX = 256;

struct Turn {
  const float* freq;         // null: rows are not turned
  const long long* base;     // [B], null: 0
  const int* offset;         // null: the node's number
  long long offset_stride;
  int half, pairs;           // pairs of elements; neighbours are pairs (else half a head apart)
  int columns;               // units with pairs
  int units, lanes;          // of a row
  int norm;
  float eps, inv_dim;
  int dim;
};

// A token's table: cos, then sin, of angle c * VE + j (pair j of unit c) at ((j / 4) * columns + c) * 4 + j % 4, so that the lanes of a row read 16
// bytes each without conflict (VE = 1: one after the other).  Places past the last pair hold 1 and 0.
template <int VE> __host__ __device__ __forceinline__ int turn_floats(int columns) { return (columns * VE + 3) & ~3; }  // cos alone
template <int VE> __device__ __forceinline__ int turn_at(int columns, int i) {
  const int c = i / VE, j = i % VE;
  if (VE < 4) return i;
  return ((j >> 2) * columns + c) * 4 + (j & 3);
}

__device__ __forceinline__ long long turn_position(const Turn& t, int b, int n) {
  return (t.base ? t.base[b] : 0) + (t.offset ? t.offset[b * t.offset_stride + n] : n);
}

// The angle in turns, in 64 bits: positions go far beyond a turn.  What the 32-bit remainder lacks is added to first order.
__device__ __forceinline__ void turn_angle(long long position, float freq, float& c, float& s) {
  const double turns = (double)position * (double)freq * 0.15915494309189535;
  const double rest = 2.0 * (turns - rint(turns));  // in half turns
  const float x = (float)rest, left = (float)(rest - (double)x) * 3.14159265358979f;
  float s0, c0;
  sincospif(x, &s0, &c0);
  c = fmaf(-s0, left, c0);
  s = fmaf(c0, left, s0);
}

// VE elements as they lie: 16, 8 or 4 (2) bytes at a time.
template <typename T, int VE> __device__ __forceinline__ void load_vec(const T* p, float* v) {
  if constexpr (sizeof(T) * VE >= 8) {
    using W = typename std::conditional<(sizeof(T) * VE >= 16), uint4, uint2>::type;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * VE / sizeof(W)); ++i) {
      const W w = reinterpret_cast<const W*>(p)[i];
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int k = 0; k < (int)(sizeof(W) / sizeof(T)); ++k) v[i * (sizeof(W) / sizeof(T)) + k] = to_float(e[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < VE; ++k) v[k] = to_float(p[k]);
  }
}
template <typename T, int VE> __device__ __forceinline__ void store_vec(T* p, const float* y) {
  if constexpr (sizeof(T) * VE >= 8) {
    using W = typename std::conditional<(sizeof(T) * VE >= 16), uint4, uint2>::type;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * VE / sizeof(W)); ++i) {
      W w;
      T* e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int k = 0; k < (int)(sizeof(W) / sizeof(T)); ++k) e[k] = from_float<T>(y[i * (sizeof(W) / sizeof(T)) + k]);
      reinterpret_cast<W*>(p)[i] = w;
    }
  } else {
#pragma unroll
    for (int k = 0; k < VE; ++k) p[k] = from_float<T>(y[k]);
  }
}

// Where unit u of a row lies: elements a .. and b .. (each VE of them, if below dim).  turn: of this row.
template <int VE> __device__ __forceinline__ bool unit_place(const Turn& t, bool turn, int u, int& a, int& b) {
  const bool turned = turn && u < t.columns;
  a = u * 2 * VE;
  b = a + VE;
  if (turn && !t.pairs) {
    if (turned) a = u * VE, b = t.half + a;
    else a = 2 * t.half + (u - t.columns) * 2 * VE, b = a + VE;
  }
  return turned;
}

// 1 / the root of the mean square of a row, of whose squares this lane has `sum`.  All lanes of the warp.
__device__ __forceinline__ float row_scale(const Turn& t, float sum) {
  for (int o = 1; o < t.lanes; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
  return rsqrtf(fmaf(sum, t.inv_dim, t.eps));
}

template <int VE> __device__ __forceinline__ void turn_unit(const Turn& t, const float* cs, int u, float (&y)[2 * VE]) {
  const float* sn = cs + turn_floats<VE>(t.columns);
  float c[VE], s[VE];
  if constexpr (VE >= 4) {
#pragma unroll
    for (int q = 0; q < VE / 4; ++q) {
      const float4 cq = *reinterpret_cast<const float4*>(cs + (q * t.columns + u) * 4), sq = *reinterpret_cast<const float4*>(sn + (q * t.columns + u) * 4);
      c[4 * q] = cq.x, c[4 * q + 1] = cq.y, c[4 * q + 2] = cq.z, c[4 * q + 3] = cq.w;
      s[4 * q] = sq.x, s[4 * q + 1] = sq.y, s[4 * q + 2] = sq.z, s[4 * q + 3] = sq.w;
    }
  } else {
    c[0] = cs[u];
    s[0] = sn[u];
  }
  if (t.pairs) {
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = fmaf(a, c[i], -b * s[i]);
      y[2 * i + 1] = fmaf(a, s[i], b * c[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const float a = y[i], b = y[VE + i];
      y[i] = fmaf(a, c[i], -b * s[i]);
      y[VE + i] = fmaf(a, s[i], b * c[i]);
    }
  }
}

// Every unit of a row that this lane has, read, normalised by `weight` (null: ones) and turned by the table `cs`, given to put(y, a, b) with
// the places of its two vectors.  All lanes of the warp call it; in: the row is there.  norm, turn: of this row.
template <typename T, int VE, typename WT, typename F>
__device__ __forceinline__ void row_units(const Turn& t, const T* row, const WT* weight, const float* cs, int lane, bool in, bool norm, bool turn, F put) {
  constexpr int K = VE == 1 ? 4 : 1;  // units of a lane
  float y[K][2 * VE];
  int a[K], b[K];
  bool turned[K];
  float sum = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int u = lane + k * t.lanes;
    turned[k] = unit_place<VE>(t, turn, u, a[k], b[k]);
    if (!in) a[k] = b[k] = t.dim;
#pragma unroll
    for (int i = 0; i < 2 * VE; ++i) y[k][i] = 0.0f;
    if (a[k] < t.dim) load_vec<T, VE>(row + a[k], y[k]);
    if (b[k] < t.dim) load_vec<T, VE>(row + b[k], y[k] + VE);
  }
  if (t.norm) {  // of the call; rows of a warp may differ in `norm`, the exchange is everybody's
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 2 * VE; ++i) sum = fmaf(y[k][i], y[k][i], sum);
    const float r = row_scale(t, sum);
    if (norm) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        float w[2 * VE];
#pragma unroll
        for (int i = 0; i < 2 * VE; ++i) w[i] = 1.0f;
        if (weight && a[k] < t.dim) load_vec<WT, VE>(weight + a[k], w);
        if (weight && b[k] < t.dim) load_vec<WT, VE>(weight + b[k], w + VE);
#pragma unroll
        for (int i = 0; i < 2 * VE; ++i) y[k][i] = y[k][i] * r * w[i];
      }
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if (a[k] >= t.dim) continue;
    if (turned[k]) turn_unit<VE>(t, cs, lane + k * t.lanes, y[k]);
    put(y[k], a[k], b[k]);
  }
}

// Units of VE elements: every vector lies within one kind of element.
inline bool turn_fits(const Turn& t, int ve) { return t.dim % ve == 0 && (!t.freq || t.pairs || t.half % ve == 0); }
inline void turn_units(Turn& t, int ve) {
  t.columns = (t.half + ve - 1) / ve;
  t.units = (t.dim + 2 * ve - 1) / (2 * ve);
  if (t.freq && !t.pairs) t.units = t.columns + (t.dim - 2 * t.half + 2 * ve - 1) / (2 * ve);
  t.lanes = 1;
  while (t.lanes < t.units && t.lanes < 32) t.lanes *= 2;
}

}  // namespace stand
