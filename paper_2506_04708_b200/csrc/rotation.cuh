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
// bytes each without conflict (VE = 1: one after the other).  Places past the last pair hold
// 1 and 0 and turn nothing.
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

// VE elements, 16, 8 or 4 (2) bytes at a time: as they lie, and as floats.
template <typename T, int VE> __device__ __forceinline__ void copy_vec(T* to, const T* from) {
  if constexpr (sizeof(T) * VE >= 8) {
    using W = typename std::conditional<(sizeof(T) * VE >= 16), uint4, uint2>::type;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) * VE / sizeof(W)); ++i) reinterpret_cast<W*>(to)[i] = reinterpret_cast<const W*>(from)[i];
  } else {
#pragma unroll
    for (int k = 0; k < VE; ++k) to[k] = from[k];
  }
}
template <typename T, int VE> __device__ __forceinline__ void load_vec(const T* p, float* v) {
  alignas(16) T e[VE];
  copy_vec<T, VE>(e, p);
#pragma unroll
  for (int k = 0; k < VE; ++k) v[k] = to_float(e[k]);
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

__device__ __forceinline__ unsigned long long mul2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
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
    // A last unit may have fewer pairs than vectors have room for; what is not turned stays as it is (a turn by nothing would
    // multiply it by 0, and its neighbour need not be finite).
    const int left = t.half - u * VE;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const float a = y[2 * i], b = y[2 * i + 1];
      y[2 * i] = i < left ? fmaf(a, c[i], -b * s[i]) : a;
      y[2 * i + 1] = i < left ? fmaf(a, s[i], b * c[i]) : b;
    }
  } else {
    if constexpr (VE >= 4) {
#pragma unroll
      for (int i = 0; i < VE; i += 2) {
        const unsigned long long a = pack2(y[i], y[i + 1]), b = pack2(y[VE + i], y[VE + i + 1]), c2 = pack2(c[i], c[i + 1]), s2 = pack2(s[i], s[i + 1]);
        unpack2(fma2(mul2(b, s2), pack2(-1.0f, -1.0f), mul2(a, c2)), y[i], y[i + 1]);
        unpack2(fma2(a, s2, mul2(b, c2)), y[VE + i], y[VE + i + 1]);
      }
    } else {
      const float a = y[0], b = y[1];
      y[0] = fmaf(a, c[0], -b * s[0]);
      y[1] = fmaf(a, s[0], b * c[0]);
    }
  }
}

// What a lane does in every row of one kind (queries, keys, values): the places of its units.
template <typename T, int VE> struct RowLane {
  static constexpr int K = VE == 1 ? 4 : 1;  // units
  int unit, a[K], b[K];                      // elements a .. and b .. (each VE of them)
  bool turned[K], has_a[K], has_b[K];        // where there is nothing the row's first elements are read and not used: loads have no conditions

  __device__ __forceinline__ RowLane(const Turn& t, int lane, bool turn) : unit(lane) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = lane + k * t.lanes;
      turned[k] = turn && u < t.columns;
      a[k] = u * 2 * VE;
      b[k] = a[k] + VE;
      if (turn && !t.pairs) {
        if (turned[k]) a[k] = u * VE, b[k] = t.half + a[k];
        else a[k] = 2 * t.half + (u - t.columns) * 2 * VE, b[k] = a[k] + VE;
      }
      has_a[k] = a[k] < t.dim;
      has_b[k] = b[k] < t.dim;
      if (!has_a[k]) a[k] = 0;
      if (!has_b[k]) b[k] = 0;
    }
  }
  // A row's elements as they lie.
  struct Raw {
    alignas(16) T e[K][2 * VE];
  };
  __device__ __forceinline__ void read(const T* from, Raw& raw) const {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      copy_vec<T, VE>(raw.e[k], from + a[k]);
      copy_vec<T, VE>(raw.e[k] + VE, from + b[k]);
    }
  }
  // The row normalised (weighted: by what weights(w, k) gives for unit k), turned by the table cs and, if it is there (in; else any row was read),
  // given to put(y, a, b, whether there is a second vector) unit by unit.  All lanes of the warp.
  template <typename W, typename F>
  __device__ __forceinline__ void row(const Turn& t, const Raw& raw, bool weighted, W weights, const float* cs, bool in, bool norm, F put) const {
    float y[K][2 * VE];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < 2 * VE; ++i) y[k][i] = to_float(raw.e[k][i]);
    if (norm) {
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float part;
          const float* v = y[k] + h * VE;
          if constexpr (VE >= 4) {
            unsigned long long sum2 = mul2(pack2(v[0], v[1]), pack2(v[0], v[1]));
#pragma unroll
            for (int i = 2; i < VE; i += 2) sum2 = fma2(pack2(v[i], v[i + 1]), pack2(v[i], v[i + 1]), sum2);
            float lo, hi;
            unpack2(sum2, lo, hi);
            part = lo + hi;
          } else {
            part = v[0] * v[0];
          }
          sum += (h ? has_b[k] : has_a[k]) ? part : 0.0f;
        }
      for (int o = 1; o < t.lanes; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
      const float r = rsqrtf(fmaf(sum, t.inv_dim, t.eps));
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < 2 * VE; i += 2) unpack2(mul2(pack2(y[k][i], y[k][i + 1]), pack2(r, r)), y[k][i], y[k][i + 1]);
      if (weighted) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
          alignas(16) float w[2 * VE];
          weights(w, k);
#pragma unroll
          for (int i = 0; i < 2 * VE; i += 2) unpack2(mul2(pack2(y[k][i], y[k][i + 1]), pack2(w[i], w[i + 1])), y[k][i], y[k][i + 1]);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (turned[k]) turn_unit<VE>(t, cs, unit + k * t.lanes, y[k]);
      if (in && has_a[k]) put(y[k], a[k], b[k], has_b[k]);
    }
  }
};

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
