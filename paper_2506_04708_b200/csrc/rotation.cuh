// A head's row, normalised and turned by its token's position: what head rotation and cache append share.
//
// y = x * rsqrt(mean(x^2) + eps) * w;  pair i: (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = position * freq[i].
// A lane has 16 neighbouring elements of a row, as many lanes as that takes (a power of two, up to 16) have the row; where the
// pairs lie half a head apart a lane reads its partners' elements too, which are on their way to another lane of the warp anyway.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "attention.cuh"
#include "common.cuh"

namespace stand {

constexpr int ROT_DIM_MAX = 256;
constexpr int ROT_E = 16;  // elements of a lane

struct Turn {
  const float* freq;         // null: rows are not turned
  const long long* base;     // [B], null: 0
  const int* offset;         // null: the node's number
  long long offset_stride;
  int half, pairs;           // pairs of elements; neighbours are pairs (else half a head apart)
  int columns;               // of the table below
  int norm;
  float eps, inv_dim;
  int dim, lanes;            // lanes of a row
};

// cos and sin of a token: [2][4 * columns * 4] floats.  Angle i belongs to lane column c and place j of it; four places lie
// together, columns side by side, so that the lanes of a row read 16 bytes each without conflict.
__host__ __device__ __forceinline__ int turn_columns(int half, int pairs) { return pairs ? (half + 7) / 8 : (half + 15) / 16; }
__device__ __forceinline__ int turn_at(const Turn& t, int i) {
  const int c = t.pairs ? i >> 3 : i >> 4, j = t.pairs ? i & 7 : i & 15;
  return ((j >> 2) * t.columns + c) * 4 + (j & 3);
}
__host__ __device__ __forceinline__ int turn_floats(int columns, int pairs) { return columns * (pairs ? 8 : 16); }  // cos alone

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

template <typename T> __device__ __forceinline__ void load_row16(const T* p, float* v) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint4 w = reinterpret_cast<const uint4*>(p)[i];
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[8 * i + k] = to_float(e[k]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 w = reinterpret_cast<const float4*>(p)[i];
      v[4 * i] = w.x, v[4 * i + 1] = w.y, v[4 * i + 2] = w.z, v[4 * i + 3] = w.w;
    }
  }
}

template <typename T> __device__ __forceinline__ void store_row16(T* p, const float* y) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint4 w;
      T* e = reinterpret_cast<T*>(&w);
#pragma unroll
      for (int k = 0; k < 8; ++k) e[k] = from_float<T>(y[8 * i + k]);
      reinterpret_cast<uint4*>(p)[i] = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
  }
}

// Elements 16 c .. of `row` in y: read, normalised by `weight` (null: ones), turned by the table `cs`.  All lanes of the warp call
// it; `there`: this lane has such elements.  WIDE: 16 elements lie within 16-byte pieces and pairs within or between whole
// lanes' elements; else element by element.  norm, turn: of this row (the same for all lanes of it).
template <typename T, bool WIDE>
__device__ __forceinline__ void row_group(const Turn& t, const T* row, const T* weight, const float* cs, int c, bool there, bool norm, bool turn,
                                          float (&y)[ROT_E]) {
  const int e0 = c * ROT_E, rotary = 2 * t.half;
  const bool turned = turn && there && e0 < rotary;
  float other[ROT_E];
  int partner = 0;  // first of the partners' elements (WIDE, halves)
  if (WIDE) {
    if (there) load_row16(row + e0, y);
    if (turned && !t.pairs) {
      partner = e0 < t.half ? e0 + t.half : e0 - t.half;
      load_row16(row + partner, other);
    }
  } else {
#pragma unroll
    for (int i = 0; i < ROT_E; ++i) {
      const int e = e0 + i;
      y[i] = there && e < t.dim ? to_float(row[e]) : 0.0f;
      other[i] = 0.0f;
      if (turned && e < rotary) other[i] = to_float(row[t.pairs ? e ^ 1 : (e < t.half ? e + t.half : e - t.half)]);
    }
  }
  if (t.norm) {  // of the call; rows of a warp may differ in `norm`, the exchange is everybody's
    float sum = 0.0f;
    if (there) {
#pragma unroll
      for (int i = 0; i < ROT_E; ++i) sum = fmaf(y[i], y[i], sum);
    }
    for (int o = 1; o < t.lanes; o <<= 1) sum += __shfl_xor_sync(FULL, sum, o);
    if (norm && there) {
      const float r = rsqrtf(fmaf(sum, t.inv_dim, t.eps));
      if (WIDE) {
        float w[ROT_E];
#pragma unroll
        for (int i = 0; i < ROT_E; ++i) w[i] = 1.0f;
        if (weight) load_row16(weight + e0, w);
#pragma unroll
        for (int i = 0; i < ROT_E; ++i) y[i] = y[i] * r * w[i];
        if (turned && !t.pairs) {
          if (weight) load_row16(weight + partner, w);
#pragma unroll
          for (int i = 0; i < ROT_E; ++i) other[i] = other[i] * r * w[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < ROT_E; ++i) {
          const int e = e0 + i;
          if (e < t.dim) y[i] = y[i] * r * (weight ? to_float(weight[e]) : 1.0f);
          if (turned && e < rotary)
            other[i] = other[i] * r * (weight ? to_float(weight[t.pairs ? e ^ 1 : (e < t.half ? e + t.half : e - t.half)]) : 1.0f);
        }
      }
    }
  }
  if (!turned) return;
  const float* sn = cs + turn_floats(t.columns, t.pairs);
  if (WIDE) {
    if (t.pairs) {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float4 co = *reinterpret_cast<const float4*>(cs + (q * t.columns + c) * 4), si = *reinterpret_cast<const float4*>(sn + (q * t.columns + c) * 4);
        const float cv[4] = {co.x, co.y, co.z, co.w}, sv[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = y[8 * q + 2 * i], b = y[8 * q + 2 * i + 1];
          y[8 * q + 2 * i] = fmaf(a, cv[i], -b * sv[i]);
          y[8 * q + 2 * i + 1] = fmaf(a, sv[i], b * cv[i]);
        }
      }
    } else {
      const bool second = e0 >= t.half;
      const int col = second ? c - t.half / ROT_E : c;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 co = *reinterpret_cast<const float4*>(cs + (q * t.columns + col) * 4), si = *reinterpret_cast<const float4*>(sn + (q * t.columns + col) * 4);
        const float cv[4] = {co.x, co.y, co.z, co.w}, sv[4] = {si.x, si.y, si.z, si.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) y[4 * q + i] = fmaf(y[4 * q + i], cv[i], other[4 * q + i] * (second ? sv[i] : -sv[i]));
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < ROT_E; ++i) {
      const int e = e0 + i;
      if (e >= rotary) continue;
      const bool second = t.pairs ? e & 1 : e >= t.half;
      const int at = turn_at(t, t.pairs ? e >> 1 : (second ? e - t.half : e));
      y[i] = fmaf(y[i], cs[at], other[i] * (second ? sn[at] : -sn[at]));
    }
  }
}

// Where a lane's 16 elements can be read and written at once, and pairs are whole lanes' elements or within one's.
inline bool turn_wide(const Turn& t) { return t.dim % ROT_E == 0 && (!t.freq || (t.pairs ? 2 * t.half : t.half) % ROT_E == 0); }
inline int row_lanes(int dim) {
  int n = 1;
  while (n * ROT_E < dim) n *= 2;
  return n;
}

}  // namespace stand
