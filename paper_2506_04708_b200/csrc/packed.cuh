// The 4-bit form of cached rows.
//
// A row's elements in groups of 16: a scale s of 8 bits - 5 exponent bits (bias 15), 3 fraction bits, no sign, subnormals, the
// bits of a half between its sign and its last seven - and 16 whole numbers k of -8 .. 7 as k + 8 in 4 bits; an element is k s.
// That has at most 7 significant bits: exact in bfloat16 and, within its range, in half, so products of values are those of the definition.
// s is the smallest with 7 s >= the group's largest magnitude, k the nearest whole number (even in a tie).  Exponent 31: not finite,
// the whole group reads as NaN.
// Four bytes hold 8 elements: the even ones in the low half, the odd ones in the high half, each from the low bits on, so that one
// mask brings two neighbours into the two halves of a word.  (Codes in the last bits of a float that begins at a power of two, less that power: published for
// weights of 4 bits by Kim, Henry, Fahim and Awadalla, arXiv 2211.10017.  Layout, powers and scales are this form's.)
// A block is one head's tokens of one page: the codes of all tokens (dim / 2 bytes each), then their scales (dim / 16 each).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include "attention.cuh"
#include "common.cuh"

namespace stand {

constexpr int PK_GROUP = 16;
constexpr uint32_t PK_BAD = 0xF8;         // scales from here on are not finite
constexpr uint32_t PK_LAST = 0xF7;        // the largest scale: 61440
constexpr float PK_MOST = 7.0f * 61440.0f;

__device__ __forceinline__ float pk_scale(uint32_t byte) {
  return byte >= PK_BAD ? __uint_as_float(0x7FC00000u) : __half2float(__ushort_as_half((unsigned short)(byte << 7)));
}

// The scale of a group whose largest magnitude has these bits (of a 32-bit float without its sign; NaN and infinity are the
// largest): amax / 7 rounded up to 4 significant bits.  SHORT: amax has at most 11 of them, so it is either 7 s exactly or 2^-11 away
// from it, and the product with a constant just below 1 / 7 rounds up to the right one.  32 bits: a first guess, put right by the definition.
template <bool SHORT> __device__ __forceinline__ uint32_t pk_scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 0xFF;
  const float amax = __uint_as_float(amax_bits), t = amax * __uint_as_float(0x3E124924u);  // 1 / 7 (1 - 2^-24)
  uint32_t b;
  if (t >= 0x1p-14f) {
    b = (__float_as_uint(t) + 0xFFFFFu) >> 20;
    b -= 112u << 3;
    b = b > PK_LAST ? PK_LAST : b;
  } else {
    b = (uint32_t)ceilf(t * 0x1p17f);
  }
  if (SHORT) return b;
  if (b < PK_LAST && 7.0f * pk_scale(b) < amax) ++b;
  else if (b > 0 && 7.0f * pk_scale(b - 1) >= amax) --b;
  return b;
}

// The codes of 16 elements.  SHORT: an element has at most 11 significant bits and s has 4, so a quotient that is
// no tie is at least 2^-12 from one; the product with the reciprocal is off by 7 * 2^-23 at most, and rounding it to multiples
// of 2^-13 (the sum with 1536) makes a tie one again; the second sum rounds to whole numbers.  32 bits: the quotient rounded to 32
// bits, then to a whole number.  Four whole numbers + 8 are put together as digits of a float, which costs less than shifts and masks.
template <bool SHORT>
__device__ __forceinline__ uint2 pk_codes(float (&y)[PK_GROUP], uint32_t amax_bits, uint32_t byte) {
  if (byte == 0 || byte >= PK_BAD) return make_uint2(0x88888888u, 0x88888888u);
  if (amax_bits > __float_as_uint(PK_MOST)) {
#pragma unroll
    for (int i = 0; i < PK_GROUP; ++i) y[i] = fminf(fmaxf(y[i], -PK_MOST), PK_MOST);
  }
  const float s = pk_scale(byte), inv = __frcp_rn(s);
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (SHORT) e[i] = fmaf(y[8 * h + i], inv, 1536.0f) + (12582912.0f + 8.0f - 1536.0f);
      else e[i] = __fdiv_rn(y[8 * h + i], s) + (12582912.0f + 8.0f);
      e[i] -= 12582912.0f;
    }
    const float even = fmaf(fmaf(fmaf(e[6], 16.0f, e[4]), 16.0f, e[2]), 16.0f, e[0]), odd = fmaf(fmaf(fmaf(e[7], 16.0f, e[5]), 16.0f, e[3]), 16.0f, e[1]);
    w[h] = __byte_perm(__float_as_uint(even + 8388608.0f), __float_as_uint(odd + 8388608.0f), 0x5410);
  }
  return make_uint2(w[0], w[1]);
}

// A group as it lies: 16 elements of type T in words.  Its codes and its scale's byte.
template <typename T> struct PkGroup {
  static constexpr int WORDS = PK_GROUP * sizeof(T) / 4;
  alignas(16) uint32_t w[WORDS];

  __device__ __forceinline__ uint2 codes(uint32_t& byte) const {
    uint32_t most = 0;
    float y[PK_GROUP];
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < WORDS; ++i) most = __vmaxu2(most, w[i] & 0x7FFF7FFFu);
      most = max(most & 0xFFFFu, most >> 16);
      const unsigned short bits = (unsigned short)most;
      most = __float_as_uint(to_float(*reinterpret_cast<const T*>(&bits)));
#pragma unroll
      for (int i = 0; i < PK_GROUP; ++i) y[i] = to_float(reinterpret_cast<const T*>(w)[i]);
    } else {
#pragma unroll
      for (int i = 0; i < PK_GROUP; ++i) most = max(most, w[i] & 0x7FFFFFFFu), y[i] = __uint_as_float(w[i]);
    }
    byte = pk_scale_byte<sizeof(T) == 2>(most);
    return pk_codes<sizeof(T) == 2>(y, most, byte);
  }
};

__device__ __forceinline__ uint32_t pk_two(float f) {  // twice, as bfloat16
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(f));
  return r;
}
// A word of 8 codes as 8 values of the call's type (16 bytes), with the scale of its group.  bfloat16: a code n in bits 1 - 4 of a bfloat16
// that begins at 64 is 64 + n, and (64 + n) s - 72 s is exact, 72 s having at most 8 significant bits (9 x 15); an infinite scale gives infinity less infinity.
// Half: 1024 + n, less 1032, times s.  SHARED (half): an eighth of each value, 128 + n / 8 less 129, times s.  A half ends at 65,504 and k s at 8 * 61,440; k s / 8 is
// exact for every scale and code.
template <bool BF16, bool SHARED = false> struct PkScale {
  uint32_t s, c;
  __device__ __forceinline__ explicit PkScale(uint32_t byte) {
    if constexpr (BF16) {
      const float f = __half2float(__ushort_as_half((unsigned short)(byte << 7)));
      s = pk_two(f);
      c = pk_two(-72.0f * f);
    } else {
      s = (byte >= PK_BAD ? 0x7E00u : byte << 7) * 0x10001u;
      c = 0;
    }
  }
};
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) {  // one instruction
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
  return r;
}
template <bool BF16, bool SHARED> __device__ __forceinline__ uint4 pk_word(uint32_t w, const PkScale<BF16, SHARED>& p) {
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (BF16) {
      const uint32_t x = and_or(i == 0 ? w << 1 : w >> (4 * i - 1), 0x001E001Eu, 0x42804280u);
      asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i]) : "r"(x), "r"(p.s), "r"(p.c));
    } else {
      const uint32_t from = SHARED ? 0x58005800u : 0x64006400u, x = and_or(w >> (4 * i), 0x000F000Fu, from);
      uint32_t k;
      asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(k) : "r"(x), "r"(from + 0x00080008u));
      asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(v[i]) : "r"(k), "r"(p.s));
    }
  }
  return make_uint4(v[0], v[1], v[2], v[3]);
}

// 8 elements of a word as floats.
__device__ __forceinline__ void pk_values(uint32_t w, float s, float* v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (float)((int)(w >> (4 * i) & 15u) - 8) * s;
    v[2 * i + 1] = (float)((int)(w >> (4 * i + 16) & 15u) - 8) * s;
  }
}

}  // namespace stand
