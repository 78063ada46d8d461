// Attention of few rows (up to 16 per key head: single tokens, short chains) over a packed cache; bfloat16 and half, heads of
// 64 and 128.
//
// With few rows the text's bytes are all there is to it, so the kernel is made for the shortest way from them to the sums.  Codes
// become 16-bit values in the registers of a matrix instruction's first operand and nowhere else:
//   S^T [16 keys x 8 rows] = K Q^T: a lane has two keys and a quarter of the head size, as whole words of codes;
//   O^T [head size x 8 rows] += V^T P^T: a lane has four keys and an eighth of the head size; two keys' words are woven into pairs.
// Which element is which index of the summed dimension does not matter as long as both operands agree, so both read their words as
// they lie.  P goes from the first product's result to the second's operand by a transposition in registers.  So a warp needs no
// other: it takes 16 keys (one part of a page) of each tile of 64, has its own maximum, sum and O, and the four are joined at the end of a
// piece.  A fifth warp copies codes and scales of the tiles ahead into a ring, across the ends of pieces.
// The matrix instructions are the warp-wide ones: 16 x 8 is all that these rows fill, and tcgen05 would need the values in shared memory.
//
// Unpacking is most of the work, and its logic instructions, which issue every other cycle, are what counts: in half a word of 8 codes is
// one shift and four masks (a code n in the low bits of a half that begins at 1024 is 1024 + n, in the next four bits of one that begins at 64
// is 64 + n; bfloat16 has room for the first only, so it would take four shifts).  So cached keys and values enter the products as halves whatever the call's type, with scales s / 128, where all that the
// form can hold is exact in a half: s / 128 is at least 2^-24 and 72 s / 128 at most 34,560.  Rows of bfloat16 are brought into the range of a half by
// a power of two of their own; weights are halves with the lift that TA_LIFT describes.  The nodes' own keys and values are of the call's type, and so are the
// products with them.
//
// Measured, 32 / 8 heads of 128, bfloat16: 64 single tokens over 500 - 8,000 91 us = 3.4 TB/s (floor 48), 256 over 130 - 4,100 182 us, 64 sequences of 4 nodes
// 136 us, one token over 700 9.7 us; heads of 64 in half 60 us for 64 tokens.  Bound by issue: the logic unit at 45 % and the half products at 48 % share
// it, and with all pages in L2 the first case took 88 us where it took 94 without.  Products of two or three tiles interleaved, and sums beside the next scores: no change.
#pragma once
#include "async.cuh"
#include "attention_plain.cuh"
#include "attention_split.cuh"
#include "attention_tensor.cuh"
#include "launch.cuh"
#include "packed.cuh"

namespace stand {

constexpr int PR_WARPS = 4, PR_THREADS = (PR_WARPS + 1) * 32;
constexpr int PR_BOX = TA_KT / PR_WARPS;  // keys of a warp: 16, the least part of a page
static_assert(PR_BOX == 16, "a warp's keys are the rows of one product");

template <int DP, int NB> struct PrShape {
  // Per SM.  Measured with 3 / 4 (one block of rows): 256 single tokens over 130 - 4,100, 32 / 8 heads of 128: 187 / 197 us, one over 100,000: 51 / 55;
  // heads of 64, 64 tokens over 500 - 8,000: 95 / 84.
  static constexpr int CTAS = NB == 1 ? (DP == 64 ? 4 : 3) : (DP == 64 ? 3 : 2);
  static constexpr int CODES = DP / 2, SCALES = DP / 16;     // bytes of a row
  static constexpr int HALF = TA_KT * (CODES + SCALES);      // bytes of a tile's keys, then of its values
  static constexpr int SLOT = 2 * HALF;
  static constexpr int STAGES = DP == 128 ? 6 : 8;
  static constexpr int ROWS = 8 * NB;
  static constexpr int TREE = 2 * 16 * DP * 2;               // the tree's keys and values, up to 16 nodes
  static constexpr int PITCH = DP + 4;
  static constexpr int X = PR_WARPS * ROWS * PITCH * 4;      // exchange between the warps, in the same place once those are done with
  static constexpr int SMEM = STAGES * SLOT + X;
  static_assert(X >= TREE + 16 * ROWS * 4 + ROWS * DP * 2, "the tree, its weights and rows");
  static_assert(CTAS * (SMEM + 3 * 1024) <= 228 * 1024, "shared memory");
};

struct PrParams {
  TaSplit s;
  unsigned wait_limit;
};

// ---- unpacking to pairs of halves ------------------------------------------------------------
constexpr float PK_SHARE = 128.0f;  // values come out as this part of themselves
// Scales (/ 128) of two elements, of one key or of two, from two bytes in the halves of a word.
struct PkPair {
  uint32_t s, c, z;  // the scale; -72 times it; 0, or NaN where it is not finite
  __device__ __forceinline__ explicit PkPair(uint32_t bytes) {
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(s) : "r"(bytes << 7), "r"(0x20002000u));
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(c) : "r"(s), "r"(0xD480D480u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(z) : "r"(s), "r"(0x54805480u), "r"(c));
  }
};
// The codes of a word as pairs of values: 8 neighbours, or (woven) 4 elements of two keys.
__device__ __forceinline__ void pk_pairs(uint32_t w, const PkPair& p, uint32_t (&v)[4]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t x = h ? w >> 8 : w, lo = and_or(x, 0x000F000Fu, 0x64006400u), hi = and_or(x, 0x00F000F0u, 0x54005400u);  // 1024 + n, 64 + n
    uint32_t k;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(k) : "r"(lo), "r"(0x64086408u));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(v[2 * h]) : "r"(k), "r"(p.s), "r"(p.z));
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(v[2 * h + 1]) : "r"(hi), "r"(p.s), "r"(p.c));
  }
}

template <bool BF16> __device__ __forceinline__ void mma_16x8(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16x8_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {  // halves; d = rather than +=
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// ---- the kernel -----------------------------------------------------------------------------
template <int DP, int NB, bool BF16>
__global__ void __launch_bounds__(PR_THREADS, PrShape<DP, NB>::CTAS) packed_rows_kernel(const __grid_constant__ PrParams p) {
  using Sh = PrShape<DP, NB>;
  using T = typename std::conditional<BF16, __nv_bfloat16, __half>::type;
  constexpr int STAGES = Sh::STAGES, KD = DP / 4, VD = DP / 8;  // elements of a lane: of a key, of a value
  constexpr int STEPS = DP / 16;                                // products per 16 keys, both times
  extern __shared__ __align__(128) char pr_smem[];
  struct Shared {
    uint64_t full[STAGES], empty[STAGES];
    TaRange<PR_THREADS> range;
    float2 ml[PR_WARPS][Sh::ROWS];
    int abort;
  };
  __shared__ Shared sh;
  char* const tree_k = pr_smem + STAGES * Sh::SLOT;
  char* const tree_v = tree_k + Sh::TREE / 2;
  char* const tree_q = tree_k + Sh::TREE + 16 * Sh::ROWS * 4;
  float* const exchange = reinterpret_cast<float*>(tree_k);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_addr(&sh.full[i]), 32);
      mbar_init(smem_addr(&sh.empty[i]), PR_WARPS);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.abort = p.wait_limit == 0;  // no waiting allowed
  }
  pdl_trigger();
  pdl_wait();
  TaWalk walk;
  ta_begin<PR_THREADS>(p.s, walk, sh.range, [] {}, [] {});
  volatile int* abort_flag = &sh.abort;
  const unsigned limit = p.wait_limit;
  auto wait_warp = [&](uint32_t bar, uint32_t parity) {
    if (__all_sync(FULL, mbar_try_wait(bar, parity))) return true;
    return ta_wait_on(bar, parity, abort_flag, limit);
  };
  const AttnParams& a = p.s.a;
  bool ok = *abort_flag == 0;

  if (warp == PR_WARPS) {
    // ---- copies ------------------------------------------------------------------------------
    const uint32_t ring = smem_addr(pr_smem);
    uint32_t stage = 0, phase = 1;
    TaSeg s;
    TaNote note(walk);
    PkCopies copies;
    while (walk.next(p.s, s)) {
      note.piece(walk, s, sh.range.total, sh.range.groups, blockIdx.x);
      if (!ok) continue;  // gave up: only the record is still to be found
      const int end = s.end < s.p_tiles ? s.end : s.p_tiles;
      if (s.begin >= end) continue;
      copies.begin(a, s, lane);
      for (int tile = s.begin; tile < end; ++tile) {
        if (!(ok = wait_warp(smem_addr(&sh.empty[stage]), phase))) break;
        copies.tile<DP>(a, DP, lane, ring + stage * Sh::SLOT, Sh::HALF, smem_addr(&sh.full[stage]));
        if (++stage == STAGES) stage = 0, phase ^= 1u;
      }
    }
    if (lane == 0) p.s.records[blockIdx.x] = note.r;
    cp_wait<0>();
    return;
  }

  // ---- the warps that compute ---------------------------------------------------------------
  const int g = lane >> 2, t = lane & 3;
  const int key0 = g ^ (g >> 1 & 1);  // the product's key g is this one of the box: neighbouring lanes' values then lie in other banks
  auto sync_rows = [] { asm volatile("bar.sync 1, %0;" ::"n"(PR_WARPS * 32) : "memory"); };
  uint32_t stage = 0, phase = 0;
  TaSeg s;
  while (walk.next(p.s, s)) {
    const bool tree = warp == 0 && s.end > s.p_tiles && s.begin < s.end;  // the first warp takes the nodes as well
    // rows: queries as the second operand (row g), results by columns (rows 2 t and 2 t + 1)
    uint32_t q[NB][STEPS][2];
    float factor[NB][2];  // from a product to the logarithm of a weight
    bool live[NB][2];
    int node[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = n * 8 + g, u = r / a.group;
      const T* src = reinterpret_cast<const T*>(a.q) + s.b * a.q_stride[0] + u * a.q_stride[1] + (s.g * a.group + r - u * a.group) * a.q_stride[2] + t * KD;
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < KD / 8; ++i) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < p.s.rows) v = *reinterpret_cast<const uint4*>(src + 8 * i);
        if (tree) *reinterpret_cast<uint4*>(tree_q + (r * DP + t * KD + 8 * i) * 2) = v;
        q[n][2 * i][0] = v.x, q[n][2 * i][1] = v.y, q[n][2 * i + 1][0] = v.z, q[n][2 * i + 1][1] = v.w;
      }
      float share = 1.0f;
      if constexpr (BF16) {
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) most = max(most, max(q[n][i][e] & 0x7F80u, q[n][i][e] >> 16 & 0x7F80u));
#pragma unroll
        for (int d = 1; d < 4; d *= 2) most = max(most, __shfl_xor_sync(FULL, most, d));
        // the row's largest power of two becomes 2^14: what is below 2^-29 of it loses bits, none is lost above 2^-38.  (Rows below 2^-112 are brought up by
        // 2^126, the most that a float has together with its inverse; what is least in the type then is 2^-7.)
        int up = 14 + 127 - (int)(most >> 7);
        up = most >= 0x7F80u ? 0 : (up > 126 ? 126 : up);
        const float by = __int_as_float((127 + up) << 23);
        share = __int_as_float((127 - up) << 23);
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            q[n][i][e] = ta_pack<false>(__uint_as_float(q[n][i][e] << 16) * by, __uint_as_float(q[n][i][e] & 0xFFFF0000u) * by);
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = n * 8 + 2 * t + c;
        // (not zero, which would make NaN of the masked scores' -inf; 2^-126 makes nothing of any product here as well)
        factor[n][c] = fmaxf(__shfl_sync(FULL, share, (2 * t + c) * 4) * PK_SHARE * a.scale2, 0x1p-126f);
        node[n][c] = row / a.group;
        live[n][c] = row < p.s.rows && !(a.tree && a.tree[(long long)s.b * a.N + node[n][c]] < 0);
      }
    }
    if (tree) {  // on their way while the text is read
      constexpr int PIECES = DP / 8;
      for (int i = lane; i < 2 * 16 * PIECES; i += 32) {
        const int row = i / PIECES, at = i - row * PIECES, v = row & 15;
        const bool is_v = row >= 16;
        char* dst = (is_v ? tree_v : tree_k) + (v * PIECES + at) * 16;
        const long long* stride = is_v ? a.v_stride : a.k_stride;
        if (v < a.N) {
          const T* src = reinterpret_cast<const T*>(is_v ? a.v : a.k) + s.b * stride[0] + v * stride[1] + s.g * stride[2] + at * 8;
          cp_async16(smem_addr(dst), src);
        } else {
          *reinterpret_cast<uint4*>(dst) = make_uint4(0, 0, 0, 0);
        }
      }
      cp_commit();
    }
    float o[NB][STEPS][4], m[NB][2], l[NB][2];
    float base[NB][2], limit_x[NB][2];  // by m: what is added to a logarithm; the product above which m is raised
#pragma unroll
    for (int n = 0; n < NB; ++n) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][i][e] = 0.0f;
#pragma unroll
      for (int c = 0; c < 2; ++c) m[n][c] = -INFINITY, l[n][c] = 0.0f, base[n][c] = TA_LIFT<false>, limit_x[n][c] = live[n][c] ? -INFINITY : INFINITY;
    }

    // Products x of 16 keys (masked ones -inf), times `by` -> weights e, 2^lift of them, and w, the second product's operand: with the maximum as
    // it is; true: some row's wants to be raised first.
    auto guess = [&](const float (&x)[NB][4], const float (&by)[NB][2], float (&e)[NB][4], uint32_t (&w)[NB][2], auto of_text) {
      constexpr bool TEXT = decltype(of_text)::value;
      bool up = false;
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          up = up || fmaxf(x[n][c], x[n][c + 2]) > limit_x[n][c];
          e[n][c] = ta_ex2(fmaf(x[n][c], by[n][c], base[n][c]));
          e[n][c + 2] = ta_ex2(fmaf(x[n][c + 2], by[n][c], base[n][c]));
        }
        w[n][0] = transpose_8x8(ta_pack<TEXT ? false : BF16>(e[n][0], e[n][1]));
        w[n][1] = transpose_8x8(ta_pack<TEXT ? false : BF16>(e[n][2], e[n][3]));
      }
      return up;
    };
    // The rest of it.  As in the other kernels the maximum is raised when scores pass it by a good deal.
    auto settle = [&](const float (&x)[NB][4], const float (&by)[NB][2], float (&e)[NB][4], uint32_t (&w)[NB][2], bool up, auto of_text) {
      constexpr bool TEXT = decltype(of_text)::value;
      constexpr float LIFT = TA_LIFT<TEXT ? false : BF16>;
      if (__any_sync(FULL, up)) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = fmaxf(x[n][c], x[n][c + 2]);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(FULL, top, d));
            const float raised = fmaxf(m[n][c], top * by[n][c]), keep = raised == -INFINITY ? 1.0f : ta_ex2(m[n][c] - raised);
            m[n][c] = raised;
            l[n][c] *= keep;
            base[n][c] = LIFT - (raised == -INFINITY ? 0.0f : raised);
            if (live[n][c]) limit_x[n][c] = (raised + TA_SLACK) / by[n][c];
#pragma unroll
            for (int i = 0; i < STEPS; ++i) o[n][i][c] *= keep, o[n][i][c + 2] *= keep;
          }
        guess(x, by, e, w, of_text);
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) l[n][c] += e[n][c] + e[n][c + 2];
    };

    // Products of the rows with this warp's 16 keys of a tile.
    auto products = [&](const char* tile, float (&x)[NB][4]) {
      const char *codes = tile + warp * 9 * DP + t * (KD / 2), *scales = tile + warp * 9 * DP + 8 * DP + t * (KD / 16);
      // keys key0 and key0 + 8: words of 8 elements, two products each
      uint32_t k[2][KD / 8], scale[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if constexpr (KD == 32) {
          const uint4 v = *reinterpret_cast<const uint4*>(codes + (key0 + 8 * h) * Sh::CODES);
          k[h][0] = v.x, k[h][1] = v.y, k[h][2] = v.z, k[h][3] = v.w;
          scale[h] = *reinterpret_cast<const unsigned short*>(scales + (key0 + 8 * h) * Sh::SCALES);
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(codes + (key0 + 8 * h) * Sh::CODES);
          k[h][0] = v.x, k[h][1] = v.y;
          scale[h] = *reinterpret_cast<const unsigned char*>(scales + (key0 + 8 * h) * Sh::SCALES);
        }
      }
#pragma unroll
      for (int i = 0; i < KD / 8; i += 2) {
        const PkPair s0(__byte_perm(scale[0], 0, i ? 0x4141 : 0x4040)), s1(__byte_perm(scale[1], 0, i ? 0x4141 : 0x4040));
#pragma unroll
        for (int j = i; j < i + 2; ++j) {
          uint32_t lo[4], hi[4];
          pk_pairs(k[0][j], s0, lo);
          pk_pairs(k[1][j], s1, hi);
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            if (j == 0) mma_16x8_first(x[n], lo[0], hi[0], lo[1], hi[1], q[n][0][0], q[n][0][1]);
            else mma_16x8<false>(x[n], lo[0], hi[0], lo[1], hi[1], q[n][2 * j][0], q[n][2 * j][1]);
            mma_16x8<false>(x[n], lo[2], hi[2], lo[3], hi[3], q[n][2 * j + 1][0], q[n][2 * j + 1][1]);
          }
        }
      }
    };
    // O += V^T P^T of this warp's keys, `left` of them there.  Keys (2 t, 2 t + 1) and the same + 8 of the product, in the order of key0.
    auto sums = [&](const char* tile, const uint32_t (&w)[NB][2], int left, auto whole) {
      constexpr bool WHOLE = decltype(whole)::value;
      const char *codes = tile + Sh::HALF + warp * 9 * DP + g * (VD / 2), *scales = tile + Sh::HALF + warp * 9 * DP + 8 * DP + g * VD / 16;
      uint32_t v[2][2][VD / 8], sv[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int key = 2 * t + (e ^ (t & 1)) + 8 * h;
          sv[h][e] = *reinterpret_cast<const unsigned char*>(scales + key * Sh::SCALES);
          if (!WHOLE && key >= left) sv[h][e] = 0;  // past the end there may be anything
          if constexpr (VD == 16) {
            const uint2 c = *reinterpret_cast<const uint2*>(codes + key * Sh::CODES);
            v[h][e][0] = c.x, v[h][e][1] = c.y;
          } else {
            v[h][e][0] = *reinterpret_cast<const uint32_t*>(codes + key * Sh::CODES);
          }
        }
      const PkPair s0(__byte_perm(sv[0][0], sv[0][1], 0x5410)), s1(__byte_perm(sv[1][0], sv[1][1], 0x5410));
#pragma unroll
      for (int i = 0; i < VD / 8; ++i) {
        uint32_t a0[4], a1[4], a2[4], a3[4];  // even and odd elements of the first keys, of the second
        pk_pairs(__byte_perm(v[0][0][i], v[0][1][i], 0x5410), s0, a0);
        pk_pairs(__byte_perm(v[0][0][i], v[0][1][i], 0x7632), s0, a1);
        pk_pairs(__byte_perm(v[1][0][i], v[1][1][i], 0x5410), s1, a2);
        pk_pairs(__byte_perm(v[1][0][i], v[1][1][i], 0x7632), s1, a3);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int n = 0; n < NB; ++n) mma_16x8<false>(o[n][4 * i + c], a0[c], a1[c], a2[c], a3[c], w[n][0], w[n][1]);
      }
    };

    const int cached = s.end < s.p_tiles ? s.end : s.p_tiles;
    float x[NB][4], e[NB][4];
    uint32_t w[NB][2];
    constexpr std::true_type TEXT{}, WHOLE{};
    for (int j = s.begin; j < cached && ok; ++j) {
      if (!(ok = wait_warp(smem_addr(&sh.full[stage]), phase))) break;
      const int left = s.len - j * TA_KT - warp * PR_BOX;  // of the text from this warp's keys on
      const char* tile = pr_smem + stage * Sh::SLOT;
      if (left >= PR_BOX) {
        products(tile, x);
        settle(x, factor, e, w, guess(x, factor, e, w, TEXT), TEXT);
        sums(tile, w, left, WHOLE);
      } else if (left > 0) {
        products(tile, x);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (key0 + (i >> 1) * 8 >= left) x[n][i] = -INFINITY;
        settle(x, factor, e, w, guess(x, factor, e, w, TEXT), TEXT);
        sums(tile, w, left, std::false_type{});
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_addr(&sh.empty[stage]));
      if (++stage == STAGES) stage = 0, phase ^= 1u;
    }

    // from here on as the nodes' products want it: values whole, weights of the call's type
    constexpr float TO = BF16 ? 0x1p-15f : 1.0f;  // 2^(TA_LIFT<BF16> - TA_LIFT<false>)
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        l[n][c] *= TO;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) o[n][i][c] *= PK_SHARE * TO, o[n][i][c + 2] *= PK_SHARE * TO;
      }
    if (tree) {
      cp_wait<0>();
      __syncwarp();
      uint32_t seen[NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = 0.0f;
#pragma unroll
        for (int c = 0; c < 2; ++c) seen[n][c] = live[n][c] ? attn_nodes_seen(a, s.b, node[n][c], 0) : 0u;
      }
#pragma unroll
      for (int i = 0; i < KD / 8; ++i) {
        const uint4 lo = *reinterpret_cast<const uint4*>(tree_k + key0 * DP * 2 + (t * KD + 8 * i) * 2);
        const uint4 hi = *reinterpret_cast<const uint4*>(tree_k + (key0 + 8) * DP * 2 + (t * KD + 8 * i) * 2);
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          const uint4 row = *reinterpret_cast<const uint4*>(tree_q + ((n * 8 + g) * DP + t * KD + 8 * i) * 2);
          mma_16x8<BF16>(x[n], lo.x, hi.x, lo.y, hi.y, row.x, row.y);
          mma_16x8<BF16>(x[n], lo.z, hi.z, lo.w, hi.w, row.z, row.w);
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[n][e] = seen[n][e & 1] >> (key0 + (e >> 1) * 8) & 1u ? x[n][e] : -INFINITY;
      float by[NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          by[n][c] = a.scale2;
          base[n][c] = TA_LIFT<BF16> - (m[n][c] == -INFINITY ? 0.0f : m[n][c]);
          limit_x[n][c] = live[n][c] ? (m[n][c] + TA_SLACK) / a.scale2 : INFINITY;
        }
      settle(x, by, e, w, guess(x, by, e, w, std::false_type{}), std::false_type{});
      uint32_t v[2][2][VD / 2];  // pairs of neighbouring elements
      constexpr uint32_t EXP = BF16 ? 0x7F80u : 0x7C00u;
      bool odd = false;  // a value that is not finite: some rows may see it, others not
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < VD / 8; ++i) {
            const int key = 2 * t + (e ^ (t & 1)) + 8 * h;
            const uint4 c = *reinterpret_cast<const uint4*>(tree_v + key * DP * 2 + (g * VD + 8 * i) * 2);
            v[h][e][4 * i] = c.x, v[h][e][4 * i + 1] = c.y, v[h][e][4 * i + 2] = c.z, v[h][e][4 * i + 3] = c.w;
#pragma unroll
            for (int k = 0; k < 4; ++k) odd = odd || (v[h][e][4 * i + k] & EXP) == EXP || (v[h][e][4 * i + k] & EXP << 16) == EXP << 16;
          }
      if (!__any_sync(FULL, odd)) {
#pragma unroll
        for (int i = 0; i < VD / 2; ++i) {
          const uint32_t a0 = __byte_perm(v[0][0][i], v[0][1][i], 0x5410), a1 = __byte_perm(v[0][0][i], v[0][1][i], 0x7632);
          const uint32_t a2 = __byte_perm(v[1][0][i], v[1][1][i], 0x5410), a3 = __byte_perm(v[1][0][i], v[1][1][i], 0x7632);
#pragma unroll
          for (int n = 0; n < NB; ++n) mma_16x8<BF16>(o[n][i], a0, a1, a2, a3, w[n][0], w[n][1]);
        }
      } else {  // node by node, only what a row sees; a value that is not finite counts whatever its weight
        float* weights = reinterpret_cast<float*>(tree_k + Sh::TREE);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) weights[(key0 + (i >> 1) * 8) * Sh::ROWS + n * 8 + 2 * t + (i & 1)] = e[n][i];
        __syncwarp();
#pragma unroll 1
        for (int key = 0; key < a.N; ++key) {
          const T* row = reinterpret_cast<const T*>(tree_v + key * DP * 2) + g * VD;
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              if (seen[n][c] >> key & 1u) {
                const float f = weights[key * Sh::ROWS + n * 8 + 2 * t + c];
#pragma unroll
                for (int i = 0; i < STEPS; ++i) {
                  const float v0 = to_float(row[2 * i]), v1 = to_float(row[2 * i + 1]);
                  o[n][i][c] = isfinite(v0) ? fmaf(f, v0, o[n][i][c]) : o[n][i][c] + v0;
                  o[n][i][c + 2] = isfinite(v1) ? fmaf(f, v1, o[n][i][c + 2]) : o[n][i][c + 2] + v1;
                }
              }
        }
        __syncwarp();
      }
    }

    // ---- the warps' results joined ------------------------------------------------------------
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[n][c] += __shfl_xor_sync(FULL, l[n][c], d);
        m[n][c] -= TA_LIFT<BF16>;                    // what l and o are relative to
        if (*abort_flag) l[n][c] = NAN;              // a wait ran out: nothing is to be trusted
        if (!live[n][c]) m[n][c] = -INFINITY, l[n][c] = 0.0f;
        if (g == 0) sh.ml[warp][n * 8 + 2 * t + c] = make_float2(m[n][c], l[n][c]);
      }
    sync_rows();
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = n * 8 + 2 * t + c;
        float top = sh.ml[0][row].x;
#pragma unroll
        for (int k = 1; k < PR_WARPS; ++k) top = fmaxf(top, sh.ml[k][row].x);
        // a weight too small for its type may still meet an infinity
        const float f = live[n][c] && l[n][c] != 0.0f ? fmaxf(ta_ex2(m[n][c] - (top == -INFINITY ? 0.0f : top)), 1.2e-38f) : 0.0f;
        float* to = exchange + (warp * Sh::ROWS + row) * Sh::PITCH + g * VD;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          float2 pair = make_float2(0.0f, 0.0f);
          if (f != 0.0f) pair = make_float2(o[n][i][c] * f, o[n][i][c + 2] * f);
          *reinterpret_cast<float2*>(to + 2 * i) = pair;
        }
      }
    sync_rows();
    constexpr int QUADS = DP / 4;
    for (int i = tid; i < p.s.rows * QUADS; i += PR_WARPS * 32) {
      const int row = i / QUADS, col = (i - row * QUADS) * 4;
      float top = sh.ml[0][row].x, total = 0.0f;
#pragma unroll
      for (int k = 1; k < PR_WARPS; ++k) top = fmaxf(top, sh.ml[k][row].x);
      const float base = top == -INFINITY ? 0.0f : top;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < PR_WARPS; ++k) {
        const float2 v = sh.ml[k][row];
        total += v.y * ta_ex2(v.x - base);
        const float4 f = *reinterpret_cast<const float4*>(exchange + (k * Sh::ROWS + row) * Sh::PITCH + col);
        sum.x += f.x, sum.y += f.y, sum.z += f.z, sum.w += f.w;
      }
      const int u = row / a.group, h = s.g * a.group + row - u * a.group;
      const long long out_row = ((long long)s.b * a.N + u) * a.heads_q + h, at = ta_part_row(p.s, s, row);
      const bool empty = total == 0.0f;
      if (!s.whole) {
        *reinterpret_cast<float4*>(p.s.part_o + at * DP + col) = sum;
        if (col == 0) p.s.part_ml[at] = make_float2(empty ? -INFINITY : top, total);
      } else {
        const float inv = empty ? 0.0f : 1.0f / total;
        *reinterpret_cast<uint2*>(a.out + 2 * (out_row * DP + col)) =
            empty ? make_uint2(0, 0) : make_uint2(ta_pack<BF16>(sum.x * inv, sum.y * inv), ta_pack<BF16>(sum.z * inv, sum.w * inv));
        if (a.lse && col == 0) a.lse[out_row] = empty ? -INFINITY : 0.6931471805599453f * (top + log2f(total));
      }
    }
    sync_rows();  // all have read
  }
}

// ---- launch --------------------------------------------------------------------------------
constexpr int PR_ROWS_MOST = 16;
inline int rows_ctas(int rows, int dim) { return tensor_dim(dim) == 64 ? (rows <= 8 ? 4 : 3) : (rows <= 8 ? 3 : 2); }

// Rows of 16-byte pieces; whole heads of 64 or 128.
inline bool rows_takes(const AttnParams& a, int dtype) {
  if (dtype == STAND_DTYPE_F32 || (a.dim != 64 && a.dim != 128) || (long long)a.N * a.group > PR_ROWS_MOST) return false;
  uintptr_t bits = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out;
  for (int i = 0; i < 3; ++i) bits |= (uintptr_t)((a.q_stride[i] | a.k_stride[i] | a.v_stride[i]) * 2);
  return (bits & 15) == 0;
}

template <int DP, int NB, bool BF16> int launch_packed_rows(const AttnParams& a, void* scratch, int sms, unsigned wait_limit, cudaStream_t st) {
  using Sh = PrShape<DP, NB>;
  PrParams p;
  // A piece's beginning and join as 8 tiles.  As 4 / 6 / 8 / 12: 64 sequences of 4 nodes over 500 - 8,000, 32 / 8 heads of 128: 155 / 144 / 136 / 137 us;
  // 64 single tokens 93 / 93 / 94 / 98; 256 over 130 - 4,100 186 / 183 / 186 / 192.
  ta_split(p.s, a, a.N * a.group, DP, sms, Sh::CTAS, 8, scratch);
  p.wait_limit = wait_limit;
  static SmemLimit limit;
  int rc = limit.raise(packed_rows_kernel<DP, NB, BF16>, Sh::SMEM);
  if (rc) return rc;
  rc = launch_dependent(packed_rows_kernel<DP, NB, BF16>, dim3((unsigned)p.s.groups), PR_THREADS, st, p, Sh::SMEM);
  if (rc) return rc;
  return launch_join<DP, typename std::conditional<BF16, __nv_bfloat16, __half>::type>(p.s, st);
}
template <int DP, bool BF16> int launch_packed_rows(const AttnParams& a, void* scratch, int sms, unsigned wait_limit, cudaStream_t st) {
  if (a.N * a.group <= 8) return launch_packed_rows<DP, 1, BF16>(a, scratch, sms, wait_limit, st);
  return launch_packed_rows<DP, 2, BF16>(a, scratch, sms, wait_limit, st);
}

}  // namespace stand
