// Tree attention on the tensor cores (tcgen05, sm_100a): bfloat16 and half, head sizes that are a multiple of 8, 16-byte
// aligned rows, up to 128 query heads per key head.
//
// A block (CTA) of seven warps works on up to 128 rows of one (sequence, key head) pair and walks over its keys in tiles of
// 64:
//   warps 4 and 6  copy tiles of keys and of values from the pages (and from the tree's own) with TMA, each into a ring,
//   warp 5  issues the matrix products S = Q K^T and O += P V, and copies the rows Q,
//   warps 0-3  own one row per thread: read S, keep the running maximum and sum, write P, finally write O / l.
// S and O live in tensor memory (a row is a lane).  P, in 16 bits, takes the place of S as the first operand of the second
// product.  There are two places for S, so the scores of the next tile are computed while the softmax works on this
// one, and the softmax waits for nothing but its own arithmetic; O is only touched by it when the maximum has risen a
// good deal.  Two CTAs share an SM (256 of the 512 columns of tensor memory and half of the shared memory each; head
// size 256: one CTA).
//
// Head sizes up to 64 with at most 32 (64) rows: the four (two) parts of the lanes hold the same rows, each takes a
// quarter (half) of a tile's keys, has its own maximum, sum and O, and they are joined at the end.  The product computes 128
// rows anyway; the exponentials of a tile then take all four warps instead of one.
//
// The keys of all pairs, laid end to end in tiles, are cut into as many equal ranges as there are CTAs (or groups of
// CTAs: the row tiles of a pair with more than 128 rows go to neighbours that walk over the same keys at the same time,
// so that those come from memory once and from L2 after that).  A range may begin and end inside a pair: such pieces
// leave (m, l, O) in scratch and a second, small kernel joins them.  So long texts with few rows fill the GPU, and so do
// batches of ragged lengths, without the host knowing a length.
//
// Measured (keys and values read once, over the time): 256 sequences x 24 nodes, texts of 130 - 4,100, 32 / 8 heads of 128:
// 390 - 404 us in short bursts = 5.8 - 6.0 TB/s (0.89 - 0.92 of the copy bandwidth), 460 - 480 us in loops of seconds, where the
// board's power limit holds the clock at 1.24 - 1.4 GHz; 64 nodes over 32,001 tokens, 28 / 4 heads of 128: 52 us = 0.57 PFLOP/s;
// one token over 700: 11 us.  64 x 24 nodes, 130 - 4,100 tokens, 16 / 4 heads of 256: 117 us = 5.0 TB/s (one CTA per SM: nothing
// overlaps the chain named below).  Prompts without a cache, 32 / 8 heads of 128: 4 x 4,096 rows 1,360 us, 1 x 16,384 4,950 us = 0.40 -
// 0.44 PFLOP/s of the visible half.  In the first case no unit is near its limit (tensor pipe 35 %, exponentials 27 %, issue 29 %, memory 82 % of
// a copy): what bounds a tile is the chain scores - maximum - exponentials - product, about 2,200 cycles, which two CTAs overlap.
//
// PACKED: the cache is in 4 bits.  Ten warps: 0-3 as above; 4, 5 make a tile's keys and 6, 7 its values from codes, each half a tile, in the places
// that TMA fills otherwise; 8 issues the products; 9 copies codes and scales, tiles ahead, into stages of 9 bytes for 16 elements (and has TMA fetch the
// tree's own).  What the unpacking warps write and the products read meets at the same barriers, after a fence between the two kinds of access.  A key's values
// (in half: an eighth of them) are exact in 16 bits, so the products are those of the definition.
// Measured: 256 x 24 nodes as above: 380 us in short bursts, 438 in loops of seconds (floor 128: products; with a cache of 16 bits 400 and 469), in half 388 - 396; 64 nodes over
// 32,001: 61 us (floor 18; 16 bits 52); 16 x 32 nodes, 16 / 16 heads of 64, half, 1 - 8,190: 63 us (16 bits 59); 64 x 24 of 16 / 4 heads of 256: 129 us (118).  Memory is no longer the
// bound (0.3 of a copy), the chain of a tile is, of 2,100 - 2,600 cycles with 96 registers a thread: tensor pipe 31 %, exponentials 24 %, logic unit 41 %,
// issue 50 %, shared memory 57 %.  Codes read by the unpacking warps straight from memory took 664 us, bulk copies by one lane 387 (950 - 1,480 cycles
// a tile to issue them); weights by the maximum of the tile before, in one pass over the scores, 495; scores kept in registers between the two passes 452.
#pragma once
#include <cuda.h>

#include "async.cuh"
#include "attention_split.cuh"
#include "launch.cuh"
#include "packed.cuh"

namespace stand {

constexpr int TA_ROWS = 128;              // rows of a CTA: lanes of tensor memory
template <bool PACKED> constexpr int TA_THREADS_OF = PACKED ? 320 : 224;
constexpr float TA_SLACK = 8.0f;          // the maximum is raised only when scores pass it by 2^8 (below)
// Weights of the second product are rounded to the input's type, since both operands of a 16-bit product have one type: each
// is off by 2^-8 (bfloat16) or 2^-11 (half) of itself at most, independently, which is what rounding the result costs anyway;
// their sum l is taken before the rounding, in fp32.  Half has few exponents: there weights are 2^7 times larger (at most 2^15,
// with the slack), as are l and o, so that those down to 2^-21 of the largest keep all bits and none above 2^-32 is lost
// (unlifted, 40,000 keys of 2^-26 beside a dominant one were lost from o while they stayed in l).  Bfloat16 has the exponents of
// fp32 and values as large: there the slack is taken off, so that no weight is above 1 and o passes fp32's range only
// where the plain sum of the values does.
template <bool BF16> constexpr float TA_LIFT = BF16 ? -TA_SLACK : 7.0f;
constexpr int TA_XCOLS = 16;              // columns of O that the parts exchange at a time

template <int DP, int C, bool PACKED> struct TaShape {
  static constexpr int CTAS = DP == 256 ? 1 : 2;              // per SM
  static constexpr int SLOT = TA_KT * DP * 2;                 // bytes of a tile of keys or values
  static constexpr int K_SLOTS = PACKED ? (DP == 64 ? 3 : 1) : (DP == 64 ? (C > 1 ? 5 : 6) : 2);
  static constexpr int V_SLOTS = PACKED ? (DP == 64 ? 3 : 2) : (DP == 64 ? K_SLOTS : 3);
  static constexpr int SLOTS = K_SLOTS + V_SLOTS;
  static constexpr int Q = TA_ROWS * DP * 2;
  static constexpr int COL_O = 0, COL_S = DP;                 // two places for S
  static constexpr int COLS = DP == 256 ? 512 : 256;          // tensor memory columns allocated
  static constexpr int X = C > 1 ? TA_ROWS * (TA_XCOLS + 1) * 4 : 0;  // exchange between the parts
  static constexpr int STAGES = PACKED ? (DP == 64 ? 4 : 3) : 0;      // of packed tiles
  static constexpr int STAGE_HALF = TA_KT * (DP / 2 + DP / 16);       // keys, then values
  static constexpr int STAGE = 2 * STAGE_HALF;
  static constexpr int SHARED = C > 1 || PACKED ? 1536 : 512; // barriers and the like
  static constexpr int SMEM = Q + SLOTS * SLOT + X + STAGES * STAGE + SHARED;
  static_assert(C == 1 || DP == 64, "parts of the lanes: small heads only");
  static_assert(COL_S + 2 * TA_KT <= COLS, "tensor memory");
  static_assert(CTAS * (SMEM + 1024) <= 228 * 1024, "shared memory");
};

struct alignas(64) TaParams {
  CUtensorMap cache_k, cache_v, tree_k, tree_v, q;
  TaSplit s;
  int box_rows;       // rows of a page that one copy takes
  unsigned wait_limit;
};

// ---- tcgen05 ----------------------------------------------------------------------
__device__ __forceinline__ void tc_alloc(uint32_t smem_dst, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tc_dealloc(uint32_t tmem, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t elect_one() {  // 1 in one lane of the (whole) warp
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
// The whole warp calls these (and the copies below), the elected lane acts: the operands then sit in uniform registers, where the unit wants
// them.  (In a branch of one lane each product took 60 cycles to issue, most of it moving five operands there.)
__device__ __forceinline__ void tc_commit(uint32_t bar, uint32_t elected) {
  asm volatile(
      "{\n\t.reg .pred e;\n\tsetp.ne.u32 e, %1, 0;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(elected)
      : "memory");
}
// D (tensor memory, fp32) = or += A (tensor memory, 16 bit) * B (shared memory).  The descriptor of B in two words: only
// the low one changes, by an addition; one thread issues all products, so each instruction that it spends counts.
__device__ __forceinline__ void tc_mma(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, uint32_t accumulate,
                                       uint32_t elected) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 b;\n\tmov.b64 b, {%2, %3};\n\tsetp.ne.u32 p, %5, 0;\n\tsetp.ne.u32 e, %6, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n\t}" ::"r"(d), "r"(a), "r"(b_lo), "r"(b_hi), "r"(idesc),
      "r"(accumulate), "r"(elected)
      : "memory");
}
// The same with A in shared memory.
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate,
                                          uint32_t elected) {
  asm volatile(
      "{\n\t.reg .pred p, e;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %3};\n\tmov.b64 b, {%2, %3};\n\tsetp.ne.u32 p, %5, 0;\n\t"
      "setp.ne.u32 e, %6, 0;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi),
      "r"(idesc), "r"(accumulate), "r"(elected)
      : "memory");
}
// 16 or 32 columns of this warp's 32 lanes: one row per thread
__device__ __forceinline__ void tc_ld16(uint32_t* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t addr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]),
      "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]),
        "=r"(r[30]), "=r"(r[31])
      : "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
      "%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle.  A tile lies as [dim / 64][keys][64 elements]: rows of 128 bytes
// whose 16-byte pieces are permuted in groups of eight rows (1024 bytes), as the copy unit writes them.
//   keys as rows (K: the head size is the summed dimension): stride 1024 between groups of eight keys;
//   keys as the summed dimension (V: rows are the head size): stride 1024 between groups of eight keys, and `chunk`
//   bytes between chunks of 64 of the head size.
// Low word: address and `chunk`, both in units of 16 bytes; high word: the stride, the version, the swizzle.
__device__ __forceinline__ uint32_t smem_desc_lo(uint32_t addr, uint32_t chunk) { return (addr & 0x3FFFF) >> 4 | (chunk >> 4) << 16; }
constexpr uint32_t SMEM_DESC_HI = (1024 >> 4) | 1u << 14 | 2u << 29;
// Instruction descriptor: fp32 accumulator, both operands of type `bf16` or half, M = 128.
__host__ __device__ constexpr uint32_t mma_desc(bool bf16, bool b_transposed, int n) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (b_transposed ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (128u >> 4) << 24;
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z, int w, uint32_t elected) {
  asm volatile(
      "{\n\t.reg .pred e;\n\tsetp.ne.u32 e, %7, 0;\n\t"
      "@e cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];\n\t}" ::"r"(dst),
      "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w), "r"(elected)
      : "memory");
}
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(FULL, v, 0); }  // the compiler then knows that it is
__device__ __forceinline__ float ta_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
template <bool BF16> __device__ __forceinline__ uint32_t ta_pack(float lo, float hi) {
  uint32_t r;
  if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <int N> __device__ __forceinline__ void tc_ld(uint32_t* r, uint32_t addr) {
  if constexpr (N == 32) tc_ld32(r, addr);
  else tc_ld16(r, addr);
}
template <int N> __device__ __forceinline__ void tc_st(uint32_t addr, const uint32_t* r) {
  if constexpr (N == 32) tc_st32(addr, r);
  else if constexpr (N == 16) tc_st16(addr, r);
  else tc_st8(addr, r);
}

// The rest of a wait that did not end at once; out of line, since each role's code should stay small: the roles share the
// instruction caches, and a warp whose code is fetched anew takes several cycles per instruction.
__device__ __noinline__ bool ta_wait_on(uint32_t bar, uint32_t parity, volatile int* abort_flag, unsigned limit) {
  const bool there = __all_sync(FULL, mbar_wait_timed(bar, parity, abort_flag, limit));
  if (!there) *abort_flag = 1;
  return there;
}

// Values that are not finite, for the rows of a warp: a lane has E elements of the row of node u, at o, the first of them in
// column c0 + at.  Elements with a bit in `lost` (NaN, though the row's weights are in order) become the sum of such cached values
// k0 .. k1 - 1, if there are any; to those of live rows come such values of the visible nodes n0 .. n1 - 1, which were taken out of
// the product.  A lane reads column c0 + lane, so that a value is read once for all rows: other warps wait meanwhile, and a sequence
// of such values must not make them give up on others (one NaN in a prompt of 4,096 rows: 8 ms; 226 when each row read for itself).
template <typename T, int E, bool PACKED>
__device__ __noinline__ void ta_settle(const AttnParams& p, int b, int g, int c0, int k0, int k1, int n0, int n1, float* o, int u, int at,
                                       uint32_t lost, bool live) {
  const int lane = threadIdx.x & 31, d = c0 + lane;
  if (__any_sync(FULL, lost != 0)) {
    const float mine = d < p.dim ? attn_odd_cached<T, PACKED>(p, b, g, d, k0, k1) : 0.0f;
    __syncwarp();
    for (int j = 0; j < 32; ++j) {
      const float sum = __shfl_sync(FULL, mine, j);
      const int e = j - at;
      if (e >= 0 && e < E && (lost >> e & 1u) && sum != 0.0f) o[e] = sum;
    }
  }
  const T* tree = reinterpret_cast<const T*>(p.v) + b * p.v_stride[0] + g * p.v_stride[2] + d;
  if (n1 > p.N) n1 = p.N;
  constexpr int NONE = 0x7FFFFFFF;
  int first = NONE, other = NONE;  // without a mask: the column's first such node, the first after it with another value
  float value1 = 0.0f;
  for (int v0 = n0; v0 < n1; v0 += 8) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v0 + i < n1 && d < p.dim ? to_float(tree[(v0 + i) * p.v_stride[1]]) : 0.0f;
    if (!p.mask) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (isfinite(f[i])) continue;
        if (first == NONE) {
          first = v0 + i;
          value1 = f[i];
        } else if (other == NONE && f[i] != value1) {
          other = v0 + i;
        }
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      for (uint32_t bits = __ballot_sync(FULL, !isfinite(f[i])); bits; bits &= bits - 1) {
        const int j = __ffs(bits) - 1, e = j - at;
        const float value = __shfl_sync(FULL, f[i], j);
        if (live && e >= 0 && e < E && attn_sees(p, b, u, v0 + i)) o[e] += value;
        __syncwarp();
      }
  }
  if (!p.mask && n1 > n0) {  // node u sees all up to itself: the sum changes at those two
    __syncwarp();
    for (int j = 0; j < 32; ++j) {
      const int from = __shfl_sync(FULL, first, j), from2 = __shfl_sync(FULL, other, j), e = j - at;
      const float value = __shfl_sync(FULL, value1, j);
      if (live && e >= 0 && e < E && u >= from) o[e] += u >= from2 ? NAN : value;
    }
  }
}

// ---- the kernel -----------------------------------------------------------------------
template <int DP, int C, bool BF16, bool PACKED>
__global__ void __launch_bounds__(TA_THREADS_OF<PACKED>, TaShape<DP, C, PACKED>::CTAS) tensor_attention_kernel(const __grid_constant__ TaParams p) {
  using Sh = TaShape<DP, C, PACKED>;
  constexpr int TA_THREADS = TA_THREADS_OF<PACKED>;
  // Halves do not hold all that codes stand for: there cached keys and values lie in the slots as 1 / 8 of themselves.  The text's scores are
  // brought back by their scale, its part of O by weights 2^3 larger than the tree's; so that these still fit, the maximum is raised that much earlier.
  // All of it by powers of two, so no bit changes but those of weights that were too small for a half.
  constexpr bool SHARED = PACKED && !BF16;
  constexpr float SHARE = SHARED ? 8.0f : 1.0f, SHARE_LOG = SHARED ? 3.0f : 0.0f, SLACK = TA_SLACK - SHARE_LOG;
  constexpr int MMA_WARP = PACKED ? 8 : 5;  // packed: warps 4 - 7 unpack, one for each scheduler as the softmax warps are (with two of those beside one: 387 us rather than 378)
  constexpr int KT = TA_KT, HALVES = DP / 64, SLOTS = Sh::SLOTS, K_SLOTS = Sh::K_SLOTS, V_SLOTS = Sh::V_SLOTS;
  constexpr int PART_ROWS = TA_ROWS / C, W = KT / C, CH = W < 32 ? W : 32;  // rows of a part; keys of a tile that it takes
  extern __shared__ __align__(1024) char ta_smem[];
  struct Shared {
    uint64_t full[SLOTS], empty[SLOTS], q, s[2], p[2], o[2], x, drain;  // s, p, o: by the place of a tile's scores
    TaRange<TA_THREADS> range;
    float2 ml[C > 1 ? TA_ROWS : 1];
    TaSeg seg;         // the piece that the rows in shared memory belong to; b < 0: no more
    uint64_t staged[PACKED ? Sh::STAGES : 1], taken[PACKED ? Sh::STAGES : 1];
    unsigned odd[2];   // 1 + the last piece (even ones, odd ones) whose tree has values that are not finite
    uint32_t tmem;
    int abort;
  };
  static_assert(sizeof(Shared) <= Sh::SHARED, "barriers");
  float* const exchange = reinterpret_cast<float*>(ta_smem + Sh::Q + SLOTS * Sh::SLOT);
  Shared& sh = *reinterpret_cast<Shared*>(ta_smem + Sh::SMEM - Sh::SHARED);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t q_smem = smem_addr(ta_smem), ring = q_smem + Sh::Q;
  if (warp == MMA_WARP) {
    tc_alloc(smem_addr(&sh.tmem), Sh::COLS);
  } else if (tid == 0) {
    for (int i = 0; i < SLOTS; ++i) {
      mbar_init(smem_addr(&sh.full[i]), PACKED ? 2 : 1);  // packed: two warps fill a slot
      mbar_init(smem_addr(&sh.empty[i]), 1);
    }
    mbar_init(smem_addr(&sh.q), 1);
    mbar_init(smem_addr(&sh.s[0]), 1);
    mbar_init(smem_addr(&sh.s[1]), 1);
    mbar_init(smem_addr(&sh.p[0]), 4);  // a lane of each warp arrives for it
    mbar_init(smem_addr(&sh.p[1]), 4);
    mbar_init(smem_addr(&sh.o[0]), 1);
    mbar_init(smem_addr(&sh.o[1]), 1);
    mbar_init(smem_addr(&sh.x), 4);
    if constexpr (PACKED)
      for (int i = 0; i < Sh::STAGES; ++i) {
        mbar_init(smem_addr(&sh.staged[i]), 32);
        mbar_init(smem_addr(&sh.taken[i]), 4);
      }
    mbar_init(smem_addr(&sh.drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.abort = (q_smem & 1023) != 0 || p.wait_limit == 0;  // the swizzle goes by address bits; no waiting allowed
    sh.odd[0] = sh.odd[1] = 0;
  }
  pdl_wait();

  TaWalk walk;
  // Dependents are released here, when the CTA has its tensor memory (behind ta_begin's barriers): a later launch of such a
  // kernel may hold tensor memory while it waits for this one, so it must not come to the allocation first.
  ta_begin<TA_THREADS>(p.s, walk, sh.range, [] { tc_fence_before(); }, [] {
    tc_fence_after();
    pdl_trigger();
  });
  const uint32_t tmem = sh.tmem;
  volatile int* abort_flag = &sh.abort;
  const unsigned limit = p.wait_limit;
  auto wait_warp = [&](uint32_t bar, uint32_t parity) {  // the whole warp calls it; false: gave up, as all others soon will
    if (__all_sync(FULL, mbar_try_wait(bar, parity))) return true;
    return ta_wait_on(bar, parity, abort_flag, limit);
  };
  const uint32_t bar_full = smem_addr(sh.full), bar_empty = smem_addr(sh.empty), bar_q = smem_addr(&sh.q), bar_s = smem_addr(sh.s),
                 bar_p = smem_addr(sh.p), bar_o = smem_addr(sh.o), bar_x = smem_addr(&sh.x);
  auto part_row = [&](const TaSeg& s, int row) { return ta_part_row(p.s, s, row); };

  if (PACKED && warp == 9) {
    // ---- packed tiles into stages --------------------------------------------------------
    constexpr int STAGES = Sh::STAGES;
    const uint32_t stages = q_smem + Sh::Q + SLOTS * Sh::SLOT + Sh::X, bar_staged = smem_addr(sh.staged), bar_taken = smem_addr(sh.taken);
    TaSeg s;
    PkCopies copies;
    uint32_t stage = 0, phase = 1;
    bool ok = *abort_flag == 0;
    while (ok && walk.next(p.s, s)) {
      const int end = s.end < s.p_tiles ? s.end : s.p_tiles;
      if (s.begin >= end) continue;
      copies.begin(p.s.a, s, lane);
      for (int tile = s.begin; tile < end; ++tile) {
        if (!(ok = wait_warp(bar_taken + 8 * stage, phase))) break;
        copies.tile<DP>(p.s.a, p.s.a.dim, lane, stages + stage * Sh::STAGE, Sh::STAGE_HALF, bar_staged + 8 * stage);
        if (++stage == STAGES) stage = 0, phase ^= 1u;
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
  } else if (PACKED && warp >= 4 && warp < 8) {
    // ---- packed keys (warps 4 and 5), packed values (6 and 7): half a tile each into its slot ---------
    // A lane has the 16 elements of a group of some keys.  Past the text's end a scale of zero makes zeros.
    constexpr int GROUPS = DP / 16, KEYS = 32 / GROUPS, UNITS = GROUPS;  // keys of a step, steps
    constexpr int STAGES = Sh::STAGES, BATCH = UNITS < 8 ? UNITS : 8;
    const bool value = warp >= 6, second = warp & 1;
    const CUtensorMap* tree_map = value ? &p.tree_v : &p.tree_k;
    const uint32_t slot0 = value ? K_SLOTS : 0, slots = value ? V_SLOTS : K_SLOTS;
    const uint32_t elected = elect_one(), bar_staged = smem_addr(sh.staged), bar_taken = smem_addr(sh.taken);
    const int D = p.s.a.dim, row0 = (second ? 32 : 0) + lane / GROUPS, group = lane % GROUPS;
    const bool has = group * 16 < D;
    // where the unit's two pieces lie in a slot; half of the lanes write them the other way round, for the banks
    const int swap = DP > 64 ? group >> 2 & 1 : 0, piece = (group & 3) * 2 + swap;
    const uint32_t column = (group >> 2) * (KT * 128) + row0 * 128;
    // this lane's codes and scales in the first of the warp's two lots of 16 keys; the second lies 9 D further on
    const char* const lot = ta_smem + Sh::Q + SLOTS * Sh::SLOT + Sh::X + (value ? Sh::STAGE_HALF : 0) + (second ? 18 * D : 0);
    const char* const codes0 = lot + lane / GROUPS * (D / 2) + (has ? group * 8 : 0);
    const char* const scales0 = lot + 8 * D + lane / GROUPS * (D / 16) + (has ? group : 0);
    TaSeg s;
    uint32_t slot = 0, phase = 1, used = 0, stage = 0, stage_phase = 0, tree_from = 0, tree_to = 0;  // tree: uses of slots with a copy of its rows
    bool ok = *abort_flag == 0;
    TaNote note(walk);
    while (walk.next(p.s, s)) {
      if (warp == 4) note.piece(walk, s, sh.range.total, sh.range.groups, blockIdx.x / p.s.group_ctas);
      if (!ok) continue;  // gave up: only the record is still to be found
      if (s.begin >= s.end) {
        if (s.rows && !s.whole && warp == 4)  // a piece of others that this CTA's rows do not see
          for (int i = lane; i < p.s.tile_rows; i += 32) p.s.part_ml[part_row(s, i)] = make_float2(-INFINITY, 0.0f);
        continue;
      }
      const int b = uniform(s.b), g = uniform(s.g), p_tiles = uniform(s.p_tiles), begin = uniform(s.begin), end = uniform(s.end);
      for (int tile = begin; tile < end; ++tile) {
        const uint32_t bar = bar_full + 8 * (slot0 + slot), dst = ring + (slot0 + slot) * Sh::SLOT;
        if (tile < p_tiles) {
          if (!(ok = wait_warp(bar_staged + 8 * stage, stage_phase))) break;
          const char *codes = codes0 + stage * Sh::STAGE, *scales = scales0 + stage * Sh::STAGE;
          char* to = ta_smem + Sh::Q + (slot0 + slot) * Sh::SLOT + column;
          const int left = s.len - tile * KT;  // of the text from this tile on
#pragma unroll
          for (int i0 = 0; i0 < UNITS; i0 += BATCH) {
            // all are read before the first is written: the compiler cannot know that they lie apart
            uint2 w[BATCH];
            uint32_t byte[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
              const int row = (i0 + i) % (UNITS / 2) * KEYS, at = (i0 + i) / (UNITS / 2) * 9 * D;
              w[i] = *reinterpret_cast<const uint2*>(codes + at + row * (D / 2));
              byte[i] = *reinterpret_cast<const unsigned char*>(scales + at + row * (D / 16));
            }
            if (!has || left < KT) {
#pragma unroll
              for (int i = 0; i < BATCH; ++i) {
                const int row = row0 + (i0 + i) * KEYS;
                if (!has || row >= left) byte[i] = 0;
              }
            }
            if (i0 == 0 && !(ok = wait_warp(bar_empty + 8 * (slot0 + slot), phase))) break;
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
              const int row = row0 + (i0 + i) * KEYS;
              const PkScale<BF16, SHARED> scale(byte[i]);
              const uint4 v0 = pk_word(swap ? w[i].y : w[i].x, scale), v1 = pk_word(swap ? w[i].x : w[i].y, scale);
              *reinterpret_cast<uint4*>(to + (i0 + i) * KEYS * 128 + ((piece ^ (row & 7)) << 4)) = v0;
              *reinterpret_cast<uint4*>(to + (i0 + i) * KEYS * 128 + ((piece ^ 1 ^ (row & 7)) << 4)) = v1;
            }
          }
          if (!ok) break;
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(bar);
            mbar_arrive(bar_taken + 8 * stage);
          }
          if (++stage == STAGES) stage = 0, stage_phase ^= 1u;
        } else {
          if (!(ok = wait_warp(bar_empty + 8 * (slot0 + slot), phase))) break;
          if (second) {
            if (lane == 0) mbar_arrive(bar);
          } else {
            if (elected) mbar_expect_tx(bar, Sh::SLOT);
#pragma unroll
            for (int half = 0; half < HALVES; ++half)
              tma_load_4d(dst + half * (KT * 128), tree_map, bar, half * 64, (tile - p_tiles) * KT, g, b, elected);
            if (tree_to != used) tree_from = used;
            tree_to = used + 1;
          }
        }
        ++used;
        if (++slot == slots) slot = 0, phase ^= 1u;
      }
    }
    if (warp == 4 && lane == 0 && blockIdx.x % p.s.group_ctas == 0) p.s.records[blockIdx.x / p.s.group_ctas] = note.r;
    if (!ok && lane == 0 && !second) {  // copies in flight land before the block ends
      for (unsigned i = tree_to > tree_from + slots ? tree_to - slots : tree_from; i < tree_to; ++i)
        mbar_wait_timed(bar_full + 8 * (slot0 + i % slots), (i / slots) & 1u, nullptr, SPIN_LIMIT);
    }
    __syncwarp();
  } else if (!PACKED && (warp == 4 || warp == 6)) {
    // ---- keys (warp 4), values (warp 6) --------------------------------------------------
    // A tile is copied in boxes of box_rows rows of one page; lane i keeps the place of the tile's i-th box and reads its
    // page's number a tile ahead.
    const bool value = warp == 6;
    const CUtensorMap* cache_map = value ? &p.cache_v : &p.cache_k;
    const CUtensorMap* tree_map = value ? &p.tree_v : &p.tree_k;
    const uint32_t slot0 = value ? K_SLOTS : 0, slots = value ? V_SLOTS : K_SLOTS;
    const int n_boxes = KT / p.box_rows;
    const uint32_t elected = elect_one();
    TaSeg s;
    uint32_t slot = 0, phase = 1, used = 0;  // phase: parity of the wait for the slot's last use
    bool ok = *abort_flag == 0;
    TaNote note(walk);
    while (walk.next(p.s, s)) {
      if (!value) note.piece(walk, s, sh.range.total, sh.range.groups, blockIdx.x / p.s.group_ctas);
      if (!ok) continue;  // gave up: only the record is still to be found
      if (s.begin >= s.end) {
        if (s.rows && !s.whole && !value)  // a piece of others that this CTA's rows do not see
          for (int i = lane; i < p.s.tile_rows; i += 32) p.s.part_ml[part_row(s, i)] = make_float2(-INFINITY, 0.0f);
        continue;
      }
      const int b = uniform(s.b), g = uniform(s.g), len = uniform(s.len), p_tiles = uniform(s.p_tiles), begin = uniform(s.begin), end = uniform(s.end);
      int pos = begin * KT + lane * p.box_rows, col = pos / p.s.a.page, in_page = pos - col * p.s.a.page;
      const int* table = p.s.a.table + (long long)b * p.s.a.cols;
      int next = lane < n_boxes && pos < len ? __ldg(table + col) : 0;
      for (int tile = begin; tile < end; ++tile) {
        const int page = next >= 0 && next < p.s.a.pages ? next : p.s.a.pages, at = in_page;  // past the pool: the copy unit fills in zeros
        pos += KT;
        for (in_page += KT; in_page >= p.s.a.page; in_page -= p.s.a.page) ++col;
        if (lane < n_boxes && pos < len) next = __ldg(table + col);
        if (!(ok = wait_warp(bar_empty + 8 * (slot0 + slot), phase))) break;
        const uint32_t bar = bar_full + 8 * (slot0 + slot), dst = ring + (slot0 + slot) * Sh::SLOT;
        if (tile < p_tiles) {
          const int left = len - tile * KT, boxes = left >= KT ? n_boxes : (left + p.box_rows - 1) / p.box_rows;
          if (elected) mbar_expect_tx(bar, boxes * HALVES * p.box_rows * 128);
          int from[KT / 16], row[KT / 16];
#pragma unroll
          for (int i = 0; i < KT / 16; ++i) from[i] = __shfl_sync(FULL, page, i), row[i] = __shfl_sync(FULL, at, i);
#pragma unroll
          for (int i = 0; i < KT / 16; ++i) {
            if (i >= boxes) break;
#pragma unroll
            for (int half = 0; half < HALVES; ++half)
              tma_load_4d(dst + half * (KT * 128) + i * p.box_rows * 128, cache_map, bar, half * 64, row[i], g, from[i], elected);
          }
        } else {
          if (elected) mbar_expect_tx(bar, Sh::SLOT);
#pragma unroll
          for (int half = 0; half < HALVES; ++half)
            tma_load_4d(dst + half * (KT * 128), tree_map, bar, half * 64, (tile - p_tiles) * KT, g, b, elected);
        }
        ++used;
        if (++slot == slots) slot = 0, phase ^= 1u;
      }
    }
    if (!value && lane == 0 && blockIdx.x % p.s.group_ctas == 0) p.s.records[blockIdx.x / p.s.group_ctas] = note.r;
    if (!ok && lane == 0) {  // copies in flight land before the block ends
      for (unsigned i = used > slots ? used - slots : 0; i < used; ++i)
        mbar_wait_timed(bar_full + 8 * (slot0 + i % slots), (i / slots) & 1u, nullptr, SPIN_LIMIT);
    }
    __syncwarp();
  } else if (warp == MMA_WARP) {
    // ---- products -----------------------------------------------------------------------
    constexpr uint32_t IDESC_S = mma_desc(BF16, false, KT), IDESC_O = mma_desc(BF16, true, DP);
    TaSeg s;
    uint32_t k_slot = 0, k_phase = 0, v_slot = 0, v_phase = 0, n = 0, q_phase = 0, buf = 0;  // n: tiles so far
    const uint32_t elected = elect_one(), base = __shfl_sync(FULL, tmem, 0);
    const uint32_t q_desc = smem_desc_lo(q_smem, 16), k_desc = smem_desc_lo(ring, 16), v_desc = smem_desc_lo(ring, KT * 128);
    const uint32_t d_s = base + Sh::COL_S, d_o = base + Sh::COL_O;
    bool ok = *abort_flag == 0, copying = false;
    while (ok) {
      bool more;
      do more = walk.next(p.s, s);  // the next piece with keys
      while (more && s.begin >= s.end);
      // Its rows into shared memory, and its description to the softmax warps, which wait for the same barrier.  They
      // have written P of the last tile before, so its scores are done with the rows that lie there.
      if (elected) {
        sh.seg = s;
        if (!more) sh.seg.b = -1;
        if (more) mbar_expect_tx(bar_q, C * HALVES * p.s.tile_rows * 128);
        else mbar_arrive(bar_q);
      }
      if (!more) break;
      copying = true;
      const int head = uniform(s.g * p.s.a.group), node0 = uniform(s.row0 / p.s.a.group), b = uniform(s.b);
#pragma unroll
      for (int i = 0; i < C * HALVES; ++i)
        tma_load_4d(q_smem + i % HALVES * (TA_ROWS * 128) + i / HALVES * (PART_ROWS * 128), &p.q, bar_q, i % HALVES * 64, head, node0, b, elected);
      const int tiles = uniform(s.end - s.begin);
      if (!(ok = wait_warp(bar_q, q_phase))) break;
      copying = false;
      q_phase ^= 1u;
      for (int j = -1; j < tiles; ++j) {
        if (j + 1 < tiles) {  // S of tile j + 1.  Its place was that of tile j - 1, whose P V is issued: products run in order.
          if (!(ok = wait_warp(bar_full + 8 * k_slot, k_phase))) break;
          tc_fence_after();
          const uint32_t bk = k_desc + k_slot * (Sh::SLOT >> 4);
#pragma unroll
          for (int k = 0; k < DP / 16; ++k)
            tc_mma_ss(d_s + buf * KT, q_desc + (((k >> 2) * (TA_ROWS * 128) + (k & 3) * 32) >> 4),
                      bk + (((k >> 2) * (KT * 128) + (k & 3) * 32) >> 4), SMEM_DESC_HI, IDESC_S, k > 0, elected);
          tc_commit(bar_s + 8 * buf, elected);
          tc_commit(bar_empty + 8 * k_slot, elected);
          if (++k_slot == K_SLOTS) k_slot = 0, k_phase ^= 1u;
          buf ^= 1u;
        }
        if (j >= 0) {  // O += P V of tile j
          if (!(ok = wait_warp(bar_full + 8 * (K_SLOTS + v_slot), v_phase) && wait_warp(bar_p + 8 * (n & 1), (n >> 1) & 1u))) break;
          tc_fence_after();
          const uint32_t bv = v_desc + (K_SLOTS + v_slot) * (Sh::SLOT >> 4), d_p = d_s + (n & 1) * KT;
#pragma unroll
          for (int k = 0; k < KT / 16; ++k) tc_mma(d_o, d_p + k * 8, bv + k * (2048 >> 4), SMEM_DESC_HI, IDESC_O, k > 0 || j > 0, elected);
          tc_commit(bar_o + 8 * (n & 1), elected);
          tc_commit(bar_empty + 8 * (K_SLOTS + v_slot), elected);
          if (++v_slot == V_SLOTS) v_slot = 0, v_phase ^= 1u;
          ++n;
        }
      }
    }
    if (!ok) {  // what is in flight ends before the block does
      if (copying) mbar_wait_timed(bar_q, q_phase, nullptr, SPIN_LIMIT);
      __syncwarp();
      tc_commit(smem_addr(&sh.drain), elected);
      mbar_wait_timed(smem_addr(&sh.drain), 0, nullptr, SPIN_LIMIT);
    }
    __syncwarp();
  } else {
    // ---- softmax: thread = row (of a part) -------------------------------------------------
    const uint32_t my = tmem + ((uint32_t)(warp * 32) << 16);
    const int part = tid / PART_ROWS, row = tid % PART_ROWS;  // a warp lies in one part
    const bool in_tile = row < p.s.tile_rows, warp_in = (warp * 32) % PART_ROWS < p.s.tile_rows;
    const int up = in_tile ? row / p.s.a.group : 0, head = in_tile ? row - up * p.s.a.group : 0;
    const float scale2 = p.s.a.scale2;
    unsigned n = 0, n_seg = 0, x_phase = 0;  // tiles and pieces so far
    bool ok = *abort_flag == 0;
    auto sync_rows = [&]() {  // all rows' threads
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_x);
      ok = wait_warp(bar_x, x_phase) && ok;
      x_phase ^= 1u;
    };
    while (ok) {
      ok = wait_warp(bar_q, n_seg & 1u);
      if (!ok) break;
      const TaSeg s = sh.seg;
      if (s.b < 0) break;
      const int u = s.row0 / p.s.a.group + up, h = s.g * p.s.a.group + head;
      const bool in = in_tile && u < p.s.a.N;
      const bool live = in && !(p.s.a.tree && p.s.a.tree[(long long)s.b * p.s.a.N + u] < 0);
      float m = -INFINITY, l = 0.0f;
      for (int j = s.begin; j < s.end; ++j, ++n) {
        const bool tree = j >= s.p_tiles;
        const int left = s.len - j * KT;  // cached tokens from this tile on
        const bool partial = !tree && left < KT;
        const float by = SHARED && !tree ? scale2 * SHARE : scale2;
        ok = wait_warp(bar_s + 8 * (n & 1), (n >> 1) & 1u);
        if (!ok) break;
        tc_fence_after();
        if (warp_in) {
          // Twice over the scores, 32 (or all W) at a time, from tensor memory both times: little code, few registers.
          const uint32_t s_addr = my + Sh::COL_S + (n & 1) * KT + part * W;
          float top = -INFINITY, top1 = -INFINITY;
#pragma unroll 1
          for (int c = 0; c < W / CH; ++c) {
            uint32_t x[CH];
            tc_ld<CH>(x, s_addr + c * CH);
            tc_wait_ld();
            if (tree || partial) {
              const int key = part * W + c * CH;  // of the tile
              uint32_t seen;                      // by this row
              if (tree) {
                seen = attn_nodes_seen(p.s.a, s.b, u, (j - s.p_tiles) * KT + key);
              } else {
                const int below = left - key;
                seen = below >= 32 ? FULL : (below > 0 ? (1u << below) - 1 : 0u);
              }
#pragma unroll
              for (int i = 0; i < CH; ++i) x[i] = seen >> i & 1u ? x[i] : 0xFF800000u;
              __syncwarp();
              tc_st<CH>(s_addr + c * CH, x);
              tc_wait_st();
            }
#pragma unroll
            for (int i = 0; i < CH; i += 4) {
              top = max3(top, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
              top1 = max3(top1, __uint_as_float(x[i + 2]), __uint_as_float(x[i + 3]));
            }
          }
          top = fmaxf(top, top1) * by;
          // Any m near the maximum will do, since o and l carry the same factor: it is left where it is until scores pass
          // it by SLACK, so that o is seldom read, scaled and written (TA_LIFT keeps the weights within their type).  The warp's rows move together, as live rows want it: what lies in the lanes of others is
          // left from earlier kernels or belongs to nodes that were not drafted, and would enter the roundings of the weights.
          if (__any_sync(FULL, live && top > m + SLACK)) {
            const float raised = fmaxf(m, top);
            const float keep = raised == -INFINITY ? 1.0f : ta_ex2(m - raised);
            m = raised;
            l *= keep;
            if (j > s.begin) {
              ok = wait_warp(bar_o + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1u);  // P V of the tile before
              if (!ok) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < DP / 32; ++c) {
                uint32_t o[32];
                tc_ld32(o, my + Sh::COL_O + c * 32);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
                tc_st32(my + Sh::COL_O + c * 32, o);
              }
            }
          }
          const float base = (m == -INFINITY ? 0.0f : m) - (TA_LIFT<BF16> + (tree ? 0.0f : SHARE_LOG));
          const unsigned long long scale_2 = pack2(by, by), base_2 = pack2(-base, -base);
          unsigned long long sum_2 = pack2(0.0f, 0.0f);
#pragma unroll 1
          for (int c = 0; c < W / CH; ++c) {
            uint32_t x[CH], w[CH / 2];
            tc_ld<CH>(x, s_addr + c * CH);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < CH / 2; ++i) {
              float a, b;
              unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), scale_2, base_2), a, b);
              a = ta_ex2(a);
              b = ta_ex2(b);
              sum_2 = add2(sum_2, pack2(a, b));
              w[i] = ta_pack<BF16>(a, b);
            }
            tc_st<CH / 2>(s_addr - part * W + part * (W / 2) + c * (CH / 2), w);
          }
          if constexpr (C > 1) {  // the other parts' keys have no weight in these lanes
            const uint32_t zero[W / 2] = {};
#pragma unroll
            for (int k = 1; k < C; ++k) tc_st<W / 2>(s_addr - part * W + (part + k) % C * (W / 2), zero);
          }
          float sum0, sum1;
          unpack2(sum_2, sum0, sum1);
          if constexpr (SHARED) l = fmaf(sum0 + sum1, tree ? 1.0f : 1.0f / SHARE, l);
          else l += sum0 + sum1;
          tc_wait_st();
        }
        if (tree || (partial && !PACKED)) {
          // Values that no row sees must not enter the product, 0 times them included: those past the text's end become
          // zero.  In the tree some rows may see what others do not: there, elements that are not finite become zero and
          // are added at the end to the rows that do see them.
          // (Not before the scores are there: until then the slot may still await the values of two tiles before.)
          const unsigned slot = K_SLOTS + n % V_SLOTS;
          ok = wait_warp(bar_full + 8 * slot, (n / V_SLOTS) & 1u);
          if (!ok) break;
          char* v0 = ta_smem + Sh::Q + slot * Sh::SLOT;
          if (partial) {  // (not packed: there they are zeros already)
            for (int i = left * 8 + tid; i < KT * 8; i += TA_ROWS)
#pragma unroll
              for (int hh = 0; hh < HALVES; ++hh) *reinterpret_cast<uint4*>(v0 + hh * (KT * 128) + i * 16) = make_uint4(0, 0, 0, 0);
          } else {
            constexpr uint32_t EXP = BF16 ? 0x7F80u : 0x7C00u;
            const int nodes = p.s.a.N - (j - s.p_tiles) * KT, pieces = (nodes < KT ? nodes : KT) * 8;  // the rest are zeros
            for (int k = tid; k < HALVES * pieces; k += TA_ROWS) {
              const int i = k + (HALVES > 1 ? k / pieces * (KT * 8 - pieces) : 0);
              uint4 v = *reinterpret_cast<uint4*>(v0 + i * 16);
              uint32_t* e = reinterpret_cast<uint32_t*>(&v);
              bool odd = false;
#pragma unroll
              for (int c = 0; c < 4; ++c) {
                if ((e[c] & EXP) == EXP) { e[c] &= 0xFFFF0000u; odd = true; }
                if ((e[c] & (EXP << 16)) == (EXP << 16)) { e[c] &= 0xFFFFu; odd = true; }
              }
              if (odd) {
                *reinterpret_cast<uint4*>(v0 + i * 16) = v;
                sh.odd[n_seg & 1] = n_seg + 1;
              }
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_p + 8 * (n & 1));
      }
      if (!ok) break;
      ok = wait_warp(bar_o + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1u);
      if (!ok) break;
      tc_fence_after();
      const bool odd = sh.odd[n_seg & 1] == n_seg + 1;
      ++n_seg;
      m -= TA_LIFT<BF16>;  // what l and o are relative to

      // ---- the piece's result ---------------------------------------------------------------
      float factor = 1.0f;  // of this part's o
      if constexpr (C > 1) {
        sh.ml[tid] = make_float2(m, l);
        sync_rows();
        if (!ok) break;
        float top = m, total = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) top = fmaxf(top, sh.ml[c * PART_ROWS + row].x);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int c = 0; c < C; ++c) {
          const float2 v = sh.ml[c * PART_ROWS + row];
          total += v.y * ta_ex2(v.x - base);
        }
        factor = ta_ex2(m - base);
        m = top;
        l = total;
        sync_rows();  // all have read
        if (!ok) break;
        if (part == 0) sh.ml[row] = make_float2(!live || l == 0.0f ? 0.0f : 1.0f / l, live ? 1.0f : 0.0f);
      }
      const long long out_row = ((long long)s.b * p.s.a.N + u) * p.s.a.heads_q + h, at = part_row(s, row);
      const bool empty = !live || l == 0.0f;
      const float inv = empty ? 0.0f : 1.0f / l;
      if (in && part == 0) {
        if (!s.whole) p.s.part_ml[at] = live ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
        else if (p.s.a.lse) p.s.a.lse[out_row] = empty ? -INFINITY : 0.6931471805599453f * (m + log2f(l));
      }
      using T = typename std::conditional<BF16, __nv_bfloat16, __half>::type;
      const int k0 = s.begin * KT, k1 = s.end * KT < s.len ? s.end * KT : s.len;  // cached tokens and nodes of the piece
      const int n0 = (s.begin > s.p_tiles ? s.begin - s.p_tiles : 0) * KT, n1 = odd && s.end > s.p_tiles ? (s.end - s.p_tiles) * KT : 0;
      if constexpr (C == 1) {
        if (warp_in) {
#pragma unroll 1
          for (int c = 0; c < DP / 32; ++c) {
            uint32_t o[32];
            __syncwarp();  // rows that do not exist have gone another way
            tc_ld32(o, my + Sh::COL_O + c * 32);
            tc_wait_ld();
            float zero[4] = {};  // NaN if one of them is not finite
#pragma unroll
            for (int i = 0; i < 32; ++i) zero[i & 3] = fmaf(__uint_as_float(o[i]), 0.0f, zero[i & 3]);
            if (__any_sync(FULL, live && (odd || isnan(zero[0] + zero[1] + zero[2] + zero[3])))) {
              float f[32];
              uint32_t lost = 0;
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                f[i] = __uint_as_float(o[i]);
                if (live && isfinite(l) && isnan(f[i])) lost |= 1u << i;
              }
              ta_settle<T, 32, PACKED>(p.s.a, s.b, s.g, c * 32, k0, k1, n0, n1, f, u, 0, lost, live);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(f[i]);
            }
            if (!in) continue;
            if (!s.whole) {
              float4* dst = reinterpret_cast<float4*>(p.s.part_o + at * DP + c * 32);
#pragma unroll
              for (int i = 0; i < 8; ++i)
                dst[i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]),
                                     __uint_as_float(o[4 * i + 3]));
            } else {
              uint4* dst = reinterpret_cast<uint4*>(p.s.a.out + 2 * (out_row * p.s.a.dim + c * 32));
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  w[e] = empty ? 0u : ta_pack<BF16>(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                if (c * 32 + i * 8 < p.s.a.dim) dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
        }
      } else {
        // Some columns at a time through shared memory, as many as fit (with few rows all of them); then each thread
        // sums four columns of a row over the parts.
        const int rows = p.s.tile_rows;
        int cols = TA_XCOLS;
        while (cols < DP && C * rows * (2 * cols + 1) <= TA_ROWS * (TA_XCOLS + 1)) cols *= 2;
        const int pitch = cols + 1;
#pragma unroll 1
        for (int c0 = 0; c0 < DP; c0 += cols) {
          if (warp_in) {
#pragma unroll 1
            for (int c = 0; c < cols; c += 16) {
              uint32_t o[16];
              __syncwarp();
              tc_ld16(o, my + Sh::COL_O + c0 + c);
              tc_wait_ld();
              if (in_tile) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  exchange[(part * rows + row) * pitch + c + i] = factor == 0.0f ? 0.0f : __uint_as_float(o[i]) * factor;
              }
            }
          }
          sync_rows();
          if (!ok) break;
          const int quads = cols / 4;
          for (int i0 = 0; i0 < rows * quads; i0 += TA_ROWS) {  // whole warps
            const int i = i0 + tid, r = i / quads, q = i - r * quads, col = c0 + q * 4;
            const int ru = s.row0 / p.s.a.group + r / p.s.a.group, rh = s.g * p.s.a.group + r % p.s.a.group;
            const bool there = r < rows && ru < p.s.a.N;
            float v[4] = {};
            float2 ml = make_float2(0.0f, 0.0f);
            if (there) {
              ml = sh.ml[r];  // 1 / l, and whether the row is there at all
#pragma unroll
              for (int k = 0; k < C; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += exchange[(k * rows + r) * pitch + q * 4 + e];
            }
            if (__any_sync(FULL, ml.y != 0.0f && (odd || !isfinite(v[0] + v[1] + v[2] + v[3])))) {
              float f[4];
              uint32_t lost = 0;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                f[e] = v[e];
                if (ml.y != 0.0f && ml.x > 0.0f && isnan(f[e])) lost |= 1u << e;
              }
              for (int at = 0; at < cols; at += 32)
                ta_settle<T, 4, PACKED>(p.s.a, s.b, s.g, c0 + at, k0, k1, n0, n1, f, ru, q * 4 - at, lost, ml.y != 0.0f);
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = f[e];
            }
            if (!there) continue;
            if (!s.whole) {
              *reinterpret_cast<float4*>(p.s.part_o + part_row(s, r) * DP + col) = make_float4(v[0], v[1], v[2], v[3]);
            } else if (col < p.s.a.dim) {
              const bool none = ml.x == 0.0f;
              *reinterpret_cast<uint2*>(p.s.a.out + 2 * ((((long long)s.b * p.s.a.N + ru) * p.s.a.heads_q + rh) * p.s.a.dim + col)) =
                  make_uint2(none ? 0u : ta_pack<BF16>(v[0] * ml.x, v[1] * ml.x), none ? 0u : ta_pack<BF16>(v[2] * ml.x, v[3] * ml.x));
            }
          }
          sync_rows();
          if (!ok) break;
        }
        if (!ok) break;
      }
      tc_fence_before();
    }
    if (!ok) {  // a wait ran out: nothing that this block had to do is to be trusted
      TaSeg s;
      while (walk.next(p.s, s)) {
        const int u = s.row0 / p.s.a.group + up, h = s.g * p.s.a.group + head;
        if (!in_tile || part != 0 || u >= p.s.a.N) continue;
        p.s.part_ml[part_row(s, row)] = make_float2(0.0f, NAN);
        if (!s.whole) continue;
        const long long out_row = ((long long)s.b * p.s.a.N + u) * p.s.a.heads_q + h;
        if (p.s.a.lse) p.s.a.lse[out_row] = NAN;
        for (int d = 0; d < p.s.a.dim; ++d) reinterpret_cast<unsigned short*>(p.s.a.out)[out_row * p.s.a.dim + d] = 0x7FFFu;  // NaN in both types
      }
    }
  }
  __syncthreads();
  if (warp == MMA_WARP) tc_dealloc(tmem, Sh::COLS);
}

// ---- launch ------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) f = nullptr;
    return reinterpret_cast<EncodeTiled>(f);
  }();
  return fn;
}

// A tensor [w][z][y][dim] of 16-bit elements (strides in elements) that is copied ny x nz rows at a time, 64 elements wide.
inline bool encode_map(CUtensorMap* map, const void* base, bool bf16, int dim, const long long (&n)[3], const long long (&stride)[3], int ny,
                       int nz) {
  cuuint64_t dims[4] = {(cuuint64_t)dim, 1, 1, 1}, strides[3];
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = (cuuint64_t)n[i];
    strides[i] = n[i] == 1 ? 16 : (cuuint64_t)stride[i] * 2;  // a dimension of extent 1 may have any stride
    if (strides[i] == 0 || (strides[i] & 15) != 0 || strides[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)ny, (cuuint32_t)nz, 1}, step[4] = {1, 1, 1, 1};
  return encode_tiled()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides,
                        box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Row tiles hold whole nodes, so that one copy brings a tile's rows.
inline int tensor_tile_rows(int n, int group) { return (long long)n * group <= TA_ROWS ? n * group : TA_ROWS / group * group; }
inline int tensor_ctas(int dim) { return tensor_dim(dim) == 256 ? 1 : 2; }

// STAND_E_ARG: not a call for these kernels (what the copy unit cannot address); nothing was launched.
template <int DP, int C, bool BF16, bool PACKED> int launch_tensor_attention(const AttnParams& a, void* scratch, int sms, unsigned wait_limit, cudaStream_t st) {
  using Sh = TaShape<DP, C, PACKED>;
  TaParams p;
  // A piece's fixed cost in tiles, measured by trying 3 to 9: 16 sequences of 1 - 8,190 tokens with heads of 64 take 81, 71, 59,
  // 58 us with 3, 5, 7, 9; 256 sequences of 130 - 4,100 with heads of 128 take 393, 389, 391, 398; 64 of them with 16 / 4 heads of 256
  // 149, 124, 117, 117 with 0, 2, 5, 8.
  ta_split(p.s, a, tensor_tile_rows(a.N, a.group), DP, sms, Sh::CTAS, DP == 64 ? 8 : 5, scratch);
  p.box_rows = 16;
  while (p.box_rows < TA_KT && a.page % (p.box_rows * 2) == 0) p.box_rows *= 2;
  p.wait_limit = wait_limit;

  const long long tree_n[3] = {a.N, a.heads_kv, a.B}, k_stride[3] = {a.k_stride[1], a.k_stride[2], a.k_stride[0]};
  const long long v_stride[3] = {a.v_stride[1], a.v_stride[2], a.v_stride[0]};
  const long long q_n[3] = {a.heads_q, a.N, a.B}, q_stride[3] = {a.q_stride[2], a.q_stride[1], a.q_stride[0]};
  if (!encode_map(&p.q, a.q, BF16, a.dim, q_n, q_stride, a.group, p.s.tile_rows / a.group) ||
      !encode_map(&p.tree_k, a.k, BF16, a.dim, tree_n, k_stride, TA_KT, 1) ||
      !encode_map(&p.tree_v, a.v, BF16, a.dim, tree_n, v_stride, TA_KT, 1))
    return STAND_E_ARG;
  if (!PACKED && a.cols > 0) {
    const long long n[3] = {a.page, a.heads_kv, a.pages}, stride[3] = {a.cache_stride[2], a.cache_stride[1], a.cache_stride[0]};
    if (a.pages < 1 || !encode_map(&p.cache_k, a.cache_k, BF16, a.dim, n, stride, p.box_rows, 1) ||
        !encode_map(&p.cache_v, a.cache_v, BF16, a.dim, n, stride, p.box_rows, 1))
      return STAND_E_ARG;
  } else {  // no cache, or not by these: never read
    p.cache_k = p.tree_k;
    p.cache_v = p.tree_v;
  }
  static SmemLimit limit;
  int rc = limit.raise(tensor_attention_kernel<DP, C, BF16, PACKED>, Sh::SMEM);
  if (rc) return STAND_E_CUDA;
  rc = launch_dependent(tensor_attention_kernel<DP, C, BF16, PACKED>, dim3((unsigned)(p.s.groups * p.s.group_ctas)), TA_THREADS_OF<PACKED>, st, p, Sh::SMEM);
  if (rc) return rc;
  return launch_join<DP, typename std::conditional<BF16, __nv_bfloat16, __half>::type>(p.s, st);
}

template <int DP, bool BF16, bool PACKED = false> int launch_tensor_parts(const AttnParams& a, void* scratch, int sms, unsigned wait_limit, cudaStream_t st) {
  // Few rows of small heads in four (two) parts.  Measured, parts / none: 16 sequences of 1 - 8,190 tokens, 16 / 16 heads of
  // 64, with 1 node 52 / 63 us, 32 nodes 59 / 66, 48 nodes 68 / 80.  Not for larger heads, whose tiles wait for memory and not
  // for the softmax, and where the exchange takes room from the rings: head size 128, 48 rows, 129 / 108; 16 rows, 193 / 184.
  if constexpr (DP == 64) {
    const int rows = tensor_tile_rows(a.N, a.group);
    if (rows <= TA_ROWS / 4) return launch_tensor_attention<DP, 4, BF16, PACKED>(a, scratch, sms, wait_limit, st);
    if (rows <= TA_ROWS / 2) return launch_tensor_attention<DP, 2, BF16, PACKED>(a, scratch, sms, wait_limit, st);
  }
  return launch_tensor_attention<DP, 1, BF16, PACKED>(a, scratch, sms, wait_limit, st);
}

// Rows of 16-byte pieces (strides are looked at when they are encoded).
inline bool tensor_takes(const AttnParams& a, int dtype) {
  if (dtype == STAND_DTYPE_F32 || a.dim % 8 != 0 || a.group > TA_ROWS || !encode_tiled()) return false;
  uintptr_t bits = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out;
  if (a.cols > 0) bits |= (uintptr_t)a.cache_k | (uintptr_t)a.cache_v;
  return (bits & 15) == 0;
}

}  // namespace stand
