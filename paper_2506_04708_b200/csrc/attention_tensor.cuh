// Tree attention on the tensor cores (tcgen05, sm_100a): bfloat16 and half, head sizes that are a multiple of 8, 16-byte
// aligned rows.
//
// A block (CTA) of six warps works on 128 rows of one (sequence, key head) pair and walks over its keys in tiles:
//   warp 4  copies tiles of keys and of values from the pages (and from the tree's own keys) with TMA into a ring,
//   warp 5  issues the matrix products S = Q K^T and O += P V, one thread for all,
//   warps 0-3  own one row per thread: read S, keep the running maximum and sum, write P, finally write O / l.
// Q, S and O live in tensor memory (a row is a lane): Q as the first operand of the first product, P, in 16 bits and in
// the place of S, as that of the second, so that shared memory holds nothing but the ring of keys and values and is read
// once per product.  What a tile costs in sequence (product, softmax, product) is hidden by the second CTA of the SM: the
// two take 256 of the 512 columns of tensor memory and half of the shared memory each (head size 256: one CTA per SM).
//
// The keys of all pairs, laid end to end in tiles, are cut into as many equal ranges as there are CTAs (or groups of
// CTAs: the row tiles of a pair with more than 128 rows go to neighbours that walk over the same keys at the same time,
// so that those come from memory once and from L2 after that).  A range may begin and end inside a pair: such pieces
// leave (m, l, O) in scratch and a second, small kernel joins them.  So long texts with few rows fill the GPU, and so do
// batches of ragged lengths, without the host knowing a length.
#pragma once
#include <cuda.h>

#include "async.cuh"
#include "attention.cuh"
#include "launch.cuh"

namespace stand {

constexpr int TA_ROWS = 128;              // rows of a CTA: lanes of tensor memory
constexpr int TA_THREADS = 192;
constexpr int TA_SMS = 148;               // B200; scratch is laid out for that many
constexpr int TA_GROUP = 4;               // row tiles that walk together, at most
constexpr float TA_SLACK = 8.0f;          // the maximum is raised only when scores pass it by 2^8 (below)

template <int DP> struct TaShape {
  static constexpr int KT = DP == 64 ? 128 : 64;              // keys per tile
  static constexpr int CTAS = DP == 256 ? 1 : 2;              // per SM
  static constexpr int SLOT = KT * DP * 2;                    // bytes of a tile of keys or values
  static constexpr int SLOTS = 6;
  static constexpr int COL_O = 0, COL_S = DP, COL_Q = DP + KT;
  static constexpr int COLS = DP == 256 ? 512 : 256;          // tensor memory columns allocated
  static constexpr int SMEM = SLOTS * SLOT + 1024;            // and room to align the ring
  static_assert(COL_Q + DP / 2 <= COLS, "tensor memory");
};

struct TaRecord {  // what the joining kernel has to do for the last pair that a group began
  int n_parts;     // 0: nothing (that pair ends within the group)
  int first_which, b, g, rb;
  int pad[3];
};

struct alignas(64) TaParams {
  CUtensorMap cache_k, cache_v, tree_k, tree_v;
  AttnParams a;
  int rows;           // N * group
  int row_blocks;     // groups of row tiles
  int group_ctas;     // row tiles per group
  int groups;
  int min_tiles;      // fewest tiles worth a group of their own
  int box_rows;       // rows of a page that one copy takes
  int part_rows;      // rows of a piece in scratch
  long long tree_tiles;  // sum over the row blocks of a pair
  TaRecord* records;
  float2* part_ml;
  float* part_o;
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
// The whole warp calls these two, the elected lane acts: the operands then sit in uniform registers, where the unit wants
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
// 32 columns of this warp's 32 lanes: one row per thread
__device__ __forceinline__ void tc_ld32(uint32_t (&r)[32], uint32_t addr) {
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
__device__ __forceinline__ void tc_st32(uint32_t addr, const uint32_t (&r)[32]) {
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

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z, int w) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(dst),
               "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
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

// ---- the walk over a group's range of tiles -----------------------------------------
struct TaSeg {
  int b, g, rb, row0;      // pair, row block, first row of this CTA
  int len, p_tiles;        // cached tokens, their tiles
  int begin, end;          // this CTA's tiles of the pair (cached ones, then the tree's)
  bool whole, rows;        // the range covers the pair; the CTA has rows in this block
  int which;               // the group's first piece or a later one
};

template <int KT> struct TaWalk {
  long long t, hi, b_start;
  int b;
  bool first;

  // tree tiles that rows before row_end see
  __device__ static __forceinline__ int tree_tiles(const TaParams& p, long long row_end) {
    const long long last = (row_end < p.rows ? row_end : p.rows) - 1;
    return (int)(last / p.a.group) / KT + 1;
  }
  __device__ static __forceinline__ long long tiles_of(const TaParams& p, int b) {
    const long long tiles = (attn_len(p.a, b) + KT - 1) / KT;
    return p.a.heads_kv * (p.row_blocks * tiles + p.tree_tiles);
  }
  __device__ __forceinline__ bool next(const TaParams& p, TaSeg& s) {
    while (t < hi) {
      s.len = (int)attn_len(p.a, b);
      s.p_tiles = (s.len + KT - 1) / KT;
      const long long per_head = (long long)p.row_blocks * s.p_tiles + p.tree_tiles;
      long long off = t - b_start;
      if (off >= p.a.heads_kv * per_head) {
        b_start += p.a.heads_kv * per_head;
        ++b;
        continue;
      }
      s.b = b;
      s.g = (int)(off / per_head);
      off -= s.g * per_head;
      s.rb = 0;
      int n;
      while (true) {
        n = s.p_tiles + tree_tiles(p, (long long)(s.rb + 1) * p.group_ctas * TA_ROWS);
        if (off < n) break;
        off -= n;
        ++s.rb;
      }
      s.begin = (int)off;
      s.end = n - s.begin < hi - t ? n : (int)(s.begin + (hi - t));
      s.whole = s.begin == 0 && s.end == n;
      s.which = first ? 0 : 1;
      first = false;
      t += s.end - s.begin;
      const long long row0 = ((long long)s.rb * p.group_ctas + blockIdx.x % p.group_ctas) * TA_ROWS;
      s.rows = row0 < p.rows;
      s.row0 = (int)row0;
      if (s.rows) {
        const int own = s.p_tiles + tree_tiles(p, row0 + TA_ROWS);  // later tree tiles are above all of this CTA's rows
        if (s.end > own) s.end = own;
        if (s.end < s.begin) s.end = s.begin;
      } else {
        s.end = s.begin;
      }
      return true;
    }
    return false;
  }
};

// ---- the kernel -----------------------------------------------------------------------
template <int DP, bool BF16>
__global__ void __launch_bounds__(TA_THREADS, TaShape<DP>::CTAS) tensor_attention_kernel(const __grid_constant__ TaParams p) {
  using Sh = TaShape<DP>;
  constexpr int KT = Sh::KT, HALVES = DP / 64;
  extern __shared__ char ta_smem[];
  __shared__ alignas(8) uint64_t s_full[Sh::SLOTS], s_empty[Sh::SLOTS], s_q, s_s, s_p, s_o, s_drain;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ unsigned s_odd[2];  // 1 + the last piece (even ones, odd ones) whose tree has values that are not finite
  __shared__ long long s_sum[TA_THREADS / 32], s_b_start;
  __shared__ int s_b;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t ring = (smem_addr(ta_smem) + 1023u) & ~1023u;
  pdl_trigger();
  if (warp == 5) {
    tc_alloc(smem_addr(&s_tmem), Sh::COLS);
  } else if (tid == 0) {
    for (int i = 0; i < Sh::SLOTS; ++i) {
      mbar_init(smem_addr(&s_full[i]), 1);
      mbar_init(smem_addr(&s_empty[i]), 1);
    }
    mbar_init(smem_addr(&s_q), TA_ROWS);
    mbar_init(smem_addr(&s_s), 1);
    mbar_init(smem_addr(&s_p), TA_ROWS);
    mbar_init(smem_addr(&s_o), 1);
    mbar_init(smem_addr(&s_drain), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    s_abort = 0;
    s_odd[0] = s_odd[1] = 0;
    s_b = 0;
    s_b_start = 0;
  }
  pdl_wait();

  // this group's range of tiles, and the sequence in which it begins
  TaWalk<KT> walk;
  const int group = blockIdx.x / p.group_ctas;
  {
    const int per = (p.a.B + TA_THREADS - 1) / TA_THREADS;
    const int b0 = tid * per, b1 = b0 + per < p.a.B ? b0 + per : p.a.B;
    long long mine = 0;
    for (int b = b0; b < b1; ++b) mine += TaWalk<KT>::tiles_of(p, b);
    long long upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(FULL, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) s_sum[warp] = upto;
    __syncthreads();
    long long total = 0;
    for (int w = 0; w < TA_THREADS / 32; ++w) {
      if (w < warp) upto += s_sum[w];
      total += s_sum[w];
    }
    long long groups = (total + p.min_tiles - 1) / p.min_tiles;
    if (groups > p.groups) groups = p.groups;
    const long long lo = group < groups ? total * group / groups : total;
    const long long hi = group < groups ? total * (group + 1) / groups : total;
    if (lo < hi && upto - mine <= lo && lo < upto) {
      long long at = upto - mine;
      for (int b = b0; b < b1; ++b) {
        const long long n = TaWalk<KT>::tiles_of(p, b);
        if (lo < at + n) {
          s_b = b;
          s_b_start = at;
          break;
        }
        at += n;
      }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    walk.t = lo;
    walk.hi = hi;
    walk.b = s_b;
    walk.b_start = s_b_start;
    walk.first = true;
    if (tid == 0 && blockIdx.x % p.group_ctas == 0) {
      // the pair in which the range ends, if it began here and goes on in the next groups
      TaRecord r;
      r.n_parts = 0;
      r.first_which = r.b = r.g = r.rb = 0;
      if (lo < hi && group + 1 < groups) {
        TaWalk<KT> w = walk;
        TaSeg s;
        long long from = w.t;
        while (w.next(p, s)) {
          const int n = s.p_tiles + TaWalk<KT>::tree_tiles(p, (long long)(s.rb + 1) * p.group_ctas * TA_ROWS);
          if (w.t == hi && s.begin == 0 && hi - from < n) {
            r.n_parts = (int)(((from + n) * groups - 1) / total) - group + 1;
            r.first_which = s.which;
            r.b = s.b;
            r.g = s.g;
            r.rb = s.rb;
          }
          from = w.t;
        }
      }
      p.records[group] = r;
    }
  }
  const uint32_t tmem = s_tmem;
  volatile int* abort_flag = &s_abort;
  const unsigned limit = p.wait_limit;
  auto wait = [&](uint32_t bar, uint32_t parity) {
    if (limit && mbar_try_wait(bar, parity)) return true;
    if (mbar_wait_bounded(bar, parity, abort_flag, limit)) return true;
    *abort_flag = 1;
    return false;
  };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(FULL, wait(bar, parity)); };
  const uint32_t bar_full = smem_addr(s_full), bar_empty = smem_addr(s_empty), bar_q = smem_addr(&s_q), bar_s = smem_addr(&s_s),
                 bar_p = smem_addr(&s_p), bar_o = smem_addr(&s_o);

  if (warp == 4) {
    // ---- copies: a lane per box (rows of one page x 64 elements) -------------------------
    const int n_boxes = KT / p.box_rows;
    const int half = lane % HALVES, box = lane / HALVES;
    TaSeg s;
    unsigned it = 0, slot = 0, phase = 1;  // phase: parity of the wait for the slot's last use
    bool ok = true;
    while (ok && walk.next(p, s)) {
      auto page_of = [&](int j) {  // the page that this lane's box of tile j lies in; -1: none
        const int pos = j * KT + box * p.box_rows;
        if (j >= s.p_tiles || box >= n_boxes || pos >= s.len) return -1;
        const int page = __ldg(p.a.table + (long long)s.b * p.a.cols + pos / p.a.page);
        return page >= 0 && page < p.a.pages ? page : p.a.pages;  // past the pool: the copy unit fills in zeros
      };
      int page_next = s.begin < s.end ? page_of(s.begin) : -1;
      for (int j = s.begin; ok && j < s.end; ++j) {
        const int page = page_next;
        if (j + 1 < s.end) page_next = page_of(j + 1);
        const bool tree = j >= s.p_tiles;
        int boxes = 1;
        if (!tree) {
          const int left = s.len - j * KT;
          boxes = left >= KT ? n_boxes : (left + p.box_rows - 1) / p.box_rows;
        }
        const uint32_t bytes = tree ? Sh::SLOT : (uint32_t)(boxes * HALVES * p.box_rows * 128);
        const int row = box * p.box_rows;
        const int in_page = tree ? 0 : (j * KT + row) % p.a.page;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv, ++it) {
          ok = wait_warp(bar_empty + 8 * slot, phase);
          if (!ok) break;
          const uint32_t bar = bar_full + 8 * slot;
          if (lane == 0) mbar_expect_tx(bar, bytes);
          __syncwarp();
          const uint32_t dst = ring + slot * Sh::SLOT + half * (KT * 128);
          if (tree) {
            if (lane < HALVES) tma_load_4d(dst, kv ? &p.tree_v : &p.tree_k, bar, half * 64, (j - s.p_tiles) * KT, s.g, s.b);
          } else if (page >= 0) {
            tma_load_4d(dst + row * 128, kv ? &p.cache_v : &p.cache_k, bar, half * 64, in_page, s.g, page);
          }
          if (++slot == Sh::SLOTS) slot = 0, phase ^= 1u;
        }
      }
    }
    if (!ok && lane == 0) {  // copies in flight land before the block ends
      for (unsigned i = it > Sh::SLOTS ? it - Sh::SLOTS : 0; i < it; ++i)
        for (unsigned spin = 0; spin < SPIN_LIMIT && !mbar_try_wait(smem_addr(&s_full[i % Sh::SLOTS]), (i / Sh::SLOTS) & 1u); ++spin) {}
    }
    __syncwarp();
  } else if (warp == 5) {
    // ---- products -----------------------------------------------------------------------
    constexpr uint32_t IDESC_S = mma_desc(BF16, false, KT), IDESC_O = mma_desc(BF16, true, DP);
    TaSeg s;
    uint32_t slot = 0, phase = 0, tile_phase = 0, seg_phase = 0;
    const uint32_t elected = elect_one(), base = __shfl_sync(FULL, tmem, 0);
    const uint32_t k_desc = smem_desc_lo(ring, 16), v_desc = smem_desc_lo(ring, KT * 128);
    const uint32_t d_s = base + Sh::COL_S, d_o = base + Sh::COL_O, a_q = base + Sh::COL_Q;
    bool ok = true;
    while (ok && walk.next(p, s)) {
      const int tiles = __shfl_sync(FULL, s.end - s.begin, 0);
      if (tiles <= 0) continue;
      ok = wait_warp(bar_q, seg_phase);
      seg_phase ^= 1u;
      for (int j = 0; ok && j < tiles; ++j, tile_phase ^= 1u) {
        ok = wait_warp(bar_full + 8 * slot, phase);
        if (!ok) break;
        tc_fence_after();
        const uint32_t bk = k_desc + slot * (Sh::SLOT >> 4);
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          tc_mma(d_s, a_q + k * 8, bk + (((k >> 2) * (KT * 128) + (k & 3) * 32) >> 4), SMEM_DESC_HI, IDESC_S, k > 0, elected);
        tc_commit(bar_s, elected);
        tc_commit(bar_empty + 8 * slot, elected);
        if (++slot == Sh::SLOTS) slot = 0, phase ^= 1u;
        ok = wait_warp(bar_full + 8 * slot, phase) && wait_warp(bar_p, tile_phase);
        if (!ok) break;
        tc_fence_after();
        const uint32_t bv = v_desc + slot * (Sh::SLOT >> 4);
#pragma unroll
        for (int k = 0; k < KT / 16; ++k) tc_mma(d_o, d_s + k * 8, bv + k * (2048 >> 4), SMEM_DESC_HI, IDESC_O, k > 0 || j > 0, elected);
        if (j + 1 == tiles) tc_commit(bar_o, elected);
        tc_commit(bar_empty + 8 * slot, elected);
        if (++slot == Sh::SLOTS) slot = 0, phase ^= 1u;
      }
    }
    if (!ok) {  // products in flight end before tensor memory is given back
      tc_commit(smem_addr(&s_drain), elected);
      for (unsigned spin = 0; spin < SPIN_LIMIT && !mbar_try_wait(smem_addr(&s_drain), 0); ++spin) {}
    }
    __syncwarp();
  } else {
    // ---- softmax: thread = row ------------------------------------------------------------
    const uint32_t my = tmem + ((uint32_t)(warp * 32) << 16);
    const float scale2 = p.a.scale2;
    // The next piece's rows are read into tensor memory as soon as this piece's last scores are there, before its result
    // is written: so the first product of the next piece runs beside that.
    TaSeg s, s_next;
    unsigned n = 0, n_seg = 0;
    bool ok = true;
    auto row_of = [&](const TaSeg& s, int& u, int& h) {
      const int r = s.row0 + tid;
      const bool in = r < p.rows;
      u = in ? r / p.a.group : 0;
      h = s.g * p.a.group + (in ? r - u * p.a.group : 0);
      return in;
    };
    auto next_piece = [&](TaSeg& s) {  // the next one with keys
      while (walk.next(p, s)) {
        if (!s.rows) continue;
        if (s.begin < s.end) return true;
        const long long part = ((long long)blockIdx.x * 2 + s.which) * p.part_rows + tid;
        if (s.row0 + tid < p.rows) p.part_ml[part] = make_float2(-INFINITY, 0.0f);  // a piece of others that this CTA's rows do not see
      }
      return false;
    };
    auto load_q = [&](const TaSeg& s) {
      if (s.row0 + warp * 32 < p.rows) {
        int u, h;
        const bool in = row_of(s, u, h);
        const uint4* src = reinterpret_cast<const uint4*>(
            p.a.q + 2 * ((long long)s.b * p.a.q_stride[0] + (long long)u * p.a.q_stride[1] + (long long)h * p.a.q_stride[2]));
#pragma unroll
        for (int hh = 0; hh < HALVES; ++hh) {
          uint32_t w[32];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (in && hh * 64 + c * 8 < p.a.dim) v = __ldg(src + hh * 8 + c);
            w[4 * c] = v.x;
            w[4 * c + 1] = v.y;
            w[4 * c + 2] = v.z;
            w[4 * c + 3] = v.w;
          }
          tc_st32(my + Sh::COL_Q + hh * 32, w);
        }
        tc_wait_st();
      }
      tc_fence_before();
      mbar_arrive(bar_q);
    };
    bool more = next_piece(s);
    if (more) load_q(s);
    for (; more; s = s_next) {
      int u, h;
      const bool in = row_of(s, u, h);
      const bool warp_in = s.row0 + warp * 32 < p.rows;
      const bool live = in && !(p.a.tree && p.a.tree[(long long)s.b * p.a.N + u] < 0);
      float m = -INFINITY, l = 0.0f;
      bool odd = false;
      if (ok) {
        for (int j = s.begin; j < s.end; ++j, ++n) {
          const bool tree = j >= s.p_tiles;
          const int left = s.len - j * KT;  // cached tokens from this tile on
          const bool partial = !tree && left < KT;
          if (tree || partial) {
            // Values that no row sees must not enter the product, 0 times them included: those past the text's end
            // become zero.  In the tree some rows may see what others do not: there, elements that are not finite become
            // zero and are added at the end to the rows that do see them.
            const unsigned iv = 2 * n + 1, slot = iv % Sh::SLOTS;
            ok = wait_warp(bar_full + 8 * slot, (iv / Sh::SLOTS) & 1u);
            if (!ok) break;
            char* v0 = ta_smem + (ring - smem_addr(ta_smem)) + slot * Sh::SLOT;
            if (partial) {
              for (int i = left * 8 + tid; i < KT * 8; i += TA_ROWS)
#pragma unroll
                for (int hh = 0; hh < HALVES; ++hh) *reinterpret_cast<uint4*>(v0 + hh * (KT * 128) + i * 16) = make_uint4(0, 0, 0, 0);
            } else {
              constexpr uint32_t EXP = BF16 ? 0x7F80u : 0x7C00u;
              const int nodes = p.a.N - (j - s.p_tiles) * KT, pieces = (nodes < KT ? nodes : KT) * 8;  // the rest are zeros
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
                  s_odd[n_seg & 1] = n_seg + 1;
                }
              }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          }
          ok = wait_warp(bar_s, n & 1u);
          if (!ok) break;
          tc_fence_after();
          if (warp_in) {
            uint32_t x[KT / 32][32];
#pragma unroll
            for (int c = 0; c < KT / 32; ++c) tc_ld32(x[c], my + Sh::COL_S + c * 32);
            tc_wait_ld();
            if (tree || partial) {
#pragma unroll
              for (int c = 0; c < KT / 32; ++c) {
                uint32_t seen;
                if (tree) {
                  const int first = (j - s.p_tiles) * KT + c * 32, below = u + 1 - first;  // nodes first .. u
                  seen = below >= 32 ? FULL : (below > 0 ? (1u << below) - 1 : 0u);
                  if (p.a.mask && seen)
                    seen &= __ldg(p.a.mask + (long long)s.b * p.a.mask_stride + (long long)u * p.a.mask_words + (first >> 5));
                } else {
                  const int below = left - c * 32;
                  seen = below >= 32 ? FULL : (below > 0 ? (1u << below) - 1 : 0u);
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) x[c][i] = seen >> i & 1u ? x[c][i] : 0xFF800000u;
              }
            }
            float top = -INFINITY, top1 = -INFINITY;
#pragma unroll
            for (int c = 0; c < KT / 32; ++c)
#pragma unroll
              for (int i = 0; i < 32; i += 4) {
                top = max3(top, __uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1]));
                top1 = max3(top1, __uint_as_float(x[c][i + 2]), __uint_as_float(x[c][i + 3]));
              }
            top = fmaxf(top, top1) * scale2;
            // Any m near the maximum will do, since o and l carry the same factor: it is left where it is until scores
            // pass it by TA_SLACK, so that o is seldom read, scaled and written (weights up to 2^8 lose nothing in
            // either 16-bit type, sums are fp32).
            if (__any_sync(FULL, top > m + TA_SLACK)) {
              const float raised = fmaxf(m, top);
              const float keep = raised == -INFINITY ? 1.0f : ta_ex2(m - raised);
              m = raised;
              l *= keep;
              if (j > s.begin) {
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
            const float base = m == -INFINITY ? 0.0f : m;
            float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
            for (int c = 0; c < KT / 64; ++c) {
              uint32_t w[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) {
                const int at = 2 * i;
                const float a = ta_ex2(fmaf(__uint_as_float(x[2 * c + at / 32][at % 32]), scale2, -base));
                const float b = ta_ex2(fmaf(__uint_as_float(x[2 * c + at / 32][at % 32 + 1]), scale2, -base));
                sum0 += a;
                sum1 += b;
                w[i] = ta_pack<BF16>(a, b);
              }
              tc_st32(my + Sh::COL_S + c * 32, w);
            }
            l += sum0 + sum1;
            tc_wait_st();
          }
          tc_fence_before();
          mbar_arrive(bar_p);
        }
      }
      more = next_piece(s_next);
      if (ok) {
        if (more) load_q(s_next);
        ok = wait_warp(bar_o, n_seg & 1u);
        tc_fence_after();
        odd = ok && s_odd[n_seg & 1] == n_seg + 1;
        ++n_seg;
      }
      if (!warp_in) continue;
      // ---- the piece's result ---------------------------------------------------------------
      if (!ok) l = NAN;  // a wait ran out: nothing of this piece is to be trusted
      const long long row = ((long long)s.b * p.a.N + u) * p.a.heads_q + h;
      const long long part = ((long long)blockIdx.x * 2 + s.which) * p.part_rows + tid;
      const bool empty = !live || l == 0.0f;
      const float inv = !ok ? NAN : (empty ? 0.0f : 1.0f / l);
      if (in) {
        if (!s.whole) p.part_ml[part] = live || !ok ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
        else if (p.a.lse) p.a.lse[row] = !ok ? NAN : (empty ? -INFINITY : 0.6931471805599453f * (m + log2f(l)));
      }
#pragma unroll 1
      for (int c = 0; c < DP / 32; ++c) {
        uint32_t o[32];
        if (ok) {
          tc_ld32(o, my + Sh::COL_O + c * 32);
          tc_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0;
        }
        if (!in) continue;
        if (odd && live) {
          const int n0 = (s.begin > s.p_tiles ? s.begin - s.p_tiles : 0) * KT;
          const int n1 = s.end > s.p_tiles ? (s.end - s.p_tiles) * KT : 0;
          for (int v = n0; v < n1 && v <= u; ++v) {
            if (!attn_sees(p.a, s.b, u, v)) continue;
            const unsigned short* src = reinterpret_cast<const unsigned short*>(p.a.v) + (long long)s.b * p.a.kv_stride[0] +
                                        (long long)v * p.a.kv_stride[1] + (long long)s.g * p.a.kv_stride[2] + c * 32;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              if (c * 32 + i >= p.a.dim) break;
              const unsigned short raw = src[i];
              const float f = BF16 ? __uint_as_float((uint32_t)raw << 16) : __half2float(__ushort_as_half(raw));
              if (!isfinite(f)) o[i] = __float_as_uint(__uint_as_float(o[i]) + f);
            }
          }
        }
        if (!s.whole) {
          float4* dst = reinterpret_cast<float4*>(p.part_o + part * DP + c * 32);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            dst[i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]),
                                 __uint_as_float(o[4 * i + 3]));
        } else {
          uint4* dst = reinterpret_cast<uint4*>(p.a.out + 2 * (row * p.a.dim + c * 32));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float lo = empty && ok ? 0.0f : __uint_as_float(o[8 * i + 2 * e]) * inv;
              const float hi = empty && ok ? 0.0f : __uint_as_float(o[8 * i + 2 * e + 1]) * inv;
              w[e] = ta_pack<BF16>(lo, hi);
            }
            if (c * 32 + i * 8 < p.a.dim) dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
      tc_fence_before();
    }
  }
  __syncthreads();
  if (warp == 5) tc_dealloc(tmem, Sh::COLS);
}

// ---- joining the pieces ---------------------------------------------------------------
constexpr int TJ_WARPS = 8;

// One warp per row: the factors 2^(m_i - M) of the pieces by lane, then the sum over the pieces of factor * o, each lane
// DP / 32 elements.  The pieces were written just before and come from L2.
template <int DP, bool BF16> __global__ void __launch_bounds__(TJ_WARPS * 32) join_attention_kernel(const __grid_constant__ TaParams p) {
  constexpr int E = DP / 32;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const TaRecord rec = p.records[blockIdx.x];
  if (rec.n_parts == 0) return;
  const int tiles_y = (p.part_rows + TJ_WARPS - 1) / TJ_WARPS;
  const int rt = blockIdx.y / tiles_y, in_tile = (blockIdx.y % tiles_y) * TJ_WARPS + warp;
  const long long r = ((long long)rec.rb * p.group_ctas + rt) * TA_ROWS + in_tile;
  if (in_tile >= p.part_rows || r >= p.rows) return;
  auto at = [&](int i) {  // row of piece i in scratch
    const long long cta = (long long)(blockIdx.x + i) * p.group_ctas + rt;
    return (cta * 2 + (i == 0 ? rec.first_which : 0)) * p.part_rows + in_tile;
  };
  float top = -INFINITY;
  for (int i = lane; i < rec.n_parts; i += 32) top = fmaxf(top, p.part_ml[at(i)].x);
  top = warp_max_f(top);
  const float base = top == -INFINITY ? 0.0f : top;
  float total = 0.0f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  for (int i0 = 0; i0 < rec.n_parts; i0 += 32) {
    const int n = rec.n_parts - i0 < 32 ? rec.n_parts - i0 : 32;
    float w = 0.0f, l = 0.0f;
    if (lane < n) {
      const float2 ml = p.part_ml[at(i0 + lane)];
      w = ta_ex2(ml.x - base);
      l = ml.y * w;
      if (ml.y == 0.0f) w = 0.0f;
    }
    total += warp_sum_f(l);
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float wi = __shfl_sync(FULL, w, i);
      if (wi == 0.0f) continue;  // no weight; a piece without keys has written no o
      const float* src = p.part_o + at(i0 + i) * DP + lane * E;
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float2 v = *reinterpret_cast<const float2*>(src + e);
        o[e] = fmaf(wi, v.x, o[e]);
        o[e + 1] = fmaf(wi, v.y, o[e + 1]);
      }
    }
  }
  const int u = (int)(r / p.a.group), h = rec.g * p.a.group + (int)(r % p.a.group);
  const long long row = ((long long)rec.b * p.a.N + u) * p.a.heads_q + h;
  const bool empty = total == 0.0f;
  const float inv = empty ? 0.0f : 1.0f / total;
  uint32_t* dst = reinterpret_cast<uint32_t*>(p.a.out + 2 * row * p.a.dim);
#pragma unroll
  for (int e = 0; e < E; e += 2)
    if (lane * E + e < p.a.dim) dst[(lane * E + e) >> 1] = empty ? 0u : ta_pack<BF16>(o[e] * inv, o[e + 1] * inv);
  if (p.a.lse && lane == 0) p.a.lse[row] = empty ? -INFINITY : 0.6931471805599453f * (top + log2f(total));
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

// A tensor [w][z][y][dim] of 16-bit elements (strides in elements) that is copied `rows` y at a time, 64 of dim wide.
inline bool encode_map(CUtensorMap* map, const void* base, bool bf16, int dim, const long long (&n)[3], const long long (&stride)[3], int rows) {
  cuuint64_t dims[4] = {(cuuint64_t)dim, 1, 1, 1}, strides[3];
  for (int i = 0; i < 3; ++i) {
    dims[i + 1] = (cuuint64_t)n[i];
    strides[i] = n[i] == 1 ? 16 : (cuuint64_t)stride[i] * 2;
    if (strides[i] == 0 || (strides[i] & 15) != 0 || strides[i] >= (1ull << 40)) return false;
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)rows, 1, 1}, step[4] = {1, 1, 1, 1};
  return encode_tiled()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base), dims, strides,
                        box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline int tensor_dim(int dim) { return dim <= 64 ? 64 : (dim <= 128 ? 128 : 256); }
inline size_t tensor_scratch_bytes(int rows, int dim) {
  const size_t dp = tensor_dim(dim), ctas = dp == 256 ? TA_SMS : 2 * TA_SMS, part_rows = rows < TA_ROWS ? rows : TA_ROWS;
  const size_t pieces = ctas * 2 * part_rows;
  return ctas * sizeof(TaRecord) + ((pieces * sizeof(float2) + 255) & ~(size_t)255) + pieces * dp * sizeof(float);
}

// STAND_E_ARG: not a call for these kernels (alignment, or what the copy unit cannot address); nothing was launched.
template <int DP, bool BF16> int launch_tensor_attention(const AttnParams& a, void* scratch, int sms, unsigned wait_limit, cudaStream_t st) {
  using Sh = TaShape<DP>;
  TaParams p;
  p.a = a;
  const long long rows = (long long)a.N * a.group;
  p.rows = (int)rows;
  const int row_tiles = (int)((rows + TA_ROWS - 1) / TA_ROWS);
  p.row_blocks = (row_tiles + TA_GROUP - 1) / TA_GROUP;
  p.group_ctas = (row_tiles + p.row_blocks - 1) / p.row_blocks;
  p.row_blocks = (row_tiles + p.group_ctas - 1) / p.group_ctas;
  p.tree_tiles = 0;
  for (int rb = 0; rb < p.row_blocks; ++rb) {
    long long end = (long long)(rb + 1) * p.group_ctas * TA_ROWS;
    if (end > rows) end = rows;
    p.tree_tiles += (end - 1) / a.group / Sh::KT + 1;
  }
  p.min_tiles = 4;
  p.groups = (sms < TA_SMS ? sms : TA_SMS) * Sh::CTAS / p.group_ctas;
  const long long most = (long long)a.B * a.heads_kv * (p.row_blocks * (((long long)a.cols * a.page + Sh::KT - 1) / Sh::KT) + p.tree_tiles);
  if (p.groups > (most + p.min_tiles - 1) / p.min_tiles) p.groups = (int)((most + p.min_tiles - 1) / p.min_tiles);
  p.box_rows = 16;
  while (p.box_rows < Sh::KT && a.page % (p.box_rows * 2) == 0) p.box_rows *= 2;
  p.part_rows = rows < TA_ROWS ? (int)rows : TA_ROWS;
  p.wait_limit = wait_limit;

  char* at = (char*)scratch;
  const size_t ctas = DP == 256 ? TA_SMS : 2 * TA_SMS, pieces = ctas * 2 * p.part_rows;
  p.records = (TaRecord*)at;
  at += ctas * sizeof(TaRecord);
  p.part_ml = (float2*)at;
  at += (pieces * sizeof(float2) + 255) & ~(size_t)255;
  p.part_o = (float*)at;

  const long long tree_n[3] = {a.N, a.heads_kv, a.B}, tree_stride[3] = {a.kv_stride[1], a.kv_stride[2], a.kv_stride[0]};
  if (!encode_map(&p.tree_k, a.k, BF16, a.dim, tree_n, tree_stride, Sh::KT) || !encode_map(&p.tree_v, a.v, BF16, a.dim, tree_n, tree_stride, Sh::KT))
    return STAND_E_ARG;
  if (a.cols > 0) {
    const long long n[3] = {a.page, a.heads_kv, a.pages}, stride[3] = {a.cache_stride[2], a.cache_stride[1], a.cache_stride[0]};
    if (a.pages < 1 || !encode_map(&p.cache_k, a.cache_k, BF16, a.dim, n, stride, p.box_rows) ||
        !encode_map(&p.cache_v, a.cache_v, BF16, a.dim, n, stride, p.box_rows))
      return STAND_E_ARG;
  } else {  // no cache: never read
    p.cache_k = p.tree_k;
    p.cache_v = p.tree_v;
  }
  static SmemLimit limit;
  int rc = limit.raise(tensor_attention_kernel<DP, BF16>, Sh::SMEM);
  if (rc) return STAND_E_CUDA;
  rc = launch_dependent(tensor_attention_kernel<DP, BF16>, dim3((unsigned)(p.groups * p.group_ctas)), TA_THREADS, st, p, Sh::SMEM);
  if (rc) return rc;
  const unsigned tiles_y = (unsigned)((p.part_rows + TJ_WARPS - 1) / TJ_WARPS);
  return launch_dependent(join_attention_kernel<DP, BF16>, dim3((unsigned)p.groups, tiles_y * p.group_ctas), TJ_WARPS * 32, st, p);
}

// Rows and strides of 16-byte pieces; a dimension of extent 1 may have any stride.
inline bool tensor_takes(const AttnParams& a, int dtype) {
  if (dtype == STAND_DTYPE_F32 || a.dim % 8 != 0 || !encode_tiled()) return false;
  uintptr_t bits = (uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.out;
  if (a.cols > 0) bits |= (uintptr_t)a.cache_k | (uintptr_t)a.cache_v;
  if (bits & 15) return false;
  const long long n[3] = {a.B, a.N, a.heads_q};
  for (int i = 0; i < 3; ++i)
    if (n[i] > 1 && a.q_stride[i] % 8 != 0) return false;
  return true;
}

}  // namespace stand
