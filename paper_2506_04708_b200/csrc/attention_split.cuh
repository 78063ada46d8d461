// How the keys of all pairs are shared out over the GPU, and how the pieces are joined: common to the attention kernels.
//
// The keys of a (sequence, key head) pair - the cached ones, then the tree's - are cut into tiles of TA_KT, its rows
// (nodes x query heads) into row tiles.  Up to TA_GROUP row tiles of a pair are walked by a group of as many CTAs at the
// same time.  All tiles of all pairs, end to end, are cut into equal ranges, one per group; the lengths are read on the
// device, so the host need not know them.  A range may begin and end inside a pair: such pieces leave (m, l, o) in scratch
// and join_attention_kernel makes the rows of them.
#pragma once
#include "attention.cuh"
#include "launch.cuh"

namespace stand {

constexpr int TA_SMS = 148;               // B200; scratch is laid out for that many
constexpr int TA_GROUP = 4;               // row tiles that walk together, at most
constexpr int TA_KT = 64;                 // keys per tile
// Fewest tiles worth a CTA of their own.  With 1, 2, 3, 4: one token over 700 (32 / 8 heads of 128) 10.9, 11.0, 11.9, 14.0 us; one over
// 3,000 (28 / 4 heads) 17.4, 13.4, 13.0, 13.9; 4 x 8 nodes over 300 (8 / 2 heads) 10.0, 12.5, 13.7, 14.2.
constexpr int TA_MIN_TILES = 2;

struct TaRecord {  // what the joining kernel has to do for the last pair that a group began
  int n_parts;     // 0: nothing (that pair ends within the group)
  int first_which, b, g, rb;
  int pad[3];
};

struct TaSplit {
  AttnParams a;
  int rows;              // of a pair: N * group
  int tile_rows;         // of a row tile: rows of a piece in scratch
  int row_blocks;        // groups of row tiles
  int group_ctas;        // row tiles per group
  int groups;
  int piece_cost;        // what beginning and ending a piece costs, in tiles
  long long tree_tiles;  // sum over the row blocks of a pair
  TaRecord* records;
  float2* part_ml;
  float* part_o;         // rows of DP
};

// ---- the walk over a group's range of tiles -----------------------------------------
struct TaSeg {
  int b, g, rb, row0;      // pair, row block, first row of this CTA
  int len, p_tiles;        // cached tokens, their tiles
  int begin, end;          // this CTA's tiles of the pair (cached ones, then the tree's)
  int whole;               // the range covers the pair
  int rows;                // the CTA has rows in this block
  int which;               // the group's first piece or a later one
  int starts, units;       // the pair begins in this group's range; its length there (cost and tiles)
};

struct TaWalk {
  long long t, hi, b_start;
  int b, cost;  // cost: of a piece, in tiles
  bool first;

  // tree tiles that rows before row_end see
  __device__ static __forceinline__ int tree_tiles(const TaSplit& p, int row_end) {
    return ((row_end < p.rows ? row_end : p.rows) - 1) / p.a.group / TA_KT + 1;
  }
  // tiles of all row blocks of a (sequence, key head)
  __device__ static __forceinline__ long long tiles_of(const TaSplit& p, long long len) {
    return p.row_blocks * ((len + TA_KT - 1) / TA_KT) + p.tree_tiles;
  }
  __device__ __forceinline__ bool next(const TaSplit& p, TaSeg& s) {
    while (t < hi) {
      s.len = (int)attn_len(p.a, b);
      s.p_tiles = (s.len + TA_KT - 1) / TA_KT;
      const long long head = tiles_of(p, s.len) + p.row_blocks * cost;
      long long off = t - b_start;
      if (off >= p.a.heads_kv * head) {
        b_start += p.a.heads_kv * head;
        ++b;
        continue;
      }
      s.b = b;
      s.g = head <= 0x7FFFFFFF && off <= 0x7FFFFFFF ? (int)((uint32_t)off / (uint32_t)head) : (int)(off / head);
      off -= s.g * head;
      s.rb = 0;
      while (true) {
        s.units = cost + s.p_tiles + tree_tiles(p, (s.rb + 1) * p.group_ctas * p.tile_rows);
        if (off < s.units) break;
        off -= s.units;
        ++s.rb;
      }
      const int from = (int)off, to = s.units - from < hi - t ? s.units : (int)(from + (hi - t));
      s.starts = from == 0;
      s.whole = from == 0 && to == s.units;
      s.which = first ? 0 : 1;
      first = false;
      t += to - from;
      s.begin = from > cost ? from - cost : 0;
      s.end = to > cost ? to - cost : 0;
      s.row0 = (s.rb * p.group_ctas + blockIdx.x % p.group_ctas) * p.tile_rows;
      s.rows = s.row0 < p.rows;
      const int own = s.rows ? s.p_tiles + tree_tiles(p, s.row0 + p.tile_rows) : 0;  // later tree tiles are above all of this CTA's rows
      if (s.end > own) s.end = own;
      if (s.end < s.begin) s.end = s.begin;
      return true;
    }
    return false;
  }
};

// Scratch row of `row` of this CTA's piece.
__device__ __forceinline__ long long ta_part_row(const TaSplit& p, const TaSeg& s, int row) {
  return ((long long)blockIdx.x * 2 + s.which) * p.tile_rows + row;
}

template <int THREADS> struct TaRange {
  long long sum[THREADS / 32], b_start, total;
  int b, groups;
};

// Whoever walks over all pieces of a group's first CTA keeps its record: what has to be joined is the pair in which the
// range ends, if it began in the range and goes on in the next groups.
struct TaNote {
  long long from;  // where the piece to come begins
  TaRecord r;

  __device__ __forceinline__ explicit TaNote(const TaWalk& walk) : from(walk.t) { r.n_parts = r.first_which = r.b = r.g = r.rb = 0; }
  __device__ __forceinline__ void piece(const TaWalk& walk, const TaSeg& s, long long total, int groups, int group) {
    if (walk.t == walk.hi && s.starts && walk.hi - from < s.units) {
      r.n_parts = (int)(((from + s.units) * groups - 1) / total) - group + 1;
      r.first_which = s.which;
      r.b = s.b;
      r.g = s.g;
      r.rb = s.rb;
    }
    from = walk.t;
  }
};

// This group's range and the sequence in which it begins.  All threads call it; `before` and `after` run around the second
// of its two barriers.
template <int THREADS, typename F, typename G>
__device__ __forceinline__ void ta_begin(const TaSplit& p, TaWalk& walk, TaRange<THREADS>& sh, F before, G after) {
  const int group = blockIdx.x / p.group_ctas, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int per = (p.a.B + THREADS - 1) / THREADS;
  const int b0 = tid * per, b1 = b0 + per < p.a.B ? b0 + per : p.a.B;
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += p.a.heads_kv * TaWalk::tiles_of(p, attn_len(p.a, b));
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(FULL, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sh.sum[warp] = upto;
  __syncthreads();
  long long total = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) upto += sh.sum[w];
    total += sh.sum[w];
  }
  // Where every CTA has enough to do, beginning and ending a piece (its rows, its result) counts as piece_cost tiles, so
  // that a CTA with many short pairs gets fewer tiles.  Where there are few tiles they are shared out as they are.
  const int cost = total >= 4ll * p.groups ? p.piece_cost : 0;
  const long long per_b = (long long)p.a.heads_kv * p.row_blocks * cost;
  total += per_b * p.a.B;
  upto += per_b * b1;
  mine += per_b * (b1 > b0 ? b1 - b0 : 0);
  long long groups = (total + TA_MIN_TILES - 1) / TA_MIN_TILES;
  if (groups > p.groups) groups = p.groups;
  const long long lo = group < groups ? total * group / groups : total;
  const long long hi = group < groups ? total * (group + 1) / groups : total;
  if (lo < hi && upto - mine <= lo && lo < upto) {
    long long at = upto - mine;
    for (int b = b0; b < b1; ++b) {
      const long long n = p.a.heads_kv * TaWalk::tiles_of(p, attn_len(p.a, b)) + per_b;
      if (lo < at + n) {
        sh.b = b;
        sh.b_start = at;
        break;
      }
      at += n;
    }
  }
  if (tid == 0) {  // for whoever keeps the record: read behind the barrier
    sh.total = total;
    sh.groups = (int)groups;
  }
  before();
  __syncthreads();
  after();
  walk.t = lo;
  walk.hi = hi;
  walk.b = sh.b;
  walk.b_start = sh.b_start;
  walk.first = true;
  walk.cost = cost;
}

// ---- packed tiles ---------------------------------------------------------------------
__device__ __forceinline__ void cp_async16_or_zero(uint32_t dst, const void* src, bool there) {  // zeros are written where it is not
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
// The copies of packed tiles by one warp, for both kernels that unpack them.  A stage holds the keys' four lots of 16 tokens (the least part of a page), then
// the values': a lot is 16 rows of codes, then 16 of scales.  Eight lanes copy a lot in 16-byte pieces, so no lane needs another's address; lots
// past the text's end and of pages outside the pool become zeros, which are values of zero.  (By bulk copies, whose operands one
// lane has to gather, this warp took 1,100 - 1,500 cycles a tile and held the others up.)
struct PkCopies {
  const char *k, *v;  // of the pair's head
  const int* table;
  int len, pos, col, in_page, next;

  __device__ __forceinline__ void begin(const AttnParams& a, const TaSeg& s, int lane) {
    k = a.cache_k + s.g * a.cache_stride[1];
    v = a.cache_v + s.g * a.cache_stride[1];
    table = a.table + (long long)s.b * a.cols;
    len = s.len;
    pos = s.begin * TA_KT + (lane >> 3) * 16;
    col = pos / a.page;
    in_page = pos - col * a.page;
    next = pos < len ? __ldg(table + col) : -1;
  }
  // One tile to `to`; DIM: the head size, at most DP.  The barrier, of 32 arrivals, completes when the pieces are there.
  template <int DP> __device__ __forceinline__ void tile(const AttnParams& a, int dim, int lane, uint32_t to, int half, uint32_t bar) {
    const bool there = next >= 0 && next < a.pages;
    const int c = lane & 7;
    const long long block = there ? next * a.cache_stride[0] : 0;
    const int code = (there ? in_page * (dim / 2) : 0) + c * 16, scale = (there ? a.page * (dim / 2) + in_page * (dim / 16) : 0) + c * 16;
    const char *pk = k + block, *pv = v + block;
    pos += TA_KT;
    for (in_page += TA_KT; in_page >= a.page; in_page -= a.page) ++col;
    next = pos < len ? __ldg(table + col) : -1;
    to += (lane >> 3) * 9 * dim + c * 16;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i)
      if (i * 16 < dim) {
        cp_async16_or_zero(to + i * 128, pk + code + i * 128, there);
        cp_async16_or_zero(to + half + i * 128, pv + code + i * 128, there);
      }
#pragma unroll
    for (int i = 0; i < (DP + 127) / 128; ++i)
      if ((c + 8 * i) * 16 < dim) {
        cp_async16_or_zero(to + 8 * dim + i * 128, pk + scale + i * 128, there);
        cp_async16_or_zero(to + half + 8 * dim + i * 128, pv + scale + i * 128, there);
      }
    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
  }
};

// ---- joining the pieces ---------------------------------------------------------------
constexpr int TJ_WARPS = 8;

// One warp per row: the factors 2^(m_i - M) of the pieces by lane, then the sum over the pieces of factor * o, each lane
// DP / 32 elements, eight pieces asked for at a time (one by one the 20 pieces of a long text took 4 us more).  The pieces were
// written just before and come from L2.  About 6 us with its launch; bound by the chain record - m and l - o.
template <int DP, typename T> __global__ void __launch_bounds__(TJ_WARPS * 32) join_attention_kernel(const __grid_constant__ TaSplit p) {
  constexpr int E = DP / 32;
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const TaRecord rec = p.records[blockIdx.x];
  if (rec.n_parts == 0) return;
  const int tiles_y = (p.tile_rows + TJ_WARPS - 1) / TJ_WARPS;
  const int rt = blockIdx.y / tiles_y, in_tile = (blockIdx.y % tiles_y) * TJ_WARPS + warp;
  const int r = (rec.rb * p.group_ctas + rt) * p.tile_rows + in_tile, u = r / p.a.group, h = rec.g * p.a.group + r - u * p.a.group;
  if (in_tile >= p.tile_rows || r >= p.rows) return;
  auto at = [&](int i) {  // row of piece i in scratch
    const long long cta = (long long)(blockIdx.x + i) * p.group_ctas + rt;
    return (cta * 2 + (i == 0 ? rec.first_which : 0)) * p.tile_rows + in_tile;
  };
  // up to 32 pieces: one read of their m and l
  float2 mine = make_float2(-INFINITY, 0.0f);
  if (lane < rec.n_parts) mine = p.part_ml[at(lane)];
  float top = mine.x;
  for (int i = lane + 32; i < rec.n_parts; i += 32) top = fmaxf(top, p.part_ml[at(i)].x);
  top = warp_max_f(top);
  const float base = top == -INFINITY ? 0.0f : top;
  float total = 0.0f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  for (int i0 = 0; i0 < rec.n_parts; i0 += 32) {
    const int n = rec.n_parts - i0 < 32 ? rec.n_parts - i0 : 32;
    if (i0 > 0) mine = lane < n ? p.part_ml[at(i0 + lane)] : make_float2(-INFINITY, 0.0f);
    float w = exp2f(mine.x - base);
    total += warp_sum_f(mine.y * w);
    // A piece without keys has written no o.  Another's weight may be too small for its type: its o may still hold infinities.
    w = mine.y == 0.0f ? 0.0f : fmaxf(w, 1.4e-45f);
    constexpr int AT_ONCE = E > 4 ? 4 : 8;  // pieces whose o is asked for together
    for (int i = 0; i < n; i += AT_ONCE) {
      float wi[AT_ONCE], v[AT_ONCE][E];
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        wi[k] = __shfl_sync(FULL, w, i + k < n ? i + k : i);
        if (i + k >= n) wi[k] = 0.0f;
        const float* src = p.part_o + at(i0 + i + k) * DP + lane * E;
#pragma unroll
        for (int e = 0; e < E; e += 2) {
          float2 t = make_float2(0.0f, 0.0f);
          if (wi[k] != 0.0f) t = *reinterpret_cast<const float2*>(src + e);
          v[k][e] = t.x;
          v[k][e + 1] = t.y;
        }
      }
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = fmaf(wi[k], v[k][e], o[e]);
    }
  }
  const long long row = ((long long)rec.b * p.a.N + u) * p.a.heads_q + h;
  const bool empty = total == 0.0f;
  const float inv = empty ? 0.0f : 1.0f / total;
  T* dst = reinterpret_cast<T*>(p.a.out) + row * p.a.dim + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    o[e] = empty ? 0.0f : o[e] * inv;
    if (lane * E + e < p.a.dim) dst[e] = from_float<T>(o[e]);
  }
  if (p.a.lse && lane == 0) p.a.lse[row] = empty ? -INFINITY : 0.6931471805599453f * (top + log2f(total));
}

template <int DP, typename T> int launch_join(const TaSplit& p, cudaStream_t st) {
  const unsigned tiles_y = (unsigned)((p.tile_rows + TJ_WARPS - 1) / TJ_WARPS);
  return launch_dependent(join_attention_kernel<DP, T>, dim3((unsigned)p.groups, tiles_y * p.group_ctas), TJ_WARPS * 32, st, p);
}

// ---- host ---------------------------------------------------------------------------------
inline int tensor_dim(int dim) { return dim <= 64 ? 64 : (dim <= 128 ? 128 : 256); }
inline size_t ta_scratch_bytes(int tile_rows, int dim, int ctas_per_sm) {
  const size_t ctas = (size_t)TA_SMS * ctas_per_sm, pieces = ctas * 2 * tile_rows;
  return ctas * sizeof(TaRecord) + ((pieces * sizeof(float2) + 255) & ~(size_t)255) + pieces * tensor_dim(dim) * sizeof(float);
}
inline void ta_split(TaSplit& p, const AttnParams& a, int tile_rows, int dp, int sms, int ctas_per_sm, int piece_cost, void* scratch) {
  p.a = a;
  p.rows = a.N * a.group;
  p.tile_rows = tile_rows;
  p.piece_cost = piece_cost;
  const int row_tiles = (p.rows + tile_rows - 1) / tile_rows;
  p.row_blocks = (row_tiles + TA_GROUP - 1) / TA_GROUP;
  p.group_ctas = (row_tiles + p.row_blocks - 1) / p.row_blocks;
  p.row_blocks = (row_tiles + p.group_ctas - 1) / p.group_ctas;
  p.tree_tiles = 0;
  for (int rb = 0; rb < p.row_blocks; ++rb) {
    const long long end = (long long)(rb + 1) * p.group_ctas * tile_rows;
    p.tree_tiles += ((end < p.rows ? end : p.rows) - 1) / a.group / TA_KT + 1;
  }
  p.groups = (sms < TA_SMS ? sms : TA_SMS) * ctas_per_sm / p.group_ctas;
  const long long most = (long long)a.B * a.heads_kv * (p.row_blocks * (((long long)a.cols * a.page + TA_KT - 1) / TA_KT) + p.tree_tiles);
  if (p.groups > (most + TA_MIN_TILES - 1) / TA_MIN_TILES) p.groups = (int)((most + TA_MIN_TILES - 1) / TA_MIN_TILES);
  const size_t ctas = (size_t)TA_SMS * ctas_per_sm, pieces = ctas * 2 * tile_rows;
  char* at = (char*)scratch;
  p.records = (TaRecord*)at;
  at += ctas * sizeof(TaRecord);
  p.part_ml = (float2*)at;
  at += (pieces * sizeof(float2) + 255) & ~(size_t)255;
  p.part_o = (float*)at;
}

}  // namespace stand
