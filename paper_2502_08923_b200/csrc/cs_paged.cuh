// Shared by the operators around the paged KV cache: the handle, what kernels get of a cache and its blocks, and how the
// attention kernels deal their work out.
#pragma once

#include <cuda_fp16.h>

#include "cs_common.cuh"

static constexpr int kPagedMaxCtas = 160;      // CTAs of an attention launch at most
static constexpr int kPagedMaxRows = 256;      // query rows (rows x heads of a group) of one work item at most
static constexpr int kPagedTile = 128;         // keys of a tile, the unit work is dealt out in
static constexpr int kPagedMaxSeqs = 512;      // sequences of one attention launch; more are further launches

struct PagedView {
  char *k, *v;
  long long page_stride, head_stride, slot_stride;   // elements
  int n_pages, page_size, page_shift, n_kv_heads;
};

struct BlocksView {
  const int *start, *len, *kv_len, *table;
  int n_seqs, table_width, rows;
};

// What a CTA leaves for the launch that adds pieces up: the item whose first tiles are its last ones; the CTAs behind it, up to `last`, have the rest (kPagedNone: there is no such item,
// kPagedGaveUp: a wait of this CTA ran out)
struct PagedSplit {
  int last, rows;              // query rows
  int first_row, head, start;  // of the block (row x head of the group), KV head, the block's first row
};
static constexpr int kPagedNone = -1, kPagedGaveUp = -2;

struct cs_paged_cache {
  cs_paged_config cfg;
  PagedView view;
  CUtensorMap tmK, tmV;        // [page][head][slot][dim], boxes of up to 64 dims x up to 128 slots
  void* workspace;
  size_t workspace_bytes;
  int* status;                 // device status word
  int* counters;               // pieces of an item that are done, by the CTA that holds its first tile; 0 between launches
  PagedSplit* splits;          // of the last launch on the tensor cores, by CTA [kPagedMaxCtas]
  float* parts;                // un-normalised pieces [kPagedMaxCtas][2][kPagedMaxRows][head_dim]
  float* parts_ml;             // their (reference point, sum) [kPagedMaxCtas][2][kPagedMaxRows][2]
  int num_sms;
  unsigned attr_set;           // shared-memory opt-ins made, a bit per kernel instance
  unsigned long long wait_limit_ns;
  int drop;                    // test hook: the next tall launch leaves out this K tile of every CTA (-1 = none)
  char err[256];
};

// x / d for 0 <= x < 2^31: the high half of a product, a sum and a shift (Granlund and Montgomery 1994, "Division by invariant integers using multiplication")
struct PagedDivisor {
  unsigned mul, shift;
#ifdef __CUDACC__
  __device__ __forceinline__ int of(int x) const { return (int)((__umulhi((unsigned)x, mul) + (unsigned)x) >> shift); }
#endif
  static PagedDivisor by(unsigned d) {
    unsigned l = 0;
    while ((1ull << l) < d) ++l;
    return PagedDivisor{(unsigned)((((1ull << l) - d) << 32) / d + 1), l};
  }
};

// what an attention launch is about
struct PagedAttnArgs {
  PagedView kv;
  BlocksView blk;
  const char* q;
  long long q_row, q_head;     // strides, elements
  char* out;
  float* lse;
  int n_heads, group;          // query heads, and per KV head
  int mask, window;
  float scale_log2e, scale;
  int item_rows;               // query rows (row of the block x head of the group) per work item
  int item_cost;               // what an item costs beside its tiles, in tiles
  int keep;                    // items of up to so many tiles are not shared where a CTA has no more than that to do
  PagedDivisor by_group, by_item_rows;
  float *parts, *parts_ml;
  int *counters, *status;
  PagedSplit* splits;
  unsigned long long wait_ns;
  int drop;
  // a cache of 4 bits: kv.k and kv.v are its numbers, kv.page_stride bytes; scales, from page to page in elements
  const unsigned short *ks, *vs;
  long long scale_page;
};

cs_status cs_launch_paged_few(cs_paged_cache* c, const PagedAttnArgs& a, cudaStream_t st);
cs_status cs_launch_paged_tc(cs_paged_cache* c, const PagedAttnArgs& a, cudaStream_t st);
cs_status cs_launch_quant_tc(cs_paged_cache* c, const PagedAttnArgs& a, cudaStream_t st);   // over a cache of 4 bits; `c`: type, workspace
cs_status cs_paged_tc_maps(cs_paged_cache* c);   // the pools' operand maps

#ifdef __CUDACC__
namespace {

// What is wrong with a sequence's block (0: nothing).  `own_rows`: its own rows need room in the pages.
__device__ __forceinline__ int paged_block_flag(const BlocksView& s, int page_size, bool own_rows, int start, int len, int kv) {
  if (len < 0 || kv < 0 || (len > 0 && (start < 0 || (long long)start + len > s.rows))) return CS_DEV_BADARG;
  const long long keys = (long long)kv + (own_rows ? len : 0), room = (long long)s.table_width * page_size;
  return len > 0 && (keys > room || (long long)kv + len > 0x7fffff00ll) ? CS_DEV_CAPACITY : 0;
}

// Keys [lo, hi) that rows r0 .. r1 of a block attend to between them.
__device__ __forceinline__ void paged_range(int mask, int window, int len, int kv, int r0, int r1, int& lo, int& hi) {
  hi = mask == CS_MASK_CAUSAL ? kv + r1 + 1 : mask == CS_MASK_PREFIX ? kv : kv + len;
  lo = window > 0 ? max(0, kv + r0 + 1 - window) : 0;
}

// Work is dealt out in key tiles.  An item is one (sequence, KV head, group of item_rows query rows); its tiles are the
// kPagedTile-aligned ones its rows attend to, one at least (a row without keys is written too).  Items in the order
// (sequence, head, row group) make one line, of which every CTA takes an equal run: CTA i of n the places
// [total * i / n, total * (i + 1) / n).  So no CTA waits for another, none has more to do than the others whatever the
// lengths are, and at most two items of a CTA are shared with others.  An item takes item_cost places, in front of one for each
// tile: changing from one to the next costs time as well (64 single tokens over 500 - 4,097 keys of the 8B shape,
// one / two places: 73.1 / 71.9 us; by no place CTAs with many short items ended up to 20 us behind the others).
// places of an item in the line (rows x heads stay below 2^31)
__device__ __forceinline__ int paged_item_places(const PagedAttnArgs& a, int len, int kv, int rg) {
  const int r0 = a.by_group.of(rg * a.item_rows), r1 = min(len - 1, a.by_group.of(rg * a.item_rows + a.item_rows - 1));
  int lo, hi;
  paged_range(a.mask, a.window, len, kv, r0, r1, lo, hi);
  return a.item_cost + (hi > lo ? (hi + kPagedTile - 1) / kPagedTile - lo / kPagedTile : 1);
}
__device__ __forceinline__ int paged_row_groups(const PagedAttnArgs& a, int len) {
  return a.by_item_rows.of(len * a.group + a.item_rows - 1);
}
// (a 64-bit division is some hundred instructions, and nearly always need not be one)
__device__ __forceinline__ long long paged_div(long long x, long long y) {
  return ((x | y) >> 32) == 0 ? (long long)((unsigned)x / (unsigned)y) : x / y;
}

// a block's items of one KV head, by a whole warp: their places together
__device__ __forceinline__ long long paged_block_tiles(const PagedAttnArgs& a, int len, int kv, int lane) {
  const int n = paged_row_groups(a, len);
  long long sum = 0;
  for (int g = lane; g < n; g += 32) sum += paged_item_places(a, len, kv, g);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  return sum;
}

template <int kSeqs>
struct PagedPlanOf {                            // in shared memory; of up to kSeqs sequences
  long long before[kSeqs + 1];                  // places of the sequences before this one
  long long per_head[kSeqs];                    // places of one of its KV heads
  int start[kSeqs], len[kSeqs], kv[kSeqs];
  long long warp_sum[32];
  int tall[kSeqs], n_tall;                      // sequences whose row groups a warp adds up
};
typedef PagedPlanOf<kPagedMaxSeqs> PagedPlan;

// one sequence's block, left out (length 0) if something is wrong with it
template <int kSeqs>
__device__ __forceinline__ void paged_load_block(const PagedAttnArgs& a, PagedPlanOf<kSeqs>& p, int b, bool report, int& len, int& kv) {
  const int start = __ldcg(a.blk.start + b);
  len = __ldcg(a.blk.len + b);
  kv = __ldcg(a.blk.kv_len + b);
  const int flag = paged_block_flag(a.blk, a.kv.page_size, a.mask != CS_MASK_PREFIX, start, len, kv);
  if (flag != 0) {
    if (report && blockIdx.x == 0) atomicOr(a.status, flag);
    len = 0;
  }
  p.start[b] = start; p.len[b] = len; p.kv[b] = kv;
}

// By all threads of a CTA (a multiple of 32, 128 at least).  Up to 32 sequences every warp works the plan out for itself - all write the same - and
// nothing is waited for; else it ends with a barrier.
template <int kSeqs>
__device__ __forceinline__ void paged_plan(const PagedAttnArgs& a, PagedPlanOf<kSeqs>& p) {
  const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31, B = a.blk.n_seqs;
  if (B <= 32) {
    int len = 0, kv = 0, n = 0;
    long long t = 0;
    if (lane < B) {
      paged_load_block(a, p, lane, warp == 0, len, kv);
      n = paged_row_groups(a, len);
      if (n <= 2) for (int g = 0; g < n; ++g) t += paged_item_places(a, len, kv, g);
    }
    for (unsigned tall = __ballot_sync(0xffffffffu, n > 2); tall != 0; tall &= tall - 1) {
      const int b = __ffs(tall) - 1;
      const long long s = paged_block_tiles(a, __shfl_sync(0xffffffffu, len, b), __shfl_sync(0xffffffffu, kv, b), lane);
      if (lane == b) t = s;
    }
    if (lane < B) p.per_head[lane] = t;
    t *= a.kv.n_kv_heads;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long v = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += v;
    }
    if (lane < B) p.before[lane + 1] = t;
    if (lane == 0) p.before[0] = 0;
    __syncwarp();
    return;
  }
  if (tid == 0) p.n_tall = 0;
  __syncthreads();
  for (int b = tid; b < B; b += nt) {
    int len, kv;
    paged_load_block(a, p, b, true, len, kv);
    const int n = paged_row_groups(a, len);
    long long t = 0;
    if (n <= 2) {
      for (int g = 0; g < n; ++g) t += paged_item_places(a, len, kv, g);
    } else {
      p.tall[atomicAdd(&p.n_tall, 1)] = b;
    }
    p.per_head[b] = t;
    p.before[b + 1] = t * a.kv.n_kv_heads;
  }
  __syncthreads();
  for (int i = warp; i < p.n_tall; i += nt >> 5) {
    const int b = p.tall[i];
    const long long t = paged_block_tiles(a, p.len[b], p.kv[b], lane);
    if (lane == 0) { p.per_head[b] = t; p.before[b + 1] = t * a.kv.n_kv_heads; }
  }
  if (tid == 0) p.before[0] = 0;
  __syncthreads();
  // running sums, in the same order whoever takes part: a thread's run, the warp's, the CTA's
  const int per = (B + nt - 1) / nt, first = tid * per, last = min(B, first + per);
  long long run = 0;
  for (int b = first; b < last; ++b) run += p.before[b + 1];
  long long inc = run;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += v;
  }
  if (lane == 31) p.warp_sum[warp] = inc;
  __syncthreads();
  long long at = inc - run;
  for (int w = 0; w < warp; ++w) at += p.warp_sum[w];
  for (int b = first; b < last; ++b) {
    at += p.before[b + 1];
    p.before[b + 1] = at;
  }
  __syncthreads();
}

// A CTA's share of one item.
struct PagedPiece {
  int start, len, kv;          // the block
  int seq, head, rg;
  int lo, hi;                  // keys the item's rows attend to between them
  int tile0, n_tiles;          // first tile (absolute: key / kPagedTile) and how many are this CTA's
  int item_tiles;
  long long item_at;           // where the item begins in the line
  bool opens, whole;           // has the item's first tile; has all of them
};

// Piece that begins at place `at` of the line, by a whole warp (all lanes get it); `end`: where the CTA's run ends.  It may be empty: n_tiles 0.
template <int kSeqs>
__device__ __forceinline__ PagedPiece paged_piece(const PagedAttnArgs& a, const PagedPlanOf<kSeqs>& p, long long at, long long end, int lane) {
  PagedPiece o;
  // the last sequence that begins at or before it (32 at a time)
  const int B = a.blk.n_seqs;
  int b = 0;
  if (B > 32) b = 32 * (__popc(__ballot_sync(0xffffffffu, 32 * lane < B && p.before[min(32 * lane, B)] <= at)) - 1);
  b += __popc(__ballot_sync(0xffffffffu, b + lane < B && p.before[min(b + lane, B)] <= at)) - 1;
  o.seq = b; o.start = p.start[b]; o.len = p.len[b]; o.kv = p.kv[b];
  const long long per_head = p.per_head[b];
  long long rest = at - p.before[b];
  o.head = a.kv.n_kv_heads <= 32 ? __popc(__ballot_sync(0xffffffffu, lane < a.kv.n_kv_heads && (lane + 1) * per_head <= rest)) : (int)paged_div(rest, per_head);
  rest -= o.head * per_head;
  // row group: 32 at a time
  const int n = paged_row_groups(a, o.len);
  int g0 = 0, places = (int)per_head;
  for (; n > 1; g0 += 32) {
    const int t = g0 + lane < n ? paged_item_places(a, o.len, o.kv, g0 + lane) : 0;
    int inc = t;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, s);
      if (lane >= s) inc += v;
    }
    const unsigned ends_behind = __ballot_sync(0xffffffffu, (long long)inc > rest);
    if (ends_behind != 0 || g0 + 32 >= n) {
      const int l = ends_behind != 0 ? __ffs(ends_behind) - 1 : 0;
      places = __shfl_sync(0xffffffffu, t, l);
      rest -= __shfl_sync(0xffffffffu, inc, l) - places;
      g0 += l;
      break;
    }
    rest -= __shfl_sync(0xffffffffu, inc, 31);
  }
  o.rg = g0;
  const int r0 = a.by_group.of(g0 * a.item_rows), r1 = min(o.len - 1, a.by_group.of(g0 * a.item_rows + a.item_rows - 1));
  paged_range(a.mask, a.window, o.len, o.kv, r0, r1, o.lo, o.hi);
  o.item_tiles = places - a.item_cost;
  o.item_at = at - rest;
  const int skip = max(0, (int)rest - a.item_cost);            // tiles that the CTAs before have
  o.tile0 = (o.hi > o.lo ? o.lo / kPagedTile : 0) + skip;
  o.n_tiles = (int)min((long long)(o.item_tiles - skip), max(0ll, end - o.item_at - a.item_cost - skip));
  o.opens = skip == 0;
  o.whole = o.n_tiles == o.item_tiles;
  return o;
}
// The piece after one, if the CTA's run goes on behind it.
template <int kSeqs>
__device__ __forceinline__ bool paged_next(const PagedAttnArgs& a, const PagedPlanOf<kSeqs>& plan, PagedPiece& p, long long end) {
  const long long at = p.item_at + p.item_tiles + a.item_cost;
  if (at + a.item_cost >= end) return false;
  if (p.rg + 1 < paged_row_groups(a, p.len)) ++p.rg;
  else {
    p.rg = 0;
    if (++p.head == a.kv.n_kv_heads) {
      p.head = 0;
      do ++p.seq; while (plan.before[p.seq + 1] <= at);
      p.start = plan.start[p.seq]; p.len = plan.len[p.seq]; p.kv = plan.kv[p.seq];
    }
  }
  const int r0 = a.by_group.of(p.rg * a.item_rows), r1 = min(p.len - 1, a.by_group.of(p.rg * a.item_rows + a.item_rows - 1));
  paged_range(a.mask, a.window, p.len, p.kv, r0, r1, p.lo, p.hi);
  p.tile0 = p.hi > p.lo ? p.lo / kPagedTile : 0;
  p.item_tiles = p.hi > p.lo ? (p.hi + kPagedTile - 1) / kPagedTile - p.tile0 : 1;
  p.item_at = at;
  p.n_tiles = (int)min((long long)p.item_tiles, end - at - a.item_cost);
  p.opens = true;
  p.whole = p.n_tiles == p.item_tiles;
  return true;
}
// The CTA (of n) whose run holds place x of a line of `total`; the first and the last one of an item's CTAs.
__device__ __forceinline__ int paged_owner(long long x, long long total, int n) { return (int)paged_div((x + 1) * n - 1, total); }

__device__ __forceinline__ int paged_first_cta(const PagedAttnArgs& a, const PagedPiece& p, long long total, int n) { return paged_owner(p.item_at + a.item_cost, total, n); }
__device__ __forceinline__ int paged_last_cta(const PagedAttnArgs& a, const PagedPiece& p, long long total, int n) { return paged_owner(p.item_at + a.item_cost + p.item_tiles - 1, total, n); }

// The first piece of a CTA's run, by a whole warp, and where the run ends; empty (n_tiles 0) if there is nothing to do.  Where CTAs have little to do, items of up to `keep` tiles are left
// to the CTA that has the last place of them: reading a few more tiles takes less time than adding pieces up.  (The small model's 11 rows over 512 keys, five
// tiles a head, cut / whole: 8.7 / 7.9 us.)
template <int kSeqs>
__device__ __forceinline__ PagedPiece paged_run(const PagedAttnArgs& a, const PagedPlanOf<kSeqs>& plan, long long total, int n_cta, int cta, int lane, long long& end) {
  const long long begin = paged_div(total * cta, n_cta);
  end = paged_div(total * (cta + 1), n_cta);
  PagedPiece p = paged_piece(a, plan, begin, end, lane);
  if (total > (long long)gridDim.x * a.keep) return p;
  PagedPiece q = p;
  for (;;) {                                     // the item that the run ends in
    const long long behind = q.item_at + a.item_cost + q.item_tiles;
    if (end < behind && q.item_tiles <= a.keep) end = q.item_at;
    if (end <= behind || !paged_next(a, plan, q, total)) break;
  }
  if (p.item_tiles <= a.keep) {
    p.tile0 = p.hi > p.lo ? p.lo / kPagedTile : 0;
    p.opens = p.whole = true;
    p.n_tiles = end > p.item_at ? p.item_tiles : 0;
  } else {
    // (the end may have moved to the end of this item)
    p.whole = p.n_tiles == p.item_tiles;
  }
  return p;
}

// 2^x, hardware approximation (relative error about 2^-22; -inf gives 0)
__device__ __forceinline__ float paged_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float paged_lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// two fp32 values in one 64-bit register and the packed fp32 arithmetic of this architecture
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack2(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(f32x2 r, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(r)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <typename T> struct PagedType;
template <> struct PagedType<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
};
template <> struct PagedType<__half> {
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ float2 unpack(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
};

}  // namespace
#endif
