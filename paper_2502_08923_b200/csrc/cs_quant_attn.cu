// Attention of few query rows per KV head over a paged cache held in 4 bits: single tokens, verification blocks, and what is too short for the tensor cores' kernel to pay (Sec. 3.2; App. B.2),
// on mma.sync.  (Which calls come here: cs_quant_attention in cs_quant.cu.)
//
// out = softmax(scale Q K^T) V by one pass over the keys with a running reference point m and sum l per row, as in cs_paged_attn.cu.  What differs comes from the cache: a value costs 4.5 bits of
// HBM and two to three instructions, so that what a key costs an SM is counted in instructions, and the products are laid out so that every value is expanded once for up to 32 query rows:
//     S^T [16 keys x 8 rows]  = K Q^T      A = keys as they come out of their words, B = queries
//     O^T [16 dims x 8 rows] += V^T P^T    A = values, two keys of one element in a register, B = weights
// Keys and head dims are the M of m16n8k16, query rows the N: 8, 16, 24 or 32 of them, a template parameter.
// The MMA's sums over k do not care which element stands where: lane t's k are those of its own words, the t-th word of every group of 32 elements.  Keys go in as whole numbers (exact in either type), a group's two MMAs make a
// partial sum of their own, and the group's scale comes in where that is added up: queries need no second term, and no chain of MMAs is longer than two.  Values: neighbouring keys of one element
// come of two keys' words by a byte permutation, and with their scales, since those differ from key to key, exact in bf16 (cs_quant.cuh); weights as two bf16 terms (value = hi + lo), which change places by a
// transposition of 8 x 8 blocks (movmatrix).  So nothing but the result is rounded to 16 bits.
//
// Persistent: CTAs of four warps take equal runs of the line of key tiles (cs_paged.cuh).  A tile's 128 keys are four slices of 32, one for each warp; a slice lies in two pages at most.
// Every warp has its own ring of slices, fetched by cp.async, its own reference points, sums and output; the warps' results meet in shared memory where the item ends, and items that
// CTAs share are added up, in the order of the keys, by a launch behind (k_quant_merge).
// The reference point moves only past 2^8, by a vote; where no score is above, no maximum is worked out.
//
// What bounds it.  Contexts of many sequences: instructions.  A slice costs a warp some 800 of them (one row tile; of 285 us for 983,040 keys of eight heads of 128 the expansion of K takes 40, that of V 36, weights' second terms 22, the
// copies 19), the schedulers issue in 67 of 100 clocks, the ALU is busy in 57, the tensor cores in 24 - 32: 3.9 TB/s where contexts differ in length.  64 ragged tokens of the 8B shape (32 query heads, 8 of keys, up to 4,097) 41 us: first data
// after 6, SMs done after 31 to 38, the pieces' sums 4.6.  A token over 30,720 keys 21 us, the length of the chain: plan and page entries 3, first data 3, slices 7, the warps' results 1.5, the pieces' sums 4.  11 rows over 512 keys of the smallest
// shape 8 us, 3 of them for fetching instructions.
// Tried and not kept: units of a warp with claims by a counter (44 -> 60 us: warps out of step miss the instruction cache), CTAs of eight warps, sixteen keys at a time for more than eight rows (5 - 11 % slower), more CTAs an SM for heads of 64
// (spills).
//
// Masked keys: scores become -inf.  Slices that lie outside of [lo, hi) of the item's rows are not fetched; of one that lies partly outside, V scales out there become 0 whatever they are (nobody may have written those
// slots, and 0 x inf is not 0).  In slices that some rows see and others do not, so do V scales that values cannot be worked out with, and the rows that see such a key are given NaN.
#include <type_traits>
#include <utility>

#include "cs_quant.cuh"

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32, kSlice = 32;
static_assert(kWarps * kSlice == kPagedTile, "a warp has a slice of every tile");
typedef PagedPlanOf<kQuantMaxSeqs> Plan;

template <int DH, int NT> struct Few {
  static constexpr int kCols = 8 * NT;                       // query rows of an item
  static constexpr int kCtas = NT == 1 ? 4 : NT == 2 ? 3 : 2;   // on an SM
  static constexpr int kStages = 2, kPieces = 4;             // slices in flight; descriptions of pieces: the one at hand and those that the fetching side has got to, kStages slices and one piece ahead at most
  static constexpr int kKeyBytes = DH / 2, kScaleBytes = DH / 16;
  static constexpr int kData = kSlice * kKeyBytes, kScales = kSlice * kScaleBytes, kStage = 2 * (kData + kScales);
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kPass = DH < 64 ? DH : 64;            // columns of the results that warps exchange at a time
  static constexpr int kLd = kPass + 4;
  static constexpr int kExchange = kWarps * kCols * kLd * 4;
  static constexpr int kQRow = DH * 2 + (DH == 32 ? 0 : 64); // bytes of a query row (the rest keeps rows out of each other's banks)
  static constexpr int kQ = kCols * kQRow;
  static constexpr int kMl = (kWarps + 1) * kCols * 8;
  static constexpr int kPiece = (sizeof(PagedPiece) + 15) / 16 * 16;
  static constexpr int kSmem = kRing + kExchange + kQ + kMl + kWarps * kPieces * kPiece + (int)sizeof(Plan) + 16 + 128;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same with nothing added
template <typename T>
__device__ __forceinline__ void mma_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// shared memory by 32-bit addresses, with the constant part of one in the instruction
template <int kAt> __device__ __forceinline__ uint32_t lds16(uint32_t a) {
  unsigned short x;
  asm volatile("ld.shared.u16 %0, [%1 + %2];" : "=h"(x) : "r"(a), "n"(kAt) : "memory");
  return x;
}
template <int kAt> __device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared.u32 %0, [%1 + %2];" : "=r"(x) : "r"(a), "n"(kAt) : "memory");
  return x;
}
template <int kAt> __device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 x;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2 + %3];" : "=r"(x.x), "=r"(x.y) : "r"(a), "n"(kAt) : "memory");
  return x;
}
template <int kAt> __device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4 + %5];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(a), "n"(kAt) : "memory");
  return x;
}
// fn(0), .., fn(N - 1), of constants
template <int I> struct Constant { __device__ constexpr operator int() const { return I; } };
template <int N, typename Fn, int... I> __device__ __forceinline__ void each(Fn&& fn, std::integer_sequence<int, I...>) { (fn(Constant<I>{}), ...); }
template <int N, typename Fn> __device__ __forceinline__ void each(Fn&& fn) { each<N>(fn, std::make_integer_sequence<int, N>{}); }
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Where 16-byte chunk c of key j of a slice lies, in chunks, so that neither the keys' loads (a word of one chunk of eight neighbouring keys) nor the values' (keys t of four, all chunks) meet in a bank.
template <int DH>
__device__ __forceinline__ uint32_t at_chunk(uint32_t j, uint32_t c) {
  if constexpr (DH == 128) return (j * 4 + c) ^ ((j >> 1 & 1) * 2) ^ (j >> 2 & 1);
  else if constexpr (DH == 64) return (j * 2 + c) ^ (j >> 2 & 1);
  else return j;
}
template <typename T, int DH, int NT>
__global__ void __launch_bounds__(kThreads, Few<DH, NT>::kCtas)
k_quant_few(const __grid_constant__ QuantAttnArgs qa) {
  CS_PDL_PROLOGUE();
  typedef Few<DH, NT> F;
  constexpr int kStages = F::kStages, kCols = F::kCols, kGroups = DH / 32, kTiles = DH / 16, kChunks = DH / 32;      // groups of a key, a word of each for a lane; tiles of 16 head dims; 16-byte chunks of a key
  const PagedAttnArgs& a = qa.p;
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* ring = smem + (((uint32_t)__cvta_generic_to_shared(smem) + 127u & ~127u) - (uint32_t)__cvta_generic_to_shared(smem));      // [warp][stage]: K, V, K scales, V scales; of 128 bytes
  float* s_x = reinterpret_cast<float*>(ring + F::kRing);                        // [warp][row][kLd]
  uint8_t* s_q = reinterpret_cast<uint8_t*>(s_x) + F::kExchange;                 // [row][DH]
  float2* s_ml = reinterpret_cast<float2*>(s_q + F::kQ);                         // [warp][row]
  float2* s_row = s_ml + kWarps * kCols;                                         // [row]
  uint8_t* s_piece = reinterpret_cast<uint8_t*>(s_ml) + F::kMl;                  // [warp][piece]
  Plan& plan = *reinterpret_cast<Plan*>(s_piece + kWarps * F::kPieces * F::kPiece);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

  // (One warp where one can do it: sixteen of an SM's at the same thing take twice as long.)
  if (a.blk.n_seqs > 32 || warp == 0) paged_plan(a, plan);
  if (a.blk.n_seqs <= 32) __syncthreads();
  const long long total = plan.before[a.blk.n_seqs];
  const int n_cta = (int)min((long long)gridDim.x, total), cta = blockIdx.x;
  if (cta >= n_cta) {
    if (tid == 0) a.splits[cta].last = kPagedNone;
    return;
  }
  long long& s_end = *reinterpret_cast<long long*>(&plan + 1);                    // where the run ends
  // Pieces are described in shared memory, for each warp by itself, and read where they are used: kept in registers they would spill.  (Piece number k in place k % kPieces.)
  uint8_t* my_pieces = s_piece + warp * F::kPieces * F::kPiece;
  auto piece = [&](int k) -> PagedPiece& { return *reinterpret_cast<PagedPiece*>(my_pieces + (k & (F::kPieces - 1)) * F::kPiece); };
  if (warp == 0) {
    long long end;
    const PagedPiece first = paged_run(a, plan, total, n_cta, cta, lane, end);
    if (lane == 0) s_end = end;
    for (int w = 0; w < kWarps; ++w) *reinterpret_cast<PagedPiece*>(s_piece + w * F::kPieces * F::kPiece) = first;
  }
  __syncthreads();
  const long long run1 = s_end;
  if (piece(0).n_tiles == 0) {
    if (tid == 0) a.splits[cta].last = kPagedNone;
    return;
  }
  int n_known = 1, n_pieces = 0x7fffffff;        // pieces described; pieces of the run, once that is known
  // is there a piece k?  (k is at most n_known)
  auto exists = [&](int k) -> bool {
    if (k < n_known) return true;
    if (k >= n_pieces) return false;
    PagedPiece x = piece(k - 1);
    if (!paged_next(a, plan, x, run1)) {
      n_pieces = k;
      return false;
    }
    __syncwarp();
    piece(k) = x;
    __syncwarp();
    ++n_known;
    return true;
  };
  const int G = a.group;

  // ---- queries: of the piece behind the one at hand, in registers until that one is done
  constexpr int kQWords = (kCols * DH / 8 + kThreads - 1) / kThreads;      // eight elements each
  uint4 q_next[kQWords];
  auto ask = [&](const PagedPiece& x) {
#pragma unroll
    for (int i = 0; i < kQWords; ++i) {
      const int e = tid + i * kThreads, row = e / (DH / 8), c = e % (DH / 8), m = x.rg * kCols + row, r = a.by_group.of(m);
      q_next[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row < kCols && m < x.len * G) q_next[i] = __ldcg(reinterpret_cast<const uint4*>(a.q + ((x.start + r) * a.q_row + (x.head * G + m - r * G) * a.q_head + c * 8) * 2));
    }
  };
  auto keep = [&]() {
#pragma unroll
    for (int i = 0; i < kQWords; ++i) {
      const int e = tid + i * kThreads, row = e / (DH / 8), c = e % (DH / 8);
      if (row >= kCols) continue;
      *reinterpret_cast<uint4*>(s_q + row * F::kQRow + c * 16) = q_next[i];
    }
  };
  ask(piece(0));

  // ---- the fetching side: runs kStages slices ahead, across pieces.  Sixteen lanes fetch a slice's first half, sixteen the second: each half lies in one page, row after row.
  const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(warp * kStages * F::kStage);
  // Addresses of this lane's words and scales of a slice's first keys.  The other keys' are constants away, those of other chunks of a key (for keys) and of keys 4 - 7 of eight (for values) are these with a bit or two the other way round.
  const uint32_t a_k = my_ring + at_chunk<DH>((g >> 1) + 4 * (g & 1), 0) * 16 + t * 4, a_ks = my_ring + 2 * F::kData + ((g >> 1) + 4 * (g & 1)) * F::kScaleBytes;
  const int vg = DH == 128 ? g >> 1 : DH == 64 ? g >> 2 : 0;      // the group of this lane's values
  const uint32_t a_v = my_ring + F::kData + at_chunk<DH>(t, vg) * 16 + (DH == 128 ? (g & 1) * 8 : DH == 64 ? (g & 3) * 4 : (g >> 1) * 4), a_vs = my_ring + 2 * F::kData + F::kScales + t * F::kScaleBytes + vg * 2;
  const uint32_t a_q = (uint32_t)__cvta_generic_to_shared(s_q) + g * F::kQRow + t * 16;
  const int f_half = lane >> 4, f_in = lane & 15;
  // this lane's chunks of a half: f_in, f_in + 16, ...; where the first lies in the ring, and what its turn over four keys changes
  const uint32_t d_first = at_chunk<DH>(16 * f_half + f_in / kChunks, f_in % kChunks) * 16;
  constexpr int kScaleChunks = DH / 16;          // of a half
  const bool f_scales = f_in < 2 * kScaleChunks;
  const int f_which = f_in / kScaleChunks & 1, f_c = f_in % kScaleChunks;
  const char* f_scale_pool = reinterpret_cast<const char*>(f_which ? qa.kv.vs : qa.kv.ks) + f_c * 16;
  const uint32_t d_scale = 2 * F::kData + f_which * F::kScales + (f_half * kScaleChunks + f_c) * 16;
  int f_piece = 0;
  int f_key = 0, f_end = 0, f_lo = 0, f_hi = 0;  // first key of this lane's half of the next slice; where the piece ends; keys its rows attend to
  int f_row = 0, f_entry = 0, f_n = 0;           // rows of a page before its head's; page-table entry of this lane; slices before, of this piece
  uint32_t f_stage = 0;
  bool f_more = true;
  // entries of this warp's next sixteen slices' halves, one per lane
  auto entries = [&]() {
    const long long k = (long long)f_key - 16 * f_half + kPagedTile * (lane >> 1) + (lane & 1) * 16;      // (the last lanes' may lie behind 2^31)
    f_entry = k < f_hi && k + 16 > f_lo ? __ldcg(a.blk.table + (long long)piece(f_piece).seq * a.blk.table_width + (k >> a.kv.page_shift)) : 0;
  };
  auto open = [&]() {
    const PagedPiece& f = piece(f_piece);
    f_key = f.tile0 * kPagedTile + warp * kSlice + 16 * f_half;
    f_end = (f.tile0 + f.n_tiles) * kPagedTile;
    f_lo = f.lo; f_hi = f.hi;
    f_row = f.head * a.kv.page_size;
    f_n = 0;
  };
  open();
  entries();
  auto fetch = [&]() {
    if (f_more) {
      const int page = __shfl_sync(0xffffffffu, f_entry, (f_n & 15) * 2 + f_half);
      const bool used = f_key < f_hi && f_key + 16 > f_lo, on = used && (unsigned)page < (unsigned)a.kv.n_pages;
      if (used && !on) atomicOr(a.status, CS_DEV_BADARG);
      // (in units of 16 bytes; a half's rows are 16 or more of those, of its scales 2 or more)
      const uint32_t row = on ? (uint32_t)(f_row + (f_key & (a.kv.page_size - 1))) : 0u, at = on ? (uint32_t)page : 0u;
      const unsigned long long d = (unsigned long long)at * qa.kv.data_units + row * (F::kKeyBytes / 16) + f_in;
      const char *k = reinterpret_cast<const char*>(qa.kv.k) + d * 16, *v = reinterpret_cast<const char*>(qa.kv.v) + d * 16;
      const uint32_t dst = my_ring + f_stage;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const uint32_t x = dst + (DH == 128 && (i & 1) ? d_first ^ 16 : d_first) + i * 256;      // (sixteen chunks on: 4, 8 or 16 keys)
        cp16(x, k + i * 256, on);
        cp16(x + F::kData, v + i * 256, on);
      }
      if (f_scales) cp16(dst + d_scale, f_scale_pool + ((unsigned long long)at * qa.kv.scale_units * 16 + row * F::kScaleBytes), on);
      f_stage = f_stage == (kStages - 1) * F::kStage ? 0 : f_stage + F::kStage;
      f_key += kPagedTile;
      ++f_n;
      if (f_key >= f_end) {
        f_more = exists(++f_piece);
        if (f_more) open();
      }
      if (f_more && (f_n & 15) == 0) entries();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) fetch();
  keep();
  __syncthreads();

  bool opened = false;                           // has this CTA begun an item that others go on with?
  uint32_t stage = 0;
  for (int number = 0;; ++number) {
    const PagedPiece& p = piece(number);
    const bool more = exists(number + 1);
    if (more) ask(piece(number + 1));
    const int rows = min(kCols, p.len * G - p.rg * kCols);
    int all_lo, all_hi;                           // keys that every row of the item sees
    {
      int x;
      const int r0 = a.by_group.of(p.rg * kCols), r1 = a.by_group.of(p.rg * kCols + rows - 1);
      paged_range(a.mask, a.window, p.len, p.kv, r0, r0, x, all_hi);
      paged_range(a.mask, a.window, p.len, p.kv, r1, r1, all_lo, x);
    }
    float o[kTiles][NT][4];
    float m[NT][2], l[NT][2];                     // of rows 8 nt + 2 t + e
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i) o[i][nt][0] = o[i][nt][1] = o[i][nt][2] = o[i][nt][3] = 0.f;
      m[nt][0] = m[nt][1] = -INFINITY;
      l[nt][0] = l[nt][1] = 0.f;
    }

    const int end = (p.tile0 + p.n_tiles) * kPagedTile;
    for (int key0 = p.tile0 * kPagedTile + warp * kSlice; key0 < end; key0 += kPagedTile) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      if (key0 < p.hi && key0 + kSlice > p.lo) {
        const bool mixed = key0 < all_lo || key0 + kSlice > all_hi;      // some row does not see all of it
        // ---- S^T = K Q^T
        float s[2][NT][4];
        uint32_t ksc[2][2][kGroups > 1 ? kGroups / 2 : 1];      // scales of the keys of rows g, g + 8, two groups a register
        each<2>([&](auto mt) {
          each<2>([&](auto b) {
            constexpr int kAt = (16 * mt + 8 * b) * F::kScaleBytes;
            if constexpr (DH == 128) {
              const uint2 x = lds64<kAt>(a_ks + stage);
              ksc[mt][b][0] = x.x; ksc[mt][b][kGroups / 2 - 1] = x.y;
            } else if constexpr (DH == 64) ksc[mt][b][0] = lds32<kAt>(a_ks + stage);
            else ksc[mt][b][0] = lds16<kAt>(a_ks + stage);
          });
        });
        each<kGroups>([&](auto w) {
          uint4 q[NT];
          each<NT>([&](auto nt) { q[nt] = lds128<nt * 8 * F::kQRow + w * 64>(a_q); });
          const uint32_t kd = (a_k + stage) ^ (DH == 128 ? w * 16 : DH == 64 ? w * 16 : 0);
          each<2>([&](auto mt) {
            uint32_t x[2][4];                     // [key of row g, g + 8]
            float sc[2];
            each<2>([&](auto b) {
              expand_numbers<T>(lds32<(16 * mt + 8 * b) * F::kKeyBytes>(kd), x[b]);
              sc[b] = __uint_as_float(w & 1 ? ksc[mt][b][w / 2] & 0xffff0000u : ksc[mt][b][w / 2] << 16);
            });
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float part[4];
              mma_first<T>(part, x[0][0], x[1][0], x[0][1], x[1][1], q[nt].x, q[nt].y);
              mma<T>(part, x[0][2], x[1][2], x[0][3], x[1][3], q[nt].z, q[nt].w);
#pragma unroll
              for (int e = 0; e < 4; ++e) s[mt][nt][e] = w == 0 ? sc[e >> 1] * part[e] : fmaf(sc[e >> 1], part[e], s[mt][nt][e]);
            }
          });
        });
        // ---- masks  (key of row g + 8 b of S^T: as loaded)
        if (mixed) {
          // (in shared memory, a key a lane: compared where scales are taken out, 64 ragged tokens took 42.0 us)
          if (key0 < p.lo || key0 + kSlice > p.hi) {
            if (key0 + lane < p.lo || key0 + lane >= p.hi) {
              const uint32_t at = my_ring + stage + 2 * F::kData + F::kScales + lane * F::kScaleBytes;
              if constexpr (DH == 128) asm volatile("st.shared.v2.u32 [%0], {%1, %1};" ::"r"(at), "r"(0) : "memory");
              else if constexpr (DH == 64) asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(0) : "memory");
              else asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"((unsigned short)0) : "memory");
            }
            __syncwarp();
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              int lo = 0, hi = 0;
              const int n = 8 * nt + 2 * t + e;
              if (n < rows) {
                const int r = a.by_group.of(p.rg * kCols + n);
                paged_range(a.mask, a.window, p.len, p.kv, r, r, lo, hi);
              }
#pragma unroll
              for (int mt = 0; mt < 2; ++mt)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const int key = key0 + 16 * mt + 8 * b + (g >> 1) + 4 * (g & 1);
                  if (key < lo || key >= hi) s[mt][nt][2 * b + e] = -INFINITY;
                }
            }
        }
        // ---- reference points (the same in a column's eight lanes), weights, sums
        bool moves = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float x = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e])) * a.scale_log2e;
            moves |= m[nt][e] == -INFINITY ? x > m[nt][e] : x > m[nt][e] + 8.f;
          }
        if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float x = fmaxf(fmaxf(s[0][nt][e], s[0][nt][2 + e]), fmaxf(s[1][nt][e], s[1][nt][2 + e]));
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
              x *= a.scale_log2e;
              if (m[nt][e] == -INFINITY ? x > m[nt][e] : x > m[nt][e] + 8.f) {
                const float corr = paged_ex2(m[nt][e] - x);      // (from -inf: 0)
                m[nt][e] = x;
                l[nt][e] *= corr;
#pragma unroll
                for (int k = 0; k < kTiles; ++k) { o[k][nt][e] *= corr; o[k][nt][2 + e] *= corr; }
              }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float base = m[nt][e] == -INFINITY ? 0.f : -m[nt][e];
#pragma unroll
            for (int mt = 0; mt < 2; ++mt)
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const float w = paged_ex2(fmaf(s[mt][nt][2 * b + e], a.scale_log2e, base));
                s[mt][nt][2 * b + e] = w;
                l[nt][e] += w;
              }
          }
        // ---- O^T += V^T P^T
        bool odd = false;
        each<2>([&](auto mt) {
          uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const float w0 = s[mt][nt][2 * b], w1 = s[mt][nt][2 * b + 1];
              const uint32_t hi = PagedType<__nv_bfloat16>::pack(w0, w1);
              const float2 x = PagedType<__nv_bfloat16>::unpack(hi);
              ph[nt][b] = transposed(hi);
              pl[nt][b] = transposed(PagedType<__nv_bfloat16>::pack(w0 - x.x, w1 - x.y));
            }
          constexpr int kW = DH == 128 ? 2 : 1;   // words of a key for this lane
          uint32_t vw[4][kW], sv[4];              // keys t, t + 4, t + 8, t + 12: MMA keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
          each<4>([&](auto j) {
            constexpr int kKey = 16 * mt + 4 * j;
            const uint32_t at = (a_v + stage) ^ (DH > 32 && (j & 1) ? 16 : 0);
            if constexpr (DH == 128) {
              const uint2 w = lds64<kKey * F::kKeyBytes>(at);
              vw[j][0] = w.x; vw[j][kW - 1] = w.y;
            } else {
              vw[j][0] = lds32<kKey * F::kKeyBytes>(at);
              if constexpr (DH == 32) vw[j][0] >>= 8 * (g & 1);
            }
            sv[j] = lds16<kKey * F::kScaleBytes>(a_vs + stage);
          });
          if (mixed) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (quant_odd(sv[j])) { odd = true; sv[j] = 0; }
          }
          const QuantScale s01 = QuantScale::of(sv[0] | sv[1] << 16), s23 = QuantScale::of(sv[2] | sv[3] << 16);
#pragma unroll
          for (int w = 0; w < kW; ++w) {
            // [keys 2 t, 2 t + 1; 2 t + 8, 2 t + 9][even, odd elements][field]
            uint32_t x[2][2][4];
            quant_expand(__byte_perm(vw[0][w], vw[1][w], 0x5410), s01, x[0][0]);
            quant_expand(__byte_perm(vw[0][w], vw[1][w], 0x7632), s01, x[0][1]);
            quant_expand(__byte_perm(vw[2][w], vw[3][w], 0x5410), s23, x[1][0]);
            quant_expand(__byte_perm(vw[2][w], vw[3][w], 0x7632), s23, x[1][1]);
#pragma unroll
            for (int term = 0; term < 2; ++term)
#pragma unroll
              for (int k = 0; k < (DH == 32 ? 2 : 4); ++k)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                  mma<__nv_bfloat16>(o[w * 4 + k][nt], x[0][0][k], x[0][1][k], x[1][0][k], x[1][1][k], term ? pl[nt][0] : ph[nt][0], term ? pl[nt][1] : ph[nt][1]);
          }
        });
        if (mixed && __any_sync(0xffffffffu, odd)) {
          // values that are not finite: the rows that see them become NaN there
#pragma unroll 1
          for (int j = 0; j < kSlice; ++j) {
            if (!quant_odd(lds16<2 * F::kData + F::kScales>(my_ring + stage + j * F::kScaleBytes + vg * 2))) continue;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                int lo = 0, hi = 0;
                const int n = 8 * nt + 2 * t + e;
                if (n < rows) {
                  const int r = a.by_group.of(p.rg * kCols + n);
                  paged_range(a.mask, a.window, p.len, p.kv, r, r, lo, hi);
                }
                if (key0 + j >= lo && key0 + j < hi) {
#pragma unroll
                  for (int k = 0; k < kTiles; ++k) o[k][nt][e] = o[k][nt][2 + e] = __int_as_float(0x7fc00000);
                }
              }
          }
        }
      }
      __syncwarp();                              // (every lane has read the slice)
      stage = stage == (kStages - 1) * F::kStage ? 0 : stage + F::kStage;
      fetch();
    }

    // ---- the warps' results meet
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], d);
        if (g == 0) s_ml[warp * kCols + 8 * nt + 2 * t + e] = make_float2(m[nt][e], l[nt][e]);
      }
    constexpr int kPasses = DH / F::kPass, kMine = F::kPass / 8;      // passes; elements of a lane in one
#pragma unroll
    for (int w = 0; w < kPasses; ++w) {
      // elements kMine kPasses g + kMine w + i of rows 8 nt + 2 t + e are number kMine g + i of the pass
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (8 * nt + 2 * t + e >= rows) continue;
          float4* dst = reinterpret_cast<float4*>(s_x + (warp * kCols + 8 * nt + 2 * t + e) * F::kLd + kMine * g);
#pragma unroll
          for (int i = 0; i < kMine / 4; ++i) {
            const int k = w * 4 + 2 * i;
            dst[i] = make_float4(o[k][nt][e], o[k][nt][2 + e], o[k + 1][nt][e], o[k + 1][nt][2 + e]);
          }
        }
      __syncthreads();
      if (w == 0) {
        // a row's common reference point and sum, and what each warp's share of it counts
        if (tid < rows) {
          float2 ml[kWarps];
          float M = -INFINITY, L = 0.f;
#pragma unroll
          for (int v = 0; v < kWarps; ++v) {
            ml[v] = s_ml[v * kCols + tid];
            M = fmaxf(M, ml[v].x);
          }
#pragma unroll
          for (int v = 0; v < kWarps; ++v) {
            const float k = ml[v].x == -INFINITY ? 0.f : paged_ex2(ml[v].x - M);
            L += ml[v].x == -INFINITY && ml[v].y == 0.f ? 0.f : k * ml[v].y;      // (without a maximum, but a sum: NaN)
            s_ml[v * kCols + tid] = make_float2(k, ml[v].y);
          }
          s_row[tid] = make_float2(M, L);
        }
        __syncthreads();
      }
      constexpr int kQuads = F::kPass / 4;       // four columns of a row a thread
#pragma unroll 2
      for (int i = tid; i < rows * kQuads; i += kThreads) {
        const int n = i / kQuads, c = i % kQuads;
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < kWarps; ++v) {
          const float2 k = s_ml[v * kCols + n];
          const float4 y = *reinterpret_cast<const float4*>(s_x + (v * kCols + n) * F::kLd + 4 * c);
          if (k.x == 0.f && k.y == 0.f) continue;                  // (it saw nothing)
          acc[0] = fmaf(k.x, y.x, acc[0]); acc[1] = fmaf(k.x, y.y, acc[1]); acc[2] = fmaf(k.x, y.z, acc[2]); acc[3] = fmaf(k.x, y.w, acc[3]);
        }
        const float2 row = s_row[n];
        const int d = 4 * c / kMine * (kMine * kPasses) + kMine * w + 4 * c % kMine;
        if (p.whole) {
          const float inv = row.y == 0.f ? 0.f : 1.f / row.y;
          const int mrow = p.rg * kCols + n, r = a.by_group.of(mrow);
          const long long at = (long long)(p.start + r) * a.n_heads + p.head * G + (mrow - r * G);
          *reinterpret_cast<uint2*>(a.out + (at * DH + d) * 2) = make_uint2(PagedType<T>::pack(acc[0] * inv, acc[1] * inv), PagedType<T>::pack(acc[2] * inv, acc[3] * inv));
          if (a.lse != nullptr && c == 0 && w == 0) a.lse[at] = row.y == 0.f ? -INFINITY : (row.x + log2f(row.y)) * 0.6931471805599453f;
        } else {
          const long long at = ((long long)cta * 2 + (p.opens ? 1 : 0)) * kCols + n;
          *reinterpret_cast<float4*>(a.parts + at * DH + d) = make_float4(acc[0], acc[1], acc[2], acc[3]);
          if (c == 0 && w == 0) *(reinterpret_cast<float2*>(a.parts_ml) + at) = row;
        }
      }
      __syncthreads();                           // (the exchange rows are free again)
    }
    if (p.opens && !p.whole) {                   // (the run ends with this item)
      opened = true;
      if (tid == 0) a.splits[cta] = PagedSplit{paged_last_cta(a, p, total, n_cta), rows, p.rg * kCols, p.head, p.start};
    }
    if (!more) break;
    keep();                                      // (nobody reads the queries of the piece before any more)
    __syncthreads();
  }
  if (!opened && tid == 0) a.splits[cta].last = kPagedNone;
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Items that several CTAs share: a row's pieces added up, in the order of the keys.  A block looks at some of those CTAs and has one row of all items that begin in them, a warp each, or its warps an eighth of the pieces of one that has many.  (Added
// up by the last CTA to arrive, inside the kernel, ten pieces of 22 rows took 14 us and 74 of four rows 11: all of them come through one SM.)
constexpr int kMergeWarps = 8;
template <typename T, int DH>
__global__ void __launch_bounds__(kMergeWarps * 32)
k_quant_merge(const __grid_constant__ PagedAttnArgs a, int cols, int n_ctas, int per_block) {
  CS_PDL_PROLOGUE();
  constexpr int kV = DH / 32, kBatch = 8;         // columns of a lane; pieces in flight
  __shared__ float2 s_ml[kMergeWarps];
  __shared__ __align__(16) float s_o[kMergeWarps][DH];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.y, first = blockIdx.x * per_block;
  float M, L, acc[kV];
  auto none = [&]() {
    M = -INFINITY; L = 0.f;
#pragma unroll
    for (int e = 0; e < kV; ++e) acc[e] = 0.f;
  };
  auto add = [&](float2 ml, const float (&v)[kV]) {
    if (ml.x == -INFINITY && ml.y == 0.f) return;                  // (it saw nothing)
    const float top = fmaxf(M, ml.x), keep = M == -INFINITY ? (L == 0.f ? 0.f : L) : paged_ex2(M - top), k = ml.x == -INFINITY ? 0.f : paged_ex2(ml.x - top);   // (a sum without a maximum is NaN)
    M = top;
    L = fmaf(k, ml.y, L * keep);
#pragma unroll
    for (int e = 0; e < kV; ++e) acc[e] = fmaf(k, v[e], acc[e] * keep);
  };
  auto load = [&](const float* p, float (&v)[kV]) {
    if constexpr (kV == 4) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p));
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
    } else if constexpr (kV == 2) {
      const float2 x = __ldcg(reinterpret_cast<const float2*>(p));
      v[0] = x.x; v[1] = x.y;
    } else {
      v[0] = __ldcg(p);
    }
  };
  int last = kPagedNone, n_rows = 0;
  if (lane < per_block && first + lane < n_ctas) { last = __ldcg(&a.splits[first + lane].last); n_rows = __ldcg(&a.splits[first + lane].rows); }
  // every so-manieth piece of an item
  auto gather = [&](int c0, int c1, int from, int step) {
    none();
    for (int cb = c0 + from; cb <= c1; cb += kBatch * step) {
      float2 ml[kBatch];
      float v[kBatch][kV];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int c = cb + i * step;
        if (c > c1) continue;
        const long long at = ((long long)c * 2 + (c == c0 ? 1 : 0)) * cols + row;
        ml[i] = __ldcg(reinterpret_cast<const float2*>(a.parts_ml) + at);
        load(a.parts + at * DH + lane * kV, v[i]);
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i)
        if (cb + i * step <= c1) add(ml[i], v[i]);
    }
  };
  auto write = [&](int c0) {
    const PagedSplit* d = a.splits + c0;
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const int m = __ldcg(&d->first_row) + row, r = a.by_group.of(m);
    const long long at = (long long)(__ldcg(&d->start) + r) * a.n_heads + __ldcg(&d->head) * a.group + (m - r * a.group);
    char* dst = a.out + (at * DH + lane * kV) * 2;
    if constexpr (kV == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(PagedType<T>::pack(acc[0] * inv, acc[1] * inv), PagedType<T>::pack(acc[2] * inv, acc[3] * inv));
    else if constexpr (kV == 2) *reinterpret_cast<uint32_t*>(dst) = PagedType<T>::pack(acc[0] * inv, acc[1] * inv);
    else *reinterpret_cast<unsigned short*>(dst) = (unsigned short)PagedType<T>::pack(acc[0] * inv, 0.f);
    if (a.lse != nullptr && lane == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
  };
  const bool some = last >= 0 && row < n_rows, many = last - (first + lane) >= kBatch;
  int nth = 0;
  for (unsigned todo = __ballot_sync(0xffffffffu, some && !many); todo != 0; todo &= todo - 1) {
    const int c0 = first + __ffs(todo) - 1, c1 = __shfl_sync(0xffffffffu, last, c0 - first);
    if (nth++ % kMergeWarps != warp) continue;
    gather(c0, c1, 0, 1);
    write(c0);
  }
  for (unsigned todo = __ballot_sync(0xffffffffu, some && many); todo != 0; todo &= todo - 1) {
    const int c0 = first + __ffs(todo) - 1, c1 = __shfl_sync(0xffffffffu, last, c0 - first);
    gather(c0, c1, warp, kMergeWarps);
    s_ml[warp] = make_float2(M, L);
#pragma unroll
    for (int e = 0; e < kV; ++e) s_o[warp][lane * kV + e] = acc[e];
    __syncthreads();
    if (warp == 0) {
      none();
#pragma unroll 1
      for (int i = 0; i < kMergeWarps; ++i) {
        float v[kV];
#pragma unroll
        for (int e = 0; e < kV; ++e) v[e] = s_o[i][lane * kV + e];
        add(s_ml[i], v);
      }
      write(c0);
    }
    __syncthreads();
  }
}

template <typename T, int DH, int NT>
cs_status launch_few(cs_quant_cache* c, const QuantAttnArgs& a, unsigned bit, cudaStream_t st) {
  typedef Few<DH, NT> F;
  static_assert(F::kCtas * (F::kSmem + 1024) <= 228 * 1024 && F::kCols <= kQuantMaxRows && F::kCtas * F::kCols <= kQuantRowsPerSm && F::kCtas <= kQuantCtasPerSm, "");
  if (!(c->attr_set & bit)) {
    CS_CUDA_OK(c, cudaFuncSetAttribute(k_quant_few<T, DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem));
    c->attr_set |= bit;
  }
  // (no more CTAs than the page table's room has places for)
  const BlocksView& b = a.p.blk;
  const long long groups = ((long long)b.rows * a.p.group + F::kCols - 1) / F::kCols + b.n_seqs, tiles = (long long)b.table_width * a.p.kv.page_size / kPagedTile + 2 + a.p.item_cost;
  int ctas = c->num_sms * F::kCtas;
  if (groups < ctas && tiles < ctas && a.p.kv.n_kv_heads < ctas && groups * tiles * a.p.kv.n_kv_heads < ctas) ctas = (int)(groups * tiles * a.p.kv.n_kv_heads);
  CS_CUDA_OK(c, cs_launch_pdl(k_quant_few<T, DH, NT>, dim3(ctas), dim3(kThreads), F::kSmem, st, a));
  // (eight or sixteen CTAs' items a block, us: 64 ragged tokens of the 8B shape 41.6 / 42.8, 11 rows over 4,096 keys 18.2 / 17.7)
  const int per_block = NT == 1 ? 8 : 16;
  CS_CUDA_OK(c, cs_launch_pdl(k_quant_merge<T, DH>, dim3((ctas + per_block - 1) / per_block, F::kCols), dim3(kMergeWarps * 32), 0, st, a.p, F::kCols, ctas, per_block));
  return CS_OK;
}
template <typename T, int DH>
cs_status launch_few_rows(cs_quant_cache* c, const QuantAttnArgs& a, int tiles, unsigned bit, cudaStream_t st) {
  switch (tiles) {
    case 1: return launch_few<T, DH, 1>(c, a, bit, st);
    case 2: return launch_few<T, DH, 2>(c, a, bit << 1, st);
    case 3: return launch_few<T, DH, 3>(c, a, bit << 2, st);
    default: return launch_few<T, DH, 4>(c, a, bit << 3, st);
  }
}
template <typename T>
cs_status launch_few_type(cs_quant_cache* c, const QuantAttnArgs& a, int tiles, unsigned bit, cudaStream_t st) {
  switch (c->cfg.head_dim) {
    case 32: return launch_few_rows<T, 32>(c, a, tiles, bit, st);
    case 64: return launch_few_rows<T, 64>(c, a, tiles, bit << 4, st);
    default: return launch_few_rows<T, 128>(c, a, tiles, bit << 8, st);
  }
}

}  // namespace

cs_status cs_launch_quant_few(cs_quant_cache* c, const QuantAttnArgs& args, long long rows, cudaStream_t st) {
  QuantAttnArgs a = args;
  // Items of as few query rows as leave no fewer items: a KV head's rows (on the average of the call's sequences, which is what the host knows; a launch may have part of them, but has all rows at hand) in equal shares of up to 32
  const long long items = (rows + kQuantMaxRows - 1) / kQuantMaxRows;
  const int tiles = (int)(((rows + items - 1) / items + 7) / 8);
  a.p.item_rows = 8 * tiles;
  a.p.by_item_rows = PagedDivisor::by(a.p.item_rows);
  // (what changing items takes, in tiles.  One / two, us: 64 ragged tokens of the 8B shape 42.8 / 43.7, 32 x 4 rows over 2,000 keys 31.1 / 30.2)
  a.p.item_cost = tiles == 1 ? 1 : 2;
  a.p.keep = 4;
  return a.half ? launch_few_type<__half>(c, a, tiles, 1u << 12, st) : launch_few_type<__nv_bfloat16>(c, a, tiles, 1u, st);
}
