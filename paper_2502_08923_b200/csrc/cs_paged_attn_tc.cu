// Attention of tall blocks over a paged KV cache, in 16 bits or in 4, on the 5th-generation tensor cores (Sec. 3.2; App. B.2).
//
// The mathematics is that of cs_paged_attn.cu.  Query rows (row of the block x head of the group) are the M = 128 of both products, so that TMEM
// lane = query row and one thread has a whole row of scores:
//     S [128 x 128 keys] = Q K_tile^T      (both from shared memory)
//     O [128 x D]       += P V_tile        (P in tensor memory, over the scores it comes from; V as it lies in the cache, MN-major)
// A CTA (one per SM, persistent, runs of tiles as cs_paged.cuh deals them out) has two slots of S/P and O columns, each with a warpgroup for its softmax, so
// that the tensor cores work on one slot while the other's weights are made.  An item of more than 128 rows fills both slots with
// different rows over the same tiles (each K and V tile is fetched once for 256 rows); of fewer, the slots take the tiles
// in turn and are added up at the end, from tensor memory.
//
// Steps s = 0, 1, ... alternate between the slots.  With heads of 128 the MMA warp issues S(0) S(1), then P V(s) and S(s + 2) for every s: S(s + 2) overwrites P(s), which the
// products' order keeps.  (Smaller heads leave room for weights beside the scores: S(s + 2) goes ahead of P V(s), see kApart; 1,184 rows over 8,192 keys 158 -> 148 us.)  A slot's scores being there means that its product before is done, so a softmax that moves its reference point may
// rescale O at once.  The reference point moves only past 2^8 (softmax does not depend on it, and weights up to 2^8 are as exact as weights up
// to 1), which leaves rescaling to a few tiles.  Weights are rounded once, to the cache's type, on their way into the second product; their sum is
// taken before.  In fp16 they are 2^7 (to 2^15) times as large, by a reference point that much lower: those below 2^-25 become 0, and 131,072 of them at 2^-25 of the largest would be 4e-3 of the sum, eight times what the
// type resolves; below 2^-32 they are 3e-5 at most.
//
// Warps 0-7 softmax, 8 issues MMAs, 9 and 10 fetch K and V tiles (a copy per page and 64 dims, page-table entries 32 at a time), 11 fetches queries.
//
// Keys no row of the item sees may hold anything: their scores are masked, their V rows set to zero in shared memory.  A value that is not finite at a key that some rows
// of the item see and others do not reaches the others' sums too (0 x inf is not 0).  Looking for such values ahead of every product makes tiles of such keys three times as long.  So that is left to a second pass:
// where a result is not finite, the CTA goes through that piece once more, with those values left out of the products and added to the rows that see them at the end: one NaN in a 2,048-row chunk behind 30,720 keys makes
// the call 2.0 ms long instead of 0.91.  (The same instructions run both passes.  A launch of its own for such rows, or a branch of the launch behind, costs calls without any 1 - 10 us for its code
// alone.)
//
// Every wait is bounded: on expiry the CTA flags CS_DEV_TIMEOUT, stops issuing, walks through its barriers, drains what is in flight, frees its TMEM and returns.  Items that it had not
// finished, shared ones among them whatever their other CTAs have done, stay unwritten.
//
// What bounds it.  Long chunks: 2,950 clocks for a pair of 128 x 128 tiles with heads of 128 (1,184 rows, what 4,096 to 16,384 keys differ by), of which the products take 2,048 at their peak rate.  A slot's chain, measured with some
// registers spilled and 3,350 a pair: scores into registers 190, maxima 300, weights 1,200 (ex2, 16 a clock, is 1,024 of it), into tensor memory 200, product 512, next scores 512, hand-overs 400.  A 2,048-row chunk
// behind 30,720 keys of the 8B shape: 0.91 ms in short runs (1.17 PFLOP/s), 1.03 - 1.06 ms at the power cap (1.49 GHz, 990 W).  Heads of 64: 2,700 clocks a pair, all of it the softmax warps' way through their instructions (two
// warps a scheduler, one instruction in three clocks, no unit above 35 %): 8 x 21 rows over 16,384 keys 64 us; measured at 65: 63.5 without the exponentials, 65 with half of the products, 64 with all pages in L2.  11 rows over
// 4,096 keys 16 us, a chain of latencies (plan and piece 1.5, page entries, first tiles 3, one step 1.8, results 1.4, sums of pieces 5).
// Tried and not kept: maxima left out, with reference points that follow the sums (3,350 -> 3,400 clocks: they hide behind ex2); a quarter of the exponentials by a polynomial in
// packed arithmetic (-2 % of the clocks, +1 % of the time at the power cap); products with the first 64 keys only when all weights are there (no slower by themselves); sixteen softmax
// warps, two to a row with half of the keys each (104 registers; heads of 128 166 -> 180 us for 1,184 rows over 8,192 keys, heads of 64 138 -> 145: a barrier a tile for the common reference
// point, and no phase shorter for it); slots that keep out of each other's exponentials (141 -> 154); exponentials in blocks of 16 (138 -> 142).
#include <type_traits>

#include "cs_quant.cuh"
#include "cs_tcgen.cuh"

namespace {

constexpr int kMmaWarp = 8, kKWarp = 9, kQWarp = 11, kExpandWarp = 12;   // (10: V; 12, 13: out of four bits, K; 14, 15: V)
template <bool kQuant> constexpr int kThreads = kQuant ? 512 : 384;
constexpr int kM = 128;                                            // query rows of a slot
// Tensor memory: scores of slot s at 128 s, output from 256 on.  With heads of 128 that is all there is, and weights lie over the scores they come from; with smaller heads
// they have 64 columns of their own, and a slot's next scores are made while the softmax is at work on the last ones, which it has in registers.
constexpr uint32_t kTmemCols = 512;
template <int DH> constexpr bool kApart = DH <= 64;
template <typename T> constexpr float kUp = std::is_same<T, __half>::value ? 7.f : 0.f;      // how far below a row's largest score its reference point is put
constexpr uint32_t kOCol = 256;
template <int DH> constexpr uint32_t kPCol = kApart<DH> ? 384 : 0;
template <int DH> constexpr uint32_t kPStep = kApart<DH> ? 64 : 128;
template <int DH> constexpr int kTileBytes = kPagedTile * DH * 2;  // of K, of V, and of a slot's queries
template <int DH, bool kQuant> constexpr int kStages = DH == 128 ? (kQuant ? 3 : 4) : 8;
// In a cache of 4 bits: tiles as they lie there, numbers, then scales; so many for keys and for values (four with heads of 64: no faster)
constexpr int kPackedTiles = 2;
template <int DH> constexpr int kPackedData = kPagedTile * DH / 2;
template <int DH> constexpr int kPacked = kPackedData<DH> + kPagedTile * DH / 16;
template <int DH> constexpr int kRowBytes = DH == 32 ? 64 : 128;    // of a row in shared memory, swizzled over so many bytes; heads of 128 are two halves one behind the other
// Registers of the warpgroups: two of the softmax and one of the others share the 384 x 168 that the block is launched with.  (What the softmax spills it fetches again for every tile: heads of 128 with 72 / 216, 68 bytes spilled,
// windowed chunks 110 us, with 56 / 224 and none 102; heads of 64 the other way round, 32 bytes and 64 us against 88 and 69.)
// Over 4 bits there is a warpgroup more, and 512 x 128 registers: 2,048 rows over 30,720 keys 931 us with 56 for both of the others and 200, 968 with 48 and 208, 1,046 with 40 and 216, 959 with 56, 40 and 208, 915 with these.
template <int DH, bool kQuant> constexpr int kOtherRegs = kQuant ? 56 : DH == 128 ? 56 : 72;
constexpr int kExpandRegs = 48;
template <int DH, bool kQuant> constexpr int kSoftmaxRegs = kQuant ? 200 : DH == 128 ? 224 : 216;
constexpr int kCtl = 512;
// Descriptors of pieces.  A slot that is still at a piece's results holds the others up four pieces on at the latest: the other slot waits for it at the next piece whose tiles the slots take in turn, but the
// scores of the piece after that may be made (of one tile each, they need neither slot), which frees the queries and makes two more known.
constexpr int kPieces = 8;
constexpr int kPieceBytes = 72;
template <int DH, bool kQuant> constexpr int kTcSmem = 1024 + (kStages<DH, kQuant> + 2) * kTileBytes<DH> + kCtl + 2 * kM * 8 + kPieces * kPieceBytes + (kQuant ? 2 * kPackedTiles * kPacked<DH> : 0) + (int)sizeof(PagedPlan);

// Operand descriptors as in cs_tcgen.cuh, for rows of 128 or (heads of 32) 64 bytes: eight of them a group, and the swizzle as wide
template <int kRow> __device__ __forceinline__ uint64_t desc_rows(uint32_t saddr, uint32_t lbo) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(8 * kRow >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)(kRow == 128 ? 2 : 4) << 61);
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
               ::"r"(dst), "l"(tm), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void umma_ta(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
               ::"r"(tmem_d), "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(acc) : "memory");
}
#define CS_R32(v) "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), \
  "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), \
  "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
// 32 columns of this thread's lane; valid after ld_wait and ld_valid
__device__ __forceinline__ void ld32(uint32_t taddr, float* v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : CS_R32(v) : "r"(taddr));
}
__device__ __forceinline__ void ld16(uint32_t taddr, float* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]),
                 "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]) : "r"(taddr));
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void ld_valid(float* v) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+f"(v[i]), "+f"(v[i + 1]), "+f"(v[i + 2]), "+f"(v[i + 3]), "+f"(v[i + 4]), "+f"(v[i + 5]), "+f"(v[i + 6]), "+f"(v[i + 7])::"memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                 "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// a word of a piece's description, read where it is used: kept in registers across the loop they would spill
__device__ __forceinline__ int fresh(const int& x) { return *const_cast<const volatile int*>(&x); }
__device__ __forceinline__ uint32_t flag(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void set_flag(uint32_t addr, uint32_t v) { asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void or_flag(uint32_t addr, uint32_t v) { asm volatile("red.shared.or.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void store32b(void* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}
// barrier of a slot's four softmax warps that also ORs a predicate
__device__ __forceinline__ bool slot_any(int slot, bool pred) {
  uint32_t out;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %2, 0;\nbar.red.or.pred q, %1, 128, p;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(out) : "r"(slot + 1), "r"((uint32_t)pred) : "memory");
  return out != 0;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Weights 2^(score scale - m) of 32 keys, rounded to T, to tensor memory, and their sum, of the weights as they were.  One term of 16 bits is a choice: a second one would make half as many products again (2,048 rows over
// 30,720 keys 757 -> 1,135 us at the rate that the power cap leaves a library's product) and as much more to pack, for errors of 2.2e-3 (bf16) and 2.8e-4 (fp16) against 64 bits, of which 1.7e-3 and 2.1e-4 are the result's own
// rounding.  (The 16-a-clock unit behind ex2 is busy for half of the loop's
// time.  A polynomial in packed arithmetic for a quarter to three eighths of them was no faster in short runs and 2 - 4 % slower at the power cap.)
template <typename T>
__device__ __forceinline__ void weights(const float* v, uint32_t taddr, f32x2 sc2, f32x2 nm2, f32x2& l2) {
  uint32_t w[16];
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    float x0, x1;
    unpack2(fma2(pack2(v[2 * j], v[2 * j + 1]), sc2, nm2), x0, x1);
    x0 = paged_ex2(x0);
    x1 = paged_ex2(x1);
    l2 = add2(l2, pack2(x0, x1));
    w[j] = PagedType<T>::pack(x0, x1);
  }
  st16(taddr, w);
}

// What the roles need to know of a piece; worked out by one warp and left in shared memory, since the softmax threads have no register to spare (what they
// spill lies beyond L1, which shared memory leaves next to nothing of: 350 bytes of it made the tile loop a third slower).
struct TcPiece {
  int start, len, kv, seq, head, rg;
  int lo, hi, all_lo, all_hi;      // keys that some row of the item attends to, that all do
  int tile0, steps;                // steps 0: there is no further piece
  int both, opens, whole, last;    // both slots have rows of their own; has the item's first tile; all; the CTA with the last
  int again;                       // second pass
};

// a word of two 16-bit values with zeros for those that are not finite
template <typename T>
__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
  constexpr uint32_t e = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
  return ((w & e) == e ? 0u : w & 0xffffu) | ((w >> 16 & e) == e ? 0u : w & 0xffff0000u);
}

// In a second pass: 32 columns of a row, as stored (`part`: fp32, else T), get the values that are not finite at keys the row sees and others of its item do not.  (Any positive weight makes the same of them.)
template <typename T, int DH, bool kQuant>
__device__ __noinline__ void add_odd(const PagedAttnArgs& a, const TcPiece& p, int n_tiles, int lo, int hi, int c0, void* dst, bool part) {
  const int last = min(hi, (p.tile0 + n_tiles) * kPagedTile);
  float sum[32] = {};
  for (int key = max(lo, p.tile0 * kPagedTile); key < last; ++key) {
    if (key >= p.all_lo && key < p.all_hi) {
      key = p.all_hi - 1;
      continue;
    }
    const int page = __ldcg(a.blk.table + (long long)p.seq * a.blk.table_width + (key >> a.kv.page_shift));
    if ((unsigned)page >= (unsigned)a.kv.n_pages) continue;
    if constexpr (kQuant) {                      // (32 columns are a group: all of it, or nothing)
      const unsigned short s = __ldcg(a.vs + (page * a.scale_page + ((long long)p.head * a.kv.page_size + (key & (a.kv.page_size - 1))) * (DH / kQuantGroup) + c0 / kQuantGroup));
      if (quant_odd(s)) {
#pragma unroll
        for (int i = 0; i < 32; ++i) sum[i] = __int_as_float(0x7fc00000);
      }
      continue;
    }
    const uint4* src = reinterpret_cast<const uint4*>(a.kv.v + (page * a.kv.page_stride + p.head * a.kv.head_stride + (long long)(key & (a.kv.page_size - 1)) * a.kv.slot_stride + c0) * 2);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 v = __ldcg(src + j);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 x = PagedType<T>::unpack(w[i] ^ finite_only<T>(w[i]));
        sum[8 * j + 2 * i] += x.x;
        sum[8 * j + 2 * i + 1] += x.y;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    if (sum[i] == 0.f) continue;
    if (part) reinterpret_cast<float*>(dst)[i] += sum[i];
    else {
      unsigned short* o = reinterpret_cast<unsigned short*>(dst) + i;
      *o = (unsigned short)PagedType<T>::pack(PagedType<T>::unpack(*o).x + sum[i], 0.f);
    }
  }
}

// Sixteen-bit values of a group's four words, each as the 16-byte chunk of eight elements that it is in a row of 16 bits.  fp16 ends at 65504: what lies beyond it becomes that.
template <typename T>
__device__ __forceinline__ void expand_group(const uint4& words, unsigned scale, uint4 (&out)[4]) {
  const uint32_t w[4] = {words.x, words.y, words.z, words.w};
  if constexpr (std::is_same<T, __nv_bfloat16>::value) {
    const QuantScale s = QuantScale::of(scale * 0x10001u);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t r[4];
      quant_expand(w[i], s, r);
      out[i] = make_uint4(r[0], r[1], r[2], r[3]);
    }
  } else {
    const float s = __uint_as_float(scale << 16);
    const __half2 h = __float2half2_rn(s);
    const uint32_t hs = *reinterpret_cast<const uint32_t*>(&h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t r[4];
      expand_numbers<__half>(w[i], r);
      out[i] = make_uint4(h2_mul(r[0], hs), h2_mul(r[1], hs), h2_mul(r[2], hs), h2_mul(r[3], hs));
    }
    // (eight of it are beyond 65504; five bits of it go below 2^-24: worked out in 32 bits, rounded once)
    if (fabsf(s) > 8192.f || (fabsf(s) < 0x1p-20f && s != 0.f)) {
      auto far = [&](int i, int k) { return fminf(fmaxf((float)((int)(w[i] >> (4 * k) & 15) - 8) * s, -65504.f), 65504.f); };
#pragma unroll
      for (int i = 0; i < 4; ++i)
        out[i] = make_uint4(PagedType<__half>::pack(far(i, 0), far(i, 4)), PagedType<__half>::pack(far(i, 1), far(i, 5)), PagedType<__half>::pack(far(i, 2), far(i, 6)), PagedType<__half>::pack(far(i, 3), far(i, 7)));
    }
  }
}

// kQuant: over a cache of 4 bits (cs_quant.cuh).  The warps that fetch keys and values have tiles copied as they lie there, and two warps more for either write them out in 16 bits, half of the rows each, where the other kind has
// TMA put them; all else is the same.  8 x 21 rows of heads of 64 over 16,384 keys (us): 133 with keys and values written out by the warp that fetches them, 94 with warps of their own, 76 with a page's copies by a lane each (one after
// the other they took 150 clocks apiece); the softmax alone takes 64.  84 rows of heads of 128 over 30,720 keys 39 (by the kernel for few rows 85).
template <typename T, int DH, bool kQuant>
__global__ void __launch_bounds__(kThreads<kQuant>, 1)
k_paged_tc(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ PagedAttnArgs a, int q_box_bytes) {
  constexpr int kTB = kTileBytes<DH>, kNS = kStages<DH, kQuant>, kRow = kRowBytes<DH>, kHalves = DH == 128 ? 2 : 1, kHalf = kPagedTile * 128;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* ring = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));   // [stage][64 dims][128 keys][128 B]
  uint8_t* sq = ring + kNS * kTB;                                       // [slot][64 dims][128 rows][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sq + 2 * kTB);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * kNS + 13 + kPieces + 2);
  float2* s_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(bars) + kCtl);      // [slot][128 rows]
  TcPiece* s_piece = reinterpret_cast<TcPiece*>(s_ml + 2 * kM);
  static_assert(sizeof(TcPiece) <= kPieceBytes, "");
  uint8_t* packed = reinterpret_cast<uint8_t*>(s_piece) + kPieces * kPieceBytes;        // [keys, values][kPackedTiles]
  PagedPlan& plan = *reinterpret_cast<PagedPlan*>(packed + (kQuant ? 2 * kPackedTiles * kPacked<DH> : 0));
  const uint32_t b_packed = smem_u32(bars) + kCtl - 16 * 2 * kPackedTiles, b_unpacked = b_packed + 8 * 2 * kPackedTiles;    // [keys, values][kPackedTiles]
  static_assert(8 * (2 * kNS + 25) <= kCtl - 16 * 2 * kPackedTiles && (kPieces * kPieceBytes) % 16 == 0 && kPacked<DH> % 16 == 0, "");
  const uint32_t b_full = smem_u32(bars), b_empty = b_full + 8 * kNS, b_s = b_empty + 8 * kNS, b_p = b_s + 16, b_p2 = b_p + 16, b_o = b_p2 + 16, b_taken = b_o + 16, b_qfull = b_taken + 16, b_qfree = b_qfull + 8,
                 b_drain = b_qfree + 8, b_piece = b_drain + 8, b_ml = b_piece + 8 * kPieces, b_read = b_ml + 8;
  // flags, by 32-bit addresses: a wait has run out; an item has been announced; results that are not finite, a bit a piece (the last one for all from there on)
  const uint32_t f_abort = b_read + 12, f_shares = f_abort + 4, f_odd = f_shares + 4;
  // All weights are there.  (Those of the first 64 keys are announced ahead where their product is on the way to the slot's next scores; elsewhere that only costs: 1,184 rows of heads
  // of 64 over 8,192 keys 141 -> 138 us without.)
  const uint32_t b_all = kApart<DH> ? b_p : b_p2;
  const int tid = threadIdx.x, warp = (int)uniform(tid >> 5), lane = tid & 31;

  // (nothing of this depends on the kernel before, so it is done while that one ends)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    if constexpr (!kQuant) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmK) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(&tmV) : "memory");
    }
    asm volatile("prefetch.tensormap [%0];" ::"l"(&tmQ) : "memory");
    for (int s = 0; s < kNS; ++s) { mbar_init(b_full + 8 * s, kQuant ? 2 : 1); mbar_init(b_empty + 8 * s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(b_s + 8 * s, 1); mbar_init(b_p + 8 * s, 4); mbar_init(b_p2 + 8 * s, 4); mbar_init(b_o + 8 * s, 1); mbar_init(b_taken + 8 * s, 4); }
    mbar_init(b_qfull, 1); mbar_init(b_qfree, 1); mbar_init(b_drain, 1);
    for (int s = 0; s < kPieces; ++s) mbar_init(b_piece + 8 * s, 1);
    mbar_init(b_ml, 8); mbar_init(b_read, 8);
    if constexpr (kQuant) for (int s = 0; s < 2 * kPackedTiles; ++s) { mbar_init(b_packed + 8 * s, 1); mbar_init(b_unpacked + 8 * s, 2); }
    set_flag(f_abort, 0);
    set_flag(f_shares, 0);
    set_flag(f_odd, 0);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  paged_plan(a, plan);
  __syncthreads();
  fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  const long long total = plan.before[a.blk.n_seqs];
  const int n_cta = (int)min((long long)gridDim.x, total), cta = blockIdx.x;

  // Bounded waits, in few instructions (see the MMA issuer).  Once one has run out all others return.
  auto wait = [&](uint32_t bar, uint32_t parity) -> bool {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = globaltimer_ns();
    for (;;) {
      if (mbar_try_wait(bar, parity)) return true;
      if (flag(f_abort)) return false;
      if (globaltimer_ns() - t0 > a.wait_ns) {
        set_flag(f_abort, 1);
        atomicOr(a.status, CS_DEV_TIMEOUT);
        return false;
      }
    }
  };
  auto wait_warp = [&](uint32_t bar, uint32_t parity) -> bool { return __all_sync(0xffffffffu, wait(bar, parity)); };
  const int slot_rows = a.item_rows / 2;          // query rows of a slot
  // the next piece, once it is known (by a warp; false: a wait has run out)
  auto known = [&](uint32_t piece) -> bool { return wait_warp(b_piece + 8 * (piece % kPieces), (piece / kPieces) & 1) && !__any_sync(0xffffffffu, flag(f_abort) != 0); };
  // Order of the ring, that of first use: where the slots share tiles K0 V0 K1 V1 .., else K0 K1 V0 K2 V1 ..; with scores made ahead (kApart) K0 K1 V0 K2 V1 .. and
  // K0 K1 K2 V0 K3 V1 ..  (Entry of step s, of n steps.)
  auto k_entry = [](bool both, int s) {
    const int i = both ? s >> 1 : s, ahead = (both ? 1 : 2) + (kApart<DH> ? 1 : 0);      // K tiles in front of the first V tile
    return i < ahead ? i : 2 * i - ahead + 1;
  };
  auto v_entry = [](bool both, int s, int n) {
    const int i = both ? s >> 1 : s, tiles = both ? n >> 1 : n, ahead = (both ? 1 : 2) + (kApart<DH> ? 1 : 0);
    return i + min(i + ahead, tiles);
  };

  // The end of a pass, where all roles meet once, whatever has become of their waits: is there a second one?  Only if no role has given up: one that has leaves here, and must not be
  // waited for again.  (Nobody adds to f_odd between here and a second pass.)
  auto again = [&](bool second) -> bool {
    uint32_t fine;
    fence_before();
    asm volatile("{\n.reg .pred p, q;\nsetp.eq.b32 p, %1, 0;\nbar.red.and.pred q, 0, p;\nselp.u32 %0, 1, 0, q;\n}" : "=r"(fine) : "r"(flag(f_abort)) : "memory");
    fence_after();
    return !second && fine != 0 && flag(f_odd) != 0;
  };
  if (warp >= 8) {
    if (kQuant && warp >= kExpandWarp) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kExpandRegs));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs<DH, kQuant>));
    uint32_t base = 0, piece = 0;                 // ring entries before this piece; pieces
    bool ok = true, met = false;
    if (warp == kMmaWarp) {
      // ------------------------------------------------------------------ MMA issuer
      constexpr uint32_t kType = std::is_same<T, __nv_bfloat16>::value ? (1u << 7) | (1u << 10) : 0u;
      constexpr uint32_t idesc_s = (1u << 4) | kType | ((uint32_t)(kPagedTile >> 3) << 17) | ((uint32_t)(kM >> 4) << 24);
      constexpr uint32_t idesc_o = (1u << 4) | kType | (1u << 16) | ((uint32_t)(DH >> 3) << 17) | ((uint32_t)(kM >> 4) << 24);   // B (= V) is MN-major
      const uint64_t dq0 = desc_rows<kRow>(smem_u32(sq), 16), dk0 = desc_rows<kRow>(smem_u32(ring), 16), dv0 = desc_rows<kRow>(smem_u32(ring), kHalf);
      // One lane runs a piece's steps by itself, and every instruction counts: this warp comes by once in 900 clocks, when the softmax warps have filled the instruction cache with
      // their unrolled loops, so that its instructions are fetched anew each time.  (All lanes with votes, ring places worked out from the step, waits in
      // line: 900 clocks a step of its own, and the tensor cores waited for it.)
      uint32_t p_phase = 0, t_phase = 0;          // bit s: of slot s
      for (;; ++piece) {
        ok = known(piece);
        if (!ok) break;
        const TcPiece& d = s_piece[piece % kPieces];
        const int n = (int)uniform((uint32_t)d.steps);
        const bool both = uniform((uint32_t)d.both) != 0;
        const uint32_t second = uniform((uint32_t)d.again);
        if (n == 0) {
          if (again(second)) continue;
          met = true;
          break;
        }
        ok = wait_warp(b_qfull, (piece - second) & 1);   // (the end of the first pass had no queries)
        if (!ok) break;
        fence_after();
        bool fine = true;
        if (elect_one()) {
          uint32_t at = base, k_at = 0, v_at = 0;   // next ring entry, in the order of first use; entries of the K and V tile at hand
          auto scores = [&](int s) {
            if (!both || !(s & 1)) {
              k_at = at++;
              if (!wait(b_full + 8 * (k_at % kNS), (k_at / kNS) & 1)) { fine = false; return; }
            }
            const uint64_t dk = dk0 + (k_at % kNS) * (kTB >> 4), dq = dq0 + (both && (s & 1) ? kTB >> 4 : 0);
            const uint32_t acc = tmem + (s & 1) * 128;
#pragma unroll
            for (int h = 0; h < kHalves; ++h)
#pragma unroll
              for (int k = 0; k < kRow / 32; ++k) umma_bf16(acc, dq + h * (kHalf >> 4) + 2 * k, dk + h * (kHalf >> 4) + 2 * k, idesc_s, (h | k) ? 1u : 0u);
            umma_commit(b_s + 8 * (s & 1));
            if (!both || (s & 1)) umma_commit(b_empty + 8 * (k_at % kNS));
            if (s == n - 1) umma_commit(b_qfree);
          };
          scores(0);
          if (fine && n > 1) scores(1);
          for (int s = 0; s < n && fine; ++s) {
            const uint32_t slot = s & 1;
            if (kApart<DH> && s + 2 < n) {
              if (!wait(b_taken + 8 * slot, t_phase >> slot & 1)) { fine = false; break; }      // (the softmax has the scores in registers)
              fence_after();
              scores(s + 2);
              if (!fine) break;
            }
            if (kApart<DH>) t_phase ^= 1u << slot;
            if (!both || !slot) {
              v_at = at++;
              if (!wait(b_full + 8 * (v_at % kNS), (v_at / kNS) & 1)) { fine = false; break; }
            }
            if (!wait(b_p + 8 * slot, p_phase >> slot & 1)) { fine = false; break; }
            fence_after();
            const uint64_t dv = dv0 + (v_at % kNS) * (kTB >> 4);
            const uint32_t acc = tmem + kOCol + slot * DH, w = tmem + kPCol<DH> + slot * kPStep<DH>;
#pragma unroll
            for (int k = 0; k < 4; ++k) umma_ta(acc, w + k * 8, dv + k * (16 * kRow >> 4), idesc_o, (s > 1 || k > 0) ? 1u : 0u);   // 16 keys per instruction
            if constexpr (!kApart<DH>) {
              if (!wait(b_p2 + 8 * slot, p_phase >> slot & 1)) { fine = false; break; }
              fence_after();
            }
            p_phase ^= 1u << slot;
#pragma unroll
            for (int k = 4; k < 8; ++k) umma_ta(acc, w + k * 8, dv + k * (16 * kRow >> 4), idesc_o, 1u);
            if (!both || slot) umma_commit(b_empty + 8 * (v_at % kNS));
            umma_commit(b_o + 8 * slot);
            if (!kApart<DH> && s + 2 < n) scores(s + 2);
          }
        }
        ok = __all_sync(0xffffffffu, fine);
        p_phase = __reduce_xor_sync(0xffffffffu, elect_one() ? p_phase : 0u);
        t_phase = __reduce_xor_sync(0xffffffffu, elect_one() ? t_phase : 0u);
        base += both ? n : 2 * n;
        if (!ok) break;
      }
      if (!ok) {                                   // what was issued must be done before its memory goes away
        if (elect_one()) umma_commit(b_drain);
        __syncwarp();
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try_wait(b_drain, 0) && globaltimer_ns() - t0 < a.wait_ns) {}
      }
    } else if (warp == kQWarp) {
      // ------------------------------------------------------------------ pieces and queries
      uint32_t todo = 0xffffffffu;                 // pieces that the pass has to go through, a bit each (the last one for all from there on)
      for (uint32_t second = 0; ; ++second, ++piece) {
        PagedPiece p;
        p.n_tiles = 0;
        long long run1 = 0;
        if (cta < n_cta) p = paged_run(a, plan, total, n_cta, cta, lane, run1);
        bool more = p.n_tiles > 0;
        for (uint32_t nth = 0; ; ++piece, ++nth) {
          for (; more && !(todo >> min(nth, 31u) & 1); ++nth) more = paged_next(a, plan, p, run1);
          const bool both = more && p.len * a.group - p.rg * a.item_rows > slot_rows;
          if (lane == 0) {
            TcPiece d;
            d.steps = more ? (both ? 2 * p.n_tiles : p.n_tiles) : 0;
            d.again = second;
            if (more) {
              int x;
              const int last_row = min(p.len * a.group, (p.rg + 1) * a.item_rows) - 1, r0 = a.by_group.of(p.rg * a.item_rows), r1 = a.by_group.of(last_row);
              paged_range(a.mask, a.window, p.len, p.kv, r0, r0, x, d.all_hi);
              paged_range(a.mask, a.window, p.len, p.kv, r1, r1, d.all_lo, x);
              d.start = p.start; d.len = p.len; d.kv = p.kv; d.seq = p.seq; d.head = p.head; d.rg = p.rg;
              d.lo = p.lo; d.hi = p.hi; d.tile0 = p.tile0; d.both = both; d.opens = p.opens; d.whole = p.whole;
              d.last = p.whole ? cta : paged_last_cta(a, p, total, n_cta);
            }
            s_piece[piece % kPieces] = d;
            mbar_arrive(b_piece + 8 * (piece % kPieces));
          }
          __syncwarp();
          if (!more) break;
          if (piece - second > 0) ok = wait_warp(b_qfree, (piece - second - 1) & 1);
          if (!ok) break;
          if (elect_one()) {
            mbar_expect_tx(b_qfull, (uint32_t)(q_box_bytes * kHalves * (both ? 2 : 1)));
            for (int s = 0; s < (both ? 2 : 1); ++s)
              for (int h = 0; h < kHalves; ++h)
                tma_load_3d(smem_u32(sq) + s * kTB + h * kHalf, &tmQ, b_qfull, 64 * h, p.head * a.group, p.start + a.by_group.of(p.rg * a.item_rows + s * slot_rows));
          }
          more = paged_next(a, plan, p, run1);
        }
        if (!ok) {
          // (every role meets a last piece, and a copy that nobody waited for must land before the shared memory goes away)
          const unsigned long long t0 = globaltimer_ns();
          while (piece - second > 0 && !mbar_try_wait(b_qfull, (piece - second - 1) & 1) && globaltimer_ns() - t0 < a.wait_ns) {}
          break;
        }
        if (!again(second)) {
          met = true;
          break;
        }
        todo = flag(f_odd);
      }
    } else {
      // ------------------------------------------------------------------ K tiles, V tiles
      const bool is_k = kQuant ? warp == kKWarp || (warp & ~1) == kExpandWarp : warp == kKWarp;
      const CUtensorMap* tm = is_k ? &tmK : &tmV;
      const int rows = min(a.kv.page_size, kPagedTile), per_tile = kPagedTile / rows, shift = a.kv.page_shift;
      uint32_t asked = 0;                          // entries this warp has started copies for, + 1
      uint32_t packed_no = 0;                      // kQuant: tiles asked for, or written out
      int tile_no = 0;
      for (;; ++piece) {
        if (!known(piece)) break;
        const TcPiece& d = s_piece[piece % kPieces];
        const int n = (int)uniform((uint32_t)d.steps), tile0 = (int)uniform((uint32_t)d.tile0), head = (int)uniform((uint32_t)d.head), lo = (int)uniform((uint32_t)d.lo),
                  hi = (int)uniform((uint32_t)d.hi), seq = (int)uniform((uint32_t)d.seq);
        const bool both = uniform((uint32_t)d.both) != 0;
        if (n == 0) {
          if (again(uniform((uint32_t)d.again))) continue;
          met = true;
          break;
        }
        const int inc = both ? 2 : 1;
        int entry = 0, first = -64;                // this lane's page-table entry, and of which page the first lane has one
        const int* table = a.blk.table + (long long)seq * a.blk.table_width;
        // pages of a step's tile that hold keys of the item: [j0, j1) from page0 on
        auto pages_of = [&](int s, int& key0, int& page0, int& j0, int& j1) {
          key0 = (tile0 + (both ? s >> 1 : s)) * kPagedTile;
          page0 = key0 >> shift;
          const int pa = max(key0, lo), pz = min(key0 + kPagedTile, hi);
          j0 = j1 = 0;
          if (pz > pa) { j0 = (pa >> shift) - page0; j1 = ((pz - 1) >> shift) - page0 + 1; }
          if (page0 < first || page0 + per_tile > first + 32) {
            first = page0;
            const int page = first + lane;
            entry = -1;
            if (((long long)(page + 1) << shift) > lo && ((long long)page << shift) < hi) entry = __ldcg(table + page);
          }
        };
        if constexpr (kQuant) {
          constexpr uint32_t kTiles = kPackedTiles;
          const uint32_t first_buffer = is_k ? 0 : kTiles;
          if (warp < kExpandWarp) {
            // tiles as they lie in the cache (scales of pages that do not exist: zeros)
            for (int s = 0; s < n && ok; s += inc, ++packed_no) {
              int key0, page0, j0, j1;
              pages_of(s, key0, page0, j0, j1);
              const uint32_t buffer = first_buffer + packed_no % kTiles, bar = b_packed + 8 * buffer;
              ok = wait_warp(b_unpacked + 8 * buffer, ((packed_no / kTiles) & 1) ^ 1);
              if (!ok) break;
              // (a page's numbers by one lane, its scales by another: one after the other by the same lane, 8 x 21 rows of heads of 64 over 16,384 keys in pages of 32 takes 94 us)
              const int j = lane & 7;
              const int page = (int)__shfl_sync(0xffffffffu, entry, page0 + j - first);
              const bool here = lane < 16 && j >= j0 && j < j1, there = (unsigned)page < (unsigned)a.kv.n_pages;
              uint8_t* numbers = packed + buffer * kPacked<DH> + j * rows * (DH / 2);
              uint8_t* scales = packed + buffer * kPacked<DH> + kPackedData<DH> + j * rows * (DH / 16);
              if (here && !there) {
                if (lane < 8) for (int x = 0; x < rows * DH / 64; ++x) reinterpret_cast<uint32_t*>(scales)[x] = 0u;
                atomicOr(a.status, CS_DEV_BADARG);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // (copies follow in the same place later)
              }
              __syncwarp();
              const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, here && there && lane < 8)) * (uint32_t)(rows * (DH / 2 + DH / 16));
              if (lane == 0) mbar_expect_tx(bar, bytes);
              __syncwarp();
              if (here && there) {
                const long long row = (long long)head * a.kv.page_size + ((key0 + j * rows) & (a.kv.page_size - 1));
                if (lane < 8) bulk_load(smem_u32(numbers), (is_k ? a.kv.k : a.kv.v) + page * a.kv.page_stride + row * (DH / 2), rows * (DH / 2), bar);
                else bulk_load(smem_u32(scales), (is_k ? a.ks : a.vs) + page * a.scale_page + row * (DH / kQuantGroup), rows * (DH / 16), bar);
              }
              __syncwarp();
            }
          } else {
            // half of a tile's rows, out of four bits
            for (int s = 0; s < n && ok; s += inc, ++packed_no) {
              const uint32_t e = base + (is_k ? k_entry(both, s) : v_entry(both, s, n)), st = e % kNS, buffer = first_buffer + packed_no % kTiles;
              ok = wait_warp(b_packed + 8 * buffer, (packed_no / kTiles) & 1);
              if (!ok) break;
              ok = wait_warp(b_empty + 8 * st, ((e / kNS) & 1) ^ 1);
              if (!ok) break;
              // Groups of a row go two to a lane's neighbour, rows on: eight lanes write all eight places of 16 bytes that 128 bytes of banks have
              constexpr int kPerRow = DH >= 64 ? 2 : 1, kRowsAtOnce = 32 / kPerRow;
              const uint8_t* src = packed + buffer * kPacked<DH>;
              uint8_t* out = ring + st * kTB;
              const int c = lane % kPerRow, r0 = (warp & 1) * (kPagedTile / 2) + lane / kPerRow;
#pragma unroll 2
              for (int i = 0; i < kPagedTile / 2 / kRowsAtOnce * kHalves; ++i) {
                const int h = i % kHalves, r = r0 + i / kHalves * kRowsAtOnce, group = h * 2 + c;
                uint4 v[4];
                expand_group<T>(*reinterpret_cast<const uint4*>(src + r * (DH / 2) + group * 16), *reinterpret_cast<const unsigned short*>(src + kPackedData<DH> + (r * (DH / kQuantGroup) + group) * 2), v);
#pragma unroll
                for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(out + h * kHalf + r * kRow + (DH >= 64 ? (c * 4 + k) ^ (r & 7) : k ^ (r >> 1 & 3)) * 16) = v[k];
              }
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(b_unpacked + 8 * buffer);
              if (is_k && tile_no++ == a.drop) continue;           // (test hook: these keys never arrive)
              if (lane == 0) mbar_arrive(b_full + 8 * st);
            }
          }
        } else {
          for (int s = 0; s < n && ok; s += inc) {
            const uint32_t e = base + (is_k ? k_entry(both, s) : v_entry(both, s, n)), st = e % kNS;
            int key0, page0, j0, j1;
            pages_of(s, key0, page0, j0, j1);
            ok = wait_warp(b_empty + 8 * st, ((e / kNS) & 1) ^ 1);
            if (!ok) break;
            if (is_k && tile_no++ == a.drop) continue;             // (test hook: these keys never arrive)
            if (elect_one()) mbar_expect_tx(b_full + 8 * st, (uint32_t)((j1 - j0) * rows * kRow * kHalves));
            __syncwarp();
            for (int j = j0; j < j1; ++j) {
              int page = (int)__shfl_sync(0xffffffffu, entry, page0 + j - first);
              if ((unsigned)page >= (unsigned)a.kv.n_pages) {      // (a page behind the last one reads as zeros)
                page = a.kv.n_pages;
                if (lane == 0) atomicOr(a.status, CS_DEV_BADARG);
              }
              const int slot = (key0 + j * rows) & (a.kv.page_size - 1);
              if (elect_one()) {
                const uint32_t dst = smem_u32(ring) + st * kTB + j * rows * kRow;
#pragma unroll
                for (int h = 0; h < kHalves; ++h) tma_load_4d(dst + h * kHalf, tm, b_full + 8 * st, 64 * h, slot, head, page);
              }
            }
            asked = e + 1;
          }
        }
        base += both ? n : 2 * n;
        if (!ok) break;
      }
      if (flag(f_abort)) {                              // copies that nobody will consume must land before the shared memory goes away
        if constexpr (kQuant) {
          if (warp < kExpandWarp) {
            constexpr uint32_t kTiles = kPackedTiles;
            for (uint32_t e = packed_no > kTiles ? packed_no - kTiles : 0; e < packed_no; ++e) {
              const unsigned long long t0 = globaltimer_ns();
              while (!mbar_try_wait(b_packed + 8 * ((is_k ? 0 : kTiles) + e % kTiles), (e / kTiles) & 1) && globaltimer_ns() - t0 < a.wait_ns) {}
            }
          }
        }
        for (uint32_t e = asked > kNS ? asked - kNS : 0; e < asked; ++e) {
          // (entries of the other warp's are waited for as well; one that was never started runs into the limit)
          const unsigned long long t0 = globaltimer_ns();
          while (!mbar_try_wait(b_full + 8 * (e % kNS), (e / kNS) & 1) && globaltimer_ns() - t0 < a.wait_ns) {}
        }
      }
    }
    if (!met) again(true);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs<DH, kQuant>));
    // -------------------------------------------------------------------- softmax and results: one thread per query row
    const int slot = warp >> 2, row = tid & 127, G = a.group;
    const bool out_32 = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;      // (rows are multiples of 32 bytes)
    const uint32_t lanes = tmem + ((uint32_t)(warp & 3) << 21), s_col = lanes + slot * 128, o_col = lanes + kOCol + slot * DH, p_col = lanes + kPCol<DH> + slot * kPStep<DH>;
    uint32_t base = 0, s_phase = 0, piece = 0, turns = 0;      // (turns: pieces whose tiles the slots took in turn)
    uint32_t o_mine = 0, o_other = 0;                          // products of this slot, of the other one, so far
    bool met = false;
    for (;; ++piece) {
      if (slot_any(slot, !known(piece))) break;
      const TcPiece& p = s_piece[piece % kPieces];
      const int n = p.steps;
      if (n == 0) {
        if (again(p.again != 0)) continue;
        met = true;
        break;
      }
      const bool both = p.both != 0;
      const int mrow = p.rg * a.item_rows + (both ? slot * slot_rows : 0) + row;
      const bool live = row < slot_rows && mrow < p.len * G;
      const bool some = __any_sync(0xffffffffu, live);         // (a warp without rows leaves its lanes to chance: nobody reads them)
      auto range = [&](int& lo, int& hi) {                     // keys that the row sees  (worked out where they are needed: in registers they would spill)
        lo = hi = 0;
        if (live) {
          const int r = a.by_group.of(mrow);
          paged_range(a.mask, a.window, fresh(p.len), fresh(p.kv), r, r, lo, hi);
        }
      };
      float m = live ? -INFINITY : 0.f;
      f32x2 l2 = pack2(0.f, 0.f);
      const f32x2 sc2 = pack2(a.scale_log2e, a.scale_log2e);

      for (int s = slot; s < n; s += 2) {
        const int key0 = (fresh(p.tile0) + (both ? s >> 1 : s)) * kPagedTile;
        const bool mixed = key0 < fresh(p.all_lo) || key0 + kPagedTile > fresh(p.all_hi);
        bool ok = wait(b_s + 8 * slot, s_phase);
        s_phase ^= 1;
        ok = __all_sync(0xffffffffu, ok);
        fence_after();
        if (mixed && ok && (p.again || key0 < p.lo || key0 + kPagedTile > p.hi)) {
          // V rows that no row of the item sees become zeros (whatever lies there: its weight is 0, but 0 x inf is not); in a second pass also what is not finite in rows that only some see
          const uint32_t e = base + v_entry(both, s, n), st = e % kNS;
          const bool none = key0 + row < p.lo || key0 + row >= p.hi;
          if (wait(b_full + 8 * st, (e / kNS) & 1) && (none || (p.again && (key0 + row < p.all_lo || key0 + row >= p.all_hi)))) {
            uint8_t* vrow = ring + st * kTB + row * kRow;
#pragma unroll 1
            for (int h = 0; h < kHalves; ++h)
#pragma unroll 1
              for (int c = 0; c < kRow / 16; ++c) {
                uint4* x = reinterpret_cast<uint4*>(vrow + h * kHalf + ((c + lane) & (kRow / 16 - 1)) * 16);
                uint4 y = make_uint4(0u, 0u, 0u, 0u);
                if (!none) {
                  y = *x;
                  y = make_uint4(finite_only<T>(y.x), finite_only<T>(y.y), finite_only<T>(y.z), finite_only<T>(y.w));
                }
                *x = y;
              }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        float v[128];
        if (some && ok) {
#pragma unroll
          for (int c = 0; c < 4; ++c) ld32(s_col + 32 * c, v + 32 * c);
          ld_wait();
#pragma unroll
          for (int c = 0; c < 4; ++c) ld_valid(v + 32 * c);
        }
        if constexpr (kApart<DH>) {
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b_taken + 8 * slot);
        }
        if (mixed && ok) {
          // a bit for each of 32 keys that the row sees
          int lo, hi;
          range(lo, hi);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int from = min(max(lo - key0 - 32 * c, 0), 32), to = min(max(hi - key0 - 32 * c, 0), 32);
            const uint32_t bits = (to == 32 ? 0xffffffffu : (1u << to) - 1u) & ~(from == 32 ? 0xffffffffu : (1u << from) - 1u);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[32 * c + j] = bits & (1u << j) ? v[32 * c + j] : -INFINITY;
          }
        }
        if (some && ok) {
          float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int j = 4; j < 124; j += 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], v[j + i], v[j + 4 + i]);
          }
          const float top = max3(max3(mx[0], mx[1], v[124]), max3(mx[2], mx[3], v[125]), max3(v[126], v[127], v[127])) * a.scale_log2e;
          // (O and the weights' columns: the product before must be done.  With scores over the weights they would not be there otherwise.)
          if constexpr (kApart<DH>) {
            if (s > 1) {
              wait(b_o + 8 * slot, (o_mine - 1) & 1);
              __syncwarp();
              fence_after();
            }
          }
          const bool moves = live && (m == -INFINITY ? top > m : top > m + (8.f + kUp<T>));
          if (__any_sync(0xffffffffu, moves)) {
            const float corr = !moves ? 1.f : m == -INFINITY ? 0.f : paged_ex2(m - (top - kUp<T>));
            if (moves) m = top - kUp<T>;
            float l0, l1;
            unpack2(l2, l0, l1);
            l2 = pack2(l0 * corr, l1 * corr);
            if (s > 1) {
#pragma unroll 1
              for (int c = 0; c < DH / 16; ++c) {      // (sixteen columns at a time: all scores are in registers)
                float o[16];
                ld16(o_col + 16 * c, o);
                ld_wait();
                asm volatile("" : "+f"(o[0]), "+f"(o[1]), "+f"(o[2]), "+f"(o[3]), "+f"(o[4]), "+f"(o[5]), "+f"(o[6]), "+f"(o[7])::"memory");
                asm volatile("" : "+f"(o[8]), "+f"(o[9]), "+f"(o[10]), "+f"(o[11]), "+f"(o[12]), "+f"(o[13]), "+f"(o[14]), "+f"(o[15])::"memory");
#pragma unroll
                for (int j = 0; j < 16; ++j) o[j] *= corr;
                st16(o_col + 16 * c, reinterpret_cast<const uint32_t*>(o));
              }
            }
          }
          const float nm = m == -INFINITY ? 0.f : -m;
          const f32x2 nm2 = pack2(nm, nm);
          weights<T>(v, p_col, sc2, nm2, l2);
          weights<T>(v + 32, p_col + 16, sc2, nm2, l2);
          if constexpr (!kApart<DH>) {
            st_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(b_p + 8 * slot);    // (the products with the first 64 keys may begin)
          }
          weights<T>(v + 64, p_col + 32, sc2, nm2, l2);
          weights<T>(v + 96, p_col + 48, sc2, nm2, l2);
          st_wait();
          fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(b_all + 8 * slot);
        } else {
          // (nor may a warp without rows run ahead: its arrivals would count for the step before)
          if constexpr (kApart<DH>) { if (s > 1) wait(b_o + 8 * slot, (o_mine - 1) & 1); }
          fence_before();
          __syncwarp();
          if (lane == 0) {
            if constexpr (!kApart<DH>) mbar_arrive(b_p + 8 * slot);
            mbar_arrive(b_all + 8 * slot);
          }
        }
        ++o_mine;
      }

      // ---- results
      float l0, l1;
      unpack2(l2, l0, l1);
      float l = l0 + l1;
      const bool mine = n > slot, other = n > 1 - slot;        // did this slot, the other slot have a step?
      o_other += (n + slot) >> 1;
      if (mine) wait(b_o + 8 * slot, (o_mine - 1) & 1);
      if (!both && other) wait(b_o + 8 * (1 - slot), (o_other - 1) & 1);
      fence_after();
      float k_mine = 1.f, k_other = 0.f;
      if (!both) {
        // the slots' rows are the same: each warpgroup adds up half of the columns, from tensor memory
        s_ml[slot * kM + row] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(b_ml);
        wait(b_ml, turns & 1);
        const float2 o_ml = s_ml[(1 - slot) * kM + row];
        const bool nothing = o_ml.x == -INFINITY && o_ml.y == 0.f;
        const float M = fmaxf(m, o_ml.x);
        k_mine = m == -INFINITY ? 0.f : paged_ex2(m - M);
        k_other = o_ml.x == -INFINITY ? 0.f : paged_ex2(o_ml.x - M);
        l = (m == -INFINITY && l == 0.f ? 0.f : l * k_mine) + (nothing ? 0.f : o_ml.y * k_other);
        m = M;
      }
      const bool good = flag(f_abort) == 0;
      // (32 columns at a time; heads of 32 have no half for the second warpgroup)
      const int c_first = both || DH == 32 ? 0 : slot * (DH / 2), c_last = both ? DH : DH == 32 ? (slot == 0 ? 32 : 0) : c_first + DH / 2;
      const long long part = ((long long)cta * 2 + (p.opens ? 1 : 0)) * kPagedMaxRows + (both ? slot * slot_rows : 0) + row;
      const int r = live ? a.by_group.of(mrow) : 0, head = p.head * G + (live ? mrow - r * G : 0);
      const long long out_row = (long long)(p.start + r) * a.n_heads + head;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const bool whole = p.whole != 0;
      if (some && good) {
#pragma unroll 1
        for (int c0 = c_first; c0 < c_last; c0 += 32) {
          float o[32];
          ld32(o_col + c0, o);
          if (both) {
            ld_wait();
            ld_valid(o);
          } else {
            float o2[32];
            ld32(lanes + kOCol + (1 - slot) * DH + c0, o2);
            ld_wait();
            ld_valid(o);
            ld_valid(o2);
            // (a slot without steps holds what an earlier item left)
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = (mine ? o[j] * k_mine : 0.f) + (other ? o2[j] * k_other : 0.f);
          }
          if (live) {
            f32x2 z = pack2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 16; ++j) z = fma2(pack2(o[2 * j], o[2 * j + 1]), pack2(0.f, 0.f), z);      // (NaN if one is not finite)
            void* dst;
            if (whole) {
              uint32_t w[16];
#pragma unroll
              for (int j = 0; j < 16; ++j) w[j] = PagedType<T>::pack(o[2 * j] * inv, o[2 * j + 1] * inv);
              dst = a.out + (out_row * DH + c0) * 2;
              if (out_32) {
                store32b(dst, w);
                store32b(reinterpret_cast<char*>(dst) + 32, w + 8);
              } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(dst) + 16 * j) = make_uint4(w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
              }
            } else {
              dst = a.parts + part * DH + c0;
#pragma unroll
              for (int j = 0; j < 4; ++j) store32b(reinterpret_cast<float*>(dst) + 8 * j, reinterpret_cast<const uint32_t*>(o) + 8 * j);
            }
            float z0, z1;
            unpack2(z, z0, z1);
            if (!(z0 + z1 == 0.f)) or_flag(f_odd, 1u << min(piece, 31u));
            if (p.again) {
              int lo, hi;
              range(lo, hi);
              add_odd<T, DH, kQuant>(a, p, both ? n >> 1 : n, lo, hi, c0, dst, !whole);
            }
          }
          __syncwarp();
        }
        if (live && (both || slot == 0)) {
          if (!whole) __stcg(reinterpret_cast<float2*>(a.parts_ml) + part, make_float2(m, l));
          else if (a.lse != nullptr) a.lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
        }
      }
      fence_before();
      if (p.opens && !whole && tid == 0) {               // (the run ends with this item)
        PagedSplit d;
        d.last = p.last;
        d.rows = min(a.item_rows, p.len * G - p.rg * a.item_rows);
        d.first_row = p.rg * a.item_rows; d.head = p.head; d.start = p.start;
        a.splits[cta] = d;
        set_flag(f_shares, 1);
      }
      if (!both) {                                       // both warpgroups have read both slots' O and the exchange rows
        __syncwarp();
        if (lane == 0) mbar_arrive(b_read);
        wait(b_read, turns & 1);
        ++turns;
        __syncwarp();
      }
      base += both ? n : 2 * n;
    }
    if (!met) again(true);
  }
  // ---------------------------------------------------------------------- teardown (all have met)
  if (tid == 0 && (flag(f_shares) == 0 || flag(f_abort) != 0)) a.splits[cta].last = flag(f_abort) != 0 ? kPagedGaveUp : kPagedNone;
  if (warp == kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Items that several CTAs share: their pieces added up, in the order of the keys, by a launch of its own.  (The last CTA to arrive did this inside the kernel at first: 430 KB through
// one SM, 5 us with its loads in flight together and 14 without.)  Bound by latencies: a list, a search, the pieces.  All rows are dealt out over all warps, two at a
// time for each (a 2,048-row prompt of the 8B shape, whose 148 CTAs share nearly every item: 69.7 us with one row at a time, 64.3 with two); where there are few rows a CTA has one at a time, its warps an eighth of the pieces each.
constexpr int kMergeWarps = 8, kMergeCtas = 3;    // CTAs per SM

// where output row `g` of the line of all split rows is kept, and by whom
struct MergeRow {
  int c0, c1, r;
};
struct MergeSum {
  float M, L;
};
template <int kV>
__device__ __forceinline__ void load_part(const PagedAttnArgs& a, int dh, int c, const MergeRow& w, int lane, float2& ml, float (&v)[kV]) {
  const long long at = ((long long)c * 2 + (c == w.c0 ? 1 : 0)) * kPagedMaxRows + w.r;
  ml = __ldcg(reinterpret_cast<const float2*>(a.parts_ml) + at);
  const float* src = a.parts + at * dh + lane * kV;
  if constexpr (kV == 4) {
    const float4 x = __ldcg(reinterpret_cast<const float4*>(src));
    v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
  } else if constexpr (kV == 2) {
    const float2 x = __ldcg(reinterpret_cast<const float2*>(src));
    v[0] = x.x; v[1] = x.y;
  } else {
    v[0] = __ldcg(src);
  }
}
// a piece to a sum with its own reference point
template <int kV>
__device__ __forceinline__ void add_part(MergeSum& s, float (&acc)[kV], float2 ml, const float (&v)[kV]) {
  if (ml.x == -INFINITY && ml.y == 0.f) return;                  // (it saw nothing)
  const float top = fmaxf(s.M, ml.x), keep = s.M == -INFINITY ? (s.L == 0.f ? 0.f : s.L) : paged_ex2(s.M - top), k = ml.x == -INFINITY ? 0.f : paged_ex2(ml.x - top);   // (a sum without a maximum is NaN)
  s.M = top;
  s.L = fmaf(k, ml.y, s.L * keep);
#pragma unroll
  for (int e = 0; e < kV; ++e) acc[e] = fmaf(k, v[e], acc[e] * keep);
}

template <typename T, int DH>
__global__ void __launch_bounds__(kMergeWarps * 32, kMergeCtas)
k_paged_merge(PagedAttnArgs a, int n_cta) {
  CS_PDL_PROLOGUE();
  constexpr int kV = DH / 32, kPerLane = kPagedMaxCtas / 32;     // columns of a lane; splits of a lane
  __shared__ PagedSplit s_split[kPagedMaxCtas];
  __shared__ int s_before[kPagedMaxCtas];         // rows of the items before
  __shared__ float2 s_ml[kMergeWarps];
  __shared__ __align__(16) float s_o[kMergeWarps][DH];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kGaveUp = 1 << 20;                // more rows than all items can have
  if (tid < kPagedMaxCtas) {
    PagedSplit d;
    d.last = kPagedNone; d.rows = 0;
    if (tid < n_cta) {
      const int* src = reinterpret_cast<const int*>(a.splits + tid);
      d.last = __ldcg(src); d.rows = __ldcg(src + 1); d.first_row = __ldcg(src + 2); d.head = __ldcg(src + 3); d.start = __ldcg(src + 4);
      if (d.last < 0) d.rows = d.last == kPagedGaveUp ? kGaveUp : 0;
    }
    s_split[tid] = d;
  }
  __syncthreads();
  // (every warp adds up for itself, all the same)
  int mine[kPerLane], total;
  for (;;) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) { mine[i] = sum; sum += s_split[lane * kPerLane + i].rows; }
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    total = __shfl_sync(0xffffffffu, inc, 31);
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) mine[i] += inc - sum;
    if (total < kGaveUp) break;
    // an item that one of its CTAs gave up on stays as it was: a piece is missing, and what lies in its place is an earlier call's
    __syncthreads();
    if (tid < n_cta) {
      bool whole = s_split[tid].last >= 0;
      for (int c = tid + 1; c <= s_split[tid].last; ++c) whole &= s_split[c].last != kPagedGaveUp;
      if (!whole) s_split[tid].rows = 0;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) s_before[lane * kPerLane + i] = mine[i];
  __syncwarp();
  auto find = [&](int g) -> MergeRow {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) n += mine[i] <= g;
    const int c0 = (int)__reduce_add_sync(0xffffffffu, (unsigned)n) - 1;            // the last item that begins at or before it (those without rows come first)
    return MergeRow{c0, s_split[c0].last, g - s_before[c0]};
  };
  auto write = [&](const MergeRow& w, const MergeSum& s, const float (&acc)[kV]) {
    const PagedSplit& d = s_split[w.c0];
    const float inv = s.L == 0.f ? 0.f : 1.f / s.L;
    const int m = d.first_row + w.r, q = a.by_group.of(m);
    const long long row = (long long)(d.start + q) * a.n_heads + d.head * a.group + (m - q * a.group);
    if constexpr (kV == 4)
      *reinterpret_cast<uint2*>(a.out + row * DH * 2 + lane * 8) = make_uint2(PagedType<T>::pack(acc[0] * inv, acc[1] * inv), PagedType<T>::pack(acc[2] * inv, acc[3] * inv));
    else if constexpr (kV == 2) *reinterpret_cast<uint32_t*>(a.out + row * DH * 2 + lane * 4) = PagedType<T>::pack(acc[0] * inv, acc[1] * inv);
    else *reinterpret_cast<unsigned short*>(a.out + row * DH * 2 + lane * 2) = (unsigned short)PagedType<T>::pack(acc[0] * inv, 0.f);
    if (a.lse != nullptr && lane == 0) a.lse[row] = s.L == 0.f ? -INFINITY : (s.M + log2f(s.L)) * 0.6931471805599453f;
  };

  if (total <= 2 * (int)gridDim.x) {
    for (int g = blockIdx.x; g < total; g += gridDim.x) {
      const MergeRow w = find(g);
      MergeSum s{-INFINITY, 0.f};
      float acc[kV] = {};
      constexpr int kBatch = 4;
      for (int cb = w.c0 + warp; cb <= w.c1; cb += kBatch * kMergeWarps) {
        float2 ml[kBatch];
        float v[kBatch][kV];
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (cb + i * kMergeWarps <= w.c1) load_part<kV>(a, DH, cb + i * kMergeWarps, w, lane, ml[i], v[i]);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
          if (cb + i * kMergeWarps <= w.c1) add_part<kV>(s, acc, ml[i], v[i]);
      }
      s_ml[warp] = make_float2(s.M, s.L);
#pragma unroll
      for (int e = 0; e < kV; ++e) s_o[warp][lane * kV + e] = acc[e];
      __syncthreads();
      if (warp == 0) {
        s = MergeSum{-INFINITY, 0.f};
#pragma unroll
        for (int e = 0; e < kV; ++e) acc[e] = 0.f;
#pragma unroll 1
        for (int i = 0; i < kMergeWarps; ++i) {
          float v[kV];
#pragma unroll
          for (int e = 0; e < kV; ++e) v[e] = s_o[i][lane * kV + e];
          add_part<kV>(s, acc, s_ml[i], v);
        }
        write(w, s, acc);
      }
      __syncthreads();
    }
    return;
  }
  constexpr int kAtOnce = 2, kPieces2 = 3;
  for (int g = (blockIdx.x * kMergeWarps + warp) * kAtOnce; g < total; g += gridDim.x * kMergeWarps * kAtOnce) {
    MergeRow w[kAtOnce];
    MergeSum s[kAtOnce];
    float acc[kAtOnce][kV];
    int most = 0;
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      w[j] = find(min(g + j, total - 1));
      s[j] = MergeSum{-INFINITY, 0.f};
      most = max(most, w[j].c1 - w[j].c0);
#pragma unroll
      for (int e = 0; e < kV; ++e) acc[j][e] = 0.f;
    }
    for (int i = 0; i <= most; i += kPieces2) {
      float2 ml[kAtOnce][kPieces2];
      float v[kAtOnce][kPieces2][kV];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int k = 0; k < kPieces2; ++k)
          if (w[j].c0 + i + k <= w[j].c1) load_part<kV>(a, DH, w[j].c0 + i + k, w[j], lane, ml[j][k], v[j][k]);
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
        for (int k = 0; k < kPieces2; ++k)
          if (w[j].c0 + i + k <= w[j].c1) add_part<kV>(s[j], acc[j], ml[j][k], v[j][k]);
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (g + j < total) write(w[j], s[j], acc[j]);
  }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                             CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static EncodeFn fn = []() -> EncodeFn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(p) : nullptr;
  }();
  return fn;
}
cs_status encode(cs_paged_cache* c, CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box, CUtensorMapL2promotion promote) {
  EncodeFn enc = encoder();
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  const CUresult r = enc == nullptr ? CUDA_ERROR_NOT_FOUND
                                    : enc(tm, c->cfg.dtype == CS_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void*>(base), dims, strides, box,
                                          ones, CU_TENSOR_MAP_INTERLEAVE_NONE, box[0] == 32 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, promote, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r == CUDA_SUCCESS) return CS_OK;
  snprintf(c->err, sizeof(c->err), "cuTensorMapEncodeTiled (rank %d) failed with %d", rank, (int)r);
  return CS_ERR_CUDA;
}

template <typename T, int DH, bool kQuant>
cs_status launch_tc(cs_paged_cache* c, const PagedAttnArgs& a, const CUtensorMap& tmQ, int q_box_bytes, unsigned bit, cudaStream_t st) {
  static_assert(kTcSmem<DH, kQuant> <= 227 * 1024, "");
  if (!(c->attr_set & bit)) {
    CS_CUDA_OK(c, cudaFuncSetAttribute(k_paged_tc<T, DH, kQuant>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTcSmem<DH, kQuant>));
    c->attr_set |= bit;
  }
  CS_CUDA_OK(c, cs_launch_pdl(k_paged_tc<T, DH, kQuant>, dim3(c->num_sms), dim3(kThreads<kQuant>), kTcSmem<DH, kQuant>, st, c->tmK, c->tmV, tmQ, a, q_box_bytes));
  CS_CUDA_OK(c, cs_launch_pdl(k_paged_merge<T, DH>, dim3(c->num_sms * kMergeCtas), dim3(kMergeWarps * 32), 0, st, a, c->num_sms));
  return CS_OK;
}

}  // namespace

cs_status cs_paged_tc_maps(cs_paged_cache* c) {
  const cs_paged_config& f = c->cfg;
  const cuuint64_t dims[4] = {(cuuint64_t)f.head_dim, (cuuint64_t)f.page_size, (cuuint64_t)f.n_kv_heads, (cuuint64_t)f.n_pages};
  const cuuint64_t strides[3] = {(cuuint64_t)f.slot_stride * 2, (cuuint64_t)f.head_stride * 2, (cuuint64_t)f.page_stride * 2};
  const cuuint32_t box[4] = {f.head_dim == 32 ? 32u : 64u, (cuuint32_t)(f.page_size < kPagedTile ? f.page_size : kPagedTile), 1, 1};
  // (rows of 128 bytes between those of other heads: 256 bytes at a time would fetch those as well: 8 x 21 rows over 16,384 keys, heads of 64, 78 / 67 us)
  const CUtensorMapL2promotion promote = f.slot_stride == f.head_dim || f.head_dim == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B
                                         : f.head_dim == 64                             ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B
                                                                                        : CU_TENSOR_MAP_L2_PROMOTION_L2_64B;
  const cs_status s = encode(c, &c->tmK, f.k, 4, dims, strides, box, promote);
  return s != CS_OK ? s : encode(c, &c->tmV, f.v, 4, dims, strides, box, promote);
}

namespace {
template <bool kQuant>
cs_status launch_any(cs_paged_cache* c, const PagedAttnArgs& args, cudaStream_t st) {
  PagedAttnArgs a = args;
  const int tokens = kM / a.group;                 // rows of the block in a slot, with all heads of the group
  a.item_rows = 2 * tokens * a.group;
  a.by_item_rows = PagedDivisor::by(a.item_rows);
  a.item_cost = 2;                                 // (one: 2 us more for the three windowed chunks)
  a.keep = 5;                                      // (a step takes 0.9 us, adding pieces up 5)
  const int box_rows = tokens < a.blk.rows ? tokens : a.blk.rows, dh = c->cfg.head_dim;
  CUtensorMap tmQ;
  // (a stride that no second row or head uses may be anything)
  const cuuint64_t dims[3] = {(cuuint64_t)dh, (cuuint64_t)a.n_heads, (cuuint64_t)a.blk.rows};
  const cuuint64_t strides[2] = {(cuuint64_t)(a.n_heads > 1 ? a.q_head : dh) * 2, (cuuint64_t)(a.blk.rows > 1 ? a.q_row : (long long)dh * a.n_heads) * 2};
  const cuuint32_t box[3] = {dh == 32 ? 32u : 64u, (cuuint32_t)a.group, (cuuint32_t)box_rows};
  const cs_status s = encode(c, &tmQ, a.q, 3, dims, strides, box, CU_TENSOR_MAP_L2_PROMOTION_L2_128B);
  if (s != CS_OK) return s;
  const int bytes = (dh == 32 ? 64 : 128) * a.group * box_rows;
  const bool bf = c->cfg.dtype == CS_BF16;
  constexpr unsigned kFirst = kQuant ? 4096 : 64;  // (bits of the instances)
  if (dh == 32) return bf ? launch_tc<__nv_bfloat16, 32, kQuant>(c, a, tmQ, bytes, kFirst * 16, st) : launch_tc<__half, 32, kQuant>(c, a, tmQ, bytes, kFirst * 32, st);
  if (dh == 64) return bf ? launch_tc<__nv_bfloat16, 64, kQuant>(c, a, tmQ, bytes, kFirst, st) : launch_tc<__half, 64, kQuant>(c, a, tmQ, bytes, kFirst * 2, st);
  return bf ? launch_tc<__nv_bfloat16, 128, kQuant>(c, a, tmQ, bytes, kFirst * 4, st) : launch_tc<__half, 128, kQuant>(c, a, tmQ, bytes, kFirst * 8, st);
}
}  // namespace

cs_status cs_launch_paged_tc(cs_paged_cache* c, const PagedAttnArgs& a, cudaStream_t st) { return launch_any<false>(c, a, st); }
cs_status cs_launch_quant_tc(cs_paged_cache* c, const PagedAttnArgs& a, cudaStream_t st) { return launch_any<true>(c, a, st); }
