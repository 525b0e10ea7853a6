// Attention of few query rows per KV head over a paged cache held in 4 bits: single tokens, verification blocks, and taller blocks where there is no room for copies (Sec. 3.2; App. B.2),
// on mma.sync.  (Which calls come here: cs_quant_attention in cs_quant.cu.)
//
// out = softmax(scale Q K^T) V by one pass over the keys with a running reference point m and sum l per row, as in cs_paged_attn.cu.  What differs comes from the cache: a value costs 4.5 bits of
// HBM and about two instructions, so that what a key costs an SM is counted in instructions, and the products are laid out so that every value is expanded once for up to 32 query rows:
//     S^T [16 keys x 8 rows]  = K Q^T      A = keys as they come out of their words, B = queries
//     O^T [16 dims x 8 rows] += V^T P^T    A = values, two keys of one element in a register, B = weights
// Keys and head dims are the M of m16n8k16, query rows the N: 8, 16, 24 or 32 of them, a template parameter.  A lane's words of a key hold elements of one group, so that it needs one scale of each key.
// The MMA's sums over k do not care which element stands where: lane t's k are those of its own words.  Values: neighbouring keys of one element come of two keys' words by a byte
// permutation.  Weights change places with a transposition of 8 x 8 blocks (movmatrix).
// Values are exact in bf16 (cs_quant.cuh).  Queries of fp16 go in as two bf16 terms (value = hi + lo, exact), weights as two (16 bits of them), so nothing but the result is rounded to 16 bits.
//
// Persistent: CTAs take equal runs of the line of key tiles (cs_paged.cuh).  A tile's 128 keys are four slices of 32, dealt out to the warps in turn; a slice lies in two pages at most.
// Every warp has its own ring of slices, fetched by cp.async, its own reference points, sums and output; the warps' results meet in shared memory where the item ends, and items that
// CTAs share meet in global memory: the last one to arrive adds the pieces up in the order of the keys.
// The reference point moves only past 2^8, by a vote; where no score is above, no maximum is worked out.
//
// Masked keys: scores become -inf.  Slices that lie outside of [lo, hi) of the item's rows are not fetched.  In slices that some rows see and others do not, V scales that are not
// finite become 0 and the rows that see such a key are given NaN (0 x NaN is not 0).
#include "cs_quant.cuh"

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32, kSlice = 32;
typedef PagedPlanOf<kQuantMaxSeqs> Plan;

template <int DH, int NT> struct Few {
  static constexpr int kCols = 8 * NT;                       // query rows of an item
  static constexpr int kCtas = NT == 1 ? 2 : 1;              // on an SM
  static constexpr int kStages = NT == 1 ? 2 : 3;
  static constexpr int kKeyBytes = DH / 2, kScaleBytes = DH / 16;
  static constexpr int kData = kSlice * kKeyBytes, kScales = kSlice * kScaleBytes, kStage = 2 * (kData + kScales);
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kPass = DH < 64 ? DH : 64;            // columns of the results that warps exchange at a time
  static constexpr int kLd = kPass + 4;
  static constexpr int kExchange = kWarps * 8 * kLd * 4;
  static constexpr int kQRow = DH * 2 + (DH == 32 ? 0 : 64); // bytes of a query row (the rest keeps rows out of each other's banks)
  static constexpr int kQ = kCols * kQRow;                   // one of two terms
  static constexpr int kMl = kWarps * kCols * 8;
  static constexpr int kSmem = kRing + kExchange + 2 * kQ + kMl + (int)sizeof(Plan) + 16;
};

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Where 16-byte chunk c of key j of a slice lies, in chunks, so that neither the keys' loads (keys g / 2 + 4 (g % 2) of eight) nor the values' (keys 0 - 3) meet in a bank.
template <int DH>
__device__ __forceinline__ uint32_t at_chunk(uint32_t j, uint32_t c) {
  if constexpr (DH == 128) return (j * 4 + c) ^ ((j >> 1 & 1) * 2) ^ ((j >> 2 & 1) * 4);
  else if constexpr (DH == 64) return (j * 2 + c) ^ ((j >> 2 & 1) * 4);
  else return j;
}

template <int DH, int NT>
__global__ void __launch_bounds__(kThreads, Few<DH, NT>::kCtas)
k_quant_few(const __grid_constant__ QuantAttnArgs qa) {
  CS_PDL_PROLOGUE();
  typedef Few<DH, NT> F;
  constexpr int kStages = F::kStages, kCols = F::kCols, kWordsK = DH / 32, kTiles = DH / 16, kChunks = DH / 32;      // words of a key for a lane; tiles of 16 head dims; 16-byte chunks of a key
  const PagedAttnArgs& a = qa.p;
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* ring = smem;                                                          // [warp][stage]: K, V, K scales, V scales
  float* s_x = reinterpret_cast<float*>(ring + F::kRing);                        // [warp][8 rows][kLd]
  uint8_t* s_q = reinterpret_cast<uint8_t*>(s_x) + F::kExchange;                 // [term][row][word of a lane][lane t][8 elements]
  float2* s_ml = reinterpret_cast<float2*>(s_q + 2 * F::kQ);                     // [warp][row]
  Plan& plan = *reinterpret_cast<Plan*>(reinterpret_cast<uint8_t*>(s_ml) + F::kMl);
  int* s_last = reinterpret_cast<int*>(&plan + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

  paged_plan(a, plan);
  const long long total = plan.before[a.blk.n_seqs];
  const int n_cta = (int)min((long long)gridDim.x, total), cta = blockIdx.x;
  if (cta >= n_cta) return;
  long long run1;
  PagedPiece p = paged_run(a, plan, total, n_cta, cta, lane, run1), f = p;
  if (p.n_tiles == 0) return;
  const int G = a.group;

  // ---- queries: of the piece behind the one at hand, in registers until that one is done
  constexpr int kQWords = (kCols * DH / 8 + kThreads - 1) / kThreads;      // eight elements each
  uint4 q_next[kQWords];
  auto ask = [&](const PagedPiece& x) {
#pragma unroll
    for (int i = 0; i < kQWords; ++i) {
      const int e = tid + i * kThreads, row = e / (DH / 8), c = e % (DH / 8), m = x.rg * kCols + row, r = a.by_group.of(m);
      q_next[i] = make_uint4(0u, 0u, 0u, 0u);
      if (row < kCols && m < x.len * G) q_next[i] = __ldg(reinterpret_cast<const uint4*>(a.q + ((x.start + r) * a.q_row + (x.head * G + m - r * G) * a.q_head + c * 8) * 2));
    }
  };
  auto keep = [&]() {
#pragma unroll
    for (int i = 0; i < kQWords; ++i) {
      const int e = tid + i * kThreads, row = e / (DH / 8), c = e % (DH / 8);
      if (row >= kCols) continue;
      uint4* dst = reinterpret_cast<uint4*>(s_q + row * F::kQRow + (c % kWordsK * 4 + c / kWordsK) * 16);
      if (!qa.half) {
        *dst = q_next[i];
        continue;
      }
      uint32_t w[4] = {q_next[i].x, q_next[i].y, q_next[i].z, q_next[i].w}, hi[4], lo[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 x = PagedType<__half>::unpack(w[j]);
        hi[j] = PagedType<__nv_bfloat16>::pack(x.x, x.y);
        const float2 y = PagedType<__nv_bfloat16>::unpack(hi[j]);
        lo[j] = PagedType<__nv_bfloat16>::pack(isfinite(x.x) ? x.x - y.x : 0.f, isfinite(x.y) ? x.y - y.y : 0.f);
      }
      dst[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(dst) + F::kQ) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
  };
  ask(p);

  // ---- the fetching side: runs kStages slices ahead, across pieces
  const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(warp * kStages * F::kStage);
  const uint8_t* my_ring_p = ring + warp * kStages * F::kStage;
  int f_turn = 0, f_slice = warp, f_n = 0, f_entry = 0, f_stage = 0;    // slices of the pieces before, modulo the warps; next slice of the piece; how many of them before; page-table entry of this lane
  bool f_more = true;
  // entries of this warp's next sixteen slices' halves, one per lane
  auto entries = [&]() {
    const long long k = ((long long)f.tile0 * 4 + f_slice + kWarps * (lane >> 1)) * kSlice + (lane & 1) * 16;      // (the last lanes' may lie behind 2^31)
    f_entry = k < f.hi && k + 16 > f.lo ? __ldcg(a.blk.table + (long long)f.seq * a.blk.table_width + (k >> a.kv.page_shift)) : 0;
  };
  // on to a piece that has slices for this warp
  auto settle = [&]() {
    while (f_more && f_slice >= 4 * f.n_tiles) {
      f_turn = (f_turn + 4 * f.n_tiles) % kWarps;
      f_more = paged_next(a, plan, f, run1);
      f_slice = (warp + kWarps - f_turn) % kWarps;
      f_n = 0;
    }
  };
  settle();
  if (f_more) entries();
  auto fetch = [&]() {
    if (f_more) {
      const int key0 = (f.tile0 * 4 + f_slice) * kSlice;
      const uint32_t dst = my_ring + (uint32_t)(f_stage * F::kStage);
      const char *src[2][2], *scl[2][2];          // [K, V][half]
      bool on[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = key0 + 16 * h, page = __shfl_sync(0xffffffffu, f_entry, (f_n & 15) * 2 + h);
        const bool used = k < f.hi && k + 16 > f.lo, exists = (unsigned)page < (unsigned)a.kv.n_pages;
        if (used && !exists && lane == 0) atomicOr(a.status, CS_DEV_BADARG);
        on[h] = used && exists;
        const long long row = on[h] ? (long long)f.head * a.kv.page_size + (k & (a.kv.page_size - 1)) : 0, at = on[h] ? page : 0;
        const long long d = (at * qa.kv.data_page + row * (DH / 8)) * 4, s = (at * qa.kv.scale_page + row * (DH / kQuantGroup)) * 2;
        src[0][h] = reinterpret_cast<const char*>(qa.kv.k) + d; src[1][h] = reinterpret_cast<const char*>(qa.kv.v) + d;
        scl[0][h] = reinterpret_cast<const char*>(qa.kv.ks) + s; scl[1][h] = reinterpret_cast<const char*>(qa.kv.vs) + s;
      }
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int e = i * 32 + lane, j = e / kChunks, c = e % kChunks, h = j >> 4, in = (e - h * 16 * kChunks) * 16;
        const uint32_t at = at_chunk<DH>(j, c) * 16;
        cp16(dst + at, (h ? src[0][1] : src[0][0]) + in, h ? on[1] : on[0]);
        cp16(dst + F::kData + at, (h ? src[1][1] : src[1][0]) + in, h ? on[1] : on[0]);
      }
      constexpr int kN = DH / 16;                 // 16-byte chunks of a half's scales
      if (lane < 4 * kN) {
        const int which = lane / (2 * kN), h = lane / kN & 1, c = lane % kN;
        const char* s = which ? (h ? scl[1][1] : scl[1][0]) : (h ? scl[0][1] : scl[0][0]);
        cp16(dst + 2 * F::kData + which * F::kScales + (h * kN + c) * 16, s + c * 16, h ? on[1] : on[0]);
      }
      if (++f_stage == kStages) f_stage = 0;
      f_slice += kWarps;
      ++f_n;
      const bool same = f_slice < 4 * f.n_tiles;
      if (!same) settle();
      if (f_more && (!same || (f_n & 15) == 0)) entries();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) fetch();
  keep();
  __syncthreads();

  // items shared with other CTAs, at most two: the run's first and its last
  struct Shared { int c0, c1, start, len, rg, head; } shared[2] = {{-1, 0, 0, 0, 0, 0}, {-1, 0, 0, 0, 0, 0}};
  int stage = 0, turn = 0;
  for (bool more = true; more;) {
    PagedPiece next = p;
    more = paged_next(a, plan, next, run1);
    if (more) ask(next);
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

    for (int i = (warp + kWarps - turn) % kWarps; i < 4 * p.n_tiles; i += kWarps) {
      const int key0 = (p.tile0 * 4 + i) * kSlice;
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      if (key0 < p.hi && key0 + kSlice > p.lo) {
        const uint8_t* st = my_ring_p + stage * F::kStage;
        const uint8_t *kd = st, *vd = st + F::kData, *ks = st + 2 * F::kData, *vs = ks + F::kScales;
        const bool mixed = key0 < all_lo || key0 + kSlice > all_hi;      // some row does not see all of it
        // ---- S^T = K Q^T
        float s[2][NT][4];
        uint32_t kw[2][2][kWordsK];               // [16 keys][row g, g + 8]
        QuantScale sc[2][2];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const uint32_t j = 16 * mt + 8 * b + (g >> 1) + 4 * (g & 1);
            if constexpr (DH == 128) {
              const uint4 w = *reinterpret_cast<const uint4*>(kd + at_chunk<DH>(j, t) * 16);
              kw[mt][b][0] = w.x; kw[mt][b][1] = w.y; kw[mt][b][2] = w.z; kw[mt][b][3] = w.w;
            } else if constexpr (DH == 64) {
              const uint2 w = *reinterpret_cast<const uint2*>(kd + at_chunk<DH>(j, t >> 1) * 16 + (t & 1) * 8);
              kw[mt][b][0] = w.x; kw[mt][b][1] = w.y;
            } else {
              kw[mt][b][0] = *reinterpret_cast<const uint32_t*>(kd + at_chunk<DH>(j, 0) * 16 + t * 4);
            }
            sc[mt][b] = QuantScale::of(*reinterpret_cast<const unsigned short*>(ks + j * F::kScaleBytes + (DH == 128 ? t : DH == 64 ? t >> 1 : 0) * 2) * 0x10001u);
          }
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) s[mt][nt][0] = s[mt][nt][1] = s[mt][nt][2] = s[mt][nt][3] = 0.f;
#pragma unroll
        for (int w = 0; w < kWordsK; ++w) {
          uint32_t x[2][2][4];
#pragma unroll
          for (int mt = 0; mt < 2; ++mt) {
            quant_expand(kw[mt][0][w], sc[mt][0], x[mt][0]);
            quant_expand(kw[mt][1][w], sc[mt][1], x[mt][1]);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            const uint8_t* qp = s_q + (8 * nt + g) * F::kQRow + (w * 4 + t) * 16;
            const uint4 hi = *reinterpret_cast<const uint4*>(qp);
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
              mma(s[mt][nt], x[mt][0][0], x[mt][1][0], x[mt][0][1], x[mt][1][1], hi.x, hi.y);
              mma(s[mt][nt], x[mt][0][2], x[mt][1][2], x[mt][0][3], x[mt][1][3], hi.z, hi.w);
            }
            if (qa.half) {
              const uint4 lo = *reinterpret_cast<const uint4*>(qp + F::kQ);
#pragma unroll
              for (int mt = 0; mt < 2; ++mt) {
                mma(s[mt][nt], x[mt][0][0], x[mt][1][0], x[mt][0][1], x[mt][1][1], lo.x, lo.y);
                mma(s[mt][nt], x[mt][0][2], x[mt][1][2], x[mt][0][3], x[mt][1][3], lo.z, lo.w);
              }
            }
          }
        }
        // ---- masks  (key of row g + 8 b of S^T: as loaded)
        if (mixed) {
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
        const int vg = DH == 128 ? g >> 1 : DH == 64 ? g >> 2 : 0;      // this lane's group of the values
        bool odd = false;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) {
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
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t key = 16 * mt + t + 4 * j;
            if constexpr (DH == 128) {
              const uint2 w = *reinterpret_cast<const uint2*>(vd + at_chunk<DH>(key, g >> 1) * 16 + (g & 1) * 8);
              vw[j][0] = w.x; vw[j][1] = w.y;
            } else if constexpr (DH == 64) {
              vw[j][0] = *reinterpret_cast<const uint32_t*>(vd + at_chunk<DH>(key, g >> 2) * 16 + (g & 3) * 4);
            } else {
              vw[j][0] = *reinterpret_cast<const uint32_t*>(vd + at_chunk<DH>(key, 0) * 16 + (g >> 1) * 4) >> (8 * (g & 1));
            }
            sv[j] = *reinterpret_cast<const unsigned short*>(vs + key * F::kScaleBytes + vg * 2);
          }
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
            for (int k = 0; k < (DH == 32 ? 2 : 4); ++k)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma(o[w * 4 + k][nt], x[0][0][k], x[0][1][k], x[1][0][k], x[1][1][k], ph[nt][0], ph[nt][1]);
                mma(o[w * 4 + k][nt], x[0][0][k], x[0][1][k], x[1][0][k], x[1][1][k], pl[nt][0], pl[nt][1]);
              }
          }
        }
        if (mixed && __any_sync(0xffffffffu, odd)) {
          // values that are not finite: the rows that see them become NaN there
#pragma unroll 1
          for (int j = 0; j < kSlice; ++j) {
            if (!quant_odd(*reinterpret_cast<const unsigned short*>(vs + j * F::kScaleBytes + vg * 2))) continue;
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
      if (++stage == kStages) stage = 0;
      fetch();
    }
    turn = (turn + 4 * p.n_tiles) % kWarps;

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
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int w = 0; w < kPasses; ++w) {
        // elements kMine kPasses g + kMine w + i of rows 2 t + e are number kMine g + i of the pass
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float4* dst = reinterpret_cast<float4*>(s_x + (warp * 8 + 2 * t + e) * F::kLd + kMine * g);
#pragma unroll
          for (int i = 0; i < kMine / 4; ++i) {
            const int k = w * 4 + 2 * i;
            dst[i] = make_float4(o[k][nt][e], o[k][nt][2 + e], o[k + 1][nt][e], o[k + 1][nt][2 + e]);
          }
        }
        __syncthreads();
        const int n = 8 * nt + warp;             // a warp has one of the eight rows
        if (n < rows && 2 * lane < F::kPass) {
          float M = -INFINITY, L = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll
          for (int v = 0; v < kWarps; ++v) M = fmaxf(M, s_ml[v * kCols + n].x);
#pragma unroll
          for (int v = 0; v < kWarps; ++v) {
            const float2 ml = s_ml[v * kCols + n];
            const float2 y = *reinterpret_cast<const float2*>(s_x + (v * 8 + warp) * F::kLd + 2 * lane);
            if (ml.x == -INFINITY && ml.y == 0.f) continue;      // (it saw nothing)
            const float k = ml.x == -INFINITY ? 0.f : paged_ex2(ml.x - M);
            L = fmaf(k, ml.y, L);
            x0 = fmaf(k, y.x, x0);
            x1 = fmaf(k, y.y, x1);
          }
          const int d = 2 * lane / kMine * (kMine * kPasses) + kMine * w + 2 * lane % kMine;
          if (p.whole) {
            const float inv = L == 0.f ? 0.f : 1.f / L;
            const int mrow = p.rg * kCols + n, r = a.by_group.of(mrow);
            const long long at = (long long)(p.start + r) * a.n_heads + p.head * G + (mrow - r * G);
            *reinterpret_cast<uint32_t*>(a.out + (at * DH + d) * 2) = qa.half ? PagedType<__half>::pack(x0 * inv, x1 * inv) : PagedType<__nv_bfloat16>::pack(x0 * inv, x1 * inv);
            if (a.lse != nullptr && lane == 0 && w == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
          } else {
            const long long at = ((long long)cta * 2 + (p.opens ? 1 : 0)) * kQuantMaxRows + n;
            __stcg(reinterpret_cast<float2*>(a.parts + at * DH + d), make_float2(x0, x1));
            if (lane == 0 && w == 0) __stcg(reinterpret_cast<float2*>(a.parts_ml) + at, make_float2(M, L));
          }
        }
        __syncthreads();                         // (the exchange rows are free again)
      }
    if (!p.whole) {
      const Shared s = {paged_first_cta(a, p, total, n_cta), paged_last_cta(a, p, total, n_cta), p.start, p.len, p.rg, p.head};
      if (p.opens) shared[1] = s;
      else shared[0] = s;
    }
    p = next;
    if (more) {
      keep();                                    // (nobody reads the queries of the piece before any more)
      __syncthreads();
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- shared items: the CTA that arrives last adds the pieces up, in the order of the keys
  if (shared[0].c0 < 0 && shared[1].c0 < 0) return;
  __threadfence();
  __syncthreads();
  if (tid < 2) {
    const int c0 = tid == 0 ? shared[0].c0 : shared[1].c0, c1 = tid == 0 ? shared[0].c1 : shared[1].c1;
    int last = 0;
    if (c0 >= 0) {
      last = atomicAdd(a.counters + c0, 1) == c1 - c0;
      if (last) a.counters[c0] = 0;
    }
    s_last[tid] = last;
  }
  __syncthreads();
#pragma unroll 1
  for (int which = 0; which < 2; ++which) {
    if (!s_last[which]) continue;
    __threadfence();
    const Shared s = which == 0 ? shared[0] : shared[1];
    // The pieces come into the ring, all in flight together, and are added up from there.
    const int rows = min(kCols, s.len * G - s.rg * kCols), fit = min(F::kRing / (rows * DH * 4), F::kExchange / (kCols * 8));
    constexpr int kTasks = (kCols * DH / 4 + kThreads - 1) / kThreads;      // (row, four columns) of a thread
    const uint32_t s_parts = (uint32_t)__cvta_generic_to_shared(ring), s_pml = (uint32_t)__cvta_generic_to_shared(s_x);
    float2* pml = reinterpret_cast<float2*>(s_x);      // [piece][row]: reference point, then weight; sum
    float acc[kTasks][4];
#pragma unroll
    for (int k = 0; k < kTasks; ++k) acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.f;
    if (tid < kCols) s_ml[tid] = make_float2(-INFINITY, 0.f);               // a row's reference point and sum so far
#pragma unroll 1
    for (int cb = s.c0; cb <= s.c1; cb += fit) {
      const int n = min(fit, s.c1 - cb + 1);
#pragma unroll 1
      for (int i = warp; i < n; i += kWarps) {
        const long long at = ((long long)(cb + i) * 2 + (cb + i == s.c0 ? 1 : 0)) * kQuantMaxRows;
        const float* src = a.parts + at * DH + lane * 4;
        const uint32_t dst = s_parts + (uint32_t)((i * rows * (DH / 4) + lane) * 16);
        if (2 * lane < rows) cp16(s_pml + (uint32_t)((i * kCols + 2 * lane) * 8), a.parts_ml + (at + 2 * lane) * 2, true);
#pragma unroll 4
        for (int j = lane; j < rows * (DH / 4); j += 32) cp16(dst + (uint32_t)((j - lane) * 16), src + (j - lane) * 4, true);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
#pragma unroll 1
      for (int row = warp; row < rows; row += kWarps) {
        const float2 old = s_ml[row];
        float top = old.x, sum = 0.f;
        for (int j = lane; j < n; j += 32) top = fmaxf(top, pml[j * kCols + row].x);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        for (int j = lane; j < n; j += 32) {
          const float2 x = pml[j * kCols + row];
          const float w = x.x == -INFINITY ? 0.f : paged_ex2(x.x - top);
          sum += x.x == -INFINITY && x.y == 0.f ? 0.f : w * x.y;           // (without a maximum, but a sum: NaN)
          pml[j * kCols + row].x = w;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) {
          const float kept = old.x == -INFINITY ? 1.f : paged_ex2(old.x - top);
          s_ml[row] = make_float2(top, old.y * kept + sum);
          s_ml[kCols + row].x = kept;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kTasks; ++k) {
        const int row = (tid + k * kThreads) / (DH / 4), c4 = (tid + k * kThreads) % (DH / 4);
        if (row >= rows) continue;
        const float kept = s_ml[kCols + row].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] *= kept;
        const float4* v = reinterpret_cast<const float4*>(ring) + row * (DH / 4) + c4;
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
          const float2 x = pml[j * kCols + row];
          const float4 y = v[j * rows * (DH / 4)];
          if (x.x == 0.f && x.y == 0.f) continue;                          // (a piece that saw nothing)
          acc[k][0] = fmaf(x.x, y.x, acc[k][0]); acc[k][1] = fmaf(x.x, y.y, acc[k][1]); acc[k][2] = fmaf(x.x, y.z, acc[k][2]); acc[k][3] = fmaf(x.x, y.w, acc[k][3]);
        }
      }
      __syncthreads();                           // (the ring is free again)
    }
#pragma unroll
    for (int k = 0; k < kTasks; ++k) {
      const int row = (tid + k * kThreads) / (DH / 4), c4 = (tid + k * kThreads) % (DH / 4) * 4;
      if (row >= rows) continue;
      const float2 ml = s_ml[row];
      const float inv = ml.y == 0.f ? 0.f : 1.f / ml.y;
      const int mrow = s.rg * kCols + row, r = a.by_group.of(mrow);
      const long long at = (long long)(s.start + r) * a.n_heads + s.head * G + (mrow - r * G);
      const float x0 = acc[k][0] * inv, x1 = acc[k][1] * inv, x2 = acc[k][2] * inv, x3 = acc[k][3] * inv;
      *reinterpret_cast<uint2*>(a.out + (at * DH + c4) * 2) = qa.half ? make_uint2(PagedType<__half>::pack(x0, x1), PagedType<__half>::pack(x2, x3))
                                                                      : make_uint2(PagedType<__nv_bfloat16>::pack(x0, x1), PagedType<__nv_bfloat16>::pack(x2, x3));
      if (a.lse != nullptr && c4 == 0) a.lse[at] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

template <int DH, int NT>
cs_status launch_few(cs_quant_cache* c, const QuantAttnArgs& a, unsigned bit, cudaStream_t st) {
  typedef Few<DH, NT> F;
  static_assert(F::kCtas * (F::kSmem + 1024) <= 227 * 1024 + 1024 && kQuantMaxRows >= F::kCols, "");
  if (!(c->attr_set & bit)) {
    CS_CUDA_OK(c, cudaFuncSetAttribute(k_quant_few<DH, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::kSmem));
    c->attr_set |= bit;
  }
  CS_CUDA_OK(c, cs_launch_pdl(k_quant_few<DH, NT>, dim3(c->num_sms * F::kCtas), dim3(kThreads), F::kSmem, st, a));
  return CS_OK;
}
template <int DH>
cs_status launch_few_rows(cs_quant_cache* c, const QuantAttnArgs& a, int tiles, unsigned bit, cudaStream_t st) {
  switch (tiles) {
    case 1: return launch_few<DH, 1>(c, a, bit, st);
    case 2: return launch_few<DH, 2>(c, a, bit << 1, st);
    case 3: return launch_few<DH, 3>(c, a, bit << 2, st);
    default: return launch_few<DH, 4>(c, a, bit << 3, st);
  }
}

}  // namespace

cs_status cs_launch_quant_few(cs_quant_cache* c, const QuantAttnArgs& args, cudaStream_t st) {
  QuantAttnArgs a = args;
  // Items of as few query rows as leave no fewer items: a KV head's rows (on the average of the sequences, which is what the host knows) in equal shares of up to 32
  const long long rows = ((long long)a.p.blk.rows * a.p.group + a.p.blk.n_seqs - 1) / a.p.blk.n_seqs, items = (rows + kQuantMaxRows - 1) / kQuantMaxRows;
  const int tiles = (int)(((rows + items - 1) / items + 7) / 8);
  a.p.item_rows = 8 * tiles;
  a.p.by_item_rows = PagedDivisor::by(a.p.item_rows);
  a.p.item_cost = 2;
  a.p.keep = 4;
  switch (c->cfg.head_dim) {
    case 32: return launch_few_rows<32>(c, a, tiles, 1, st);
    case 64: return launch_few_rows<64>(c, a, tiles, 16, st);
    default: return launch_few_rows<128>(c, a, tiles, 256, st);
  }
}
