// Attention of few query rows per KV head over a paged KV cache: single tokens and short verification blocks
// (Sec. 3.2; App. B.2), on mma.sync.  (Which calls come here: cs_paged_attention in cs_paged.cu.)
//
// out = softmax(scale Q K^T) V by one pass over the keys with a running maximum m and sum l per row:
//     m' = max(m, max_j s_j),  l' = l 2^(m - m') + sum_j 2^(s_j - m'),  O' = O 2^(m - m') + sum_j 2^(s_j - m') V_j   (base-2 scores).
//
// Persistent: a CTA per SM takes an equal run of the line of key tiles (cs_paged.cuh).  A tile's 128 keys are cut into eight slices
// of 16, one for each warp: a slice never crosses a page (pages are powers of two from 16 on).  Every warp has its own ring of slices, fetched by cp.async
// with a page-table entry each, its own running maximum, sum and output, so nothing is waited for inside the CTA until the item ends; then the warps'
// results meet in shared memory.  Items that several CTAs share meet in global memory: each leaves its un-normalised
// piece, the last one to arrive (a counter) adds the pieces up in the order of the keys, so results do not depend on who was last.
// Sixteen query rows (token x head of the group) are the M of m16n8k16; the softmax weights, in the layout the scores come in, are the
// second product's A operand, as two 16-bit terms (value = hi + lo): the tensor pipe has the room, and the weights stay as
// exact as the scores.  In fp16 they are 2^14 times as large, by a reference point that much lower: of weights up to 1 both terms of one below 2^-25 are 0, and tens of thousands of such are more than the type's rounding.
//
// Masked keys: scores become -inf.  Keys outside [lo, hi) of the item's rows are never fetched (cp.async fills zeros), so
// what lies there, freed pages included, does not matter.  Slices that some rows see and others do not are looked through for
// values that are not finite, since 0 x inf is not 0: with any, the second product is done by plain arithmetic over the keys each row sees.
//
// Bound by HBM (K and V once) where the cache is long, by a chain of latencies (plan 1.5 us, piece 0.5, page entries and first slices 1.4, results 1.3, adding pieces up 4) where it is
// short.  8B shape, bf16 or fp16: one token over 30,720 keys 29 us (126 MB, 19.2 at the copy rate; the keys themselves come in 18), 64 over 500 - 4,097 keys 72 us (404 MB, 62; 78 among calls on other caches); the small model's 11
// rows over 512 keys 8.0 us.  What made it: queries fetched with their piece instead of behind all keys in flight (3 us a piece), shared items settled after the run and added up from shared
// memory (10 -> 4 us), two places of the line for changing items.  ex2 and the products take a third of the issue slots at most.
#include <type_traits>

#include "cs_paged.cuh"

namespace {

constexpr int kWarps = 8, kThreads = kWarps * 32, kSlice = 16, kRows = 16;
template <typename T> constexpr float kUp = std::is_same<T, __half>::value ? 14.f : 0.f;      // how far below a row's largest score its reference point is put
template <int DH> constexpr int kFewStages = DH == 128 ? 2 : 4;
template <int DH> constexpr int kFewSmem = kWarps * kFewStages<DH> * 2 * kSlice * DH * 2 + kWarps * kRows * (DH + 8) * 4 + kWarps * kRows * 8 +
                                         (kFewStages<DH> + 1) * kRows * DH * 2 + (int)sizeof(PagedPlan) + 16;

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// where 16-byte chunk c of row j of a slice lies, so that eight rows' chunks of one column fall into different banks
template <int DH>
__device__ __forceinline__ uint32_t at_chunk(int j, int c) {
  return DH == 32 ? (uint32_t)(j * 64 + ((c ^ ((j >> 1) & 3)) << 4)) : (uint32_t)(j * DH * 2 + ((c ^ (j & 7)) << 4));
}
// a word of two 16-bit values: is one of them not finite?
template <typename T>
__device__ __forceinline__ bool odd_pair(uint32_t w) {
  constexpr uint32_t e = std::is_same<T, __nv_bfloat16>::value ? 0x7f80u : 0x7c00u;
  return (w & e) == e || ((w >> 16) & e) == e;
}

template <typename T, int DH>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_few(PagedAttnArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kStages = kFewStages<DH>, CPR = DH / 8, kSliceBytes = kSlice * DH * 2, kSteps = DH / 16, kLd = DH + 8;
  constexpr int kIter = kSlice * CPR / 32;       // 16-byte copies per lane of K, and of V
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* ring = smem;                                                                  // [warp][stage][K, V][16 keys][DH]
  float* s_o = reinterpret_cast<float*>(ring + kWarps * kStages * 2 * kSliceBytes);        // [warp][16 rows][kLd]
  float2* s_ml = reinterpret_cast<float2*>(s_o + kWarps * kRows * kLd);                      // [warp][16 rows]
  uint8_t* s_q = reinterpret_cast<uint8_t*>(s_ml + kWarps * kRows);                          // [kStages + 1][16 rows][DH]: queries of the pieces being fetched
  PagedPlan& plan = *reinterpret_cast<PagedPlan*>(s_q + (kStages + 1) * kRows * DH * 2);
  int* s_last = reinterpret_cast<int*>(&plan + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;

  paged_plan(a, plan);
  const long long total = plan.before[a.blk.n_seqs];
  const int n_cta = (int)min((long long)gridDim.x, total), cta = blockIdx.x;
  if (cta >= n_cta) return;

  const uint32_t my_ring = (uint32_t)__cvta_generic_to_shared(ring) + (uint32_t)(warp * kStages * 2 * kSliceBytes);
  const uint8_t* my_ring_p = ring + warp * kStages * 2 * kSliceBytes;

  // ---- the fetching side: runs kStages slices ahead, across pieces
  long long run1;
  PagedPiece p = paged_run(a, plan, total, n_cta, cta, lane, run1), f = p;
  if (p.n_tiles == 0) return;
  const int G = a.group;
  int f_tile = 0, f_entry = 0, f_stage = 0, f_q = 0, q_at = 0;
  // Queries go through shared memory, with the fetched piece: two rows by every warp.  (Loaded where the piece begins they waited behind all keys in flight: 2.5 us.)
  auto queries = [&]() {
    const int row = lane / CPR + warp * 2, c = lane % CPR, m = f.rg * kRows + row, r = a.by_group.of(m);
    if (lane < 2 * CPR) {
      const bool live = m < f.len * G;
      const char* src = a.q + (live ? (f.start + r) * a.q_row + (f.head * G + m - r * G) * a.q_head + c * 8 : 0) * 2;
      cp16((uint32_t)__cvta_generic_to_shared(s_q) + (uint32_t)(f_q * kRows * DH * 2) + at_chunk<DH>(row, c), src, live);
    }
    if (++f_q == kStages + 1) f_q = 0;
  };
  queries();
  bool f_more = true;
  // page-table entries of this warp's slices of the next 32 tiles, one per lane: asked for a slice before the first is needed
  auto entries = [&]() {
    const long long k = (long long)(f.tile0 + f_tile + lane) * kPagedTile + warp * kSlice;      // (the last lanes' may lie behind 2^31)
    f_entry = k < f.hi && k + kSlice > f.lo ? __ldcg(a.blk.table + (long long)f.seq * a.blk.table_width + (k >> a.kv.page_shift)) : 0;
  };
  const long long lane_off = (lane / CPR * a.kv.slot_stride + lane % CPR * 8) * 2, hop = 32 / CPR * a.kv.slot_stride * 2;   // this lane's chunks of a slice, bytes
  entries();
  auto fetch = [&]() {
    if (f_more) {
      const int key0 = (f.tile0 + f_tile) * kPagedTile + warp * kSlice;
      const int page = __shfl_sync(0xffffffffu, f_entry, f_tile & 31);
      const bool used = key0 < f.hi && key0 + kSlice > f.lo, exists = (unsigned)page < (unsigned)a.kv.n_pages;
      if (used && !exists && lane == 0) atomicOr(a.status, CS_DEV_BADARG);
      const uint32_t dst = my_ring + (uint32_t)(f_stage * 2 * kSliceBytes);
      if (used && exists) {
        const long long off = (page * a.kv.page_stride + f.head * a.kv.head_stride + (long long)(key0 & (a.kv.page_size - 1)) * a.kv.slot_stride) * 2 + lane_off;
        const char *k = a.kv.k + off, *v = a.kv.v + off;
        const bool all = key0 >= f.lo && key0 + kSlice <= f.hi;
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          const int j = (i * 32 + lane) / CPR, c = lane % CPR;
          const bool on = all || (key0 + j >= f.lo && key0 + j < f.hi);
          cp16(dst + at_chunk<DH>(j, c), on ? k + i * hop : a.kv.k, on);
          cp16(dst + kSliceBytes + at_chunk<DH>(j, c), on ? v + i * hop : a.kv.v, on);
        }
      } else {
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
          cp16(dst + (i * 32 + lane) * 16, a.kv.k, false);
          cp16(dst + kSliceBytes + (i * 32 + lane) * 16, a.kv.v, false);
        }
      }
      if (++f_stage == kStages) f_stage = 0;
      if (++f_tile == f.n_tiles) {
        f_tile = 0;
        f_more = paged_next(a, plan, f, run1);
        if (f_more) queries();
      }
      if ((f_tile & 31) == 0 && f_more) entries();
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < kStages; ++s) fetch();

  uint32_t qf[kSteps][4];
  int lo[2], hi[2], all_lo, all_hi;              // what this thread's two rows attend to; keys every live row of the item sees
  auto begin = [&]() {
    all_lo = 0; all_hi = 0x7fffffff;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int m = p.rg * kRows + g + 8 * h;
      lo[h] = hi[h] = 0;
      if (m < p.len * G) {
        const int r = a.by_group.of(m);
        paged_range(a.mask, a.window, p.len, p.kv, r, r, lo[h], hi[h]);
        all_lo = max(all_lo, lo[h]);
        all_hi = min(all_hi, hi[h]);
      }
    }
    all_lo = __reduce_max_sync(0xffffffffu, all_lo);
    all_hi = __reduce_min_sync(0xffffffffu, all_hi);
    const uint32_t q = (uint32_t)__cvta_generic_to_shared(s_q) + (uint32_t)(q_at * kRows * DH * 2);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) ldm4(q + at_chunk<DH>((lane & 7) + (((lane >> 3) & 1) << 3), 2 * s + (lane >> 4)), qf[s]);
    if (++q_at == kStages + 1) q_at = 0;
  };
  asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
  __syncthreads();
  // A piece's queries are read by every warp (all sixteen rows) before any warp fetches again: of pieces of one tile each the ring holds this one and the kStages behind it, so the next queries
  // go to this one's place.
  begin();
  __syncthreads();

  // items shared with other CTAs, at most two: the run's first and its last
  struct Shared { int c0, c1, start, len, rg, head; } shared[2] = {{-1, 0, 0, 0, 0, 0}, {-1, 0, 0, 0, 0, 0}};
  int stage = 0;
  for (bool more = true; more;) {
    float o[DH / 8][4];
#pragma unroll
    for (int n = 0; n < DH / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int i = 0; i < p.n_tiles; ++i) {
      const int key0 = (p.tile0 + i) * kPagedTile + warp * kSlice;
      asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
      __syncwarp();
      if (key0 < p.hi && key0 + kSlice > p.lo) {
        const uint32_t ks = my_ring + (uint32_t)(stage * 2 * kSliceBytes), vs = ks + kSliceBytes;
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
          uint32_t b[4];
          ldm4(ks + at_chunk<DH>((lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), b);
          mma<T>(s[0], qf[k], b[0], b[1]);
          mma<T>(s[1], qf[k], b[2], b[3]);
        }
        const bool mixed = key0 < all_lo || key0 + kSlice > all_hi;    // some live row does not see all of it
        if (mixed) {
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int key = key0 + 8 * n + 2 * t + (e & 1);
              if (key < lo[e >> 1] || key >= hi[e >> 1]) s[n][e] = -INFINITY;
            }
        }
        // ---- running maxima (of a row's four threads), weights, sums
        float nm[2];
        bool moves = false;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float x = fmaxf(fmaxf(s[0][2 * h], s[0][2 * h + 1]), fmaxf(s[1][2 * h], s[1][2 * h + 1]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
          x = fmaf(fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2)), a.scale_log2e, -kUp<T>);
          nm[h] = fmaxf(m[h], x);
          moves |= nm[h] > m[h];
        }
        if (__any_sync(0xffffffffu, moves)) {
          float corr[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            corr[h] = nm[h] > m[h] ? paged_ex2(m[h] - nm[h]) : 1.f;      // (from -inf: 0)
            m[h] = nm[h];
            l[h] *= corr[h];
          }
#pragma unroll
          for (int n = 0; n < DH / 8; ++n) {
            o[n][0] *= corr[0]; o[n][1] *= corr[0];
            o[n][2] *= corr[1]; o[n][3] *= corr[1];
          }
        }
        uint32_t ph[4], pl[4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float base = m[h] == -INFINITY ? 0.f : -m[h];
            const float w0 = paged_ex2(fmaf(s[n][2 * h], a.scale_log2e, base)), w1 = paged_ex2(fmaf(s[n][2 * h + 1], a.scale_log2e, base));
            l[h] += w0 + w1;
            s[n][2 * h] = w0; s[n][2 * h + 1] = w1;
            const uint32_t hi16 = PagedType<T>::pack(w0, w1);
            const float2 f2 = PagedType<T>::unpack(hi16);
            ph[2 * n + h] = hi16;
            pl[2 * n + h] = PagedType<T>::pack(w0 - f2.x, w1 - f2.y);
          }
        // ---- O += P V
        bool plain = false;
        if (mixed) {
          bool odd = false;
#pragma unroll
          for (int i2 = 0; i2 < kIter; ++i2) {
            const uint4 w = *reinterpret_cast<const uint4*>(my_ring_p + (stage * 2 + 1) * kSliceBytes + (i2 * 32 + lane) * 16);
            odd |= odd_pair<T>(w.x) || odd_pair<T>(w.y) || odd_pair<T>(w.z) || odd_pair<T>(w.w);
          }
          plain = __any_sync(0xffffffffu, odd);
        }
        if (!plain) {
#pragma unroll
          for (int n = 0; n < DH / 16; ++n) {
            uint32_t b[4];
            ldm4t(vs + at_chunk<DH>((lane & 7) + (((lane >> 3) & 1) << 3), 2 * n + (lane >> 4)), b);
            mma<T>(o[2 * n], ph, b[0], b[1]);
            mma<T>(o[2 * n + 1], ph, b[2], b[3]);
            mma<T>(o[2 * n], pl, b[0], b[1]);
            mma<T>(o[2 * n + 1], pl, b[2], b[3]);
          }
        } else {
          for (int j = 0; j < kSlice; ++j) {
            const int src = (lane & ~3) | ((j & 7) >> 1);
            float w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float x0 = j & 8 ? s[1][2 * h] : s[0][2 * h], x1 = j & 8 ? s[1][2 * h + 1] : s[0][2 * h + 1];
              w[h] = __shfl_sync(0xffffffffu, j & 1 ? x1 : x0, src);
            }
            const bool see0 = key0 + j >= lo[0] && key0 + j < hi[0], see1 = key0 + j >= lo[1] && key0 + j < hi[1];
#pragma unroll
            for (int n = 0; n < DH / 8; ++n) {
              const uint32_t v2 = *reinterpret_cast<const uint32_t*>(my_ring_p + (stage * 2 + 1) * kSliceBytes + at_chunk<DH>(j, n) + 4 * t);
              const float2 v = PagedType<T>::unpack(v2);
              if (see0) { o[n][0] = fmaf(w[0], v.x, o[n][0]); o[n][1] = fmaf(w[0], v.y, o[n][1]); }
              if (see1) { o[n][2] = fmaf(w[1], v.x, o[n][2]); o[n][3] = fmaf(w[1], v.y, o[n][3]); }
            }
          }
        }
      }
      __syncwarp();                              // (every lane has read the slice)
      if (++stage == kStages) stage = 0;
      fetch();
    }

    // ---- the warps' results meet: eight columns of a row per thread
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
      l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
      float* dst = s_o + (warp * kRows + g + 8 * h) * kLd + 2 * t;
#pragma unroll
      for (int n = 0; n < DH / 8; ++n) *reinterpret_cast<float2*>(dst + 8 * n) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
      if (t == 0) s_ml[warp * kRows + g + 8 * h] = make_float2(m[h], l[h]);
    }
    PagedPiece next = p;
    more = paged_next(a, plan, next, run1);
    __syncthreads();
    const int row = tid / CPR, c8 = tid % CPR * 8, mrow = p.rg * kRows + row;
    if (row < kRows && mrow < p.len * G) {
      float acc[8], M = -INFINITY, L = 0.f;
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_ml[w * kRows + row].x);
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = s_ml[w * kRows + row];
        const float k = ml.x == -INFINITY ? 0.f : paged_ex2(ml.x - M);
        if (ml.x == -INFINITY && ml.y == 0.f) continue;      // (it saw nothing)
        L = fmaf(k, ml.y, L);
        const float4 v0 = *reinterpret_cast<const float4*>(s_o + (w * kRows + row) * kLd + c8), v1 = *reinterpret_cast<const float4*>(s_o + (w * kRows + row) * kLd + c8 + 4);
        acc[0] = fmaf(k, v0.x, acc[0]); acc[1] = fmaf(k, v0.y, acc[1]); acc[2] = fmaf(k, v0.z, acc[2]); acc[3] = fmaf(k, v0.w, acc[3]);
        acc[4] = fmaf(k, v1.x, acc[4]); acc[5] = fmaf(k, v1.y, acc[5]); acc[6] = fmaf(k, v1.z, acc[6]); acc[7] = fmaf(k, v1.w, acc[7]);
      }
      if (p.whole) {
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int r = a.by_group.of(mrow);
        const long long at = (long long)(p.start + r) * a.n_heads + p.head * G + (mrow - r * G);
        *reinterpret_cast<uint4*>(a.out + (at * DH + c8) * 2) =
            make_uint4(PagedType<T>::pack(acc[0] * inv, acc[1] * inv), PagedType<T>::pack(acc[2] * inv, acc[3] * inv),
                       PagedType<T>::pack(acc[4] * inv, acc[5] * inv), PagedType<T>::pack(acc[6] * inv, acc[7] * inv));
        if (a.lse != nullptr && c8 == 0) a.lse[at] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.6931471805599453f;
      } else {
        const long long at = ((long long)cta * 2 + (p.opens ? 1 : 0)) * kPagedMaxRows + row;
        float* dst = a.parts + at * DH + c8;
        __stcg(reinterpret_cast<float4*>(dst), make_float4(acc[0], acc[1], acc[2], acc[3]));
        __stcg(reinterpret_cast<float4*>(dst + 4), make_float4(acc[4], acc[5], acc[6], acc[7]));
        if (c8 == 0) __stcg(reinterpret_cast<float2*>(a.parts_ml) + at, make_float2(M, L));
      }
    }
    if (!p.whole) {
      const Shared s = {paged_first_cta(a, p, total, n_cta), paged_last_cta(a, p, total, n_cta), p.start, p.len, p.rg, p.head};
      if (p.opens) shared[1] = s;
      else shared[0] = s;
    }
    p = next;
    if (more) {
      begin();                                   // (its queries came with the last slice of the piece before)
      __syncthreads();                           // (they are read, and the exchange rows are free again)
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- shared items: the CTA that arrives last adds the pieces up, in the order of the keys.  (Both at the end of the run: arriving takes 1.5 us of waiting for
  // writes and the counter, during which the next piece's keys would not be fetched.)
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
    // The pieces come into the ring, all in flight together, and are added up from there.  (Through registers it is either one piece after the other, 10 us
    // for 18, or a body of some thousand instructions that nobody has run yet: 5 us.)
    const int rows = min(kRows, s.len * G - s.rg * kRows), fit = kWarps * kStages * 2 * kSliceBytes / (rows * DH * 4);
    constexpr int kTasks = (kRows * DH / 4 + kThreads - 1) / kThreads;      // (row, four columns) of a thread
    const uint32_t s_parts = (uint32_t)__cvta_generic_to_shared(ring), s_pml = (uint32_t)__cvta_generic_to_shared(s_o);
    float2* pml = reinterpret_cast<float2*>(s_o);      // [piece][16 rows]: reference point, then weight; sum
    float acc[kTasks][4];
#pragma unroll
    for (int k = 0; k < kTasks; ++k) acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.f;
    if (tid < kRows) s_ml[tid] = make_float2(-INFINITY, 0.f);              // a row's reference point and sum so far
#pragma unroll 1
    for (int cb = s.c0; cb <= s.c1; cb += fit) {
      const int n = min(fit, s.c1 - cb + 1);
#pragma unroll 1
      for (int i = warp; i < n; i += kWarps) {
        const long long at = ((long long)(cb + i) * 2 + (cb + i == s.c0 ? 1 : 0)) * kPagedMaxRows;
        const float* src = a.parts + at * DH + lane * 4;
        const uint32_t dst = s_parts + (uint32_t)((i * rows * (DH / 4) + lane) * 16);
        if (2 * lane < rows) cp16(s_pml + (uint32_t)((i * kRows + 2 * lane) * 8), a.parts_ml + (at + 2 * lane) * 2, true);
#pragma unroll 4
        for (int j = lane; j < rows * (DH / 4); j += 32) cp16(dst + (uint32_t)((j - lane) * 16), src + (j - lane) * 4, true);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncthreads();
#pragma unroll 1
      for (int row = warp; row < rows; row += kWarps) {
        const float2 old = s_ml[row];
        float top = old.x, sum = 0.f;
        for (int j = lane; j < n; j += 32) top = fmaxf(top, pml[j * kRows + row].x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        for (int j = lane; j < n; j += 32) {
          const float2 x = pml[j * kRows + row];
          const float w = x.x == -INFINITY ? 0.f : paged_ex2(x.x - top);
          sum += x.x == -INFINITY && x.y == 0.f ? 0.f : w * x.y;           // (without a maximum, but a sum: NaN)
          pml[j * kRows + row].x = w;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) {
          const float keep = old.x == -INFINITY ? 1.f : paged_ex2(old.x - top);
          s_ml[row] = make_float2(top, old.y * keep + sum);
          s_ml[kRows + row].x = keep;
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < kTasks; ++k) {
        const int row = (tid + k * kThreads) / (DH / 4), c4 = (tid + k * kThreads) % (DH / 4);
        if (row >= rows) continue;
        const float keep = s_ml[kRows + row].x;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[k][e] *= keep;
        const float4* v = reinterpret_cast<const float4*>(ring) + row * (DH / 4) + c4;
#pragma unroll 4
        for (int j = 0; j < n; ++j) {
          const float2 x = pml[j * kRows + row];
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
      const int mrow = s.rg * kRows + row, r = a.by_group.of(mrow);
      const long long at = (long long)(s.start + r) * a.n_heads + s.head * G + (mrow - r * G);
      *reinterpret_cast<uint2*>(a.out + (at * DH + c4) * 2) = make_uint2(PagedType<T>::pack(acc[k][0] * inv, acc[k][1] * inv), PagedType<T>::pack(acc[k][2] * inv, acc[k][3] * inv));
      if (a.lse != nullptr && c4 == 0) a.lse[at] = ml.y == 0.f ? -INFINITY : (ml.x + log2f(ml.y)) * 0.6931471805599453f;
    }
    __syncthreads();
  }
}

template <typename T, int DH>
cs_status launch_few(cs_paged_cache* c, const PagedAttnArgs& a, unsigned bit, cudaStream_t st) {
  if (!(c->attr_set & bit)) {
    CS_CUDA_OK(c, cudaFuncSetAttribute(k_paged_few<T, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem<DH>));
    c->attr_set |= bit;
  }
  CS_CUDA_OK(c, cs_launch_pdl(k_paged_few<T, DH>, dim3(c->num_sms), dim3(kThreads), kFewSmem<DH>, st, a));
  return CS_OK;
}

}  // namespace

cs_status cs_launch_paged_few(cs_paged_cache* c, const PagedAttnArgs& args, cudaStream_t st) {
  PagedAttnArgs a = args;
  a.item_rows = kRows;
  a.by_item_rows = PagedDivisor::by(kRows);
  a.item_cost = 2;
  // (a tile takes 0.6, 0.4 or 0.3 us where a CTA has few, adding pieces up some 4)
  a.keep = c->cfg.head_dim == 128 ? 6 : c->cfg.head_dim == 64 ? 10 : 16;
  const bool bf = c->cfg.dtype == CS_BF16;
  switch (c->cfg.head_dim) {
    case 32: return bf ? launch_few<__nv_bfloat16, 32>(c, a, 1, st) : launch_few<__half, 32>(c, a, 2, st);
    case 64: return bf ? launch_few<__nv_bfloat16, 64>(c, a, 4, st) : launch_few<__half, 64>(c, a, 8, st);
    default: return bf ? launch_few<__nv_bfloat16, 128>(c, a, 16, st) : launch_few<__half, 128>(c, a, 32, st);
  }
}
