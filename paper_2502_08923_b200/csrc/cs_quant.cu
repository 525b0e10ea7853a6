// Rows quantised into a paged cache of 4 bits, and read back; the host side of that cache.  (The format: cs_quant.cuh.)
//
// Append: keys are normed and rotated as in cs_paged.cu, u = x rsqrt(mean(x^2) + eps) gain, y_i = u_i c_i - u_{i+h} s_i, y_{i+h} = u_{i+h} c_i + u_i s_i, then quantised; values are
// quantised; queries are normed and rotated.  A lane holds eight elements of a head's first half and their eight partners, which are a word each; a group's maximum is that of four words,
// by way of shared memory.  Keys that are normed or rotated are worked out in 64 bits up to their level: which of fifteen levels an element goes to is then decided by its value, not by
// the order of some sums (in 32 bits one element in some three million ends up a whole step from where another order puts it).  Elements that come as they are need no more than 32 bits: a correctly rounded quotient
// of numbers of 24 and 5 bits is a whole number and a half only where it is one.
#include <algorithm>
#include <type_traits>

#include "cs_quant.cuh"

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;

struct QuantAppendArgs {
  const char *q, *k, *v;             // sources; no queries: n_q = 0
  char* yq;
  long long q_row, q_head, k_row, k_head, v_row, v_head, yq_row, yq_head;   // elements
  const char *q_gain, *k_gain;
  int n_q, n_kv, n_rows;
  int warps_per_row;                 // 1, 2 or 4
  const float* rope;
  int n_positions, rot_dim;
  float eps;
  QuantView kv;
  BlocksView blk;
  int* status;
};

template <typename T> __device__ __forceinline__ void load8(const char* p, float (&f)[8]) {
  const uint4 x = __ldg(reinterpret_cast<const uint4*>(p));
  if constexpr (sizeof(T) == 4) {
    const uint4 y = __ldg(reinterpret_cast<const uint4*>(p) + 1);
    f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
    f[4] = __uint_as_float(y.x); f[5] = __uint_as_float(y.y); f[6] = __uint_as_float(y.z); f[7] = __uint_as_float(y.w);
  } else {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = PagedType<T>::unpack(w[i]);
      f[2 * i] = y.x; f[2 * i + 1] = y.y;
    }
  }
}
// the same from shared memory
template <typename T> __device__ __forceinline__ void lds8(const char* p, float (&f)[8]) {
  const uint4 x = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  if constexpr (sizeof(T) == 4) {
    const uint4 y = *(reinterpret_cast<const uint4*>(p) + 1);
    f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
    f[4] = __uint_as_float(y.x); f[5] = __uint_as_float(y.y); f[6] = __uint_as_float(y.z); f[7] = __uint_as_float(y.w);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = PagedType<T>::unpack(w[i]);
      f[2 * i] = y.x; f[2 * i + 1] = y.y;
    }
  }
}
template <typename T> __device__ __forceinline__ void store8(char* p, const float (&f)[8]) {
  *reinterpret_cast<uint4*>(p) = make_uint4(PagedType<T>::pack(f[0], f[1]), PagedType<T>::pack(f[2], f[3]), PagedType<T>::pack(f[4], f[5]), PagedType<T>::pack(f[6], f[7]));
}

// Quotients are products with a reciprocal in two terms, 1 / d = hi + lo up to 2^-48: what that gives in 32 bits is a whole number and a half, or halfway between two scales, only where the quotient is.  (A quotient
// of a number of 24 bits by one of five is farther from those than half a unit in the last place, unless it is one of them.)
struct Reciprocal {
  float hi, lo;
  __device__ __forceinline__ static Reciprocal of(float d) {
    Reciprocal r;
    r.hi = __fdiv_rn(1.f, d);
    r.lo = fmaf(-d, r.hi, 1.f) * r.hi;
    return r;
  }
  __device__ __forceinline__ float times(float x) const { return fmaf(x, hi, x * lo); }
};
constexpr float kMostScale = 1.0633823966279327e37f;         // 2^123: 24 times it is finite
// The scale of a group whose largest element is `most`, which may be inf or NaN: five significant bits, halves to even, below 2^-126 the nearest multiple of 2^-133; at most 2^123
__device__ __forceinline__ float scale_of(double most) {
  const double x = most / 7.0;
  if (!(x <= (double)kMostScale)) return x <= 1e300 ? kMostScale : __uint_as_float(0x7fc00000u);
  long long b = __double_as_longlong(x);
  b += 0x7fffffffffffll + (b >> 48 & 1);
  return __bfloat162float(__float2bfloat16_rn((float)__longlong_as_double(b >> 48 << 48)));
}
__device__ __forceinline__ float scale_of(float most) {
  const Reciprocal seventh{0.14285714924335479736328125f, -6.386212e-9f};      // 1 / 7: rounded, and what that leaves out
  const bool small = most < 0x1p-60f;            // (the quotient's second term, and near 2^-126 the quotient, would have fewer bits there)
  uint32_t b = __float_as_uint(seventh.times(most * (small ? 0x1p64f : 1.f)));
  if ((b & 0x7f800000u) == 0x7f800000u) return __uint_as_float(0x7fc00000u);
  b += 0x3ffffu + (b >> 19 & 1u);
  return __bfloat162float(__float2bfloat16_rn(fminf(__uint_as_float(b & 0xfff80000u), kMostScale) * (small ? 0x1p-64f : 1.f)));
}
constexpr uint32_t kZeros = 0x88888888u;
__device__ __forceinline__ constexpr int field_at(int i) { return 4 * (i / 2 + 4 * (i & 1)); }
// Eight elements of a group as a word.  The sum with 1.5 2^23 + 8 rounds to a whole number, halves to even, and leaves n + 8 in its last bits; what stands above them is taken out of the word at the end.
__device__ __forceinline__ uint32_t word_of(const float (&y)[8], float s) {
  if (!(s >= 1.17549435e-38f && s < kMostScale)) {           // (nothing to divide by, or elements that have to be held back)
    uint32_t w = 0;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      float x = y[0];
#pragma unroll
      for (int k = 1; k < 8; ++k) x = i == k ? y[k] : x;
      w |= (uint32_t)((s > 0.f ? min(max(__float2int_rn(__fdiv_rn(x, s)), -7), 7) : 0) + 8) << field_at(i);
    }
    return w;
  }
  const Reciprocal r = Reciprocal::of(s);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) w += (__float_as_uint(r.times(y[i]) + 12582920.f) - 0x4b400000u) << field_at(i);
  return w;
}
// In 64 bits: the quotient, by the product with the reciprocal, is rounded to a multiple of 2^-44 first (the sum with 384 does that), which makes a whole number and a half of one that is a rounding beside it, and
// then to a whole number (the sum with 1.5 2^52 + 8).
__device__ __forceinline__ uint32_t word_of(const double (&y)[8], float s) {
  if (!(s > 0.f)) return kZeros;
  uint32_t w = 0;
  const double inv = 1.0 / (double)s;
  const bool held_back = s >= kMostScale || s < 1.17549435e-38f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    int u = __double2loint(fma(y[i], inv, 384.0) + (6755399441055752.0 - 384.0));
    if (held_back) u = min(max(u, 1), 15);
    w += (uint32_t)u << field_at(i);
  }
  return w;
}
// the largest of some, inf or NaN if one is not finite
template <int N> __device__ __forceinline__ float most_of(const float* y) {
  float m = fabsf(y[0]);
#pragma unroll
  for (int i = 1; i < N; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(y[i])));
  return m;
}
template <int N> __device__ __forceinline__ double most_of(const double* y) {
  double m = fabs(y[0]), z = y[0] * 0.0;
#pragma unroll
  for (int i = 1; i < N; ++i) {
    const double x = fabs(y[i]);
    m = x > m ? x : m;
    z = fma(x, 0.0, z);
  }
  return m + z;                                  // (0 x inf is NaN)
}

__device__ __forceinline__ void fetch16(uint32_t dst, const char* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// A unit is 512 elements: up to kPer neighbouring heads of the queries, the keys or the values of a row.  Units lie in a ring of shared memory for each warp, as in memory; three are in flight.
// What bounds it: instructions.  Four chunks of up to 2,048 rows (32 query heads, 8 of keys, norms and rotation) with their positions read back: 50 us (from rows in 32 bits 56), 44 of them here; 26 M instructions, the schedulers issue in 62 of 100 clocks; 7 us are the
// keys' 64-bit arithmetic, in what an SM has units for.  (87 us with rows fetched as they are needed, 66 with the ring, 54 with factors and quotients worked out once, 50 with four blocks of four warps an SM; five of them: no faster, nor
// several rows a warp.)  A token each of 64 sequences and one verification block: 4 us, a chain of loads (whose row, which page) and one row's arithmetic.
template <typename S, typename D, int DH>
__global__ void __launch_bounds__(kThreads, 4)
k_quant_append(const __grid_constant__ QuantAppendArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kLanes = DH / 16, kPer = 32 / kLanes, kWords = DH / 8;      // lanes of a head, heads of a unit, words of a head
  constexpr int kSize = (int)sizeof(S), kUnit = 512 * kSize, kPieces = kUnit / 512, kHeadPieces = DH * kSize / 16, kSlots = 4;      // bytes of a unit; 16-byte pieces of a lane, of a head
  __shared__ __align__(16) uint8_t s_ring[kWarps][kSlots][kUnit];
  __shared__ int s_seq[kWarps], s_pos[kWarps];
  __shared__ double s_most[kWarps][64];          // [head][word]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = lane % kLanes, sub = lane / kLanes;
  const int n_here = kWarps / a.warps_per_row;
  const long long row0 = (long long)blockIdx.x * n_here, row = row0 + warp / a.warps_per_row;
  const int uq = (a.n_q + kPer - 1) / kPer, uk = uq + (a.n_kv + kPer - 1) / kPer, units = row < a.n_rows ? uk + (a.n_kv + kPer - 1) / kPer : 0;
  const int step = a.warps_per_row, u0 = warp % step;
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(&s_ring[warp][0][0]);
  int fu = u0;
  uint32_t f_at = 0;
  auto fetch = [&]() {
    if (fu < units) {
      const int kind = fu < uq ? 0 : fu < uk ? 1 : 2, h0 = (fu - (kind == 0 ? 0 : kind == 1 ? uq : uk)) * kPer, n = kind == 0 ? a.n_q : a.n_kv;
      const long long head = kind == 0 ? a.q_head : kind == 1 ? a.k_head : a.v_head;
      const char* src = kind == 0 ? a.q + row * a.q_row * kSize : kind == 1 ? a.k + row * a.k_row * kSize : a.v + row * a.v_row * kSize;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int e = i * 32 + lane, h = h0 + e / kHeadPieces, c = e % kHeadPieces;
        if (h < n) fetch16(ring + f_at + e * 16, src + h * head * kSize + c * 16);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    fu += step;
    f_at = f_at == (kSlots - 1) * kUnit ? 0 : f_at + kUnit;
  };
#pragma unroll
  for (int i = 0; i < kSlots - 1; ++i) fetch();  // (whose row it is, and where it goes, takes three loads in a row: these are under way meanwhile)

  // the blocks these rows belong to
  if (threadIdx.x < kWarps) s_seq[threadIdx.x] = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.blk.n_seqs; b += kThreads) {
    const int start = __ldcg(a.blk.start + b), len = __ldcg(a.blk.len + b), kv = __ldcg(a.blk.kv_len + b);
    const int flag = paged_block_flag(a.blk, a.kv.page_size, true, start, len, kv);
    if (flag != 0) {
      if (blockIdx.x == 0) atomicOr(a.status, flag);
    } else {
      for (int i = 0; i < n_here; ++i)
        if (row0 + i >= start && row0 + i - start < len) { s_seq[i] = b; s_pos[i] = kv + (int)(row0 + i - start); }
    }
  }
  __syncthreads();
  const int b = s_seq[warp / a.warps_per_row], pos = s_pos[warp / a.warps_per_row];
  const bool lost = b >= 0 && a.rot_dim > 0 && pos >= a.n_positions;
  if (lost && lane == 0) atomicOr(a.status, CS_DEV_CAPACITY);
  if (b < 0 || lost) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  const int page = __ldcg(a.blk.table + (long long)b * a.blk.table_width + (pos >> a.kv.page_shift)), slot = pos & (a.kv.page_size - 1);

  // this lane's words: partners of the rotation, or two neighbours behind what is rotated
  const int half = a.rot_dim >> 4;
  const bool rotated = pair < half;
  const int c0 = rotated ? pair : 2 * pair, c1 = rotated ? pair + half : c0 + 1;
  float cs[8], sn[8];
  if (rotated) {
    load8<float>(reinterpret_cast<const char*>(a.rope + (long long)pos * a.rot_dim + c0 * 8), cs);
    load8<float>(reinterpret_cast<const char*>(a.rope + (long long)pos * a.rot_dim + (c0 + half) * 8), sn);
  }
  const bool kept = (unsigned)page < (unsigned)a.kv.n_pages;
  if (!kept && lane == 0) atomicOr(a.status, CS_DEV_BADARG);
  // The next unit's two words of this lane, once they are there; the one behind those in flight is asked for.
  uint32_t at = 0;
  auto take = [&](float (&x0)[8], float (&x1)[8]) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 2) : "memory");
    __syncwarp();
    const char* mine = reinterpret_cast<const char*>(&s_ring[warp][0][0]) + at + sub * DH * kSize;
    lds8<S>(mine + c0 * 8 * kSize, x0);
    lds8<S>(mine + c1 * 8 * kSize, x1);
    __syncwarp();
    fetch();                                     // (into the place of the unit before: all lanes have read it)
    at = at == (kSlots - 1) * kUnit ? 0 : at + kUnit;
  };
  auto gains = [&](const char* gain, int word, float (&g)[8]) {
    if (gain != nullptr) load8<D>(gain + word * 8 * (int)sizeof(D), g);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = 1.f;
    }
  };
  int u = u0;
  // ---- queries: y0 = r (x0 C0 - x1 S0), y1 = r (x1 C1 + x0 S1), C = gain cos, S = gain sin worked out once
  if (u < uq) {
    f32x2 C0[4], C1[4], S0[4], S1[4];
    {
      float g0[8], g1[8];
      gains(a.q_gain, c0, g0);
      gains(a.q_gain, c1, g1);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 a0 = pack2(g0[2 * i], g0[2 * i + 1]), a1 = pack2(g1[2 * i], g1[2 * i + 1]);
        const f32x2 c = rotated ? pack2(cs[2 * i], cs[2 * i + 1]) : pack2(1.f, 1.f), s = rotated ? pack2(sn[2 * i], sn[2 * i + 1]) : pack2(0.f, 0.f);
        C0[i] = mul2(a0, c); C1[i] = mul2(a1, c);
        S1[i] = mul2(a0, s); S0[i] = mul2(a1, mul2(s, pack2(-1.f, -1.f)));
      }
    }
    const bool norm = a.q_gain != nullptr;
    char* dst = a.yq + (row * a.yq_row + (u * kPer + sub) * a.yq_head) * (long long)sizeof(D);
    const long long dst_step = step * kPer * a.yq_head * (long long)sizeof(D);
    for (; u < uq; u += step, dst += dst_step) {
      float x0[8], x1[8];
      take(x0, x1);
      f32x2 p0[4], p1[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { p0[i] = pack2(x0[2 * i], x0[2 * i + 1]); p1[i] = pack2(x1[2 * i], x1[2 * i + 1]); }
      if (norm) {
        f32x2 s2 = mul2(p0[0], p0[0]);
#pragma unroll
        for (int i = 1; i < 4; ++i) s2 = fma2(p0[i], p0[i], s2);
#pragma unroll
        for (int i = 0; i < 4; ++i) s2 = fma2(p1[i], p1[i], s2);
        float lo, hi;
        unpack2(s2, lo, hi);
        float sq = lo + hi;
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        const float r = rsqrtf(sq * (1.f / DH) + a.eps);
#pragma unroll
        for (int i = 0; i < 4; ++i) { p0[i] = mul2(p0[i], pack2(r, r)); p1[i] = mul2(p1[i], pack2(r, r)); }
      }
      // (what is not rotated has no partner: its product with a sine of 0 would make NaN of an inf)
      if (a.rot_dim > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x2 t0 = mul2(p0[i], C0[i]), t1 = mul2(p1[i], C1[i]);
          const f32x2 y0 = rotated ? fma2(p1[i], S0[i], t0) : t0, y1 = rotated ? fma2(p0[i], S1[i], t1) : t1;
          unpack2(y0, x0[2 * i], x0[2 * i + 1]);
          unpack2(y1, x1[2 * i], x1[2 * i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          unpack2(mul2(p0[i], C0[i]), x0[2 * i], x0[2 * i + 1]);
          unpack2(mul2(p1[i], C1[i]), x1[2 * i], x1[2 * i + 1]);
        }
      }
      if (u * kPer + sub < a.n_q) {
        store8<D>(dst + c0 * 8 * (int)sizeof(D), x0);
        store8<D>(dst + c1 * 8 * (int)sizeof(D), x1);
      }
    }
  }
  // ---- keys, values
  const bool plain_keys = a.k_gain == nullptr && a.rot_dim == 0;
  for (; u < units; u += step) {
    const bool keys = u < uk;
    const int h = (u - (keys ? uq : uk)) * kPer + sub;
    const bool live = h < a.n_kv;
    float x0[8], x1[8];
    take(x0, x1);
    if (!live) {                                 // (what lies in the ring there is another unit's)
#pragma unroll
      for (int i = 0; i < 8; ++i) x0[i] = x1[i] = 0.f;
    }
    uint32_t w0, w1;
    float s0, s1;
    if (keys && !plain_keys) {
      double y0[8], y1[8], r = 1.0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { y0[i] = (double)x0[i]; y1[i] = (double)x1[i]; }
      if (a.k_gain != nullptr) {
        double sq = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = fma(y0[i], y0[i], fma(y1[i], y1[i], sq));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
        r = rsqrt(sq * (1.0 / DH) + (double)a.eps);
        float g[8];
        gains(a.k_gain, c0, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y0[i] *= r * (double)g[i];
        gains(a.k_gain, c1, g);
#pragma unroll
        for (int i = 0; i < 8; ++i) y1[i] *= r * (double)g[i];
      }
      if (rotated) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const double c = (double)cs[i], s = (double)sn[i], y = fma(y0[i], c, -(y1[i] * s));
          y1[i] = fma(y1[i], c, y0[i] * s);
          y0[i] = y;
        }
      }
      double* most = &s_most[warp][sub * kWords];
      most[c0] = most_of<8>(y0);
      most[c1] = most_of<8>(y1);
      __syncwarp();
      s0 = scale_of(most_of<4>(most + (c0 & ~3)));
      s1 = scale_of(most_of<4>(most + (c1 & ~3)));
      __syncwarp();
      w0 = word_of(y0, s0);
      w1 = word_of(y1, s1);
    } else {
      float* most = reinterpret_cast<float*>(&s_most[warp][0]) + sub * kWords;
      most[c0] = most_of<8>(x0);
      most[c1] = most_of<8>(x1);
      __syncwarp();
      s0 = scale_of(most_of<4>(most + (c0 & ~3)));
      s1 = scale_of(most_of<4>(most + (c1 & ~3)));
      __syncwarp();
      w0 = word_of(x0, s0);
      w1 = word_of(x1, s1);
    }
    if (live && kept) {
      const long long in_page = (long long)h * a.kv.page_size + slot;
      uint32_t* data = (keys ? a.kv.k : a.kv.v) + page * a.kv.data_page + in_page * kWords;
      unsigned short* scale = (keys ? a.kv.ks : a.kv.vs) + page * a.kv.scale_page + in_page * (DH / kQuantGroup);
      data[c0] = w0;
      data[c1] = w1;
      if ((c0 & 3) == 0) scale[c0 >> 2] = __bfloat16_as_ushort(__float2bfloat16_rn(s0));
      if ((c1 & 3) == 0) scale[c1 >> 2] = __bfloat16_as_ushort(__float2bfloat16_rn(s1));
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// ------------------------------------------------------------------ reading back
// A group, a lane: 16 bytes side by side with its neighbours' and a scale make 32 elements, which are two whole sectors of 16 bits (stored 32 bytes at a time where that is aligned), in some 16 instructions for eight
// of them.  (A word, a lane: 59, most of them addresses.)  Bound by HBM and by how much is in flight: two sequences of 16,384 positions of the 8B shape 31.9 us (171 MB, 5.4 TB/s).
constexpr int kReadRows = 8;
struct QuantReadArgs {
  QuantView kv;
  BlocksView blk;
  char *k, *v;                       // destinations of rows, or of copies
  long long k_row, k_head, v_row, v_head;      // elements; copies: page, head (of both)
  int mask, window;                  // copies: which keys the blocks attend to
  int rows_per_warp;                 // up to kReadRows
  int copy_pages, copy_shift;        // pages of a sequence's copies, their size
  int shares;                        // warps that share the heads of sixteen positions
  int* copy_len;                     // lengths of blocks that nothing is wrong with
  int* status;
};

// a group's 32 values in type T.  (fp16 ends at 65504: what lies beyond it becomes that.)
template <typename T> __device__ __forceinline__ void put_group(char* dst, const uint4& words, unsigned scale, bool by_32) {
  const QuantScale s = QuantScale::of(scale * 0x10001u);
  const uint32_t w[4] = {words.x, words.y, words.z, words.w};
  uint32_t r[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) quant_expand(w[i], s, r[i]);
  auto store = [&](int at, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, uint32_t b2, uint32_t b3) {
    if (by_32) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + at), "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(b2), "r"(b3) : "memory");
    } else {
      *reinterpret_cast<uint4*>(dst + at) = make_uint4(a0, a1, a2, a3);
      *reinterpret_cast<uint4*>(dst + at + 16) = make_uint4(b0, b1, b2, b3);
    }
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      store(32 * i, r[i][0] << 16, r[i][0] & 0xffff0000u, r[i][1] << 16, r[i][1] & 0xffff0000u, r[i][2] << 16, r[i][2] & 0xffff0000u, r[i][3] << 16, r[i][3] & 0xffff0000u);
    } else {
      if constexpr (std::is_same<T, __half>::value) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 y = PagedType<__nv_bfloat16>::unpack(r[i][k]);
          const float lo = fabsf(y.x) > 65504.f ? copysignf(65504.f, y.x) : y.x, hi = fabsf(y.y) > 65504.f ? copysignf(65504.f, y.y) : y.y;      // (NaN stays)
          r[i][k] = PagedType<__half>::pack(lo, hi);
        }
      }
      if (i & 1) store(32 * (i / 2), r[i - 1][0], r[i - 1][1], r[i - 1][2], r[i - 1][3], r[i][0], r[i][1], r[i][2], r[i][3]);
    }
  }
}
__device__ __forceinline__ bool whole_sectors(const void* p, long long row, long long head, int size) { return ((reinterpret_cast<unsigned long long>(p) | (unsigned long long)(row * size) | (unsigned long long)(head * size)) & 31) == 0; }

constexpr int kReadWarps = 8;

// A warp has rows_per_warp neighbouring rows: what finding a row takes (whose block, which page, one load after the other) is under way for all of them at once, and so are two rows' groups.
// Traffic bounds it, what is written above all: a lane has a whole group (16 bytes of numbers, one scale) and stores whole sectors.  Two sequences of 16,384 positions of eight heads of 128: 31.9 us, 5.4 TB/s of the
// 172 MB that are read and written, in 32 bits 68.7 us, 4.5 TB/s of 306; 36.6 with eight elements a lane, 16 bytes a store.  Three short blocks: 3.1 us, what finding a row takes.
template <typename T, int DH>
__global__ void __launch_bounds__(kReadWarps * 32)
k_quant_read(const __grid_constant__ QuantReadArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kGroups = DH / kQuantGroup, kAhead = 4;
  __shared__ int s_seq[kReadWarps * kReadRows], s_pos[kReadWarps * kReadRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, here = kReadWarps * a.rows_per_warp;
  const long long row0 = (long long)blockIdx.x * here;
  if (threadIdx.x < here) s_seq[threadIdx.x] = -1;
  __syncthreads();
  for (int b = threadIdx.x; b < a.blk.n_seqs; b += kReadWarps * 32) {
    const int start = __ldcg(a.blk.start + b), len = __ldcg(a.blk.len + b), kv = __ldcg(a.blk.kv_len + b);
    const int flag = paged_block_flag(a.blk, a.kv.page_size, true, start, len, kv);
    if (flag != 0) {
      if (blockIdx.x == 0) atomicOr(a.status, flag);
    } else {
      // (rows of this CTA that are the block's)
      const int from = (int)max(0ll, start - row0), to = (int)min((long long)here, (long long)start + len - row0);
      for (int i = from; i < to; ++i) { s_seq[i] = b; s_pos[i] = kv + (int)(row0 + i - start); }
    }
  }
  __syncthreads();
  int b = -1, pos = 0, page = -1;
  if (lane < a.rows_per_warp) {
    b = s_seq[warp * a.rows_per_warp + lane];
    pos = s_pos[warp * a.rows_per_warp + lane];
    if (b >= 0) {
      page = __ldcg(a.blk.table + (long long)b * a.blk.table_width + (pos >> a.kv.page_shift));
      if ((unsigned)page >= (unsigned)a.kv.n_pages) atomicOr(a.status, CS_DEV_BADARG);
    }
  }
  // groups of the rows: keys of all heads, then values
  const int n = a.kv.n_kv_heads * kGroups, per_row = 2 * n, total = per_row * a.rows_per_warp;
  const bool by_32 = whole_sectors(a.k, a.k_row, a.k_head, sizeof(T)) && whole_sectors(a.v, a.v_row, a.v_head, sizeof(T));
  for (int i0 = 0; i0 < total; i0 += 32 * kAhead) {
    uint4 w[kAhead];
    unsigned s[kAhead];
    char* dst[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const int i = i0 + 32 * j + lane, r = min(i, total - 1) / per_row;
      const int rb = __shfl_sync(0xffffffffu, b, r), rp = __shfl_sync(0xffffffffu, page, r), slot = __shfl_sync(0xffffffffu, pos, r) & (a.kv.page_size - 1);
      const int e = i - r * per_row, g = e < n ? e : e - n, h = g / kGroups, c = g % kGroups;
      dst[j] = nullptr;
      w[j] = make_uint4(kZeros, kZeros, kZeros, kZeros);
      s[j] = 0;
      if (i < total && rb >= 0) {
        const long long row = row0 + warp * a.rows_per_warp + r;
        dst[j] = e < n ? a.k + (row * a.k_row + h * a.k_head + c * kQuantGroup) * (long long)sizeof(T) : a.v + (row * a.v_row + h * a.v_head + c * kQuantGroup) * (long long)sizeof(T);
        if ((unsigned)rp < (unsigned)a.kv.n_pages) {
          const uint32_t in_page = ((uint32_t)h * a.kv.page_size + slot) * kGroups + c;
          w[j] = __ldcg(reinterpret_cast<const uint4*>(e < n ? a.kv.k : a.kv.v) + ((unsigned long long)rp * a.kv.data_units + in_page));
          s[j] = __ldcg((e < n ? a.kv.ks : a.kv.vs) + ((unsigned long long)rp * a.kv.scale_page + in_page));
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (dst[j] != nullptr) put_group<T>(dst[j], w[j], s[j], by_32);
  }
}

// Copies in 16 bits of the positions that blocks attend to, for the attention of tall blocks: sequence b's in the pages from b copy_pages on.  Sixteen positions of a head are one run of words, of scales and of copied
// elements; a warp has several heads of them, so that finding them (lengths, page) is paid once.  8 x 16,405 positions of eight heads of 64: 62 us, 5.5 TB/s.
template <typename T, int DH>
__global__ void __launch_bounds__(kReadWarps * 32)
k_quant_copy(const __grid_constant__ QuantReadArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kRun = 16 * DH / kQuantGroup, kEach = (kRun + 31) / 32;      // groups of a run, of a lane
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (blockIdx.x == 0)
    for (int b = threadIdx.x; b < a.blk.n_seqs; b += kReadWarps * 32) {
      const int len = __ldcg(a.blk.len + b), flag = paged_block_flag(a.blk, a.kv.page_size, a.mask != CS_MASK_PREFIX, __ldcg(a.blk.start + b), len, __ldcg(a.blk.kv_len + b));
      if (flag != 0) atomicOr(a.status, flag);
      a.copy_len[b] = flag != 0 ? 0 : len;
    }
  const int runs = (a.copy_pages << a.copy_shift) / 16, H = a.kv.n_kv_heads;
  // tasks: (sequence, sixteen positions, share of the heads)
  const long long n = (long long)a.blk.n_seqs * runs * a.shares;
  for (long long i = (long long)blockIdx.x * kReadWarps + warp; i < n; i += (long long)gridDim.x * kReadWarps) {
    const int share = (int)(i % a.shares), b = (int)(i / a.shares / runs), pos = (int)(i / a.shares - (long long)b * runs) * 16;
    const int start = __ldcg(a.blk.start + b), len = __ldcg(a.blk.len + b), kv = __ldcg(a.blk.kv_len + b);
    if (len <= 0 || paged_block_flag(a.blk, a.kv.page_size, a.mask != CS_MASK_PREFIX, start, len, kv) != 0) continue;
    int lo, hi;
    paged_range(a.mask, a.window, len, kv, 0, len - 1, lo, hi);
    if (pos + 16 <= lo || pos >= hi) continue;
    const int page = __ldcg(a.blk.table + (long long)b * a.blk.table_width + (pos >> a.kv.page_shift));
    const bool exists = (unsigned)page < (unsigned)a.kv.n_pages;
    if (!exists && lane == 0) atomicOr(a.status, CS_DEV_BADARG);
    const int slot = pos & (a.kv.page_size - 1);
    const long long at = ((long long)b * a.copy_pages + (pos >> a.copy_shift)) * a.k_row + (long long)(pos & ((1 << a.copy_shift) - 1)) * DH;
    for (int h = share; h < H; h += a.shares) {
      const uint32_t in_page = ((uint32_t)h * a.kv.page_size + slot) * (DH / kQuantGroup);
      const long long to = (at + h * a.k_head) * (long long)sizeof(T);
      uint4 w[2][kEach];
      unsigned s[2][kEach];
#pragma unroll
      for (int j = 0; j < kEach; ++j) {
        w[0][j] = w[1][j] = make_uint4(kZeros, kZeros, kZeros, kZeros);
        s[0][j] = s[1][j] = 0;
        if (exists && j * 32 + lane < kRun) {
          const unsigned long long d = (unsigned long long)page * a.kv.data_units + in_page + j * 32 + lane, g = (unsigned long long)page * a.kv.scale_page + in_page + j * 32 + lane;
          w[0][j] = __ldcg(reinterpret_cast<const uint4*>(a.kv.k) + d); s[0][j] = __ldcg(a.kv.ks + g);
          w[1][j] = __ldcg(reinterpret_cast<const uint4*>(a.kv.v) + d); s[1][j] = __ldcg(a.kv.vs + g);
        }
      }
#pragma unroll
      for (int j = 0; j < kEach; ++j)
        if (j * 32 + lane < kRun) {
          put_group<T>(a.k + to + (j * 32 + lane) * kQuantGroup * (int)sizeof(T), w[0][j], s[0][j], true);      // (the copies are whole multiples of 32 bytes from aligned bases on)
          put_group<T>(a.v + to + (j * 32 + lane) * kQuantGroup * (int)sizeof(T), w[1][j], s[1][j], true);
        }
    }
  }
}

__global__ void k_quant_iota(int* p, int n) {
  CS_PDL_PROLOGUE();
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) p[i] = i;
}

// Query rows per KV head (on the average of a call's sequences) that the kernel for few rows always has, up to 32: a pass over the keys; the tensor cores always have, more than 128; that are worked out
// from copies there, where they fit, more than 2,560.  In between it is the work that decides, rows x positions x KV heads x sequences: the tensor cores' kernel has more to set up (32 query heads in groups of four, us here
// and there; 84 rows over 512 keys 16.7 and 20.9, over 4,096 27.9 and 21.3; 44 rows over 4,096 keys 17.9 and 18.6, over 30,720 48 and 37; 24 rows 30 and 36; 8 sequences over 16,384 keys, 24 rows 54 and 73, 44 rows 97 and 74,
// 84 rows 168 and 76; 132 rows over 200 keys 17.5 and 18.0, of four sequences 19.3 and 18.6, of sixteen 48 and 19; 512 rows over 200 keys 21.7 and 22.8, heads of 64 15.1 and 19.2).  Expanded by the kernel and from copies: 84 rows over 8 x 16,384 keys 76 and 129, 2,400 rows over 30,720 keys 307 and 308, 8,192 rows 936 and 896; windows of 1,000 keys, 2,400 rows 61 and 63, 4,500 rows 124 and 113.
constexpr long long kFewRows = 32, kTallRows = 128, kTallWork = 3 << 19, kCopyRows = 2560;

thread_local char t_quant_err[256] = "";

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int bytes_of(int dtype) { return dtype == CS_F32 ? 4 : 2; }

cs_status fail(cs_quant_cache* c, cs_status s, const char* text) {
  snprintf(c->err, sizeof(c->err), "%s", text);
  return s;
}
// source rows (of type `in`) and, where out >= 0, destination rows
cs_status check_rows(const cs_heads* h, int in, int out) {
  if (h->n_heads < 0) return CS_ERR_ARG;
  if (h->n_heads == 0) return CS_OK;
  if (in >= 0 && (h->x == nullptr || !aligned16(h->x) || h->row_stride % (16 / bytes_of(in)) != 0 || h->head_stride % (16 / bytes_of(in)) != 0 || !aligned16(h->gain))) return CS_ERR_ARG;
  if (out >= 0 && (h->y == nullptr || !aligned16(h->y) || h->y_row_stride % (16 / bytes_of(out)) != 0 || h->y_head_stride % (16 / bytes_of(out)) != 0)) return CS_ERR_ARG;
  return CS_OK;
}
cs_status check_blocks(const cs_blocks* b) {
  if (b->n_seqs < 0 || b->rows < 0 || b->table_width < 0) return CS_ERR_ARG;
  if (b->n_seqs == 0 || b->rows == 0) return CS_OK;
  return b->start == nullptr || b->len == nullptr || b->kv_len == nullptr || (b->page_table == nullptr && b->table_width > 0) ? CS_ERR_ARG : CS_OK;
}
BlocksView view_of(const cs_blocks* b) { return BlocksView{b->start, b->len, b->kv_len, b->page_table, b->n_seqs, b->table_width, b->rows}; }

// why a configuration is refused (CS_OK: it is not)
cs_status check_config(const cs_quant_config* c, const char** why) {
  *why = "";
  if (c == nullptr) { *why = "NULL argument"; return CS_ERR_ARG; }
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128) { *why = "head_dim must be 32, 64 or 128"; return CS_ERR_SHAPE; }
  if (c->page_size < 16 || (c->page_size & (c->page_size - 1)) != 0) { *why = "page_size must be a power of two from 16 on"; return CS_ERR_SHAPE; }
  if (c->n_pages < 1 || c->n_kv_heads < 1 || c->n_kv_heads > 0x0fffffff) { *why = "no pages or no heads"; return CS_ERR_ARG; }
  const int64_t row = (int64_t)c->n_kv_heads * c->page_size;         // rows of a page
  if (c->page_stride % 16 != 0 || c->scale_page_stride % 8 != 0 || (c->n_pages > 1 && (c->page_stride < row * (c->head_dim / 2) || c->scale_page_stride < row * (c->head_dim / kQuantGroup)))) {
    *why = "pages must not overlap, their strides must be multiples of 16 bytes";
    return CS_ERR_ARG;
  }
  // (rows of a page times 64 bytes, and strides in 16 bytes, in 32 bits)
  if (row > (1 << 26) || c->page_stride > (1ll << 35) || c->scale_page_stride > (1ll << 34)) { *why = "pages of more than 2^26 rows, or farther apart than 2^35 bytes"; return CS_ERR_SHAPE; }
  if (c->tall_positions < 0 || c->tall_positions > (1ll << 30)) { *why = "tall_positions must be between 0 and 2^30"; return CS_ERR_ARG; }
  return CS_OK;
}

struct QuantLayout {
  size_t status, splits, parts, parts_ml, table, len, k, v, paged, total;
  size_t paged_bytes;
  long long positions;         // room for copies
};
// a cache of 16 bits over the copies, with pages of 128 >> i slots
cs_paged_config copies_config(const cs_quant_config& c, long long positions, char* k, char* v, int i, int dtype) {
  cs_paged_config p = {};
  p.page_size = kQuantCopyPage >> i;
  p.k = k; p.v = v;
  p.slot_stride = c.head_dim; p.head_stride = (int64_t)p.page_size * c.head_dim; p.page_stride = p.head_stride * c.n_kv_heads;
  p.n_pages = (int32_t)(positions >> (7 - i)); p.n_kv_heads = c.n_kv_heads; p.head_dim = c.head_dim; p.dtype = dtype;
  return p;
}
QuantLayout layout_of(const cs_quant_config& c) {
  QuantLayout l = {};
  size_t at = 0;
  auto put = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) & ~(size_t)255; return o; };
  l.status = put(256);
  l.splits = put(kQuantMaxSms * kQuantCtasPerSm * sizeof(PagedSplit));
  l.parts = put((size_t)kQuantMaxSms * kQuantRowsPerSm * 2 * c.head_dim * 4);
  l.parts_ml = put((size_t)kQuantMaxSms * kQuantRowsPerSm * 2 * 8);
  // (a page of copies at least: the caches over them are also what tall blocks have their sums in)
  l.positions = c.tall_positions > 0 ? (c.tall_positions + 15) & ~15ll : 16;
  const cs_paged_config p = copies_config(c, l.positions, nullptr, nullptr, 3, CS_BF16);
  const size_t pool = (size_t)l.positions * c.n_kv_heads * c.head_dim * 2;
  l.paged_bytes = cs_paged_workspace_bytes(&p);
  l.table = put((size_t)l.positions / 16 * 4);
  l.len = put((size_t)l.positions / 16 * 4);
  l.k = put(pool);
  l.v = put(pool);
  l.paged = put(l.paged_bytes);
  l.total = at;
  return l;
}

// `first`: the cache whose workspace it is already (nullptr: nobody's)
cs_status create(const char* name, cs_quant_cache** out, const cs_quant_config* cfg, void* workspace, size_t workspace_bytes, const cs_quant_cache* first, void* stream) {
  auto refuse = [&](cs_status s, const char* text) {
    snprintf(t_quant_err, sizeof(t_quant_err), "%s: %s", name, text);
    return s;
  };
  t_quant_err[0] = 0;
  const char* why;
  if (out == nullptr) return refuse(CS_ERR_ARG, "NULL argument");
  *out = nullptr;
  const cs_status s = check_config(cfg, &why);
  if (s != CS_OK) return refuse(s, why);
  if (cfg->k == nullptr || cfg->v == nullptr || cfg->k_scale == nullptr || cfg->v_scale == nullptr || workspace == nullptr) return refuse(CS_ERR_ARG, "NULL pointer");
  if (!aligned16(cfg->k) || !aligned16(cfg->v) || !aligned16(cfg->k_scale) || !aligned16(cfg->v_scale)) return refuse(CS_ERR_ARG, "the pools must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return refuse(CS_ERR_ARG, "the workspace must be 256-byte aligned");
  const QuantLayout l = layout_of(*cfg);
  if (workspace_bytes < l.total) return refuse(CS_ERR_CAPACITY, "the workspace is too small");
  if (first != nullptr && (first->cfg.head_dim != cfg->head_dim || first->cfg.n_kv_heads != cfg->n_kv_heads || first->cfg.tall_positions != cfg->tall_positions))
    return refuse(CS_ERR_SHAPE, "caches that share a workspace need the same heads and tall_positions");
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return refuse(CS_ERR_CUDA, "no device");
  cs_quant_cache* c = static_cast<cs_quant_cache*>(calloc(1, sizeof(cs_quant_cache)));
  if (c == nullptr) return refuse(CS_ERR_CAPACITY, "out of host memory");
  c->cfg = *cfg;
  c->num_sms = sms < kQuantMaxSms ? sms : kQuantMaxSms;
  int shift = 0;
  while ((1 << shift) < cfg->page_size) ++shift;
  c->view = QuantView{static_cast<uint32_t*>(cfg->k), static_cast<uint32_t*>(cfg->v), static_cast<unsigned short*>(cfg->k_scale), static_cast<unsigned short*>(cfg->v_scale),
                      cfg->page_stride / 4, cfg->scale_page_stride, (uint32_t)(cfg->page_stride / 16), (uint32_t)(cfg->scale_page_stride / 8), cfg->n_pages, cfg->page_size, shift, cfg->n_kv_heads};
  char* ws = static_cast<char*>(workspace);
  c->workspace = workspace;
  c->workspace_bytes = workspace_bytes;
  c->status = reinterpret_cast<int*>(ws + l.status);
  c->splits = reinterpret_cast<PagedSplit*>(ws + l.splits);
  c->parts = reinterpret_cast<float*>(ws + l.parts);
  c->parts_ml = reinterpret_cast<float*>(ws + l.parts_ml);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (first == nullptr) {
    const cudaError_t e = cudaMemsetAsync(ws, 0, l.splits, st);
    if (e != cudaSuccess) {
      free(c);
      return refuse(CS_ERR_CUDA, cudaGetErrorString(e));
    }
  }
  c->drop = -1;
  c->tall_positions = cfg->tall_positions > 0 ? l.positions : 0;
  c->tall_k = ws + l.k;
  c->tall_v = ws + l.v;
  c->tall_table = reinterpret_cast<int*>(ws + l.table);
  c->tall_len = reinterpret_cast<int*>(ws + l.len);
  // (the smallest pages first: there is one at least)
  const cs_paged_cache* beside = first != nullptr ? first->tall[0][3] : nullptr;
  cs_status r = CS_OK;
  for (int i = 3; i >= 0; --i)
    for (int type = 0; type < 2 && r == CS_OK; ++type) {
      const cs_paged_config p = copies_config(*cfg, l.positions, c->tall_k, c->tall_v, i, type == 0 ? CS_BF16 : CS_F16);
      if (p.n_pages < 1) continue;
      r = beside != nullptr ? cs_paged_create_beside(&c->tall[type][i], &p, beside) : cs_paged_create(&c->tall[type][i], &p, ws + l.paged, l.paged_bytes, stream);
      if (beside == nullptr) beside = c->tall[type][i];
    }
  const int n = (int)(l.positions / 16);
  if (r == CS_OK && first == nullptr && cs_launch_pdl(k_quant_iota, dim3((unsigned)(n < 1 << 18 ? (n + 1023) / 1024 : 256)), dim3(256), 0, st, c->tall_table, n) != cudaSuccess) r = CS_ERR_CUDA;
  if (r != CS_OK) {
    refuse(r, cs_paged_last_error(nullptr)[0] != 0 ? cs_paged_last_error(nullptr) : "launch failed");
    cs_quant_destroy(c);
    return r;
  }
  *out = c;
  return CS_OK;
}

template <typename S, typename D>
cudaError_t launch_append(QuantAppendArgs a, int head_dim, int sms, cudaStream_t st) {
  const int per = 512 / head_dim, units = cs_ceil_div(a.n_q, per) + 2 * cs_ceil_div(a.n_kv, per);
  a.warps_per_row = kWarps;
  while (a.warps_per_row > 1 && (a.warps_per_row >= 2 * units || (long long)a.n_rows * a.warps_per_row > 16 * sms)) a.warps_per_row /= 2;
  const dim3 grid((unsigned)(((long long)a.n_rows * a.warps_per_row + kWarps - 1) / kWarps)), block(kThreads);
  switch (head_dim) {
    case 32: return cs_launch_pdl(k_quant_append<S, D, 32>, grid, block, 0, st, a);
    case 64: return cs_launch_pdl(k_quant_append<S, D, 64>, grid, block, 0, st, a);
    default: return cs_launch_pdl(k_quant_append<S, D, 128>, grid, block, 0, st, a);
  }
}
template <typename T>
cudaError_t launch_read(QuantReadArgs a, int head_dim, int sms, cudaStream_t st) {
  // (as many rows a warp as leave every SM its warps)
  a.rows_per_warp = kReadRows;
  while (a.rows_per_warp > 1 && (long long)a.blk.rows < (long long)sms * 32 * a.rows_per_warp) a.rows_per_warp /= 2;
  const int here = kReadWarps * a.rows_per_warp;
  const dim3 grid((unsigned)(((long long)a.blk.rows + here - 1) / here)), block(kReadWarps * 32);
  switch (head_dim) {
    case 32: return cs_launch_pdl(k_quant_read<T, 32>, grid, block, 0, st, a);
    case 64: return cs_launch_pdl(k_quant_read<T, 64>, grid, block, 0, st, a);
    default: return cs_launch_pdl(k_quant_read<T, 128>, grid, block, 0, st, a);
  }
}
template <typename T>
cudaError_t launch_copy(QuantReadArgs a, int head_dim, int sms, cudaStream_t st) {
  const long long runs = (long long)a.blk.n_seqs * ((a.copy_pages << a.copy_shift) / 16);
  a.shares = 1;
  while (2 * a.shares <= a.kv.n_kv_heads && runs * a.shares < 64ll * sms) a.shares *= 2;
  const long long ctas = (runs * a.shares + kReadWarps - 1) / kReadWarps;
  const dim3 grid((unsigned)(ctas < 8 * sms ? (ctas > 0 ? ctas : 1) : 8 * sms)), block(kReadWarps * 32);
  switch (head_dim) {
    case 32: return cs_launch_pdl(k_quant_copy<T, 32>, grid, block, 0, st, a);
    case 64: return cs_launch_pdl(k_quant_copy<T, 64>, grid, block, 0, st, a);
    default: return cs_launch_pdl(k_quant_copy<T, 128>, grid, block, 0, st, a);
  }
}

}  // namespace

size_t cs_quant_workspace_bytes(const cs_quant_config* cfg) {
  const char* why;
  return check_config(cfg, &why) == CS_OK ? layout_of(*cfg).total : 0;
}

cs_status cs_quant_create(cs_quant_cache** out, const cs_quant_config* cfg, void* workspace, size_t workspace_bytes, void* stream) {
  return create("cs_quant_create", out, cfg, workspace, workspace_bytes, nullptr, stream);
}

cs_status cs_quant_create_beside(cs_quant_cache** out, const cs_quant_config* cfg, const cs_quant_cache* first) {
  if (first == nullptr) {
    snprintf(t_quant_err, sizeof(t_quant_err), "cs_quant_create_beside: NULL argument");
    if (out != nullptr) *out = nullptr;
    return CS_ERR_ARG;
  }
  return create("cs_quant_create_beside", out, cfg, first->workspace, first->workspace_bytes, first, nullptr);
}

void cs_quant_destroy(cs_quant_cache* c) {
  if (c == nullptr) return;
  for (int type = 0; type < 2; ++type)
    for (int i = 0; i < 4; ++i) cs_paged_destroy(c->tall[type][i]);
  free(c);
}

int cs_quant_head_dim(const cs_quant_cache* c) { return c != nullptr ? c->cfg.head_dim : 0; }

const char* cs_quant_last_error(const cs_quant_cache* c) { return c != nullptr ? c->err : t_quant_err; }

cs_status cs_quant_debug_drop_tile(cs_quant_cache* c, int tile) {
  if (c == nullptr) return CS_ERR_ARG;
  c->drop = tile < 0 ? -1 : tile;
  return CS_OK;
}

cs_status cs_quant_status(cs_quant_cache* c, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int bits = 0;
  CS_CUDA_OK(c, cudaMemcpyAsync(&bits, c->status, sizeof(int), cudaMemcpyDeviceToHost, st));
  CS_CUDA_OK(c, cudaStreamSynchronize(st));
  const cs_status tall = cs_paged_status(c->tall[0][3], stream);
  if (tall != CS_OK) fail(c, tall, cs_paged_last_error(c->tall[0][3]));
  if (bits == 0 || tall == CS_ERR_TIMEOUT || tall == CS_ERR_CUDA) {
    if (bits != 0) CS_CUDA_OK(c, cudaMemsetAsync(c->status, 0, sizeof(int), st));
    return tall;
  }
  CS_CUDA_OK(c, cudaMemsetAsync(c->status, 0, sizeof(int), st));
  CS_CUDA_OK(c, cudaStreamSynchronize(st));
  if (bits & CS_DEV_TIMEOUT) return fail(c, CS_ERR_TIMEOUT, "a bounded wait ran out");
  if (bits & CS_DEV_CAPACITY) return fail(c, CS_ERR_CAPACITY, "a block does not fit its row of the page table, or the rotation table is too short");
  return fail(c, CS_ERR_ARG, "a length is negative, rows lie outside the tensors, or a page does not exist");
}

cs_status cs_quant_append(cs_quant_cache* c, const cs_blocks* blocks, const cs_heads* k, const cs_heads* v, const cs_heads* q, cs_dtype in, cs_dtype out, const float* rope, int n_positions,
                          int rot_dim, float eps, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  if (blocks == nullptr || k == nullptr || v == nullptr) return fail(c, CS_ERR_ARG, "NULL argument");
  if ((out != CS_BF16 && out != CS_F16) || (in != out && in != CS_F32)) return fail(c, CS_ERR_ARG, "queries and gains are CS_BF16 or CS_F16, rows of the same type or CS_F32");
  cs_status s = check_blocks(blocks);
  if (s != CS_OK) return fail(c, s, "bad blocks");
  if (blocks->n_seqs == 0 || blocks->rows == 0) return CS_OK;
  if (rot_dim < 0 || !(eps >= 0.f) || (rot_dim > 0 && (rope == nullptr || n_positions < 1 || !aligned16(rope)))) return fail(c, CS_ERR_ARG, "bad rotation table or eps");
  if (rot_dim % 16 != 0 || rot_dim > c->cfg.head_dim) return fail(c, CS_ERR_SHAPE, "rot_dim must be a multiple of 16, at most head_dim");
  if (k->n_heads != c->cfg.n_kv_heads || v->n_heads != c->cfg.n_kv_heads) return fail(c, CS_ERR_SHAPE, "keys and values need the cache's heads");
  if ((q != nullptr && (s = check_rows(q, in, out)) != CS_OK) || (s = check_rows(k, in, -1)) != CS_OK || (s = check_rows(v, in, -1)) != CS_OK)
    return fail(c, s, "rows need 16-byte aligned bases and strides of multiples of 16 bytes");
  if ((q != nullptr ? q->n_heads : 0) > 0x0fffffff) return fail(c, CS_ERR_SHAPE, "too many heads");
  QuantAppendArgs a = {};
  if (q != nullptr && q->n_heads > 0) {
    a.q = static_cast<const char*>(q->x); a.q_row = q->row_stride; a.q_head = q->head_stride;
    a.yq = static_cast<char*>(q->y); a.yq_row = q->y_row_stride; a.yq_head = q->y_head_stride;
    a.q_gain = static_cast<const char*>(q->gain); a.n_q = q->n_heads;
  }
  a.k = static_cast<const char*>(k->x); a.k_row = k->row_stride; a.k_head = k->head_stride;
  a.k_gain = static_cast<const char*>(k->gain); a.n_kv = k->n_heads;
  a.v = static_cast<const char*>(v->x); a.v_row = v->row_stride; a.v_head = v->head_stride;
  a.n_rows = blocks->rows;
  a.rope = rope; a.n_positions = n_positions; a.rot_dim = rot_dim; a.eps = eps;
  a.kv = c->view; a.blk = view_of(blocks); a.status = c->status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int dh = c->cfg.head_dim;
  if (out == CS_BF16) CS_CUDA_OK(c, in == CS_F32 ? (launch_append<float, __nv_bfloat16>(a, dh, c->num_sms, st)) : (launch_append<__nv_bfloat16, __nv_bfloat16>(a, dh, c->num_sms, st)));
  else CS_CUDA_OK(c, in == CS_F32 ? (launch_append<float, __half>(a, dh, c->num_sms, st)) : (launch_append<__half, __half>(a, dh, c->num_sms, st)));
  return CS_OK;
}

cs_status cs_quant_read(cs_quant_cache* c, const cs_blocks* blocks, const cs_heads* k, const cs_heads* v, cs_dtype out, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  if (blocks == nullptr || k == nullptr || v == nullptr) return fail(c, CS_ERR_ARG, "NULL argument");
  if (out < CS_BF16 || out > CS_F32) return fail(c, CS_ERR_ARG, "rows are CS_BF16, CS_F16 or CS_F32");
  cs_status s = check_blocks(blocks);
  if (s != CS_OK) return fail(c, s, "bad blocks");
  if (blocks->n_seqs == 0 || blocks->rows == 0) return CS_OK;
  if (k->n_heads != c->cfg.n_kv_heads || v->n_heads != c->cfg.n_kv_heads) return fail(c, CS_ERR_SHAPE, "keys and values need the cache's heads");
  if ((s = check_rows(k, -1, out)) != CS_OK || (s = check_rows(v, -1, out)) != CS_OK) return fail(c, s, "rows need 16-byte aligned bases and strides of multiples of 16 bytes");
  QuantReadArgs a = {};
  a.kv = c->view; a.blk = view_of(blocks); a.status = c->status;
  a.k = static_cast<char*>(k->y); a.k_row = k->y_row_stride; a.k_head = k->y_head_stride;
  a.v = static_cast<char*>(v->y); a.v_row = v->y_row_stride; a.v_head = v->y_head_stride;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int dh = c->cfg.head_dim;
  CS_CUDA_OK(c, out == CS_F32 ? launch_read<float>(a, dh, c->num_sms, st) : out == CS_BF16 ? launch_read<__nv_bfloat16>(a, dh, c->num_sms, st) : launch_read<__half>(a, dh, c->num_sms, st));
  return CS_OK;
}

cs_status cs_quant_attention(cs_quant_cache* c, const cs_blocks* blocks, const void* q, int64_t q_row_stride, int64_t q_head_stride, int n_heads, cs_dtype dtype, cs_mask mask, int window,
                             float scale, void* out, float* lse, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  if (blocks == nullptr) return fail(c, CS_ERR_ARG, "NULL argument");
  const cs_status s = check_blocks(blocks);
  if (s != CS_OK) return fail(c, s, "bad blocks");
  if (dtype != CS_BF16 && dtype != CS_F16) return fail(c, CS_ERR_ARG, "queries are CS_BF16 or CS_F16");
  if (mask < CS_MASK_CAUSAL || mask > CS_MASK_FULL || window < 0 || !(scale > 0.f) || !(scale <= 2.0e38f)) return fail(c, CS_ERR_ARG, "bad mask, window or scale");
  if ((long long)blocks->table_width * c->cfg.page_size > (1ll << 30)) return fail(c, CS_ERR_SHAPE, "a sequence has room for 2^30 positions at most");
  if (n_heads < 1 || n_heads % c->cfg.n_kv_heads != 0 || n_heads / c->cfg.n_kv_heads > 128) return fail(c, CS_ERR_SHAPE, "n_heads must be a multiple of the cache's heads, at most 128 per KV head");
  if ((long long)blocks->rows * n_heads > 0x7fffff00ll) return fail(c, CS_ERR_SHAPE, "too many rows");
  if (blocks->n_seqs == 0 || blocks->rows == 0) return CS_OK;
  if (q == nullptr || out == nullptr) return fail(c, CS_ERR_ARG, "NULL pointer");
  if (!aligned16(q) || !aligned16(out) || q_row_stride % 8 != 0 || q_head_stride % 8 != 0) return fail(c, CS_ERR_ARG, "q and out need 16-byte aligned bases, q strides of multiples of 8 elements");
  if ((reinterpret_cast<uintptr_t>(lse) & 3) != 0) return fail(c, CS_ERR_ARG, "lse must be aligned to its type");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int group = n_heads / c->cfg.n_kv_heads;
  const long long per_seq = ((long long)blocks->rows * group + blocks->n_seqs - 1) / blocks->n_seqs;      // query rows of a KV head, on the average
  const long long room = (long long)blocks->table_width * c->cfg.page_size;
  const long long seen = window > 0 ? std::min(room, (long long)window + blocks->rows / blocks->n_seqs) : room;      // positions of a sequence, at most about
  // (queries that repeat one row have no operand map)
  const bool tall = per_seq > kFewRows && (per_seq > kTallRows || per_seq * blocks->n_seqs * c->cfg.n_kv_heads * seen > kTallWork) && (blocks->rows == 1 || q_row_stride > 0) && (n_heads == 1 || q_head_stride > 0);
  // Copies in pages as large as fit: a tile of 128 keys is fetched page by page
  int size = 0;
  long long copy_pages = 0;
  for (; size < 4; ++size) {
    copy_pages = (room + (kQuantCopyPage >> size) - 1) >> (7 - size);
    if ((copy_pages << (7 - size)) <= c->tall_positions / blocks->n_seqs) break;
  }
  if (tall && per_seq > kCopyRows && size < 4 && copy_pages > 0) {
    QuantReadArgs r = {};
    r.kv = c->view; r.blk = view_of(blocks); r.status = c->status;
    r.k = c->tall_k; r.v = c->tall_v;
    r.k_head = (long long)(kQuantCopyPage >> size) * c->cfg.head_dim; r.k_row = r.k_head * c->cfg.n_kv_heads;
    r.mask = mask; r.window = window; r.copy_pages = (int)copy_pages; r.copy_shift = 7 - size; r.copy_len = c->tall_len;
    CS_CUDA_OK(c, dtype == CS_BF16 ? launch_copy<__nv_bfloat16>(r, c->cfg.head_dim, c->num_sms, st) : launch_copy<__half>(r, c->cfg.head_dim, c->num_sms, st));
    cs_blocks b = *blocks;
    b.len = c->tall_len;
    b.page_table = c->tall_table;
    b.table_width = (int)copy_pages;
    cs_paged_cache* const copies = c->tall[dtype == CS_BF16 ? 0 : 1][size];
    cs_paged_debug_drop_tile(copies, c->drop);
    c->drop = -1;
    const cs_status t = cs_paged_attention(copies, &b, q, q_row_stride, q_head_stride, n_heads, mask, window, scale, out, lse, stream);
    return t == CS_OK ? t : fail(c, t, cs_paged_last_error(copies));
  }
  QuantAttnArgs a = {};
  a.kv = c->view;
  a.half = dtype == CS_F16;
  cs_paged_cache* const paged = c->tall[a.half][3];
  PagedAttnArgs& p = a.p;
  p.kv.n_pages = c->view.n_pages; p.kv.page_size = c->view.page_size; p.kv.page_shift = c->view.page_shift; p.kv.n_kv_heads = c->view.n_kv_heads;
  p.blk = view_of(blocks);
  p.q = static_cast<const char*>(q); p.q_row = q_row_stride; p.q_head = q_head_stride;
  p.out = static_cast<char*>(out); p.lse = lse;
  p.n_heads = n_heads; p.group = group;
  p.by_group = PagedDivisor::by(group);
  p.mask = mask; p.window = window;
  p.scale = scale; p.scale_log2e = (float)(1.4426950408889634 * (double)scale);
  p.status = c->status;
  p.wait_ns = paged->wait_limit_ns;
  p.drop = -1;
  if (tall) {
    p.drop = c->drop;
    c->drop = -1;
    p.kv.k = reinterpret_cast<char*>(c->view.k); p.kv.v = reinterpret_cast<char*>(c->view.v); p.kv.page_stride = c->view.data_page * 4;
    p.ks = c->view.ks; p.vs = c->view.vs; p.scale_page = c->view.scale_page;
    p.parts = paged->parts; p.parts_ml = paged->parts_ml; p.splits = paged->splits;
  } else {
    p.parts = c->parts; p.parts_ml = c->parts_ml; p.splits = c->splits;
  }
  const int most = tall ? kPagedMaxSeqs : kQuantMaxSeqs;
  for (int b = 0; b < blocks->n_seqs; b += most) {      // (a launch's plan holds so many)
    QuantAttnArgs part = a;
    part.p.blk.n_seqs = blocks->n_seqs - b < most ? blocks->n_seqs - b : most;
    part.p.blk.start += b; part.p.blk.len += b; part.p.blk.kv_len += b;
    part.p.blk.table += (long long)b * blocks->table_width;
    const cs_status r = tall ? cs_launch_quant_tc(paged, part.p, st) : cs_launch_quant_few(c, part, per_seq, st);
    if (r != CS_OK) return tall ? fail(c, r, cs_paged_last_error(paged)) : r;
  }
  return CS_OK;
}
