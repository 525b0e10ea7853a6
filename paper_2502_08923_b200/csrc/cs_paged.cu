// Norms and rotation of queries and keys, rows appended to a paged KV cache, and the host side of the paged cache.
//
// For a row at position p and a head x of D elements, h = rot_dim / 2, c_i = cos(p w_i), s_i = sin(p w_i) from a table:
//     u = x rsqrt(mean(x^2) + eps) gain,   y_i = u_i c_i - u_{i+h} s_i,   y_{i+h} = u_{i+h} c_i + u_i s_i   (i < h).
// A lane holds eight elements of a head's first half and their eight partners (16 bytes each of the 16-bit types; behind rot_dim two neighbouring chunks), a head is D / 16 lanes.  With C = gain cos and
// S = gain sin, worked out once per row for the queries and once for the keys, an element is r (x0 C - x1 S), r the head's reciprocal norm (a
// reduction over its lanes), and nothing is exchanged.  Warps take a row each, or 2, 4 or 8 share one where there are few; three units of 32 / (D / 16) heads are in flight, in
// a ring of shared memory for each warp (in registers instead, four of them, 16 warps fit on an SM and not 20, and the setup is there four times: 34 us for the 29 below).
//
// Bound by HBM where there are many rows: 8,192 of the 8B shape 29.3 us (172 MB, 5.9 TB/s of the 6.5 that a copy reaches), an append of 6k rows 30.0 us (150 MB, 5.0).  With an
// element's partner in another lane, fetched by shuffles, and the factors worked out for each head 61 us.  Few rows: launch and a chain of loads (whose block is the row's, which
// page and, at the same time, its rotation): 2.4 - 4.3 us.
#include "cs_paged.cuh"

namespace {

constexpr int kThreads = 256;

// what k_heads does with a row
struct HeadsArgs {
  const char *q, *k, *v;             // sources; head counts 0 = left out
  char *yq, *yk;                     // destinations of rows (yk: unless they go to pages)
  long long q_row, q_head, k_row, k_head, v_row, v_head, yq_row, yq_head, yk_row, yk_head;   // elements
  const char *q_gain, *k_gain;
  int n_q, n_k, n_v, n_rows;
  int warps_per_row;                 // 1, 2, 4 or 8
  const int* pos;                    // positions of rows, unless blocks give them
  const float* rope;
  int n_positions, rot_dim;
  float eps;
  PagedView kv;
  BlocksView blk;
  int* status;
};

__device__ __forceinline__ void fetch16(uint32_t dst, const char* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void fetch_drain() { asm volatile("cp.async.wait_all;" ::: "memory"); }   // before a warp leaves
template <typename T, int N> __device__ __forceinline__ void widen(const uint32_t (&w)[N], f32x2 (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (N == 8) {
      f[i] = pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    } else {
      const float2 x = PagedType<T>::unpack(w[i]);
      f[i] = pack2(x.x, x.y);
    }
  }
}
template <typename T> __device__ __forceinline__ void store8(char* p, const f32x2 (&v)[4]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) unpack2(v[i], f[2 * i], f[2 * i + 1]);
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(PagedType<T>::pack(f[0], f[1]), PagedType<T>::pack(f[2], f[3]), PagedType<T>::pack(f[4], f[5]), PagedType<T>::pack(f[6], f[7]));
  }
}
__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fc00000); }
// eight gains
template <typename T> __device__ __forceinline__ void gain8(const char* g, int chunk, float (&f)[8]) {
  uint32_t w[sizeof(T) == 4 ? 8 : 4];
  const uint4* p = reinterpret_cast<const uint4*>(g + chunk * 8 * (int)sizeof(T));
  const uint4 x = p[0];
  w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  if constexpr (sizeof(T) == 4) {
    const uint4 y = p[1];
    w[4] = y.x; w[5] = y.y; w[6] = y.z; w[7] = y.w;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      f[2 * i] = __uint_as_float(w[2 * i]); f[2 * i + 1] = __uint_as_float(w[2 * i + 1]);
    } else {
      const float2 y = PagedType<T>::unpack(w[i]);
      f[2 * i] = y.x; f[2 * i + 1] = y.y;
    }
  }
}

template <typename S, typename D, int DH, bool kPaged, int kBlock>
__global__ void __launch_bounds__(kBlock * 32, kBlock == 8 ? 2 : 5)
k_heads(HeadsArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kLanes = DH / 16, kPer = 32 / kLanes, kW = sizeof(S) == 4 ? 8 : 4;    // lanes of a head, heads of a unit, words of a chunk
  constexpr bool kWide = sizeof(S) == 4;
  constexpr int kSlots = kWide && kBlock == 8 ? 2 : 4, kPieces = kW / 2, kSlotBytes = kPieces * 512;      // slots of a warp's ring; 16-byte pieces of a lane's two chunks
  __shared__ uint4 s_ring[kBlock][kSlots][kPieces][32];
  __shared__ int s_seq[kBlock], s_pos[kBlock];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = lane % kLanes, sub = lane / kLanes;
  const int n_here = kBlock / a.warps_per_row;
  const long long row0 = (long long)blockIdx.x * n_here, row = row0 + warp / a.warps_per_row;
  // a row's units: up to kPer neighbouring heads, of queries, then keys, then values
  const int uq = (a.n_q + kPer - 1) / kPer, uk = uq + (a.n_k + kPer - 1) / kPer, units = row < a.n_rows ? uk + (a.n_v + kPer - 1) / kPer : 0;
  const int step = a.warps_per_row, u0 = warp % step;
  // this lane's chunks: partners of the rotation, or two neighbours behind what is rotated
  const int half = a.rot_dim >> 4;
  const bool rotated = pair < half;
  const int c0 = rotated ? pair : 2 * pair, c1 = rotated ? pair + half : c0 + 1;

  // Fetching runs kSlots - 1 units ahead of the rest.  16-bit rows: a lane reads from the ring only what it fetched itself.  32-bit rows lie in the ring as in memory, fetched 16 bytes a
  // lane side by side (each lane its own 32 bytes in two fetches asked L2 for every sector twice: 8,192 rows of the 8B shape 61.5 us, so 40.6).
  int fu = u0, f_end = 0, f_h = 0, f_n = 0;      // next unit, where its kind's units end, this lane's head of it, the kind's heads
  const char* f_p = a.q;
  long long f_step = 0;
  const int f_first = kWide ? pair * 16 : c0 * 16;                                         // byte of the head where this lane's first piece begins
  const char* mine = reinterpret_cast<const char*>(&s_ring[warp][0][0][kWide ? 0 : lane]) + (kWide ? sub * DH * 4 : 0);
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(mine) + (kWide ? pair * 16 : 0);
  auto fetch = [&](uint32_t place) {
    if (fu >= f_end && fu < units) {             // (the same in the whole warp)
      const int kind = fu < uq ? 0 : fu < uk ? 1 : 2;
      const long long rs = kind == 0 ? a.q_row : kind == 1 ? a.k_row : a.v_row, hs = kind == 0 ? a.q_head : kind == 1 ? a.k_head : a.v_head;
      f_h = (fu - (kind == 0 ? 0 : kind == 1 ? uq : uk)) * kPer + sub;
      f_n = kind == 0 ? a.n_q : kind == 1 ? a.n_k : a.n_v;
      f_end = kind == 0 ? uq : kind == 1 ? uk : units;
      f_p = (kind == 0 ? a.q : kind == 1 ? a.k : a.v) + (row * rs + f_h * hs) * (long long)sizeof(S) + f_first;
      f_step = step * kPer * hs * (long long)sizeof(S);
    }
    if (fu < units && f_h < f_n) {
      const uint32_t d = ring + place;
      if constexpr (kWide) {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) fetch16(d + j * kLanes * 16, f_p + j * kLanes * 16);
      } else {
        fetch16(d, f_p);
        fetch16(d + 512, f_p + (c1 - c0) * 16);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    fu += step; f_h += step * kPer; f_p += f_step;
  };
#pragma unroll
  for (int i = 0; i < kSlots - 1; ++i) fetch(i * kSlotBytes); // (whose row it is, and where it goes, takes three loads in a row: these are under way meanwhile)

  int pos = 0;
  int page = 0;                                  // (not looked at before the first factors have been asked for)
  if constexpr (kPaged) {
    // the blocks these rows belong to
    if (threadIdx.x < kBlock) s_seq[threadIdx.x] = -1;
    __syncthreads();
    for (int b = threadIdx.x; b < a.blk.n_seqs; b += kBlock * 32) {
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
    const int b = s_seq[warp / a.warps_per_row];
    if (b < 0 || row >= a.n_rows) {
      fetch_drain();
      return;
    }
    pos = s_pos[warp / a.warps_per_row];
    if (a.rot_dim > 0 && pos >= a.n_positions) {
      if (lane == 0) atomicOr(a.status, CS_DEV_CAPACITY);
      fetch_drain();
      return;
    }
    page = __ldcg(a.blk.table + (long long)b * a.blk.table_width + (pos >> a.kv.page_shift));
  } else {
    if (row >= a.n_rows) return;
    if (a.rot_dim > 0) pos = __ldcg(a.pos + row);
  }

  // y0 = r (x0 C0 - x1 S1), y1 = r (x1 C1 + x0 S0), C = gain cos, S = gain sin: worked out once for the queries and once for the keys.  (Table
  // and gains are read through L1: all warps of a row want the same.)
  f32x2 C0[4], C1[4], S0[4], S1[4];
  uint32_t place = 0;                            // of this unit in the ring, bytes
  for (int u = u0; u < units;) {
    const int kind = u < uq ? 0 : u < uk ? 1 : 2;
    const int n = kind == 0 ? a.n_q : kind == 1 ? a.n_k : a.n_v, end = kind == 0 ? uq : kind == 1 ? uk : units;
    const bool plain = kind == 2;                // (values are neither normed nor rotated)
    const char* gain = kind == 0 ? a.q_gain : kind == 1 ? a.k_gain : nullptr;
    const bool norm = gain != nullptr;
    if (!plain) {
      float g0[8], g1[8];
      if (norm) {
        gain8<D>(gain, c0, g0);
        gain8<D>(gain, c1, g1);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g0[j] = g1[j] = 1.f;
      }
      if (!rotated) {
#pragma unroll
        for (int j = 0; j < 4; ++j) { C0[j] = pack2(g0[2 * j], g0[2 * j + 1]); C1[j] = pack2(g1[2 * j], g1[2 * j + 1]); }
      } else {
        float4 cs[2], sn[2];
        if ((unsigned)pos < (unsigned)a.n_positions) {
          const float4* r = reinterpret_cast<const float4*>(a.rope + (long long)pos * a.rot_dim + c0 * 8);
          cs[0] = r[0]; cs[1] = r[1]; sn[0] = r[2 * half]; sn[1] = r[2 * half + 1];
        } else {
          cs[0] = cs[1] = sn[0] = sn[1] = make_float4(nan_f(), nan_f(), nan_f(), nan_f());
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x2 x = pack2(cs[j].x, cs[j].y), y = pack2(cs[j].z, cs[j].w), sx = pack2(sn[j].x, sn[j].y), sy = pack2(sn[j].z, sn[j].w);
          const f32x2 ga = pack2(g0[4 * j], g0[4 * j + 1]), gb = pack2(g0[4 * j + 2], g0[4 * j + 3]), ha = pack2(g1[4 * j], g1[4 * j + 1]), hb = pack2(g1[4 * j + 2], g1[4 * j + 3]);
          C0[2 * j] = mul2(ga, x); C0[2 * j + 1] = mul2(gb, y);
          C1[2 * j] = mul2(ha, x); C1[2 * j + 1] = mul2(hb, y);
          S0[2 * j] = mul2(ga, sx); S0[2 * j + 1] = mul2(gb, sy);
          S1[2 * j] = mul2(pack2(-g1[4 * j], -g1[4 * j + 1]), sx); S1[2 * j + 1] = mul2(pack2(-g1[4 * j + 2], -g1[4 * j + 3]), sy);
        }
      }
    }
    int h = (u - (kind == 0 ? 0 : kind == 1 ? uq : uk)) * kPer + sub;
    char* dst;
    long long dst_step;
    bool kept = true;
    if (kind == 0) {
      dst = a.yq + (row * a.yq_row + h * a.yq_head + c0 * 8) * (long long)sizeof(D);
      dst_step = step * kPer * a.yq_head * (long long)sizeof(D);
    } else if constexpr (kPaged) {
      // the element of the pools where this row's slot of head 0 begins
      const long long at = page * a.kv.page_stride + (long long)(pos & (a.kv.page_size - 1)) * a.kv.slot_stride;
      dst = (kind == 1 ? a.kv.k : a.kv.v) + (at + h * a.kv.head_stride + c0 * 8) * (long long)sizeof(D);
      dst_step = step * kPer * a.kv.head_stride * (long long)sizeof(D);
      kept = (unsigned)page < (unsigned)a.kv.n_pages;
      if (!kept && lane == 0) atomicOr(a.status, CS_DEV_BADARG);
    } else {
      dst = a.yk + (row * a.yk_row + h * a.yk_head + c0 * 8) * (long long)sizeof(D);
      dst_step = step * kPer * a.yk_head * (long long)sizeof(D);
    }
    for (; u < end; u += step) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kSlots - 2) : "memory");
      if constexpr (kWide) __syncwarp();
      uint32_t w[2][kW];
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        const int at = kWide ? (j < 2 ? c0 : c1) * 32 + j % 2 * 16 : j * 512;
        const uint4 v = *reinterpret_cast<const uint4*>(mine + place + at);
        uint32_t* d = &w[j / (kPieces / 2)][j % (kPieces / 2) * 4];
        d[0] = v.x; d[1] = v.y; d[2] = v.z; d[3] = v.w;
      }
      fetch((place + (kSlots - 1) * kSlotBytes) % (kSlots * kSlotBytes));      // (into the slot whose unit is done)
      place = (place + kSlotBytes) % (kSlots * kSlotBytes);
      f32x2 x0[4], x1[4];
      widen<S>(w[0], x0);
      widen<S>(w[1], x1);
      if (!plain) {
        if (norm) {
          f32x2 s2 = mul2(x0[0], x0[0]);
#pragma unroll
          for (int j = 1; j < 4; ++j) s2 = fma2(x0[j], x0[j], s2);
#pragma unroll
          for (int j = 0; j < 4; ++j) s2 = fma2(x1[j], x1[j], s2);
          float lo, hi;
          unpack2(s2, lo, hi);
          float sq = lo + hi;
#pragma unroll
          for (int o = 1; o < kLanes; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
          const float r = rsqrtf(sq * (1.f / DH) + a.eps);
          const f32x2 r2 = pack2(r, r);
#pragma unroll
          for (int j = 0; j < 4; ++j) { x0[j] = mul2(x0[j], r2); x1[j] = mul2(x1[j], r2); }
        }
        if (rotated) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x2 y0 = fma2(x0[j], C0[j], mul2(x1[j], S1[j]));
            x1[j] = fma2(x1[j], C1[j], mul2(x0[j], S0[j]));
            x0[j] = y0;
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) { x0[j] = mul2(x0[j], C0[j]); x1[j] = mul2(x1[j], C1[j]); }
        }
      }
      if (kept && h < n) {
        store8<D>(dst, x0);
        store8<D>(dst + (c1 - c0) * 8 * (int)sizeof(D), x1);
      }
      h += step * kPer; dst += dst_step;
    }
  }
}

__global__ void __launch_bounds__(kThreads)
k_rope_table(float* table, int n_positions, int rot_dim, double log_theta) {
  CS_PDL_PROLOGUE();
  const int h = rot_dim / 2;
  const long long n = (long long)n_positions * h;
  for (long long i = blockIdx.x * (long long)kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
    const long long p = i / h;
    const int j = (int)(i % h);
    double s, c;
    sincos((double)p * exp(-2.0 * j / rot_dim * log_theta), &s, &c);
    table[p * rot_dim + j] = (float)c;
    table[p * rot_dim + h + j] = (float)s;
  }
}

thread_local char t_paged_err[256] = "";

template <typename S, typename D, bool kPaged, int kBlock>
cudaError_t launch_heads_of(const HeadsArgs& a, int head_dim, cudaStream_t st) {
  const dim3 grid((unsigned)(((long long)a.n_rows * a.warps_per_row + kBlock - 1) / kBlock)), block(kBlock * 32);
  switch (head_dim) {
    case 32: return cs_launch_pdl(k_heads<S, D, 32, kPaged, kBlock>, grid, block, 0, st, a);
    case 64: return cs_launch_pdl(k_heads<S, D, 64, kPaged, kBlock>, grid, block, 0, st, a);
    default: return cs_launch_pdl(k_heads<S, D, 128, kPaged, kBlock>, grid, block, 0, st, a);
  }
}

template <typename S, typename D, bool kPaged>
cudaError_t launch_heads(HeadsArgs a, int rows, int head_dim, cudaStream_t st) {
  const int per = 512 / head_dim, units = cs_ceil_div(a.n_q, per) + cs_ceil_div(a.n_k, per) + cs_ceil_div(a.n_v, per);
  a.n_rows = rows;
  // As many warps a row as run at the same time on 148 SMs (two blocks of 8 warps, or five of 4, on each), each with a unit at least: what is worked out per row is worked out by each of its
  // warps.  Rows of the 8B shape, us with 8 / 4 / 2 / 1 warps: 256 3.6 / 3.9 / 4.1 / -, 350 6.0 / 4.3 / 4.8 / 5.5, 700 - / 4.7 / 5.6 / 6.5, 2,048 - / 12.9 / 11.2 / 10.2.
  a.warps_per_row = 8;
  while (a.warps_per_row > 1 && (a.warps_per_row >= 2 * units || (long long)rows * a.warps_per_row > 148 * (a.warps_per_row == 8 ? 16 : 20))) a.warps_per_row /= 2;
  return a.warps_per_row == 8 ? launch_heads_of<S, D, kPaged, 8>(a, head_dim, st) : launch_heads_of<S, D, kPaged, 4>(a, head_dim, st);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool known_dim(int d) { return d == 32 || d == 64 || d == 128; }
int bytes_of(int dtype) { return dtype == CS_F32 ? 4 : 2; }

// source (and, with `out` >= 0, destination) of a call's heads
cs_status check_heads(const cs_heads* h, int in, int out, bool gain) {
  if (h->n_heads < 0) return CS_ERR_ARG;
  if (h->n_heads == 0) return CS_OK;
  const int ui = 16 / bytes_of(in);
  if (h->x == nullptr || !aligned16(h->x) || h->row_stride % ui != 0 || h->head_stride % ui != 0) return CS_ERR_ARG;
  if (gain && !aligned16(h->gain)) return CS_ERR_ARG;
  if (out >= 0) {
    const int uo = 16 / bytes_of(out);
    if (h->y == nullptr || !aligned16(h->y) || h->y_row_stride % uo != 0 || h->y_head_stride % uo != 0) return CS_ERR_ARG;
  }
  return CS_OK;
}
cs_status check_rope(const float* rope, int n_positions, int rot_dim, int head_dim, float eps) {
  if (rot_dim < 0 || !(eps >= 0.f)) return CS_ERR_ARG;
  if (rot_dim == 0) return CS_OK;
  if (rope == nullptr || n_positions < 1 || !aligned16(rope)) return CS_ERR_ARG;
  return rot_dim % 16 != 0 || rot_dim > head_dim ? CS_ERR_SHAPE : CS_OK;
}
cs_status check_blocks(const cs_blocks* b) {
  if (b->n_seqs < 0 || b->rows < 0 || b->table_width < 0) return CS_ERR_ARG;
  if (b->n_seqs == 0 || b->rows == 0) return CS_OK;
  return b->start == nullptr || b->len == nullptr || b->kv_len == nullptr || (b->page_table == nullptr && b->table_width > 0) ? CS_ERR_ARG : CS_OK;
}
BlocksView view_of(const cs_blocks* b) { return BlocksView{b->start, b->len, b->kv_len, b->page_table, b->n_seqs, b->table_width, b->rows}; }

struct PagedLayout {
  size_t status, counters, splits, parts, parts_ml, total;
};
PagedLayout layout_of(const cs_paged_config& c) {
  PagedLayout l;
  size_t at = 0;
  auto put = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) & ~(size_t)255; return o; };
  l.status = put(256);
  l.counters = put(kPagedMaxCtas * sizeof(int));
  l.splits = put(kPagedMaxCtas * sizeof(PagedSplit));
  l.parts = put((size_t)kPagedMaxCtas * 2 * kPagedMaxRows * c.head_dim * 4);
  l.parts_ml = put((size_t)kPagedMaxCtas * 2 * kPagedMaxRows * 8);
  l.total = at;
  return l;
}
// why a configuration is refused (CS_OK: it is not)
cs_status check_config(const cs_paged_config* c, const char** why) {
  *why = "";
  if (c == nullptr) { *why = "NULL argument"; return CS_ERR_ARG; }
  if (!known_dim(c->head_dim)) { *why = "head_dim must be 32, 64 or 128"; return CS_ERR_SHAPE; }
  if (c->page_size < 16 || (c->page_size & (c->page_size - 1)) != 0) { *why = "page_size must be a power of two from 16 on"; return CS_ERR_SHAPE; }
  if (c->dtype != CS_BF16 && c->dtype != CS_F16) { *why = "a cache is CS_BF16 or CS_F16"; return CS_ERR_SHAPE; }
  if (c->n_pages < 1 || c->n_kv_heads < 1) { *why = "no pages or no heads"; return CS_ERR_ARG; }
  if (c->page_stride < 1 || c->head_stride < 1 || c->slot_stride < c->head_dim || c->page_stride % 8 != 0 || c->head_stride % 8 != 0 || c->slot_stride % 8 != 0) {
    *why = "strides must be positive multiples of 8 elements";
    return CS_ERR_ARG;
  }
  return CS_OK;
}

cs_status fail(cs_paged_cache* c, cs_status s, const char* text) {
  snprintf(c->err, sizeof(c->err), "%s", text);
  return s;
}

}  // namespace

cs_status cs_rope_table(float* table, int n_positions, int rot_dim, float theta, void* stream) {
  if (n_positions < 0 || rot_dim < 0 || rot_dim % 2 != 0 || !(theta > 0.f)) return CS_ERR_ARG;
  if (n_positions == 0 || rot_dim == 0) return CS_OK;
  if (table == nullptr) return CS_ERR_ARG;
  const long long n = (long long)n_positions * (rot_dim / 2), ctas = (n + kThreads - 1) / kThreads;
  return cs_launch_pdl(k_rope_table, dim3((unsigned)(ctas < 4096 ? ctas : 4096)), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), table, n_positions, rot_dim,
                       log((double)theta)) == cudaSuccess ? CS_OK : CS_ERR_CUDA;
}

cs_status cs_qk_norm_rope(const cs_heads* q, const cs_heads* k, int rows, int head_dim, cs_dtype in, cs_dtype out, const int32_t* pos,
                          const float* rope, int n_positions, int rot_dim, float eps, void* stream) {
  if (rows < 0 || in < CS_BF16 || in > CS_F32 || out < CS_BF16 || out > CS_F32 || (in != out && in != CS_F32)) return CS_ERR_ARG;
  if (!known_dim(head_dim)) return CS_ERR_SHAPE;
  if (rows == 0) return CS_OK;
  cs_status s = check_rope(rope, n_positions, rot_dim, head_dim, eps);
  if (s != CS_OK) return s;
  HeadsArgs a = {};
  if (q != nullptr) {
    if ((s = check_heads(q, in, out, true)) != CS_OK) return s;
    a.q = static_cast<const char*>(q->x); a.q_row = q->row_stride; a.q_head = q->head_stride;
    a.yq = static_cast<char*>(q->y); a.yq_row = q->y_row_stride; a.yq_head = q->y_head_stride;
    a.q_gain = static_cast<const char*>(q->gain); a.n_q = q->n_heads;
  }
  if (k != nullptr) {
    if ((s = check_heads(k, in, out, true)) != CS_OK) return s;
    a.k = static_cast<const char*>(k->x); a.k_row = k->row_stride; a.k_head = k->head_stride;
    a.yk = static_cast<char*>(k->y); a.yk_row = k->y_row_stride; a.yk_head = k->y_head_stride;
    a.k_gain = static_cast<const char*>(k->gain); a.n_k = k->n_heads;
  }
  if ((long long)a.n_q + a.n_k > 0x3fffffff) return CS_ERR_ARG;
  if (a.n_q + a.n_k == 0) return CS_OK;
  if (rot_dim > 0 && pos == nullptr) return CS_ERR_ARG;
  a.pos = pos; a.rope = rope; a.n_positions = n_positions; a.rot_dim = rot_dim; a.eps = eps;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (in == CS_BF16) e = launch_heads<__nv_bfloat16, __nv_bfloat16, false>(a, rows, head_dim, st);
  else if (in == CS_F16) e = launch_heads<__half, __half, false>(a, rows, head_dim, st);
  else if (out == CS_BF16) e = launch_heads<float, __nv_bfloat16, false>(a, rows, head_dim, st);
  else if (out == CS_F16) e = launch_heads<float, __half, false>(a, rows, head_dim, st);
  else e = launch_heads<float, float, false>(a, rows, head_dim, st);
  return e == cudaSuccess ? CS_OK : CS_ERR_CUDA;
}

size_t cs_paged_workspace_bytes(const cs_paged_config* cfg) {
  const char* why;
  return check_config(cfg, &why) == CS_OK ? layout_of(*cfg).total : 0;
}

namespace {
// `clear`: the workspace is nobody's yet
cs_status create(const char* name, cs_paged_cache** out, const cs_paged_config* cfg, void* workspace, size_t workspace_bytes, bool clear, void* stream) {
  auto refuse = [&](cs_status s, const char* text) {
    snprintf(t_paged_err, sizeof(t_paged_err), "%s: %s", name, text);
    return s;
  };
  t_paged_err[0] = 0;
  const char* why;
  if (out == nullptr) return refuse(CS_ERR_ARG, "NULL argument");
  *out = nullptr;
  const cs_status s = check_config(cfg, &why);
  if (s != CS_OK) return refuse(s, why);
  if (cfg->k == nullptr || cfg->v == nullptr || workspace == nullptr) return refuse(CS_ERR_ARG, "NULL pointer");
  if (!aligned16(cfg->k) || !aligned16(cfg->v)) return refuse(CS_ERR_ARG, "the pools must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(workspace) & 255) != 0) return refuse(CS_ERR_ARG, "the workspace must be 256-byte aligned");
  const PagedLayout l = layout_of(*cfg);
  if (workspace_bytes < l.total) return refuse(CS_ERR_CAPACITY, "the workspace is too small");
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return refuse(CS_ERR_CUDA, "no device");
  cs_paged_cache* c = static_cast<cs_paged_cache*>(aligned_alloc(64, (sizeof(cs_paged_cache) + 63) / 64 * 64));   // (operand maps: 64 bytes)
  if (c == nullptr) return refuse(CS_ERR_CAPACITY, "out of host memory");
  memset(c, 0, sizeof(*c));
  c->drop = -1;
  c->cfg = *cfg;
  c->num_sms = sms < kPagedMaxCtas ? sms : kPagedMaxCtas;
  int shift = 0;
  while ((1 << shift) < cfg->page_size) ++shift;
  c->view = PagedView{static_cast<char*>(cfg->k), static_cast<char*>(cfg->v), cfg->page_stride, cfg->head_stride, cfg->slot_stride, cfg->n_pages, cfg->page_size, shift, cfg->n_kv_heads};
  char* ws = static_cast<char*>(workspace);
  c->workspace = workspace;
  c->workspace_bytes = workspace_bytes;
  c->status = reinterpret_cast<int*>(ws + l.status);
  c->counters = reinterpret_cast<int*>(ws + l.counters);
  c->splits = reinterpret_cast<PagedSplit*>(ws + l.splits);
  c->parts = reinterpret_cast<float*>(ws + l.parts);
  c->parts_ml = reinterpret_cast<float*>(ws + l.parts_ml);
  const char* wl = getenv("CS_WAIT_LIMIT_US");
  const long long us = wl != nullptr ? atoll(wl) : 0;
  c->wait_limit_ns = us > 0 ? (unsigned long long)us * 1000ull : 2000000000ull;
  if (cs_paged_tc_maps(c) != CS_OK) {
    snprintf(t_paged_err, sizeof(t_paged_err), "%s: %.200s", name, c->err);
    free(c);
    return CS_ERR_CUDA;
  }
  const cudaError_t e = clear ? cudaMemsetAsync(ws, 0, l.parts, static_cast<cudaStream_t>(stream)) : cudaSuccess;
  if (e != cudaSuccess) {
    free(c);
    return refuse(CS_ERR_CUDA, cudaGetErrorString(e));
  }
  *out = c;
  return CS_OK;
}
}  // namespace

cs_status cs_paged_create(cs_paged_cache** out, const cs_paged_config* cfg, void* workspace, size_t workspace_bytes, void* stream) {
  return create("cs_paged_create", out, cfg, workspace, workspace_bytes, true, stream);
}

cs_status cs_paged_create_beside(cs_paged_cache** out, const cs_paged_config* cfg, const cs_paged_cache* first) {
  return create("cs_paged_create_beside", out, cfg, first != nullptr ? first->workspace : nullptr, first != nullptr ? first->workspace_bytes : 0, false, nullptr);
}

void cs_paged_destroy(cs_paged_cache* cache) { free(cache); }

int cs_paged_head_dim(const cs_paged_cache* cache) { return cache != nullptr ? cache->cfg.head_dim : 0; }

const char* cs_paged_last_error(const cs_paged_cache* cache) { return cache != nullptr ? cache->err : t_paged_err; }

cs_status cs_paged_status(cs_paged_cache* c, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int bits = 0;
  CS_CUDA_OK(c, cudaMemcpyAsync(&bits, c->status, sizeof(int), cudaMemcpyDeviceToHost, st));
  CS_CUDA_OK(c, cudaStreamSynchronize(st));
  if (bits == 0) return CS_OK;
  // (the counters too: a launch whose wait ran out may have left pieces uncounted)
  CS_CUDA_OK(c, cudaMemsetAsync(c->status, 0, sizeof(int), st));
  CS_CUDA_OK(c, cudaMemsetAsync(c->counters, 0, kPagedMaxCtas * sizeof(int), st));
  CS_CUDA_OK(c, cudaStreamSynchronize(st));
  if (bits & CS_DEV_TIMEOUT) return fail(c, CS_ERR_TIMEOUT, "a bounded wait ran out");
  if (bits & CS_DEV_SMEM) return fail(c, CS_ERR_CUDA, "a kernel found its shared memory too small");
  if (bits & CS_DEV_CAPACITY) return fail(c, CS_ERR_CAPACITY, "a block does not fit its row of the page table, or the rotation table is too short");
  return fail(c, CS_ERR_ARG, "a length is negative, rows lie outside the tensors, or a page does not exist");
}

cs_status cs_paged_debug_drop_tile(cs_paged_cache* c, int tile) {
  if (c == nullptr) return CS_ERR_ARG;
  c->drop = tile < 0 ? -1 : tile;
  return CS_OK;
}

cs_status cs_paged_append(cs_paged_cache* c, const cs_blocks* blocks, const cs_heads* k, const cs_heads* v, const cs_heads* q, cs_dtype in,
                          const float* rope, int n_positions, int rot_dim, float eps, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  if (blocks == nullptr || k == nullptr || v == nullptr) return fail(c, CS_ERR_ARG, "NULL argument");
  if (in != c->cfg.dtype && in != CS_F32) return fail(c, CS_ERR_ARG, "rows come in the cache's type or in CS_F32");
  cs_status s = check_blocks(blocks);
  if (s != CS_OK) return fail(c, s, "bad blocks");
  if (blocks->n_seqs == 0 || blocks->rows == 0) return CS_OK;
  s = check_rope(rope, n_positions, rot_dim, c->cfg.head_dim, eps);
  if (s != CS_OK) return fail(c, s, "bad rotation table, eps or rot_dim (a multiple of 16, at most head_dim)");
  if (k->n_heads != c->cfg.n_kv_heads || v->n_heads != c->cfg.n_kv_heads) return fail(c, CS_ERR_SHAPE, "keys and values need the cache's heads");
  if ((q != nullptr && (s = check_heads(q, in, c->cfg.dtype, true)) != CS_OK) || (s = check_heads(k, in, -1, true)) != CS_OK || (s = check_heads(v, in, -1, false)) != CS_OK)
    return fail(c, s, "rows need 16-byte aligned bases and strides of multiples of 16 bytes");
  if ((long long)(q != nullptr ? q->n_heads : 0) + 2ll * c->cfg.n_kv_heads > 0x3fffffff) return fail(c, CS_ERR_SHAPE, "too many heads");
  HeadsArgs a = {};
  if (q != nullptr) {
    a.q = static_cast<const char*>(q->x); a.q_row = q->row_stride; a.q_head = q->head_stride;
    a.yq = static_cast<char*>(q->y); a.yq_row = q->y_row_stride; a.yq_head = q->y_head_stride;
    a.q_gain = static_cast<const char*>(q->gain); a.n_q = q->n_heads;
  }
  a.k = static_cast<const char*>(k->x); a.k_row = k->row_stride; a.k_head = k->head_stride;
  a.k_gain = static_cast<const char*>(k->gain); a.n_k = k->n_heads;
  a.v = static_cast<const char*>(v->x); a.v_row = v->row_stride; a.v_head = v->head_stride; a.n_v = v->n_heads;
  a.rope = rope; a.n_positions = n_positions; a.rot_dim = rot_dim; a.eps = eps;
  a.kv = c->view; a.blk = view_of(blocks); a.status = c->status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int rows = blocks->rows, dh = c->cfg.head_dim;
  if (c->cfg.dtype == CS_BF16)
    CS_CUDA_OK(c, in == CS_F32 ? (launch_heads<float, __nv_bfloat16, true>(a, rows, dh, st)) : (launch_heads<__nv_bfloat16, __nv_bfloat16, true>(a, rows, dh, st)));
  else
    CS_CUDA_OK(c, in == CS_F32 ? (launch_heads<float, __half, true>(a, rows, dh, st)) : (launch_heads<__half, __half, true>(a, rows, dh, st)));
  return CS_OK;
}

cs_status cs_paged_attention(cs_paged_cache* c, const cs_blocks* blocks, const void* q, int64_t q_row_stride, int64_t q_head_stride, int n_heads, cs_mask mask,
                             int window, float scale, void* out, float* lse, void* stream) {
  if (c == nullptr) return CS_ERR_ARG;
  if (blocks == nullptr) return fail(c, CS_ERR_ARG, "NULL argument");
  const cs_status s = check_blocks(blocks);
  if (s != CS_OK) return fail(c, s, "bad blocks");
  if (mask < CS_MASK_CAUSAL || mask > CS_MASK_FULL || window < 0 || !(scale > 0.f) || !(scale <= 3.0e38f)) return fail(c, CS_ERR_ARG, "bad mask, window or scale");
  if (n_heads < 1 || n_heads % c->cfg.n_kv_heads != 0 || n_heads / c->cfg.n_kv_heads > 128) return fail(c, CS_ERR_SHAPE, "n_heads must be a multiple of the cache's heads, at most 128 per KV head");
  if ((long long)blocks->rows * n_heads > 0x7fffff00ll) return fail(c, CS_ERR_SHAPE, "too many rows");
  if (blocks->n_seqs == 0 || blocks->rows == 0) return CS_OK;
  if (q == nullptr || out == nullptr) return fail(c, CS_ERR_ARG, "NULL pointer");
  if (!aligned16(q) || !aligned16(out) || q_row_stride % 8 != 0 || q_head_stride % 8 != 0) return fail(c, CS_ERR_ARG, "q and out need 16-byte aligned bases, q strides of multiples of 8 elements");
  if ((reinterpret_cast<uintptr_t>(lse) & 3) != 0) return fail(c, CS_ERR_ARG, "lse must be aligned to its type");
  PagedAttnArgs a = {};
  a.kv = c->view; a.blk = view_of(blocks);
  a.q = static_cast<const char*>(q); a.q_row = q_row_stride; a.q_head = q_head_stride;
  a.out = static_cast<char*>(out); a.lse = lse;
  a.n_heads = n_heads; a.group = n_heads / c->cfg.n_kv_heads;
  a.by_group = PagedDivisor::by(a.group);
  a.mask = mask; a.window = window;
  a.scale = scale; a.scale_log2e = (float)(1.4426950408889634 * (double)scale);
  a.parts = c->parts; a.parts_ml = c->parts_ml; a.counters = c->counters; a.splits = c->splits; a.status = c->status;
  a.wait_ns = c->wait_limit_ns;
  a.drop = -1;
  // 16 query rows per KV head are a tile of the kernel for few rows, and the average is what the host knows: where blocks differ much, some are in the other kernel's hands, more slowly, and a row's weights
  // are rounded as the kernel of its call does it.  (On tensor cores / by it, us: 11 rows of the 8B shape over 1,024 keys 15.0 / 13.0, over 4,096 16.0 / 18.3, over 16,384 26.4 / 40.4; 16 x 5 over 1,024
  // 28.8 / 36.2.  By the first it would be the better one for short contexts with 44 rows too; how long they are stands on the device.)  Queries that repeat one row have no operand map
  const bool few = (long long)blocks->rows * a.group <= 16ll * blocks->n_seqs || (blocks->rows > 1 && q_row_stride <= 0) || (n_heads > 1 && q_head_stride <= 0);
  if (!few) {
    a.drop = c->drop;
    c->drop = -1;
  }
  for (int b = 0; b < blocks->n_seqs; b += kPagedMaxSeqs) {      // (a launch's plan holds so many)
    PagedAttnArgs p = a;
    p.blk.n_seqs = blocks->n_seqs - b < kPagedMaxSeqs ? blocks->n_seqs - b : kPagedMaxSeqs;
    p.blk.start += b; p.blk.len += b; p.blk.kv_len += b;
    p.blk.table += (long long)b * blocks->table_width;
    const cs_status r = few ? cs_launch_paged_few(c, p, static_cast<cudaStream_t>(stream)) : cs_launch_paged_tc(c, p, static_cast<cudaStream_t>(stream));
    if (r != CS_OK) return r;
  }
  return CS_OK;
}
