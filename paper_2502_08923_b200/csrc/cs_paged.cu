// Norms and rotation of queries and keys, rows appended to a paged KV cache, and the host side of the paged cache.
//
// For a row at position p and a head x of D elements, h = rot_dim / 2, c_i = cos(p w_i), s_i = sin(p w_i) from a table:
//     u = x rsqrt(mean(x^2) + eps) gain,   y_i = u_i c_i - u_{i+h} s_i,   y_{i+h} = u_{i+h} c_i + u_i s_i   (i < h).
// A lane holds eight neighbouring elements (16 bytes of the 16-bit types), a head is D / 8 lanes.  An element's partner is h away, so it lies in the
// same place of another lane of the head: one exchange of the raw words.  With A = gain_i c_i and B = -/+ gain_{partner} s_i the rest is
// y = r (x A + partner B), r the head's reciprocal norm (a reduction over its lanes).
//
// One CTA per row, all of its heads (queries, keys, values) in one go with the loads of up to four heads per lane in flight: bound by HBM
// where there are many rows, by launch and two dependent loads (whose block is the row's, which page) where there are few.
#include "cs_paged.cuh"

namespace {

constexpr int kThreads = 256, kUnroll = 4;

// what k_heads does with a row
struct HeadsArgs {
  const char *q, *k, *v;             // sources; head counts 0 = left out
  char *yq, *yk;                     // destinations of rows (yk: unless they go to pages)
  long long q_row, q_head, k_row, k_head, v_row, v_head, yq_row, yq_head, yk_row, yk_head;   // elements
  const char *q_gain, *k_gain;
  int n_q, n_k, n_v;
  const int* pos;                    // positions of rows, unless blocks give them
  const float* rope;
  int n_positions, rot_dim;
  float eps;
  PagedView kv;
  BlocksView blk;
  int* status;
};

template <typename T> __device__ __forceinline__ void load8(const char* p, uint32_t (&w)[sizeof(T) == 4 ? 8 : 4]) {
  const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p));
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  if constexpr (sizeof(T) == 4) {
    const uint4 b = __ldcg(reinterpret_cast<const uint4*>(p) + 1);
    w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}
template <typename T, int N> __device__ __forceinline__ void widen(const uint32_t (&w)[N], float (&f)[8]) {
  if constexpr (N == 8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = PagedType<T>::unpack(w[i]);
      f[2 * i] = x.x; f[2 * i + 1] = x.y;
    }
  }
}
template <typename T> __device__ __forceinline__ void store8(char* p, const float (&f)[8]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    *reinterpret_cast<uint4*>(p) = make_uint4(PagedType<T>::pack(f[0], f[1]), PagedType<T>::pack(f[2], f[3]), PagedType<T>::pack(f[4], f[5]), PagedType<T>::pack(f[6], f[7]));
  }
}
// eight gains; without any, ones
template <typename T> __device__ __forceinline__ void gain8(const char* g, int chunk, float (&f)[8]) {
  if (g == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 1.f;
  } else {
    uint32_t w[sizeof(T) == 4 ? 8 : 4];
    load8<T>(g + (long long)chunk * 8 * sizeof(T), w);
    widen<T>(w, f);
  }
}

template <typename S, typename D, int DH, bool kPaged>
__global__ void __launch_bounds__(kThreads)
k_heads(HeadsArgs a) {
  CS_PDL_PROLOGUE();
  constexpr int kLanes = DH / 8, kGroups = kThreads / kLanes, kW = sizeof(S) == 4 ? 8 : 4;
  __shared__ int s_seq;
  const int tid = threadIdx.x, grp = tid / kLanes, c = tid % kLanes;
  const long long row = blockIdx.x;
  const int n_heads = a.n_q + a.n_k + a.n_v;

  uint32_t w[kUnroll][kW];
  auto source = [&](int h) -> const char* {
    if (h < a.n_q) return a.q + (row * a.q_row + h * a.q_head) * (long long)sizeof(S) + c * 8 * sizeof(S);
    h -= a.n_q;
    if (h < a.n_k) return a.k + (row * a.k_row + h * a.k_head) * (long long)sizeof(S) + c * 8 * sizeof(S);
    h -= a.n_k;
    return a.v + (row * a.v_row + h * a.v_head) * (long long)sizeof(S) + c * 8 * sizeof(S);
  };
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      const int h = h0 + i * kGroups;
      if (h < n_heads) load8<S>(source(h), w[i]);
    }
  };
  load(grp);                                     // (whose row it is takes two loads in a row: these are under way meanwhile)

  int pos;
  long long at = 0;                              // element of the pools where slot (page, head 0) of this row begins
  bool stored = true;
  if constexpr (kPaged) {
    // the block this row belongs to
    if (tid == 0) s_seq = -1;
    __syncthreads();
    for (int b = tid; b < a.blk.n_seqs; b += kThreads) {
      const int start = __ldcg(a.blk.start + b), len = __ldcg(a.blk.len + b);
      if (row >= start && row - start < len) s_seq = b;
    }
    if (row == 0)                                // one CTA reports blocks that are left out
      for (int b = tid; b < a.blk.n_seqs; b += kThreads) {
        PagedBlock k;
        paged_block(a.blk, a.kv.page_size, b, true, k, a.status);
      }
    __syncthreads();
    const int b = s_seq;
    if (b < 0) return;
    PagedBlock k;
    if (!paged_block(a.blk, a.kv.page_size, b, true, k, a.status)) return;
    pos = k.kv + (int)(row - k.start);
    const int page = __ldcg(a.blk.table + (long long)b * a.blk.table_width + (pos >> a.kv.page_shift));
    if ((unsigned)page >= (unsigned)a.kv.n_pages) {
      stored = false;
      if (tid == 0) atomicOr(a.status, CS_DEV_BADARG);
    } else {
      at = page * a.kv.page_stride + (long long)(pos & (a.kv.page_size - 1)) * a.kv.slot_stride;
    }
    if (a.rot_dim > 0 && pos >= a.n_positions) {
      if (tid == 0) atomicOr(a.status, CS_DEV_CAPACITY);
      return;
    }
  } else {
    pos = a.rot_dim > 0 ? __ldcg(a.pos + row) : 0;
  }

  // rotation factors of this lane's elements; its partner's lane; what a chunk that is not rotated has: y = r x gain
  const int half = a.rot_dim >> 4;               // chunks of h elements
  const int pc = c < half ? c + half : c < 2 * half ? c - half : c;
  float cs[8], sn[8];
  if (pc == c) {
#pragma unroll
    for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  } else if ((unsigned)pos >= (unsigned)a.n_positions) {
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = sn[i] = __int_as_float(0x7fc00000);
  } else {
    const float* r = a.rope + (long long)pos * a.rot_dim + (c < half ? c : c - half) * 8;
    const float sign = c < half ? -1.f : 1.f;
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(r + i)), y = __ldcg(reinterpret_cast<const float4*>(r + 8 * half + i));
      cs[i] = x.x; cs[i + 1] = x.y; cs[i + 2] = x.z; cs[i + 3] = x.w;
      sn[i] = sign * y.x; sn[i + 1] = sign * y.y; sn[i + 2] = sign * y.z; sn[i + 3] = sign * y.w;
    }
  }
  const int lane = tid & 31, partner = (lane & ~(kLanes - 1)) | pc;

  for (int h0 = grp; h0 - grp < n_heads; h0 += kUnroll * kGroups) {
    if (h0 != grp) load(h0);
#pragma unroll
    for (int i = 0; i < kUnroll; ++i) {
      if (h0 - grp + i * kGroups >= n_heads) break;          // (the same in the whole CTA)
      const int h = h0 + i * kGroups;
      const bool is_v = h >= a.n_q + a.n_k, is_q = h < a.n_q, live = h < n_heads;
      float x[8], y[8], p[8];
      uint32_t pw[kW];
#pragma unroll
      for (int j = 0; j < kW; ++j) {
        if (!live) w[i][j] = 0u;
        pw[j] = __shfl_sync(0xffffffffu, w[i][j], partner);
      }
      widen<S>(w[i], x);
      widen<S>(pw, p);
      const char* gain = is_v ? nullptr : is_q ? a.q_gain : a.k_gain;
      float sq = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sq = fmaf(x[j], x[j], sq);
#pragma unroll
      for (int o = 1; o < kLanes; o <<= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
      if (!live) continue;
      if (is_v) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[j];
      } else {
        const float r = gain != nullptr ? 1.f / sqrtf(sq * (1.f / DH) + a.eps) : 1.f;
        float g[8], gp[8];
        gain8<D>(gain, c, g);
        gain8<D>(gain, pc, gp);
        // (a chunk that is not rotated takes no part of its "partner", or infinities would make NaN of it)
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = pc == c ? x[j] * r * g[j] : fmaf(x[j] * r * g[j], cs[j], p[j] * r * gp[j] * sn[j]);
      }
      if (is_q) {
        store8<D>(a.yq + (row * a.yq_row + h * a.yq_head + c * 8) * (long long)sizeof(D), y);
      } else if constexpr (kPaged) {
        if (stored) {
          const long long e = at + (long long)(is_v ? h - a.n_q - a.n_k : h - a.n_q) * a.kv.head_stride + c * 8;
          store8<D>((is_v ? a.kv.v : a.kv.k) + e * (long long)sizeof(D), y);
        }
      } else {
        store8<D>(a.yk + (row * a.yk_row + (h - a.n_q) * a.yk_head + c * 8) * (long long)sizeof(D), y);
      }
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

template <typename S, typename D, bool kPaged>
cudaError_t launch_heads(const HeadsArgs& a, int rows, int head_dim, cudaStream_t st) {
  switch (head_dim) {
    case 32: return cs_launch_pdl(k_heads<S, D, 32, kPaged>, dim3(rows), dim3(kThreads), 0, st, a);
    case 64: return cs_launch_pdl(k_heads<S, D, 64, kPaged>, dim3(rows), dim3(kThreads), 0, st, a);
    default: return cs_launch_pdl(k_heads<S, D, 128, kPaged>, dim3(rows), dim3(kThreads), 0, st, a);
  }
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
  size_t status, counters, parts, parts_ml, total;
};
PagedLayout layout_of(const cs_paged_config& c) {
  PagedLayout l;
  size_t at = 0;
  auto put = [&](size_t bytes) { const size_t o = at; at += (bytes + 255) & ~(size_t)255; return o; };
  l.status = put(256);
  l.counters = put(kPagedMaxCtas * sizeof(int));
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

cs_status cs_paged_create(cs_paged_cache** out, const cs_paged_config* cfg, void* workspace, size_t workspace_bytes, void* stream) {
  auto refuse = [](cs_status s, const char* text) {
    snprintf(t_paged_err, sizeof(t_paged_err), "cs_paged_create: %s", text);
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
  cs_paged_cache* c = static_cast<cs_paged_cache*>(calloc(1, sizeof(cs_paged_cache)));
  if (c == nullptr) return refuse(CS_ERR_CAPACITY, "out of host memory");
  c->cfg = *cfg;
  c->num_sms = sms < kPagedMaxCtas ? sms : kPagedMaxCtas;
  int shift = 0;
  while ((1 << shift) < cfg->page_size) ++shift;
  c->view = PagedView{static_cast<char*>(cfg->k), static_cast<char*>(cfg->v), cfg->page_stride, cfg->head_stride, cfg->slot_stride, cfg->n_pages, cfg->page_size, shift, cfg->n_kv_heads};
  char* ws = static_cast<char*>(workspace);
  c->status = reinterpret_cast<int*>(ws + l.status);
  c->counters = reinterpret_cast<int*>(ws + l.counters);
  c->parts = reinterpret_cast<float*>(ws + l.parts);
  c->parts_ml = reinterpret_cast<float*>(ws + l.parts_ml);
  const char* wl = getenv("CS_WAIT_LIMIT_US");
  const long long us = wl != nullptr ? atoll(wl) : 0;
  c->wait_limit_ns = us > 0 ? (unsigned long long)us * 1000ull : 2000000000ull;
  const cudaError_t e = cudaMemsetAsync(ws, 0, l.parts, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) {
    free(c);
    return refuse(CS_ERR_CUDA, cudaGetErrorString(e));
  }
  *out = c;
  return CS_OK;
}

void cs_paged_destroy(cs_paged_cache* cache) { free(cache); }

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
  a.mask = mask; a.window = window;
  a.scale = scale; a.scale_log2e = (float)(1.4426950408889634 * (double)scale);
  a.parts = c->parts; a.parts_ml = c->parts_ml; a.counters = c->counters; a.status = c->status;
  a.wait_ns = c->wait_limit_ns;
  for (int b = 0; b < blocks->n_seqs; b += kPagedMaxSeqs) {      // (a launch's plan holds so many)
    PagedAttnArgs p = a;
    p.blk.n_seqs = blocks->n_seqs - b < kPagedMaxSeqs ? blocks->n_seqs - b : kPagedMaxSeqs;
    p.blk.start += b; p.blk.len += b; p.blk.kv_len += b;
    p.blk.table += (long long)b * blocks->table_width;
    const cs_status r = cs_launch_paged_few(c, p, static_cast<cudaStream_t>(stream));
    if (r != CS_OK) return r;
  }
  return CS_OK;
}
