// Shared by the operators around the paged cache held in 4 bits: the handle, the format, what kernels get of a cache.
//
// A row (one position, one KV head) is cut into groups of 32 neighbouring elements.  With a = max |x| of a group,
//     s = a / 7 rounded to five significant bits,   n = x / s rounded to a whole number, |n| <= 7;
// the group is held as s (bf16) and 4-bit numbers n + 8, and stands for s n.  Five bits and three make eight, so every value that the cache stands for is exactly a bf16 number: reading back in bf16 is
// exact, and keys and values go into the tensor cores as they are held, without a further rounding, in the kernel for few rows whatever the queries' type, in tall blocks of bf16 queries.  (Tall blocks of fp16 queries have them
// in fp16, which ends at 65504 and has steps of 2^-24 below 2^-14.)  Scales below 2^-126 are multiples of 2^-133, where bf16 ends.  Rounding the scale (by 1/32 at most) makes
// x / s at most 7.22, so the largest element still is off by less than half a step, as all others.  A group with an element that is not finite has the scale NaN, and all of it reads as NaN.
//
// Eight elements make a word: 2i and 2i + 1 are its fields i and i + 4, field f begins at bit 4f, so that a mask takes neighbouring elements out as the two halves of a register.
// Pools: [page][KV head][slot] rows of words, and of scales; 4.5 bits an element.
#pragma once

#include <type_traits>

#include "cs_paged.cuh"

static constexpr int kQuantGroup = 32;
static constexpr int kQuantMaxSms = 160;
static constexpr int kQuantCtasPerSm = 4;      // of an attention launch, at most
static constexpr int kQuantMaxRows = 32;       // query rows of one work item at most
static constexpr int kQuantRowsPerSm = 64;     // query rows of the items that CTAs of an SM have at hand, at most
static constexpr int kQuantMaxSeqs = 128;      // sequences of one attention launch; more are further launches.  (The plan of 512 takes 17 KB of shared memory a CTA, which four of them on an SM have not got.  Ragged tokens over up
                                               // to 4,097 keys of the 8B shape: 128 of them 77 us, 256 in two pairs of launches 159.)
static constexpr int kQuantCopyPage = 128;     // slots of a page of the copies that prompts' chunks are worked out from; 64, 32 or 16 where sequences in whole pages would not fit

struct QuantView {
  uint32_t *k, *v;                   // words of eight elements
  unsigned short *ks, *vs;           // scales, bf16
  long long data_page, scale_page;   // from page to page, in words and in scales
  uint32_t data_units, scale_units;  // the same in 16 bytes
  int n_pages, page_size, page_shift, n_kv_heads;
};

struct cs_quant_cache {
  cs_quant_config cfg;
  QuantView view;
  void* workspace;
  size_t workspace_bytes;
  int* status;                 // device status word
  PagedSplit* splits;          // of the last launch of few rows, by CTA
  float* parts;                // un-normalised pieces [CTA][2][query rows of an item][head_dim]
  float* parts_ml;             // their (reference point, sum)
  int num_sms;
  unsigned attr_set;           // shared-memory opt-ins made, a bit per kernel instance
  // copies in 16 bits of the positions that a call of prompts' chunks attends to
  long long tall_positions;    // room asked for, a multiple of 16; 0: none
  char *tall_k, *tall_v;       // [page][KV head][slot][head_dim]
  int *tall_table, *tall_len;  // 0, 1, 2, ...; lengths of the blocks that nothing is wrong with
  cs_paged_cache* tall[2][4];  // over the copies, by the queries' type (CS_BF16, CS_F16) and the size of a page (128 >> i); tall blocks without copies have their sums in the last one's workspace
  int drop;                    // test hook: K tile that the next call of tall blocks leaves out; -1: none
  char err[256];
};

// what an attention launch of few rows is about: what cs_paged.cuh deals work out by (pools left out), and the cache
struct QuantAttnArgs {
  PagedAttnArgs p;
  QuantView kv;
  int half;                    // queries and results are fp16 (else bf16)
};

cs_status cs_launch_quant_few(cs_quant_cache* c, const QuantAttnArgs& a, long long rows, cudaStream_t st);   // `rows`: query rows of a KV head, on the average of the call's sequences

#ifdef __CUDACC__
namespace {

__device__ __forceinline__ uint32_t bf2_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t bf2_sub(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t h2_mul(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
// (a & b) | c in one instruction
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}

// The scales of a register's two halves, and what the conversion makes of them once.
struct QuantScale {
  uint32_t s, c;               // s, -24 s: both exact in bf16, where it ends as well (a multiple of 2^-133 stays one)
  __device__ __forceinline__ static QuantScale of(uint32_t pair) { return QuantScale{pair, bf2_mul(pair, 0xc1c0c1c0u)}; }
};
// Two 16-bit halves of four fields u = n + 8 each -> field i of both, times their scales: exact.  A field at bits 3 - 6 under the exponent of 16 reads 16 + u, and one product and sum make s (u - 8) of it.
// (Without a shift, at bits 0 - 3 under the exponent of 128, the first field takes a difference and a product, and two more constants: as many instructions, and registers that heads of 128 have not got.  64 ragged tokens
// 42.4 us, so 41.4.)
__device__ __forceinline__ void quant_expand(uint32_t w, const QuantScale& q, uint32_t (&r)[4]) {
  r[0] = bf2_fma(and_or(w << 3, 0x00780078u, 0x41804180u), q.s, q.c);
  r[1] = bf2_fma(and_or(w >> 1, 0x00780078u, 0x41804180u), q.s, q.c);
  r[2] = bf2_fma(and_or(w >> 5, 0x00780078u, 0x41804180u), q.s, q.c);
  r[3] = bf2_fma(and_or(w >> 9, 0x00780078u, 0x41804180u), q.s, q.c);
}

// Eight fields u = n + 8 of a word -> whole numbers n in type T: field i and i + 4 as the halves of register i.  (bf16 has room for a field at bits 0 - 3 under the exponent of 128, fp16 at bits 0 - 3 under that of 1024 and at
// 4 - 7 under that of 64.)
template <typename T>
__device__ __forceinline__ void expand_numbers(uint32_t w, uint32_t (&r)[4]) {
  if constexpr (std::is_same<T, __half>::value) {
    const uint32_t v = w >> 8;
    r[0] = h2_sub(and_or(w, 0x000f000fu, 0x64006400u), 0x64086408u);
    r[1] = h2_sub(and_or(w, 0x00f000f0u, 0x54005400u), 0x54805480u);
    r[2] = h2_sub(and_or(v, 0x000f000fu, 0x64006400u), 0x64086408u);
    r[3] = h2_sub(and_or(v, 0x00f000f0u, 0x54005400u), 0x54805480u);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = bf2_sub(and_or(w >> (4 * i), 0x000f000fu, 0x43004300u), 0x43084308u);
  }
}

// is a scale not finite, or so far beyond the format's 2^123 that what it is expanded with (24 s) is not?
__device__ __forceinline__ bool quant_odd(unsigned scale) { return (scale & 0x7fffu) > 0x7d2au; }

}  // namespace
#endif
