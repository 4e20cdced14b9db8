// The paged cache: what its kernels share.  A page holds page_size slots of every key head (or of one head); a
// sequence (or a head of a sequence) has a row of the page table and a length.  Slot s of head h of sequence b is
// row s % page_size of page table[b, h][s / page_size].
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ssd_device.cuh"
#include "ssd_internal.cuh"

namespace ssd {

// Bits of the cache's device status word: what a kernel met in device data and left out.
constexpr uint32_t kPagedBadPage = 1u;     // a page number outside the pool: the slot counts as masked, is not written
constexpr uint32_t kPagedBadLength = 2u;   // a length outside [0, capacity]: it is cut to that range
constexpr uint32_t kPagedBadScores = 4u;   // a slot behind the end of the score row: its weight is dropped

struct PagedView {
  char* k;                  // pages
  char* v;
  float* ks;                // row scales (8-bit rows), else null
  float* vs;
  const int32_t* table;
  int32_t* lens;
  float* scores;            // accumulated weights, or null
  uint32_t* status;         // or null
  long long page_b, head_b, slot_b;          // strides of the pages, bytes
  long long sc_page, sc_head, sc_slot;       // strides of the row scales, elements
  long long t_seq, t_head;                   // strides of the table
  long long n_seq, n_head;                   // strides of the lengths
  long long w_seq, w_head;                   // strides of the scores
  int n_seqs, H, page_size, page_shift;      // page_shift: log2(page_size), -1 where that is no power of two
  int n_pages, cap;                          // cap: slots that a table row can name
  int score_slots;
};

#if defined(__CUDACC__)
__device__ __forceinline__ void paged_flag(const PagedView& c, uint32_t bit) {
  if (c.status) atomicOr(c.status, bit);
}
__device__ __forceinline__ int paged_length(const PagedView& c, int seq, int head) {
  const int n = c.lens[seq * c.n_seq + head * c.n_head];
  if (n < 0 || n > c.cap) {
    paged_flag(c, kPagedBadLength);
    return n < 0 ? 0 : c.cap;
  }
  return n;
}
__device__ __forceinline__ void paged_split(const PagedView& c, int slot, int& index, int& row) {
  if (c.page_shift >= 0) {
    index = slot >> c.page_shift;
    row = slot & (c.page_size - 1);
  } else {
    index = (int)((uint32_t)slot / (uint32_t)c.page_size);
    row = slot - index * c.page_size;
  }
}
// Page and row of a slot in [0, cap); page -1 where the table names none of the pool.
__device__ __forceinline__ int paged_lookup(const PagedView& c, const int32_t* table, int slot, int& row) {
  int index;
  paged_split(c, slot, index, row);
  const int page = __ldg(table + index);
  if ((uint32_t)page < (uint32_t)c.n_pages) return page;
  paged_flag(c, kPagedBadPage);
  return -1;
}
__device__ __forceinline__ const int32_t* paged_table(const PagedView& c, int seq, int head) {
  return c.table + seq * c.t_seq + head * c.t_head;
}
__device__ __forceinline__ float* paged_scores(const PagedView& c, int seq, int head) {
  return c.scores + seq * c.w_seq + head * c.w_head;
}

// ------------------------------------------------------------------ 8-bit rows: scale = max|x| / 448, code = E4M3(x / scale)
__device__ __forceinline__ void widen8(const uint4& raw, bool bf16, float (&x)[8]) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 f;
    if (bf16) {
      f = widen2(w[i]);
    } else {
      __half2 h;
      memcpy(&h, &w[i], 4);
      f = __half22float2(h);
    }
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint32_t paged_e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}
// A row is held by kLanes consecutive lanes, 8 values each (16-bit, in raw): its codes, and its scale in all of them.
template <int kLanes>
__device__ __forceinline__ uint2 paged_quantize(const uint4& raw, bool bf16, float& scale) {
  float x[8], m = 0.f;
  widen8(raw, bf16, x);
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(x[i]));
#pragma unroll
  for (int o = kLanes / 2; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  scale = __fdiv_rn(m, 448.f);
  const float by = scale > 0.f ? scale : 1.f;
  uint32_t c[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] = paged_e4m3x2(__fdiv_rn(x[2 * i], by), __fdiv_rn(x[2 * i + 1], by));
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
#endif

// ------------------------------------------------------------------ attention of one new token
// n / d for n < 2^31 by a multiplication (the round-up method of Granlund and Montgomery, PLDI 1994: with s = ceil(log2 d)
// and m = floor(2^32 (2^s - d) / d) + 1, the quotient is (n + floor(m n / 2^32)) >> s)
struct FastDiv {
  uint32_t m, s;
#if defined(__CUDACC__)
  __device__ __forceinline__ uint32_t div(uint32_t n) const { return (n + __umulhi(n, m)) >> s; }
#endif
};
inline FastDiv fast_div(uint32_t d) {
  FastDiv f = {0u, 0u};
  while ((1ull << f.s) < d) ++f.s;
  f.m = (uint32_t)(((1ull << 32) * ((1ull << f.s) - d)) / d + 1u);
  return f;
}

struct PagedDecodeParams {
  PagedView c;
  const char* q;            // [n_seqs, H * g, D], strides in bytes
  long long q_seq, q_head;
  char* out;
  long long o_seq, o_head;
  const char* k_new;        // fused append: the rows of slot length - 1, [n_seqs, H, D]; else null
  const char* v_new;
  long long new_seq, new_head;
  float* lse;               // [n_seqs, H * g], or null
  float* logits;            // weights wanted: [n_seqs * H * g, logit_row]; else null
  float2* ml;               // weights wanted: [n_seqs * H * g] (max, sum)
  long long logit_row;
  uint32_t* counters;       // [workers], zero between launches
  float* partial;           // [workers][2][paged_part_floats(rows, D)]
  float scale_log2;
  int g, qt, rows;          // query heads per key head; groups of at most `rows` of them that one worker takes together
  FastDiv by_qt, by_heads;  // n / qt, n / H
  int whole_tiles;          // the page size is a multiple of the tile's slots
  int bf16;                 // type of q, out, k_new, v_new: 1 bf16, 0 fp16
};

enum { kPagedBf16 = 0, kPagedFp16 = 1, kPagedE4m3 = 2 };

// query heads that one pass over a key head's rows serves
inline int paged_rows(int g) { return g < 16 ? g : 16; }

// a state in memory: O [rows][D], m [rows], l [rows], whole float4s
#if defined(__CUDACC__)
__host__ __device__
#endif
inline int paged_part_floats(int rows, int head_dim) { return (rows * (head_dim + 2) + 3) / 4 * 4; }

cudaError_t launch_paged_decode_16(const PagedDecodeParams& p, int head_dim, int sms, cudaStream_t st);
cudaError_t launch_paged_decode_8(const PagedDecodeParams& p, int head_dim, int sms, cudaStream_t st);
cudaError_t launch_paged_weights(const PagedDecodeParams& p, cudaStream_t st);
size_t paged_max_workers(int sms);

}  // namespace ssd
