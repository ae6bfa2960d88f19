// The paged key/value cache and the plan of a step as the kernels see them (kv_cache.hip, kv_plan.hip, the attend files).
#pragma once

#include "grinqh_internal.h"

namespace grinqh {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));

constexpr long kMaxTokens = 1L << 30;   // of a sequence: token indices and a tile beyond them fit 32 bits

// A validated cache, passed to kernels by value.
struct KvCache {
  char* k;
  char* v;
  float* ks;        // scales, GRINQH_KV_I8; GRINQH_KV_I4: a word per group, step below base
  float* vs;
  int format, H, D;
  int shift;        // tokens per page = 1 << shift
  int n_pages;
};

// A validated batch, passed to kernels by value.
struct KvBatch {
  const int* table;
  const int* lens;
  const int* offs;
  int B, width, rows;
};

// Dense rows, strides in elements.
struct DenseRows {
  char* p;
  long row, head;
};

// A validated plan, passed to kernels by value.
struct KvPlan {
  int* free_pages;
  int* n_free;
  int capacity, B, width, rows, shift, n_pages;
  const int* new_rows;
  int* table;
  int* lens;
  int* offs;
  int* positions;
  long* slots;
  int* granted;
  int* space;       // the workspace: four words (the list's pages first), then two arrays [B], which kv_plan.hip describes
};

struct Attend {
  int heads, G;     // query heads, and those that share a kv head
  int type;
  float scale;
  int window, sinks;
  int max_rows, max_len;
};

// One sequence: rows r0 .. r0 + n - 1 are its last n tokens of L.  The device
// arrays are clamped so that no value in them leads outside the buffers.
struct Seq {
  int r0, n, L;
};

__device__ __forceinline__ int kv_capacity(const KvCache& c, const KvBatch& b) {
  const long cap = (long)b.width << c.shift;
  return cap < kMaxTokens ? (int)cap : (int)kMaxTokens;
}

__device__ __forceinline__ Seq kv_seq(const KvCache& c, const KvBatch& b, int s) {
  Seq q;
  q.r0 = min(max(b.offs[s], 0), b.rows);
  q.n = min(max(b.offs[s + 1], q.r0), b.rows) - q.r0;
  q.L = min(max(b.lens[s], 0), kv_capacity(c, b));
  return q;
}

// The page of token t (0 <= t < capacity), -1 if its id is out of range.
__device__ __forceinline__ int kv_page(const KvCache& c, const KvBatch& b, int s, int t) {
  const int id = b.table[(long)s * b.width + (t >> c.shift)];
  return (unsigned)id < (unsigned)c.n_pages ? id : -1;
}

// Index of (page, head, token) among the cache's rows of head_dim values.
__device__ __forceinline__ long kv_slot(const KvCache& c, int page, int h, int t) {
  return (((long)page * c.H + h) << c.shift) + (t & ((1 << c.shift) - 1));
}

__device__ __forceinline__ float bf2f(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }
// round to nearest even; a NaN keeps its sign and becomes quiet
__device__ __forceinline__ uint16_t f2bf_rn(float f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, f);
  if (!(fabsf(f) <= INFINITY)) return (uint16_t)((u >> 16) | 0x40u);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

int launch_kv_write(const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v, hipStream_t s);
int launch_kv_read(const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v, hipStream_t s);
size_t plan_workspace(int B);
int launch_kv_plan(const KvPlan& p, hipStream_t s);
size_t attend_workspace(const KvCache& c, const Attend& a, int B, int rows);
int launch_attend(const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q, const DenseRows& out,
                  float* lse, void* workspace, hipStream_t s);

// GRINQH_KV_I4: channels that share a step and a base, and the largest magnitude of a group that is not NaN.
constexpr int kKvGroup = 32;
constexpr float kKvLargest = 0x1p15f;

// The masks and the exponents of nibbles() in registers: an instruction that takes both at once takes them from there alone.
struct Nibbles { uint32_t low, high, exponents; };
__device__ __forceinline__ Nibbles nibble_masks() {
  Nibbles n = {0x000f000fu, 0x00f000f0u, 0x64006400u};
  asm("" : "+s"(n.low), "+s"(n.high), "+v"(n.exponents));
  return n;
}

// The codes at bits 4 I .. 4 I + 3 of w's halves as fp16, exact: beside 0x64 a nibble reads as 1024 + code, or 1024 + 16 code.
template <int I>
__device__ __forceinline__ half2 nibbles(uint32_t w, const Nibbles& in) {
  const uint32_t x = I & 2 ? w >> 8 : w;
  if constexpr (I & 1) {
    const half2 by = {(_Float16)0.0625f, (_Float16)0.0625f}, off = {(_Float16)-64.0f, (_Float16)-64.0f};
    return __builtin_elementwise_fma(__builtin_bit_cast(half2, (x & in.high) | in.exponents), by, off);
  } else {
    const half2 off = {(_Float16)1024.0f, (_Float16)1024.0f};
    return __builtin_bit_cast(half2, (x & in.low) | in.exponents) - off;
  }
}

// The 8 channels of a word of GRINQH_KV_I4 as fp16: code * step + base, rounded once.
__device__ __forceinline__ u32x4 values8(uint32_t w, uint32_t group, const Nibbles& in) {
  const half2 g = __builtin_bit_cast(half2, group), step = {g[0], g[0]}, base = {g[1], g[1]};
  return u32x4{__builtin_bit_cast(uint32_t, __builtin_elementwise_fma(nibbles<0>(w, in), step, base)),
               __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(nibbles<1>(w, in), step, base)),
               __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(nibbles<2>(w, in), step, base)),
               __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(nibbles<3>(w, in), step, base))};
}

// The larger of each half, as unsigned numbers.
__device__ __forceinline__ uint32_t max_halves(uint32_t x, uint32_t y) {
  typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, x), __builtin_bit_cast(ushort2v, y)));
}

}  // namespace grinqh
