// The paged key/value cache as the kernels see it (kv_cache.hip, attend.hip).
#pragma once

#include "grinqh_internal.h"

namespace grinqh {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr long kMaxTokens = 1L << 30;   // of a sequence: token indices and a tile beyond them fit 32 bits

// A validated cache, passed to kernels by value.
struct KvCache {
  char* k;
  char* v;
  float* ks;        // scales, GRINQH_KV_I8 only
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
size_t attend_workspace(const KvCache& c, const Attend& a, int B, int rows);
int launch_attend(const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q, const DenseRows& out,
                  float* lse, void* workspace, hipStream_t s);

// The larger of each half, as unsigned numbers.
__device__ __forceinline__ uint32_t max_halves(uint32_t x, uint32_t y) {
  typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2v, x), __builtin_bit_cast(ushort2v, y)));
}

}  // namespace grinqh
