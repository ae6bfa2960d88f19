// Writing rows of K and V into the paged cache, and reading them back.
#include "kv.h"

namespace grinqh {


// Eight consecutive values of a dense row.
template <int TYPE>
__device__ __forceinline__ void load8(const char* p, float* x) {
  if constexpr (TYPE == GRINQH_F32) {
    for (int i = 0; i < 2; ++i) {
      const u32x4 w = *(const u32x4*)(p + 16 * i);
      for (int j = 0; j < 4; ++j) x[4 * i + j] = __builtin_bit_cast(float, (uint32_t)w[j]);
    }
  } else {
    const u32x4 w = *(const u32x4*)p;
    for (int j = 0; j < 8; ++j) {
      const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
      x[j] = TYPE == GRINQH_F16 ? h2f(h) : bf2f(h);
    }
  }
}

template <int TYPE>
__device__ __forceinline__ void store8(char* p, const float* x) {
  if constexpr (TYPE == GRINQH_F32) {
    for (int i = 0; i < 2; ++i) {
      u32x4 w;
      for (int j = 0; j < 4; ++j) w[j] = __builtin_bit_cast(uint32_t, x[4 * i + j]);
      *(u32x4*)(p + 16 * i) = w;
    }
  } else {
    u32x4 w;
    for (int j = 0; j < 4; ++j) {
      const uint16_t lo = TYPE == GRINQH_F16 ? f2h_rn(x[2 * j]) : f2bf_rn(x[2 * j]);
      const uint16_t hi = TYPE == GRINQH_F16 ? f2h_rn(x[2 * j + 1]) : f2bf_rn(x[2 * j + 1]);
      w[j] = lo | (uint32_t)hi << 16;
    }
    *(u32x4*)p = w;
  }
}

// The sequence whose rows hold `row`: the last one that starts at or before it.
__device__ __forceinline__ int kv_find(const KvBatch& b, int row) {
  int lo = 0, hi = b.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (b.offs[mid] <= row) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// Position of a dense row and its page: pos < 0 for a row of no slot,
// page < 0 for a page id out of range.  False if no sequence has the row.
__device__ __forceinline__ bool kv_place(const KvCache& c, const KvBatch& b, int row, int* pos, int* page) {
  const int s = kv_find(b, row);
  const Seq q = kv_seq(c, b, s);
  if (row < q.r0 || row >= q.r0 + q.n) return false;
  *pos = q.L - q.n + (row - q.r0);
  *page = *pos >= 0 ? kv_page(c, b, s, *pos) : -1;
  return true;
}

constexpr int kRowThreads = 256;

// D / 8 lanes hold a row of a head; K in the first half of the grid's y, V in the second.
template <int D, int FORMAT, int TYPE>
__global__ void k_kv_write(KvCache c, KvBatch b, DenseRows k, DenseRows v) {
  constexpr int LPR = D / 8;
  const long r = ((long)blockIdx.x * kRowThreads + threadIdx.x) / LPR;
  const int lane = threadIdx.x % LPR;
  const bool in = r < (long)b.rows * c.H;
  const int row = in ? (int)(r / c.H) : 0, h = in ? (int)(r % c.H) : 0;
  const DenseRows& src = blockIdx.y ? v : k;
  float x[8] = {};
  if (in) load8<TYPE>(src.p + (row * src.row + h * src.head + lane * 8) * (TYPE == GRINQH_F32 ? 4 : 2), x);
  float scale = 0, r127 = 0;
  if constexpr (FORMAT == GRINQH_KV_I8) {
    float a = 0;
    bool bad = false;
    for (int i = 0; i < 8; ++i) {
      bad |= !(fabsf(x[i]) < INFINITY);
      a = fmaxf(a, fabsf(x[i]));
    }
    if (bad) a = INFINITY;
    for (int m = LPR / 2; m; m >>= 1) a = fmaxf(a, __shfl_xor(a, m, LPR));
    if (a < INFINITY && a >= 0x1p-100f) { scale = a / 127.0f; r127 = 127.0f / a; }
    if (!(a < INFINITY)) scale = NAN;
  }
  int pos, page;
  if (!in || !kv_place(c, b, row, &pos, &page) || page < 0) return;
  const long slot = kv_slot(c, page, h, pos);
  char* dst = blockIdx.y ? c.v : c.k;
  if constexpr (FORMAT == GRINQH_KV_I8) {
    u32x2 w = {0, 0};
    if (r127 > 0)
      for (int i = 0; i < 8; ++i) w[i / 4] |= (uint32_t)(uint8_t)(int)rintf(x[i] * r127) << (8 * (i & 3));
    *(u32x2*)(dst + slot * D + lane * 8) = w;
    if (lane == 0) (blockIdx.y ? c.vs : c.ks)[slot] = scale;
  } else {
    store8<FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16>(dst + (slot * D + lane * 8) * 2, x);
  }
}

template <int D, int FORMAT, int TYPE>
__global__ void k_kv_read(KvCache c, KvBatch b, DenseRows k, DenseRows v) {
  constexpr int LPR = D / 8;
  const long r = ((long)blockIdx.x * kRowThreads + threadIdx.x) / LPR;
  const int lane = threadIdx.x % LPR;
  if (r >= (long)b.rows * c.H) return;
  const int row = (int)(r / c.H), h = (int)(r % c.H);
  const DenseRows& dst = blockIdx.y ? v : k;
  int pos, page;
  if (!kv_place(c, b, row, &pos, &page)) return;
  float x[8];
  if (page < 0) {
    for (int i = 0; i < 8; ++i) x[i] = pos < 0 ? 0.0f : NAN;
  } else {
    const long slot = kv_slot(c, page, h, pos);
    const char* src = blockIdx.y ? c.v : c.k;
    if constexpr (FORMAT == GRINQH_KV_I8) {
      const u32x2 w = *(const u32x2*)(src + slot * D + lane * 8);
      const float scale = (blockIdx.y ? c.vs : c.ks)[slot];
      for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(w[i / 4] >> (8 * (i & 3))) * scale;
    } else {
      load8<FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16>(src + (slot * D + lane * 8) * 2, x);
    }
  }
  store8<TYPE>(dst.p + (row * dst.row + h * dst.head + lane * 8) * (TYPE == GRINQH_F32 ? 4 : 2), x);
}

template <int D, int FORMAT, int TYPE>
static void launch_rows(bool write, const KvCache& c, const KvBatch& b, const DenseRows& k, const DenseRows& v, hipStream_t s) {
  const long lanes = (long)b.rows * c.H * (D / 8);
  const dim3 grid((unsigned)((lanes + kRowThreads - 1) / kRowThreads), 2);
  if (write) k_kv_write<D, FORMAT, TYPE><<<grid, kRowThreads, 0, s>>>(c, b, k, v);
  else k_kv_read<D, FORMAT, TYPE><<<grid, kRowThreads, 0, s>>>(c, b, k, v);
}

static int dispatch_rows(bool write, const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v,
                         hipStream_t s) {
  if ((long)b.rows * c.H * (c.D / 8) / kRowThreads > 0x7ffffff0L)
    return fail(GRINQH_EUNSUPPORTED, "rows=%d of %d heads exceed one launch", b.rows, c.H);
  auto on_type = [&](auto d, auto format) {
    constexpr int D = decltype(d)::value, F = decltype(format)::value;
    if (type == GRINQH_F16) launch_rows<D, F, GRINQH_F16>(write, c, b, k, v, s);
    else if (type == GRINQH_BF16) launch_rows<D, F, GRINQH_BF16>(write, c, b, k, v, s);
    else launch_rows<D, F, GRINQH_F32>(write, c, b, k, v, s);
  };
  auto on_format = [&](auto d) {
    if (c.format == GRINQH_KV_F16) on_type(d, std::integral_constant<int, GRINQH_KV_F16>{});
    else if (c.format == GRINQH_KV_BF16) on_type(d, std::integral_constant<int, GRINQH_KV_BF16>{});
    else on_type(d, std::integral_constant<int, GRINQH_KV_I8>{});
  };
  if (c.D == 64) on_format(std::integral_constant<int, 64>{});
  else on_format(std::integral_constant<int, 128>{});
  return check_launch(write ? "kv_write" : "kv_read");
}

int launch_kv_write(const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v, hipStream_t s) {
  return dispatch_rows(true, c, b, type, k, v, s);
}

int launch_kv_read(const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v, hipStream_t s) {
  return dispatch_rows(false, c, b, type, k, v, s);
}

}  // namespace grinqh
