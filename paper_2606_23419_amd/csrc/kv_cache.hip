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

// Where a dense row's token lies: its slot among the rows of head 0, or what keeps it from having one.
constexpr long kNoSequence = -1, kNoToken = -2, kNoPage = -3;

__device__ __forceinline__ long kv_place(const KvCache& c, const KvBatch& b, int row) {
  const int s = kv_find(b, row);
  const Seq q = kv_seq(c, b, s);
  if (row < q.r0 || row >= q.r0 + q.n) return kNoSequence;
  const int pos = q.L - q.n + (row - q.r0);
  if (pos < 0) return kNoToken;
  const int page = kv_page(c, b, s, pos);
  return page < 0 ? kNoPage : kv_slot(c, page, 0, pos);
}

// A workgroup takes `tokens` rows of K (grid y = 0) or V (1), all heads of each: D / 8 lanes hold 8 channels
// each of one head, and a thread has kItems such pieces in flight.  The rows' places are looked up once per
// row, while what does not depend on them is loaded.
constexpr int kRowThreads = 256;
constexpr int kItems = 4;

struct Piece {
  int row, head, lane;   // row counted from the workgroup's first; lane = piece of 8 channels
  bool in;
};

template <int D>
__device__ __forceinline__ Piece piece_of(const KvCache& c, int item, int left) {
  constexpr int LPR = D / 8;
  Piece p;
  const int hl = item / LPR;
  p.row = hl / c.H;
  p.head = hl - p.row * c.H;
  p.lane = item % LPR;
  p.in = p.row < left;
  return p;
}

template <int D, int FORMAT, int TYPE>
__global__ __launch_bounds__(kRowThreads) void k_kv_write(KvCache c, KvBatch b, DenseRows k, DenseRows v, int tokens) {
  constexpr int LPR = D / 8, SIZE = TYPE == GRINQH_F32 ? 4 : 2;
  __shared__ long place[kRowThreads];
  const DenseRows& src = blockIdx.y ? v : k;
  char* dst = blockIdx.y ? c.v : c.k;
  float* scales = blockIdx.y ? c.vs : c.ks;
  const int r0 = blockIdx.x * tokens, left = min(tokens, b.rows - r0), items = tokens * c.H * LPR;
  for (int i0 = 0; i0 < items; i0 += kRowThreads * kItems) {
    Piece p[kItems];
    float x[kItems][8] = {};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      p[i] = piece_of<D>(c, i0 + i * kRowThreads + threadIdx.x, left);
      if (p[i].in) load8<TYPE>(src.p + ((long)(r0 + p[i].row) * src.row + p[i].head * src.head + p[i].lane * 8) * SIZE, x[i]);
    }
    if (i0 == 0) {
      if ((int)threadIdx.x < left) place[threadIdx.x] = kv_place(c, b, r0 + threadIdx.x);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const long at = p[i].in ? place[p[i].row] : kNoSequence, slot = at + ((long)p[i].head << c.shift);
      if constexpr (FORMAT == GRINQH_KV_I8) {
        float a = 0, scale = 0, r127 = 0;
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          bad |= !(fabsf(x[i][j]) < INFINITY);
          a = fmaxf(a, fabsf(x[i][j]));
        }
        if (bad) a = INFINITY;
#pragma unroll
        for (int m = LPR / 2; m; m >>= 1) a = fmaxf(a, __shfl_xor(a, m, LPR));
        if (a < INFINITY && a >= 0x1p-100f) { scale = a / 127.0f; r127 = 127.0f / a; }
        if (!(a < INFINITY)) scale = NAN;
        u32x2 w = {0, 0};
        if (r127 > 0)
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j / 4] |= (uint32_t)(uint8_t)(int)rintf(x[i][j] * r127) << (8 * (j & 3));
        if (at >= 0) {
          *(u32x2*)(dst + slot * D + p[i].lane * 8) = w;
          if (p[i].lane == 0) scales[slot] = scale;
        }
      } else if (at >= 0) {
        store8<FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16>(dst + (slot * D + p[i].lane * 8) * 2, x[i]);
      }
    }
  }
}

template <int D, int FORMAT, int TYPE>
__global__ __launch_bounds__(kRowThreads) void k_kv_read(KvCache c, KvBatch b, DenseRows k, DenseRows v, int tokens) {
  constexpr int LPR = D / 8, SIZE = TYPE == GRINQH_F32 ? 4 : 2;
  __shared__ long place[kRowThreads];
  const DenseRows& dst = blockIdx.y ? v : k;
  const char* src = blockIdx.y ? c.v : c.k;
  const float* scales = blockIdx.y ? c.vs : c.ks;
  const int r0 = blockIdx.x * tokens, left = min(tokens, b.rows - r0), items = tokens * c.H * LPR;
  if ((int)threadIdx.x < left) place[threadIdx.x] = kv_place(c, b, r0 + threadIdx.x);
  __syncthreads();
  for (int i0 = 0; i0 < items; i0 += kRowThreads * kItems) {
    Piece p[kItems];
    long at[kItems];
    u32x2 codes[kItems];
    float scale[kItems], x[kItems][8];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      p[i] = piece_of<D>(c, i0 + i * kRowThreads + threadIdx.x, left);
      at[i] = p[i].in ? place[p[i].row] : kNoSequence;
      const long slot = at[i] + ((long)p[i].head << c.shift);
      if (at[i] >= 0) {
        if constexpr (FORMAT == GRINQH_KV_I8) {
          codes[i] = *(const u32x2*)(src + slot * D + p[i].lane * 8);
          scale[i] = scales[slot];
        } else {
          load8<FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16>(src + (slot * D + p[i].lane * 8) * 2, x[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (at[i] == kNoSequence) continue;
      if (at[i] < 0) {
        for (int j = 0; j < 8; ++j) x[i][j] = at[i] == kNoToken ? 0.0f : NAN;
      } else if constexpr (FORMAT == GRINQH_KV_I8) {
        for (int j = 0; j < 8; ++j) x[i][j] = (float)(int8_t)(codes[i][j / 4] >> (8 * (j & 3))) * scale[i];
      }
      store8<TYPE>(dst.p + ((long)(r0 + p[i].row) * dst.row + p[i].head * dst.head + p[i].lane * 8) * SIZE, x[i]);
    }
  }
}

template <int D, int FORMAT, int TYPE>
static void launch_rows(bool write, const KvCache& c, const KvBatch& b, const DenseRows& k, const DenseRows& v, hipStream_t s) {
  // one pass of kItems pieces per thread where a row's heads allow it
  const int per_pass = kRowThreads * kItems / (c.H * (D / 8)), tokens = per_pass < 1 ? 1 : per_pass < kRowThreads ? per_pass : kRowThreads;
  const dim3 grid((unsigned)((b.rows + tokens - 1) / tokens), 2);
  if (write) k_kv_write<D, FORMAT, TYPE><<<grid, kRowThreads, 0, s>>>(c, b, k, v, tokens);
  else k_kv_read<D, FORMAT, TYPE><<<grid, kRowThreads, 0, s>>>(c, b, k, v, tokens);
}

static int dispatch_rows(bool write, const KvCache& c, const KvBatch& b, int type, const DenseRows& k, const DenseRows& v,
                         hipStream_t s) {
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
