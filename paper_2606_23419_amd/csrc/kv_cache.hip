// Writing rows of K and V into the paged cache, and reading them back.
#include "kv.h"

namespace grinqh {

// Eight consecutive values, as they lie in memory.
template <int TYPE>
struct Eight { u32x4 w[TYPE == GRINQH_F32 ? 2 : 1]; };

template <int TYPE>
__device__ __forceinline__ Eight<TYPE> load8(const char* p) {
  Eight<TYPE> e;
  for (int i = 0; i < (TYPE == GRINQH_F32 ? 2 : 1); ++i) e.w[i] = *(const u32x4*)(p + 16 * i);
  return e;
}

template <int TYPE>
__device__ __forceinline__ float value(const Eight<TYPE>& e, int j) {
  if constexpr (TYPE == GRINQH_F32) return __builtin_bit_cast(float, (uint32_t)e.w[j >> 2][j & 3]);
  const uint16_t h = (uint16_t)(e.w[0][j >> 1] >> (16 * (j & 1)));
  return TYPE == GRINQH_F16 ? h2f(h) : bf2f(h);
}

// The largest magnitude of the values of the lanes that hold a row of 8 LPR channels: magnitudes are ordered as their
// bits are, with NaN above infinity.  Lanes exchange within fours, then mirrored within 8 and 16.
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true));
}

template <int TYPE, int LPR>
__device__ __forceinline__ float row_max(const Eight<TYPE>& e) {
  uint32_t m = 0;
  if constexpr (TYPE == GRINQH_F32) {
    for (int j = 0; j < 8; ++j) m = max(m, (uint32_t)e.w[j >> 2][j & 3] & 0x7fffffffu);
  } else {
    for (int j = 0; j < 4; ++j) m = max_halves(m, e.w[0][j] & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);
  }
  static_assert(LPR == 8 || LPR == 16);
  m = max_dpp<0xb1>(m);                      // quad_perm: the neighbour, then the other two
  m = max_dpp<0x4e>(m);
  m = max_dpp<0x141>(m);                     // row_half_mirror
  if constexpr (LPR == 16) m = max_dpp<0x140>(m);   // row_mirror
  return TYPE == GRINQH_F32 ? __builtin_bit_cast(float, m) : TYPE == GRINQH_F16 ? h2f((uint16_t)m) : bf2f((uint16_t)m);
}

// rne(fp32(x r)) as a code, |x r| <= 127: the low byte of the product added to 1.5 2^23, where the spacing is one.
__device__ __forceinline__ uint32_t code(float x, float r) {
#pragma clang fp contract(off)
  const float y = x * r;
  return __builtin_bit_cast(uint32_t, y + 12582912.0f);
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
// each of one head, and a thread has kItems such pieces in flight.  The rows' places are looked up once per row: in
// writing by a wave of its own, so that the chain of lookups (sequence, length, page) runs while the rows are loaded.
//
// Rounding (8 bits): a = max |x| of a row's head, scale = a / 127 and 127 / a in fp32, codes to nearest even.
// Bound by memory.  34642 tokens of 8 heads of 128, bf16 into 8 bits (216 MB): 51 us, 4.2 TB/s where a copy of 2 GiB reaches
// 4.9 (64 us with the places looked up by the loading waves, 59 with shuffles and conversions one value at a time); read
// back as bf16 40 us.  One 8-bit context of 131072 tokens as fp16 (814 MB): 167 .. 186 us.  A single token of 8 heads: 3.0 us
// written, 2.6 read, latency.
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
__global__ __launch_bounds__(kRowThreads + 64) void k_kv_write(KvCache c, KvBatch b, DenseRows k, DenseRows v, int tokens) {
  constexpr int LPR = D / 8, SIZE = TYPE == GRINQH_F32 ? 4 : 2;
  __shared__ long place[kRowThreads];
  const DenseRows& src = blockIdx.y ? v : k;
  char* dst = blockIdx.y ? c.v : c.k;
  float* scales = blockIdx.y ? c.vs : c.ks;
  const int r0 = blockIdx.x * tokens, left = min(tokens, b.rows - r0), items = tokens * c.H * LPR;
  const bool looks_up = threadIdx.x >= kRowThreads;
  if (looks_up)
    for (int t = threadIdx.x - kRowThreads; t < left; t += 64) place[t] = kv_place(c, b, r0 + t);
  for (int i0 = 0; i0 < items; i0 += kRowThreads * kItems) {
    Piece p[kItems];
    Eight<TYPE> x[kItems] = {};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      p[i] = piece_of<D>(c, i0 + i * kRowThreads + threadIdx.x, left);
      p[i].in &= !looks_up;
      if (p[i].in) x[i] = load8<TYPE>(src.p + ((long)(r0 + p[i].row) * src.row + p[i].head * src.head + p[i].lane * 8) * SIZE);
    }
    if (i0 == 0) __syncthreads();
    if (looks_up) return;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const long at = p[i].in ? place[p[i].row] : kNoSequence, slot = at + ((long)p[i].head << c.shift);
      if constexpr (FORMAT == GRINQH_KV_I8) {
        const float a = row_max<TYPE, LPR>(x[i]);
        float scale = 0, r127 = 0;
        if (a < INFINITY && a >= 0x1p-100f) { scale = a / 127.0f; r127 = 127.0f / a; }
        if (!(a < INFINITY)) scale = NAN;
        u32x2 w = {0, 0};
        if (r127 > 0)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t b[4];
            for (int k = 0; k < 4; ++k) b[k] = code(value<TYPE>(x[i], 4 * j + k), r127);
            w[j] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u), __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u), 0x05040100u);
          }
        if (at >= 0) {
          *(u32x2*)(dst + slot * D + p[i].lane * 8) = w;
          if (p[i].lane == 0) scales[slot] = scale;
        }
      } else if (at >= 0) {
        constexpr int HELD = FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16;
        char* to = dst + (slot * D + p[i].lane * 8) * 2;
        if constexpr (TYPE == HELD) {
          *(u32x4*)to = x[i].w[0];
        } else {
          float y[8];
          for (int j = 0; j < 8; ++j) y[j] = value<TYPE>(x[i], j);
          store8<HELD>(to, y);
        }
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
          constexpr int HELD = FORMAT == GRINQH_KV_F16 ? GRINQH_F16 : GRINQH_BF16;
          const Eight<HELD> e = load8<HELD>(src + (slot * D + p[i].lane * 8) * 2);
          for (int j = 0; j < 8; ++j) x[i][j] = value<HELD>(e, j);
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
  if (write) k_kv_write<D, FORMAT, TYPE><<<grid, kRowThreads + 64, 0, s>>>(c, b, k, v, tokens);
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
