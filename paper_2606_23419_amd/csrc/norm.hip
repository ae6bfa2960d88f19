// Between the blocks of a layer: a block's output is normed, gated and added to the scaled residual stream, and the sum's norm
// is what the next block reads.
//   a = post(y),  h' = residual_scale h + gate a,  x = pre(h')
//   RMS    v / sqrt(sum v^2 / n + eps) w + b
//   LAYER  (v - m) / sqrt(sum (v - m)^2 / n + eps) w + b,  m = sum v / n
// A row stays in registers from its loads to its stores, so every input is read once.  Sums are fp32: of a lane's values, then
// of the wave's lanes, then of the waves.  How many there are follows the channels alone, so a row's bits do not depend on the others.
//
// Bound by memory: 8192 rows of 4096, both norms and a gate (336 MB), 71 us; 1777 rows of 5001, two means, a gate per row, 39 us
// (34 where the last-level cache holds them), where rows that start at odd elements and the barriers of four sums cost; one row 3.9 us,
// latency.
#include <cmath>

#include "kv.h"

namespace grinqh {

namespace {

constexpr int kMaxChannels = 32768;          // 16 waves of 4 pieces a lane: what the registers of a workgroup hold

// Sixteen bytes of a row, whose rows may start at any element.
typedef u32x4 u32x4u __attribute__((aligned(2)));

struct Norm {
  int rows, n;
  int post, pre;
  int y_type, h_type, x_type, gate_type, weight_type;
  float scale, eps;
  const char *y, *h, *gate;
  char *h_out, *x;
  long y_stride, h_stride, gate_stride, h_out_stride, x_stride;
  const char *post_weight, *post_bias, *weight, *bias;
};

__device__ __forceinline__ int type_size(int type) { return type == GRINQH_F32 ? 4 : 2; }

// Eight values as they lie in memory.
struct Raw { u32x4 w[2]; };

// This lane's pieces of a row: piece v is channels 8 (v LANES + lane) .. + 7.
template <int NV>
struct Pieces { Raw r[NV]; };

template <int LANES, int NV>
__device__ __forceinline__ Pieces<NV> load_row(const char* p, int type, int lane, int n) {
  Pieces<NV> out;
#pragma unroll
  for (int v = 0; v < NV; ++v) out.r[v].w[0] = out.r[v].w[1] = u32x4{0, 0, 0, 0};
  if (type == GRINQH_F32) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int at = 8 * (v * LANES + lane);
      if (at + 8 <= n) {
        out.r[v].w[0] = *(const u32x4u*)(p + 4L * at);
        out.r[v].w[1] = *(const u32x4u*)(p + 4L * at + 16);
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (at + j < n) out.r[v].w[j >> 2][j & 3] = ((const uint32_t*)p)[at + j];
      }
    }
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int at = 8 * (v * LANES + lane);
      if (at + 8 <= n) {
        out.r[v].w[0] = *(const u32x4u*)(p + 2L * at);
      } else {
#pragma unroll
        for (int j = 0; j < 7; ++j)
          if (at + j < n) out.r[v].w[0][j >> 1] |= (uint32_t)((const uint16_t*)p)[at + j] << (16 * (j & 1));
      }
    }
  }
  return out;
}

template <int NV>
__device__ __forceinline__ void to_float(const Pieces<NV>& in, int type, float (*to)[8]) {
  if (type == GRINQH_F32) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) to[v][j] = __builtin_bit_cast(float, (uint32_t)in.r[v].w[j >> 2][j & 3]);
  } else if (type == GRINQH_F16) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) to[v][j] = h2f((uint16_t)(in.r[v].w[0][j >> 1] >> (16 * (j & 1))));
  } else {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int j = 0; j < 8; ++j) to[v][j] = bf2f((uint16_t)(in.r[v].w[0][j >> 1] >> (16 * (j & 1))));
  }
}

template <int LANES, int NV>
__device__ __forceinline__ void store_row(char* p, int type, int lane, int n, const float (*from)[8]) {
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int at = 8 * (v * LANES + lane);
    Raw r;
    if (type == GRINQH_F32) {
#pragma unroll
      for (int j = 0; j < 8; ++j) r.w[j >> 2][j & 3] = __builtin_bit_cast(uint32_t, from[v][j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float lo = from[v][2 * j], hi = from[v][2 * j + 1];
        r.w[0][j] = type == GRINQH_F16 ? f2h_rn(lo) | (uint32_t)f2h_rn(hi) << 16 : f2bf_rn(lo) | (uint32_t)f2bf_rn(hi) << 16;
      }
    }
    if (at + 8 <= n) {
      if (type == GRINQH_F32) {
        *(u32x4u*)(p + 4L * at) = r.w[0];
        *(u32x4u*)(p + 4L * at + 16) = r.w[1];
      } else {
        *(u32x4u*)(p + 2L * at) = r.w[0];
      }
    } else {
#pragma unroll
      for (int j = 0; j < 7; ++j)
        if (at + j < n) {
          if (type == GRINQH_F32) ((uint32_t*)p)[at + j] = r.w[j >> 2][j & 3];
          else ((uint16_t*)p)[at + j] = (uint16_t)(r.w[0][j >> 1] >> (16 * (j & 1)));
        }
    }
  }
}

// Sum (or maximum) over the lanes of a row.
template <int WAVES, bool MAX>
__device__ __forceinline__ float row_reduce(float x, float* lds) {
#pragma unroll
  for (int s = 32; s; s >>= 1) {
    const float y = __shfl_xor(x, s);
    x = MAX ? fmaxf(x, y) : x + y;
  }
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                         // the last reduction has been read
    if ((threadIdx.x & 63) == 0) lds[wave] = x;
    __syncthreads();
    x = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) x = MAX ? fmaxf(x, lds[w]) : x + lds[w];
  }
  return x;
}
template <int CTRL>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// The waves' two sums come back one to a lane, which meet in the order of a tree.
template <int WAVES>
__device__ __forceinline__ void row_sums(float* x, float* y, float* lds) {
#pragma unroll
  for (int s = 32; s; s >>= 1) { *x += __shfl_xor(*x, s); *y += __shfl_xor(*y, s); }
  if constexpr (WAVES > 1) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();                         // the last reduction has been read
    if ((threadIdx.x & 63) == 0) { lds[2 * wave] = *x; lds[2 * wave + 1] = *y; }
    __syncthreads();
    static_assert(WAVES == 4 || WAVES == 8 || WAVES == 16);
    auto meet = [](float v) {
      v = add_dpp<0x4e>(add_dpp<0xb1>(v));   // quad_perm: the neighbour, then the other two
      if constexpr (WAVES >= 8) v = add_dpp<0x141>(v);    // row_half_mirror
      if constexpr (WAVES == 16) v = add_dpp<0x140>(v);   // row_mirror
      return v;
    };
    const int from = 2 * (threadIdx.x & (WAVES - 1));
    *x = meet(lds[from]);
    *y = meet(lds[from + 1]);
  }
}

// v becomes its norm, weight and bias not yet applied.  Channels from n on are 0 and stay out of the sums.
// LAYER takes its mean off in two parts: the sum's, m, which is off by its roundings, and the mean r of what that leaves, so the variance
// is mean((v - m)^2) - r^2.  With the first alone a row of one value would be 1 or -1 throughout wherever m is not that value.  Of equal
// values v - m is exact and so is the sum of a few units in the last place; r is a quotient, not a product with 1 / n, so nothing
// is left.  Where r is no small part of what is left, the centred squares are summed once more.
template <int LANES, int NV, int WAVES>
__device__ __forceinline__ void normalise(int kind, float eps, int n, int lane, float (*v)[8], float* lds) {
  const float inv_n = 1.0f / n;
  float mean, rest, factor;
  // f(t) of the channels' t = v - mean - less, 0 from n on.  (Behind the assembly nothing that another pass made is kept: registers
  // are scarce.)
  auto centred = [&](float less, auto f) __attribute__((always_inline)) {
    int here = n - 8 * lane;
    float m = mean;
    asm volatile("" : "+v"(here), "+v"(m));
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) f(v[i][j], 8 * i * LANES + j < here ? v[i][j] - m - less : 0.0f);
  };
  auto spread = [&]() __attribute__((always_inline)) {
    float s = 0;
    mean = rest = 0;
    if (kind != GRINQH_NORM_LAYER) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[i][j] * v[i][j];
      return row_reduce<WAVES, false>(s, lds) * inv_n;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[i][j];
    mean = row_reduce<WAVES, false>(s, lds) * inv_n;
    float left = 0;
    s = 0;
    centred(0.0f, [&](float, float t) { left += t; s += t * t; });
    row_sums<WAVES>(&left, &s, lds);
    rest = left / n;
    const float square = s * inv_n;
    if (!(rest * rest > square * 0x1p-6f)) return square - rest * rest;
    s = 0;
    centred(rest, [&](float, float t) { s += t * t; });
    return row_reduce<WAVES, false>(s, lds) * inv_n;
  };
  const float var = spread() + eps;
  if (var >= 0x1p-100f && var < INFINITY) {
    factor = 1.0f / sqrtf(var);
  } else {
    // squares, or sums, that have left fp32's range, in either direction: the row times a power of two that brings its largest
    // magnitude to 1..2, or eps times the power's square, which is under the root then, to under 2^127 (where it outweighs all squares)
    float top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(v[i][j]));
    top = row_reduce<WAVES, true>(top, lds);
    int e = top > 0 && top < INFINITY ? min(-ilogbf(top), 126) : 0;
    if (eps > 0) e = min(e, (126 - ilogbf(eps)) >> 1);
    const float up = ldexpf(1.0f, e);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= up;
    const float root = spread() + ldexpf(eps, 2 * e);
    factor = root == 0 && eps > 0 ? 0.0f : 1.0f / sqrtf(root);   // one value, whose eps is lost here: zeros times anything finite
  }
  centred(rest, [&](float& to, float t) { to = t * factor; });
}

template <int LANES, int NV>
__device__ __forceinline__ void scale_and_shift(const char* weight, const char* bias, int type, int lane, int n, float (*v)[8]) {
  if (weight) {
    float w[NV][8];
    to_float<NV>(load_row<LANES, NV>(weight, type, lane, n), type, w);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= w[i][j];
  }
  if (bias) {
    float w[NV][8];
    to_float<NV>(load_row<LANES, NV>(bias, type, lane, n), type, w);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += w[i][j];
  }
}

// WAVES waves take a row, NV pieces of 8 channels a lane; with one wave a row a workgroup takes four.  With eight waves a SIMD, whose 64
// registers suffice without scratch, rows of 5001 take 0.82 to 0.92 of the time that seven take and 16384 channels 0.93.
template <int WAVES, int NV>
__global__ __launch_bounds__(WAVES == 1 ? 256 : 64 * WAVES) __attribute__((amdgpu_waves_per_eu(NV <= 2 ? 8 : 4))) void k_norm(Norm a) {
  constexpr int LANES = 64 * WAVES;
  __shared__ float lds[2 * WAVES];
  const int lane = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
  const long block = (long)blockIdx.y * gridDim.x + blockIdx.x, row = WAVES == 1 ? block * 4 + (threadIdx.x >> 6) : block;
  if (row >= a.rows) return;
  float v[NV][8];
  Pieces<NV> ry, rh;
  if (a.y) ry = load_row<LANES, NV>(a.y + row * a.y_stride * type_size(a.y_type), a.y_type, lane, a.n);
  if (a.h) rh = load_row<LANES, NV>(a.h + row * a.h_stride * type_size(a.h_type), a.h_type, lane, a.n);
  if (a.y) {
    to_float<NV>(ry, a.y_type, v);
    if (a.post != GRINQH_NORM_NONE) {
      normalise<LANES, NV, WAVES>(a.post, a.eps, a.n, lane, v, lds);
      scale_and_shift<LANES, NV>(a.post_weight, a.post_bias, a.weight_type, lane, a.n, v);
    }
    if (a.gate) scale_and_shift<LANES, NV>(a.gate + row * a.gate_stride * type_size(a.gate_type), nullptr, a.gate_type, lane, a.n, v);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = 0;
  }
  if (a.h) {
    float h[NV][8];
    to_float<NV>(rh, a.h_type, h);
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = fmaf(a.scale, h[i][j], v[i][j]);
  }
  if (a.h_out) store_row<LANES, NV>(a.h_out + row * a.h_out_stride * type_size(a.h_type), a.h_type, lane, a.n, v);
  if (a.x) {
    normalise<LANES, NV, WAVES>(a.pre, a.eps, a.n, lane, v, lds);
    scale_and_shift<LANES, NV>(a.weight, a.bias, a.weight_type, lane, a.n, v);
    store_row<LANES, NV>(a.x + row * a.x_stride * type_size(a.x_type), a.x_type, lane, a.n, v);
  }
}

// Fused sum and norm in fp16, us of 8192 rows: 512 channels by one wave 9, by four 21; 1024 by one 15, by four 21; 2048 by four 25, by
// one of four pieces 28; 4096 by four 43, by eight of one piece 46, by two of four 45; 8192 by eight 98, by sixteen of one piece 103.  (Of
// one row 4096 by four 4.7, by eight 4.2.)
void launch_norm(const Norm& a, hipStream_t s) {
  const int pieces = (a.n + 7) / 8;
  auto go = [&](auto waves, auto nv) {
    constexpr int W = decltype(waves)::value, NV = decltype(nv)::value;
    // an axis of the grid has less than 2^32 threads: 2^20 workgroups and less, and the rest along the other one
    const int threads = W == 1 ? 256 : 64 * W, blocks = W == 1 ? (a.rows + 3) / 4 : a.rows;
    const int y = (blocks + (1 << 20) - 1) >> 20, x = (blocks + y - 1) / y;
    k_norm<W, NV><<<dim3(x, y), threads, 0, s>>>(a);
  };
  using std::integral_constant;
  if (pieces <= 64) go(integral_constant<int, 1>{}, integral_constant<int, 1>{});
  else if (pieces <= 128) go(integral_constant<int, 1>{}, integral_constant<int, 2>{});
  else if (pieces <= 256) go(integral_constant<int, 4>{}, integral_constant<int, 1>{});
  else if (pieces <= 512) go(integral_constant<int, 4>{}, integral_constant<int, 2>{});
  else if (pieces <= 1024) go(integral_constant<int, 8>{}, integral_constant<int, 2>{});
  else if (pieces <= 2048) go(integral_constant<int, 16>{}, integral_constant<int, 2>{});
  else go(integral_constant<int, 16>{}, integral_constant<int, 4>{});
}

}  // namespace

}  // namespace grinqh

using namespace grinqh;

extern "C" int grinqh_norm(const grinqh_norm_desc* d, const grinqh_norm_arrays* p, void* stream) {
  clear_error();
  if (!d || !p) return fail(GRINQH_EINVAL, "desc and arrays must not be NULL");
  if (d->rows < 0 || d->rows > (1 << 24)) return fail(GRINQH_EINVAL, "rows=%d outside 0..2^24", d->rows);
  if (d->n < 1) return fail(GRINQH_EINVAL, "n=%d must be positive", d->n);
  if (d->n > kMaxChannels) return fail(GRINQH_EUNSUPPORTED, "n=%d: at most %d channels are implemented", d->n, kMaxChannels);
  for (int kind : {d->post, d->pre})
    if (kind < GRINQH_NORM_NONE || kind > GRINQH_NORM_LAYER) return fail(GRINQH_EINVAL, "%d is not a known norm", kind);
  for (int type : {d->y_type, d->h_type, d->x_type, d->gate_type, d->weight_type})
    if (type < GRINQH_F16 || type > GRINQH_F32) return fail(GRINQH_EINVAL, "type=%d is not a known type", type);
  if (!std::isfinite(d->residual_scale)) return fail(GRINQH_EINVAL, "residual_scale must be finite");
  if (!(d->eps >= 0) || !std::isfinite(d->eps)) return fail(GRINQH_EINVAL, "eps must be finite and not negative");
  if (!d->rows) return GRINQH_OK;            // whatever the arrays are: those of no elements have no address
  if (!p->y && !p->h) return fail(GRINQH_EINVAL, "y and h are both NULL");
  if (!p->h_out && !p->x) return fail(GRINQH_EINVAL, "h_out and x are both NULL");
  if ((d->pre != GRINQH_NORM_NONE) != (p->x != nullptr)) return fail(GRINQH_EINVAL, "x is the pre norm's output: both or neither");
  if (d->post == GRINQH_NORM_NONE && (p->post_weight || p->post_bias)) return fail(GRINQH_EINVAL, "post_weight and post_bias without a post norm");
  if (d->pre == GRINQH_NORM_NONE && (p->weight || p->bias)) return fail(GRINQH_EINVAL, "weight and bias without a pre norm");
  if (!p->y && (d->post != GRINQH_NORM_NONE || p->gate)) return fail(GRINQH_EINVAL, "a post norm or a gate without y");
  struct { const char* name; const void* at; int64_t stride; int type; bool written, row; } const rows[] = {
      {"y", p->y, p->y_stride, d->y_type, false, true},       {"h", p->h, p->h_stride, d->h_type, false, true},
      {"gate", p->gate, p->gate_stride, d->gate_type, false, true}, {"h_out", p->h_out, p->h_out_stride, d->h_type, true, true},
      {"x", p->x, p->x_stride, d->x_type, true, true},         {"post_weight", p->post_weight, 0, d->weight_type, false, false},
      {"post_bias", p->post_bias, 0, d->weight_type, false, false}, {"weight", p->weight, 0, d->weight_type, false, false},
      {"bias", p->bias, 0, d->weight_type, false, false}};
  for (const auto& r : rows) {
    if (!r.at) continue;
    if ((uintptr_t)r.at & (r.type == GRINQH_F32 ? 3u : 1u)) return fail(GRINQH_EINVAL, "%s must be aligned to its elements", r.name);
    if (!r.row || d->rows < 2) continue;     // the stride of an axis of one entry says nothing
    if ((r.stride < d->n && (r.written || r.stride)) || r.stride > (int64_t)1 << 36)
      return fail(GRINQH_EINVAL, "%s: the stride of rows is outside %d..2^36", r.name, d->n);
  }
  const Norm a = {d->rows, d->n, d->post, d->pre, d->y_type, d->h_type, d->x_type, d->gate_type, d->weight_type,
                  d->residual_scale, d->eps, (const char*)p->y, (const char*)p->h, (const char*)p->gate, (char*)p->h_out, (char*)p->x,
                  p->y_stride, p->h_stride, p->gate_stride, p->h_out_stride, p->x_stride, (const char*)p->post_weight,
                  (const char*)p->post_bias, (const char*)p->weight, (const char*)p->bias};
  launch_norm(a, (hipStream_t)stream);
  return check_launch("norm");
}
