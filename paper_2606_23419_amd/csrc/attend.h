// What the attention kernels share (attend.hip, attend_rows.hip, attend_tile.hip).
#pragma once

#include "kv.h"

namespace grinqh {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half2 __attribute__((ext_vector_type(2)));
typedef __bf16 bhalf8 __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf2 __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));
// Four scales, whose arrays are 4-byte aligned (such a load needs no more).
typedef float float4s __attribute__((ext_vector_type(4), aligned(4)));

// Results of the splits of a block of rows that has more than one (Span::splits): o [split][row * heads + head][D],
// normalised, and lse (base 2) [split][row * heads + head]; o is not written where lse is -inf.
struct Partial {
  float* o;
  float* lse;
  long rows;        // rows * heads
};

// How a call is launched (attend.hip).
struct AttendPlan {
  bool tile;        // k_attend_tile, else k_attend_rows
  int nb;           // k_attend_rows: blocks of 16 rows per wave
  int rows_log2;    // rows of a block: 16 or 32, and 256
  int blocks;       // row blocks of the longest sequence, as far as the caller's estimate goes
  int splits;       // parts of a sequence's tiles, and tiles per part (the last takes the rest)
  int per_split;
};

// A load known to be from device memory: through a pointer that may point to more than one array the
// compiler would use a flat load, which every wait for LDS would wait for as well.
template <typename T>
__device__ __forceinline__ T load_global(const void* p) {
  return *(const __attribute__((address_space(1))) T*)p;
}

// Between a wave's writes to LDS and its reads of them.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The attention kernels' argument.  What only the start or the end of a kernel needs is read there (late()):
// held in scalar registers throughout, it would push other values out of them.
struct AttendArgs {
  KvCache c;
  KvBatch b;
  Attend a;
  int splits, per_split;
  DenseRows q, out;
  float* lse;
  Partial part;
};

__device__ __forceinline__ const AttendArgs& late() {
  auto p = (const __attribute__((address_space(4))) AttendArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));   // keeps the loads where they are asked for
  return *(const AttendArgs*)p;
}

// Waves per workgroup of k_attend_rows, and per SIMD: of one block of 16 rows three (8-bit) or two workgroups of
// four waves share a CU, so that one's start and end overlap with the others' loads.  One token over 131072 tokens,
// 8 bits, whole call: 60 us, with workgroups of 8, 12 and 16 waves 59 .. 93; 32 sequences up to 8191 tokens 67 .. 75
// and 75 .. 130 (over the numbers of parts).
constexpr int rows_waves(int nb) { return nb == 1 ? 4 : 8; }
constexpr int rows_per_simd(int format, int nb) { return format == GRINQH_KV_I8 && nb == 1 ? 3 : 2; }

// What is read for tokens that are not there, a block of 16 rows each: zeros behind the last token, NaN for K of a page
// id out of range.  (A scale reads the first words.)
constexpr int kFill = 16 * 256 / 4;
static __device__ const uint32_t g_zeros[kFill] = {0};
#define NAN4 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff
#define NAN64 NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4, NAN4
static __device__ const uint32_t g_nans[kFill] = {NAN64, NAN64, NAN64, NAN64, NAN64, NAN64, NAN64, NAN64,
                                           NAN64, NAN64, NAN64, NAN64, NAN64, NAN64, NAN64, NAN64};
#undef NAN64
#undef NAN4

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// What a row's scores are held against follows their maximum once that has risen by kSlack powers of two, so weights stay under
// 2^6 of the maximum's and the sums are rescaled a few times instead of at every tile.  For an fp16 cache it stands kLift
// powers of two below the maximum: weights are at most 2^15 then, 11 bits of them stay down to 2^-23 of a row's largest, and what
// is below is off by at most 2^-34 of it.  (Held against the maximum itself, a long tail 17 nats below a first token would be
// rounded to nothing and stay in the sum that divides.)
template <int FORMAT>
constexpr float kLift = FORMAT == GRINQH_KV_F16 ? 9.0f : 0.0f;
template <int FORMAT>
constexpr float kSlack = 6.0f + kLift<FORMAT>;

// A score times its factor, rounded to fp32 whatever is done with it next.
__device__ __forceinline__ float rounded_product(float x, float factor) {
#pragma clang fp contract(off)
  return x * factor;
}
// From 2^22 on the spacing of fp32 is half a power of two and more.  exp2(fma(score, factor, -m)) would see the rest by which the
// largest product was rounded to m, and make that token's weight anything from nothing to infinity: the products of a row
// that is held against such an m, which is not lifted, are rounded first, as m was.  Its slack is -inf, so every tile takes the
// branch that does so.
__device__ __forceinline__ bool far_out(float m) { return fabsf(m) >= 0x1p22f && fabsf(m) < INFINITY; }
template <int FORMAT>
__device__ __forceinline__ float held_against(float mx) { return far_out(mx) ? mx : mx - kLift<FORMAT>; }
// 1 / factor for factors of 2^-124 and more (those of such rows are 2^-105 and more), to rcp's last bit; the instruction
// itself makes zero of a quotient under 2^-126.
__device__ __forceinline__ float inverse(float factor) { return __builtin_amdgcn_rcpf(0.25f * factor) * 0.25f; }

// The tiles of TK tokens that some of the rows at positions first .. last see: those of the sinks, then
// from the window's start on.
struct Span {
  int sink_tiles, lo_tile, tiles, hi;   // hi: tokens from here on are seen by no row
  __device__ __forceinline__ int tile(int v) const { return v < sink_tiles ? v : v - sink_tiles + lo_tile; }
  // how many of a call's `most` splits have tiles; a block of one writes its rows itself
  __device__ __forceinline__ int splits(int most, int per_split) const { return max(1, min(most, (tiles + per_split - 1) / per_split)); }
};

template <int TK>
__device__ __forceinline__ Span attend_span(const Attend& a, int first, int last) {
  Span s;
  s.hi = max(last + 1, 0);
  const int lo = a.window ? min(max(first - a.window + 1, 0), s.hi) : 0;
  s.lo_tile = lo / TK;
  s.sink_tiles = min((min(a.sinks, s.hi) + TK - 1) / TK, s.lo_tile);
  s.tiles = s.sink_tiles + (s.hi + TK - 1) / TK - s.lo_tile;
  return s;
}

// What a row at position pos sees: token t if t <= pos and t lies past behind_window or before the sinks' end.
__device__ __forceinline__ int behind_window(const Attend& a, int pos) { return a.window ? pos - a.window : -0x7fffffff - 1; }
__device__ __forceinline__ bool row_sees(int t, int pos, int behind, int sinks) {
  return (t <= pos) & ((t > behind) | (t < sinks));   // without branches
}

// Whether every row at positions first .. last sees every token of t0 .. t0 + n - 1.
__device__ __forceinline__ bool all_visible(const Attend& a, int first, int last, int t0, int n) {
  return t0 + n - 1 <= first && (!a.window || t0 > last - a.window || t0 + n <= a.sinks);
}

template <int TYPE>
__device__ __forceinline__ uint32_t pack2(float x, float y) {   // to nearest even
  if constexpr (TYPE == GRINQH_F16) {
    half2 r;
    r[0] = (_Float16)x; r[1] = (_Float16)y;
    return __builtin_bit_cast(uint32_t, r);
  } else {
    bhalf2 r;
    r[0] = (__bf16)x; r[1] = (__bf16)y;
    return __builtin_bit_cast(uint32_t, r);
  }
}

// 16-bit formats: whether a dword holds a value that is not finite, as a mask of its halves.
template <int FORMAT>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  constexpr uint32_t e = FORMAT == GRINQH_KV_F16 ? 0x7c00u : 0x7f80u;
  return ((w & e) == e ? 0xffffu : 0u) | ((w >> 16 & e) == e ? 0xffff0000u : 0u);
}


template <int FORMAT>
__device__ __forceinline__ float4v mfma16(u32x4 a, u32x4 b, float4v c) {
  if constexpr (FORMAT == GRINQH_KV_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

template <int FORMAT>
__device__ __forceinline__ float16v mfma32(u32x4 a, u32x4 b, float16v c) {
  if constexpr (FORMAT == GRINQH_KV_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// Maximum over the lanes that differ in bit 5, and in bit 4, of the lane number.
__device__ __forceinline__ float max_xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float max_xor16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float sum_xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ float sum_xor16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

// Two int8 codes as fp16, exact: bytes a and b of w ^ 0x80808080 beside 0x64 read as 1024 + code + 128.
__device__ __forceinline__ uint32_t codes2(uint32_t offset_binary, uint32_t a, uint32_t b) {
  const uint32_t v = __builtin_amdgcn_perm(0x64646464u, offset_binary, a | 0x0400u | (b << 16) | 0x04000000u);
  const half2 c = {(_Float16)1152.0f, (_Float16)1152.0f};
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(half2, v) - c);
}

// Queries of a row for the products with an 8-bit cache: fp16 as they are, bf16 as fp16 times the power of
// two that brings the row's largest finite magnitude to 2^14..2^15 (exact but for what lies 2^28 below it).  The scores' factor, which
// takes it back, stays a normal number: a row's power is held back where the factor would be under 2^-126, what that costs a score
// is under 2^-137 of the keys' scale.  A factor of zero would make NaN of the masked scores, -inf.
__device__ __forceinline__ int row_shift(float amax, float factor) {
  return amax > 0 ? min(14 - ilogbf(amax), 126 + ilogbf(factor)) : 0;
}
// And it is finite: zero times infinity would make NaN of scores of zero.
__device__ __forceinline__ float bounded(float factor) { return fminf(factor, 0x1.fffffep127f); }

// The exponent a scale >= 0 is held against: scale <= 2^e.  (An infinite one makes every channel of the rows that
// see it infinite or NaN, whatever it is held against.)
__device__ __forceinline__ int scale_exponent(float s) {
  return (int)(__builtin_bit_cast(uint32_t, s) >> 23 & 0xffu) - 126;
}
// Values of an 8-bit cache are weighed by exp(s - m) * scale * 2^(kUp - e), e the exponent of the largest
// scale that the row has seen so far: at most 2^15 in fp16, and 11 bits stay down to scales 2^23
// below it.  Stored scales reach down to 2^-107.
constexpr int kUp = 9;
constexpr int kLowestExponent = -110;

void launch_attend_rows(const AttendPlan& p, const AttendArgs& args, hipStream_t s);
void launch_attend_tile(const AttendPlan& p, const AttendArgs& args, hipStream_t s);

}  // namespace grinqh
