// Attention of chunks: many rows over the paged cache.
//
// A workgroup takes 32 rows per wave (token i, head g of one kv head's group) and walks tiles of 64 tokens, which
// all its waves share through LDS; a wave computes S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16, its
// rows being the columns.
//   - S^T leaves a lane with 16 of a block's 32 tokens for ONE row: maximum and sum are in the lane but for one
//     exchange of the two half waves, and the rescaling factor of O^T is the lane's own.
//   - the weights come out of the first product where the second wants them: its contraction is over tokens in
//     any order, and ds_read_b64_tr_b16 hands V over in the order of S^T's registers, channel per lane.
//   - 16-byte chunks of K's and V's rows are swizzled in LDS so that neither read conflicts.  (The rows that codes become are
//     written every second chunk at a time, which does: 0.15 of the cycles that LDS is busy.)
// 16-bit rows go to LDS directly; int8 rows pass through registers and become fp16 codes (exact), K's scales
// multiply the scores and V's the weights, each lane holding the scale of one token that the multiplication
// broadcasts by DPP.  Tiles are copied several slots ahead, and the waves run in two halves half a tile apart: one
// half's products meet the other's softmax.
//
// 4096 rows of 32 heads behind 32768 tokens of an 8-bit cache (2.34 Tflop): 2.69 .. 2.84 ms, 825 .. 870 TFLOP/s, where a library
// product of 8192^3 reaches 1200.  Neither pipe is full: a SIMD takes 89 cycles a product, of which the product holds its pipe
// 32, and about nine other vector instructions that go with it at 8 bits (scales, maximum, exponential, sum, packing, codes to
// fp16) take 38 to 50.  That is near the sum of the two, which the halves of the workgroup are there to overlap; waves wait in a
// third of their cycles, and what for is not known.  16-bit caches pay for the staging (page addresses, issue of the copies, a
// workgroup's first tile): without it in the loop they came to 1300; copies spread among the products were faster at D = 64
// (541 -> 472 us) and slower at D = 128, so they stand together.  A call of one tile takes 12 us, and 1.8 to 2.2 us go with every
// further one: a prompt of 2048 tokens from its start (34 Gflop, 8 kv heads of 4) is 256 workgroups of 4 to 32 tiles, and the
// longest makes its 76 us.
#include "attend.h"

namespace grinqh {

namespace {

constexpr int kTile = 64;
constexpr int kWaves = 8;

template <int N, int I = 0, typename F>
__device__ __forceinline__ void unroll(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unroll<N, I + 1>(f);
  }
}

// x of lane I of the lane's 16.
template <int I>
__device__ __forceinline__ float bcast16(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), 0x150 + I, 0xf, 0xf, true));
}

// Physical 16-byte chunk of a row's logical one.  K's rows are read 32 at a time at one chunk, V's 4 at a time
// over 64 bytes; either way 16 lanes meet 16 chunk places.
template <int D>
__device__ __forceinline__ int k_swizzle(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D>
__device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? (row & 3) << 2 : (row >> 1 & 1) << 2; }

// Tiles of fp16 or bf16 rows; an 8-bit cache's codes as they come, and its scales.
template <int D, bool I8>
struct TileLds {
  static constexpr int kBuffers = I8 ? 3 : 4;
  uint8_t k[kBuffers][kTile][2 * D];
  uint8_t v[kBuffers][kTile][2 * D];
  uint8_t raw_k[I8 ? 2 : 1][I8 ? kTile * D : 16];
  uint8_t raw_v[I8 ? 2 : 1][I8 ? kTile * D : 16];
  float ks[4][kTile], vs[4][kTile];
  int vmax[4];
  int odd[4][kWaves];   // per wave: what it staged of V held a value that is not finite
};

typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef short short4v __attribute__((ext_vector_type(4)));

template <int D, int FORMAT, int TYPE, bool SMALL>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_attend_tile(AttendArgs args) {
  const KvCache& c = args.c;
  const KvBatch& b = args.b;
  const Attend& a = args.a;
  const int splits = args.splits, per_split = args.per_split;
  constexpr bool I8 = FORMAT == GRINQH_KV_I8;
  constexpr int MF = I8 ? GRINQH_KV_F16 : FORMAT;   // type of the products
  constexpr int RB = 2 * D;                         // bytes of a row in LDS
  constexpr int ES = I8 ? 1 : 2;
  constexpr int LPR = D * ES / 16;                  // lanes per row of a staged load
  constexpr int LOADS = kTile * LPR / (64 * kWaves) > 0 ? kTile * LPR / (64 * kWaves) : 1;   // per lane, for K and for V
  constexpr int KS = D / 16, VB = D / 32;
  __shared__ __attribute__((aligned(1024))) TileLds<D, I8> lds;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, i16 = lane & 15;
  const int h = blockIdx.x % c.H, split = blockIdx.x / c.H, s = blockIdx.z;
  const Seq sq = kv_seq(c, b, s);
  const int all = sq.n * a.G, blocks = (all + 32 * kWaves - 1) / (32 * kWaves);
  const int* table = b.table + (long)s * b.width;

  for (int block = blockIdx.y; block < blocks; block += gridDim.y) {
    // the last rows see the most tokens: they start first
    const int r0 = (blocks - 1 - block) * 32 * kWaves;
    const int first = sq.L - sq.n + r0 / a.G, last = sq.L - sq.n + min(r0 + 32 * kWaves - 1, all - 1) / a.G;
    const Span span = attend_span<kTile>(a, first, last);
    const int v0 = split * per_split, used = span.splits(splits, per_split);
    if (split >= used) continue;
    const int v_end = split == splits - 1 ? span.tiles : min(span.tiles, v0 + per_split);

    // this lane's row (both halves of the wave have the same 32), and the span of the wave's rows
    const int w0 = r0 + 32 * wave, r = min(w0 + (lane & 31), all - 1);
    const int row = sq.r0 + r / a.G, head = h * a.G + r % a.G, pos = sq.L - sq.n + r / a.G;
    const int behind = behind_window(a, pos);
    const int wfirst = __builtin_amdgcn_readfirstlane(sq.L - sq.n + min(w0, all - 1) / a.G);
    const int wlast = __builtin_amdgcn_readfirstlane(sq.L - sq.n + min(w0 + 31, all - 1) / a.G);

    const DenseRows q = late().q;
    u32x4 qf[KS];
    float factor = bounded(a.scale * kLog2e);
    {
      const char* qp = q.p + (row * q.row + head * q.head) * 2 + 16 * half;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = *(const u32x4*)(qp + 32 * k);
      if constexpr (I8 && TYPE == GRINQH_BF16) {
        float amax = 0;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = bf2f((uint16_t)(qf[k][e >> 1] >> (16 * (e & 1))));
            amax = fmaxf(amax, fabsf(x) < INFINITY ? fabsf(x) : 0.0f);
          }
        const int up = row_shift(max_xor32(amax), factor);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            qf[k][e] = pack2<GRINQH_F16>(ldexpf(bf2f((uint16_t)qf[k][e]), up), ldexpf(bf2f((uint16_t)(qf[k][e] >> 16)), up));
        factor = bounded(ldexpf(factor, -up));
      }
    }

    float m = -INFINITY, l = 0, slack = kSlack<FORMAT>;
    int ev = kLowestExponent;
    float16v o[VB];
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = 0;

    // ---- staging: load i of a lane is chunk lane % LPR of row (64 kWaves i + thread) / LPR of the tile.  The rows of
    // one load of a wave lie in one page of 16 tokens or more: its address is scalar and the lanes' offsets do
    // not change.  Smaller pages (SMALL) are looked up by the lanes.  Page ids are read a tile ahead.
    constexpr int RPW = 64 / LPR;            // rows of a load of a wave
    static_assert(RPW <= 16);
    const int N = v_end - v0;                // tiles, counted from 0 from here on
    auto start = [&](int i) { const int v = v0 + i; return i < N ? span.tile(v) * kTile : 0x7fffffc0; };
    auto first_row = [&](int i) { return (kWaves * i + wave) * RPW % kTile; };
    const int my_row = lane / LPR, my_chunk = lane % LPR;
    const bool stages = (kWaves * (LOADS - 1) + wave) * RPW < kTile;   // else it repeats others' rows
    // byte offset of a load's first row (SMALL: of this lane's) in the arrays, or what is read in its place
    constexpr long kAbsent = -1, kBad = -2;
    int id[LOADS];                           // page ids of the next tile of K
    long at[LOADS];                          // offsets of the last tile of K: V's next
    int sid[4];                              // page ids of the next tile's scales (SMALL: this lane's)
    auto page_of = [&](int t) { return t < span.hi ? table[t >> c.shift] : -1; };
    auto offset_of = [&](int t, int page, int size) {
      return t >= span.hi ? kAbsent : (unsigned)page >= (unsigned)c.n_pages ? kBad : kv_slot(c, page, h, t) * size;
    };
    auto row_at = [&](int i, int x) { return start(i) + first_row(x) + (SMALL ? my_row : 0); };
    auto look = [&](int i) {
#pragma unroll
      for (int x = 0; x < LOADS; ++x) id[x] = page_of(row_at(i, x));
      if constexpr (I8) {
        if (wave < 2) {
#pragma unroll
          for (int x = 0; x < (SMALL ? 1 : 4); ++x) sid[x] = page_of(start(i) + (SMALL ? lane : 16 * x));
        }
      }
    };
    // a lane's chunk from there: SMALL adds none for the row
    uint32_t kat[LOADS], vat[LOADS];
#pragma unroll
    for (int x = 0; x < LOADS; ++x) {
      const int rw = first_row(x) + my_row, from = SMALL ? 0 : my_row * D * ES;
      kat[x] = from + 16 * (I8 ? my_chunk : my_chunk ^ k_swizzle<D>(rw));
      vat[x] = from + 16 * (I8 ? my_chunk : my_chunk ^ v_swizzle<D>(rw));
    }
    auto copy = [&](const char* from, uint8_t* to, int x) {
      if (stages) __builtin_amdgcn_global_load_lds((global_ptr)from, (lds_ptr)(to + (64 * kWaves * x + 64 * wave) * 16), 16, 0, 0);
    };
    // V of the tile that at[] stands for, into buffer or raw slot `to`
    auto fetch_v = [&](int to) {
#pragma unroll
      for (int x = 0; x < LOADS; ++x)
        copy((at[x] >= 0 ? c.v + at[x] : (const char*)g_zeros) + vat[x], I8 ? lds.raw_v[to] : &lds.v[I8 ? 0 : to][0][0], x);
    };
    // K of tile i, whose page ids look(i) has read, and its scales
    auto fetch_k = [&](int i, int to) {
#pragma unroll
      for (int x = 0; x < LOADS; ++x) {
        at[x] = offset_of(row_at(i, x), id[x], D * ES);
        copy((at[x] >= 0 ? c.k + at[x] : (const char*)(at[x] == kBad ? g_nans : g_zeros)) + kat[x],
             I8 ? lds.raw_k[to] : &lds.k[I8 ? 0 : to][0][0], x);
      }
      if constexpr (I8) {
        if (wave < 2) {   // a token per lane
          const int t = start(i) + lane, page = SMALL ? sid[0] : lane < 32 ? lane < 16 ? sid[0] : sid[1] : lane < 48 ? sid[2] : sid[3];
          const long o = offset_of(t, page, 4);
          const char* from = o >= 0 ? (const char*)(wave ? c.vs : c.ks) + o : (const char*)(o == kBad && !wave ? g_nans : g_zeros);
          __builtin_amdgcn_global_load_lds((global_ptr)from, (lds_ptr)(wave ? lds.vs[i & 3] : lds.ks[i & 3]), 4, 0, 0);
        }
      }
    };
    // This wave's part of raw codes as fp16 into LDS; its scales' largest exponent.
    auto convert = [&](const uint8_t* raw, uint8_t (*to)[RB], auto swizzle) {
      if (stages) {
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
          const u32x4 r = *(const u32x4*)(raw + (64 * kWaves * x + (int)threadIdx.x) * 16);
          const int rw = first_row(x) + my_row, ch = 2 * my_chunk;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = codes2(r[2 * y + (e >> 1)] ^ 0x80808080u, 2 * (e & 1), 2 * (e & 1) + 1);
            *(u32x4*)&to[rw][16 * ((ch + y) ^ swizzle(rw))] = w;
          }
        }
      }
    };
    auto convert_k = [&](int i, int raw, int to) {
      convert(lds.raw_k[raw], lds.k[to], [](int rw) { return k_swizzle<D>(rw); });
      if (wave == 1) {
        const float sr = lds.vs[i & 3][lane];
        int big = sr > 0 && sr < INFINITY ? scale_exponent(sr) : kLowestExponent;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) big = max(big, __shfl_xor(big, x));
        if (lane == 0) lds.vmax[i & 3] = big;
      }
    };
    auto convert_v = [&](int raw, int to) { convert(lds.raw_v[raw], lds.v[to], [](int rw) { return v_swizzle<D>(rw); }); };

    // Tiles that every row of the workgroup, or of the wave, sees whole: those inside the sinks, and from the last
    // row's window start to the first row's position.
    const int inner = a.sinks / kTile, shift_i = span.sink_tiles - span.lo_tile - v0;   // tile of tokens t is i = t / 64 + shift_i
    auto tiles_from = [&](int p) { return (a.window ? max(p - a.window + 1 + kTile - 1, 0) / kTile : 0) + shift_i; };
    auto tiles_to = [&](int p) { return max(p + 1, 0) / kTile + shift_i; };
    const int full_from = max(tiles_from(last), span.sink_tiles - v0), full_to = tiles_to(first);
    const int wave_from = max(tiles_from(wlast), span.sink_tiles - v0), wave_to = tiles_to(wfirst);
    const int sinks_to = min(inner, span.sink_tiles) - v0;
    auto full = [&](int i) { return i < sinks_to || (i >= full_from && i < full_to); };

    // A tile that not all rows see whole: values of this wave's part of V that are not finite are set to zero (and
    // lds.odd says so), since their products with weights of zero would reach rows that do not see them.
    auto check = [&](int i, int buf) {
      if constexpr (!I8) {
        if (i < N && !full(i)) {
          uint32_t top = 0;
          u32x4 w[LOADS];
#pragma unroll
          for (int x = 0; x < LOADS; ++x) {
            w[x] = *(const u32x4*)(&lds.v[buf][0][0] + (64 * kWaves * x + (int)threadIdx.x) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) top = max_halves(top, w[x][e] & 0x7fff7fffu);
          }
          const int odd = __any(not_finite<FORMAT>(top) != 0);
          if (lane == 0) lds.odd[i & 3][wave] = odd;
          if (odd) {
#pragma unroll
            for (int x = 0; x < LOADS; ++x) {
#pragma unroll
              for (int e = 0; e < 4; ++e) w[x][e] &= ~not_finite<FORMAT>(w[x][e]);
              *(u32x4*)(&lds.v[buf][0][0] + (64 * kWaves * x + (int)threadIdx.x) * 16) = w[x];
            }
          }
        }
      }
    };

    // ---- the work on a tile for the wave's rows: products() on the matrix cores, softmax() beside them
    float16v sc[2];
    u32x4 pf[2][2];
    // values(i) of the tile before and scores of tile i, one step at a time: PS steps of 16 tokens and 64 channels of V
    // (no accumulator twice in a row), then KS steps of 16 channels of K.  The operands are read AHEAD steps ahead,
    // which is about LDS's latency, and no further: registers are scarce.
    constexpr int PS = 2 * VB, AHEAD = 4;
    auto products = [&](int i, int vbuf, int kbuf, auto values_c, auto scores_c) __attribute__((always_inline)) {
      constexpr int FROM = decltype(values_c)::value ? 0 : PS, TO = decltype(scores_c)::value ? PS + KS : PS;
      const uint8_t* kb = &lds.k[kbuf][lane & 31][0];
      const uint8_t* vb = &lds.v[vbuf][4 * half + (i16 >> 2)][32 * (lane >> 4 & 1) + 8 * (i16 & 3)];
      u32x4 f[AHEAD + 1][2];
      auto read = [&](auto step_c) __attribute__((always_inline)) {
        constexpr int step = decltype(step_c)::value;
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          u32x4& to = f[step % (AHEAD + 1)][y];
          if constexpr (step < PS) {
            const int j = 2 * (step % (VB / 2)) + y, t = step / (VB / 2), at = 16 * ((4 * j) ^ v_swizzle<D>(i16 >> 2));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (__attribute__((address_space(3))) short4v*)(vb + (16 * t + 8 * x) * RB + at)));
              to[2 * x] = w[0]; to[2 * x + 1] = w[1];
            }
          } else {
            to = *(const u32x4*)(kb + 32 * RB * y + 16 * ((2 * (step - PS) + half) ^ k_swizzle<D>(lane & 31)));
          }
        }
      };
      if constexpr (TO > PS) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 16; ++e) sc[t][e] = 0;
      }
      unroll<AHEAD>([&](auto x) { read(std::integral_constant<int, FROM + decltype(x)::value>{}); });
      __builtin_amdgcn_sched_barrier(0);
      unroll<TO - FROM>([&](auto x) {
        constexpr int step = FROM + decltype(x)::value;
        if constexpr (step + AHEAD < TO) read(std::integral_constant<int, step + AHEAD>{});
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const u32x4 w = f[step % (AHEAD + 1)][y];
          if constexpr (step < PS) {
            constexpr int j = 2 * (step % (VB / 2)), t = step / (VB / 2);
            o[j + y] = mfma32<MF>(w, pf[t >> 1][t & 1], o[j + y]);
          } else {
            sc[y] = mfma32<MF>(w, qf[step - PS], sc[y]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      if constexpr (!I8 && FROM == 0) {
        // 0 times an infinity must not reach rows that do not see it: the products took what check() left, and the
        // rows that see a token get its other values here, from memory
        bool odd = false;
        const int t0 = start(i - 1);
        if (!full(i - 1))
          for (int w = 0; w < kWaves; ++w) odd |= lds.odd[(i - 1) & 3][w] != 0;
        if (__any(odd)) {
#pragma unroll 1
          for (int x = 0; x < kTile && t0 + x < span.hi; ++x) {
            const int id = table[(t0 + x) >> c.shift];
            if ((unsigned)id >= (unsigned)c.n_pages) continue;
            const bool see = row_sees(t0 + x, pos, behind, a.sinks);
            const char* from = c.v + kv_slot(c, id, h, t0 + x) * RB + 8 * half;
#pragma unroll
            for (int j = 0; j < VB; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const u32x2 w = load_global<u32x2>(from + 16 * (4 * j + e));   // channels 32 j + 8 e + 4 half .. + 3
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                  const uint16_t u = (uint16_t)(w[n >> 1] >> (16 * (n & 1)));
                  const float y = FORMAT == GRINQH_KV_F16 ? h2f(u) : bf2f(u);
                  o[j][4 * e + n] += see && !(fabsf(y) < INFINITY) ? y : 0.0f;
                }
              }
          }
        }
      }
    };
    // masked: some row of the wave does not see some token.  Branches rather than a second copy of the code: with
    // two, the 64 registers of o are held twice where they meet.
    auto softmax = [&](int i) __attribute__((always_inline)) {
      const int t0 = start(i);
      const bool masked = !(i < sinks_to || (i >= wave_from && i < wave_to));
      float kst[2], vst[2];
      int big = kLowestExponent;
      if constexpr (I8) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int tk = 32 * t + 8 * (i16 >> 2) + 4 * half + (i16 & 3);
          kst[t] = lds.ks[i & 3][tk];
          vst[t] = lds.vs[i & 3][tk];
        }
        big = lds.vmax[i & 3];
        unroll<16>([&](auto ec) {
          constexpr int e = decltype(ec)::value;
          sc[0][e] *= bcast16<e>(kst[0]);
          sc[1][e] *= bcast16<e>(kst[1]);
        });
      }
      uint32_t vis[2] = {0xffffu, 0xffffu};
      if (masked) {
        float vmax = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          vis[t] = 0;
          unroll<16>([&](auto ec) {
            constexpr int e = decltype(ec)::value;
            const bool see = row_sees(t0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3), pos, behind, a.sinks);
            vis[t] |= see ? 1u << e : 0u;
            sc[t][e] = see ? sc[t][e] : -INFINITY;
            if constexpr (I8) {
              const float w = bcast16<e>(vst[t]);
              vmax = fmaxf(vmax, see && w < INFINITY ? w : 0.0f);   // rows share a factor below
            }
          });
        }
        if constexpr (I8) big = scale_exponent(max_xor32(vmax));
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[t][e]);
      mx = rounded_product(max_xor32(mx), factor);
      look(i + 4);   // here: a scalar load among reads of LDS would make every wait for them a wait for all
      // a row's own scores and values alone decide what it is held against
      const bool grows = I8 && big > ev;
      float held = m;
      if (__any(mx - m > slack || grows)) {
        const bool rises = mx - m > kSlack<FORMAT>;
        const float was = m;
        if (rises) m = held_against<FORMAT>(mx);
        float alpha = rises ? exp2f(was - m) : 1.0f;
        l *= alpha;
        if (grows) { alpha *= ldexpf(1.0f, max(ev - big, -126)); ev = big; }
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[j][e] *= alpha;
        held = m;
        slack = far_out(held) ? -INFINITY : kSlack<FORMAT>;
        if (far_out(held)) {   // what exp2 is to see, over the factor that it will be multiplied by
          const float inv = inverse(factor);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 16; ++e) sc[t][e] = (rounded_product(sc[t][e], factor) - held) * inv;
          held = 0;
        }
      }
      const float base = held == -INFINITY ? 0.0f : held;
      // the factor 2^(kUp - ev) goes into the tokens' scales, which the wave shares, where its rows have one ev, else into
      // the weights: of rows whose ev lie far apart no common factor would leave all in range.  (A scale is at most 2^121.01,
      // the largest fp32 over 127, so its product with a weight of up to 2^6 is finite.  Exact either way, but that of values
      // under 2^-80 such a product can be subnormal and lose bits 2^-43 below the row's largest.)
      float down = 1, own = 1;
      bool shared = true;
      if constexpr (I8) {
        shared = __all(ev == __builtin_amdgcn_readfirstlane(ev));
        (shared ? down : own) = ldexpf(1.0f, kUp - ev);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float p[16], sum = 0;
        unroll<16>([&](auto ec) {
          constexpr int e = decltype(ec)::value;
          p[e] = __builtin_amdgcn_exp2f(fmaf(sc[t][e], factor, -base));
          sum += p[e];
        });
        if constexpr (I8) {
          const float w = vst[t] * down;
          unroll<16>([&](auto ec) {
            constexpr int e = decltype(ec)::value;
            p[e] *= bcast16<e>(w);
          });
          if (!shared) {
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] *= own;
          }
          if (masked) {   // a scale that is not finite stays with the rows that see it
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = vis[t] >> e & 1 ? p[e] : 0.0f;
          }
        }
        l += sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[t][e >> 2][e & 3] = pack2<MF == GRINQH_KV_BF16 ? GRINQH_BF16 : GRINQH_F16>(p[2 * e], p[2 * e + 1]);
      }
      // the weights are made here and not, as the compiler would have it, where the products take them
      asm volatile("" : "+v"(pf[0][0]), "+v"(pf[0][1]), "+v"(pf[1][0]), "+v"(pf[1][1]), "+v"(l));
    };
    // ---- the schedule.  Time runs in slots that end in a barrier.  The waves of the first half take the products of
    // tile i (its scores, and the values of i - 1) in slot 2 i and softmax(i) in slot 2 i + 1, the others a slot later, so
    // that on every SIMD one wave's softmax runs beside the other's products.  With softmax(i) a wave asks for its part of K
    // of i + 3 and V of i + 2, and with its products of i + 2 it sees to it that they are there: four slots, for all
    // workgroups of an XCD walk the same tokens abreast and wait for them to come from HBM.  16-bit rows take
    // the buffers of tiles i - 1 and i - 2, last read in slot 2 i - 1; codes pass through a slot of their own and become rows in
    // three buffers with the products of i + 2.  What is there by the end of slot 2 i + 5 is first read in slot 2 i + 6.
    // Behind the last tile come fillers.
    auto wait = [&](bool all) {   // a barrier does not wait for copies into LDS: until those of the last softmax, or none, are left
      if (all || SMALL) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      else if (!I8) { if constexpr (LOADS == 2) asm volatile("s_waitcnt vmcnt(4)" ::: "memory"); else asm volatile("s_waitcnt vmcnt(2)" ::: "memory"); }
      else if (wave < 2) asm volatile("s_waitcnt vmcnt(3)" ::: "memory");
      else asm volatile("s_waitcnt vmcnt(2)" ::: "memory");
    };
    static_assert(LOADS == 1 || (!I8 && LOADS == 2));
    auto end_slot = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    if (N > 0) {
      const bool second = wave >= kWaves / 2;
      look(0);
      fetch_k(0, 0);
      fetch_v(0);
      look(1);
      fetch_k(1, 1);
      look(2);
      if constexpr (I8) {
        wait(true);
        convert_k(0, 0, 0);
        convert_v(0, 0);
        convert_k(1, 1, 1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the slots have been read
      }
      fetch_v(1);
      fetch_k(2, I8 ? 1 : 2);
      look(3);
      if constexpr (!I8) {
        wait(false);
        check(0, 0);
      }
      end_slot();
      if (second) end_slot();
      products(0, 0, 0, std::false_type{}, std::true_type{});
      end_slot();
      int b3 = 0;                            // i modulo 3
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const int n3 = b3 == 2 ? 0 : b3 + 1, nn3 = 3 - b3 - n3;
        fetch_v(I8 ? i & 1 : (i + 2) & 3);
        fetch_k(i + 3, I8 ? i & 1 : (i + 3) & 3);
        softmax(i);
        end_slot();
        if constexpr (I8) products(i + 1, b3, n3, std::true_type{}, std::true_type{});
        else products(i + 1, i & 3, (i + 1) & 3, std::true_type{}, std::true_type{});
        wait(false);
        if constexpr (I8) {
          convert_k(i + 2, (i + 1) & 1, nn3);
          convert_v((i + 1) & 1, n3);
        } else {
          check(i + 1, (i + 1) & 3);
        }
        end_slot();
        b3 = n3;
      }
      if (!second) end_slot();
      wait(true);
      __syncthreads();
    }

    const DenseRows out = late().out;
    const Partial part = late().part;
    float* lse = late().lse;
    // ---- results: lane = row, 4 channels per quad of registers
    l += __builtin_bit_cast(float, __shfl_xor(__builtin_bit_cast(int, l), 32));
    const float inv = l == 0 ? 0.0f : 1.0f / l;
    const float back = ldexpf(1.0f, ev - kUp);   // of its own: with 1 / l it could leave fp32
    auto result = [&](int j, int e) { return I8 ? o[j][e] * inv * back : o[j][e] * inv; };
    const float lse2 = l == 0 ? -INFINITY : m + log2f(l);
    if (w0 + (lane & 31) < all) {
      const long at = (long)row * a.heads + head;
      if (used > 1) {
        if (half == 0) part.lse[split * part.rows + at] = lse2;
        if (lse2 != -INFINITY) {
          float* p = part.o + (split * part.rows + at) * D + 4 * half;
#pragma unroll
          for (int j = 0; j < VB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *(float4v*)(p + 32 * j + 8 * e) = float4v{result(j, 4 * e), result(j, 4 * e + 1), result(j, 4 * e + 2), result(j, 4 * e + 3)};
        }
      } else {
        if (lse && half == 0) lse[at] = lse2 * kLn2;
      }
    }
    if (used == 1) {
      // Rows of the output are written whole, through LDS: from the lanes' own pieces of 8 bytes every store would touch 32
      // rows, 2 us of a workgroup's end.  (`rows` begins where no copy is under way any more.)
      constexpr int STRIDE = RB + 16;        // 16 rows of pieces meet 64 banks
      static_assert(kWaves * 32 * STRIDE <= sizeof(lds.k) + sizeof(lds.v));
      uint8_t* rows = &lds.k[0][0][0] + wave * 32 * STRIDE;
#pragma unroll
      for (int j = 0; j < VB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *(u32x2*)(rows + (lane & 31) * STRIDE + 2 * (32 * j + 8 * e + 4 * half)) =
              u32x2{pack2<TYPE>(result(j, 4 * e), result(j, 4 * e + 1)), pack2<TYPE>(result(j, 4 * e + 2), result(j, 4 * e + 3))};
      const long to = (row * out.row + head * out.head) * 2;
      wave_sync();
      constexpr int LANES = RB / 16;         // of a row
#pragma unroll
      for (int x = 0; x < LANES / 2; ++x) {
        const int n = x * (64 / LANES) + lane / LANES, piece = 16 * (lane % LANES);
        const u32x4 w = *(const u32x4*)(rows + n * STRIDE + piece);
        const long at = __shfl(to, n);
        if (w0 + n < all) *(u32x4*)(out.p + at + piece) = w;
      }
    }
    __syncthreads();
  }
}

template <int D, int FORMAT, int TYPE>
void go(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  const dim3 grid(args.c.H * p.splits, p.blocks, args.b.B);
  if (args.c.shift >= 4) k_attend_tile<D, FORMAT, TYPE, false><<<grid, 64 * kWaves, 0, s>>>(args);
  else k_attend_tile<D, FORMAT, TYPE, true><<<grid, 64 * kWaves, 0, s>>>(args);
}

}  // namespace

void launch_attend_tile(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  auto on = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (args.c.format == GRINQH_KV_F16) go<D, GRINQH_KV_F16, GRINQH_F16>(p, args, s);
    else if (args.c.format == GRINQH_KV_BF16) go<D, GRINQH_KV_BF16, GRINQH_BF16>(p, args, s);
    else if (args.a.type == GRINQH_F16) go<D, GRINQH_KV_I8, GRINQH_F16>(p, args, s);
    else go<D, GRINQH_KV_I8, GRINQH_BF16>(p, args, s);
  };
  if (args.c.D == 64) on(std::integral_constant<int, 64>{});
  else on(std::integral_constant<int, 128>{});
}

}  // namespace grinqh
