// Attention of chunks: many rows over the paged cache.
//
// A workgroup takes 32 rows per wave (token i, head g of one kv head's group) and walks tiles of 64 tokens, which
// all its waves share through LDS; a wave computes S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_32x32x16, its
// rows being the columns.
//   - S^T leaves a lane with 16 of a block's 32 tokens for ONE row: maximum and sum are in the lane but for one
//     exchange of the two half waves, and the rescaling factor of O^T is the lane's own.
//   - the weights come out of the first product where the second wants them: its contraction is over tokens in
//     any order, and ds_read_b64_tr_b16 hands V over in the order of S^T's registers, channel per lane.
//   - 16-byte chunks of K's and V's rows are swizzled in LDS so that neither read conflicts.
// 16-bit rows go to LDS directly; int8 rows pass through registers and become fp16 codes (exact), K's scales
// multiply the scores and V's the weights, each lane holding the scale of one token that the multiplication
// broadcasts by DPP.  The next tile's rows are under way while one is multiplied; one barrier per tile.
#include "attend.h"

namespace grinqh {

namespace {

constexpr int kTile = 64;

__device__ const uint32_t g_zeros[64] = {0};
__device__ const uint32_t g_nans[64] = {
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
    0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff};

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

template <int D>
struct TileLds {
  uint8_t k[2][kTile][2 * D];
  uint8_t v[2][kTile][2 * D];
  float ks[2][kTile], vs[2][kTile];
  int vmax[2];
  int odd[2][8];     // per wave: what it staged of V holds a value that is not finite
};

typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;
typedef short short4v __attribute__((ext_vector_type(4)));

template <int D, int FORMAT, int TYPE, int NW>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2)))
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
  constexpr int LOADS = kTile * LPR / (64 * NW) > 0 ? kTile * LPR / (64 * NW) : 1;   // per lane, for K and for V
  constexpr int KS = D / 16, VB = D / 32;
  __shared__ __attribute__((aligned(1024))) TileLds<D> lds;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, i16 = lane & 15;
  const int h = blockIdx.x % c.H, split = blockIdx.x / c.H, s = blockIdx.z;
  const Seq sq = kv_seq(c, b, s);
  const int all = sq.n * a.G, blocks = (all + 32 * NW - 1) / (32 * NW);
  const int* table = b.table + (long)s * b.width;

  for (int block = blockIdx.y; block < blocks; block += gridDim.y) {
    // the last rows see the most tokens: they start first, and with two workgroups per CU the lightest join
    // the heaviest
    const int order = block < (blocks + 1) / 2 || gridDim.z * gridDim.y * gridDim.x > 512 ? blocks - 1 - block : block - (blocks + 1) / 2;
    const int r0 = order * 32 * NW;
    const int first = sq.L - sq.n + r0 / a.G, last = sq.L - sq.n + min(r0 + 32 * NW - 1, all - 1) / a.G;
    const Span span = attend_span<kTile>(a, first, last);
    const int v0 = split * per_split;
    const int v_end = split == splits - 1 ? span.tiles : min(span.tiles, v0 + per_split);

    // this lane's row (both halves of the wave have the same 32), and the span of the wave's rows
    const int w0 = r0 + 32 * wave, r = min(w0 + (lane & 31), all - 1);
    const int row = sq.r0 + r / a.G, head = h * a.G + r % a.G, pos = sq.L - sq.n + r / a.G;
    const int behind = behind_window(a, pos);
    const int wfirst = __builtin_amdgcn_readfirstlane(sq.L - sq.n + min(w0, all - 1) / a.G);
    const int wlast = __builtin_amdgcn_readfirstlane(sq.L - sq.n + min(w0 + 31, all - 1) / a.G);
    const bool idle = w0 >= all;

    const DenseRows q = late().q;
    u32x4 qf[KS];
    float factor = a.scale * kLog2e;
    {
      const char* qp = q.p + (row * q.row + head * q.head) * 2 + 16 * half;
#pragma unroll
      for (int k = 0; k < KS; ++k) qf[k] = *(const u32x4*)(qp + 32 * k);
      if constexpr (I8 && TYPE == GRINQH_BF16) {
        float amax = 0;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float x = bf2f((uint16_t)(qf[k][e >> 1] >> (16 * (e & 1))));
            bad |= !(fabsf(x) < INFINITY);
            amax = fmaxf(amax, fabsf(x));
          }
        if (bad) amax = INFINITY;
        const int up = row_shift(max_xor32(amax));
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            qf[k][e] = pack2<GRINQH_F16>(ldexpf(bf2f((uint16_t)qf[k][e]), up), ldexpf(bf2f((uint16_t)(qf[k][e] >> 16)), up));
        factor = ldexpf(factor, -up);
      }
    }

    float m = -INFINITY, l = 0;
    int ev = kLowestExponent;
    float16v o[VB];
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = 0;

    // ---- staging: load i of a lane is chunk lane % LPR of row (64 NW i + thread) / LPR of the tile
    int ids[LOADS], sid = 0;
    u32x4 kr[LOADS], vr[LOADS];
    float sr = 0;
    const bool stages = LOADS > 1 || (int)threadIdx.x < kTile * LPR;
    auto token = [&](int v, int t) { return v < v_end ? span.tile(v) * kTile + t : 0x7fffffff; };
    auto lookup = [&](int v, int t) { const int x = token(v, t); return x < span.hi ? table[x >> c.shift] : -1; };
    auto row_of = [&](int i) { return (64 * NW * i + (int)threadIdx.x) / LPR; };
    auto look = [&](int v) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) ids[i] = lookup(v, row_of(i) % kTile);
      if constexpr (I8) if (wave < 2) sid = lookup(v, lane);
    };
    auto fetch = [&](int v, int buf) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int t = token(v, row_of(i) % kTile);
        const bool in = t < span.hi, ok = in && (unsigned)ids[i] < (unsigned)c.n_pages;
        const long at = ok ? kv_slot(c, ids[i], h, t) * (D * ES) : 0;
        const char* kp = ok ? c.k + at : (const char*)(in ? g_nans : g_zeros);
        const char* vp = ok ? c.v + at : (const char*)g_zeros;
        if constexpr (I8) {
          kr[i] = load_global<u32x4>(kp + 16 * (lane % LPR));
          vr[i] = load_global<u32x4>(vp + 16 * (lane % LPR));
        } else {
          const int rw = row_of(i), to = (64 * NW * i + 64 * wave) * 16;
          __builtin_amdgcn_global_load_lds((global_ptr)(kp + 16 * ((lane % LPR) ^ k_swizzle<D>(rw))),
                                           (lds_ptr)(&lds.k[buf][0][0] + to), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((global_ptr)(vp + 16 * ((lane % LPR) ^ v_swizzle<D>(rw))),
                                           (lds_ptr)(&lds.v[buf][0][0] + to), 16, 0, 0);
        }
      }
      if constexpr (I8) {
        if (wave < 2) {
          const int t = token(v, lane);
          const bool in = t < span.hi, ok = in && (unsigned)sid < (unsigned)c.n_pages;
          const float* src = wave ? c.vs : c.ks;
          const float* none = (const float*)(in && !wave ? g_nans : g_zeros);
          sr = load_global<float>(ok ? src + kv_slot(c, sid, h, t) : none);
        }
      }
    };
    // int8 codes as fp16 into LDS
    auto put = [&](int buf) {
      if constexpr (I8) {
        if (stages) {
#pragma unroll
          for (int i = 0; i < LOADS; ++i) {
            const int rw = row_of(i), ch = 2 * (lane % LPR);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              u32x4 kk, vv;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                kk[e] = codes2(kr[i][2 * x + (e >> 1)] ^ 0x80808080u, 2 * (e & 1), 2 * (e & 1) + 1);
                vv[e] = codes2(vr[i][2 * x + (e >> 1)] ^ 0x80808080u, 2 * (e & 1), 2 * (e & 1) + 1);
              }
              *(u32x4*)&lds.k[buf][rw][16 * ((ch + x) ^ k_swizzle<D>(rw))] = kk;
              *(u32x4*)&lds.v[buf][rw][16 * ((ch + x) ^ v_swizzle<D>(rw))] = vv;
            }
          }
        }
        if (wave == 0) lds.ks[buf][lane] = sr;
        if (wave == 1) {
          lds.vs[buf][lane] = sr;
          int big = sr > 0 && sr < INFINITY ? scale_exponent(sr) : kLowestExponent;
#pragma unroll
          for (int x = 1; x < 64; x <<= 1) big = max(big, __shfl_xor(big, x));
          if (lane == 0) lds.vmax[buf] = big;
        }
      }
    };

    // a tile that not all rows see whole: whether this wave's part of V is finite throughout
    auto check = [&](int v, int buf) {
      if constexpr (!I8) {
        if (v < v_end && !all_visible(a, first, last, span.tile(v) * kTile, kTile)) {
          uint32_t any = 0;
#pragma unroll
          for (int i = 0; i < LOADS; ++i) {
            const u32x4 w = *(const u32x4*)(&lds.v[buf][0][0] + (64 * NW * i + (int)threadIdx.x) % (kTile * LPR) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) any |= not_finite<FORMAT>(w[e]);
          }
          const int odd = __any(any != 0);
          if (lane == 0) lds.odd[buf][wave] = odd;
        }
      }
    };

    // ---- one tile for the wave's rows.  masked: some row does not see some token; odd: that tile's V holds a
    // value that is not finite (16-bit formats).  Branches rather than a second copy of the code: with two,
    // the 64 registers of o are held twice where they meet.
    auto compute = [&](int buf, int t0, bool masked, bool odd) __attribute__((always_inline)) {
      float16v sc[2];
      const uint8_t* kb = &lds.k[buf][lane & 31][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] = 0;
      u32x4 kf[2][2];
      auto read_k = [&](int k) __attribute__((always_inline)) {
        const int at = 16 * ((2 * k + half) ^ k_swizzle<D>(lane & 31));
#pragma unroll
        for (int t = 0; t < 2; ++t) kf[k & 1][t] = *(const u32x4*)(kb + 32 * RB * t + at);
      };
      read_k(0);
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        if (k + 1 < KS) read_k(k + 1);
        __builtin_amdgcn_sched_barrier(0);   // one step ahead and no further: registers are scarce
#pragma unroll
        for (int t = 0; t < 2; ++t) sc[t] = mfma32<MF>(kf[k & 1][t], qf[k], sc[t]);
        __builtin_amdgcn_sched_barrier(0);
      }
      float kst[2], vst[2];
      int big = kLowestExponent;
      if constexpr (I8) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int tk = 32 * t + 8 * (i16 >> 2) + 4 * half + (i16 & 3);
          kst[t] = lds.ks[buf][tk];
          vst[t] = lds.vs[buf][tk];
        }
        big = lds.vmax[buf];
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
            const int tk = t0 + 32 * t + 8 * (e >> 2) + 4 * half + (e & 3);
            const bool see = row_sees(tk, pos, behind, a.sinks);
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
      mx = max_xor32(mx) * factor;
      // a row's own scores and values alone decide what it is held against
      const bool rises = mx > m + kSlack, grows = I8 && big > ev;
      if (__any(rises || grows)) {
        float alpha = rises ? exp2f(m - mx) : 1.0f;
        if (rises) m = mx;
        l *= alpha;
        if (grows) { alpha *= ldexpf(1.0f, max(ev - big, -126)); ev = big; }
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[j][e] *= alpha;
      }
      const float base = m == -INFINITY ? 0.0f : m;
      // the factor 2^(kUp - ev) goes into the tokens' scales, which the wave shares: that of the largest ev,
      // and where rows differ what is left of theirs (powers of two: exact)
      float down = 1, fix = 1;
      bool shared = true;
      if constexpr (I8) {
        int top = __builtin_amdgcn_readfirstlane(ev);
        shared = __all(ev == top);
        if (!shared) {
          top = ev;
#pragma unroll
          for (int x = 1; x < 32; x <<= 1) top = max(top, __shfl_xor(top, x));
          fix = ldexpf(1.0f, min(top - ev, 127));
        }
        down = ldexpf(1.0f, kUp - top);
      }
      u32x4 pf[2][2];
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
            for (int e = 0; e < 16; ++e) p[e] *= fix;
          }
        }
        if constexpr (I8) {
          if (masked) {   // a scale that is not finite stays with the rows that see it
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = vis[t] >> e & 1 ? p[e] : 0.0f;
          }
        }
        l += sum;
#pragma unroll
        for (int e = 0; e < 8; ++e) pf[t][e >> 2][e & 3] = pack2<MF == GRINQH_KV_BF16 ? GRINQH_BF16 : GRINQH_F16>(p[2 * e], p[2 * e + 1]);
      }
      const uint8_t* vb = &lds.v[buf][4 * half + (i16 >> 2)][32 * (lane >> 4 & 1) + 8 * (i16 & 3)];
      u32x4 vf[2][2];   // two steps of 16 tokens, read two ahead
      auto read_v = [&](int step) __attribute__((always_inline)) {
        const int j = step >> 1, at = 16 * ((4 * j) ^ v_swizzle<D>(i16 >> 2));
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int t = 2 * (step & 1) + y;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) short4v*)(vb + (16 * t + 8 * x) * RB + at)));
            vf[step & 1][y][2 * x] = w[0]; vf[step & 1][y][2 * x + 1] = w[1];
          }
        }
      };
      read_v(0);
#pragma unroll
      for (int step = 0; step < 2 * VB; ++step) {
        if (step + 1 < 2 * VB) read_v(step + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const int j = step >> 1, t = 2 * (step & 1) + y;
          u32x4 f = vf[step & 1][y];
          if constexpr (!I8) {
            if (odd) {
#pragma unroll
              for (int e = 0; e < 4; ++e) f[e] &= ~not_finite<FORMAT>(f[e]);
            }
          }
          o[j] = mfma32<MF>(f, pf[t >> 1][t & 1], o[j]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!I8) {
        if (odd) {
          // 0 times an infinity must not reach rows that do not see it: the products above took the finite
          // values, and the rows that see a token now get its others
#pragma unroll 1
          for (int x = 0; x < kTile; ++x) {
            const int tk = t0 + x;
            const bool see = row_sees(tk, pos, behind, a.sinks);
#pragma unroll
            for (int j = 0; j < VB; ++j)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                // channels 32 j + 8 e + 4 half .. + 3
                const u32x2 w = *(const u32x2*)&lds.v[buf][x][16 * ((4 * j + e) ^ v_swizzle<D>(x)) + 8 * half];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const uint16_t u = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
                  const float y = FORMAT == GRINQH_KV_F16 ? h2f(u) : bf2f(u);
                  o[j][4 * e + i] += see && !(fabsf(y) < INFINITY) ? y : 0.0f;
                }
              }
          }
        }
      }
    };

    if (v0 < v_end) {
      look(v0);
      fetch(v0, 0);
      look(v0 + 1);
      put(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // a barrier does not wait for copies into LDS
      check(v0, 0);
      __syncthreads();
      for (int v = v0; v < v_end; ++v) {
        const int buf = (v - v0) & 1, t0 = span.tile(v) * kTile;
        fetch(v + 1, buf ^ 1);   // past the end: fillers, never used
        look(v + 2);
        if (!idle && t0 <= wlast && (!a.window || t0 + kTile > wfirst - a.window + 1 || t0 < a.sinks)) {
          bool odd = false;
          if (!I8 && !all_visible(a, first, last, t0, kTile))
            for (int w = 0; w < NW; ++w) odd |= lds.odd[buf][w] != 0;
          compute(buf, t0, !all_visible(a, wfirst, wlast, t0, kTile), __any(odd));
        }
        put(buf ^ 1);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        check(v + 1, buf ^ 1);
        __syncthreads();
      }
    }

    const DenseRows out = late().out;
    const Partial part = late().part;
    float* lse = late().lse;
    // ---- results: lane = row, 4 channels per quad of registers
    l += __builtin_bit_cast(float, __shfl_xor(__builtin_bit_cast(int, l), 32));
    const float inv = l == 0 ? 0.0f : (I8 ? ldexpf(1.0f, ev - kUp) : 1.0f) / l;
    const float lse2 = l == 0 ? -INFINITY : m + log2f(l);
    if (w0 + (lane & 31) < all) {
      const long at = (long)row * a.heads + head;
      if (splits > 1) {
        if (half == 0) part.lse[split * part.rows + at] = lse2;
        if (lse2 != -INFINITY) {
          float* p = part.o + (split * part.rows + at) * D + 4 * half;
#pragma unroll
          for (int j = 0; j < VB; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              *(float4v*)(p + 32 * j + 8 * e) = float4v{o[j][4 * e] * inv, o[j][4 * e + 1] * inv, o[j][4 * e + 2] * inv, o[j][4 * e + 3] * inv};
        }
      } else {
        if (lse && half == 0) lse[at] = lse2 * kLn2;
        char* p = out.p + (row * out.row + head * out.head + 4 * half) * 2;
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *(u32x2*)(p + 2 * (32 * j + 8 * e)) = u32x2{pack2<TYPE>(o[j][4 * e] * inv, o[j][4 * e + 1] * inv),
                                                        pack2<TYPE>(o[j][4 * e + 2] * inv, o[j][4 * e + 3] * inv)};
      }
    }
    __syncthreads();
  }
}

template <int D, int FORMAT, int TYPE>
void go(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  const dim3 grid(args.c.H * p.splits, p.blocks, args.b.B);
  if (p.nb == 4) k_attend_tile<D, FORMAT, TYPE, 4><<<grid, 256, 0, s>>>(args);
  else k_attend_tile<D, FORMAT, TYPE, 8><<<grid, 512, 0, s>>>(args);
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
