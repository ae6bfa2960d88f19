// Attention of a few rows over a long cache: decoding, and short chunks.
//
// The rows (token i, head g of the group) of a kv head are the columns of S^T = K Q^T and O^T = V^T P^T, 16 NB
// of them.  A wave walks its own tiles of 32 tokens, K and V straight from memory into the operands of
// v_mfma_f32_16x16x32: no LDS copy of K or V, no barrier until the waves' results meet.
//   - S^T leaves a lane with 4 tokens of each of the tile's two 16-token blocks for ONE row, so the softmax is
//     in the lane but for one maximum over the four lanes of the row, and the weights are where the second
//     product wants them: its contraction is over tokens in any order, as long as V's rows follow the same one.
//   - a lane loads D / 16 consecutive values of each of those 8 tokens of V; byte permutes turn the 8 x D / 16
//     block round into D / 16 operands whose row is the channel (D / 16) (lane % 16) + j.
//   - int8 codes become fp16 on the way (exact); K's scales multiply the scores, V's the weights.
//   - pages of 16 tokens or more hold a block whole: its address is scalar, the lanes' offsets are constant.
//     Smaller pages (SMALL) pass the 32 tokens' addresses and scales through LDS.
// The next tile's K is loaded while the softmax runs, its V behind the second product.
//
// Bound by memory: every visible K and V row is read once.  One token over 131072 tokens of an 8-bit cache, 8 kv heads
// of 128 (277 MB): 44.4 us in this kernel, 6.2 TB/s where a plain read of 2 GiB reaches 6.9, and 5.1 us joining 64
// parts; 32 sequences up to 8191 tokens, bf16 rows (269 MB): 51 and 5 us.  A part of a few tiles is a chain of latencies
// (page id, loads, two products): one token after 76 takes 6.2 us, of which its 0.2 MB are nothing.  With NB = 2 it is far
// from that bound (64 rows of a kv head over 8190 tokens of 4 sequences, 69 MB: 43 us): 33 rows and more are two workgroups
// that each read the cache, and at D = 128 over a 16-bit one the kernel needs more than 256 registers and keeps 12 to 15
// values in scratch.
#include "attend.h"

namespace grinqh {

namespace {

constexpr int kTile = 32;

// What a value that is not finite adds where it is seen: 1 in the halves of w that are +inf or NaN
// (sign = 0), -inf or NaN (sign = 1).
template <int FORMAT>
__device__ __forceinline__ uint32_t infinite_ones(uint32_t w, int sign) {
  constexpr uint32_t one = FORMAT == GRINQH_KV_F16 ? 0x3c00u : 0x3f80u;
  constexpr uint32_t inf = FORMAT == GRINQH_KV_F16 ? 0x7c00u : 0x7f80u;
  uint32_t r = 0;
  for (int i = 0; i < 2; ++i) {
    const uint32_t h = w >> (16 * i) & 0xffffu;
    const bool nan = (h & 0x7fffu) > inf;
    if (nan || h == (inf | (uint32_t)sign << 15)) r |= one << (16 * i);
  }
  return r;
}

// LDS of one wave: where the tile's 32 tokens lie, and their scales.
struct alignas(16) WaveTokens {
  const char* k[kTile];
  const char* v[kTile];
  float ks[kTile];
  float vs[kTile];
};

template <int D, int NB, int WAVES>
struct RowsLds {
  WaveTokens tokens[WAVES];
  float m[WAVES][16 * NB], l[WAVES][16 * NB];
  float o[WAVES][16][D + 4];   // one block of 16 rows at a time
};

template <int W>
struct Words { uint32_t w[W]; };

template <int W>
__device__ __forceinline__ Words<W> load_words(const char* p) {
  Words<W> r;
  if constexpr (W == 1) r.w[0] = load_global<uint32_t>(p);
  else if constexpr (W == 2) { const u32x2 x = load_global<u32x2>(p); r.w[0] = x[0]; r.w[1] = x[1]; }
  else { const u32x4 x = load_global<u32x4>(p); for (int i = 0; i < 4; ++i) r.w[i] = x[i]; }
  return r;
}

template <int D, int FORMAT, int TYPE, int NB, bool SMALL>
__global__ __launch_bounds__(64 * rows_waves(NB)) __attribute__((amdgpu_waves_per_eu(rows_per_simd(FORMAT, NB))))
void k_attend_rows(AttendArgs args) {
  const KvCache& c = args.c;
  const KvBatch& b = args.b;
  const Attend& a = args.a;
  const int splits = args.splits, per_split = args.per_split;
  constexpr bool I8 = FORMAT == GRINQH_KV_I8;
  constexpr int ES = I8 ? 1 : 2;             // bytes of a cached value
  constexpr int KS = D / 32;                 // steps of the first product
  constexpr int KL = I8 ? D / 64 : D / 32;   // 16-byte loads of a K row per lane
  constexpr int VC = D / 16;                 // channels of V per lane, blocks of the second product
  constexpr int VW = VC * ES / 4;            // dwords of those
  constexpr int WAVES = rows_waves(NB);
  __shared__ RowsLds<D, NB, WAVES> lds;

  const int lane = threadIdx.x & 63, i16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = blockIdx.x % c.H, split = blockIdx.x / c.H, s = blockIdx.z;
  const Seq sq = kv_seq(c, b, s);
  const int all = sq.n * a.G;                // rows of this kv head
  WaveTokens& tok = lds.tokens[wave];

  for (int r0 = blockIdx.y * 16 * NB; r0 < all; r0 += gridDim.y * 16 * NB) {
    const int first = sq.L - sq.n + r0 / a.G, last = sq.L - sq.n + min(r0 + 16 * NB - 1, all - 1) / a.G;
    const Span span = attend_span<kTile>(a, first, last);
    const int used = span.splits(splits, per_split);
    if (split >= used) continue;
    const int v_end = split == splits - 1 ? span.tiles : min(span.tiles, (split + 1) * per_split);
    const int v0 = split * per_split + wave;

    // this lane's rows and their queries
    const DenseRows q = late().q;
    int pos[NB], behind[NB];
    float factor[NB];
    u32x4 qf[NB][KS];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(r0 + 16 * n + i16, all - 1);   // rows past the last repeat it and are not stored
      pos[n] = sq.L - sq.n + r / a.G;
      behind[n] = behind_window(a, pos[n]);
      const char* qp = q.p + ((sq.r0 + r / a.G) * q.row + (h * a.G + r % a.G) * q.head) * 2;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int d = I8 ? (k >> 1) * 64 + 16 * quad + 8 * (k & 1) : 32 * k + 8 * quad;
        qf[n][k] = *(const u32x4*)(qp + 2 * d);
      }
      factor[n] = bounded(a.scale * kLog2e);
      if constexpr (I8 && TYPE == GRINQH_BF16) {
        float amax = 0;
        for (int k = 0; k < KS; ++k)
          for (int e = 0; e < 8; ++e) {
            const float x = bf2f((uint16_t)(qf[n][k][e >> 1] >> (16 * (e & 1))));
            amax = fmaxf(amax, fabsf(x) < INFINITY ? fabsf(x) : 0.0f);
          }
        amax = max_xor16(max_xor32(amax));
        const int up = row_shift(amax, factor[n]);
        for (int k = 0; k < KS; ++k)
          for (int e = 0; e < 4; ++e)
            qf[n][k][e] = pack2<GRINQH_F16>(ldexpf(bf2f((uint16_t)qf[n][k][e]), up), ldexpf(bf2f((uint16_t)(qf[n][k][e] >> 16)), up));
        factor[n] = bounded(ldexpf(factor[n], -up));
      }
    }

    float m[NB], l[NB], slack[NB];
    float4v o[NB][VC];
    int ev[NB];                              // of the values' scales that the row has seen (8-bit cache)
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      m[n] = -INFINITY; l[n] = 0; ev[n] = kLowestExponent; slack[n] = kSlack<FORMAT>;
#pragma unroll
      for (int j = 0; j < VC; ++j) o[n][j] = float4v{0, 0, 0, 0};
    }

    // ---- where virtual tile v's tokens lie: their page ids a tile ahead, then their addresses
    const int* table = b.table + (long)s * b.width;
    auto start = [&](int v) { return v < v_end ? span.tile(v) * kTile : 0x7fffffc0; };   // its first token
    // lane's token: of the tile (SMALL), else the first of its block of 16 (lanes 0 and 16 are asked)
    auto page_id = [&](int v) {
      const int t = start(v) + (SMALL ? lane & 31 : lane & 16);
      return t < span.hi ? load_global<int>(table + (t >> c.shift)) : -1;
    };
    const char* kp[2];
    const char* vp[2];
    const float* ksp[2];
    const float* vsp[2];
    float ks1 = 0, vs1 = 0;
    auto locate = [&](int v, int id) {
      if constexpr (SMALL) {
        const int t = start(v) + (lane & 31);
        const bool in = t < span.hi, ok = in && (unsigned)id < (unsigned)c.n_pages;
        const long slot = ok ? kv_slot(c, id, h, t) : 0;
        wave_sync();
        if (lane < 32) {
          tok.k[lane] = ok ? c.k + slot * D * ES : (const char*)(in ? g_nans : g_zeros);
          tok.v[lane] = ok ? c.v + slot * D * ES : (const char*)g_zeros;
        }
        if constexpr (I8) {
          ks1 = load_global<float>(ok ? c.ks + slot : (const float*)(in ? g_nans : g_zeros));
          vs1 = load_global<float>(ok ? c.vs + slot : (const float*)g_zeros);
        }
        wave_sync();
      } else {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int t = start(v) + 16 * x, pid = __builtin_amdgcn_readlane(id, 16 * x);
          const bool in = t < span.hi, ok = in && (unsigned)pid < (unsigned)c.n_pages;
          const long slot = ok ? kv_slot(c, pid, h, t) : 0;
          kp[x] = ok ? c.k + slot * (D * ES) : (const char*)(in ? g_nans : g_zeros);
          vp[x] = ok ? c.v + slot * (D * ES) : (const char*)g_zeros;
          if constexpr (I8) {
            ksp[x] = ok ? c.ks + slot : (const float*)(in ? g_nans : g_zeros);
            vsp[x] = ok ? c.vs + slot : (const float*)g_zeros;
          }
        }
      }
    };
    u32x4 kr[2][KL];
    Words<VW> vr[8];
    float4v kst[2], vst[2];                  // scales of this lane's tokens 16 t + 4 quad ..+ 3
    auto load_k = [&] {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* p = SMALL ? tok.k[16 * t + i16] + 16 * quad : kp[t] + (uint32_t)(i16 * D * ES + 16 * quad);
#pragma unroll
        for (int k = 0; k < KL; ++k) kr[t][k] = load_global<u32x4>(p + 64 * k);
      }
    };
    auto load_v = [&] {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int tk = 4 * quad + (j & 3);
        const char* p = SMALL ? tok.v[4 * (j & 4) + tk] + i16 * VC * ES : vp[j >> 2] + (uint32_t)((4 * quad * D + i16 * VC) * ES);
        vr[j] = load_words<VW>(p + (SMALL ? 0 : (j & 3) * D * ES));
      }
      if constexpr (I8 && !SMALL) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          kst[t] = load_global<float4s>((const char*)ksp[t] + (uint32_t)(16 * quad));
          vst[t] = load_global<float4s>((const char*)vsp[t] + (uint32_t)(16 * quad));
        }
      }
    };

    if (v0 < v_end) {
      locate(v0, page_id(v0));
      load_k();
      load_v();
    }
    int next_id = page_id(v0 + WAVES);
#pragma unroll 1
    for (int v = v0; v < v_end; v += WAVES) {
      // ---- S^T = K Q^T
      float4v sc[NB][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int n = 0; n < NB; ++n) sc[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          u32x4 f;
          if constexpr (I8) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              f[e] = codes2(kr[t][k >> 1][2 * (k & 1) + (e >> 1)] ^ 0x80808080u, 2 * (e & 1), 2 * (e & 1) + 1);
          } else {
            f = kr[t][k];
          }
#pragma unroll
          for (int n = 0; n < NB; ++n) sc[n][t] = mfma16<I8 ? GRINQH_KV_F16 : FORMAT>(f, qf[n][k], sc[n][t]);
        }
      }
      if constexpr (I8 && SMALL) {
        wave_sync();
        if (lane < 32) { tok.ks[lane] = ks1; tok.vs[lane] = vs1; }
        wave_sync();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          kst[t] = *(const float4v*)&tok.ks[16 * t + 4 * quad];
          vst[t] = *(const float4v*)&tok.vs[16 * t + 4 * quad];
        }
      }
      const int t0 = start(v);
      const bool masked = !all_visible(a, first, last, t0, kTile);
      // ---- the next tile's K
      locate(v + WAVES, next_id);
      load_k();
      next_id = page_id(v + 2 * WAVES);
      // ---- softmax
      u32x4 pf[NB];
      uint32_t vis[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        vis[n] = 0xffu;
        float vmax = 0;
        if constexpr (I8) {
#pragma unroll
          for (int t = 0; t < 2; ++t) sc[n][t] *= kst[t];
#pragma unroll
          for (int e = 0; e < 8; ++e) vmax = fmaxf(vmax, vst[e >> 2][e & 3]);
        }
        if (masked) {
          vis[n] = 0;
          vmax = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const int tk = t0 + 16 * (e >> 2) + 4 * quad + (e & 3);
            const bool see = row_sees(tk, pos[n], behind[n], a.sinks);
            vis[n] |= see ? 1u << e : 0u;
            sc[n][e >> 2][e & 3] = see ? sc[n][e >> 2][e & 3] : -INFINITY;
            if constexpr (I8) vmax = fmaxf(vmax, see ? vst[e >> 2][e & 3] : 0.0f);
          }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, sc[n][e >> 2][e & 3]);
        mx = rounded_product(max_xor16(max_xor32(mx)), factor[n]);
        const int big = I8 ? scale_exponent(max_xor16(max_xor32(vmax))) : kLowestExponent;
        // what a row is held against follows its own scores and values alone: other rows, and what
        // they see, never change its bits
        const bool grows = I8 && big > ev[n];
        float held = m[n];
        if (__any(mx > m[n] + slack[n] || grows)) {
          const bool rises = mx - m[n] > kSlack<FORMAT>;
          const float was = m[n];
          if (rises) m[n] = held_against<FORMAT>(mx);
          float alpha = rises ? exp2f(was - m[n]) : 1.0f;
          l[n] *= alpha;
          if (grows) { alpha *= ldexpf(1.0f, max(ev[n] - big, -126)); ev[n] = big; }
#pragma unroll
          for (int j = 0; j < VC; ++j) o[n][j] *= alpha;
          held = m[n];
          slack[n] = far_out(held) ? -INFINITY : kSlack<FORMAT>;
          if (far_out(held)) {   // what exp2 is to see, over the factor that it will be multiplied by
            const float inv = inverse(factor[n]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[n][e >> 2][e & 3] = (rounded_product(sc[n][e >> 2][e & 3], factor[n]) - held) * inv;
            held = 0;
          }
        }
        const float down = I8 ? ldexpf(1.0f, kUp - ev[n]) : 1.0f;
        const float base = held == -INFINITY ? 0.0f : held;
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(sc[n][e >> 2][e & 3], factor[n], -base));
          l[n] += p[e];
          if constexpr (I8) p[e] *= vst[e >> 2][e & 3] * down;
        }
        if constexpr (I8) {
          if (masked) {   // a scale that is not finite stays with the rows that see it
#pragma unroll
            for (int e = 0; e < 8; ++e) p[e] = vis[n] >> e & 1 ? p[e] : 0.0f;
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[n][e] = pack2<FORMAT == GRINQH_KV_BF16 ? GRINQH_BF16 : GRINQH_F16>(p[2 * e], p[2 * e + 1]);
      }
      // ---- O^T += V^T P^T
      bool odd = false;   // values that are not finite, in a tile that not all rows see whole
      if constexpr (!I8) {
        if (masked) {
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int w = 0; w < VW; ++w) top = max_halves(top, vr[j].w[w] & 0x7fff7fffu);
          odd = __any(not_finite<FORMAT>(top) != 0);
        }
      }
#pragma unroll
      for (int j = 0; j < VC; ++j) {
        u32x4 f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if constexpr (I8) {
            // byte j of two tokens, as fp16 subnormals 2^-24 (code + 128); times 2^15 less 2^-2: code 2^-9
            const uint32_t x = vr[2 * e].w[j >> 2] ^ 0x80808080u, y = vr[2 * e + 1].w[j >> 2] ^ 0x80808080u;
            const uint32_t u = __builtin_amdgcn_perm(y, x, (uint32_t)(j & 3) | 0x0c00u | (uint32_t)((j & 3) + 4) << 16 | 0x0c000000u);
            const half2 up = {(_Float16)32768.0f, (_Float16)32768.0f}, off = {(_Float16)-0.25f, (_Float16)-0.25f};
            f[e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(half2, u), up, off));
          } else {
            f[e] = __builtin_amdgcn_perm(vr[2 * e + 1].w[j >> 1], vr[2 * e].w[j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
          }
        }
        if (I8 || !odd) {
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][j] = mfma16<I8 ? GRINQH_KV_F16 : FORMAT>(f, pf[n], o[n][j]);
        } else if constexpr (!I8) {
          // 0 times an infinity must not reach rows that do not see it: the finite values as ever, then
          // how many infinities of either sign (a NaN counts as both) a row sees
          constexpr uint32_t one = FORMAT == GRINQH_KV_F16 ? 0x3c00u : 0x3f80u;
          u32x4 fine, inf[2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            fine[e] = f[e] & ~not_finite<FORMAT>(f[e]);
            inf[0][e] = infinite_ones<FORMAT>(f[e], 0);
            inf[1][e] = infinite_ones<FORMAT>(f[e], 1);
          }
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            u32x4 seen;
#pragma unroll
            for (int e = 0; e < 4; ++e) seen[e] = (vis[n] >> (2 * e) & 1 ? one : 0u) | (vis[n] >> (2 * e) & 2 ? one << 16 : 0u);
            o[n][j] = mfma16<FORMAT>(fine, pf[n], o[n][j]);
#pragma unroll
            for (int sign = 0; sign < 2; ++sign) {
              const float4v count = mfma16<FORMAT>(inf[sign], seen, float4v{0, 0, 0, 0});
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][j][e] += count[e] > 0 ? (sign ? -INFINITY : INFINITY) : 0.0f;
            }
          }
        }
      }
      load_v();
    }

    // ---- the waves' results meet
    const DenseRows out = late().out;
    const Partial part = late().part;
    float* lse = late().lse;
    float up[NB];   // what brings the sums over the values back
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      l[n] = sum_xor16(sum_xor32(l[n]));
      up[n] = I8 ? ldexpf(1.0f, ev[n]) : 1.0f;
      if (quad == 0) { lds.m[wave][16 * n + i16] = m[n]; lds.l[wave][16 * n + i16] = l[n]; }
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      __syncthreads();
      float top = -INFINITY;
      for (int w = 0; w < WAVES; ++w) top = fmaxf(top, lds.m[w][16 * n + i16]);
      const float base = top == -INFINITY ? 0.0f : top, f = exp2f(m[n] - base);   // 0 for a wave that saw nothing; a NaN passes
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VC; ++j)
          lds.o[wave][i16][VC * (4 * quad + e) + j] = o[n][j][e] * up[n] * f;
      __syncthreads();
      // CH channels of a row per thread
      constexpr int CH = 16 * D / (64 * WAVES) > 2 ? 16 * D / (64 * WAVES) : 2;
      const int rr = threadIdx.x / (D / CH), ch = (threadIdx.x % (D / CH)) * CH, r = r0 + 16 * n + rr;
      if (rr < 16 && r < all) {
        float rm = -INFINITY, rl = 0, y[CH] = {};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) rm = fmaxf(rm, lds.m[w][16 * n + rr]);
        const float rb = rm == -INFINITY ? 0.0f : rm;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          rl += lds.l[w][16 * n + rr] * exp2f(lds.m[w][16 * n + rr] - rb);
#pragma unroll
          for (int j = 0; j < CH; ++j) y[j] += lds.o[w][rr][ch + j];
        }
        const float inv = rl == 0 ? 0.0f : 1.0f / rl;
        const int rw = sq.r0 + r / a.G, hd = h * a.G + r % a.G;
        const long at = (long)rw * a.heads + hd;
        const float lse2 = rl == 0 ? -INFINITY : rm + log2f(rl);
        if (used > 1) {
          if (ch == 0) part.lse[split * part.rows + at] = lse2;
          if (lse2 != -INFINITY) {
            float* p = part.o + (split * part.rows + at) * D + ch;
#pragma unroll
            for (int j = 0; j < CH; ++j) p[j] = y[j] * inv;
          }
        } else {
          if (lse && ch == 0) lse[at] = lse2 * kLn2;
          uint32_t* p = (uint32_t*)(out.p + (rw * out.row + hd * out.head + ch) * 2);
#pragma unroll
          for (int j = 0; j < CH / 2; ++j) p[j] = pack2<TYPE>(y[2 * j] * inv, y[2 * j + 1] * inv);
        }
      }
    }
    __syncthreads();
  }
}

template <int D, int FORMAT, int TYPE>
void go(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  const dim3 grid(args.c.H * p.splits, p.blocks, args.b.B);
  auto run = [&](auto nb, auto small) {
    constexpr int NB = decltype(nb)::value;
    k_attend_rows<D, FORMAT, TYPE, NB, decltype(small)::value>
        <<<grid, 64 * rows_waves(NB), 0, s>>>(args);
  };
  if (args.c.shift >= 4) {
    if (p.nb == 1) run(std::integral_constant<int, 1>{}, std::false_type{});
    else run(std::integral_constant<int, 2>{}, std::false_type{});
  } else {
    if (p.nb == 1) run(std::integral_constant<int, 1>{}, std::true_type{});
    else run(std::integral_constant<int, 2>{}, std::true_type{});
  }
}

}  // namespace

void launch_attend_rows(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
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
