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
// The next tile's K is loaded while the softmax runs, its V behind the second product.
#include "attend.h"

namespace grinqh {

namespace {

constexpr int kWaves = 4;
constexpr int kTile = 32;

// What a token that is not there reads: zeros past the last token, NaN for a page id out of range.
__device__ const uint32_t g_filler[2][64] = {
    {0},
    {0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff,
     0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff, 0x7fff7fff}};

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

__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// LDS of one wave: where the tile's 32 tokens lie, and their scales.
struct alignas(16) WaveTokens {
  const char* k[kTile];
  const char* v[kTile];
  float ks[kTile];
  float vs[kTile];
};

template <int D, int NB>
struct RowsLds {
  WaveTokens tokens[kWaves];
  float m[kWaves][16 * NB], l[kWaves][16 * NB];
  float o[kWaves][16][D + 4];   // one block of 16 rows at a time
};

template <int W>
struct Words { uint32_t w[W]; };

template <int W>
__device__ __forceinline__ Words<W> load_words(const char* p) {
  Words<W> r;
  if constexpr (W == 1) r.w[0] = *(const uint32_t*)p;
  else if constexpr (W == 2) { const u32x2 x = *(const u32x2*)p; r.w[0] = x[0]; r.w[1] = x[1]; }
  else { const u32x4 x = *(const u32x4*)p; for (int i = 0; i < 4; ++i) r.w[i] = x[i]; }
  return r;
}

template <int D, int FORMAT, int TYPE, int NB>
__global__ __launch_bounds__(64 * kWaves) void k_attend_rows(KvCache c, KvBatch b, Attend a, DenseRows q, DenseRows out,
                                                             float* lse, Partial part, int splits, int per_split) {
  constexpr bool I8 = FORMAT == GRINQH_KV_I8;
  constexpr int ES = I8 ? 1 : 2;             // bytes of a cached value
  constexpr int KS = D / 32;                 // steps of the first product
  constexpr int KL = I8 ? D / 64 : D / 32;   // 16-byte loads of a K row per lane
  constexpr int VC = D / 16;                 // channels of V per lane, blocks of the second product
  constexpr int VW = VC * ES / 4;            // dwords of those
  __shared__ RowsLds<D, NB> lds;

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, quad = lane >> 4;
  const int h = blockIdx.x % c.H, split = blockIdx.x / c.H, s = blockIdx.z;
  const Seq sq = kv_seq(c, b, s);
  const int all = sq.n * a.G;                // rows of this kv head
  WaveTokens& tok = lds.tokens[wave];

  for (int r0 = blockIdx.y * 16 * NB; r0 < all; r0 += gridDim.y * 16 * NB) {
    const int first = sq.L - sq.n + r0 / a.G, last = sq.L - sq.n + min(r0 + 16 * NB - 1, all - 1) / a.G;
    const Span span = attend_span<kTile>(a, first, last);
    const int v_end = split == splits - 1 ? span.tiles : min(span.tiles, (split + 1) * per_split);
    const int v0 = split * per_split + wave;

    // this lane's rows and their queries
    int pos[NB], row[NB], head[NB];
    float factor[NB];
    u32x4 qf[NB][KS];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int r = min(r0 + 16 * n + i16, all - 1);   // rows past the last repeat it and are not stored
      row[n] = sq.r0 + r / a.G;
      head[n] = h * a.G + r % a.G;
      pos[n] = sq.L - sq.n + r / a.G;
      const char* qp = q.p + (row[n] * q.row + head[n] * q.head) * 2;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int d = I8 ? (k >> 1) * 64 + 16 * quad + 8 * (k & 1) : 32 * k + 8 * quad;
        qf[n][k] = *(const u32x4*)(qp + 2 * d);
      }
      factor[n] = a.scale * kLog2e;
      if constexpr (I8 && TYPE == GRINQH_BF16) {
        float amax = 0;
        bool bad = false;
        for (int k = 0; k < KS; ++k)
          for (int e = 0; e < 8; ++e) {
            const float x = bf2f((uint16_t)(qf[n][k][e >> 1] >> (16 * (e & 1))));
            bad |= !(fabsf(x) < INFINITY);
            amax = fmaxf(amax, fabsf(x));
          }
        if (bad) amax = INFINITY;
        amax = max_xor16(max_xor32(amax));
        const int up = row_shift(amax);
        for (int k = 0; k < KS; ++k)
          for (int e = 0; e < 4; ++e)
            qf[n][k][e] = pack2<GRINQH_F16>(ldexpf(bf2f((uint16_t)qf[n][k][e]), up), ldexpf(bf2f((uint16_t)(qf[n][k][e] >> 16)), up));
        factor[n] = ldexpf(factor[n], -up);
      }
    }

    float m[NB], l[NB];
    float4v o[NB][VC];
    int ev[NB];                              // of the values' scales that the row has seen (8-bit cache)
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      m[n] = -INFINITY; l[n] = 0; ev[n] = kLowestExponent;
#pragma unroll
      for (int j = 0; j < VC; ++j) o[n][j] = float4v{0, 0, 0, 0};
    }

    // token lane % 32 of virtual tile v: its page id (kept a tile ahead), then where it lies
    const int* table = b.table + (long)s * b.width;
    auto token = [&](int v) { return v < v_end ? span.tile(v) * kTile + (lane & 31) : 0x7fffffff; };
    auto page_id = [&](int v) { const int t = token(v); return t < span.hi ? table[t >> c.shift] : -1; };
    float ks = 0, vs = 0;
    auto locate = [&](int v, int id) {
      const int t = token(v);
      const bool in = t < span.hi, ok = in && (unsigned)id < (unsigned)c.n_pages;
      const long slot = ok ? kv_slot(c, id, h, t) : 0;
      wave_sync();
      if (lane < 32) {
        tok.k[lane] = ok ? c.k + slot * D * ES : (const char*)g_filler[in ? 1 : 0];
        tok.v[lane] = ok ? c.v + slot * D * ES : (const char*)g_filler[0];
      }
      if constexpr (I8) {
        const float* filler = (const float*)g_filler[in ? 1 : 0];
        ks = ok ? c.ks[slot] : *filler;
        vs = ok ? c.vs[slot] : 0.0f;
      }
      wave_sync();
    };
    u32x4 kr[2][KL];
    Words<VW> vr[8];
    auto load_k = [&] {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const char* p = tok.k[16 * t + i16];
#pragma unroll
        for (int k = 0; k < KL; ++k) kr[t][k] = *(const u32x4*)(p + 64 * k + 16 * quad);
      }
    };
    auto load_v = [&] {
#pragma unroll
      for (int j = 0; j < 8; ++j) vr[j] = load_words<VW>(tok.v[(j & 4) * 4 + 4 * quad + (j & 3)] + i16 * VC * ES);
    };

    if (v0 < v_end) {
      locate(v0, page_id(v0));
      load_k();
      load_v();
    }
    int next_id = page_id(v0 + kWaves);
    for (int v = v0; v < v_end; v += kWaves) {
      // ---- S^T = K Q^T
      float4v sc[NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          sc[n][t] = float4v{0, 0, 0, 0};
        }
#pragma unroll
      for (int t = 0; t < 2; ++t)
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
      // ---- this tile's scales, then the next tile's K
      float kst[2][4], vst[2][4];
      if constexpr (I8) {
        wave_sync();
        if (lane < 32) { tok.ks[lane] = ks; tok.vs[lane] = vs; }
        wave_sync();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const float4v kk = *(const float4v*)&tok.ks[16 * t + 4 * quad], vv = *(const float4v*)&tok.vs[16 * t + 4 * quad];
#pragma unroll
          for (int e = 0; e < 4; ++e) { kst[t][e] = kk[e]; vst[t][e] = vv[e]; }
        }
      }
      const int t0 = span.tile(v) * kTile;
      const bool whole = all_visible(a, first, last, t0, kTile);
      locate(v + kWaves, next_id);
      load_k();
      next_id = page_id(v + 2 * kWaves);
      // ---- softmax
      u32x4 pf[NB], seen[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        bool vis[2][4];
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = sc[n][t][e];
            if constexpr (I8) x *= kst[t][e];
            if (!whole) {
              const int tk = t0 + 16 * t + 4 * quad + e;
              vis[t][e] = tk <= pos[n] && (!a.window || tk > pos[n] - a.window || tk < a.sinks);
              if (!vis[t][e]) x = -INFINITY;
            }
            sc[n][t][e] = x;
            mx = fmaxf(mx, x);
          }
        mx = max_xor16(max_xor32(mx)) * factor[n];
        int big = kLowestExponent;
        if constexpr (I8) {
          float vmax = 0;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) vmax = fmaxf(vmax, (whole || vis[t][e]) && vst[t][e] < INFINITY ? vst[t][e] : 0.0f);
          big = scale_exponent(max_xor16(max_xor32(vmax)));
        }
        // what a row is held against follows its own scores and values alone: other rows, and what
        // they see, never change its bits
        const bool rises = mx > m[n] + kSlack, grows = I8 && big > ev[n];
        if (__any(rises || grows)) {
          float alpha = rises ? exp2f(m[n] - mx) : 1.0f;
          if (rises) m[n] = mx;
          l[n] *= alpha;
          if (grows) { alpha *= ldexpf(1.0f, max(ev[n] - big, -126)); ev[n] = big; }
#pragma unroll
          for (int j = 0; j < VC; ++j) o[n][j] *= alpha;
        }
        const float base = m[n] == -INFINITY ? 0.0f : m[n], down = I8 ? ldexpf(1.0f, kUp - ev[n]) : 1.0f;
        float p[8];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = __builtin_amdgcn_exp2f(fmaf(sc[n][t][e], factor[n], -base));
            l[n] += x;
            if constexpr (I8) {
              x *= vst[t][e] * down;
              if (!whole && !vis[t][e]) x = 0;   // a scale that is not finite stays with the rows that see it
            }
            p[4 * t + e] = x;
          }
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[n][e] = pack2<FORMAT == GRINQH_KV_BF16 ? GRINQH_BF16 : GRINQH_F16>(p[2 * e], p[2 * e + 1]);
        if constexpr (!I8) {
          if (!whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              constexpr uint32_t one = FORMAT == GRINQH_KV_F16 ? 0x3c00u : 0x3f80u;
              seen[n][e] = (vis[e >> 1][2 * (e & 1)] ? one : 0u) | (vis[e >> 1][2 * (e & 1) + 1] ? one << 16 : 0u);
            }
          }
        }
      }
      // ---- O^T += V^T P^T
      bool odd = false;   // values that are not finite, in a tile that not all rows see whole
      if constexpr (!I8) {
        if (!whole) {
          uint32_t any = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            for (int w = 0; w < VW; ++w) any |= not_finite<FORMAT>(vr[j].w[w]);
          odd = __any(any != 0);
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
        if constexpr (I8) {
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][j] = mfma16<GRINQH_KV_F16>(f, pf[n], o[n][j]);
        } else if (!odd) {
#pragma unroll
          for (int n = 0; n < NB; ++n) o[n][j] = mfma16<FORMAT>(f, pf[n], o[n][j]);
        } else {
          // 0 times an infinity must not reach rows that do not see it: the finite values as ever, then
          // how many infinities of either sign (a NaN counts as both) a row sees
          u32x4 fine, inf[2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            fine[e] = f[e] & ~not_finite<FORMAT>(f[e]);
            inf[0][e] = infinite_ones<FORMAT>(f[e], 0);
            inf[1][e] = infinite_ones<FORMAT>(f[e], 1);
          }
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            o[n][j] = mfma16<FORMAT>(fine, pf[n], o[n][j]);
#pragma unroll
            for (int sign = 0; sign < 2; ++sign) {
              const float4v count = mfma16<FORMAT>(inf[sign], seen[n], float4v{0, 0, 0, 0});
#pragma unroll
              for (int e = 0; e < 4; ++e) o[n][j][e] += count[e] > 0 ? (sign ? -INFINITY : INFINITY) : 0.0f;
            }
          }
        }
      }
      load_v();
    }

    // ---- the waves' results meet
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
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.m[w][16 * n + i16]);
      const float base = top == -INFINITY ? 0.0f : top, f = exp2f(m[n] - base);   // 0 for a wave that saw nothing; a NaN passes
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int j = 0; j < VC; ++j)
          lds.o[wave][i16][VC * (4 * quad + e) + j] = o[n][j][e] * up[n] * f;
      __syncthreads();
      // 16 lanes per row, D / 16 channels each
      const int rr = threadIdx.x / 16, ch = (threadIdx.x % 16) * VC, r = r0 + 16 * n + rr;
      if (r < all) {
        float rm = -INFINITY, rl = 0;
        for (int w = 0; w < kWaves; ++w) rm = fmaxf(rm, lds.m[w][16 * n + rr]);
        const float rb = rm == -INFINITY ? 0.0f : rm;
        for (int w = 0; w < kWaves; ++w) rl += lds.l[w][16 * n + rr] * exp2f(lds.m[w][16 * n + rr] - rb);
        float y[VC];
#pragma unroll
        for (int j = 0; j < VC; ++j) {
          float x = 0;
          for (int w = 0; w < kWaves; ++w) x += lds.o[w][rr][ch + j];
          y[j] = rl == 0 ? 0.0f : x / rl;
        }
        const int rw = sq.r0 + r / a.G, hd = h * a.G + r % a.G;
        const long at = (long)rw * a.heads + hd;
        const float lse2 = rl == 0 ? -INFINITY : rm + log2f(rl);
        if (splits > 1) {
          if (ch == 0) part.lse[split * part.rows + at] = lse2;
          if (lse2 != -INFINITY) {
            float* p = part.o + (split * part.rows + at) * D + ch;
#pragma unroll
            for (int j = 0; j < VC; j += 4) *(float4v*)(p + j) = float4v{y[j], y[j + 1], y[j + 2], y[j + 3]};
          }
        } else {
          if (lse && ch == 0) lse[at] = lse2 * kLn2;
          char* p = out.p + (rw * out.row + hd * out.head + ch) * 2;
          uint32_t w[VC / 2];
#pragma unroll
          for (int j = 0; j < VC / 2; ++j) w[j] = pack2<TYPE>(y[2 * j], y[2 * j + 1]);
          if constexpr (VC == 8) *(u32x4*)p = u32x4{w[0], w[1], w[2], w[3]};
          else *(u32x2*)p = u32x2{w[0], w[1]};
        }
      }
    }
    __syncthreads();
  }
}

template <int D, int FORMAT, int TYPE>
void go(const AttendPlan& p, const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q, const DenseRows& out,
        float* lse, const Partial& part, hipStream_t s) {
  const dim3 grid(c.H * p.splits, p.blocks, b.B);
  if (p.nb == 1) k_attend_rows<D, FORMAT, TYPE, 1><<<grid, 64 * kWaves, 0, s>>>(c, b, a, q, out, lse, part, p.splits, p.per_split);
  else k_attend_rows<D, FORMAT, TYPE, 2><<<grid, 64 * kWaves, 0, s>>>(c, b, a, q, out, lse, part, p.splits, p.per_split);
}

}  // namespace

void launch_attend_rows(const AttendPlan& p, const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q,
                        const DenseRows& out, float* lse, const Partial& part, hipStream_t s) {
  auto on = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (c.format == GRINQH_KV_F16) go<D, GRINQH_KV_F16, GRINQH_F16>(p, c, b, a, q, out, lse, part, s);
    else if (c.format == GRINQH_KV_BF16) go<D, GRINQH_KV_BF16, GRINQH_BF16>(p, c, b, a, q, out, lse, part, s);
    else if (a.type == GRINQH_F16) go<D, GRINQH_KV_I8, GRINQH_F16>(p, c, b, a, q, out, lse, part, s);
    else go<D, GRINQH_KV_I8, GRINQH_BF16>(p, c, b, a, q, out, lse, part, s);
  };
  if (c.D == 64) on(std::integral_constant<int, 64>{});
  else on(std::integral_constant<int, 128>{});
}

}  // namespace grinqh
