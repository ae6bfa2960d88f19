// Attention of a few rows over a long 4-bit cache: k_attend_rows (attend_rows.hip) for codes with a step and a base per group.
//
// The same plan: rows are the columns of S^T = K Q^T and O^T = V^T P^T, a wave walks its own tiles of 32 tokens, nothing of K
// or V goes through LDS.  What the format asks for:
//   - codes become the fp16 values that they stand for in registers: a byte 0000cccc read as an 8-bit float of 4 exponent and 3
//     mantissa bits is c 2^-9, subnormal or not, so one conversion makes two exact codes, and a packed multiply-add with step and
//     base rounds once, as the format's definition does.  Eight values are 11 instructions (with masks beside an exponent and a
//     subtraction 13: 131072 tokens took 34.4 us).
//   - a lane holds a quarter of a K row, which one group covers (a half of it at 64 channels), so the row is one load of codes and
//     one of step and base; the first product's contraction runs over the quarters' words.
//   - of V a lane holds one word (a half at 64 channels) of each of its eight tokens.  Halves of two tokens' words are put side by
//     side before they are decoded, so what comes out is the operand.  The four lanes of a group load the steps and bases of
//     four tokens between them and pass them round by DPP.
//   - pages of 16 tokens or more are read by buffer loads: base and size are scalar, a page that is not there has size 0 and reads
//     as zeros without an access, and a lane's offsets are the same for all tiles.
// A tile's loads are issued a whole tile ahead, into the other of two sets of registers, and the page ids of the one after it
// before them (a microsecond in 32).
//
// Registers: one block of 16 rows a wave, which decoding uses, takes 128 to 192 and nothing in scratch.  Two blocks of 128 channels
// have all 256 and keep 15 to 30 more in scratch, of which every tile reads some again: 10 to 12 with pages of 32 tokens and more or
// of less than 16, 4 to 6 with pages of 16.
//
// Bound by memory, and by vector instructions close behind: one token of 32 heads over 131072 tokens of 8 kv heads of 128 (168 MB)
// takes 30.6 us, 5.5 TB/s, where a large read reaches 6.9; its loads alone took 26.2 and everything but the loads, still with the
// older conversions, 28.8.  32 sequences of up to 8191 tokens in pages of 16 take 47: unequal lengths.
#include "attend.h"

namespace grinqh {

namespace {

constexpr int kTile = 32;

// LDS of one wave: where the tile's 32 tokens lie, and their groups (pages under 16 tokens).
struct WaveTokens4 {
  const char* k[kTile];
  const char* v[kTile];
  const char* kg[kTile];
  const char* vg[kTile];
};

template <int D, int NB, int WAVES, bool SMALL>
struct Rows4Lds {
  WaveTokens4 tokens[SMALL ? WAVES : 1];
  float m[WAVES][16 * NB], l[WAVES][16 * NB];
  float o[WAVES][16][D + 4];   // one block of 16 rows at a time
};

// PAGES: of 32 tokens and more (2): a tile lies in one; of 16 (1): in two; smaller ones (0) are looked up by the lanes.
template <int D, int TYPE, int NB, int PAGES>
__global__ __launch_bounds__(64 * rows_waves(NB)) __attribute__((amdgpu_waves_per_eu(rows_per_simd(GRINQH_KV_I4, NB))))
void k_attend_rows4(AttendArgs args) {
  constexpr int F4 = GRINQH_KV_I4;
  constexpr bool SMALL = PAGES == 0;
  const KvCache& c = args.c;
  const KvBatch& b = args.b;
  const Attend& a = args.a;
  const int splits = args.splits, per_split = args.per_split;
  constexpr int RB = D / 2;                  // bytes of a row's codes
  constexpr int GB = D / kKvGroup * 4;       // and of its steps and bases
  constexpr int KS = D / 32;                 // words of a lane's quarter of a K row, steps of the first product
  constexpr int VC = D / 16;                 // channels of V per lane, blocks of the second product
  constexpr int WAVES = rows_waves(NB);
  __shared__ Rows4Lds<D, NB, WAVES, SMALL> lds;

  const int lane = threadIdx.x & 63, i16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int h = blockIdx.x % c.H, split = blockIdx.x / c.H, s = blockIdx.z;
  const Seq sq = kv_seq(c, b, s);
  const int all = sq.n * a.G;                // rows of this kv head
  WaveTokens4& tok = lds.tokens[SMALL ? wave : 0];
  // this lane's group in a row of K, whose quarter it holds, and of V; the channel of the j-th value of V in lane i
  const int k_group = quad * (D / 4) / kKvGroup, v_group = i16 * VC / kKvGroup;
  auto channel = [](int i, int j) { return D == 64 ? 8 * (i >> 1) + (i & 1) + 2 * j : 8 * i + j; };
  // byte offsets in the 16 tokens of a page
  const int k_at = i16 * RB + 4 * KS * quad, kg_at = i16 * GB + 4 * k_group;
  const int v_at = 4 * quad * RB + i16 * (VC / 2), vg_at = (4 * quad + (i16 & 3)) * GB + 4 * v_group;
  const uint32_t steps_or_bases = lane & 1 ? 0x03020706u : 0x05040100u;
  // what is made of such a value inside a branch stays there: before the loop it would hold registers
  auto rarely = [](int x) { asm volatile("" : "+v"(x)); return x; };

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
      for (int k = 0; k < KS; ++k) qf[n][k] = mix8(*(const u32x4*)(qp + 2 * (D / 4 * quad + 8 * k)));
      factor[n] = bounded(a.scale * kLog2e);
      if constexpr (TYPE == GRINQH_BF16) {
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
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      m[n] = -INFINITY; l[n] = 0; slack[n] = kSlack<F4>;
#pragma unroll
      for (int j = 0; j < VC; ++j) o[n][j] = float4v{0, 0, 0, 0};
    }

    // ---- a tile's loads
    const int* table = b.table + (long)s * b.width;
    auto start = [&](int v) { return v < v_end ? span.tile(v) * kTile : 0x7fffffc0; };   // its first token
    // page id of a lane's token of the tile (SMALL), else of its block of 16 (lanes 0 and 16 are asked), or of the tile
    auto page_id = [&](int v) {
      const int t = start(v) + (SMALL ? lane & 31 : PAGES == 1 ? lane & 16 : 0);
      return t < span.hi ? load_global<int>(table + (t >> c.shift)) : -1;
    };
    uint32_t kr[2][2][KS], kg[2][2], vr[2][8], vg[2][2];   // by set, then block of 16 tokens, or token of this lane
    auto load = [&](int v, int id, auto set_c) __attribute__((always_inline)) {
      constexpr int S = decltype(set_c)::value;
      if constexpr (SMALL) {
        const int t = start(v) + (lane & 31);
        const bool in = t < span.hi, ok = in && (unsigned)id < (unsigned)c.n_pages;
        const long slot = ok ? kv_slot(c, id, h, t) : 0;
        const char* none = (const char*)(in ? g_nans : g_zeros);
        wave_sync();
        if (lane < 32) {
          tok.k[lane] = ok ? c.k + slot * RB : none;
          tok.v[lane] = ok ? c.v + slot * RB : (const char*)g_zeros;
          tok.kg[lane] = ok ? (const char*)c.ks + slot * GB : none;
          tok.vg[lane] = ok ? (const char*)c.vs + slot * GB : (const char*)g_zeros;
        }
        wave_sync();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const char* p = tok.k[16 * t + i16] + 4 * KS * quad;
#pragma unroll
          for (int k = 0; k < KS; ++k) kr[S][t][k] = load_global<uint32_t>(p + 4 * k);
          kg[S][t] = load_global<uint32_t>(tok.kg[16 * t + i16] + 4 * k_group);
          vg[S][t] = load_global<uint32_t>(tok.vg[16 * t + 4 * quad + (i16 & 3)] + 4 * v_group);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const char* p = tok.v[16 * (j >> 2) + 4 * quad + (j & 3)] + i16 * (VC / 2);
          vr[S][j] = D == 64 ? load_global<uint16_t>(p) : load_global<uint32_t>(p);
        }
      } else {
        constexpr int PER = PAGES == 1 ? 1 : 2;   // blocks of 16 tokens that share a page
        __amdgpu_buffer_rsrc_t kb, kgb, vb[2], vgb[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (t % PER == 0) {
            const int t0 = start(v) + 16 * t, pid = PAGES == 1 ? __builtin_amdgcn_readlane(id, 16 * t) : __builtin_amdgcn_readfirstlane(id);
            const bool in = t0 < span.hi, ok = in && (unsigned)pid < (unsigned)c.n_pages;
            const long slot = ok ? kv_slot(c, pid, h, t0) : 0;
            kb = buffer_of(c.k + slot * RB, ok ? 16 * PER * RB : 0);
            // codes of 0 with a step and a base of NaN are NaN
            kgb = buffer_of(ok || !in ? (const char*)c.ks + slot * GB : (const char*)g_nans, in ? 16 * PER * GB : 0);
            vb[t] = buffer_of(c.v + slot * RB, ok ? 16 * PER * RB : 0);
            vgb[t] = buffer_of((const char*)c.vs + slot * GB, ok ? 16 * PER * GB : 0);
          } else {
            vb[t] = vb[0];
            vgb[t] = vgb[0];
          }
          const int block = t % PER * 16;
          if constexpr (D == 64) {
            const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(kb, k_at + block * RB, 0, 0));
            kr[S][t][0] = w[0]; kr[S][t][1] = w[1];
          } else {
            const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(kb, k_at + block * RB, 0, 0));
#pragma unroll
            for (int k = 0; k < KS; ++k) kr[S][t][k] = w[k];
          }
          kg[S][t] = __builtin_amdgcn_raw_buffer_load_b32(kgb, kg_at + block * GB, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (D == 64) vr[S][4 * t + j] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(vb[t], v_at + (t % PER * 16 + j) * RB, 0, 0);
            else vr[S][4 * t + j] = __builtin_amdgcn_raw_buffer_load_b32(vb[t], v_at + (t % PER * 16 + j) * RB, 0, 0);
          }
          vg[S][t] = __builtin_amdgcn_raw_buffer_load_b32(vgb[t], vg_at + t % PER * 16 * GB, 0, 0);
        }
      }
    };

    // ---- a tile: its loads lie in set S, those of the next go to the other one
    int next_id = 0;
    auto tile = [&](int v, auto set_c) __attribute__((always_inline)) {
      constexpr int S = decltype(set_c)::value;
      // the page after the next one's first: loads come in order, and it is waited for without those that follow it
      const int id = page_id(v + 2 * WAVES);
      load(v + WAVES, next_id, std::integral_constant<int, 1 - S>{});
      next_id = id;
      // ---- S^T = K Q^T
      float4v sc[NB][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int n = 0; n < NB; ++n) sc[n][t] = float4v{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const u32x4 f = mixed8(kr[S][t][k], kg[S][t]);
#pragma unroll
          for (int n = 0; n < NB; ++n) sc[n][t] = mfma16<GRINQH_KV_F16>(f, qf[n][k], sc[n][t]);
        }
      }
      const int t0 = start(v);
      const bool masked = !all_visible(a, first, last, t0, kTile);
      // ---- softmax
      u32x4 pf[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        if (masked) {
          const int q4 = rarely(4 * quad);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            sc[n][e >> 2][e & 3] = row_sees(t0 + 16 * (e >> 2) + q4 + (e & 3), pos[n], behind[n], a.sinks) ? sc[n][e >> 2][e & 3] : -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int e = 0; e < 8; ++e) mx = fmaxf(mx, sc[n][e >> 2][e & 3]);
        // what a row is held against follows its own scores alone: other rows, and what they see, never change its bits.  The
        // four lanes of a row meet where one of them has something to say.
        float held = m[n];
        if (__any(rounded_product(mx, factor[n]) > m[n] + slack[n])) {
          mx = rounded_product(max_xor16(max_xor32(mx)), factor[n]);
          const bool rises = mx - m[n] > kSlack<F4>;
          const float was = m[n];
          if (rises) m[n] = held_against<F4>(mx);
          const float alpha = rises ? exp2f(was - m[n]) : 1.0f;
          l[n] *= alpha;
#pragma unroll
          for (int j = 0; j < VC; ++j) o[n][j] *= alpha;
          held = m[n];
          slack[n] = far_out(held) ? -INFINITY : kSlack<F4>;
          if (far_out(held)) {   // what exp2 is to see, over the factor that it will be multiplied by
            const float inv = inverse(factor[n]);
#pragma unroll
            for (int e = 0; e < 8; ++e) sc[n][e >> 2][e & 3] = (rounded_product(sc[n][e >> 2][e & 3], factor[n]) - held) * inv;
            held = 0;
          }
        }
        const float base = held == -INFINITY ? 0.0f : held;
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(sc[n][e >> 2][e & 3], factor[n], -base));
          l[n] += p[e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) pf[n][e] = pack2<GRINQH_F16>(p[2 * e], p[2 * e + 1]);
      }
      // ---- O^T += V^T P^T: tokens 2 e and 2 e + 1 of this lane's eight side by side
      uint32_t w[4][D == 64 ? 1 : 2];   // bytes x, y, x, y: the tokens' first two, and last two
      half2 step[4], base[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e][0] = __builtin_amdgcn_perm(vr[S][2 * e + 1], vr[S][2 * e], 0x05010400u);
        if constexpr (D == 128) w[e][1] = __builtin_amdgcn_perm(vr[S][2 * e + 1], vr[S][2 * e], 0x07030602u);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        // of four lanes with a token each the first makes the first two tokens' steps, the second their bases, and so on; then
        // all four get them (quad_perm)
        const int own = (int)vg[S][t], other = __builtin_amdgcn_update_dpp(0, own, 0xb1, 0xf, 0xf, true);
        const int made = (int)__builtin_amdgcn_perm((uint32_t)other, (uint32_t)own, steps_or_bases);
        step[2 * t] = __builtin_bit_cast(half2, __builtin_amdgcn_update_dpp(0, made, 0x00, 0xf, 0xf, true));
        base[2 * t] = __builtin_bit_cast(half2, __builtin_amdgcn_update_dpp(0, made, 0x55, 0xf, 0xf, true));
        step[2 * t + 1] = __builtin_bit_cast(half2, __builtin_amdgcn_update_dpp(0, made, 0xaa, 0xf, 0xf, true));
        base[2 * t + 1] = __builtin_bit_cast(half2, __builtin_amdgcn_update_dpp(0, made, 0xff, 0xf, 0xf, true));
      }
      // Channels that stand in the low, or the high, nibbles of two of those bytes: operands and products.
      auto products = [&](auto finite_only) __attribute__((always_inline)) {
#pragma unroll
        for (int x = 0; x < VC / 2; ++x) {
          const int half = x >> 1, high = x & 1;
          u32x4 f[2];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t bytes = (high ? w[e][half] >> 4 : w[e][half]) & kLow;
            f[0][e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(codes_of<false>(bytes), step[e], base[e]));
            f[1][e] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(codes_of<true>(bytes), step[e], base[e]));
            if constexpr (decltype(finite_only)::value) {
              f[0][e] &= ~not_finite<GRINQH_KV_F16>(f[0][e]);
              f[1][e] &= ~not_finite<GRINQH_KV_F16>(f[1][e]);
            }
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int j = D == 64 ? high + 2 * y : 2 * (high + 2 * y) + half;
#pragma unroll
            for (int n = 0; n < NB; ++n) o[n][j] = mfma16<GRINQH_KV_F16>(f[y], pf[n], o[n][j]);
          }
          __builtin_amdgcn_sched_barrier(0);   // the operands of one step at a time: registers are scarce
        }
      };
      bool odd = false;   // values that may not be finite, in a tile that not all rows see whole
      if (masked) {       // steps under 2^11 and bases under 2^15 leave 15 step + base finite
        const uint32_t top = max_halves(vg[S][0] & 0x7fff7fffu, vg[S][1] & 0x7fff7fffu);
        odd = __any((top & 0xffffu) >= 0x6800u || (top >> 16) >= 0x7800u);
      }
      if (!odd) {
        products(std::false_type{});
      } else {
        // 0 times an infinity must not reach rows that do not see it: the finite values as ever, then what is not finite, from
        // memory, to the rows that see it
        products(std::true_type{});
#pragma unroll 1
        for (int t = t0; t < t0 + kTile && t < span.hi; ++t) {
          const int qd = rarely(quad), id = load_global<int>(table + (t >> c.shift));
          if ((unsigned)id >= (unsigned)c.n_pages) continue;
          const long slot = kv_slot(c, id, h, t);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int word = D == 64 ? 2 * qd + (e >> 1) : 4 * qd + e;
            const u32x4 v8 = values8(load_global<uint32_t>(c.v + slot * RB + 4 * word),
                                    load_global<uint32_t>((const char*)c.vs + slot * GB + 4 * (word * 8 / kKvGroup)), nibble_masks());
#pragma unroll
            for (int j = 0; j < VC; ++j) {
              const float y = h2f((uint16_t)(D == 64 ? v8[j] >> (16 * (e & 1)) : v8[j >> 1] >> (16 * (j & 1))));
#pragma unroll
              for (int n = 0; n < NB; ++n)
                o[n][j][e] += row_sees(t, pos[n], behind[n], a.sinks) && !(fabsf(y) < INFINITY) ? y : 0.0f;
            }
          }
        }
      }
    };

    if (v0 < v_end) {
      const int id = page_id(v0);
      next_id = page_id(v0 + WAVES);
      load(v0, id, std::integral_constant<int, 0>{});
#pragma unroll 1
      for (int v = v0;;) {
        tile(v, std::integral_constant<int, 0>{});
        if ((v += WAVES) >= v_end) break;
        tile(v, std::integral_constant<int, 1>{});
        if ((v += WAVES) >= v_end) break;
      }
    }

    // ---- the waves' results meet
    const DenseRows out = late().out;
    const Partial part = late().part;
    float* lse = late().lse;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      l[n] = sum_xor16(sum_xor32(l[n]));
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
          lds.o[wave][i16][channel(4 * quad + e, j)] = o[n][j][e] * f;
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

template <int D, int TYPE>
void go(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  const dim3 grid(args.c.H * p.splits, p.blocks, args.b.B);
  auto run = [&](auto pages) {
    constexpr int PAGES = decltype(pages)::value;
    if (p.nb == 1) k_attend_rows4<D, TYPE, 1, PAGES><<<grid, 64 * rows_waves(1), 0, s>>>(args);
    else k_attend_rows4<D, TYPE, 2, PAGES><<<grid, 64 * rows_waves(2), 0, s>>>(args);
  };
  if (args.c.shift >= 5) run(std::integral_constant<int, 2>{});
  else if (args.c.shift == 4) run(std::integral_constant<int, 1>{});
  else run(std::integral_constant<int, 0>{});
}

}  // namespace

void launch_attend_rows4(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  auto on = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (args.a.type == GRINQH_F16) go<D, GRINQH_F16>(p, args, s);
    else go<D, GRINQH_BF16>(p, args, s);
  };
  if (args.c.D == 64) on(std::integral_constant<int, 64>{});
  else on(std::integral_constant<int, 128>{});
}

}  // namespace grinqh
