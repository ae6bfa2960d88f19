// Attention of chunks over a 4-bit cache: many rows.
//
// As k_attend_tile (attend_tile.hip) has it, a workgroup takes 32 rows per wave (token i, head g of one kv head's group) and walks
// tiles of 64 tokens that its waves share through LDS as fp16 rows; S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_32x32x16, rows being
// the columns, so that a lane holds 16 of a block's 32 scores of ONE row and the weights leave the first product where the second
// wants them.  What differs:
//   - codes wait in registers and become rows on their way into LDS (mixed8): eight channels in the order 0, 4, 1, 5, 2, 6, 3, 7, which
//     the queries are brought into, and which is taken back when the results leave.  No scale multiplies a score or a weight.
//   - a wave's own products and softmax run side by side: the scores of tile i + 1 are multiplied while the weights of tile i are
//     made, the values of tile i while the maximum of the next scores is taken and codes become rows.  One wave alone issues a vector
//     instruction every 6 to 9 cycles, two of a SIMD together one every 4, so the waves must not take turns at it.  (Waves half a
//     tile apart, one's products beside the other's softmax, took 3950 cycles a tile at 64 channels for 1080 of vector
//     instructions and 512 of products a wave.)
//   - so one barrier a tile, and two buffers.
// At 64 channels a wave takes 195 to 208 registers; at 128 it has all 256, and 1 to 19 more in scratch (small pages and bf16 rows the
// most), which are read at a workgroup's start and end and not in the tiles' loop: 4096 rows of bf16 take as long as of fp16.
//
// Bound by neither pipe alone.  4096 rows of 32 heads behind 32768 tokens (2.34 Tflop) take 2250 to 2370 us, 990 to 1040 TFLOP/s;
// the products' pipe is busy in 0.47 of the cycles and the vector one in 0.46, which are the same cycles in part only.  6 chunks
// of 28 heads on 4 of 64 channels, window 2048: 67 to 70 us at the card's first clocks, which the next figures are of, 61 after 10 ms
// of work; 1.44 us a tile of 64 tokens and 17 for the call of a few tiles.  What was
// tried and took as long: three K buffers and codes fetched two tiles ahead, operands of both products in one ring, half the
// waves bringing K and half V (2300, 66), the weights summed in two chains (2320, 67).
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

// Physical 16-byte chunk of a row's logical one: neither K's reads, 32 rows at one chunk, nor V's, 4 rows over 64 bytes, conflict.
template <int D>
__device__ __forceinline__ int k_swizzle(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
template <int D>
__device__ __forceinline__ int v_swizzle(int row) { return D == 128 ? (row & 3) << 2 : (row >> 1 & 1) << 2; }

template <int D>
struct Tile4Lds {
  uint8_t k[2][kTile][2 * D];
  uint8_t v[2][kTile][2 * D];
  uint8_t more[8192];   // the rows of the results are padded: they need more than both
  int odd[2][kWaves];   // per wave: what it made of V held a value that is not finite
};

typedef short short4v __attribute__((ext_vector_type(4)));

template <int D, int TYPE, bool SMALL>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void k_attend_tile4(AttendArgs args) {
  constexpr int F4 = GRINQH_KV_I4, MF = GRINQH_KV_F16;
  const KvCache& c = args.c;
  const KvBatch& b = args.b;
  const Attend& a = args.a;
  const int splits = args.splits, per_split = args.per_split;
  constexpr int RB = 2 * D;                         // bytes of a row in LDS
  constexpr int CB = D / 2;                         // of its codes
  constexpr int GB = D / kKvGroup * 4;              // and of its steps and bases
  constexpr int WORDS = D / 64;                     // words of codes of a lane: eight lanes a row
  constexpr int RPW = 8;                            // rows of a wave
  constexpr int KS = D / 16, VB = D / 32;
  __shared__ __attribute__((aligned(1024))) Tile4Lds<D> lds;

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
      for (int k = 0; k < KS; ++k) qf[k] = mix8(*(const u32x4*)(qp + 32 * k));
      if constexpr (TYPE == GRINQH_BF16) {
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

    float m = -INFINITY, l = 0, slack = kSlack<F4>;
    float16v o[VB];
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[j][e] = 0;

    // ---- staging: lane x of wave w has words WORDS (x % 8) .. of row 8 w + x / 8 of the tile.  A wave's eight rows lie in one page of
    // 16 tokens or more, whose address is scalar; smaller ones (SMALL) are looked up by the lanes.
    const int N = v_end - v0;                // tiles, counted from 0 from here on
    auto start = [&](int i) { const int v = v0 + i; return i < N ? span.tile(v) * kTile : 0x7fffffc0; };
    const int my_row = lane / 8, my_chunk = lane % 8, tile_row = RPW * wave + my_row;
    auto row_at = [&](int i) { return start(i) + RPW * wave + (SMALL ? my_row : 0); };
    // A scalar load whatever the compiler knows of other arrays: one into a vector register would be waited for, and with it all
    // loads before it, as soon as it is made a scalar.
    auto page_at = [&](int i) {
      const int t = row_at(i);
      if constexpr (SMALL) return t < span.hi ? table[t >> c.shift] : -1;
      const int at = __builtin_amdgcn_readfirstlane(t < span.hi ? t >> c.shift : 0);
      const int page = *((const __attribute__((address_space(4))) int*)table + at);
      return t < span.hi ? page : -1;
    };
    uint32_t rk[WORDS], rv[WORDS], gk, gv;   // codes, and step and base
    long v_slot = -1;                        // of the rows whose K was fetched last: V's next (-1: none)
    const int code_at = (SMALL ? 0 : my_row * CB) + 4 * WORDS * my_chunk, group_at = (SMALL ? 0 : my_row * GB) + 8 * WORDS * my_chunk / kKvGroup * 4;
    auto fetch = [&](const char* codes, const char* groups, long slot, bool bad, uint32_t* r, uint32_t& g) __attribute__((always_inline)) {
      if constexpr (SMALL) {
        const char* fill = (const char*)(bad ? g_nans : g_zeros);
        const char* p = (slot >= 0 ? codes + slot * CB : fill) + code_at;
#pragma unroll
        for (int x = 0; x < WORDS; ++x) r[x] = load_global<uint32_t>(p + 4 * x);
        g = load_global<uint32_t>((slot >= 0 ? groups + slot * GB : fill) + group_at);
      } else {
        const long at = slot >= 0 ? slot : 0;   // size 0 reads as zeros without an access; codes of 0 with a NaN base are NaN
        const __amdgpu_buffer_rsrc_t cb = buffer_of(codes + at * CB, slot >= 0 ? RPW * CB : 0);
        const __amdgpu_buffer_rsrc_t gb = buffer_of(bad ? (const char*)g_nans : groups + at * GB, slot >= 0 || bad ? RPW * GB : 0);
        if constexpr (WORDS == 2) {
          const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(cb, code_at, 0, 0));
          r[0] = w[0]; r[WORDS - 1] = w[1];
        } else {
          r[0] = __builtin_amdgcn_raw_buffer_load_b32(cb, code_at, 0, 0);
        }
        g = __builtin_amdgcn_raw_buffer_load_b32(gb, group_at, 0, 0);
      }
    };
    auto fetch_v = [&] { fetch(c.v, (const char*)c.vs, v_slot, false, rv, gv); };
    auto fetch_k = [&](int i, int page) {
      const int t = row_at(i);
      const bool in = t < span.hi, ok = in && (unsigned)page < (unsigned)c.n_pages;
      v_slot = ok ? kv_slot(c, page, h, t) : -1;
      fetch(c.k, (const char*)c.ks, v_slot, in && !ok, rk, gk);
    };

    // Tiles that every row of the workgroup, or of the wave, sees whole: those inside the sinks, and from the last
    // row's window start to the first row's position.
    const int inner = a.sinks / kTile, shift_i = span.sink_tiles - span.lo_tile - v0;   // tile of tokens t is i = t / 64 + shift_i
    auto tiles_from = [&](int p) { return (a.window ? max(p - a.window + 1 + kTile - 1, 0) / kTile : 0) + shift_i; };
    auto tiles_to = [&](int p) { return max(p + 1, 0) / kTile + shift_i; };
    const int full_from = max(tiles_from(last), span.sink_tiles - v0), full_to = tiles_to(first);
    const int wave_from = max(tiles_from(wlast), span.sink_tiles - v0), wave_to = tiles_to(wfirst);
    const int sinks_to = min(inner, span.sink_tiles) - v0;
    auto full = [&](int i) { return i < sinks_to || (i >= full_from && i < full_to); };

    // Codes that have come become rows of K in buffer `to`, one word at a time; and of V, whose values that are not finite are set
    // to zero in a tile that not all rows see whole (and lds.odd says so): their products with weights of zero would reach rows
    // that do not see them.
    auto decode_k = [&](int to, int x) __attribute__((always_inline)) {
      *(u32x4*)&lds.k[to][tile_row][16 * ((WORDS * my_chunk + x) ^ k_swizzle<D>(tile_row))] = mixed8(rk[x], gk);
    };
    auto decode_v = [&](int to, int x, u32x4 w) __attribute__((always_inline)) {
      *(u32x4*)&lds.v[to][tile_row][16 * ((WORDS * my_chunk + x) ^ v_swizzle<D>(tile_row))] = w;
    };
    auto check_v = [&](int i, int to) {      // behind decode_v, where it was not whole
      if (i < N && !full(i)) {
        int odd = 0;
#pragma unroll
        for (int x = 0; x < WORDS; ++x) {
          u32x4 w = mixed8(rv[x], gv);
          uint32_t top = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max_halves(top, w[e] & 0x7fff7fffu);
          if (__any(not_finite<MF>(top) != 0)) {
            odd = 1;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] &= ~not_finite<MF>(w[e]);
            decode_v(to, x, w);
          }
        }
        if (lane == 0) lds.odd[i & 1][wave] = odd;
      }
    };

    // ---- scores of a tile, 2 KS products, with aside(product) among them; the operands are read AHEAD steps ahead
    constexpr int AHEAD = 3;
    auto scores = [&](int buf, float16v* sc, auto&& aside) __attribute__((always_inline)) {
      const uint8_t* kb = &lds.k[buf][lane & 31][0];
      u32x4 f[AHEAD + 1][2];
      auto read = [&](auto step_c) __attribute__((always_inline)) {
        constexpr int step = decltype(step_c)::value;
#pragma unroll
        for (int y = 0; y < 2; ++y)
          f[step % (AHEAD + 1)][y] = *(const u32x4*)(kb + 32 * RB * y + 16 * ((2 * step + half) ^ k_swizzle<D>(lane & 31)));
      };
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[y][e] = 0;
      unroll<(AHEAD < KS ? AHEAD : KS)>([&](auto x) { read(x); });
      __builtin_amdgcn_sched_barrier(0);
      unroll<KS>([&](auto x) {
        constexpr int step = decltype(x)::value;
        if constexpr (step + AHEAD < KS) read(std::integral_constant<int, step + AHEAD>{});
        unroll<2>([&](auto y) {
          constexpr int Y = decltype(y)::value;
          sc[Y] = mfma32<MF>(f[step % (AHEAD + 1)][Y], qf[step], sc[Y]);
          aside(std::integral_constant<int, 2 * step + Y>{});
          __builtin_amdgcn_sched_barrier(0);
        });
      });
    };
    // ---- values of a tile, 4 VB products, likewise.  Product p takes block j = p % VB of the channels (no accumulator twice in a row)
    // and tokens 16 (p / VB) ..
    u32x4 pf[2][2];
    auto values = [&](int buf, auto&& aside) __attribute__((always_inline)) {
      constexpr int PRODUCTS = 4 * VB, FAR = 2 * AHEAD;
      const uint8_t* vb = &lds.v[buf][4 * half + (i16 >> 2)][32 * (lane >> 4 & 1) + 8 * (i16 & 3)];
      u32x4 f[FAR + 1];
      auto read = [&](auto p_c) __attribute__((always_inline)) {
        constexpr int p = decltype(p_c)::value, j = p % VB, t = p / VB;
        const int at = 16 * ((4 * j) ^ v_swizzle<D>(i16 >> 2));
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const u32x2 w = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              (__attribute__((address_space(3))) short4v*)(vb + (16 * t + 8 * x) * RB + at)));
          f[p % (FAR + 1)][2 * x] = w[0]; f[p % (FAR + 1)][2 * x + 1] = w[1];
        }
      };
      unroll<FAR>([&](auto x) { read(x); });
      __builtin_amdgcn_sched_barrier(0);
      unroll<PRODUCTS>([&](auto x) {
        constexpr int p = decltype(x)::value, j = p % VB, t = p / VB;
        if constexpr (p + FAR < PRODUCTS) read(std::integral_constant<int, p + FAR>{});
        o[j] = mfma32<MF>(f[p % (FAR + 1)], pf[t >> 1][t & 1], o[j]);
        aside(x);
        __builtin_amdgcn_sched_barrier(0);
      });
    };
    // Values that are not finite, which check_v() took out: from memory, to the rows that see them.
    auto odd_values = [&](int i) {
      bool odd = false;
      const int t0 = start(i);
      if (!full(i))
        for (int w = 0; w < kWaves; ++w) odd |= lds.odd[i & 1][w] != 0;
      if (__any(odd)) {
#pragma unroll 1
        for (int x = 0; x < kTile && t0 + x < span.hi; ++x) {
          const int id = table[(t0 + x) >> c.shift];
          if ((unsigned)id >= (unsigned)c.n_pages) continue;
          const bool see = row_sees(t0 + x, pos, behind, a.sinks);
          const long slot = kv_slot(c, id, h, t0 + x);
#pragma unroll
          for (int j = 0; j < VB; ++j) {
            const uint32_t group = load_global<uint32_t>((const char*)c.vs + slot * GB + 4 * j);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const u32x4 w = mixed8(load_global<uint32_t>(c.v + slot * CB + 4 * (4 * j + e)), group);
#pragma unroll
              for (int n = 0; n < 4; ++n) {
                const float y = h2f((uint16_t)((half ? w[2 + (n >> 1)] : w[n >> 1]) >> (16 * (n & 1))));
                o[j][4 * e + n] += see && !(fabsf(y) < INFINITY) ? y : 0.0f;
              }
            }
          }
        }
      }
    };
    auto mask = [&](int i, float16v* sc) {
      const int t0 = start(i) + 4 * half;
#pragma unroll
      for (int t = 0; t < 2; ++t)
        unroll<16>([&](auto ec) {
          constexpr int e = decltype(ec)::value;
          sc[t][e] = row_sees(t0 + 32 * t + 8 * (e >> 2) + (e & 3), pos, behind, a.sinks) ? sc[t][e] : -INFINITY;
        });
    };
    auto masked = [&](int i) { return !(i < sinks_to || (i >= wave_from && i < wave_to)); };
    auto end_tile = [] { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    // ---- tile i, whose scores lie in sc and their largest, of this lane, in mx; leaves those of tile i + 1 in next and mx
    float mx = -INFINITY;
    int page = -1;                           // of tile i + 3's rows
    auto tile = [&](int i, int parity, float16v* sc, float16v* next) __attribute__((always_inline)) {
      // what a row is held against follows its own scores alone; its two lanes meet where one has something to say
      float held = m;
      if (__any(rounded_product(mx, factor) - m > slack)) {
        const float top = rounded_product(max_xor32(mx), factor), was = m;
        const bool rises = top - m > kSlack<F4>;
        if (rises) m = held_against<F4>(top);
        const float alpha = rises ? exp2f(was - m) : 1.0f;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < VB; ++j)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[j][e] *= alpha;
        held = m;
        slack = far_out(held) ? -INFINITY : kSlack<F4>;
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
      // weights, E of the 32 beside a product
      float sum = 0;
      constexpr int E = 32 / (2 * KS);
      scores(parity ^ 1, next, [&](auto product) __attribute__((always_inline)) {
        unroll<E / 2>([&](auto x) {
          constexpr int at = decltype(product)::value * E + 2 * decltype(x)::value, t = at / 16, e = at % 16;
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[t][e], factor, -base));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[t][e + 1], factor, -base));
          sum += p0;
          sum += p1;
          uint32_t w = pack2<GRINQH_F16>(p0, p1);
          asm volatile("" : "+v"(w), "+v"(sum));   // here, beside the product, and not where it is used
          pf[t][e >> 3][e >> 1 & 3] = w;
        });
      });
      l += sum;
      if (masked(i + 1)) mask(i + 1, next);
      // the next maximum, and rows of what has come, V of i + 1 and K of i + 2
      mx = -INFINITY;
      constexpr int PRODUCTS = 4 * VB, M = 32 / PRODUCTS, AT = PRODUCTS / (2 * WORDS);
      values(parity, [&](auto product) __attribute__((always_inline)) {
        constexpr int p = decltype(product)::value;
#pragma unroll
        for (int x = 0; x < M; x += 2) {
          constexpr int from = p * M;
          mx = fmaxf(fmaxf(next[from / 16][(from + x) % 16], next[from / 16][(from + x) % 16 + 1]), mx);
        }
        asm volatile("" : "+v"(mx));
        if constexpr (p % AT == 0) {
          constexpr int x = p / AT;
          if constexpr (x < WORDS) decode_v(parity ^ 1, x, mixed8(rv[x], gv));
          else decode_k(parity, x - WORDS);
        }
      });
      check_v(i + 1, parity ^ 1);
      odd_values(i);
      fetch_v();
      fetch_k(i + 3, page);
      page = page_at(i + 4);
      end_tile();
    };

    if (N > 0) {
      float16v sc[2][2];
      fetch_k(0, page_at(0));
      fetch_v();
      page = page_at(1);
      for (int x = 0; x < WORDS; ++x) { decode_k(0, x); decode_v(0, x, mixed8(rv[x], gv)); }
      check_v(0, 0);
      fetch_k(1, page);
      fetch_v();
      page = page_at(2);
      for (int x = 0; x < WORDS; ++x) decode_k(1, x);
      fetch_k(2, page);
      page = page_at(3);
      end_tile();
      scores(0, sc[0], [](auto) {});
      if (masked(0)) mask(0, sc[0]);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[0][t][e]);
      end_tile();                            // K of tile 0 has been read: that of tile 2 goes there
#pragma unroll 1
      for (int i = 0;;) {
        tile(i, 0, sc[0], sc[1]);
        if (++i >= N) break;
        tile(i, 1, sc[1], sc[0]);
        if (++i >= N) break;
      }
      __syncthreads();
    }

    const DenseRows out = late().out;
    const Partial part = late().part;
    float* lse = late().lse;
    // ---- results: lane = row; channels 0, 4, 1, 5 of each eight in one half of the wave and 2, 6, 3, 7 in the other become 0 .. 3 and 4 .. 7
    l += __builtin_bit_cast(float, __shfl_xor(__builtin_bit_cast(int, l), 32));
    const float inv = l == 0 ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < VB; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t x[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) x[n] = __builtin_bit_cast(uint32_t, (float)o[j][4 * e + n] * inv);
        const auto s0 = __builtin_amdgcn_permlane32_swap(x[0], x[1], false, false), s1 = __builtin_amdgcn_permlane32_swap(x[2], x[3], false, false);
        o[j][4 * e] = __builtin_bit_cast(float, (uint32_t)s0[0]);
        o[j][4 * e + 1] = __builtin_bit_cast(float, (uint32_t)s1[0]);
        o[j][4 * e + 2] = __builtin_bit_cast(float, (uint32_t)s0[1]);
        o[j][4 * e + 3] = __builtin_bit_cast(float, (uint32_t)s1[1]);
      }
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
              *(float4v*)(p + 32 * j + 8 * e) = float4v{o[j][4 * e], o[j][4 * e + 1], o[j][4 * e + 2], o[j][4 * e + 3]};
        }
      } else {
        if (lse && half == 0) lse[at] = lse2 * kLn2;
      }
    }
    if (used == 1) {
      // rows of the output are written whole, through LDS
      constexpr int STRIDE = RB + 16;        // 16 rows of pieces meet 64 banks
      static_assert(kWaves * 32 * STRIDE <= sizeof(lds.k) + sizeof(lds.v) + sizeof(lds.more));
      uint8_t* rows = &lds.k[0][0][0] + wave * 32 * STRIDE;
#pragma unroll
      for (int j = 0; j < VB; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *(u32x2*)(rows + (lane & 31) * STRIDE + 2 * (32 * j + 8 * e + 4 * half)) =
              u32x2{pack2<TYPE>(o[j][4 * e], o[j][4 * e + 1]), pack2<TYPE>(o[j][4 * e + 2], o[j][4 * e + 3])};
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

template <int D, int TYPE>
void go(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  const dim3 grid(args.c.H * p.splits, p.blocks, args.b.B);
  if (args.c.shift >= 4) k_attend_tile4<D, TYPE, false><<<grid, 64 * kWaves, 0, s>>>(args);
  else k_attend_tile4<D, TYPE, true><<<grid, 64 * kWaves, 0, s>>>(args);
}

}  // namespace

void launch_attend_tile4(const AttendPlan& p, const AttendArgs& args, hipStream_t s) {
  auto on = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (args.a.type == GRINQH_F16) go<D, GRINQH_F16>(p, args, s);
    else go<D, GRINQH_BF16>(p, args, s);
  };
  if (args.c.D == 64) on(std::integral_constant<int, 64>{});
  else on(std::integral_constant<int, 128>{});
}

}  // namespace grinqh
