// A step's plan: pages for the tokens that come, pages back from those that are taken back, and the batch's arrays.
//
// With len and d = new_rows of sequence b, P tokens a page and pages(x) = ceil(x / P):
//   back   d < 0: len' = max(len + d, 0), pages(len) - pages(len') table entries leave, from the first sequence's first on
//          to the list's end downwards: stacked up from the last sequence's last page
//   come   d > 0: need_b = pages(len + d) - pages(len); b gets d rows iff sum_{i <= b} need_i <= the list's pages and
//          sum_{i <= b} d_i <= rows, over the sequences whose own table holds len + d tokens
//   row i  of b stands at position len + i; its page is the table's, or where that is one of the need_b new ones, the
//          (sum_{j < b} need_j + its number)-th from the list's end
// Sums are unsigned 32-bit numbers that stay at 2^32 - 1 once they get there, far past any limit that they are held against.
//
// Up to kSmall sequences are one workgroup's, a thread a sequence, with everything read at once and kept (k_plan_small): bound by
// latency, 3 to 4 us for 64.  More are counted by a grid (k_plan_count), summed up by one workgroup (k_plan_sums) and their pages
// stacked by a grid (k_plan_back).  Rows that are more than a few per thread of that one workgroup are a grid's (k_plan_rows).
//   One workgroup : grid, us, L tokens for each of B sequences in pages of 16, planned and taken back again: B = 64 10 : 20 (L = 1),
//   15 : 22 (256); 256 14 : 21, 19 : 22; 512 18 : 23, 23 : 23; 1024 26 : 27, 33 : 24.
//   Rows by it : by a grid: 16384 of 64 sequences 25 : 15, of 256 30 : 19, 65536 of 256 80 : 19.
// 2.5 million rows of 1500 sequences (30 MB) and some taken back: 35 us in seven launches, of which counts 2 to 4, sums 5, rows 13.
#include "kv.h"

namespace grinqh {

namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kSmall = 512;                  // sequences of the one workgroup
constexpr int kSmallRows = 4 * kThreads;     // rows that it also does itself
constexpr int kItems = 4;                    // sequences of a thread of k_plan_sums
constexpr int kChunk = kThreads * kItems;

__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_dpp(uint32_t x) {
  return add(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false));
}

// The sum of the lanes' values up to this one's.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x = add_dpp<0x111, 0xf>(x);                // from 1, 2, 4 and 8 lanes before it in its row of 16
  x = add_dpp<0x112, 0xf>(x);
  x = add_dpp<0x114, 0xf>(x);
  x = add_dpp<0x118, 0xf>(x);
  x = add_dpp<0x142, 0xa>(x);                // the first row's sum into the second, the third's into the fourth
  return add_dpp<0x143, 0xc>(x);             // the first two rows' into the others
}

struct Sums { uint32_t a, b; };

// The sums of the threads' values before this one's, and of all.  One barrier; tot is another's only after the next.  (The value
// before, not the value up to it less its own: a sum at its end would lose what lies before it.)
__device__ __forceinline__ Sums block_scan(Sums x, Sums* tot, Sums* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums s = {wave_scan(x.a), wave_scan(x.b)};
  if (lane == 63) tot[wave] = s;
  __syncthreads();
  Sums before = {0, 0}, sum = {0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = sum;
    sum = {add(sum.a, tot[w].a), add(sum.b, tot[w].b)};
  }
  *all = sum;
  auto shifted = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xf, 0xf, false); };   // wave_shr:1
  return {add(before.a, shifted(s.a)), add(before.b, shifted(s.b))};
}

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (int)(((uint32_t)tokens + (1u << shift) - 1) >> shift); }

__device__ __forceinline__ int plan_capacity(const KvPlan& p) {
  const long cap = (long)p.width << p.shift;
  return cap < kMaxTokens ? (int)cap : (int)kMaxTokens;
}

// Tokens left of len after d < 0 more.
__device__ __forceinline__ int left_of(int len, int d) { return (int)max((long)len + d, 0L); }

// LANES lanes take a sequence's pages, entries first .. end - 1, four each at a time so that a long sequence is no chain of loads.
constexpr int kAtOnce = 4;

// How many there are, in every lane.
template <int LANES>
__device__ __forceinline__ uint32_t count_pages(const KvPlan& p, int b, int first, int end) {
  const int* table = p.table + (long)b * p.width;
  uint32_t n = 0;
  for (int j0 = first + (int)(threadIdx.x % LANES); j0 < end; j0 += kAtOnce * LANES) {
    int id[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) id[u] = j0 + u * LANES < end ? table[j0 + u * LANES] : -1;
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) n += (unsigned)id[u] < (unsigned)p.n_pages;
  }
#pragma unroll
  for (int s = LANES / 2; s; s >>= 1) n += (uint32_t)__shfl_xor((int)n, s);
  return n;
}

// They go to the list from place `at` on, the last one first, and leave the table.
template <int LANES>
__device__ __forceinline__ void stack_pages(const KvPlan& p, int b, int first, int end, long at) {
  const int lane = threadIdx.x % LANES;
  int* table = p.table + (long)b * p.width;
  for (int j0 = end - 1; j0 >= first; j0 -= kAtOnce * LANES) {
    int id[kAtOnce];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int j = j0 - u * LANES - lane;
      id[u] = j >= first ? table[j] : -1;
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
      const int j = j0 - u * LANES - lane;
      const bool is = (unsigned)id[u] < (unsigned)p.n_pages;
      unsigned long long mask = __ballot(is);
      if constexpr (LANES < 64) mask = mask >> (threadIdx.x & 63 & ~(LANES - 1)) & ((1ull << LANES) - 1);
      const long to = at + __popcll(mask & ((1ull << lane) - 1));
      if (is && to < p.capacity) p.free_pages[to] = id[u];
      if (j >= first) table[j] = -1;
      at += __popcll(mask);
    }
  }
}

// A row of a sequence whose rows start at `offset`, behind `was` tokens, and whose new pages begin `base` from the list's end.
struct Row { int position, id; int* entry; };   // entry: of a new page, whose first row writes it

__device__ __forceinline__ Row plan_row(const KvPlan& p, int list, int row, int b, int offset, int was, int base) {
  const int first_new = pages_of(was, p.shift);
  Row r;
  r.position = was + row - offset;
  const int page = r.position >> p.shift;
  int* entry = p.table + (long)b * p.width + page;
  const bool is_new = page >= first_new;
  r.entry = is_new && (r.position & ((1 << p.shift) - 1)) == 0 ? entry : nullptr;
  r.id = *(is_new ? p.free_pages + (list - 1 - (base + page - first_new)) : entry);
  return r;
}

__device__ __forceinline__ void store_row(const KvPlan& p, int row, const Row& r) {
  if (r.entry) *r.entry = r.id;
  if (p.positions) p.positions[row] = r.position;
  if (p.slots)
    p.slots[row] = (unsigned)r.id < (unsigned)p.n_pages ? ((long)r.id << p.shift) + (r.position & ((1 << p.shift) - 1)) : -1;
}
constexpr int kNoRow = -1;                   // position and, as a page, id of what is behind the last row

// What a sequence asks for, and whether it gets it.
__device__ __forceinline__ Sums asked(const KvPlan& p, int cap, int len, int d) {
  if (d <= 0 || (long)len + d > cap) return {0, 0};
  return {(uint32_t)(pages_of(len + d, p.shift) - pages_of(len, p.shift)), (uint32_t)d};
}
__device__ __forceinline__ bool granted(const KvPlan& p, long list, Sums upto) { return upto.a <= (uint32_t)list && upto.b <= (uint32_t)p.rows; }

// Of sums that grow from thread to thread, those of the last one that is ok, in every thread (0 if none is).  One barrier.
__device__ __forceinline__ Sums last_ok(bool ok, Sums upto, Sums* lds) {
  const unsigned long long mask = __ballot(ok);
  const int last = 63 - __clzll(mask);
  if ((int)(threadIdx.x & 63) == (mask ? last : 0)) lds[threadIdx.x >> 6] = mask ? upto : Sums{0, 0};
  __syncthreads();
  Sums most = {0, 0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) most = {max(most.a, lds[w].a), max(most.b, lds[w].b)};
  return most;
}

template <bool ROWS>
__global__ __launch_bounds__(kThreads) void k_plan_small(KvPlan p) {
  __shared__ Sums tot[4][kWaves];
  __shared__ int listed[kThreads], first[kThreads], end[kThreads], count[kThreads];
  const int b = threadIdx.x, cap = plan_capacity(p);
  const bool in = b < p.B;
  int d = 0, len = 0;
  if (in) { d = p.new_rows[b]; len = p.lens[b]; }
  long list = min(max(*p.n_free, 0), p.capacity);
  len = min(max(len, 0), cap);

  // ---- tokens taken back
  const int now = d < 0 ? left_of(len, d) : len, from = pages_of(now, p.shift), to = pages_of(len, p.shift);
  const bool gives = to > from;
  if (d < 0) {
    p.lens[b] = now;
    if (p.granted) p.granted[b] = now - len;
  }
  if (__syncthreads_or(gives)) {
    Sums all;
    const uint32_t before_it = block_scan({gives, 0}, tot[0], &all).a;
    const int n = (int)all.a;
    if (gives) {
      const int x = n - 1 - (int)before_it;  // last first
      listed[x] = b; first[x] = from; end[x] = to;
    }
    __syncthreads();
    // a wave a sequence as long as there are no more of them, else a quarter of one
    auto each = [&](auto f) {
      if (n <= kWaves) {
        if (b / 64 < n) f(b / 64, std::integral_constant<int, 64>{});
      } else {
        for (int x = b / 16; x < n; x += kThreads / 16) f(x, std::integral_constant<int, 16>{});
      }
    };
    each([&](int x, auto lanes) {
      constexpr int LANES = decltype(lanes)::value;
      const uint32_t k = count_pages<LANES>(p, listed[x], first[x], end[x]);
      if (b % LANES == 0) count[x] = (int)k;
    });
    __syncthreads();
    const uint32_t own = b < n ? (uint32_t)count[b] : 0;
    const uint32_t before = block_scan({own, 0}, tot[1], &all).a;
    if (b < n) count[b] = (int)before;
    __syncthreads();
    each([&](int x, auto lanes) {
      stack_pages<decltype(lanes)::value>(p, listed[x], first[x], end[x], list + (uint32_t)count[x]);
    });
    list = min(list + (long)all.a, (long)p.capacity);
    __syncthreads();
  }

  // ---- tokens that come
  const Sums need = asked(p, cap, len, d);
  Sums all;
  const Sums before = block_scan(need, tot[2], &all), upto = {add(before.a, need.a), add(before.b, need.b)};
  const bool ok = granted(p, list, upto);
  const Sums most = last_ok(ok, upto, tot[3]);
  const int got = ok ? (int)need.b : 0, behind = (int)(ok ? upto.b : most.b);
  if (in) {
    p.offs[b + 1] = behind;
    if (p.granted && d >= 0) p.granted[b] = got;
    if (got) p.lens[b] = len + got;
  }
  if (b == 0) {
    p.offs[0] = 0;
    *p.n_free = (int)(list - most.a);
  }
  if constexpr (ROWS) {
    // rows look their sequence up among those that have any, one behind the other
    int* offset = first; int* was = end; int* base = count;
    const bool has = got > 0;
    const unsigned long long mask = __ballot(has);
    int* per_wave = (int*)tot[0];
    if ((threadIdx.x & 63) == 0) per_wave[threadIdx.x >> 6] = __popcll(mask);
    __syncthreads();
    int at = __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1)), n = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < (int)(threadIdx.x >> 6)) at += per_wave[w];
      n += per_wave[w];
    }
    if (has) { listed[at] = b; offset[at] = behind - got; was[at] = len; base[at] = (int)before.a; }
    __syncthreads();
    for (int row = threadIdx.x; row < p.rows; row += kThreads) {
      Row r = {kNoRow, kNoRow, nullptr};
      if (row < (int)most.b) {
        int lo = 0, hi = n - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (offset[mid] <= row) lo = mid; else hi = mid - 1;
        }
        r = plan_row(p, (int)list, row, listed[lo], offset[lo], was[lo], base[lo]);
      }
      store_row(p, row, r);
    }
  } else {
    if (in) { p.space[4 + b] = (int)before.a; p.space[4 + p.B + b] = len; }
    if (b == 0) p.space[0] = (int)list;
  }
}

// ---- more sequences.  Workspace: [0] the list's pages before any are handed out, [1] those before any came back, [2] those that came
// back, [3] unused; from [4] on base [B], a sequence's pages from the list's end (d < 0: pages that came back from the sequences before
// it), and old length [B] (d < 0: its own pages that came back).  k_plan_small leaves [0], base and old length there for k_plan_rows.
constexpr int kSeqThreads = 256, kSeqs = kSeqThreads / 64;   // a wave a sequence

__global__ __launch_bounds__(kSeqThreads) void k_plan_count(KvPlan p) {
  const int b = blockIdx.x * kSeqs + threadIdx.x / 64;
  if (b >= p.B) return;
  const int d = p.new_rows[b];
  uint32_t n = 0;
  if (d < 0) {
    const int len = min(max(p.lens[b], 0), plan_capacity(p));
    n = count_pages<64>(p, b, pages_of(left_of(len, d), p.shift), pages_of(len, p.shift));
  }
  if (threadIdx.x % 64 == 0) p.space[4 + p.B + b] = (int)n;
}

__global__ __launch_bounds__(kThreads) void k_plan_sums(KvPlan p) {
  __shared__ Sums tot[3][kWaves];
  __shared__ Sums ends[2][kWaves];
  const int cap = plan_capacity(p), free_now = min(max(*p.n_free, 0), p.capacity);
  int* base = p.space + 4;
  int* old = base + p.B;
  int d[kItems], len[kItems];
  uint32_t back[kItems];
  auto load = [&](int c0) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = c0 + threadIdx.x * kItems + i;
      d[i] = b < p.B ? p.new_rows[b] : 0;
      len[i] = b < p.B ? p.lens[b] : 0;
      back[i] = b < p.B ? (uint32_t)old[b] : 0;
    }
  };
  load(0);
  // all the pages that come back: the first chunk's are here
  uint32_t mine = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) mine = add(mine, back[i]);
  for (int b = kChunk + threadIdx.x; b < p.B; b += kThreads) mine = add(mine, (uint32_t)old[b]);
  Sums all;
  block_scan({mine, 0}, tot[2], &all);
  const uint32_t came = all.a;
  const long list = min(free_now + (long)came, (long)p.capacity);
  Sums sum0 = {0, 0}, most = {0, 0};
  uint32_t back0 = 0;
  int turn = 0;                              // of two arrays of sums: a thread behind may still read the other one
  for (int c0 = 0; c0 < p.B; c0 += kChunk, turn ^= 1) {
    Sums own = {0, 0}, need[kItems];
    uint32_t own_back = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      len[i] = min(max(len[i], 0), cap);
      need[i] = asked(p, cap, len[i], d[i]);
      own = {add(own.a, need[i].a), add(own.b, need[i].b)};
      own_back = add(own_back, back[i]);
    }
    const Sums before = block_scan(own, tot[turn], &all);
    Sums sum = {add(sum0.a, before.a), add(sum0.b, before.b)}, ok_sum = {0, 0}, upto[kItems];
    bool ok[kItems], any = false;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      sum = {add(sum.a, need[i].a), add(sum.b, need[i].b)};
      upto[i] = sum;
      ok[i] = granted(p, list, sum);
      if (ok[i]) { ok_sum = sum; any = true; }
    }
    sum0 = {add(sum0.a, all.a), add(sum0.b, all.b)};
    const Sums here = last_ok(any, ok_sum, ends[turn]);
    most = {max(most.a, here.a), max(most.b, here.b)};
    uint32_t back_before = 0;
    if (came) {                              // else none has a place in the list to be told
      back_before = add(back0, block_scan({own_back, 0}, tot[2], &all).a);
      back0 = add(back0, all.a);
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int b = c0 + threadIdx.x * kItems + i;
      if (b >= p.B) continue;
      p.offs[b + 1] = (int)(ok[i] ? upto[i].b : most.b);
      if (d[i] < 0) {                        // the rest is k_plan_back's
        base[b] = (int)back_before;
        back_before = add(back_before, back[i]);
        continue;
      }
      const int got = ok[i] ? (int)need[i].b : 0;
      if (p.granted) p.granted[b] = got;
      if (got) p.lens[b] = len[i] + got;
      base[b] = (int)(upto[i].a - need[i].a);   // of one that is granted something exact
      old[b] = len[i];
    }
    if (c0 + kChunk < p.B) load(c0 + kChunk);
  }
  if (threadIdx.x == 0) {
    p.offs[0] = 0;
    p.space[0] = (int)list;
    p.space[1] = free_now;
    p.space[2] = (int)came;
    *p.n_free = (int)(list - most.a);
  }
}

__global__ __launch_bounds__(kSeqThreads) void k_plan_back(KvPlan p) {
  const int b = blockIdx.x * kSeqs + threadIdx.x / 64;
  if (b >= p.B) return;
  const int d = p.new_rows[b];
  if (d >= 0) return;
  const int len = min(max(p.lens[b], 0), plan_capacity(p)), now = left_of(len, d);
  const uint32_t at = (uint32_t)p.space[2] - (uint32_t)p.space[4 + b] - (uint32_t)p.space[4 + p.B + b];   // what lies behind it
  stack_pages<64>(p, b, pages_of(now, p.shift), pages_of(len, p.shift), p.space[1] + (long)at);
  if (threadIdx.x % 64 == 0) {
    p.lens[b] = now;
    if (p.granted) p.granted[b] = now - len;
  }
}

constexpr int kRowThreads = 256;
constexpr int kRowItems = 4;                 // rows of a thread
constexpr int kWindow = 1024;                // sequences whose offsets a workgroup keeps

// The number of offs[0 .. B - 1] at or below each of two rows, which the workgroup counts together: every 256th first, of which a
// thread brings its own, o, then those between.  (offs ascend from 0, so at least one.)
__device__ __forceinline__ void count_offsets(const int* offs, int B, int o, int row0, int row1, int* lds, int* n0, int* n1) {
  static_assert(kRowThreads == 256);
  const int wave = threadIdx.x >> 6, i = threadIdx.x;
  auto sum = [&](unsigned long long m0, unsigned long long m1, int* s0, int* s1) {
    if ((i & 63) == 0) { lds[wave] = __popcll(m0); lds[4 + wave] = __popcll(m1); }
    __syncthreads();
    *s0 = lds[0] + lds[1] + lds[2] + lds[3];
    *s1 = lds[4] + lds[5] + lds[6] + lds[7];
    __syncthreads();
  };
  int c0, c1;
  sum(__ballot(o <= row0), __ballot(o <= row1), &c0, &c1);
  const int a0 = (c0 - 1) * 256 + i, a1 = (c1 - 1) * 256 + i;
  const int o0 = a0 < B ? offs[a0] : 0x7fffffff, o1 = a1 < B ? offs[a1] : 0x7fffffff;
  sum(__ballot(o0 <= row0), __ballot(o1 <= row1), n0, n1);
  *n0 += (c0 - 1) * 256;
  *n1 += (c1 - 1) * 256;
}

// A thread's chain of loads: the offsets' sample, those between, what the workgroup's sequences have, the row's page.
__global__ __launch_bounds__(kRowThreads) void k_plan_rows(KvPlan p) {
  __shared__ int offset[kWindow], was[kWindow], based[kWindow], counts[8];
  const int* base = p.space + 4;
  const int* old = base + p.B;
  const int sample = (int)threadIdx.x * 256 < p.B ? p.offs[threadIdx.x * 256] : 0x7fffffff;
  const int list = p.space[0], total = p.offs[p.B];
  const int r0 = blockIdx.x * kRowThreads * kRowItems, r1 = min(r0 + kRowThreads * kRowItems, total) - 1;
  int lo0 = 0, hi0 = 0;
  if (r0 < total) {
    count_offsets(p.offs, p.B, sample, r0, r1, counts, &lo0, &hi0);
    --lo0; --hi0;
    if (hi0 - lo0 < kWindow)
      for (int i = threadIdx.x; i <= hi0 - lo0; i += kRowThreads) {
        offset[i] = p.offs[lo0 + i]; was[i] = old[lo0 + i]; based[i] = base[lo0 + i];
      }
    __syncthreads();
  }
  const bool near = hi0 - lo0 < kWindow;
  Row r[kRowItems];
#pragma unroll
  for (int i = 0; i < kRowItems; ++i) {
    const int row = r0 + i * kRowThreads + threadIdx.x;
    r[i] = {kNoRow, kNoRow, nullptr};
    if (row < total) {
      int lo = lo0, hi = hi0;                // the last sequence whose rows start at or before this one
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((near ? offset[mid - lo0] : p.offs[mid]) <= row) lo = mid; else hi = mid - 1;
      }
      r[i] = near ? plan_row(p, list, row, lo, offset[lo - lo0], was[lo - lo0], based[lo - lo0])
                  : plan_row(p, list, row, lo, p.offs[lo], old[lo], base[lo]);
    }
  }
#pragma unroll
  for (int i = 0; i < kRowItems; ++i) {
    const int row = r0 + i * kRowThreads + threadIdx.x;
    if (row < p.rows) store_row(p, row, r[i]);
  }
}

}  // namespace

size_t plan_workspace(int B) { return (4 + 2 * (size_t)B) * sizeof(int); }

int launch_kv_plan(const KvPlan& p, hipStream_t s) {
  const int seq_blocks = (p.B + kSeqs - 1) / kSeqs;
  if (p.B <= kSmall) {
    if (p.rows <= kSmallRows) {
      k_plan_small<true><<<1, kThreads, 0, s>>>(p);
      return check_launch("kv_plan");
    }
    k_plan_small<false><<<1, kThreads, 0, s>>>(p);
  } else {
    k_plan_count<<<seq_blocks, kSeqThreads, 0, s>>>(p);
    k_plan_sums<<<1, kThreads, 0, s>>>(p);
    k_plan_back<<<seq_blocks, kSeqThreads, 0, s>>>(p);
  }
  constexpr int rows = kRowThreads * kRowItems;
  if (p.rows) k_plan_rows<<<(p.rows + rows - 1) / rows, kRowThreads, 0, s>>>(p);
  return check_launch("kv_plan");
}

}  // namespace grinqh
