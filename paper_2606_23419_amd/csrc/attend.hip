// Attention of a batch's rows over the paged cache: how a call is launched,
// and the joining of sequences that were split.
#include "attend.h"

#include <algorithm>

namespace grinqh {

namespace {

// The splits' results of a row and head, weighed by their sums.  D / 8 lanes hold the channels; `groups` such
// groups of a workgroup take every groups-th split of one row and meet in LDS, so a row of many splits is not
// one chain of loads.  Bound by latency: 64 parts of one token's 32 heads (1 MB) take 4.8 us.
constexpr int kJoinThreads = 256;

template <int D, int TYPE, int TK>
__global__ __launch_bounds__(kJoinThreads) void k_attend_join(KvCache c, KvBatch b, Attend a, DenseRows out, float* lse,
                                                              Partial part, int most, int per_split, int rows_log2, int groups) {
  constexpr int LPR = D / 8, GROUPS = kJoinThreads / LPR;
  __shared__ float sm[GROUPS], ssum[GROUPS], sy[GROUPS][D];
  const int s = blockIdx.z, lane = threadIdx.x % LPR, group = threadIdx.x / LPR, g = group % groups;
  const Seq sq = kv_seq(c, b, s);
  const long all = (long)sq.n * a.heads;
  const int per_block = GROUPS / groups;
  for (long r0 = (long)blockIdx.x * per_block; r0 < all; r0 += (long)gridDim.x * per_block) {
    const long r = r0 + group / groups, rc = min(r, all - 1), at = (long)sq.r0 * a.heads + rc;
    // the row's block, as the kernel before took it, and how many splits that had
    const int of_group = (int)(rc / a.heads) * a.G + (int)(rc % a.heads) % a.G, first_row = of_group >> rows_log2 << rows_log2;
    const int last_row = min(first_row + (1 << rows_log2), sq.n * a.G) - 1;
    const int splits = attend_span<TK>(a, sq.L - sq.n + first_row / a.G, sq.L - sq.n + last_row / a.G).splits(most, per_split);
    float m = -INFINITY, sum = 0, y[8] = {};
    // four splits in flight; past the last one the last is read again and weighs nothing
    for (int i0 = splits > 1 ? g : splits; i0 < splits; i0 += 4 * groups) {
      float z[4];
      float4v p[4][2];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const long i = min(i0 + u * groups, splits - 1);
        z[u] = part.lse[i * part.rows + at];
        const float4v* src = (const float4v*)(part.o + (i * part.rows + at) * D + lane * 8);
        p[u][0] = src[0];
        p[u][1] = src[1];
      }
      float top = m;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (i0 + u * groups >= splits) z[u] = -INFINITY;
        top = fmaxf(top, z[u]);
      }
      const float base = top == -INFINITY ? 0.0f : top, old = exp2f(m - base);
      m = top;
      sum *= old;
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] *= old;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool any = z[u] != -INFINITY;   // else nothing was written there
        const float w = any ? exp2f(z[u] - base) : 0.0f;
        sum += w;
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] += any ? w * p[u][j >> 2][j & 3] : 0.0f;
      }
    }
    if (groups > 1) {
      if (lane == 0) { sm[group] = m; ssum[group] = sum; }
      for (int j = 0; j < 8; ++j) sy[group][lane * 8 + j] = y[j];
      __syncthreads();
      float top = -INFINITY;
      for (int i = 0; i < groups; ++i) top = fmaxf(top, sm[group - g + i]);
      m = top;
      sum = 0;
      for (int j = 0; j < 8; ++j) y[j] = 0;
      for (int i = 0; i < groups; ++i) {
        const float w = exp2f(sm[group - g + i] - (top == -INFINITY ? 0.0f : top));
        sum += w * ssum[group - g + i];
        for (int j = 0; j < 8; ++j) y[j] += w * sy[group - g + i][lane * 8 + j];
      }
      __syncthreads();
    }
    if (g == 0 && r < all && splits > 1) {   // else the row is there already
      const float inv = sum == 0 ? 0.0f : 1.0f / sum;
      uint32_t w[4];
      for (int j = 0; j < 4; ++j) w[j] = pack2<TYPE>(y[2 * j] * inv, y[2 * j + 1] * inv);
      *(u32x4*)(out.p + ((sq.r0 + r / a.heads) * out.row + (r % a.heads) * out.head + lane * 8) * 2) = u32x4{w[0], w[1], w[2], w[3]};
      if (lse && lane == 0) lse[at] = sum == 0 ? -INFINITY : (m + log2f(sum)) * kLn2;
    }
  }
}

AttendPlan attend_plan(const KvCache& c, const Attend& a, int B, int rows) {
  AttendPlan p = {};
  const int forced = option(&Options::attend_kernel), forced_splits = option(&Options::attend_splits);
  const long n = std::min(a.max_rows, rows), R = n * a.G;
  // R rows of a kv head share its K and V.  Up to 32 of them are one workgroup's in k_attend_rows, the next read the cache
  // again, from L2 at first.  8 bits, rows kernel against tile kernel, us: R = 64 over 8190 tokens of 1 sequence 27 : 37, of
  // 4 44 : 59; 500 tokens of 4 17 : 34; 2000 of 32 101 : 98; 16 bits, 8190 of 8 90 : 102.  R = 128: 34 : 39, 62 : 66,
  // 19 : 34, 188 : 100, 212 : 110.  Past 64 rows it depends on the number of sequences, which the rule does not look at: few
  // short ones of 65 to 128 rows pay up to 1.8 times.
  p.tile = forced ? forced != GRINQH_ATTEND_ROWS : R > 64;
  p.nb = R > 16 ? 2 : 1;
  const long per_block = p.tile ? 256 : 16 * p.nb, tile = p.tile ? 64 : 32;
  p.rows_log2 = __builtin_ctzl(per_block);
  p.blocks = (int)std::min<long>((R + per_block - 1) / per_block, 65535);
  // tiles that the longest sequence's last block sees
  const long seen = a.window ? std::min<long>(a.max_len, (long)a.window + per_block / a.G + a.sinks + 2 * tile) : a.max_len;
  const long tiles = (seen + tile - 1) / tile, groups = (long)B * c.H * p.blocks;
  // Sequences too few to fill the device are split: one workgroup per CU in k_attend_tile (its LDS), two and more in
  // k_attend_rows.  One token over 131072 tokens is 64 parts: 16 parts 71 us, 32 62, 64 58, 128 64.  Prompts that fill half
  // the CUs stay whole: 2048 rows of 32 heads from the start 74 us, in two parts 85 and 23 joining, in three 71 and 25.
  const long fill = p.tile ? device_cus() : 2 * device_cus();
  const long unit = p.tile ? 1 : rows_waves(p.nb), least = p.tile ? 8 : unit;
  long splits = forced_splits ? forced_splits : std::min(std::max<long>(1, fill / groups), std::max<long>(1, tiles / least));
  // Sequences enough to fill the CUs without splitting are as a rule of unequal length, which the host does not see:
  // parts of about 700 tokens keep the longest from being waited for.  32 sequences up to 8191 tokens: 1 part each 99 us,
  // 3 81, 6 73, 12 65; 16 sequences of 4100 visible tokens 2 57, 4 58, 12 62 (2 and 4 are what filling twice gives there).
  if (!forced_splits && !p.tile && groups >= device_cus()) splits = std::max(splits, std::min<long>(16, (tiles + 21) / 22));
  long per = (tiles + splits - 1) / splits;
  per = (per + unit - 1) / unit * unit;
  p.per_split = (int)per;
  p.splits = (int)((tiles + per - 1) / per);
  return p;
}

}  // namespace

static size_t partial_bytes(const AttendPlan& p, const KvCache& c, const Attend& a, int rows) {
  return p.splits > 1 ? (size_t)p.splits * rows * a.heads * (c.D + 1) * sizeof(float) : 0;
}

size_t attend_workspace(const KvCache& c, const Attend& a, int B, int rows) {
  return partial_bytes(attend_plan(c, a, B, rows), c, a, rows);
}

int launch_attend(const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q, const DenseRows& out,
                  float* lse, void* workspace, hipStream_t s) {
  const AttendPlan p = attend_plan(c, a, b.B, b.rows);
  Partial part = {(float*)workspace, nullptr, (long)b.rows * a.heads};
  part.lse = part.o + p.splits * part.rows * c.D;
  const AttendArgs args = {c, b, a, p.splits, p.per_split, q, out, lse, part};
  (p.tile ? launch_attend_tile : launch_attend_rows)(p, args, s);
  int st = check_launch("attend");
  if (st || p.splits == 1) return st;
  int groups = 1;
  while (groups < 16 && groups * 2 <= p.splits) groups *= 2;
  const long per_block = kJoinThreads / (c.D / 8) / groups, per_seq = (long)std::min(a.max_rows, b.rows) * a.heads;
  const dim3 grid((unsigned)std::min<long>((per_seq + per_block - 1) / per_block, 1 << 20), 1, b.B);
  auto go = [&](auto d, auto tk) {
    constexpr int D = decltype(d)::value, TK = decltype(tk)::value;
    if (a.type == GRINQH_F16)
      k_attend_join<D, GRINQH_F16, TK><<<grid, kJoinThreads, 0, s>>>(c, b, a, out, lse, part, p.splits, p.per_split, p.rows_log2, groups);
    else
      k_attend_join<D, GRINQH_BF16, TK><<<grid, kJoinThreads, 0, s>>>(c, b, a, out, lse, part, p.splits, p.per_split, p.rows_log2, groups);
  };
  auto on = [&](auto d) {
    if (p.tile) go(d, std::integral_constant<int, 64>{});
    else go(d, std::integral_constant<int, 32>{});
  };
  if (c.D == 64) on(std::integral_constant<int, 64>{});
  else on(std::integral_constant<int, 128>{});
  return check_launch("attend");
}

}  // namespace grinqh
