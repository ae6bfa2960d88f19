// Attention of a batch's rows over the paged cache: how a call is launched,
// and the joining of sequences that were split.
#include "attend.h"

#include <algorithm>

namespace grinqh {

namespace {

// One group of D / 8 lanes per row and head: the splits' results weighed by their sums.
template <int D, int TYPE>
__global__ void k_attend_join(KvCache c, KvBatch b, Attend a, DenseRows out, float* lse, Partial part, int splits) {
  constexpr int LPR = D / 8;
  const int s = blockIdx.z, lane = threadIdx.x % LPR;
  const Seq sq = kv_seq(c, b, s);
  const long all = (long)sq.n * a.heads;
  const int per_block = blockDim.x / LPR;
  for (long r = (long)blockIdx.x * per_block + threadIdx.x / LPR; r < all; r += (long)gridDim.x * per_block) {
    const long at = (long)sq.r0 * a.heads + r;
    float m = -INFINITY;
    for (int i = lane; i < splits; i += LPR) m = fmaxf(m, part.lse[i * part.rows + at]);
    for (int x = LPR / 2; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, LPR));
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0, y[8] = {};
    for (int i = 0; i < splits; ++i) {
      const float z = part.lse[i * part.rows + at];
      if (z == -INFINITY) continue;
      const float w = exp2f(z - base);
      const float4v* p = (const float4v*)(part.o + (i * part.rows + at) * D + lane * 8);
      sum += w;
      for (int j = 0; j < 8; ++j) y[j] += w * p[j / 4][j % 4];
    }
    const float inv = sum == 0 ? 0.0f : 1.0f / sum;
    uint32_t w[4];
    for (int j = 0; j < 4; ++j) w[j] = pack2<TYPE>(y[2 * j] * inv, y[2 * j + 1] * inv);
    *(u32x4*)(out.p + ((sq.r0 + r / a.heads) * out.row + (r % a.heads) * out.head + lane * 8) * 2) = u32x4{w[0], w[1], w[2], w[3]};
    if (lse && lane == 0) lse[at] = sum == 0 ? -INFINITY : (m + log2f(sum)) * kLn2;
  }
}

AttendPlan attend_plan(const KvCache& c, const Attend& a, int B, int rows) {
  AttendPlan p = {};
  const int forced = option(&Options::attend_kernel), forced_splits = option(&Options::attend_splits);
  const long n = std::min(a.max_rows, rows), R = n * a.G;
  p.tile = forced ? forced != GRINQH_ATTEND_ROWS : R > 32;
  p.nb = p.tile ? (forced == GRINQH_ATTEND_TILE_4 ? 4 : 8) : R > 16 ? 2 : 1;
  const long per_block = p.tile ? 32 * p.nb : 16 * p.nb, tile = p.tile ? 64 : 32;
  p.blocks = (int)std::min<long>((R + per_block - 1) / per_block, 65535);
  // tiles that the longest sequence's last block sees
  const long seen = a.window ? std::min<long>(a.max_len, (long)a.window + per_block / a.G + a.sinks + 2 * tile) : a.max_len;
  const long tiles = (seen + tile - 1) / tile, groups = (long)B * c.H * p.blocks;
  const long fill = p.tile ? (p.nb == 4 ? 2 : 1) * device_cus() : 2 * device_cus();
  long splits = forced_splits ? forced_splits : std::min(std::max<long>(1, fill / groups), std::max<long>(1, tiles / 8));
  long per = (tiles + splits - 1) / splits;
  if (!p.tile) per = (per + 3) / 4 * 4;
  p.per_split = (int)per;
  p.splits = (int)((tiles + per - 1) / per);
  return p;
}

}  // namespace

size_t partial_bytes(const AttendPlan& p, const KvCache& c, const Attend& a, int rows) {
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
  (p.tile ? launch_attend_tile : launch_attend_rows)(p, c, b, a, q, out, lse, part, s);
  int st = check_launch("attend");
  if (st || p.splits == 1) return st;
  const long per_seq = (long)std::min(a.max_rows, b.rows) * a.heads * (c.D / 8);
  const dim3 grid((unsigned)std::min<long>((per_seq + 255) / 256, 1 << 20), 1, b.B);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (a.type == GRINQH_F16) k_attend_join<D, GRINQH_F16><<<grid, 256, 0, s>>>(c, b, a, out, lse, part, p.splits);
    else k_attend_join<D, GRINQH_BF16><<<grid, 256, 0, s>>>(c, b, a, out, lse, part, p.splits);
  };
  if (c.D == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return check_launch("attend");
}

}  // namespace grinqh
