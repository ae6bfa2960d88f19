// Attention of a batch's rows over the paged cache.
#include "kv.h"

namespace grinqh {

// One wave per row and query head: lane = token for the scores, lane = channel
// for the sum over the values.  Running maximum and sum in fp32.
template <int D, int FORMAT, int TYPE>
__global__ void k_attend_simple(KvCache c, KvBatch b, Attend a, DenseRows q, DenseRows out, float* lse) {
  const int lane = threadIdx.x, head = blockIdx.x, s = blockIdx.z, h = head / a.G;
  const Seq sq = kv_seq(c, b, s);
  for (int i = blockIdx.y; i < sq.n; i += gridDim.y) {
    const int row = sq.r0 + i, p = sq.L - sq.n + i;
    const uint16_t* qp = (const uint16_t*)q.p + row * q.row + head * q.head;
    const int lo = a.window ? max(0, p - a.window + 1) : 0, first = min(a.sinks, lo);
    float m = -INFINITY, l = 0, o[D / 64] = {};
    for (int t0 = 0; t0 <= p; t0 += 64) {
      if (t0 >= first && t0 + 63 < lo) continue;
      const int t = t0 + lane;
      const bool sees = t <= p && (t >= lo || t < first);
      const int page = sees ? kv_page(c, b, s, t) : -1;
      const long slot = page >= 0 ? kv_slot(c, page, h, t) : 0;
      float x = sees ? NAN : -INFINITY;
      if (page >= 0) {
        x = 0;
        for (int d = 0; d < D; ++d) {
          const float qd = TYPE == GRINQH_F16 ? h2f(qp[d]) : bf2f(qp[d]);
          if (FORMAT == GRINQH_KV_I8) x += qd * (float)((const int8_t*)c.k)[slot * D + d];
          else {
            const uint16_t kd = ((const uint16_t*)c.k)[slot * D + d];
            x += qd * (FORMAT == GRINQH_KV_F16 ? h2f(kd) : bf2f(kd));
          }
        }
        x *= a.scale;
        if (FORMAT == GRINQH_KV_I8) x *= c.ks[slot];
      }
      float mx = x;
      for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
      const float mn = fmaxf(m, mx), base = mn == -INFINITY ? 0.0f : mn;
      const float alpha = expf(m - base);
      const float e = sees ? expf(x - base) : 0.0f;
      float sum = e;
      for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
      l = l * alpha + sum;
      m = mn;
      for (int j = 0; j < D / 64; ++j) o[j] *= alpha;
      for (int u = 0; u < 64; ++u) {
        const float pu = __shfl(e, u);
        const long su = __shfl(slot, u);
        if (!__shfl((int)sees, u)) continue;
        const float w = FORMAT == GRINQH_KV_I8 ? pu * c.vs[su] : pu;
        for (int j = 0; j < D / 64; ++j) {
          const long at = su * D + j * 64 + lane;
          float vd;
          if (FORMAT == GRINQH_KV_I8) vd = (float)((const int8_t*)c.v)[at];
          else vd = FORMAT == GRINQH_KV_F16 ? h2f(((const uint16_t*)c.v)[at]) : bf2f(((const uint16_t*)c.v)[at]);
          o[j] += w * vd;
        }
      }
    }
    const float inv = l == 0 ? 0.0f : 1.0f / l;
    uint16_t* op = (uint16_t*)out.p + row * out.row + head * out.head;
    for (int j = 0; j < D / 64; ++j) {
      const float y = o[j] * inv;
      op[j * 64 + lane] = TYPE == GRINQH_F16 ? f2h_rn(y) : f2bf_rn(y);
    }
    if (lse && lane == 0) lse[(long)row * a.heads + head] = l == 0 ? -INFINITY : m + logf(l);
  }
}

size_t attend_workspace(const KvCache&, const Attend&, int, int) { return 0; }

int launch_attend(const KvCache& c, const KvBatch& b, const Attend& a, const DenseRows& q, const DenseRows& out,
                  float* lse, void*, hipStream_t s) {
  const dim3 grid(a.heads, min(min(a.max_rows, b.rows), 32768), b.B);
  auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (c.format == GRINQH_KV_F16) k_attend_simple<D, GRINQH_KV_F16, GRINQH_F16><<<grid, 64, 0, s>>>(c, b, a, q, out, lse);
    else if (c.format == GRINQH_KV_BF16) k_attend_simple<D, GRINQH_KV_BF16, GRINQH_BF16><<<grid, 64, 0, s>>>(c, b, a, q, out, lse);
    else if (a.type == GRINQH_F16) k_attend_simple<D, GRINQH_KV_I8, GRINQH_F16><<<grid, 64, 0, s>>>(c, b, a, q, out, lse);
    else k_attend_simple<D, GRINQH_KV_I8, GRINQH_BF16><<<grid, 64, 0, s>>>(c, b, a, q, out, lse);
  };
  if (c.D == 64) go(std::integral_constant<int, 64>{});
  else go(std::integral_constant<int, 128>{});
  return check_launch("attend");
}

}  // namespace grinqh
