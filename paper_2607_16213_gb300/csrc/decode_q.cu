// How a decode over an 8-bit cache is split (the kernels are in decode_q.cuh, a file for each type).
#include <algorithm>

#include "quant.cuh"

namespace selkv {

// Warps of a CTA, splits of a (sequence, KV head) and how many of them make a cluster, from the shape alone.
//
// A CTA goes through its rows in rounds of 32 a warp; a round takes about 1.2 us, longer where CTAs share
// an SM, a further wave of CTAs starts 2 us late, and all rows together take no less than HBM gives.  Splits have to be folded: in a cluster about 1.5 us,
// through global memory about 3 us and 50 ns a partial; both, for the few heads that need many splits.
// Measured (one token, us; rows x KV heads of all sequences, d 128):
//   25000 x 8    splits through memory 19: 15.3, 38: 16.8; clusters of 8: 21, 2 x 9: 17.0, 4 x 4: 17.3
//   2000 x 8     clusters of 8: 8.3; through memory 8: 9.4; one split: 14.2
//   100000 x 1   64 through memory: 16.8; 36 clusters of 4: 13.7
//   12000 x 32   through memory 4: 24.4, 9: 19.6; clusters of 8: 20.4
//   819 x 512    CTAs of 4 warps: 22, of 8: 27 (four and two on an SM; one CTA of 8 warps: 43)
//   256 x 2      one split: 4.9, two: 5.9
// Clusters of more than 64 CTAs in all are placed two CTAs to an SM although others are free (25000 x 16
// as clusters of 8: 29 us, split through memory 24), and larger ones than 8 are not placed everywhere.
namespace {
QDecodePlan plan_of(const selkv_shape& s) {
  const long n = (long)s.batch * s.num_kv_heads, rows = s.m_cap;
  const bool wide = s.num_q_heads / s.num_kv_heads > 8 || s.dtype == SELKV_FP32;
  const int warps = n >= kPlanSMs / 2 ? 4 : 8;
  const long per_sm = ctas_of(warps, wide);
  // ns of a round with 1, 2, 3 and 4 CTAs on an SM
  static const long kRound[2][4] = {{900, 1200, 1600, 2000}, {1200, 1900, 0, 0}};
  const long hbm_ns = 9 * n * rows * s.head_dim * 2 / (10 * 6300);
  QDecodePlan best{};
  long best_ns = -1;
  for (int cluster = 1; cluster <= 8; cluster *= 2) {
    const long most = std::min<long>(kMaxSplits, (rows + 63) / 64) / cluster;
    for (long groups = 1; groups <= most; ++groups) {
      const long S = cluster * groups;
      const long ctas = n * S, sms = cluster > 1 && ctas > 64 ? kPlanSMs / 2 : kPlanSMs;
      const long share = std::min(per_sm, (ctas + sms - 1) / sms);
      // CTAs placed at once (clusters of 8 with an SM for each CTA: 15)
      const long slots = cluster < 4 ? kPlanSMs * share : cluster == 8 && share == 1 ? 120 : 144 * share;
      const long waves = (ctas + slots - 1) / slots;
      const long cta_rows = ((rows + S - 1) / S + 63) / 64 * 64, round = kRound[warps == 8][share - 1];
      const long idle = std::max(0L, slots - ctas);  // places without a CTA: HBM gives up to a quarter less
      const long ns = std::max(waves * (cta_rows * round / (warps * 32) + round / 2), hbm_ns + hbm_ns * idle / (4 * slots)) +
                      2000 * (waves - 1) + (cluster > 1 ? 1500 : 0) + (groups > 1 ? 3000 + 50 * groups : 0);
      if (best_ns < 0 || ns < best_ns) {
        best_ns = ns;
        best = {warps, (int)S, cluster};
      }
      if (n * S > 16L * kPlanSMs) break;
    }
  }
  return best;
}
}  // namespace

// (The search takes some microseconds; a decode comes back with the same shape call after call.)
QDecodePlan decode_q_plan(const selkv_shape& s) {
  static thread_local selkv_shape of{};
  static thread_local QDecodePlan plan{};
  if (plan.warps == 0 || of.dtype != s.dtype || of.batch != s.batch || of.num_q_heads != s.num_q_heads ||
      of.num_kv_heads != s.num_kv_heads || of.head_dim != s.head_dim || of.m_cap != s.m_cap) {
    plan = plan_of(s);
    of = s;
  }
  return plan;
}

cudaError_t launch_decode_q(const QDecodeArgs& a, cudaStream_t st) {
  return a.c.type == SELKV_Q_E4M3 ? launch_decode_q_e4m3(a, st) : launch_decode_q_int8(a, st);
}

}  // namespace selkv
