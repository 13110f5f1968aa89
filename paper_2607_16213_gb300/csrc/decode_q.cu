// How a decode over an 8-bit cache is split (the kernels are in decode_q.cuh, a file for each type).
#include <algorithm>
#include <cmath>

#include "quant.cuh"

namespace selkv {

// Warps of a CTA, splits of a (sequence, KV head) and how many of them make a cluster, from the shape alone.
//
// A CTA goes through its rows in rounds of 32 a warp; a round takes longer where CTAs share an SM, and all rows
// together take no less than HBM gives.  Splits have to be folded: in a cluster, or through global memory, which
// costs more, the more partials there are; or both, for the few heads that need many splits.
// Measured (one token, us; rows x KV heads of all sequences, d 128, four query heads each):
//   2000 x 8     a cluster of 8: 6.6; 8 through memory: 7.5; one split: 13.3
//   25000 x 8    19 through memory: 15.5; a cluster of 8: 21
//   100000 x 1   32 clusters of 4: 12.8; 64 through memory: 15.4
//   16000 x 64   clusters of 4: 43.5, with CTAs of 4 warps 45.8; 4 through memory: 45.3
//   2000 x 192   one split, CTAs of 8 warps: 20.6, of 4: 23.7; clusters of 2: 28.3, of 4 warps 21.6
//   2000 x 512   one split, CTAs of 4 warps: 43.3, of 8: 45.8
//   256 x 2      one split: 4.1; a cluster of 2: 4.9
// The constants below were fitted to the times of all plans (caches larger than L2, a row appended) for 744 batches:
// 1 to 1024 heads, 90 to 130000 rows, 1 to 16 query heads, d 64 and 128, both types, full and ragged.  The plan that
// they choose takes 0.9 percent more than the best one on average and 15 percent at most; of 80 other batches 1.7 and 12.
// (The caches were full to within 100 rows of m_cap, or ragged from a half up: the split follows m_cap, not the lengths,
// so that shorter ones are split further than they need.)
namespace {
double plan_us(const selkv_shape& s, int warps, int S, int cluster) {
  const bool wide = s.num_q_heads / s.num_kv_heads > 8, fp32 = s.dtype == SELKV_FP32;
  const double n = (double)s.batch * s.num_kv_heads, rows = s.m_cap, ctas = n * S;
  const double partial = s.num_q_heads / s.num_kv_heads * s.head_dim / 512.0;  // size of one
  const int groups = S / cluster;
  // CTAs on an SM, and places for CTAs at once (not every SM has room for a whole cluster)
  const double share = std::min((double)ctas_of(warps, wide, fp32, s.head_dim),
                                std::ceil(ctas / (cluster > 1 && ctas > 64 ? 150 : kPlanSMs)));
  const double slots = cluster < 4 ? kPlanSMs * share : cluster == 8 && share == 1 ? 127 : 144 * share;
  const double waves = std::ceil(ctas / slots), idle = std::max(0.0, slots - ctas) / slots;
  static const double kRound[2][4] = {{0.71, 0.78, 0.92, 0.74}, {0.83, 0.99, 0.99, 0.99}};
  const double cta_rows = std::ceil(std::ceil(rows / S) / 64) * 64;
  const double work = waves * cta_rows / (warps * 32) * kRound[warps == 8][(int)share - 1] *
                      (s.head_dim == 64 ? 0.89 : 1) * (fp32 ? 0.89 : 1) * (wide ? 1.1 : 1);
  // (what an SM has in flight, in 64 KB: more than that queues up; 131072 x 8 rows: 44.7 us with 64 KB, 45.6 with 128)
  const double flight = share * warps * s.head_dim / 1024;
  const double hbm = 0.9 * n * rows * s.head_dim * 2 / 6.4e6 * (1 + 0.29 * idle) * (1 + 0.04 * std::max(0.0, flight - 1));
  const double both = std::cbrt(work * work * work + hbm * hbm * hbm);  // (the larger of the two, rounded off)
  return both + 2.6 * (waves - 1) + 0.26 * (share - 1) +
         (cluster == 1 ? 0 : (cluster == 2 ? 1.0 : cluster == 4 ? 1.1 : 1.5) + 0.11 * (partial - 1)) +
         (groups > 1 ? 1.7 + 0.019 * groups * partial : 0);
}

QDecodePlan plan_of(const selkv_shape& s) {
  static const int kGroups[] = {1, 2, 3, 4, 5, 6, 8, 9, 12, 16, 19, 24, 32, 38, 48, 64};
  const bool wide = s.num_q_heads / s.num_kv_heads > 8, fp32 = s.dtype == SELKV_FP32;
  const long n = (long)s.batch * s.num_kv_heads, most = std::min<long>(kMaxSplits, ((long)s.m_cap + 63) / 64);
  QDecodePlan best{};
  double best_us = 0;
  for (int warps = 4; warps <= 8; warps += 4)
    for (int cluster = 1; cluster <= 8; cluster *= 2)
      for (int groups : kGroups) {
        const int S = cluster * groups;
        if (S > 1 && (S > most || n * S > 2 * kPlanSMs * ctas_of(warps, wide, fp32, s.head_dim))) continue;
        const double us = plan_us(s, warps, S, cluster);
        if (best.warps == 0 || us < best_us) {
          best_us = us;
          best = {warps, S, cluster};
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
