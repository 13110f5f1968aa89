// Compensated decode attention over an 8-bit cache.
//
//   out[b][h] = sum_i softmax_i(q_h . k_i / sqrt(d) + bias_i) v_i,   k_i = code * scale, v_i = code * scale
//
// Split-K flash decoding: CTA (split, KV head, sequence) walks a slice of the rows, a row a warp at a
// time, all query heads of the group together; the splits are folded as in decode_simt.cu.
#include <algorithm>

#include "decode_common.cuh"
#include "quant.cuh"

namespace selkv {
namespace {

constexpr int kWarps = 4;

// Bias in base 2.  The lowest finite numbers stay finite: rows that all have them share the weight.
__device__ __forceinline__ float bias_log2(float b) {
  return b == -INFINITY ? b : fmaxf(b * kLog2e, -3.402823466e38f);
}

template <int TYPE, typename T, int D, int GM>
__global__ __launch_bounds__(kWarps * 32) void decode_q_kernel(QDecodeArgs a) {
  constexpr int N = D / 32;
  __shared__ float wm[kWarps][GM], wl[kWarps][GM];
  __shared__ __align__(16) float wo[kWarps][GM][D];
  __shared__ bool s_last;
  const int s = blockIdx.x, kv = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = a.G, S = a.splits;
  const size_t bk = (size_t)b * a.Hkv + kv;
  int L = a.lengths[b];
  if (L < 0 || L > a.m_cap) {
    if (tid == 0 && s == 0 && kv == 0) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = L < 0 ? 0 : a.m_cap;
  }
  bool app = a.k_new != nullptr;
  if (app && L + 1 > a.m_cap) {
    if (tid == 0 && s == 0 && kv == 0) raise_flag(a.flags, SELKV_DEVERR_CAPACITY);
    app = false;
  }
  const int total = L + (app ? 1 : 0);
  const int chunk = (total + S - 1) / S;
  const int lo = min(total, s * chunk), hi = min(total, lo + chunk);
  const uint8_t *Kb = a.c.K + bk * a.m_cap * D, *Vb = a.c.V + bk * a.m_cap * D;
  const float* bias = a.bias != nullptr ? a.bias + bk * a.m_cap : nullptr;
  float q[GM][N], m[GM], l[GM], o[GM][N];
#pragma unroll
  for (int g = 0; g < GM; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
    if (g < G) load_row<T, D>(static_cast<const T*>(a.q) + ((size_t)b * a.Hq + kv * G + g) * D, q[g]);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      q[g][e] = g < G ? q[g][e] * a.scale_log2 : 0.f;
      o[g][e] = 0.f;
    }
  }
  for (int key = lo + warp; key < hi; key += kWarps) {
    float k[N], v[N];
    float bv = 0.f;
    if (key < L) {
      const int blk = key >> a.c.block_log2;
      const float ks = a.c.ks[bk * a.c.nblk + blk], vs = a.c.vs[bk * a.c.nblk + blk];
      uint32_t kw, vw;
      if constexpr (N == 4) {
        kw = *reinterpret_cast<const uint32_t*>(Kb + (size_t)key * D + lane * 4);
        vw = *reinterpret_cast<const uint32_t*>(Vb + (size_t)key * D + lane * 4);
      } else {
        kw = *reinterpret_cast<const uint16_t*>(Kb + (size_t)key * D + lane * 2);
        vw = *reinterpret_cast<const uint16_t*>(Vb + (size_t)key * D + lane * 2);
      }
      float k4[4], v4[4];
      Code<TYPE>::unpack4(kw, k4);
      Code<TYPE>::unpack4(vw, v4);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        k[e] = k4[e] * ks;
        v[e] = v4[e] * vs;
      }
      if (bias != nullptr) bv = bias_log2(bias[key]);
    } else {
      load_row<T, D>(static_cast<const T*>(a.k_new) + bk * D, k);
      load_row<T, D>(static_cast<const T*>(a.v_new) + bk * D, v);
    }
#pragma unroll
    for (int g = 0; g < GM; ++g) {
      if (g >= G) break;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) x = fmaf(q[g][e], k[e], x);
      x = warp_sum(x) + bv;
      const float mn = fmaxf(m[g], x);
      const float mref = mn == -INFINITY ? 0.f : mn;
      const float corr = exp2f(m[g] - mref), p = exp2f(x - mref);
      l[g] = l[g] * corr + p;
#pragma unroll
      for (int e = 0; e < N; ++e) o[g][e] = fmaf(p, v[e], o[g][e] * corr);
      m[g] = mn;
    }
  }
#pragma unroll
  for (int g = 0; g < GM; ++g) {
    if (g >= G) break;
    if (lane == 0) {
      wm[warp][g] = m[g];
      wl[warp][g] = l[g];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) wo[warp][g][lane * N + e] = o[g][e];
  }
  __syncthreads();
  write_split_partial<kWarps>(a, b, kv, s, &wo[0][0][0], &wm[0][0], &wl[0][0], GM, D, false);
  if (!arrive_last(a, bk, &s_last)) return;
  combine_splits<T>(a, b, kv, nullptr);
  if (app) {  // every split of this KV head has read its rows
    if (warp == 0)
      append_row<TYPE, T, D>(static_cast<const T*>(a.k_new) + bk * D, a.c.K + bk * a.m_cap * D, a.c.ks + bk * a.c.nblk,
                             a.c.block_log2, L, a.flags);
    if (warp == 1)
      append_row<TYPE, T, D>(static_cast<const T*>(a.v_new) + bk * D, a.c.V + bk * a.m_cap * D, a.c.vs + bk * a.c.nblk,
                             a.c.block_log2, L, a.flags);
    if (tid == 0 && a.bias != nullptr) a.bias[bk * a.m_cap + L] = 0.f;
  }
  finish_lengths(a, b, bk, L, app);
}

template <int TYPE, typename T, int D>
cudaError_t launch_t(const QDecodeArgs& a, cudaStream_t st) {
  const dim3 grid(a.splits, a.Hkv, a.B);
  if (a.G <= 4) decode_q_kernel<TYPE, T, D, 4><<<grid, kWarps * 32, 0, st>>>(a);
  else decode_q_kernel<TYPE, T, D, 16><<<grid, kWarps * 32, 0, st>>>(a);
  return cudaGetLastError();
}

template <int TYPE>
cudaError_t launch_type(const QDecodeArgs& a, cudaStream_t st) {
  if (a.dtype == SELKV_BF16)
    return a.D == 128 ? launch_t<TYPE, __nv_bfloat16, 128>(a, st) : launch_t<TYPE, __nv_bfloat16, 64>(a, st);
  return a.D == 128 ? launch_t<TYPE, float, 128>(a, st) : launch_t<TYPE, float, 64>(a, st);
}

}  // namespace

int decode_q_splits(const selkv_shape& s) { return decode_splits(s.batch, s.num_kv_heads, s.m_cap, kPlanSMs, false); }

cudaError_t launch_decode_q(const QDecodeArgs& a, cudaStream_t st) {
  return a.c.type == SELKV_Q_E4M3 ? launch_type<SELKV_Q_E4M3>(a, st) : launch_type<SELKV_Q_INT8>(a, st);
}

}  // namespace selkv
