// Caches held in 8 bits: a code per element and one fp32 scale per `block` rows of a KV head;
// element = code * scale.
//
// Scale of a block that a call writes from its first row on, with A the largest finite magnitude of the
// rows: the smallest s of a grid with s * qmax >= A, at least 2^-100 (blocks of zeros).  The grids
// are the powers of two for e4m3 (qmax 448: a finer scale gains a floating-point code nothing) and the
// numbers m/8 * 2^e, m = 8..15, for int8 (qmax 127: at most an eighth of the codes' range is lost).
// On these grids a product of code and scale is exact in fp32, the quotient of a bf16
// element never rounds onto the border between two codes, and scaling e4m3 codes by a power of two is exact
// above the subnormals.
// A block that holds rows already keeps its scale s0 times 2^k, k >= 0 the smallest that covers the
// new rows; with k > 0 the old codes become RNE(code * 2^-k).
#pragma once

#include <cuda_fp16.h>

#include "ptx.cuh"
#include "selkv_internal.cuh"

namespace selkv {

constexpr float kMinScale = 7.888609052210118e-31f;  // 2^-100

template <int TYPE>
struct Code;

__device__ __forceinline__ uint32_t cvt_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// Two e4m3 codes as two halves (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t codes16) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)codes16));
  return r;
}

template <>
struct Code<SELKV_Q_E4M3> {
  static constexpr float kMax = 448.f;
  // Smallest power of two s with 448 s >= a: 448 = 1.75 * 2^8.
  __device__ static __forceinline__ float fresh_scale(float a) {
    const int bits = __float_as_int(a);
    const int e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
    return a > 448.f * kMinScale ? __int_as_float(e << 23) : kMinScale;
  }
  // Four elements, as they are after the division by the scale.
  __device__ static __forceinline__ uint32_t pack4(const float (&y)[4]) {
    return cvt_e4m3x2(y[0], y[1]) | cvt_e4m3x2(y[2], y[3]) << 16;
  }
  __device__ static __forceinline__ void unpack4(uint32_t w, float (&y)[4]) {
    const uint32_t a = e4m3x2_to_f16x2(w), b = e4m3x2_to_f16x2(w >> 16);
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&a));
    const float2 hi = __half22float2(*reinterpret_cast<const __half2*>(&b));
    y[0] = lo.x, y[1] = lo.y, y[2] = hi.x, y[3] = hi.y;
  }
  // Element over scale.  1 / s is a power of two unless the caller brought the scale.
  __device__ static __forceinline__ float quotient(float x, float s, float rcp, bool any_scale) {
    return any_scale ? __fdiv_rn(x, s) : x * rcp;
  }
};

template <>
struct Code<SELKV_Q_INT8> {
  static constexpr float kMax = 127.f;
  // a = F 2^(k-23), F of 24 bits: s = M 2^(k-10) with the smallest M such that 127 * 2^13 M >= F; M = 16
  // and 17 (round up to 18) belong to the next power of two.
  __device__ static __forceinline__ float fresh_scale(float a) {
    const uint32_t bits = __float_as_uint(a);
    const uint32_t F = (bits & 0x7fffffu) | 0x800000u;
    uint32_t M = (F + 127u * 8192u - 1u) / (127u * 8192u);
    uint32_t e = (bits >> 23) - 7u;  // biased exponent of M/8 * 2^(k-7) for M = 8..15
    if (M >= 16u) {
      M = (M + 1u) >> 1;
      ++e;
    }
    return a > 127.f * kMinScale ? __uint_as_float(e << 23 | (M - 8u) << 20) : kMinScale;
  }
  // The codes are integers already (quotient rounds).
  __device__ static __forceinline__ uint32_t pack4(const float (&y)[4]) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= (uint32_t)(max(-127, min(127, __float2int_rn(y[i]))) & 0xff) << (8 * i);
    return w;
  }
  __device__ static __forceinline__ void unpack4(uint32_t w, float (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (float)(int8_t)(w >> (8 * i));
  }
  // Element over scale, still to be rounded to an integer.  With a scale of the grid and a bf16 element
  // the quotient is one of an 8-bit by a 4-bit number: where it lies on a border of two codes it is
  // exact in fp32, else at least 2^-9 of itself away from one.  The product with the rounded 1 / s misses some of the borders
  // by its last place; with its remainder added back it rounds as the quotient in every case (all
  // were gone through on the host).  Otherwise the integer itself is checked against the remainder.
  __device__ static __forceinline__ float quotient(float x, float s, float rcp, bool any_scale) {
    const float q = x * rcp;
    if (!(fabsf(q) < 1024.f)) return q;  // an infinity or NaN
    if (!any_scale) return fmaf(fmaf(-q, s, x), rcp, q);
    const float c = rintf(q), r = fmaf(-c, s, x), h = 0.5f * s;
    const bool odd = ((int)c & 1) != 0;
    return fabsf(r) > h || (fabsf(r) == h && odd) ? c + copysignf(1.f, r) : c;
  }
};

// Scale of a block with rows in it: any normal number, as the caller may have set it.  (Anything smaller or a NaN, which no
// block with rows has, counts as the smallest fresh one.)
__device__ __forceinline__ float held_scale(float s) { return s >= 1.1754943508222875e-38f ? s : kMinScale; }
// The same for new rows of largest magnitude a.
template <int TYPE>
__device__ __forceinline__ float grown_scale(float old, float a) {
  const float most = old * Code<TYPE>::kMax;
  if (!(a > most)) return old;
  int k = (int)(__float_as_uint(a) >> 23) - (int)(__float_as_uint(most) >> 23);
  if (ldexpf(most, k) < a) ++k;
  return ldexpf(old, k);
}

// |x| where it is finite, else 0; *odd is set where it is not.
__device__ __forceinline__ float finite_abs(float x, bool* odd) {
  const float a = fabsf(x);
  if (a < INFINITY) return a;
  *odd = true;
  return 0.f;
}

// ---- arguments ----------------------------------------------------------------------------
struct QCache {
  int type, block_log2, nblk;  // nblk = ceil(m_cap / block)
  uint8_t *K, *V;              // [B][Hkv][m_cap][d]
  float *ks, *vs;              // [B][Hkv][nblk]
  float* bias;                 // [B][Hkv][m_cap] or null
  int32_t* lengths;            // [B]
};

struct QAppendArgs {
  QCache c;
  int dtype, B, Hkv, D, m_cap, rows;
  const void *k_new, *v_new;  // [B][Hkv][rows][d]
  const float* bias_new;      // [B][Hkv][rows] or null (zeros)
  const int32_t* counts;      // [B] or null (all rows)
  uint32_t* flags;
  uint32_t* cnt_seq;          // [B] arrivals (self-resetting)
};
cudaError_t launch_qappend(const QAppendArgs& a, cudaStream_t s);

struct QReadArgs {
  QCache c;
  int dtype, B, Hkv, D, m_cap, row0, rows;
  void *k_out, *v_out;  // [B][Hkv][rows][d]
  uint32_t* flags;
};
cudaError_t launch_qread(const QReadArgs& a, cudaStream_t s);

// Decode over an 8-bit cache: DecodeArgs without Kc and Vc.
struct QDecodeArgs : DecodeArgs {
  QCache c;
  int warps;
  int cluster;  // CTAs of a cluster: 1, 2, 4 or 8; divides the splits
};
// Warps of a CTA and splits of a (sequence, KV head)'s rows.
struct QDecodePlan {
  int warps, splits, cluster;
};
QDecodePlan decode_q_plan(const selkv_shape& s);
// CTA sizes: few (sequence, KV head) pairs get large CTAs, one or two on an SM (few splits to fold); many get small
// ones.  CTAs on an SM, as registers allow (wide: more than eight heads).
constexpr int kMaxQCtas = 4;
constexpr int ctas_of(int warps, bool wide, bool fp32, int d) {
  if (!wide && !fp32) return warps == 8 ? 2 : kMaxQCtas;
  return warps == 8 ? 1 : d == 64 && !(wide && fp32) ? 3 : 2;
}
constexpr int kMaxSplits = kPlanSMs;
// CTAs of a decode whose (sequence, KV head) pairs are split, all together: two waves (plan_of).
constexpr int kMaxQSplitCtas = 2 * kPlanSMs * kMaxQCtas;
// Floats of a (sequence, KV head)'s record of partials, where there are several clusters (Sg).
__host__ __device__ constexpr size_t decode_q_record_floats(int G, int Sc, int Sg, int D) {
  return (size_t)G * Sg * D + (((size_t)Sc * G * Sg * 2 + 3) & ~(size_t)3);
}
cudaError_t launch_decode_q(const QDecodeArgs& a, cudaStream_t s);
cudaError_t launch_decode_q_e4m3(const QDecodeArgs& a, cudaStream_t s);
cudaError_t launch_decode_q_int8(const QDecodeArgs& a, cudaStream_t s);

// One lane's elements of a row of D, as fp32, by a whole warp: lane l holds l * D / 32 onwards.
template <typename T, int D>
__device__ __forceinline__ void load_row(const T* row, float (&x)[D / 32]) {
  const int lane = threadIdx.x & 31;
  if constexpr (D == 128) load4(row + lane * 4, x);
  else load2(row + lane * 2, x);
}

// One warp puts the row `x` (one of K or V of a KV head) into row L of its codes: its block's scale covers
// it, and if that had to grow the block's rows are encoded anew.  No one else may be reading the block.
template <int TYPE, typename T, int D>
__device__ __forceinline__ void append_row(const T* x, uint8_t* codes, float* scales, int block_log2, int L,
                                           uint32_t* flags) {
  using C = Code<TYPE>;
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  float v[N], a = 0.f;
  load_row<T, D>(x, v);
  bool odd = false;
#pragma unroll
  for (int i = 0; i < N; ++i) a = fmaxf(a, finite_abs(v[i], &odd));
  a = warp_max(a);
  if (odd) raise_flag(flags, SELKV_DEVERR_VALUE);
  const int blk = L >> block_log2, first = blk << block_log2;
  const bool holds = L > first;
  const float s0 = holds ? held_scale(scales[blk]) : 0.f;
  const float s = holds ? grown_scale<TYPE>(s0, a) : C::fresh_scale(a);
  if (holds && s != s0) {
    const float f = s0 / s;  // 2^-k
    uint32_t* w = reinterpret_cast<uint32_t*>(codes + (size_t)first * D);
    for (int i = lane; i < (L - first) * (D / 4); i += 32) {
      float y[4];
      C::unpack4(w[i], y);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] *= f;
      w[i] = C::pack4(y);
    }
  }
  __syncwarp();
  if (lane == 0) scales[blk] = s;
  const float rcp = 1.f / s;
  float y[4] = {};
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = C::quotient(v[i], s, rcp, holds || sizeof(T) == 4);
  const uint32_t w = C::pack4(y);
  uint8_t* dst = codes + (size_t)L * D + lane * N;
  if constexpr (N == 4) *reinterpret_cast<uint32_t*>(dst) = w;
  else *reinterpret_cast<uint16_t*>(dst) = (uint16_t)w;
}

}  // namespace selkv
