// Rotary positions of queries and keys (selkv_rotary_apply).
//
// Pair f of a row at position p turns by p w_f.  The angle in turns is p times the plan's 64-bit fraction of a
// turn per position, and the product's wrap modulo 2^64 takes whole turns off exactly: its upper half is the angle in
// [-1/2, 1/2) turns, right to 2^-31 for any 32-bit position (the plan's fraction to 2^-65, and what is cut off), without 64-bit
// floating point (which this GPU has little of).  The sine's argument is that in fp32: right to 2^-26 turns.
//
// Bound by memory: each element is read and written once (16384 tokens x 40 heads, d 128, bf16: 56 us, 88% of the copy rate; 8
// tokens: 3.3, a launch's latency).  A thread has the same pairs of one token in all heads of its
// CTA: their sines and cosines are computed once and stay in its registers.
#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kThreads = 256;
constexpr int kMostHeads = 32, kFewestHeads = 4;  // heads of a CTA (16384 tokens: 32 56.2 us, 8 58.9; 8 tokens: 4 3.3, 32 12.0)

// VEC elements of a thread at a time (16 bytes where the pairs allow it).
template <typename T, int VEC>
struct Chunk {
  float x[VEC];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (VEC == 8) load8(p, x);
    else if constexpr (VEC == 4) load4(p, reinterpret_cast<float(&)[4]>(x));
    else if constexpr (VEC == 2) load2(p, reinterpret_cast<float(&)[2]>(x));
    else x[0] = load1(p);
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (VEC == 8) {
      uint4 u = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
      *reinterpret_cast<uint4*>(p) = u;
    } else if constexpr (VEC == 4) {
      store4(p, reinterpret_cast<const float(&)[4]>(x));
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) store1(p + e, x[e]);
    }
  }
};

// HALF layout: an item is VEC elements of the first half and their partners; INTERLEAVED: 2 VEC
// elements in a row, VEC pairs.  Behind the pairs, items of 2 VEC elements that stay.  A thread an item of a token.
template <typename T, int VEC, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const __grid_constant__ RotaryArgs a, int nheads) {
  const int half = a.rot / 2, pairs = half / VEC, items = pairs + (a.D - a.rot) / (2 * VEC), tokens = kThreads / items;
  const int ti = threadIdx.x / items, it = threadIdx.x - ti * items, b = blockIdx.z;
  const uint32_t t = blockIdx.x * tokens + ti;  // (the last CTA's may pass 2^31)
  if (ti >= tokens || t >= (uint32_t)a.T) return;
  const bool turns = it < pairs;
  float c[VEC], s[VEC];
  if (turns) {
    const int64_t p = a.positions[(size_t)b * a.T + t];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const int32_t turn = (int32_t)(((uint64_t)p * a.turns[it * VEC + e]) >> 32);
      sincospif((float)turn * 0x1p-31f, &s[e], &c[e]);
      c[e] *= a.amplitude;
      s[e] *= a.amplitude * a.sign;
    }
  }
  const int e0 = turns && HALF ? it * VEC : turns ? it * 2 * VEC : a.rot + (it - pairs) * 2 * VEC;
  const int e1 = turns && HALF ? e0 + half : e0 + VEC;
  const int nq = a.q != nullptr ? a.Hq : 0, heads = nq + (a.k != nullptr ? a.Hkv : 0);
  const int h0 = blockIdx.y * nheads, h1 = min(heads, h0 + nheads);
#pragma unroll 4
  for (int h = h0; h < h1; ++h) {
    const bool isq = h < nq;
    const size_t at = ((isq ? (size_t)b * a.Hq + h : (size_t)b * a.Hkv + (h - nq)) * a.T + t) * a.D;
    const T* src = static_cast<const T*>(isq ? a.q : a.k) + at;
    T* dst = static_cast<T*>(isq ? a.q_out : a.k_out) + at;
    Chunk<T, VEC> x, y;
    x.load(src + e0);
    y.load(src + e1);
    if (turns) {
      if constexpr (HALF || VEC == 1) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float u = x.x[e], v = y.x[e];
          x.x[e] = u * c[e] - v * s[e];
          y.x[e] = v * c[e] + u * s[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const int f0 = e / 2, f1 = (VEC + e) / 2;
          const float u0 = x.x[e], v0 = x.x[e + 1], u1 = y.x[e], v1 = y.x[e + 1];
          x.x[e] = u0 * c[f0] - v0 * s[f0];
          x.x[e + 1] = v0 * c[f0] + u0 * s[f0];
          y.x[e] = u1 * c[f1] - v1 * s[f1];
          y.x[e + 1] = v1 * c[f1] + u1 * s[f1];
        }
      }
    }
    x.store(dst + e0);
    y.store(dst + e1);
  }
}

template <typename T, int VEC>
cudaError_t launch(const RotaryArgs& a, cudaStream_t s) {
  const int heads = (a.q != nullptr ? a.Hq : 0) + (a.k != nullptr ? a.Hkv : 0);
  const int items = a.rot / (2 * VEC) + (a.D - a.rot) / (2 * VEC), tokens = kThreads / items;
  const int64_t across = ((int64_t)a.T + tokens - 1) / tokens, tiles = across * a.B;
  // many heads share a thread's angles, but not so many that SMs stay empty
  int each = kMostHeads;
  while (each > kFewestHeads && tiles * ((heads + each - 1) / each) < 4 * kPlanSMs) each /= 2;
  const dim3 grid((unsigned)across, (unsigned)((heads + each - 1) / each), (unsigned)a.B);
  if (a.layout == SELKV_ROPE_HALF) rotary_kernel<T, VEC, true><<<grid, kThreads, 0, s>>>(a, each);
  else rotary_kernel<T, VEC, false><<<grid, kThreads, 0, s>>>(a, each);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t s) {
  // whole vectors where both the pairs and what is behind them come in them
  const int vec = a.dtype == SELKV_BF16 ? 8 : 4;
  const bool whole = a.rot % (2 * vec) == 0;
  if (a.dtype == SELKV_BF16) return whole ? launch<__nv_bfloat16, 8>(a, s) : launch<__nv_bfloat16, 1>(a, s);
  return whole ? launch<float, 4>(a, s) : launch<float, 1>(a, s);
}

}  // namespace selkv
