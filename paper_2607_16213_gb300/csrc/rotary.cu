// Rotary positions of queries and keys (selkv_rotary_apply).
//
// Pair f of a row at position p turns by p w_f.  The angle in turns is p times the plan's 64-bit fraction of a
// turn per position, and the product's wrap modulo 2^64 takes whole turns off exactly: its upper half is the angle in
// [-1/2, 1/2) turns, right to 2^-33, for any 32-bit position, without 64-bit floating point (which this GPU has little of).
//
// Bound by memory: each element is read and written once.  A CTA takes a tile of tokens and some of the heads: the
// sines and cosines of the tile are computed once and shared by its heads.
#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 16;  // tokens of a tile
constexpr int kHeads = 8;    // heads that share a tile's angles

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
// elements in a row, VEC pairs.  Behind the pairs, items of 2 VEC elements that stay.
template <typename T, int VEC, bool HALF>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const __grid_constant__ RotaryArgs a) {
  __shared__ float2 cs[kTokens][SELKV_ROTARY_MAX_DIM / 2 + 1];
  const int t0 = blockIdx.x * kTokens, nt = min(kTokens, a.T - t0), b = blockIdx.z;
  const int half = a.rot / 2;
  for (int i = threadIdx.x; i < nt * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    const int64_t p = a.positions[(size_t)b * a.T + t0 + t];
    const int32_t turn = (int32_t)(((uint64_t)p * a.turns[f]) >> 32);
    float s, c;
    sincospif((float)turn * 0x1p-31f, &s, &c);
    cs[t][f] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
  }
  __syncthreads();
  const int nq = a.q != nullptr ? a.Hq : 0, heads = nq + (a.k != nullptr ? a.Hkv : 0);
  const int h0 = blockIdx.y * kHeads, nh = min(kHeads, heads - h0);
  const int pairs = half / VEC, items = pairs + (a.D - a.rot) / (2 * VEC);
  const int all = nh * nt * items;
#pragma unroll 2
  for (int i = threadIdx.x; i < all; i += kThreads) {
    const int rest = i / items, it = i - rest * items;
    const int hh = rest / nt, t = rest - hh * nt, h = h0 + hh;
    const bool isq = h < nq;
    const size_t row = isq ? ((size_t)b * a.Hq + h) * a.T : ((size_t)b * a.Hkv + (h - nq)) * a.T;
    const size_t at = (row + t0 + t) * a.D;
    const T* src = static_cast<const T*>(isq ? a.q : a.k) + at;
    T* dst = static_cast<T*>(isq ? a.q_out : a.k_out) + at;
    const bool turns = it < pairs;
    const int e0 = turns && HALF ? it * VEC : turns ? it * 2 * VEC : a.rot + (it - pairs) * 2 * VEC;
    const int e1 = turns && HALF ? e0 + half : e0 + VEC;
    Chunk<T, VEC> x, y;
    x.load(src + e0);
    y.load(src + e1);
    if (turns) {
      const float2* w = cs[t] + it * VEC;
      if constexpr (HALF) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float u = x.x[e], v = y.x[e];
          const float2 c = w[e];
          x.x[e] = u * c.x - v * c.y;
          y.x[e] = v * c.x + u * c.y;
        }
      } else if constexpr (VEC == 1) {
        const float u = x.x[0], v = y.x[0];
        x.x[0] = u * w[0].x - v * w[0].y;
        y.x[0] = v * w[0].x + u * w[0].y;
      } else {
#pragma unroll
        for (int e = 0; e < VEC; e += 2) {
          const float2 c0 = w[e / 2], c1 = w[(VEC + e) / 2];
          const float u0 = x.x[e], v0 = x.x[e + 1], u1 = y.x[e], v1 = y.x[e + 1];
          x.x[e] = u0 * c0.x - v0 * c0.y;
          x.x[e + 1] = v0 * c0.x + u0 * c0.y;
          y.x[e] = u1 * c1.x - v1 * c1.y;
          y.x[e + 1] = v1 * c1.x + u1 * c1.y;
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
  const dim3 grid((unsigned)((a.T + kTokens - 1) / kTokens), (unsigned)((heads + kHeads - 1) / kHeads), (unsigned)a.B);
  if (a.layout == SELKV_ROPE_HALF) rotary_kernel<T, VEC, true><<<grid, kThreads, 0, s>>>(a);
  else rotary_kernel<T, VEC, false><<<grid, kThreads, 0, s>>>(a);
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
