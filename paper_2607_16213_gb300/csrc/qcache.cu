// Writing rows into an 8-bit cache and reading them back (quant.cuh has the scales and codes).
//
// Append: a CTA takes 128 rows of the cache at a time, aligned to 128, of one KV head's K or V: whole blocks, so
// no two CTAs share a scale.  A warp takes 8 or 16 of the rows and keeps them in registers between the
// largest magnitude and the codes: an element is read once and a code written once.  Read: a thread takes 16
// codes at a time.  Both are bound by HBM: 131072 x 8 rows of bf16 and d 128 are written in 122 us (805 MB, 6.6
// TB/s), eight ragged caches of 8192-16384 x 8 read in 84 us (557 MB, 6.6 TB/s).
#include <algorithm>

#include "quant.cuh"

namespace selkv {
namespace {

constexpr int kTileRows = 128;
// Rows of a warp: at most 32 registers of elements a lane, and no more than the smallest block.  CTAs of a tile on an
// SM: as many as registers hold (25000 x 8 rows of bf16, d 128: two or three CTAs 33.9 us, four 30.8,
// five 29.7, six 35.5).
template <typename T, int D>
struct ACfg {
  static constexpr bool kLight = D * sizeof(T) == 128;
  static constexpr int kWarpRows = D * sizeof(T) == 512 ? 8 : 16;
  static constexpr int kThreads = kTileRows / kWarpRows * 32;
  static constexpr int kCtas = (kLight ? 2048 : 1280) / kThreads;
};

// Four consecutive elements of 16 loaded bytes.
__device__ __forceinline__ void elements4(const uint4& w, int half, __nv_bfloat16, float (&x)[4]) {
  const uint32_t a = half ? w.z : w.x, b = half ? w.w : w.y;
  x[0] = bf16_lo(a), x[1] = bf16_hi(a), x[2] = bf16_lo(b), x[3] = bf16_hi(b);
}
__device__ __forceinline__ void elements4(const uint4& w, int, float, float (&x)[4]) {
  x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
}
// Bits of the largest magnitude of 16 loaded bytes as an fp32 number (magnitudes order as their bits do;
// infinities and NaN above the finite ones).
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
template <typename T, int N>
__device__ __forceinline__ uint32_t max_bits(const uint4 (&w)[N]) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 2) m = max_u16x2(m, u[k] & 0x7fff7fffu);
      else m = max(m, u[k] & 0x7fffffffu);
    }
  }
  if constexpr (sizeof(T) == 2) m = max(m << 16, m & 0xffff0000u);
  return m;
}
// The largest finite magnitude (where some elements are not).
template <typename T, int N>
__device__ __forceinline__ uint32_t max_finite_bits(const uint4 (&w)[N]) {
  float m = 0.f;
  bool odd = false;
  for (int i = 0; i < N; ++i)
    for (int k = 0; k < (sizeof(T) == 2 ? 2 : 1); ++k) {
      float x[4];
      elements4(w[i], k, T{}, x);
      for (int e = 0; e < 4; ++e) m = fmaxf(m, finite_abs(x[e], &odd));
    }
  return __float_as_uint(m);
}
// Four finite elements as codes under a scale of the grid.  For int8 the integer is in the low bits of
// quotient + 1.5 * 2^23; for fp32 elements it is then checked against the remainder.
template <int TYPE, typename T>
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], float s, float rcp) {
  if constexpr (TYPE == SELKV_Q_E4M3) {
    return cvt_e4m3x2(x[0] * rcp, x[1] * rcp) | cvt_e4m3x2(x[2] * rcp, x[3] * rcp) << 16;
  } else {
    constexpr float kBig = 12582912.f;
    uint32_t t[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float q = x[e] * rcp;
      if constexpr (sizeof(T) == 2) {
        t[e] = __float_as_uint(fmaf(fmaf(-q, s, x[e]), rcp, q) + kBig);
      } else {
        const float c = q + kBig, r = fmaf(-(c - kBig), s, x[e]), h = 0.5f * s;
        const bool off = fabsf(r) > h || (fabsf(r) == h && (__float_as_uint(c) & 1u));
        t[e] = __float_as_uint(off ? c + copysignf(1.f, r) : c);
      }
    }
    return __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
  }
}

// LOOP: a CTA goes through every gridDim.x-th tile of its KV head's K or V, else it has one.
template <int TYPE, typename T, int D, bool LOOP>
__global__ __launch_bounds__(ACfg<T, D>::kThreads, ACfg<T, D>::kCtas) void qappend_kernel(QAppendArgs a) {
  using C = Code<TYPE>;
  constexpr int kWarpRows = ACfg<T, D>::kWarpRows, kThreads = ACfg<T, D>::kThreads;
  constexpr int kEl = 16 / sizeof(T);           // elements of a 16-byte load
  constexpr int kLpr = D / kEl;                 // lanes per row
  constexpr int kRpl = 32 / kLpr;               // rows per load
  constexpr int kLoads = kWarpRows / kRpl;
  __shared__ uint32_t wmax[kTileRows / kWarpRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int h = blockIdx.y, b = blockIdx.z >> 1, isv = blockIdx.z & 1;
  const size_t bk = (size_t)b * a.Hkv + h;
  __shared__ int s_len, s_n;
  chain_begin();
  if (tid == kThreads - 1) {  // (the CTA's only thread to read the length)
    s_len = a.c.lengths[b];
    s_n = a.counts != nullptr ? a.counts[b] : a.rows;
  }
  __syncthreads();
  int L = s_len, n = s_n;
  const bool first_cta = blockIdx.x == 0 && h == 0 && isv == 0;
  if (L < 0 || L > a.m_cap || n < 0 || n > a.rows) {
    if (tid == 0 && first_cta) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = min(max(L, 0), a.m_cap);
    n = min(max(n, 0), a.rows);
  }
  if (n > a.m_cap - L) {
    if (tid == 0 && first_cta) raise_flag(a.flags, SELKV_DEVERR_CAPACITY);
    n = 0;
  }
  const T* src = static_cast<const T*>(isv ? a.v_new : a.k_new) + bk * a.rows * D;
  uint8_t* codes = (isv ? a.c.V : a.c.K) + bk * a.m_cap * D;
  float* scales = (isv ? a.c.vs : a.c.ks) + bk * a.c.nblk;
  const int at = lane % kLpr * kEl;  // this lane's elements of its rows
  int tile0 = (L / kTileRows + (int)blockIdx.x) * kTileRows;
  for (bool first = true;; first = false, tile0 += gridDim.x * kTileRows) {
    const int row0 = tile0 + warp * kWarpRows;  // this warp's first row
    uint4 x[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + i * kRpl + lane / kLpr;
      x[i] = row >= L && row < L + n ? *reinterpret_cast<const uint4*>(src + (size_t)(row - L) * D + at) : make_uint4(0, 0, 0, 0);
    }
    // The last CTA of the sequence to have read its length moves it.  (Behind the loads: the thread waits for the
    // counter, and its warp with it.)
    if (first && tid == kThreads - 1) {
      const uint32_t all = gridDim.x * gridDim.y * 2u;
      if (atom_add_acq_rel_gpu(&a.cnt_seq[b], 1u) == all - 1u) {
        a.cnt_seq[b] = 0u;
        if (n > 0) a.c.lengths[b] = L + n;
      }
    }
    if (n == 0 || tile0 >= L + n) return;
    uint32_t m = __reduce_max_sync(0xffffffffu, max_bits<T>(x));
    const bool finite = __syncthreads_or(m >= 0x7f800000u) == 0;
    if (!finite) {
      if (lane == 0 && m >= 0x7f800000u) raise_flag(a.flags, SELKV_DEVERR_VALUE);
      m = __reduce_max_sync(0xffffffffu, max_finite_bits<T>(x));
    }
    if (lane == 0) wmax[warp] = m;
    const int blk = row0 >> a.c.block_log2, bfirst = blk << a.c.block_log2;
    const bool live = bfirst < L + n && bfirst + (1 << a.c.block_log2) > L;  // the block takes new rows
    const bool holds = live && L > bfirst;
    const float s0 = holds ? held_scale(scales[blk]) : 0.f;  // read by every warp before one writes it
    __syncthreads();
    if (!isv && a.c.bias != nullptr) {
      const int row = row0 + lane;
      if (lane < kWarpRows && row >= L && row < L + n)
        a.c.bias[bk * a.m_cap + row] = a.bias_new != nullptr ? a.bias_new[bk * a.rows + row - L] : 0.f;
    }
    if (!live) {
      if (LOOP) continue;
      return;
    }
    const int wpb = (1 << a.c.block_log2) / kWarpRows, w0 = warp / wpb * wpb;  // warps of the block
    m = 0u;
    for (int w = w0; w < w0 + wpb; ++w) m = max(m, wmax[w]);
    const float amax = __uint_as_float(m);
    const float s = holds ? grown_scale<TYPE>(s0, amax) : C::fresh_scale(amax);
    if (warp == w0 && lane == 0) scales[blk] = s;
    if (holds && s != s0) {  // this warp's rows among those the block holds, under the new scale
      const float f = s0 / s;
      uint32_t* w = reinterpret_cast<uint32_t*>(codes + (size_t)row0 * D);
      const int old = min(L - row0, kWarpRows);
      for (int i = lane; i < old * (D / 4); i += 32) {
        float y[4];
        C::unpack4(w[i], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] *= f;
        w[i] = C::pack4(y);
      }
    }
    const float rcp = 1.f / s;
    const bool quick = finite && !holds;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int row = row0 + i * kRpl + lane / kLpr;
      if (row < L || row >= L + n) continue;
      uint32_t w[kEl / 4];
#pragma unroll
      for (int j = 0; j < kEl / 4; ++j) {
        float y[4];
        elements4(x[i], j, T{}, y);
        if (quick) {
          w[j] = encode4<TYPE, T>(y, s, rcp);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = C::quotient(y[e], s, rcp, holds || sizeof(T) == 4);
          w[j] = C::pack4(y);
        }
      }
      uint8_t* dst = codes + (size_t)row * D + at;
      if constexpr (kEl == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(dst) = w[0];
    }
    if (!LOOP) return;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]);
template <>
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float (&x)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
template <>
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

constexpr int kReadThreads = 256;

template <int TYPE, typename T, int D>
__global__ __launch_bounds__(kReadThreads) void qread_kernel(QReadArgs a) {
  using C = Code<TYPE>;
  const int h = blockIdx.y, b = blockIdx.z >> 1, isv = blockIdx.z & 1;
  const size_t bk = (size_t)b * a.Hkv + h;
  chain_begin();
  int L = a.c.lengths[b];
  if (L < 0 || L > a.m_cap) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && h == 0 && isv == 0) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = min(max(L, 0), a.m_cap);
  }
  const int n = max(0, min(a.rows, L - a.row0));  // rows to read
  const uint8_t* codes = (isv ? a.c.V : a.c.K) + (bk * a.m_cap + a.row0) * D;
  const float* scales = (isv ? a.c.vs : a.c.ks) + bk * a.c.nblk;
  T* out = static_cast<T*>(isv ? a.v_out : a.k_out) + bk * a.rows * D;
  const size_t end = (size_t)n * (D / 16);  // 16 codes each
  for (size_t i = blockIdx.x * kReadThreads + threadIdx.x; i < end; i += gridDim.x * kReadThreads) {
    const uint4 w = *reinterpret_cast<const uint4*>(codes + i * 16);
    const float s = scales[(a.row0 + (int)(i / (D / 16))) >> a.c.block_log2];
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float y[8], t[4];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        C::unpack4(ws[j * 2 + p], t);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[p * 4 + e] = t[e] * s;
      }
      store8(out + i * 16 + j * 8, y);
    }
  }
}

// The last kernel of a read into bf16 rows: it ends when they are in place.  A decode over them that follows loads rows
// before it waits for the kernel in front of it, so that must not be the one that writes them.
__global__ void qread_end_kernel() { pdl_wait(); }

template <int TYPE, typename T>
cudaError_t qappend_t(const QAppendArgs& a, cudaStream_t st) {
  // The rows behind any length touch at most this many tiles.  Beyond 24 CTAs for each SM a CTA takes several
  // tiles, which saves starts, and those that find no rows in a ragged batch (131072 x 8 rows: 122.0 us, with a
  // tile a CTA 127.7; 64 x 1024-2048 x 8: 108.7 and 116.1); below, the code for one is faster (25000 x 8: 30.2 us, 31.5).
  const long tiles = (a.rows + kTileRows - 2) / kTileRows + 1, units = 2L * a.B * a.Hkv, most = 24 * kPlanSMs;
  const bool loop = tiles * units > most;
  const dim3 grid((unsigned)(loop ? std::min(tiles, (most + units - 1) / units) : tiles), a.Hkv, 2 * a.B);
  if (a.D == 128)
    return loop ? launch_chained(true, qappend_kernel<TYPE, T, 128, true>, grid, dim3(ACfg<T, 128>::kThreads), 0, st, a)
                : launch_chained(true, qappend_kernel<TYPE, T, 128, false>, grid, dim3(ACfg<T, 128>::kThreads), 0, st, a);
  return loop ? launch_chained(true, qappend_kernel<TYPE, T, 64, true>, grid, dim3(ACfg<T, 64>::kThreads), 0, st, a)
              : launch_chained(true, qappend_kernel<TYPE, T, 64, false>, grid, dim3(ACfg<T, 64>::kThreads), 0, st, a);
}

template <int TYPE, typename T>
cudaError_t qread_t(const QReadArgs& a, cudaStream_t st) {
  // A CTA goes through its share of the rows: at most 128 CTAs for each SM in all (8 ragged caches of 8192-16384 x 8
  // rows: 84.1 us, with 64: 86.5, with 32: 95.0, with a CTA for every 4 KB: 88.5).
  const int per = kReadThreads * 16 / a.D;  // rows of a step
  const long steps = (a.rows + per - 1) / per, units = 2L * a.B * a.Hkv;
  const dim3 grid((unsigned)std::min(steps, (128L * kPlanSMs + units - 1) / units), a.Hkv, 2 * a.B);
  const cudaError_t e = a.D == 128 ? launch_chained(true, qread_kernel<TYPE, T, 128>, grid, dim3(kReadThreads), 0, st, a)
                                   : launch_chained(true, qread_kernel<TYPE, T, 64>, grid, dim3(kReadThreads), 0, st, a);
  if (sizeof(T) == 4 || e != cudaSuccess) return e;
  return launch_chained(true, qread_end_kernel, dim3(1), dim3(32), 0, st);
}

}  // namespace

cudaError_t launch_qappend(const QAppendArgs& a, cudaStream_t st) {
  if (a.c.type == SELKV_Q_E4M3)
    return a.dtype == SELKV_BF16 ? qappend_t<SELKV_Q_E4M3, __nv_bfloat16>(a, st) : qappend_t<SELKV_Q_E4M3, float>(a, st);
  return a.dtype == SELKV_BF16 ? qappend_t<SELKV_Q_INT8, __nv_bfloat16>(a, st) : qappend_t<SELKV_Q_INT8, float>(a, st);
}

cudaError_t launch_qread(const QReadArgs& a, cudaStream_t st) {
  if (a.c.type == SELKV_Q_E4M3)
    return a.dtype == SELKV_BF16 ? qread_t<SELKV_Q_E4M3, __nv_bfloat16>(a, st) : qread_t<SELKV_Q_E4M3, float>(a, st);
  return a.dtype == SELKV_BF16 ? qread_t<SELKV_Q_INT8, __nv_bfloat16>(a, st) : qread_t<SELKV_Q_INT8, float>(a, st);
}

}  // namespace selkv
