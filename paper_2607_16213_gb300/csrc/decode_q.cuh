// Compensated decode attention over an 8-bit cache.
//
//   out[b][h] = sum_i softmax_i(q_h . k_i / sqrt(d) + bias_i) v_i,   k_i = kc_i ks, v_i = vc_i vs
//
// with codes kc, vc of 8 bits and scales ks, vs of a block of rows.  Split-K flash decoding: CTA (split,
// KV head, sequence) takes a contiguous slice of the rows, cut at multiples of 64.  Each of its warps is
// a stream of its own: it takes every kWarps-th tile of 32 rows, which its lane 0 brings into the warp's own
// shared memory with two 2D TMA loads (K and V; the next K as soon as this one is multiplied, the next V
// likewise), so no warp waits for another in the loop.  64 KB in flight on an SM is as much as helps:
// with 128 KB one token over 131072 x 8 rows takes 45.6 us instead of 44.7, with 192 KB 49.8, as whatever is
// asked for queues behind it.
//
// Per tile S^T = K Q^T and O^T += V^T P^T run on the tensor cores (mma.sync m16n8k16): the rows and the
// elements of the cache are the 16 of the product and the heads of a group its 8 (one step for up to
// eight heads, two for up to 16).  Each row of the cache is used by at most 16 heads, an eighth of the smallest
// tcgen05 tile, and its codes have to pass through registers to become fp16.
//
// Numbers.  A code is exact in fp16.  A query row is scaled by a power of two to a largest magnitude in [2^14, 2^15)
// and held in fp16: exactly for bf16; an fp32 query as the sum of two halves (22 bits).  The
// weights p = 2^(x - largest x so far) are summed in fp32, and go into O as
//   fp16(p * vs * 2^(largest x so far - ref)),
// ref a reference that only grows and keeps these below 2^15: the scales of V never meet O, and
// weights (times their scales) down to 2^-24 of the largest keep 11 bits.  fp32 caches hold them as two halves: 22 bits down
// to 2^-12 of the largest, and an error of at most 2^-35 of the largest below that.
//
// A key row costs 2 d + 4 bytes of HBM and 4 G d flops.  What bounds it: for bf16, d 128 and up to eight heads a group HBM
// from some tens of MB on (131072 x 8 rows, 269 MB: 45.2 us, 5.9 TB/s of 6.8 measured for a copy); below that the way in
// (length, queries and the first tiles: 3 us) and out (fold of warps and splits: 2 to 4 us).  The other forms are
// bound by the instructions of a tile (floor 39 to 40 us each; 8 caches of 16000 x 8 rows of d 128 or 32000 x 8 of d 64, fp32 d 128
// 4 of 32000 x 8): d 64, whose tile costs as d 128's but for half of the products, 48 to 51 us; nine to sixteen heads, whose
// registers leave room for eight to twelve warps on an SM, 54 to 77; fp32, with each product twice, 50 to 67, and 78 to 94
// with both.
#pragma once

#include "decode_common.cuh"
#include "quant.cuh"

namespace selkv {
namespace {

constexpr int kTileRows = 32;  // rows of a warp's tile: one bias a lane

template <int D, int NT, int NW>
struct QCfg {
  static constexpr int kWarps = NW, kThreads = NW * 32;
  static constexpr int kSlot = kTileRows * D;
  static constexpr int kFoldLd = D + 4;               // fold row stride (floats): conflict-free float2 stores
  static constexpr int kFold = NW * 8 * NT * kFoldLd * 4;
  static constexpr int kPart = 8 * NT * D * 4;         // a cluster's CTA: its folded output
  static constexpr int kTiles = NW * 2 * kSlot;  // the rings, and the fold in their place
  static constexpr int kRing = kTiles > kFold + kPart ? kTiles : kFold + kPart;
  static constexpr int kSmem = 1024 + kRing + kWarps * 2 * 8;
};

// Byte offset of 16-byte chunk c of row r in a tile written by TMA with 128-byte (D = 128) or
// 64-byte (D = 64) swizzling.
template <int D>
__device__ __forceinline__ uint32_t tile_at(int r, int c) {
  return D == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

// Four consecutive elements as they are stored, zeros where `in` is false.
template <typename T>
struct Row4;
template <>
struct Row4<__nv_bfloat16> {
  uint2 w;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, bool in) {
    w = in ? *reinterpret_cast<const uint2*>(p) : make_uint2(0u, 0u);
  }
  __device__ __forceinline__ void get(float (&x)[4]) const {
    x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
  }
};
template <>
struct Row4<float> {
  float4 w;
  __device__ __forceinline__ void load(const float* p, bool in) {
    w = in ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __device__ __forceinline__ void get(float (&x)[4]) const { x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w; }
};

// The four codes of a word as two pairs of halves: (0, 1), (2, 3), or with kSplit (0, 2), (1, 3).
template <int TYPE, bool kSplit>
__device__ __forceinline__ void to_halves(uint32_t w, uint32_t& a, uint32_t& b) {
  if constexpr (TYPE == SELKV_Q_E4M3) {
    if constexpr (kSplit) w = __byte_perm(w, 0u, 0x3120);
    a = e4m3x2_to_f16x2(w & 0xffffu);
    b = e4m3x2_to_f16x2(w >> 16);
  } else {
    // 0x64uu is the half 1024 + u, with u = code + 128
    const uint32_t u = w ^ 0x80808080u;
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1152
    const uint32_t x = __byte_perm(u, 0x64646464u, kSplit ? 0x4240 : 0x4140);
    const uint32_t y = __byte_perm(u, 0x64646464u, kSplit ? 0x4341 : 0x4342);
    const __half2 xs = __hsub2(*reinterpret_cast<const __half2*>(&x), off);
    const __half2 ys = __hsub2(*reinterpret_cast<const __half2*>(&y), off);
    a = *reinterpret_cast<const uint32_t*>(&xs);
    b = *reinterpret_cast<const uint32_t*>(&ys);
  }
}

// D(16x8, fp32) += A(16x16, fp16) B(16x8, fp16).
__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// Transpose of an 8x8 matrix of halves held by a warp, a pair of a row in each lane.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// What is left of the pair after pack_f16, as halves.
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t packed) {
  const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&packed));
  return pack_f16(lo - t.x, hi - t.y);
}

// Bias in base 2.  The lowest finite numbers stay finite: rows that all have them share the weight.  A NaN stays one.
__device__ __forceinline__ float bias_log2(float b) {
  float x;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(x) : "f"(b * kLog2e), "f"(-3.402823466e38f));
  return b == -INFINITY ? b : x;
}

// NT: steps of eight heads.  fp32: queries and weights as two halves each.
template <int TYPE, typename T, int D, int NT, int NW>
__global__ __launch_bounds__(NW * 32, ctas_of(NW, NT == 2, sizeof(T) == 4, D)) void decode_q_kernel(
    const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, QDecodeArgs a) {
  using C = QCfg<D, NT, NW>;
  constexpr int kWarps = C::kWarps, kThreads = C::kThreads;
  constexpr int NC = D / 16;                    // 16-byte chunks of a code row
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;    // halves of a query or weight
  constexpr int GU = 8 * NT;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kRing);  // [kWarps][K, V]
  __shared__ float wm[kWarps][GU], wl[kWarps][GU];
  __shared__ float apm[GU], s_M[GU];  // the appended row's logits; the largest logits
  __shared__ float s_inv[GU];
  __shared__ __align__(16) float s_vnew[D];  // the appended row's values
  __shared__ float2 s_ml[GU];  // (largest logit, sum) of the CTA's rows
  __shared__ int s_abort, s_len;
  __shared__ bool s_last;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int S = a.splits, s = blockIdx.x, kv = blockIdx.y, b = blockIdx.z;
  const int G = a.G;
  // split s: CTA `rank` of `Sc` in cluster `sg` of `Sg`
  const int Sc = a.cluster, Sg = S / Sc, rank = s % Sc, sg = s / Sc;
  const size_t bk = (size_t)b * a.Hkv + kv, bh0 = bk * G;
  uint64_t* bar = full + warp * 2;

  if (lane == 0) {
    for (int i = 0; i < 2; ++i) mbar_init(&bar[i], 1);
    fence_mbar_init();
    if (warp == 0) {
      s_abort = 0;
      prefetch_tensormap(&tmK);
      prefetch_tensormap(&tmV);
    }
  }
  pdl_wait();
  pdl_launch_dependents();

  // The length, this lane's part of the queries (elements 16 c + 4 j .. + 3 of head n * 8 + g) and, once the
  // slice is known, the first tile's scales are asked for before the tiles: behind those they would
  // wait for the whole ring (25000 rows x 8 heads: queries there after 5.1 us instead of 1.7).
  const int g = lane >> 2, j = lane & 3;
  if (tid == kThreads - 1) s_len = a.lengths[b];  // (the CTA's only thread to read it)
  Row4<T> qr[NT][NC];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < NC; ++c)
      qr[n][c].load(static_cast<const T*>(a.q) + (bh0 + n * 8 + g) * D + j * 4 + c * 16, n * 8 + g < G);
  if (a.k_new != nullptr && s == S - 1 && warp == kWarps - 1) {  // (most likely the split that takes the new row)
    constexpr int kLines = D * (int)sizeof(T) / 128;
    if (lane < 2 * kLines)
      prefetch_l2(static_cast<const char*>(lane < kLines ? a.k_new : a.v_new) + bk * D * sizeof(T) + lane % kLines * 128);
  }
  __syncthreads();
  int L = s_len;
  if (L < 0 || L > a.m_cap) {
    if (tid == 0 && s == 0 && kv == 0) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = L < 0 ? 0 : a.m_cap;
  }
  bool app = a.k_new != nullptr;
  if (app && L + 1 > a.m_cap) {
    if (tid == 0 && s == 0 && kv == 0) raise_flag(a.flags, SELKV_DEVERR_CAPACITY);
    app = false;
  }
  // whole blocks: the one that takes the new row is read by one split only
  const int cut = max(64, 1 << a.c.block_log2);
  const int chunk = ((L + S - 1) / S + cut - 1) / cut * cut;
  const int lo = min(L, s * chunk), hi = min(L, lo + chunk);
  const int ntiles = (hi - lo + kTileRows - 1) / kTileRows;
  const int nt = warp < ntiles ? (ntiles - warp + kWarps - 1) / kWarps : 0;  // this warp's
  // the warp's tiles: i is rows row0 + i * kStep .. + 31; K in slot 0 of its ring, V in slot 1
  constexpr int kStep = kWarps * kTileRows;
  const int row0 = lo + warp * kTileRows, y0 = (int)(bk * a.m_cap) + row0;
  unsigned char *ring_k = smem + warp * 2 * C::kSlot, *ring_v = ring_k + C::kSlot;
  auto issue_k = [&](int i) {  // (lane 0)
    mbar_arrive_expect_tx(&bar[0], C::kSlot);
    tma_load_2d(ring_k, &tmK, 0, y0 + i * kStep, &bar[0]);
  };
  auto issue_v = [&](int i) {
    mbar_arrive_expect_tx(&bar[1], C::kSlot);
    tma_load_2d(ring_v, &tmV, 0, y0 + i * kStep, &bar[1]);
  };
  float* ksp = a.c.ks + bk * a.c.nblk;
  float* vsp = a.c.vs + bk * a.c.nblk;
  // Bias (of row `lane`; -inf: no weight) and scales (of each half) of a tile, fetched one tile ahead.  A step
  // is a whole number of blocks, so that all of them are a fixed way from the tile before.
  struct Side {
    float bias, ks[2], vs[2];
  };
  const bool halves = a.c.block_log2 == 4;  // a tile's halves have scales of their own
  const int blk0 = row0 >> a.c.block_log2, blk_step = kStep >> a.c.block_log2;
  const float *bias_at = a.bias != nullptr ? a.bias + bk * a.m_cap + row0 + lane : nullptr;
  const float *ks_at = ksp + blk0, *vs_at = vsp + blk0;
  int left = hi - row0;  // rows of the slice from the tile on
  auto fetch = [&](Side& f) {
    f.bias = lane < left ? (bias_at != nullptr ? *bias_at : 0.f) : -INFINITY;
    f.ks[0] = f.ks[1] = *ks_at;
    f.vs[0] = f.vs[1] = *vs_at;
    if (halves && left > 16) {
      f.ks[1] = ks_at[1];
      f.vs[1] = vs_at[1];
    }
    if (bias_at != nullptr) bias_at += kStep;
    ks_at += blk_step;
    vs_at += blk_step;
    left -= kStep;
  };
  // the appended row joins the split that reads its block
  const bool joins = app && s == (L > 0 ? (L - 1) / chunk : 0);
  float kn[D / 32], vn = 0.f;
  if (joins) {
    load_row<T, D>(static_cast<const T*>(a.k_new) + bk * D, kn);
    if (tid < D) vn = load1(static_cast<const T*>(a.v_new) + bk * D + tid);
  }
  Side next{};
  if (nt > 0) fetch(next);
  if (lane == 0 && nt > 0) {
    issue_k(0);
    issue_v(0);
  }

  // The last CTA of the sequence to have read its length moves it (while the first tiles are on their way).
  if (app && tid == kThreads - 1 && atom_add_acq_rel_gpu(&a.cnt_seq[b], 1u) == (uint32_t)(S * a.Hkv) - 1u) {
    a.lengths[b] = L + 1;
    a.cnt_seq[b] = 0u;
  }

  // queries as halves, and the factor of the logits of the heads n * 8 + 2 j + e
  uint32_t qb[NT][NP][NC][2];
  float qsc[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float x[NC][4], m = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      qr[n][c].get(x[c]);
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(x[c][e]));
    }
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    int e2 = 0;
    if (m > 0.f && m < INFINITY) e2 = min(100, 14 + 127 - (int)(__float_as_uint(m) >> 23));
    const float up = __uint_as_float((uint32_t)(e2 + 127) << 23);
    const float down = a.scale_log2 * __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll
    for (int e = 0; e < 2; ++e) qsc[n][e] = __shfl_sync(0xffffffffu, down, (2 * j + e) * 4);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float x0 = x[c][2 * p] * up, x1 = x[c][2 * p + 1] * up;
        const uint32_t w = pack_f16(x0, x1);
        qb[n][0][c][p] = w;
        if constexpr (NP == 2) qb[n][NP - 1][c][p] = pack_rest(x0, x1, w);
      }
  }

  if (joins) {
    float q[D / 32];
    for (int h = warp; h < G; h += kWarps) {
      load_row<T, D>(static_cast<const T*>(a.q) + (bh0 + h) * D, q);
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) x = fmaf(q[e], kn[e], x);
      x = warp_sum(x) * a.scale_log2;
      if (lane == 0) apm[h] = x;
    }
    if (tid < D) s_vnew[tid] = vn;
  }

  // heads n * 8 + 2 j + (i & 1), elements 16 c + 2 g + (i >> 1)
  float o[NT][NC][4];
  float mrow[NT][2], lrow[NT][2], xref[NT][2], kref[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][c][i] = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      mrow[n][e] = xref[n][e] = -INFINITY;
      lrow[n][e] = kref[n][e] = 0.f;
    }
  }

  int got_k = 0, got_v = 0;  // tiles read
  for (int i = 0; i < nt; ++i) {
    const Side cur = next;
    if (i + 1 < nt) fetch(next);
    if (!__all_sync(0xffffffffu, mbar_wait(&bar[0], i & 1))) {
      if (lane == 0) {
        s_abort = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      break;
    }
    const uint32_t Kt = smem_u32(ring_k), Vt = smem_u32(ring_v);
    const float bl = bias_log2(cur.bias);
    const uint32_t dead = __ballot_sync(0xffffffffu, bl == -INFINITY);
    // S^T = K Q^T: the bytes 4 j .. 4 j + 3 of chunk c are the k indexes 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of step c
    // (The tensor cores cut sums off instead of rounding them.  With fp32 caches the products with the second halves
    // of the queries therefore have sums of their own here, and a tile's share of O is added to it below: errors of
    // 2e-7 to 6e-7 of the output instead of 2e-7 to 1.3e-6.  Many equal rows near 2^-24 of the largest weight would all be
    // rounded the same way: 100000 of them to some 3e-6 of the output.)
    float x[NT][2][4], x2[NT][2][4] = {};  // heads n * 8 + 2 j + (i & 1), rows 16 h + 8 (i >> 1) + g
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) x[n][h][k] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint32_t kw[4];
      ldmatrix_x4(kw, Kt + tile_at<D>(lane, c));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t ka[4];
        to_halves<TYPE, false>(kw[2 * h], ka[0], ka[2]);
        to_halves<TYPE, false>(kw[2 * h + 1], ka[1], ka[3]);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int p = 0; p < NP; ++p) mma_f16_16816(p == 0 ? x[n][h] : x2[n][h], ka, qb[n][p][c]);
      }
    }
    got_k = i + 1;
    __syncwarp();
    if (lane == 0 && i + 1 < nt) issue_k(i + 1);
    // logits in base 2
    float tm[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) tm[n][0] = tm[n][1] = -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const float bv = __shfl_sync(0xffffffffu, bl, h * 16 + q * 8 + g);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float& v = x[n][h][q * 2 + e];
            if constexpr (NP == 2) v += x2[n][h][q * 2 + e];
            v = fmaf(v, qsc[n][e] * cur.ks[h], bv);
            if (dead && bv == -INFINITY) v = bv;  // (the codes may be NaN)
            tm[n][e] = fmaxf(tm[n][e], v);
          }
      }
    // v scale = mantissa * 2^ve
    float ve[2], vm[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      ve[h] = (float)((int)(__float_as_uint(cur.vs[h]) >> 23) - 127);
      vm[h] = __uint_as_float((__float_as_uint(cur.vs[h]) & 0x7fffffu) | 0x3f800000u);
    }
    // The largest logit, and (tr, vr) that of the half of the tile whose largest weight times scale sets the units.
    float tr[NT][2], vr[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float& t = tm[n][e];
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
        tr[n][e] = t;
        vr[n][e] = ve[0];
      }
    if (ve[0] != ve[1]) {  // (all lanes alike)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float th[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            th[h] = fmaxf(x[n][h][e], x[n][h][2 + e]);
#pragma unroll
            for (int m = 4; m < 32; m *= 2) th[h] = fmaxf(th[h], __shfl_xor_sync(0xffffffffu, th[h], m));
          }
          const bool first = (th[0] - th[1]) + (ve[0] - ve[1]) > 0.f;  // (no: neither half has a weight)
          tr[n][e] = first ? th[0] : th[1];
          vr[n][e] = first ? ve[0] : ve[1];
        }
    }
    float corr[NT][2];
    bool grew = false;
    float most = -INFINITY;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float t = tm[n][e];
        const float mn = fmaxf(mrow[n][e], t), mnr = mn == -INFINITY ? 0.f : mn;
        float sum = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float& v = x[n][h][q * 2 + e];
            v = ex2_approx(v - mnr);
            sum += v;
          }
        lrow[n][e] = lrow[n][e] * ex2_approx(mrow[n][e] - mnr) + sum;
        mrow[n][e] = mn;
        // O is in units of 2^(xref + kref - 10); the units grow only when a weight would pass 2^15.
        // (The logits are subtracted first: next to the lowest numbers ve would vanish.)
        corr[n][e] = 1.f;
        if ((tr[n][e] - xref[n][e]) + vr[n][e] > kref[n][e] + 4.f) {  // (never with tr = -inf)
          corr[n][e] = ex2_approx((xref[n][e] - tr[n][e]) + (kref[n][e] - vr[n][e]));
          xref[n][e] = tr[n][e];
          kref[n][e] = vr[n][e];
          grew = true;
        }
        const float d = mnr - xref[n][e] - kref[n][e] + 10.f;
        most = fmaxf(most, d);  // (+inf while no row has had a weight: the weights are 0)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float up = d + ve[h], f = vm[h] * ex2_approx(fminf(up, 120.f));
#pragma unroll
          for (int q = 0; q < 2; ++q) x[n][h][q * 2 + e] *= f;
        }
      }
    // Weights are 2^-126 and more and their products with f below 2^15, so the exponent of f is below 142 where there are
    // any: what is beyond its range is a second factor.
    if (most + fmaxf(ve[0], ve[1]) > 120.f) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float up = (mrow[n][e] == -INFINITY ? 0.f : mrow[n][e]) - xref[n][e] - kref[n][e] + 10.f + ve[h];
            const float f2 = ex2_approx(fminf(fmaxf(up - 120.f, 0.f), 22.f));
#pragma unroll
            for (int q = 0; q < 2; ++q) x[n][h][q * 2 + e] *= f2;
          }
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int k = 0; k < 4; ++k) o[n][c][k] *= corr[n][k & 1];
    }
    // weights with the rows along k
    uint32_t pb[NT][NP][2][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float p0 = x[n][h][q * 2], p1 = x[n][h][q * 2 + 1];
          const uint32_t w = pack_f16(p0, p1);
          pb[n][0][h][q] = transpose8(w);
          if constexpr (NP == 2) pb[n][NP - 1][h][q] = transpose8(pack_rest(p0, p1, w));
        }
    if (!__all_sync(0xffffffffu, mbar_wait(&bar[1], i & 1))) {
      if (lane == 0) {
        s_abort = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      break;
    }
    if (dead) {
      // rows without weight may hold anything: their values are zeroed
      for (uint32_t rest = dead; rest != 0; rest &= rest - 1) {
        const int r = __ffs(rest) - 1;
        if (lane < NC)
          *reinterpret_cast<uint4*>(ring_v + tile_at<D>(r, lane)) = make_uint4(0, 0, 0, 0);
      }
      __syncwarp();
    }
    // O^T += V^T P^T: a transposed load gives, of 16 rows and a chunk, two rows' bytes 2 g and 2 g + 1,
    // which are rows g and g + 8 of the product
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NC; c += 2) {
        uint32_t vw[4];
        ldmatrix_x4_trans(vw, Vt + tile_at<D>(h * 16 + (lane & 15), c + (lane >> 4)));
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t va[4];
          to_halves<TYPE, true>(vw[q * 2], va[0], va[1]);
          to_halves<TYPE, true>(vw[q * 2 + 1], va[2], va[3]);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            if constexpr (NP == 1) {
              mma_f16_16816(o[n][c + q], va, pb[n][0][h]);
            } else {
              float t[4] = {};
              mma_f16_16816(t, va, pb[n][0][h]);
              mma_f16_16816(t, va, pb[n][NP - 1][h]);
#pragma unroll
              for (int k = 0; k < 4; ++k) o[n][c + q][k] += t[k];
            }
          }
        }
      }
    if (dead) fence_proxy_async_smem();
    __syncwarp();
    got_v = i + 1;
    if (lane == 0 && i + 1 < nt) issue_v(i + 1);
  }
  // every copy has landed before the ring is used again or the CTA leaves (tile i's K is asked for when that
  // of i - 1 has been read)
  if (got_k < nt) mbar_wait(&bar[0], got_k & 1);
  if (got_v < nt) mbar_wait(&bar[1], got_v & 1);

  // Fold of the warps, the lanes' sums of a head first.
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float& l = lrow[n][e];
      l += __shfl_xor_sync(0xffffffffu, l, 4);
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
      if (g == 0) wm[warp][n * 8 + 2 * j + e] = mrow[n][e];
    }
  __syncthreads();
  const bool aborted = s_abort != 0;
  float* wo = reinterpret_cast<float*>(smem);  // [kWarps][GU][kFoldLd] outputs, in units of 2^(largest logit of all)
  float* part = wo + C::kFold / 4;             // [G][D]: a cluster's CTA's output
  // the KV head's record in the workspace: outputs [G][Sg][D], (largest logit, sum) pairs [Sc][G][Sg]
  float* po = a.partial + bk * decode_q_record_floats(G, Sc, Sg, D);
  float2* pml = reinterpret_cast<float2*>(po + (size_t)G * Sg * D) + rank * G * Sg;
  // Float4 d4 of head hd, folded over a cluster or a CTA of its own: the output, or this cluster's partial.
  auto emit = [&](int hd, int d4, float2 ml, float4 v) {
    if (Sg == 1) {
      const float iv = ml.y > 0.f || ml.y != ml.y ? 1.f / ml.y : 0.f;
      const float r[4] = {v.x * iv, v.y * iv, v.z * iv, v.w * iv};
      store4(static_cast<T*>(a.out) + (bh0 + hd) * D + d4 * 4, r);
    } else {
      reinterpret_cast<float4*>(po + ((size_t)hd * Sg + sg) * D)[d4] = v;
      if (d4 == rank) pml[hd * Sg + sg] = ml;  // (its first one)
    }
  };
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int hd = n * 8 + 2 * j + e;
      if (hd >= G) continue;
      float M = joins ? apm[hd] : -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w][hd]);
      const bool none = mrow[n][e] == -INFINITY;  // this warp has no row with a weight
      const float down = (xref[n][e] - M) + (kref[n][e] - 10.f);
      const float f = none ? 0.f : ex2_approx(fmaxf(down, -100.f));
      if (down < -100.f) {  // two factors where one may be below 2^-126: a weight is as small as that, and a row's scale too
        const float f2 = ex2_approx(down + 100.f);
#pragma unroll
        for (int c = 0; c < NC; ++c) o[n][c][e] *= f2, o[n][c][2 + e] *= f2;
      }
#pragma unroll
      for (int c = 0; c < NC; ++c)
        *reinterpret_cast<float2*>(wo + (warp * GU + hd) * C::kFoldLd + c * 16 + 2 * g) =
            make_float2(o[n][c][e] * f, o[n][c][2 + e] * f);
      if (g == 0) {
        wl[warp][hd] = none ? lrow[n][e] : lrow[n][e] * ex2_approx(mrow[n][e] - M);
        if (warp == 0) s_M[hd] = M;
      }
    }
  __syncthreads();
  constexpr int D4 = D / 4;
  for (int i = tid; i < G * D4; i += kThreads) {
    const int hd = i / D4, d4 = i % D4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(wo + (w * GU + hd) * C::kFoldLd + d4 * 4);
      acc.x += v.x;
      acc.y += v.y;
      acc.z += v.z;
      acc.w += v.w;
      l += wl[w][hd];
    }
    if (joins) {
      const float4 v = *reinterpret_cast<const float4*>(s_vnew + d4 * 4);
      const float wa = ex2_approx(apm[hd] - s_M[hd]);
      l += wa;
      acc.x = fmaf(wa, v.x, acc.x);
      acc.y = fmaf(wa, v.y, acc.y);
      acc.z = fmaf(wa, v.z, acc.z);
      acc.w = fmaf(wa, v.w, acc.w);
    }
    if (aborted) {
      acc = make_float4(0.f, 0.f, 0.f, 0.f);
      l = 0.f;
    }
    const float2 ml = make_float2(aborted ? -INFINITY : s_M[hd], l);
    if (Sc == 1) {
      emit(hd, d4, ml, acc);
    } else {
      reinterpret_cast<float4*>(part)[i] = acc;
      if (d4 == 0) s_ml[hd] = ml;
    }
  }
  // The split that has read the new row's block puts it into the cache, behind its own reads, and after
  // anything that another CTA waits for.
  auto append = [&]() {
    if (!joins) return;
    if (warp == kWarps - 2)
      append_row<TYPE, T, D>(static_cast<const T*>(a.k_new) + bk * D, a.c.K + bk * a.m_cap * D, ksp, a.c.block_log2, L,
                             a.flags);
    if (warp == kWarps - 1)
      append_row<TYPE, T, D>(static_cast<const T*>(a.v_new) + bk * D, a.c.V + bk * a.m_cap * D, vsp, a.c.block_log2, L,
                             a.flags);
    if (tid == 0 && a.bias != nullptr) a.bias[bk * a.m_cap + L] = 0.f;
  };
  if (Sc > 1) {
    // The CTAs of a cluster share out the float4s of the output: rank r takes those with d4 = r modulo Sc, Sc
    // lanes for each, lane t with CTA t's part.
    cluster_arrive();
    cluster_wait();
    const int t = lane & (Sc - 1);
    const uint32_t ml0 = peer_smem(smem_u32(s_ml), t), part0 = peer_smem(smem_u32(part), t);
    for (int base = rank; base < G * D4; base += kThreads) {
      const int i = base + tid / Sc * Sc, ic = min(i, G * D4 - 1), hd = ic / D4;
      const float2 ml = ld_peer_f2(ml0 + hd * 8);
      float4 v = ld_peer_f4(part0 + ic * 16);
      float M = ml.x;
      for (int d = 1; d < Sc; d <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
      const float w = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - M);
      float l = ml.y * w;
      v.x *= w, v.y *= w, v.z *= w, v.w *= w;
      for (int d = 1; d < Sc; d <<= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, d);
        v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
        v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
        v.z += __shfl_xor_sync(0xffffffffu, v.z, d);
        v.w += __shfl_xor_sync(0xffffffffu, v.w, d);
      }
      if (t == 0 && i < G * D4) emit(hd, ic % D4, make_float2(M, l), v);
    }
    cluster_arrive();  // no CTA leaves (cluster_wait) while another may still read its shared memory
  }
  bool last = false;
  if (Sg > 1) {
    __syncthreads();
    if (tid == 0) s_last = atom_add_acq_rel_gpu(&a.cnt_head[bk * Sc + rank], 1u) == (uint32_t)Sg - 1u;
    __syncthreads();
    last = s_last;
  }
  if (!last) {
    append();
    if (Sc > 1) cluster_wait();
    return;
  }
  if (tid == 0) a.cnt_head[bk * Sc + rank] = 0u;
  // The last CTA of its rank folds the clusters, in their order: two lanes a float4 of the output, each
  // with half of the clusters.  The outputs are on their way while the weights are computed.
  float* wts = wo;  // [G][Sg] weights of the clusters
  constexpr int kBatch = 16, kItems = kThreads / 2;
  const int half = lane >> 4, Sh = (Sg + 1) / 2, t0 = half * Sh, t1 = min(Sg, t0 + Sh);
  for (int base = 0; base < G * D4 / Sc; base += kItems) {
    const int k0 = base + warp * 16 + (lane & 15), i = rank + k0 * Sc, hd = i / D4, d4 = i % D4;
    const bool in = k0 < G * D4 / Sc;
    const float4* op = reinterpret_cast<const float4*>(po + (size_t)hd * Sg * D) + d4;
    float4 v[kBatch];
    auto load = [&](int t) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k)
        v[k] = in && t + k < t1 ? __ldcg(op + (size_t)(t + k) * D4) : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    load(t0);
    if (base == 0) {
      constexpr int kMl = (kMaxSplits + 31) / 32;
      for (int h = warp; h < G; h += kWarps) {
        float2 ml[kMl];
        float M = -INFINITY, Ls = 0.f;
#pragma unroll
        for (int k = 0; k < kMl; ++k) {
          const int t = lane + 32 * k;
          ml[k] = t < Sg ? __ldcg(pml + h * Sg + t) : make_float2(-INFINITY, 0.f);
        }
#pragma unroll
        for (int k = 0; k < kMl; ++k) M = fmaxf(M, ml[k].x);
        M = warp_max(M);
#pragma unroll
        for (int k = 0; k < kMl; ++k) {
          const int t = lane + 32 * k;
          if (t >= Sg) break;
          const float w = M == -INFINITY ? 0.f : ex2_approx(ml[k].x - M);
          wts[h * Sg + t] = w;
          Ls = fmaf(ml[k].y, w, Ls);
        }
        Ls = warp_sum(Ls);
        if (lane == 0) s_inv[h] = Ls > 0.f || Ls != Ls ? 1.f / Ls : 0.f;
      }
      __syncthreads();
    }
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int t = t0;;) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float w = in && t + k < t1 ? wts[hd * Sg + t + k] : 0.f;
        acc.x = fmaf(v[k].x, w, acc.x);
        acc.y = fmaf(v[k].y, w, acc.y);
        acc.z = fmaf(v[k].z, w, acc.z);
        acc.w = fmaf(v[k].w, w, acc.w);
      }
      t += kBatch;
      if (t >= t1) break;
      load(t);
    }
    acc.x += __shfl_xor_sync(0xffffffffu, acc.x, 16);
    acc.y += __shfl_xor_sync(0xffffffffu, acc.y, 16);
    acc.z += __shfl_xor_sync(0xffffffffu, acc.z, 16);
    acc.w += __shfl_xor_sync(0xffffffffu, acc.w, 16);
    if (in && half == 0) {
      const float iv = s_inv[hd];
      const float r[4] = {acc.x * iv, acc.y * iv, acc.z * iv, acc.w * iv};
      store4(static_cast<T*>(a.out) + (bh0 + hd) * D + d4 * 4, r);
    }
  }
  append();
  if (Sc > 1) cluster_wait();
}

template <int TYPE, typename T, int D, int NT, int NW>
cudaError_t launch_warps(const QDecodeArgs& a, cudaStream_t st) {
  using C = QCfg<D, NT, NW>;
  CUtensorMap tk, tv;
  const uint64_t rows = (uint64_t)a.B * a.Hkv * a.m_cap;
  if (!encode_rows_u8(&tk, a.c.K, rows, D, kTileRows) || !encode_rows_u8(&tv, a.c.V, rows, D, kTileRows))
    return cudaErrorInvalidValue;
  constexpr auto kern = decode_q_kernel<TYPE, T, D, NT, NW>;
  if (const cudaError_t e = set_smem_once<kern>(C::kSmem); e != cudaSuccess) return e;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.splits, a.Hkv, a.B);
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = st;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, tk, tv, a);
}

template <int TYPE, typename T, int D>
cudaError_t launch_heads(const QDecodeArgs& a, cudaStream_t st) {
  if (a.G <= 8) return a.warps == 8 ? launch_warps<TYPE, T, D, 1, 8>(a, st) : launch_warps<TYPE, T, D, 1, 4>(a, st);
  return a.warps == 8 ? launch_warps<TYPE, T, D, 2, 8>(a, st) : launch_warps<TYPE, T, D, 2, 4>(a, st);
}

template <int TYPE>
cudaError_t launch_type(const QDecodeArgs& a, cudaStream_t st) {
  if (a.dtype == SELKV_FP32) return a.D == 128 ? launch_heads<TYPE, float, 128>(a, st) : launch_heads<TYPE, float, 64>(a, st);
  return a.D == 128 ? launch_heads<TYPE, __nv_bfloat16, 128>(a, st) : launch_heads<TYPE, __nv_bfloat16, 64>(a, st);
}

}  // namespace
}  // namespace selkv
