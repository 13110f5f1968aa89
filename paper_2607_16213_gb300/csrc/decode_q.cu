// Compensated decode attention over an 8-bit cache.
//
//   out[b][h] = sum_i softmax_i(q_h . k_i / sqrt(d) + bias_i) v_i,   k_i = kc_i ks, v_i = vc_i vs
//
// with codes kc, vc of 8 bits and scales ks, vs of a block of rows.  Split-K flash decoding: CTA (split,
// KV head, sequence) takes a contiguous slice of the rows, cut at multiples of 64.  Each of its warps is
// a stream of its own: it takes every kWarps-th tile of 32 rows, which its lane 0 brings into the warp's own
// ring of shared memory with two 2D TMA loads (K and V), so no warp waits for another in the loop.
// Per tile S = Q K^T and O += P V run on the tensor cores with all query heads of the group as
// the M rows (mma.sync m16n8k16: a decode has at most 16 rows, an eighth of the smallest tcgen05 tile, and
// the codes have to pass through registers to become fp16).
//
// Numbers.  A code is exact in fp16.  A query row is scaled by a power of two to a largest magnitude in [2^14, 2^15) and
// held in fp16: exactly for bf16; an fp32 query is held as two halves in two of the 16 rows (22 bits).
// A tile's weights p = 2^(x - largest x of the tile) are summed in fp32, and go into O as
//   fp16(p * vs * 2^(largest x - ref)),
// ref a reference that only grows and keeps these below 2^15: the scales of V never meet O, and
// weights down to 2^-24 of the largest keep 11 bits (fp32 caches: 22, as two halves).
//
// A key row costs 2 d + 4 bytes of HBM and 4 G d flops.
#include <algorithm>

#include "decode_common.cuh"
#include "quant.cuh"

namespace selkv {
namespace {

constexpr int kTileRows = 32;  // rows of a warp's tile: one bias a lane
constexpr int kWarps = 8;
constexpr int kStages = 3;     // tiles in flight per warp
constexpr int kThreads = kWarps * 32;

// How the 16 rows of the matrix product are used: 8 heads; 16 heads; 8 heads of fp32 as two halves each.
enum Rows { kRows8, kRows16, kHalves };

template <int D>
struct QCfg {
  static constexpr int kSide = kTileRows * D;        // K or V of a tile
  static constexpr int kStage = 2 * kSide;
  static constexpr int kRing = kWarps * kStages * kStage;
  static constexpr int kFoldLd = D + 4;              // fold row stride (floats)
  static constexpr int kSmem = 1024 + kRing + kWarps * kStages * 8;
  static_assert(kWarps * 16 * kFoldLd * 4 <= kRing, "fold scratch fits");
};

// Byte offset of 16-byte chunk c of row r in a tile written by TMA with 128-byte (D = 128) or
// 64-byte (D = 64) swizzling.
template <int D>
__device__ __forceinline__ uint32_t tile_at(int r, int c) {
  return D == 128 ? (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)) : (uint32_t)(r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
}

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

// D(16x8, fp32) += A(16x16, fp16) B(16x8, fp16).  With eight rows in use the other half of A is zero
// and of D is not kept.
template <int N>
__device__ __forceinline__ void mma_rows(float (&d)[N], const uint32_t (&a)[N], uint32_t b0, uint32_t b1) {
  if constexpr (N == 4) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  } else {
    float t0, t1;
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %6, %5, %6}, {%7, %8}, "
        "{%0, %1, %9, %9};"
        : "+f"(d[0]), "+f"(d[1]), "=f"(t0), "=f"(t1)
        : "r"(a[0]), "r"(a[1]), "r"(0), "r"(b0), "r"(b1), "f"(0.f));
  }
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

// Bias in base 2.  The lowest finite numbers stay finite: rows that all have them share the weight.
__device__ __forceinline__ float bias_log2(float b) {
  return b == -INFINITY ? b : fmaxf(b * kLog2e, -3.402823466e38f);
}

template <int TYPE, typename T, int D, int ROWS>
__global__ __launch_bounds__(kThreads, 1) void decode_q_kernel(const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV, QDecodeArgs a) {
  using C = QCfg<D>;
  constexpr int NC = D / 16;                    // 16-byte chunks of a code row
  constexpr int NR = ROWS == kRows16 ? 2 : 1;   // heads of a lane
  constexpr int NA = ROWS == kRows8 ? 2 : 4;    // registers of an A fragment and of an accumulator
  constexpr int GU = ROWS == kRows16 ? 16 : 8;  // most heads of a unit
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kRing);  // [kWarps][kStages]
  __shared__ float wm[kWarps][GU], wl[kWarps][GU];
  __shared__ float apm[GU], apw[GU];  // the appended row's logit and weight
  __shared__ float s_inv[GU];
  __shared__ int s_abort;
  __shared__ bool s_last, s_kv_last;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int S = a.splits, s = blockIdx.x, b = blockIdx.z;
  // unit: the heads of a group that go together (all of them but for fp32 groups of more than eight)
  const int units = gridDim.y, HG = units / a.Hkv;
  const int kv = blockIdx.y / HG, hg = blockIdx.y % HG;
  const int h0 = kv * a.G + hg * GU, G = min(GU, a.G - hg * GU);
  const size_t bk = (size_t)b * a.Hkv + kv, bu = (size_t)b * units + blockIdx.y;
  uint64_t* bar = full + warp * kStages;
  unsigned char* ring = smem + warp * kStages * C::kStage;

  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(&bar[i], 1);
    fence_mbar_init();
    if (warp == 0) {
      s_abort = 0;
      prefetch_tensormap(&tmK);
      prefetch_tensormap(&tmV);
    }
  }
  __syncthreads();
  pdl_wait();
  pdl_launch_dependents();

  int L = a.lengths[b];
  if (L < 0 || L > a.m_cap) {
    if (tid == 0 && s == 0 && blockIdx.y == 0) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = L < 0 ? 0 : a.m_cap;
  }
  bool app = a.k_new != nullptr;
  if (app && L + 1 > a.m_cap) {
    if (tid == 0 && s == 0 && blockIdx.y == 0) raise_flag(a.flags, SELKV_DEVERR_CAPACITY);
    app = false;
  }
  const int chunk = ((L + S - 1) / S + 63) / 64 * 64;
  const int lo = min(L, s * chunk), hi = min(L, lo + chunk);
  const int ntiles = (hi - lo + kTileRows - 1) / kTileRows;
  const int nt = warp < ntiles ? (ntiles - warp + kWarps - 1) / kWarps : 0;  // this warp's
  auto issue = [&](int i) {  // (lane 0)
    const int st = i % kStages, y = (int)(bk * a.m_cap) + lo + (warp + i * kWarps) * kTileRows;
    unsigned char* base = ring + st * C::kStage;
    mbar_arrive_expect_tx(&bar[st], C::kStage);
    tma_load_2d(base, &tmK, 0, y, &bar[st]);
    tma_load_2d(base + C::kSide, &tmV, 0, y, &bar[st]);
  };
  if (lane == 0)
    for (int i = 0; i < min(nt, kStages); ++i) issue(i);

  const int g0 = lane >> 2, j = lane & 3;
  // this lane's part of the queries: elements 16 c + 4 j .. + 3 of row g0 (and g0 + 8)
  uint32_t qa[NC][NA];
  float qsc[NR];
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int g = g0 + r * 8;
    const T* qp = static_cast<const T*>(a.q) + ((size_t)b * a.Hq + h0 + g) * D + j * 4;
    float x[NC][4], m = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      if (g < G) {
        load4(qp + c * 16, x[c]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[c][e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(x[c][e]));
    }
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
    int e2 = 0;
    if (m > 0.f && m < INFINITY) e2 = min(100, 14 + 127 - (int)(__float_as_uint(m) >> 23));
    const float up = __uint_as_float((uint32_t)(e2 + 127) << 23);
    qsc[r] = a.scale_log2 * __uint_as_float((uint32_t)(127 - e2) << 23);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const uint32_t p0 = pack_f16(x[c][0] * up, x[c][1] * up), p1 = pack_f16(x[c][2] * up, x[c][3] * up);
      if constexpr (ROWS == kRows8) {
        qa[c][0] = p0;
        qa[c][1] = p1;
      } else {
        qa[c][r] = p0;
        qa[c][2 + r] = p1;
        if constexpr (ROWS == kHalves) {
          qa[c][1] = pack_rest(x[c][0] * up, x[c][1] * up, p0);
          qa[c][3] = pack_rest(x[c][2] * up, x[c][3] * up, p1);
        }
      }
    }
  }

  const float* brow = a.bias != nullptr ? a.bias + bk * a.m_cap : nullptr;
  const float* ksp = a.c.ks + bk * a.c.nblk;
  const float* vsp = a.c.vs + bk * a.c.nblk;
  // bias (of row `lane`; -inf: no weight) and scales (of each half) of a tile, fetched one tile ahead
  struct Side {
    float bias, ks[2], vs[2];
  };
  auto fetch = [&](int i) {
    Side f;
    const int row = lo + (warp + i * kWarps) * kTileRows;
    f.bias = row + lane < hi ? (brow != nullptr ? brow[row + lane] : 0.f) : -INFINITY;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int blk = min(row + h * 16, hi - 1) >> a.c.block_log2;
      f.ks[h] = ksp[blk];
      f.vs[h] = vsp[blk];
    }
    return f;
  };

  float o[NC][2][NA];  // [chunk][even or odd element]
  float mrow[NR], lrow[NR], xref[NR], kref[NR];
#pragma unroll
  for (int c = 0; c < NC; ++c)
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int e = 0; e < NA; ++e) o[c][p][e] = 0.f;
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    mrow[r] = xref[r] = -INFINITY;
    lrow[r] = kref[r] = 0.f;
  }

  Side next{};
  if (nt > 0) next = fetch(0);
  int done = 0;
  for (int i = 0; i < nt; ++i) {
    const Side cur = next;
    if (i + 1 < nt) next = fetch(i + 1);
    const int st = i % kStages;
    const bool ok = mbar_wait(&bar[st], (i / kStages) & 1);
    if (!__all_sync(0xffffffffu, ok)) {
      if (lane == 0) {
        s_abort = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      break;
    }
    const uint32_t Kt = smem_u32(ring + st * C::kStage), Vt = Kt + C::kSide;
    const float bl = bias_log2(cur.bias);
    const uint32_t dead = __ballot_sync(0xffffffffu, bl == -INFINITY);
    if (dead) {
      // rows without weight may hold anything: their values are zeroed before P V
      for (uint32_t rest = dead; rest != 0; rest &= rest - 1) {
        const int r = __ffs(rest) - 1;
        if (lane < NC)
          *reinterpret_cast<uint4*>(ring + st * C::kStage + C::kSide + tile_at<D>(r, lane)) = make_uint4(0, 0, 0, 0);
      }
      __syncwarp();
    }
    // S = Q K^T: the bytes 4 j .. 4 j + 3 of chunk c are the k indexes 2 j, 2 j + 1, 2 j + 8, 2 j + 9 of step c
    float sacc[4][NA];
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < NA; ++e) sacc[n][e] = 0.f;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      uint32_t kw[4];
      ldmatrix_x4(kw, Kt + tile_at<D>(lane, c));
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        uint32_t b0, b1;
        to_halves<TYPE, false>(kw[n], b0, b1);
        mma_rows<NA>(sacc[n], qa[c], b0, b1);
      }
    }
    // logits in base 2; key n * 8 + 2 j + e
    float x[NR][4][2], tm[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) tm[r] = -INFINITY;
#pragma unroll
    for (int n = 0; n < 4; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float bv = __shfl_sync(0xffffffffu, bl, n * 8 + j * 2 + e);
#pragma unroll
        for (int r = 0; r < NR; ++r) {
          const float dot = ROWS == kHalves ? sacc[n][e] + sacc[n][NA - 2 + e] : sacc[n][r * 2 + e];
          const float v = bv == -INFINITY ? bv : fmaf(dot, qsc[r] * cur.ks[n >> 1], bv);
          x[r][n][e] = v;
          tm[r] = fmaxf(tm[r], v);
        }
      }
    uint32_t pa[2][NA];  // weights of the keys 16 h .. 16 h + 15
    float corr[NR];
    bool grew = false;
#pragma unroll
    for (int r = 0; r < NR; ++r) {
      tm[r] = fmaxf(tm[r], __shfl_xor_sync(0xffffffffu, tm[r], 1));
      tm[r] = fmaxf(tm[r], __shfl_xor_sync(0xffffffffu, tm[r], 2));
      const float tref = tm[r] == -INFINITY ? 0.f : tm[r];
      const float mn = fmaxf(mrow[r], tm[r]), mnr = mn == -INFINITY ? 0.f : mn;
      float sum = 0.f;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          x[r][n][e] = ex2_approx(x[r][n][e] - tref);
          sum += x[r][n][e];
        }
      lrow[r] = lrow[r] * ex2_approx(mrow[r] - mnr) + sum * ex2_approx(tm[r] - mnr);
      mrow[r] = mn;
      // v scale = mantissa * 2^e.  O is in units of 2^(xref + kref - 10); the units grow only when a weight
      // would pass 2^15.  (tm - xref is taken first: at logits near the lowest number e would vanish.)
      float ve[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) ve[h] = (float)((int)(__float_as_uint(cur.vs[h]) >> 23) - 127);
      const float vmax = fmaxf(ve[0], ve[1]);
      float d = tm[r] == -INFINITY ? tm[r] : tm[r] - xref[r];
      corr[r] = 1.f;
      if (d + vmax > kref[r] + 4.f) {
        corr[r] = ex2_approx((xref[r] - tm[r]) + (kref[r] - vmax));
        xref[r] = tm[r];
        kref[r] = vmax;
        d = 0.f;
        grew = true;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float f = __uint_as_float((__float_as_uint(cur.vs[h]) & 0x7fffffu) | 0x3f800000u) *
                        ex2_approx(d + (ve[h] - kref[r] + 10.f));
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) {
          const int n = h * 2 + q2;
          const float p0 = x[r][n][0] * f, p1 = x[r][n][1] * f;
          const uint32_t w = pack_f16(p0, p1);
          if constexpr (ROWS == kRows8) {
            pa[h][q2] = w;
          } else {
            pa[h][q2 * 2 + r] = w;
            if constexpr (ROWS == kHalves) pa[h][q2 * 2 + 1] = pack_rest(p0, p1, w);
          }
        }
      }
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int e = 0; e < NA; ++e) o[c][p][e] *= corr[NR == 2 ? e >> 1 : 0];
    }
    // O += P V: a transposed load gives, of 16 keys and a chunk, two keys' bytes 2 g0 and 2 g0 + 1
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < NC; c += 2) {
        uint32_t vw[4];
        ldmatrix_x4_trans(vw, Vt + tile_at<D>(h * 16 + (lane & 15), c + (lane >> 4)));
#pragma unroll
        for (int q2 = 0; q2 < 2; ++q2) {
          uint32_t e0, o0, e1, o1;
          to_halves<TYPE, true>(vw[q2 * 2], e0, o0);
          to_halves<TYPE, true>(vw[q2 * 2 + 1], e1, o1);
          mma_rows<NA>(o[c + q2][0], pa[h], e0, e1);
          mma_rows<NA>(o[c + q2][1], pa[h], o0, o1);
        }
      }
    if (dead) fence_proxy_async_smem();
    __syncwarp();
    done = i + 1;
    if (lane == 0 && i + kStages < nt) issue(i + kStages);
  }
  // every copy has landed before the ring is used again or the CTA leaves
  for (int i = done; i < min(nt, done + kStages); ++i) mbar_wait(&bar[i % kStages], (i / kStages) & 1);

  // O in units of 2^mrow; the sums of a row's four lanes
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    lrow[r] += __shfl_xor_sync(0xffffffffu, lrow[r], 1);
    lrow[r] += __shfl_xor_sync(0xffffffffu, lrow[r], 2);
    if (j == 0 && g0 + r * 8 < GU) {
      wm[warp][g0 + r * 8] = mrow[r];
      wl[warp][g0 + r * 8] = lrow[r];
    }
  }
  // the appended row joins the last split
  const bool joins = app && s == S - 1;
  if (joins) {
    float k[D / 32], q[D / 32];
    load_row<T, D>(static_cast<const T*>(a.k_new) + bk * D, k);
    for (int g = warp; g < G; g += kWarps) {
      load_row<T, D>(static_cast<const T*>(a.q) + ((size_t)b * a.Hq + h0 + g) * D, q);
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < D / 32; ++e) x = fmaf(q[e], k[e], x);
      x = warp_sum(x) * a.scale_log2;
      if (lane == 0) apm[g] = x;
    }
  }
  __syncthreads();
  const bool aborted = s_abort != 0;
  float* wo = reinterpret_cast<float*>(smem);  // [kWarps][GU][kFoldLd]
  const size_t rec = decode_record_floats(GU < a.G ? GU : a.G, S, D);  // record of a unit
  float* po = a.partial + bu * rec;
  float2* pml = reinterpret_cast<float2*>(po + (size_t)G * S * D);
#pragma unroll
  for (int r = 0; r < NR; ++r) {
    const int g = g0 + r * 8;
    if (g >= G) continue;
    float M = joins ? apm[g] : -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w][g]);
    const float f = xref[r] == -INFINITY ? 0.f : exp2f((xref[r] - M) + (kref[r] - 10.f));
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int e = NR == 2 ? r * 2 : 0;
      float4 v = make_float4(o[c][0][e], o[c][1][e], o[c][0][e + 1], o[c][1][e + 1]);
      if constexpr (ROWS == kHalves) {
        v.x += o[c][0][2];
        v.y += o[c][1][2];
        v.z += o[c][0][3];
        v.w += o[c][1][3];
      }
      *reinterpret_cast<float4*>(wo + (warp * GU + g) * C::kFoldLd + c * 16 + j * 4) =
          make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
    }
    if (warp == 0 && j == 0) {
      float Ls = 0.f;
      if (M != -INFINITY) {
#pragma unroll
        for (int w = 0; w < kWarps; ++w) Ls = fmaf(wl[w][g], exp2f(wm[w][g] - M), Ls);
      }
      const float wa = joins ? exp2f(apm[g] - M) : 0.f;
      Ls += wa;
      apw[g] = wa;
      s_inv[g] = Ls > 0.f || Ls != Ls ? 1.f / Ls : 0.f;
      if (S > 1) pml[g * S + s] = aborted ? make_float2(-INFINITY, 0.f) : make_float2(M, Ls);
    }
  }
  __syncthreads();
  constexpr int D4 = D / 4;
  for (int i = tid; i < G * D4; i += kThreads) {
    const int g = i / D4, d4 = i % D4;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(wo + (w * GU + g) * C::kFoldLd + d4 * 4);
      acc.x += v.x;
      acc.y += v.y;
      acc.z += v.z;
      acc.w += v.w;
    }
    if (joins) {
      float v[4];
      load4(static_cast<const T*>(a.v_new) + bk * D + d4 * 4, v);
      const float wa = apw[g];
      acc.x = fmaf(wa, v[0], acc.x);
      acc.y = fmaf(wa, v[1], acc.y);
      acc.z = fmaf(wa, v[2], acc.z);
      acc.w = fmaf(wa, v[3], acc.w);
    }
    if (aborted) acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (S == 1) {
      const float iv = s_inv[g];
      const float r[4] = {acc.x * iv, acc.y * iv, acc.z * iv, acc.w * iv};
      store4(static_cast<T*>(a.out) + ((size_t)b * a.Hq + h0 + g) * D + d4 * 4, r);
    } else {
      reinterpret_cast<float4*>(po + ((size_t)g * S + s) * D)[d4] = acc;
    }
  }
  // the last CTA of the unit folds its splits
  __syncthreads();
  if (S > 1) {
    if (tid == 0) s_last = atom_add_acq_rel_gpu(&a.cnt_head[bu], 1u) == (uint32_t)S - 1u;
    __syncthreads();
    if (!s_last) return;
    float* wts = wo;  // [G][S] weights of the splits
    for (int g = warp; g < G; g += kWarps) {
      float M = -INFINITY;
      for (int t = lane; t < S; t += 32) M = fmaxf(M, __ldcg(pml + g * S + t).x);
      M = warp_max(M);
      float Ls = 0.f;
      for (int t = lane; t < S; t += 32) {
        const float2 ml = __ldcg(pml + g * S + t);
        const float w = M == -INFINITY ? 0.f : exp2f(ml.x - M);
        wts[g * S + t] = w;
        Ls = fmaf(ml.y, w, Ls);
      }
      Ls = warp_sum(Ls);
      if (lane == 0) s_inv[g] = Ls > 0.f || Ls != Ls ? 1.f / Ls : 0.f;
    }
    __syncthreads();
    for (int i = tid; i < G * D4; i += kThreads) {
      const int g = i / D4, d4 = i % D4;
      const float4* op = reinterpret_cast<const float4*>(po + (size_t)g * S * D) + d4;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
      for (int t = 0; t < S; ++t) {
        const float4 v = __ldcg(op + (size_t)t * D4);
        const float w = wts[g * S + t];
        acc.x = fmaf(v.x, w, acc.x);
        acc.y = fmaf(v.y, w, acc.y);
        acc.z = fmaf(v.z, w, acc.z);
        acc.w = fmaf(v.w, w, acc.w);
      }
      const float iv = s_inv[g];
      const float r[4] = {acc.x * iv, acc.y * iv, acc.z * iv, acc.w * iv};
      store4(static_cast<T*>(a.out) + ((size_t)b * a.Hq + h0 + g) * D + d4 * 4, r);
    }
  }
  // The last unit of the KV head puts the new row into the cache: every CTA that reads its blocks has read
  // them.  The last KV head of the sequence moves the length.
  if (tid == 0) {
    a.cnt_head[bu] = 0u;
    bool last = true;
    if (HG > 1) {
      last = atom_add_acq_rel_gpu(&a.cnt_kv[bk], 1u) == (uint32_t)HG - 1u;
      if (last) a.cnt_kv[bk] = 0u;
    }
    s_kv_last = last;
  }
  if (!app) return;
  __syncthreads();
  if (!s_kv_last) return;
  if (warp == 0)
    append_row<TYPE, T, D>(static_cast<const T*>(a.k_new) + bk * D, a.c.K + bk * a.m_cap * D, a.c.ks + bk * a.c.nblk,
                           a.c.block_log2, L, a.flags);
  if (warp == 1)
    append_row<TYPE, T, D>(static_cast<const T*>(a.v_new) + bk * D, a.c.V + bk * a.m_cap * D, a.c.vs + bk * a.c.nblk,
                           a.c.block_log2, L, a.flags);
  if (tid == 64) {
    if (a.bias != nullptr) a.bias[bk * a.m_cap + L] = 0.f;
    if (atom_add_acq_rel_gpu(&a.cnt_seq[b], 1u) == (uint32_t)a.Hkv - 1u) {
      a.lengths[b] = L + 1;
      a.cnt_seq[b] = 0u;
    }
  }
}

template <int TYPE, typename T, int D, int ROWS>
cudaError_t launch_rows(const QDecodeArgs& a, cudaStream_t st) {
  using C = QCfg<D>;
  CUtensorMap tk, tv;
  const uint64_t rows = (uint64_t)a.B * a.Hkv * a.m_cap;
  if (!encode_rows_u8(&tk, a.c.K, rows, D, kTileRows) || !encode_rows_u8(&tv, a.c.V, rows, D, kTileRows))
    return cudaErrorInvalidValue;
  constexpr auto kern = decode_q_kernel<TYPE, T, D, ROWS>;
  if (const cudaError_t e = set_smem_once<kern>(C::kSmem); e != cudaSuccess) return e;
  const dim3 grid(a.splits, a.Hkv * decode_q_units(a.dtype, a.G), a.B);
  return launch_chained(true, kern, grid, dim3(kThreads), C::kSmem, st, tk, tv, a);
}

template <int TYPE, int D>
cudaError_t launch_dtype(const QDecodeArgs& a, cudaStream_t st) {
  if (a.dtype == SELKV_FP32) return launch_rows<TYPE, float, D, kHalves>(a, st);
  return a.G > 8 ? launch_rows<TYPE, __nv_bfloat16, D, kRows16>(a, st) : launch_rows<TYPE, __nv_bfloat16, D, kRows8>(a, st);
}

}  // namespace

int decode_q_units(int dtype, int G) { return dtype == SELKV_FP32 ? (G + 7) / 8 : 1; }

int decode_q_splits(const selkv_shape& s) {
  const int units = s.num_kv_heads * decode_q_units(s.dtype, s.num_q_heads / s.num_kv_heads);
  const long n = (long)s.batch * units, slots = kPlanSMs;
  const int smax = std::max(1, std::min(64, (s.m_cap + 63) / 64));
  int best = 1;
  long best_cost = -1;
  for (int S = 1; S <= smax; ++S) {
    const long waves = (n * S + slots - 1) / slots;
    const long rows = ((long)(s.m_cap + S - 1) / S + 63) / 64 * 64;
    const long cost = waves * (rows + 512);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      best = S;
    }
  }
  return best;
}

cudaError_t launch_decode_q(const QDecodeArgs& a, cudaStream_t st) {
  if (a.c.type == SELKV_Q_E4M3)
    return a.D == 128 ? launch_dtype<SELKV_Q_E4M3, 128>(a, st) : launch_dtype<SELKV_Q_E4M3, 64>(a, st);
  return a.D == 128 ? launch_dtype<SELKV_Q_INT8, 128>(a, st) : launch_dtype<SELKV_Q_INT8, 64>(a, st);
}

}  // namespace selkv
