// Verification of a tree's tokens against the target's probabilities (selkv_tree_verify).
//
// A walk from the root: the tests of a node's children need two numbers each until one is rejected; a rejection
// and the draw of the next token need sums over the vocabulary.  All the tests' numbers are fetched at once at the
// start, and a cluster of CTAs holds a part of the vocabulary each, so the walk costs a memory round trip and a
// pass for each rejection; the passes read the distributions of the nodes they are at and no others.
//
// Weights are held in 64-bit fixed point, units of 2^-62: an fp32 probability above 2^-39 is exact, differences and
// sums are exact in any order, and so the token that a given number draws does not depend on how the vocabulary is
// split.  (Sums in fp32 would move the borders between tokens by 2^-24 of the whole: one draw in a hundred
// over a flat vocabulary of 128k.)
#include "tree.cuh"

namespace selkv {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kSpan = 1024;             // entries of a warp's step: a sum is kept for each
constexpr int kMaxVocab = 1 << 20;
constexpr u64 kOne = 1ull << 62;

// a * b in units of 2^-62, for a < 2^64 and b < 2^62.
__device__ __forceinline__ u64 mul_fix(u64 a, u64 b) { return (__umul64hi(a, b) << 2) | ((a * b) >> 62); }
// A probability in fixed point; one that is none counts as 0.
__device__ __forceinline__ u64 to_fix(float p, bool& bad) {
  const bool ok = p >= 0.f && p < 2.f;
  bad = bad || !ok;
  return __float2ull_rz((ok ? p : 0.f) * 0x1p62f);
}

struct Smem {
  u64 span[kMaxVocab / kSpan + 1];  // sums of the CTA's spans
  u64 pt[SELKV_MAX_TREE];           // target probability of token t at its parent
  u64 qt[SELKV_MAX_TREE];           // draft's
  u64 mult[SELKV_MAX_TREE];         // masses that the node's rejections were taken with
  u64 warp[kWarps];
  u64 part[2];                      // the CTA's sum, read by the cluster
  float u[SELKV_MAX_TREE];
  int parent[SELKV_MAX_TREE];
  int token[SELKV_MAX_TREE];
  int out[SELKV_MAX_TREE];          // tokens taken out at the node (picked drafts)
  int path[SELKV_MAX_TREE];
};

__device__ __forceinline__ u64 ld_peer_u64(uint32_t peer) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer) : "memory");
  return v;
}
__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The vocabulary's entries at one node, after the node's rejections.
template <bool DRAWN>
struct Weights {
  const float* p;
  const float* q;
  const Smem* sm;
  int rejected;
  bool vec;  // rows 16-byte aligned

  __device__ __forceinline__ void load4x(const float* row, int i, int hi, float (&x)[4]) const {
    if (vec && i + 3 < hi) {
      const float4 v = *reinterpret_cast<const float4*>(row + i);
      x[0] = v.x;
      x[1] = v.y;
      x[2] = v.z;
      x[3] = v.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = i + e < hi ? row[i + e] : 0.f;
    }
  }
  __device__ __forceinline__ void of(int i, int hi, u64 (&r)[4], bool& bad) const {
    float x[4], y[4];
    load4x(p, i, hi, x);
    if (DRAWN && rejected > 0) load4x(q, i, hi, y);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      r[e] = to_fix(x[e], bad);
      if (DRAWN) {
        if (rejected > 0) {
          const u64 f = to_fix(y[e], bad);
          for (int j = 0; j < rejected; ++j) {
            const u64 m = j == 0 ? f : mul_fix(sm->mult[j], f);  // (the first mass is 1)
            r[e] = r[e] > m ? r[e] - m : 0;
          }
        }
      } else {
        for (int j = 0; j < rejected; ++j)
          if (sm->out[j] == i + e) r[e] = 0;
      }
    }
  }
};

// The sum of the weights over the vocabulary: this CTA's entries lo .. hi - 1 span by span, then the cluster's CTAs.
template <bool DRAWN>
__device__ u64 sum_weights(const Weights<DRAWN>& w, Smem* sm, int lo, int hi, int ctas, int& phase, bool& bad) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 mine = 0;
  for (int s0 = lo + warp * kSpan, s = warp; s0 < hi; s0 += kWarps * kSpan, s += kWarps) {
    u64 sum = 0;
#pragma unroll
    for (int k = 0; k < kSpan / 128; ++k) {
      u64 r[4];
      w.of(s0 + k * 128 + lane * 4, hi, r, bad);
      sum += (r[0] + r[1]) + (r[2] + r[3]);
    }
    sum = warp_sum_u64(sum);
    if (lane == 0) sm->span[s] = sum;
    mine += sum;
  }
  if (lane == 0) sm->warp[warp] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    u64 t = 0;
    for (int i = 0; i < kWarps; ++i) t += sm->warp[i];
    sm->part[phase & 1] = t;
  }
  cluster_arrive();
  cluster_wait();
  u64 total = 0;
  for (int c = 0; c < ctas; ++c) total += ld_peer_u64(peer_smem(smem_u32(&sm->part[phase & 1]), c));
  ++phase;
  return total;
}

template <bool DRAWN>
__global__ __launch_bounds__(kThreads) void tree_verify_kernel(VerifyArgs a, int part) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  Smem* sm = reinterpret_cast<Smem*>(smem_raw);
  const int tid = threadIdx.x, rank = blockIdx.x, ctas = gridDim.x, b = blockIdx.y;
  const int lo = min(a.V, rank * part), hi = min(a.V, lo + part);
  bool bad = false;
  uint32_t flags = 0;

  int n = a.counts != nullptr ? a.counts[b] : a.T;
  if (n < 0 || n > a.T) {
    flags |= SELKV_DEVERR_LENGTH;
    n = min(max(n, 0), a.T);
  }
  const float* target = a.target + (size_t)b * a.T * a.V;
  const float* draft = DRAWN ? a.draft + (size_t)b * a.T * a.V : nullptr;
  if (tid < n) {
    int p = -1;
    if (tid > 0) {
      p = a.parents != nullptr ? a.parents[(size_t)b * a.T + tid] : tid - 1;
      if (p < -1 || p >= tid) {
        flags |= SELKV_DEVERR_TREE;
        p = -1;
      }
    }
    float u = a.uniforms[(size_t)b * a.T + tid];
    if (!(u >= 0.f && u < 1.f)) {
      bad = true;
      u = u >= 1.f ? 0x1.fffffep-1f : 0.f;
    }
    const int x = tid > 0 ? a.tokens[(size_t)b * a.T + tid] : 0;
    u64 pt = 0, qt = kOne;
    if (p >= 0) {
      if (x >= 0 && x < a.V) {
        pt = to_fix(target[(size_t)p * a.V + x], bad);
        if (DRAWN) qt = to_fix(draft[(size_t)p * a.V + x], bad);
      } else {
        bad = true;
      }
    }
    sm->parent[tid] = p;
    sm->token[tid] = x;
    sm->u[tid] = u;
    sm->pt[tid] = pt;
    sm->qt[tid] = qt;
  }
  if (tid == 0) {
    sm->mult[0] = kOne;
    // (the token of rows without mass; another CTA's draw comes behind the cluster's first barrier)
    if (rank == 0) a.next[b] = n > 0 ? a.V - 1 : -1;
  }
  __syncthreads();

  // The walk; every thread of the cluster takes the same way.
  int node = 0, taken = n > 0 ? 1 : 0, rejected = 0, phase = 0;
  u64 M = kOne, Z = 0;  // the mass of the tests, and the sum over the vocabulary where it is known
  bool known = false;
  const bool vec = (a.V & 3) == 0;
  auto weights = [&](int rej) {
    return Weights<DRAWN>{target + (size_t)node * a.V, DRAWN ? draft + (size_t)node * a.V : nullptr, sm, rej, vec};
  };
  if (tid == 0) sm->path[0] = 0;
  for (int t = 1; t < n; ++t) {
    if (sm->parent[t] != node) continue;
    bool bu = false;
    const u64 u = to_fix(sm->u[t], bu);
    u64 r = sm->pt[t];
    const int x = sm->token[t];
    if (DRAWN) {
      for (int j = 0; j < rejected; ++j) {
        const u64 m = mul_fix(sm->mult[j], sm->qt[t]);
        r = r > m ? r - m : 0;
      }
    } else {
      for (int j = 0; j < rejected; ++j)
        if (sm->out[j] == x) r = 0;
    }
    if (mul_fix(u, DRAWN ? mul_fix(M, sm->qt[t]) : M) < r) {
      if (tid == 0) sm->path[taken] = t;
      ++taken;
      node = t;
      rejected = 0;
      M = kOne;
      known = false;
      continue;
    }
    // a rejection: the weights that are left, and their mass
    if (DRAWN) {
      const u64 left = sum_weights(weights(rejected + 1), sm, lo, hi, ctas, phase, bad);
      known = left > 0;
      if (known) {
        Z = M = left;
        ++rejected;
        if (rejected < SELKV_MAX_TREE && tid == 0) sm->mult[rejected] = left;
      }
    } else if (M > r) {
      M -= r;
      if (tid == 0) sm->out[rejected] = x;
      ++rejected;
    }
    __syncthreads();
  }
  if (n > 0) {
    if (!known) Z = sum_weights(weights(rejected), sm, lo, hi, ctas, phase, bad);
    // the CTA and the span that the number falls into, then the entry
    bool bu = false;
    const u64 at = mul_fix(Z, to_fix(sm->u[0], bu));
    u64 below = 0, own = 0;
    for (int c = 0; c <= rank; ++c) {
      below += own;
      own = ld_peer_u64(peer_smem(smem_u32(&sm->part[(phase - 1) & 1]), c));
    }
    if (Z == 0) bad = true;
    else if (tid < 32 && at >= below && at - below < own) {
      const int spans = (hi - lo + kSpan - 1) / kSpan;
      u64 rest = at - below;  // mass before the entry
      int s = 0;
      for (int s0 = 0; s0 < spans; s0 += 32) {
        const u64 v = s0 + tid < spans ? sm->span[s0 + tid] : 0;
        u64 inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
          if (tid >= o) inc += y;
        }
        const uint32_t over = __ballot_sync(0xffffffffu, inc > rest);
        const int k = over != 0 ? __ffs(over) - 1 : 31;
        const u64 inck = __shfl_sync(0xffffffffu, inc, k), vk = __shfl_sync(0xffffffffu, v, k);
        if (over != 0) {
          s = s0 + k;
          rest -= inck - vk;
          break;
        }
        rest -= inck;
      }
      const Weights<DRAWN> w = weights(rejected);
      for (int k = 0; k < kSpan / 128; ++k) {
        const int i = lo + s * kSpan + k * 128 + tid * 4;
        u64 r[4];
        w.of(i, hi, r, bad);
        const u64 v = (r[0] + r[1]) + (r[2] + r[3]);
        u64 inc = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const u64 y = __shfl_up_sync(0xffffffffu, inc, o);
          if (tid >= o) inc += y;
        }
        const uint32_t over = __ballot_sync(0xffffffffu, inc > rest);
        if (over != 0) {
          if (tid == __ffs(over) - 1) {
            u64 left = rest - (inc - v);
            int e = 0;
            while (e < 3 && r[e] <= left) left -= r[e++];
            a.next[b] = min(i + e, a.V - 1);
          }
          break;
        }
        rest -= __shfl_sync(0xffffffffu, inc, 31);
      }
    }
  }
  __syncthreads();
  if (rank == 0) {
    if (tid < a.T) a.path[(size_t)b * a.T + tid] = tid < taken ? sm->path[tid] : -1;
    if (tid == 0) a.accepted[b] = taken;
  }
  if (bad) flags |= SELKV_DEVERR_VALUE;
  if (flags != 0) raise_flag(a.flags, flags);
  // no CTA leaves while another reads its sum
  cluster_arrive();
  cluster_wait();
}

template <bool DRAWN>
cudaError_t launch(const VerifyArgs& a, cudaStream_t s) {
  constexpr int smem = (int)sizeof(Smem);
  if (const cudaError_t e = set_smem_once<tree_verify_kernel<DRAWN>>(smem); e != cudaSuccess) return e;
  // CTAs of a sequence: up to the eight of a portable cluster while there is a span for each of its warps
  int ctas = 1;
  while (ctas < 8 && (long long)a.B * ctas < 2 * kPlanSMs && a.V > ctas * kSpan) ctas *= 2;
  const int part = ((a.V + ctas - 1) / ctas + kSpan - 1) / kSpan * kSpan;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ctas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas, (unsigned)a.B, 1);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, tree_verify_kernel<DRAWN>, a, part);
}

}  // namespace

cudaError_t launch_tree_verify(const VerifyArgs& a, cudaStream_t s) {
  return a.draft != nullptr ? launch<true>(a, s) : launch<false>(a, s);
}

}  // namespace selkv
