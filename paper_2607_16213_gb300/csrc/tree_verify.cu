// Verification of a tree's tokens against the target's probabilities (selkv_tree_verify).
//
// A walk from the root: the tests of a node's children need two numbers each until one is rejected; a rejection
// and the draw of the next token need sums over the vocabulary.  All the tests' numbers are fetched at once at the
// start, and a cluster of CTAs holds a part of the vocabulary each, so the walk costs a memory round trip and a
// pass for each rejection; the passes read the distributions of the nodes they are at and no others.
//
// Tests and sums are held in 64-bit fixed point, units of 2^-62.  A pass adds up each thread's few weights as an fp32 number and its
// error (an exact difference of three operations and an exact sum of six, where a 64-bit sum took 70 instructions an entry)
// and goes on in fixed point from there.  So the token that a given number draws depends on how the vocabulary is split for
// borders right beside it alone.  (Sums in fp32 would move the borders between tokens by 2^-24 of the whole: one draw in a hundred
// over a flat vocabulary of 128k.)  After k rejections the weights are max(p - A q, 0) with A the sum of the masses that they were
// taken with (max(max(x, 0) - y, 0) is max(x - y, 0) for y >= 0), so a pass costs the same however many there were.
//
// How far a border may be off, u = 2^-24.  Eight entries in a Pair: errors of up to u of the sum each, whose own sum is rounded to u
// of itself: at most (2 + .. + 8 + 8) u^2 = 43 u^2 of the sum; whole units: 1.5 x 2^-62 an eight, 2^-44.4 for 2^20 entries.  Together
// below 2^-42.2 of the mass m.  From the second rejection on, an entry p - A q cancels: A as two numbers, l and e rounded,
// 2^-45.4 of p, so that of the whole.  A takes on the errors of the masses in it, but not more (a larger A leaves a smaller mass,
// by less).  So after k rejections sums and tests are right to 2^-42 (m + k), and in parts of m, as the numbers count, to
// 2^-42 (1 + k / m).  Met, for 8192 entries and two rejections: 2^-48.7 of m = 0.0023, 2^-38.5 of m = 0.00023.
//
// 1 x 32000 entries, 8 tokens: 8.7 us on the GPU, latencies (tests, pass, draw).  64 x 128000, 16 tokens: 41 us where the rows of the
// 1.5 passes a sequence takes would need 14: latencies, and sequences with up to four passes (about 25 instructions
// an entry and pass: 8 us of all issue slots).
#include "tree.cuh"
#include "tree_fixed.h"

namespace selkv {
namespace {

typedef unsigned long long u64;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kSpan = 256;              // entries of a warp's step: a sum is kept for each
constexpr u64 kOne = 1ull << 62;

// a * b in units of 2^-62, for a < 2^64 and b < 2^62.
__device__ __forceinline__ u64 mul_fix(u64 a, u64 b) { return (__umul64hi(a, b) << 2) | ((a * b) >> 62); }
// A q in units of 2^-62, for A in units of 2^-kTimes below 2^(64 - kTimes) and q < 2^63; all ones where it is 4 or more (no weight
// is left there: p < 2).
constexpr int kTimes = 56;
__device__ __forceinline__ u64 times_fix(u64 A, u64 q) {
  const u64 hi = __umul64hi(A, q), lo = A * q;
  return hi >> kTimes != 0 ? ~0ull : (hi << (64 - kTimes)) | (lo >> kTimes);
}
struct Smem {
  u64 span[kMaxVocab / kSpan + 1];  // sums of the CTA's spans
  u64 pt[SELKV_MAX_TREE];           // target probability of token t at its parent
  u64 qt[SELKV_MAX_TREE];           // draft's
  u64 warp[kWarps];
  u64 part[2];                      // the CTA's sum, read by the cluster
  float mine[kThreads];             // each thread's sum in fp32 (registers are short)
  float warp_about[kWarps];
  float about[2];                   // the CTA's in fp32: where the cluster's is 4 or more the fixed point has wrapped
  float u[SELKV_MAX_TREE];
  int parent[SELKV_MAX_TREE];
  uint32_t first[SELKV_MAX_TREE / 32];  // tokens that are accepted when no child of their parent was rejected before, as bits
  int token[SELKV_MAX_TREE];
  int out[SELKV_MAX_TREE];          // tokens taken out at the node (picked drafts)
  int path[SELKV_MAX_TREE];
  // where the walk stands, from the warp that takes it to the others
  int node, rejected, taken, more;  // more: it goes on behind the pass
  u64 A;
};

__device__ __forceinline__ u64 ld_peer_u64(uint32_t peer) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(peer) : "memory");
  return v;
}
__device__ __forceinline__ float ld_peer_f32(uint32_t peer) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(peer) : "memory");
  return v;
}
__device__ __forceinline__ u64 warp_sum_u64(u64 v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A sum of fp32 numbers as the rounded sum and what it is short of.
struct Pair {
  float s, e;
  __device__ __forceinline__ void add(float x, float more) {
    const float t = s + x, b = t - s;
    e += (s - (t - b)) + (x - b) + more;
    s = t;
  }
  __device__ __forceinline__ u64 fixed() const { return __float2ull_rz(s * 0x1p62f) + (u64)__float2ll_rn(e * 0x1p62f); }
};

// The vocabulary's entries at one node, after the node's rejections.
template <bool DRAWN>
struct Weights {
  const float* p;
  const float* q;
  const Smem* sm;
  int rejected;
  u64 A;         // sum of the masses that the rejections were taken with, units of 2^-kTimes
  float Ah, Al;  // the same as an fp32 number and the rest
  bool vec;      // rows 16-byte aligned

  __device__ __forceinline__ static float4 four(const float* row, int i, int hi, bool whole) {
    if (whole) return *reinterpret_cast<const float4*>(row + i);
    return make_float4(i < hi ? row[i] : 0.f, i + 1 < hi ? row[i + 1] : 0.f, i + 2 < hi ? row[i + 2] : 0.f, i + 3 < hi ? row[i + 3] : 0.f);
  }
  __device__ __forceinline__ bool uses_q() const { return DRAWN && rejected > 0; }
  // What is no probability counts as 0.
  __device__ __forceinline__ static void clean(float4& v, bool& bad) {
    if (((__float_as_uint(v.x) | __float_as_uint(v.y) | __float_as_uint(v.z) | __float_as_uint(v.w)) >> 30) == 0u) return;
    float* x = reinterpret_cast<float*>(&v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool ok = x[e] >= 0.f && x[e] < 2.f;
      bad = bad || !ok;
      x[e] = ok ? x[e] : 0.f;
    }
  }
  __device__ __forceinline__ u64 weight(float x, float y) const {
    bool bad = false;
    u64 r = to_fix(x, bad);
    if (DRAWN && rejected > 0) {
      const u64 f = to_fix(y, bad), m = rejected == 1 ? f : times_fix(A, f);  // (the first mass is 1)
      r = r > m ? r - m : 0;
    }
    return r;
  }
  __device__ __forceinline__ bool is_out(int i) const {
    for (int j = 0; j < rejected; ++j)
      if (sm->out[j] == i) return true;
    return false;
  }
  // The weight of one entry onto a sum, after no (kAfter 0), one or more rejections of drawn drafts.
  template <int kAfter>
  __device__ __forceinline__ void onto(Pair& sum, float x, float y) const {
    if (kAfter == 0) {
      sum.add(x, 0.f);
    } else if (kAfter == 1) {
      const float z = fmaxf(x, y), s = z - y, e = (z - s) - y;  // exact for x > y >= 0, and 0 for the others
      sum.add(s, e);
    } else {
      const float h = __fmul_rn(Ah, y), l = fmaf(Ah, y, -h) + Al * y;
      const float s = x - h, b = s - x, e = ((x - (s - b)) - (h + b)) - l;
      const bool pos = s + e > 0.f;
      sum.add(pos ? s : 0.f, pos ? e : 0.f);
    }
  }
  // Whether a token between s0 and s0 + kSpan is taken out (the warp's).
  __device__ __forceinline__ bool takes(int s0) const {
    bool t = false;
    if (!DRAWN)
      for (int j = threadIdx.x & 31; j < rejected; j += 32) t = t || (sm->out[j] >= s0 && sm->out[j] < s0 + kSpan);
    return !DRAWN && rejected > 0 && __any_sync(0xffffffffu, t);
  }
};

// This warp's part of the sum of the weights over the CTA's entries lo .. hi - 1, span by span; two spans' loads are on
// their way together.
template <bool DRAWN, int kAfter>
__device__ __forceinline__ u64 sum_spans(const Weights<DRAWN>& w, Smem* sm, int lo, int hi, bool& bad) {
  constexpr int kRows = kSpan / 128;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, spans = (hi - lo + kSpan - 1) / kSpan;
  u64 mine = 0;
#pragma unroll 1
  for (int s = warp; s < spans; s += 2 * kWarps) {
    float4 x[2][kRows], y[2][kRows];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int s0 = lo + (s + h * kWarps) * kSpan;
      if (w.vec && s0 + kSpan <= hi) {
        const float4* p = reinterpret_cast<const float4*>(w.p + s0) + lane;
        const float4* q = reinterpret_cast<const float4*>(w.q + s0) + lane;
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          x[h][k] = p[k * 32];
          if (kAfter > 0) y[h][k] = q[k * 32];
        }
      } else {
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
          x[h][k] = Weights<DRAWN>::four(w.p, s0 + k * 128 + lane * 4, hi, false);
          if (kAfter > 0) y[h][k] = Weights<DRAWN>::four(w.q, s0 + k * 128 + lane * 4, hi, false);
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = s + h * kWarps;
      if (at >= spans) continue;
      const bool taken = w.takes(lo + at * kSpan);
      Pair sum{0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float4 a = x[h][k], c = kAfter > 0 ? y[h][k] : make_float4(0.f, 0.f, 0.f, 0.f);
        Weights<DRAWN>::clean(a, bad);
        if (kAfter > 0) Weights<DRAWN>::clean(c, bad);
        if (taken) {
          const int i = lo + at * kSpan + k * 128 + lane * 4;
          a.x = w.is_out(i) ? 0.f : a.x;
          a.y = w.is_out(i + 1) ? 0.f : a.y;
          a.z = w.is_out(i + 2) ? 0.f : a.z;
          a.w = w.is_out(i + 3) ? 0.f : a.w;
        }
        w.template onto<kAfter>(sum, a.x, c.x);
        w.template onto<kAfter>(sum, a.y, c.y);
        w.template onto<kAfter>(sum, a.z, c.z);
        w.template onto<kAfter>(sum, a.w, c.w);
      }
      sm->mine[threadIdx.x] += sum.s;
      const u64 f = warp_sum_u64(sum.fixed());
      if (lane == 0) sm->span[at] = f;
      mine += f;
    }
  }
  return mine;
}

// The sum of the weights over the vocabulary: this CTA's entries, then the cluster's CTAs.
template <bool DRAWN>
__device__ u64 sum_weights(const Weights<DRAWN>& w, Smem* sm, int lo, int hi, int ctas, int& phase, bool& bad) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 mine;
  sm->mine[threadIdx.x] = 0.f;
  if (!DRAWN || w.rejected == 0) mine = sum_spans<DRAWN, 0>(w, sm, lo, hi, bad);
  else if (w.rejected == 1) mine = sum_spans<DRAWN, 1>(w, sm, lo, hi, bad);
  else mine = sum_spans<DRAWN, 2>(w, sm, lo, hi, bad);
  float about = warp_sum(sm->mine[threadIdx.x]);
  if (lane == 0) {
    sm->warp[warp] = mine;
    sm->warp_about[warp] = about;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const u64 t = warp_sum_u64(threadIdx.x < kWarps ? sm->warp[threadIdx.x] : 0);
    const float x = warp_sum(threadIdx.x < kWarps ? sm->warp_about[threadIdx.x] : 0.f);
    if (threadIdx.x == 0) {
      sm->part[phase & 1] = t;
      sm->about[phase & 1] = x;
    }
  }
  cluster_arrive();
  cluster_wait();
  u64 total = 0;
  about = 0.f;
  for (int c = 0; c < ctas; ++c) {
    total += ld_peer_u64(peer_smem(smem_u32(&sm->part[phase & 1]), c));
    about += ld_peer_f32(peer_smem(smem_u32(&sm->about[phase & 1]), c));
  }
  bad = bad || about >= 3.99f;
  ++phase;
  return total;
}

template <bool DRAWN>
__global__ __launch_bounds__(kThreads, 2) void tree_verify_kernel(VerifyArgs a, int part) {
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
  bool yes = false;
  if (tid < a.T) {
    // (what the count does not decide is asked for beside it)
    int p = tid > 0 ? (a.parents != nullptr ? a.parents[(size_t)b * a.T + tid] : tid - 1) : -1;
    float u = a.uniforms[(size_t)b * a.T + tid];
    const int x = tid > 0 ? a.tokens[(size_t)b * a.T + tid] : 0;
    u64 pt = 0, qt = kOne;
    if (tid < n) {
      if (p < -1 || p >= tid) {
        if (tid > 0) flags |= SELKV_DEVERR_TREE;
        p = -1;
      }
      if (!(u >= 0.f && u < 1.f)) {
        bad = true;
        u = u >= 1.f ? 0x1.fffffep-1f : 0.f;
      }
      if (p >= 0) {
        if (x >= 0 && x < a.V) {
          pt = to_fix(target[(size_t)p * a.V + x], bad);
          if (DRAWN) qt = to_fix(draft[(size_t)p * a.V + x], bad);
        } else {
          bad = true;
        }
      }
    }
    sm->parent[tid] = p;
    sm->token[tid] = x;
    sm->u[tid] = u;
    sm->pt[tid] = pt;
    sm->qt[tid] = qt;
    bool none = false;
    yes = mul_fix(to_fix(u, none), qt) < pt;
  }
  if (tid < SELKV_MAX_TREE) {
    const uint32_t bits = __ballot_sync(0xffffffffu, yes);
    if ((tid & 31) == 0) sm->first[tid >> 5] = bits;
  }
  // (the token of rows without mass; another CTA's draw comes behind the cluster's first barrier)
  if (tid == 0 && rank == 0) a.next[b] = n > 0 ? a.V - 1 : -1;
  __syncthreads();

  // The walk, by the first warp of each CTA of the cluster in the same way, from one pass over the vocabulary to the next.
  // The others take part in the passes.
  int phase = 0;
  const bool vec = (a.V & 3) == 0;
  auto weights = [&](int node, int rej, u64 times) {
    const float high = __ull2float_rn(times) * 0x1p-56f;
    const float low = __ll2float_rn((long long)(times - __float2ull_rz(high * 0x1p56f))) * 0x1p-56f;
    return Weights<DRAWN>{target + (size_t)node * a.V, DRAWN ? draft + (size_t)node * a.V : nullptr, sm, rej, times, high, low, vec};
  };
  int node = 0, taken = n > 0 ? 1 : 0, rejected = 0;
  u64 M = kOne, Z = 0;  // the mass of the tests, and the sum over the vocabulary where it is known
  u64 A = 0;            // the sum of the masses that the node's rejections were taken with
  if (n > 0) {
    uint32_t kids[SELKV_MAX_TREE / 32];  // the node's children that are not tried yet, as bits
    auto children = [&] {
#pragma unroll
      for (int k = 0; k < SELKV_MAX_TREE / 32; ++k) {
        kids[k] = 0u;
        if (k * 32 >= n) continue;
        const int t = k * 32 + (tid & 31);
        kids[k] = __ballot_sync(0xffffffffu, t > node && t < n && sm->parent[t] == node);
      }
    };
    if (tid < 32) {
      children();
      if (tid == 0) sm->path[0] = 0;
    }
    bool known = false;  // Z is the sum of the weights as they are
    for (;;) {
      if (tid < 32) {
        bool pass = false;
        for (;;) {
          int t = -1;
#pragma unroll
          for (int k = SELKV_MAX_TREE / 32 - 1; k >= 0; --k)
            if (kids[k] != 0u) t = k * 32 + __ffs(kids[k]) - 1;
          if (t < 0) break;
#pragma unroll
          for (int k = 0; k < SELKV_MAX_TREE / 32; ++k)
            if (t >> 5 == k) kids[k] &= kids[k] - 1u;
          bool accept;
          u64 r = 0;
          const int x = sm->token[t];
          if (rejected == 0) {
            accept = (sm->first[t >> 5] >> (t & 31)) & 1u;
            if (!DRAWN && !accept) r = sm->pt[t];
          } else {
            bool none = false;
            const u64 u = to_fix(sm->u[t], none);
            r = sm->pt[t];
            if (DRAWN) {
              const u64 m = rejected == 1 ? sm->qt[t] : times_fix(A, sm->qt[t]);
              r = r > m ? r - m : 0;
            } else {
              for (int j = 0; j < rejected; ++j)
                if (sm->out[j] == x) r = 0;
            }
            accept = mul_fix(u, DRAWN ? mul_fix(M, sm->qt[t]) : M) < r;
          }
          if (accept) {
            if (tid == 0) sm->path[taken] = t;
            ++taken;
            node = t;
            rejected = 0;
            M = kOne;
            A = 0;
            known = false;
            children();
            continue;
          }
          // a rejection: the weights that are left, and their mass
          if (DRAWN) {
            pass = true;
            break;
          }
          if (M > r) {
            M -= r;
            if (tid == 0) sm->out[rejected] = x;
            ++rejected;
          }
          __syncwarp();
        }
        __syncwarp();  // (every lane has read the last round's A)
        if (tid == 0) {
          sm->node = node;
          sm->rejected = rejected + (pass ? 1 : 0);
          sm->taken = taken;
          sm->more = pass ? 1 : known ? -1 : 0;
          sm->A = pass ? A + (M >> (62 - kTimes)) : A;
        }
      }
      __syncthreads();
      const int more = sm->more;
      if (more < 0) break;
      const u64 sum = sum_weights(weights(sm->node, sm->rejected, sm->A), sm, lo, hi, ctas, phase, bad);
      if (more == 0) {
        Z = sum;
        break;
      }
      if (tid < 32) {
        known = sum > 0;
        if (known) {
          Z = M = sum;
          A = sm->A;
          ++rejected;
        }
      }
      // (sm's words are read: the cluster's barrier of the sum lies behind them)
    }
    node = sm->node;
    taken = sm->taken;
    // the CTA and the span that the number falls into, then the entry
    bool bu = false;
    const u64 at = mul_fix(Z, to_fix(sm->u[0], bu));
    u64 below = 0, own = 0;
    for (int c = 0; c <= rank; ++c) {
      below += own;
      own = ld_peer_u64(peer_smem(smem_u32(&sm->part[(phase - 1) & 1]), c));
    }
    // (no CTA leaves or goes on while another reads its sum; from here on they need one another no more)
    cluster_arrive();
    cluster_wait();
    // (the first warp's from here on: it knows the sum)
    // (a row without mass is none; one whose picked drafts took all that its sum, a rounding below 1, had is)
    if (tid < 32 && Z == 0) bad = bad || M == kOne;
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
      const Weights<DRAWN> w = weights(node, rejected, A);
      const int s0 = lo + s * kSpan;
      const bool whole = vec && s0 + kSpan <= hi, taken = w.takes(s0);
#pragma unroll 1
      for (int k = 0; k < kSpan / 128; ++k) {
        const int i = s0 + k * 128 + tid * 4;
        float4 x = Weights<DRAWN>::four(w.p, i, hi, whole);
        float4 y = w.uses_q() ? Weights<DRAWN>::four(w.q, i, hi, whole) : make_float4(0.f, 0.f, 0.f, 0.f);
        Weights<DRAWN>::clean(x, bad);
        Weights<DRAWN>::clean(y, bad);
        u64 r[4] = {w.weight(x.x, y.x), w.weight(x.y, y.y), w.weight(x.z, y.z), w.weight(x.w, y.w)};
        if (taken) {
#pragma unroll
          for (int e = 0; e < 4; ++e) r[e] = w.is_out(i + e) ? 0 : r[e];
        }
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
        // (the entries' sum may fall short of the span's by its rounding: then the last one that has weight)
        const uint32_t some = __ballot_sync(0xffffffffu, v > 0);
        if (some != 0 && tid == 31 - __clz(some)) a.next[b] = min(i + (r[3] > 0 ? 3 : r[2] > 0 ? 2 : r[1] > 0 ? 1 : 0), a.V - 1);
        __syncwarp();
      }
    }
  }
  if (rank == 0) {
    __syncthreads();  // the path is written
    if (tid < a.T) a.path[(size_t)b * a.T + tid] = tid < taken ? sm->path[tid] : -1;
    if (tid == 0) a.accepted[b] = taken;
  }
  if (bad) flags |= SELKV_DEVERR_VALUE;
  if (flags != 0) raise_flag(a.flags, flags);
}

template <bool DRAWN>
cudaError_t launch(const VerifyArgs& a, cudaStream_t s) {
  constexpr int smem = (int)sizeof(Smem);
  if (const cudaError_t e = set_smem_once<tree_verify_kernel<DRAWN>>(smem); e != cudaSuccess) return e;
  // CTAs of a sequence: up to the eight of a portable cluster while SMs are left and there is work for each (64 x 128000 entries: 8
  // 42.6 us, 4 44.1)
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
