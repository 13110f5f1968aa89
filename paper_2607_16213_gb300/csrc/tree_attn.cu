// Compensated attention of a tree of drafted tokens (selkv_tree_attn): fp32 on CUDA cores, and for both
// types the kernel that joins the pieces of a unit.
//
//   out[t] = sum_i p_i v_i,  p = softmax(q_t . k_i / sqrt(d) + bias_i) over the cached rows, token t's ancestors and t.
//
// The G T query rows of a KV head meet its rows together: the cache is read once per block of rows.  The list
// of all (sequence, KV head, row block, key tile) is cut into pieces, or into equal shares of consecutive tiles, one a
// CTA (tree.cuh), so ragged lengths leave no CTA idle; a unit that lies in one is finished there, the others' pieces go through memory as (reference, sum, output) and are joined in list order by tree_join_kernel: results
// do not depend on scheduling.
#include <cfloat>

#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kThreads = 256;

// Finish row `row` of a unit: elements d .. d + 3.
template <typename T>
__device__ __forceinline__ void put_out(const TreeArgs& a, int b, int kv, int r, int d, const float (&x)[4]) {
  store4(static_cast<T*>(a.out) + (((size_t)b * a.Hq + kv * a.G) * a.T + r) * a.D + d, x);
}

// fp32: tiles of 64 keys, a thread holds RPT rows x 4 keys of the logits and RPT rows x D / 16 elements of the
// output; 16 threads share a row, so its statistics and probabilities stay within half a warp.
// The products run on the FMA units: R rows cost 4 R d operations per key for 8 d bytes, so above about 20 rows
// a KV head the arithmetic bounds it, below the loads.  2 heads, d 64, 7 tokens, a pass on the GPU: 2 x 101-201 rows 11.1 us, 2 x 1000
// 13.5, the join 3 us of it: latency (list, tile, statistics, partials); 16000 rows 37.8, 2 x 16000 51.7 (no copy is under way
// while a tile is worked on).
template <int D, int RPT>
__global__ __launch_bounds__(kThreads) void tree_simt_kernel(TreeArgs a) {
  constexpr int RT = RPT * 16, KEYS = kTreeSimtKeys;
  constexpr int LD = D + 4, PLD = KEYS + 4;  // (padded: 16 rows' float4 in different banks)
  constexpr int NE = D / 64;                 // float4 of the output per thread and row
  extern __shared__ __align__(16) float sm[];
  float* Qs = sm;                 // [RT][LD]
  float* Ks = Qs + RT * LD;       // [KEYS][LD]; the probabilities [RT][PLD] lie over it once it is read
  float* Vs = Ks + KEYS * LD;     // [KEYS][D]
  float* bs = Vs + KEYS * D;      // [KEYS] bias in base 2, -inf: the key is out
  uint4* seen = reinterpret_cast<uint4*>(bs + KEYS);  // [SELKV_MAX_TREE]
  const TreeList list = tree_list_at(seen + SELKV_MAX_TREE, a.B);
  __shared__ int8_t up[SELKV_MAX_TREE];
  float* Ps = Ks;
  static_assert(RT * PLD <= KEYS * LD, "probabilities fit the keys' place");
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;

  chain_begin();
  tree_list<KEYS, kTreeSimtMinTiles>(a, list, blockIdx.x, gridDim.x);
  if (blockIdx.x == 0) tree_list_store(a, list);
  for (TreePiece p = *list.first; p.left > 0; tree_next<KEYS>(a, list, p)) {
    const size_t bk = (size_t)p.b * a.Hkv + p.kv;
    const int cache_tiles = (p.L + KEYS - 1) / KEYS;
    const int row0 = p.blk * RT, rows = min(RT, a.R - row0);
    __syncthreads();  // the last piece's rows are read
    const float* q = static_cast<const float*>(a.q) + (((size_t)p.b * a.Hq + p.kv * a.G) * a.T + row0) * D;
    for (int i = tid; i < RT * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (r < rows) load4(q + (size_t)r * D + d, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= a.scale_log2;
      store4(Qs + r * LD + d, x);
    }
    if (p.first + p.count > cache_tiles && tid < 32) tree_ancestors(a, p.b, p.n, seen, up);  // (the tile loop's barrier is behind it)
    float m[RPT], l[RPT], o[RPT][NE * 4];
    int tok[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
      tok[i] = (row0 + ty * RPT + i) % a.T;
#pragma unroll
      for (int e = 0; e < NE * 4; ++e) o[i][e] = 0.f;
    }
    for (int t = p.first; t < p.first + p.count; ++t) {
      const bool drafts = t >= cache_tiles;
      const int key0 = (drafts ? t - cache_tiles : t) * KEYS, keys = min(KEYS, (drafts ? p.n : p.L) - key0);
      const float* kp = static_cast<const float*>(drafts ? a.k_new : a.Kc) + (bk * (drafts ? a.T : a.m_cap) + key0) * D;
      const float* vp = static_cast<const float*>(drafts ? a.v_new : a.Vc) + (bk * (drafts ? a.T : a.m_cap) + key0) * D;
      const float* bias = drafts || a.bias == nullptr ? nullptr : a.bias + bk * a.m_cap + key0;
      __syncthreads();  // the last tile is read (and Q is there)
      for (int i = tid; i < KEYS * (D / 4); i += kThreads) {
        const int r = i / (D / 4), d = i % (D / 4) * 4;
        float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
        // (a row without weight may hold anything)
        if (r < keys && (bias == nullptr || bias[r] != -INFINITY)) {
          load4(kp + (size_t)r * D + d, x);
          load4(vp + (size_t)r * D + d, y);
        }
        store4(Ks + r * LD + d, x);
        store4(Vs + r * D + d, y);
      }
      if (tid < KEYS) bs[tid] = tid >= keys ? -INFINITY : bias != nullptr ? bias[tid] * kLog2e : 0.f;
      __syncthreads();
      // logits of rows ty RPT + i and keys tx + 16 j
      float s[RPT][4];
#pragma unroll
      for (int i = 0; i < RPT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int d = 0; d < D; d += 4) {
        float kx[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) load4(Ks + (tx + 16 * j) * LD + d, kx[j]);
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
          float qx[4];
          load4(Qs + (ty * RPT + i) * LD + d, qx);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][j] = fmaf(qx[e], kx[j][e], s[i][j]);
        }
      }
      __syncthreads();  // the keys are read: the probabilities go there
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        float mx = -INFINITY;
        const uint4 sees = drafts ? seen[tok[i]] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = tx + 16 * j;
          const float b = bs[key];
          bool in = b != -INFINITY;
          if (drafts) {
            const uint32_t w = key0 == 0 ? (key < 32 ? sees.x : sees.y) : (key < 32 ? sees.z : sees.w);
            in = in && ((w >> (key & 31)) & 1u);
          }
          s[i][j] = in ? s[i][j] + b : -INFINITY;
          mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
        const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.f : mn;
        const float f = exp2f(m[i] - ref);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float x = exp2f(s[i][j] - ref);
          Ps[(ty * RPT + i) * PLD + tx + 16 * j] = x;
          sum += x;
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        m[i] = mn;
        l[i] = l[i] * f + sum;
#pragma unroll
        for (int e = 0; e < NE * 4; ++e) o[i][e] *= f;
      }
      __syncwarp();  // a row's probabilities are written and read by the same half warp
#pragma unroll 2
      for (int k = 0; k < KEYS; k += 4) {
        float px[RPT][4];
#pragma unroll
        for (int i = 0; i < RPT; ++i) load4(Ps + (ty * RPT + i) * PLD + k, px[i]);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          float v[NE * 4];
#pragma unroll
          for (int e = 0; e < NE; ++e) load4(Vs + (k + kk) * D + tx * 4 + 64 * e, reinterpret_cast<float(&)[4]>(v[e * 4]));
#pragma unroll
          for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int e = 0; e < NE * 4; ++e) {
              // (an unseen token's row may hold infinities or NaN)
              const float x = drafts && px[i][kk] == 0.f ? 0.f : v[e];
              o[i][e] = fmaf(px[i][kk], x, o[i][e]);
            }
        }
      }
    }
    if (p.whole()) {
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = ty * RPT + i;
        if (r < rows && tok[i] < p.n) {
          const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const float x[4] = {o[i][e * 4] * inv, o[i][e * 4 + 1] * inv, o[i][e * 4 + 2] * inv, o[i][e * 4 + 3] * inv};
            put_out<float>(a, p.b, p.kv, row0 + r, tx * 4 + 64 * e, x);
          }
        }
      }
    } else {
      float* rec = tree_record(a, blockIdx.x, p);
#pragma unroll
      for (int i = 0; i < RPT; ++i) {
        const int r = ty * RPT + i;
        if (r < rows) {
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            const float x[4] = {o[i][e * 4], o[i][e * 4 + 1], o[i][e * 4 + 2], o[i][e * 4 + 3]};
            store4(rec + ((size_t)(tx + 16 * e) * a.rec_rows + r) * 4, x);
          }
          if (tx == 0) reinterpret_cast<float2*>(rec + (size_t)a.rec_rows * D)[r] = make_float2(m[i], l[i]);
        }
      }
    }
  }
}

template <int D, int RPT>
cudaError_t launch_simt(const TreeArgs& a, int ctas, cudaStream_t s) {
  constexpr int RT = RPT * 16, KEYS = kTreeSimtKeys;
  constexpr int fixed = (RT * (D + 4) + KEYS * (D + 4) + KEYS * D + KEYS) * 4 + SELKV_MAX_TREE * 16;
  if (const cudaError_t e = set_smem_once<tree_simt_kernel<D, RPT>>(fixed + tree_list_bytes(SELKV_MAX_BATCH)); e != cudaSuccess) return e;
  return launch_chained(true, tree_simt_kernel<D, RPT>, dim3((unsigned)ctas), dim3(kThreads), (size_t)(fixed + tree_list_bytes(a.B)), s, a);
}

// ---- joining the pieces of a unit ----------------------------------------------------------
// Eight rows of a unit a CTA; a thread four elements of one.  Units that one CTA finished have nothing to join.  Bound
// by latency (7 to 9 us by itself, less behind the kernel in front): the pieces' references and sums come in one round, and the
// first outputs with them.  Joined by the last CTA of a unit instead, it took as long and the others waited.
constexpr int kJoinRows = 8, kJoinAhead = 8;
template <typename T, int D>
__global__ __launch_bounds__(kJoinRows * D / 4) void tree_join_kernel(TreeArgs a, int unit_rows) {
  constexpr int kMost = 2 * kPlanSMs;  // CTAs, and so pieces of a unit
  __shared__ float2 ml[kMost][kJoinRows];
  chain_begin();
  const int per = (unit_rows + kJoinRows - 1) / kJoinRows;
  const int blk = blockIdx.x / per, lr = threadIdx.x % kJoinRows, r = (blockIdx.x - blk * per) * kJoinRows + lr;
  const int d4 = threadIdx.x / kJoinRows, kv = blockIdx.y, b = blockIdx.z;
  const int lo = a.before[b], share = a.before[a.B + 1], mine = (a.before[b + 1] - lo) / (a.Hkv * a.blocks);
  if (mine == 0) return;
  // the CTAs that hold the unit's pieces
  const int u0 = lo + (kv * a.blocks + blk) * mine;
  const bool piece = a.before[a.B + 2] != 0;
  const int c0 = piece ? u0 : u0 / share, c1 = piece ? u0 + mine - 1 : (u0 + mine - 1) / share;
  const int S = c1 - c0 + 1;
  if (S == 1) return;
  const size_t rec = tree_record_floats(a.rec_rows, D);
  // the first piece lies in its CTA's second record, the others in their CTAs' first
  auto record = [&](int t) { return a.partial + (size_t)((c0 + t) * 2 + (t == 0 ? 1 : 0)) * rec; };
  const int row = blk * unit_rows + r, n = min(a.counts != nullptr ? a.counts[b] : a.T, a.T);
  const bool on = r < unit_rows && row < a.R && row % a.T < n;
  auto out_of = [&](int t) {
    return on && t < S ? __ldcg(reinterpret_cast<const float4*>(record(t)) + (size_t)d4 * a.rec_rows + r) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  float4 v[kJoinAhead];
#pragma unroll
  for (int k = 0; k < kJoinAhead; ++k) v[k] = out_of(k);
  for (int t = d4; t < S; t += D / 4)
    ml[t][lr] = on ? __ldcg(reinterpret_cast<const float2*>(record(t) + (size_t)a.rec_rows * D) + r) : make_float2(-INFINITY, 0.f);
  __syncthreads();
  float M = -INFINITY;
  for (int t = 0; t < S; ++t) M = fmaxf(M, ml[t][lr].x);
  const float ref = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int t0 = 0; t0 < S; t0 += kJoinAhead) {
#pragma unroll
    for (int k = 0; k < kJoinAhead; ++k) {
      if (t0 + k < S) {
        const float2 e = ml[t0 + k][lr];
        const float w = exp2f(e.x - ref);  // (a piece without weight has outputs 0)
        L = fmaf(e.y, w, L);
        x[0] = fmaf(v[k].x, w, x[0]);
        x[1] = fmaf(v[k].y, w, x[1]);
        x[2] = fmaf(v[k].z, w, x[2]);
        x[3] = fmaf(v[k].w, w, x[3]);
      }
      v[k] = out_of(t0 + kJoinAhead + k);
    }
  }
  if (!on) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  put_out<T>(a, b, kv, row, d4 * 4, x);
}

template <typename T, int D>
cudaError_t launch_join(const TreeArgs& a, cudaStream_t s) {
  const int unit_rows = tree_block_rows(a.dtype, a.R);
  const int used = a.blocks > 1 ? unit_rows : a.R;
  const dim3 grid((unsigned)(((used + kJoinRows - 1) / kJoinRows) * a.blocks), (unsigned)a.Hkv, (unsigned)a.B);
  return launch_chained(true, tree_join_kernel<T, D>, grid, dim3(kJoinRows * D / 4), 0, s, a, used);
}

}  // namespace

int tree_ctas(int dtype) { return dtype == SELKV_BF16 ? kPlanSMs : 2 * kPlanSMs; }

cudaError_t launch_tree_attn(const TreeArgs& a, cudaStream_t s) {
  const int ctas = tree_ctas(a.dtype);
  cudaError_t e;
  if (a.dtype == SELKV_BF16) {
    e = launch_tree_tc(a, ctas, s);
    if (e != cudaSuccess) return e;
    return a.D == 128 ? launch_join<__nv_bfloat16, 128>(a, s) : launch_join<__nv_bfloat16, 64>(a, s);
  }
  if (a.R <= 16)
    e = a.D == 128 ? launch_simt<128, 1>(a, ctas, s) : launch_simt<64, 1>(a, ctas, s);
  else
    e = a.D == 128 ? launch_simt<128, 4>(a, ctas, s) : launch_simt<64, 4>(a, ctas, s);
  if (e != cudaSuccess) return e;
  return a.D == 128 ? launch_join<float, 128>(a, s) : launch_join<float, 64>(a, s);
}

}  // namespace selkv
