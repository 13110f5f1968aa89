// A tree of drafted tokens over a cache: arguments, the walk over key tiles that both attention kernels
// share, and the ancestor sets.
#pragma once

#include "ptx.cuh"
#include "selkv_internal.cuh"

namespace selkv {

struct TreeArgs {
  int dtype, B, Hq, Hkv, G, D, m_cap, T;
  int R;         // query rows of a KV head: G * T, row g * T + t
  int blocks;    // row blocks of a KV head
  int rec_rows;  // rows of a partial record
  float scale_log2;
  const void* q;
  const void* Kc;
  const void* Vc;
  const float* bias;
  const int32_t* lengths;
  const void* k_new;
  const void* v_new;
  const int32_t* parents;
  const int32_t* counts;
  void* out;
  uint32_t* flags;
  int32_t* before;  // [B + 1] key tiles of the sequences before b, and of all; then tiles a CTA takes
  float* partial;   // [CTA][2] records of tree_record_floats
};

// A partial record: outputs relative to the row's reference [D / 4][rows] of four, then (reference in base 2,
// sum) [rows].  Rows side by side: the lanes of a warp hold a row each.
__host__ __device__ constexpr size_t tree_record_floats(int rows, int D) { return (size_t)rows * (D + 2); }

// Fewest tiles a CTA takes of a call (below it a partial's way through memory costs more than the tiles).
constexpr int kTreeMinTiles = 2;

// What a sequence has: cached rows, tokens, and its key tiles (the tokens' own rows are one more), 0 without tokens.
struct TreeSeq {
  int L, n, tiles;
};
template <int KEYS>
__device__ __forceinline__ TreeSeq tree_seq(const TreeArgs& a, int b, bool tell) {
  int L = a.lengths[b], n = a.counts != nullptr ? a.counts[b] : a.T;
  if (L < 0 || L > a.m_cap || n < 0 || n > a.T) {
    if (tell) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
    L = min(max(L, 0), a.m_cap);
    n = min(max(n, 0), a.T);
  }
  return {L, n, n > 0 ? (L + KEYS - 1) / KEYS + (n + KEYS - 1) / KEYS : 0};
}

// The list of all (sequence, KV head, row block, key tile) in that order is cut into equal shares, one a
// CTA.  `before` [B + 1] in shared memory: entries of the list before each sequence.  All threads come here.
template <int KEYS>
__device__ __forceinline__ void tree_list(const TreeArgs& a, int32_t* before, bool tell) {
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) before[b + 1] = tree_seq<KEYS>(a, b, tell).tiles * a.Hkv * a.blocks;
  if (threadIdx.x == 0) before[0] = 0;
  __syncthreads();
  if (threadIdx.x < 32) {
    int sum = 0;
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int b = b0 + threadIdx.x;
      int x = b < a.B ? before[b + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if ((int)threadIdx.x >= o) x += y;
      }
      if (b < a.B) before[b + 1] = sum + x;
      sum += __shfl_sync(0xffffffffu, x, 31);
    }
  }
  __syncthreads();
}
__device__ __forceinline__ int tree_share(int total, int ctas) { return max(kTreeMinTiles, (total + ctas - 1) / ctas); }

// One piece of a CTA's share: tiles of one (sequence, KV head, row block).
struct TreePiece {
  int b, kv, blk;
  int L, n;      // cached rows, tokens
  int tiles;     // key tiles of the unit
  int first, count;
  __device__ __forceinline__ bool whole() const { return count == tiles; }
};
template <int KEYS>
__device__ __forceinline__ TreePiece tree_piece(const TreeArgs& a, const int32_t* before, int pos, int end) {
  int lo = 0, hi = a.B;  // before[lo] <= pos < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (before[mid] <= pos) lo = mid;
    else hi = mid;
  }
  const TreeSeq s = tree_seq<KEYS>(a, lo, false);
  const int at = pos - before[lo], unit = at / s.tiles;
  TreePiece p;
  p.b = lo;
  p.kv = unit / a.blocks;
  p.blk = unit - p.kv * a.blocks;
  p.L = s.L;
  p.n = s.n;
  p.tiles = s.tiles;
  p.first = at - unit * s.tiles;
  p.count = min(s.tiles - p.first, end - pos);
  return p;
}
__device__ __forceinline__ float* tree_record(const TreeArgs& a, int cta, const TreePiece& p) {
  return a.partial + (size_t)(cta * 2 + (p.first > 0 ? 0 : 1)) * tree_record_floats(a.rec_rows, a.D);
}

// Ancestors of each token of sequence b and the token itself, as bits, into `seen`; by paths of doubling length.
// Called by threads 0 .. kN - 1 of a barrier `bar` over them (kN >= SELKV_MAX_TREE).
template <int kN>
__device__ __forceinline__ void tree_ancestors(const TreeArgs& a, int b, int n, uint4* seen, int8_t* up, int i, int bar) {
  if (i < SELKV_MAX_TREE) {
    int p = -1;
    if (i < n) {
      p = a.parents != nullptr ? a.parents[(size_t)b * a.T + i] : i - 1;
      if (p < -1 || p >= i) {
        raise_flag(a.flags, SELKV_DEVERR_TREE);
        p = -1;
      }
    }
    up[i] = (int8_t)p;
    const uint32_t bit = 1u << (i & 31);
    seen[i] = make_uint4(i < 32 ? bit : 0u, (i >> 5) == 1 ? bit : 0u, (i >> 5) == 2 ? bit : 0u, (i >> 5) == 3 ? bit : 0u);
  }
  named_bar_sync(bar, kN);
  for (int reach = 1; reach < n; reach <<= 1) {
    int p = -1, far = -1;
    uint4 s = make_uint4(0u, 0u, 0u, 0u);
    if (i < n) {
      p = up[i];
      if (p >= 0) {
        s = seen[p];
        far = up[p];
      }
    }
    named_bar_sync(bar, kN);
    if (p >= 0) {
      seen[i] = make_uint4(seen[i].x | s.x, seen[i].y | s.y, seen[i].z | s.z, seen[i].w | s.w);
      up[i] = (int8_t)far;
    }
    named_bar_sync(bar, kN);
  }
}

constexpr int kTreeTcKeys = 128, kTreeSimtKeys = 64;  // keys of a tile
// Rows of a block (tensor cores: two accumulators of 128 rows where one does not hold them).
inline int tree_block_rows(int dtype, int R) {
  if (dtype == SELKV_BF16) return R <= 128 ? 128 : 256;
  return R <= 16 ? 16 : 64;
}
int tree_ctas(int dtype, int D, int R);  // CTAs of a launch
cudaError_t launch_tree_attn(const TreeArgs& a, cudaStream_t s);
cudaError_t launch_tree_tc(const TreeArgs& a, int ctas, cudaStream_t s);

// ---- the other steps ----------------------------------------------------------------------
struct RotaryArgs {
  int dtype, B, Hq, Hkv, D, T;
  int rot, layout;
  float amplitude, sign;
  const int32_t* positions;
  const void* q;
  const void* k;
  void* q_out;
  void* k_out;
  uint64_t turns[SELKV_ROTARY_MAX_DIM / 2];
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t s);

struct VerifyArgs {
  int B, T, V;
  const int32_t* parents;
  const int32_t* counts;
  const int32_t* tokens;
  const float* uniforms;
  const float* target;
  const float* draft;
  int32_t* accepted;
  int32_t* path;
  int32_t* next;
  uint32_t* flags;
};
cudaError_t launch_tree_verify(const VerifyArgs& a, cudaStream_t s);

struct CommitLayers {
  const void* k_new[kMaxLayers];
  const void* v_new[kMaxLayers];
  void* K[kMaxLayers];
  void* V[kMaxLayers];
  float* bias[kMaxLayers];
  int32_t* lengths[kMaxLayers];
};
struct CommitArgs {
  int B, Hkv, T, m_cap, layers;
  int row_bytes;
  const int32_t* path;
  const int32_t* accepted;
  uint32_t* flags;
};
cudaError_t launch_tree_commit(const CommitArgs& a, const CommitLayers& layers, cudaStream_t s);

}  // namespace selkv
