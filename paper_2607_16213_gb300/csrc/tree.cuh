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
  int32_t* before;  // [B + 3] the list (TreeList::before and head)
  float* partial;   // [CTA][2] records of tree_record_floats
};

// A partial record: outputs relative to the row's reference [D / 4][rows] of four, then (reference in base 2,
// sum) [rows].  Rows side by side: the lanes of a warp hold a row each.
__host__ __device__ constexpr size_t tree_record_floats(int rows, int D) { return (size_t)rows * (D + 2); }

// Fewest tiles of a piece where a unit is cut: below it a partial's way through memory costs more than the tiles do (bf16, 1000 rows
// x 8 heads, 8 tokens: 1 tile 13.5 us, 2 12.4, 4 12.8; fp32, 2 heads, d 64, 7 tokens, where a tile takes longer: 2 x 1000 rows 1 tile
// 13.5, 2 16.8, 4 24.2; 2 x 101-201 rows 11.1, 15.2, 20.3; 16000 rows 37.8, 37.8, 41.2).
constexpr int kTreeTcMinTiles = 2, kTreeSimtMinTiles = 1;
// What ending one piece and beginning another costs a CTA, in tiles (bf16, 4 x 5000 rows x 8 heads, 8 tokens: 6 or 12 25.6 us, 0
// 27.5).
constexpr int kTreePieceTiles = 6;

// The work is the list of all units (sequence, KV head, row block) and their key tiles: those of the cached rows,
// then those of the tokens' own.  Each CTA finds its part from the lengths, in one of two ways.
//   Equal shares: the tiles of all units in a row, `share` consecutive ones a CTA, so that ragged lengths leave
//   none idle; a CTA may end one unit and begin another.
//   A piece a CTA: a unit of t tiles is cut into ceil(t / share) even pieces, with the smallest share that leaves no more
//   pieces than CTAs.  Taken where there are no more units than CTAs and that share is at most kTreePieceTiles more, what a
//   second piece costs (one sequence of 25000 rows, 8 KV heads, 152 CTAs: a CTA with two pieces took 36 us, the others 25).
// In shared memory: the CTA's first piece, the sequences' (cached rows, tokens), and the pieces or tiles of the sequences
// before each.
struct TreePiece {
  int b, kv, blk;
  int L, n;          // cached rows, tokens
  int tiles;         // key tiles of the unit
  int first, count;  // tiles first .. first + count - 1 of it
  int left;          // places of the CTA's part of the list from here on, this piece's among them
  __device__ __forceinline__ bool whole() const { return count == tiles; }
};
struct TreeList {
  TreePiece* first;
  int2* seq;        // [B]
  int32_t* before;  // [B + 1]
  int32_t* head;    // [2] share, 1: a piece a CTA
};
__host__ __device__ constexpr int tree_list_bytes(int B) { return 40 + B * 12 + 12; }
__device__ __forceinline__ TreeList tree_list_at(void* smem, int B) {  // 8-byte aligned
  static_assert(sizeof(TreePiece) <= 40, "the piece comes first");
  int2* seq = reinterpret_cast<int2*>(static_cast<char*>(smem) + 40);
  int32_t* before = reinterpret_cast<int32_t*>(seq + B);
  return {static_cast<TreePiece*>(smem), seq, before, before + B + 1};
}
template <int KEYS>
__device__ __forceinline__ int tree_tiles(int2 seq) {
  return seq.y > 0 ? (seq.x + KEYS - 1) / KEYS + (seq.y + KEYS - 1) / KEYS : 0;
}
// A warp's running sum of `before`'s entries 1 .. B, in place.
__device__ __forceinline__ void tree_prefix(int32_t* before, int B) {
  const int lane = threadIdx.x & 31;
  int sum = 0;
  for (int b0 = 0; b0 < B; b0 += 32) {
    const int b = b0 + lane;
    int x = b < B ? before[b + 1] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += y;
    }
    if (b < B) before[b + 1] = sum + x;
    sum += __shfl_sync(0xffffffffu, x, 31);
  }
}
// All threads of the CTA come here.  (The first CTA reports lengths and counts out of range.)
template <int KEYS, int MIN>
__device__ __forceinline__ void tree_list(const TreeArgs& a, const TreeList& w, int cta, int ctas) {
  const int per = a.Hkv * a.blocks;  // units of a sequence
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    int L = a.lengths[b], n = a.counts != nullptr ? a.counts[b] : a.T;
    if (L < 0 || L > a.m_cap || n < 0 || n > a.T) {
      if (cta == 0) raise_flag(a.flags, SELKV_DEVERR_LENGTH);
      L = min(max(L, 0), a.m_cap);
      n = min(max(n, 0), a.T);
    }
    w.seq[b] = make_int2(L, n);
    w.before[b + 1] = tree_tiles<KEYS>(make_int2(L, n)) * per;
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int units = 0, total = 0;
    for (int b = lane; b < a.B; b += 32) {
      const int t = w.before[b + 1];
      units += t > 0 ? per : 0;
      total += t;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      units += __shfl_xor_sync(0xffffffffu, units, o);
      total += __shfl_xor_sync(0xffffffffu, total, o);
    }
    int share = max(MIN, (total + ctas - 1) / ctas);
    bool piece = false;
    if (units <= ctas) {
      // (a candidate a lane)
      const int mine = share + min(lane, kTreePieceTiles);
      int pieces = 0;
      for (int b = 0; b < a.B; ++b) pieces += (tree_tiles<KEYS>(w.seq[b]) + mine - 1) / mine * per;
      const uint32_t fits = __ballot_sync(0xffffffffu, pieces <= ctas);
      if (fits != 0) {
        piece = true;
        share += __ffs(fits) - 1;
        for (int b = lane; b < a.B; b += 32) w.before[b + 1] = (tree_tiles<KEYS>(w.seq[b]) + share - 1) / share * per;
      }
    }
    if (lane == 0) {
      w.before[0] = 0;
      w.head[0] = share;
      w.head[1] = piece;
    }
    __syncwarp();
    tree_prefix(w.before, a.B);
    __syncwarp();
    // the CTA's part of the list, and its first piece
    const int places = w.before[a.B];
    const int pos = piece ? min(cta, places) : (int)min((long long)places, (long long)cta * share);
    const int end = piece ? min(cta + 1, places) : min(places, pos + share);
    int b = 0;  // before[b] <= pos < before[b + 1]
    for (int b0 = 0; b0 < a.B; b0 += 32) b += __popc(__ballot_sync(0xffffffffu, b0 + lane < a.B && w.before[b0 + lane + 1] <= pos));
    if (lane == 0) {
      TreePiece p{};
      p.left = end - pos;
      if (p.left > 0) {
        const int2 q = w.seq[b];
        p.b = b;
        p.L = q.x;
        p.n = q.y;
        p.tiles = tree_tiles<KEYS>(q);
        const int at = pos - w.before[b], pieces = piece ? (p.tiles + share - 1) / share : p.tiles, unit = at / pieces;
        const int j = at - unit * pieces;
        if (piece) {
          const int each = p.tiles / pieces, more = p.tiles - each * pieces;  // `more` pieces have one more
          p.first = j * each + min(j, more);
          p.count = each + (j < more ? 1 : 0);
        } else {
          p.first = j;
          p.count = min(p.tiles - j, p.left);
        }
        p.kv = unit / a.blocks;
        p.blk = unit - p.kv * a.blocks;
      }
      *w.first = p;
    }
  }
  __syncthreads();
}
// The piece behind `p`: the next unit's first tiles (a CTA with a single place has no other piece).
template <int KEYS>
__device__ __forceinline__ void tree_next(const TreeArgs& a, const TreeList& w, TreePiece& p) {
  p.left -= w.head[1] ? 1 : p.count;
  if (p.left <= 0) return;
  if (++p.blk == a.blocks) {
    p.blk = 0;
    if (++p.kv == a.Hkv) {
      p.kv = 0;
      do ++p.b;
      while (w.before[p.b + 1] == w.before[p.b]);  // (the list goes on)
      const int2 s = w.seq[p.b];
      p.L = s.x;
      p.n = s.y;
      p.tiles = tree_tiles<KEYS>(s);
    }
  }
  p.first = 0;
  p.count = min(p.tiles, p.left);
}
// The list for the kernel that joins (by one CTA).
__device__ __forceinline__ void tree_list_store(const TreeArgs& a, const TreeList& w) {
  for (int b = threadIdx.x; b < a.B + 3; b += blockDim.x) a.before[b] = w.before[b];  // (head lies behind)
}

__device__ __forceinline__ float* tree_record(const TreeArgs& a, int cta, const TreePiece& p) {
  return a.partial + (size_t)(cta * 2 + (p.first > 0 ? 0 : 1)) * tree_record_floats(a.rec_rows, a.D);
}

// The warp's: ancestors of each token of sequence b and the token itself, as bits, into `seen`, by paths of doubling length.
__device__ __forceinline__ void tree_ancestors(const TreeArgs& a, int b, int n, uint4* seen, int8_t* up) {
  constexpr int kPer = SELKV_MAX_TREE / 32;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = lane + 32 * k;
    int p = -1;
    if (i < n) {
      p = a.parents != nullptr ? a.parents[(size_t)b * a.T + i] : i - 1;
      if (p < -1 || p >= i) {
        raise_flag(a.flags, SELKV_DEVERR_TREE);
        p = -1;
      }
    }
    up[i] = (int8_t)p;
    const uint32_t bit = 1u << lane;
    seen[i] = make_uint4(k == 0 ? bit : 0u, k == 1 ? bit : 0u, k == 2 ? bit : 0u, k == 3 ? bit : 0u);
  }
  __syncwarp();
  for (int reach = 1; reach < n; reach <<= 1) {
    int far[kPer];
    uint4 s[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      const int i = lane + 32 * k, p = i < n ? up[i] : -1;
      s[k] = seen[i];
      far[k] = -1;
      if (p >= 0) {
        const uint4 t = seen[p];
        s[k] = make_uint4(s[k].x | t.x, s[k].y | t.y, s[k].z | t.z, s[k].w | t.w);
        far[k] = up[p];
      }
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      seen[lane + 32 * k] = s[k];
      up[lane + 32 * k] = (int8_t)far[k];
    }
    __syncwarp();
  }
}

constexpr int kTreeTcKeys = 64, kTreeSimtKeys = 64;  // keys of a tile
// Rows of a block.  Tensor cores: two accumulators of 128 rows where one does not hold them.  CUDA cores: 16 where they hold all (14
// rows, 2 heads, d 64: blocks of 16 over 2 x 101-201 cached rows 11.1 us, of 64 14.9; 2 x 1000: 13.5 and 17.8; 16000: 37.8 and
// 50.3; 2 x 16000: 51.7 and 73.8).
inline int tree_block_rows(int dtype, int R) {
  if (dtype == SELKV_BF16) return R <= 128 ? 128 : 256;
  return R <= 16 ? 16 : 64;
}
int tree_ctas(int dtype);  // CTAs of a launch
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

constexpr int kMaxVocab = 1 << 20;  // (the sums of a CTA's spans have places in shared memory for that many)
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
