// Compensated attention of a tree of drafted tokens over a bf16 cache, on the 5th-generation tensor cores.
//
// The R = G T query rows of a KV head are the 128 rows of an accumulator (two accumulators above 128), so the
// cache is read once for all of them.  Per key tile: S = Q K^T into tensor memory, the softmax warps read a row
// each (a thread a row: no exchange for the maximum), write P = 2^(s - ref) back over S as bf16, and O += P V takes P
// from there.  V lies in shared memory as it came, keys by d, and is the MN-major operand.
//
// Two such chains run side by side, each with its S, P and O, so the tensor cores work on one while the other is in its
// softmax: with up to 128 rows they take every other key tile of a piece and are joined at its end, above it they take
// 128 rows each of the same tiles.  The reference is a running maximum that moves only when a tile's maximum
// passes it by more than 8 (a factor of 256, far inside the range of bf16 and fp32): O is rescaled in those tiles alone.
//
// Arithmetic per byte is 4 R d / (4 d) = R operations: with up to 256 rows the cache's bytes bound it (281 a byte at the
// measured peaks).  All CTAs have equal shares of the list of key tiles (tree.cuh).
#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kKeys = kTreeTcKeys;
constexpr int kSoftWarps = 8, kProducerWarp = 8, kMmaWarp = 9, kThreads = 384;
constexpr int kBox = 32;       // rows of a copy
// Registers: a softmax thread holds a row of 128 logits.  384 threads start with 168 each; the two softmax warpgroups take
// 216 of them and the third keeps 72 (together what the launch had).
constexpr int kSoftRegs = 216, kIssueRegs = 72;
static_assert(2 * kSoftRegs + kIssueRegs == 3 * 168, "the launch's registers");
constexpr int kTmemCols = 512;
constexpr float kSlack = 8.f;  // how far a maximum may pass the reference, in powers of two

template <int D, int MT>
struct Cfg {
  static constexpr int kHalves = D / 64;           // 128-byte wide halves of a row
  static constexpr int kSlot = kKeys * D * 2;      // a tile of K or V
  static constexpr int kQ = 128 * MT * D * 2;
  static constexpr int kSlots = D == 128 ? (MT == 1 ? 5 : 4) : 8;
  // barriers | bias of a tile, a copy a warp | (reference, sum) of the chains' rows | ancestors | parents | unfit tokens
  static constexpr int kBars = 0, kBias = 256, kMl = kBias + kSoftWarps * kKeys * 4, kSeen = kMl + 2 * 128 * 8,
                       kUp = kSeen + SELKV_MAX_TREE * 16, kBad = kUp + SELKV_MAX_TREE, kBefore = kBad + 16;
  static constexpr int kFixed = 1024 + kQ + kSlots * kSlot + kBefore;
  static_assert(kFixed + (SELKV_MAX_BATCH + 1) * 4 <= 232448, "227 KB of shared memory");
  static_assert((2 * kSlots + 9) * 8 + 8 <= 256, "barriers and flags");
};

// D (fp32, tensor memory) += A (bf16 pairs, tensor memory) * B (shared memory).
__device__ __forceinline__ void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// Descriptor of an MN-major operand written by TMA with 128-byte swizzling: rows of 64 elements of N, 8 rows of K an
// atom of 1024 bytes; `next_n` bytes to the next 64 elements of N.
__device__ __forceinline__ uint64_t umma_desc_mn_sw128(uint32_t addr, uint32_t next_n) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(next_n >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kBMnMajor = 1u << 16;

__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, float (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, "
      "%14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]),
        "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]),
        "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr)
      : "memory");
}
// (names the registers, so that no use of them can be scheduled before it)
__device__ __forceinline__ void tmem_wait_ld32(float (&v)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                 "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
                 "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                 "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
          taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&f)[32]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t u[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) u[i] = __float_as_uint(f[h * 16 + i]);
    tmem_st16(taddr + h * 16, u);
  }
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Place in the ring (a count over the piece's copies) of K and V of tile i of n: one chain of tiles behind the other
// has the next tile's K before this one's V.
template <int MT>
__device__ __forceinline__ int k_place(int i) { return MT == 1 ? (i == 0 ? 0 : 2 * i - 1) : 2 * i; }
template <int MT>
__device__ __forceinline__ int v_place(int i, int n) { return MT == 1 ? (i == n - 1 ? 2 * n - 1 : 2 * i + 2) : 2 * i + 1; }

__device__ __forceinline__ bool unfit16(uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u; }

template <int D, int MT>
__global__ __launch_bounds__(kThreads, 1) void tree_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                              const __grid_constant__ CUtensorMap tmK,
                                                              const __grid_constant__ CUtensorMap tmV,
                                                              const __grid_constant__ CUtensorMap tmKn,
                                                              const __grid_constant__ CUtensorMap tmVn, TreeArgs a) {
  using C = Cfg<D, MT>;
  constexpr int kSlots = C::kSlots;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* Qs = smem;              // [halves][128 MT rows][128 B]
  unsigned char* ring = Qs + C::kQ;      // [slots][halves][128 keys][128 B]
  unsigned char* misc = ring + kSlots * C::kSlot;
  uint64_t* full = reinterpret_cast<uint64_t*>(misc + C::kBars);
  uint64_t* empty = full + kSlots;
  uint64_t* sfull = empty + kSlots;  // [2] S of a chain is there
  uint64_t* pfull = sfull + 2;       // [2] its P is
  uint64_t* ofull = pfull + 2;       // [2] its O of the piece is done
  uint64_t* qfull = ofull + 2;
  uint64_t* qfree = qfull + 1;
  uint64_t* done = qfree + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* bias_s = reinterpret_cast<float*>(misc + C::kBias);
  float2* ml_s = reinterpret_cast<float2*>(misc + C::kMl);
  uint4* seen = reinterpret_cast<uint4*>(misc + C::kSeen);
  int8_t* up = reinterpret_cast<int8_t*>(misc + C::kUp);
  uint32_t* bad = reinterpret_cast<uint32_t*>(misc + C::kBad);
  int32_t* before = reinterpret_cast<int32_t*>(misc + C::kBefore);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_launch_dependents();
  if (threadIdx.x == kProducerWarp * 32) {
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[i], 4);
      mbar_init(&ofull[i], 1);
    }
    mbar_init(qfull, 1);
    mbar_init(qfree, 1);
    mbar_init(done, 1);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tensormap(&tmQ);
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
    prefetch_tensormap(&tmKn);
    prefetch_tensormap(&tmVn);
  }
  __syncwarp();
  if (warp == kMmaWarp) tmem_alloc(tmem_slot, kTmemCols);
  tree_list<kKeys>(a, before, blockIdx.x == 0);
  const int total = before[a.B], share = tree_share(total, gridDim.x);
  if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b <= a.B; b += kThreads) a.before[b] = before[b];
    if (threadIdx.x == 0) a.before[a.B + 1] = share;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int pos0 = (int)min((long long)total, (long long)blockIdx.x * share), end = min(total, pos0 + share);

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kIssueRegs));
  if (warp == kProducerWarp) {
    if (lane == 0) {
      int used = 0, pieces = 0;  // copies into the ring, pieces
      bool ok = true;
      for (int pos = pos0; ok && pos < end; ++pieces) {
        const TreePiece p = tree_piece<kKeys>(a, before, pos, end);
        pos += p.count;
        const int bk = p.b * a.Hkv + p.kv, cache_tiles = (p.L + kKeys - 1) / kKeys;
        // K (or V) of the piece's tile i
        auto load = [&](bool v, int i) -> bool {
          const int t = p.first + i, slot = used % kSlots;
          const bool drafts = t >= cache_tiles;
          const int keys = drafts ? p.n : min(kKeys, p.L - t * kKeys), boxes = (keys + kBox - 1) / kBox;
          const int row = drafts ? bk * a.T : bk * a.m_cap + t * kKeys;
          const CUtensorMap* map = drafts ? (v ? &tmVn : &tmKn) : (v ? &tmV : &tmK);
          if (used >= kSlots && (!mbar_wait(&empty[slot], ((used / kSlots) & 1) ^ 1) || *abort_flag)) return false;
          mbar_arrive_expect_tx(&full[slot], (uint32_t)boxes * kBox * D * 2);
          for (int h = 0; h < C::kHalves; ++h)
            for (int x = 0; x < boxes; ++x)
              tma_load_2d(ring + slot * C::kSlot + h * (kKeys * 128) + x * (kBox * 128), map, h * 64, row + x * kBox, &full[slot]);
          ++used;
          return true;
        };
        ok = load(false, 0);
        if (ok && pieces > 0) ok = mbar_wait(qfree, (pieces - 1) & 1) && !*abort_flag;
        if (!ok) break;
        {
          const int row0 = p.blk * 128 * MT, boxes = (min(128 * MT, a.R - row0) + kBox - 1) / kBox;
          const int row = (p.b * a.Hq + p.kv * a.G) * a.T + row0;
          mbar_arrive_expect_tx(qfull, (uint32_t)boxes * kBox * D * 2);
          for (int h = 0; h < C::kHalves; ++h)
            for (int x = 0; x < boxes; ++x)
              tma_load_2d(Qs + h * (128 * MT * 128) + x * (kBox * 128), &tmQ, h * 64, row + x * kBox, qfull);
        }
        if (MT == 1) {
          for (int i = 1; ok && i < p.count; ++i) ok = load(false, i) && load(true, i - 1);
          ok = ok && load(true, p.count - 1);
        } else {
          ok = load(true, 0);
          for (int i = 1; ok && i < p.count; ++i) ok = load(false, i) && load(true, i);
        }
      }
      if (!ok) {
        *abort_flag = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      // no copy of this CTA is in flight when it ends
      for (int t = max(0, used - kSlots); t < used; ++t) mbar_wait(&full[t % kSlots], (t / kSlots) & 1);
      if (!ok && pieces > 0) mbar_wait(qfull, (pieces - 1) & 1);
    }
  } else if (warp == kMmaWarp) {
    if (lane == 0 && pos0 < end) {
      bool ok = true;
      const uint32_t qbase = smem_u32(Qs), rbase = smem_u32(ring);
      int base = 0, pieces = 0;  // ring places before the piece, pieces
      int cnt[2] = {0, 0};       // tiles of each chain
      for (int pos = pos0; ok && pos < end; ++pieces) {
        const TreePiece p = tree_piece<kKeys>(a, before, pos, end);
        pos += p.count;
        const int n = p.count, cache_tiles = (p.L + kKeys - 1) / kKeys;
        const bool two = MT == 2 && a.R - p.blk * 256 > 128;  // (rows for the second accumulator)
        auto cols = [&](int i) {
          const int t = p.first + i, keys = t >= cache_tiles ? p.n : min(kKeys, p.L - t * kKeys);
          return (keys + 31) / 32 * 32;
        };
        auto wait_slot = [&](int place) {
          const int u = base + place;
          ok = ok && mbar_wait(&full[u % kSlots], (u / kSlots) & 1) && !*abort_flag;
          return rbase + (uint32_t)(u % kSlots) * C::kSlot;
        };
        auto release = [&](int place) { umma_commit(&empty[(base + place) % kSlots]); };
        auto qk = [&](int i, int c, uint32_t kaddr) {
          const uint32_t idesc = umma_idesc_bf16(128, cols(i));
          tc_fence_after();
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t qoff = (ks >> 2) * (128 * MT * 128) + (ks & 3) * 32 + (MT == 2 ? c * 128 * 128 : 0);
            const uint32_t koff = (ks >> 2) * (kKeys * 128) + (ks & 3) * 32;
            umma_bf16(tmem + c * 128, umma_desc_sw128(qbase + qoff), umma_desc_sw128(kaddr + koff), idesc, ks > 0);
          }
          umma_commit(&sfull[c]);
        };
        auto pv = [&](int i, int c, uint32_t vaddr, bool first, bool last) {
          ok = ok && mbar_wait(&pfull[c], cnt[c] & 1) && !*abort_flag;
          if (!ok) return;
          ++cnt[c];
          const uint32_t idesc = umma_idesc_bf16(128, D) | kBMnMajor;
          const int steps = cols(i) / 16;
          tc_fence_after();
          for (int ks = 0; ks < steps; ++ks)
            umma_bf16_ta(tmem + 256 + c * 128, tmem + c * 128 + ks * 8, umma_desc_mn_sw128(vaddr + ks * 2048, kKeys * 128), idesc,
                         !first || ks > 0);
          if (last) umma_commit(&ofull[c]);
        };
        ok = mbar_wait(qfull, pieces & 1) && !*abort_flag;
        if (MT == 1) {
          for (int i = 0; ok && i <= n; ++i) {
            if (i < n) {
              const uint32_t k = wait_slot(k_place<MT>(i));
              if (!ok) break;
              qk(i, i & 1, k);
              release(k_place<MT>(i));
              if (i == n - 1) umma_commit(qfree);
            }
            if (i > 0) {
              const uint32_t v = wait_slot(v_place<MT>(i - 1, n));
              if (!ok) break;
              pv(i - 1, (i - 1) & 1, v, i <= 2, i - 1 >= n - 2);
              if (!ok) break;
              release(v_place<MT>(i - 1, n));
            }
          }
        } else if (ok) {
          uint32_t k = wait_slot(k_place<MT>(0));
          if (ok) {
            qk(0, 0, k);
            if (two) qk(0, 1, k);
            release(k_place<MT>(0));
            if (n == 1) umma_commit(qfree);
          }
          for (int i = 0; ok && i < n; ++i) {
            const uint32_t v = wait_slot(v_place<MT>(i, n));
            if (!ok) break;
            for (int c = 0; ok && c < (two ? 2 : 1); ++c) {
              pv(i, c, v, i == 0, i == n - 1);
              if (!ok) break;
              const bool last = c == (two ? 1 : 0);
              if (last) release(v_place<MT>(i, n));
              if (i + 1 < n) {
                if (c == 0) k = wait_slot(k_place<MT>(i + 1));
                if (!ok) break;
                qk(i + 1, c, k);
                if (last) {
                  release(k_place<MT>(i + 1));
                  if (i + 1 == n - 1) umma_commit(qfree);
                }
              }
            }
          }
        }
        base += 2 * n;
      }
      if (!ok) {
        *abort_flag = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      umma_commit(done);  // every MMA issued above has completed once this arrives
      mbar_wait(done, 0);
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---------------- softmax: chain c, lane quarter w4 of tensor memory ----------------
    const int c = warp >> 2, w4 = warp & 3;
    const uint32_t tl = tmem + ((uint32_t)(w4 * 32) << 16);
    const uint32_t ts = tl + c * 128;
    float* bw = bias_s + warp * kKeys;
    const float sc = a.scale_log2;
    const uint64_t sc2 = pack_f2(sc, sc);
    auto warp_wait = [&](uint64_t* bar, uint32_t parity) -> bool {
      int ok = 0;
      if (lane == 0) {
        ok = !*abort_flag && mbar_wait(bar, parity);
        if (!ok && !*abort_flag) {
          *abort_flag = 1;
          raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
        }
      }
      return __shfl_sync(0xffffffffu, ok, 0) != 0;
    };
    int base = 0;
    int cnt = 0;              // tiles of this chain
    int oc[2] = {0, 0};       // pieces that each chain had tiles of
    for (int pos = pos0; pos < end;) {
      const TreePiece p = tree_piece<kKeys>(a, before, pos, end);
      pos += p.count;
      const int n = p.count, cache_tiles = (p.L + kKeys - 1) / kKeys;
      const int row0 = p.blk * 128 * MT, rows = min(128 * MT, a.R - row0);
      const int r = (MT == 2 ? c * 128 : 0) + w4 * 32 + lane;  // this thread's row of the block
      const bool chain_on = MT == 1 || c * 128 < rows;
      const bool warp_on = (MT == 2 ? c * 128 : 0) + w4 * 32 < rows;
      const int tok = (row0 + r) % a.T;
      const size_t bk = (size_t)p.b * a.Hkv + p.kv;
      const bool has_drafts = p.first + n > cache_tiles;
      if (has_drafts) {
        named_bar_sync(1, 256);  // the last piece's sets are read
        if (threadIdx.x < 4) bad[threadIdx.x] = 0u;
        tree_ancestors<256>(a, p.b, p.n, seen, up, threadIdx.x, 1);
      }
      const float* bias = a.bias != nullptr ? a.bias + bk * a.m_cap : nullptr;
      float ref = -INFINITY, sum = 0.f;
      bool fresh = true;  // no tile of the chain yet
      const int i0 = MT == 1 ? c : 0, step = MT == 1 ? 2 : 1;
      float bnext[4];
      auto fetch_bias = [&](int i) {
        const int t = p.first + i;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int key = t * kKeys + k * 32 + lane;
          bnext[k] = i < n && t < cache_tiles && key < p.L ? (bias != nullptr ? bias[key] * kLog2e : 0.f) : -INFINITY;
        }
      };
      if (chain_on) fetch_bias(i0);
      for (int i = i0; chain_on && i < n; i += step) {
        const int t = p.first + i;
        const bool drafts = t >= cache_tiles;
        const int keys = drafts ? p.n : min(kKeys, p.L - t * kKeys), cols = (keys + 31) / 32 * 32;
        // the tile's bias, and keys that are out (behind the last one, or with a bias of -inf)
        bool out = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) out = out || bnext[k] == -INFINITY;
        const bool plain = !drafts && !__any_sync(0xffffffffu, out);
        const int key_here = w4 * 32 + lane;
        bool gone = drafts ? key_here >= keys : false;
        if (!drafts) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            bw[k * 32 + lane] = bnext[k];
            if (k == w4) gone = bnext[k] == -INFINITY;
          }
        }
        __syncwarp();
        fetch_bias(i + step);
        if (!plain && (MT == 1 || c == 0) && w4 * 32 < cols) {
          // rows of V that have no weight become zeros, and so do elements of drafted tokens' rows that are no
          // numbers (0 times an infinity is none): the epilogue gives those to the tokens that see them
          const int u = base + v_place<MT>(i, n), slot = u % kSlots;
          if (warp_wait(&full[slot], (u / kSlots) & 1)) {
            uint4* v = reinterpret_cast<uint4*>(ring + slot * C::kSlot + key_here * 128);
            if (gone) {
#pragma unroll
              for (int h = 0; h < C::kHalves; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[h * (kKeys * 8) + e] = make_uint4(0u, 0u, 0u, 0u);
            } else if (drafts) {
              bool any = false;
              for (int e = 0; e < C::kHalves * 8; ++e) {
                uint4 x = v[(e >> 3) * (kKeys * 8) + (e & 7)];
                uint32_t w[4] = {x.x, x.y, x.z, x.w};
                bool hit = false;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  if (unfit16(w[k])) {
                    w[k] &= 0xffff0000u;
                    hit = true;
                  }
                  if (unfit16(w[k] >> 16)) {
                    w[k] &= 0x0000ffffu;
                    hit = true;
                  }
                }
                if (hit) v[(e >> 3) * (kKeys * 8) + (e & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
                any = any || hit;
              }
              if (any) atomicOr(&bad[key_here >> 5], 1u << (key_here & 31));
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
        }
        const bool ok = warp_wait(&sfull[c], cnt & 1);
        ++cnt;
        tc_fence_after();
        if (ok && warp_on) {
          float x[4][32];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q * 32 < cols) tmem_ld32_issue(ts + q * 32, x[q]);
          float mx = -INFINITY;
          if (plain) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              tmem_wait_ld32(x[q]);
              const uint32_t ba = smem_u32(bw + q * 32);
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 b4 = lds_f4(ba + e * 4);
                unpack_f2(ffma2(pack_f2(x[q][e], x[q][e + 1]), sc2, pack_f2(b4.x, b4.y)), x[q][e], x[q][e + 1]);
                unpack_f2(ffma2(pack_f2(x[q][e + 2], x[q][e + 3]), sc2, pack_f2(b4.z, b4.w)), x[q][e + 2], x[q][e + 3]);
              }
              mx = fmaxf(mx, max32(x[q]));
            }
          } else {
            const uint4 sees = drafts ? seen[tok] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if (q * 32 < cols) {
                tmem_wait_ld32(x[q]);
                const uint32_t w = q == 0 ? sees.x : q == 1 ? sees.y : q == 2 ? sees.z : sees.w;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const float b = drafts ? ((w >> e) & 1u ? 0.f : -INFINITY) : bw[q * 32 + e];
                  x[q][e] = b == -INFINITY ? -INFINITY : fmaf(x[q][e], sc, b);
                }
                mx = fmaxf(mx, max32(x[q]));
              }
            }
          }
          const bool move = fresh ? true : mx > ref + kSlack;
          if (!fresh && __any_sync(0xffffffffu, move)) {
            // (the chain's O is done: this tile's S came behind it)
            const float f = move ? ex2_approx(ref - mx) : 1.f;
            sum *= f;
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
              float o[32];
              tmem_ld32_issue(tl + 256 + c * 128 + d, o);
              tmem_wait_ld32(o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= f;
              tmem_st32(tl + 256 + c * 128 + d, o);
            }
          }
          if (move) ref = mx;
          fresh = false;
          const float neg = ref == -INFINITY ? 0.f : -ref;
          const uint64_t neg2 = pack_f2(neg, neg);
          uint64_t s01 = pack_f2(0.f, 0.f), s23 = s01;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (q * 32 < cols) {
              uint32_t w[16];
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                float y0, y1, y2, y3;
                unpack_f2(fadd2(pack_f2(x[q][e], x[q][e + 1]), neg2), y0, y1);
                unpack_f2(fadd2(pack_f2(x[q][e + 2], x[q][e + 3]), neg2), y2, y3);
                y0 = ex2_approx(y0);
                y1 = ex2_approx(y1);
                y2 = ex2_approx(y2);
                y3 = ex2_approx(y3);
                s01 = fadd2(s01, pack_f2(y0, y1));
                s23 = fadd2(s23, pack_f2(y2, y3));
                w[e / 2] = pack_bf16(y0, y1);
                w[e / 2 + 1] = pack_bf16(y2, y3);
              }
              tmem_st16(ts + q * 16, w);
            }
          }
          float a0, a1, a2, a3;
          unpack_f2(s01, a0, a1);
          unpack_f2(s23, a2, a3);
          sum += (a0 + a1) + (a2 + a3);
          tmem_wait_st();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[c]);
      }
      base += 2 * n;

      // ---------------- the piece's rows ----------------
      bool ok = true;
      float f[2] = {c == 0 ? 1.f : 0.f, c == 0 ? 0.f : 1.f};
      bool use[2] = {MT == 1 || c == 0, MT == 1 ? n > 1 : c == 1};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (!use[k] || !chain_on) continue;
        ok = warp_wait(&ofull[k], oc[k] & 1) && ok;
        ++oc[k];
      }
      tc_fence_after();
      if (warp_on) {
        if (MT == 1) {
          ml_s[c * 128 + r] = make_float2(ref, sum);
          named_bar_sync(2 + w4, 64);
          const float2 other = ml_s[(c ^ 1) * 128 + r];
          const float top = fmaxf(ref, other.x), base2 = top == -INFINITY ? 0.f : top;
          const float mine = ex2_approx(ref - base2), its = ex2_approx(other.x - base2);
          f[c] = mine;
          f[c ^ 1] = its;
          sum = sum * mine + other.y * its;
          ref = top;
        }
        const int d0 = MT == 1 ? c * (D / 2) : 0, d1 = MT == 1 ? d0 + D / 2 : D;
        const bool whole = p.whole();
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint32_t unfit[4] = {0u, 0u, 0u, 0u};
        bool any_unfit = false;
        if (has_drafts && (bad[0] | bad[1] | bad[2] | bad[3]) != 0u) {
          const uint4 sees = seen[tok];
          unfit[0] = sees.x & bad[0];
          unfit[1] = sees.y & bad[1];
          unfit[2] = sees.z & bad[2];
          unfit[3] = sees.w & bad[3];
          any_unfit = (unfit[0] | unfit[1] | unfit[2] | unfit[3]) != 0u && tok < p.n;
        }
        float* rec = whole ? nullptr : tree_record(a, blockIdx.x, p);
        __nv_bfloat16* orow = static_cast<__nv_bfloat16*>(a.out) + (((size_t)p.b * a.Hq + p.kv * a.G) * a.T + row0 + r) * D;
        const bool write = ok && r < rows && tok < p.n;
#pragma unroll 1
        for (int d = d0; d < d1; d += 32) {
          float o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0.f;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if (!use[k]) continue;
            float y[32];
            tmem_ld32_issue(tl + 256 + k * 128 + d, y);
            tmem_wait_ld32(y);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(y[e], f[k], o[e]);
          }
          if (any_unfit) {
            for (int u = 0; u < p.n; ++u)
              if ((unfit[u >> 5] >> (u & 31)) & 1u) {
                const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v_new) + (bk * a.T + u) * D + d;
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                  const float y = __bfloat162float(v[e]);
                  if (!(fabsf(y) < INFINITY)) o[e] += y;
                }
              }
          }
          if (!write) continue;
          if (whole) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
              uint4 w;
              w.x = pack_bf16(o[e] * inv, o[e + 1] * inv);
              w.y = pack_bf16(o[e + 2] * inv, o[e + 3] * inv);
              w.z = pack_bf16(o[e + 4] * inv, o[e + 5] * inv);
              w.w = pack_bf16(o[e + 6] * inv, o[e + 7] * inv);
              *reinterpret_cast<uint4*>(orow + d + e) = w;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              reinterpret_cast<float4*>(rec)[(size_t)((d + e) / 4) * a.rec_rows + r] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (write && !whole && (MT == 2 || c == 0)) reinterpret_cast<float2*>(rec + (size_t)a.rec_rows * D)[r] = make_float2(ref, sum);
        tc_fence_before();
        if (MT == 1) named_bar_sync(2 + w4, 64);  // both chains' O and sums are read
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

template <int D, int MT>
cudaError_t launch(const TreeArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<D, MT>;
  CUtensorMap q, k, v, kn, vn;
  const uint64_t bk = (uint64_t)a.B * a.Hkv;
  if (!encode_rows_bf16(&q, a.q, (uint64_t)a.B * a.Hq * a.T, D, kBox) || !encode_rows_bf16(&k, a.Kc, bk * a.m_cap, D, kBox) ||
      !encode_rows_bf16(&v, a.Vc, bk * a.m_cap, D, kBox) || !encode_rows_bf16(&kn, a.k_new, bk * a.T, D, kBox) ||
      !encode_rows_bf16(&vn, a.v_new, bk * a.T, D, kBox))
    return cudaErrorInvalidValue;
  constexpr int most = C::kFixed + (SELKV_MAX_BATCH + 1) * 4;
  if (const cudaError_t e = set_smem_once<tree_tc_kernel<D, MT>>(most); e != cudaSuccess) return e;
  tree_tc_kernel<D, MT><<<ctas, kThreads, C::kFixed + (a.B + 1) * 4, s>>>(q, k, v, kn, vn, a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_tree_tc(const TreeArgs& a, int ctas, cudaStream_t s) {
  if (a.R <= 128) return a.D == 128 ? launch<128, 1>(a, ctas, s) : launch<64, 1>(a, ctas, s);
  return a.D == 128 ? launch<128, 2>(a, ctas, s) : launch<64, 2>(a, ctas, s);
}

}  // namespace selkv
