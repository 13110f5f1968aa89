// Compensated attention of a tree of drafted tokens over a bf16 cache, on the 5th-generation tensor cores.
//
// The R = G T query rows of a KV head are the 128 rows of an accumulator (two accumulators above 128), so the
// cache is read once for all of them.  Per tile of 64 keys: S = Q K^T into tensor memory, the softmax warps read a row
// each (a thread a row: no exchange for the maximum), write P = 2^(s - ref) back over S as bf16, and O += P V takes P
// from there.  V lies in shared memory as it came, keys by d, and is the MN-major operand.
//
// Two such chains run side by side, each with its O and two places for S and P, so that a chain's next S is there when
// its softmax ends: with up to 128 rows they take every other key tile of a piece and are joined at its end, above it
// they take 128 rows each of the same tiles.  The reference is a running maximum that moves only when a tile's maximum
// passes it by more than 8 (a factor of 256, far inside the range of bf16 and fp32): O is rescaled in those tiles alone.
//
// Arithmetic per byte is 4 R d / (4 d) = R operations: with up to 256 rows the cache's bytes bound it (281 a byte at the
// measured peaks).  A CTA takes a piece of a unit, or an equal share of the list of all key tiles (tree.cuh).
//
// A pass with the join, 8 KV heads, d 128: 25000 rows and 4 tokens (16 rows a head) 28.7 us, 32 tokens 30.7 (floor 15.2:
// start, list and the first copies take 4 us, the end and the join 6); 8 x 8192-16384 rows, 25 tokens 73.9 (55); 131072 rows, 64
// tokens 128 (79: the chain from S over the softmax to P V takes 2100 cycles a tile of 64 keys, its copies 1400); 64 x
// 410-819 rows, 9 tokens 72 (25: a CTA goes through 3.4 units, and what is run once a unit, masks, the rows' end, the next
// piece's start, waits for its instructions).
#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kKeys = kTreeTcKeys;
constexpr int kSoftWarps = 8, kProducerWarp = 8, kMmaWarp = 9, kTreeWarp = 11, kThreads = 384;  // (an MMA warp a chain)
constexpr int kBox = 32;       // rows of a copy where a tile is not whole
constexpr int kTmemCols = 512;
// A reference is at least this: rows with the lowest number for a bias, or none at all, have weight 0 beside a token's own
// logit, and the reference's product with log2 e stays a number.
constexpr float kLowest = -1e37f;
constexpr float kSlack = 8.f;  // how far a maximum may pass the reference (powers of two, or of e)

template <int D, int MT>
struct Cfg {
  static constexpr int kHalves = D / 64;           // 128-byte wide halves of a row
  static constexpr int kSlot = kKeys * D * 2;      // a tile of K or V
  static constexpr int kQ = 128 * MT * D * 2;
  // Q of the next piece is fetched behind this one's rows where there is room for it (a copy waits for some us behind those
  // under way)
  static constexpr int kQs = MT == 1 ? 2 : 1;
  // Rings of K and V tiles: one for each set of tiles that is consumed in order (a chain's own, or what both take), so that
  // every wait for a copy comes after the one for the last copy in its place: a phase later would read as done.
  static constexpr int kRings = MT == 1 ? 2 : 1;
  static constexpr int kRing = (D == 128 ? 8 : 16) / kRings;  // places of a ring
  static_assert(kRing >= 4, "V of a tile comes at most 3 places behind its K");
  static constexpr int kSlots = kRings * kRing;
  // barriers | bias of a tile, a copy a warp | sums and references of the chains' rows | ancestors, parents and unfit
  // tokens, twice | the list
  static constexpr int kBars = 0, kBias = 512, kSum = kBias + kSoftWarps * kKeys * 4, kSeen = kSum + 2 * 128 * 8,
                       kUp = kSeen + 2 * SELKV_MAX_TREE * 16, kBad = kUp + SELKV_MAX_TREE, kList = kBad + 2 * 16;
  static constexpr int kFixed = 1024 + kQs * kQ + kSlots * kSlot + kList;
  static_assert(kFixed + tree_list_bytes(SELKV_MAX_BATCH) <= 232448, "227 KB of shared memory");
  static_assert((2 * kSlots + 22) * 8 + 8 <= 512, "barriers and flags");
};
// Shared-memory matrix descriptors, 128-byte swizzling, 8 rows of 128 bytes an atom: the upper word is the same for
// all operands here; the lower one holds the address and, for the MN-major V, the distance to the next 64 elements of N.
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t next_n = 16) { return addr >> 4 | (next_n >> 4) << 16; }
constexpr uint32_t kBMnMajor = 1u << 16;

// The MMA warp runs as one and its elected lane issues: operands stay uniform (with the loops in one thread an
// instruction took about 120 cycles to issue, twice what it runs).
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t l;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(l));
  return l;
}
// D (fp32, tensor memory) (+)= A B with A and B in shared memory, and with A (bf16 pairs) in tensor memory.
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, l;\n .reg .b64 da, db;\n setp.ne.b32 l, %5, 0;\n setp.ne.b32 p, %4, 0;\n mov.b64 da, {%1, %6};\n"
      " mov.b64 db, {%2, %6};\n @l tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}\n" ::"r"(d),
      "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(leader), "n"(kDescHi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p, l;\n .reg .b64 db;\n setp.ne.b32 l, %5, 0;\n setp.ne.b32 p, %4, 0;\n mov.b64 db, {%2, %6};\n"
      " @l tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}\n" ::"r"(d),
      "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "r"(leader), "n"(kDescHi)
      : "memory");
}
__device__ __forceinline__ void commit_to(uint32_t leader, uint64_t* bar) {
  asm volatile(
      "{\n .reg .pred l;\n setp.ne.b32 l, %1, 0;\n"
      " @l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(smem_u32(bar)),
      "r"(leader)
      : "memory");
}

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
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Place in the ring (a count over the piece's copies) of K and V of the ring's tile i of n: the first two K, then a V and
// the next K in turn.
constexpr int kAhead = 2;
__device__ __forceinline__ int k_place(int i) { return i + max(0, i - kAhead + 1); }
__device__ __forceinline__ int v_place(int i, int n) { return i + min(i + kAhead, n); }
// Tiles of a piece of n that chain c takes (MT 1: every other one).
template <int MT>
__device__ __forceinline__ int chain_tiles(int n, int c) { return MT == 1 ? (n + 1 - c) >> 1 : n; }

// The bf16 of a pair that are no numbers, as ones (an exponent of ones carries into the sign's place).
__device__ __forceinline__ uint32_t unfit2(uint32_t pair) { return ((((pair & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15) * 0xffffu; }

template <int D, int MT>
__global__ __launch_bounds__(kThreads, 1) void tree_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                              const __grid_constant__ CUtensorMap tmK,
                                                              const __grid_constant__ CUtensorMap tmV,
                                                              const __grid_constant__ CUtensorMap tmK32,
                                                              const __grid_constant__ CUtensorMap tmV32,
                                                              const __grid_constant__ CUtensorMap tmKn,
                                                              const __grid_constant__ CUtensorMap tmVn, TreeArgs a) {
  using C = Cfg<D, MT>;
  constexpr int kRing = C::kRing;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem =
      reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  unsigned char* Qs = smem;              // [kQs][halves][128 MT rows][128 B]
  unsigned char* ring = Qs + C::kQs * C::kQ;      // [rings][places][halves][keys][128 B]
  unsigned char* misc = ring + C::kSlots * C::kSlot;
  uint64_t* full = reinterpret_cast<uint64_t*>(misc + C::kBars);
  uint64_t* empty = full + C::kSlots;
  uint64_t* sfull = empty + C::kSlots;  // [chain][2] S is there
  uint64_t* pfull = sfull + 4;       // [chain][2] P is
  uint64_t* odone = pfull + 4;       // [chain] a tile's P V is in O
  uint64_t* ofull = odone + 2;       // [chain] its last one of a piece
  uint64_t* qfull = ofull + 2;       // [kQs]
  uint64_t* qfree = qfull + 2;
  uint64_t* done = qfree + 2;        // [chain]
  uint64_t* tfull = done + 2;        // [2] a piece's ancestors are there
  uint64_t* tfree = tfull + 2;       // [2] they are read
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tfree + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  float* bias_s = reinterpret_cast<float*>(misc + C::kBias);
  float2* sum_s = reinterpret_cast<float2*>(misc + C::kSum);  // [chain][128] (reference, sum)
  uint4* seen_s = reinterpret_cast<uint4*>(misc + C::kSeen);
  int8_t* up = reinterpret_cast<int8_t*>(misc + C::kUp);
  uint32_t* bad_s = reinterpret_cast<uint32_t*>(misc + C::kBad);
  const TreeList list = tree_list_at(misc + C::kList, a.B);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == kProducerWarp * 32) {
    for (int i = 0; i < C::kSlots; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], MT);  // (the chains that take a tile)
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[i], kSoftWarps / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&odone[i], 1);
      mbar_init(&ofull[i], 1);
      mbar_init(&tfull[i], 1);
      mbar_init(&done[i], 1);
      mbar_init(&qfull[i], 1);
      mbar_init(&qfree[i], 2);
      mbar_init(&tfree[i], kSoftWarps);
    }
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
  pdl_wait();  // (no early start for what follows: its CTAs, waiting, cost this kernel 4 us of 34)
  tree_list<kKeys, kTreeTcMinTiles>(a, list, blockIdx.x, gridDim.x);
  if (blockIdx.x == 0) tree_list_store(a, list);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == kProducerWarp) {
    if (lane == 0) {
      int used[2] = {0, 0}, pieces = 0;  // copies into the rings, pieces
      bool ok = true;
      int asked = 0;  // pieces whose Q is
      auto load_q = [&](const TreePiece& p) -> bool {
        const int k = asked % C::kQs;
        if (asked >= C::kQs && (!mbar_wait(&qfree[k], ((asked / C::kQs) & 1) ^ 1) || *abort_flag)) return false;
        const int row0 = p.blk * 128 * MT, boxes = (min(128 * MT, a.R - row0) + kBox - 1) / kBox;
        const int row = (p.b * a.Hq + p.kv * a.G) * a.T + row0;
        mbar_arrive_expect_tx(&qfull[k], (uint32_t)boxes * kBox * D * 2);
        for (int h = 0; h < C::kHalves; ++h)
          for (int x = 0; x < boxes; ++x)
            tma_load_2d(Qs + k * C::kQ + h * (128 * MT * 128) + x * (kBox * 128), &tmQ, h * 64, row + x * kBox, &qfull[k]);
        ++asked;
        return true;
      };
      for (TreePiece p = *list.first; ok && p.left > 0; ++pieces, tree_next<kKeys>(a, list, p)) {
        const int n = p.count, bk = p.b * a.Hkv + p.kv, cache_tiles = (p.L + kKeys - 1) / kKeys;
        // K (or V) of the piece's tile i
        auto load = [&](bool v, int i) -> bool {
          const int t = p.first + i;
          const bool drafts = t >= cache_tiles;
          const int key0 = (drafts ? t - cache_tiles : t) * kKeys, keys = min(kKeys, (drafts ? p.n : p.L) - key0);
          const int row = bk * (drafts ? a.T : a.m_cap) + key0, boxes = (keys + kBox - 1) / kBox;
          const int ri = C::kRings == 2 ? i & 1 : 0, u = used[ri], slot = ri * kRing + u % kRing;
          if (u >= kRing && (!mbar_wait(&empty[slot], ((u / kRing) & 1) ^ 1) || *abort_flag)) return false;
          mbar_arrive_expect_tx(&full[slot], (uint32_t)boxes * kBox * D * 2);
          unsigned char* to = ring + slot * C::kSlot;
          if (boxes == kKeys / kBox && !drafts) {
#pragma unroll
            for (int h = 0; h < C::kHalves; ++h) tma_load_2d(to + h * (kKeys * 128), v ? &tmV : &tmK, h * 64, row, &full[slot]);
          } else {
            const CUtensorMap* map = drafts ? (v ? &tmVn : &tmKn) : (v ? &tmV32 : &tmK32);
            for (int h = 0; h < C::kHalves; ++h)
              for (int x = 0; x < boxes; ++x)
                tma_load_2d(to + h * (kKeys * 128) + x * (kBox * 128), map, h * 64, row + x * kBox, &full[slot]);
          }
          ++used[ri];
          return true;
        };
        ok = load(false, 0);
        if (ok && asked == pieces) ok = load_q(p);
        constexpr int kFirst = kAhead * C::kRings;
        for (int i = 1; ok && i < min(kFirst, n); ++i) ok = load(false, i);
        for (int i = 0; ok && i < n; ++i) {
          ok = load(true, i);
          if (ok && i + kFirst < n) ok = load(false, i + kFirst);
        }
        if (C::kQs == 2 && ok) {
          TreePiece behind = p;
          tree_next<kKeys>(a, list, behind);
          if (behind.left > 0) ok = load_q(behind);
        }
      }
      if (!ok) {
        *abort_flag = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      // no copy of this CTA is in flight when it ends
      for (int ri = 0; ri < C::kRings; ++ri)
        for (int u = max(0, used[ri] - kRing); u < used[ri]; ++u) mbar_wait(&full[ri * kRing + u % kRing], (u / kRing) & 1);
      for (int q = max(0, asked - C::kQs); q < asked; ++q) mbar_wait(&qfull[q % C::kQs], (q / C::kQs) & 1);
    }
  } else if (warp == kMmaWarp || warp == kMmaWarp + 1) {
    // ---------------- matrix products of chain c ----------------
    if (list.first->left > 0) {
      const int c = warp - kMmaWarp;
      bool ok = true;
      const uint32_t leader = elect_one();
      const uint32_t q0 = desc_lo(smem_u32(Qs)) + (MT == 2 ? c * (128 * 128 >> 4) : 0), rbase = smem_u32(ring);
      const uint32_t o = tmem + 256 + c * 128;
      int base = 0, pieces = 0, cnt = 0;  // copies into the chain's ring before the piece; pieces; tiles of the chain whose P V is issued
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        ok = __all_sync(0xffffffffu, !*abort_flag && mbar_wait(bar, parity) && !*abort_flag);
        return ok;
      };
      for (TreePiece p = *list.first; ok && p.left > 0; ++pieces, tree_next<kKeys>(a, list, p)) {
        const int n = p.count, cache_tiles = (p.L + kKeys - 1) / kKeys;
        const bool on = MT == 1 || c == 0 || a.R - p.blk * 256 > 128;  // (rows for the second accumulator)
        auto cols = [&](int i) {
          const int t = p.first + i, keys = t >= cache_tiles ? p.n - (t - cache_tiles) * kKeys : p.L - t * kKeys;
          return (min(kKeys, keys) + 31) / 32 * 32;
        };
        const int qi = pieces % C::kQs;
        const uint32_t qbase = q0 + qi * (C::kQ >> 4);
        if (!wait(&qfull[qi], (pieces / C::kQs) & 1)) break;
        // round i: P V of the chain's tile i, whose P the softmax gives, and S of tile i + kAhead in its place; the rounds
        // before the first tile bring the first S's
        const int nc = chain_tiles<MT>(n, c);
        auto tile = [&](int i) { return MT == 1 ? 2 * i + c : i; };  // of the piece
        const int r0 = (C::kRings == 2 ? c : 0) * kRing;
        for (int i = -kAhead; i < nc; ++i) {
          if (i >= 0) {
            const int u = base + v_place(i, nc), slot = r0 + u % kRing;
            if (!wait(&full[slot], (u / kRing) & 1)) break;
            if (on) {
              const uint32_t s = (cnt & 1) * 64;
              if (!wait(&pfull[c * 2 + (cnt & 1)], (cnt >> 1) & 1)) break;
              const uint32_t idesc = umma_idesc_bf16(128, D) | kBMnMajor, v0 = desc_lo(rbase + slot * C::kSlot, kKeys * 128);
              const uint32_t p0 = tmem + c * 128 + s;
              const int steps = cols(tile(i)) / 16;
              tc_fence_after();
#pragma unroll
              for (int ks = 0; ks < kKeys / 16; ++ks)
                if (ks < steps) mma_ts(leader, o, p0 + ks * 8, v0 + ks * (2048 >> 4), idesc, ks > 0 ? 1u : (i == 0 ? 0u : 1u));
              ++cnt;
              commit_to(leader, &odone[c]);
              if (i + 1 == nc) commit_to(leader, &ofull[c]);
            }
            commit_to(leader, &empty[slot]);  // (a chain that is off has nothing under way)
          }
          const int k = i + kAhead;
          if (k < nc) {
            const int u = base + k_place(k), slot = r0 + u % kRing;
            if (!wait(&full[slot], (u / kRing) & 1)) break;
            if (on) {
              const int j = cnt + (i >= 0 ? 1 : k);  // the chain's tile, over all pieces
              const uint32_t idesc = umma_idesc_bf16(128, cols(tile(k))), k0 = desc_lo(rbase + slot * C::kSlot);
              const uint32_t d = tmem + c * 128 + (j & 1) * 64;
              tc_fence_after();
#pragma unroll
              for (int ks = 0; ks < D / 16; ++ks)
                mma_ss(leader, d, qbase + (((ks >> 2) * (128 * MT * 128) + (ks & 3) * 32) >> 4),
                       k0 + (((ks >> 2) * (kKeys * 128) + (ks & 3) * 32) >> 4), idesc, ks > 0);
              commit_to(leader, &sfull[c * 2 + (j & 1)]);
            }
            commit_to(leader, &empty[slot]);
          }
          if (i == nc - 1 - kAhead || (nc == 0 && i == -1)) commit_to(leader, &qfree[qi]);  // the last S that there is
        }
        base += 2 * nc;
      }
      if (!ok && leader) {
        *abort_flag = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      commit_to(leader, &done[c]);  // every MMA issued above has completed once this arrives
      mbar_wait(&done[c], 0);
      __syncwarp();
    }
  } else if (warp == kTreeWarp) {
    // ---------------- the ancestors, a piece ahead of the softmax ----------------
    int trees = 0;
    for (TreePiece p = *list.first; p.left > 0; tree_next<kKeys>(a, list, p)) {
      if (p.first + p.count <= (p.L + kKeys - 1) / kKeys) continue;
      const int k = trees & 1;
      if (trees >= 2 && (!__all_sync(0xffffffffu, mbar_wait(&tfree[k], ((trees >> 1) & 1) ^ 1) && !*abort_flag))) {
        if (lane == 0) {
          *abort_flag = 1;
          raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
        }
        break;
      }
      if (lane < 4) bad_s[k * 4 + lane] = 0u;
      tree_ancestors(a, p.b, p.n, seen_s + k * SELKV_MAX_TREE, up);
      if (lane == 0) mbar_arrive(&tfull[k]);
      ++trees;
    }
  } else if (warp < kSoftWarps) {
    // ---------------- softmax: chain c, lane quarter w4 of tensor memory ----------------
    const int c = warp >> 2, w4 = warp & 3;
    const uint32_t tl = tmem + ((uint32_t)(w4 * 32) << 16);
    float* bw = bias_s + warp * kKeys;
    // Without a bias the logits and the reference are in base 2, and the scale goes in with the reference.  With one they
    // are in base e, as the bias is, and their factor to base 2 goes in with the reference.
    const bool added = a.bias != nullptr;
    const float sc = added ? a.scale_log2 * kLn2 : a.scale_log2, to2 = added ? kLog2e : 1.f;
    const int rl = w4 * 32 + lane;         // this thread's row of the chain
    const int pair_bar = 1 + w4;           // of the two chains' warps for the same lanes
    // (the whole warp looks; one that has to give up takes the others along)
    auto warp_wait = [&](uint64_t* bar, uint32_t parity) -> bool {
      if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
      const bool ok = __all_sync(0xffffffffu, !*abort_flag && mbar_wait(bar, parity));
      if (!ok && lane == 0 && !*abort_flag) {
        *abort_flag = 1;
        raise_flag(a.flags, SELKV_DEVERR_TIMEOUT);
      }
      __syncwarp();
      return ok;
    };
    int base = 0;        // copies into the chain's ring before the piece
    int cnt = 0;         // tiles of the chain
    int oc[2] = {0, 0};  // pieces that each chain had tiles of
    int trees = 0;       // pieces with tokens' rows
    float bnext[2];      // bias of the chain's next tile; -inf: the key is out
    auto fetch_bias = [&](const TreePiece& p, int i) {
      if (!added) return;
      const int key0 = (p.first + i) * kKeys + lane;
      const float* bias = a.bias + ((size_t)p.b * a.Hkv + p.kv) * a.m_cap;
#pragma unroll
      for (int k = 0; k < 2; ++k) bnext[k] = i < p.count && key0 + k * 32 < p.L ? bias[key0 + k * 32] : -INFINITY;
    };
    const int i0 = MT == 1 ? c : 0, step = MT == 1 ? 2 : 1;
    if (list.first->left > 0) fetch_bias(*list.first, i0);
    for (TreePiece p = *list.first; p.left > 0; tree_next<kKeys>(a, list, p)) {
      // bias of the chain's tile behind tile i, be it the next piece's
      auto fetch_behind = [&](int i) {
        if (!added) return;
        if (i + step < p.count) {
          fetch_bias(p, i + step);
        } else {
          TreePiece behind = p;
          tree_next<kKeys>(a, list, behind);
          if (behind.left > 0) fetch_bias(behind, i0);
        }
      };
      const int n = p.count, cache_tiles = (p.L + kKeys - 1) / kKeys;
      const int row0 = p.blk * 128 * MT, rows = min(128 * MT, a.R - row0);
      const int r = (MT == 2 ? c * 128 : 0) + rl;  // this thread's row of the block
      const bool chain_on = MT == 1 || c * 128 < rows;
      const bool warp_on = (MT == 2 ? c * 128 : 0) + w4 * 32 < rows;
      const int tok = (row0 + r) % a.T;
      const bool has_drafts = p.first + n > cache_tiles;
      const uint4* seen = seen_s + (trees & 1) * SELKV_MAX_TREE;
      uint32_t* bad = bad_s + (trees & 1) * 4;
      float ref = -INFINITY, sum = 0.f;
      bool fresh = true;  // no tile of the chain yet
      for (int i = i0; chain_on && i < n; i += step) {
        const int t = p.first + i, j = cnt++;
        const bool drafts = t >= cache_tiles;
        const int key0 = (drafts ? t - cache_tiles : t) * kKeys, keys = min(kKeys, (drafts ? p.n : p.L) - key0);
        const int chunks = (keys + 31) >> 5;  // of 32 columns
        const uint32_t ts = tl + c * 128 + (j & 1) * 64;
        // no key is out (behind the last one, or with a bias of -inf)
        bool plain = !drafts && keys == kKeys;
        if (added) {
          plain = plain && !__any_sync(0xffffffffu, bnext[0] == -INFINITY || bnext[1] == -INFINITY);
          bw[lane] = drafts ? 0.f : bnext[0];
          bw[32 + lane] = drafts ? 0.f : bnext[1];
          fetch_behind(i);
          __syncwarp();
        }
        uint32_t live[2];  // where the tile is not plain: the columns that the row sees, as bits
        if (drafts) {
          warp_wait(&tfull[trees & 1], (trees >> 1) & 1);
          const uint2 sees = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint32_t*>(seen + tok) + (key0 >> 5));
          live[0] = sees.x;
          live[1] = sees.y;
        } else if (!plain) {
          live[0] = __ballot_sync(0xffffffffu, lane < keys && !(added && bw[lane] == -INFINITY));
          live[1] = __ballot_sync(0xffffffffu, 32 + lane < keys && !(added && bw[32 + lane] == -INFINITY));
        }
        bool ok = warp_wait(&sfull[c * 2 + (j & 1)], (j >> 1) & 1);
        tc_fence_after();
        auto void_rows = [&]() {
          // rows of V that have no weight become zeros, and so do elements of drafted tokens' rows that are no
          // numbers (0 times an infinity is none): the epilogue gives those to the tokens that see them.  (Where both
          // chains take the tile, both do so, with the same values.)  Behind the wait for S: the copy that had V's place
          // before is done.  Behind P, too: V comes later than K.
          const int u = base + v_place(MT == 1 ? i >> 1 : i, chain_tiles<MT>(n, c)), slot = (C::kRings == 2 ? c : 0) * kRing + u % kRing;
          ok = warp_wait(&full[slot], (u / kRing) & 1) && ok;
          const int key = w4 * 16 + (lane & 15);  // a row and, with two halves of d, one of them
          if (ok && key < chunks * 32 && (lane >> 4) < C::kHalves) {
            uint4* v = reinterpret_cast<uint4*>(ring + slot * C::kSlot + (lane >> 4) * (kKeys * 128) + key * 128);
            if (key >= keys || (added && !drafts && bw[key] == -INFINITY)) {
#pragma unroll
              for (int e = 0; e < 8; ++e) v[e ^ (lane & 7)] = make_uint4(0u, 0u, 0u, 0u);  // (the lanes' rows lie 128 bytes apart)
            } else if (drafts) {
              uint32_t hit = 0;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint4 w = v[e ^ (lane & 7)];
                hit |= unfit2(w.x) | unfit2(w.y) | unfit2(w.z) | unfit2(w.w);
              }
              if (hit != 0) {
                atomicOr(&bad[(key0 + key) >> 5], 1u << (key & 31));
                __threadfence_block();  // (the other chain may find the element gone)
#pragma unroll 1
                for (int e = 0; e < 8; ++e) {
                  const uint4 w = v[e];
                  v[e] = make_uint4(w.x & ~unfit2(w.x), w.y & ~unfit2(w.y), w.z & ~unfit2(w.z), w.w & ~unfit2(w.w));
                }
              }
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
        };
        if (MT == 2 && !plain) void_rows();
        if (ok && warp_on) {
          // the reference moves to `mx` where that passes it by more than the slack; returns what is added to the logits
          auto settle = [&](float mx) {
            mx = fmaxf(mx, kLowest);
            const bool move = fresh || mx > ref + kSlack;
            if (!fresh && __any_sync(0xffffffffu, move)) {
              warp_wait(&odone[c], (j - 1) & 1);  // the tile before is in O (this tile's S came behind the one before that)
              tc_fence_after();
              const float f = move ? ex2_approx((ref - mx) * to2) : 1.f;
              sum *= f;
#pragma unroll 1
              for (int d = 0; d < D; d += 16) {
                float o[16];
                tmem_ld16_issue(tl + 256 + c * 128 + d, o);
                tmem_wait_ld16(o);
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[e] * f);
                tmem_st16(tl + 256 + c * 128 + d, w);
              }
            }
            if (move) ref = mx;
            fresh = false;
            return -ref * to2;
          };
          float x[2][32];
#pragma unroll
          for (int q = 0; q < 2; ++q) tmem_ld32_issue(ts + q * 32, x[q]);
          float mx = -INFINITY;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            tmem_wait_ld32(x[q]);
            if (added) {
              const uint32_t ba = smem_u32(bw + q * 32);
              const uint64_t sc2 = pack_f2(sc, sc);
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 b4 = lds_f4(ba + e * 4);
                unpack_f2(ffma2(pack_f2(x[q][e], x[q][e + 1]), sc2, pack_f2(b4.x, b4.y)), x[q][e], x[q][e + 1]);
                unpack_f2(ffma2(pack_f2(x[q][e + 2], x[q][e + 3]), sc2, pack_f2(b4.z, b4.w)), x[q][e + 2], x[q][e + 3]);
              }
            }
            if (!plain) {  // (whatever S and the bias are there)
#pragma unroll
              for (int e = 0; e < 32; ++e) x[q][e] = (live[q] & (1u << e)) != 0u ? x[q][e] : -INFINITY;
            }
            mx = fmaxf(mx, max32(x[q]));
          }
          // (without a bias the scale, which is positive, goes in with the reference)
          const float neg = settle(added ? mx : mx * sc), by = added ? kLog2e : sc;
          const uint64_t neg2 = pack_f2(neg, neg), by2 = pack_f2(by, by);
          uint64_t s01 = pack_f2(0.f, 0.f), s23 = s01;
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              float y0, y1, y2, y3;
              unpack_f2(ffma2(pack_f2(x[q][e], x[q][e + 1]), by2, neg2), y0, y1);
              unpack_f2(ffma2(pack_f2(x[q][e + 2], x[q][e + 3]), by2, neg2), y2, y3);
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
          float a0, a1, a2, a3;
          unpack_f2(s01, a0, a1);
          unpack_f2(s23, a2, a3);
          sum += (a0 + a1) + (a2 + a3);
          tmem_wait_st();
        }
        if (MT == 1 && !plain) void_rows();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pfull[c * 2 + (j & 1)]);
      }
      if (!chain_on || i0 >= n) fetch_behind(n);
      base += 2 * chain_tiles<MT>(n, c);

      // ---------------- the piece's rows ----------------
      bool ok = true;
      const bool use[2] = {MT == 1 || c == 0, MT == 1 ? n > 1 : c == 1};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (!use[k] || !chain_on) continue;
        if (warp_on) ok = warp_wait(&ofull[k], oc[k] & 1) && ok;  // (others might come too late for the phase)
        ++oc[k];
      }
      if (has_drafts) ok = warp_wait(&tfull[trees & 1], (trees >> 1) & 1) && ok;
      tc_fence_after();
      if (warp_on) {
        float f[2] = {1.f, 1.f};
        ref *= to2;  // (as it was used)
        if (MT == 1) {  // the row's sum in both chains
          sum_s[c * 128 + rl] = make_float2(ref, sum);
          named_bar_sync(pair_bar, 64);
          const float2 s0 = sum_s[rl], s1 = sum_s[128 + rl];
          const float top = fmaxf(s0.x, s1.x);  // (a number: the first chain has a tile)
          f[0] = ex2_approx(s0.x - top);
          f[1] = ex2_approx(s1.x - top);
          sum = s0.y * f[0] + s1.y * f[1];
          ref = top;
        }
        constexpr int kCols = MT == 1 ? D / 2 : D;  // columns of O a warp takes
        const int d0 = MT == 1 ? c * kCols : 0;
        const bool whole = p.whole();
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        bool any_unfit = false;  // the row sees a token whose values are not all numbers
        if (has_drafts && tok < p.n) {
          const uint4 sees = seen[tok];
          any_unfit = ((sees.x & bad[0]) | (sees.y & bad[1]) | (sees.z & bad[2]) | (sees.w & bad[3])) != 0u;
        }
        float* rec = whole ? nullptr : tree_record(a, blockIdx.x, p);
        __nv_bfloat16* orow = static_cast<__nv_bfloat16*>(a.out) + (((size_t)p.b * a.Hq + p.kv * a.G) * a.T + row0 + r) * D;
        const bool write = ok && r < rows && tok < p.n;
        const size_t new_row = ((size_t)p.b * a.Hkv + p.kv) * a.T;
#pragma unroll 1
        for (int d = d0; d < d0 + kCols; d += 16) {
          float o[16];
          tmem_ld16_issue(tl + 256 + (MT == 2 ? c * 128 : 0) + d, o);
          tmem_wait_ld16(o);
          if (MT == 1) {
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] *= f[0];
            if (n > 1) {
              float y[16];
              tmem_ld16_issue(tl + 384 + d, y);
              tmem_wait_ld16(y);
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = fmaf(y[e], f[1], o[e]);
            }
          }
          if (any_unfit) {
#pragma unroll 1
            for (int u = 0; u < p.n; ++u)
              if ((reinterpret_cast<const uint32_t*>(seen + tok)[u >> 5] & bad[u >> 5]) >> (u & 31) & 1u) {
                const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v_new) + (new_row + u) * D + d;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  const float g = __bfloat162float(v[e]);
                  if (!(fabsf(g) < INFINITY)) o[e] += g;
                }
              }
          }
          if (write && whole) {
#pragma unroll
            for (int e = 0; e < 16; e += 8) {
              uint4 w;
              w.x = pack_bf16(o[e] * inv, o[e + 1] * inv);
              w.y = pack_bf16(o[e + 2] * inv, o[e + 3] * inv);
              w.z = pack_bf16(o[e + 4] * inv, o[e + 5] * inv);
              w.w = pack_bf16(o[e + 6] * inv, o[e + 7] * inv);
              *reinterpret_cast<uint4*>(orow + d + e) = w;
            }
          } else if (write) {
#pragma unroll
            for (int e = 0; e < 16; e += 4)
              reinterpret_cast<float4*>(rec)[(size_t)((d + e) / 4) * a.rec_rows + r] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
          __syncwarp();  // (rows that are written and rows that are not go on together: the next loads are the whole warp's)
        }
        if (write && !whole && d0 == 0) reinterpret_cast<float2*>(rec + (size_t)a.rec_rows * D)[r] = make_float2(ref, sum);
        tc_fence_before();
        __syncwarp();  // (the barrier is, too)
        if (MT == 1) named_bar_sync(pair_bar, 64);  // both chains' O, and the rows' sums, are read
      }
      if (has_drafts) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&tfree[trees & 1]);
        ++trees;
      }
    }
  }
  tc_fence_before();
  __syncwarp();
  __syncthreads();
  tc_fence_after();
  if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

template <int D, int MT>
cudaError_t launch(const TreeArgs& a, int ctas, cudaStream_t s) {
  using C = Cfg<D, MT>;
  CUtensorMap q, k, v, k32, v32, kn, vn;
  const uint64_t bk = (uint64_t)a.B * a.Hkv;
  if (!encode_rows_bf16(&q, a.q, (uint64_t)a.B * a.Hq * a.T, D, kBox) || !encode_rows_bf16(&k, a.Kc, bk * a.m_cap, D, kKeys) ||
      !encode_rows_bf16(&v, a.Vc, bk * a.m_cap, D, kKeys) || !encode_rows_bf16(&k32, a.Kc, bk * a.m_cap, D, kBox) ||
      !encode_rows_bf16(&v32, a.Vc, bk * a.m_cap, D, kBox) || !encode_rows_bf16(&kn, a.k_new, bk * a.T, D, kBox) ||
      !encode_rows_bf16(&vn, a.v_new, bk * a.T, D, kBox))
    return cudaErrorInvalidValue;
  if (const cudaError_t e = set_smem_once<tree_tc_kernel<D, MT>>(C::kFixed + tree_list_bytes(SELKV_MAX_BATCH)); e != cudaSuccess) return e;
  return launch_chained(true, tree_tc_kernel<D, MT>, dim3((unsigned)ctas), dim3(kThreads), C::kFixed + tree_list_bytes(a.B), s, q, k, v, k32, v32,
                        kn, vn, a);
}

}  // namespace

cudaError_t launch_tree_tc(const TreeArgs& a, int ctas, cudaStream_t s) {
  if (a.R <= 128) return a.D == 128 ? launch<128, 1>(a, ctas, s) : launch<64, 1>(a, ctas, s);
  return a.D == 128 ? launch<128, 2>(a, ctas, s) : launch<64, 2>(a, ctas, s);
}

}  // namespace selkv
