// The accepted path of a tree into the caches of a model's layers (selkv_tree_commit).
//
// A copy of a few rows a sequence, KV head and layer: bound by latency, so all layers go in one launch.  The lengths
// move in a second kernel: a decode that follows may come up while the call's last kernel still runs and load rows below the
// lengths that it finds, so the rows are complete before the lengths move.  32 layers x 8 heads: 5 us for the rows, 4 for the
// lengths.
#include "tree.cuh"

namespace selkv {
namespace {

constexpr int kThreads = 128;

// What sequence b takes in a layer whose length is `len`: `rows` of it to row `at` (none where they do not fit).
struct Take {
  int at, rows;
  uint32_t flags;
};
__device__ __forceinline__ Take take_of(const CommitArgs& a, int len, int acc, bool bad_path) {
  uint32_t f = 0;
  if (len < 0 || len > a.m_cap || acc < 0 || acc > a.T) f |= SELKV_DEVERR_LENGTH;
  len = min(max(len, 0), a.m_cap);
  acc = min(max(acc, 0), a.T);
  if (bad_path) return {len, 0, f | SELKV_DEVERR_TREE};
  if (acc > a.m_cap - len) return {len, 0, f | SELKV_DEVERR_CAPACITY};
  return {len, acc, f};
}

__global__ __launch_bounds__(kThreads) void commit_rows_kernel(const __grid_constant__ CommitLayers layers, CommitArgs a) {
  const int kv = blockIdx.x, b = blockIdx.y, l = blockIdx.z, tid = threadIdx.x;
  __shared__ int path[SELKV_MAX_TREE];
  pdl_launch_dependents();  // (the lengths' kernel waits for this one's end)
  const int acc = a.accepted[b], len = layers.lengths[l][b];
  int entry = 0;
  if (tid < a.T) {
    entry = a.path[(size_t)b * a.T + tid];
    path[tid] = entry;
  }
  const bool bad = __syncthreads_or(tid < min(acc, a.T) && (entry < 0 || entry >= a.T));
  const Take t = take_of(a, len, acc, bad);
  const size_t bk = (size_t)b * a.Hkv + kv;
  const int per = a.row_bytes / 16;
  const uint4* ks = static_cast<const uint4*>(layers.k_new[l]) + bk * a.T * per;
  const uint4* vs = static_cast<const uint4*>(layers.v_new[l]) + bk * a.T * per;
  uint4* kd = static_cast<uint4*>(layers.K[l]) + (bk * a.m_cap + t.at) * per;
  uint4* vd = static_cast<uint4*>(layers.V[l]) + (bk * a.m_cap + t.at) * per;
  for (int i = tid; i < t.rows * per; i += kThreads) {
    const int r = i / per, e = i - r * per;
    const size_t from = (size_t)path[r] * per + e;
    const uint4 k = ks[from], v = vs[from];
    kd[i] = k;
    vd[i] = v;
  }
  if (layers.bias[l] != nullptr && tid < t.rows) layers.bias[l][bk * a.m_cap + t.at + tid] = 0.f;
}

// A warp a sequence, a lane a layer.
__global__ __launch_bounds__(kThreads) void commit_lengths_kernel(const __grid_constant__ CommitLayers layers, CommitArgs a) {
  const int b = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  pdl_wait();
  if (b >= a.B) return;
  const int acc = a.accepted[b];
  bool bad = false;
  for (int i = lane; i < min(acc, a.T); i += 32) {
    const int e = a.path[(size_t)b * a.T + i];
    bad = bad || e < 0 || e >= a.T;
  }
  bad = __any_sync(0xffffffffu, bad);
  for (int l = lane; l < a.layers; l += 32) {
    const Take t = take_of(a, layers.lengths[l][b], acc, bad);
    if (t.rows > 0) layers.lengths[l][b] = t.at + t.rows;
    if (t.flags != 0) raise_flag(a.flags, t.flags);
  }
}

}  // namespace

cudaError_t launch_tree_commit(const CommitArgs& a, const CommitLayers& layers, cudaStream_t s) {
  static_assert(kThreads >= SELKV_MAX_TREE, "a thread an entry of the path");
  const dim3 grid((unsigned)a.Hkv, (unsigned)a.B, (unsigned)a.layers);
  commit_rows_kernel<<<grid, kThreads, 0, s>>>(layers, a);
  if (const cudaError_t e = cudaGetLastError(); e != cudaSuccess) return e;
  return launch_chained(true, commit_lengths_kernel, dim3((unsigned)((a.B + kThreads / 32 - 1) / (kThreads / 32))), dim3(kThreads), 0, s,
                        layers, a);
}

}  // namespace selkv
