// The two ends of a tree step: visibility words and positions from the
// nodes' parents (mkv_tree_build) and the accepted path into the caches of
// all layers (mkv_tree_commit).  Both move kilobytes and are bounded by their
// launch and a few dependent reads: 4 x 64 nodes 1.8 us and 64 x 251 nodes 3.3 us;
// 36 layers of 4 x 8 heads 4.1 us, 8 layers of 32 x 8 heads 6.3 us.
#include "common.cuh"
#include "kernels.h"
#include "tree.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

// One CTA per batch item, one thread per node.  Pointer doubling: after round
// r a node's word set holds its 2^r nearest ancestors and `up` the next one
// above them, so 8 rounds reach the root of any tree of 256 nodes (a walk up
// the parents would take a round per level, 255 in a chain).
__global__ void __launch_bounds__(kTreeNodes) tree_build_kernel(const TreeBuildArgs a) {
  constexpr int kW = kTreeNodes / 32;
  __shared__ uint32_t bits[kW][kTreeNodes];
  __shared__ int16_t up[kTreeNodes];
  const int b = blockIdx.x, i = threadIdx.x, W = tree_words(a.N);
  grid_dependency_wait();
  grid_launch_dependents();
  int n = a.count != nullptr ? a.count[b] : a.N;
  if (n < 0 || n > a.N) {
    if (i == 0) record_error(a.ws, MKV_ERR_INVALID_ARG, b);
    n = n < 0 ? 0 : a.N;
  }
  int p = -1;
  if (i < n) {
    p = a.parents[(size_t)b * a.N + i];
    if (p < -1 || p >= i) {
      record_error(a.ws, MKV_ERR_INVALID_ARG, b);
      p = -1;
    }
  }
  uint32_t own[kW];
#pragma unroll
  for (int w = 0; w < kW; ++w) own[w] = (i < n && (i >> 5) == w) ? 1u << (i & 31) : 0u;
  int far = p;  // the first ancestor that `own` does not hold
  for (int reach = 1; reach < n; reach *= 2) {
#pragma unroll
    for (int w = 0; w < kW; ++w) bits[w][i] = own[w];
    up[i] = static_cast<int16_t>(far);
    __syncthreads();
    if (far >= 0) {
#pragma unroll
      for (int w = 0; w < kW; ++w) own[w] |= bits[w][far];
      far = up[far];
    }
    __syncthreads();
  }
  if (i >= a.N) return;
  int seen = 0;
#pragma unroll
  for (int w = 0; w < kW; ++w) {
    if (w < W) a.mask[((size_t)b * a.N + i) * W + w] = own[w];
    seen += __popc(own[w]);
  }
  if (a.pos != nullptr)
    a.pos[(size_t)b * a.N + i] = (a.base != nullptr ? a.base[b * a.base_stride] : 0) + (seen > 0 ? seen - 1 : 0);
}

// One CTA per (unit, layer): path_len rows of K and V, 16 bytes per thread.
// It writes caches, so it releases no later launch before it is done (one that
// loads its cache early would read it half written).
constexpr int kCommitThreads = 128;
__global__ void __launch_bounds__(kCommitThreads) tree_commit_kernel(const __grid_constant__ CommitArgs a) {
  const int u = blockIdx.x, b = u / a.n_kv, kv = u % a.n_kv, tid = threadIdx.x;
  const CommitLayer& l = a.layer[blockIdx.y];
  grid_dependency_wait();
  const int n = a.n_path[b], len = l.len[u], seen = l.seen[u];
  const int32_t* path = a.path + (size_t)b * a.path_len;
  const bool range = n >= 0 && n <= a.path_len;
  bool bad = !range;
  for (int j = tid; range && j < n; j += kCommitThreads) bad |= path[j] < 0 || path[j] >= a.N;
  // (the barrier also holds every thread's reads of len and seen before their update)
  if (__syncthreads_or(bad)) {
    if (tid == 0) record_error(a.ws, MKV_ERR_INVALID_ARG, u);
    return;
  }
  if (len < 0 || (int64_t)len + n > l.cap) {
    if (tid == 0) record_error(a.ws, MKV_ERR_CAPACITY, u);
    return;
  }
  const int pieces = a.D / 8;  // 16-byte pieces of a row
  for (int i = tid; i < n * pieces * 2; i += kCommitThreads) {
    const int row = i / (2 * pieces), r = i % (2 * pieces), p = r % pieces;
    const bool val = r >= pieces;
    const int64_t from = b * a.kv_batch + path[row] * a.kv_node + kv * a.D;
    const int64_t to = ((int64_t)u * l.cap + len + row) * a.D;
    reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(val ? l.V : l.K) + to)[p] =
        reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(val ? l.v : l.k) + from)[p];
  }
  for (int j = tid; j < n; j += kCommitThreads) l.pos[(int64_t)u * l.cap + len + j] = seen + j;
  if (tid == 0) {
    l.len[u] = len + n;
    l.seen[u] = seen + n;
  }
}

}  // namespace

cudaError_t launch_tree_build(const TreeBuildArgs& a, int batch, cudaStream_t stream) {
  return launch_pdl(tree_build_kernel, dim3(batch), dim3((a.N + 31) / 32 * 32), 0, stream, a);
}

cudaError_t launch_tree_commit(const CommitArgs& a, int layers, int units, cudaStream_t stream) {
  return launch_pdl(tree_commit_kernel, dim3(units, layers), dim3(kCommitThreads), 0, stream, a);
}

}  // namespace mkv
