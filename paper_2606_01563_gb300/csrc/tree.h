// Internal launcher interface of the calls in include/mkv_tree.h.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/mkv_tree.h"

namespace mkv {

// A launch that may be placed while its predecessor in the stream still runs
// (its kernel waits for it with griddepcontrol.wait before anything else).
template <typename Kernel, typename... Args>
cudaError_t launch_pdl(Kernel kernel, dim3 grid, dim3 block, size_t smem, cudaStream_t stream, const Args&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

constexpr int kTreeNodes = MKV_TREE_MAX_NODES;

__host__ __device__ constexpr int tree_words(int n) { return (n + 31) / 32; }

// -------------------------------------------------------------------- step
struct TreeArgs {
  const void* q;  // bf16 [b, N, Hkv*G, D], strides in elements
  const void* k;  // bf16 [b, N, Hkv, D]
  const void* v;
  int64_t q_node, q_batch, kv_node, kv_batch;
  int32_t N;
  const int32_t* count;  // [b] or null
  const uint32_t* mask;  // [b, N, tree_words(N)]
  const void* K;         // bf16 [b, Hkv, cap, D]
  const void* V;
  const int32_t* len;
  int32_t cap;
  const int32_t* n;  // null: no moment term
  const float* mu_k;
  const float* mu_v;
  const float* C;
  const __nv_bfloat16* C16;
  const uint2* Cs;
  int32_t order;
  float tau;
  int32_t early;
  __nv_bfloat16* out;  // [b, N, Hkv*G, D]
  float* lse;
  uint32_t polls;  // poll limit of the pipeline waits
  void* ws;
  int32_t batch;
  int32_t n_kv;
};

size_t tree_workspace_bytes(const mkv_geom& g, int32_t n_nodes, int32_t capacity, int num_sms);
cudaError_t launch_tree_step(const TreeArgs& a, const mkv_geom& g, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------- build and commit
struct TreeBuildArgs {
  const int32_t* parents;  // [b, N]
  const int32_t* count;
  const int32_t* base;
  int64_t base_stride;
  uint32_t* mask;
  int32_t* pos;
  int32_t N;
  void* ws;
};
cudaError_t launch_tree_build(const TreeBuildArgs& a, int batch, cudaStream_t stream);

constexpr int kCommitLayers = 64;  // layers per launch: their pointers travel in the launch's arguments (4 KB)
struct CommitLayer {
  void* K;
  void* V;
  int32_t* pos;
  int32_t* len;
  int32_t* seen;
  const void* k;
  const void* v;
  int64_t cap;
};
struct CommitArgs {
  CommitLayer layer[kCommitLayers];
  const int32_t* path;
  const int32_t* n_path;
  int32_t path_len;
  int32_t N;
  int64_t kv_node, kv_batch;
  int32_t n_kv;
  int32_t D;
  void* ws;
};
cudaError_t launch_tree_commit(const CommitArgs& a, int layers, int units, cudaStream_t stream);

// -------------------------------------------------------------------- rope
constexpr int kRopeFreqs = 64;
struct RopeTensor {
  const void* in;
  void* out;
  int64_t in_batch, in_token, in_head;
  int64_t out_batch, out_token, out_head;
  int32_t heads;
};
struct RopeArgs {
  uint64_t turn[kRopeFreqs];  // turns per position, modulo one turn, in units of 2^-64
  uint8_t axis[kRopeFreqs];
  RopeTensor x[MKV_ROPE_MAX_TENSORS];
  const int32_t* pos;
  int64_t pos_axis, pos_batch;
  int32_t heads;  // of all tensors
  int32_t batch;
  int32_t tokens;
  int32_t rot;
  int32_t neighbours;
};
cudaError_t launch_rope(const RopeArgs& a, int head_dim, int num_sms, cudaStream_t stream);

}  // namespace mkv
