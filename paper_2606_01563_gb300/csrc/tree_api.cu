// C-ABI entry points declared in include/mkv_tree.h: argument validation,
// workspace sizing and kernel dispatch.
#include <cmath>

#include "common.cuh"
#include "kernels.h"
#include "tree.h"
#include "validate.h"

using namespace mkv;

namespace {

mkv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MKV_OK : MKV_ERR_CUDA; }

bool header_ok(const void* ws, size_t bytes) { return ws && bytes >= kHeaderBytes && aligned(ws, 256); }

// A stride as used: the dense value for 0, else the caller's, which 16-byte
// copies must be able to step by and tensor maps to hold (below 2^40 bytes).
bool stride_of(int64_t given, int64_t dense, int64_t* used) {
  *used = given == 0 ? dense : given;
  return *used >= dense && *used % 8 == 0 && *used < ((int64_t)1 << 38);
}

// 1 / 2 pi as the sum of two doubles
constexpr double kTurnHi = 0x1.45f306dc9c883p-3, kTurnLo = -0x1.6b01ec5417056p-57;

// Turns per position of w radians, modulo one, in units of 2^-64: the product
// with the first part is split exactly (fma), whole turns drop out, and the
// sign is that of two's complement.
uint64_t turns_of(float w, bool inverse) {
  const double p = static_cast<double>(w) * kTurnHi;
  const double rest = std::fma(static_cast<double>(w), kTurnHi, -p) + static_cast<double>(w) * kTurnLo;
  const double frac = p - std::rint(p);  // [-1/2, 1/2], exact
  const double head = std::rint(frac * 0x1p62);
  const int64_t lead = static_cast<int64_t>(head);  // within +-2^61
  const int64_t tail = std::llrint((frac * 0x1p62 - head) * 4.0 + rest * 0x1p64);
  const uint64_t t = (static_cast<uint64_t>(lead) << 2) + static_cast<uint64_t>(tail);
  return inverse ? ~t + 1 : t;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------- build
mkv_status mkv_tree_build(int32_t batch, int32_t n_nodes, const int32_t* parents, const int32_t* count,
                          const int32_t* base, int64_t base_stride, uint32_t* mask, int32_t* pos, void* workspace,
                          size_t workspace_bytes, void* stream) {
  NvtxRange nvtx("mkv_tree_build");
  if (batch < 1 || batch > 65535 || n_nodes < 1 || n_nodes > MKV_TREE_MAX_NODES) return MKV_ERR_SHAPE;
  if (!parents || !mask || base_stride < 0 || !aligned(parents, 4) || !aligned(count, 4) || !aligned(base, 4) ||
      !aligned(mask, 4) || !aligned(pos, 4))
    return MKV_ERR_INVALID_ARG;
  if (!header_ok(workspace, workspace_bytes)) return MKV_ERR_WORKSPACE;
  TreeBuildArgs a{};
  a.parents = parents;
  a.count = count;
  a.base = base;
  a.base_stride = base_stride;
  a.mask = mask;
  a.pos = pos;
  a.N = n_nodes;
  a.ws = workspace;
  return cuda_status(launch_tree_build(a, batch, static_cast<cudaStream_t>(stream)));
}

// -------------------------------------------------------------------- step
size_t mkv_tree_workspace_size(mkv_geom geom, int32_t n_nodes, int32_t capacity) {
  if (!geom_ok(geom) || n_nodes < 1 || n_nodes > MKV_TREE_MAX_NODES || capacity < 1) return 0;
  return tree_workspace_bytes(geom, n_nodes, capacity, num_sms_current());
}

mkv_status mkv_tree_step(mkv_geom geom, const mkv_tree* tree, const void* q, const void* k, const void* v,
                         const mkv_cache* cache, const mkv_moments* mom, const mkv_decode_params* p, void* out,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  NvtxRange nvtx("mkv_tree_step");
  if (!tree || !k || !v) return geom_ok(geom) ? MKV_ERR_INVALID_ARG : geom_status(geom);
  const mkv_status chk =
      decode_args_status(geom, q, k, v, cache, mom, p, static_cast<const float*>(out));
  if (chk != MKV_OK) return chk;
  if (tree->n_nodes < 1 || tree->n_nodes > MKV_TREE_MAX_NODES) return MKV_ERR_SHAPE;
  if (!tree->mask || !aligned(tree->mask, 4) || !aligned(tree->count, 4) || !aligned(lse, 4))
    return MKV_ERR_INVALID_ARG;
  TreeArgs a{};
  const int64_t kv = (int64_t)geom.n_kv_heads * geom.head_dim, N = tree->n_nodes;
  if (!stride_of(tree->q_node, kv * geom.group, &a.q_node) || !stride_of(tree->q_batch, N * a.q_node, &a.q_batch) ||
      !stride_of(tree->kv_node, kv, &a.kv_node) || !stride_of(tree->kv_batch, N * a.kv_node, &a.kv_batch))
    return MKV_ERR_INVALID_ARG;
  const int sms = num_sms_current();
  if (!workspace || workspace_bytes < tree_workspace_bytes(geom, tree->n_nodes, cache->capacity, sms) ||
      !aligned(workspace, 256))
    return MKV_ERR_WORKSPACE;
  a.q = q;
  a.k = k;
  a.v = v;
  a.N = tree->n_nodes;
  a.count = tree->count;
  a.mask = tree->mask;
  a.K = cache->K;
  a.V = cache->V;
  a.len = cache->len;
  a.cap = cache->capacity;
  if (p->correction) {
    a.n = mom->n;
    a.mu_k = mom->mu_k;
    a.mu_v = mom->mu_v;
    a.C = mom->C;
    a.C16 = static_cast<const __nv_bfloat16*>(p->C16);
    a.Cs = static_cast<const uint2*>(p->C_split);
  }
  a.order = p->order;
  a.tau = p->tau;
  a.early = p->early_load;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = lse;
  a.ws = workspace;
  a.batch = geom.batch;
  a.n_kv = geom.n_kv_heads;
  return cuda_status(launch_tree_step(a, geom, sms, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ commit
mkv_status mkv_tree_commit(mkv_geom geom, const mkv_tree* tree, int32_t n_layers, const mkv_tree_layer* layers,
                           const int32_t* path, int32_t path_len, const int32_t* n_path, void* workspace,
                           size_t workspace_bytes, void* stream) {
  NvtxRange nvtx("mkv_tree_commit");
  if (!geom_ok(geom)) return geom_status(geom);
  if (!tree || !layers || !path || !n_path || n_layers < 0 || !aligned(path, 4) || !aligned(n_path, 4))
    return MKV_ERR_INVALID_ARG;
  if (tree->n_nodes < 1 || tree->n_nodes > MKV_TREE_MAX_NODES || path_len < 1 || path_len > MKV_TREE_MAX_NODES)
    return MKV_ERR_SHAPE;
  CommitArgs a{};
  const int64_t N = tree->n_nodes;
  if (!stride_of(tree->kv_node, (int64_t)geom.n_kv_heads * geom.head_dim, &a.kv_node) ||
      !stride_of(tree->kv_batch, N * a.kv_node, &a.kv_batch))
    return MKV_ERR_INVALID_ARG;
  for (int i = 0; i < n_layers; ++i)
    if (!cache_ok(&layers[i].cache) || !layers[i].k || !layers[i].v || !aligned(layers[i].k, 16) ||
        !aligned(layers[i].v, 16))
      return MKV_ERR_INVALID_ARG;
  if (!header_ok(workspace, workspace_bytes)) return MKV_ERR_WORKSPACE;
  a.path = path;
  a.n_path = n_path;
  a.path_len = path_len;
  a.N = tree->n_nodes;
  a.n_kv = geom.n_kv_heads;
  a.D = geom.head_dim;
  a.ws = workspace;
  const int units = geom.batch * geom.n_kv_heads;
  for (int first = 0; first < n_layers; first += kCommitLayers) {
    const int n = n_layers - first < kCommitLayers ? n_layers - first : kCommitLayers;
    for (int i = 0; i < n; ++i) {
      const mkv_tree_layer& l = layers[first + i];
      a.layer[i] = CommitLayer{l.cache.K, l.cache.V, l.cache.pos, l.cache.len, l.cache.seen, l.k, l.v,
                               l.cache.capacity};
    }
    const cudaError_t e = launch_tree_commit(a, n, units, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_status(e);
  }
  return MKV_OK;
}

// -------------------------------------------------------------------- rope
mkv_status mkv_rope(int32_t batch, int32_t tokens, int32_t head_dim, const int32_t* pos, int64_t pos_axis,
                    int64_t pos_batch, const mkv_rope_params* p, int32_t n_tensors, const mkv_rope_tensor* tensors,
                    void* stream) {
  NvtxRange nvtx("mkv_rope");
  if (head_dim != 64 && head_dim != 128) return MKV_ERR_UNSUPPORTED;
  if (batch < 1 || tokens < 0 || (int64_t)batch * tokens > ((int64_t)1 << 31) || n_tensors < 1 ||
      n_tensors > MKV_ROPE_MAX_TENSORS)
    return MKV_ERR_SHAPE;
  if (!p || !tensors || pos_axis < 0 || pos_batch < 0) return MKV_ERR_INVALID_ARG;
  if (p->rot_dim < 16 || p->rot_dim > head_dim || p->rot_dim % 16 != 0 || p->n_axes < 1 ||
      p->n_axes > MKV_ROPE_MAX_AXES || (p->neighbours != 0 && p->neighbours != 1) ||
      (p->inverse != 0 && p->inverse != 1))
    return MKV_ERR_INVALID_ARG;
  RopeArgs a{};
  for (int f = 0; f < p->rot_dim / 2; ++f) {
    if (!(std::fabs(p->inv_freq[f]) <= 0x1p20f) || p->axis[f] < 0 || p->axis[f] >= p->n_axes)
      return MKV_ERR_INVALID_ARG;
    a.turn[f] = turns_of(p->inv_freq[f], p->inverse != 0);
    a.axis[f] = static_cast<uint8_t>(p->axis[f]);
  }
  if (tokens == 0) return MKV_OK;  // (empty tensors may have no address)
  if (!pos || !aligned(pos, 4)) return MKV_ERR_INVALID_ARG;
  int64_t heads = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const mkv_rope_tensor& t = tensors[i];
    if (!t.in || !t.out || !aligned(t.in, 16) || !aligned(t.out, 16) || t.heads < 1) return MKV_ERR_INVALID_ARG;
    for (const int64_t s : {t.in_batch, t.in_token, t.in_head, t.out_batch, t.out_token, t.out_head})
      if (s % 8 != 0 || s < 0) return MKV_ERR_INVALID_ARG;
    // two tokens or heads that are written to one place
    if ((batch > 1 && t.out_batch == 0) || (tokens > 1 && t.out_token == 0) || (t.heads > 1 && t.out_head == 0))
      return MKV_ERR_INVALID_ARG;
    heads += t.heads;
    a.x[i] = RopeTensor{t.in,        t.out,       t.in_batch, t.in_token, t.in_head,
                        t.out_batch, t.out_token, t.out_head, t.heads};
  }
  if (heads > 65536) return MKV_ERR_SHAPE;
  a.pos = pos;
  a.pos_axis = pos_axis;
  a.pos_batch = pos_batch;
  a.heads = static_cast<int32_t>(heads);
  a.batch = batch;
  a.tokens = tokens;
  a.rot = p->rot_dim;
  a.neighbours = p->neighbours;
  return cuda_status(launch_rope(a, head_dim, num_sms_current(), static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
