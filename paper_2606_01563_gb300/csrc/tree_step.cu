// Attention of drafted nodes over the retained cache, the nodes they see and
// the moment term, in one normaliser (mkv_tree_step).
//
// One CTA per (node, KV head, batch item): its warps take the keys in turn, a
// lane holds D / 32 dims of the group's queries and of each key and value,
// and every warp keeps a running maximum, sum and output per head; the warps'
// states and the moment term merge at the end.  Simple and slow: K and V are
// read once per node.
#include "common.cuh"
#include "kernels.h"
#include "tree.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kWarps = 4;

template <int D, int G>
__global__ void __launch_bounds__(kWarps * 32) tree_step_kernel(const TreeArgs a) {
  constexpr int E = D / 32;  // dims per lane
  const int i = blockIdx.x, kv = blockIdx.y, b = blockIdx.z, u = b * a.n_kv + kv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  __shared__ float sm[kWarps + 1][G], sl[kWarps + 1][G], so[kWarps + 1][G][D], sq[G][D];
  grid_dependency_wait();
  const int HQ = a.n_kv * G;
  __nv_bfloat16* out = a.out + (((size_t)b * a.N + i) * HQ + kv * G) * D;
  float* lse = a.lse != nullptr ? a.lse + ((size_t)b * a.N + i) * HQ + kv * G : nullptr;
  int nodes = a.count != nullptr ? a.count[b] : a.N;
  if (nodes < 0 || nodes > a.N) {
    if (tid == 0) record_error(a.ws, MKV_ERR_INVALID_ARG, u);
    nodes = nodes < 0 ? 0 : a.N;
  }
  int len = a.len[u];
  if (len < 0 || len > a.cap) {
    if (tid == 0) record_error(a.ws, MKV_ERR_CAPACITY, u);
    len = len < 0 ? 0 : a.cap;
  }
  if (i >= nodes) {
    for (int j = tid; j < G * D; j += kWarps * 32) out[j] = __float2bfloat16_rn(0.f);
    if (lse != nullptr && tid < G) lse[tid] = -INFINITY;
    return;
  }
  const float qs = rsqrtf(static_cast<float>(D)) * kLog2e;
  float q[G][E], o[G][E] = {}, m[G], l[G];
  const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch + i * a.q_node + kv * G * D;
#pragma unroll
  for (int h = 0; h < G; ++h) {
    load_bf16<E>(qp + h * D + lane * E, q[h]);
    m[h] = -INFINITY;
    l[h] = 0.f;
    if (warp == 0)
#pragma unroll
      for (int e = 0; e < E; ++e) sq[h][lane * E + e] = q[h][e];
  }
  auto take = [&](const __nv_bfloat16* kp, const __nv_bfloat16* vp) {
    float k[E], v[E];
    load_bf16<E>(kp + lane * E, k);
    load_bf16<E>(vp + lane * E, v);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) x = fmaf(q[h][e], k[e], x);
      x = warp_sum(x) * qs;
      const float mn = fmaxf(m[h], x);
      const float f = mn == -INFINITY ? 1.f : fast_exp2(m[h] - mn), p = mn == -INFINITY ? 0.f : fast_exp2(x - mn);
      m[h] = mn;
      l[h] = fmaf(l[h], f, p);
#pragma unroll
      for (int e = 0; e < E; ++e) o[h][e] = fmaf(o[h][e], f, p * v[e]);
    }
  };
  const __nv_bfloat16* K = static_cast<const __nv_bfloat16*>(a.K) + (size_t)u * a.cap * D;
  const __nv_bfloat16* V = static_cast<const __nv_bfloat16*>(a.V) + (size_t)u * a.cap * D;
  for (int j = warp; j < len; j += kWarps) take(K + (size_t)j * D, V + (size_t)j * D);
  const uint32_t* row = a.mask + ((size_t)b * a.N + i) * tree_words(a.N);
  for (int j = warp; j < nodes; j += kWarps)
    if ((row[j >> 5] >> (j & 31)) & 1u) {
      const int64_t off = b * a.kv_batch + j * a.kv_node + kv * D;
      take(static_cast<const __nv_bfloat16*>(a.k) + off, static_cast<const __nv_bfloat16*>(a.v) + off);
    }
#pragma unroll
  for (int h = 0; h < G; ++h) {
#pragma unroll
    for (int e = 0; e < E; ++e) so[warp][h][lane * E + e] = o[h][e];
    if (lane == 0) {
      sm[warp][h] = m[h];
      sl[warp][h] = l[h];
    }
  }
  __syncthreads();
  // the moment term as one more state: m = its logit, l = 1, o = its value
  const int n_e = a.n != nullptr ? a.n[u] : 0;
  for (int t = tid; t < G * D; t += kWarps * 32) {
    const int h = t / D, c = t % D;
    float f = 0.f;
    if (n_e > 0) {
      if (a.order == 1)
        for (int j = 0; j < D; ++j) {
          const size_t at = ((size_t)u * D + c) * D + j;
          float x;
          if (a.Cs != nullptr) {
            const uint2 w = a.Cs[at / 2];
            const __nv_bfloat162 hi = *reinterpret_cast<const __nv_bfloat162*>(&w.x);
            const __nv_bfloat162 lo = *reinterpret_cast<const __nv_bfloat162*>(&w.y);
            x = (j & 1) ? __high2float(hi) + __high2float(lo) : __low2float(hi) + __low2float(lo);
          } else {
            x = a.C16 != nullptr ? __bfloat162float(a.C16[at]) : a.C[at];
            if (fabsf(x * static_cast<float>(n_e)) < a.tau) x = 0.f;
          }
          f = fmaf(x, sq[h][j], f);
        }
      f = fmaf(f, rsqrtf(static_cast<float>(D)), a.mu_v[(size_t)u * D + c]);
    }
    so[kWarps][h][c] = f;
  }
  if (tid < G) {
    float x = 0.f;
    for (int j = 0; n_e > 0 && j < D; ++j) x = fmaf(a.mu_k[(size_t)u * D + j], sq[tid][j], x);
    sm[kWarps][tid] = n_e > 0 ? fmaf(x, qs, log2f(static_cast<float>(n_e))) : -INFINITY;
    sl[kWarps][tid] = n_e > 0 ? 1.f : 0.f;
  }
  __syncthreads();
  for (int t = tid; t < G * D; t += kWarps * 32) {
    const int h = t / D, c = t % D;
    float M = -INFINITY, L = 0.f, acc = 0.f;
    for (int w = 0; w <= kWarps; ++w)
      if (sl[w][h] > 0.f) M = fmaxf(M, sm[w][h]);
    for (int w = 0; w <= kWarps; ++w)
      if (sl[w][h] != 0.f) {  // (a NaN sum passes on)
        const float f = fast_exp2(sm[w][h] - M);
        L = fmaf(sl[w][h], f, L);
        acc = fmaf(so[w][h][c], f, acc);
      }
    out[t] = __float2bfloat16_rn(L != 0.f ? acc / L : 0.f);
    if (c == 0 && lse != nullptr) lse[h] = L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
  }
}

}  // namespace

size_t tree_workspace_bytes(const mkv_geom&, int32_t, int32_t, int) { return kHeaderBytes; }

cudaError_t launch_tree_step(const TreeArgs& a, const mkv_geom& g, int, cudaStream_t stream) {
  const dim3 grid(a.N, g.n_kv_heads, g.batch);
#define MKV_TREE_CASE(D_, G_)                                                 \
  if (g.head_dim == D_ && g.group == G_) {                                    \
    tree_step_kernel<D_, G_><<<grid, kWarps * 32, 0, stream>>>(a);            \
    return cudaGetLastError();                                                \
  }
  MKV_TREE_CASE(128, 1)
  MKV_TREE_CASE(128, 2)
  MKV_TREE_CASE(128, 4)
  MKV_TREE_CASE(128, 8)
  MKV_TREE_CASE(64, 1)
  MKV_TREE_CASE(64, 2)
  MKV_TREE_CASE(64, 4)
  MKV_TREE_CASE(64, 8)
#undef MKV_TREE_CASE
  return cudaErrorInvalidValue;
}

}  // namespace mkv
