// Norms of queries and keys per head with the rotation by position in the
// same pass (mkv_norm_rope), and the gradient of both (mkv_norm_rope_grad).
//
// Mathematics.  A row is one head of one token, d values x.  With r = (mean
// x^2 + eps)^(-1/2) and xh = x r, the result is y = R (w xh), R the rotation of
// rope.cu (its angles reduced exactly).  Backwards, from the gradient dy of y:
// dn = R^T dy (the rotation by the negative angle), dw = sum over rows of
// dn xh, and with gain = w dn
//   dx = r (gain - xh mean(gain xh)).
// All of it is fp32; y and dx are rounded once.  A sum of squares that passes
// fp32's range is taken again of the values times 2^-70.
//
// A row is spread over d / 16 neighbouring lanes, 16 dims each in the pairs
// that rotate together, so a row's sums are 2 or 3 shuffles, its angles serve
// the thread's other heads, and nothing goes through shared memory but the
// weights' gradient at the end.
//
// The weights' gradient: a thread sums its rows' terms in registers, a block its
// threads', and each block leaves one row in the workspace, which a second
// launch sums in a fixed order: no atomics, the same bits on every run.
//
// Bounded by HBM at 4 bytes a value forward and 6 backward, in so far as enough
// rows are in flight: a row's sum stands between its loads and its stores, so
// the forward kernel is held to 64 registers, four blocks an SM, at the cost of
// 24 spilled bytes (4 x 32768 tokens, 40 heads of 128 dims: 494 us, 0.80 of 6.8 TB/s; 526 with 72 registers and three; 505 with the next
// head's values loaded ahead and 80; 516 with weight times cosine and sine
// kept in pairs for two operations an instruction, and 80).  The gradient, 127
// registers and two blocks: 16382 tokens 122 us, 0.61.
#include <algorithm>

#include "kernels.h"
#include "rope.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kGradBlocks = 2;  // of the gradient per SM, by their registers
constexpr float kShrink = 0x1p-70f;

// Sum over the lanes that share a row (aligned groups of N lanes; `mask` the group's).
template <int N>
__device__ __forceinline__ float row_sum(float v, uint32_t mask) {
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) v += __shfl_xor_sync(mask, v, o);
  return v;
}

__device__ __forceinline__ float dot8(const float (&a)[8], const float (&b)[8], float s) {
#pragma unroll
  for (int i = 0; i < 8; ++i) s = fmaf(a[i], b[i], s);
  return s;
}

// 8 weights from element `at` of a row that starts at element `row`.
__device__ __forceinline__ void load_weights(const NormWeight& w, int64_t row, int at, float (&x)[8]) {
  if (w.p == nullptr) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 1.f;
  } else if (w.f32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(w.p) + row + at);
    const float4 a = __ldg(p), b = __ldg(p + 1);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else {
    unpack8(__ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(w.p) + row + at)), x);
  }
}

// r of a row, whose values become xh = x r.
template <int D>
__device__ __forceinline__ float normalise(float (&x0)[8], float (&x1)[8], float eps, uint32_t mask) {
  constexpr int N = D / 16;
  float ss = row_sum<N>(dot8(x0, x0, dot8(x1, x1, 0.f)), mask), shrink = 1.f;
  if (!(ss < INFINITY)) {  // (uniform over the row)
    shrink = kShrink;
#pragma unroll
    for (int i = 0; i < 8; ++i) x0[i] *= kShrink, x1[i] *= kShrink;
    ss = row_sum<N>(dot8(x0, x0, dot8(x1, x1, 0.f)), mask);
    eps *= kShrink * kShrink;
  }
  const float r = rsqrtf(fmaf(ss, 1.f / D, eps));
#pragma unroll
  for (int i = 0; i < 8; ++i) x0[i] *= r, x1[i] *= r;
  return r * shrink;
}

// A thread has one chunk of one token and the heads slot, slot + slots, ... of all tensors (as many as in rope.cu).
template <int D>
__global__ void __launch_bounds__(kThreads, 4) norm_rope_kernel(const __grid_constant__ NormRopeArgs a, int slots) {
  constexpr int kChunks = D / 16;
  grid_dependency_wait();
  const int per = kChunks * slots;  // threads of a token
  const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t tok = id / per;
  if (tok >= (int64_t)a.batch * a.tokens) return;
  const uint32_t mask = ((1u << kChunks) - 1u) << (threadIdx.x & 31 & ~(kChunks - 1));
  const int r = static_cast<int>(id % per), c = r % kChunks, slot = r / kChunks;
  const int b = static_cast<int>(tok / a.tokens), t = static_cast<int>(tok % a.tokens);
  const bool turn = c < a.rot / 16;
  float cs[8], sn[8];
  if (turn) chunk_angles(a, c, b, t, cs, sn);
  const int o0 = turn ? (a.neighbours ? c * 16 : c * 8) : c * 16;
  const int o1 = turn && !a.neighbours ? o0 + a.rot / 2 : o0 + 8;
  for (int h = slot; h < a.heads; h += slots) {
    int i = 0, hh = h;
    while (hh >= a.x[i].heads) hh -= a.x[i++].heads;
    const RopeTensor& x = a.x[i];
    const __nv_bfloat16* src =
        static_cast<const __nv_bfloat16*>(x.in) + b * x.in_batch + t * x.in_token + hh * x.in_head;
    __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(x.out) + b * x.out_batch + t * x.out_token + hh * x.out_head;
    const uint4 v0 = *reinterpret_cast<const uint4*>(src + o0), v1 = *reinterpret_cast<const uint4*>(src + o1);
    float x0[8], x1[8], w0[8], w1[8];
    load_weights(a.w[i], hh * a.w[i].head, o0, w0);
    load_weights(a.w[i], hh * a.w[i].head, o1, w1);
    unpack8(v0, x0);
    unpack8(v1, x1);
    (void)normalise<D>(x0, x1, a.eps, mask);
#pragma unroll
    for (int j = 0; j < 8; ++j) x0[j] *= w0[j], x1[j] *= w1[j];
    if (turn) {
      float y0[8], y1[8];
      turn_chunk<false>(a.neighbours != 0, cs, sn, x0, x1, y0, y1);
      *reinterpret_cast<uint4*>(dst + o0) = pack8(y0);
      *reinterpret_cast<uint4*>(dst + o1) = pack8(y1);
    } else {
      *reinterpret_cast<uint4*>(dst + o0) = pack8(x0);
      *reinterpret_cast<uint4*>(dst + o1) = pack8(x1);
    }
  }
}

// The rows that share a weight row (a tensor's, or one head's) are a group; its
// blocks share the group's (token, head slot) units evenly.
template <int D>
__global__ void __launch_bounds__(kThreads) norm_rope_grad_kernel(const __grid_constant__ NormRopeGradArgs a) {
  constexpr int kChunks = D / 16, kRows = kThreads / kChunks;  // rows at a time
  __shared__ float sums[kThreads / 32][D];
  grid_dependency_wait();
  grid_launch_dependents();
  int i = 0, block = blockIdx.x;
  while (i + 1 < a.tensors && block >= a.x[i + 1].first_block) ++i;
  const NormRopeGradTensor& x = a.x[i];
  block -= x.first_block;
  const int group = block / x.blocks, mine = block - group * x.blocks;  // the group within the tensor, the block within the group
  const uint32_t mask = ((1u << kChunks) - 1u) << (threadIdx.x & 31 & ~(kChunks - 1));
  const int c = threadIdx.x % kChunks;
  const bool turn = c < a.rot / 16;
  const int o0 = turn ? (a.neighbours ? c * 16 : c * 8) : c * 16;
  const int o1 = turn && !a.neighbours ? o0 + a.rot / 2 : o0 + 8;
  const int heads = x.per_head ? 1 : x.heads;
  float w0[8], w1[8];
  load_weights(x.w, group * x.w.head, o0, w0);
  load_weights(x.w, group * x.w.head, o1, w1);
  float d0[8] = {}, d1[8] = {};
  const int64_t units = (int64_t)a.batch * a.tokens * x.slots;
  for (int64_t u = (int64_t)mine * kRows + threadIdx.x / kChunks; u < units; u += (int64_t)x.blocks * kRows) {
    const int64_t tok = u / x.slots;
    const int slot = static_cast<int>(u - tok * x.slots);
    const int b = static_cast<int>(tok / a.tokens), t = static_cast<int>(tok % a.tokens);
    float cs[8], sn[8];
    if (turn) chunk_angles(a, c, b, t, cs, sn);
    for (int h = slot; h < heads; h += x.slots) {
      const int hh = x.per_head ? group : h;
      const __nv_bfloat16* px =
          static_cast<const __nv_bfloat16*>(x.x) + b * x.x_batch + t * x.x_token + hh * x.x_head;
      const __nv_bfloat16* py =
          static_cast<const __nv_bfloat16*>(x.dy) + b * x.dy_batch + t * x.dy_token + hh * x.dy_head;
      const uint4 v0 = *reinterpret_cast<const uint4*>(px + o0), v1 = *reinterpret_cast<const uint4*>(px + o1);
      const uint4 u0 = *reinterpret_cast<const uint4*>(py + o0), u1 = *reinterpret_cast<const uint4*>(py + o1);
      float x0[8], x1[8], y0[8], y1[8];
      unpack8(v0, x0);
      unpack8(v1, x1);
      unpack8(u0, y0);
      unpack8(u1, y1);
      if (turn) {
        float n0[8], n1[8];
        turn_chunk<true>(a.neighbours != 0, cs, sn, y0, y1, n0, n1);
#pragma unroll
        for (int j = 0; j < 8; ++j) y0[j] = n0[j], y1[j] = n1[j];
      }
      const float r = normalise<D>(x0, x1, a.eps, mask);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        d0[j] = fmaf(y0[j], x0[j], d0[j]);
        d1[j] = fmaf(y1[j], x1[j], d1[j]);
        y0[j] *= w0[j];
        y1[j] *= w1[j];
      }
      const float mean = row_sum<kChunks>(dot8(y0, x0, dot8(y1, x1, 0.f)), mask) * (1.f / D);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y0[j] = r * fmaf(-x0[j], mean, y0[j]);
        y1[j] = r * fmaf(-x1[j], mean, y1[j]);
      }
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(x.dx) + b * x.dx_batch + t * x.dx_token + hh * x.dx_head;
      *reinterpret_cast<uint4*>(dst + o0) = pack8(y0);
      *reinterpret_cast<uint4*>(dst + o1) = pack8(y1);
    }
  }
  if (x.dw == nullptr) return;
  // the block's sums: over the rows of a warp by shuffles, over the warps through shared memory
#pragma unroll
  for (int j = 0; j < 8; ++j) {
#pragma unroll
    for (int o = kChunks; o < 32; o <<= 1) {
      d0[j] += __shfl_xor_sync(0xffffffffu, d0[j], o);
      d1[j] += __shfl_xor_sync(0xffffffffu, d1[j], o);
    }
  }
  if ((threadIdx.x & 31) < kChunks) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sums[threadIdx.x / 32][o0 + j] = d0[j];
      sums[threadIdx.x / 32][o1 + j] = d1[j];
    }
  }
  __syncthreads();
  if (threadIdx.x < D) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) s += sums[w][threadIdx.x];
    a.parts[(size_t)blockIdx.x * D + threadIdx.x] = s;
  }
}

// dw of one group and 32 dims: its blocks' rows, 8 runs of them at once, then
// the runs one after another.
template <int D>
__global__ void __launch_bounds__(kThreads) norm_rope_dw_kernel(const __grid_constant__ NormRopeGradArgs a) {
  __shared__ float sums[kThreads / 32][32];
  grid_dependency_wait();
  int i = 0, group = blockIdx.x / (D / 32);
  while (group >= a.x[i].groups) group -= a.x[i++].groups;
  const NormRopeGradTensor& x = a.x[i];
  if (x.dw == nullptr) return;
  const int lane = threadIdx.x & 31, run = threadIdx.x >> 5, at = blockIdx.x % (D / 32) * 32 + lane;
  const float* part = a.parts + ((size_t)x.first_block + (size_t)group * x.blocks) * D + at;
  float s = 0.f;
#pragma unroll 8
  for (int p = run; p < x.blocks; p += kThreads / 32) s += part[(size_t)p * D];
  sums[run][lane] = s;
  __syncthreads();
  if (run != 0) return;
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) s += sums[w][lane];
  x.dw[(size_t)group * D + at] = s;
}

}  // namespace

cudaError_t launch_norm_rope(const NormRopeArgs& a, int head_dim, int num_sms, cudaStream_t stream) {
  const int64_t chunks = (int64_t)a.batch * a.tokens * a.heads * (head_dim / 16);
  const int64_t per = std::clamp<int64_t>(chunks / (5ll * 5 * kThreads * num_sms), 3, 20);
  const int slots = static_cast<int>((a.heads + per - 1) / per);
  const int64_t threads = (int64_t)a.batch * a.tokens * slots * (head_dim / 16);
  const int64_t blocks = (threads + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  return head_dim == 128 ? launch_pdl(norm_rope_kernel<128>, grid, block, 0, stream, a, slots)
                         : launch_pdl(norm_rope_kernel<64>, grid, block, 0, stream, a, slots);
}

// Blocks of every group, and where each tensor's start: as many as the GPU
// holds, dealt out by the rows of the groups.
int norm_rope_grad_plan(NormRopeGradArgs& a, int head_dim, int num_sms) {
  const int64_t tokens = (int64_t)a.batch * a.tokens, rows = kThreads / (head_dim / 16);
  int64_t all = 0;
  for (int i = 0; i < a.tensors; ++i) all += a.x[i].heads;
  int first = 0;
  for (int i = 0; i < a.tensors; ++i) {
    NormRopeGradTensor& x = a.x[i];
    x.groups = x.per_head ? x.heads : 1;
    const int64_t heads = x.per_head ? 1 : x.heads, share = kGradBlocks * num_sms * heads / all;
    // A unit's angles serve its heads, but there should be a unit for every row
    // that the blocks work on at a time, and with four heads or more eight of
    // them, so that the last ones do not leave most blocks idle.
    const int64_t fill = (share * rows + tokens) / std::max<int64_t>(tokens, 1);
    x.slots = static_cast<int>(std::clamp<int64_t>(std::max(std::min(fill, heads), std::min(8 * fill, heads / 4)), 1, heads));
    const int64_t units = tokens * x.slots;
    x.blocks = static_cast<int>(std::clamp<int64_t>((units + rows - 1) / rows, 1, std::max<int64_t>(share, 1)));
    x.first_block = first;
    first += x.groups * x.blocks;
  }
  return first;
}

cudaError_t launch_norm_rope_grad(const NormRopeGradArgs& a, int head_dim, int blocks, cudaStream_t stream) {
  const auto run = [&](auto kernel, int grid) {
    return launch_pdl(kernel, dim3(static_cast<unsigned>(grid)), dim3(kThreads), 0, stream, a);
  };
  cudaError_t e = head_dim == 128 ? run(norm_rope_grad_kernel<128>, blocks) : run(norm_rope_grad_kernel<64>, blocks);
  if (e != cudaSuccess) return e;
  int groups = 0;
  bool wanted = false;
  for (int i = 0; i < a.tensors; ++i) groups += a.x[i].groups, wanted |= a.x[i].dw != nullptr;
  if (!wanted) return cudaSuccess;
  const int grid = groups * (head_dim / 32);
  return head_dim == 128 ? run(norm_rope_dw_kernel<128>, grid) : run(norm_rope_dw_kernel<64>, grid);
}

}  // namespace mkv
