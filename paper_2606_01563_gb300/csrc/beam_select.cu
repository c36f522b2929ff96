// Beam search's selection over beams and vocabulary (mkv_beam_select).
//
// Mathematics.  A live beam's continuation by token t has the score
// score[beam] + (logit[t] - L), L the log of the sum of the beam's exponentials;
// a beam that has ended continues only as itself.  Wanted are the best n_out of a
// batch item's beams x vocabulary continuations, equal ones by the lower beam,
// then the lower token.
//
// Two launches.  The first reads the logits once: a block has a run of one
// beam's tokens, keeps the sum of exponentials about a reference per thread,
// and the run's n_out best logits.  Within a beam the order of logits is the order
// of scores, so nothing of the sum is needed for that.  The second has a
// block per batch item, which joins the runs' sums and selects among the runs'
// lists by score.
//
// The best of a run.  A logit and its token make one 64-bit key, so no two are
// equal.  Of the groups of a few threads each, the n_out-th largest of the groups'
// best keys is a bound with at least n_out keys at or above it, and only keys of n_out groups
// at most reach it: they fit a buffer whatever the logits are.  Once a list
// is full its last key is the bound for what follows, which nearly nothing
// passes.
//
// Rounding.  Terms are fp32 about a reference that is a whole number at or
// above the largest logit (a term of weight has a small exponent, and sums about different references
// join by factors that depend on whole numbers alone), sums of a thread fp32,
// the joined sum, its log and the scores fp64: which of two continuations is
// better is decided to about 1e-7, and the scores that come back are rounded once.
//
// Bounded by HBM over many beams: each logit is read once.
#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kVec = 16;                   // elements of a thread and chunk
constexpr int kChunk = kThreads * kVec;    // elements of a chunk
constexpr int kMaxOut = MKV_BEAM_MAX_OUT;  // 64
constexpr int kBuffer = 2048 + 2 * kMaxOut;
constexpr int kMaxLists = 128;  // of a batch item
constexpr float kNegInf = -INFINITY;

// Order-preserving key of a logit and the token that has it: larger is better,
// of equal logits the lower token.  0: none (a logit of -infinity).
__device__ __forceinline__ uint64_t make_key(float x, uint32_t token) {
  return x > kNegInf ? static_cast<uint64_t>(float_key(x + 0.f)) << 32 | ~token : 0ull;  // (-0 is 0)
}
__device__ __forceinline__ float key_logit(uint64_t k) {
  const uint32_t u = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((u & 0x80000000u) ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint32_t key_token(uint64_t k) { return ~static_cast<uint32_t>(k); }

__device__ __forceinline__ uint64_t shfl_max(uint64_t k, int o) {
  const uint64_t other = __shfl_xor_sync(0xffffffffu, k, o);
  return other > k ? other : k;
}

struct RowShared {
  uint64_t keys[kBuffer];
  uint64_t groups[256];
  uint64_t bound;  // the least key that is still wanted
  int fill;
  float ref[kWarps];
  float sum[kWarps];
};

// The buffer's best `out` keys (all, if there are fewer) in order, at its start.
__device__ __forceinline__ void keep_best(RowShared& sh, int out) {
  __syncthreads();
  const int n = sh.fill;
  uint64_t mine[(kBuffer + kThreads - 1) / kThreads];
  int rank[(kBuffer + kThreads - 1) / kThreads];
#pragma unroll 1
  for (int j = 0; j * kThreads < n; ++j) {
    const int i = j * kThreads + threadIdx.x;
    uint64_t k = i < n ? sh.keys[i] : 0;
    int r = 0;
    if (i < n)
#pragma unroll 4
      for (int m = 0; m < n; ++m) r += sh.keys[m] > k;
    mine[j] = k, rank[j] = i < n ? r : kBuffer;
  }
  __syncthreads();
#pragma unroll 1
  for (int j = 0; j * kThreads < n; ++j)
    if (rank[j] < out) {
      sh.keys[rank[j]] = mine[j];
      if (rank[j] == out - 1) sh.bound = mine[j] + 1;
    }
  if (threadIdx.x == 0) sh.fill = min(n, out);
  __syncthreads();
}

// The chunk's element that x[i] of a thread is: in vectors of 16 bytes, dealt out
// in turn, or (rows that do not all start at 16 bytes) one by one.  The same in every row of a call, so
// that beams with the same logits have the same sum to the last bit.
template <bool F32, bool Vec>
__device__ __forceinline__ int element_of(int i) {
  constexpr int V = !Vec ? 1 : F32 ? 4 : 8;
  return ((i / V) * kThreads + threadIdx.x) * V + i % V;
}

// A thread's elements of the chunk that starts at element `first` of the row; from `end` on they are
// -infinity and not read.
template <bool F32, bool Vec>
__device__ __forceinline__ void load_chunk(const void* row, int first, int end, float (&x)[kVec]) {
  constexpr int V = !Vec ? 1 : F32 ? 4 : 8;
#pragma unroll
  for (int j = 0; j < kVec / V; ++j) {
    const int v = first + element_of<F32, Vec>(j * V);
    if (Vec && v + V <= end) {
      const uint4 w = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(row) + (size_t)v * (F32 ? 4 : 2)));
      const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
          x[j * V + (Vec ? i : 0)] = __uint_as_float(u[i]);
        } else if constexpr (Vec) {
          x[j * V + 2 * i] = __uint_as_float(u[i] << 16);
          x[j * V + 2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (F32)
          x[j * V + i] = v + i < end ? __ldcs(static_cast<const float*>(row) + v + i) : kNegInf;
        else
          x[j * V + i] = v + i < end ? __uint_as_float(static_cast<uint32_t>(__ldcs(static_cast<const uint16_t*>(row) + v + i)) << 16)
                                     : kNegInf;
      }
    }
  }
}

template <bool F32, bool Vec>
__global__ void __launch_bounds__(kThreads) beam_rows_kernel(const __grid_constant__ SelectArgs a) {
  __shared__ RowShared sh;
  grid_dependency_wait();
  grid_launch_dependents();
  const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits, tid = threadIdx.x, lane = tid & 31;
  const float score = a.score[row];
  float4* stat = a.stats + (size_t)row * a.splits + split;
  if (split == 0 && tid == 0 && !(score < INFINITY)) record_error(a.ws, MKV_ERR_INVALID_ARG, row);
  if (!(score > kNegInf && score < INFINITY) || (a.done != nullptr && a.done[row] != 0)) {
    if (tid == 0) *stat = make_float4(kNegInf, 0.f, __int_as_float(0), 0.f);
    return;
  }
  const int item = row / a.beams;
  const uint8_t* base = static_cast<const uint8_t*>(a.logits) +
                        (item * a.s_batch + (row - item * a.beams) * a.s_beam) * (F32 ? 4 : 2);
  const int lo = split * a.per, end = min(lo + a.per, a.vocab);
  if (tid == 0) sh.fill = 0, sh.bound = 1;
  float ref = kNegInf, sum = 0.f;
  bool odd = false;
  const int span = a.out <= 32 ? 4 : 2, groups = kThreads / span;  // threads of a group
  __syncthreads();
  for (int first = lo; first < end; first += kChunk) {
    float x[kVec];
    load_chunk<F32, Vec>(base, first, end, x);
    float top = kNegInf;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      top = fmaxf(top, x[i]);
      odd |= !(x[i] < INFINITY);
    }
    if (top > kNegInf && !odd) {
      if (top > ref) {
        const float r = ceilf(top);
        sum = ref == kNegInf ? 0.f : sum * expf(ref - r);
        ref = r;
      }
#pragma unroll
      for (int i = 0; i < kVec; ++i) sum += fast_exp2((x[i] - ref) * kLog2e);
    }
    // what is still wanted of the chunk
    uint64_t bound = sh.bound;
    const float least = key_logit(bound);
    const bool any = bound == 1 ? top > kNegInf : top >= least;
    const int wanted = __syncthreads_count(any);
    if (wanted == 0) continue;
    if (sh.fill + wanted * kVec > kBuffer) {
      if (sh.fill > a.out) keep_best(sh, a.out);
      uint64_t best = 0;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const uint64_t k = make_key(x[i], first + element_of<F32, Vec>(i));
        best = k > best ? k : best;
      }
      for (int o = 1; o < span; o <<= 1) best = shfl_max(best, o);
      if (tid % span == 0) sh.groups[tid / span] = best;
      __syncthreads();
      if (tid < groups) {
        const uint64_t mine = sh.groups[tid];
        int r = 0;
#pragma unroll 8
        for (int g = 0; g < groups; ++g) r += sh.groups[g] > mine;
        if (r == a.out - 1 && mine > sh.bound) sh.bound = mine;
      }
      __syncthreads();
      bound = sh.bound;
    }
    if (any) {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const uint64_t k = make_key(x[i], first + element_of<F32, Vec>(i));
        if (k >= bound) sh.keys[atomicAdd(&sh.fill, 1)] = k;
      }
    }
    __syncthreads();
    // (a full list's last key is the bound from here on)
    if (sh.fill > 4 * a.out || (sh.fill >= a.out && bound == 1)) keep_best(sh, a.out);
  }
  // the sums of the warps, then of the block
  float r = warp_max(ref);
  sum = warp_sum(ref == kNegInf ? 0.f : sum * expf(ref - r));
  if (lane == 0) sh.ref[tid >> 5] = r, sh.sum[tid >> 5] = sum;
  odd = __syncthreads_or(odd);
  keep_best(sh, a.out);
  const int n = odd ? 0 : sh.fill;
  if (tid < n) a.keys[((size_t)row * a.splits + split) * a.out + tid] = sh.keys[tid];
  if (tid < 32) {
    r = tid < kWarps ? sh.ref[tid] : kNegInf;
    sum = tid < kWarps ? sh.sum[tid] : 0.f;
    const float m = warp_max(r);
    sum = warp_sum(r == kNegInf ? 0.f : sum * expf(r - m));
    if (tid == 0) {
      *stat = make_float4(m, sum, __int_as_float(n), odd ? 1.f : 0.f);
      if (odd) record_error(a.ws, MKV_ERR_INVALID_ARG, row);
    }
  }
}

// A continuation: larger is better, of equal scores the lower place.
struct Cand {
  double v;
  uint32_t at;  // beam * vocab + token
  uint32_t pad;
};
__device__ __forceinline__ bool better(const Cand& a, const Cand& b) { return a.v > b.v || (a.v == b.v && a.at < b.at); }

// A block per batch item.  Its lists (a run of one beam's tokens each, or an ended beam's
// one continuation) are in order, so a bound with n_out continuations at or above it is
// the n_out-th best of the lists' first ones, or any list's n_out-th one.
__global__ void __launch_bounds__(kThreads) beam_join_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) uint8_t raw[];
  Cand* cand = reinterpret_cast<Cand*>(raw);  // [lists * out]
  __shared__ Cand heads[kMaxLists];
  __shared__ Cand bound, deep[kMaxLists];
  __shared__ float refs[MKV_BEAM_MAX_BEAMS];     // a beam's reference
  __shared__ double offset[MKV_BEAM_MAX_BEAMS];  // its score less the log of its sum about that
  __shared__ int count[kMaxLists], over[MKV_BEAM_MAX_BEAMS], fill;
  __shared__ float scores[MKV_BEAM_MAX_BEAMS];
  grid_dependency_wait();
  grid_launch_dependents();
  const int item = blockIdx.x, tid = threadIdx.x, lists = a.beams * a.splits;
  if (tid == 0) fill = 0, bound = Cand{-INFINITY, 0xffffffffu, 0};
  for (int b = tid; b < a.beams; b += kThreads) {
    const int row = item * a.beams + b;
    scores[b] = a.score[row];
    over[b] = a.done != nullptr && a.done[row] != 0;
    const float4* st = a.stats + (size_t)row * a.splits;
    float m = kNegInf, odd = 0.f;
    for (int s = 0; s < a.splits; ++s) m = fmaxf(m, st[s].x), odd += st[s].w;
    double sum = 0;
    for (int s = 0; s < a.splits; ++s)
      if (st[s].x > kNegInf) sum += static_cast<double>(st[s].y * expf(st[s].x - m));
    const bool ok = !over[b] && odd == 0.f && sum > 0;
    refs[b] = m;
    offset[b] = ok ? static_cast<double>(scores[b]) - log(sum) : 0;
    for (int s = 0; s < a.splits; ++s) count[b * a.splits + s] = ok ? __float_as_int(st[s].z) : 0;
    // an ended beam's one continuation is its first list's
    if (over[b] && scores[b] > kNegInf && scores[b] < INFINITY && a.end >= 0) count[b * a.splits] = 1;
  }
  __syncthreads();
  auto get = [&](int list, int i) {
    const int b = list / a.splits;
    if (over[b]) return Cand{static_cast<double>(scores[b]), static_cast<uint32_t>(b) * a.vocab + a.end, 0};
    const uint64_t k = a.keys[((size_t)item * lists + list) * a.out + i];
    // (a logit less its reference first: exact, where both are far from 0)
    return Cand{(static_cast<double>(key_logit(k)) - refs[b]) + offset[b], static_cast<uint32_t>(b) * a.vocab + key_token(k), 0};
  };
  const Cand none{-INFINITY, 0xffffffffu, 0};
  if (tid < lists) {
    heads[tid] = count[tid] > 0 ? get(tid, 0) : none;
    deep[tid] = count[tid] == a.out ? get(tid, a.out - 1) : none;
  }
  __syncthreads();
  if (tid < lists) {
    const Cand h = heads[tid], d = deep[tid];
    int r = 0, rd = 0;
    for (int l = 0; l < lists; ++l) {
      r += better(heads[l], h);
      rd += better(deep[l], d);
    }
    // (both may hold: the better one is the bound)
    if (r == a.out - 1 && h.v > -INFINITY) heads[tid].pad = 1;
    if (rd == 0 && d.v > -INFINITY) deep[tid].pad = 1;
  }
  __syncthreads();
  if (tid < lists) {
    if (heads[tid].pad) bound = heads[tid];
  }
  __syncthreads();
  if (tid < lists && deep[tid].pad && better(deep[tid], bound)) bound = deep[tid];
  __syncthreads();
  const Cand least = bound;
  for (int i = tid; i < lists * a.out; i += kThreads) {
    const int list = i / a.out, k = i - list * a.out;
    if (k >= count[list]) continue;
    const Cand c = get(list, k);
    if (!better(least, c)) cand[atomicAdd(&fill, 1)] = c;
  }
  __syncthreads();
  const int n = fill;
  for (int i = tid; i < n; i += kThreads) {
    const Cand c = cand[i];
    int r = 0;
#pragma unroll 4
    for (int j = 0; j < n; ++j) r += better(cand[j], c);
    if (r >= a.out) continue;
    const size_t o = (size_t)item * a.out + r;
    const int b = static_cast<int>(c.at / a.vocab), t = static_cast<int>(c.at - static_cast<uint32_t>(b) * a.vocab);
    a.parent[o] = b;
    a.token[o] = t;
    a.score_out[o] = static_cast<float>(c.v);
    if (a.done_out != nullptr) a.done_out[o] = over[b] || t == a.end;
  }
  for (int r = n + tid; r < a.out; r += kThreads) {
    const size_t o = (size_t)item * a.out + r;
    a.parent[o] = -1;
    a.token[o] = -1;
    a.score_out[o] = kNegInf;
    if (a.done_out != nullptr) a.done_out[o] = 0;
  }
}

}  // namespace

size_t select_plan(SelectArgs& a, int batch, int num_sms, void* ws) {
  // Blocks of 512 threads, four to an SM, as many as there are places, but no
  // split below a chunk, and lists of a batch item that the second launch can hold.
  const int64_t rows = (int64_t)batch * a.beams;
  const int64_t most = std::min<int64_t>(kMaxLists / a.beams, ((int64_t)a.vocab + kChunk - 1) / kChunk);
  a.splits = static_cast<int>(std::clamp<int64_t>(4ll * num_sms / rows, 1, most));
  a.per = static_cast<int>((((int64_t)a.vocab + a.splits - 1) / a.splits + 7) / 8 * 8);
  const size_t stats = align_up((size_t)rows * a.splits * sizeof(float4), 256);
  if (ws != nullptr) {
    a.ws = ws;
    a.stats = reinterpret_cast<float4*>(static_cast<uint8_t*>(ws) + kHeaderBytes);
    a.keys = reinterpret_cast<uint64_t*>(static_cast<uint8_t*>(ws) + kHeaderBytes + stats);
  }
  return kHeaderBytes + stats + (size_t)rows * a.splits * a.out * sizeof(uint64_t);
}

cudaError_t launch_beam_select(const SelectArgs& a, int batch, bool f32, cudaStream_t stream) {
  const int64_t blocks = (int64_t)batch * a.beams * a.splits;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kThreads);
  const int size = f32 ? 4 : 2;
  const bool vec = reinterpret_cast<uintptr_t>(a.logits) % 16 == 0 && a.s_batch * size % 16 == 0 && a.s_beam * size % 16 == 0;
  const auto rows = [&](auto kernel) { return launch_pdl(kernel, grid, block, 0, stream, a); };
  cudaError_t e = f32 ? (vec ? rows(beam_rows_kernel<true, true>) : rows(beam_rows_kernel<true, false>))
                      : (vec ? rows(beam_rows_kernel<false, true>) : rows(beam_rows_kernel<false, false>));
  if (e != cudaSuccess) return e;
  const size_t smem = (size_t)a.beams * a.splits * a.out * sizeof(Cand);
  e = cudaFuncSetAttribute(beam_join_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           kMaxLists * kMaxOut * static_cast<int>(sizeof(Cand)));
  if (e != cudaSuccess) return e;
  return launch_pdl(beam_join_kernel, dim3(batch), block, smem, stream, a);
}

}  // namespace mkv
