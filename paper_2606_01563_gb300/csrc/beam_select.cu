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
// equal.  The n_out-th largest of the threads' best keys of a chunk is a bound
// with at least n_out keys at or above it, and only keys of n_out threads
// at most reach it: they fit a buffer whatever the logits are.  Once a list
// is full its last key is the bound for what follows, which nearly nothing
// passes.
//
// Rounding.  Terms, and the sum of 16 of them, are fp32 about a reference that is a whole number at or
// above the largest logit (a term of weight has a small exponent, and sums about different references
// join by factors that depend on whole numbers alone).  From there on sums are pairs of fp32
// values: a thread may add 4096 such sums, whose roundings in one value came to 2e-5.
// The log of the joined sum and the scores are fp64: which of two continuations is
// better is decided to a few 1e-7 whatever the vocabulary, and the scores that come back are rounded once.
//
// Each logit is read once.  What bounds it over many beams is waiting more than
// issue (32 x 8 of 150001 bf16 logits: 44 us, HBM's floor 9.6; with blocks of 512 threads
// 72): an SM that has blocks issues in 0.58 of its cycles, 20 instructions a logit,
// and of the 8.8 cycles from one of a warp's issues to its next 2.3 go to the
// chunk's barrier and 1.8 to the instruction before; the join, 11 us, has a block an item.
// Over few it is the two launches' chains (4 beams of 32000: 9.8-10.3 us).  Of the
// same logits fp32 take 46 us, rows of an odd length that are not padded to 16 bytes 56 (bf16)
// and 46 (fp32); one item of 64 beams 74 us (n_out 64), of 8 beams 21.
#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 128, kWarps = kThreads / 32;  // of a run's block
constexpr int kJoinThreads = 512;
constexpr int kVec = 16;                   // elements of a thread and chunk (32 and six blocks an SM: 51 us for 42.6)
constexpr int kChunk = kThreads * kVec;    // elements of a chunk
constexpr int kMaxOut = MKV_BEAM_MAX_OUT;  // 64
constexpr int kBuffer = kMaxOut * kVec + 2 * kMaxOut;
constexpr int kMaxLists = 128;  // of a batch item
constexpr int64_t kBlocks = 8;  // of an SM (measured at 32 x 8 beams of 150001: 4, 8, 16 and 32: 57, 47, 55 and 76 us)
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

// A sum that is kept to more than 32 bits: hi, with what its roundings lost in lo.
// (fp64 units are few: a warp's addition holds them for 16 cycles.)
struct Sum {
  float hi, lo;
};
__device__ __forceinline__ Sum add(const Sum& a, const Sum& b) {
  const float s = a.hi + b.hi, t = s - a.hi;
  return Sum{s, ((a.hi - (s - t)) + (b.hi - t)) + (a.lo + b.lo)};
}
// a += x, four operations: exact where a is the larger.  Where x is, the sum at least
// doubles, so that what such steps lose is at most 2^-23 of the result, however many there are.
__device__ __forceinline__ void add_to(Sum& a, float x) {
  const float y = x + a.lo, s = a.hi + y;
  a.lo = y - (s - a.hi);
  a.hi = s;
}
__device__ __forceinline__ Sum scaled(const Sum& a, float f) {
  const float hi = a.hi * f;
  return Sum{hi, fmaf(a.hi, f, -hi) + a.lo * f};
}
// The sum of a warp's first `lanes` lanes (those after them hold 0), in each of them.
__device__ __forceinline__ Sum lanes_sum(Sum s, int lanes) {
  for (int o = 1; o < lanes; o <<= 1)
    s = add(s, Sum{__shfl_xor_sync(0xffffffffu, s.hi, o), __shfl_xor_sync(0xffffffffu, s.lo, o)});
  return s;
}

struct RowShared {
  uint64_t keys[kBuffer];
  uint64_t best[kMaxOut];
  uint64_t tops[kThreads];
  uint64_t bound;  // the least key that is still wanted
  int fill;
  float ref[kWarps];
  Sum sum[kWarps];
};

// The buffer's best `out` keys (all, if there are fewer) in order, at its start.
__device__ __forceinline__ void keep_best(RowShared& sh, int out) {
  __syncthreads();
  const int n = sh.fill;
  // the ranks' keys by way of a second place (a rank below `out` is one thread's)
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const uint64_t k = sh.keys[i];
    int r = 0;
#pragma unroll 8
    for (int m = 0; m < n; ++m) r += sh.keys[m] > k;
    if (r < out) {
      sh.best[r] = k;
      if (r == out - 1) sh.bound = k + 1;
    }
  }
  __syncthreads();
  if (threadIdx.x < min(n, out)) sh.keys[threadIdx.x] = sh.best[threadIdx.x];
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

// A thread's elements of the chunk that starts at element `first` of the row, as
// they lie in memory (a chunk ahead); from `end` on they are -infinity and not read.
template <bool F32, bool Vec>
struct Chunk {
  uint32_t w[F32 ? kVec : kVec / 2];
  __device__ __forceinline__ void load(const void* row, int first, int end) {
    constexpr int V = F32 ? 4 : 8;
    constexpr uint32_t kNone = F32 ? 0xff800000u : 0xff80u;  // -infinity
    if constexpr (Vec) {
#pragma unroll
      for (int j = 0; j < kVec / V; ++j) {
        const int v = first + element_of<F32, Vec>(j * V);
        if (v + V <= end) {
          const uint4 x = __ldcs(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(row) + (size_t)v * (F32 ? 4 : 2)));
          w[4 * j] = x.x, w[4 * j + 1] = x.y, w[4 * j + 2] = x.z, w[4 * j + 3] = x.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if constexpr (F32) {
              w[4 * j + i] = v + i < end ? static_cast<const uint32_t*>(row)[v + i] : kNone;
            } else {
              const int e = v + 2 * i;
              const uint32_t lo = e < end ? static_cast<const uint16_t*>(row)[e] : kNone;
              w[4 * j + i] = lo | (e + 1 < end ? static_cast<const uint16_t*>(row)[e + 1] : kNone) << 16;
            }
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const int v = first + element_of<F32, Vec>(i);
        if constexpr (F32) {
          w[i] = v < end ? __ldcs(static_cast<const uint32_t*>(row) + v) : kNone;
        } else {
          const uint32_t x = v < end ? __ldcs(static_cast<const uint16_t*>(row) + v) : kNone;
          w[i / 2] = i % 2 == 0 ? x : w[i / 2] | x << 16;
        }
      }
    }
  }
  __device__ __forceinline__ void floats(float (&x)[kVec]) const {
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      if constexpr (F32)
        x[i] = __uint_as_float(w[i]);
      else
        x[i] = __uint_as_float(i % 2 == 0 ? w[i / 2] << 16 : w[i / 2] & 0xffff0000u);
    }
  }
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
static_assert(kVec == 16, "four fours");
// Two floats in one 64-bit register, and two operations per instruction.
__device__ __forceinline__ uint64_t pack2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t x, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x));
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <bool F32, bool Vec>
__global__ void __launch_bounds__(kThreads) beam_rows_kernel(const __grid_constant__ SelectArgs a) {
  __shared__ RowShared sh;
  grid_dependency_wait();
  grid_launch_dependents();
  const int row = blockIdx.x / a.splits, split = blockIdx.x - row * a.splits, tid = threadIdx.x, lane = tid & 31;
  const int item = row / a.beams, lo = split * a.per, end = min(lo + a.per, a.vocab);
  const uint8_t* base = static_cast<const uint8_t*>(a.logits) +
                        (item * a.s_batch + (row - item * a.beams) * a.s_beam) * (F32 ? 4 : 2);
  Chunk<F32, Vec> next;  // on its way while the beam's state is read
  next.load(base, lo, end);
  const float score = a.score[row];
  float4* stat = a.stats + (size_t)row * a.splits + split;
  if (split == 0 && tid == 0 && !(score < INFINITY)) record_error(a.ws, MKV_ERR_INVALID_ARG, row);
  if (!(score > kNegInf && score < INFINITY) || (a.done != nullptr && a.done[row] != 0)) {
    if (tid == 0) *stat = make_float4(kNegInf, 0.f, 0.f, __int_as_float(0));
    return;
  }
  if (tid == 0) sh.fill = 0, sh.bound = 1;
  float ref = kNegInf;
  Sum sum{0.f, 0.f};
  __syncthreads();
  for (int first = lo; first < end; first += kChunk) {
    float x[kVec];
    next.floats(x);
    if (first + kChunk < end) next.load(base, first + kChunk, end);
    float tops[kVec / 4];  // of four elements each
#pragma unroll
    for (int i = 0; i < kVec / 4; ++i) tops[i] = fmaxf(max3(x[4 * i], x[4 * i + 1], x[4 * i + 2]), x[4 * i + 3]);
    const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]);
    if (top > ref) {
      const float r = ceilf(top);
      if (ref != kNegInf) sum = scaled(sum, expf(ref - r));  // (else it is 0, or NaN for good)
      ref = r;
    }
    {
      // (about a reference of 0 where there is nothing yet; a NaN or +infinity makes the sum one)
      const float r = ref == kNegInf ? 0.f : ref;
      const uint64_t nref = pack2(-r, -r), scale = pack2(kLog2e, kLog2e);
      uint64_t sums = 0;
#pragma unroll
      for (int i = 0; i < kVec; i += 2) {
        float t0, t1;
        unpack2(mul2(add2(pack2(x[i], x[i + 1]), nref), scale), t0, t1);
        sums = add2(sums, pack2(fast_exp2(t0), fast_exp2(t1)));
      }
      float s0, s1;
      unpack2(sums, s0, s1);
      add_to(sum, s0 + s1);
    }
    // what is still wanted of the chunk
    uint64_t bound = sh.bound;
    const float least = key_logit(bound);
    const bool any = bound == 1 ? top > kNegInf : top >= least;
    // (read before the barrier: behind it other warps may already be adding keys,
    // and all threads must take the same side, which has barriers of its own)
    const int fill = sh.fill;
    const int wanted = __syncthreads_count(any);
    if (wanted == 0) continue;
    if (fill + wanted * kVec > kBuffer) {
      if (fill > a.out) keep_best(sh, a.out);
      uint64_t best = 0;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const uint64_t k = make_key(x[i], first + element_of<F32, Vec>(i));
        best = k > best ? k : best;
      }
      sh.tops[tid] = best;
      __syncthreads();
      int r = 0;
#pragma unroll 16
      for (int t = 0; t < kThreads; ++t) r += sh.tops[t] > best;
      if (r == a.out - 1 && best > sh.bound) sh.bound = best;
      __syncthreads();
      bound = sh.bound;
    }
    if (any) {
      const float wanted_from = bound == 1 ? kNegInf : key_logit(bound);
#pragma unroll
      for (int j = 0; j < kVec / 4; ++j) {
        if (!(tops[j] >= wanted_from)) continue;  // (most are not)
#pragma unroll
        for (int i = 4 * j; i < 4 * j + 4; ++i) {
          const uint64_t k = make_key(x[i], first + element_of<F32, Vec>(i));
          if (k >= bound) sh.keys[atomicAdd(&sh.fill, 1)] = k;
        }
      }
    }
    __syncthreads();
    // (a full list's last key is the bound from here on)
    if (sh.fill > 2 * a.out) keep_best(sh, a.out);
  }
  // the sums of the warps, then of the block
  float r = warp_max(ref);
  bool odd = !(sum.hi < INFINITY);
  sum = lanes_sum(ref == kNegInf ? Sum{0.f, 0.f} : scaled(sum, expf(ref - r)), 32);
  if (lane == 0) sh.ref[tid >> 5] = r, sh.sum[tid >> 5] = sum;
  odd = __syncthreads_or(odd);
  keep_best(sh, a.out);
  const int n = odd ? 0 : sh.fill;
  if (tid < n) a.keys[((size_t)row * a.splits + split) * a.out + tid] = sh.keys[tid];
  if (tid < 32) {
    r = tid < kWarps ? sh.ref[tid] : kNegInf;
    const float m = warp_max(r);
    sum = lanes_sum(r == kNegInf ? Sum{0.f, 0.f} : scaled(sh.sum[tid], expf(r - m)), kWarps);  // (lanes past the warps have no reference)
    if (tid == 0) {
      *stat = make_float4(m, sum.hi, sum.lo, __int_as_float(odd ? -1 : n));
      if (odd) record_error(a.ws, MKV_ERR_INVALID_ARG, row);
    }
  }
}

// A continuation: larger is better, of equal scores the lower place.  (Scores
// are compared as order-preserving integers: the fp64 units are few, and ranks are many comparisons.)
struct Cand {
  uint64_t key;
  uint32_t at;  // beam * vocab + token
  uint32_t pad;
};
__device__ __forceinline__ uint64_t score_key(double v) {
  const int64_t u = __double_as_longlong(v + 0.0);  // (-0 is 0)
  return static_cast<uint64_t>(u) ^ (u < 0 ? ~0ull : 1ull << 63);
}
__device__ __forceinline__ float key_score(uint64_t k) {
  return static_cast<float>(__longlong_as_double(static_cast<int64_t>(k >> 63 ? k ^ 1ull << 63 : ~k)));
}
// (without branches: ranks are many comparisons)
__device__ __forceinline__ int better(const Cand& a, const Cand& b) {
  return static_cast<int>(a.key > b.key) | (static_cast<int>(a.key == b.key) & static_cast<int>(a.at < b.at));
}

// A block per batch item.  Its lists (a run of one beam's tokens each, or an ended beam's
// one continuation) are in order, so a bound with n_out continuations at or above it is
// the n_out-th best of the lists' first ones, or any list's n_out-th one.
__global__ void __launch_bounds__(kJoinThreads) beam_join_kernel(const __grid_constant__ SelectArgs a) {
  extern __shared__ __align__(16) uint8_t raw[];
  Cand* cand = reinterpret_cast<Cand*>(raw);  // [lists * out]
  __shared__ Cand heads[kMaxLists];
  __shared__ Cand bound, deep[kMaxLists];
  __shared__ float refs[MKV_BEAM_MAX_BEAMS];     // a beam's reference
  __shared__ double offset[MKV_BEAM_MAX_BEAMS];  // its score less the log of its sum about that
  __shared__ int count[kMaxLists], over[MKV_BEAM_MAX_BEAMS], fill;
  __shared__ float scores[MKV_BEAM_MAX_BEAMS];
  __shared__ Sum sums[MKV_BEAM_MAX_BEAMS];
  grid_dependency_wait();
  grid_launch_dependents();
  const int item = blockIdx.x, tid = threadIdx.x, lists = a.beams * a.splits;
  if (tid == 0) fill = 0, bound = Cand{0, 0xffffffffu, 0};
  // a warp a beam, a lane a split (at most 128 of them, where there is one beam)
  for (int b = tid >> 5; b < a.beams; b += kJoinThreads / 32) {
    const int row = item * a.beams + b, lane = tid & 31;
    const float score = a.score[row];
    const bool ended = a.done != nullptr && a.done[row] != 0;
    float4 st[kMaxLists / 32];
    float m = kNegInf;
    Sum sum{0.f, 0.f};
    bool odd = false;
#pragma unroll
    for (int i = 0; i < kMaxLists / 32; ++i) {
      const int s = i * 32 + lane;
      st[i] = s < a.splits ? a.stats[(size_t)row * a.splits + s] : make_float4(kNegInf, 0.f, 0.f, 0.f);
      m = fmaxf(m, st[i].x);
      odd |= __float_as_int(st[i].w) < 0;
    }
    m = warp_max(m);
    odd = __any_sync(0xffffffffu, odd);
#pragma unroll
    for (int i = 0; i < kMaxLists / 32; ++i)
      if (st[i].x > kNegInf) sum = add(sum, scaled(Sum{st[i].y, st[i].z}, expf(st[i].x - m)));
    sum = lanes_sum(sum, min(a.splits, 32));
    const bool ok = !ended && !odd && sum.hi > 0.f;
#pragma unroll
    for (int i = 0; i < kMaxLists / 32; ++i) {
      const int s = i * 32 + lane;
      // an ended beam's one continuation is its first list's
      if (s < a.splits)
        count[b * a.splits + s] = ended ? (s == 0 && score > kNegInf && score < INFINITY && a.end >= 0 ? 1 : 0)
                                  : ok  ? __float_as_int(st[i].w)
                                        : 0;
    }
    if (lane == 0) {
      scores[b] = score;
      over[b] = ended;
      refs[b] = m;
      sums[b] = ok ? sum : Sum{1.f, 0.f};
    }
  }
  __syncthreads();
  // (all beams' at once: a warp's fp64 instruction takes as long for one lane as for 32)
  if (tid < a.beams) offset[tid] = static_cast<double>(scores[tid]) - log(static_cast<double>(sums[tid].hi) + sums[tid].lo);
  __syncthreads();
  auto get = [&](int list, int i) {
    const int b = list / a.splits;
    if (over[b]) return Cand{score_key(static_cast<double>(scores[b])), static_cast<uint32_t>(b) * a.vocab + a.end, 0};
    const uint64_t k = a.keys[((size_t)item * lists + list) * a.out + i];
    // (a logit less its reference first: exact, where both are far from 0)
    return Cand{score_key((static_cast<double>(key_logit(k)) - refs[b]) + offset[b]), static_cast<uint32_t>(b) * a.vocab + key_token(k), 0};
  };
  const Cand none{0, 0xffffffffu, 0};  // (no finite score has key 0)
  if (tid < lists) {
    heads[tid] = count[tid] > 0 ? get(tid, 0) : none;
    deep[tid] = count[tid] == a.out ? get(tid, a.out - 1) : none;
  }
  __syncthreads();
  if (tid < lists) {
    const Cand h = heads[tid], d = deep[tid];
    int r = 0, rd = 0;
#pragma unroll 8
    for (int l = 0; l < lists; ++l) {
      r += better(heads[l], h);
      rd += better(deep[l], d);
    }
    // (both may hold: the better one is the bound)
    if (r == a.out - 1 && h.key != 0) heads[tid].pad = 1;
    if (rd == 0 && d.key != 0) deep[tid].pad = 1;
  }
  __syncthreads();
  if (tid < lists) {
    if (heads[tid].pad) bound = heads[tid];
  }
  __syncthreads();
  if (tid < lists && deep[tid].pad && better(deep[tid], bound)) bound = deep[tid];
  __syncthreads();
  const Cand least = bound;
  for (int i = tid; i < lists * a.out; i += kJoinThreads) {
    const int list = i / a.out, k = i - list * a.out;
    if (k >= count[list]) continue;
    const Cand c = get(list, k);
    if (!better(least, c)) cand[atomicAdd(&fill, 1)] = c;
  }
  __syncthreads();
  const int n = fill;
  for (int i = tid; i < n; i += kJoinThreads) {
    const Cand c = cand[i];
    int r = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) r += better(cand[j], c);
    if (r >= a.out) continue;
    const size_t o = (size_t)item * a.out + r;
    const int b = static_cast<int>(c.at / a.vocab), t = static_cast<int>(c.at - static_cast<uint32_t>(b) * a.vocab);
    a.parent[o] = b;
    a.token[o] = t;
    a.score_out[o] = key_score(c.key);
    if (a.done_out != nullptr) a.done_out[o] = over[b] || t == a.end;
  }
  for (int r = n + tid; r < a.out; r += kJoinThreads) {
    const size_t o = (size_t)item * a.out + r;
    a.parent[o] = -1;
    a.token[o] = -1;
    a.score_out[o] = kNegInf;
    if (a.done_out != nullptr) a.done_out[o] = 0;
  }
}

}  // namespace

size_t select_plan(SelectArgs& a, int batch, int num_sms, void* ws) {
  // As many blocks as there are places for eight on an SM, but no split below a
  // chunk, and lists of a batch item that the second launch can hold.
  const int64_t rows = (int64_t)batch * a.beams;
  const int64_t most = std::min<int64_t>(kMaxLists / a.beams, ((int64_t)a.vocab + kChunk - 1) / kChunk);
  a.splits = static_cast<int>(std::clamp<int64_t>(kBlocks * num_sms / rows, 1, most));
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
  return launch_pdl(beam_join_kernel, dim3(batch), dim3(kJoinThreads), smem, stream, a);
}

}  // namespace mkv
