// The selected beams' states, in place (mkv_beam_reorder): slot j of a batch
// item takes the state that slot parent[j] had, in every layer.
//
// A state is copied by byte ranges: a block takes a range of the item's
// slots in one layer and KV head, loads it from every slot that is another one's
// parent into shared memory (each is read once, however many slots it goes to),
// waits, and stores it to the slots.  Ranges do not depend on one another,
// so nothing else is needed for any parents, and a slot that stays as it is costs nothing.
// Loads and stores are bulk copies; one warp issues them, a range
// loading while the one before is stored.
//
// Positions and means, which need not start at 16 bytes, are blocks of their own
// that go through shared memory word by word.  Lengths and counts change last: a
// second launch, after every block of the first has read the lengths.
//
// Bounded by HBM: the bytes of the parents read and of the changed slots written
// (8 layers, 4 x 16 slots of 8 heads, 512 rows and moments: 278 us, 0.91 of 6.8 TB/s).
#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kThreads = 128;
constexpr int kRing = 96 * 1024;  // of a block: two fit an SM
constexpr int kStages = 2;
constexpr int kSmallThreads = 256;

__device__ __forceinline__ void bulk_s2g(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_addr(src)), "r"(bytes)
               : "memory");
}

// What both launches know of an item's slots in one layer and head.
struct Slots {
  int parent[kReorderSeqs];   // -1: stays
  int length[kReorderSeqs];   // rows in use, 0..cap
  int y_len[kReorderSeqs];
  int place[kReorderSeqs];    // of a slot that is read: its place among those; -1
  int reads;                  // slots that are read
  int longest;                // of those
  int bad;
};

// Reads an item's parents and lengths; false: nothing to do (no slot changes, or a parent is out of
// range: recorded by the caller's first block).
template <int Threads>
__device__ __forceinline__ bool read_slots(const ReorderArgs& a, const ReorderLayer& l, int item, int kv, bool first,
                                           Slots& s) {
  const int tid = threadIdx.x;
  if (tid == 0) s.reads = s.longest = s.bad = 0;
  for (int j = tid; j < a.N; j += Threads) s.place[j] = -1;
  __syncthreads();
  for (int j = tid; j < a.N; j += Threads) {
    const int p = a.parent[(size_t)item * a.N + j], unit = (item * a.N + j) * a.n_kv + kv;
    if (p < -1 || p >= a.N) s.bad = 1;
    s.parent[j] = p == j ? -1 : p;
    const int len = l.len[unit], y = l.y_len != nullptr ? l.y_len[unit] : 0;
    if (first && max(static_cast<uint32_t>(len), static_cast<uint32_t>(y)) > static_cast<uint32_t>(l.cap))
      record_error(a.ws, MKV_ERR_CAPACITY, unit);
    s.length[j] = min(max(len, 0), l.cap);
    s.y_len[j] = min(max(y, 0), l.cap);
  }
  __syncthreads();
  if (s.bad) {
    if (first && tid == 0) record_error(a.ws, MKV_ERR_INVALID_ARG, item);
    return false;
  }
  for (int j = tid; j < a.N; j += Threads)
    if (s.parent[j] >= 0) s.place[s.parent[j]] = 0;
  __syncthreads();
  if (tid < 32) {
    int n = 0, most = 0;
    for (int j0 = 0; j0 < a.N; j0 += 32) {
      const int j = j0 + tid;
      const bool read = j < a.N && s.place[j] == 0;
      const uint32_t all = __ballot_sync(0xffffffffu, read);
      if (read) {
        s.place[j] = n + __popc(all & ((1u << tid) - 1u));
        most = max(most, s.length[j]);
      }
      n += __popc(all);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (tid == 0) s.reads = n, s.longest = most;
  }
  __syncthreads();
  return s.reads > 0;
}

// `stride` words of an array per unit, of which slot j holds have(j), at most
// `most`: from the slots that are read into shared memory, then to the others.
template <typename Have>
__device__ __forceinline__ void move_words(const ReorderArgs& a, const Slots& s, int item, int kv, int32_t* base,
                                           size_t stride, int most, int32_t* words, Have have) {
  if (base == nullptr) return;
  const int per = kRing / 4 / s.reads;  // words of a slot at a time (at least 96)
  auto unit = [&](int j) { return (size_t)((item * a.N + j) * a.n_kv + kv); };
  for (int w0 = 0; w0 < most; w0 += per) {
    const int n = min(per, most - w0);
    __syncthreads();
    for (int j = 0; j < a.N; ++j)
      if (s.place[j] >= 0)
        for (int w = threadIdx.x; w < min(n, have(j) - w0); w += kThreads) words[s.place[j] * per + w] = base[unit(j) * stride + w0 + w];
    __syncthreads();
    for (int j = 0; j < a.N; ++j) {
      const int p = s.parent[j];
      if (p >= 0)
        for (int w = threadIdx.x; w < min(n, have(p) - w0); w += kThreads) base[unit(j) * stride + w0 + w] = words[s.place[p] * per + w];
    }
  }
}

__global__ void __launch_bounds__(kThreads) reorder_kernel(const __grid_constant__ ReorderArgs a) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ Slots s;
  __shared__ __align__(8) uint64_t full[kStages];
  const int tid = threadIdx.x, item = blockIdx.y / a.n_kv, kv = blockIdx.y - item * a.n_kv;
  const ReorderLayer& l = a.layer[blockIdx.z];
  if (tid < kStages) mbar_init(&full[tid], 1);
  mbar_fence_init();
  grid_dependency_wait();
  grid_launch_dependents();
  if (!read_slots<kThreads>(a, l, item, kv, blockIdx.x == 0, s)) return;
  if (blockIdx.x >= a.split) {
    int32_t* words = reinterpret_cast<int32_t*>(ring);
    if (blockIdx.x == a.split) {
      move_words(a, s, item, kv, l.pos, l.cap, s.longest, words, [&](int j) { return s.length[j]; });
    } else {
      move_words(a, s, item, kv, l.mu_k, a.D, a.D, words, [&](int) { return a.D; });
      move_words(a, s, item, kv, l.mu_v, a.D, a.D, words, [&](int) { return a.D; });
    }
    return;
  }
  if (tid >= 32) return;
  // one warp from here on
  const uint32_t range = kRing / kStages / s.reads / 128 * 128;  // bytes of a slot (at least 128: 256 slots)
  const uint32_t row = a.D * 2;
  // the arrays' ranges in one list: K, V, y, C
  uint32_t ranges[4], total = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint64_t bytes = l.big[k] == nullptr ? 0
                           : k < 2             ? (uint64_t)s.longest * row
                           : k == 2            ? (uint64_t)l.cap * row * 2  // (y_len of the parents, below)
                                               : (uint64_t)a.D * a.D * 4;
    ranges[k] = static_cast<uint32_t>((bytes + range - 1) / range);
  }
  if (l.big[2] != nullptr) {
    int most = 0;
    for (int j = tid; j < a.N; j += 32)
      if (s.place[j] >= 0) most = max(most, s.y_len[j]);
    most = __reduce_max_sync(0xffffffffu, most);
    ranges[2] = static_cast<uint32_t>(((uint64_t)most * row * 2 + range - 1) / range);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) total += ranges[k];
  // range i: which array, its first byte, the bytes of a slot's array and of its content
  struct Range {
    int k;
    uint64_t at;
  };
  auto find = [&](uint32_t i) {
    int k = 0;
    while (i >= ranges[k]) i -= ranges[k++];
    return Range{k, (uint64_t)i * range};
  };
  auto unit_bytes = [&](int k) -> uint64_t {
    return k == 3 ? (uint64_t)a.D * a.D * 4 : (uint64_t)l.cap * row * (k == 2 ? 2 : 1);
  };
  auto content = [&](const Range& r, int j) -> uint32_t {  // bytes of slot j's range
    const uint64_t have = r.k == 3 ? (uint64_t)a.D * a.D * 4
                          : r.k == 2 ? (uint64_t)s.y_len[j] * row * 2
                                     : (uint64_t)s.length[j] * row;
    return have <= r.at ? 0u : static_cast<uint32_t>(min((uint64_t)range, have - r.at));
  };
  auto at = [&](const Range& r, int j) {
    return l.big[r.k] + (size_t)((item * a.N + j) * a.n_kv + kv) * unit_bytes(r.k) + r.at;
  };
  auto load = [&](uint32_t i, int stage) {
    const Range r = find(i);
    uint32_t bytes = 0;
    for (int j = tid; j < a.N; j += 32)
      if (s.place[j] >= 0) bytes += content(r, j);
    bytes = __reduce_add_sync(0xffffffffu, bytes);
    if (tid == 0) mbar_arrive_expect_tx(&full[stage], bytes);
    __syncwarp();
    for (int j = tid; j < a.N; j += 32) {
      const uint32_t n = s.place[j] >= 0 ? content(r, j) : 0;
      if (n > 0) bulk_g2s(ring + (size_t)stage * (kRing / kStages) + (size_t)s.place[j] * range, at(r, j), n, &full[stage]);
    }
  };
  uint32_t i = blockIdx.x, phase[kStages] = {};  // (of a.split blocks)
  int stage = 0;
  if (i < total) load(i, 0);
  for (; i < total; i += a.split) {
    const uint32_t next = i + a.split;
    if (next < total) {
      // (the next stage's stores have read shared memory)
      asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      __syncwarp();
      load(next, stage ^ 1);
    }
    const bool got = mbar_wait(&full[stage], phase[stage], a.polls);
    phase[stage] ^= 1;
    if (!__all_sync(0xffffffffu, got)) {
      if (tid == 0) {
        record_error(a.ws, MKV_ERR_TIMEOUT, item);
        // the copies in flight land before the block's shared memory goes
        (void)mbar_wait(&full[stage], phase[stage] ^ 1);
        if (next < total) (void)mbar_wait(&full[stage ^ 1], phase[stage ^ 1]);
      }
      break;
    }
    const Range r = find(i);
    for (int j = tid; j < a.N; j += 32) {
      const int p = s.parent[j];
      const uint32_t n = p >= 0 ? content(r, p) : 0;
      if (n > 0) bulk_s2g(at(r, j), ring + (size_t)stage * (kRing / kStages) + (size_t)s.place[p] * range, n);
    }
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    stage ^= 1;
  }
  asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncwarp();
}

// Lengths and counts: a block per item, layer and head, a thread a slot.
__global__ void __launch_bounds__(kSmallThreads) reorder_small_kernel(const __grid_constant__ ReorderArgs a) {
  __shared__ int bad;
  const int j = threadIdx.x, item = blockIdx.y / a.n_kv, kv = blockIdx.y - item * a.n_kv;
  const ReorderLayer& l = a.layer[blockIdx.z];
  if (j == 0) bad = 0;
  grid_dependency_wait();
  __syncthreads();
  const int p = j < a.N ? a.parent[(size_t)item * a.N + j] : -1;
  if (p < -1 || p >= a.N) bad = 1;
  int32_t* const array[4] = {l.n, l.seen, l.len, l.y_len};
  const bool moves = p >= 0 && p < a.N && p != j;
  const size_t from = (size_t)((item * a.N + p) * a.n_kv + kv), to = (size_t)((item * a.N + j) * a.n_kv + kv);
  int32_t x[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = moves && array[k] != nullptr ? array[k][from] : 0;
  __syncthreads();
  if (bad || !moves) return;
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (array[k] != nullptr) array[k][to] = x[k];
}

}  // namespace

cudaError_t launch_beam_reorder(const ReorderArgs& args, int layers, int batch, int num_sms, cudaStream_t stream) {
  ReorderArgs a = args;
  a.polls = pipeline_poll_limit();
  cudaError_t e = cudaFuncSetAttribute(reorder_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRing);
  if (e != cudaSuccess) return e;
  // two blocks to an SM; more of an item's ranges side by side where there are few items
  const int64_t units = (int64_t)batch * a.n_kv * layers;
  int cap = 0;
  for (int i = 0; i < layers; ++i) cap = std::max(cap, a.layer[i].cap);
  const int64_t ranges = std::max<int64_t>(1, (int64_t)cap * a.D * 4 * a.N / (kRing / kStages));
  const int split = static_cast<int>(std::clamp<int64_t>((4ll * num_sms + units - 1) / units, 1, std::min<int64_t>(ranges, 256)));
  bool means = false;
  for (int i = 0; i < layers; ++i) means |= a.layer[i].mu_k != nullptr;
  a.split = split;
  const dim3 grid(split + (means ? 2 : 1), batch * a.n_kv, layers);
  e = launch_pdl(reorder_kernel, grid, dim3(kThreads), kRing, stream, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(reorder_small_kernel, dim3(1, batch * a.n_kv, layers), dim3(kSmallThreads), 0, stream, a);
}

}  // namespace mkv
