// Attention of drafted nodes over the retained cache, the nodes they see and
// the moment term, in one normaliser (mkv_tree_step), on the fifth-generation
// tensor cores.
//
// Mathematics.  A unit's query rows are (node, head of the group).  A block
// of 128 rows keeps a reference m, a sum l and an output O per row and takes
// the keys 128 at a time: S = Q K^T, P = 2^(S scale log2 e - m), l += sum P,
// O += P V.  The retained rows are tiles without a mask, the nodes are tiles
// whose bits the mask words give.  The moment term is one more key of every
// row, with logit e = log n + scale q.mu_k and value mu_v + scale C' q: its
// weight starts m and l, and its value joins at the end, the product Q C'^T
// running on the tensor cores with C' as bf16 hi + lo parts.  m only has to be
// common to a row's keys, so it is set 32 above the largest score so far in log2
// units and moves (by a whole number, with a rescaling of O and l) only when a
// score exceeds it: weights are at most 1, so that no sum overflows whose terms
// do not, and above 2^-33 for the largest score, which a floating-point sum
// holds as exactly (with 8 some row of a warp moved in most tiles of a long
// cache, 700 cycles each).  P enters
// the second product rounded to bf16 (2^-8 relative, the output's own
// rounding); l is summed from the unrounded weights, and O is scaled by the
// ratio of that sum to the rounded weights' (where a few weights dominate,
// their roundings then cancel: error against 64 bits 0.0023 without it).
//
// Work.  The tiles of all (unit, row block) items form one list that is cut
// into equal runs, one per CTA, wherever the run ends; an item cut by a
// boundary leaves (m, l, O) of its parts in the workspace, and
// tree_merge_kernel joins them.  Lengths of any raggedness so cost what their
// tiles cost.  Where one CTA per item would leave few tiles idle, that is taken
// instead (make_plan).  A CTA holds one or two row blocks: with two every K and V tile
// is read once for 256 rows, with one the two softmax groups take the tiles
// alternately and merge at the end.
//
// One CTA, four warpgroups: warps 0-3 and 4-7 are the softmax groups, a thread
// a row; warp 8 issues TMA copies (Q, and K and V tiles into a ring), warps 9
// and 10 the MMAs of a group each: S of its first tile, then in turn its product
// with V and its next S, so that one group's softmax runs beside the other's
// products (one thread for both groups: its own instructions, some 10 cycles
// each, left the tensor cores idle between the batches); warp 11 looks after
// sizes that were read early; warps 12-15 turn C'
// into operands, in slots of the ring, while the last tiles are worked on.  Code
// that runs once per item is kept in loops: unrolled, it waited for its own
// instructions (a masked tile took 9000 cycles instead of 2000).  Tensor memory: S (then P over it, at last Q C'^T) of the two groups,
// 128 columns each, and O of the two, D columns each.
//
// What bounds it: with few query rows HBM (16 x 8 heads, 8 nodes of 4 heads, 8192
// rows: 89 us, 0.90 of the copy rate); with 256 rows per tile the chain of a tile
// in each group, between the floors of HBM and the tensor cores (8 heads, 33
// nodes, 131072 rows: 112 us, HBM's floor 79; 8 x 8 heads, 256 nodes, 4096 rows: 163
// us, the tensor cores' floor 77); short items an item's start and end (4 x 8 heads,
// 64 nodes, 1024 rows: 19.5 us).
//
// The same kernel serves mkv_prefix_step (prefix_step.cu): its sequences are nodes without keys
// (no mask), and with PARTS a row's state (m, l, O), not yet divided by l, is what it leaves.
#include <limits.h>
#include <stddef.h>

#include <algorithm>
#include <mutex>

#include "common.cuh"
#include "kernels.h"
#include "tc.cuh"
#include "tree.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kTile = 128;                   // keys per tile, rows per block
constexpr int kBox = kTile * 128;            // bytes of 128 rows x 64 bf16
constexpr int kWarpTma = 8, kWarpMma = 9, kWarpCheck = 11, kWarpC = 12;
constexpr int kThreads = 512;                // 2 softmax groups; a TMA warp, two MMA warps, one for early loads; four for C'
constexpr int kScanUnits = 4096;             // units (and 2^30 tiles) above which every item has a CTA of its own
constexpr int kMinRun = 2;                   // tiles of a list's run at least
constexpr float kSlack = 32.f;               // the reference lies this far (log2) above the score that set it
constexpr float kNegInf = -INFINITY;
constexpr uint32_t kAll = 0xffffffffu;

__host__ __device__ constexpr int slot_bytes(int D) { return kTile * D * 2; }
__host__ __device__ constexpr int ring_slots(int D, int blocks) { return D == 128 ? (blocks == 2 ? 5 : 6) : 10; }
constexpr int kMaxSlots = 10;

struct Plan {
  int32_t blocks;   // row blocks per CTA: 1 or 2
  int32_t mb;       // items per unit
  int32_t g_shift;  // log2 of the group
  int32_t list;     // 1: runs of the tile list, 0: one item per CTA
  int32_t grid;
  int32_t min_run;  // tiles per CTA at least
  int32_t words;    // mask words per node
  uint64_t kv_inv;  // 2^40 / KV heads, rounded up: units (below 2^22) divided by a product, u * n_kv < 2^40
};

// A part of a split item (m, l, O of `blocks` x 128 rows).
struct Parts {
  int2* desc;   // [items]: the CTAs of its first and of its last part (the same: it is whole)
  float2* ml;   // [2 grid][blocks 128]
  float4* o;    // [2 grid][D / 4][blocks 128]
};

struct Raw {  // a unit's sizes as read
  int len, count, n_e;
};

struct Shared {
  uint64_t full[kMaxSlots], empty[kMaxSlots];
  uint64_t q_full, q_empty, c_grant, c_full, s_full[2], p_ready[2], turn[2], p_half[2], o_full, mma_done;
  uint32_t tmem;
  int32_t abort, issued, q_issued;
  int32_t unit, mb, t0, start, end;  // the CTA's run of the list: first item, tile in it, the list's tiles [start, end)
  Raw raw;                     // of the first unit
  int32_t run;                 // tiles per CTA before the ends are moved
  uint32_t seen[kThreads / 32];  // (early loads) the sizes that the run was made from, summed with weights
  uint32_t odd[2][8];          // nodes with a value that is not finite, of this segment and the next
  union {
    float2 ml[kTile];          // (one row block) group 1's (m, l), then the two groups' factors
    int32_t scan[kThreads / 32];  // (find_run, before that)
  };
  union alignas(16) {   // (read as float4)
    float mu_k[kTile];  // from a segment's start
    float w[kTile];     // (one row block) at its end: the moment term's factor
  };
};
constexpr int kSharedBytes = 2048;
static_assert(kSlack == 32.f, "log_sum");
static_assert(sizeof(Shared) <= kSharedBytes, "shared variables");
static_assert(offsetof(Shared, mu_k) % 16 == 0 && kSharedBytes % 16 == 0, "mu_k is read 16 bytes at a time");
__host__ __device__ constexpr int smem_bytes(int D, int blocks) {
  return (blocks + ring_slots(D, blocks)) * slot_bytes(D) + kSharedBytes + 1024;
}
static_assert(smem_bytes(128, 2) <= 232448 && smem_bytes(128, 1) <= 232448 && smem_bytes(64, 2) <= 232448, "227 KB");

// D[tmem] (+)= A[tmem] B over one k-step (16 elements, 8 columns of A).
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t db, uint32_t idesc,
                                             uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(db), "r"(idesc), "r"(accumulate));
}

// 32 columns of this warp's lanes, without waiting (tmem_wait_ld, then keep()).
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// The loaded registers may only be read from here on (orders their uses after the wait).
__device__ __forceinline__ void keep16(uint32_t* r) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
               "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Shared memory written by threads, next read by the tensor cores.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w,
                                            uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::
          "r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_addr(bar))
      : "memory");
}

// Two floats in one 64-bit register, and two operations per instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t x, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// s += two bf16 values, each in one instruction without widening it first
// (131072 rows, 33 nodes: 119 -> 112 us against shifts, masks and a sum of pairs).
__device__ __forceinline__ void add_rounded(float (&s)[2], uint32_t w) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.bf16 %0, a, %0;\n\tadd.rn.f32.bf16 %1, b, %1;\n\t}"
      : "+f"(s[0]), "+f"(s[1])
      : "r"(w));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// 2^d of a whole number d <= 0, exactly (0 below the smallest normal number).
__device__ __forceinline__ float pow2(float d) {
  return d < -126.f ? 0.f : __int_as_float((127 + static_cast<int>(d)) << 23);
}
// The natural log of a normaliser l about the reference m (the reference's headroom goes into l, exactly).
__device__ __forceinline__ float log_sum(float m, float l) {
  return l != 0.f ? (m - kSlack + log2f(l * 0x1p32f)) * kLn2 : kNegInf;
}
// O's columns of this warp's rows times the row's factor.  (Stores to tensor
// memory are not ordered before loads that follow them: those of an earlier
// scaling of the same tile are waited for.)
template <int D>
__device__ __forceinline__ void scale_columns(uint32_t tO, float f) {
  tmem_wait_st();
#pragma unroll 1
  for (int c = 0; c < D; c += 16) {
    uint32_t o[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]), "=r"(o[8]),
          "=r"(o[9]), "=r"(o[10]), "=r"(o[11]), "=r"(o[12]), "=r"(o[13]), "=r"(o[14]), "=r"(o[15])
        : "r"(tO + c));
    tmem_wait_ld();
    keep16(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
    tmem_st16(tO + c, o);
  }
}
// The weights (pairs of bf16) of the first n times 32 columns times the row's factor, a power of two.
// (They were stored by this warp a moment ago, which has to be complete.)
__device__ __forceinline__ void scale_weights(uint32_t tS, int n, float f) {
  tmem_wait_st();
#pragma unroll 1
  for (int c = 0; c < n; ++c) {
    uint32_t o[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]), "=r"(o[8]),
          "=r"(o[9]), "=r"(o[10]), "=r"(o[11]), "=r"(o[12]), "=r"(o[13]), "=r"(o[14]), "=r"(o[15])
        : "r"(tS + c * 16));
    tmem_wait_ld();
    keep16(o);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&o[i]));
      o[i] = pack_bf16x2(x.x * f, x.y * f);
    }
    tmem_st16(tS + c * 16, o);
  }
}

// Eight words of a row, at once where the address is a multiple of 32 bytes (the
// rows of a warp lie 256 bytes apart: the fewer stores the better).
__device__ __forceinline__ void store8(void* dst, const uint32_t* x, bool aligned32) {
  if (aligned32) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(x[0]), "r"(x[1]), "r"(x[2]),
                 "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(dst)[0] = make_uint4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<uint4*>(dst)[1] = make_uint4(x[4], x[5], x[6], x[7]);
  }
}

// Whether any of a word's two bf16 values is infinite or NaN.
__device__ __forceinline__ bool odd2(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}

// What a unit's items consist of.
struct Item {
  int len, count, n_e;
  int cache, nodes, tail;  // tiles: the cache, the nodes, the moment term (0 or 1)
};

__device__ __forceinline__ int batch_of(const Plan& p, int u) {
  return static_cast<int>((static_cast<uint64_t>(u) * p.kv_inv) >> 40);
}
__device__ __forceinline__ Raw load_raw(const TreeArgs& a, const Plan& p, int u) {
  return Raw{a.len[u], a.count != nullptr ? a.count[batch_of(p, u)] : a.N, a.n != nullptr ? a.n[u] : 0};
}
// The same from L2: what an early load left in L1 may be old.
__device__ __forceinline__ Raw reload_raw(const TreeArgs& a, const Plan& p, int u) {
  return Raw{__ldcg(a.len + u), a.count != nullptr ? __ldcg(a.count + batch_of(p, u)) : a.N,
             a.n != nullptr ? __ldcg(a.n + u) : 0};
}
// A unit's share of the sum by which sizes that changed under an early load are
// found: lengths that grow always change it, whichever they are (the sum of odd
// multiples stays below 2^32), anything else but for one case in 2^32.
__device__ __forceinline__ uint32_t raw_sum(int u, const Raw& r) {
  return (2u * u + 1u) * (static_cast<uint32_t>(r.len) + 0x9e3779b1u * static_cast<uint32_t>(r.count) +
                          0x85ebca6bu * static_cast<uint32_t>(r.n_e));
}
__device__ __forceinline__ Item make_item(const TreeArgs& a, const Raw& r) {
  Item it;
  it.len = min(max(r.len, 0), a.cap);
  it.count = min(max(r.count, 0), a.N);
  it.n_e = r.n_e;
  it.tail = a.n != nullptr ? 1 : 0;
  it.cache = (it.len + kTile - 1) / kTile;
  it.nodes = a.mask != nullptr ? (it.count + kTile - 1) / kTile : 0;
  return it;
}
// Tiles of an item whose rows start at node `first` (at least one: its outputs have to be written).
__device__ __forceinline__ int item_tiles(const Item& it, int first) {
  return first < it.count ? max(1, it.cache + it.nodes + it.tail) : 1;
}

// A CTA's next segment: tiles [begin, end) of item (unit, mb).
struct Segment {
  int unit, mb, first;  // first node of the item's rows
  int begin, end, tiles;
  int k0, k1;  // key tiles: the cache's, then the nodes'
  // Ring: K and V of every key tile, and before the last one or two tiles the
  // operands of C' (0 to 2 slots), so that they are made while those tiles run.
  int c_slots, c_tile;
  Item it;
  bool live, mom;  // rows in use; the moment term belongs to this segment
  __device__ __forceinline__ int slot(int j) const { return 2 * (j - k0) + (j >= c_tile ? c_slots : 0); }  // of K
  __device__ __forceinline__ int c_slot() const { return 2 * (c_tile - k0); }
  __device__ __forceinline__ int slots() const { return 2 * (k1 - k0) + c_slots; }
  // keys in use of key tile j
  __device__ __forceinline__ int valid(int j) const {
    return min(kTile, (j < it.cache ? it.len : it.count + it.cache * kTile) - j * kTile);
  }
};

struct Walk {
  int unit, mb, t, left;
  Raw raw;  // (read while the segment before is worked on)
  // With early loads the first unit's sizes are those that find_run read, the
  // same for every role, and the others are read when they are due, after the
  // dependency wait: the roles cannot disagree about sizes that changed.
  static constexpr int kDue = INT_MIN;  // as a count
  __device__ __forceinline__ bool next(const TreeArgs& a, const Plan& p, Segment& s) {
    if (left <= 0) return false;
    if (a.early && raw.count == kDue) {
      grid_dependency_wait();
      raw = reload_raw(a, p, unit);
    }
    s.unit = unit;
    s.mb = mb;
    s.first = mb * ((p.blocks * kTile) >> p.g_shift);
    s.it = make_item(a, raw);
    s.live = s.first < s.it.count;
    s.tiles = item_tiles(s.it, s.first);
    s.begin = t;
    s.end = min(s.tiles, t + left);
    const int keys = s.live ? s.it.cache + s.it.nodes : 0;
    s.mom = s.live && s.end == s.tiles && s.it.tail > 0 && s.it.n_e > 0;
    s.k0 = min(s.begin, keys);
    s.k1 = min(s.end, keys);
    s.c_slots = s.mom && a.order == 1 ? (a.C16 != nullptr ? 1 : 2) : 0;
    s.c_tile = max(s.k0, s.k1 - (p.blocks == 1 ? 2 : 1));
    left -= s.end - s.begin;
    t = 0;
    if (++mb == p.mb) {
      mb = 0;
      // (lengths written while the call runs cannot lead past the last unit)
      if (++unit == a.batch * a.n_kv) left = 0;
    }
    if (a.early) raw.count = kDue;
    else if (left > 0) raw = load_raw(a, p, unit);
    return true;
  }
};

// Pipeline wait that gives up after `polls` polls: records the timeout once and
// raises the CTA's abort flag; every later wait that has to poll then passes.
__device__ __noinline__ void record_bad(void* ws, uint32_t code, int32_t info) { record_error(ws, code, info); }
__device__ __noinline__ bool pwait_slow(uint64_t* bar, uint32_t parity, int32_t* abort, void* ws, uint32_t polls) {
  volatile int32_t* flag = abort;
  if (*flag) return false;
  if (mbar_wait(bar, parity, polls)) return true;
  *flag = 1;
  record_error(ws, MKV_ERR_TIMEOUT, static_cast<int32_t>(blockIdx.x));
  return false;
}
__device__ __forceinline__ bool pwait(uint64_t* bar, uint32_t parity, Shared& sh, const TreeArgs& a) {
  return (a.polls > 0 && mbar_try_wait(bar, parity)) || pwait_slow(bar, parity, &sh.abort, a.ws, a.polls);
}

// Where this CTA's run starts in the list of all items' tiles, and whether its
// start cuts an item
// (`mine`: the sizes of unit threadIdx.x, read ahead).
__device__ __forceinline__ void find_run(const TreeArgs& a, const Plan& p, Shared& sh, const Raw& mine) {
  const int tid = threadIdx.x, units = a.batch * a.n_kv;
  const int nodes = (p.blocks * kTile) >> p.g_shift;  // of an item
  auto record = [&](int u, const Raw& r) {
    if (static_cast<uint32_t>(r.len) > static_cast<uint32_t>(a.cap)) record_bad(a.ws, MKV_ERR_CAPACITY, u);
    if (static_cast<uint32_t>(r.count) > static_cast<uint32_t>(a.N)) record_bad(a.ws, MKV_ERR_INVALID_ARG, u);
  };
  if (!p.list) {
    if (tid == 0) {
      sh.unit = blockIdx.x / p.mb;
      sh.mb = blockIdx.x % p.mb;
      sh.t0 = 0;
      sh.raw = load_raw(a, p, sh.unit);
      sh.start = 0;
      sh.end = item_tiles(make_item(a, sh.raw), sh.mb * nodes);
      if (sh.mb == 0) record(sh.unit, sh.raw);
    }
    __syncthreads();
    return;
  }
  // a unit's items with rows in use (the others weigh one tile each), and the tiles of one
  auto weigh = [&](const Raw& r, int& tiles) {
    const Item it = make_item(a, r);
    tiles = item_tiles(it, 0);
    return (it.count + nodes - 1) / nodes;
  };
  const int chunk = (units + kThreads - 1) / kThreads, u0 = min(units, tid * chunk), u1 = min(units, u0 + chunk);
  int sum = 0;
  uint32_t seen = 0;
#pragma unroll 1
  for (int u = u0; u < u1; ++u) {
    const Raw r = chunk == 1 ? mine : load_raw(a, p, u);
    int tiles;
    const int alive = weigh(r, tiles);
    sum += alive * tiles + (p.mb - alive);
    seen += raw_sum(u, r);
    if (blockIdx.x == 0) record(u, r);
  }
  if (a.early) {
    seen = __reduce_add_sync(kAll, seen);
    if ((tid & 31) == 0) sh.seen[tid >> 5] = seen;
  }
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, incl, o);
    if ((tid & 31) >= o) incl += x;
  }
  if ((tid & 31) == 31) sh.scan[tid >> 5] = incl;
  if (tid == 0) {
    sh.start = sh.end = 0;
  }
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    const int x = sh.scan[w];
    if (w < (tid >> 5)) before += x;
    total += x;
  }
  const int run = max(p.min_run, (total + p.grid - 1) / p.grid);
  const int at = before + incl - sum;  // of this thread's first unit
  if (tid == 0) sh.run = run;
  // The run is [start, end) with both ends moved off an item's first and last
  // tile, to the item's edge: no CTA is left with the moment term alone or with
  // one tile to begin with.
#pragma unroll 1
  for (int edge = 0; edge < 2; ++edge) {
    const int pos = run * (blockIdx.x + edge);
    if (tid == 0 && pos >= total) (edge == 0 ? sh.start : sh.end) = total;
    if (pos < at || pos >= at + sum) continue;
    int u = u0, tiles, alive, w, base = at;
    Raw r;
#pragma unroll 1
    for (;; ++u) {
      r = chunk == 1 ? mine : load_raw(a, p, u);
      alive = weigh(r, tiles);
      w = alive * tiles + (p.mb - alive);
      if (pos < base + w || u + 1 == u1) break;  // (sizes read anew may have changed: no further)
      base += w;
    }
    int in = pos - base, mb = 0;  // the unit's tiles before `pos`
    while (mb < alive && in >= tiles) in -= tiles, ++mb;
    if (mb == alive) mb = min(mb + in, p.mb - 1), in = 0;
    const int item = pos - in;  // where the item starts
    int snap = pos;
    if (in > 0) {
      if (tiles - in <= 1) snap = item + tiles;
      else if (in <= 1) snap = item;
    }
    if (edge == 1) {
      sh.end = min(snap, total);
      continue;
    }
    if (snap == item + tiles && in > 0) {  // the next item
      if (++mb == p.mb) {
        mb = 0;
        if (++u == units) {  // there is none
          sh.start = total;
          continue;
        }
        r = load_raw(a, p, u);
      }
    }
    sh.unit = u;
    sh.mb = mb;
    sh.t0 = in > 0 && snap == pos ? in : 0;
    sh.raw = r;
    sh.start = snap;
  }
  __syncthreads();
}

// With early loads, one warp after the dependency wait: sizes that differ from
// those that this CTA's run was made from are recorded.
__device__ __noinline__ void check_early(const TreeArgs& a, const Plan& p, const Shared& sh) {
  const int lane = threadIdx.x & 31, units = a.batch * a.n_kv;
  grid_dependency_wait();
  uint32_t diff = 0;
  if (p.list) {
    if (lane < kThreads / 32) diff = 0u - sh.seen[lane];
#pragma unroll 4
    for (int u = lane; u < units; u += 32) diff += raw_sum(u, reload_raw(a, p, u));
    diff = __reduce_add_sync(kAll, diff);
  }
  if (lane != 0) return;
  if (sh.end > sh.start) {
    const Raw r = reload_raw(a, p, sh.unit);
    diff |= (r.len ^ sh.raw.len) | (r.count ^ sh.raw.count) | (r.n_e ^ sh.raw.n_e);
  }
  if (diff != 0) record_bad(a.ws, MKV_ERR_INVALID_ARG, sh.end > sh.start ? sh.unit : 0);
}

template <int D, int BLOCKS, bool PARTS>
__global__ void __launch_bounds__(kThreads, 1)
    tree_step_kernel(const __grid_constant__ TreeArgs a, const __grid_constant__ Plan p,
                     const __grid_constant__ Parts parts, const __grid_constant__ CUtensorMap tmQ,
                     const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ CUtensorMap tmKt, const __grid_constant__ CUtensorMap tmVt) {
  constexpr int kSlot = slot_bytes(D), NS = ring_slots(D, BLOCKS), BX = D / 64;
  // With two row blocks P is handed over in halves, so that its product with V
  // starts during the second half's exponentials (131072 rows: 123 us without,
  // 112 with it; with one block, where the ring is the limit, 2% slower).
  constexpr bool kHalf = BLOCKS == 2;
  constexpr uint32_t cS = 0, cO = 256;  // TMEM columns: S / P of group s at 128 s, O at 256 + D s
  extern __shared__ __align__(1024) uint8_t smraw[];
  uint8_t* sm = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smraw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = sm;
  uint8_t* ring = sm + BLOCKS * kSlot;
  Shared& sh = *reinterpret_cast<Shared*>(ring + NS * kSlot);

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (warp == kWarpTma && lane < 5) {
    const CUtensorMap* map = lane == 0 ? &tmQ : lane == 1 ? &tmK : lane == 2 ? &tmV : lane == 3 ? &tmKt : &tmVt;
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
  }
  if (!a.early) grid_dependency_wait();
  Raw mine{};  // in flight while the barriers are set up
  if (tid < a.batch * a.n_kv) mine = load_raw(a, p, tid);
  if (tid < NS) {
    mbar_init(&sh.full[tid], 1);
    mbar_init(&sh.empty[tid], BLOCKS);  // the groups that read a slot
  } else if (tid >= 32 && tid < 34) {
    mbar_init(&sh.s_full[tid - 32], 1);
    mbar_init(&sh.p_ready[tid - 32], 4);
    mbar_init(&sh.turn[tid - 32], 4);
    mbar_init(&sh.p_half[tid - 32], 4);
  } else if (tid == 64) {
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_empty, 2 + 8);
    mbar_init(&sh.c_grant, 1);
    mbar_init(&sh.c_full, 4);
    mbar_init(&sh.o_full, 2);
    mbar_init(&sh.mma_done, 2);
    sh.abort = 0;
    sh.issued = 0;
    sh.q_issued = 0;
  } else if (tid >= 96 && tid < 112) {
    (&sh.odd[0][0])[tid - 96] = 0;
  }
  mbar_fence_init();
  if (warp == kWarpMma) tmem_alloc(&sh.tmem, 512);
  tc_fence_before();
  find_run(a, p, sh, mine);  // (ends with a barrier)
  tc_fence_after();
  const uint32_t tm = sh.tmem;
  Walk walk{sh.unit, sh.mb, sh.t0, sh.end - sh.start, sh.raw};
  Segment s;

  if (warp == kWarpTma) {
    if (lane == 0) {  // ---- TMA
      int seq = 0, nq = 0, c_last = -1;  // c_last: the last slot given to C'
      bool ok = true, waited = !a.early;
      const uint64_t pol = l2_evict_first();
      auto wait_prior = [&] {
        if (!waited) grid_dependency_wait();
        waited = true;
        grid_launch_dependents();
      };
      auto slot = [&]() -> int {  // the next slot of the ring, free
        const int i = seq % NS;
        if (seq >= NS && !pwait(&sh.empty[i], ((seq / NS) - 1) & 1, sh, a)) ok = false;
        return i;
      };
      while (ok && walk.next(a, p, s)) {
        if (!s.mom && s.k1 == s.k0) continue;
        const int b = batch_of(p, s.unit), kv = s.unit - b * a.n_kv;
        if (s.c_slots > 0) {  // C' is read when slots are free: into L2 now
          const size_t at = (size_t)s.unit * D * D;
          const void* c = a.C16 != nullptr ? static_cast<const void*>(a.C16 + at)
                          : a.Cs != nullptr ? static_cast<const void*>(a.Cs + at / 2)
                                            : static_cast<const void*>(a.C + at);
          asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(c), "r"(D * D * (a.C16 != nullptr ? 2 : 4))
                       : "memory");
        }
        bool q_due = true;
        for (int j = s.k0; ok && j <= s.k1; ++j) {
          const bool cache = j < s.it.cache;
          // Q as soon as it may be replaced, but after the first tile at the
          // latest; before what precedes this launch is done, only the cache's
          // tiles, as many as the ring holds
          if (q_due && (!waited ? (!cache || j == s.k1 || j == s.c_tile || seq + 2 > NS)
                                : (j != s.k0 || j == s.k1 || nq == 0 || mbar_try_wait(&sh.q_empty, (nq - 1) & 1)))) {
            wait_prior();
            if (nq > 0 && !pwait(&sh.q_empty, (nq - 1) & 1, sh, a)) {
              ok = false;
              break;
            }
            mbar_arrive_expect_tx(&sh.q_full, BLOCKS * kSlot);
            for (int r = 0; r < BLOCKS; ++r)
              for (int x = 0; x < BX; ++x)
                tma_load_4d(sQ + r * kSlot + x * kBox, &tmQ, x * 64, kv << p.g_shift, s.first + r * (kTile >> p.g_shift), b,
                            &sh.q_full);
            sh.q_issued = ++nq;
            q_due = false;
          }
          if (j == s.c_tile && s.c_slots > 0) {
            // one C' at a time: the phases of c_grant and c_full do not tell one
            // from the next but one (a slot used again since has been waited for)
            if (c_last >= 0 && seq <= c_last + NS && !pwait(&sh.empty[c_last % NS], (c_last / NS) & 1, sh, a)) {
              ok = false;
              break;
            }
            for (int k = 0; ok && k < s.c_slots; ++k) {
              const int i = slot();
              if (!ok) break;
              mbar_arrive(&sh.full[i]);
              sh.issued = ++seq;
            }
            if (!ok) break;
            c_last = seq - 1;
            mbar_arrive(&sh.c_grant);
          }
          if (j == s.k1) break;
#pragma unroll 1
          for (int v = 0; ok && v < 2; ++v) {
            const int i = slot();
            if (!ok) break;
            mbar_arrive_expect_tx(&sh.full[i], kSlot);
            for (int x = 0; x < BX; ++x) {
              uint8_t* dst = ring + i * kSlot + x * kBox;
              if (cache)
                tma_load_3d_hint(dst, v ? &tmV : &tmK, x * 64, j * kTile, s.unit, &sh.full[i], pol);
              else
                tma_load_4d(dst, v ? &tmVt : &tmKt, x * 64, kv, (j - s.it.cache) * kTile, b, &sh.full[i]);
            }
            sh.issued = ++seq;
          }
        }
      }
      wait_prior();
    }
  } else if (warp == kWarpMma || warp == kWarpMma + 1) {
    if (lane == 0) {  // ---- MMA, a thread per group
      const int g = warp - kWarpMma;
      const bool reads_c = BLOCKS == 2 || g == 0;  // the moment term counts in this group's state
      const uint64_t dQ = sdesc_sw128(smem_addr(sQ) + (BLOCKS == 2 ? g * kSlot : 0), 16, 1024);
      const uint64_t dR = sdesc_sw128(smem_addr(ring), 16, 1024), dV = sdesc_sw128(smem_addr(ring), kBox, 1024);
      const uint32_t tP = tm + cS + g * 128, tO = tm + cO + g * D;
      constexpr uint32_t idS = idesc_bf16(128, kTile, 0, 0), idP = idesc_bf16(128, D, 0, 1);
      constexpr int kStep = BLOCKS == 2 ? 2 : 4;  // ring slots from one K tile of this group to the next
      int seq = 0;                                // ring slots of the segments before
      uint32_t qph = 0, cph = 0, pph = 0, f_ph = 0;  // (with halves: pph is p_half's, f_ph p_ready's)
      bool ok = true, f_read = false;
      // S = Q K^T of the tile in slot i (n16 keys)
      auto issue_s = [&](int i, int n16) {
        const uint64_t db = dR + i * (kSlot >> 4);
        const uint32_t id = idS - ((uint32_t)(kTile - n16) >> 3 << 17);
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          umma_bf16(tP, dQ + (kk >> 2) * (kBox >> 4) + (kk & 3) * 2, db + (kk >> 2) * (kBox >> 4) + (kk & 3) * 2, id,
                    kk > 0 ? 1u : 0u);
        umma_commit(&sh.s_full[g]);
        umma_commit(&sh.empty[i]);
      };
      while (ok && walk.next(a, p, s)) {
        const int k0 = s.k0, k1 = s.k1;
        if (!s.mom && k0 == k1) continue;
        ok = pwait(&sh.q_full, qph, sh, a);
        qph ^= 1;
        if (f_read && reads_c) {  // the last segment's Q C'^T has been read
          uint32_t& ready = kHalf ? f_ph : pph;
          ok = ok && pwait(&sh.p_ready[g], ready, sh, a);
          ready ^= 1;
        }
        f_read = false;
        int t = k0 + (BLOCKS == 2 ? 0 : g);
        int i = seq + s.slot(t);  // slot and phase of the K tile; V is in the next slot
        uint32_t ph = (i / NS) & 1;
        i %= NS;
        uint32_t add = 0;
        int n16 = (s.valid(t) + 15) & ~15;
        if (ok && t < k1) {
          ok = pwait(&sh.full[i], ph, sh, a);
          tc_fence_after();
          if (ok) issue_s(i, n16);
        }
#pragma unroll 1
        while (ok && t < k1) {
          const int steps = n16 >> 4;
          int vi = i + 1, ni = i + s.slot(t + kStep / 2) - s.slot(t);
          uint32_t vph = ph, nph = ph;
          if (vi >= NS) vi -= NS, vph ^= 1;
          if (ni >= NS) ni -= NS, nph ^= 1;
          t += kStep / 2;
          n16 = t < k1 ? (s.valid(t) + 15) & ~15 : 0;
          const uint64_t db = dV + vi * (kSlot >> 4);
          // (P first: it is ready only after the slot's use before has been
          // consumed -- with one row block that is the other thread's, and a
          // phase's parity alone would not tell the two apart)
          ok = pwait(kHalf ? &sh.p_half[g] : &sh.p_ready[g], pph, sh, a) && pwait(&sh.full[vi], vph, sh, a);
          if (!ok) break;
          tc_fence_after();
          if (steps == 8) {
            umma_bf16_ts(tO, tP, db, idP, add);
#pragma unroll
            for (int kk = 1; kk < 4; ++kk) umma_bf16_ts(tO, tP + kk * 8, db + kk * 128, idP, 1u);
          }
          if (kHalf) {
            ok = pwait(&sh.p_ready[g], f_ph, sh, a);
            f_ph ^= 1;
            if (!ok) break;
            tc_fence_after();
          }
          pph ^= 1;
          if (steps == 8) {
#pragma unroll
            for (int kk = 4; kk < 8; ++kk) umma_bf16_ts(tO, tP + kk * 8, db + kk * 128, idP, 1u);
          } else {
#pragma unroll 1
            for (int kk = 0; kk < steps; ++kk) umma_bf16_ts(tO, tP + kk * 8, db + kk * 128, idP, kk == 0 ? add : 1u);
          }
          add = 1;
          umma_commit(&sh.empty[vi]);
          if (n16 > 0) {
            // (K's slot: with one row block and one slot of C' the ring is shifted
            // by an odd number, so that V of the other thread's tile t - 3 had it,
            // which nothing this thread has waited for implies.  Until that use is
            // released K's phase must not be asked for: its parity is that of the
            // use before.  With 0 or 2 slots of C', or 10 in the ring, this thread's
            // or an earlier tile had the slot, and S or P of t - 2 implies its release.)
            if (BLOCKS == 1 && s.c_slots == 1 && seq + s.slot(t) >= NS)
              ok = pwait(&sh.empty[ni], nph ^ 1, sh, a);
            ok = ok && pwait(&sh.full[ni], nph, sh, a);
            if (!ok) break;
            tc_fence_after();
            issue_s(ni, n16);
          }
          i = ni, ph = nph;
        }
        if (ok && s.c_slots > 0) {  // the moment term's value, Q C'^T, in the place of S
          if (reads_c) {
            ok = pwait(&sh.c_full, cph, sh, a);
            cph ^= 1;
            if (!ok) break;
            tc_fence_after();
            constexpr uint32_t id = idesc_bf16(128, D, 0, 0);
#pragma unroll 1
            for (int j = 0; j < s.c_slots; ++j) {
              const int ci = (seq + s.c_slot() + j) % NS;
              const uint64_t db = dR + ci * (kSlot >> 4);
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk)
                umma_bf16(tP, dQ + (kk >> 2) * (kBox >> 4) + (kk & 3) * 2, db + (kk >> 2) * (D * 128 >> 4) + (kk & 3) * 2,
                          id, (j > 0 || kk > 0) ? 1u : 0u);
              umma_commit(&sh.empty[ci]);
            }
          }
          f_read = true;
        }
        seq += s.slots();
        umma_commit(&sh.q_empty);
        umma_commit(&sh.o_full);
      }
      umma_commit(&sh.mma_done);
    }
  } else if (warp >= kWarpC) {
    // ---- C' as the operand of Q C'^T: 16-byte chunks of 8 columns, hi and lo parts
    constexpr int kBatch = 4, kRounds = D * D / 8 / 128 / kBatch;
    const int t = tid - kWarpC * 32;
    uint32_t seq = 0, cph = 0;
    while (walk.next(a, p, s)) {
      if (!s.mom && s.k0 == s.k1) continue;
      const uint32_t c_seq = seq + s.c_slot();
      seq += s.slots();
      if (s.c_slots == 0) continue;
      const float nf = static_cast<float>(s.it.n_e);
      uint8_t* hi = ring + (c_seq % NS) * kSlot;
      uint8_t* lo = ring + ((c_seq + 1) % NS) * kSlot;
      const size_t base = (size_t)s.unit * D * D;
#pragma unroll 1
      for (int k = 0; k < kRounds; ++k) {
        uint4 x[kBatch], y[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const size_t at = base + ((k * kBatch + j) * 128 + t) * 8;
          const uint4* src = a.C16 != nullptr ? reinterpret_cast<const uint4*>(a.C16 + at)
                             : a.Cs != nullptr ? reinterpret_cast<const uint4*>(a.Cs + at / 2)
                                               : reinterpret_cast<const uint4*>(a.C + at);
          x[j] = src[0];
          y[j] = a.C16 == nullptr ? src[1] : make_uint4(0, 0, 0, 0);
        }
        if (k == 0) {
          (void)pwait(&sh.c_grant, cph, sh, a);
          cph ^= 1;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int c = (k * kBatch + j) * 128 + t;
          const uint32_t off = swz_off(c / (D / 8), (c % (D / 8)) * 8, D);
          if (a.Cs != nullptr) {
            *reinterpret_cast<uint4*>(hi + off) = make_uint4(x[j].x, x[j].z, y[j].x, y[j].z);
            *reinterpret_cast<uint4*>(lo + off) = make_uint4(x[j].y, x[j].w, y[j].y, y[j].w);
            continue;
          }
          uint32_t w[8] = {x[j].x, x[j].y, x[j].z, x[j].w, y[j].x, y[j].y, y[j].z, y[j].w}, h[4];
          if (a.C16 != nullptr) {
#pragma unroll
            for (int i = 3; i >= 0; --i) {
              w[2 * i + 1] = w[i] & 0xffff0000u;
              w[2 * i] = w[i] << 16;
            }
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (fabsf(__uint_as_float(w[i]) * nf) < a.tau) w[i] = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) h[i] = pack_bf16x2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
          *reinterpret_cast<uint4*>(hi + off) = make_uint4(h[0], h[1], h[2], h[3]);
          if (a.C16 == nullptr) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              h[i] = pack_bf16x2(__uint_as_float(w[2 * i]) - __uint_as_float(h[i] << 16),
                                 __uint_as_float(w[2 * i + 1]) - __uint_as_float(h[i] & 0xffff0000u));
            *reinterpret_cast<uint4*>(lo + off) = make_uint4(h[0], h[1], h[2], h[3]);
          }
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.c_full);
    }
  } else if (warp == kWarpCheck) {
    if (a.early) check_early(a, p, sh);
  } else if (warp < kWarpTma) {
    // ---- softmax groups: thread r of group g has row r of a block
    const int g = warp >> 2, r = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // this warp's 32 TMEM lanes
    const uint32_t tS = tm + lanes + cS + g * 128, tO = tm + lanes + cO + g * D;
    const float scale = rsqrtf(static_cast<float>(D)), qs = scale * kLog2e;
    const int G = 1 << p.g_shift, HQ = a.n_kv << p.g_shift;
    constexpr int kCols = BLOCKS == 2 ? D : D / 2;  // columns of the output that a thread writes, from c_lo on
    const int c_lo = BLOCKS == 2 ? 0 : g * (D / 2);
    uint32_t nq = 0, ns = 0, no = 0, vseq = 0;  // phases passed; ring slots of the segments before
    uint32_t tph = 0;
    const bool aligned_out = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
    if (g == 1 && lane == 0) mbar_arrive(&sh.turn[0]);  // group 0 begins
    int seg = 0, at = sh.start;  // the list's tile that the segment begins with
    while (walk.next(a, p, s)) {
      const bool mom = s.mom;
      const int k0 = s.k0, k1 = s.k1, b = batch_of(p, s.unit), kv = s.unit - b * a.n_kv;
      const bool active = mom || k1 > k0;
      const int node = s.first + ((BLOCKS == 2 ? g * kTile + r : r) >> p.g_shift), h = r & (G - 1);
      const bool live = node < s.it.count;
      const bool warp_live = __any_sync(kAll, live);
      const bool mine = BLOCKS == 2 || g == 0;  // the moment term counts in this group's state
      float m = kNegInf, l = 0.f, lr = 0.f, e = kNegInf;  // lr: the sum of the rounded weights
      bool filled = false;  // O holds something
      float mv[kCols / 32] = {};  // mu_v: this lane's columns of those that the thread writes
      if (mom) {
        if (tid < D) sh.mu_k[tid] = a.mu_k[(size_t)s.unit * D + tid];
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k) mv[k] = a.mu_v[(size_t)s.unit * D + c_lo + k * 32 + lane];
        named_sync(1, 256);
        (void)pwait(&sh.q_full, nq & 1, sh, a);
        if (mine) {
          float e0 = 0.f, e1 = 0.f;
          const uint8_t* row = sQ + (BLOCKS == 2 ? g * kSlot : 0) + r * 128;
#pragma unroll 2
          for (int c = 0; c < D / 8; ++c) {
            const uint4 w = *reinterpret_cast<const uint4*>(row + (c >> 3) * kBox + (((c & 7) ^ (r & 7)) << 4));
            const uint32_t x[4] = {w.x, w.y, w.z, w.w};
            const float4 ka = *reinterpret_cast<const float4*>(&sh.mu_k[c * 8]);
            const float4 kb = *reinterpret_cast<const float4*>(&sh.mu_k[c * 8 + 4]);
            const float k[8] = {ka.x, ka.y, ka.z, ka.w, kb.x, kb.y, kb.z, kb.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x[i]));
              e0 = fmaf(f.x, k[2 * i], e0);
              e1 = fmaf(f.y, k[2 * i + 1], e1);
            }
          }
          e = fmaf(e0 + e1, qs, log2f(static_cast<float>(s.it.n_e)));
          m = ceilf(e) + kSlack;
          l = lr = e != kNegInf ? fast_exp2(e - m) : 0.f;  // (without weight no term; a NaN passes on)
        }
      }
      if (active) {
        ++nq;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_empty);  // (with the MMA threads' commits: Q may be replaced)
      }
      const uint32_t seg_seq = vseq;  // of the first K tile
      vseq += s.slots();
      // The groups take turns at the exponentials: left to themselves they fell
      // into step, and both waited for the special-function units and then for
      // the tensor cores (4200 cycles a tile of 256 rows instead of 3000).
      const int turns = BLOCKS == 2 ? k1 - k0 : (k1 - k0 + 1) >> 1;
      for (int turn = 0; turn < turns; ++turn) {
        const int j = BLOCKS == 2 ? k0 + turn : k0 + 2 * turn + g;
        if (BLOCKS == 1 && j >= k1) {  // (an odd number of tiles: group 1 passes)
          (void)pwait(&sh.turn[g], tph, sh, a);
          tph ^= 1;
          if (lane == 0) mbar_arrive(&sh.turn[g ^ 1]);
          break;
        }
        const int valid = s.valid(j);
        const bool tree = j >= s.it.cache;
        uint32_t words[4];  // the keys of this tile that the row sees
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int n = valid - i * 32;
          words[i] = n >= 32 ? kAll : n <= 0 ? 0u : (1u << n) - 1u;
        }
        if (tree) {
          const int w0 = (j - s.it.cache) * 4;
          const uint32_t* row = a.mask + ((size_t)b * a.N + node) * p.words + w0;
#pragma unroll
          for (int i = 0; i < 4; ++i) words[i] &= live && w0 + i < p.words ? row[i] : 0u;
        }
        (void)pwait(&sh.s_full[g], ns & 1, sh, a);
        ++ns;
        (void)pwait(&sh.turn[g], tph, sh, a);
        tph ^= 1;
        if (tree || valid % 16 != 0) {
          // (in turn: the other group's products with what the slot held before
          // are complete.)  V rows past the keys in use must be finite (their weights are 0),
          // and so must a node's value where its weight is 0: elements that
          // are not are taken out here and reach the nodes that see them at
          // the end
          const uint32_t sv = seg_seq + s.slot(j) + 1;
          uint8_t* tv = ring + (sv % NS) * kSlot;
          (void)pwait(&sh.full[sv % NS], (sv / NS) & 1, sh, a);
          const int end = (valid + 15) & ~15;
          for (int c = r; c < (end - valid) * (D / 8); c += kTile) {
            const int row = valid + c / (D / 8), x = c % (D / 8);
            *reinterpret_cast<uint4*>(tv + (x >> 3) * kBox + row * 128 + ((x & 7) << 4)) = make_uint4(0, 0, 0, 0);
          }
          if (tree) {
            for (int c = r; c < valid * (D / 8); c += kTile) {
              const int row = c / (D / 8), x = c % (D / 8);
              uint4* at = reinterpret_cast<uint4*>(tv + (x >> 3) * kBox + row * 128 + ((x & 7) << 4));
              uint4 w = *at;
              if (odd2(w.x) || odd2(w.y) || odd2(w.z) || odd2(w.w)) {
                const int n = (j - s.it.cache) * kTile + row;
                atomicOr(&sh.odd[seg & 1][n >> 5], 1u << (n & 31));
                __threadfence_block();  // (the other group may find the zeros instead)
                uint32_t* y = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  if ((y[i] & 0x7f80u) == 0x7f80u) y[i] &= 0xffff0000u;
                  if ((y[i] & 0x7f800000u) == 0x7f800000u) y[i] &= 0xffffu;
                }
                *at = w;
              }
            }
          }
          fence_async_smem();
        }
        tc_fence_after();
        if (warp_live && !tree && valid == kTile) {
          // a tile without a mask: its maximum, then its weights, the next 32
          // columns on their way while 32 are worked on
          uint32_t x[4][32];
          float mx[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
          tmem_ld32_async(tS, x[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_wait_ld();
            keep16(x[c]), keep16(x[c] + 16);
            if (c < 3) tmem_ld32_async(tS + (c + 1) * 32, x[c + 1]);
#pragma unroll
            for (int i = 0; i < 32; i += 2)
              mx[(i >> 1) & 3] = max3(mx[(i >> 1) & 3], __uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1]));
          }
          const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * qs;
          if (__any_sync(kAll, top > m)) {
            const float mn = fmaxf(m, ceilf(top) + kSlack);
            const float f = m == kNegInf ? 1.f : pow2(m - mn);
            m = mn;
            l *= f, lr *= f;
            if (filled) scale_columns<D>(tO, f);  // (S of this tile is complete, so every product into O is)
          }
          const float ref = m == kNegInf ? 0.f : m;
          const uint64_t qs2 = pair(qs, qs), nref = pair(-ref, -ref);
          uint64_t sum2[2] = {0, 0};
          float sumr[2] = {0.f, 0.f};
          uint32_t y[4][32];
          tmem_ld32_async(tS, y[0]);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            tmem_wait_ld();
            keep16(y[c]), keep16(y[c] + 16);
            if (c < 3) tmem_ld32_async(tS + (c + 1) * 32, y[c + 1]);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float t0, t1;
              unpair(fma2(pair(__uint_as_float(y[c][i]), __uint_as_float(y[c][i + 1])), qs2, nref), t0, t1);
              const float p0 = fast_exp2(t0), p1 = fast_exp2(t1);
              const uint32_t pr = pack_bf16x2(p0, p1);
              sum2[(i >> 1) & 1] = add2(sum2[(i >> 1) & 1], pair(p0, p1));
              add_rounded(sumr, pr);
              y[c][i >> 1] = pr;
            }
            tmem_st16(tS + c * 16, y[c]);
            if (kHalf && c == 1) {  // the first half of the product with V may begin
              tmem_wait_st();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.p_half[g]);
            }
          }
          float lo, hi;
          unpair(add2(sum2[0], sum2[1]), lo, hi);
          l += lo + hi;
          lr += sumr[0] + sumr[1];
          tmem_wait_st();
        } else if (warp_live) {
          // 32 columns at a time; a reference that has to move (by a whole
          // number: the factor is exact) takes O, l and the weights already
          // written of this tile along.  (P's columns lie below those of S that
          // are still to be read.)
          const uint64_t qs2 = pair(qs, qs);
#pragma unroll 1
          for (int c = 0; c * 32 < valid; ++c) {
            uint64_t sum2 = 0;
            float sumr[2] = {0.f, 0.f};
            uint32_t x[32];
            tmem_ld32_async(tS + c * 32, x);
            const uint32_t word = c == 0 ? words[0] : c == 1 ? words[1] : c == 2 ? words[2] : words[3];
            tmem_wait_ld();
            keep16(x);
            keep16(x + 16);
            if (word != kAll) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!((word >> i) & 1u)) x[i] = 0xff800000u;  // -inf
            }
            float mx[4] = {kNegInf, kNegInf, kNegInf, kNegInf};
#pragma unroll
            for (int i = 0; i < 32; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(x[i]));
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * qs;
            if (__any_sync(kAll, top > m)) {
              const float mn = fmaxf(m, ceilf(top) + kSlack);
              const float f = m == kNegInf ? 1.f : pow2(m - mn);
              m = mn;
              l *= f, lr *= f;
              if (filled) scale_columns<D>(tO, f);  // (S of this tile is complete, so every product into O is)
              scale_weights(tS, c, f);
            }
            const float ref = m == kNegInf ? 0.f : m;
            const uint64_t nref = pair(-ref, -ref);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              float t0, t1;
              unpair(fma2(pair(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), qs2, nref), t0, t1);
              const float p0 = fast_exp2(t0), p1 = fast_exp2(t1);
              const uint32_t pr = pack_bf16x2(p0, p1);
              sum2 = add2(sum2, pair(p0, p1));
              add_rounded(sumr, pr);
              x[i >> 1] = pr;
            }
            tmem_st16(tS + c * 16, x);
            float lo, hi;
            unpair(sum2, lo, hi);
            l += lo + hi;
            lr += sumr[0] + sumr[1];
          }
          tmem_wait_st();
        }
        filled = true;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (kHalf && (!warp_live || tree || valid < kTile)) mbar_arrive(&sh.p_half[g]);
          mbar_arrive(&sh.p_ready[g]);
          mbar_arrive(&sh.turn[g ^ 1]);
        }
      }

      // ---- the segment's state: into the output (a whole item) or the workspace
      if (active) {
        (void)pwait(&sh.o_full, no & 1, sh, a);
        ++no;
        tc_fence_after();
      }
      grid_dependency_wait();  // (a no-op unless the loads went early)
      const bool whole = s.begin == 0 && s.end == s.tiles;
      // An item's first part says where the others are: the last boundary that
      // stays inside it is the last at or below its tile tiles - 2.
      if (p.list && s.begin == 0 && tid == 0)
        parts.desc[s.unit * p.mb + s.mb] = make_int2(blockIdx.x, whole ? blockIdx.x : min((at + s.tiles - 2) / sh.run, p.grid - 1));
      at += s.end - s.begin;
      const int part = 2 * blockIdx.x + (s.begin == 0 ? 1 : 0);  // an item's start: this CTA's last segment; else its first
      constexpr int R = BLOCKS * kTile;
      bool any_odd = false;
      const float even = lr != 0.f ? l / lr : 1.f;  // what O lacks for the weights' roundings
      if (BLOCKS == 1 && g == 1) {
        sh.ml[r] = make_float2(m, l);
        if (k1 > k0 + 1) sh.w[r] = even;  // (group 0 is past its use of mu_k: it has taken a turn)
      }
      named_sync(1, 256);  // the other group's state; the nodes' odd values are known
      auto seen_odd = [&](int w) {
        return w < p.words ? sh.odd[seg & 1][w] & a.mask[((size_t)b * a.N + node) * p.words + w] : 0u;
      };
      if (live && k1 > s.it.cache) {
#pragma unroll
        for (int i = 0; i < 8; ++i) any_odd |= sh.odd[seg & 1][i] != 0;
      }
      // output = f0 O_0 + f1 O_1 + w (mu_v + scale F) over the columns this thread writes
      float M = m, L = l, f0 = L != 0.f ? even : 0.f, f1 = 0.f;
      if (BLOCKS == 1 && g == 0) {
        const float2 y = sh.ml[r];
        M = fmaxf(L != 0.f ? m : kNegInf, y.y != 0.f ? y.x : kNegInf);
        const float ref = M == kNegInf ? 0.f : M;
        f0 = L != 0.f ? fast_exp2(m - ref) : 0.f;
        f1 = y.y != 0.f ? fast_exp2(y.x - ref) : 0.f;
        L = (L != 0.f ? L * f0 : 0.f) + (y.y != 0.f ? y.y * f1 : 0.f);
        f0 *= even;
        if (k1 > k0 + 1) f1 *= sh.w[r];
      }
      float w = mom && mine && e != kNegInf ? fast_exp2(e - M) * even : 0.f;
      if (whole && !PARTS) {
        const float inv = L != 0.f ? 1.f / L : 0.f;
        f0 *= inv, f1 *= inv, w *= inv;
      }
      if (BLOCKS == 1) {
        if (g == 0) {
          sh.ml[r] = make_float2(f0, f1);
          sh.w[r] = w;
        }
        named_sync(1, 256);
        f0 = sh.ml[r].x, f1 = sh.ml[r].y, w = sh.w[r];
      }
      // a factor of 0 stands for a state without content: its columns may hold anything
      const bool use0 = f0 != 0.f && k1 > k0, use1 = f1 != 0.f && k1 > k0 + 1, use_f = mom && a.order == 1;
      const float wf = w * scale;
      const bool absent = __any_sync(kAll, wf == 0.f);  // a term without weight is absent, whatever Q C'^T came to
      const bool put = node < a.N;
      const size_t orow = ((size_t)b * a.N + node) * HQ + (kv << p.g_shift) + h;
      const uint32_t tA = tm + lanes + cO + (BLOCKS == 2 ? g * D : 0) + c_lo, tB = tA + D;
      const uint32_t tF = tm + lanes + cS + (BLOCKS == 2 ? g * 128 : 0) + c_lo;
#pragma unroll 1
      for (int c = 0; c < kCols; c += 32) {
        uint32_t x[32], y[32];
        tmem_ld32_async(tA + c, x);
        if (BLOCKS == 1) tmem_ld32_async(tB + c, y);
        tmem_wait_ld();
        keep16(x), keep16(x + 16);
        if (BLOCKS == 1) keep16(y), keep16(y + 16);
        float o[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          o[i] = use0 ? __uint_as_float(x[i]) * f0 : 0.f;
          if (BLOCKS == 1 && use1) o[i] = fmaf(__uint_as_float(y[i]), f1, o[i]);
        }
        if (mom) {
          if (use_f) {
            tmem_ld32_async(tF + c, x);
            tmem_wait_ld();
            keep16(x), keep16(x + 16);
            if (absent) {
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = wf == 0.f ? 0u : x[i];
            }
          }
          float m32 = mv[0];
#pragma unroll
          for (int k = 1; k < kCols / 32; ++k)
            if (c == 32 * k) m32 = mv[k];
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            o[i] = fmaf(__shfl_sync(kAll, m32, i), w, o[i]);
            if (use_f) o[i] = fmaf(__uint_as_float(x[i]), wf, o[i]);
          }
        }
        if (PARTS && whole) {
          if (live) {
            float* dst = a.state_o + orow * D + c_lo + c;
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(o[i]);
#pragma unroll
            for (int i = 0; i < 32; i += 8) store8(dst + i, x + i, true);
          }
        } else if (whole) {
          if (put) {
            __nv_bfloat16* dst = a.out + orow * D + c_lo + c;
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] = live ? pack_bf16x2(o[2 * i], o[2 * i + 1]) : 0u;
            store8(dst, x, aligned_out);
            store8(dst + 16, x + 8, aligned_out);
          }
        } else if (warp_live) {  // (rows that are not in use are not joined)
          const int row = BLOCKS == 2 ? g * kTile + r : r;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            parts.o[((size_t)part * (D / 4) + (c_lo + c) / 4 + i) * R + row] =
                make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
        }
      }
      if (any_odd && (put || !whole)) {
        // the values that are not finite join the row's columns one by one
        const int row = BLOCKS == 2 ? g * kTile + r : r;
#pragma unroll 1
        for (int n = 0; n < s.it.count; ++n) {
          const int j = s.it.cache + (n >> 7);
          if (j < k0 || j >= k1 || !((seen_odd(n >> 5) >> (n & 31)) & 1u)) continue;
          const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(a.v) + b * a.kv_batch + n * a.kv_node + kv * D;
#pragma unroll 1
          for (int c = c_lo; c < c_lo + kCols; ++c) {
            const float z = __bfloat162float(v[c]);
            if (isfinite(z)) continue;
            if (whole) {
              a.out[orow * D + c] = __float2bfloat16_rn(__bfloat162float(a.out[orow * D + c]) + z);
            } else {
              float* o = reinterpret_cast<float*>(&parts.o[((size_t)part * (D / 4) + c / 4) * R + row]) + (c & 3);
              *o += z;
            }
          }
        }
      }
      if (BLOCKS == 2 || g == 0) {
        if (PARTS && whole) {
          if (live) a.state_ml[orow] = make_float2(M, L);
        } else if (whole) {
          if (put && a.lse != nullptr) a.lse[orow] = live ? log_sum(M, L) : kNegInf;
        } else if (warp_live) {
          parts.ml[(size_t)part * R + (BLOCKS == 2 ? g * kTile + r : r)] = make_float2(M, L);
        }
      }
      if (tid < 8) sh.odd[(seg + 1) & 1][tid] = 0;  // (read last in the segment before)
      ++seg;
      tc_fence_before();
      named_sync(1, 256);  // both groups are done with O, Q C'^T and the exchange
      if (use_f && mine && lane == 0) mbar_arrive(&sh.p_ready[g]);
    }
  }

  __syncthreads();
  if (warp == kWarpMma) {
    if (lane == 0) {
      if (sh.abort) {  // wait, with the full limit, for the copies in flight
        for (int i = 0; i < NS; ++i) {
          const int last = sh.issued - 1 - ((sh.issued - 1 - i) % NS + NS) % NS;  // the last use of slot i
          if (last >= 0) (void)mbar_wait(&sh.full[i], (last / NS) & 1);
        }
        if (sh.q_issued > 0) (void)mbar_wait(&sh.q_full, (sh.q_issued - 1) & 1);
      }
      (void)mbar_wait(&sh.mma_done, 0);  // no product or arrival is left
    }
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tm, 512);
  }
}

// Joins the parts of the items that a boundary of the list cuts.  Bounded by
// latency: as many threads as the GPU holds at once are best, each with all of
// its loads in flight.  A warp has 32 rows x 4 Q columns of an item; P warps
// share them where there are few, every P-th part each.
template <int D, int P, int Q, bool PARTS>
__global__ void __launch_bounds__(256) tree_merge_kernel(const __grid_constant__ TreeArgs a,
                                                         const __grid_constant__ Plan p,
                                                         const __grid_constant__ Parts parts) {
  constexpr int kCols = D / (4 * Q);  // column groups of an item
  __shared__ float2 s_ml[P > 1 ? 8 : 1][32];
  __shared__ float4 s_o[P > 1 ? 8 : 1][Q][32];
  grid_dependency_wait();
  grid_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wp = warp % P;
  const int id = blockIdx.x * (8 / P) + warp / P;  // (item, row block, column group, 32 rows)
  const int c4 = (id >> 2) % kCols * Q, z = (id >> 2) / kCols % p.blocks, item = (id >> 2) / kCols / p.blocks;
  const int u = item / p.mb, mb = item - u * p.mb;
  const int2 d = parts.desc[item];  // (the same item in all warps of a block: it has at least 16 groups)
  if (d.x == d.y) return;
  // (an item that no CTA began, as lengths that changed during the call can leave it, has an old record)
  if (static_cast<uint32_t>(d.x) >= static_cast<uint32_t>(p.grid) || static_cast<uint32_t>(d.y) >= static_cast<uint32_t>(p.grid))
    return;
  const int R = p.blocks * kTile, row = z * kTile + (id & 3) * 32 + lane;
  const int G = 1 << p.g_shift, b = batch_of(p, u), kv = u - b * a.n_kv;
  const int node = mb * (R >> p.g_shift) + (row >> p.g_shift), h = row & (G - 1);
  const int n = d.y - d.x + 1;
  float M = kNegInf, L = 0.f, acc[4 * Q] = {};
  if (node < a.N && node < (a.count != nullptr ? a.count[b] : a.N)) {
    // parts: the end of CTA d.x, then the starts of those up to d.y
    auto part = [&](int i) { return (size_t)(2 * (d.x + i) + (i == 0 ? 1 : 0)); };
#pragma unroll 4
    for (int i = wp; i < n; i += P) {
      const float2 x = parts.ml[part(i) * R + row];
      const float4* src = parts.o + (part(i) * (D / 4) + c4) * R + row;
      float4 o[Q];
#pragma unroll
      for (int k = 0; k < Q; ++k) o[k] = src[k * R];
      if (x.y != 0.f) {  // (a part without content may hold anything)
        const float mn = fmaxf(M, x.x), ref = mn == kNegInf ? 0.f : mn;
        const float f0 = L != 0.f ? fast_exp2(M - ref) : 0.f, f = fast_exp2(x.x - ref);
        M = mn;
        L = L * f0 + x.y * f;
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          acc[4 * k] = fmaf(o[k].x, f, acc[4 * k] * f0);
          acc[4 * k + 1] = fmaf(o[k].y, f, acc[4 * k + 1] * f0);
          acc[4 * k + 2] = fmaf(o[k].z, f, acc[4 * k + 2] * f0);
          acc[4 * k + 3] = fmaf(o[k].w, f, acc[4 * k + 3] * f0);
        }
      }
    }
  }
  if constexpr (P > 1) {
    s_ml[warp][lane] = make_float2(M, L);
#pragma unroll
    for (int k = 0; k < Q; ++k) s_o[warp][k][lane] = make_float4(acc[4 * k], acc[4 * k + 1], acc[4 * k + 2], acc[4 * k + 3]);
    __syncthreads();
    if (wp != 0) return;
    for (int w = 1; w < min(P, n); ++w) {
      const float2 x = s_ml[warp + w][lane];
      if (x.y == 0.f) continue;
      const float mn = fmaxf(M, x.x), ref = mn == kNegInf ? 0.f : mn;
      const float f0 = L != 0.f ? fast_exp2(M - ref) : 0.f, f = fast_exp2(x.x - ref);
      M = mn;
      L = L * f0 + x.y * f;
#pragma unroll
      for (int k = 0; k < Q; ++k) {
        const float4 o = s_o[warp + w][k][lane];
        acc[4 * k] = fmaf(o.x, f, acc[4 * k] * f0);
        acc[4 * k + 1] = fmaf(o.y, f, acc[4 * k + 1] * f0);
        acc[4 * k + 2] = fmaf(o.z, f, acc[4 * k + 2] * f0);
        acc[4 * k + 3] = fmaf(o.w, f, acc[4 * k + 3] * f0);
      }
    }
  }
  if (node >= a.N) return;
  const size_t orow = ((size_t)b * a.N + node) * (a.n_kv << p.g_shift) + (kv << p.g_shift) + h;
  if constexpr (PARTS) {
#pragma unroll
    for (int k = 0; k < Q; ++k)
      reinterpret_cast<float4*>(a.state_o + orow * D)[c4 + k] =
          make_float4(acc[4 * k], acc[4 * k + 1], acc[4 * k + 2], acc[4 * k + 3]);
    if (c4 == 0) a.state_ml[orow] = make_float2(M, L);
    return;
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;
#pragma unroll
  for (int k = 0; k < Q; ++k)
    reinterpret_cast<uint2*>(a.out + orow * D)[c4 + k] =
        L != 0.f ? make_uint2(pack_bf16x2(acc[4 * k] * inv, acc[4 * k + 1] * inv),
                              pack_bf16x2(acc[4 * k + 2] * inv, acc[4 * k + 3] * inv))
                 : make_uint2(0, 0);
  if (c4 == 0 && a.lse != nullptr) a.lse[orow] = log_sum(M, L);
}

// Tiles of an item at most.
long max_tiles(int key_nodes, int capacity) {
  return 1 + ((long)capacity + kTile - 1) / kTile + (key_nodes + kTile - 1) / kTile;
}
// CTAs of a list of so many tiles at most.
int list_grid(long tiles, int num_sms) {
  return static_cast<int>(std::min<long>(num_sms, (tiles + kMinRun - 1) / kMinRun));
}

// (key_nodes: the nodes that are keys too, all or none)
Plan make_plan(const mkv_geom& g, int n_nodes, int key_nodes, int capacity, int num_sms) {
  Plan p{};
  const int rows = n_nodes * g.group;
  p.g_shift = g.group == 8 ? 3 : g.group == 4 ? 2 : g.group == 2 ? 1 : 0;
  p.words = tree_words(n_nodes);
  p.kv_inv = ((1ull << 40) + g.n_kv_heads - 1) / g.n_kv_heads;
  p.min_run = kMinRun;
  const long units = (long)g.batch * g.n_kv_heads;
  const long tiles = max_tiles(key_nodes, capacity);
  const auto items = [&](int blocks) { return units * ((rows + blocks * kTile - 1) / (blocks * kTile)); };
  // One row block per CTA spreads few, short items over more SMs; two read K and
  // V once for 256 rows.  Measured, one and two: 4 x 8 heads, 64 nodes of 4
  // heads, 1024 rows 19.6 and 28.2 us, 4096 rows 41.7 and 40.5; 16 x 8 heads,
  // 512 rows 35.1 and 25.5; 8 heads, 33 nodes, 131072 rows 164 and 112; 8 x 8
  // heads, 256 nodes, 4096 rows 203 and 165.
  p.blocks = rows > kTile && (items(1) > num_sms || items(2) * tiles >= 8l * num_sms) ? 2 : 1;
  const long n = items(p.blocks);
  p.mb = static_cast<int>(n / units);
  // One CTA per item leaves SMs idle in the last wave, by the tiles that even
  // runs would save; the list costs its records, the cut items' second ends and
  // the merge.  A tile takes 0.9 us with one row block (1.4 where HBM bounds
  // it).  Measured, list and whole items, (idle tiles): 8 items of 5 tiles 13.9
  // and 11.7 us (3), of 10 14.5 and 16.7 (8), of 18 15.3 and 23.8 (16); 64 items
  // of 10 22.0 and 19.5 (6), of 18 33.7 and 27.1 (11); 32 items of 35 29.8 and
  // 40.0 (28); 128 items of 18 42.5 and 32.1 (3).  More items than SMs: 256 of
  // 10 56.2 and 42.3 (4), of 34 ragged 93.5 and 89.7 (11), of 66 170 and 174
  // (21); 512 of 18 135 and 123 (12); 320 of 18 87.9 and 89.1 (17); 192 of 34
  // 82.5 and 92.3 (26); with two row blocks 256 of 18 105 and 93 (6), of 35 164
  // and 163 (12), 320 of 18 122 and 131 (17).
  const long run = std::max<long>(p.min_run, n * tiles / num_sms), waves = (n + num_sms - 1) / num_sms;
  const bool whole = waves * tiles - run <= (n <= num_sms ? 3 + n / 5 : 13);
  p.list = units <= kScanUnits && n * tiles < (1L << 30) && !whole ? 1 : 0;
  p.grid = p.list ? list_grid(n * tiles, num_sms) : static_cast<int>(n);
  return p;
}

// Bytes of the parts' records of a list plan.
size_t parts_bytes(long items, int blocks, int grid, int D) {
  return align_up(static_cast<size_t>(items) * sizeof(int2), 256) +
         2 * static_cast<size_t>(grid) * blocks * kTile * (8 + static_cast<size_t>(D) * 4);
}

// bf16 [n3][n2][n1][inner] with the strides of n1, n2, n3 in elements; boxes of b1 x b2 rows of 64 elements.
bool encode_4d(CUtensorMap* map, const void* base, uint64_t inner, uint64_t n1, uint64_t n2, uint64_t n3, uint64_t s1,
               uint64_t s2, uint64_t s3, uint32_t b1, uint32_t b2) {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(f);
  });
  if (fn == nullptr) return false;
  const cuuint64_t dims[4] = {inner, n1, n2, n3}, strides[3] = {s1 * 2, s2 * 2, s3 * 2};
  const cuuint32_t box[4] = {64, b1, b2, 1}, step[4] = {1, 1, 1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int BLOCKS, bool PARTS>
cudaError_t launch_step(const TreeArgs& a, const Plan& p, const Parts& parts, const CUtensorMap (&tm)[5],
                        int num_sms, cudaStream_t stream) {
  constexpr int smem = smem_bytes(D, BLOCKS);
  cudaError_t e = cudaFuncSetAttribute(tree_step_kernel<D, BLOCKS, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  e = launch_pdl(tree_step_kernel<D, BLOCKS, PARTS>, dim3(p.grid), dim3(kThreads), smem, stream, a, p, parts, tm[0], tm[1], tm[2],
                 tm[3], tm[4]);
  if (e != cudaSuccess || !p.list) return e;
  // threads if each had 4 columns of a row: at most grid - 1 items are cut, and
  // the GPU holds 2048 threads per SM
  const long items = (long)a.batch * a.n_kv * p.mb, units = items * BLOCKS * (D / 4) * 4;
  const long cut = std::min<long>(items, p.grid) * BLOCKS * kTile * (D / 4), most = 2048l * num_sms;
  const auto merge = [&](auto kernel, int P, int Q) {
    return launch_pdl(kernel, dim3(static_cast<unsigned>(units * P / Q / 8)), dim3(256), 0, stream, a, p, parts);
  };
  if (cut * 8 <= most) return merge(tree_merge_kernel<D, 8, 1, PARTS>, 8, 1);
  if (cut * 4 <= most) return merge(tree_merge_kernel<D, 4, 1, PARTS>, 4, 1);
  if (cut * 2 <= most) return merge(tree_merge_kernel<D, 2, 1, PARTS>, 2, 1);
  if (cut <= most) return merge(tree_merge_kernel<D, 1, 1, PARTS>, 1, 1);
  return merge(tree_merge_kernel<D, 1, 4, PARTS>, 1, 4);
}

template <bool PARTS>
cudaError_t launch_tree(const TreeArgs& args, const mkv_geom& g, int num_sms, cudaStream_t stream) {
  TreeArgs a = args;
  a.polls = pipeline_poll_limit();
  const Plan p = make_plan(g, a.N, a.mask != nullptr ? a.N : 0, a.cap, num_sms);
  Parts parts{};
  const int D = g.head_dim, R = p.blocks * kTile;
  uint8_t* w = static_cast<uint8_t*>(a.parts);
  parts.desc = reinterpret_cast<int2*>(w);
  w += align_up((size_t)a.batch * a.n_kv * p.mb * sizeof(int2), 256);
  parts.o = reinterpret_cast<float4*>(w);
  w += 2 * (size_t)p.grid * R * D * 4;
  parts.ml = reinterpret_cast<float2*>(w);
  const uint64_t hq = (uint64_t)a.n_kv * g.group, units = (uint64_t)a.batch * a.n_kv, d = D;
  CUtensorMap tm[5];
  if (!encode_4d(&tm[0], a.q, d, hq, a.N, a.batch, d, a.q_node, a.q_batch, g.group, kTile / g.group) ||
      !encode_tmap_bf16_3d(&tm[1], a.K, d, a.cap, units, d * 2, (uint64_t)a.cap * d * 2, kTile) ||
      !encode_tmap_bf16_3d(&tm[2], a.V, d, a.cap, units, d * 2, (uint64_t)a.cap * d * 2, kTile))
    return cudaErrorInvalidValue;
  tm[3] = tm[4] = tm[0];  // (nodes without keys: not read)
  if (a.mask != nullptr &&
      (!encode_4d(&tm[3], a.k, d, a.n_kv, a.N, a.batch, d, a.kv_node, a.kv_batch, 1, kTile) ||
       !encode_4d(&tm[4], a.v, d, a.n_kv, a.N, a.batch, d, a.kv_node, a.kv_batch, 1, kTile)))
    return cudaErrorInvalidValue;
  if (D == 128)
    return p.blocks == 2 ? launch_step<128, 2, PARTS>(a, p, parts, tm, num_sms, stream)
                         : launch_step<128, 1, PARTS>(a, p, parts, tm, num_sms, stream);
  return p.blocks == 2 ? launch_step<64, 2, PARTS>(a, p, parts, tm, num_sms, stream)
                       : launch_step<64, 1, PARTS>(a, p, parts, tm, num_sms, stream);
}

// Bytes of the parts' records, enough for the plan of every batch, number of
// nodes and capacity up to these: plans change with each of them, and only
// lists have parts, so that a smaller tree can need more than a larger one.
size_t tree_parts_bytes(const mkv_geom& g, int32_t n_nodes, int32_t key_nodes, int32_t capacity, int num_sms) {
  const long units = std::min<long>((long)g.batch * g.n_kv_heads, kScanUnits), rows = (long)n_nodes * g.group;
  const long tiles = max_tiles(key_nodes, capacity);
  size_t most = 0;
  for (int blocks = 1; blocks <= (rows > kTile ? 2 : 1); ++blocks) {
    const long items = units * ((rows + blocks * kTile - 1) / (blocks * kTile));
    most = std::max(most, parts_bytes(items, blocks, list_grid(items * tiles, num_sms), g.head_dim));
  }
  return most;
}

}  // namespace

size_t tree_workspace_bytes(const mkv_geom& g, int32_t n_nodes, int32_t capacity, int num_sms) {
  return kHeaderBytes + tree_parts_bytes(g, n_nodes, n_nodes, capacity, num_sms);
}

cudaError_t launch_tree_step(const TreeArgs& args, const mkv_geom& g, int num_sms, cudaStream_t stream) {
  TreeArgs a = args;
  a.parts = static_cast<uint8_t*>(a.ws) + kHeaderBytes;
  return launch_tree<false>(a, g, num_sms, stream);
}

size_t prefix_tree_bytes(const mkv_geom& g, int32_t n_seqs, int32_t capacity, int num_sms) {
  return tree_parts_bytes(g, n_seqs, 0, capacity, num_sms);
}

cudaError_t launch_prefix_tree(const TreeArgs& a, const mkv_geom& g, int num_sms, cudaStream_t stream) {
  return launch_tree<true>(a, g, num_sms, stream);
}

}  // namespace mkv
