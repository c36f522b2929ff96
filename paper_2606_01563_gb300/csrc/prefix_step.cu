// One decoding step of several sequences that share a prompt's retained rows
// and moments, each with a tail of its own (mkv_prefix_step).
//
// Mathematics.  A query row (sequence, head) attends over the shared rows, its
// sequence's tail, its new token and the moment term of the shared prompt's
// evicted tokens, in one normaliser.  Any set of keys is a state (m, l, O): a
// reference, the sum of 2^(x - m) over its logits x (log2 domain) and the sum of
// values so weighted; states join by rescaling to the larger reference.  The
// moment term is a state too: m = log2 n + scale log2 e q.mu_k, l = 1, O = mu_v +
// scale C' q; and so is the new token.
//
// Two launches, or three to four.  prefix_parts_kernel leaves states ("parts") of every query row in
// the workspace: a block takes a run of the shared rows for up to 8 NT query
// rows of a unit (all sequences' heads side by side, so that a shared row is read
// once for all of them), or 64 dims of the moment term for as many, or tails, one
// a warp.  prefix_join_kernel joins each row's parts and the new token and
// appends that token to its tail.  For many query rows over many shared rows the kernels of
// tree_step.cu (one, and a second where it cuts items) take the shared rows, between the two.
//
// A run: a warp issues 64-row TMA copies into a ring; four warps work on every
// tile together.  Each takes the logits of 16 of its rows, S^T = K q^T with the keys on
// the 16-row side and the query rows on the 8-column side, and writes their
// weights, rounded to bf16, to shared memory; then each takes a quarter of the
// value dims over all 64 rows, O^T += V^T P^T.  So a query row's O is held once (8 NT registers a thread at
// 128 dims), up to 32 query rows share a shared row's one trip, and no states of
// warps are merged.  One barrier a tile: the weights have two buffers.  A reference
// lies 32 (log2) above the score that set it and moves when a score exceeds it, which every warp learns
// at that barrier.  O is scaled by the ratio of the unrounded weights' sum to the
// rounded ones', so that roundings that are common cancel; those that are not
// leave the output off by up to 2^-8 of the values' mean magnitude, half a step of its own
// type (measured against 64 bits 0.0017, a form with weights in 32 bits 0.0016-0.0017).
//
// What bounds it: HBM with few query rows over a long prompt (4 sequences of 8 x 4
// heads, 65536 rows: 43.5-45 us, 0.88-0.91 of 6.8 TB/s); with 32 the chain of a tile, 1
// us (8 sequences, 65536 rows: 50 us; its kernel, with four column tiles at 128 dims,
// has 168 registers and spills 80 bytes); short prompts the two launches' chains
// (4 sequences, 128 rows: 6.0 us; 8 sequences of 4 prompts, 1024 rows, tails of 100: 15).
// Splits follow capacities, since the host does not know the lengths: tails of
// capacity 1024 or 4096 that hold 4 rows cost those 8 sequences 16.6-16.9 us, of
// capacity 8 11.3 (13 sequences of 8 prompts, 4001 rows: 49.6 and 42.8).
#include <algorithm>
#include <cmath>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "tree.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kWarps = 4;                   // that attend
constexpr int kThreads = (kWarps + 1) * 32;  // and one that loads
constexpr int kRows = 64;                   // rows of a tile
constexpr int kMinTiles = 2;   // of a run, where there are as many
constexpr int kMaxSplits = 64;
constexpr int kMaxTails = 8;   // tails of a warp
// Visits of 64-row tiles by blocks of up to 32 query rows, per place and at 128
// dims, above which several such blocks of a unit give way to tcgen05.  Measured
// at 8 heads of 4, here and there (visits a place): 16 sequences over 16384
// rows 26 and 34 us (14), 24 over 8192 23 and 26 (10), 32 x 2 prompts over 2048 21
// and 26 (7); 64 over 4096 32 and 28 (14), 64 x 4 over 1024 44 and 39 (14), 32 x 2
// over 8192 55 and 38 (27), 24 over 32768 61 and 45 (40).  A unit's only block
// keeps its rows: 8 sequences over 65536 49 and 59 (27).  The first of these cases is on
// the wrong side: visits alone do not tell two blocks of a unit, which do well here
// for longer, from eight.
constexpr long kVisits = 12;
constexpr float kSlack = 32.f;  // log2 headroom of a reference above the score that set it (weights at most 1)
constexpr float kNegInf = -INFINITY;
constexpr int kJoinThreads = 256;

__host__ __device__ constexpr int tile_bytes(int D) { return kRows * D * 2; }
__host__ __device__ constexpr int stages(int D) { return D == 64 ? 4 : 3; }
constexpr int kMaxStages = 4;
// Rows of q and of the weights lie 16 bytes apart beyond their length: ldmatrix meets no bank twice.
__host__ __device__ constexpr int q_pitch(int D) { return D * 2 + 16; }
constexpr int kPPitch = kRows * 2 + 16;
// The query rows go into registers, and their place in shared memory is one of the weights' two buffers.
__host__ __device__ constexpr int p_offset(int D, int NT, int buffer) { return buffer == 0 ? 0 : 8 * NT * q_pitch(D); }
__host__ __device__ constexpr int qp_bytes(int D, int NT) { return p_offset(D, NT, 1) + 8 * NT * kPPitch; }
__host__ __device__ constexpr int parts_smem(int D, int NT) { return stages(D) * 2 * tile_bytes(D) + qp_bytes(D, NT) + 1024; }
static_assert(2 * (parts_smem(128, 4) + 3 * 1024) <= 228 * 1024, "two blocks to an SM");

// A query row of a unit: sequence r / G, head r % G.
__device__ __forceinline__ int out_row(const PrefixArgs& a, int b, int kv, int r) {
  return (((b * a.N + (r >> a.g_shift)) * a.n_kv + kv) << a.g_shift) + (r & (a.group - 1));
}
__device__ __forceinline__ int live_seqs(const PrefixArgs& a, int b) {
  return a.count != nullptr ? min(max(a.count[b], 0), a.N) : a.N;
}

constexpr int kMaxCols = 32;  // query rows of a block at most
struct PartsShared {
  uint64_t full[kMaxStages], empty[kMaxStages];
  uint64_t own[kWarps][kMaxStages];  // tails: a ring a warp
  float l[kWarps][kMaxCols][2];  // of a warp and column: the weights' sum and the rounded ones'
  float top[kWarps][kMaxCols];   // a moving reference: the warps' largest scores
  float mu_k[128];
  int moved[2];  // the last tile (counted from 1) of either buffer in which a score passed its reference
  int fail;
};

__device__ __forceinline__ bool failed(const PartsShared& sh) { return *reinterpret_cast<const volatile int*>(&sh.fail) != 0; }
// A warp's wait on a tile (every lane's, and the lanes stay together: what follows
// is the warp's as one).  One that runs out fails the block, whose later waits then
// end at once.  From there on no tile is asked for: a copy into a place
// whose last one was not waited for would count against that one's phase, and the
// block could end with copies in flight.  (The warps of a run meet their barriers
// as ever; what they compute is not used.)
__device__ __forceinline__ bool wait_tile(uint64_t* bar, uint32_t parity, PartsShared& sh, uint32_t polls) {
  for (uint32_t i = 0; i < polls; ++i) {
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    if ((i & 63) == 63 && __any_sync(0xffffffffu, failed(sh))) return false;
  }
  *reinterpret_cast<volatile int*>(&sh.fail) = 1;
  __syncwarp();
  return false;
}

// The loading warp's part of a run of n rows: one thread, tiles seq, seq + 1, ... of the block.
template <int D, int NS>
__device__ __forceinline__ void load_run(const PrefixArgs& a, const CUtensorMap* tmK, const CUtensorMap* tmV, int row0, int n,
                                         uint8_t* ring, PartsShared& sh, uint32_t& seq) {
  constexpr int kTile = tile_bytes(D);
  const uint64_t pol = l2_evict_first();
  for (int i = 0; i * kRows < n; ++i) {
    const uint32_t st = seq % NS;
    // (a place may have been released by warps whose own wait had given up)
    if (seq >= NS && (!mbar_wait(&sh.empty[st], ((seq / NS) - 1) & 1, a.polls) || failed(sh))) {
      *reinterpret_cast<volatile int*>(&sh.fail) = 1;
      return;
    }
    uint8_t* dst = ring + (size_t)st * 2 * kTile;
    mbar_arrive_expect_tx(&sh.full[st], 2u * kTile);
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
      tma_load_2d_hint(dst + x * kRows * 128, tmK, x * 64, row0 + i * kRows, &sh.full[st], pol);
      tma_load_2d_hint(dst + kTile + x * kRows * 128, tmV, x * 64, row0 + i * kRows, &sh.full[st], pol);
    }
    ++seq;
  }
}

// s += two bf16 values, each in one instruction without widening it first.
__device__ __forceinline__ void add_rounded(float (&s)[2], uint32_t w) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tadd.rn.f32.bf16 %0, a, %0;\n\tadd.rn.f32.bf16 %1, b, %1;\n\t}"
      : "+f"(s[0]), "+f"(s[1])
      : "r"(w));
}

// Shared memory read or written by threads, next written by a bulk copy.
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Columns nt (and nt + 1, with four registers) of rows of q or of the weights as B
// operands: 8 columns x 16 values of their rows.
__device__ __forceinline__ void ldsm_b2(uint32_t& r0, uint32_t& r1, const uint8_t* p) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0,%1}, [%2];" : "=r"(r0), "=r"(r1) : "r"(smem_addr(p)));
}

// The state of a run of n rows for `cols` query rows (in sm, zeros past cols) into
// part `part`; row_of(c) is column c's output row.  The four attending warps.
template <int D, int NT, int NS, typename RowOf>
__device__ __forceinline__ void attend_run(const PrefixArgs& a, int n, int cols, int part, uint8_t* ring, uint8_t* sm,
                                           PartsShared& sh, uint32_t& seq, RowOf row_of) {
  constexpr int KS = D / 16, MW = D / 64, kTile = tile_bytes(D);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int tiles = (n + kRows - 1) / kRows, r0 = warp * 16;
  const float qscale = rsqrtf(static_cast<float>(D)) * kLog2e;
  // A column's reference, before scaling: kSlack above the score that set it.
  const float slack = kSlack / qscale;
  auto reference = [&](float x) { return x == kNegInf ? 0.f : x * qscale; };
  float most[NT][2], l[NT][2], lr[NT][2], o[NT][MW][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    most[nt][0] = most[nt][1] = kNegInf;
    l[nt][0] = l[nt][1] = lr[nt][0] = lr[nt][1] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MW; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
  }
  const uint8_t* q_at = sm + (lane & 7) * q_pitch(D) + ((lane >> 3) & 1) * 16;  // (lanes 0-15)
  uint32_t qf[NT][KS][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) ldsm_b2(qf[nt][kk][0], qf[nt][kk][1], q_at + nt * 8 * q_pitch(D) + kk * 32);
  named_sync(1, kWarps * 32);  // (the weights may be written over q)
  const int kr = r0 + (lane & 7) + ((lane >> 3) & 1) * 8, kc = (lane >> 4) * 8;
  const int vr = (lane & 7) + (lane >> 4) * 8, vc = warp * (D / 4) + ((lane >> 3) & 1) * 8;
  for (int it = 0; it < tiles; ++it, ++seq) {
    (void)wait_tile(&sh.full[seq % NS], (seq / NS) & 1, sh, a.polls);
    const int rows = min(kRows, n - it * kRows);
    const uint8_t* tK = ring + (size_t)(seq % NS) * 2 * kTile;
    uint8_t* tV = ring + (size_t)(seq % NS) * 2 * kTile + kTile;
    uint8_t* sP = sm + p_offset(D, NT, it & 1);
    if (rows < r0 + 16) {  // V rows past the end are zeroed: their weights are 0, but they may hold anything
      const int from = max(rows, r0);
      for (int i = lane; i < (r0 + 16 - from) * (D / 8); i += 32) {
        const int r = from + i / (D / 8), c = (i % (D / 8)) * 8;
        *reinterpret_cast<uint4*>(tV + (c >> 6) * kRows * 128 + r * 128 + (c & 63) * 2) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    float s[NT][4];
    if constexpr (NT == 1) {  // two chains: one would wait for itself
      float c[2][4] = {};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        uint32_t k4[4];
        ldsm_x4(k4, tK + swz_off(kr, kk * 16 + kc, kRows));
        mma_m16n8k16(c[kk & 1], k4[0], k4[1], k4[2], k4[3], qf[0][kk][0], qf[0][kk][1]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[0][i] = c[0][i] + c[1][i];
    } else {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        uint32_t k4[4];
        ldsm_x4(k4, tK + swz_off(kr, kk * 16 + kc, kRows));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          mma_m16n8k16(s[nt], k4[0], k4[1], k4[2], k4[3], qf[nt][kk][0], qf[nt][kk][1]);
        }
      }
    }
    // lane (g, t): keys r0 + g (0, 1) and r0 + g + 8 (2, 3), columns 2t (0, 2) and 2t + 1 (1, 3)
    bool moves = false;
    if (rows < kRows) {
      const bool va = r0 + g < rows, vb = r0 + g + 8 < rows;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        s[nt][0] = va ? s[nt][0] : kNegInf, s[nt][1] = va ? s[nt][1] : kNegInf;
        s[nt][2] = vb ? s[nt][2] : kNegInf, s[nt][3] = vb ? s[nt][3] : kNegInf;
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
      moves |= fmaxf(s[nt][0], s[nt][2]) > most[nt][0] || fmaxf(s[nt][1], s[nt][3]) > most[nt][1];
    // the weights, and what they add to the sums (taken once the references are known to hold)
    float dl[NT][2], dr[NT][2];
    auto weigh = [&]() {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float ma = reference(most[nt][0]), mb = reference(most[nt][1]);
        const float x0 = fast_exp2(fmaf(s[nt][0], qscale, -ma)), x1 = fast_exp2(fmaf(s[nt][1], qscale, -mb));
        const float x2 = fast_exp2(fmaf(s[nt][2], qscale, -ma)), x3 = fast_exp2(fmaf(s[nt][3], qscale, -mb));
        const uint32_t h0 = pack_bf16x2(x0, x1), h1 = pack_bf16x2(x2, x3);
        dl[nt][0] = x0 + x2;
        dl[nt][1] = x1 + x3;
        dr[nt][0] = dr[nt][1] = 0.f;
        add_rounded(dr[nt], h0);
        add_rounded(dr[nt], h1);
        uint8_t* p = sP + (nt * 8 + g) * kPPitch + (r0 + 2 * t) * 2;  // [column][key]
        *reinterpret_cast<uint32_t*>(p) = movmatrix_t(h0);
        *reinterpret_cast<uint32_t*>(p + 16) = movmatrix_t(h1);
      }
    };
    if (__any_sync(0xffffffffu, moves)) {
      if (lane == 0) *reinterpret_cast<volatile int*>(&sh.moved[it & 1]) = it + 1;
      __syncwarp();
    } else {
      weigh();
    }
    named_sync(1, kWarps * 32);
    // Past the barrier all four warps have read the tile before.  (Released by each warp
    // after its own reads, with a barrier arrival that nothing but its order ties to them, a tile's last
    // rows were now and then those of the copy that took its place: in some 4 of
    // 100 processes, in the first run.)
    if (it > 0 && tid == 0) mbar_arrive(&sh.empty[(seq - 1) % NS]);
    if (*reinterpret_cast<volatile int*>(&sh.moved[it & 1]) == it + 1) {
      // some column's reference moves: to the largest score of the four warps'
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float mx = fmaxf(s[nt][j], s[nt][j + 2]);
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
          if (g == 0) sh.top[warp][nt * 8 + 2 * t + j] = mx;
        }
      named_sync(1, kWarps * 32);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int c = nt * 8 + 2 * t + j;
          const float mx = fmaxf(fmaxf(sh.top[0][c], sh.top[1][c]), fmaxf(sh.top[2][c], sh.top[3][c]));
          // (selects: the lanes stay together)
          const float mn = mx > most[nt][j] ? mx + slack : most[nt][j];
          const float f = mx > most[nt][j] ? fast_exp2((most[nt][j] - mn) * qscale) : 1.f;
          most[nt][j] = mn;
          l[nt][j] *= f, lr[nt][j] *= f;
#pragma unroll
          for (int mt = 0; mt < MW; ++mt) o[nt][mt][j] *= f, o[nt][mt][j + 2] *= f;
        }
      weigh();
      named_sync(1, kWarps * 32);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) l[nt][j] += dl[nt][j], lr[nt][j] += dr[nt][j];
    // O^T += V^T P^T over this warp's dims
    const uint8_t* p_at = sP + (lane & 7) * kPPitch + (lane >> 3) * 16;
#pragma unroll
    for (int kk = 0; kk < kRows / 32; ++kk) {
      uint32_t v4[2][MW][4];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int mt = 0; mt < MW; ++mt) ldsm_x4_t(v4[x][mt], tV + swz_off(kk * 32 + x * 16 + vr, vc + mt * 16, kRows));
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        uint32_t b[4];
        ldsm_x4(b, p_at + nt * 8 * kPPitch + kk * 64);
#pragma unroll
        for (int mt = 0; mt < MW; ++mt) {
          mma_m16n8k16(o[nt][mt], v4[0][mt][0], v4[0][mt][1], v4[0][mt][2], v4[0][mt][3], b[0], b[1]);
          mma_m16n8k16(o[nt][mt], v4[1][mt][0], v4[1][mt][1], v4[1][mt][2], v4[1][mt][3], b[2], b[3]);
        }
      }
    }
  }
  // the columns' sums over the warps, and the state
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], off);
        lr[nt][j] += __shfl_xor_sync(0xffffffffu, lr[nt][j], off);
      }
      if (g == 0) {
        sh.l[warp][nt * 8 + 2 * t + j][0] = l[nt][j];
        sh.l[warp][nt * 8 + 2 * t + j][1] = lr[nt][j];
      }
    }
  named_sync(1, kWarps * 32);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int c = nt * 8 + 2 * t + j;
      if (c >= cols) continue;
      float L = 0.f, LR = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) L += sh.l[w][c][0], LR += sh.l[w][c][1];
      const size_t at = (size_t)part * a.rows + row_of(c);
      if (warp == 0 && g == 0) a.ml[at] = make_float2(reference(most[nt][j]), L);
      if (L == 0.f) continue;
      const float even = LR != 0.f ? L / LR : 1.f;
      float* dst = a.o + at * D + warp * (D / 4) + g;
#pragma unroll
      for (int mt = 0; mt < MW; ++mt) {
        dst[mt * 16] = o[nt][mt][j] * even;
        dst[mt * 16 + 8] = o[nt][mt][j + 2] * even;
      }
    }
}

// The moment term's state of unit u for `cols` query rows (sQ, being written): 64
// dims of it from 64 `piece` on, 16 of C' q to a warp, C' (clamped) as bf16 hi + lo
// parts, or in the forms it was packed in; the logits with the first piece.
template <int D, int NT, typename RowOf>
__device__ __forceinline__ void moment_run(const PrefixArgs& a, int u, int n_e, int piece, int cols, const uint8_t* sQ,
                                           PartsShared& sh, RowOf row_of) {
  constexpr int KS = D / 16;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const float scale = rsqrtf(static_cast<float>(D));
  const int ra = piece * 64 + warp * 16 + g, rb = ra + 8;
  float2 cf[KS][4] = {};
  float va = 0.f, vb = 0.f;
  if (n_e > 0) {
    va = a.mu_v[(size_t)u * D + ra], vb = a.mu_v[(size_t)u * D + rb];
    if (piece == 0)
      for (int i = tid; i < D; i += kWarps * 32) sh.mu_k[i] = a.mu_k[(size_t)u * D + i];
    if (a.order == 1) {
#pragma unroll
      for (int kk = 0; kk < KS; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const size_t off = ((size_t)u * D + (i & 1 ? rb : ra)) * D + kk * 16 + 2 * t + (i >> 1) * 8;
          cf[kk][i] = a.C16 != nullptr ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(a.C16 + off))
                      : a.Cs != nullptr ? *reinterpret_cast<const float2*>(a.Cs + off / 2)
                                        : *reinterpret_cast<const float2*>(a.C + off);
        }
    }
  }
  named_sync(1, kWarps * 32);
  if (piece == 0) {
    // four threads a column (a warp has eight: all of them take every turn, for the shuffles)
    for (int c = tid >> 2; c < 8 * NT; c += kWarps * 8) {
      float e = 0.f;
      if (n_e > 0) {
#pragma unroll 4
        for (int i = (tid & 3) * 2; i < D; i += 8) {
          const float2 q = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(sQ + c * q_pitch(D) + i * 2));
          e = fmaf(q.x, sh.mu_k[i], fmaf(q.y, sh.mu_k[i + 1], e));
        }
      }
      e += __shfl_xor_sync(0xffffffffu, e, 1);
      e += __shfl_xor_sync(0xffffffffu, e, 2);
      if ((tid & 3) == 0 && c < cols) {
        const float x = n_e > 0 ? fmaf(e, scale * kLog2e, log2f(static_cast<float>(n_e))) : kNegInf;
        a.ml[(size_t)a.moments * a.rows + row_of(c)] = make_float2(x, x != kNegInf ? 1.f : 0.f);
      }
    }
  }
  if (n_e <= 0) return;
  const float nf = static_cast<float>(n_e), tau = a.tau;
  float f[NT][4] = {};
#pragma unroll
  for (int kk = 0; kk < KS; ++kk) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (a.Cs != nullptr) {
        hi[i] = __float_as_uint(cf[kk][i].x);
        lo[i] = __float_as_uint(cf[kk][i].y);
      } else {
        const float x = fabsf(cf[kk][i].x * nf) < tau ? 0.f : cf[kk][i].x;
        const float y = fabsf(cf[kk][i].y * nf) < tau ? 0.f : cf[kk][i].y;
        hi[i] = pack_bf16x2(x, y);
        lo[i] = pack_bf16x2(bf16_residual(x), bf16_residual(y));  // (0 of a 16-bit C)
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const uint8_t* p = sQ + (nt * 8 + g) * q_pitch(D) + kk * 32 + t * 4;
      const uint32_t b0 = *reinterpret_cast<const uint32_t*>(p), b1 = *reinterpret_cast<const uint32_t*>(p + 16);
      mma_m16n8k16(f[nt], hi[0], hi[1], hi[2], hi[3], b0, b1);
      mma_m16n8k16(f[nt], lo[0], lo[1], lo[2], lo[3], b0, b1);
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = nt * 8 + 2 * t + (i & 1);
      if (c < cols)
        a.o[((size_t)a.moments * a.rows + row_of(c)) * D + (i >> 1 ? rb : ra)] = fmaf(scale, f[nt][i], i >> 1 ? vb : va);
    }
}

// Tails, one to a warp: its items are first, first + 4, ... below `end` (tail
// unit, split), `mine` of them at most 32.  A warp has a ring of its own, of 16-row
// tiles that it asks for itself, ahead over its items; the keys and then the value dims are the 16-row side,
// the weights stay in registers, and no warp waits for another.
template <int D>
__device__ __forceinline__ void tail_warp(const PrefixArgs& a, const CUtensorMap* tmK, const CUtensorMap* tmV, int first,
                                          int end, uint8_t* ring, PartsShared& sh) {
  constexpr int KS = D / 16, MT = D / 16, NS = stages(D), kKeys = 16, kTile = kKeys * D * 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  uint64_t* full = sh.own[warp];
  ring += warp * NS * 2 * kTile;
  const int mine = end > first ? (end - first + kWarps - 1) / kWarps : 0;
  // an item each lane: its rows, none of a sequence that is not in use
  int n_all = -1, row_all = 0;
  if (lane < mine) {
    const int item = first + kWarps * lane, u = item / a.splits_t, split = item - u * a.splits_t, b = u / a.n_kv / a.N;
    const int have = a.len_t[u];
    if (u / a.n_kv - b * a.N < (a.count != nullptr ? a.count[b] : a.N)) {
      const int len = min(max(have, 0), a.cap_t);
      if (have != len && split == 0) record_error(a.ws, MKV_ERR_CAPACITY, u);
      const int tiles = (len + kKeys - 1) / kKeys, per = (tiles + a.splits_t - 1) / a.splits_t;
      const int t0 = min(tiles, split * per), t1 = min(tiles, t0 + per);
      n_all = max(0, min(len, t1 * kKeys) - t0 * kKeys);
      row_all = u * a.cap_t + t0 * kKeys;
    }
  }
  uint32_t asked = 0, seq = 0;  // tiles asked for and used
  int ask_item = 0, ask_row = 0;
  const uint64_t pol = l2_evict_first();
  auto ask = [&]() {  // the next tile of the warp's items, if there is one
    int n = 0;
    while (ask_item < mine && ask_row >= (n = __shfl_sync(0xffffffffu, n_all, ask_item))) ++ask_item, ask_row = 0;
    if (ask_item == mine) return;
    const int row = __shfl_sync(0xffffffffu, row_all, ask_item) + ask_row;
    if (lane == 0) {
      if (ask_row == 0 && n > kKeys) {  // the next tiles into L2 now (further ahead they would crowd it)
        const size_t off = (size_t)(row + kKeys) * D * 2;
        const uint32_t bytes = static_cast<uint32_t>(min(n, 6 * kKeys) - kKeys) * D * 2;
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(static_cast<const uint8_t*>(a.Kt) + off), "r"(bytes) : "memory");
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(static_cast<const uint8_t*>(a.Vt) + off), "r"(bytes) : "memory");
      }
      uint8_t* dst = ring + (asked % NS) * 2 * kTile;
      uint64_t* bar = &full[asked % NS];
      mbar_arrive_expect_tx(bar, 2u * kTile);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        tma_load_2d_hint(dst + x * kKeys * 128, tmK, x * 64, row, bar, pol);
        tma_load_2d_hint(dst + kTile + x * kKeys * 128, tmV, x * 64, row, bar, pol);
      }
    }
    ++asked;
    ask_row += kKeys;
  };
  auto query = [&](int i, uint32_t (&q)[KS][2]) {  // item i's query rows as the B operand
    const int u = (first + kWarps * i) / a.splits_t, pair = u / a.n_kv, kv = u - pair * a.n_kv, b = pair / a.N;
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch + (pair - b * a.N) * a.q_seq +
                             ((kv << a.g_shift) + g) * D + 2 * t;
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      q[kk][0] = i < mine && g < a.group ? *reinterpret_cast<const uint32_t*>(p + kk * 16) : 0u;
      q[kk][1] = i < mine && g < a.group ? *reinterpret_cast<const uint32_t*>(p + kk * 16 + 8) : 0u;
    }
  };
  for (int i = 0; i < NS; ++i) ask();
  const float qscale = rsqrtf(static_cast<float>(D)) * kLog2e, slack = kSlack / qscale;
  uint32_t next[KS][2];
  query(0, next);
  bool waited = true;
  for (int i = 0; waited && i < mine; ++i) {
    uint32_t q[KS][2];
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) q[kk][0] = next[kk][0], q[kk][1] = next[kk][1];
    if (i + 1 < mine) query(i + 1, next);
    const int n = __shfl_sync(0xffffffffu, n_all, i);
    if (n < 0) continue;  // (not in use: nothing is joined)
    float most[2] = {kNegInf, kNegInf}, l[2] = {}, lr[2] = {}, o[MT][4] = {};
    for (int r0 = 0; r0 < n; r0 += kKeys, ++seq) {
      waited = wait_tile(&full[seq % NS], (seq / NS) & 1, sh, a.polls);
      if (!waited) break;  // (a state of part of a tail is not used)
      const uint8_t* tK = ring + (seq % NS) * 2 * kTile;
      uint8_t* tV = ring + (seq % NS) * 2 * kTile + kTile;
      const int rows = min(kKeys, n - r0);
      if (rows < kKeys) {  // V rows past the end are zeroed: their weights are 0, but they may hold anything
        for (int x = lane; x < (kKeys - rows) * (D / 8); x += 32) {
          const int r = rows + x / (D / 8), c = (x % (D / 8)) * 8;
          *reinterpret_cast<uint4*>(tV + (c >> 6) * kKeys * 128 + r * 128 + (c & 63) * 2) = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
      }
      const int kr = (lane & 7) + ((lane >> 3) & 1) * 8, kc = (lane >> 4) * 8;
      float c[2][4] = {};
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) {
        uint32_t k4[4];
        ldsm_x4(k4, tK + swz_off(kr, kk * 16 + kc, kKeys));
        mma_m16n8k16(c[kk & 1], k4[0], k4[1], k4[2], k4[3], q[kk][0], q[kk][1]);
      }
      // lane (g, t): keys g (0, 1) and g + 8 (2, 3), columns 2t (0, 2) and 2t + 1 (1, 3)
      float s[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) s[x] = (x < 2 ? g : g + 8) < rows ? c[0][x] + c[1][x] : kNegInf;
      const float m0 = fmaxf(s[0], s[2]), m1 = fmaxf(s[1], s[3]);
      if (__any_sync(0xffffffffu, m0 > most[0] || m1 > most[1])) {
        float mx[2] = {m0, m1};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], off));
          const float mn = mx[j] > most[j] ? mx[j] + slack : most[j];
          const float f = mx[j] > most[j] ? fast_exp2((most[j] - mn) * qscale) : 1.f;
          most[j] = mn;
          l[j] *= f, lr[j] *= f;
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) o[mt][j] *= f, o[mt][j + 2] *= f;
        }
      }
      const float ra = most[0] == kNegInf ? 0.f : most[0] * qscale, rb = most[1] == kNegInf ? 0.f : most[1] * qscale;
      const float x0 = fast_exp2(fmaf(s[0], qscale, -ra)), x1 = fast_exp2(fmaf(s[1], qscale, -rb));
      const float x2 = fast_exp2(fmaf(s[2], qscale, -ra)), x3 = fast_exp2(fmaf(s[3], qscale, -rb));
      const uint32_t h0 = pack_bf16x2(x0, x1), h1 = pack_bf16x2(x2, x3);
      l[0] += x0 + x2;
      l[1] += x1 + x3;
      add_rounded(lr, h0);
      add_rounded(lr, h1);
      const uint32_t p0 = movmatrix_t(h0), p1 = movmatrix_t(h1);
      const int vr = (lane & 7) + (lane >> 4) * 8, vc = ((lane >> 3) & 1) * 8;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t v4[4];
        ldsm_x4_t(v4, tV + swz_off(vr, mt * 16 + vc, kKeys));
        mma_m16n8k16(o[mt], v4[0], v4[1], v4[2], v4[3], p0, p1);
      }
      fence_proxy_async();  // every lane has read the tile (and written its zeros) before a copy takes its place
      __syncwarp();
      ask();
    }
    const int u = (first + kWarps * i) / a.splits_t, split = first + kWarps * i - u * a.splits_t;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        l[j] += __shfl_xor_sync(0xffffffffu, l[j], off);
        lr[j] += __shfl_xor_sync(0xffffffffu, lr[j], off);
      }
      if (2 * t + j >= a.group) continue;
      const size_t at = (size_t)(a.tail + split) * a.rows + ((size_t)u << a.g_shift) + 2 * t + j;
      if (g == 0) a.ml[at] = make_float2(most[j] == kNegInf ? 0.f : most[j] * qscale, l[j]);
      const float even = lr[j] != 0.f ? l[j] / lr[j] : 1.f;
      if (l[j] != 0.f)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          a.o[at * D + mt * 16 + g] = o[mt][j] * even;
          a.o[at * D + mt * 16 + g + 8] = o[mt][j + 2] * even;
        }
    }
  }
  // after a wait that gave up: the copies in flight land before the block ends
  if (failed(sh) && lane == 0)
    for (uint32_t j = asked > NS ? asked - NS : 0; j < asked; ++j) (void)mbar_wait(&full[j % NS], (j / NS) & 1);
}

// Query rows of unit (b, kv) from row `first` on into shared memory, `wide` of them, zeros where there is none.
template <int D>
__device__ __forceinline__ void stage_q(const PrefixArgs& a, int b, int kv, int first, int wide, uint8_t* sm) {
  for (int i = threadIdx.x; i < wide * (D / 8); i += kWarps * 32) {
    const int c = i / (D / 8), k = i % (D / 8), r = first + c, seq = r >> a.g_shift;
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (seq < a.N)
      w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch + seq * a.q_seq +
                                          ((kv << a.g_shift) + (r & (a.group - 1))) * D + k * 8);
    *reinterpret_cast<uint4*>(sm + c * q_pitch(D) + k * 16) = w;
  }
}

// Blocks: the shared rows' runs (unit, column block, split) and the moment terms
// (unit, column block, piece), where they are this launch's, and the tails.
template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 2)
    prefix_parts_kernel(const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKt,
                        const __grid_constant__ CUtensorMap tmVt) {
  constexpr int NS = stages(D);
  extern __shared__ __align__(128) uint8_t raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sm = ring + NS * 2 * tile_bytes(D);  // the query rows and the weights
  __shared__ PartsShared sh;
  const int tid = threadIdx.x, lane = tid & 31;
  const bool loads = tid >= kWarps * 32;
  if (tid < NS) {
    mbar_init(&sh.full[tid], 1);
    mbar_init(&sh.empty[tid], 1);
    for (int w = 0; w < kWarps; ++w) mbar_init(&sh.own[w][tid], 1);
  }
  if (tid == 0) sh.fail = sh.moved[0] = sh.moved[1] = 0;
  mbar_fence_init();
  // what this block's work is: in one wave the short ones' loads go first, in several the long runs
  const int units = a.batch * a.n_kv, shared_blocks = units * a.blocks * a.splits;
  const int moment_blocks = a.moments >= 0 ? units * a.blocks * (D / 64) : 0;
  int x = blockIdx.x, kind = 0;
  if (a.shared_last) x = x < static_cast<int>(gridDim.x) - shared_blocks ? x + shared_blocks : x - (gridDim.x - shared_blocks);
  if (x >= shared_blocks) x -= shared_blocks, kind = 1;
  if (kind == 1 && x >= moment_blocks) x -= moment_blocks, kind = 2;
  const int each = kind == 0 ? a.splits : kind == 1 ? D / 64 : 1;  // blocks of an item: its runs, or the moment term's pieces
  const int item = x / each, split = x - item * each;
  const int u = kind == 2 ? 0 : a.blocks > 1 ? item / a.blocks : item;
  const int b = kind == 2 ? 0 : u / a.n_kv, kv = u - b * a.n_kv, first = kind == 2 ? 0 : (item - u * a.blocks) * 8 * NT;
  __syncthreads();
  grid_dependency_wait();
  grid_launch_dependents();
  uint32_t seq = 0;
  auto run_of = [](int len, int splits, int split, int& row) {  // this split's rows of `len`
    const int tiles = (len + kRows - 1) / kRows, per = (tiles + splits - 1) / splits;
    const int t0 = min(tiles, split * per), t1 = min(tiles, t0 + per);
    row = t0 * kRows;
    return max(0, min(len, t1 * kRows) - t0 * kRows);
  };
  if (kind < 2) {
    const int counted = a.count != nullptr ? a.count[b] : a.N, have = kind == 0 ? a.len[u] : a.n[u];
    if (!loads) stage_q<D>(a, b, kv, first, 8 * NT, sm);
    const int count = min(max(counted, 0), a.N), cols = min(8 * NT, count * a.group - first);
    const int len = min(max(have, 0), a.cap);
    if (kind == 0 && split == 0 && first == 0 && tid == 0) {
      if (kv == 0 && count != counted) record_error(a.ws, MKV_ERR_INVALID_ARG, b);
      if (have != len) record_error(a.ws, MKV_ERR_CAPACITY, u);
    }
    if (cols > 0) {  // (else no sequence is in use: nothing is joined)
      int row, n = 0;
      if (kind == 0) n = run_of(len, a.splits, split, row);
      if (loads) {
        if (lane == 0 && kind == 0) load_run<D, NS>(a, &tmK, &tmV, u * a.cap + row, n, ring, sh, seq);
        __syncwarp();
      } else {
        auto row_of = [&](int c) { return out_row(a, b, kv, first + c); };
        if (kind == 0) {
          named_sync(1, kWarps * 32);
          attend_run<D, NT, NS>(a, n, cols, split, ring, sm, sh, seq, row_of);
        } else {
          moment_run<D, NT>(a, u, have, split, cols, sm, sh, row_of);
        }
      }
    }
  } else if (!loads) {
    const int from = x * kWarps * a.tails, all = units * a.N * a.splits_t;
    tail_warp<D>(a, &tmKt, &tmVt, from + (tid >> 5), min(all, from + kWarps * a.tails), ring, sh);
  }
  __syncthreads();
  if (failed(sh) && loads && lane == 0) {
    record_error(a.ws, MKV_ERR_TIMEOUT, static_cast<int>(blockIdx.x));
    // the copies in flight land before the block ends
    for (uint32_t j = seq > NS ? seq - NS : 0; j < seq; ++j) (void)mbar_wait(&sh.full[j % NS], (j / NS) & 1);
  }
}

struct State {
  float m, l, o[4];
};
__device__ __forceinline__ void join(State& s, float m, float l, const float4& v) {
  const float mn = fmaxf(s.m, m), ref = mn == kNegInf ? 0.f : mn;
  const float f0 = s.l != 0.f ? fast_exp2(s.m - ref) : 0.f, f = fast_exp2(m - ref);
  s.m = mn;
  s.l = s.l * f0 + l * f;
  s.o[0] = fmaf(v.x, f, s.o[0] * f0);
  s.o[1] = fmaf(v.y, f, s.o[1] * f0);
  s.o[2] = fmaf(v.z, f, s.o[2] * f0);
  s.o[3] = fmaf(v.w, f, s.o[3] * f0);
}

// P threads share 4 dims of a query row, every P-th part each; the first joins
// theirs and the new token, and a unit's first row appends that token to its tail.
template <int D, int P>
__global__ void __launch_bounds__(kJoinThreads) prefix_join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int kLanes = D / 4, kPer = kJoinThreads / kLanes / P;  // rows of a block
  __shared__ State others[P > 1 ? P - 1 : 1][P > 1 ? kPer * kLanes : 1];
  const int at_row = threadIdx.x / kLanes % kPer, slice = threadIdx.x / kLanes / kPer, lane = threadIdx.x % kLanes;
  const int64_t row = (int64_t)blockIdx.x * kPer + at_row;
  const int d0 = lane * 4;
  const bool in = row < a.rows;
  const int h = static_cast<int>(row) & (a.group - 1), ut = static_cast<int>(row >> a.g_shift);  // head, tail unit
  const int kv = ut % a.n_kv, pair = ut / a.n_kv, b = pair / a.N, seq = pair - b * a.N;
  grid_dependency_wait();
  grid_launch_dependents();
  // four parts' loads at a time in flight, whether they hold anything or not
  State s{kNegInf, 0.f, {}};
  const bool token = a.k_new != nullptr && slice == 0 && in;
  uint2 kw{}, vw{}, qw{};
  int len = 0, seen = 0;
  if (token) {
    const int64_t at = b * a.kv_batch + seq * a.kv_seq + kv * D + d0;
    kw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.k_new) + at);
    vw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.v_new) + at);
    qw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch + seq * a.q_seq +
                                         (kv * a.group + h) * D + d0);
    if (h == 0) len = a.len_t[ut], seen = a.seen_t[ut];
  }
  const bool live = in && seq < live_seqs(a, b);
  if (live) {
    for (int p0 = slice; p0 < a.parts; p0 += 4 * P) {
      float2 ml[4];
      float4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const size_t at = (size_t)min(p0 + i * P, a.parts - 1) * a.rows + row;
        ml[i] = a.ml[at];
        v[i] = *reinterpret_cast<const float4*>(a.o + at * D + d0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (p0 + i * P < a.parts && ml[i].y != 0.f) join(s, ml[i].x, ml[i].y, v[i]);
    }
  }
  if constexpr (P > 1) {
    if (slice > 0) others[slice - 1][at_row * kLanes + lane] = s;
    __syncthreads();
    if (slice > 0) return;
#pragma unroll
    for (int i = 0; i < P - 1; ++i) {
      const State& x = others[i][at_row * kLanes + lane];
      if (x.l != 0.f) join(s, x.m, x.l, make_float4(x.o[0], x.o[1], x.o[2], x.o[3]));
    }
  }
  if (!in) return;
  uint2* dst = reinterpret_cast<uint2*>(a.out + row * D + d0);
  if (!live) {
    *dst = make_uint2(0u, 0u);
    if (d0 == 0 && a.lse != nullptr) a.lse[row] = kNegInf;
    return;
  }
  if (token) {
    const uint32_t mask = kLanes == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);  // the row's lanes
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    float x = lo(qw.x) * lo(kw.x) + hi(qw.x) * hi(kw.x) + lo(qw.y) * lo(kw.y) + hi(qw.y) * hi(kw.y);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) x += __shfl_xor_sync(mask, x, off);
    join(s, x * rsqrtf(static_cast<float>(D)) * kLog2e, 1.f, make_float4(lo(vw.x), hi(vw.x), lo(vw.y), hi(vw.y)));
    if (h == 0) {
      len = min(max(len, 0), a.cap_t);
      __syncwarp(mask);  // (all have read the length)
      if (len < a.cap_t) {
        const size_t slot = (size_t)ut * a.cap_t + len;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.Kt) + slot * D + d0) = kw;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.Vt) + slot * D + d0) = vw;
        if (d0 == 0) {
          a.pos_t[slot] = seen;
          a.seen_t[ut] = seen + 1;
          a.len_t[ut] = len + 1;
        }
      } else if (d0 == 0) {
        record_error(a.ws, MKV_ERR_CAPACITY, ut);
      }
    }
  }
  const float inv = s.l != 0.f ? 1.f / s.l : 0.f;
  *dst = s.l != 0.f ? make_uint2(pack_bf16x2(s.o[0] * inv, s.o[1] * inv), pack_bf16x2(s.o[2] * inv, s.o[3] * inv))
                    : make_uint2(0u, 0u);
  if (d0 == 0 && a.lse != nullptr) a.lse[row] = s.l != 0.f ? (s.m + log2f(s.l)) * kLn2 : kNegInf;
}

// The 8-column tiles of a block (1, 2 or 4; 0: the shared rows run on tcgen05, whose
// state is part 0), the parts of a query row and the splits.
int plan(PrefixArgs& a, const mkv_geom& g, int num_sms) {
  const long units = (long)g.batch * g.n_kv_heads, rows = (long)a.N * g.group, places = 2 * num_sms;
  long tiles = ((long)a.cap + kRows - 1) / kRows;
  const long tiles_t = ((long)a.cap_t + kRows - 1) / kRows;
  int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  long blocks = (rows + 8 * nt - 1) / (8 * nt);
  if (blocks > 1 && units * blocks * tiles * g.head_dim > kVisits * 128 * places) nt = 0, blocks = 0, tiles = 0;
  const long moments = nt > 0 && a.n != nullptr ? 1 : 0;
  // Tails are a warp's; long ones are split, so that their items are more than the places (13 x 8
  // tails of up to 300 rows: 208 blocks on 152 SMs took 25 us, three times as many 20).
  const long items = units * a.N;
  const long splits_t = std::clamp<long>((5 * kWarps * places / 2 + items - 1) / items, 1, std::min<long>(kMaxSplits, (tiles_t + 1) / 2));
  const long item_tiles = (tiles_t + splits_t - 1) / splits_t;
  // Splits of the shared rows and tails of a warp: the least of an estimate (in
  // us, from clock stamps of blocks): the longest block, or all blocks over the
  // places and half of the longest for the last wave's end, and the join's traffic.
  const float tile = (nt == 4 ? 1.1f : 0.85f) * g.head_dim / 128;
  float best = INFINITY;
  long best_splits = 1, in_warp = 1;
  for (const int s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64}) {
    // (and no more parts than the workspace was sized for)
    if (s > 1 && (s * kMinTiles > tiles + kMinTiles - 1 || units * blocks * (s - 1) > places)) break;
    for (int w = 1; w <= kMaxTails; w *= 2) {
      const float run = nt > 0 ? 3.f + tile * ((tiles + s - 1) / s) : 0.f, tail = 2.f + w * (0.8f + 2.f * item_tiles);
      const long runs = units * blocks * s, terms = units * blocks * moments * (g.head_dim / 64);
      const long tails = (items * splits_t + kWarps * w - 1) / (kWarps * w);
      const float longest = std::max(run, tail), all = (runs * run + terms * 3.f + tails * tail) / places;
      const float us = (runs + terms + tails <= places ? longest : std::max(longest, all + 0.5f * longest)) +
                       units * rows * (s + moments + splits_t) * g.head_dim * 1e-6f;
      if (us < best) best = us, best_splits = s, in_warp = w, a.shared_last = runs + terms + tails <= places;
    }
    if (nt == 0) break;
  }
  a.splits = static_cast<int>(best_splits);
  a.splits_t = static_cast<int>(splits_t);
  a.tails = static_cast<int>(in_warp);
  a.blocks = static_cast<int>(blocks);
  a.moments = moments > 0 ? a.splits : -1;
  a.tail = a.splits + static_cast<int>(moments);
  a.parts = a.tail + a.splits_t;
  a.rows = static_cast<int>(units * rows);
  a.g_shift = g.group == 8 ? 3 : g.group == 4 ? 2 : g.group == 2 ? 1 : 0;
  return nt;
}

template <int D, int NT>
cudaError_t launch_parts(const PrefixArgs& a, cudaStream_t stream) {
  CUtensorMap tm[4];
  const uint64_t rows = (uint64_t)a.batch * a.n_kv * a.cap, rows_t = (uint64_t)a.batch * a.N * a.n_kv * a.cap_t;
  if (!encode_tmap_bf16(&tm[0], a.K, D, rows, (uint64_t)D * 2, 64, kRows) ||
      !encode_tmap_bf16(&tm[1], a.V, D, rows, (uint64_t)D * 2, 64, kRows) ||
      !encode_tmap_bf16(&tm[2], a.Kt, D, rows_t, (uint64_t)D * 2, 64, 16) ||
      !encode_tmap_bf16(&tm[3], a.Vt, D, rows_t, (uint64_t)D * 2, 64, 16))
    return cudaErrorInvalidValue;
  constexpr int smem = parts_smem(D, NT);
  cudaError_t e = cudaFuncSetAttribute(prefix_parts_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const long units = (long)a.batch * a.n_kv;
  const long blocks = units * a.blocks * (a.splits + (a.moments >= 0 ? D / 64 : 0)) +
                      (units * a.N * a.splits_t + kWarps * a.tails - 1) / (kWarps * a.tails);
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_pdl(prefix_parts_kernel<D, NT>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), smem, stream, a,
                    tm[0], tm[1], tm[2], tm[3]);
}

// The shared rows' and the moment term's states by the kernels of tree_step.cu, the
// sequences as nodes that are no keys.  It loads early: what precedes it is the
// tails' launch, which writes nothing that it reads and has waited for what did.
cudaError_t launch_shared(const PrefixArgs& a, const mkv_geom& g, int num_sms, void* parts, cudaStream_t stream) {
  TreeArgs t{};
  t.q = a.q;
  t.q_node = a.q_seq;
  t.q_batch = a.q_batch;
  t.N = a.N;
  t.count = a.count;
  t.K = a.K;
  t.V = a.V;
  t.len = a.len;
  t.cap = a.cap;
  t.n = a.n;
  t.mu_k = a.mu_k;
  t.mu_v = a.mu_v;
  t.C = a.C;
  t.C16 = a.C16;
  t.Cs = a.Cs;
  t.order = a.order;
  t.tau = a.tau;
  t.early = 1;
  t.ws = a.ws;
  t.parts = parts;
  t.state_o = a.o;
  t.state_ml = a.ml;
  t.batch = a.batch;
  t.n_kv = a.n_kv;
  return launch_prefix_tree(t, g, num_sms, stream);
}

template <int D>
cudaError_t launch(const PrefixArgs& a, const mkv_geom& g, int nt, int num_sms, void* parts, cudaStream_t stream) {
  cudaError_t e = nt == 4 ? launch_parts<D, 4>(a, stream) : nt == 2 ? launch_parts<D, 2>(a, stream) : launch_parts<D, 1>(a, stream);
  if (e == cudaSuccess && nt == 0) e = launch_shared(a, g, num_sms, parts, stream);
  if (e != cudaSuccess) return e;
  // threads of a row: one round of loads each, where the GPU holds them all at once
  const auto run = [&](auto kernel, int P) {
    const int per = kJoinThreads / (D / 4) / P;
    return launch_pdl(kernel, dim3((a.rows + per - 1) / per), dim3(kJoinThreads), 0, stream, a);
  };
  const long all = (long)a.rows * (D / 4), most = 1024l * num_sms;
  if (a.parts > 16 && all * 8 <= most) return run(prefix_join_kernel<D, 8>, 8);
  if (a.parts > 8 && all * 4 <= most) return run(prefix_join_kernel<D, 4>, 4);
  if (a.parts > 4 && all * 2 <= most) return run(prefix_join_kernel<D, 2>, 2);
  return run(prefix_join_kernel<D, 1>, 1);
}

}  // namespace

// Bytes of the parts: of every query row one of the shared rows, the moment
// term's and one of its tail, as many more as there are places (of up to 32 rows
// each), and a warp of every place for a tail's (8 rows each); more than any smaller call needs.
size_t prefix_workspace_bytes(const mkv_geom& g, int32_t n_seqs, int32_t capacity, int num_sms) {
  const long rows = (long)g.batch * g.n_kv_heads * n_seqs * g.group;
  const long part_rows = 3 * rows + 2l * num_sms * (kMaxCols + 5 * kWarps / 2 * 8);
  const size_t tree = prefix_tree_bytes(g, n_seqs, capacity, num_sms);
  return kHeaderBytes + 256 + tree + align_up(part_rows * sizeof(float2), 256) + (size_t)part_rows * g.head_dim * 4;
}

cudaError_t launch_prefix_step(const PrefixArgs& args, const mkv_geom& g, int num_sms, cudaStream_t stream) {
  PrefixArgs a = args;
  a.polls = pipeline_poll_limit();
  const int nt = plan(a, g, num_sms);
  uint8_t* w = static_cast<uint8_t*>(a.ws) + kHeaderBytes;
  a.ml = reinterpret_cast<float2*>(w);
  w += align_up((size_t)a.parts * a.rows * sizeof(float2), 256);
  a.o = reinterpret_cast<float*>(w);
  w += (size_t)a.parts * a.rows * g.head_dim * 4;
  void* parts = reinterpret_cast<void*>(align_up(reinterpret_cast<uintptr_t>(w), 256));
  return g.head_dim == 128 ? launch<128>(a, g, nt, num_sms, parts, stream) : launch<64>(a, g, nt, num_sms, parts, stream);
}

}  // namespace mkv
