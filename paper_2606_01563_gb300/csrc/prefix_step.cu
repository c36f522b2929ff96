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
// Two launches.  prefix_parts_kernel leaves states ("parts") of every query row in
// the workspace: a block takes a run of the shared rows for up to 8 NT query
// rows of a unit (all sequences' heads side by side, so that a shared row is read
// once for all of them), or the moment term for as many, or a run of one tail for
// its unit's heads.  prefix_join_kernel joins each row's parts and the new token and
// appends that token to its tail.
//
// A run, as in decode_cl.cu: a warp issues 64-row TMA copies into a ring; four
// warps take 16 rows of every tile each, S^T = K q^T with the keys on the 16-row
// side and the query rows on the 8-column side, then O^T += V^T P^T with P rounded
// to bf16.  O is scaled by the ratio of the unrounded weights' sum to the rounded
// ones', so that roundings that are common cancel.
#include <algorithm>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "warp_mma.cuh"

namespace mkv {

namespace {

constexpr int kWarps = 4;                   // that attend
constexpr int kThreads = (kWarps + 1) * 32;  // and one that loads
constexpr int kRows = 64;                   // rows of a tile
constexpr int kStages = 3;
constexpr int kMinTiles = 2;   // of a run, where there are as many
constexpr int kMaxSplits = 64;
constexpr float kSlack = 8.f;  // log2 headroom of a reference (weights at most 2^8)
constexpr float kNegInf = -INFINITY;
constexpr int kJoinThreads = 256;

__host__ __device__ constexpr int tile_bytes(int D) { return kRows * D * 2; }
// q rows in shared memory lie 16 bytes apart beyond their length: ldmatrix meets no bank twice
__host__ __device__ constexpr int q_pitch(int D) { return D * 2 + 16; }
__host__ __device__ constexpr int parts_smem(int D, int NT) {
  return kStages * 2 * tile_bytes(D) + 8 * NT * q_pitch(D) + 1024;
}
static_assert(2 * (parts_smem(128, 4) + 1024) <= 228 * 1024, "two blocks to an SM");

// A query row of a unit: sequence r / G, head r % G.
__device__ __forceinline__ int64_t out_row(const PrefixArgs& a, int b, int kv, int r) {
  const int seq = r / a.group;
  return ((int64_t)(b * a.N + seq) * a.n_kv + kv) * a.group + (r - seq * a.group);
}
__device__ __forceinline__ int live_seqs(const PrefixArgs& a, int b) {
  return a.count != nullptr ? min(max(a.count[b], 0), a.N) : a.N;
}

struct PartsShared {
  uint64_t full[kStages], empty[kStages];
  float ml[kWarps][32][3];  // of a warp and column: reference, sum, sum of the rounded weights
  float e[32];              // the moment term's logits
  float mu_k[128];
  int fail;
};

// The state of the `n` keys from row `row0` of the maps' matrices on, for `cols`
// query rows (sQ) into part `part`; `row_of(c)` is column c's output row.
template <int D, int NT, typename RowOf>
__device__ __forceinline__ void attend_run(const PrefixArgs& a, const CUtensorMap* tmK, const CUtensorMap* tmV, int row0,
                                           int n, int cols, int part, uint8_t* ring, const uint8_t* sQ,
                                           PartsShared& sh, RowOf row_of) {
  constexpr int MT = D / 16, KS = D / 16, kTile = tile_bytes(D);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int tiles = (n + kRows - 1) / kRows;
  const float qscale = rsqrtf(static_cast<float>(D)) * kLog2e;
  if (warp == kWarps) {
    int i = 0;  // tiles asked for
    if (lane == 0) {
      const uint64_t pol = l2_evict_first();
      for (; i < tiles; ++i) {
        const int st = i % kStages;
        if (i >= kStages && !mbar_wait(&sh.empty[st], ((i / kStages) - 1) & 1, a.polls)) {
          *reinterpret_cast<volatile int*>(&sh.fail) = 1;
          break;
        }
        uint8_t* dst = ring + (size_t)st * 2 * kTile;
        mbar_arrive_expect_tx(&sh.full[st], 2u * kTile);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          tma_load_2d_hint(dst + x * kRows * 128, tmK, x * 64, row0 + i * kRows, &sh.full[st], pol);
          tma_load_2d_hint(dst + kTile + x * kRows * 128, tmV, x * 64, row0 + i * kRows, &sh.full[st], pol);
        }
      }
    }
    __syncwarp();
    named_sync(2, kThreads);
    // after a wait that gave up: the copies in flight land before the block ends
    if (lane == 0 && *reinterpret_cast<volatile int*>(&sh.fail))
      for (int j = max(0, i - kStages); j < i; ++j) (void)mbar_wait(&sh.full[j % kStages], (j / kStages) & 1);
    return;
  }
  const int r0 = warp * 16;
  float m[NT][2], l[NT][2], lr[NT][2], o[NT][MT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = kNegInf;
    l[nt][0] = l[nt][1] = lr[nt][0] = lr[nt][1] = 0.f;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) o[nt][mt][0] = o[nt][mt][1] = o[nt][mt][2] = o[nt][mt][3] = 0.f;
  }
  // the query rows as the B operand: kept in registers where they are few
  constexpr bool kKeep = NT <= 2;
  uint32_t qf[kKeep ? NT : 1][KS][2];
  auto load_q = [&](int nt, int kk, uint32_t (&b)[2]) {
    const uint8_t* p = sQ + (nt * 8 + g) * q_pitch(D) + kk * 32 + t * 4;
    b[0] = *reinterpret_cast<const uint32_t*>(p);
    b[1] = *reinterpret_cast<const uint32_t*>(p + 16);
  };
  if constexpr (kKeep) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int kk = 0; kk < KS; ++kk) load_q(nt, kk, qf[nt][kk]);
  }
  bool ok = true;
  for (int it = 0; it < tiles; ++it) {
    const int st = it % kStages;
    const bool got = mbar_wait(&sh.full[st], (it / kStages) & 1, a.polls);
    if (!__all_sync(0xffffffffu, got)) {
      ok = false;
      break;
    }
    const int rows = min(kRows, n - it * kRows);
    const uint8_t* tK = ring + (size_t)st * 2 * kTile;
    uint8_t* tV = ring + (size_t)st * 2 * kTile + kTile;
    if (rows > r0) {
      if (rows < r0 + 16) {  // V rows past the end are zeroed: their weights are 0, but they may hold anything
        for (int i = lane; i < (r0 + 16 - rows) * (D / 8); i += 32) {
          const int r = rows + i / (D / 8), c = (i % (D / 8)) * 8;
          *reinterpret_cast<uint4*>(tV + (c >> 6) * kRows * 128 + r * 128 + (c & 63) * 2) = make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
      }
      float s[NT][4];
      const int kr = r0 + (lane & 7) + ((lane >> 3) & 1) * 8, kc = (lane >> 4) * 8;
      if constexpr (NT == 1) {  // four chains: one would wait for itself
        float c[4][4] = {};
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          uint32_t k4[4];
          ldsm_x4(k4, tK + swz_off(kr, kk * 16 + kc, kRows));
          mma_m16n8k16(c[kk & 3], k4[0], k4[1], k4[2], k4[3], qf[0][kk][0], qf[0][kk][1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[0][i] = (c[0][i] + c[2][i]) + (c[1][i] + c[3][i]);
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          uint32_t k4[4];
          ldsm_x4(k4, tK + swz_off(kr, kk * 16 + kc, kRows));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if constexpr (kKeep) {
              mma_m16n8k16(s[nt], k4[0], k4[1], k4[2], k4[3], qf[nt][kk][0], qf[nt][kk][1]);
            } else {
              uint32_t b[2];
              load_q(nt, kk, b);
              mma_m16n8k16(s[nt], k4[0], k4[1], k4[2], k4[3], b[0], b[1]);
            }
          }
        }
      }
      // lane (g, t): keys r0 + g (0, 1) and r0 + g + 8 (2, 3), columns 2t (0, 2) and 2t + 1 (1, 3)
      const bool va = r0 + g < rows, vb = r0 + g + 8 < rows;
      bool moves = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[nt][i] = (i < 2 ? va : vb) ? s[nt][i] * qscale : kNegInf;
        moves |= fmaxf(s[nt][0], s[nt][2]) > m[nt][0] + kSlack || fmaxf(s[nt][1], s[nt][3]) > m[nt][1] + kSlack;
      }
      // A reference only has to be common to a column's keys: it moves when a score
      // exceeds it by more than kSlack, so most tiles skip the maximum over the lanes.
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float mx = fmaxf(s[nt][j], s[nt][j + 2]);
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
            const float mn = fmaxf(m[nt][j], mx);
            const float f = mn == kNegInf ? 1.f : fast_exp2(m[nt][j] - mn);
            m[nt][j] = mn;
            l[nt][j] *= f, lr[nt][j] *= f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[nt][mt][j] *= f, o[nt][mt][j + 2] *= f;
          }
        }
      }
      uint32_t p0[NT], p1[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float ma = m[nt][0] == kNegInf ? 0.f : m[nt][0], mb = m[nt][1] == kNegInf ? 0.f : m[nt][1];
        const float x0 = fast_exp2(s[nt][0] - ma), x1 = fast_exp2(s[nt][1] - mb);
        const float x2 = fast_exp2(s[nt][2] - ma), x3 = fast_exp2(s[nt][3] - mb);
        l[nt][0] += x0 + x2;
        l[nt][1] += x1 + x3;
        const uint32_t h0 = pack_bf16x2(x0, x1), h1 = pack_bf16x2(x2, x3);
        lr[nt][0] += __uint_as_float(h0 << 16) + __uint_as_float(h1 << 16);
        lr[nt][1] += __uint_as_float(h0 & 0xffff0000u) + __uint_as_float(h1 & 0xffff0000u);
        p0[nt] = movmatrix_t(h0);
        p1[nt] = movmatrix_t(h1);
      }
      const int vr = r0 + (lane & 7) + (lane >> 4) * 8, vc = ((lane >> 3) & 1) * 8;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t v4[4];
        ldsm_x4_t(v4, tV + swz_off(vr, mt * 16 + vc, kRows));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) mma_m16n8k16(o[nt][mt], v4[0], v4[1], v4[2], v4[3], p0[nt], p1[nt]);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.empty[st]);
  }
  if (!ok && lane == 0) *reinterpret_cast<volatile int*>(&sh.fail) = 1;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int off = 4; off < 32; off <<= 1) {
        l[nt][j] += __shfl_xor_sync(0xffffffffu, l[nt][j], off);
        lr[nt][j] += __shfl_xor_sync(0xffffffffu, lr[nt][j], off);
      }
  // the four warps' states into one, through the ring (free once every warp is
  // past its tiles, unless a wait gave up and copies may still land there)
  named_sync(2, kThreads);
  const bool bad = *reinterpret_cast<volatile int*>(&sh.fail) != 0;
  float* sW = reinterpret_cast<float*>(ring);  // [4][8 NT][D]
  if (!bad) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sW[(size_t)(warp * 8 * NT + nt * 8 + 2 * t + (i & 1)) * D + mt * 16 + g + (i >> 1) * 8] = o[nt][mt][i];
    if (g == 0) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float* x = sh.ml[warp][nt * 8 + 2 * t + j];
          x[0] = m[nt][j], x[1] = l[nt][j], x[2] = lr[nt][j];
        }
    }
  } else if (tid == 0) {
    record_error(a.ws, MKV_ERR_TIMEOUT, static_cast<int>(blockIdx.x));
  }
  named_sync(1, kWarps * 32);
  for (int i = tid; i < cols * (D / 4); i += kWarps * 32) {
    const int c = i / (D / 4), d0 = (i % (D / 4)) * 4;
    float M = kNegInf, L = 0.f, LR = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (!bad) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        if (sh.ml[w][c][1] != 0.f) M = fmaxf(M, sh.ml[w][c][0]);
      const float ref = M == kNegInf ? 0.f : M;
#pragma unroll
      for (int w = 0; w < kWarps; ++w)
        if (sh.ml[w][c][1] != 0.f) {
          const float f = fast_exp2(sh.ml[w][c][0] - ref);
          const float4 v = *reinterpret_cast<const float4*>(sW + (size_t)(w * 8 * NT + c) * D + d0);
          L = fmaf(sh.ml[w][c][1], f, L);
          LR = fmaf(sh.ml[w][c][2], f, LR);
          acc.x = fmaf(f, v.x, acc.x);
          acc.y = fmaf(f, v.y, acc.y);
          acc.z = fmaf(f, v.z, acc.z);
          acc.w = fmaf(f, v.w, acc.w);
        }
    }
    const size_t at = (size_t)part * a.rows + row_of(c);
    if (d0 == 0) a.ml[at] = make_float2(M, L);
    if (L != 0.f) {
      const float even = LR != 0.f ? L / LR : 1.f;
      *reinterpret_cast<float4*>(a.o + at * D + d0) = make_float4(acc.x * even, acc.y * even, acc.z * even, acc.w * even);
    }
  }
}

// The moment term's state of unit u for `cols` query rows (sQ): a warp has 16
// dims of C' q at a time, C' (clamped) as bf16 hi + lo parts, or in the forms it was packed in.
template <int D, int NT, typename RowOf>
__device__ __forceinline__ void moment_run(const PrefixArgs& a, int u, int n_e, int cols, const uint8_t* sQ,
                                           PartsShared& sh, RowOf row_of) {
  constexpr int KS = D / 16;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  if (warp == kWarps) return;
  const float scale = rsqrtf(static_cast<float>(D));
  if (n_e > 0)
    for (int i = tid; i < D; i += kWarps * 32) sh.mu_k[i] = a.mu_k[(size_t)u * D + i];
  named_sync(1, kWarps * 32);
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
      sh.e[c] = x;
      a.ml[(size_t)a.moments * a.rows + row_of(c)] = make_float2(x, x != kNegInf ? 1.f : 0.f);
    }
  }
  if (n_e <= 0) return;
  named_sync(1, kWarps * 32);
  const float nf = static_cast<float>(n_e), tau = a.tau;
  for (int mt = warp; mt < D / 16; mt += kWarps) {
    const int ra = mt * 16 + g, rb = ra + 8;
    float f[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) f[nt][0] = f[nt][1] = f[nt][2] = f[nt][3] = 0.f;
    if (a.order == 1) {
      float2 cf[KS][4];
#pragma unroll
      for (int kk = 0; kk < KS; ++kk)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const size_t off = ((size_t)u * D + (i & 1 ? rb : ra)) * D + kk * 16 + 2 * t + (i >> 1) * 8;
          cf[kk][i] = a.C16 != nullptr ? __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(a.C16 + off))
                      : a.Cs != nullptr ? *reinterpret_cast<const float2*>(a.Cs + off / 2)
                                        : *reinterpret_cast<const float2*>(a.C + off);
        }
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
    }
    const float va = a.mu_v[(size_t)u * D + ra], vb = a.mu_v[(size_t)u * D + rb];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = nt * 8 + 2 * t + (i & 1);
        if (c < cols)
          a.o[((size_t)a.moments * a.rows + row_of(c)) * D + (i >> 1 ? rb : ra)] = fmaf(scale, f[nt][i], i >> 1 ? vb : va);
      }
  }
}

// Blocks: the shared rows' runs (unit, column block, split), the moment terms (unit, column
// block), the tails' runs (tail unit, split).
template <int D, int NT>
__global__ void __launch_bounds__(kThreads, 2)
    prefix_parts_kernel(const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap tmK,
                        const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmKt,
                        const __grid_constant__ CUtensorMap tmVt) {
  extern __shared__ __align__(128) uint8_t raw[];
  uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = ring + kStages * 2 * tile_bytes(D);
  __shared__ PartsShared sh;
  const int tid = threadIdx.x;
  if (tid < kStages) {
    mbar_init(&sh.full[tid], 1);
    mbar_init(&sh.empty[tid], kWarps);
  }
  if (tid == 0) sh.fail = 0;
  mbar_fence_init();
  // what this block's work is
  const int units = a.batch * a.n_kv, shared_blocks = units * a.blocks * a.splits;
  const int moment_blocks = a.moments >= 0 ? units * a.blocks : 0;
  int x = blockIdx.x, kind = 0;
  if (x >= shared_blocks) x -= shared_blocks, kind = 1;
  if (kind == 1 && x >= moment_blocks) x -= moment_blocks, kind = 2;
  const int split = kind == 0 ? x % a.splits : kind == 2 ? x % a.splits_t : 0;
  const int item = kind == 0 ? x / a.splits : kind == 2 ? x / a.splits_t : x;
  // kinds 0 and 1: unit and column block; kind 2: tail unit (prompt, sequence, head)
  const int u = kind == 2 ? item : item / a.blocks;
  const int pair = u / a.n_kv, kv = u - pair * a.n_kv;  // (prompt, or prompt and sequence)
  const int b = kind == 2 ? pair / a.N : pair;
  const int first = kind == 2 ? (pair - b * a.N) * a.group : (item - u * a.blocks) * 8 * NT;
  grid_dependency_wait();
  grid_launch_dependents();
  const int count = live_seqs(a, b);
  if (kind == 0 && split == 0 && kv == 0 && first == 0 && tid == 0 && a.count != nullptr && a.count[b] != count)
    record_error(a.ws, MKV_ERR_INVALID_ARG, b);
  const int cols = min(kind == 2 ? a.group : 8 * NT, count * a.group - first);
  if (cols <= 0) return;  // (no sequence in use: nothing is joined)
  const int cap = kind == 2 ? a.cap_t : a.cap;
  const int have = kind == 1 ? 0 : kind == 2 ? a.len_t[u] : a.len[u];
  const int len = min(max(have, 0), cap);
  if (have != len && split == 0 && (kind == 2 || first == 0) && tid == 0) record_error(a.ws, MKV_ERR_CAPACITY, u);
  // the query rows into shared memory, zeros past `cols`
  const int wide = kind == 2 ? 8 : 8 * NT;
  for (int i = tid; i < wide * (D / 8); i += kThreads) {
    const int c = i / (D / 8), k = i % (D / 8);
    uint4 w = make_uint4(0u, 0u, 0u, 0u);
    if (c < cols) {
      const int r = first + c, seq = r / a.group;
      w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch + seq * a.q_seq +
                                          (kv * a.group + r - seq * a.group) * D + k * 8);
    }
    *reinterpret_cast<uint4*>(sQ + c * q_pitch(D) + k * 16) = w;
  }
  __syncthreads();
  auto row_of = [&](int c) { return out_row(a, b, kv, first + c); };
  // this split's run of tiles
  const int splits = kind == 2 ? a.splits_t : a.splits;
  const int tiles = (len + kRows - 1) / kRows, per = (tiles + splits - 1) / splits;
  const int t0 = min(tiles, split * per), t1 = min(tiles, t0 + per);
  const int n = max(0, min(len, t1 * kRows) - t0 * kRows), row0 = u * cap + t0 * kRows;
  if (kind == 0)
    attend_run<D, NT>(a, &tmK, &tmV, row0, n, cols, split, ring, sQ, sh, row_of);
  else if (kind == 1)
    moment_run<D, NT>(a, u, a.n[u], cols, sQ, sh, row_of);
  else
    attend_run<D, 1>(a, &tmKt, &tmVt, row0, n, cols, a.tail + split, ring, sQ, sh, row_of);
}

// A thread has 4 dims of a query row: the parts, then the new token, joined; the
// first row of a unit appends the token to the tail.
template <int D>
__global__ void __launch_bounds__(kJoinThreads) prefix_join_kernel(const __grid_constant__ PrefixArgs a) {
  constexpr int kLanes = D / 4;
  grid_dependency_wait();
  grid_launch_dependents();
  const int64_t row = (int64_t)blockIdx.x * (kJoinThreads / kLanes) + threadIdx.x / kLanes;
  const int d0 = (threadIdx.x % kLanes) * 4;
  if (row >= a.rows) return;
  const uint32_t mask = kLanes == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16);
  const int h = static_cast<int>(row % a.group), ut = static_cast<int>(row / a.group);  // head, tail unit
  const int kv = ut % a.n_kv, pair = ut / a.n_kv, b = pair / a.N, seq = pair - b * a.N;
  uint2* dst = reinterpret_cast<uint2*>(a.out + row * D + d0);
  if (seq >= live_seqs(a, b)) {
    *dst = make_uint2(0u, 0u);
    if (d0 == 0 && a.lse != nullptr) a.lse[row] = kNegInf;
    return;
  }
  float M = kNegInf, L = 0.f, acc[4] = {};
  auto join = [&](float m, float l, const float4& v) {
    const float mn = fmaxf(M, m), ref = mn == kNegInf ? 0.f : mn;
    const float f0 = L != 0.f ? fast_exp2(M - ref) : 0.f, f = fast_exp2(m - ref);
    M = mn;
    L = L * f0 + l * f;
    acc[0] = fmaf(v.x, f, acc[0] * f0);
    acc[1] = fmaf(v.y, f, acc[1] * f0);
    acc[2] = fmaf(v.z, f, acc[2] * f0);
    acc[3] = fmaf(v.w, f, acc[3] * f0);
  };
#pragma unroll 4
  for (int p = 0; p < a.parts; ++p) {
    const size_t at = (size_t)p * a.rows + row;
    const float2 ml = a.ml[at];
    if (ml.y != 0.f) join(ml.x, ml.y, *reinterpret_cast<const float4*>(a.o + at * D + d0));
  }
  if (a.k_new != nullptr) {
    const int64_t at = b * a.kv_batch + seq * a.kv_seq + kv * D + d0;
    const uint2 kw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.k_new) + at);
    const uint2 vw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.v_new) + at);
    const uint2 qw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.q) + b * a.q_batch +
                                                     seq * a.q_seq + (kv * a.group + h) * D + d0);
    auto lo = [](uint32_t w) { return __uint_as_float(w << 16); };
    auto hi = [](uint32_t w) { return __uint_as_float(w & 0xffff0000u); };
    float s = lo(qw.x) * lo(kw.x) + hi(qw.x) * hi(kw.x) + lo(qw.y) * lo(kw.y) + hi(qw.y) * hi(kw.y);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) s += __shfl_xor_sync(mask, s, off);
    join(s * rsqrtf(static_cast<float>(D)) * kLog2e, 1.f, make_float4(lo(vw.x), hi(vw.x), lo(vw.y), hi(vw.y)));
    if (h == 0) {
      const int len = min(max(a.len_t[ut], 0), a.cap_t);
      __syncwarp(mask);
      if (len < a.cap_t) {
        const size_t slot = (size_t)ut * a.cap_t + len;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.Kt) + slot * D + d0) = kw;
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.Vt) + slot * D + d0) = vw;
        if (d0 == 0) {
          const int seen = a.seen_t[ut];
          a.pos_t[slot] = seen;
          a.seen_t[ut] = seen + 1;
          a.len_t[ut] = len + 1;
        }
      } else if (d0 == 0) {
        record_error(a.ws, MKV_ERR_CAPACITY, ut);
      }
    }
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;
  *dst = L != 0.f ? make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv))
                  : make_uint2(0u, 0u);
  if (d0 == 0 && a.lse != nullptr) a.lse[row] = L != 0.f ? (M + log2f(L)) * kLn2 : kNegInf;
}

// Columns of a block (8, 16 or 32), the parts of a query row and the splits.
int plan(PrefixArgs& a, const mkv_geom& g, int num_sms) {
  const long units = (long)g.batch * g.n_kv_heads, rows = (long)a.N * g.group;
  const int nt = rows <= 8 ? 1 : rows <= 16 ? 2 : 4;
  a.blocks = static_cast<int>((rows + 8 * nt - 1) / (8 * nt));
  const long tiles = ((long)a.cap + kRows - 1) / kRows, tiles_t = ((long)a.cap_t + kRows - 1) / kRows;
  // runs of equal length, as many as there are places
  const long all = units * a.blocks * tiles + units * a.N * tiles_t;
  const long per = std::max<long>(kMinTiles, (all + 2 * num_sms - 1) / (2 * num_sms));
  a.splits = static_cast<int>(std::min<long>(kMaxSplits, (tiles + per - 1) / per));
  a.splits_t = static_cast<int>(std::min<long>(kMaxSplits, (tiles_t + per - 1) / per));
  a.moments = a.n != nullptr ? a.splits : -1;
  a.tail = a.splits + (a.n != nullptr ? 1 : 0);
  a.parts = a.tail + a.splits_t;
  a.rows = static_cast<int>(units * rows);
  return nt;
}

template <int D, int NT>
cudaError_t launch_parts(const PrefixArgs& a, cudaStream_t stream) {
  CUtensorMap tm[4];
  const uint64_t rows = (uint64_t)a.batch * a.n_kv * a.cap, rows_t = (uint64_t)a.batch * a.N * a.n_kv * a.cap_t;
  if (!encode_tmap_bf16(&tm[0], a.K, D, rows, (uint64_t)D * 2, 64, kRows) ||
      !encode_tmap_bf16(&tm[1], a.V, D, rows, (uint64_t)D * 2, 64, kRows) ||
      !encode_tmap_bf16(&tm[2], a.Kt, D, rows_t, (uint64_t)D * 2, 64, kRows) ||
      !encode_tmap_bf16(&tm[3], a.Vt, D, rows_t, (uint64_t)D * 2, 64, kRows))
    return cudaErrorInvalidValue;
  constexpr int smem = parts_smem(D, NT);
  cudaError_t e = cudaFuncSetAttribute(prefix_parts_kernel<D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const long units = (long)a.batch * a.n_kv;
  const long blocks = units * a.blocks * (a.splits + (a.moments >= 0 ? 1 : 0)) + units * a.N * a.splits_t;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  return launch_pdl(prefix_parts_kernel<D, NT>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), smem, stream, a,
                    tm[0], tm[1], tm[2], tm[3]);
}

template <int D>
cudaError_t launch(const PrefixArgs& a, int nt, cudaStream_t stream) {
  const cudaError_t e = nt == 1   ? launch_parts<D, 1>(a, stream)
                        : nt == 2 ? launch_parts<D, 2>(a, stream)
                                  : launch_parts<D, 4>(a, stream);
  if (e != cudaSuccess) return e;
  constexpr int kPer = kJoinThreads / (D / 4);
  return launch_pdl(prefix_join_kernel<D>, dim3((a.rows + kPer - 1) / kPer), dim3(kJoinThreads), 0, stream, a);
}

}  // namespace

// Bytes of the parts: at most one run a place and one more of every column block
// and tail, and the moment terms'; more than any smaller call needs.
size_t prefix_workspace_bytes(const mkv_geom& g, int32_t n_seqs, int32_t capacity, int32_t tail_capacity, int num_sms) {
  (void)capacity, (void)tail_capacity;
  const long units = (long)g.batch * g.n_kv_heads, rows = units * n_seqs * g.group;
  // a column block's parts have at most 32 rows, a tail's at most 8
  const long part_rows = 3 * rows + 2l * num_sms * 32 + 2l * num_sms * 8;
  return kHeaderBytes + align_up(part_rows * sizeof(float2), 256) + (size_t)part_rows * g.head_dim * 4;
}

cudaError_t launch_prefix_step(const PrefixArgs& args, const mkv_geom& g, int num_sms, cudaStream_t stream) {
  PrefixArgs a = args;
  a.polls = pipeline_poll_limit();
  const int nt = plan(a, g, num_sms);
  uint8_t* w = static_cast<uint8_t*>(a.ws) + kHeaderBytes;
  a.ml = reinterpret_cast<float2*>(w);
  a.o = reinterpret_cast<float*>(w + align_up((size_t)a.parts * a.rows * sizeof(float2), 256));
  return g.head_dim == 128 ? launch<128>(a, nt, stream) : launch<64>(a, nt, stream);
}

}  // namespace mkv
