// Rotary positions with one or more axes (mkv_rope), forward and inverse, for
// several strided tensors of the same tokens in one launch.
//
// Mathematics: the angle of frequency f at position p is p w_f radians.  The
// host turns w_f into a 64-bit fixed-point fraction of a turn, F = frac(w_f /
// 2 pi) 2^64, so p F modulo 2^64 (one integer product) is the angle modulo a
// turn with an error of |p| 2^-64 turns; in fp32 p w_f loses a radian's
// digits with every digit of p (0.004 rad at 128K).  The upper 32 bits as a
// signed fraction lie in [-1/2, 1/2) turns, where sine and cosine need no
// range reduction.
//
// Bounded by HBM: every value is read and written once (4 bytes), and a
// position's 8 angles per thread serve the thread's heads one after another
// (4 x 32768 tokens, 40 heads of 128 dims: 404 us, 0.98 of 6.8 TB/s).
#include <algorithm>

#include "kernels.h"
#include "rope.cuh"

namespace mkv {

namespace {

constexpr int kRopeThreads = 256;

// A thread has one chunk of 16 dims of a head -- 8 pairs that rotate, or 16
// dims past rot that are copied -- for one token and the heads slot, slot +
// slots, ... of all tensors.
template <int D>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a, int slots) {
  constexpr int kChunks = D / 16;
  grid_dependency_wait();
  const int per = kChunks * slots;  // threads of a token
  const int64_t id = (int64_t)blockIdx.x * kRopeThreads + threadIdx.x;
  const int64_t tok = id / per;
  if (tok >= (int64_t)a.batch * a.tokens) return;
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
    uint4 v0 = *reinterpret_cast<const uint4*>(src + o0), v1 = *reinterpret_cast<const uint4*>(src + o1);
    if (turn) {
      float x0[8], x1[8], y0[8], y1[8];
      unpack8(v0, x0);
      unpack8(v1, x1);
      turn_chunk<false>(a.neighbours != 0, cs, sn, x0, x1, y0, y1);
      v0 = pack8(y0);
      v1 = pack8(y1);
    }
    *reinterpret_cast<uint4*>(dst + o0) = v0;
    *reinterpret_cast<uint4*>(dst + o1) = v1;
  }
}

}  // namespace

cudaError_t launch_rope(const RopeArgs& a, int head_dim, int num_sms, cudaStream_t stream) {
  // Heads per thread: its angles serve them all, so as many as leave five waves
  // of threads (five blocks per SM; fewer leave a last wave that is not full),
  // and no fewer than 3, whose loads are in flight one after another.  Measured
  // at 40 heads of 128 dims, 2, 3, 5, 8 and 20 heads per thread: 131072 tokens
  // 554, 484, 423, 413 and 405 us; 16382 tokens (half of the dims) 67.7, 62.2,
  // 56.8, 57.5 and 63.1; 256 tokens 3.8, 3.8, 4.4, 5.5 and 9.9.
  const int64_t chunks = (int64_t)a.batch * a.tokens * a.heads * (head_dim / 16);
  const int64_t per = std::clamp<int64_t>(chunks / (5ll * 5 * kRopeThreads * num_sms), 3, 20);
  const int slots = static_cast<int>((a.heads + per - 1) / per);
  const int64_t threads = (int64_t)a.batch * a.tokens * slots * (head_dim / 16);
  const int64_t blocks = (threads + kRopeThreads - 1) / kRopeThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kRopeThreads);
  return head_dim == 128 ? launch_pdl(rope_kernel<128>, grid, block, 0, stream, a, slots)
                         : launch_pdl(rope_kernel<64>, grid, block, 0, stream, a, slots);
}

}  // namespace mkv
