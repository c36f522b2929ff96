// What the kernels that rotate by position share (rope.cu, norm_rope.cu): a
// thread has one chunk of 16 dims of a head, which are 8 pairs that rotate, or
// 16 dims past rot_dim that do not.
#pragma once

#include "common.cuh"
#include "tree.h"
#include "warp_mma.cuh"

namespace mkv {

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// Cosines and sines of chunk c's 8 frequencies for batch item b's token t.
template <typename Args>
__device__ __forceinline__ void chunk_angles(const Args& a, int c, int b, int t, float (&cs)[8], float (&sn)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int f = c * 8 + i;
    const int32_t p = a.pos[a.axis[f] * a.pos_axis + b * a.pos_batch + t];
    const uint64_t ang = static_cast<uint64_t>(static_cast<int64_t>(p)) * a.turn[f];
    const float x = static_cast<float>(static_cast<int32_t>(ang >> 32)) * 0x1p-31f;  // half turns in [-1, 1)
    sincospif(x, &sn[i], &cs[i]);
  }
}

// The chunk's first and second 8 dims turned by those angles, forward or by the
// negative angle: neighbours are pairs (0, 1), (2, 3), ... of the 16 dims, halves
// pairs of the two runs.
template <bool Back>
__device__ __forceinline__ void turn_chunk(bool neighbours, const float (&cs)[8], const float (&sn)[8],
                                           const float (&x0)[8], const float (&x1)[8], float (&y0)[8], float (&y1)[8]) {
  if (neighbours) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float s0 = Back ? -sn[j] : sn[j], s1 = Back ? -sn[4 + j] : sn[4 + j];
      y0[2 * j] = x0[2 * j] * cs[j] - x0[2 * j + 1] * s0;
      y0[2 * j + 1] = x0[2 * j] * s0 + x0[2 * j + 1] * cs[j];
      y1[2 * j] = x1[2 * j] * cs[4 + j] - x1[2 * j + 1] * s1;
      y1[2 * j + 1] = x1[2 * j] * s1 + x1[2 * j + 1] * cs[4 + j];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float s = Back ? -sn[j] : sn[j];
      y0[j] = x0[j] * cs[j] - x1[j] * s;
      y1[j] = x0[j] * s + x1[j] * cs[j];
    }
  }
}

}  // namespace mkv
