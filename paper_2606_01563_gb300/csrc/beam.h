// Internal launcher interface of the calls in include/mkv_beam.h.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/mkv_beam.h"
#include "tree.h"

namespace mkv {

// ------------------------------------------------------------------ select
struct SelectArgs {
  const void* logits;  // [b, beams, vocab], strides in elements
  int64_t s_batch, s_beam;
  const float* score;   // [b, beams]
  const int32_t* done;  // [b, beams] or null
  int32_t end;
  int32_t beams, vocab, out;
  int32_t* parent;  // [b, out]
  int32_t* token;
  float* score_out;
  int32_t* done_out;  // or null
  void* ws;
  // carved from the workspace by select_plan
  float4* stats;   // [b * beams][splits]: reference, sum, candidates (int), unused
  uint64_t* keys;  // [b * beams][splits][out], best first
  int32_t splits;
  int32_t per;  // elements of a split
};
// Splits of a row, and the workspace's bytes; carves it where `ws` is given.
size_t select_plan(SelectArgs& a, int batch, int num_sms, void* ws);
cudaError_t launch_beam_select(const SelectArgs& a, int batch, bool f32, cudaStream_t stream);

// ----------------------------------------------------------------- reorder
constexpr int kReorderLayers = 64;  // layers per launch: their pointers travel in the launch's arguments
constexpr int kReorderSeqs = MKV_BEAM_MAX_SEQS;
struct ReorderLayer {
  uint8_t* big[4];     // K, V, y, C (null: absent): copied by rows of 16 bytes
  int32_t* pos;
  int32_t* len;
  int32_t* seen;
  int32_t* y_len;      // or null
  int32_t* n;          // or null, with mu_k and mu_v
  int32_t* mu_k;
  int32_t* mu_v;
  int32_t cap;
};
struct ReorderArgs {
  ReorderLayer layer[kReorderLayers];
  const int32_t* parent;  // [b, N]
  int32_t N;
  int32_t n_kv;
  int32_t D;
  uint32_t polls;
  void* ws;
};
cudaError_t launch_beam_reorder(const ReorderArgs& a, int layers, int batch, int num_sms, cudaStream_t stream);

}  // namespace mkv
