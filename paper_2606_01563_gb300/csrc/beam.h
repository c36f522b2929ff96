// Internal launcher interface of the calls in include/mkv_beam.h.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/mkv_beam.h"
#include "tree.h"

namespace mkv {

// ------------------------------------------------------------------ prefix
struct PrefixArgs {
  const void* q;  // bf16 [b, N, Hkv*G, D], strides in elements
  int64_t q_seq, q_batch;
  const void* k_new;  // bf16 [b, N, Hkv, D] or null
  const void* v_new;
  int64_t kv_seq, kv_batch;
  int32_t N;
  const int32_t* count;  // [b] or null
  const void* K;         // the shared rows: bf16 [b, Hkv, cap, D]
  const void* V;
  const int32_t* len;
  int32_t cap;
  const int32_t* n;  // null: no moment term
  const float* mu_k;
  const float* mu_v;
  const float* C;
  const __nv_bfloat16* C16;
  const uint2* Cs;
  int32_t order;
  float tau;
  void* Kt;  // the tails: bf16 [b * N, Hkv, cap_t, D]
  void* Vt;
  int32_t* pos_t;
  int32_t* len_t;
  int32_t* seen_t;
  int32_t cap_t;
  __nv_bfloat16* out;  // [b, N, Hkv*G, D]
  float* lse;
  int32_t batch;
  int32_t n_kv;
  int32_t group;
  uint32_t polls;
  void* ws;
  // filled by the launcher: parts of every query row, row-major as out's rows
  float2* ml;        // [parts][rows]: reference and sum, log2 domain
  float* o;          // [parts][rows][D]: sum of weighted values about the reference
  int32_t rows;      // b * N * Hkv * G
  int32_t blocks;    // column blocks of a unit's query rows (0: the shared rows and moments are another launch's)
  int32_t splits;    // parts of the shared rows; part 0 is the first
  int32_t moments;   // the moment term's part, or -1
  int32_t tail;      // the tails' first part
  int32_t splits_t;  // parts of a tail
  int32_t tails;     // items (a tail, or a split of one) of a warp
  int32_t g_shift;   // log2 of the group
  int32_t shared_last;  // the shared rows' blocks come last
  int32_t parts;
};
size_t prefix_workspace_bytes(const mkv_geom& g, int32_t n_seqs, int32_t capacity, int num_sms);
cudaError_t launch_prefix_step(const PrefixArgs& a, const mkv_geom& g, int num_sms, cudaStream_t stream);

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
  float4* stats;   // [b * beams][splits]: reference, sum and what its rounding lost, candidates (int; -1: a value that is not finite)
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
  int32_t split;  // blocks of the bulk copies of an item, layer and head (filled by the launcher)
  uint32_t polls;
  void* ws;
};
cudaError_t launch_beam_reorder(const ReorderArgs& a, int layers, int batch, int num_sms, cudaStream_t stream);

}  // namespace mkv
