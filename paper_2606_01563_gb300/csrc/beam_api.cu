// C-ABI entry points declared in include/mkv_beam.h: argument validation,
// workspace sizing and kernel dispatch.
#include <string.h>

#include "beam.h"
#include "common.cuh"
#include "kernels.h"
#include "validate.h"

using namespace mkv;

namespace {

mkv_status cuda_status(cudaError_t e) { return e == cudaSuccess ? MKV_OK : MKV_ERR_CUDA; }

// Sizes of a step, and rows of K and V that a tensor map's coordinates reach.
bool prefix_sizes_ok(const mkv_geom& g, int32_t n_seqs, int32_t capacity, int32_t tail_capacity) {
  const int64_t units = (int64_t)g.batch * g.n_kv_heads;
  return n_seqs >= 1 && n_seqs <= MKV_BEAM_MAX_SEQS && capacity >= 1 && tail_capacity >= 1 &&
         units * capacity < ((int64_t)1 << 31) && units * n_seqs * tail_capacity < ((int64_t)1 << 31) &&
         units * n_seqs * g.group < ((int64_t)1 << 30);
}

bool select_sizes_ok(int32_t batch, int32_t beams, int32_t vocab, int32_t n_out) {
  return batch >= 1 && batch <= 65535 && beams >= 1 && beams <= MKV_BEAM_MAX_BEAMS && vocab >= 1 &&
         vocab <= (1 << 24) && n_out >= 1 && n_out <= MKV_BEAM_MAX_OUT;
}

// Whether an array of one layer is an array of the other: it would be moved twice, at once.
// (Absent ones are null in both; keys and values, and the two means, may also be each other's.)
bool share_an_array(const mkv_beam_layer& x, const mkv_beam_layer& y) {
  const mkv_cache &a = x.cache, &b = y.cache;
  const mkv_moments &m = x.mom, &n = y.mom;
  const bool rows = (a.K == b.K) | (a.V == b.V) | (a.K == b.V) | (a.V == b.K) | (a.pos == b.pos) | (a.len == b.len) |
                    (a.seen == b.seen);
  const bool state = a.y && ((a.y == b.y) | (a.y_len == b.y_len));
  const bool moments = m.n && n.n && ((m.n == n.n) | (m.mu_k == n.mu_k) | (m.mu_v == n.mu_v) | (m.mu_k == n.mu_v) |
                                      (m.mu_v == n.mu_k) | (m.C == n.C));
  return rows | state | moments;
}

}  // namespace

extern "C" {

// ------------------------------------------------------------------ prefix
size_t mkv_prefix_workspace_size(mkv_geom geom, int32_t n_seqs, int32_t capacity, int32_t tail_capacity) {
  if (!geom_ok(geom) || !prefix_sizes_ok(geom, n_seqs, capacity, tail_capacity)) return 0;
  return prefix_workspace_bytes(geom, n_seqs, capacity, num_sms_current());
}

mkv_status mkv_prefix_step(mkv_geom geom, const mkv_seqs* seqs, const void* q, const void* k_new, const void* v_new,
                           const mkv_cache* prefix, const mkv_moments* mom, const mkv_cache* tail,
                           const mkv_decode_params* p, void* out, float* lse, void* workspace, size_t workspace_bytes,
                           void* stream) {
  NvtxRange nvtx("mkv_prefix_step");
  const mkv_status chk =
      decode_args_status(geom, q, k_new, v_new, prefix, mom, p, static_cast<const float*>(out));
  if (chk != MKV_OK) return chk;
  if (!seqs || !cache_ok(tail) || !aligned(seqs->count, 4) || !aligned(lse, 4)) return MKV_ERR_INVALID_ARG;
  if (!prefix_sizes_ok(geom, seqs->n_seqs, prefix->capacity, tail->capacity)) return MKV_ERR_SHAPE;
  PrefixArgs a{};
  const int64_t kv = (int64_t)geom.n_kv_heads * geom.head_dim, N = seqs->n_seqs;
  if (!stride_of(seqs->q_seq, kv * geom.group, &a.q_seq) || !stride_of(seqs->q_batch, N * a.q_seq, &a.q_batch) ||
      !stride_of(seqs->kv_seq, kv, &a.kv_seq) || !stride_of(seqs->kv_batch, N * a.kv_seq, &a.kv_batch))
    return MKV_ERR_INVALID_ARG;
  const int sms = num_sms_current();
  if (!workspace || !aligned(workspace, 256) ||
      workspace_bytes < prefix_workspace_bytes(geom, seqs->n_seqs, prefix->capacity, sms))
    return MKV_ERR_WORKSPACE;
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.N = seqs->n_seqs;
  a.count = seqs->count;
  a.K = prefix->K;
  a.V = prefix->V;
  a.len = prefix->len;
  a.cap = prefix->capacity;
  if (p->correction) {
    a.n = mom->n;
    a.mu_k = mom->mu_k;
    a.mu_v = mom->mu_v;
    a.C = mom->C;
    a.C16 = static_cast<const __nv_bfloat16*>(p->C16);
    a.Cs = static_cast<const uint2*>(p->C_split);
  }
  a.order = p->order;
  a.tau = p->tau;
  a.Kt = tail->K;
  a.Vt = tail->V;
  a.pos_t = tail->pos;
  a.len_t = tail->len;
  a.seen_t = tail->seen;
  a.cap_t = tail->capacity;
  a.out = static_cast<__nv_bfloat16*>(out);
  a.lse = lse;
  a.batch = geom.batch;
  a.n_kv = geom.n_kv_heads;
  a.group = geom.group;
  a.ws = workspace;
  return cuda_status(launch_prefix_step(a, geom, sms, static_cast<cudaStream_t>(stream)));
}

// ------------------------------------------------------------------ select
size_t mkv_beam_select_workspace_size(int32_t batch, int32_t beams, int32_t vocab, int32_t n_out) {
  if (!select_sizes_ok(batch, beams, vocab, n_out)) return 0;
  SelectArgs a{};
  a.beams = beams;
  a.vocab = vocab;
  a.out = n_out;
  return select_plan(a, batch, num_sms_current(), nullptr);
}

mkv_status mkv_beam_select(int32_t batch, int32_t beams, int32_t vocab, const mkv_beam_scores* s, int32_t n_out,
                           int32_t* parent, int32_t* token, float* score_out, int32_t* done_out, void* workspace,
                           size_t workspace_bytes, void* stream) {
  NvtxRange nvtx("mkv_beam_select");
  if (!select_sizes_ok(batch, beams, vocab, n_out)) return MKV_ERR_SHAPE;
  if (!s || !s->logits || !s->score || !parent || !token || !score_out) return MKV_ERR_INVALID_ARG;
  if ((s->f32 != 0 && s->f32 != 1) || !aligned(s->logits, s->f32 ? 4 : 2) || !aligned(s->score, 4) ||
      !aligned(s->done, 4) || !aligned(parent, 4) || !aligned(token, 4) || !aligned(score_out, 4) ||
      !aligned(done_out, 4))
    return MKV_ERR_INVALID_ARG;
  if (s->logits_batch < 0 || s->logits_beam < 0 || s->end_token < -1 || s->end_token >= vocab ||
      (s->done && s->end_token < 0))
    return MKV_ERR_INVALID_ARG;
  SelectArgs a{};
  a.logits = s->logits;
  a.s_batch = s->logits_batch;
  a.s_beam = s->logits_beam;
  a.score = s->score;
  a.done = s->done;
  a.end = s->end_token;
  a.beams = beams;
  a.vocab = vocab;
  a.out = n_out;
  a.parent = parent;
  a.token = token;
  a.score_out = score_out;
  a.done_out = done_out;
  if (!workspace || !aligned(workspace, 256) ||
      workspace_bytes < select_plan(a, batch, num_sms_current(), workspace))
    return MKV_ERR_WORKSPACE;
  return cuda_status(launch_beam_select(a, batch, s->f32 != 0, static_cast<cudaStream_t>(stream)));
}

// ----------------------------------------------------------------- reorder
mkv_status mkv_beam_reorder(mkv_geom geom, int32_t n_seqs, int32_t n_layers, const mkv_beam_layer* layers,
                            const int32_t* parent, void* workspace, size_t workspace_bytes, void* stream) {
  NvtxRange nvtx("mkv_beam_reorder");
  if (!geom_ok(geom)) return geom_status(geom);
  if (n_seqs < 1 || n_seqs > MKV_BEAM_MAX_SEQS || (long)geom.batch * geom.n_kv_heads > 65535) return MKV_ERR_SHAPE;
  if (n_layers < 0 || !layers || !parent || !aligned(parent, 4)) return MKV_ERR_INVALID_ARG;
  for (int i = 0; i < n_layers; ++i) {
    if (!cache_ok(&layers[i].cache) || (layers[i].mom.n && !moments_ok(&layers[i].mom))) return MKV_ERR_INVALID_ARG;
    for (int k = 0; k < i; ++k)
      if (share_an_array(layers[k], layers[i])) return MKV_ERR_INVALID_ARG;
  }
  if (!workspace || workspace_bytes < kHeaderBytes || !aligned(workspace, 256)) return MKV_ERR_WORKSPACE;
  ReorderArgs a{};
  a.parent = parent;
  a.N = n_seqs;
  a.n_kv = geom.n_kv_heads;
  a.D = geom.head_dim;
  a.ws = workspace;
  const int sms = num_sms_current();
  for (int first = 0; first < n_layers; first += kReorderLayers) {
    const int n = n_layers - first < kReorderLayers ? n_layers - first : kReorderLayers;
    for (int i = 0; i < n; ++i) {
      const mkv_cache& c = layers[first + i].cache;
      const mkv_moments& m = layers[first + i].mom;
      ReorderLayer& l = a.layer[i];
      l.big[0] = static_cast<uint8_t*>(c.K);
      l.big[1] = static_cast<uint8_t*>(c.V);
      l.big[2] = reinterpret_cast<uint8_t*>(c.y);
      l.big[3] = m.n ? reinterpret_cast<uint8_t*>(m.C) : nullptr;
      l.pos = c.pos;
      l.len = c.len;
      l.seen = c.seen;
      l.y_len = c.y_len;
      l.n = m.n;
      l.mu_k = m.n ? reinterpret_cast<int32_t*>(m.mu_k) : nullptr;
      l.mu_v = m.n ? reinterpret_cast<int32_t*>(m.mu_v) : nullptr;
      l.cap = c.capacity;
    }
    const cudaError_t e = launch_beam_reorder(a, n, geom.batch, sms, static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) return cuda_status(e);
  }
  return MKV_OK;
}

}  // extern "C"
