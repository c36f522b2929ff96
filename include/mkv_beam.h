/*
 * mkv_beam.h -- several continuations of one compressed prompt (beam search,
 * parallel sampling): the calls that sit beside mkv.h's in such a serving step.
 *
 * A batch item is a prompt; N sequences continue it.  The prompt's retained rows and
 * moments (mkv_compress) are held once per prompt and shared; each sequence has
 * a tail, an mkv_cache of its own for the tokens generated since.
 *
 *   mkv_prefix_step   one decoding step of all sequences: attention over the
 *                     shared rows and moments, read once for all of them, and
 *                     over each sequence's tail, which the new token joins
 *   mkv_beam_select   beam search's selection over beams and vocabulary
 *   mkv_beam_reorder  the selected beams' states (caches, and moments where
 *                     there are any) in every layer, in place
 *
 * In beam search a step runs mkv_norm_rope or mkv_rope (mkv_tree.h) on the new
 * tokens' queries and keys and mkv_prefix_step, for every layer, then
 * mkv_beam_select on the model's logits and mkv_beam_reorder on the tails.
 *
 * Conventions are those of mkv.h (device pointers, caller-owned memory,
 * stream order, statuses, the workspace's error word read by
 * mkv_get_device_error), except that these tensors may be strided as stated.
 */
#ifndef MKV_BEAM_H
#define MKV_BEAM_H

#include "mkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MKV_BEAM_MAX_SEQS 256 /* sequences of a prompt (mkv_prefix_step, mkv_beam_reorder) */
#define MKV_BEAM_MAX_BEAMS 64 /* beams of a batch item (mkv_beam_select)                   */
#define MKV_BEAM_MAX_OUT 64   /* continuations that it selects                             */

/*
 * The sequences of every prompt.
 *   n_seqs  N: sequences per prompt in the tensors, 1..256
 *   count   int32 [b]  optional: the sequences in use of each prompt, 0..N (NULL: all N).  The outputs of
 *           those at or above it are zeros and their lse -infinity, and their
 *           tails are neither read nor changed.  A count outside 0..N is taken
 *           as the nearer end and recorded as MKV_ERR_INVALID_ARG.
 * Strides of the tensors below, in elements; 0 stands for the dense value.
 * All are multiples of 8 and not below it.
 *   q_seq, q_batch    q [b, N, g*h_kv, d]: from sequence to sequence (dense
 *                     g*h_kv*d), from prompt to prompt (dense N * q_seq)
 *   kv_seq, kv_batch  k_new and v_new [b, N, h_kv, d] (dense h_kv*d, N * kv_seq)
 */
typedef struct {
  int32_t n_seqs;
  const int32_t* count;
  int64_t q_seq;
  int64_t q_batch;
  int64_t kv_seq;
  int64_t kv_batch;
} mkv_seqs;

/*
 * Bytes of device workspace mkv_prefix_step needs for this geometry (batch:
 * prompts), N and capacities of the shared and the tail caches on the current
 * device, and for every smaller batch, N and capacity.
 * Returns 0 if the arguments are invalid.  The workspace must be zero-filled
 * before its first use; every call leaves it ready for the next one.
 */
MKV_API size_t mkv_prefix_workspace_size(mkv_geom geom, int32_t n_seqs, int32_t capacity, int32_t tail_capacity);

/*
 * One layer's decoding step of every sequence (Algorithm 1 Phase 2 over two
 * sets of rows).  geom.batch is the number of prompts b.
 *   q             bf16 [b, N, g*h_kv, d]  the new tokens' queries
 *   k_new, v_new  bf16 [b, N, h_kv, d]    optional (both NULL or both set): the new tokens, appended to their tails
 *                                         at row len with position seen, as mkv_decode_step does
 *   prefix        the shared rows: an mkv_cache of b * h_kv units; not changed
 *   mom           their moments (b * h_kv units); may be NULL if p->correction is 0
 *   tail          the sequences' own rows: an mkv_cache of (b * N) * h_kv units; y and y_len are not used
 *   out           bf16 [b, N, g*h_kv, d]  dense
 *   lse           fp32 [b, N, g*h_kv]     optional: natural log of the normaliser
 * For query head h of sequence i, unit (b, kv): the softmax over the shared
 * rows 0..len-1, the tail's rows 0..len-1, the new token and, if p->correction
 * and n > 0, the moment term with logit log n + scale q.mu_k and value mu_v +
 * scale C' q (p->order 1) or mu_v (order 0), as in mkv_decode_step; p->C16 and
 * p->C_split have that call's meaning; p->early_load is accepted and changes
 * nothing (the shared rows are loaded early wherever that is always safe).  A
 * sequence with nothing at all to attend to gets zeros and lse -infinity.
 * An append past the tail's capacity records MKV_ERR_CAPACITY (info: the tail's
 * unit), still attends over the new token and leaves the tail as it is; a
 * length outside 0..capacity is recorded as MKV_ERR_CAPACITY and taken as the
 * nearer end.  Scores, statistics and sums are fp32; the softmax weights enter
 * the product with the values rounded to bf16 (about a normaliser of the
 * rounded weights; mkv_decode_step has them in two parts, and an fp32 output), as the output is, and the order-1 product takes an fp32 C'
 * as two bf16 parts.
 * Requirements: q, k_new, v_new and out 16-byte aligned, lse 4; p as in
 * mkv_decode_step.
 */
MKV_API mkv_status mkv_prefix_step(mkv_geom geom, const mkv_seqs* seqs, const void* q, const void* k_new,
                                   const void* v_new, const mkv_cache* prefix, const mkv_moments* mom,
                                   const mkv_cache* tail, const mkv_decode_params* p, void* out, float* lse,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* The scores of every beam's continuations, read on the host during the call. */
typedef struct {
  const void* logits;    /* bf16 or fp32 [batch, beams, vocab]: adjacent tokens, strides below      */
  int32_t f32;           /* 1: fp32 logits; 0: bf16                                                */
  int64_t logits_batch;  /* elements from batch item to batch item, any value at least 0           */
  int64_t logits_beam;   /* and from beam to beam                                                  */
  const float* score;    /* fp32 [batch, beams]: a beam's score so far; -infinity: not alive       */
  const int32_t* done;   /* int32 [batch, beams] optional: not 0 where a beam has ended            */
  int32_t end_token;     /* the token that ends a beam, 0..vocab-1, or -1: none (done is then NULL) */
} mkv_beam_scores;

/*
 * Bytes of device workspace mkv_beam_select needs on the current device.
 * Returns 0 if the arguments are invalid.  Only its first 256 bytes need to be zero before its first use.
 */
MKV_API size_t mkv_beam_select_workspace_size(int32_t batch, int32_t beams, int32_t vocab, int32_t n_out);

/*
 * The n_out best continuations of every batch item, best first.  A live beam
 * that has not ended continues with token t at score[beam] + logit[t] -
 * log sum exp(logits of the beam); one that has ended continues only with
 * end_token, at its own score (its logits do not matter).  Equal ones: the lower beam, then the lower token.
 *   parent     int32 [batch, n_out]  the beam that is continued
 *   token      int32 [batch, n_out]  by which token
 *   score_out  fp32  [batch, n_out]
 *   done_out   int32 [batch, n_out]  optional: 1 where the beam had ended or the token is end_token
 * Tokens with a logit of -infinity, and beams whose logits all are, do not take
 * part.  Where there are fewer continuations than n_out, the slots that are left have parent and
 * token -1, score -infinity and done 0.  A live beam that has not ended with a logit
 * that is NaN or +infinity, and any beam with a score that is, take no part and are
 * recorded as MKV_ERR_INVALID_ARG (info: batch item * beams + beam).
 * Exponentials, and sums of 16 of them, are fp32; their sums are kept in pairs of fp32 values, logs and
 * scores in fp64.  An error of a few 1e-7, whatever the vocabulary, decides between continuations of
 * different beams that are nearer to each other than that.
 * score_out may be score, and done_out may be done, where n_out = beams; else
 * outputs do not overlap inputs.
 * Requirements: batch 1..65535, beams 1..64, n_out 1..64, vocab 1..2^24; logits aligned to their
 * type, the others to 4 bytes; workspace 256.
 */
MKV_API mkv_status mkv_beam_select(int32_t batch, int32_t beams, int32_t vocab, const mkv_beam_scores* scores,
                                   int32_t n_out, int32_t* parent, int32_t* token, float* score_out, int32_t* done_out,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* One layer's states: (b * N) * h_kv units.  mom.n NULL: no moments. */
typedef struct {
  mkv_cache cache;
  mkv_moments mom;
} mkv_beam_layer;

/*
 * Slot j of batch item i takes the state that slot parent[i][j] has, in every
 * layer, in place: rows 0..len-1 of K, V and pos, len and seen, with y and
 * y_len where the cache has them (rows 0..y_len-1), and the moments where given.  Rows at or above the new
 * length are left as they are.  Packed copies of C (mkv_moments_pack_bf16,
 * mkv_moments_pack_split) are the caller's to make again.  geom.batch is the
 * number of batch items b; geom's group is not used.
 *   n_seqs  N: slots per batch item, 1..256
 *   parent  int32 [b, N]  0..N-1, several slots may have the same; -1: the slot stays as it is
 *   layers  HOST array of n_layers entries, copied during the call; no array of a cache or of moments in two of them (MKV_ERR_INVALID_ARG)
 * A batch item with another parent is left as it is and recorded as
 * MKV_ERR_INVALID_ARG (info: the batch item); a length (len or y_len) outside 0..capacity is
 * recorded as MKV_ERR_CAPACITY (info: the unit) and rows are copied up to the nearer end.
 * Requirements: b * h_kv <= 65535 (else MKV_ERR_SHAPE); as mkv_cache and mkv_moments.
 * The workspace is 256 bytes, zero-filled before its first use.  Two launches for every 64 layers.
 */
MKV_API mkv_status mkv_beam_reorder(mkv_geom geom, int32_t n_seqs, int32_t n_layers, const mkv_beam_layer* layers,
                                    const int32_t* parent, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MKV_BEAM_H */
