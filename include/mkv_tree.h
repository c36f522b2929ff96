/*
 * mkv_tree.h -- speculative decoding over a compressed cache, and rotary
 * positions: the calls that sit beside mkv.h's in a serving step.
 *
 * A drafted tree is N nodes per batch item, each a token that continues its
 * parent; the model verifies all of them in one pass.
 *
 *   mkv_tree_build    the nodes' visibility words and positions from their
 *                     parents, once per drafted tree
 *   mkv_rope          rotary positions with one or more axes, on queries and
 *                     keys: of the drafted nodes before mkv_tree_step, of a
 *                     prompt before mkv_compress, of one token before
 *                     mkv_decode_step; inverse = 1 is its gradient
 *   mkv_norm_rope     the same with the norms of queries and keys per head in
 *                     front, for models that have them; mkv_norm_rope_grad is
 *                     its gradient
 *   mkv_tree_step     attention of every node over the retained cache, the
 *                     nodes it sees and the moment term of the evicted tokens,
 *                     in one normaliser; the cache is not changed
 *   mkv_tree_commit   the accepted path's keys and values into the caches of
 *                     all layers, once per verified tree
 *
 * Conventions are those of mkv.h (device pointers, caller-owned memory,
 * stream order, statuses, the workspace's error word read by
 * mkv_get_device_error), except that these tensors may be strided as stated.
 */
#ifndef MKV_TREE_H
#define MKV_TREE_H

#include "mkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MKV_TREE_MAX_NODES 256
#define MKV_ROPE_MAX_AXES 4
#define MKV_ROPE_MAX_TENSORS 4

/*
 * The drafted nodes of every batch item.
 *   n_nodes  N: nodes per batch item in the tensors, 1..256
 *   count    int32 [b]  optional: the nodes in use of each item, 0..N (NULL:
 *            all N).  Nodes at or above it are not read as keys; their outputs
 *            are zeros and their lse -infinity.  A count outside 0..N is
 *            taken as the nearer end and recorded as MKV_ERR_INVALID_ARG.
 *   mask     uint32 [b, N, ceil(N / 32)]: bit a % 32 of word a / 32 of row i
 *            is set where node i sees node a (itself included); any pattern is
 *            allowed, a row without a bit sees the cache and the moments alone
 * Strides of the tensors below, in elements; 0 stands for the dense value.
 * All are multiples of 8 and not below it.
 *   q_node, q_batch    q [b, N, g*h_kv, d]: from node to node (dense g*h_kv*d),
 *                      from batch item to batch item (dense N * q_node)
 *   kv_node, kv_batch  k and v [b, N, h_kv, d] (dense h_kv*d, N * kv_node)
 */
typedef struct {
  int32_t n_nodes;
  const int32_t* count;
  const uint32_t* mask;
  int64_t q_node;
  int64_t q_batch;
  int64_t kv_node;
  int64_t kv_batch;
} mkv_tree;

/*
 * Visibility words and positions of drafted trees, one launch on `stream`.
 *   parents  int32 [b, N]  each node's parent, below the node itself, or -1
 *            for a node that continues the cache; another value is recorded
 *            as MKV_ERR_INVALID_ARG (info: the batch item) and taken as -1
 *   count    int32 [b] optional, as in mkv_tree
 *   base     optional int32, base[i * base_stride] for batch item i: the position
 *            of a node without parent (a cache's `seen` with stride h_kv);
 *            NULL: 0
 *   mask     uint32 [b, N, ceil(N / 32)]: the node and its ancestors; rows of
 *            nodes that are not in use are zeros
 *   pos      int32 [b, N]: base plus the number of ancestors (base for nodes
 *            that are not in use); NULL: not written
 * The workspace is 256 bytes, zero-filled before its first use.
 */
MKV_API mkv_status mkv_tree_build(int32_t batch, int32_t n_nodes, const int32_t* parents, const int32_t* count,
                                  const int32_t* base, int64_t base_stride, uint32_t* mask, int32_t* pos,
                                  void* workspace, size_t workspace_bytes, void* stream);

/*
 * Bytes of device workspace mkv_tree_step needs for this geometry, N and cache
 * capacity on the current device, and for every smaller batch, N and capacity
 * (one workspace sized for the largest serves them all).  Returns 0 if the
 * arguments are invalid.  The workspace must be zero-filled before its first use; every call leaves
 * it ready for the next one.
 */
MKV_API size_t mkv_tree_workspace_size(mkv_geom geom, int32_t n_nodes, int32_t capacity);

/*
 * One layer's attention of every drafted node (Algorithm 1 Phase 2 with the
 * visible nodes in place of the appended token).
 *   q     bf16 [b, N, g*h_kv, d]
 *   k, v  bf16 [b, N, h_kv, d]     keys (rotated, where the model does) and values of the nodes
 *   out   bf16 [b, N, g*h_kv, d]   dense
 *   lse   fp32 [b, N, g*h_kv]      optional: natural log of the normaliser
 * For query head h of node i, unit (b, kv): the softmax over the retained
 * rows 0..len-1, the nodes a that i sees and, if p->correction and n > 0, the
 * moment term with logit log n + scale q.mu_k and value mu_v + scale C' q
 * (p->order 1) or mu_v (order 0), as in mkv_decode_step; p->C16, p->C_split
 * and p->early_load have that call's meaning (with early_load the caller's
 * guarantee also covers tree->count and tree->mask, and a count or a number of
 * evicted tokens that changed is recorded as a length is; q, k and v are read
 * after the dependency wait).  A node that sees
 * nothing at all gets zeros and lse -infinity.  A node's key or value that is
 * not finite reaches only the nodes that see it; queries and keys of nodes
 * that are not in use and cache rows at or above len reach nothing.  A length
 * outside 0..capacity is recorded as MKV_ERR_CAPACITY and taken as the nearer
 * end.  Scores, statistics and sums are fp32; the softmax weights enter the
 * product with the values rounded to bf16, as the output is, and the order-1
 * product takes an fp32 C' as two bf16 parts (16 to 17 significant bits, those of
 * mkv_moments_pack_split).
 * Requirements: q, k, v and out 16-byte aligned, lse and mask 4; mom may be
 * NULL if p->correction is 0.
 */
MKV_API mkv_status mkv_tree_step(mkv_geom geom, const mkv_tree* tree, const void* q, const void* k, const void* v,
                                 const mkv_cache* cache, const mkv_moments* mom, const mkv_decode_params* p, void* out,
                                 float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* One layer of a commit: its cache and the nodes' keys and values (as given
 * to mkv_tree_step). */
typedef struct {
  mkv_cache cache;
  const void* k;
  const void* v;
} mkv_tree_layer;

/*
 * Takes an accepted path into the cache of every layer: for batch item i and
 * each of its KV heads, row len + j = node path[i][j] (keys, values, position
 * seen + j) for j < n_path[i]; then len and seen grow by n_path[i].  The
 * caches' y rows stay valid (rows are added above y_len).
 *   layers    HOST array of n_layers entries (new addresses at every step where
 *             k and v are new tensors), copied during the call; k and v
 *             have the strides tree->kv_node and kv_batch in every layer
 *   path      int32 [b, path_len]  node indices, root first
 *   n_path    int32 [b]            accepted nodes, 0..path_len
 * tree->count and tree->mask are not read.  geom's group is not used.
 * A unit whose rows would pass its capacity (MKV_ERR_CAPACITY), or whose item
 * has n_path or a node index out of range (MKV_ERR_INVALID_ARG), is left as it
 * is and recorded (info: batch item * h_kv + head).
 * The workspace is 256 bytes, zero-filled before its first use.  One launch
 * for every 64 layers.
 */
MKV_API mkv_status mkv_tree_commit(mkv_geom geom, const mkv_tree* tree, int32_t n_layers,
                                   const mkv_tree_layer* layers, const int32_t* path, int32_t path_len,
                                   const int32_t* n_path, void* workspace, size_t workspace_bytes, void* stream);

/* Rotation parameters, read on the host during the call. */
typedef struct {
  int32_t rot_dim;     /* dims rotated, from dim 0: a multiple of 16, at most head_dim; the others are copied */
  int32_t neighbours;  /* 0: frequency f turns dims (f, f + rot_dim / 2); 1: dims (2 f, 2 f + 1)              */
  int32_t inverse;     /* 1: by the negative angle (the gradient of the rotation, and its undoing)           */
  int32_t n_axes;      /* axes of the positions, 1..4                                                      */
  float inv_freq[64];  /* radians per position of frequency f < rot_dim / 2; finite, magnitude at most 2^20 */
  int32_t axis[64];    /* the axis whose position turns frequency f, 0..n_axes-1                           */
} mkv_rope_params;

/* One tensor: bf16 [b, tokens, heads, d] with the strides given, in elements
 * (the d values of a head are adjacent).  out may be in itself with the same
 * strides (in place); else the two must not overlap. */
typedef struct {
  const void* in;
  void* out;
  int32_t heads;
  int64_t in_batch, in_token, in_head;
  int64_t out_batch, out_token, out_head;
} mkv_rope_tensor;

/*
 * Rotary positions of up to four tensors of the same tokens (a layer's
 * queries and keys), one launch on `stream`: pair (x, y) of frequency f becomes
 * (x cos - y sin, x sin + y cos) of the angle pos[axis[f]] * inv_freq[f].
 *   pos   int32: pos[a * pos_axis + i * pos_batch + t] of axis a, batch item i,
 *         token t; strides in elements (0 repeats a position for every axis
 *         or batch item), any int32 values
 * The angle is reduced exactly (in units of 2^-64 turns), whatever the
 * position; products are fp32 and rounded once to bf16.  tokens may be 0
 * (nothing is launched).
 * Requirements: head_dim 64 or 128; pointers 16-byte aligned; strides
 * multiples of 8 elements.
 */
MKV_API mkv_status mkv_rope(int32_t batch, int32_t tokens, int32_t head_dim, const int32_t* pos, int64_t pos_axis,
                            int64_t pos_batch, const mkv_rope_params* p, int32_t n_tensors,
                            const mkv_rope_tensor* tensors, void* stream);

/* A tensor of mkv_norm_rope, with the weights of its norm. */
typedef struct {
  mkv_rope_tensor t;    /* as in mkv_rope                                                              */
  const void* weight;   /* bf16 or fp32 [d], or one row for each head; 16-byte aligned; NULL: ones     */
  int64_t weight_head;  /* elements from one head's row to the next, a multiple of 8 and at least d; 0: */
                        /* one row for all heads                                                       */
  int32_t weight_f32;   /* 1: fp32 weights; 0: bf16                                                    */
} mkv_norm_rope_tensor;

/*
 * Norms of queries and keys per head, and their rotary positions, in one pass
 * (one launch on `stream`): for every head of every token, n = x (mean x^2 +
 * eps)^(-1/2) weight over the d values, then n rotated as mkv_rope does.
 * Everything is fp32 between x and the one rounding to bf16; sums of squares
 * that pass fp32's range are taken of smaller values, so that any finite x has
 * its norm.  Arguments, layouts and requirements as in mkv_rope, with
 * p->inverse 0, no two tensors with one out, and eps a normal number above 0
 * (2^-126 or more: below fp32's range squares lose their digits).
 */
MKV_API mkv_status mkv_norm_rope(int32_t batch, int32_t tokens, int32_t head_dim, const int32_t* pos, int64_t pos_axis,
                                 int64_t pos_batch, const mkv_rope_params* p, float eps, int32_t n_tensors,
                                 const mkv_norm_rope_tensor* tensors, void* stream);

/* A tensor of mkv_norm_rope_grad: bf16 [b, tokens, heads, d] each with the strides given.  dx may be x or dy
 * with the same strides (in place); else it must not overlap them.  No two tensors have one dx or dweight
 * (the gradient of weights that tensors share is the sum of theirs, the caller's to add). */
typedef struct {
  const void* x;        /* what mkv_norm_rope read                                            */
  const void* dy;       /* the gradient of what it wrote                                     */
  void* dx;             /* the gradient of x                                                 */
  int32_t heads;
  int64_t x_batch, x_token, x_head;
  int64_t dy_batch, dy_token, dy_head;
  int64_t dx_batch, dx_token, dx_head;
  const void* weight;   /* as in mkv_norm_rope_tensor                                        */
  int64_t weight_head;
  int32_t weight_f32;
  float* dweight;       /* fp32 [d], or dense [heads, d] where weight_head is not 0: the gradient of the */
                        /* weights, overwritten; NULL: not wanted                           */
} mkv_norm_rope_grad_tensor;

/*
 * Bytes of device workspace mkv_norm_rope_grad needs for these tensors (only
 * heads and weight_head are read) on the current device.  Returns 0 if the
 * arguments are invalid.  The workspace needs no initialisation.
 */
MKV_API size_t mkv_norm_rope_grad_workspace_size(int32_t batch, int32_t tokens, int32_t head_dim, int32_t n_tensors,
                                                 const mkv_norm_rope_grad_tensor* tensors);

/*
 * The gradient of mkv_norm_rope, with that call's pos, p and eps: dx of every
 * tensor, and the sums over tokens (and over heads, where they share weights)
 * that are dweight.  The sums are fp32 in an order that is the same on every
 * call with the same sizes.  With tokens 0, dweight becomes zeros.  Two launches on `stream` (one without
 * dweight).
 */
MKV_API mkv_status mkv_norm_rope_grad(int32_t batch, int32_t tokens, int32_t head_dim, const int32_t* pos,
                                      int64_t pos_axis, int64_t pos_batch, const mkv_rope_params* p, float eps,
                                      int32_t n_tensors, const mkv_norm_rope_grad_tensor* tensors, void* workspace,
                                      size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* MKV_TREE_H */
