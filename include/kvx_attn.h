/*
 * kvx_attn.h -- decoding on a translated cache (gfx950 / MI355X).
 *
 * kvx_translate leaves the target model's K/V cache; the target model then
 * decodes on it.  Per layer it stores its new tokens' keys and values, attends
 * to the cache, and, to stay within a memory budget, drops the cached tokens
 * that received the least attention:
 *
 *   kvx_attn_append   rotary positions (one or several axes) of new queries
 *                     and keys, new keys and values into the cache
 *   kvx_attn_forward  attention of the new tokens over the cache
 *   kvx_attn_mass     attention weight that each cached token received
 *   kvx_attn_evict    keep the cached tokens of the largest weight, all layers
 *
 * Notation: context b has n = tokens[b] cached tokens, the new ones included,
 * in slots 0 .. n-1; its m new tokens are the last ones, so that new token i
 * has slot p = n - m + i.  Query head h reads KV head h / (Hq / Hkv).  New
 * tokens of all contexts stand one after another in rows, context b's from
 * row q_start[b] on.  A context may outgrow its cache (a replayed step counts
 * on without the host): slots keep their numbers, those past the capacity are
 * not stored, seen or kept, and all others stay as they are.
 *
 * Status codes and dtypes are those of kvx.h.  No function throws.  Every
 * host-visible argument is checked before anything is enqueued.  Device
 * contents (q_start, tokens, prefix, block_table) are trusted unless
 * KVX_VALIDATE=1 (then, after synchronising the stream, they are copied back
 * and checked; KVX_EDATA on a violation).  KVX_FAULT=launch applies as to
 * kvx_translate.  Calls are asynchronous on the given stream, allocate nothing
 * and can be captured into a graph: lengths are read on the device.
 */
#ifndef KVX_ATTN_H
#define KVX_ATTN_H

#include "kvx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The attention side of a target model; consumed by kvx_attn_create. */
typedef struct {
  kvx_model model;           /* cache geometry, RoPE base or inv_freq table */
  int32_t n_heads;           /* query heads, a multiple of model.n_kv_heads */
  int32_t dtype;             /* kvx_dtype of q, k, v, outputs and the cache */
  double scale;              /* score scale; 0: 1 / sqrt(head_dim) */
  double softcap;            /* c > 0: scores s become c * tanh(s / c); 0: none.  Both and
                                scale / softcap are numbers that fp32 holds */
  int32_t n_axes;            /* position axes, 1..4 */
  const uint8_t* pair_axis;  /* host [head_dim/2], position axis of rotary pair
                                (i, i + head_dim/2); NULL: all axis 0.  Copied. */
} kvx_attn_desc;

/* A cache of the target model, as kvx_translate writes it: strides in
 * elements for (layer, batch, head, token) of a contiguous cache, for (layer,
 * block, head, slot) of a paged one; all zero: [L][B][H][capacity][D], or
 * [L][num_blocks][H][block_size][D]. */
typedef struct {
  void* k;
  void* v;
  int64_t stride[4];
  int32_t capacity;           /* contiguous: tokens per context */
  const int32_t* block_table; /* paged: device [batch][max_blocks]; NULL: contiguous.
                                 Entries of slots >= tokens[b], and of slots that no
                                 new token's window reaches, are not read through */
  int32_t block_size;         /* tokens per block, > 0 */
  int32_t max_blocks;         /* table entries per context, > 0 */
  int32_t num_blocks;         /* physical blocks, > 0 */
} kvx_cache;

/* One layer's call of append, forward or mass; each reads the fields named
 * for it and ignores the others. */
typedef struct {
  int32_t batch;
  int32_t layer;             /* layer of the cache, 0-based */
  int32_t rows;              /* new tokens of all contexts */
  int32_t max_new;           /* most new tokens that any context has (>= 1; chooses
                                the kernel: results agree to the errors below) */
  const int32_t* q_start;    /* device [batch + 1], first row of each context, from 0
                                to rows; NULL: one new token each (rows == batch) */
  const int32_t* tokens;     /* device [batch], cached tokens with the new ones */
  kvx_cache cache;
  /* append: new rows [rows][heads][head_dim], strides (row, head) in elements,
   * head_dim unit-stride; new_q may be NULL (only keys and values), or
   * new_k and new_v both NULL (only queries) */
  const void* new_q;
  const void* new_k;
  const void* new_v;
  int64_t new_q_stride[2];
  int64_t new_k_stride[2];
  int64_t new_v_stride[2];
  const int32_t* pos;        /* append: device [n_axes][rows]; NULL: slots, on every axis */
  /* rotated queries: written by append (may be new_q itself), read by forward
   * and mass */
  void* q;
  int64_t q_stride[2];
  /* forward and mass: visibility.  New token of slot p >= 0 sees slot j < n if
   * (j <= p or j < prefix[b]) and (window == 0 or j > p - window).  A window counts
   * slots: after an eviction it reaches further back than as many positions. */
  int32_t window;            /* >= 0 */
  const int32_t* prefix;     /* device [batch] or NULL (none) */
  /* forward: outputs; a row that sees nothing gets out 0, lse -inf */
  void* out;
  int64_t out_stride[2];
  float* lse;                /* [rows][n_heads] log-sum-exp of the visible scores;
                                forward: written unless NULL; mass: read */
  /* mass: [batch][n_kv_heads][mass_capacity], slot-indexed; mass_in NULL is
   * zero and may be mass itself.  Slots >= n are copied from mass_in (or 0).
   * tokens[b] <= mass_capacity is wanted: slots past it get no weight. */
  const float* mass_in;
  float* mass;
  int32_t mass_capacity;
} kvx_attn_io;

/* One eviction over all layers. */
typedef struct {
  int32_t batch;
  const int32_t* tokens;     /* device [batch] */
  int32_t keep;              /* tokens kept per context, >= 1 */
  int32_t sink;              /* the first `sink` tokens are kept always */
  int32_t recent;            /* and the last `recent`; sink + recent <= keep */
  kvx_cache src;
  kvx_cache dst;             /* where kept rows go, slots 0 .. ; k == NULL: in
                                place.  Other memory than src's */
  const float* mass;         /* [layers][batch][n_kv_heads][mass_capacity]; cached
                                tokens past it count as weight 0 */
  float* mass_out;           /* same shape, or NULL: the kept tokens' weights, then
                                zeros up to min(mass_capacity, max(keep, n)); may be
                                mass itself */
  int32_t mass_capacity;
  int32_t* kept;             /* [layers][batch][n_kv_heads][keep] old slots of the
                                kept tokens in rising order, then -1 */
  int32_t* tokens_out;       /* [batch] min(n, keep), or NULL; not tokens itself */
} kvx_evict_io;

typedef struct kvx_attn kvx_attn;

/* Validate the description and copy its tables to the current device
 * (synchronous).  Errors: KVX_EINVAL, KVX_EUNSUPPORTED (head_dim not a
 * multiple of 16 or above 256), KVX_ENOMEM, KVX_EHIP.  On error *out is NULL. */
kvx_status kvx_attn_create(const kvx_attn_desc* desc, kvx_attn** out);

/* Release (NULL-safe); no call that uses it may still be running. */
void kvx_attn_destroy(kvx_attn* attn);

/* Rotate new queries into q and new keys into the cache, copy new values into
 * the cache.  Angles are formed in 64 bits, rotations computed in fp32 and
 * rounded once.  Rows of negative slots (n < m) and slots past the cache's
 * capacity are not stored.  KVX_EUNSUPPORTED: rows or buffers that are not
 * 16-byte aligned (here and below). */
kvx_status kvx_attn_append(const kvx_attn* attn, const kvx_attn_io* io, void* stream);

/* Device bytes that kvx_attn_forward needs for any call of this handle. */
kvx_status kvx_attn_workspace_bytes(const kvx_attn* attn, size_t* bytes);

/* Attention of the rows over their contexts' cache.  The workspace is device
 * memory of the caller's, 16-byte aligned, not read before it is written;
 * calls that share one must not overlap.  Scores, softmax statistics and sums
 * are fp32; weights are rounded to bf16 for their product with bf16 values.
 * Capped scores err by 2^-21 of the terms of their dot product (here and in
 * kvx_attn_mass), here those of bf16 calls with caps up to 128 by 2^-22 of the cap.
 * Values whose magnitudes add up to less than 2^104 over a context's slots give
 * finite outputs whatever the scores are.
 * Results depend on no order of execution: equal calls give equal bits. */
kvx_status kvx_attn_forward(const kvx_attn* attn, const kvx_attn_io* io, void* workspace,
                            size_t workspace_bytes, void* stream);

/* mass = mass_in + the weight exp(score - lse) of each cached token, summed
 * over the new tokens and the query heads of its KV head that see it. */
kvx_status kvx_attn_mass(const kvx_attn* attn, const kvx_attn_io* io, void* stream);

/* Keep min(n, keep) tokens per (layer, context, KV head): the protected ones,
 * and of the others those of the largest mass, ties to the lowest slot, a NaN
 * counting as -inf.  Kept rows move to the front in their order.  Every head
 * of every layer keeps the same number, so one length per context serves.
 * Keys stay rotated at their original positions.  In place, no two contexts may
 * share a block of kept or dropped tokens. */
kvx_status kvx_attn_evict(const kvx_attn* attn, const kvx_evict_io* io, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KVX_ATTN_H */
