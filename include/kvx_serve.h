/*
 * kvx_serve.h -- serving on a translated cache that is held in 8 bits, bounded
 * by a window with sinks, and decoded by drafted trees (gfx950 / MI355X).
 *
 *   kvx_attn_append_coded  new keys (rotated) and values into a cache of 8 bits
 *   kvx_attn_pack          a cache into one of 8 bits, all layers
 *   kvx_attn_unpack        a cache of 8 bits into one of the model's dtype
 *   kvx_attn_tree          what the tokens of drafted trees see, by their parents
 *   kvx_attn_forward_view  attention over caches of 8 bits, with sinks, of trees
 *   kvx_attn_accept        the accepted path of every tree, all layers
 *
 * Notation, status codes, checks, KVX_VALIDATE and KVX_FAULT are those of
 * kvx_attn.h; calls are asynchronous on the given stream, allocate nothing and
 * can be captured into a graph.
 */
#ifndef KVX_SERVE_H
#define KVX_SERVE_H

#include "kvx_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Numbers of 8 bits: integers from -127 to 127, or e4m3 floating point (up to
 * 448, a number with all of its low seven bits set is none). */
typedef enum { KVX_CODE_I8 = 0, KVX_CODE_E4M3 = 1 } kvx_code;

/* A cache of 8 bits: number = code * scale of its row (a key's or value's
 * head_dim numbers).  A row's scale is the smallest power of two, from 2^-100
 * on, under which its largest magnitude is not past the largest code (127 or
 * 448); magnitudes over 2^127 count as 2^127.  So a number is one of bf16 and
 * reading back is exact.  A row that holds an infinity or NaN has a NaN for its
 * scale and reads as NaN.  Scales are powers of two from 2^-100 to 2^122, or NaN:
 * others give unspecified numbers. */
typedef struct {
  kvx_cache codes;         /* k and v: one byte a number; as kvx_attn.h, 16-byte aligned
                              rows, strides in bytes */
  void* scale;             /* pairs of bf16, (key's, value's), 4-byte aligned */
  int64_t scale_stride[4]; /* in pairs, for (layer, batch, head, token) or (layer, block,
                              head, slot); all zero: dense */
  int32_t code;            /* kvx_code */
} kvx_cache8;

/* kvx_attn_append into a cache of 8 bits (io's own cache is ignored): keys are
 * rotated in 64 bits and rounded once, to their codes.  bf16 models only
 * (KVX_EUNSUPPORTED). */
kvx_status kvx_attn_append_coded(const kvx_attn* attn, const kvx_attn_io* io,
                                 const kvx_cache8* cache8, void* stream);

/* One conversion of the first tokens[b] slots of every context, all layers; of slots
 * past either cache's capacity nothing is read or written. */
typedef struct {
  int32_t batch;
  const int32_t* tokens;     /* device [batch] */
  kvx_cache cache;           /* of the model's dtype: pack reads it, unpack writes it */
  const kvx_cache8* cache8;  /* other memory than cache's */
} kvx_pack_io;

kvx_status kvx_attn_pack(const kvx_attn* attn, const kvx_pack_io* io, void* stream);
kvx_status kvx_attn_unpack(const kvx_attn* attn, const kvx_pack_io* io, void* stream);

/* Drafted trees: the new tokens of a context are a tree's nodes (or several
 * trees'), each behind its parent. */
typedef struct {
  int32_t batch;
  int32_t rows;              /* nodes of all contexts */
  const int32_t* q_start;    /* device [batch + 1]; NULL: one node each (rows == batch) */
  const int32_t* tokens;     /* device [batch], cached tokens with the nodes */
  const int32_t* parent;     /* device [rows], index of a node's parent among its
                                context's; negative: a root.  An index that is not less
                                than the node's own counts as negative */
  int32_t window;            /* positions that a node sees, 0: all */
  int32_t sink;              /* first positions that stay visible outside of it */
  const int32_t* shift;      /* device [batch] or NULL (0): position less slot (evictions
                                let positions run ahead of slots); added to pos only */
  int32_t words;             /* of a node's mask, 1..64; nodes of a context from 32 words on
                                see nothing drafted */
  uint32_t* mask;            /* [rows][words]: bit k % 32 of word k / 32 is set if the node
                                sees node k of its context: itself and its ancestors, fewer
                                than `window` positions before it or at a position < sink */
  int32_t* depth;            /* [rows] ancestors of the node, or NULL */
  int32_t* pos;              /* [n_axes][rows] position n - m + depth + shift, or NULL */
} kvx_tree_io;

kvx_status kvx_attn_tree(const kvx_attn* attn, const kvx_tree_io* io, void* stream);

/* What a call of kvx_attn_forward_view sees beyond its kvx_attn_io. */
typedef struct {
  const kvx_cache8* cache8;  /* the cache, instead of io's (bf16 models only); or NULL */
  int32_t sink;              /* with a window: slots j < sink are visible outside of it:
                                (j <= p or j < prefix[b]) and (window == 0 or
                                j > p - window or j < sink) */
  const uint32_t* tree;      /* NULL, or device [rows][tree_words] as kvx_attn_tree leaves
                                it: new token i, at slot p = n - m + i >= 0 and position
                                n - m + depth[i], sees of slots j < n - m those that
                                window and sink leave it, and of the new tokens those
                                of its mask.  io's prefix has to be NULL */
  int32_t tree_words;        /* >= 1, 32 tree_words >= max_new */
  const int32_t* depth;      /* device [rows], taken into 0..m - 1; NULL: i; with a tree
                                only */
} kvx_attn_view;

/* kvx_attn_forward under a view; NULL, or an empty one, is kvx_attn_forward
 * itself.  Numbers of 8 bits enter products exactly; a value's scale is applied
 * before the weight's rounding to bf16 or exactly after it. */
kvx_status kvx_attn_forward_view(const kvx_attn* attn, const kvx_attn_io* io,
                                 const kvx_attn_view* view, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* The accepted nodes of every context's tree move, in all layers, to the first
 * slots of its new tokens: node path[b][i] from slot n - m + path[b][i] to slot
 * n - m + i, i < count[b]. */
typedef struct {
  int32_t batch;
  const int32_t* q_start;    /* device [batch + 1], as the forward call's; NULL: one each */
  const int32_t* tokens;     /* device [batch], cached tokens with the nodes */
  const int32_t* path;       /* device [batch][max_path], rising; entries outside of 0..m - 1
                                and slots past the capacity move nothing */
  int32_t max_path;          /* >= 1 */
  const int32_t* count;      /* device [batch], taken into 0..min(m, max_path) */
  kvx_cache cache;           /* ignored with cache8 */
  const kvx_cache8* cache8;  /* or NULL */
  int32_t* tokens_out;       /* device [batch] n - m + count, or NULL; not memory of
                                tokens, count, path or q_start (KVX_EINVAL) */
} kvx_accept_io;

/* No two contexts may share a block of their new tokens. */
kvx_status kvx_attn_accept(const kvx_attn* attn, const kvx_accept_io* io, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KVX_SERVE_H */
