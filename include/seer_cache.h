/*
 * seer_cache.h -- C ABI of libseer.so, third part: keeping the cache of a long
 * generation small.
 *
 *   seer_kv_append_q4    keys and values of new tokens into a paged cache held in 4
 *                        bits, the keys rotated on the way
 *   seer_kv_read         tokens of a paged cache back out (a cached prefix, for the next
 *                        piece of a prompt)
 *   seer_paged_attn_q4   attention of new tokens over a cache held in 4 bits
 *   seer_kv_weights      the attention weight that each cached key gets from some queries
 *   seer_kv_evict        the keys of the largest weight, and their values, into new pages
 *
 * The conventions of seer.h and seer_decode.h hold: device pointers of the current
 * device that the caller owns, asynchronous on `stream`, validation on the host before
 * anything is launched, no state between calls, no allocation, reentrant, nothing that
 * a HIP graph cannot capture, and sizes that change from step to step read on the
 * device.
 *
 * 4 bits.  Each `group` (32 or 64) successive elements of a key or value of one head share
 * two bf16 numbers, a step and a middle; element x of code c, 0 to 15, stands for
 *   middle + step (c - 7.5).
 * A token's elements x are held so: middle = bf16(max / 2 + min / 2), in fp32 and to nearest; step the
 * least bf16 number from which 7.5 steps reach every element from the middle (0 where the
 * middle is them all, else at least 2^-100); c = floor((x - middle) / step) + 8, within 0 to
 * 15, decided exactly: the code whose value is nearest, the upper of two equally near ones.  So a value is off
 * by half a step at most, which is 1/30 of the group's range and up to 1/128 of that more (and
 * up to 2^-9 of the middle more, where bf16 rounds that).
 * A group that holds a value which is not finite, or beyond 2^127, is held as step NaN and
 * reads as NaN.  A head's codes are head_dim / 2 bytes, element 2 i in the low half of byte i;
 * its params head_dim / group (step, middle) pairs.  With 5 (group 32) or 4.5 (64) bits an element, head_dim 128
 * takes 80 or 72 bytes a token and head, where bf16 takes 256.
 */
#ifndef SEER_CACHE_H
#define SEER_CACHE_H

#include "seer_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Pages of one of K and V. */
typedef struct {
  void* data;              /* group 0: values [page][head][slot][head_dim]; else codes, bytes [page][head][slot][head_dim / 2] */
  void* params;            /* group 0: NULL; else (step, middle) pairs [page][head][slot][head_dim / group] */
  int64_t stride[3];       /* (page, head, slot) of data, in elements (codes: bytes); multiples of 16 bytes */
  int64_t param_stride[3]; /* of params, in pairs; multiples of head_dim / group */
} seer_kv_pool;

/* A paged cache: two pools and the table of the sequences' pages (seer_decode.h). */
typedef struct {
  int32_t heads_kv, head_dim;   /* head_dim 64 or 128 */
  int32_t dtype;                /* seer_dtype of the values; not read where group is 32 or 64 */
  int32_t group;                /* 0: the values themselves; 32 or 64: 4 bits */
  int32_t page_size, num_pages; /* both >= 1 */
  int32_t table_rows, max_pages;/* table: device [table_rows][max_pages], both >= 1 */
  int64_t table_stride;         /* elements between two rows of the table */
  const int32_t* table;
  seer_kv_pool k, v;
} seer_kv_cache;

/* Keys and values of tokens, [batch][heads_kv][tokens][head_dim]. */
typedef struct {
  int32_t batch, tokens, dtype;
  int32_t reserved;                 /* 0 */
  int64_t k_stride[3], v_stride[3]; /* (batch, head, token); multiples of 16 bytes */
  int64_t pos_stride;               /* elements between two batch entries of positions, rope_positions and rows */
} seer_kv_tokens;

/*
 * Token (b, s) of k and v goes to slot positions[b][s] of the sequence of table row rows[b][s]
 * (rows NULL: row b), in 4 bits.  rope (NULL: none) rotates k first, at position rope_positions[b][s] (NULL:
 * positions[b][s]), in fp32, and the rotated values are held without a rounding in between.  Padding, and what
 * is left as it is, as in seer_kv_append; two tokens of a call may not go to the same slot (its codes may be of one
 * and its params of the other then).
 * SEER_ERR_INVALID_ARG: a cache of group 0 (seer_kv_append serves it).
 * SEER_ERR_UNSUPPORTED: as seer_kv_append, and a group that head_dim is no multiple of or that is not 32 or 64.
 */
seer_status seer_kv_append_q4(const seer_kv_cache* cache, const seer_kv_tokens* desc, const seer_rope_params* rope,
                              const void* k, const void* v, const int32_t* positions, const int32_t* rope_positions,
                              const int32_t* rows, void* stream);

/*
 * What the cache holds for token (b, s), at slot positions[b][s] of the sequence of table row rows[b][s] (rows
 * NULL: row b), to k and v (desc: their layout and type; of a cache of group 0, its type).  The value of a code is
 * formed in fp32 (one rounding) and rounded to the type.  Tokens whose position or row is negative or beyond the table, or
 * whose page is none, read as 0.  k and v may not overlap the pools or each other.
 * SEER_ERR_UNSUPPORTED: as seer_kv_append.
 */
seer_status seer_kv_read(const seer_kv_cache* cache, const seer_kv_tokens* desc, void* k, void* v,
                         const int32_t* positions, const int32_t* rows, void* stream);

/* New tokens' queries, [batch][heads_q][tokens][head_dim], over a cache whose table row b is batch entry b's. */
typedef struct {
  int32_t batch, heads_q, tokens, dtype; /* heads_q % heads_kv == 0 */
  int64_t q_stride[3], o_stride[3];      /* (batch, head, token); multiples of 16 bytes */
  int64_t pos_stride;                    /* elements between two batch entries of positions and rope_positions */
} seer_kv_queries;

/* Workspace bytes of seer_paged_attn_q4 for these shapes (0 on invalid arguments). */
size_t seer_paged_attn_q4_workspace_bytes(const seer_kv_cache* cache, const seer_kv_queries* desc);

/*
 * seer_paged_attn over a cache held in 4 bits: o = softmax(sm_scale q K^T) V over the keys at slots t <=
 * positions[b][s] whose page exists; all that is said there of rows without keys, lse, the joining launch, workspace and
 * reproducibility holds.  rope rotates q at rope_positions[b][s] (NULL: positions[b][s]).  sm_scale at most 2^100.
 * K and V enter as the values that they stand for, exactly, and q whole (in fp32 or rotated: three bf16 parts); sums and
 * statistics are fp32.  A weight times the step of a value enters whole where o is fp32, and where it is bf16 in two bf16
 * parts, at most 2^-18 of it off; o is rounded once.
 * The cache is read once for each 16 query rows (heads_q / heads_kv x tokens).
 * Unseen slots and their params have no effect.  A seen key whose step is NaN makes the rows that see it NaN, a
 * value the elements of its group.
 * SEER_ERR_UNSUPPORTED: as seer_paged_attn and seer_kv_append_q4.
 */
seer_status seer_paged_attn_q4(const seer_kv_cache* cache, const seer_kv_queries* desc, const seer_rope_params* rope,
                               float sm_scale, const void* q, const int32_t* positions, const int32_t* rope_positions,
                               void* o, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* The weights of cached keys: device float [batch][heads_kv][width], key t of a sequence at element t. */
typedef struct {
  const float* in;  /* weights so far; not read when decay is 0 */
  float* out;       /* may be `in`, with its strides; any other overlap is not allowed */
  int64_t in_stride[2], out_stride[2]; /* (batch, head) */
  int32_t width;    /* keys from there on are not counted */
  float decay;      /* factor on the weights so far, finite */
} seer_kv_weight_buf;

/*
 * For every KV head h and slot t up to the largest of positions[b][.],
 *   out[b][h][t] = decay in[b][h][t] + sum over the query heads g of h and the tokens s that see t (t <= positions[b][s],
 *                  page exists) of exp(sm_scale q[b][g][s] . k[b][h][t] - lse[b][g][s]),
 * lse being what the attention of these queries returned (device float [batch][heads_q][tokens], contiguous): the softmax
 * weights that it gave to the key.  Rows whose lse is -inf count nothing.  out beyond these slots is left as it is.
 * The cache may be of either kind; only its keys are read (cache->v may hold NULLs).  rope, sm_scale, precision as in
 * seer_paged_attn_q4 (a cache of group 0: desc->dtype is its type; its bf16 products are exact, those of fp32 fp32).  No atomics: the
 * same bits every time.
 * SEER_ERR_UNSUPPORTED: as seer_paged_attn_q4.
 */
seer_status seer_kv_weights(const seer_kv_cache* cache, const seer_kv_queries* desc, const seer_rope_params* rope,
                            float sm_scale, const void* q, const int32_t* positions, const int32_t* rope_positions,
                            const float* lse, const seer_kv_weight_buf* weights, void* stream);

/* What seer_kv_evict reads and writes beside the cache. */
typedef struct {
  int32_t batch;                  /* sequences: table rows 0 .. batch - 1 */
  int32_t keep, first, last;      /* slots to keep, the first and last ones among them; first + last <= keep >= 1 */
  const int32_t* lengths;         /* device [batch]: slots in use */
  int32_t* new_lengths;           /* device [batch]; may be `lengths` */
  const int32_t* new_table;       /* device [batch][new_max_pages]: pages (of the same pools) that the kept slots go to */
  int64_t new_table_stride;
  int32_t new_max_pages;          /* page_size new_max_pages >= keep */
  int32_t width, new_width;       /* of weights (>= 1) and new_weights (>= keep) */
  int32_t reserved;               /* 0 */
  const float* weights;           /* device [batch][heads_kv][width] */
  float* new_weights;             /* device [batch][heads_kv][new_width] */
  int64_t stride[2], new_stride[2]; /* (batch, head) of weights and new_weights */
  int32_t* kept;                  /* device [batch][heads_kv][keep], contiguous */
} seer_kv_eviction;

/* Workspace bytes of seer_kv_evict for `batch` sequences of this cache (0: it needs none, or invalid arguments). */
size_t seer_kv_evict_workspace_bytes(const seer_kv_cache* cache, int32_t batch);

/*
 * Cuts every sequence to `keep` slots of each KV head: the `first` first and `last` last ones, and of the others those
 * with the largest weights, of equal ones the lower slot (-0 and 0 are equal, NaN is larger than any number; slots from `width` on
 * weigh 0).  A sequence of length n <= keep (lengths are taken within 0 and what its table has room for) keeps all n.  The
 * kept slots go to slots 0, 1, .. of new_table's rows, in their order, keys and values as they are; so do their weights, and
 * the rest of new_weights is 0.  kept says which slots they were (-1 behind them), new_lengths how many.
 * Heads keep different tokens: a cache cut so holds rotated keys, and slots are no positions any more (new tokens
 * are rotated at their positions, and stored and attended at their slots).
 * The new pages are written while the old ones are read: a page of new_table may not be one that a sequence of the call
 * holds, nor stand in it twice, and weights may not overlap new_weights.  A kept slot whose page is none is not moved.  Every other slot is left as it
 * is.  workspace: device memory of seer_kv_evict_workspace_bytes, 256-byte aligned, not shared with a call that may run at
 * the same time; its contents need no set-up.  NULL where that is 0.
 * SEER_ERR_UNSUPPORTED: as seer_kv_append, more than 65535 KV heads, 2^22 pairs of sequence and head and more.
 */
seer_status seer_kv_evict(const seer_kv_cache* cache, const seer_kv_eviction* desc, void* workspace, size_t workspace_bytes,
                          void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SEER_CACHE_H */
