/*
 * seer_decode.h -- C ABI of libseer.so, second part: what carries a prefilled
 * prompt on to generation.
 *
 *   seer_rope        rotary positions of Q and K, and their gradient.  The gate
 *                    takes Q and K before them, the attention after them
 *                    (SeerAttention section 3.1)
 *   seer_kv_append   keys and values of new tokens into a paged key-value cache,
 *                    the keys rotated on the way
 *   seer_paged_attn  attention of new tokens (one, or a few drafted ones, per
 *                    sequence) over that cache
 *
 * The conventions of seer.h hold: device pointers of the current device that
 * the caller owns, asynchronous on `stream`, validation on the host before
 * anything is launched, no state between calls, no allocation, reentrant, and
 * nothing that a HIP graph cannot capture.  Sizes that change from step to step
 * (positions, tables) are read on the device, so a captured step replays
 * with new ones.
 *
 * Rotary positions.  Plane p of rot_dim / 2 of a head at position t turns by the
 * angle t inv_freq[p]; its two elements are (p, p + rot_dim / 2), or (2p, 2p + 1)
 * when interleaved.  Elements from rot_dim on are left as they are:
 *   x' = scale (x cos a - y sin a),  y' = scale (x sin a + y cos a)
 * Angles are reduced to a turn in 64-bit fixed point before the sine: off by 2^-52 of
 * the angle and by 2^-64 of a turn per position at most (3.4e-19 radians; 7.3e-10 at position
 * 2^31), less than fp32's rounding up to 2^27 radians and 5e-7 at 2^31.  Cosine and sine are
 * within 8 steps of 2^-24 of their own size beside that, however slow the plane.
 *
 * Paged cache.  A pool of num_pages pages of page_size slots for each of K and V,
 * [page][head][slot][head_dim] with element strides given per (page, head,
 * slot), head_dim contiguous.  table[row][i] is the page that holds tokens
 * i page_size .. of the sequence of that row.  A table entry outside [0, num_pages)
 * is no page: nothing is written to it and no key is read from it.
 */
#ifndef SEER_DECODE_H
#define SEER_DECODE_H

#include "seer.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  const double* inv_freq; /* device [rot_dim / 2], finite: angle per position of each plane */
  int32_t rot_dim;        /* a multiple of 16, 16 to head_dim */
  int32_t interleaved;    /* 0: planes (p, p + rot_dim / 2); 1: planes (2p, 2p + 1) */
  float scale;            /* factor on the rotated elements (1, or a long-context method's), finite */
} seer_rope_params;

typedef struct {
  int32_t batch, heads_q, heads_kv; /* heads_kv 0: no K */
  int32_t seq_len, head_dim, dtype; /* head_dim 64 or 128; seer_dtype */
  int64_t q_stride[3], k_stride[3];         /* element strides of (batch, head, seq) */
  int64_t q_out_stride[3], k_out_stride[3]; /* multiples of 16 bytes, as all of them */
  int64_t pos_stride;                       /* elements between the positions of two batch entries */
} seer_rope_desc;

/*
 * Rotary positions of q and k into q_out and k_out (which may be q and k
 * themselves, with their strides; any other overlap is not allowed).  positions:
 * device [batch][seq], any int32; NULL: token s of every batch entry is at
 * position start + s (start is ignored otherwise).  grad != 0: the transpose
 * instead, which takes the gradient of the rotated tensors to that of the
 * unrotated ones.  Arithmetic in fp32, rounded once to dtype.
 * SEER_ERR_UNSUPPORTED: head_dim not 64 or 128, a rot_dim that is no multiple of
 * 16, strides that are no multiple of 16 bytes, more than 2^27 tokens or 65535 heads.
 */
seer_status seer_rope(const seer_rope_desc* desc, const seer_rope_params* rope, const void* q, const void* k,
                      void* q_out, void* k_out, const int32_t* positions, int32_t start, int32_t grad,
                      void* stream);

typedef struct {
  int32_t batch, tokens, heads_kv, head_dim, dtype;
  int32_t page_size, num_pages;      /* both >= 1 */
  int32_t table_rows, max_pages;     /* table: device [table_rows][max_pages], both >= 1 */
  int32_t reserved;                  /* 0 */
  int64_t k_stride[3], v_stride[3];  /* new tokens: (batch, head, token) */
  int64_t k_cache_stride[3], v_cache_stride[3]; /* (page, head, slot) */
  int64_t table_stride;              /* elements between two rows of the table */
  int64_t pos_stride;                /* elements between two batch entries of positions and rows */
} seer_append_desc;

/*
 * Token (b, s) of k and v ([batch][heads_kv][tokens][head_dim]) goes to position
 * positions[b][s] of the sequence of table row rows[b][s] (rows NULL: row b).
 * rope (NULL: none) rotates k at that position, computed in fp32 and rounded once.
 * A packed batch is batch 1 with a row for each token.  Tokens whose position or row is
 * negative or beyond the table, or whose page is none, are padding: not
 * written.  Every other slot of the cache is left as it is.  Two tokens of a call
 * may not go to the same slot (which of them stays is unspecified then), and k and v may not lie in
 * the pools.
 * SEER_ERR_UNSUPPORTED: as seer_rope, and a table whose rows have room for more than 2^30 tokens.
 */
seer_status seer_kv_append(const seer_append_desc* desc, const seer_rope_params* rope, const void* k, const void* v,
                           void* k_cache, void* v_cache, const int32_t* table, const int32_t* positions,
                           const int32_t* rows, void* stream);

typedef struct {
  int32_t batch, heads_q, heads_kv, tokens, head_dim, dtype; /* heads_q % heads_kv == 0 */
  int32_t page_size, num_pages;      /* both >= 1 */
  int32_t max_pages;                 /* table: device [batch][max_pages], >= 1 */
  int32_t reserved;                  /* 0 */
  int64_t q_stride[3], o_stride[3];  /* (batch, head, token) */
  int64_t k_cache_stride[3], v_cache_stride[3]; /* (page, head, slot) */
  int64_t table_stride;              /* elements between two rows of the table */
  int64_t pos_stride;                /* elements between the positions of two batch entries */
} seer_paged_desc;

/* Workspace bytes of seer_paged_attn for this shape (0 on invalid arguments):
 * two partial results for each workgroup of the launch, whatever the lengths,
 * and 8 bytes per (batch, KV head, 32 query rows). */
size_t seer_paged_attn_workspace_bytes(const seer_paged_desc* desc);

/*
 * Attention over the cache: the query of token (b, s) sees the keys at positions
 * t <= positions[b][s] of table row b whose page exists,
 *   o = softmax(sm_scale q K^T) V,
 * sm_scale at most 2^127, a value <= 0 selecting 1 / sqrt(head_dim).  Query head h reads KV head h / (heads_q /
 * heads_kv).  Positions beyond the table see every key it holds.  rope (NULL: none)
 * rotates q at its position first (in fp32, not rounded).  A row that sees no
 * key (position negative, or no page) yields o = 0 and lse = -inf.  lse: device float
 * [batch][heads_q][tokens], natural log, or NULL.  What unseen slots hold has no
 * effect on the results, be it NaN.  Statistics, weights and sums are fp32, o is rounded once.  Seen values
 * that are not finite make o of the rows that see them NaN or infinite, whatever their weights, and so do seen keys
 * the rows whose q is rotated here.
 *
 * The work, sequences of any lengths, is cut evenly over the workgroups: one sequence's keys
 * may be split over many of them, whose partial results a second launch joins.  Whether there is one goes by the room of a
 * table row, not by the lengths, which only the device knows: beyond 512 keys (fp32: 256), and beyond twice that with 128
 * to 512 KV heads in the batch (blocks of 32 query rows counted each).  It costs 2 to 4 us; a caller whose sequences are all
 * short avoids it by giving fewer max_pages with the same table_stride.
 * Results are the same bit for bit from run to run; they may differ by fp32 rounding
 * from those of the same sequence in another batch (the cuts lie elsewhere).
 * workspace: device memory of at least seer_paged_attn_workspace_bytes(desc) bytes, 256-byte
 * aligned, not shared with a call that may run at the same time.  Its contents need no set-up.
 * The cache is read once for each 32 query rows (heads_q / heads_kv x tokens), and the positions of a sequence one after
 * the other: made for one token or a few.  Any number up to the limits below gives right results, at a rate that falls
 * behind a matrix product's (32 / 8 heads of 128, bf16, after 16000 tokens: 512 tokens take 0.38 ms, 2048 2.4 ms, 3 to 5
 * times what their products need); a whole prompt goes through seer_bsattn or seer_dense_attn before its keys are
 * appended.  o may not overlap an input.
 * SEER_ERR_UNSUPPORTED: head_dim not 64 or 128, a rot_dim that is no multiple of 16, strides that are no multiple of 16
 * bytes, a table whose rows have room for more than 2^30 tokens, page or slot strides of 64 GB and more, more than 2^23
 * query rows a KV head (heads_q / heads_kv x tokens) or 2^23 blocks of 16 of them (the sum over batch and heads_kv, each
 * rounded up).
 */
seer_status seer_paged_attn(const seer_paged_desc* desc, const seer_rope_params* rope, float sm_scale, const void* q,
                            const void* k_cache, const void* v_cache, const int32_t* table,
                            const int32_t* positions, void* o, float* lse, void* workspace, size_t workspace_bytes,
                            void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SEER_DECODE_H */
