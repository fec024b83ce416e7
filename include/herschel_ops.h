/*
 * herschel_ops.h -- C ABI of the reference operators: the attention layer of a
 * served model, from the rows of the QKV product to the attention's output.
 *
 * The trace analyzer (herschel.h) rates an op by SOL = max(MFU, MBU) and sums
 * what its name would save at a reference SOL, "the SOL the same op reaches
 * elsewhere".  These operators are such a reference on MI355X for the op that
 * the paper's case study is about, attention over a paged cache (Section 9.4),
 * and for those around it: run them at the traced shapes, rate them with
 * HERSCHEL_OUT_SOL, and give the result as ref_sol_ppm.
 *
 *  - herschel_rope_write: rotary positions, and the write of keys and values
 *    into a paged cache, quantised on the way (one launch);
 *  - herschel_cache_read: rows of the cache back in 16 bits;
 *  - herschel_attn_prompt: attention over packed prompts;
 *  - herschel_attn_decode: attention of one or a few new tokens over the cache.
 *
 * Conventions, those of herschel.h where they apply: every array is a DEVICE
 * pointer, the caller owns every buffer, return codes are HERSCHEL_*.  Unlike
 * the analyzer, a call only enqueues: it runs on args->hip_stream (a stream of
 * the current device), waits for nothing, allocates nothing, copies nothing
 * to the host, and can be captured into a graph.  What only the device can
 * see to be wrong (a page id, a length, a position or a slot out of range)
 * touches no memory out of range; it sets a bit in *args->status (may be
 * NULL; cleared by the caller alone) and has the effect stated there.
 *
 * Numbers: inputs and outputs are bfloat16 or IEEE half; products are summed,
 * and maxima, sums and scales held, in 32 bits.  The attention operators round a
 * weight (over an 8-bit cache, the weight times its value's scale) before it
 * meets its value: prompts to the rows' type; decode to two parts of 16 bits, or
 * to one where more than 16 rows share a key head and are not half rows over an
 * 8-bit cache.  A weight too small for 32 bits counts
 * as not 0 where its value is an infinity.
 */
#ifndef HERSCHEL_OPS_H
#define HERSCHEL_OPS_H

#include "herschel.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  FP8 (4 exponent bits, 3 fraction bits, largest value 448) and
 * INT8 are cache codes only. */
enum { HERSCHEL_BF16 = 0, HERSCHEL_F16 = 1, HERSCHEL_FP8 = 2, HERSCHEL_INT8 = 3 };

/* Rotary layouts: element i is paired with i + rotary_dim / 2, or 2 i with 2 i + 1. */
enum { HERSCHEL_ROPE_HALF = 0, HERSCHEL_ROPE_INTERLEAVED = 1 };

/* Bits of *status. */
enum {
  HERSCHEL_OP_BAD_PAGE = 1,     /* a block table entry outside [0, n_pages): its keys are not seen, its rows read as 0 */
  HERSCHEL_OP_BAD_LENGTH = 2,   /* lengths that fall, are negative or exceed the buffers: taken as the nearest valid */
  HERSCHEL_OP_BAD_POSITION = 4, /* a position outside the table: the token's rotated rows are NaN, nothing is cached */
  HERSCHEL_OP_BAD_SLOT = 8      /* a slot at or beyond the cache's end: the token is not cached */
};

/* A paged cache of keys and values: page p holds, for each head, page_size
 * consecutive tokens.  Token t of a sequence is row t % page_size of the page
 * that entry t / page_size of the sequence's block table row names.
 * With 8-bit codes each row has a scale: value = code * scale, where, for the
 * row's largest magnitude a and M = 448 (FP8) or 127 (INT8),
 *   scale = max(a * (1 / M), 2^-100), code = round to nearest even(x * (1 / scale)), at most M;
 * a row that holds an infinity or a NaN has scale NaN and codes 0. */
typedef struct {
  void *k, *v;               /* [n_pages][n_heads][page_size][head_dim], 16-byte aligned */
  float *k_scale, *v_scale;  /* [n_pages][n_heads][page_size], 16-byte aligned; NULL unless kind is FP8 or INT8 */
  int64_t n_pages;           /* >= 1 */
  int32_t n_heads;           /* >= 1 */
  int32_t page_size;         /* 16, 32, 64, 128 or 256 */
  int32_t head_dim;          /* even, at most 256 (attention: 64 or 128) */
  int32_t kind;              /* HERSCHEL_BF16 ... HERSCHEL_INT8 */
} herschel_cache;

/* Rows of heads: element d of head h of row t is at base + t * row + h * head + d. */
typedef struct {
  int64_t row, head;         /* in elements, >= 0; elements of a head are contiguous */
} herschel_strides;

typedef struct {
  /* Inputs [n_tokens][heads][head_dim].  q may be NULL (keys and values only); k and v may both be NULL. */
  const void *q, *k, *v;
  herschel_strides q_strides, k_strides, v_strides;
  /* Rotated rows; q_out and k_out may each be NULL (not written), or equal q, k with equal strides. */
  void *q_out, *k_out;
  herschel_strides q_out_strides, k_out_strides;
  const int64_t *positions;  /* [n_tokens], each in [0, n_positions) */
  const float *table;        /* [n_positions][rotary_dim / 2][2]: cos and sin of each angle, with any scaling for long
                                contexts already in it; 8-byte aligned */
  int64_t n_positions;
  const int64_t *slots;      /* [n_tokens]: page * page_size + row in the page, negative for a token that is not
                                cached; with a cache only.  No two tokens share a slot. */
  int64_t n_tokens;          /* >= 0; 0: nothing is done, and the rows', positions' and slots' addresses may be NULL */
  int32_t q_heads, kv_heads, head_dim; /* kv_heads and head_dim equal the cache's */
  int32_t rotary_dim;        /* even, 0 <= rotary_dim <= head_dim: the rest of a head passes unchanged */
  int32_t layout;            /* HERSCHEL_ROPE_* */
  int32_t type;              /* HERSCHEL_BF16 or HERSCHEL_F16; a cache that is not quantised has the same */
  uint32_t *status;
  void *hip_stream;
} herschel_rope_args;

/* For each token and head, with (c, s) = table[position][i] and the pair (a, b) of index i:
 * a' = a c - b s, b' = b c + a s, in 32 bits, each product and sum rounded.
 * q_out, k_out: rounded to the type.  With a cache, the keys' rotated rows and
 * the values' rows go to slots[token] of every head (quantised from the 32-bit
 * values).  cache may be NULL: v is not read. */
int herschel_rope_write(const herschel_rope_args *args, const herschel_cache *cache);

typedef struct {
  const int32_t *block_table; /* [n_seqs][table_stride] */
  int64_t table_stride;       /* entries a sequence has room for */
  const int32_t *cu;          /* [n_seqs + 1]: sequence b's rows are cu[b] ... cu[b + 1] - 1 of the output; cu[0] = 0 */
  int32_t n_seqs;
  int64_t n_rows;             /* rows of the outputs, cu[n_seqs]; rows beyond that read as 0 */
  void *k_out, *v_out;        /* [n_rows][n_heads][head_dim] contiguous, 16-byte aligned; each may be NULL */
  int32_t type;               /* HERSCHEL_BF16 or HERSCHEL_F16; that of a cache that is not quantised */
  uint32_t *status;
  void *hip_stream;
} herschel_read_args;

/* Tokens 0 ... cu[b + 1] - cu[b] - 1 of every sequence as dense rows, rounded once.
 * head_dim must be a multiple of 16. */
int herschel_cache_read(const herschel_read_args *args, const herschel_cache *cache);

typedef struct {
  const void *q, *k, *v;      /* [n_q][q_heads][head_dim], [n_k][kv_heads][head_dim] */
  herschel_strides q_strides, k_strides, v_strides;
  void *out;                  /* [n_q][q_heads][head_dim] contiguous, 8-byte aligned */
  float *lse;                 /* [n_q][q_heads] or NULL: log of the sum of exp(scale q.k) over the keys seen */
  const int32_t *cu_q, *cu_k; /* [n_seqs + 1]: first query and first key row of each sequence; cu[0] = 0.  Rows of q
                                 from cu_q[n_seqs] on are padding: out is 0 there, lse -infinity */
  int32_t n_seqs;
  int64_t n_q, n_k;           /* rows of q and of k and v */
  int32_t max_q;              /* queries of the longest sequence: those beyond are not computed, out is 0 there */
  int32_t q_heads, kv_heads;  /* q_heads a multiple of kv_heads */
  int32_t head_dim;           /* 64 or 128 */
  int32_t type;               /* HERSCHEL_BF16 or HERSCHEL_F16 */
  int32_t causal;             /* query i of nq sees key j of nk iff j <= i + nk - nq */
  int32_t window;             /* > 0: and j > i + nk - nq - window; 0: no window */
  float scale;                /* of the scores; finite */
  void *workspace;            /* herschel_attn_prompt_workspace() bytes, 16-byte aligned, no two calls at once; or */
  size_t workspace_bytes;     /* NULL or fewer bytes: long keys are then not shared among more workgroups */
  uint32_t *status;
  void *hip_stream;
} herschel_prompt_args;

/* Bytes of workspace with which a call of these sizes is fastest; 0 for most. */
int herschel_attn_prompt_workspace(int32_t n_seqs, int64_t n_q, int64_t n_k, int32_t max_q, int32_t q_heads,
                                   int32_t kv_heads, int32_t head_dim, size_t *bytes);

/* out = softmax over the keys seen of (scale q.k) times v.  A query that sees
 * no key has out 0 and lse -infinity.  Keys not seen have no effect, whatever
 * they hold. */
int herschel_attn_prompt(const herschel_prompt_args *args);

typedef struct {
  const void *q;              /* [n_seqs][new_tokens][q_heads][head_dim] */
  int64_t q_seq_stride;       /* elements from one sequence to the next */
  herschel_strides q_strides; /* row: from one new token to the next */
  void *out;                  /* [n_seqs][new_tokens][q_heads][head_dim] contiguous, 16-byte aligned */
  float *lse;                 /* [n_seqs][new_tokens][q_heads] or NULL */
  const int32_t *block_table; /* [n_seqs][table_stride] */
  int64_t table_stride;
  const int32_t *seq_lens;    /* [n_seqs]: cached tokens, the new ones among them (0: out is 0) */
  int32_t n_seqs;             /* 1 ... HERSCHEL_MAX_DECODE_SEQS */
  int32_t new_tokens;         /* query i of a sequence is its token seq_len - new_tokens + i */
  int32_t q_heads;            /* a multiple of the cache's n_heads */
  int32_t type;               /* HERSCHEL_BF16 or HERSCHEL_F16; that of a cache that is not quantised */
  int32_t window;             /* as for herschel_attn_prompt */
  float scale;
  void *workspace;            /* herschel_attn_decode_workspace() bytes, 256-byte aligned; no two calls at once */
  size_t workspace_bytes;
  uint32_t *status;
  void *hip_stream;
} herschel_decode_args;

#define HERSCHEL_MAX_DECODE_SEQS 4096

/* Bytes of workspace for calls of at most these sizes. */
int herschel_attn_decode_workspace(int32_t n_seqs, int32_t new_tokens, int32_t q_heads,
                                   const herschel_cache *cache, size_t *bytes);

/* Causal attention of each sequence's last new_tokens tokens over its cached
 * tokens.  Keys not seen have no effect, whatever the pages hold. */
int herschel_attn_decode(const herschel_decode_args *args, const herschel_cache *cache);

#ifdef __cplusplus
}
#endif

#endif /* HERSCHEL_OPS_H */
