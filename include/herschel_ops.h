/*
 * herschel_ops.h -- C ABI of the reference operators: the attention layer of a
 * served model, from the rows of the QKV product to the attention's output, and
 * what a decoder layer has around it.
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
 *  - herschel_attn_decode: attention of one or a few new tokens over the cache;
 *  - herschel_norm_rows: root-mean-square norm with the residual's addition, to
 *    16 bits or to 8 with scales;
 *  - herschel_product4: rows, of 16 or 8 bits, times 4-bit weights with a scale
 *    for each group of a weight row;
 *  - herschel_verify_drafts: drafted tokens against the target's probabilities.
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
 * INT8 are codes, of caches and of rows; F32 is for what stays in 32 bits where
 * an operator says so. */
enum { HERSCHEL_BF16 = 0, HERSCHEL_F16 = 1, HERSCHEL_FP8 = 2, HERSCHEL_INT8 = 3, HERSCHEL_F32 = 4 };

/* Rotary layouts: element i is paired with i + rotary_dim / 2, or 2 i with 2 i + 1. */
enum { HERSCHEL_ROPE_HALF = 0, HERSCHEL_ROPE_INTERLEAVED = 1 };

/* Bits of *status. */
enum {
  HERSCHEL_OP_BAD_PAGE = 1,     /* a block table entry outside [0, n_pages): its keys are not seen, its rows read as 0 */
  HERSCHEL_OP_BAD_LENGTH = 2,   /* lengths that fall, are negative or exceed the buffers: taken as the nearest valid */
  HERSCHEL_OP_BAD_POSITION = 4, /* a position outside the table: the token's rotated rows are NaN, nothing is cached */
  HERSCHEL_OP_BAD_SLOT = 8,     /* a slot at or beyond the cache's end: the token is not cached */
  HERSCHEL_OP_BAD_TOKEN = 16,   /* a drafted token outside the vocabulary: not accepted */
  HERSCHEL_OP_BAD_ROW = 32      /* a row of probabilities without one above 0: the token drawn from it is -1 */
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

typedef struct {
  const void *x;              /* [n_rows][dim] of type */
  int64_t x_row;              /* elements from one row to the next, >= 0 */
  const void *residual;       /* [n_rows][dim] of residual_type, or NULL */
  int64_t residual_row;
  void *residual_out;         /* [n_rows][dim] of residual_type, or NULL; may be residual with the same stride */
  int64_t residual_out_row;   /* >= dim */
  const void *weight;         /* [dim] of weight_type */
  void *out;                  /* [n_rows][dim] of out_kind, contiguous; of the rows' type it may be a contiguous x */
  float *scale;               /* 8 bits: [n_rows][dim / group], or [n_rows] with group 0 */
  int64_t n_rows;             /* >= 0; 0: nothing is done */
  int32_t dim;                /* 1 ... HERSCHEL_MAX_NORM_DIM */
  int32_t group;              /* 8 bits: columns that share a scale, 32, 64 or 128 and a divisor of dim; 0: a row's */
  int32_t type;               /* HERSCHEL_BF16 or HERSCHEL_F16 */
  int32_t residual_type;      /* type or HERSCHEL_F32 */
  int32_t weight_type;        /* type or HERSCHEL_F32 */
  int32_t out_kind;           /* type, HERSCHEL_FP8 or HERSCHEL_INT8 */
  float eps;                  /* finite, >= 0 */
  void *hip_stream;
} herschel_norm_args;

#define HERSCHEL_MAX_NORM_DIM 32768

/* For each row, in 32 bits: h = x + residual, residual_out = h rounded to its
 * type, y = h / sqrt(mean(h^2) + eps) * weight, from the h that is not rounded.
 * Squares of rows whose sum would leave 32 bits are summed scaled by a power of
 * two.  out = y rounded, or codes with the scale of the row or of each group of
 * columns, by the rule of a cache row.  residual_out may be residual or x, and a
 * 16-bit out x, with the same rows; else what is written shares no memory with
 * anything (rows of one tensor may lie between those of another), or the call is
 * refused. */
int herschel_norm_rows(const herschel_norm_args *args);

/* A matrix [n][k] of 4-bit codes c, each worth (c - zero) * scale with the zero
 * and scale of its row's group of `group` columns.  Rows are held in tiles of 16,
 * columns in tiles of 128, both filled up with codes, scales and zeros of 0.  A
 * scale is a 32-bit float of at most 16 significant bits: a word holds its upper
 * 24 bits, and in its low 8 the zero, 0 ... 15 (8 where the weights have none).  Of
 * column k in its tile, g = k / group, f = k % group, r = group / 4:
 *   codes[tile][n / 16][f / r][n % 16][g * r / 8 + f % r / 8][k % 4], bytes, the
 *     column in the low half of its byte if k % 8 < 4, else in the high half;
 *   scales[tile][n / 16][n % 16 / 4][g][n % 4], words. */
typedef struct {
  const void *codes;          /* 16-byte aligned */
  const uint32_t *scales;     /* 16-byte aligned */
  int32_t n, k;               /* 1 ... HERSCHEL_MAX_WEIGHT_ROWS, 1 ... 2^30 */
  int32_t group;              /* 32, 64 or 128; the last of a row may be shorter */
} herschel_weights4;

#define HERSCHEL_MAX_WEIGHT_ROWS 715827840

typedef struct {
  const void *x;              /* [n_rows][k] of kind */
  int64_t x_row;              /* elements from one row to the next, >= 0 */
  const float *x_scale;       /* 8 bits: [n_rows][ceil(k / group)] with x_group, else [n_rows] */
  void *out;                  /* [n_rows][n], gated [n_rows][n / 2], of type, contiguous */
  int64_t n_rows;             /* 0 ... HERSCHEL_MAX_PRODUCT_ROWS; 0: nothing is done */
  int32_t kind;               /* HERSCHEL_BF16 ... HERSCHEL_INT8 */
  int32_t x_group;            /* 8 bits: 0 or the weights' group */
  int32_t type;               /* HERSCHEL_BF16 or HERSCHEL_F16; that of rows of 16 bits */
  int32_t gated;              /* n a multiple of 32: y = silu(a) b, a the first n / 2 columns of the product, b the others */
  void *workspace;            /* herschel_product4_workspace() bytes, 16-byte aligned, no two calls at once; or NULL or */
  size_t workspace_bytes;     /* fewer bytes: a product's columns are then not shared among more workgroups */
  void *hip_stream;
} herschel_product_args;

#define HERSCHEL_MAX_PRODUCT_ROWS 4194240

/* Bytes of workspace with which a call of these sizes is fastest; 0 for most. */
int herschel_product4_workspace(int64_t n_rows, int32_t kind, int32_t gated, int32_t n, int32_t k, size_t *bytes);

/* out[m] = sum over k of x[m][k] * weight[n][k], codes summed within a group
 * before they meet its scale, in 32 bits (int8 rows: whole numbers), rounded
 * once.  A row that holds an infinity or a NaN comes out as NaN.  out shares no
 * memory with x, x_scale or the weights (it may lie between rows of x), or the call
 * is refused. */
int herschel_product4(const herschel_product_args *args, const herschel_weights4 *weights);

typedef struct {
  const void *target;         /* [n_seqs][n_drafts + 1][vocab] of type: the target's probabilities at each draft and
                                 behind the last */
  int64_t target_seq, target_row; /* elements from one sequence, and one row, to the next, >= 0 */
  const void *draft;          /* [n_seqs][n_drafts][vocab] of type: those that the drafts were drawn from; or NULL: each
                                 draft had probability 1 */
  int64_t draft_seq, draft_row;
  const int64_t *tokens;      /* [n_seqs][n_drafts]: the drafted tokens */
  const int32_t *counts;      /* [n_seqs]: drafts of each sequence, 0 ... n_drafts; NULL: n_drafts */
  const float *accept_u;      /* [n_seqs][n_drafts]: a random number in [0, 1) for each draft */
  const float *final_u;       /* [n_seqs]: and one for the token behind the accepted ones */
  int64_t *out;               /* [n_seqs][n_drafts + 1]: the accepted drafts, the token drawn, -1 */
  int32_t *accepted;          /* [n_seqs] */
  int32_t n_seqs;             /* 0 ... 65535; 0: nothing is done */
  int32_t n_drafts;           /* 0 ... HERSCHEL_MAX_DRAFTS */
  int32_t vocab;              /* 1 ... 2^30 */
  int32_t type;               /* HERSCHEL_F32, HERSCHEL_BF16 or HERSCHEL_F16 */
  void *workspace;            /* herschel_verify_workspace() bytes, 16-byte aligned, or NULL with 0; no two calls at once */
  size_t workspace_bytes;
  uint32_t *status;
  void *hip_stream;
} herschel_verify_args;

#define HERSCHEL_MAX_DRAFTS 1024

/* Bytes of workspace for a call of these sizes; 0 for small vocabularies. */
int herschel_verify_workspace(int32_t n_seqs, int32_t vocab, size_t *bytes);

/* Draft t of a sequence, token x, is accepted iff those before it are and
 * accept_u[t] * draft[t][x] < target[t][x].  Behind the accepted ones one token is
 * drawn: from target - draft, where that is above 0, of the first draft that is
 * not accepted; behind the last draft from the target.  Where nothing is above 0,
 * from the target alone.  The token drawn is the lowest whose cumulative sum is
 * above final_u times the sum of all (with a final_u not below 1, the last whose
 * part is above 0).  Products, differences and sums are in 64 bits; what is not
 * above 0, a NaN among it, counts as 0.  A count out of range is taken as the
 * nearest valid one (HERSCHEL_OP_BAD_LENGTH).  What is written shares no memory with
 * anything (it may lie between rows of probabilities), or the call is refused. */
int herschel_verify_drafts(const herschel_verify_args *args);

#ifdef __cplusplus
}
#endif

#endif /* HERSCHEL_OPS_H */
