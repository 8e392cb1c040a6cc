/*
 * ebrl_kv8.h -- a paged KV cache held in 8 bits, and the operators on it.
 *
 * Paper: the generation stage's memory share m (Section 4.3.1) bounds how
 * many environments' caches a GPU holds; half the bytes a token hold twice
 * the environments.  Same conventions as ebrl.h: device pointers,
 * stream-ordered calls, status codes; a call allocates nothing, synchronises
 * nothing and may be captured into a HIP graph.
 *
 * The cache.  A page holds EBRL_KV8_PAGE tokens.  A sequence is a row of the
 * block table: its token t lies in page table[row][t / 16], slot t % 16.
 * Page p has 16 * head_dim e4m3 codes for each of K and V and each KV head,
 * and one scale 2^e for each such group: a value is code * 2^e.  e is the
 * least integer >= -100 with |values| <= 448 * 2^e when a page's first token
 * is written, and grows only while the page keeps earlier tokens, also where a
 * token that needed it is written over.  Orders inside a group
 * (the ones in which the matrix instructions' lanes take them):
 *   K: byte 1024 (d / 64) + 64 t + d % 64,
 *   V: byte 1024 (d / 64) + 256 (t / 4) + 16 (d % 64 / 4) + 4 (d % 4) + t % 4
 * for token slot t and dim d.  A value that is not finite, or 2^127 and more,
 * is stored as the format's NaN.
 *
 * Device-side data that a call cannot check on the host never leads to an
 * access out of bounds: a row of the table outside [0, table_rows) is a
 * sequence of length 0; a page id outside [0, num_blocks) holds no tokens (none
 * are written there or seen; queries at its positions are still turned); a
 * sequence ends with the table's row (queries past it are left as well); row
 * ranges are cut to [0, rows] and to the host's max_* bounds (a sequence's
 * first max_* rows and keys are what counts, also for a causal mask);
 * positions are cut to the rotary tables.
 */
#ifndef EBRL_KV8_H
#define EBRL_KV8_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define EBRL_KV8_PAGE 16

typedef struct ebrl_kv8_cache {
    void* codes;                 /* device [num_blocks][2 (K, V)][kv_heads][16 * head_dim] bytes, 16-byte aligned */
    float* scales;               /* device [num_blocks][2][kv_heads] */
    const int32_t* block_table;  /* device [table_rows][table_stride] page ids */
    int32_t num_blocks, table_rows, table_stride;
    int32_t kv_heads, head_dim;  /* kv_heads 1 to 2^20, head_dim 64 or 128 */
} ebrl_kv8_cache;

typedef struct ebrl_kv8_write_args {
    int32_t dtype;               /* EBRL_DTYPE_*: type of q, q_out, k, v */
    int32_t n;                   /* sequences */
    int32_t rows;                /* rows of q, k, v */
    int32_t max_len;             /* most new tokens of a sequence */
    int32_t q_heads;             /* heads of q, at most 2^20; 0: no q */
    int32_t n_axes;              /* rotary axes, 1 to 3; 0: no rotation (then no q) */
    int32_t sections[3];         /* pairs of each axis, >= 1, sum head_dim / 2 */
    int32_t tab_rows;            /* rows of cos_tab, sin_tab */
    const void *q, *k, *v;       /* device rows: head h's dims at h * head_dim */
    void* q_out;                 /* rotated queries; may be q itself (with ldq_out = ldq) */
    int64_t ldq, ldk, ldv, ldq_out;   /* row strides in elements; 16-byte multiples */
    const int32_t* row_start;    /* device [n + 1]: sequence i's rows are row_start[i] .. row_start[i + 1] - 1 */
    const int32_t* pos0;         /* device [n]: cache position of the first of them */
    const int32_t* seq;          /* device [n] block-table rows, or NULL: row i */
    const int32_t* axis_pos;     /* device [rows][n_axes] positions, or NULL (one axis): the cache position */
    const float *cos_tab, *sin_tab;   /* device [tab_rows][head_dim / 2] */
} ebrl_kv8_write_args;

/* Rotary positions and the cache write of the rows a projection gives, one
 * pass over them.  Pair i of a head, elements (x_i, x_{i + head_dim / 2}),
 * turns by the angle whose cosine and sine stand in column i of the tables,
 * in the row given by the position on pair i's axis (axis a has the
 * sections[a] pairs after those of the axes before it).  Q and K turn, V does
 * not.  Each result is rounded once, from 64 bits.
 *
 * Tokens pos0[i] .. of each sequence are written; tokens before pos0[i] keep
 * their values.  The bytes of slots and pages behind the last token are left as
 * they were, but a slot behind it in the same page has no value from then on:
 * the page's scale is that of the tokens up to the last.  Rows of q_out outside
 * every sequence are left as they were.  A page that holds earlier tokens keeps
 * its scale unless a new token needs a larger one: the earlier tokens' codes
 * are then divided by the power of two that it grew by, which is exact down to
 * 2^-6 of the new scale and rounded below.  Writing smaller tokens in the place
 * of larger ones gives neither the scale nor those roundings back: who writes
 * the same slots again (a denoiser's steps) copies the page first.  Two
 * sequences of a call must not write the same page.  Returns EBRL_E_INVALID on
 * bad arguments. */
int ebrl_op_kv8_write(const ebrl_kv8_cache* cache, const ebrl_kv8_write_args* args, void* stream);

typedef struct ebrl_kv8_attn_args {
    int32_t dtype;               /* EBRL_DTYPE_*: type of q and out */
    int32_t n;                   /* sequences */
    int32_t rows;                /* rows of q and out */
    int32_t max_q_len;           /* most query rows of a sequence */
    int32_t max_kv_len;          /* most keys of a sequence, at most 2^30; a longer one counts as this long */
    int32_t q_heads;             /* a multiple of kv_heads, at most 2^20: query head h reads KV head h / (q_heads / kv_heads) */
    int32_t causal;              /* 0: every row sees all keys; else row j of m sees keys 0 .. kv_len - m + j */
    float scale;                 /* of the scores, > 0 (commonly 1 / sqrt(head_dim)) */
    const void* q;               /* device rows, as in ebrl_kv8_write_args */
    void* out;                   /* device rows; not q */
    int64_t ldq, ldo;            /* row strides in elements; 16-byte multiples */
    const int32_t* row_start;    /* device [n + 1] */
    const int32_t* kv_len;       /* device [n] keys of each sequence, the query rows' own among them */
    const int32_t* seq;          /* device [n] block-table rows, or NULL: row i */
    void* workspace;             /* device, 16-byte aligned; NULL where none is needed */
    int64_t workspace_bytes;
} ebrl_kv8_attn_args;

/* Bytes of workspace that a call with these arguments needs (host arithmetic
 * on n, max_q_len, max_kv_len, the heads and the dtype; no pointer is read),
 * or EBRL_E_INVALID.  0: none.  Fewer sequences or rows may need more, since
 * their keys are cut into more parts: a workspace for calls of several sizes
 * is the largest of what each of them needs. */
int64_t ebrl_op_kv8_attn_workspace(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args);

/* out = softmax(scale q K^T + mask) V over the cache: one query row a sequence
 * (a decode step), a prompt's rows, or any ragged mix.  Keys a row does not see
 * do not count, whatever their slots hold, NaN included; a row that sees no key
 * gets zeros; one whose query is not finite (fp32: past bf16's range, 3.39e38),
 * or whose scores pass the 32-bit range (the largest upwards, or all
 * downwards), is NaN; rows outside every sequence are left as they were.
 * Scores, the softmax's maximum and sum and the weighted sum are held in 32
 * bits; bf16 rows' weights enter the product with V as bf16, in two terms where
 * a KV head has at most 16 rows a sequence.  Weights go up to 2^11: the sum
 * overflows to infinity only where the keys' values, times 2^11 and their
 * number, pass the 32-bit range.  Scores, times log2(e), are floats: from 2^24
 * on they lie whole numbers apart.  With few rows the keys are cut into parts
 * that run at the same time and are joined in their order by a second launch.
 * The cut follows n, max_q_len, max_kv_len and the heads.
 *
 * The workspace holds the parts; what is in it before a call does not matter.
 * Calls that may overlap in time (other streams, graphs replayed side by side)
 * need a workspace each.  Returns EBRL_E_INVALID on bad arguments, too small a
 * workspace, or where the bounds ask for more than 2^23 workgroups (a tile of
 * 16 to 128 query rows of a KV head each). */
int ebrl_op_kv8_attn(const ebrl_kv8_cache* cache, const ebrl_kv8_attn_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBRL_KV8_H */
