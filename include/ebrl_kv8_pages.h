/*
 * ebrl_kv8_pages.h -- the pages of an 8-bit KV cache (ebrl_kv8.h): shared by
 * sequences that start alike, copied when one of them writes, freed, compacted.
 *
 * Paper: environments of a group start from one observation (the groups of
 * Section 4.2.2), and the memory share m of Section 4.3.1 bounds the pages; a
 * prefix held once serves every action sequence sampled after it.  Same
 * conventions as ebrl_kv8.h: device pointers, stream-ordered calls, status
 * codes; a call allocates nothing, synchronises nothing and may be captured into
 * a HIP graph.
 *
 * A pool is the caches of `layers` layers that share one block table, and refs:
 * refs[p] is the number of table entries that hold page p.  A page of refs 0 is
 * free.  Entries outside [0, num_blocks) hold no page; these calls write -1.  A
 * pool starts with a table of -1 and refs of 0.  The calls keep refs right; a
 * caller that edits the table itself keeps them right too (a page of negative
 * refs counts as free).
 *
 * Calls on one pool follow one another on a stream, or are ordered by the caller:
 * each reads what the one before it has written.
 *
 * All choices are fixed by the arguments: page ids do not depend on timing.
 * Numbers on the device that a call cannot check on the host never lead to an
 * access out of bounds: rows of the table outside [0, table_rows) are left out,
 * token numbers are cut to 0 and to what a table row holds.
 */
#ifndef EBRL_KV8_PAGES_H
#define EBRL_KV8_PAGES_H

#include <stdint.h>

#include "ebrl_kv8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ebrl_kv8_pool {
    void* codes;             /* device: layer l's codes (ebrl_kv8_cache) at codes + l * layer_codes */
    float* scales;           /* device: layer l's scales at scales + l * layer_scales */
    int32_t* block_table;    /* device [table_rows][table_stride] */
    int32_t* refs;           /* device [num_blocks] */
    int64_t layer_codes;     /* bytes, a multiple of 16; any value with one layer */
    int64_t layer_scales;    /* floats */
    int32_t layers;          /* 1 to 65535 */
    int32_t num_blocks;      /* 1 to 2^30 */
    int32_t table_rows, table_stride;   /* from 1 on; table_stride below 2^27 */
    int32_t kv_heads, head_dim;         /* kv_heads 1 to 2^17, head_dim 64 or 128 */
} ebrl_kv8_pool;

/* Row dst[i] takes the pages of row src[i]'s first len[i] tokens, the last of them
 * also where it is partly filled; its other entries become -1.  Pages that dst[i]
 * held before are released (no call of ebrl_op_kv8_free is needed first).  src, dst,
 * len: device int32 [n].  A fork whose source is a destination of the call is left
 * out, and of several forks to one row all but the first.  Codes and scales are not
 * touched (codes, scales and their strides may be 0).  n: at most 65536, here and
 * below.  Returns EBRL_E_INVALID on bad arguments. */
int ebrl_op_kv8_fork(const ebrl_kv8_pool* pool, const int32_t* src, const int32_t* dst, const int32_t* len, int32_t n,
                     void* stream);

/* Row seq[i] keeps the pages of its first keep[i] tokens and releases the others:
 * their entries become -1 and their refs one less.  seq, keep: device int32 [n];
 * keep NULL: nothing is kept.  A row named twice keeps the smaller number.  Codes
 * and scales are not touched (and may be 0, as above).  Returns EBRL_E_INVALID on
 * bad arguments. */
int ebrl_op_kv8_free(const ebrl_kv8_pool* pool, const int32_t* seq, const int32_t* keep, int32_t n, void* stream);

/* Bytes of workspace for ebrl_op_kv8_reserve calls of at most n rows and max_count
 * tokens each (host arithmetic on the pool's numbers; no pointer is read), or
 * EBRL_E_INVALID: for numbers out of range, n rows whose max_count tokens lie in more
 * than 2^30 pages, or n pages of more than 2^23 pieces of 16 KB, counted once for
 * each eight layers.  A call of a size that gets a workspace is not refused for its
 * size. */
int64_t ebrl_op_kv8_reserve_workspace(const ebrl_kv8_pool* pool, int32_t n, int32_t max_count);

/* Makes ready the pages that tokens pos0[i] .. pos0[i] + count[i] - 1 of row seq[i]
 * will be written to.  In the order of i and then of the tokens, each of their
 * entries that holds no page, or one that other entries hold too (refs above 1
 * before the call), gets a page of its own: the k-th that needs one gets the k-th
 * lowest free id.  A shared page is released for it, and if it holds tokens before
 * pos0[i], its codes and scales are copied in every layer.  A pos0[i] below 0 counts
 * as 0, and count[i] is cut to max_count and to the table's row; of several i for one
 * row all but the first are left out.  Pages that this call releases are free from
 * the next one on.
 *
 * *lacking (device int32): 0, or how many pages were missing: then the call has
 * changed nothing, and a write that follows without a look at it writes nothing
 * where there is no page, but into shared pages where there is one.  seq, pos0,
 * count: device int32 [n].  Calls that may overlap in time need a workspace each;
 * what is in it before a call does not matter.  Returns EBRL_E_INVALID on bad
 * arguments or too small a workspace. */
int ebrl_op_kv8_reserve(const ebrl_kv8_pool* pool, const int32_t* seq, const int32_t* pos0, const int32_t* count,
                        int32_t n, int32_t max_count, int32_t* lacking, void* workspace, int64_t workspace_bytes,
                        void* stream);

/* Bytes of workspace for ebrl_op_kv8_compact (host arithmetic on the pool's
 * numbers), or EBRL_E_INVALID: for numbers out of range, or layers of more than 2^31
 * pieces of 16 KB. */
int64_t ebrl_op_kv8_compact_workspace(const ebrl_kv8_pool* pool);

/* Moves the used pages to ids 0 .. *used - 1: of the pages in use from id *used on
 * (refs above 0) the k-th lowest goes to the k-th lowest free id, in every layer.
 * new_table and new_refs get the table and refs that go with it; each may be the
 * pool's own.  What a moved page held stays readable in its old place until that is
 * written again, so a reader of the old table may still finish.  *used, device
 * int32: the number of used pages.  Returns EBRL_E_INVALID on bad arguments or too
 * small a workspace. */
int ebrl_op_kv8_compact(const ebrl_kv8_pool* pool, int32_t* new_table, int32_t* new_refs, int32_t* used,
                        void* workspace, int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EBRL_KV8_PAGES_H */
