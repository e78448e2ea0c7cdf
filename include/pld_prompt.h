/*
 * pld_prompt.h -- C ABI of a prompt's pass and of the pages that it fills, on
 * AMD Instinct MI355X (gfx950): prompts of different lengths read together, and
 * what the paged caches of pld_model.h need before and after.  The conventions
 * of pld.h (device pointers, streams, status codes, no allocation, no
 * synchronisation, deterministic results) and struct pld_cache of pld_model.h
 * hold here as well.
 *
 * Packed rows.  The rows of B sequences follow each other in buffers of N rows:
 * starts is int32 [B+1] on the device, non-decreasing with 0 <= starts[0] and
 * starts[B] <= N, and row r belongs to sequence b where starts[b] <= r <
 * starts[b+1]; sequences may be empty.  Rows before starts[0] and from starts[B]
 * on belong to none: they change no result and are not written, but like all N rows
 * (and their positions) they have to be memory that can be read.  (Starts that break
 * the rule give unspecified rows, and no access outside the buffers.)
 *
 * A prompt's layer: pld_cache_write_packed finishes queries and keys and puts
 * keys and values into the layer's cache, pld_prompt_attn attends, straight from
 * the packed rows.  The verification passes that follow (arXiv 2412.01447, Sec. 3)
 * read the cache by the calls of pld_model.h; where their positions are not the
 * cache's, as behind images, their rows join it by pld_cache_write_packed too.
 *
 * The pages of a pool are shared by sequences that go on from the same prompt:
 * pld_pages_take, pld_pages_fork, pld_pages_free, pld_pages_compact and
 * pld_pages_copy.
 */
#ifndef PLD_PROMPT_H
#define PLD_PROMPT_H

#include "pld_model.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Version of this header's ABI (major * 10000 + minor * 100 + patch). */
#define PLD_PROMPT_ABI_VERSION 100
int pld_prompt_version(void);

#define PLD_MAX_PACKED_ROWS 16777216   /* N: rows of a packed buffer */
#define PLD_MAX_AXES 4                 /* axes of a position */
#define PLD_MAX_LAYERS 64              /* caches of one page call */
#define PLD_MAX_PAGES 16777216         /* pages of a pool */
#define PLD_MAX_PAGE_ENTRIES 4096      /* sequences or forks of one page call */

/*
 * pld_cache_write_packed -- pld_cache_write for packed rows, with positions on
 * several axes.  Row r of sequence b goes to position first[b] + r - starts[b]
 * of the sequence's cache (its slot).  Pair t of the first rot_dim elements of a
 * query or key is turned by the row's position on axis pair_axis[t]: with
 * p = positions[pair_axis[t]*axis_stride + r], by cos = rope[p*rope_stride + t]
 * and sin = rope[p*rope_stride + rot_dim/2 + t].  So the axes (time, height and
 * width of an image's patches, say) may have sections of pairs or take turns.
 * Norm, rotation, storing and rounding are pld_cache_write's.
 *
 *   q, k, v     bf16 [N][heads][head_dim], rows row_stride apart, heads follow
 *               each other; 16-byte aligned, strides multiples of 8 elements
 *   rope, rope_stride, n_pos, rot_dim, rope_pairs   as pld_cache_write
 *   positions   int32, axis a's row r at a*axis_stride + r; NULL: the cache's
 *               position on every axis (axes and pair_axis are not used)
 *   axes        1 .. PLD_MAX_AXES;  axis_stride >= N
 *   pair_axis   int32 [rot_dim/2], 16-byte aligned, values in [0, axes-1] (others count as 0);
 *               NULL: axis 0
 *   starts, first   int32 [B+1] and [B];  B 1 .. 65535
 *   q_out       bf16 [N][Hq][head_dim]; may be q itself with q's stride
 *   k_out       bf16 [N][heads][head_dim], the finished keys as pld_prompt_attn
 *               takes them; may be k itself with k's stride; or NULL.  Outputs overlap nothing
 *               else
 * Device-side rule: a row whose position in the cache is negative or past the table
 * of pages, whose page is bad, or one of whose pairs' positions is outside [0, n_pos)
 * (with rope), is not stored, and its q_out and k_out are NaN.  Two rows of one call
 * must not have the same slot.
 * Errors: PLD_ERR_INVALID, PLD_ERR_ALIGN, PLD_ERR_LAUNCH.
 */
int pld_cache_write_packed(const pld_cache *cache, const uint16_t *q, int64_t q_row_stride,
                           const uint16_t *k, int64_t k_row_stride, const uint16_t *v,
                           int64_t v_row_stride, const uint16_t *q_norm, const uint16_t *k_norm,
                           float eps, const float *rope, int64_t rope_stride, int n_pos,
                           int rot_dim, int rope_pairs, const int32_t *positions, int axes,
                           int64_t axis_stride, const int32_t *pair_axis, const int32_t *starts,
                           const int32_t *first, int B, int N, int Hq, uint16_t *q_out,
                           int64_t o_row_stride, uint16_t *k_out, int64_t ko_row_stride,
                           void *stream);

/*
 * pld_prompt_attn -- causal attention of packed sequences to themselves.  Row r of
 * sequence b sees the keys starts[b] <= j <= r, of those r - window < j when
 * window > 0.  With the key head h / (Hq / heads) of query head h:
 *   s_j = (q . k_j) * scale;  softcap > 0: s_j = softcap * tanh(s_j / softcap)
 *   out = sum_j exp(s_j - lse) v_j,   lse = log sum_j exp(s_j)
 *
 *   q, k, v     bf16 [N][Hq or heads][head_dim], rows row_stride apart (at most
 *               2^22 elements), heads follow each other; 16-byte aligned, strides
 *               multiples of 8 elements
 *   heads       1 .. 1024;  Hq a multiple of it, up to 4096;  head_dim 64, 128 or 256
 *   scale, softcap, window   as pld_cache_attn
 *   out         bf16 [N][Hq][head_dim]; may be q itself with q's stride, not k or v
 *   lse         fp32 [N][Hq] or NULL
 * Device-side rules: rows that a row does not see do not affect it, whatever they
 * hold; a row's bits are the same from run to run.  Where a query, or a key or value that a row sees, is not finite, that head of
 * its out, and its lse, may be NaN as a whole.  The ranges of values and scores are
 * pld_cache_attn's: values up to 2^89, and a score above -1e29 for every row.  (A
 * block of rows that meets what is not finite is computed twice.)  out is summed in fp32,
 * 16 keys at a time: up to 2^22 keys of a row the roundings stay below that to bf16; of more,
 * whose weights and values are alike, out may be off by more (2% at 2^24), lse not.
 * Errors: PLD_ERR_INVALID, PLD_ERR_ALIGN, PLD_ERR_LAUNCH.
 */
int pld_prompt_attn(const uint16_t *q, int64_t q_row_stride, const uint16_t *k,
                    int64_t k_row_stride, const uint16_t *v, int64_t v_row_stride,
                    const int32_t *starts, int B, int N, int Hq, int heads, int head_dim,
                    float scale, float softcap, int window, uint16_t *out, int64_t o_row_stride,
                    float *lse, void *stream);

/*
 * A pool of pages: the table that names each sequence's pages, and for each page
 * how many entries of the table name it.  The struct is host memory, read during a
 * call and not kept; the memory it points to is the device's and the caller's.
 *
 * Page x is free where refs[x] <= 0.  A caller may hold a page that no entry names
 * by a reference of its own.  An entry of the table outside [0, num_pages) names no
 * page; calls write -1 there.  Calls on one pool have to follow each other (one
 * stream, or events between).
 */
typedef struct pld_pool {
    int32_t *table;        /* [seqs][table_stride] */
    int64_t table_stride;  /* >= max_pages */
    int32_t *refs;         /* [num_pages], 16-byte aligned */
    int seqs;              /* 1 .. 2^20 */
    int max_pages;         /* table entries per sequence; max_pages*page_size <= 2^30 */
    int num_pages;         /* 1 .. PLD_MAX_PAGES */
    int page_size;         /* a power of two in [16, 4096] */
} pld_pool;

/*
 * pld_pages_take -- pages for the next tokens: for each i, sequence seq[i]'s entries
 * for positions below need[i] that name no page get free ones, the lowest first,
 * in order of i and position.
 *   seq, need   int32 [count]
 *   status      int32 [count]: 0, or -1: seq[i] is not in [0, seqs) or is named by
 *               another i as well, or need[i] is past the table; or how many pages
 *               were lacking.  Pages go out in order: where too few are left for one
 *               i, it and all later ones that lack pages get none.
 *   count       1 .. PLD_MAX_PAGE_ENTRIES
 *   workspace   pld_pages_workspace_bytes(pool, count) bytes, 16-byte aligned,
 *               contents of no importance
 */
size_t pld_pages_workspace_bytes(const pld_pool *pool, int count);

int pld_pages_take(const pld_pool *pool, const int32_t *seq, const int32_t *need, int count,
                   int32_t *status, void *workspace, size_t workspace_bytes, void *stream);

/*
 * pld_pages_free -- sequence seq[i] gives back the pages of the entries for positions
 * from keep[i] on (keep NULL: all; a page that holds a kept position stays).  A page
 * is free again when no entry names it.  Sequences outside [0, seqs) are skipped, and
 * one may be named more than once.
 */
int pld_pages_free(const pld_pool *pool, const int32_t *seq, const int32_t *keep, int count,
                   void *stream);

/*
 * pld_pages_fork -- sequence dst[i] goes on from the first T = lens[i] tokens of
 * sequence src[i].  What dst[i] had is given back.  The pages before the one of
 * position T-1 are shared; that page, which the next pass writes (its first row is
 * position T-1), becomes a copy of its own: the slots of its positions below T, in
 * every layer, in the lowest free page (in order of i).  Later entries name no page.
 *   layers      the n_layers caches of the pool, 0 .. PLD_MAX_LAYERS: alike in all but
 *               k, v, k_scale, v_scale (their table is not used); pages and page size
 *               the pool's.  0: the integers alone
 *   status      int32 [count]: 0 or
 *               -1: src[i] or dst[i] is not in [0, seqs), dst[i] is src of any entry or
 *                   dst of another, T < 0 or past the table, or position T-1 has no page:
 *                   nothing is done;
 *               -2: no page was left: dst[i] has given back what it had, and has nothing
 *   workspace   as pld_pages_take
 * T = 0 leaves dst[i] with nothing.
 */
int pld_pages_fork(const pld_pool *pool, const pld_cache *layers, int n_layers, const int32_t *src,
                   const int32_t *dst, const int32_t *lens, int count, int32_t *status,
                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * pld_pages_compact -- pages in use move to the lowest indices.  With n pages in use
 * (refs > 0), those from index n on move, in order, to the free ones below n, whole and
 * in every layer; what they move from keeps its contents, and no page in use is written,
 * so that passes by the old table go on reading what they read.
 *   map         int32 [num_pages], written: a page's new index, -1 for a free one
 *   used        int32 [1], written: n
 *   table_out, refs_out   the new table ([seqs][table_out_stride]; entries that name no
 *               page as they were, -1 for those that name a free one) and references; may be
 *               the pool's own
 *   workspace   as pld_pages_take with count 1
 */
int pld_pages_compact(const pld_pool *pool, const pld_cache *layers, int n_layers, int32_t *map,
                      int32_t *used, int32_t *table_out, int64_t table_out_stride,
                      int32_t *refs_out, void *workspace, size_t workspace_bytes, void *stream);

/*
 * pld_pages_copy -- pages between two sets of caches (or within one): the first
 * slots[i] slots (NULL: all) of page src[i] of every layer of `from` to page dst[i] of
 * the same layer of `to`.  Pages out of range are skipped, slots outside [0, page_size]
 * count as all.  Layers of a set as in pld_pages_fork; the sets agree in type, page
 * size, heads and head_dim, not in strides or pages.  No page written may be read or
 * written by another i.
 *   count       1 .. PLD_MAX_PAGES
 */
int pld_pages_copy(const pld_cache *from, const pld_cache *to, int n_layers, const int32_t *src,
                   const int32_t *dst, const int32_t *slots, int count, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PLD_PROMPT_H */
