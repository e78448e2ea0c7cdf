/*
 * pld_model.h -- C ABI of the verification pass's model side on AMD Instinct
 * MI355X (gfx950): what the target model computes around a draft that no plain
 * matrix product covers.  The drafting and verification calls are in pld.h,
 * whose conventions (device pointers, streams, status codes, no allocation, no
 * synchronisation, deterministic results) hold here as well.
 *
 * Verifying a draft of K tokens (arXiv 2412.01447, Sec. 3 and Sec. 4.4) runs
 * the model over n = K + 1 rows per sequence.  With T = lens[b] committed
 * tokens, row i is the model's row for position p = T-1+i: the last committed
 * token, then the draft.  Row i exists when T >= 1, 0 <= draft_len[b] <= n-1
 * and i <= draft_len[b] (draft_len NULL: every sequence has n rows).  Rows that
 * do not exist are neither read nor written.  A prompt is read the same way: a
 * chunk of n tokens from position s on has lens = s + 1 and draft_len = n - 1.
 *
 * Per layer, pld_cache_write puts the rows' keys and values into the layer's
 * paged cache and pld_cache_attn attends to it; once the draft is verified,
 * pld_cache_attn_rows gives the attention weights of chosen heads at the row
 * whose position is the next step's artifact query (row accept_len[b]), in the
 * layout pld_rank_attn ranks by (Eq. 3).  pld_token_logprobs gives the log
 * probabilities of the emitted tokens with entropy and alternatives.
 *
 * A rejected draft's keys and values need no removal: the next pass's rows
 * start at the new T-1 and write over them, and no row reads past its own
 * position.
 */
#ifndef PLD_MODEL_H
#define PLD_MODEL_H

#include "pld.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Version of this header's ABI (major * 10000 + minor * 100 + patch). */
#define PLD_MODEL_ABI_VERSION 100
int pld_model_version(void);

/* Element type of a quantised cache, beside PLD_BF16: 8-bit floats of four
 * exponent and three fraction bits (finite, largest 448), with one fp32 scale
 * per slot and head. */
enum { PLD_E4M3 = 2 };

/* The elements of a head that a position's angles turn together. */
enum {
    PLD_ROPE_HALVES = 0,     /* element t with element t + rot_dim/2 */
    PLD_ROPE_NEIGHBOURS = 1  /* element 2t with element 2t + 1       */
};

#define PLD_MAX_CACHE_ROWS 65535   /* n: rows per sequence in one call */
#define PLD_MAX_TOP 64             /* alternatives per row of pld_token_logprobs */

/*
 * A layer's paged cache.  The struct itself is host memory, read during a call
 * and not kept; the memory it points to is the device's and the caller's.
 *
 * A page holds page_size consecutive positions of one sequence, for every key
 * head.  Element (page, slot, head, t) of k or v is at
 * page*page_stride + slot*slot_stride + head*head_stride + t, so pages of
 * [slot][head][t] and of [head][slot][t], and keys and values interleaved page
 * by page, are all served.  table[b*table_stride + p/page_size] is the page of
 * position p of sequence b.
 */
typedef struct pld_cache {
    void *k, *v;           /* 16-byte aligned; v is not used by pld_cache_attn_rows */
    int dtype;             /* PLD_BF16 or PLD_E4M3 */
    float *k_scale;        /* PLD_E4M3 only, else NULL: a stored element stands for   */
    float *v_scale;        /*   itself times scale[page*scale_page_stride +           */
    int64_t scale_page_stride; /* head*page_size + slot]; 16-byte aligned,            */
                           /*   scale_page_stride a multiple of 4, <= 2^31            */
    int64_t page_stride, slot_stride, head_stride;   /* elements; multiples of 16 bytes; */
                           /*   slot_stride <= 2^24, page_stride <= 2^34              */
    const int32_t *table;  /* [B][table_stride]; an entry outside [0, num_pages) is a bad page */
    int64_t table_stride;  /* >= max_pages */
    int num_pages;         /* >= 1 */
    int page_size;         /* a power of two in [16, 4096] */
    int max_pages;         /* table entries per sequence; max_pages*page_size <= 2^30 */
    int heads;             /* key heads, 1 .. 1024 */
    int head_dim;          /* 64, 128 or 256 */
} pld_cache;

/*
 * pld_cache_write -- a layer's new rows join the cache: queries and keys are
 * normed and rotated per head, keys and values stored at their positions'
 * slots, quantised where the cache is PLD_E4M3, and the queries written out.
 * For a head's row x (fp32 throughout, rounded once at the end):
 *   norm     x_t = x_t / sqrt(mean(x^2) + eps) * w_t   (q_norm / k_norm NULL: skipped)
 *            (elements of up to 2^59: the squares are summed in fp32)
 *   rotate   each pair (a, c) of the first rot_dim elements becomes
 *            (a cos - c sin, c cos + a sin) with the pair's cos and sin of the
 *            row's position (rope NULL: skipped); values are neither normed
 *            nor rotated
 *   store    bf16, or for PLD_E4M3: scale = max|x| / 448, element x_t / scale
 *            (a scale below 2^-126 is stored as 2^-126)
 *
 *   q, k, v     bf16; row i of sequence b starts at b*seq_stride + i*row_stride,
 *               heads follow each other (Hq, cache heads, cache heads); 16-byte
 *               aligned, strides multiples of 8 elements
 *   q_norm, k_norm   bf16 [head_dim], 16-byte aligned, or NULL
 *   rope        fp32; position p's row at p*rope_stride: rot_dim/2 cosines, then
 *               rot_dim/2 sines; 16-byte aligned, rope_stride a multiple of 4; or NULL
 *   n_pos       positions in the table;  rot_dim a multiple of 8, <= head_dim
 *   q_out       bf16, laid out like q; may be q itself with q's strides
 * Device-side rule: a row whose position is past the table of pages (or past
 * n_pos, with rope), or whose page is bad, is not stored, and its q_out is NaN.
 * Errors: PLD_ERR_INVALID (NULL, a size out of range, Hq not a multiple of the
 * cache's heads, eps not finite or negative, q_out at q with other strides),
 * PLD_ERR_ALIGN, PLD_ERR_LAUNCH.
 */
int pld_cache_write(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                    int64_t q_row_stride, const uint16_t *k, int64_t k_seq_stride,
                    int64_t k_row_stride, const uint16_t *v, int64_t v_seq_stride,
                    int64_t v_row_stride, const uint16_t *q_norm, const uint16_t *k_norm,
                    float eps, const float *rope, int64_t rope_stride, int n_pos, int rot_dim,
                    int rope_pairs, const int32_t *lens, const int32_t *draft_len, int B, int n,
                    int Hq, uint16_t *q_out, int64_t o_seq_stride, int64_t o_row_stride,
                    void *stream);

/*
 * pld_cache_attn -- attention of every existing row over its sequence's cache.
 * Row i (position p) sees the keys j <= p, or p - window < j <= p when
 * window > 0.  With the key head h / (Hq / heads) of query head h:
 *   s_j = (q . k_j) * scale;  softcap > 0: s_j = softcap * tanh(s_j / softcap)
 *   out = sum_j exp(s_j - lse) v_j,   lse = log sum_j exp(s_j)
 * The rows' own keys and values must be in the cache (pld_cache_write).
 *
 *   q           bf16, as pld_cache_write's q_out
 *   scale       > 0 (1 / sqrt(head_dim) as a rule);  softcap >= 0;  window >= 0
 *               (scale at most 2^127; softcap 0 or from 2^-125 to 2^126)
 *   out         bf16, laid out like q with its own strides; not q
 *   lse         fp32 [B][n][Hq] or NULL
 *   workspace   pld_cache_attn_workspace_bytes(B, n, Hq, heads, head_dim) bytes,
 *               16-byte aligned, contents of no importance; calls that overlap in
 *               time must not share it (the size never falls as n grows: one for
 *               the most rows serves fewer)
 * Device-side rules: keys that a row does not see do not affect it, whatever
 * their slots hold; a row one of whose keys lies on a bad page or past the table
 * gets NaN in out and lse.  Where a value that a row sees is not finite, that head
 * of its out, and its lse, may be NaN as a whole.  Values past 2^89 may overflow: up
 * to 2^30 of them are summed, with weights of up to 2^8, before the division by the
 * weights' sum.  A row has to see a score above -1e29 (no finite inputs of ordinary
 * size come near it).
 * Errors: PLD_ERR_INVALID (also out at q), PLD_ERR_ALIGN, PLD_ERR_WORKSPACE,
 * PLD_ERR_LAUNCH.
 */
size_t pld_cache_attn_workspace_bytes(int B, int n, int Hq, int heads, int head_dim);

int pld_cache_attn(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                   int64_t q_row_stride, const int32_t *lens, const int32_t *draft_len, int B,
                   int n, int Hq, float scale, float softcap, int window, uint16_t *out,
                   int64_t o_seq_stride, int64_t o_row_stride, float *lse, void *workspace,
                   size_t workspace_bytes, void *stream);

/*
 * pld_cache_attn_rows -- attention weights as a ranking artifact (Eq. 3, Sec.
 * 4.2.1): for one row of each sequence and R chosen query heads of the layer,
 *   attn[b][r][j] = exp(s_j - lse)  for the keys the row sees, 0 for the other j <= p,
 * over 0 <= j < min(p + 1, n_keys), with s_j and lse as pld_cache_attn has them.
 * Later entries are left as they were.  With row = accept_len of the
 * verification, attn is what pld_rank_attn (pld_draft_attn) takes for the next
 * step.  Heads chosen from several layers: one call a layer, each with its
 * rows of a shared attn buffer.
 *
 *   row         int32 [B]: the row, in [0, n-1]; a sequence with another value,
 *               or with T < 1, is left as it was
 *   heads       int32 [R]: query heads, in any order, repeated or not; a value
 *               outside [0, Hq-1] gets NaN
 *   lse         fp32 [B][n][Hq] from pld_cache_attn of the same rows
 *   attn        fp32; (b, r, j) at b*a_seq_stride + r*a_row_stride + j
 * Device-side rule: a key on a bad page or past the table gets NaN.
 * Errors: PLD_ERR_INVALID (also R outside [1, 65535], n_keys < 1 or
 * past 2^31 - 65537), PLD_ERR_ALIGN,
 * PLD_ERR_LAUNCH.
 */
int pld_cache_attn_rows(const pld_cache *cache, const uint16_t *q, int64_t q_seq_stride,
                        int64_t q_row_stride, const int32_t *lens, const int32_t *row,
                        const int32_t *heads, int R, const float *lse, int B, int n, int Hq,
                        float scale, float softcap, int window, float *attn, int64_t a_seq_stride,
                        int64_t a_row_stride, int64_t n_keys, void *stream);

/*
 * pld_token_logprobs -- log probabilities of given tokens (those a verification
 * emitted, as a rule) with entropy and the most likely alternatives, under
 * softmax(z / temperature) of the rows pld_verify_* read.  With lse the log of
 * the row's sum of exp(z_v / temperature), for the rows i < count[b]:
 *   logprob[b][i] = z_t / temperature - lse,  t = tokens[b][i];  NaN for t outside [0, V)
 *   entropy[b][i] = -sum_v p_v log p_v  (terms of p_v = 0 are 0)
 *   top_ids[b][i][k], top_logprobs[b][i][k]: the k-th largest logit's token, the
 *                   lowest id first among equals (-0 == +0); past V: -1 and -inf
 * Other rows are left as they were.  A row of -inf only has logprob and
 * top_logprobs -inf and entropy 0; NaN and +inf logits are outside the contract.
 *
 *   logits, dtype, l_seq_stride, l_row_stride, V   as pld_verify_greedy, with n rows
 *   tokens      int32 [B][n];  count int32 [B] or NULL (n rows each); a count
 *               outside [0, n] counts as 0
 *   temperature finite, > 0 (from 2^-127 on: log2(e) / temperature is taken in fp32).  Rows
 *               whose largest |z / temperature| is past 2^23 take longer: they are read again
 *   logprob     fp32 [B][n];  entropy fp32 [B][n] or NULL
 *   top         0 .. PLD_MAX_TOP;  top_ids int32 [B][n][top], top_logprobs fp32
 *               [B][n][top], both required when top > 0
 *   workspace   pld_token_logprobs_workspace_bytes(B, n, V, dtype, top) bytes,
 *               16-byte aligned, contents of no importance; calls that overlap in
 *               time must not share it
 * Errors: PLD_ERR_INVALID, PLD_ERR_ALIGN, PLD_ERR_WORKSPACE, PLD_ERR_LAUNCH.
 */
size_t pld_token_logprobs_workspace_bytes(int B, int n, int V, int dtype, int top);

int pld_token_logprobs(const void *logits, int dtype, int64_t l_seq_stride, int64_t l_row_stride,
                       int V, int n, const int32_t *tokens, const int32_t *count, int B,
                       double temperature, float *logprob, float *entropy, int top,
                       int32_t *top_ids, float *top_logprobs, void *workspace,
                       size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* PLD_MODEL_H */
