/*
 * specdec.h -- C ABI of the verification step of speculative decoding
 * (Algorithm 1: "determine the accepted token length n_t" and "verify and update
 * the draft sequence") on batches of synthetic draft / target distributions.
 *
 * A batch holds B independent steps.  Step b has k draft positions over a
 * vocabulary of V tokens:
 *   q[b][j][.]  draft distribution at position j (j < k),
 *   p[b][j][.]  target distribution at position j (j <= k; row k is used when
 *               every draft token is accepted),
 *   tok[b][j]   the draft token x_j (drawn from q[b][j] by the caller),
 *   r[b][j]     the uniform r_j in [0, 1) of the acceptance test,
 *   u[b]        a uniform 32-bit integer for the resampling draw.
 * All arrays are DEVICE pointers, row-major float32 / int32 / uint32, owned by the
 * caller and read-only; outputs are device pointers owned by the caller.  Calls
 * are asynchronous on `hip_stream` (a hipStream_t; NULL = default stream).  The
 * library allocates nothing.
 *
 * Every function returns 0 or a negative sd_status.
 */
#ifndef SPECDEC_H
#define SPECDEC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    SD_OK = 0,
    SD_EINVAL = -1,        /* null / misaligned pointer, non-positive size */
    SD_EUNSUPPORTED = -2,  /* k > SD_MAX_K or V > SD_MAX_V */
    SD_EHIP = -3,          /* HIP runtime error */
    SD_ENOMEM = -4         /* workspace too small */
} sd_status;

/* Element types of logits, keys, values and queries. */
typedef enum { SD_F32 = 0, SD_BF16 = 1, SD_F16 = 2 } sd_dtype;

#define SD_MAX_K 64         /* candidate length */
#define SD_MAX_V 262144     /* vocabulary size */
#define SD_FIXED_BITS 40    /* probabilities are summed as integers in units of 2^-40 */
#define SD_MAX_REQUESTS 4096 /* requests of one served step */
#define SD_MAX_HEAD_DIM 256 /* D of sd_attend */

/*
 * Accepted length and next token of every step (Algorithm 1):
 *   n[b]    = min({ j : r_j > p_j(x_j) / q_j(x_j) } U { k })   (0-based j: the number of
 *             accepted draft tokens); the test is evaluated as NOT(r_j * q_j(x_j) <= p_j(x_j))
 *             in float32, so q_j(x_j) = 0 accepts;
 *   next[b] ~ p' with p'(x) proportional to max(0, p_n(x) - q_n(x)) if n < k, and p' = p_k
 *             otherwise.
 * The draw is the inverse CDF in exact integer arithmetic, so it does not depend on
 * summation order: m(x) = trunc(2^40 * max(0, p_n(x) - q_n(x))) (float32 subtraction),
 * Z = sum_x m(x), target = floor(Z * u / 2^32), next = the smallest x whose inclusive prefix
 * sum exceeds target.  If Z == 0 (the residual vanishes at this resolution) p' = p_n.
 * tok values outside [0, V) are clamped.  n_dev, next_dev: device [B] int32.
 */
int sd_verify(const float *p_dev, const float *q_dev, const int32_t *tok_dev, const float *r_dev,
              const uint32_t *u_dev, int64_t B, int64_t k, int64_t V, int32_t *n_dev,
              int32_t *next_dev, void *hip_stream);

/*
 * Acceptance rate of every draft position, Eq. (1):
 *   acc[b][j] = E_{x ~ q_j} min{1, p_j(x) / q_j(x)} = sum_x min(p_j(x), q_j(x)) = 1 - TV(p_j, q_j),
 * summed in float64 in a fixed order.  acc_dev: device [B][k] float64.  p_dev has k+1 rows
 * per step as in sd_verify (row k is not read).
 */
int sd_acceptance(const float *p_dev, const float *q_dev, int64_t B, int64_t k, int64_t V,
                  double *acc_dev, void *hip_stream);

/*
 * ---- A served verification step ------------------------------------------------------------
 * The target model checks the drafts of B requests in one pass over a batch of ragged chunks:
 * request b brings m_b = cu[b+1] - cu[b] new tokens (the last emitted one and its k_b = m_b - 1
 * drafts, or a part of a prompt), whose rows are cu[b] .. cu[b+1]-1 of every array "of tokens".
 * Keys and values live in a cache of pages of `page` tokens; table[b][i] is the page that holds
 * the tokens i*page .. i*page+page-1 of request b, and token t of a page P has the slot P*page+t.
 * A step calls sd_pages, then per layer sd_cache_store and sd_attend, and sd_verify_logits last;
 * its accepted lengths go into the next step's sd_pages.
 *
 * As above: device pointers unless said otherwise, owned by the caller; asynchronous on
 * hip_stream; nothing is allocated; every argument that the host can see is checked before
 * anything is launched.  Numbers that only the device sees (lengths, table entries, slots, token
 * ids, row offsets) are clamped to what the arrays hold, so that a wrong one gives wrong results and no
 * access outside the arrays.  Strides are in elements.  All calls can be captured into a HIP graph.
 */

/*
 * Block tables and slot maps of a step.  All integers; the result does not depend on how the work is
 * divided.  With keep_b the valid tokens of request b and want_b the pages that it needs,
 *   keep_b = min(length[b] + (accepted ? max(accepted[b], -1) + 1 : 0), pages[b] * page),
 *   want_b = ceil((keep_b + add[b]) / page):
 * pages of requests with want_b < pages[b] (rejected drafts; finished requests: length = add = 0, accepted = -1 or NULL)
 * are pushed onto the stack of free pages, requests in order, pages in ascending place; then the others
 * take theirs from its top, requests in order.  A request with want_b > width is refused, and so is, from
 * the first one that finds too few pages on, every request that needs more than it holds: it keeps
 * its pages, and its tokens get slot and position -1.
 *
 * Of a refused request (kv_out[b] = length_out[b] with add[b] > 0) no new key is in the cache.  What sd_attend and sd_verify_logits
 * write for its rows then means nothing, and the caller has to give accepted[b] = -1 in the next step, which says that nothing of the last chunk stands,
 * the token before its drafts no more than they; the request stays where it was and may bring the same tokens again.
 *
 * Reads only table entries below pages[b] and stack entries below *nfree, and writes only others,
 * so a call can be repeated with the same inputs.  No output may be one of the inputs.
 * B <= SD_MAX_REQUESTS; pool * page, width * page and width * B below 2^31.  Row offsets that would pass 2^31 - 1 end there.
 */
typedef struct {
    int64_t B, page;              /* requests; tokens of a page */
    int64_t width, table_stride;  /* entries of a table row; elements from row to row */
    int64_t pool;                 /* pages there are = entries of `free` */
    int64_t tokens;               /* entries of slot_out and pos_out: the sum of add, or more (the rest gets -1), or fewer (tokens past them are left out) */
    const int32_t *pages;         /* [B] pages held */
    const int32_t *length;        /* [B] tokens that were valid before the last step's chunk */
    const int32_t *accepted;      /* [B] accepted drafts of the last step; -1 (or below), NULL: length is what is valid */
    const int32_t *add;           /* [B] new tokens */
    const int32_t *nfree;         /* [1] free pages */
    int32_t *table;               /* [B][width] in place */
    int32_t *free;                /* [pool] in place: the stack, its top at entry *nfree - 1 */
    int32_t *pages_out;           /* [B] pages held now */
    int32_t *length_out;          /* [B] keep_b */
    int32_t *kv_out;              /* [B] keep_b + add[b], or keep_b if refused: keys in the cache once the chunk is stored */
    int32_t *nfree_out;           /* [1] */
    int32_t *cu_out;              /* [B+1] */
    int32_t *slot_out;            /* [tokens] */
    int32_t *pos_out;             /* [tokens] place of the token in its request */
} sd_page_step;

int sd_pages(const sd_page_step *step, void *hip_stream);

/* A paged cache of one layer: element d of head h of token t of page P at P*page_stride + t*tok_stride +
 * h*head_stride + d, so pages may be laid out token by token or head by head. */
typedef struct {
    void *k, *v;
    int64_t pages, page, heads, D;
    int64_t k_page_stride, k_tok_stride, k_head_stride;
    int64_t v_page_stride, v_tok_stride, v_head_stride;
    int32_t dtype;                /* sd_dtype */
} sd_cache;

/*
 * Keys and values of new tokens into their slots.  k, v: [tokens][heads][D] with the given strides, of the
 * cache's type.  Tokens with a slot outside [0, pages * page) are skipped (sd_pages marks refused ones with -1);
 * the others' slots have to be distinct.
 */
int sd_cache_store(const sd_cache *cache, const void *k, int64_t k_tok_stride, int64_t k_head_stride, const void *v,
                   int64_t v_tok_stride, int64_t v_head_stride, const int32_t *slot, int64_t tokens, void *hip_stream);

/*
 * Attention of the chunk of every request over its pages.  The m_b rows of request b are its last
 * tokens: row i stands at position pos = kv[b] - m_b + i and sees the keys j with
 * max(0, pos - window + 1) <= j <= pos (window = 0: from 0 on).  Query head h reads key head h / (Hq / heads).
 *   out = sum_j softmax_j(scale <q, k_j>) v_j,      lse = log sum_j exp(scale <q, k_j>);
 * a row that sees no key (pos < 0) gets out = 0 and lse = -inf.  Rows of no request (past cu[B]) are not written.
 * Keys that no row of a chunk sees are not used, whatever they hold.  Of a key that some rows see and others do not (a later
 * token of the chunk, the edge of the window) those others see nothing if its value is finite; one that is not may turn their results
 * into NaN too, since a weight of 0 multiplies it.
 * SD_BF16 and SD_F16; scores, softmax and sums are float32, the weights are rounded to the cache's type
 * before they multiply the values (in float16 those below 2^-21 of a row's largest lose bits, and below 2^-32 they vanish there, though not
 * from the sum that divides).  D a multiple of 8, at most SD_MAX_HEAD_DIM; rows of D elements and all
 * strides 16-byte aligned.
 * Refused with SD_EUNSUPPORTED: more threads than a launch holds, 2^32 (thousands of requests with thousands of key heads each).
 * `ws` (16-byte aligned) needs sd_attend_workspace_bytes.  It holds parts of rows whose keys are split over workgroups; how
 * they are split depends on the shapes and lengths alone, so equal calls give equal bits.
 */
typedef struct {
    sd_cache cache;
    int64_t B, tokens, Hq;
    int64_t width, table_stride;  /* of table */
    const void *q;                /* [tokens][Hq][D] */
    int64_t q_tok_stride, q_head_stride;
    void *out;                    /* [tokens][Hq][D] */
    int64_t out_tok_stride, out_head_stride;
    float *lse;                   /* [tokens][Hq], or NULL */
    const int32_t *cu;            /* [B+1] */
    const int32_t *kv;            /* [B] keys of the request, its new tokens included */
    const int32_t *table;         /* [B][width] */
    int64_t window;
    double scale;                 /* > 0 */
} sd_attention;

size_t sd_attend_workspace_bytes(const sd_attention *a);   /* 0 if a call with these sizes would be refused; pointers are not read */
int sd_attend(const sd_attention *a, void *ws, size_t ws_bytes, void *hip_stream);

/*
 * Accepted length and next token of every request from logits.  Row t of p (t = cu[b] + j) holds the target's
 * logits behind the j-th of the chunk's tokens; row cu[b] - b + j of q, tok and r belongs to draft j of request b
 * (all of a batch's drafts one behind the other).  Every request has at least one row.  With
 * P_j = softmax(p_j / tau[b]) and Q_j = softmax(q_j / tau[b]) (q = NULL: drafts without a distribution, Q_j = 1 at the draft):
 *   n[b]    = min({ j : NOT(r_j Q_j(x_j) <= P_j(x_j)) } U { k_b });
 *   next[b] ~ max(0, P_n - Q_n) if n < k_b and that is not zero everywhere, and P_n otherwise, drawn as an
 *             exponential race: next = argmax_x weight(x) / noise[b][x] with noise ~ Exp(1), ties to the lowest x.
 * tau[b] <= 0 or NaN is greedy: n[b] = the drafts that are their row's first largest logit, one after the other;
 * next[b] = that of row n; r, q and noise are not used.
 * A logit that is NaN counts as -inf (probability 0), +inf as the largest float.  A row without any finite logit
 * has all probabilities 0, and gives next = 0.  tok is clamped to [0, V).
 * Rows of p and q together fewer than 2^24.
 * Sums are float64 over float32 parts, in a fixed order.  ws (16-byte aligned): sd_verify_logits_workspace_bytes.
 */
typedef struct {
    int64_t B, rows, V;           /* requests; rows of p, B of which test no draft */
    int32_t dtype;                /* sd_dtype of p and q */
    const void *p; int64_t p_stride;       /* [rows][V] */
    const void *q; int64_t q_stride;       /* [rows - B][V], or NULL */
    const int32_t *tok;                    /* [rows - B] */
    const float *r;                        /* [rows - B] uniform in [0, 1) */
    const float *noise; int64_t noise_stride;   /* [B][V], >= 0 */
    const float *tau;                      /* [B] */
    const int32_t *cu;                     /* [B+1] */
} sd_logits;

size_t sd_verify_logits_workspace_bytes(const sd_logits *a);  /* as above */
int sd_verify_logits(const sd_logits *a, int32_t *n_dev, int32_t *next_dev, void *ws, size_t ws_bytes, void *hip_stream);

/* Static, human-readable text for a status code. */
const char *sd_strerror(int status);

#ifdef __cplusplus
}
#endif
#endif /* SPECDEC_H */
