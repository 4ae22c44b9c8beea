/*
 * na_seq.h -- C ABI of the sequence operators of libna.so: the attention of a causal 1-D
 * neighbourhood with first tokens that stay visible, its gradient, and the paged cache that
 * serves it one step at a time, whose requests may share first tokens and are cut back to a
 * budget by the attention weight that their keys gathered.
 *
 * Attention.  Token i of a sequence attends to token j when
 *     j <= i   and   (i - j < kernel_size   or   j < sinks):
 * the causal window of na_forward along one axis (its kernel_size nearest tokens up to
 * itself, no dilation), and the first `sinks` tokens of the sequence.  Any kernel_size >= 1
 * is legal; one at or above the length is full causal attention.  Query heads share
 * key/value heads in groups: query head h reads key/value head h / (heads / kv_heads).
 *     s_ij = scale q_i . k_j,  lse_i = log sum_j exp s_ij,  out_i = sum_j exp(s_ij - lse_i) v_j
 *
 * Conventions, beside those of na.h (streams, statuses, ownership):
 *   - Strides count elements; the last axis is contiguous.  Every stride of an input may be 0
 *     (a broadcast axis); outputs must not overlap themselves.  A stride is a multiple of 16
 *     bytes, and a token stride below 2^26 bytes.  The stride of an axis of one entry does not
 *     matter.
 *   - Data pointers (q, k, v, out, gradients, pages, logsumexp, workspaces) are 16-byte
 *     aligned, integer arrays by their element.  Integer arrays are device memory.
 *   - Queries, keys and values of the tokens that a sequence has are finite.  What lies behind
 *     a sequence's length, on unused pages, or on pages that no new token sees, may hold
 *     anything, NaN included.  An output gradient that is not finite makes the gradients that
 *     it reaches infinite or NaN.
 *   - Outputs overlap neither the inputs nor each other.
 *   - A workspace belongs to one call until that call's work on the stream is done; calls
 *     that may run at once need one each.
 */
#ifndef NA_SEQ_H_
#define NA_SEQ_H_

#include "na.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
    int64_t batch, head, token;
} na_strides;

/* Attention over contiguous sequences. */
typedef struct {
    int64_t batch, heads, kv_heads, tokens, head_dim;
    int64_t kernel_size, sinks;
    na_strides q, k, v, out;        /* [batch, heads | kv_heads, tokens, head_dim] */
    na_strides dout, dq, dk, dv;    /* na_sink_backward only */
    int32_t dtype;                  /* na_dtype */
    float scale;
} na_sink_problem;

/*
 * Forward.  lengths: valid tokens per sequence (int32 [batch], clamped to [0, tokens]), or
 * NULL where all are; rows behind a length get out 0 and logsumexp -inf, and their keys are
 * not read.  logsumexp: contiguous [batch, heads, tokens] fp32, natural log.
 * NA_ERR_SHAPE: kv_heads does not divide heads, only one of the two is 0, an extent is negative,
 * a stride breaks the rules above, sinks is negative, tokens * (heads / kv_heads) reaches 2^30, or
 * batch * kv_heads * ceil(tokens * (heads / kv_heads) / 128) reaches 2^24.
 */
na_status na_sink_forward(const na_sink_problem* problem, const void* q, const void* k,
                          const void* v, const int32_t* lengths, void* out, float* logsumexp,
                          na_stream_t stream);

/*
 * Gradients of out with respect to q, k and v given dout, from the saved out and logsumexp of
 * na_sink_forward on the same inputs.  A shared key/value head sums the rows of its whole
 * group.  dq, dk, dv are fully overwritten (0 behind a length) and must not alias the inputs or
 * each other.  Deterministic: the same inputs give bit-identical gradients.
 * workspace: na_sink_backward_workspace(problem) bytes; NA_ERR_WORKSPACE if workspace_bytes is
 * less.  (0 for a problem that is empty or not valid.)
 * NA_ERR_SHAPE also where dk and dv would take 2^23 workgroups or more: one for 128 keys of a
 * key/value head, and one for 32 of its first tokens that rows outside their window see (up to
 * 1024 in all where those are fewer).
 */
size_t na_sink_backward_workspace(const na_sink_problem* problem);
na_status na_sink_backward(const na_sink_problem* problem, const void* q, const void* k,
                           const void* v, const int32_t* lengths, const void* out,
                           const float* logsumexp, const void* dout, void* dq, void* dk, void* dv,
                           void* workspace, size_t workspace_bytes, na_stream_t stream);

/* The paged cache.  A page holds page_size tokens (a power of two, 16 or more) of every
 * key/value head: k_pages, v_pages are contiguous [pages, kv_heads, page_size, head_dim]
 * arrays.  Row r of the page table (int32 [requests, max_pages]) lists the pages of request
 * r in the order of its tokens. */
typedef struct {
    int64_t requests, tokens;  /* requests; new tokens of all of them (rows of q, k, v) */
    int64_t heads, kv_heads, head_dim;
    int64_t pages, page_size, max_pages;
    int64_t kernel_size, sinks;
    int64_t max_new, max_context;  /* see na_cache_attention */
    na_strides q, k, v, out;       /* [tokens, heads | kv_heads, head_dim]; batch unused */
    int32_t dtype;
    float scale;
} na_cache_problem;

/*
 * Tables of a step, from request lengths: request r has context_lens[r] tokens in the cache
 * and gets new_lens[r] more (device int32 arrays; negative counts as 0,
 * more than 2^30 as 2^30).
 *   cu_new[requests + 1]  offsets of the requests' new tokens, exclusive sums of new_lens
 *   positions[tokens]     int32, position of each new token in its request
 *   slots[tokens]         int64, page * page_size + offset in the page; -1 without a page
 *   page_table            entries of pages that the new tokens begin are written, request by
 *                         request from free_pages[*head], [*head + 1], ..; others are left
 *   new_head[1]           *head plus the pages taken.  Above num_free the pool ran dry: the
 *                         last tokens' pages are -1, their slots too
 * NA_ERR_SHAPE: requests, tokens or num_free reach 2^30, page_size and the table's size as in
 * na_cache_attention, or new_head is head.
 * head may be NULL (0); new_head must be other memory than head.  `tokens` is the room in
 * slots and positions: entries behind the last new token get -1; new tokens beyond the room
 * get no entry, as those beyond max_pages pages get no page.
 */
na_status na_cache_tables(int64_t requests, int64_t tokens, int64_t page_size, int64_t max_pages,
                          int64_t num_free, const int32_t* context_lens, const int32_t* new_lens,
                          const int32_t* free_pages, const int32_t* head, int32_t* page_table,
                          int32_t* cu_new, int64_t* slots, int32_t* positions, int32_t* new_head,
                          na_stream_t stream);

/*
 * Writes row t of k and v ([tokens, kv_heads, head_dim], strided) into the pages at slots[t].
 * Slots outside [0, pages * page_size) are skipped.  Slots of one call must differ: two equal
 * ones leave a mixture of both rows.
 * NA_ERR_SHAPE: page_size as below, kv_heads or a stride out of range, tokens * kv_heads reaches
 * 2^30, or the 16-byte pieces of k do 2^31.
 */
na_status na_cache_write(const na_cache_problem* problem, const void* k, const void* v,
                         const int64_t* slots, void* k_pages, void* v_pages, na_stream_t stream);

/*
 * Attention of new tokens over a cache that already holds them: token t of request r is at
 * position context_lens[r] + t, row cu_new[r] + t of q, out and logsumexp.
 * logsumexp: contiguous [tokens, heads] fp32.  Rows from cu_new[requests] on are left as they
 * were.  A page id outside [0, pages), or a column beyond max_pages, reads as a page of zero
 * keys and values; context lengths are clamped to [0, max_pages * page_size].  A request whose
 * range of rows is not inside [0, tokens) has no rows.  (Where cu_new decreases somewhere, it is
 * left open which of the requests that have rows get them.)
 * max_new, max_context: bounds of new_lens and of context + new that the caller knows (0:
 * unknown).  They choose how the work is split, and are not relied on for the result.
 * workspace: na_cache_attention_workspace(problem) bytes (it may be 0: then NULL is fine);
 * NA_ERR_WORKSPACE if workspace_bytes is less.  It grows with the requests, those without new
 * tokens among them.
 * NA_ERR_SHAPE: what na_sink_forward refuses of heads, sinks and strides; page_size is no power of
 * two from 16 to 2^20; requests reach 2^24, max_pages * page_size passes 2^30, requests * max_pages
 * reaches 2^31 or a page's bytes do, tokens * (heads / kv_heads) reaches 2^30 - 256, or
 * (tokens * (heads / kv_heads) / 32 + requests) * kv_heads reaches 2^24.
 */
size_t na_cache_attention_workspace(const na_cache_problem* problem);
na_status na_cache_attention(const na_cache_problem* problem, const void* q, const void* k_pages,
                             const void* v_pages, const int32_t* page_table,
                             const int32_t* context_lens, const int32_t* cu_new, void* out,
                             float* logsumexp, void* workspace, size_t workspace_bytes,
                             na_stream_t stream);

/* ---- long contexts: shared first tokens, gathered weights, eviction ---- */

/* Groups of requests that share their first tokens. */
typedef struct {
    na_cache_problem cache;      /* max_context unused */
    int64_t groups;
    int64_t max_shared, max_own; /* see na_cache_shared_attention */
} na_shared_problem;

/*
 * Attention of new tokens over a cache in which groups of requests share their first tokens: what
 * na_cache_attention computes, with the shared keys read once for all rows of a group.
 *   cu_groups[groups + 1]   group g holds the requests cu_groups[g] .. cu_groups[g + 1] - 1; the
 *                           offsets do not decrease (otherwise it is left open which requests
 *                           are in which group).  Requests outside of all groups share nothing.
 *   shared_lens[groups]     the first shared_lens[g] tokens of each request of group g are the
 *                           same, on the pages that the group's first request lists: a key
 *                           before shared_lens[g] is read there, one from it on on the request's
 *                           own pages (clamped to [0, max_pages * page_size]).  It need not fill
 *                           whole pages, and may reach past a request's context.
 * Both are int32 device arrays (they may be NULL where groups is 0).  max_new bounds the new tokens
 * of a request, max_shared the shared ones of a group, max_own those of a request behind the
 * shared ones, the new ones among them (0: unknown): they choose how the work is split, and are
 * not relied on for the result.  A row that sees a key whose score is NaN or +inf (a key that is
 * not finite, or a product beyond fp32) gets NaN in out and logsumexp; a value that is not finite
 * makes its column so in the rows that see it, and may in rows beside them, as in na_cache_attention.
 * workspace: na_cache_shared_attention_workspace(problem) bytes; NA_ERR_WORKSPACE if
 * workspace_bytes is less.  (0 for a problem that is empty or not valid.)
 * NA_ERR_SHAPE: what na_cache_attention refuses; groups is negative or reaches 2^24; a bound is
 * negative; or (tokens * (heads / kv_heads) / 32 + 4 * requests + groups) * kv_heads reaches 2^24.
 */
size_t na_cache_shared_attention_workspace(const na_shared_problem* problem);
na_status na_cache_shared_attention(const na_shared_problem* problem, const void* q,
                                    const void* k_pages, const void* v_pages,
                                    const int32_t* page_table, const int32_t* context_lens,
                                    const int32_t* cu_new, const int32_t* cu_groups,
                                    const int32_t* shared_lens, void* out, float* logsumexp,
                                    void* workspace, size_t workspace_bytes, na_stream_t stream);

/* Gathered attention weights: fp32 [requests, kv_heads, capacity], contiguous; entry j belongs to
 * the token at position j of the request.  A capacity may be less than the tokens of a request:
 * those behind it gather nothing. */
typedef struct {
    na_cache_problem cache;  /* v, out unused */
    int64_t capacity;
} na_weights_problem;

/*
 * Adds to weights[r, c, j] the attention weights that the new tokens of request r gave key j:
 *     sum over new tokens i that see j, and query heads h of key/value head c, of
 *     exp(scale q_ih . k_jc - logsumexp_ih),
 * with the logsumexp ([tokens, heads], 4-byte aligned) that na_cache_attention (or the form above)
 * returned for the same tokens.  The keys of the new tokens are in the cache.  Entries before
 * first[r] (int32 [requests] or NULL: none), of keys that no new token sees, and of requests
 * without new tokens are left as they were.  (Keys before first[r] are read all the same.)  All keys are
 * read on each request's own pages.  A page outside the pool reads as zero keys.
 * Deterministic: the same inputs give the same bits.  Weights must overlap no input.
 * max_new and max_context as in na_cache_attention.
 * workspace: na_cache_weights_workspace(problem) bytes (it may be 0: then NULL is fine);
 * NA_ERR_WORKSPACE if workspace_bytes is less.
 * NA_ERR_SHAPE: what na_cache_attention refuses of these arguments; capacity is negative,
 * or requests * kv_heads * capacity reaches 2^40; or requests * kv_heads reaches 2^20.
 */
size_t na_cache_weights_workspace(const na_weights_problem* problem);
na_status na_cache_weights(const na_weights_problem* problem, const void* q,
                           const float* logsumexp, const void* k_pages, const int32_t* page_table,
                           const int32_t* context_lens, const int32_t* cu_new,
                           const int32_t* first, float* weights, void* workspace,
                           size_t workspace_bytes, na_stream_t stream);

typedef struct {
    int64_t requests, kv_heads, head_dim;
    int64_t pages, page_size, max_pages, num_free;
    int64_t capacity;        /* of weights and new_weights */
    int64_t budget, recent;  /* tokens that stay, and how many of them the last ones */
    int32_t dtype;
} na_evict_problem;

/*
 * Cuts the requests of a cache back to `budget` tokens a key/value head.  A request with
 * context_lens[r] <= budget stays as it is.  Of the others each key/value head keeps
 *   the first f = min(first[r], budget) tokens (first: int32 [requests], or NULL: 0),
 *   the last l = min(recent, budget - f), and
 *   of those between the budget - f - l of largest weight (of equal ones those of lower position;
 *   NaN is below all, and so the weights behind the capacity count as 0),
 * and the request's first `budget` positions then hold, key/value head by key/value head:
 *   the first tokens, and at their own positions those of largest weight that lie before
 *   end = budget - l;
 *   at the other positions before end, in order, those of largest weight from end on;
 *   from end on the last l tokens, in order.
 * Rows of k_pages and v_pages move in place, on the request's own pages of the first `budget`
 * positions.  Positions before f are neither read nor written, so requests may share the pages
 * of their first f tokens; a page that holds other positions belongs to one request.  A row
 * from a page outside the pool is zeros, and one to such a page goes nowhere.
 *   kept[requests, kv_heads, budget]         position at which what is there now was; -1 behind
 *                                            the tokens of a request below the budget
 *   new_weights[requests, kv_heads, capacity] the weights of what is there now, 0 behind it
 *   new_context[requests]                    min(context_lens[r], budget), context_lens[r] clamped
 *                                            to [0, max_pages * page_size]
 *   new_head[1], free_pages[num_free]        pages of the positions from budget on return to the
 *                                            list that na_cache_tables takes from: new_head is
 *                                            *head minus their number (not below 0), and they are
 *                                            entered from there on, request by request; entries
 *                                            outside [0, num_free) are dropped.  The page table is
 *                                            left as it is.
 * From then on a position is a place in the cache: na_cache_tables counts the new tokens' positions on
 * from new_context, and kernel_size counts places.  Where a token stands in its text, for keys that
 * were rotated by it, is for the caller to keep (kept says where a place's token was).
 * Outputs overlap neither the inputs nor each other.  All of it is exact, and the same inputs give
 * the same bits.
 * workspace: na_cache_evict_workspace(problem) bytes; NA_ERR_WORKSPACE if workspace_bytes is less.
 * NA_ERR_SHAPE: page_size and the table's size as in na_cache_attention; kv_heads is below 1 or
 * requests * kv_heads reaches 2^20; budget is below 1, recent or capacity negative, one of
 * budget and num_free reaches 2^30, requests * kv_heads * capacity reaches 2^40; a page's bytes
 * reach 2^31; or new_head is head, new_context context_lens, new_weights weights, or v_pages
 * k_pages.
 */
size_t na_cache_evict_workspace(const na_evict_problem* problem);
na_status na_cache_evict(const na_evict_problem* problem, const float* weights,
                         const int32_t* context_lens, const int32_t* first,
                         const int32_t* page_table, const int32_t* head, int32_t* free_pages,
                         void* k_pages, void* v_pages, int32_t* new_context, float* new_weights,
                         int32_t* kept, int32_t* new_head, void* workspace,
                         size_t workspace_bytes, na_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* NA_SEQ_H_ */
