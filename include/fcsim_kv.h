/*
 * fcsim_kv -- the paged key-value cache of one layer on the device: append, attend, prefill, evict, read.
 *
 * The simulator (fcsim.h) counts tokens of KV cache per slot; these operators are what a slot does to a real
 * cache.  A cache is a pool of n_pages pages of page_size tokens; a request owns pages through a row of a table
 * (entry i holds tokens i * page_size ..).  Token rows are [n_kv_heads][head_dim].
 *
 *   append   y = norm(x) rotated by position, for every head of q and k; q is returned, k and v go into the cache.
 *   attend   one query token per request: o = sum_t softmax_t(scale q . k_t) v_t over the request's cached tokens;
 *            optionally each token's weight grows by the attention it received (summed over the query heads that
 *            share its kv head).
 *   prefill  the same for several query tokens per request, each of which sees the tokens up to its own: a prompt, or a chunk of one.
 *   evict    per request and kv head: the oldest `first`, the newest `recent` and, of the rest, the largest
 *            weights are kept up to a budget; the kept rows move in order, with their weights, to other pages.
 *   read     the values that stand at given slots, as 16-bit rows: what append has stored, for another cache or for the eye.
 *
 * (The paper of fcsim.h has no counterpart: it counts tokens and evicts whole requests.)
 *
 * Conventions are those of fcsim.h: every function returns 0 (FCSIM_OK) or a negative code and nothing throws, aborts
 * or traps.  All pointers inside the structs are DEVICE pointers except the structs themselves; buffers are the
 * caller's.  Launches are asynchronous on `cuda_stream` (a cudaStream_t; NULL = default stream) of the current device
 * and may be captured in a graph.  No state is kept between calls.  Strides are in elements; the innermost dimension
 * (head_dim) is contiguous; addresses and strides of q, k, v and of the cache must be multiples of 16 bytes.
 *
 * What only the device can see (page numbers, lengths, positions) is checked there: a bad value never reads or
 * writes outside the buffers, its effect is stated below, and a bit is set in *status (int32, may be NULL; never
 * cleared by the library).
 */
#ifndef FCSIM_KV_H
#define FCSIM_KV_H

#include "fcsim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types.  E4M3 (8 bits, largest value 448) is for caches only. */
enum { FCSIM_KV_F16 = 0, FCSIM_KV_BF16 = 1, FCSIM_KV_E4M3 = 2 };

enum { /* bits of *status */
    FCSIM_KV_BAD_PAGE = 1,     /* page or slot outside the pool: its tokens are left out (evict: see there) */
    FCSIM_KV_BAD_LENGTH = 2,   /* length < 0 (taken as 0) or > max_length (taken as max_length) */
    FCSIM_KV_BAD_POSITION = 4, /* position outside the rope table: q_out row zero, nothing stored */
    FCSIM_KV_BAD_BUDGET = 8,   /* budget < 0 (taken as 0) or > max_budget (taken as max_budget) */
    FCSIM_KV_STUCK = 16        /* a wait inside a kernel took seconds and was given up: the call's results are wrong, and its workspace
                                  has to be cleared again before it is used */
};

/* head_dim: a multiple of 8 (16-bit caches) or 16 (E4M3), at most 256.  k and v have the same strides.
 * n_pages * page_size is below 2^31, n_kv_heads at most 65535.
 * weight: [n_pages][n_kv_heads][page_size] fp32, contiguous, 16-byte aligned, or NULL.
 * k_scale, v_scale: [n_kv_heads] fp32 of either sign, E4M3 only (else NULL): a stored value x stands for x * scale. */
typedef struct {
    void* k;
    void* v;
    float* weight;
    const float* k_scale;
    const float* v_scale;
    int64_t stride_page, stride_slot, stride_head;
    int32_t dtype, n_pages, page_size, n_kv_heads, head_dim;
    int32_t reserved;
} fcsim_kv_cache;

/* n tokens; token i of q at q + i * q_row + head * q_head.  `dtype` (F16 or BF16) is that of q, k, v, q_out and the
 * norm weights; a 16-bit cache must have the same.
 * q_norm, k_norm: [head_dim], or NULL = that norm is left out.  x <- x / sqrt(mean(x^2) + eps) * w over each head.
 * rope: fp32 [n_positions][rope_dim], the cosines of the rope_dim / 2 angles, then their sines; NULL = no rotation.
 *   The first rope_dim elements of a head turn in pairs: (i, i + rope_dim / 2) (rope_dim a multiple of 16, the table 16-byte
 *   aligned), or with
 *   `interleaved` (2i, 2i + 1) (rope_dim even); the others pass.
 * positions: [n] int32 (unused without rope).  slots: [n] int64 = page * page_size + place, negative = not stored.  No two tokens
 *   of a call may have the same slot.
 * q_out: [n][n_heads][head_dim] contiguous.  n_heads = 0: q, q_norm, q_out are not used.
 * The weights of the slots written are set to 0.  All arithmetic in fp32, one rounding at the end; values beyond
 * E4M3's range are stored as +-448.  n_tokens is at most 2^31 - 2^16. */
typedef struct {
    const void *q, *k, *v;
    void* q_out;
    const void *q_norm, *k_norm;
    const float* rope;
    const int32_t* positions;
    const int64_t* slots;
    int32_t* status;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head;
    int32_t n_tokens, n_heads, dtype, rope_dim, n_positions, interleaved;
    float eps;
    int32_t reserved;
} fcsim_kv_append_args;

int fcsim_kv_append(const fcsim_kv_cache* cache, const fcsim_kv_append_args* args, void* cuda_stream);

/* table: [n_requests] rows of table_cols int32, row r at table + r * table_row; only the entries that a request's
 *   length reaches are read.  lengths: [n_requests] int32 tokens held, 0 .. max_length <= table_cols * page_size.
 * window > 0: only the newest `window` tokens are seen, and the oldest `first` (without a window `first` has no effect).
 *   n_heads: a multiple of n_kv_heads; head h reads kv head h / (n_heads / n_kv_heads).  q: request r at q + r * q_row +
 *   head * q_head, F16 or BF16, that of a 16-bit cache.  (Of a BF16 query over E4M3, elements below 2^-31 of the head's
 *   largest finite one are rounded to 2^-38 of it.)
 * Sums over tokens are the tensor core's: in 32 bits, cut off, up to 2^-23 of the sum lost at each of 16 to 24 additions per
 *   128 tokens of one warp's share.
 * out: [n_requests][n_heads][head_dim] contiguous, in q's type.  lse: [n_requests][n_heads] fp32, the natural
 *   logarithm of the softmax sums, or NULL.  A request without tokens gives zeros and -infinity.
 * add_weight: cache->weight[token] += the softmax weights, summed over the heads of its group.  The requests of such
 *   a call must not share pages.
 * workspace: 16-byte aligned, of the size fcsim_kv_attend_workspace reports; its first `zeroed` bytes (the same for all
 *   calls) must be zero before the first call and are zero again after every call.  Calls that share it must be ordered;
 *   they may differ in everything else.
 * At most 65535 requests, n_requests * max_length below 2^36, max_length at most 2^31 - 2^16 and n_heads * head_dim below 2^31
 * (FCSIM_EINVAL).
 * The struct has no size or version in it: `first` and `reserved` stand behind what it held before there were first tokens, so what
 * was compiled against a header without them has to be compiled again. */
typedef struct {
    const void* q;
    void* out;
    float* lse;
    const int32_t* table;
    const int32_t* lengths;
    int32_t* status;
    int64_t q_row, q_head, table_row;
    int32_t n_requests, n_heads, dtype, table_cols, max_length, window, add_weight;
    float scale;
    int32_t first, reserved;
} fcsim_kv_attend_args;

typedef struct {
    size_t bytes, zeroed;
} fcsim_kv_workspace;

int fcsim_kv_attend_workspace(const fcsim_kv_cache* cache, const fcsim_kv_attend_args* args, fcsim_kv_workspace* out);
int fcsim_kv_attend(const fcsim_kv_cache* cache, const fcsim_kv_attend_args* args, void* workspace,
                    size_t workspace_bytes, void* cuda_stream);

/* q: n_rows rows, row i at q + i * q_row + head * q_head, F16 or BF16, that of a 16-bit cache.  Request r has the rows starts[r] ..
 * starts[r + 1] - 1 (starts: [n_requests + 1] int32, not falling, 0 .. n_rows): the newest of its lengths[r] tokens, which are all in
 * the cache already.  A row whose token is number p sees the tokens t <= p, with window > 0 only those of t > p - window or
 * t < first (without a window `first` has no effect).  n_heads: a multiple of n_kv_heads; head h reads kv head
 * h / (n_heads / n_kv_heads).  table, lengths, max_length, workspace: as for attend (one workspace serves both).  The cache's
 * weights do not grow by it.
 * out: [n_rows][n_heads][head_dim] contiguous, in q's type.  lse: [n_rows][n_heads] fp32, or NULL.  A row that sees nothing, or
 * belongs to no request, gives zeros and -infinity.  What a row does not see may hold anything, infinities and NaN too.
 * Rounding: a softmax weight meets v in two 16-bit parts, off by up to 2^-14 (BF16) or 2^-20 (F16) of it.  Those of F16 queries are
 * multiples of 2^-38 of the row's largest; of BF16 queries and a 16-bit cache, values below 2^-94 lose bits.  Sums over tokens
 * are the tensor core's, in 32 bits, cut off: up to 2^-12 of an output, whatever its length.
 * starts beyond 0 .. n_rows are taken as these ends, rows that two requests claim hold either's output, a request of more rows than
 * tokens has rows that see nothing (FCSIM_KV_BAD_LENGTH for either).  n_rows and max_length are at most 2^31 - 2^16, n_requests
 * 65535, n_heads * head_dim below 2^31. */
typedef struct {
    const void* q;
    void* out;
    float* lse;
    const int32_t* starts;
    const int32_t* table;
    const int32_t* lengths;
    int32_t* status;
    int64_t q_row, q_head, table_row;
    int32_t n_rows, n_requests, n_heads, dtype, table_cols, max_length, window, first;
    float scale;
    int32_t reserved;
} fcsim_kv_prefill_args;

int fcsim_kv_prefill_workspace(const fcsim_kv_cache* cache, const fcsim_kv_prefill_args* args, fcsim_kv_workspace* out);
int fcsim_kv_prefill(const fcsim_kv_cache* cache, const fcsim_kv_prefill_args* args, void* workspace,
                     size_t workspace_bytes, void* cuda_stream);

/* Request r keeps n' = min(length, budget[r]) tokens: the newest min(recent, budget), of what is left the oldest
 * min(first, budget - recent), then the largest weights (equal weights: the oldest first; NaN counts as the lowest,
 * and -0 as 0).  Kept tokens stay in order: token i of the new request is row kept[r][h][i] of the old one.  They are
 * copied with their weights to new_table's pages, which must not be among the pages read by the call.  Tokens of a page
 * outside the pool rank as NaN does; those that are kept become zeros of weight 0, and rows for one are not written.
 * new_lengths: [n_requests] int32.  kept: [n_requests][n_kv_heads][max_budget] int32, -1 beyond n'.
 * budget: [n_requests] int32, 0 .. max_budget <= new_cols * page_size.  Needs cache->weight.  At most 65535 requests; max_length
 * and max_budget are at most 2^31 - 2^16.
 * workspace: none is needed at present; fcsim_kv_evict_workspace reports {0, 0}, and NULL will do. */
typedef struct {
    const int32_t* table;
    const int32_t* lengths;
    const int32_t* budget;
    const int32_t* new_table;
    int32_t* new_lengths;
    int32_t* kept;
    int32_t* status;
    int64_t table_row, new_row;
    int32_t n_requests, table_cols, new_cols, max_length, max_budget, recent, first;
    int32_t reserved;
} fcsim_kv_evict_args;

int fcsim_kv_evict_workspace(const fcsim_kv_cache* cache, const fcsim_kv_evict_args* args, fcsim_kv_workspace* out);
int fcsim_kv_evict(const fcsim_kv_cache* cache, const fcsim_kv_evict_args* args, void* workspace,
                   size_t workspace_bytes, void* cuda_stream);

/* k_out, v_out: [n_tokens][n_kv_heads][head_dim] contiguous in `dtype` (F16 or BF16, whatever the cache's type), 16-byte aligned.  Row i
 * is what stands at slots[i] (int64, page * page_size + place), an E4M3 value as its fp32 product with its scale, rounded to `dtype`; negative: zeros.
 * A slot outside the pool gives zeros (FCSIM_KV_BAD_PAGE).  A slot may come more than once.  n_tokens is at most 2^31 - 2^16. */
typedef struct {
    const int64_t* slots;
    void *k_out, *v_out;
    int32_t* status;
    int32_t n_tokens, dtype;
} fcsim_kv_read_args;

int fcsim_kv_read(const fcsim_kv_cache* cache, const fcsim_kv_read_args* args, void* cuda_stream);

/* cudaError_t behind the last FCSIM_ECUDA of these functions on the calling thread, else 0. */
int fcsim_kv_last_cuda_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FCSIM_KV_H */
