/*
 * sim_kv.h - paged key/value cache and attention over shared prefixes (libsim.so, CUDA, sm_103a).
 *
 * The schedulers of sim.h count a worker's KV cache in tokens: a request holds s_i + (tokens generated)
 * of the M that fit (arXiv 2508.14544, eq. constraintM), a cancellation gives them back, a completion
 * too.  These calls are that memory on the GPU, in pages, and the operator that reads it, so that the
 * batches of a schedule can be run and timed (the coefficients of sim_batch_time are the caller's).
 *
 * Layout.  A cache is four arrays of the caller in DEVICE memory:
 *   pool    [n_pages][n_layers][2: keys, values][n_kv_heads][page_size][head_dim], 16-bit floats,
 *   table   int32 [max_seqs][max_pages]: the pages of each sequence in order, -1 where there is none,
 *   length  int32 [max_seqs]: tokens of each sequence (0: none),
 *   ref     int32 [n_pages]: sequences that hold the page; 0 means free.
 * Sequence i holds ceil(length[i] / page_size) pages.  A page may be held by several sequences (sim_kv_fork);
 * tokens are only ever added to a page with one holder: a shared last page is copied first.  Pages are
 * given out lowest number first, in the order of the call's entries, so results are deterministic.
 *
 * Calls.  All arguments described as DEVICE are read when the work runs.  Every call only enqueues work on
 * `cuda_stream` (a cudaStream_t of the current device, or NULL for the default stream), allocates nothing
 * and may be captured into a graph.  Host-side argument errors return SIM_E_INVAL with a message in
 * sim_last_error(NULL).  What only the device can see is reported in kv->status[0], which keeps the most
 * negative code until the caller clears it: an entry that is out of range, repeated or refused
 * (SIM_E_INVAL) is left out and the other entries take effect; a sim_kv_extend or sim_kv_copy that needs
 * more free pages than there are (SIM_E_NOMEM), or whose offsets are not in order (SIM_E_INVAL), changes
 * nothing.  SIM_E_STATE: a block of sim_kv_attend gave up a wait (nothing moved for a second, which no input should
 * cause); results that it had not written yet are left as they were.  Calls on one cache belong on one stream at a time
 * (they share kv->scratch).
 */
#ifndef SIM_KV_H_
#define SIM_KV_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SIM_KV_BF16 = 0, SIM_KV_F16 = 1 } sim_kv_dtype;

typedef struct {
    void *pool;       /* DEVICE, 16-byte aligned */
    int32_t *table;   /* DEVICE */
    int32_t *length;  /* DEVICE */
    int32_t *ref;     /* DEVICE, 16-byte aligned */
    int32_t *status;  /* DEVICE, one int32, 0 at first */
    void *scratch;    /* DEVICE, 16-byte aligned, sim_kv_scratch_bytes bytes */
    int32_t dtype;      /* sim_kv_dtype */
    int32_t n_pages;    /* 1 .. 2^28 */
    int32_t n_layers;   /* >= 1 */
    int32_t n_kv_heads; /* >= 1 */
    int32_t page_size;  /* tokens: 16, 32, 64 or 128 */
    int32_t head_dim;   /* a multiple of 8, 8 .. 128 */
    int32_t max_seqs;   /* 1 .. 2^17 */
    int32_t max_pages;  /* pages per sequence, >= 1, max_pages * page_size < 2^30 (2^37 / n_kv_heads) */
} sim_kv;

/* sim_kv_scratch_bytes: size of kv->scratch (the pointers of *kv are not read); 0 for bad sizes. */
int64_t sim_kv_scratch_bytes(const sim_kv *kv);

/*
 * sim_kv_extend: room for new tokens at the end of sequences.
 *   n        entries, 0 .. max_seqs;  seqs  DEVICE int32 [n], distinct.
 *   cu_new   DEVICE int32 [n + 1], non-decreasing: entry i gets cu_new[i + 1] - cu_new[i] tokens.
 *   n_new    tokens in all, at least cu_new[n].
 *   slots    DEVICE int64 [n_new]: page * page_size + position in the page of each new token, -1 for
 *            tokens of no valid entry.
 * length grows, full pages are followed by new ones, and a last page that other sequences hold too and
 * that has room is replaced by a copy (all layers).  An entry past max_pages is refused (SIM_E_INVAL).
 */
int sim_kv_extend(const sim_kv *kv, int32_t n, const int32_t *seqs, const int32_t *cu_new, int32_t n_new,
                  int64_t *slots, void *cuda_stream);

/*
 * sim_kv_write: keys and values of one layer into the slots of sim_kv_extend.
 *   k, v     DEVICE [n_new][n_kv_heads][head_dim] of kv->dtype; strides in elements between tokens and
 *            between heads, the last dimension contiguous; any alignment of the type.
 * Slots outside the pool are skipped.
 */
int sim_kv_write(const sim_kv *kv, int32_t layer, int32_t n_new, const int64_t *slots, const void *k,
                 int64_t k_token_stride, int64_t k_head_stride, const void *v, int64_t v_token_stride,
                 int64_t v_head_stride, void *cuda_stream);

/*
 * sim_kv_fork: dst[i] becomes the first tokens[i] tokens of src[i] (all of them if `tokens` is NULL) and
 * holds the same pages.  dst: distinct, empty (length 0), and not a src of the same call.
 */
int sim_kv_fork(const sim_kv *kv, int32_t n, const int32_t *src, const int32_t *dst, const int32_t *tokens,
                void *cuda_stream);

/* sim_kv_copy: like sim_kv_fork of whole sequences, with pages of its own for each dst. */
int sim_kv_copy(const sim_kv *kv, int32_t n, const int32_t *src, const int32_t *dst, void *cuda_stream);

/*
 * sim_kv_free: seqs[i] keeps its first keep[i] tokens (none if `keep` is NULL; at most its length) and
 * gives the other pages back; a page becomes free with its last holder.
 */
int sim_kv_free(const sim_kv *kv, int32_t n, const int32_t *seqs, const int32_t *keep, void *cuda_stream);

/*
 * sim_kv_compact: move pages so that those in use are the lowest-numbered: the i-th used page above their
 * number goes to the i-th free one below it, and every table is rewritten.
 *   to       DEVICE int32 [n_pages]: the new number of each page, -1 where it was free.
 */
int sim_kv_compact(const sim_kv *kv, int32_t *to, void *cuda_stream);

/* The queries of one batch: entry i has the query tokens cu_q[i] .. cu_q[i + 1] - 1, which are the last
 * tokens of sequence seqs[i] (already in the cache); a query sees the keys up to its own position. */
typedef struct {
    int32_t n;                /* entries, 0 .. 2^17, n * n_kv_heads <= 2^26 (an entry may have no queries, a sequence may repeat) */
    int32_t n_q;              /* query tokens in all, n_q * q_heads <= 2^30 */
    int32_t q_heads;          /* a multiple of n_kv_heads: query head h reads kv head h / (q_heads / n_kv_heads) */
    int32_t n_groups;         /* 0: none */
    const int32_t *seqs;      /* DEVICE [n] */
    const int32_t *cu_q;      /* DEVICE [n + 1], non-decreasing, 0 .. n_q */
    const int32_t *cu_group;  /* DEVICE [n_groups + 1], from 0 to n: entries that may share a prefix, or NULL */
    void *plan;               /* DEVICE, 16-byte aligned, sim_kv_plan_bytes bytes */
    void *workspace;          /* DEVICE, 16-byte aligned, sim_kv_workspace_bytes bytes */
} sim_kv_batch;

int64_t sim_kv_plan_bytes(const sim_kv *kv, const sim_kv_batch *b);
int64_t sim_kv_workspace_bytes(const sim_kv *kv, const sim_kv_batch *b);

/*
 * sim_kv_plan: divide the batch's attention among the SMs, for any number of sim_kv_attend calls (one per
 * layer) until lengths, tables or the batch change.  In each group the pages that every entry's table
 * begins with, as far as all its queries see them whole, are found by comparing the tables: they are read once for
 * all of the group's queries, where that saves work.  Groups change the time, never what is computed.  An
 * entry whose sequence is out of range sees no keys; with offsets that are not in order no query does (both
 * SIM_E_INVAL in kv->status).
 */
int sim_kv_plan(const sim_kv *kv, const sim_kv_batch *b, void *cuda_stream);

/*
 * sim_kv_attend: softmax(scale q k^T) v over the cached keys that each query sees, for one layer.
 *   q        DEVICE [n_q][q_heads][head_dim] of kv->dtype, strides in elements, last dimension contiguous.
 *   out      the same shape and type, strides multiples of 8, 16-byte aligned.
 *   lse      DEVICE float [n_q][q_heads], or NULL: log of the sum of the exponentials.
 *   scale    > 0, finite, also times log2(e).
 * A query that sees no key gets zeros, and -infinity for lse.  Cached values past a sequence's length are
 * never used, whatever they are, nor are those that a query does not see.  Sums and the softmax are in 32 bits, those
 * of the products (which cut off what does not fit) over 2^15 keys at most; the probabilities are rounded to kv->dtype for
 * the product with the values.
 */
int sim_kv_attend(const sim_kv *kv, const sim_kv_batch *b, int32_t layer, const void *q, int64_t q_token_stride,
                  int64_t q_head_stride, float scale, void *out, int64_t out_token_stride, int64_t out_head_stride,
                  float *lse, void *cuda_stream);

#ifdef __cplusplus
}
#endif

#endif /* SIM_KV_H_ */
