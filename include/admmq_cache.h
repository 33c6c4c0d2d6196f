/*
 * admmq_cache.h -- a cache of keys and values in 8 bits, and attention over it (B200, sm_100a).
 *
 * What the projections, adapters, norm and rotation of admmq_adapt.h leave of a token, its keys and values, is kept here
 * for the tokens that come after it: written as rows come, read back, and attended over by one new token of a request,
 * by a few, or by a prompt.
 *
 * The conventions of admmq_adapt.h hold: device pointers, nothing allocated, asynchronous, argument errors returned at
 * once with nothing enqueued, errors met on the device raised in d_status, sums in fp32, every call can be captured.
 */
#ifndef ADMMQ_CACHE_H_
#define ADMMQ_CACHE_H_

#include "admmq_adapt.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ADMMQ_CACHE_BLOCK 16          /* tokens that share the scale of a head */
#define ADMMQ_CACHE_MAX_HEAD 256
#define ADMMQ_CACHE_MAX_PAGE 256

/* ---- The cache -----------------------------------------------------------------------------------------
 * n_pages pages of page_size tokens (16, 32, 64, 128 or 256) for kv_heads heads of head_dim values (a multiple of 16, at
 * most 256).  16 neighbouring tokens of a page and head are a block; keys and values of a block have a scale each:
 *   value = scale * code,  code in [-127, 127],
 *   scale = (largest magnitude that the block was given) * (1 / 127) in fp32, code = round(x / scale) to nearest, ties to
 *   even.
 * Where rows that are added raise a block's scale from s to s', the codes it holds become round(code * (s / s')) (fp32).
 * A block whose first token is written starts anew, whatever it held.  One whose magnitudes all stay below 2^-40 is held
 * as zeros; one that was given a magnitude of 2^40 or more, an infinity or a NaN has scale NaN and is read as NaN, until
 * it starts anew.
 * d_codes: admmq_cache_code_bytes, d_scale: admmq_cache_scale_bytes, both in an order of the library's own, in which a
 * page is contiguous: pages may be copied whole.  They need not be initialised. */
typedef struct {
  size_t struct_size;      /* sizeof(admmq_cache) */
  int n_pages, kv_heads, head_dim, page_size;
  void* d_codes;
  float* d_scale;
} admmq_cache;
size_t admmq_cache_code_bytes(int n_pages, int kv_heads, int head_dim, int page_size);
size_t admmq_cache_scale_bytes(int n_pages, int kv_heads, int head_dim, int page_size);

/* ---- The rows of a call --------------------------------------------------------------------------------
 * Request i has lengths[i] adjacent rows, at its positions held[i] .. held[i] + lengths[i] - 1; its position p is token
 * p % page_size of page tables[i][p / page_size].  lengths are the host's, tables and held the device's (read when the
 * kernels run, so a captured call follows them).  A request with held < 0 takes no part: nothing of it is written, its
 * rows read as zero.  One that does not fit its table raises ADMMQ_ERR_SHAPE in d_status and takes no part either, and so
 * does a page outside [0, n_pages), which is not accessed.  tables and held may not change while a call runs.
 * d_index: int32 buffer of admmq_cache_plan_ints entries that admmq_cache_plan_fill fills on the host (no CUDA call is
 * made) and the caller copies to the device.  group: query heads a key head (for attend). */
typedef struct {
  size_t struct_size;      /* sizeof(admmq_cache_plan) */
  int n_requests, max_pages, group;
  int n_blocks;            /* admmq_cache_plan_fill sets these five */
  int n_small, n_big, small_rows;
  long long n_rows;
  const int* d_tables;     /* [n_requests][max_pages] */
  const int* d_held;       /* [n_requests] */
  const int* d_index;
} admmq_cache_plan;
long long admmq_cache_plan_ints(const long long* lengths, int n_requests, int group);
admmq_status admmq_cache_plan_fill(const long long* lengths, int n_requests, int group, int* index, admmq_cache_plan* plan);

/* ---- Writing and reading --------------------------------------------------------------------------------
 * k, v: [n_rows][kv_heads][head_dim] fp32 or bf16 by row and head strides (elements, inner stride 1; 16-byte aligned).
 * write: the plan's rows into the cache.  A page may be written through one entry of the tables only (else its contents are
 * unspecified); pages that requests only read may be shared.
 * read: what the cache holds at the plan's rows, as scale * code rounded to the given type; rows and heads may not overlap. */
admmq_status admmq_cache_write(const admmq_cache* cache, const admmq_cache_plan* plan, admmq_dtype dtype, const void* d_k,
                               long long k_row, long long k_head, const void* d_v, long long v_row, long long v_head,
                               int* d_status, void* cuda_stream);
admmq_status admmq_cache_read(const admmq_cache* cache, const admmq_cache_plan* plan, admmq_dtype dtype, void* d_k,
                              long long k_row, long long k_head, void* d_v, long long v_row, long long v_head, int* d_status,
                              void* cuda_stream);

/* ---- Attention ------------------------------------------------------------------------------------------
 * q, out: [n_rows][kv_heads * group][head_dim] bf16 by row and head strides (at most 65536 heads; those of out may not overlap, nor
 * out and q); query head h goes with key head h / group.
 * A row at position p sees the positions j <= p of its request that the cache holds (its own among them: write first),
 * with window > 0 those with j > p - window (pages with none of the positions that a request's rows see are not asked for,
 * so those that a window has left may be gone from the tables):
 *   out = sum_j w_j v_j,  w = softmax_j(scale q . k_j),  lse [n_rows][heads] fp32 = log sum_j exp(scale q . k_j)
 * in fp32 sums; weights (times their value scale) enter the second product as fp16, with 11 bits down to 2^-20 of the row's
 * largest at least, fewer down to 2^-31 and perhaps none below; queries as fp16 after a shift by a power of two of each row (exact for values
 * within 2^-27 of the row's largest; a query with an infinity or a NaN gives a row of NaN).  Requests
 * that take no part get out = 0 and lse = -inf.  d_lse may be NULL.  A block with scale NaN gives NaN to the rows that see
 * any of its tokens.
 * d_workspace: admmq_cache_attend_workspace bytes, not initialised; no two calls that may run at once share it. */
size_t admmq_cache_attend_workspace(const admmq_cache* cache, const admmq_cache_plan* plan);
admmq_status admmq_cache_attend(const admmq_cache* cache, const admmq_cache_plan* plan, double scale, int window,
                                const void* d_q, long long q_row, long long q_head, void* d_out, long long out_row,
                                long long out_head, float* d_lse, void* d_workspace, size_t workspace_bytes, int* d_status,
                                void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* ADMMQ_CACHE_H_ */
