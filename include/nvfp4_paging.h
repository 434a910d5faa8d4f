/*
 * nvfp4_paging.h -- C ABI of serving over the paged 8-bit cache of
 * nvfp4_attention.h: the tables of a step made on the GPU from the requests'
 * lengths, the attention of batches whose sequences share prefixes, and the attention
 * over the pages that a cheap score selects for each query.
 *
 * Conventions are those of nvfp4_attention.h: device pointers owned by the
 * caller, synchronous checks before anything is enqueued, work enqueued on
 * ``stream``, no host synchronization, no allocation, safe from several host
 * threads.  Values in device memory are not checked on the host; the kernels
 * bound every access by the sizes given here.  Every function may be captured
 * into a graph.  Sizes for which a launch would have 2^32 work-items or more are
 * refused (NVFP4_EINVAL).
 */
#ifndef NVFP4_PAGING_H
#define NVFP4_PAGING_H

#include "nvfp4_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The sequences of a serving loop, their pages and the pool of free ones.
 *
 *   page_table   device int32 [n_seqs x max_pages], row stride
 *                page_table_stride >= max_pages entries: as in nvfp4_kv_batch.
 *   kv_len       device int32 [n_seqs]: tokens that a sequence holds (cut to
 *                [0, max_pages * page_size]).
 *   free_pages   device int32 [num_pages]: the free pages' numbers are its first
 *                free_count[0] entries, the last of them the next to be taken.
 *   free_count   device int32 [1] (cut to [0, num_pages]).
 * Requirements: 0 <= n_seqs < 2^24; page_size 16, 32, 64 or 128; 0 <= max_pages,
 * max_pages * page_size <= 2^30; 1 <= num_pages < 2^31; pointers 4-byte aligned.
 */
typedef struct nvfp4_requests {
  int32_t* page_table;
  int32_t* kv_len;
  int32_t* free_pages;
  int32_t* free_count;
  int64_t page_table_stride;
  int64_t max_pages;
  int64_t n_seqs;
  int64_t num_pages;
  int64_t page_size;
} nvfp4_requests;

/* Workspace bytes of nvfp4_step_tables; 0 if the arguments are invalid. */
size_t nvfp4_step_tables_workspace(int64_t n_seqs);

/*
 * A step's tables: for each sequence b, drop[b] tokens are taken off its end (those
 * of drafts that were rejected; all of them where a request has ended), then new_rows[b]
 * new ones come, with pages of the pool.  With p = page_size, held = kv_len[b] and
 * base = max(held - drop[b], 0):
 *   given back     entries ceil(max(base, kept[b]) / p) .. ceil(held / p) - 1 of the
 *                  sequence's row of page_table, pushed onto the pool one after the
 *                  other, sequences in order (those that no longer fit into it are
 *                  dropped: num_pages of them are free already);
 *   served         a sequence whose base + new_rows[b] tokens its row holds (one of
 *                  more gets no rows), up to the first for which the pool, after all
 *                  that is given back, has too few pages, or rows too few rows; from
 *                  it on nobody gets rows (drop[b] is taken off all the same);
 *   page_table     served sequences' new entries ceil(base / p) .. ceil((base +
 *                  new_rows[b]) / p) - 1: of the pages taken from the pool's end, in
 *                  the order in which they stand there, sequences in order;
 *   kv_len[b]      base, with the new rows of a served sequence; free_count;
 *   cu_rows        0, and the sums of the rows given: what nvfp4_kv_batch takes.
 *   positions      of each new row: its token's number in its sequence, and
 *   slots          page * p + position % p (-1 where the page is not one of num_pages).
 * Whole numbers, the same in every run; entries of free_pages behind its count keep
 * the pages that were taken.  A negative new_rows, drop or kept counts as 0.
 *
 *   new_rows     device int32 [n_seqs].
 *   drop         device int32 [n_seqs], or NULL: nothing is dropped.
 *   kept         device int32 [n_seqs], or NULL: tokens in front of each sequence
 *                whose pages are never given back (a prefix that others share).
 *   cu_rows      out, device int32 [n_seqs + 1].
 *   positions    out, device int32 [rows], or NULL.
 *   slots        out, device int64 [rows], or NULL.  positions and slots of rows from
 *                cu_rows[n_seqs] on are left as they are.
 *   rows         rows of the step's tensors, < 2^24.
 *   workspace    at least nvfp4_step_tables_workspace bytes, 8-byte aligned.  Its
 *                contents on entry do not matter; calls sharing one must be ordered.
 * Buffers do not overlap.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_step_tables(const nvfp4_requests* requests, const int32_t* new_rows, const int32_t* drop, const int32_t* kept,
                      int32_t* cu_rows, int32_t* positions, int64_t* slots, int64_t rows, void* workspace,
                      size_t workspace_bytes, void* stream);

/*
 * Groups of a step's sequences that share a prefix: sequences [cu_seqs[g],
 * cu_seqs[g + 1]) of the batch begin with the same prefix[g] tokens, in the same pages
 * (their rows of page_table agree that far).  Sequences in front of cu_seqs[0] or from
 * cu_seqs[n_groups] on are in no group.
 *
 *   cu_seqs      device int32 [n_groups + 1], not decreasing.
 *   prefix       device int32 [n_groups]: tokens.
 *   n_groups     0 <= n_groups <= n_seqs.
 *   max_prefix   the largest prefix, and
 *   max_own      the largest number of tokens of a sequence behind its prefix, as far as
 *                the host knows them: work is divided by them (larger ones are computed
 *                all the same, with less of them side by side).
 */
typedef struct nvfp4_shared_prefix {
  const int32_t* cu_seqs;
  const int32_t* prefix;
  int64_t n_groups;
  int64_t max_prefix;
  int64_t max_own;
} nvfp4_shared_prefix;

/* Workspace bytes of nvfp4_kv_attention_shared (partial results); 0: none is used, or
 * the arguments are invalid. */
size_t nvfp4_kv_attention_shared_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch,
                                           const nvfp4_shared_prefix* shared, int64_t q_heads);

/*
 * nvfp4_kv_attention (without a window) of a batch whose sequences share prefixes: the
 * same result, with each prefix read once for all sequences of its group.  A sequence
 * shares where all its rows lie behind the prefix (kv_len[b] - n_b >= prefix[g]); the
 * prefix is then read through the row of page_table of the group's first sequence that
 * does.  A sequence that does not, one that is empty for instance, is computed over its
 * own row of page_table alone.  Accuracy: as stated there, for each of the two parts.
 *
 * Steps for which sharing is taken to be slower by their sizes take the kernels of
 * nvfp4_kv_attention, for all of their sequences: those whose max_prefix is below 1536, and
 * those with 64 packed rows (new rows times q_heads / kv_heads) and more for each sequence
 * on the average, be they one prompt's among single tokens.
 *
 *   workspace, workspace_bytes   at least nvfp4_kv_attention_shared_workspace bytes,
 *                16-byte aligned (NULL if that is 0).  Its contents on entry do not
 *                matter; calls sharing one must be ordered.
 * The others, and the requirements, as for nvfp4_kv_attention.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_attention_shared(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_shared_prefix* shared,
                              const void* q, int64_t ldq, int64_t q_heads, void* y, int64_t ldy, float* lse,
                              float softmax_scale, int causal, void* workspace, size_t workspace_bytes, void* stream);

/* Which kernels nvfp4_kv_attention_shared launches for a step: as nvfp4_kv_attention_kernel. */
const char* nvfp4_kv_attention_shared_kernel(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch,
                                             const nvfp4_shared_prefix* shared, int64_t q_heads, int part);

/*
 * Bounds of the keys of a cache's pages, in 8 bits: page p and head h hold 2 * head_dim
 * bytes at codes + p * page_stride + h * 2 * head_dim,
 *   codes[0][e] = rint(127 hi_e / A),  codes[1][e] = rint(127 lo_e / A)   (to nearest even)
 *   step[p * step_stride + h] = fl(fl(A * k_scale) / 127)
 * with hi_e, lo_e the largest and the smallest E4M3 value of element e among the page's
 * page_size tokens (NaN codes left out; 0 where there are no others), A the largest |hi_e|,
 * |lo_e| of the head (all 0 if A is), fl binary32.
 * Requirements: codes 16-byte aligned, int8 [num_pages]; page_stride in bytes, a
 * multiple of 16, at least 2 * kv_heads * head_dim; step float [num_pages], 4-byte aligned,
 * step_stride >= kv_heads; strides below 2^31.
 */
typedef struct nvfp4_kv_bounds {
  void* codes;
  float* step;
  int64_t page_stride;
  int64_t step_stride;
} nvfp4_kv_bounds;

/*
 * The bounds of the pages that a step's rows completed: for each sequence the pages that
 * one of its new rows lies in and that its kv_len[b] tokens fill.  Called behind the append
 * of every step, it keeps the bounds of all full pages; those of other pages stay as they are.
 * Errors: NVFP4_EINVAL, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_page_bounds(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_kv_bounds* bounds,
                         void* stream);

/* Workspace bytes of nvfp4_kv_select_pages; 0: none is used, or the arguments are
 * invalid. */
size_t nvfp4_kv_select_pages_workspace(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch);

/*
 * Chooses up to `count` pages for each row of a step and each key head, of the pages
 * 0 .. n - 1 of the row's sequence that it sees (n = t / page_size + 1 for the row's token
 * t; if not causal, t is the sequence's last token): all of them if n <= count; else the
 * `first` ones, the `recent` last ones and, of those between them, the count - first -
 * recent with the largest scores, the lowest ones first among equals.  With key head h's
 * query heads a,
 *   q_a,e in 8 bits: i_a,e = rint(127 q_a,e / Q_a) (to nearest even),  Q_a = max_e |q_a,e|
 *   score = fl(max_a fl(fl(Q_a / 127) * sum_e max(i_a,e hi_e, i_a,e lo_e)) * step)
 * with hi_e, lo_e the page's bounds (codes): but for the 8-bit roundings, the largest
 * product that a query of the head can have with a key of the page.  (The softmax scale
 * is taken to be positive.)  The sums are whole numbers, so that the choice is the same
 * in every run.  A query head that has an infinity or a NaN among its elements is left out
 * of the maximum; a score that is no number (of a page for which no head is left, too)
 * counts as -infinity.  A page outside [0, num_pages) is chosen last.
 *
 *   index        out, device int32 [rows x kv_heads x count]: the chosen pages' numbers in
 *                their sequence, ascending; -1 behind them.
 *   pages        out, the same of the pages themselves (entries of page_table).
 *   tokens       out, device int32 [rows]: tokens of the chosen pages that the row sees
 *                (all of them, but t % page_size + 1 of the last); -1 for rows from
 *                cu_rows[n_seqs] on, whose index and pages are left as they are.
 *   first, recent   first >= 0, recent >= 1, first + recent <= count.
 *   workspace, workspace_bytes   at least nvfp4_kv_select_pages_workspace bytes, 16-byte
 *                aligned (NULL if that is 0).  Its contents on entry do not matter; calls
 *                sharing one must be ordered.
 * Requirements: those of the structures; q as for nvfp4_kv_attention; 1 <= count, count *
 * page_size <= 2^30; a batch that has rows has sequences; rows * kv_heads < 2^22, and with
 * max_pages over 8192 and over count rows * kv_heads * ceil(max_pages / 1024) < 2^24.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_select_pages(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_kv_bounds* bounds,
                          const void* q, int64_t ldq, int64_t q_heads, int64_t count, int64_t first, int64_t recent, int causal,
                          int32_t* index, int32_t* pages, int32_t* tokens, void* workspace, size_t workspace_bytes,
                          void* stream);

/* Workspace bytes of nvfp4_kv_attention_selected (partial results); 0: none is used, or
 * the arguments are invalid. */
size_t nvfp4_kv_attention_selected_workspace(const nvfp4_kv_cache* cache, int64_t rows, int64_t q_heads, int64_t count);

/*
 * Attention of each row over its chosen pages: of nvfp4_kv_attention's definition, with
 * the sums over the first tokens[row] tokens of pages[row][h][0 .. count - 1], one page
 * behind the other.  A row without tokens gets y = 0 and lse = -infinity; one whose
 * tokens are below 0 is left as it is.  tokens over count * page_size count as that;
 * tokens of pages outside [0, num_pages) are masked.
 *   pages, tokens   as nvfp4_kv_select_pages leaves them, or a caller's own choice.
 *   workspace, workspace_bytes   at least nvfp4_kv_attention_selected_workspace bytes,
 *                16-byte aligned (NULL if that is 0).  Its contents on entry do not
 *                matter; calls sharing one must be ordered.
 * The others, their requirements and the accuracy: as for nvfp4_kv_attention.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_attention_selected(const nvfp4_kv_cache* cache, const void* q, int64_t ldq, int64_t q_heads, int64_t rows,
                                int64_t count, const int32_t* pages, const int32_t* tokens, void* y, int64_t ldy, float* lse,
                                float softmax_scale, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NVFP4_PAGING_H */
