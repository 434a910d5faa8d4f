/*
 * nvfp4_paging.h -- C ABI of serving over the paged 8-bit cache of
 * nvfp4_attention.h: the tables of a step made on the GPU from the requests'
 * lengths, and the attention of batches whose sequences share prefixes.
 *
 * Conventions are those of nvfp4_attention.h: device pointers owned by the
 * caller, synchronous checks before anything is enqueued, work enqueued on
 * ``stream``, no host synchronization, no allocation, safe from several host
 * threads.  Values in device memory are not checked on the host; the kernels
 * bound every access by the sizes given here.  Every function may be captured
 * into a graph.
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

/* Workspace bytes of nvfp4_kv_attention_shared (partial results); 0: the batch has no
 * rows, or the arguments are invalid. */
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
 *   workspace, workspace_bytes   at least nvfp4_kv_attention_shared_workspace bytes,
 *                16-byte aligned.  Its contents on entry do not matter; calls sharing
 *                one must be ordered.
 * The others, and the requirements, as for nvfp4_kv_attention.
 * Errors: NVFP4_EINVAL, NVFP4_EWORKSPACE, NVFP4_EUNSUPPORTED, NVFP4_EHIP.
 */
int nvfp4_kv_attention_shared(const nvfp4_kv_cache* cache, const nvfp4_kv_batch* batch, const nvfp4_shared_prefix* shared,
                              const void* q, int64_t ldq, int64_t q_heads, void* y, int64_t ldy, float* lse,
                              float softmax_scale, int causal, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* NVFP4_PAGING_H */
