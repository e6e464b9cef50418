/* earlytom_pages.h -- what a server around the decode step of earlytom_decode.h needs on the device, so that a step can be
 * captured into a CUDA graph and replayed while conversations grow, end and branch: pages of the cache handed out and taken back, and
 * beam search, whose beams share pages.  No counterpart in the paper.
 *
 * Conventions are those of earlytom_decode.h: caller-owned device buffers of the current device, asynchronous on cuda_stream, no
 * allocation, no synchronisation, capturable; shapes are checked on the host and refused with an et_status before anything is
 * launched; contents of device arrays are checked by the kernels, skipped where they cannot be used, and reported in status_dev (int,
 * may be NULL, set to 0 by the caller; a larger value stays).  Buffers that a call writes overlap no other buffer of it unless it
 * is said.
 *
 * The state: refs_dev int [n_pages], for each page of the cache how many entries of block tables (and whatever else its owner counts)
 * name it; a page is free if its count is 0.  block_table_dev int [n_seq][max_pages] as in earlytom_decode.h; a sequence of len
 * positions uses its first ceil(len / page_size) entries.  All layers' caches share the tables and the counts.  One step of beam
 * search, for n sequences:
 *
 *   et_pages_update (a place for one more token each) -> the layers of earlytom_decode.h (et_kv_append at the lengths before,
 *   et_attention_paged with the lengths after) -> et_linear_rows (output head) -> et_beam_select -> et_pages_fork -> et_kv_copy for
 *   each layer
 *
 * Pages are taken in ascending order of their numbers, by sequences in ascending order: the result depends on the state alone. */
#ifndef EARLYTOM_PAGES_H
#define EARLYTOM_PAGES_H

#include "earlytom_decode.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Values of status_dev beside those of earlytom_decode.h: no page was free; a count would have become negative; a parent is no row. */
enum { ET_PAGED_NO_PAGE = 6, ET_PAGED_BAD_COUNT = 7, ET_PAGED_BAD_ROW = 8 };

/* Sequences give positions back and get new ones.  Sequence s holds len_dev[s] positions (negative: the slot is not in use), keeps
 * the first keep_dev[s] of them (at most those that it holds; negative: it keeps none and leaves the slot; NULL: all) and gets
 * add_dev[s] more behind (negative counts as 0; NULL: one each).  A slot that is not in use comes into use with keep_dev[s] >= 0.
 *
 * Entries behind the kept positions, ceil(keep / page_size) .. ceil(len / page_size) - 1, are given back: their pages' counts go down
 * by one and the entries become -1.  Then entries up to ceil((keep + add) / page_size) - 1 are taken: free pages (those that have just
 * become free among them), whose counts become 1.  The taken pages are numbered by sequence, then by entry; the i-th is the free page
 * with i smaller ones.  A sequence whose last one there is no free page for gets no position (status ET_PAGED_NO_PAGE; its entries
 * become -1), nor does one whose positions the table cannot hold (ET_PAGED_CAPACITY; it takes no pages).  The numbers of pages that
 * were not to be had are not given to the sequences behind: those that need a page get none either, so one request for more than
 * there is belongs into a call of its own, or behind the others.
 *
 * The new positions begin in the last kept page if that one is not full, and then it has to be the sequence's own: nothing is copied and
 * no other page taken in its place, so two sequences that hold it would get the same places in it, and no status says so.  Where others
 * hold it too (a beginning in common that ends inside a page, positions given back into pages that are shared) et_pages_fork gives
 * each row one of its own: et_pages_update with add = 0, et_pages_fork with each row its own parent, et_kv_copy, then the new positions.
 *
 * new_len_dev [n_seq] (may be len_dev): keep + add, keep where it got none, -1 where the slot is not in use.
 * row_offsets_dev [n_seq + 1] (may be NULL): where the new positions' rows stand when they are packed in the order of the sequences,
 * the exclusive sum of what was asked for, whether it was got or not; et_kv_append takes it with the kept lengths as its start, and with
 * a negative start for a sequence that got none: its rows would go through the entries behind the used ones, whatever those name.
 * slots_dev [rows] (may be NULL with rows = 0): for each of these rows page * page_size + place, the place of its position in the
 * cache, or -1 for a position that was not got and for rows behind the last; rows more than that are left out (ET_PAGED_CAPACITY).
 *
 * A given-back entry that is no page is skipped (ET_PAGED_BAD_PAGE), a count that is not above 0 stays (ET_PAGED_BAD_COUNT).
 * workspace_dev: ET_PAGES_WORKSPACE(n_pages, n_seq) bytes, 16-byte aligned, contents neither needed nor kept; one call at a time.
 * Limits (ET_ERR_CAPACITY): n_pages * page_size < 2^31, max_pages * page_size <= 2^30, n_seq <= 65536, n_seq * max_pages < 2^31.  The
 * sums of what is asked for have to stay below 2^31: beyond that row_offsets and slots hold any values, while tables, counts and lengths
 * stay right. */
#define ET_PAGES_WORKSPACE(n_pages, n_seq) (4ull * (n_pages) + 8ull * (n_seq))
ET_API et_status et_pages_update(int* refs_dev, int n_pages, int page_size, int* block_table_dev, int n_seq, int max_pages,
                                 const int* len_dev, const int* keep_dev, const int* add_dev, int* new_len_dev, int* row_offsets_dev,
                                 int* slots_dev, int rows, void* workspace_dev, size_t workspace_bytes, int* status_dev,
                                 void* cuda_stream);

/* Rows of the new table follow rows of the old one: row b of new_table_dev [n_new][max_pages] continues row parent_dev[b] of
 * block_table_dev [n_old][max_pages] with its len_dev positions (negative, or no row of the old table, ET_PAGED_BAD_ROW: the slot
 * is not in use).  The old rows end with the call.  A row's used entries are copied, its others left as they were; a page's count follows
 * the entries that name it.
 *
 * Rows write into their last page as they grow, so a last page that is not full belongs to one row: the first of a parent's rows
 * keeps it if nobody but this parent's rows holds it; each other one gets a free page in its place (the lowest numbers, rows in
 * ascending order, after the counts have followed) and an entry of copies_dev [n_new][3]: old page, new page, positions in it; rows that
 * copy nothing have -1, -1, 0.  Where there is no free page left the entry becomes -1 (ET_PAGED_NO_PAGE); the row keeps its length, and
 * every later call over it reports the page that is missing.  new_len_dev [n_new] (may not be len_dev): the row's positions, -1 for
 * slots not in use.  Entries that are no pages of the cache are copied and not counted (ET_PAGED_BAD_PAGE).  No count falls
 * below 0 (ET_PAGED_BAD_COUNT); a half-filled last page whose count is not above 0 stays with its rows, as it is.
 * workspace_dev: ET_FORK_WORKSPACE(n_pages, n_new) bytes, as above.  Limits (ET_ERR_CAPACITY): n_old, n_new <= 16384, and those of
 * et_pages_update. */
#define ET_FORK_WORKSPACE(n_pages, n_new) (4ull * (n_pages) + 16ull * (n_new))
ET_API et_status et_pages_fork(int* refs_dev, int n_pages, int page_size, const int* block_table_dev, int n_old, int max_pages,
                               const int* len_dev, const int* parent_dev, int n_new, int* new_table_dev, int* new_len_dev,
                               int* copies_dev, void* workspace_dev, size_t workspace_bytes, int* status_dev, void* cuda_stream);

/* Copies positions of pages within a layer's cache, keys and values (and their scales): copies_dev [n][3] as et_pages_fork leaves it;
 * entries with a negative page are skipped, as are those that name no page (ET_PAGED_BAD_PAGE); more positions than a page has count
 * as all.  No page that is written may be read or written by another entry. */
ET_API et_status et_kv_copy(const et_kv_cache* cache, const int* copies_dev, int n, int* status_dev, void* cuda_stream);

/* The k best continuations of each request's beams: beam b of a request has the score scores_dev[b] (fp32; NULL: zeros) and may be
 * continued by each token v < vocab at score + logits[b][v] - log(sum of exp(logits[b])).  logits: fp32 (logits_fp32 = 1) or
 * bf16, row r = request * beams + beam at r * row_stride elements.  A beam that has ended (done_dev [n_req * beams], bytes, may be NULL)
 * has the token eos alone, at its score.  Scores are compared in 64 bits; among equal ones the lower beam, then the lower token
 * comes first.  Continuations at minus infinity are none: a row whose score or whose logits' sum is not finite has none.
 *
 * Out, [n_req * k], best first: parent_dev the row that is continued, token_dev, new_scores_dev fp32, new_done_dev bytes (may be
 * NULL): 1 where the token is eos.  Where there are fewer than k: -1, -1, minus infinity, 1.  (A score below fp32's range is
 * put out as minus infinity.)  eos may be -1 if done_dev is NULL.
 * beams * vocab >= 1; k need not be beams (k = 2 * beams leaves room for those that end; beams = 1 begins a search).
 * The logarithm is off by 2^-20 at most, by 2^-19 of rows whose largest logit is 2^23 or more in magnitude.  Continuations of one beam
 * are in the order of their logits.
 * workspace_dev: ET_BEAM_WORKSPACE(n_req * beams, vocab, k) bytes, 16-byte aligned, as above.
 * Limits (ET_ERR_CAPACITY): beams <= 32, k <= 64, vocab <= 2^20, n_req * beams <= 65535. */
#define ET_BEAM_CHUNK 4096
#define ET_BEAM_WORKSPACE(rows, vocab, k) ((unsigned long long)(rows) * (((vocab) + ET_BEAM_CHUNK - 1) / ET_BEAM_CHUNK) * (8ull * (k) + 16))
ET_API et_status et_beam_select(const void* logits_dev, int logits_fp32, long long row_stride, int n_req, int beams, int vocab,
                                const float* scores_dev, const unsigned char* done_dev, int eos, int k, int* parent_dev, int* token_dev,
                                float* new_scores_dev, unsigned char* new_done_dev, void* workspace_dev, size_t workspace_bytes,
                                void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* EARLYTOM_PAGES_H */
