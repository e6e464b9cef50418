/* earlytom_decode.h -- what a decode step of the language model needs beside the prefill of earlytom_llm.h: a paged
 * key / value cache (bf16, or e4m3 with one power of two per row), attention of one new token over it, and dense
 * layers for a handful of rows.  No counterpart in the paper, whose time-to-first-token ends with the prefill; the
 * architecture is the one of earlytom_llm.h (grouped-query attention, rotate-half rotary embedding, bf16 activations,
 * fp32 residual stream and statistics).
 *
 * Conventions are those of earlytom.h's single steps: caller-owned device buffers of the current device, asynchronous on
 * cuda_stream, no allocation, no synchronisation, capturable into a CUDA graph; shapes are checked on the host and refused
 * with an et_status before anything is launched.  Contents of device arrays (page numbers, lengths) are checked by the
 * kernels: what they cannot use is skipped and reported in status_dev.  One step of one layer, for n sequences:
 *
 *   et_rmsnorm -> et_linear_rows (Q | K | V, bias) -> et_kv_append (rotates Q and K, stores K and V)
 *   -> et_attention_paged -> et_linear_rows (output projection, residual) -> et_rmsnorm
 *   -> et_linear_rows (gate | up, gated) -> et_linear_rows (down projection, residual)
 *
 * status_dev (int, may be NULL, set to 0 by the caller) receives ET_PAGED_CAPACITY where a position lies behind a
 * sequence's max_pages * page_size, ET_PAGED_BAD_PAGE where a table entry in use is not a page of the cache, 1 where a
 * bounded wait expired (a larger one stays).
 *
 * Limits (ET_ERR_CAPACITY): max_pages * page_size <= 2^30; rows of a cache below 2^31 (see et_kv_cache); for attention also
 * n_seq * heads <= 2^24 and n_seq * heads * (max_pages * page_size / 64 + 16) < 2^31. */
#ifndef EARLYTOM_DECODE_H
#define EARLYTOM_DECODE_H

#include "earlytom.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ET_KV_BF16 = 0, ET_KV_E4M3 = 1 } et_kv_format;
enum { ET_PAGED_CAPACITY = 3, ET_PAGED_BAD_PAGE = 5 };

/* A paged cache of one layer.  Row t of page p holds the key (plane 0) and value (plane 1) of one position:
 *   data  [n_pages][2][kv_heads][page_size][head_dim], bf16 or e4m3 (4 exponent bits, 3 mantissa bits, no infinities);
 *   scale [n_pages][2][kv_heads][page_size], ET_KV_E4M3 only (NULL otherwise): a byte b stands for 2^(b - 127), the factor
 *         of its row of head_dim values; b is never 255.
 * Both 16-byte aligned.  Rows never written hold whatever was there; nothing reads behind a sequence's length. */
typedef struct {
  void* data;
  unsigned char* scale;
  int n_pages;     /* n_pages * 2 * kv_heads * page_size < 2^31 */
  int kv_heads;
  int page_size;   /* 16, 32, 64 or 128 */
  int head_dim;    /* 64 or 128 */
  int format;      /* et_kv_format */
} et_kv_cache;

/* Stores the keys and values of `rows` new tokens.  qkv bf16, row r at qkv + r * row_stride elements, packed
 * [Q (heads) | K (kv_heads) | V (kv_heads)] x head_dim; row_stride a multiple of 8.  heads may be 0: then a row is
 * [K | V], the layout of et_llm_result.kv_cache, whose keys are rotated already.
 *
 * Rows belong to sequences in runs: row_offsets_dev [n_seq + 1] (ascending, first 0) says that rows row_offsets[s] ..
 * row_offsets[s+1] - 1 are sequence s, at positions start[s], start[s] + 1, ...; rows from row_offsets[n_seq] on are
 * padding.  row_offsets_dev NULL: one row for each sequence (rows == n_seq).  start_dev [n_seq]: positions that the sequence
 * has in the cache; a negative one marks a slot that is not in use.  block_table_dev [n_seq][max_pages]: page of positions
 * j * page_size .. (j + 1) * page_size - 1.  Padding, slots not in use and rows that cannot be placed (see status_dev)
 * are skipped: nothing is written for them.  A page that rows of one call go to must belong to one sequence only and stand
 * in its table once; where it does not, those rows' contents are unspecified.  Offsets that are not as said put no row outside
 * the cache, but may put it at a wrong position of it; one behind `rows` counts as `rows`.
 *
 * theta > 1: Q and K are turned as et_rope does it, by the row's position; the turned Q goes to q_out_dev (bf16
 * [rows][heads * head_dim], dense, not overlapping qkv; may be NULL with heads = 0 only).  theta = 0: nothing is turned
 * and q_out_dev is not written (and must be NULL).
 *
 * ET_KV_E4M3: a row x of head_dim values is stored as x * 2^-e rounded to e4m3 (nearest, ties to even), with the smallest
 * e in [-127, 127] for which max|x| <= 448 * 2^e; scaling by a power of two is exact, so the conversion is the only
 * rounding.  Turned keys are converted from fp32, off by two roundings of that.  A value that is not finite is stored as NaN
 * and not counted in the maximum.
 *
 * new_len_dev (int [n_seq], may be NULL, not start_dev): positions in the cache after the call, start + rows but at most
 * max_pages * page_size (also where the start is behind that already), or the negative start. */
ET_API et_status et_kv_append(const et_kv_cache* cache, const void* qkv_dev, long long row_stride, int rows, int heads,
                              const int* block_table_dev, int n_seq, int max_pages, const int* row_offsets_dev,
                              const int* start_dev, float theta, void* q_out_dev, int* new_len_dev, int* status_dev,
                              void* cuda_stream);

/* Reads rows back: out bf16, row r at out + r * row_stride elements = [K (kv_heads) | V (kv_heads)] x head_dim as stored
 * (an e4m3 value times a power of two has 4 significant bits: exact from 2^-130 on, rounded to bf16's smallest steps of 2^-133
 * below, infinite from 2^128 on).  Rows are named as in et_kv_append; rows that are skipped there are left as they were here. */
ET_API et_status et_kv_read(const et_kv_cache* cache, void* out_dev, long long row_stride, int rows,
                            const int* block_table_dev, int n_seq, int max_pages, const int* row_offsets_dev,
                            const int* start_dev, int* status_dev, void* cuda_stream);

/* Attention of one token of each sequence over its cached positions: out[s] = softmax(q K^T / sqrt(head_dim)) V over
 * positions 0 .. len[s] - 1, query head h reading key / value head h / (heads / kv_heads).  q bf16, row s at
 * q + s * q_stride elements (a multiple of 8; 16-byte aligned), heads x head_dim: et_kv_append's q_out, or packed rows.
 * out bf16 [n_seq][heads * head_dim]; lse_dev fp32 [n_seq][heads] (may be NULL): natural logarithm of the sum of
 * exponentials.  len_dev [n_seq]; a length of 0 or less gives zeros and -infinity.  Positions behind max_pages * page_size
 * and on pages that are not in the cache are left out (see status_dev).  Whatever stands behind a sequence's length, NaN
 * included, has no influence.  Scores, their maximum and sum and the outputs are fp32.  A probability counts with 16 bits for a
 * bf16 cache; for e4m3 with 11 or more down to 2^-21 of the largest one, below that it is off by at most 2^-32 of the largest.
 * An infinite value is its column's result, the other columns keep theirs; below 2^-100 of the
 * largest weight it may make a NaN of its column instead (0 * infinity).
 * workspace_dev: ET_PAGED_WORKSPACE bytes, 16-byte aligned, contents neither needed nor kept; one call at a time may use
 * it (calls, captured or not, that can run at the same time need one each). */
#define ET_PAGED_WORKSPACE (4u << 20)
ET_API et_status et_attention_paged(const et_kv_cache* cache, const void* q_dev, long long q_stride, void* out_dev,
                                    float* lse_dev, int n_seq, int heads, const int* block_table_dev, int max_pages,
                                    const int* len_dev, void* workspace_dev, size_t workspace_bytes, int* status_dev,
                                    void* cuda_stream);

/* Dense layer for few rows: c = epilogue(a[M][K] * w[N][K]^T + bias[N]), M <= 32; the memory traffic of the weights
 * bounds it.  Arguments and epilogues 0, 1, 2 and 4 are those of et_linear_bf16 (the weight rows of epilogue 4 are in the
 * same order, N % 256 == 0); K % 8 == 0, a, w and c 16-byte aligned, c overlaps neither; bias may be NULL (zeros).  Sums
 * are taken in an order that depends on M, N, K and the device (on how many clusters of blocks it holds at once); a row's result
 * does not depend on the other rows' values. */
ET_API et_status et_linear_rows(const void* a_dev, const void* w_dev, const float* bias_dev, void* c_dev, int M, int N, int K,
                                int epilogue, int gelu_tanh, int* status_dev, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* EARLYTOM_DECODE_H */
