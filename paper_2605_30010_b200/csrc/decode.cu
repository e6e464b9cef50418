// C entry points of include/earlytom_decode.h: argument checks and launches.
#include <math.h>

#include "decode.cuh"

using namespace et;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

et_status check_cache(const et_kv_cache* c, PagedCache* out) {
  if (!c || !c->data) return ET_ERR_INVALID_ARG;
  if (c->format != ET_KV_BF16 && c->format != ET_KV_E4M3) return ET_ERR_INVALID_ARG;
  if ((c->format == ET_KV_E4M3) != (c->scale != nullptr)) return ET_ERR_INVALID_ARG;
  if (!aligned16(c->data) || !aligned16(c->scale)) return ET_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->kv_heads < 1 || (c->head_dim != 64 && c->head_dim != 128)) return ET_ERR_SHAPE;
  int shift = 4;
  while (shift < 7 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return ET_ERR_SHAPE;
  // row numbers of the cache are 32-bit (TMA coordinates); byte offsets are 64-bit
  if ((long long)c->n_pages > ((1ll << 31) - 1) / (2ll * c->page_size) / c->kv_heads) return ET_ERR_CAPACITY;
  *out = PagedCache{(uint8_t*)c->data, c->scale, c->n_pages, c->kv_heads, shift, c->head_dim};
  return ET_OK;
}

et_status check_table(const int* table, int n_seq, int max_pages, int page_shift) {
  if (!table) return ET_ERR_INVALID_ARG;
  if (n_seq < 1 || max_pages < 1) return ET_ERR_SHAPE;
  if ((long long)max_pages << page_shift > 1ll << 30) return ET_ERR_CAPACITY;      // positions are 32-bit, with room for tiles' ends
  return ET_OK;
}

et_status check_rows(const PagedCache& c, int rows, const int* table, int n_seq, int max_pages, const int* offsets, const int* start,
                     int* status, PagedRows* out) {
  const et_status st = check_table(table, n_seq, max_pages, c.page_shift);
  if (st != ET_OK) return st;
  if (!start) return ET_ERR_INVALID_ARG;
  if (rows < 1 || (!offsets && rows != n_seq)) return ET_ERR_SHAPE;
  *out = PagedRows{table, offsets, start, rows, n_seq, max_pages, status};
  return ET_OK;
}

// theta^(-2i/dh) / (2 pi) as a fraction of 2^64: a geometric sequence in extended precision, off by less than 2^-56 of its
// value after 64 steps, i.e. by less than 2^-24 of a turn at the largest position.  A model has one theta and head size: each
// host thread keeps the frequencies of the last ones (a microsecond of a call's five).
const RopeTurns& rope_turns(float theta, int head_dim) {
  static thread_local RopeTurns t;
  static thread_local float of_theta = 0.f;
  static thread_local int of_dim = 0;
  if (theta != of_theta || head_dim != of_dim) {
    const long double ratio = powl((long double)theta, -2.0L / head_dim);
    long double f = 0.15915494309189533576888376337251436L * 18446744073709551616.0L;     // 2^64 / (2 pi) < 2^63
    for (int i = 0; i < head_dim / 2; ++i) {
      t.f[i] = (unsigned long long)(long long)(f + 0.5L);
      f *= ratio;
    }
    of_theta = theta; of_dim = head_dim;
  }
  return t;
}

// A launch's own result: an error that an earlier call left behind is not this call's, and none is left for a later one.
et_status launched(cudaError_t e) {
  if (e == cudaSuccess) return ET_OK;
  cudaGetLastError();
  return ET_ERR_CUDA;
}

}  // namespace

extern "C" {

et_status et_kv_append(const et_kv_cache* cache, const void* qkv_dev, long long row_stride, int rows, int heads,
                       const int* block_table_dev, int n_seq, int max_pages, const int* row_offsets_dev, const int* start_dev,
                       float theta, void* q_out_dev, int* new_len_dev, int* status_dev, void* cuda_stream) {
  PagedCache c;
  PagedRows r;
  et_status st = check_cache(cache, &c);
  if (st == ET_OK) st = check_rows(c, rows, block_table_dev, n_seq, max_pages, row_offsets_dev, start_dev, status_dev, &r);
  if (st != ET_OK) return st;
  if (heads < 0 || (long long)heads + 2ll * c.kv_heads > (1 << 20)) return ET_ERR_SHAPE;
  const bool rotate = theta != 0.f;
  if (!qkv_dev || !aligned16(qkv_dev) || !aligned16(q_out_dev)) return ET_ERR_INVALID_ARG;
  if (rotate && !(theta > 1.f && theta <= 3.402823466e38f)) return ET_ERR_INVALID_ARG;
  if ((q_out_dev != nullptr) != (rotate && heads > 0)) return ET_ERR_INVALID_ARG;
  if (new_len_dev && new_len_dev == start_dev) return ET_ERR_INVALID_ARG;
  if (row_stride % 8 != 0 || row_stride < ((long long)heads + 2ll * c.kv_heads) * c.head_dim) return ET_ERR_SHAPE;
  static const RopeTurns none = {};
  return launched(launch_kv_append(c, r, (const bf16*)qkv_dev, row_stride, heads, rotate, rotate ? rope_turns(theta, c.head_dim) : none,
                                   (bf16*)q_out_dev, new_len_dev, (cudaStream_t)cuda_stream));
}

et_status et_kv_read(const et_kv_cache* cache, void* out_dev, long long row_stride, int rows, const int* block_table_dev, int n_seq,
                     int max_pages, const int* row_offsets_dev, const int* start_dev, int* status_dev, void* cuda_stream) {
  PagedCache c;
  PagedRows r;
  et_status st = check_cache(cache, &c);
  if (st == ET_OK) st = check_rows(c, rows, block_table_dev, n_seq, max_pages, row_offsets_dev, start_dev, status_dev, &r);
  if (st != ET_OK) return st;
  if (!out_dev || !aligned16(out_dev)) return ET_ERR_INVALID_ARG;
  if (c.kv_heads > (1 << 19)) return ET_ERR_SHAPE;
  if (row_stride % 8 != 0 || row_stride < 2ll * c.kv_heads * c.head_dim) return ET_ERR_SHAPE;
  return launched(launch_kv_read(c, r, (bf16*)out_dev, row_stride, (cudaStream_t)cuda_stream));
}

et_status et_attention_paged(const et_kv_cache* cache, const void* q_dev, long long q_stride, void* out_dev, float* lse_dev, int n_seq,
                             int heads, const int* block_table_dev, int max_pages, const int* len_dev, void* workspace_dev,
                             size_t workspace_bytes, int* status_dev, void* cuda_stream) {
  PagedCache c;
  et_status st = check_cache(cache, &c);
  if (st == ET_OK) st = check_table(block_table_dev, n_seq, max_pages, c.page_shift);
  if (st != ET_OK) return st;
  if (!q_dev || !out_dev || !len_dev || !workspace_dev) return ET_ERR_INVALID_ARG;
  if (!aligned16(q_dev) || !aligned16(out_dev) || !aligned16(workspace_dev)) return ET_ERR_INVALID_ARG;
  if (heads < 1 || heads % c.kv_heads != 0) return ET_ERR_SHAPE;
  if (q_stride % 8 != 0 || q_stride < (long long)heads * c.head_dim) return ET_ERR_SHAPE;
  if ((long long)n_seq * heads > (1ll << 24)) return ET_ERR_CAPACITY;
  // the work is numbered in 32 bits: tiles of 64 positions of every sequence and head
  if ((long long)n_seq * heads * ((((long long)max_pages << c.page_shift) + 63) / 64 + PAGED_ITEM_COST_MAX) >= (1ll << 31) - 256) return ET_ERR_CAPACITY;
  if (workspace_bytes < ET_PAGED_WORKSPACE) return ET_ERR_CAPACITY;
  const PagedAttention a{(const bf16*)q_dev, q_stride, (bf16*)out_dev, lse_dev, n_seq, heads, max_pages, block_table_dev, len_dev,
                         (float*)workspace_dev, status_dev};
  return launched(launch_attention_paged(c, a, (cudaStream_t)cuda_stream));
}

et_status et_linear_rows(const void* a_dev, const void* w_dev, const float* bias_dev, void* c_dev, int M, int N, int K, int epilogue,
                         int gelu_tanh, int* status_dev, void* cuda_stream) {
  if (!a_dev || !w_dev || !c_dev || !aligned16(a_dev) || !aligned16(w_dev) || !aligned16(c_dev)) return ET_ERR_INVALID_ARG;
  if (epilogue != EPI_STORE && epilogue != EPI_GELU && epilogue != EPI_RESIDUAL && epilogue != EPI_SWIGLU) return ET_ERR_INVALID_ARG;
  if (M < 1 || N < 1 || K < 8 || K % 8 != 0 || (epilogue == EPI_SWIGLU && N % 256 != 0)) return ET_ERR_SHAPE;
  if (M > LINEAR_ROWS_MAX || N > (1 << 24) || K > (1 << 24)) return ET_ERR_CAPACITY;
  return launched(launch_linear_rows((const bf16*)a_dev, (const bf16*)w_dev, bias_dev, c_dev, M, N, K, epilogue, gelu_tanh, status_dev,
                                     (cudaStream_t)cuda_stream));
}

}  // extern "C"
