// Internal declarations of the decode step's operators (kv_cache.cu, attention_paged.cu, linear_rows.cu, decode.cu).
#pragma once

#include "common.cuh"
#include "earlytom_decode.h"

namespace et {

// A checked et_kv_cache: sizes as shifts where they are powers of two.
struct PagedCache {
  uint8_t* data;
  uint8_t* scale;        // NULL: bf16
  int n_pages, kv_heads, page_shift, head_dim;
};

// The rows of a call and the pages that they go to.
struct PagedRows {
  const int* table;      // [n_seq][max_pages]
  const int* offsets;    // [n_seq + 1] or NULL: row r is sequence r
  const int* start;      // [n_seq]
  int rows, n_seq, max_pages;
  int* status;           // may be NULL
};

struct RopeTurns { unsigned long long f[64]; };   // theta^(-2i/dh) / (2 pi) as a fraction of 2^64

cudaError_t launch_kv_append(const PagedCache& c, const PagedRows& r, const bf16* qkv, long long row_stride, int heads, bool rotate,
                             const RopeTurns& turns, bf16* q_out, int* new_len, cudaStream_t s);
cudaError_t launch_kv_read(const PagedCache& c, const PagedRows& r, bf16* out, long long row_stride, cudaStream_t s);

struct PagedAttention {
  const bf16* q;
  long long q_stride;
  bf16* out;
  float* lse;            // may be NULL
  int n_seq, heads, max_pages;
  const int* table;
  const int* len;
  float* workspace;
  int* status;           // may be NULL
};
constexpr int PAGED_ITEM_COST_MAX = 16;   // units beside its tiles of 64 positions that an item (sequence, key / value head, head tile) counts for
cudaError_t launch_attention_paged(const PagedCache& c, const PagedAttention& a, cudaStream_t s);

// c = epi(a[M][K] * w[N][K]^T + bias), M <= LINEAR_ROWS_MAX
constexpr int LINEAR_ROWS_MAX = 32;
cudaError_t launch_linear_rows(const bf16* a, const bf16* w, const float* bias, void* c, int M, int N, int K, int epilogue,
                               int gelu_tanh, int* status, cudaStream_t s);

// Every kernel of the decode step is launched so that it may be set up while the kernel before it in the stream still runs
// (programmatic dependent launch), and begins, before it touches memory, by waiting for that one's end and results.  What these
// kernels read may be what the kernel before wrote while they were resident already: none of it is read with non-coherent loads
// (__ldg, .nc, const __restrict__ parameters), which may come before the wait or from a stale line.
__device__ __forceinline__ void begin_after_previous() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");    // the next kernel may be set up; it waits in turn
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

struct Launch {
  cudaLaunchAttribute attr[2];
  cudaLaunchConfig_t cfg = {};
  Launch(dim3 blocks, int threads, size_t smem, cudaStream_t s, int cluster = 1) {
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
  Launch(const Launch&) = delete;
};

// Place of a position of sequence s; false (with the status) if it has none.
__device__ __forceinline__ bool paged_place(const PagedCache& c, const int* table, int max_pages, int s, long long pos, int* status,
                                            int& page, int& place) {
  if ((pos >> c.page_shift) >= max_pages) {
    if (status) atomicMax(status, (int)ET_PAGED_CAPACITY);
    return false;
  }
  page = table[(size_t)s * max_pages + (pos >> c.page_shift)];
  place = (int)(pos & ((1 << c.page_shift) - 1));
  if ((unsigned)page >= (unsigned)c.n_pages) {
    if (status) atomicMax(status, (int)ET_PAGED_BAD_PAGE);
    return false;
  }
  return true;
}

}  // namespace et
