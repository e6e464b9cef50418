// Attention of one new token of each sequence over its paged key / value cache.
#include <cuda_fp8.h>

#include "decode.cuh"
#include "rowops.cuh"

namespace et {

namespace {

constexpr int WARPS = 4;

// The simplest form: one block per (sequence, query head), keys dealt to the warps in turn, each warp with a running
// maximum and sum of its own, joined through shared memory at the end.
template <int DH, bool E4M3>
__global__ void __launch_bounds__(WARPS * 32)
attention_paged_kernel(PagedCache c, PagedAttention g) {
  constexpr int V = DH / 32;                     // values of a row per lane
  const int s = blockIdx.x / g.heads, h = blockIdx.x % g.heads, kvh = h / (g.heads / c.kv_heads);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float scale = rsqrtf((float)DH);
  float q[V], o[V], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int k = 0; k < V; ++k) { q[k] = __bfloat162float(g.q[(size_t)s * g.q_stride + h * DH + lane * V + k]) * scale; o[k] = 0.f; }
  auto load = [&](size_t row, float (&x)[V]) {
    const float f = E4M3 ? __int_as_float(c.scale[row] ? c.scale[row] << 23 : 1 << 22) : 1.f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const size_t at = row * DH + lane * V + k;
      if (E4M3) {
        const __half_raw y = __nv_cvt_fp8_to_halfraw(c.data[at], __NV_E4M3);
        x[k] = __half2float(*reinterpret_cast<const __half*>(&y)) * f;
      } else {
        x[k] = __bfloat162float(reinterpret_cast<const bf16*>(c.data)[at]);
      }
    }
  };
  long long len = g.len[s];
  const long long cap = (long long)g.max_pages << c.page_shift;
  if (len > cap) {
    if (g.status && threadIdx.x == 0) atomicMax(g.status, (int)ET_PAGED_CAPACITY);
    len = cap;
  }
  for (long long t = warp; t < len; t += WARPS) {
    int page, place;
    if (!paged_place(c, g.table, g.max_pages, s, t, g.status, page, place)) continue;
    const size_t row = ((((size_t)page * 2) * c.kv_heads + kvh) << c.page_shift) + place;
    float k[V], v[V], d = 0.f;
    load(row, k);
    load(row + ((size_t)c.kv_heads << c.page_shift), v);
#pragma unroll
    for (int j = 0; j < V; ++j) d += q[j] * k[j];
    d = warp_sum(d);
    const float mn = fmaxf(m, d), a = expf(m - mn), p = expf(d - mn);
    l = l * a + p;
#pragma unroll
    for (int j = 0; j < V; ++j) o[j] = o[j] * a + p * v[j];
    m = mn;
  }
  __shared__ float so[WARPS][DH], sm[WARPS], sl[WARPS];
#pragma unroll
  for (int j = 0; j < V; ++j) so[warp][lane * V + j] = o[j];
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
  __syncthreads();
  float top = -INFINITY, total = 0.f;
  for (int w = 0; w < WARPS; ++w) top = fmaxf(top, sm[w]);
  for (int w = 0; w < WARPS; ++w) if (sm[w] > -INFINITY || sl[w] != 0.f) total += sl[w] * expf(sm[w] - top);
  const bool empty = total == 0.f;               // NaN is not empty
  for (int j = threadIdx.x; j < DH; j += WARPS * 32) {
    float x = 0.f;
    for (int w = 0; w < WARPS; ++w) if (sm[w] > -INFINITY || sl[w] != 0.f) x += so[w][j] * expf(sm[w] - top);
    g.out[((size_t)s * g.heads + h) * DH + j] = __float2bfloat16_rn(empty ? 0.f : x / total);
  }
  if (g.lse && threadIdx.x == 0) g.lse[(size_t)s * g.heads + h] = empty ? -INFINITY : logf(total) + top;
}

}  // namespace

cudaError_t launch_attention_paged(const PagedCache& c, const PagedAttention& a, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  const int blocks = a.n_seq * a.heads;
  if (c.head_dim == 64) {
    if (c.scale) attention_paged_kernel<64, true><<<blocks, WARPS * 32, 0, s>>>(c, a);
    else attention_paged_kernel<64, false><<<blocks, WARPS * 32, 0, s>>>(c, a);
  } else {
    if (c.scale) attention_paged_kernel<128, true><<<blocks, WARPS * 32, 0, s>>>(c, a);
    else attention_paged_kernel<128, false><<<blocks, WARPS * 32, 0, s>>>(c, a);
  }
  return cudaGetLastError();
}

}  // namespace et
