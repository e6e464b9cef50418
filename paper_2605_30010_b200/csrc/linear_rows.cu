// Dense layer for few rows.
#include "decode.cuh"
#include "rowops.cuh"

namespace et {

namespace {

constexpr int WARPS = 8;

// The simplest form: one warp per output column, all rows of a against its weight row.
__device__ __forceinline__ float dot_row(const bf16* a, const bf16* w, int K, int lane) {
  float d = 0.f;
  for (int k = lane; k < K; k += 32) d += __bfloat162float(a[k]) * __bfloat162float(w[k]);
  return warp_sum(d);
}

__global__ void __launch_bounds__(WARPS * 32)
linear_rows_kernel(const bf16* __restrict__ a, const bf16* __restrict__ w, const float* __restrict__ bias, void* c, int M, int N, int K,
                   int epilogue, int gelu_tanh) {
  const int lane = threadIdx.x & 31;
  const int outs = epilogue == EPI_SWIGLU ? N / 2 : N;
  const int j = blockIdx.x * WARPS + (threadIdx.x >> 5);
  if (j >= outs) return;
  const int n = epilogue == EPI_SWIGLU ? (j / 32) * 64 + j % 32 : j;
  for (int m = 0; m < M; ++m) {
    const bf16* ar = a + (size_t)m * K;
    float y = dot_row(ar, w + (size_t)n * K, K, lane) + (bias ? bias[n] : 0.f);
    const size_t at = (size_t)m * outs + j;
    if (epilogue == EPI_SWIGLU) {
      const float up = dot_row(ar, w + (size_t)(n + 32) * K, K, lane) + (bias ? bias[n + 32] : 0.f);
      y = y / (1.f + expf(-y)) * up;
    } else if (epilogue == EPI_GELU) {
      y = gelu_f(y, gelu_tanh);
    }
    if (lane == 0) {
      if (epilogue == EPI_RESIDUAL) reinterpret_cast<float*>(c)[at] += y;
      else reinterpret_cast<bf16*>(c)[at] = __float2bfloat16_rn(y);
    }
  }
}

}  // namespace

cudaError_t launch_linear_rows(const bf16* a, const bf16* w, const float* bias, void* c, int M, int N, int K, int epilogue,
                               int gelu_tanh, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  linear_rows_kernel<<<cdiv(epilogue == EPI_SWIGLU ? N / 2 : N, WARPS), WARPS * 32, 0, s>>>(a, w, bias, c, M, N, K, epilogue, gelu_tanh);
  return cudaGetLastError();
}

}  // namespace et
