// Dense layer for few rows (a decode step's): c[M][N] = epilogue(a[M][K] * w[N][K]^T + bias), M <= 32.
//
// Every weight is read once and used M times, so the weights' bytes over the memory bandwidth bound it and everything is
// arranged to keep loads in flight.  The product is transposed, c^T = w a^T: 16 weight rows are the tall side of mma.sync's
// m16n8k16 and 8 rows of a the narrow one.  (tcgen05's tiles would stage the weights through shared memory for tensor work
// that is a few per cent of the time.)  A weight goes from memory to the register that feeds the tensor core with one
// 16-byte load and no shuffle: the k-index of a step is permuted so that a lane's 8 consecutive weights are its operands of
// two instructions, and a is read in the same order.
//
// A block of 8 warps owns 32 weight rows; K is dealt to the warps in steps of 64, and where there are too few blocks for
// the card a cluster shares a block's K as well.  Sums meet in shared memory (of the cluster), always in the same order,
// which depends on N and K alone: a row's result does not depend on the other rows, nor on how many there are.
#include <cooperative_groups.h>

#include "decode.cuh"
#include "rowops.cuh"

namespace et {

namespace {

namespace cg = cooperative_groups;

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int BLOCK_ROWS = 32;                 // weight rows of a block: two tiles of 16
constexpr int STEP = 64;                       // k of a warp's step: 128 bytes of each row
constexpr int MAX_CLUSTER = 8;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// weights are used once: not worth a place in L1
__device__ __forceinline__ uint4 load_once(const bf16* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

struct LinearArgs {
  const bf16* a;
  const bf16* w;
  const float* bias;
  void* c;
  int M, N, K, epilogue, gelu_tanh;
};

template <int NT>
__global__ void __launch_bounds__(THREADS, NT <= 2 ? 2 : 1)
linear_rows_kernel(const LinearArgs g) {
  constexpr int COLS = 8 * NT, LD = COLS + 1;
  __shared__ float red[WARPS][BLOCK_ROWS * LD];
  __shared__ float part[BLOCK_ROWS * COLS];
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int block = blockIdx.x / ranks;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, gq = lane >> 2, tq = lane & 3;
  const bool gated = g.epilogue == EPI_SWIGLU;
  // first weight row of the block's two tiles: neighbours, or 16 gate rows and the up rows of the same outputs
  const int row0 = gated ? (block >> 1) * 64 + (block & 1) * 16 : block * BLOCK_ROWS;
  const int tile_stride = gated ? 32 : 16;

  const bf16* wp[2][2];                        // rows gq and gq + 8 of each tile; rows behind N are read as the last one and dropped
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) wp[i][j] = g.w + (size_t)min(row0 + i * tile_stride + j * 8 + gq, g.N - 1) * g.K + 8 * tq;
  const bf16* ap[NT];
  bool live[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    live[n] = n * 8 + gq < g.M;
    ap[n] = g.a + (size_t)(live[n] ? n * 8 + gq : 0) * g.K + 8 * tq;
  }
  float acc[2][NT][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;

  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 wb[2][2][2];                           // [half of the step][tile][row]
  auto load_w = [&](int k) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = k + 32 * h + 8 * tq < g.K;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) wb[h][i][j] = in ? load_once(wp[i][j] + k + 32 * h) : zero;
    }
  };
  const int stride = STEP * WARPS * ranks;
  int k = STEP * (rank * WARPS + warp);
  if (k < g.K) load_w(k);
  for (; k < g.K; k += stride) {
    uint4 ab[2][NT], cur[2][2][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool in = k + 32 * h + 8 * tq < g.K;
#pragma unroll
      for (int n = 0; n < NT; ++n) ab[h][n] = in && live[n] ? __ldg(reinterpret_cast<const uint4*>(ap[n] + k + 32 * h)) : zero;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) cur[h][i][j] = wb[h][i][j];
    }
    if (k + stride < g.K) load_w(k + stride);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          mma_bf16(acc[i][n], cur[h][i][0].x, cur[h][i][1].x, cur[h][i][0].y, cur[h][i][1].y, ab[h][n].x, ab[h][n].y);
          mma_bf16(acc[i][n], cur[h][i][0].z, cur[h][i][1].z, cur[h][i][0].w, cur[h][i][1].w, ab[h][n].z, ab[h][n].w);
        }
  }

  // ---- the warps' sums, then the cluster's
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float* dst = &red[warp][(i * 16 + j * 8 + gq) * LD + n * 8 + 2 * tq];
        dst[0] = acc[i][n][2 * j]; dst[1] = acc[i][n][2 * j + 1];
      }
  __syncthreads();
  for (int e = tid; e < BLOCK_ROWS * g.M; e += THREADS) {
    const int r = e % BLOCK_ROWS, m = e / BLOCK_ROWS;
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < WARPS; ++v) s += red[v][r * LD + m];
    part[m * BLOCK_ROWS + r] = s;
  }
  if (ranks > 1) cluster.sync(); else __syncthreads();
  auto total = [&](int r, int m) {
    float s = 0.f;
    for (int p = 0; p < ranks; ++p) s += cluster.map_shared_rank(part, p)[m * BLOCK_ROWS + r];
    return s;
  };
  if (gated) {
    for (int e = rank * THREADS + tid; e < 16 * g.M; e += ranks * THREADS) {
      const int r = e % 16, m = e / 16, n = row0 + r;
      const float gate = total(r, m) + (g.bias ? g.bias[n] : 0.f), up = total(16 + r, m) + (g.bias ? g.bias[n + 32] : 0.f);
      reinterpret_cast<bf16*>(g.c)[(size_t)m * (g.N / 2) + block * 16 + r] = __float2bfloat16_rn(gate / (1.f + expf(-gate)) * up);
    }
  } else {
    for (int e = rank * THREADS + tid; e < BLOCK_ROWS * g.M; e += ranks * THREADS) {
      const int r = e % BLOCK_ROWS, m = e / BLOCK_ROWS, n = row0 + r;
      if (n >= g.N) continue;
      float y = total(r, m) + (g.bias ? g.bias[n] : 0.f);
      const size_t at = (size_t)m * g.N + n;
      if (g.epilogue == EPI_RESIDUAL) {
        reinterpret_cast<float*>(g.c)[at] += y;
      } else {
        if (g.epilogue == EPI_GELU) y = gelu_f(y, g.gelu_tanh);
        reinterpret_cast<bf16*>(g.c)[at] = __float2bfloat16_rn(y);
      }
    }
  }
  if (ranks > 1) cluster.sync();               // a block's sums stay until its neighbours have read them
}

template <int NT>
cudaError_t launch(const LinearArgs& g, int blocks, int ranks, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ranks; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks * ranks);
  cfg.blockDim = dim3(THREADS);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, linear_rows_kernel<NT>, g);
}

}  // namespace

cudaError_t launch_linear_rows(const bf16* a, const bf16* w, const float* bias, void* c, int M, int N, int K, int epilogue,
                               int gelu_tanh, cudaStream_t s) {
  const LinearArgs g{a, w, bias, c, M, N, K, epilogue, gelu_tanh};
  const int blocks = cdiv(N, BLOCK_ROWS);
  // two blocks an SM are wanted, each with at least two steps for every warp
  int ranks = 1;
  while (ranks < MAX_CLUSTER && blocks * ranks * 2 <= 148 * 2 && K >= STEP * WARPS * 2 * ranks * 2) ranks *= 2;
  switch ((M + 7) / 8) {
    case 1: return launch<1>(g, blocks, ranks, s);
    case 2: return launch<2>(g, blocks, ranks, s);
    case 3: return launch<3>(g, blocks, ranks, s);
    default: return launch<4>(g, blocks, ranks, s);
  }
}

}  // namespace et
