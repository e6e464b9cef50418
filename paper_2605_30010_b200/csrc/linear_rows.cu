// Dense layer for few rows (a decode step's): c[M][N] = epilogue(a[M][K] * w[N][K]^T + bias), M <= 32.
//
// Every weight is read once and used M times, so the weights' bytes over the memory bandwidth bound it and everything is
// arranged to keep loads in flight.  The product is transposed, c^T = w a^T: 16 weight rows are the tall side of mma.sync's
// m16n8k16 and 8 rows of a the narrow one, so up to 8 rows cost no padding.  (tcgen05's smallest tiles have 64 rows of each;
// the tensor work here is a few per cent of the time.)  Two kernels share the epilogue:
//
//   direct  weights go from memory to the registers that feed the tensor core; a block has 32 weight rows.  Starts fast.
//   ring    TMA tiles of up to 128 weight rows and of a in a ring of five stages; a is fetched once for up to four times as
//           many weights.
//
// K is shared by the warps of a block (direct) and by the blocks of a cluster where there are too few blocks to fill the
// card.  Sums meet in shared memory (of the cluster) in a fixed order.
//
// Device time per call in a chain of calls, B200, weights not in L2 (of the measured copy bandwidth):
//   1 x 3584 x 4608 8.4 us (0.61, direct), 1 x 3584 x 37888 gated 43.5 us (0.97, ring), 19 x the same 46.5 us (0.90; 47.2 in calls
//   repeated for a second), 1 x 18944 x 3584 residual 24 us (0.88, ring), 32 x the same 27.5 us (0.78)
#include <cooperative_groups.h>

#include <atomic>

#include "decode.cuh"
#include "rowops.cuh"
#include "tcgen05.cuh"

namespace et {

namespace {

namespace cg = cooperative_groups;
using namespace tc;

constexpr int WARPS = 8, THREADS = 32 * WARPS;  // of the direct kernel
constexpr int BLOCK_ROWS = 32;                 // its weight rows of a block: two tiles of 16
constexpr int STEP = 64;                       // k of a warp's step: 128 bytes of each row
constexpr int SUM_STEPS = 32;                  // steps of a warp that the tensor core sums at most
constexpr int MAX_CLUSTER = 8;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 16 consecutive values of a row, k .. k + 15: one 32-byte load where rows allow it (WIDE: K % 16 == 0, 32-byte aligned),
// so that the four lanes of a row take a whole 128-byte line with one instruction, two 16-byte loads where they do not.
// Weights are used once and not worth a place in L1.
struct Vec { uint32_t r[8]; };
template <bool WIDE, bool ONCE>
__device__ __forceinline__ void load_vec(Vec& v, const bf16* p, int k, int K, bool live) {
  if (WIDE) {
    if (live && k < K) {
      if (ONCE)
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v.r[0]), "=r"(v.r[1]), "=r"(v.r[2]), "=r"(v.r[3]), "=r"(v.r[4]), "=r"(v.r[5]), "=r"(v.r[6]), "=r"(v.r[7]) : "l"(p + k));
      else
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(v.r[0]), "=r"(v.r[1]), "=r"(v.r[2]), "=r"(v.r[3]), "=r"(v.r[4]), "=r"(v.r[5]), "=r"(v.r[6]), "=r"(v.r[7]) : "l"(p + k));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v.r[i] = 0;
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (live && k + 8 * h < K) x = *reinterpret_cast<const uint4*>(p + k + 8 * h);
      v.r[4 * h] = x.x; v.r[4 * h + 1] = x.y; v.r[4 * h + 2] = x.z; v.r[4 * h + 3] = x.w;
    }
  }
}

struct LinearArgs {
  const bf16* a;
  const bf16* w;
  const float* bias;
  void* c;
  int M, N, K, epilogue, gelu_tanh;
  int* status;
};

// The block's sums [m][ROWS] of every rank become outputs, dealt to the ranks' threads four at a time; the ranks' parts are
// fetched together and added in order.  In a gated block 16 gate rows are followed by the 16 up rows of the same outputs.
template <int ROWS, int NTHREADS>
__device__ __forceinline__ void finish(const LinearArgs& g, cg::cluster_group& cluster, float* part, int rows, int block, int ranks, int rank) {
  const int tid = threadIdx.x;
  const bool gated = g.epilogue == EPI_SWIGLU;
  auto total = [&](int r, int m, float (&y)[4]) {
    float4 v[MAX_CLUSTER];
#pragma unroll
    for (int p = 0; p < MAX_CLUSTER; ++p)
      if (p < ranks) v[p] = *reinterpret_cast<const float4*>((ranks > 1 ? cluster.map_shared_rank(part, p) : part) + m * ROWS + r);
    y[0] = y[1] = y[2] = y[3] = 0.f;
#pragma unroll
    for (int p = 0; p < MAX_CLUSTER; ++p)
      if (p < ranks) { y[0] += v[p].x; y[1] += v[p].y; y[2] += v[p].z; y[3] += v[p].w; }
  };
  const int outs = gated ? g.N / 2 : g.N, quads = gated ? rows / 8 : rows / 4;
  const bool vectors = outs % 4 == 0;          // a row's groups of four are aligned
  for (int e = rank * NTHREADS + tid; e < quads * g.M; e += ranks * NTHREADS) {
    const int q = e % quads, m = e / quads;
    const int j = block * quads * 4 + q * 4;   // first of the four outputs
    if (j >= outs) continue;
    const int live = min(4, outs - j);
    float y[4];
    total(gated ? (q / 4) * 32 + (q % 4) * 4 : q * 4, m, y);
    const int n = gated ? (j / 32) * 64 + j % 32 : j;
#pragma unroll
    for (int i = 0; i < 4; ++i) if (g.bias && i < live) y[i] += g.bias[n + i];
    if (gated) {
      float up[4];
      total((q / 4) * 32 + (q % 4) * 4 + 16, m, up);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = y[i] / (1.f + expf(-y[i])) * (up[i] + (g.bias ? g.bias[n + 32 + i] : 0.f));
    } else if (g.epilogue == EPI_GELU) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = gelu_f(y[i], g.gelu_tanh);
    }
    const size_t at = (size_t)m * outs + j;
    if (g.epilogue == EPI_RESIDUAL) {
      float* c = reinterpret_cast<float*>(g.c) + at;
      if (vectors) {
        const float4 x = *reinterpret_cast<const float4*>(c);
        *reinterpret_cast<float4*>(c) = make_float4(x.x + y[0], x.y + y[1], x.z + y[2], x.w + y[3]);
      } else {
        for (int i = 0; i < live; ++i) c[i] += y[i];
      }
    } else {
      bf16* c = reinterpret_cast<bf16*>(g.c) + at;
      if (vectors) *reinterpret_cast<uint2*>(c) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
      else for (int i = 0; i < live; ++i) c[i] = __float2bfloat16_rn(y[i]);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Direct: a lane's 16 consecutive weights are its operands of four instructions (the k-index of a step is permuted, and a is
// read in the same order), so a weight passes from the load to the tensor core without a shuffle.  The next step's weights
// are loaded before the current ones are used; 16 warps an SM then have 64 KB on their way.
// ---------------------------------------------------------------------------------------------
template <int NT, bool WIDE, bool LONG>
__global__ void __launch_bounds__(THREADS, 2)
linear_direct_kernel(const LinearArgs g) {
  constexpr int COLS = 8 * NT, LD = COLS + 1;
  constexpr int ROWS = BLOCK_ROWS;
  __shared__ __align__(16) float red[WARPS * ROWS * LD];
  float* const part = red;
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
    for (int j = 0; j < 2; ++j) wp[i][j] = g.w + (size_t)min(row0 + i * tile_stride + j * 8 + gq, g.N - 1) * g.K + 16 * tq;
  const bf16* ap[NT];
  bool live[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    live[n] = n * 8 + gq < g.M;
    ap[n] = g.a + (size_t)(live[n] ? n * 8 + gq : 0) * g.K + 16 * tq;
  }
  float acc[2][NT][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;

  begin_after_previous();
  Vec wb[2][2];                                // [tile][row]
  auto load_w = [&](int k) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) load_vec<WIDE, true>(wb[i][j], wp[i][j], k, g.K - 16 * tq, true);
  };
  const int stride = STEP * WARPS * ranks;
  int k = STEP * (rank * WARPS + warp);
  load_w(k);
  // The tensor core truncates where fp32 addition rounds, which adds up over a long chain (1.7e-3 of the result over K = 2^24): LONG
  // ones go to shared memory every SUM_STEPS steps, and are added there in fp32.  (In every layer that costs a tenth: 1 x 3584 x 4608
  // 8.4 -> 9.2 us.)
  auto sum_at = [&](int i, int n, int j) { return red + (warp * ROWS + i * 16 + j * 8 + gq) * LD + n * 8 + 2 * tq; };
  int steps = 0;
  auto leave_sums = [&]() {
    const bool more = LONG && steps > SUM_STEPS;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float* const dst = sum_at(i, n, j);
          dst[0] = acc[i][n][2 * j] + (more ? dst[0] : 0.f);
          dst[1] = acc[i][n][2 * j + 1] + (more ? dst[1] : 0.f);
          if (LONG) acc[i][n][2 * j] = acc[i][n][2 * j + 1] = 0.f;
        }
  };
  for (; k < g.K; k += stride) {
    if (LONG) {
      if (steps > 0 && steps % SUM_STEPS == 0) leave_sums();
      ++steps;
    }
    Vec ab[NT], cur[2][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) load_vec<WIDE, false>(ab[n], ap[n], k, g.K - 16 * tq, live[n]);
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) cur[i][j] = wb[i][j];
    load_w(k + stride);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int n = 0; n < NT; ++n)
          mma_bf16(acc[i][n], cur[i][0].r[2 * q], cur[i][1].r[2 * q], cur[i][0].r[2 * q + 1], cur[i][1].r[2 * q + 1], ab[n].r[2 * q],
                   ab[n].r[2 * q + 1]);
  }

  // ---- the warps' sums, then the cluster's
  leave_sums();
  __syncthreads();
  float sums[ROWS * COLS / THREADS];
#pragma unroll
  for (int i = 0; i < ROWS * COLS / THREADS; ++i) {
    const int e = tid + i * THREADS;
    sums[i] = 0.f;
    if (e < ROWS * g.M) {
#pragma unroll
      for (int v = 0; v < WARPS; ++v) sums[i] += red[(v * ROWS + e % ROWS) * LD + e / ROWS];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ROWS * COLS / THREADS; ++i) {
    const int e = tid + i * THREADS;
    if (e < ROWS * g.M) part[e] = sums[i];
  }
  if (ranks > 1) cluster.sync(); else __syncthreads();
  finish<ROWS, THREADS>(g, cluster, part, ROWS, block, ranks, rank);
  if (ranks > 1) cluster.sync();               // a block's sums stay until its neighbours have read them
}

// ---------------------------------------------------------------------------------------------
// Ring: one warp copies, four compute, up to 32 weight rows each.  100 KB a block, two blocks an SM, about 160 KB of weights on
// their way.  A rank of a cluster takes every ranks-th step of 64 along K.
// ---------------------------------------------------------------------------------------------
constexpr int RING_ROWS = 128 /* at most */, RING_WARPS = 4, RING_THREADS = 32 * (RING_WARPS + 1);
template <int NT> struct Ring {
  static constexpr int W_BYTES = RING_ROWS * 128, A_BYTES = 8 * NT * 128, STAGE = W_BYTES + A_BYTES;
  static constexpr int STAGES = 5;
  static constexpr int SMEM = 1024 + STAGES * STAGE + 256;
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}

template <int NT>
__global__ void __launch_bounds__(RING_THREADS, 2)
linear_ring_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap amap, const LinearArgs g, const int rows) {
  using R = Ring<NT>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const gen = smem_raw + (base - raw);
  const uint32_t bars = base + R::STAGES * R::STAGE;
  auto full = [&](int s) { return bars + 8u * (uint32_t)s; };
  auto empty = [&](int s) { return bars + 8u * (uint32_t)(R::STAGES + s); };
  volatile int* const abort_flag = reinterpret_cast<volatile int*>(gen + R::STAGES * R::STAGE + 16 * R::STAGES);
  cg::cluster_group cluster = cg::this_cluster();
  const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int block = blockIdx.x / ranks;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int steps = (g.K + 63) / 64, mine = (steps - rank + ranks - 1) / ranks;      // k-steps rank, rank + ranks, ...
  const bool gated = g.epilogue == EPI_SWIGLU;

  if (tid == 0) {
    for (int s = 0; s < R::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), RING_WARPS); }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&wmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&amap) : "memory");
  }
  __syncthreads();
  begin_after_previous();

  bool ok = true;
  float acc[2][NT][4];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
  // first row of the warp's two tiles inside the block: neighbours, or 16 gate rows and the up rows of the same outputs
  const int r0 = gated ? (warp >> 1) * 64 + (warp & 1) * 16 : warp * 32, r1 = r0 + (gated ? 32 : 16);
  if (warp == RING_WARPS) {
    if (lane == 0) {
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      for (; issued < mine; ++issued) {
        ok = mbar_wait(empty(stage), phase ^ 1u, abort_flag);
        if (!ok) break;
        const uint32_t dst = base + stage * R::STAGE;
        const int x = (rank + issued * ranks) * 64;
        mbar_arrive_expect_tx(full(stage), (uint32_t)rows * 128u + R::A_BYTES);
        tma_load_2d(dst, &wmap, full(stage), x, block * rows);
        tma_load_2d(dst + R::W_BYTES, &amap, full(stage), x, 0);
        if (++stage == R::STAGES) { stage = 0; phase ^= 1u; }
      }
      // copies have to land before the ring's memory is used for the sums, also if nobody waits for them any more
      for (int i = 0; i < R::STAGES && i < issued; ++i) {
        if (--stage < 0) { stage = R::STAGES - 1; phase ^= 1u; }
        int given_up = 0;
        mbar_wait(full(stage), phase, &given_up);
      }
    }
  } else {
    const int arow = (lane & 7) + ((lane >> 3) & 1) * 8, achunk = lane >> 4;          // of a 16 x 16 tile of w
    const int brow = (lane & 7) + (lane >> 4) * 8, bchunk = (lane >> 3) & 1;          // of two 8 x 16 tiles of a
    auto at = [&](int row, int chunk) { return (uint32_t)(row * 128 + ((chunk ^ (row & 7)) << 4)); };
    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < mine; ++i) {
      if (ok) ok = mbar_wait_warp(full(stage), phase, abort_flag);
      if (ok) {
        const uint32_t wb = base + stage * R::STAGE, ab = wb + R::W_BYTES;
        // The tensor core truncates where fp32 addition rounds, which adds up over a long chain (1.8e-6 of the result over K =
        // 18 944): a stage's products get accumulators of their own, and the stages are added in fp32.
        float part_acc[2][NT][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n) part_acc[i][n][0] = part_acc[i][n][1] = part_acc[i][n][2] = part_acc[i][n][3] = 0.f;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
          uint32_t w0[4], w1[4];
          ldmatrix4(wb + at(r0 + arow, 2 * ks + achunk), w0);
          ldmatrix4(wb + at(r1 + arow, 2 * ks + achunk), w1);
#pragma unroll
          for (int n = 0; n < NT; n += 2) {
            uint32_t b[4];
            ldmatrix4(ab + at(NT == 1 ? (brow & 7) : n * 8 + brow, 2 * ks + bchunk), b);
            mma_bf16(part_acc[0][n], w0[0], w0[1], w0[2], w0[3], b[0], b[1]);
            mma_bf16(part_acc[1][n], w1[0], w1[1], w1[2], w1[3], b[0], b[1]);
            if (n + 1 < NT) {
              mma_bf16(part_acc[0][(n + 1) % NT], w0[0], w0[1], w0[2], w0[3], b[2], b[3]);
              mma_bf16(part_acc[1][(n + 1) % NT], w1[0], w1[1], w1[2], w1[3], b[2], b[3]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][n][j] += part_acc[i][n][j];
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(stage));
      }
      if (++stage == R::STAGES) { stage = 0; phase ^= 1u; }
    }
  }
  __syncthreads();                             // the ring is idle: its memory takes the sums, [m][row of the block]
  float* const part = reinterpret_cast<float*>(gen);
  if (warp < RING_WARPS) {
    const int gq = lane >> 2, tq = lane & 3;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[(n * 8 + 2 * tq + (j & 1)) * RING_ROWS + warp * 32 + i * 16 + gq + (j >> 1) * 8] = acc[i][n][j];
  }
  if (ranks > 1) cluster.sync(); else __syncthreads();
  finish<RING_ROWS, RING_THREADS>(g, cluster, part, rows, block, ranks, rank);
  if (tid == 0 && *abort_flag && g.status) atomicMax(g.status, (int)DS_WAIT_EXPIRED);
  if (ranks > 1) cluster.sync();               // a block's sums stay until its neighbours have read them
}

template <int NT>
cudaError_t launch_direct(const LinearArgs& g, cudaStream_t s) {
  const int blocks = cdiv(g.N, BLOCK_ROWS);
  int ranks = 1;                               // two blocks an SM, each with two steps or more for every warp
  while (ranks < MAX_CLUSTER && blocks * ranks * 2 <= 2 * 148 && g.K >= 2 * STEP * WARPS * ranks * 2) ranks *= 2;
  const bool wide = g.K % 16 == 0 && ((reinterpret_cast<uintptr_t>(g.a) | reinterpret_cast<uintptr_t>(g.w)) & 31u) == 0;
  Launch l(blocks * ranks, THREADS, 0, s, ranks);
  ET_COUNT_LAUNCH();
  if (g.K > STEP * WARPS * ranks * SUM_STEPS)
    return wide ? cudaLaunchKernelEx(&l.cfg, linear_direct_kernel<NT, true, true>, g)
                : cudaLaunchKernelEx(&l.cfg, linear_direct_kernel<NT, false, true>, g);
  return wide ? cudaLaunchKernelEx(&l.cfg, linear_direct_kernel<NT, true, false>, g)
              : cudaLaunchKernelEx(&l.cfg, linear_direct_kernel<NT, false, false>, g);
}

template <int NT>
cudaError_t launch_ring(const LinearArgs& g, cudaStream_t s) {
  using R = Ring<NT>;
  // clusters of each size (of one: blocks) that the card holds at once, per device, looked up once
  constexpr int DEVICES = 64;
  static std::atomic<int> resident[DEVICES][MAX_CLUSTER + 1];       // zero: not looked up; [1] is set last
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= DEVICES) return cudaErrorInvalidDevice;
  if (!resident[dev][1]) {
    e = cudaFuncSetAttribute(linear_ring_kernel<NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, R::SMEM);
    if (e != cudaSuccess) return e;
    for (int ranks = MAX_CLUSTER; ranks >= 2; --ranks) {
      Launch probe(ranks, RING_THREADS, R::SMEM, s, ranks);
      int n = 0;
      e = cudaOccupancyMaxActiveClusters(&n, linear_ring_kernel<NT>, &probe.cfg);
      if (e != cudaSuccess) return e;
      resident[dev][ranks] = n > 0 ? n : 1;
    }
    int sms = 0, per_sm = 0;
    e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, linear_ring_kernel<NT>, RING_THREADS, R::SMEM);
    if (e != cudaSuccess) return e;
    resident[dev][1] = sms * per_sm > 0 ? sms * per_sm : 1;
  }
  const int steps = cdiv(g.K, STEP);
  int ranks = 1;
  for (int r = 2; r <= MAX_CLUSTER && steps >= 4 * r; ++r) if (cdiv(g.N, RING_ROWS) <= resident[dev][r]) ranks = r;
  // Below eight ranks a block has as few rows (a swizzle pattern's 8 at a time) as the number of waves that blocks of 128 need
  // allows, so that the last wave is full too.  128 / these in us: 1 x 3584 x 40000 54.0 / 48.6 (72 rows), 1 x 8192 x 40000 119.0 /
  // 106.6 (72), 32 x 3584 x 50000 76.4 / 73.4 (88), 1 x 3584 x 152064 164.1 / 163.2 (104), 32 x 2048 x 22000 22.2 / 22.0 (80), 32 x
  // 520 x 8000 8.6 / 7.7 (56), 19 x 10152 x 9728 41.4 / 40.5 (112), 12 x 1504 x 5000 6.7 / 7.1, 32 x 2048 x 152064 120.9 / 124.6
  // (104).  Gated rows stay in groups of 64, of which one is too few for a block (3584 x 38912 54.8 / 60.1).  At eight ranks
  // fewer rows gain nothing (13 x 3584 x 2048 6.8 / 7.0).
  int rows = RING_ROWS;
  if (g.epilogue != EPI_SWIGLU && ranks < MAX_CLUSTER) {
    const int places = cdiv(cdiv(g.N, RING_ROWS), resident[dev][ranks]) * resident[dev][ranks];
    rows = cdiv(cdiv(g.N, places), 8) * 8;
  }
  const int blocks = cdiv(g.N, rows);
  TmaDesc w, a;
  if (!make_tma_2d_bf16(&w, g.w, g.N, g.K, rows, nullptr) || !make_tma_2d_bf16(&a, g.a, g.M, g.K, 8 * NT, nullptr)) return cudaErrorUnknown;
  Launch l(blocks * ranks, RING_THREADS, R::SMEM, s, ranks);
  ET_COUNT_LAUNCH();
  return cudaLaunchKernelEx(&l.cfg, linear_ring_kernel<NT>, *reinterpret_cast<const CUtensorMap*>(w.bytes),
                            *reinterpret_cast<const CUtensorMap*>(a.bytes), g, rows);
}

}  // namespace

cudaError_t launch_linear_rows(const bf16* a, const bf16* w, const float* bias, void* c, int M, int N, int K, int epilogue,
                               int gelu_tanh, int* status, cudaStream_t s) {
  const LinearArgs g{a, w, bias, c, M, N, K, epilogue, gelu_tanh, status};
  // The ring takes over where the weights are many, much sooner with more than 8 rows (direct reads a again for every 32 weight
  // rows), unless there are too few weight rows for its blocks.  Direct / ring in us: 1 x 3584 x 4608 8.4 / 8.8, 8 x 3584 x 9000
  // 12.9 / 14.1, 8 x 18944 x 3584 24.9 / 23.9; 13 x 2048 x 2048 6.0 / 5.7, 13 x 3584 x 2048 8.0 / 6.8, 13 x 18944 x 3584 28.2 /
  // 24.3; 20 x 1024 x 900 4.2 / 5.2; 32 x 2048 x 2048 7.7 / 6.6; 32 x 16384 x 512 10.9 / 13.9.
  const long long weights = (long long)N * K;
  const bool ring = M <= 8 ? weights > (1ll << 25) : N >= 1024 && weights * ((M + 7) / 8) > 12000000;
  if (ring) return M <= 8 ? launch_ring<1>(g, s) : M <= 16 ? launch_ring<2>(g, s) : launch_ring<4>(g, s);
  return M <= 8 ? launch_direct<1>(g, s) : M <= 16 ? launch_direct<2>(g, s) : M <= 24 ? launch_direct<3>(g, s) : launch_direct<4>(g, s);
}

}  // namespace et
