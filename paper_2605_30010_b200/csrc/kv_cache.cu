// The paged key / value cache: rows of a projection go in (turned and quantised on the way), rows come back.
#include <cuda_fp8.h>

#include "decode.cuh"

namespace et {

namespace {

constexpr int THREADS = 256;
constexpr int MAX_ROWS = 16;         // rows of one step of a block

// Where a row goes, found once per row by one thread of the block.
struct RowPlace {
  int seq, page, place;              // seq < 0: nothing to do for this row
  long long pos;
};

// The sequence of a row is the last one whose offset is not behind it (a binary search); a row outside its sequence's
// run is padding (or the offsets are not ascending) and is skipped.
__device__ RowPlace place_of_row(const PagedCache& c, const PagedRows& r, int row) {
  RowPlace p;
  p.seq = -1; p.page = p.place = 0; p.pos = 0;
  int s = row, first = row;
  if (r.offsets) {
    int lo = 0, hi = r.n_seq;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(r.offsets + mid) <= row) lo = mid; else hi = mid;
    }
    s = lo;
    first = __ldg(r.offsets + s);
    if (row < first || row >= __ldg(r.offsets + s + 1)) return p;
  }
  const int start = __ldg(r.start + s);
  if (start < 0) return p;
  p.pos = (long long)start + (row - first);
  if (!paged_place(c, r.table, r.max_pages, s, p.pos, r.status, p.page, p.place)) return p;
  p.seq = s;
  return p;
}

// First row of data (in rows of head_dim values) of a (page, plane, head, place).
__device__ __forceinline__ size_t cache_row(const PagedCache& c, int page, int plane, int head, int place) {
  return ((((size_t)page * 2 + plane) * c.kv_heads + head) << c.page_shift) + place;
}

// The smallest e in [-127, 127] with top <= 448 * 2^e, 448 = 1.75 * 2^8: read off the bits of top = m * 2^E.
__device__ __forceinline__ int e4m3_exponent(float top) {
  const int bits = __float_as_int(top);                      // top >= 0 and finite
  const int e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000 ? 1 : 0);
  return max(e, -127);                                       // at most 127 - 8 + 1
}
// 2^e for e in [-127, 127], exact (2^-127 is a subnormal)
__device__ __forceinline__ float pow2(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 1 << 22); }

__device__ __forceinline__ uint2 to_e4m3(const float (&x)[8], float inv) {
  uint32_t w[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float a = x[2 * k], b = x[2 * k + 1];
    // an infinity becomes NaN, like NaN itself: the saturating conversion would make it an ordinary value
    const float2 v = make_float2(fabsf(a) <= 3.402823466e38f ? a * inv : __int_as_float(0x7fffffff),
                                 fabsf(b) <= 3.402823466e38f ? b * inv : __int_as_float(0x7fffffff));
    w[k] = (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);
  }
  return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

__device__ __forceinline__ void unpack8(const uint4& v, float (&x)[8]) {
  const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
  for (int k = 0; k < 4; ++k) { const float2 f = __bfloat1622float2(p[k]); x[2 * k] = f.x; x[2 * k + 1] = f.y; }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint4 v;
  __nv_bfloat162* p = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
  for (int k = 0; k < 4; ++k) p[k] = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
  return v;
}

// ---------------------------------------------------------------------------------------------
// Append.  A thread takes elements i .. i+7 and i + d/2 .. i + d/2 + 7 of one head of one row, the two halves that the
// rotation pairs; d/16 neighbouring threads hold a head and find its maximum with shuffles, so the row is read once and
// written once.  The angle of position p and pair i is p * theta^(-2i/d): the host gives each frequency as a 64-bit
// fraction of a turn, so that p * f modulo 2^64 is the exact fraction of a turn however far p is; (cos, sin) of a block's
// rows are computed once and shared by all heads.  Bound by memory.
// ---------------------------------------------------------------------------------------------
template <int DH, bool E4M3, bool ROTATE>
__global__ void __launch_bounds__(THREADS)
kv_append_kernel(const bf16* __restrict__ qkv, long long row_stride, int heads, PagedCache c, PagedRows r,
                 const __grid_constant__ RopeTurns turns, bf16* __restrict__ q_out, int* __restrict__ new_len, int step_rows) {
  constexpr int HALF = DH / 2, CHUNKS = DH / 16;
  __shared__ RowPlace places[MAX_ROWS];
  __shared__ float2 angle[ROTATE ? MAX_ROWS * HALF : 1];
  const int tid = threadIdx.x;
  const int skip = ROTATE ? 0 : heads;                       // query heads that need nothing done
  const int units_row = (heads - skip + 2 * c.kv_heads) * CHUNKS;

  if (new_len && blockIdx.x == 0) {
    for (int s = tid; s < r.n_seq; s += THREADS) {
      const int start = r.start[s];
      const long long n = r.offsets ? max(0, r.offsets[s + 1] - r.offsets[s]) : 1;
      const long long cap = (long long)r.max_pages << c.page_shift;
      new_len[s] = start < 0 ? start : (int)min((long long)start + n, max(cap, (long long)start));
    }
  }

  for (long long row0 = (long long)blockIdx.x * step_rows; row0 < r.rows; row0 += (long long)gridDim.x * step_rows) {
    const int n = (int)min((long long)step_rows, r.rows - row0);
    if (tid < n) places[tid] = place_of_row(c, r, (int)row0 + tid);
    __syncthreads();
    if (ROTATE) {
      for (int j = tid; j < n * HALF; j += THREADS) {
        const unsigned long long turn = (unsigned long long)places[j / HALF].pos * turns.f[j % HALF];
        float sn, cs;
        sincospif(__ll2float_rn((long long)turn) * 1.0842021724855044e-19f, &sn, &cs);    // 2^-63: half turns in [-1, 1)
        angle[j] = make_float2(cs, sn);
      }
      __syncthreads();
    }
    const int total = n * units_row;
    for (int u0 = 0; u0 < total; u0 += THREADS) {            // whole warps stay together for the shuffles
      const int u = u0 + tid;
      const bool live = u < total;
      const int rl = live ? u / units_row : 0, unit = live ? u - rl * units_row : 0;
      const int head = skip + unit / CHUNKS, chunk = unit % CHUNKS;
      const RowPlace p = places[rl];
      const bool work = live && p.seq >= 0;
      float a[8] = {0, 0, 0, 0, 0, 0, 0, 0}, b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (work) {
        const bf16* src = qkv + (row0 + rl) * row_stride + (size_t)head * DH + chunk * 8;
        unpack8(__ldg(reinterpret_cast<const uint4*>(src)), a);
        unpack8(__ldg(reinterpret_cast<const uint4*>(src + HALF)), b);
      }
      if (ROTATE && head < heads + c.kv_heads) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float2 t = angle[rl * HALF + chunk * 8 + k];
          const float x = a[k], y = b[k];
          a[k] = x * t.x - y * t.y;
          b[k] = y * t.x + x * t.y;
        }
      }
      if (ROTATE && head < heads) {
        if (work) {
          uint4* dst = reinterpret_cast<uint4*>(q_out + ((size_t)(row0 + rl) * heads + head) * DH + chunk * 8);
          dst[0] = pack8(a);
          dst[HALF / 8] = pack8(b);
        }
      }
      float top = 0.f;
      if (E4M3) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = fabsf(a[k]), y = fabsf(b[k]);
          if (x <= 3.402823466e38f) top = fmaxf(top, x);
          if (y <= 3.402823466e38f) top = fmaxf(top, y);
        }
#pragma unroll
        for (int o = CHUNKS / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      }
      if (work && head >= heads) {
        const int kvh = head - heads;
        const int plane = kvh >= c.kv_heads ? 1 : 0;
        const size_t at = cache_row(c, p.page, plane, kvh - plane * c.kv_heads, p.place);
        if (E4M3) {
          const int e = e4m3_exponent(top);
          const float inv = pow2(-e);
          uint2* dst = reinterpret_cast<uint2*>(c.data + at * DH + chunk * 8);
          dst[0] = to_e4m3(a, inv);
          dst[HALF / 8] = to_e4m3(b, inv);
          if (chunk == 0) c.scale[at] = (uint8_t)(e + 127);
        } else {
          uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<bf16*>(c.data) + at * DH + chunk * 8);
          dst[0] = pack8(a);
          dst[HALF / 8] = pack8(b);
        }
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------
// Read: 16 bytes of the cache a thread (8 bf16 or 16 e4m3 values).  Bound by memory.
// ---------------------------------------------------------------------------------------------
template <int DH, bool E4M3>
__global__ void __launch_bounds__(THREADS)
kv_read_kernel(bf16* __restrict__ out, long long row_stride, PagedCache c, PagedRows r, int step_rows) {
  constexpr int VEC = E4M3 ? 16 : 8, CHUNKS = DH / VEC;
  __shared__ RowPlace places[MAX_ROWS];
  const int tid = threadIdx.x;
  const int units_row = 2 * c.kv_heads * CHUNKS;
  for (long long row0 = (long long)blockIdx.x * step_rows; row0 < r.rows; row0 += (long long)gridDim.x * step_rows) {
    const int n = (int)min((long long)step_rows, r.rows - row0);
    if (tid < n) places[tid] = place_of_row(c, r, (int)row0 + tid);
    __syncthreads();
    const int total = n * units_row;
    for (int u = tid; u < total; u += THREADS) {
      const int rl = u / units_row, unit = u - rl * units_row;
      const int head = unit / CHUNKS, chunk = unit % CHUNKS;
      const RowPlace p = places[rl];
      if (p.seq < 0) continue;
      const int plane = head >= c.kv_heads ? 1 : 0;
      const size_t at = cache_row(c, p.page, plane, head - plane * c.kv_heads, p.place);
      uint4* dst = reinterpret_cast<uint4*>(out + (row0 + rl) * row_stride + (size_t)head * DH + chunk * VEC);
      if (E4M3) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(c.data + at * DH + chunk * VEC));
        const float f = pow2((int)__ldg(c.scale + at) - 127);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        float x[16];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[k >> 1] >> (16 * (k & 1))), __NV_E4M3);
          const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&h));
          x[2 * k] = y.x * f; x[2 * k + 1] = y.y * f;
        }
        float lo[8], hi[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) { lo[k] = x[k]; hi[k] = x[8 + k]; }
        dst[0] = pack8(lo);
        dst[1] = pack8(hi);
      } else {
        *dst = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(c.data) + at * DH + chunk * VEC));
      }
    }
    __syncthreads();
  }
}

// Rows of one step: enough that a block has a few units for every thread, few enough that every SM gets rows.
int rows_per_step(int rows, int units_row) {
  const int enough = (4 * THREADS + units_row - 1) / units_row;
  const int spread = rows / (148 * 4) + 1;
  const int n = enough < spread ? enough : spread;
  return n < 1 ? 1 : n > MAX_ROWS ? MAX_ROWS : n;
}
int blocks_for(int rows, int step) { return (int)std::min<long long>(((long long)rows + step - 1) / step, 148 * 8); }

}  // namespace

void launch_kv_append(const PagedCache& c, const PagedRows& r, const bf16* qkv, long long row_stride, int heads, bool rotate,
                      const RopeTurns& turns, bf16* q_out, int* new_len, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  const int step = rows_per_step(r.rows, ((rotate ? heads : 0) + 2 * c.kv_heads) * (c.head_dim / 16));
  const int blocks = blocks_for(r.rows, step);
#define ET_APPEND(D, E, R) kv_append_kernel<D, E, R><<<blocks, THREADS, 0, s>>>(qkv, row_stride, heads, c, r, turns, q_out, new_len, step)
#define ET_APPEND_D(D)                                                       \
  do {                                                                       \
    if (c.scale) { if (rotate) ET_APPEND(D, true, true); else ET_APPEND(D, true, false); }   \
    else { if (rotate) ET_APPEND(D, false, true); else ET_APPEND(D, false, false); }         \
  } while (0)
  if (c.head_dim == 64) ET_APPEND_D(64); else ET_APPEND_D(128);
#undef ET_APPEND_D
#undef ET_APPEND
}

void launch_kv_read(const PagedCache& c, const PagedRows& r, bf16* out, long long row_stride, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  const int step = rows_per_step(r.rows, 2 * c.kv_heads * c.head_dim / (c.scale ? 16 : 8));
  const int blocks = blocks_for(r.rows, step);
#define ET_READ(D, E) kv_read_kernel<D, E><<<blocks, THREADS, 0, s>>>(out, row_stride, c, r, step)
  if (c.head_dim == 64) { if (c.scale) ET_READ(64, true); else ET_READ(64, false); }
  else { if (c.scale) ET_READ(128, true); else ET_READ(128, false); }
#undef ET_READ
}

}  // namespace et
