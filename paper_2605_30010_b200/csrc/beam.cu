// Beam search: the k best continuations of each request's beams over the vocabulary.
//
// Every logit is read once, and that bounds it: score + x - log(sum of exp(x)) orders a beam's tokens as x does, so one pass finds the
// best k of x, their largest and the sum together.  A beam's logits are cut into segments, one block each (as many as fill the card); a
// second, small kernel joins a request's segments and beams in a fixed order.
//
//   * Which of a chunk's 4 096 logits can be among the best k?  In a segment's first chunk: those that are not below the k-th largest
//     of the maxima of 32 groups of them, for k groups have at least that.  In the others: those above the k-th best so far; a lower
//     token comes first among equal ones, so later equal ones need not be looked at.  What passes goes to a list in shared memory,
//     which is cut back to k entries, in order, when it is long.
//   * The sum is a running one against a running maximum, each thread's own; a thread's maximum seldom moves after its first chunk.
//   * Scores are compared in 64 bits: a beam's logarithm of its sum is off by a few 2^-24, which the beams have alike or nearly so.
#include "decode.cuh"
#include "earlytom_pages.h"

namespace et {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, EACH = 16, CHUNK = THREADS * EACH;
static_assert(CHUNK == ET_BEAM_CHUNK, "workspace");
constexpr int K_MAX = 64, BEAMS_MAX = 32, SEGMENTS_MAX = 64;
constexpr int LONG = 192, LIST = CHUNK + LONG;      // the list is cut back when it has more than LONG entries; a chunk adds CHUNK at most
constexpr int RANKED = 1024;                        // up to so many entries each one's rank is counted
constexpr float LOG2E = 1.4426950408889634f;

struct Select {
  const void* logits;
  long long stride;
  const float* scores;            // may be NULL
  const unsigned char* done;      // may be NULL
  int beams, vocab, k, eos, segments, chunks_each;
  unsigned char* workspace;
  int* parent;
  int* token;
  float* new_scores;
  unsigned char* new_done;        // may be NULL
};

// What a segment leaves: its best k (value, token) in order, (-infinity, -1) behind the last, and (maximum, sum).
struct Entry { float value; int token; };
__host__ __device__ constexpr size_t segment_bytes(int k) { return 8 * (size_t)k + 16; }
__device__ __forceinline__ unsigned char* segment_of(const Select& a, int row, int segment) {
  return a.workspace + ((size_t)row * a.segments + segment) * segment_bytes(a.k);
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }
__device__ __forceinline__ float score_of(const Select& a, int row) { return a.scores ? a.scores[row] : 0.f; }
__device__ __forceinline__ bool done_of(const Select& a, int row) { return a.done && a.done[row]; }
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The list's best k entries, in order, to its front.  All threads; the list is complete.
__device__ __forceinline__ int cut_back(Entry* list, int n, int k, Entry* best, uint2* reduce) {
  const int tid = threadIdx.x;
  auto before = [](const Entry& a, const Entry& b) { return a.value > b.value || (a.value == b.value && a.token < b.token); };
  const int kept = min(n, k);
  if (n <= RANKED) {
    Entry mine[RANKED / THREADS];
    int rank[RANKED / THREADS];
#pragma unroll
    for (int j = 0; j < RANKED / THREADS; ++j) {
      if (j * THREADS >= n) break;
      rank[j] = k;
      const int e = tid + j * THREADS;
      if (e >= n) continue;
      mine[j] = list[e];
      int r = 0;
      for (int i = 0; i < n; ++i) r += before(list[i], mine[j]);
      rank[j] = r;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < RANKED / THREADS; ++j) {
      if (j * THREADS >= n) break;
      if (rank[j] < k) list[rank[j]] = mine[j];
    }
  } else {
    // many values that are equal or come in an unlucky order: the best one, k times
    for (int r = 0; r < kept; ++r) {
      Entry top{-INFINITY, 0x7fffffff};
      int at = -1;
      for (int e = tid; e < n; e += THREADS) if (before(list[e], top)) { top = list[e]; at = e; }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        Entry other;
        other.value = __shfl_xor_sync(0xffffffffu, top.value, o);
        other.token = __shfl_xor_sync(0xffffffffu, top.token, o);
        const int other_at = __shfl_xor_sync(0xffffffffu, at, o);
        if (before(other, top)) { top = other; at = other_at; }
      }
      if ((tid & 31) == 0) { best[WARPS + (tid >> 5)] = top; reduce[tid >> 5].x = at; }
      __syncthreads();
      if (tid == 0) {
        int w = 0;
        for (int i = 1; i < WARPS; ++i) if (before(best[WARPS + i], best[WARPS + w])) w = i;
        best[2 * WARPS + r] = best[WARPS + w];
        list[reduce[w].x] = Entry{-INFINITY, 0x7fffffff};
      }
      __syncthreads();
    }
    if (tid < kept) list[tid] = best[2 * WARPS + tid];
  }
  __syncthreads();
  return kept;
}

template <bool FP32, bool ALIGNED>
__global__ void __launch_bounds__(THREADS)
beam_scan_kernel(const __grid_constant__ Select a) {
  constexpr int SIZE = FP32 ? 4 : 2, VEC = 16 / SIZE, SLOTS = EACH / VEC;
  extern __shared__ Entry list[];                   // [LIST]
  __shared__ int listed;
  __shared__ float group_top[64];
  __shared__ Entry best[2 * WARPS + K_MAX];
  __shared__ uint2 reduce[WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, segment = blockIdx.x, row = blockIdx.y;
  begin_after_previous();
  if (done_of(a, row) || !finite(score_of(a, row))) return;
  const unsigned char* const src = static_cast<const unsigned char*>(a.logits) + (size_t)row * a.stride * SIZE;
  // Rows may begin anywhere.  Which thread takes which logit does not depend on it, so that equal rows have equal sums: where rows are
  // not aligned, a slot's elements are cut out of the two 16-byte vectors that they lie in.
  const int shift = ALIGNED ? 0 : (int)(reinterpret_cast<uintptr_t>(src) & 15) / SIZE;
  const int first = segment * a.chunks_each * CHUNK, last = (int)min((long long)first + (long long)a.chunks_each * CHUNK, (long long)a.vocab);
  auto place = [&](int j) { return (j * THREADS + tid) * VEC; };           // of this thread's j-th slot, in the chunk
  constexpr int WORDS = ALIGNED ? 4 : 8;
  auto inside = [&](int e) { return e - shift >= 0 && e - shift + (ALIGNED ? 1 : 2) * VEC <= a.vocab; };
  auto load = [&](int at, uint32_t (&raw)[SLOTS][WORDS]) {
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      const int e0 = at + place(j);
      if (inside(e0)) {
        const unsigned char* const p = src + (ptrdiff_t)(e0 - shift) * SIZE;
#pragma unroll
        for (int w = 0; w < WORDS; w += 4)
          asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(raw[j][w]), "=r"(raw[j][w + 1]), "=r"(raw[j][w + 2]), "=r"(raw[j][w + 3]) : "l"(p + 4 * w));
      } else {
        // the row's ends, one by one, as cut() leaves them
#pragma unroll
        for (int w = 0; w < 4; ++w) raw[j][w] = 0;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          uint32_t bits = FP32 ? 0xff800000u : 0xff80u;                     // minus infinity
          if (e0 + v < last) bits = FP32 ? *reinterpret_cast<const uint32_t*>(src + (size_t)(e0 + v) * SIZE) : *reinterpret_cast<const uint16_t*>(src + (size_t)(e0 + v) * SIZE);
          if (FP32) raw[j][v & 3] = bits; else raw[j][v / 2] |= bits << (16 * (v & 1));
        }
      }
    }
  };
  auto cut = [&](uint32_t (&w)[WORDS]) {
    if constexpr (!ALIGNED) {
      if (!FP32 && (shift & 1))
#pragma unroll
        for (int i = 0; i < 7; ++i) w[i] = __byte_perm(w[i], w[i + 1], 0x5432);
      const int words = FP32 ? shift : shift >> 1;
      if (words & 1)
#pragma unroll
        for (int i = 0; i < 6; ++i) w[i] = w[i + 1];
      if (words & 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = w[i + 2];
    }
  };
  uint32_t raw[SLOTS][WORDS];
  if (first < last) load(first, raw);
  if (tid == 0) listed = 0;
  float m = -INFINITY, s = 0.f, bar = -INFINITY;    // bar: what a logit has to reach or, behind the first chunk, to pass
  int n = 0;
  bool begun = false;
  for (int at = first; at < last; at += CHUNK) {
    float x[EACH];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      if (inside(at + place(j))) cut(raw[j]);
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        x[j * VEC + v] = __uint_as_float(FP32 ? raw[j][v & 3] : v & 1 ? raw[j][v / 2] & 0xffff0000u : raw[j][v / 2] << 16);
    }
    if (at + CHUNK < last) load(at + CHUNK, raw);   // on its way while this chunk is looked at
    float top = x[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) top = fmaxf(top, x[i]);
    if (top > m) { s *= exp2_fast((m - top) * LOG2E); m = top; }
    const float ref = m == -INFINITY ? 0.f : m;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EACH; ++i) sum[i & 3] += exp2_fast((x[i] - ref) * LOG2E);
    s += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    if (!begun) {
      float g = top;
      const int lanes = a.k <= 32 ? 8 : 4;          // of a group
      for (int o = 1; o < lanes; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
      if (lane % lanes == 0) group_top[(warp * 32 + lane) / lanes] = g;
      __syncthreads();
      if (a.k <= 32) {
        g = group_top[lane];
        // the 32 maxima in descending order
#pragma unroll
        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
          for (int o = size >> 1; o > 0; o >>= 1) {
            const float other = __shfl_xor_sync(0xffffffffu, g, o);
            g = ((lane & size) == 0) == ((lane & o) == 0) ? fmaxf(g, other) : fminf(g, other);
          }
        bar = __shfl_sync(0xffffffffu, g, a.k - 1);
      } else {
        g = fminf(group_top[lane], group_top[lane + 32]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) g = fminf(g, __shfl_xor_sync(0xffffffffu, g, o));
        bar = g;
      }
    }
    if (begun ? top > bar : top >= bar)
#pragma unroll
      for (int j = 0; j < SLOTS; ++j)
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
          const float y = x[j * VEC + v];
          if ((begun ? y > bar : y >= bar) && y > -INFINITY) list[atomicAdd(&listed, 1)] = Entry{y + 0.f, at + place(j) + v};
        }
    __syncthreads();
    n = listed;
    if (!begun || n > LONG) {
      n = cut_back(list, n, a.k, best, reduce);
      bar = n == a.k ? list[a.k - 1].value : -INFINITY;
      begun = true;
      if (tid == 0) listed = n;
    }
    __syncthreads();                                // listed is read before the next chunk adds to it
  }
  n = cut_back(list, n, a.k, best, reduce);
  unsigned char* const out = segment_of(a, row, segment);
  if (tid < a.k) reinterpret_cast<Entry*>(out)[tid] = tid < n ? list[tid] : Entry{-INFINITY, -1};
  float big = m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
  s *= m == big ? 1.f : exp2_fast((m - big) * LOG2E);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) reduce[warp] = make_uint2(__float_as_uint(big), __float_as_uint(s));
  __syncthreads();
  if (tid == 0) {
    for (int w = 0; w < WARPS; ++w) big = fmaxf(big, __uint_as_float(reduce[w].x));
    float all = 0.f;
    for (int w = 0; w < WARPS; ++w) {
      const float mw = __uint_as_float(reduce[w].x);
      all += __uint_as_float(reduce[w].y) * (mw == big ? 1.f : exp2_fast((mw - big) * LOG2E));
    }
    *reinterpret_cast<float2*>(out + 8 * (size_t)a.k) = make_float2(big, all);
  }
}

// Floats and doubles as whole numbers of the same order, above 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ unsigned long long ordered(double x) {
  const unsigned long long u = (unsigned long long)__double_as_longlong(x);
  return u ^ (u >> 63 ? ~0ull : 1ull << 63);
}

// The front of one segment's list, a few entries in registers.
struct Front {
  static constexpr int AHEAD = 4;
  const Entry* from;
  Entry e[AHEAD];
  int have, next;
  __device__ __forceinline__ void fill(int k) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      e[i] = Entry{-INFINITY, -1};
      if (from && next + i < k) {
        const float2 v = __ldcg(reinterpret_cast<const float2*>(from + next + i));
        e[i] = Entry{v.x, __float_as_int(v.y)};
      }
    }
    next += AHEAD;
    have = AHEAD;
  }
  __device__ __forceinline__ uint32_t key() const { return e[0].token < 0 ? 0u : ordered(e[0].value); }
  __device__ __forceinline__ void pop(int k) {
#pragma unroll
    for (int i = 0; i + 1 < AHEAD; ++i) e[i] = e[i + 1];
    e[AHEAD - 1] = Entry{-INFINITY, -1};
    if (--have == 0) fill(k);
  }
};

// A block joins a request: a warp each beam's segments, the first warp the beams.
__global__ void beam_join_kernel(const __grid_constant__ Select a) {
  extern __shared__ Entry beam_list[];              // [beams][k]
  __shared__ double base_s[BEAMS_MAX];
  __shared__ int count_s[BEAMS_MAX];
  const int lane = threadIdx.x & 31, beam = threadIdx.x >> 5, request = blockIdx.x, row = request * a.beams + beam, k = a.k;
  begin_after_previous();
  const float score = score_of(a, row);
  Entry* const mine = beam_list + beam * k;
  int count = 0;
  double base = 0.;
  if (!finite(score)) {
  } else if (done_of(a, row)) {
    if (lane == 0) mine[0] = Entry{0.f, a.eos};
    base = score;
    count = 1;
  } else {
    Front front[2];
    float2 part[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int segment = lane + 32 * i;
      const unsigned char* const at = segment_of(a, row, segment);
      front[i].from = segment < a.segments ? reinterpret_cast<const Entry*>(at) : nullptr;
      front[i].next = 0;
      part[i] = segment < a.segments ? __ldcg(reinterpret_cast<const float2*>(at + 8 * (size_t)k)) : make_float2(-INFINITY, 0.f);
      front[i].fill(k);
    }
    float big = fmaxf(part[0].x, part[1].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    double sum = 0.;
#pragma unroll
    for (int i = 0; i < 2; ++i) sum += part[i].y * (part[i].x == big ? 1. : exp((double)part[i].x - big));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    base = (double)score - ((double)big + log(sum));
    if (finite(big) && base >= -1.7e308 && base <= 1.7e308) {
      for (; count < k; ++count) {
        const uint32_t u0 = front[0].key(), u1 = front[1].key(), top = __reduce_max_sync(0xffffffffu, max(u0, u1));
        if (top == 0) break;
        const unsigned low = __ballot_sync(0xffffffffu, u0 == top), high = __ballot_sync(0xffffffffu, u1 == top);
        // lower segments have lower tokens
        if (low) {
          if (lane == __ffs(low) - 1) { mine[count] = front[0].e[0]; front[0].pop(k); }
        } else if (lane == __ffs(high) - 1) {
          mine[count] = front[1].e[0]; front[1].pop(k);
        }
        __syncwarp();
      }
    }
  }
  if (lane == 0) { base_s[beam] = base; count_s[beam] = count; }
  __syncthreads();
  if (beam != 0) return;
  const int n = lane < a.beams ? count_s[lane] : 0;
  base = lane < a.beams ? base_s[lane] : 0.;
  const Entry* const of = beam_list + lane * k;
  Entry e{};
  int next = 0;
  unsigned long long key = 0;
  auto advance = [&]() {
    key = 0;
    if (next < n) { e = of[next]; key = ordered(base + (double)e.value); }
    ++next;
  };
  advance();
  for (int i = 0; i < k; ++i) {
    const uint32_t hi = (uint32_t)(key >> 32), top = __reduce_max_sync(0xffffffffu, hi);
    const uint32_t lo = hi == top ? (uint32_t)key : 0u, top_lo = __reduce_max_sync(0xffffffffu, lo);
    const unsigned who = __ballot_sync(0xffffffffu, key != 0 && hi == top && (uint32_t)key == top_lo);
    const int winner = who ? __ffs(who) - 1 : 0;
    if (lane == winner) {
      const size_t at = (size_t)request * k + i;
      a.parent[at] = who ? request * a.beams + lane : -1;
      a.token[at] = who ? e.token : -1;
      a.new_scores[at] = who ? (float)(base + (double)e.value) : -INFINITY;
      if (a.new_done) a.new_done[at] = !who || e.token == a.eos;
      if (who) advance();
    }
    __syncwarp();
  }
}

}  // namespace

}  // namespace et

using namespace et;

extern "C" et_status et_beam_select(const void* logits_dev, int logits_fp32, long long row_stride, int n_req, int beams, int vocab,
                                    const float* scores_dev, const unsigned char* done_dev, int eos, int k, int* parent_dev,
                                    int* token_dev, float* new_scores_dev, unsigned char* new_done_dev, void* workspace_dev,
                                    size_t workspace_bytes, void* cuda_stream) {
  if (!logits_dev || !parent_dev || !token_dev || !new_scores_dev || !workspace_dev || !aligned16(workspace_dev)) return ET_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(logits_dev) & (logits_fp32 ? 3 : 1)) != 0) return ET_ERR_INVALID_ARG;
  if (new_scores_dev == scores_dev || (new_done_dev && new_done_dev == done_dev)) return ET_ERR_INVALID_ARG;
  if (n_req < 1 || beams < 1 || vocab < 1 || k < 1 || row_stride < vocab) return ET_ERR_SHAPE;
  if (eos >= vocab || eos < (done_dev ? 0 : -1)) return ET_ERR_SHAPE;
  if (beams > BEAMS_MAX || k > K_MAX || vocab > 1 << 20 || (long long)n_req * beams > 65535) return ET_ERR_CAPACITY;
  const int rows = n_req * beams, chunks = cdiv(vocab, CHUNK);
  if (workspace_bytes < ET_BEAM_WORKSPACE(rows, vocab, k)) return ET_ERR_CAPACITY;
  // six blocks an SM are there at once; more segments than that are only more lists to join
  int segments = cdiv(148 * 6, rows);
  if (segments > chunks) segments = chunks;
  if (segments > SEGMENTS_MAX) segments = SEGMENTS_MAX;
  const int each = cdiv(chunks, segments);
  segments = cdiv(chunks, each);
  const Select a{logits_dev, row_stride, scores_dev, done_dev, beams, vocab, k, eos, segments, each, (unsigned char*)workspace_dev,
                 parent_dev, token_dev, new_scores_dev, new_done_dev};
  cudaStream_t s = (cudaStream_t)cuda_stream;
  ET_COUNT_LAUNCH();
  Launch scan(dim3(segments, rows), THREADS, LIST * sizeof(Entry), s);
  const bool aligned = aligned16(logits_dev) && (rows == 1 || row_stride % (logits_fp32 ? 4 : 8) == 0);
  auto* const kernel = logits_fp32 ? aligned ? beam_scan_kernel<true, true> : beam_scan_kernel<true, false>
                                   : aligned ? beam_scan_kernel<false, true> : beam_scan_kernel<false, false>;
  cudaError_t e = cudaLaunchKernelEx(&scan.cfg, kernel, a);
  if (e != cudaSuccess) return launched(e);
  ET_COUNT_LAUNCH();
  Launch join(n_req, 32 * beams, (size_t)beams * k * sizeof(Entry), s);
  return launched(cudaLaunchKernelEx(&join.cfg, beam_join_kernel, a));
}
