// Beam search: the k best continuations of each request's beams over the vocabulary.
//
// Every logit is read once, and that bounds it: score + x - log(sum of exp(x)) orders a beam's tokens as x does, so one pass finds the
// best k of x, their largest and the sum together.  A beam's logits are cut into segments, one block each (as many as fill the card); a
// second, small kernel joins a request's segments and beams in a fixed order.
//
//   * Which of a chunk's 4 096 logits can be among the best k?  In a segment's first chunk: those that are not below the k-th largest
//     of the maxima of 32 groups of them, for k groups have at least that, or, for a large k, not below what each warp has its share
//     of k threads' maxima above.  In the others: those above the k-th best so far; a lower token comes first among equal ones, so
//     later equal ones need not be looked at.  What passes goes to a list in shared memory, which is cut back to k entries, in order,
//     when it is long.
//   * The sum is a running one against a reference near the running maximum, each thread's own; it seldom moves after a thread's first
//     chunk.  A chunk's terms are added in fp32, the chunks in 64 bits.  Additions and multiplications take two logits at once.
//   * Scores are compared in 64 bits.
//
// Device time in a chain of calls, B200, logits not in L2 (of the measured copy bandwidth), both kernels: 32 x 8 beams over 152 064,
// the best 16: fp32 42 us (0.57), bf16 40 (0.30); the best 64 of 64 rows, fp32 39 (0.15); the best 31 of 6 x 4 beams over 194 849 20;
// 1 x 4 beams, the best 4, bf16 9.1, 8 x 4 14.5 (two launches, a first chunk); 32 x 8 over 32 003, bf16, rows not aligned 19.0 (0.13).
// Instructions bound it, about 230 of a warp for 512 logits: 70 are the arithmetic, the others find candidates and keep the list;
// the blocks' barrier, one a chunk, is the longest wait.
#include "decode.cuh"
#include "earlytom_pages.h"

namespace et {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32, EACH = 16, CHUNK = THREADS * EACH;
static_assert(CHUNK == ET_BEAM_CHUNK, "workspace");
static_assert(EACH == 16, "four groups of four");
// Resident: 64 registers a thread (an unaligned row's loads take 80: 23 for 19 us; of fp32 rows they spill 168 bytes).
constexpr int BLOCKS_SM = 4;
constexpr int K_MAX = 64, BEAMS_MAX = 32, SEGMENTS_MAX = 64;
// The list is cut back when it has more than so many keys; a chunk adds CHUNK at most.  With k more than the best k the bar follows the
// segment in four or five steps, and a chunk adds few keys.
__host__ __device__ constexpr int longest(int k) { return 2 * k + 8; }
constexpr int LIST = CHUNK + longest(K_MAX);
constexpr int RANKED = 1024;                        // up to so many keys each one's rank is counted
// Up to so many of a first chunk are bounded by 32 groups of threads, more by warps: by warps 4 beams' best 4 take 20.0 us in place of
// 8.5 (too much passes), the best 18 of 155 beams 21.9 of 21.0; by groups the best 31 of 24 beams 26.3 us in place of 24.8.
constexpr int FEW = 20;
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

// What a segment leaves: its best k (value, token) in order, (-infinity, -1) behind the last, and its Sum.
struct Entry { float value; int token; };
// Floats as whole numbers of the same order, above 0.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
// A (value, token) as one number, larger for a larger value, among equal ones for the lower token; no such number is 0.
__device__ __forceinline__ unsigned long long key_of(float value, int token) {
  return (unsigned long long)ordered(value + 0.f) << 32 | (0xffffffffu - (uint32_t)token);      // (the zeros are equal)
}
__device__ __forceinline__ Entry entry_of(unsigned long long key) {
  const uint32_t u = (uint32_t)(key >> 32);
  return Entry{__uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xffffffffu)), (int)(0xffffffffu - (uint32_t)key)};
}
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

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Two floats each
__device__ __forceinline__ unsigned long long pair(float a, float b) {
  unsigned long long y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void unpair(unsigned long long x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
  unsigned long long y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}

// A sum of powers 2^(LOG2E x), held as total * 2^(LOG2E from - lift): a term is 2^(LOG2E (x - from) + lift), of an exponent that is rounded
// once.  lift puts the largest term between 2^6 and 2^14, so that those which count, down to 2^-20 of it, have exponents below 16
// whose rounding is 2^-21 at most.  `from` is 0 and lift a whole number up to logits of 2^23: then x - from is exact and a new reference
// costs no rounding.  Of larger logits `from` is the largest one when it was set.
// In units of 2^-24 the logarithm is off by 5.5 (the exponents' rounding), 4 (ex2.approx, 2^-22), 4 (a chunk's sixteen terms; chunks are
// added in 64 bits) and 2.2 (LOG2E's own rounding, at most 9.7 from the reference): less than 16, 2^-20.  Beyond 2^23 up to three new
// references count, 4 each (exp2f, two units in the last place): less than 32.  (A running fp32 sum of exponents rounded twice, 40.1 us in
// place of 42.0 for 32 x 8 beams fp32, is off by up to 2^-16 where logits are equal: its roundings do not cancel.)
struct Sum { float from, lift; double total; };
constexpr float LARGE_LOGIT = 8388608.f, LIFT = 7.f, LEEWAY = 4.f;          // LEEWAY: how far above the reference's logit one has to be for a new one
__device__ __forceinline__ double place_of(const Sum& s) { return s.total == 0. ? -1e300 : (double)LOG2E * s.from - s.lift; }
// 2^k for k <= 0, 2^-1022 at least; 1 for k > 0, where there is nothing yet that it could count for
__device__ __forceinline__ double power(int k) { return __hiloint2double((1023 + min(max(k, -1022), 0)) << 20, 0); }
// total * 2^d, d <= 0
__device__ __forceinline__ double scaled(double total, double d) {
  const double k = rint(d);
  const float f = (float)(d - k);
  double p = power((int)fmax(k, -1022.));
  if (f != 0.f) p *= exp2f(f);
  return total * p;
}
// The sums of the first N lanes, added up at the highest reference; the other lanes' are zero.
template <int N>
__device__ __forceinline__ void add_lanes(Sum& s) {
  if (__all_sync(0xffffffffu, s.from == 0.f)) {
    const int at = s.total == 0. ? -(1 << 30) : -(int)s.lift, top = __reduce_max_sync(0xffffffffu, at);
    s.total *= power(at - top);
    s.lift = (float)-top;
  } else {
    const double at = place_of(s);
    double top = at;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmax(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int who = __ffs(__ballot_sync(0xffffffffu, at == top)) - 1;
    s.from = __shfl_sync(0xffffffffu, s.from, who);
    s.lift = __shfl_sync(0xffffffffu, s.lift, who);
    s.total = scaled(s.total, at - top);
  }
#pragma unroll
  for (int o = N / 2; o > 0; o >>= 1) s.total += __shfl_xor_sync(0xffffffffu, s.total, o);
}

// The list's best k keys, in order, to its front; returns how many.  All threads; the list is complete.
__device__ __forceinline__ int cut_back(unsigned long long* list, int n, int k, unsigned long long* best) {
  const int tid = threadIdx.x, kept = min(n, k);
  if (n <= RANKED) {
    // each key's rank is how many are larger
    unsigned long long mine[RANKED / THREADS];
    int rank[RANKED / THREADS];
#pragma unroll
    for (int j = 0; j < RANKED / THREADS; ++j) {
      const int e = tid + j * THREADS;
      rank[j] = k;
      if (e >= n) continue;
      mine[j] = list[e];
      int r = 0;
#pragma unroll 4
      for (int i = 0; i < n; ++i) r += list[i] > mine[j];
      rank[j] = r;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < RANKED / THREADS; ++j) if (rank[j] < k) list[rank[j]] = mine[j];
  } else {
    // many values that are equal or come in an unlucky order: the largest one, k times
    for (int r = 0; r < kept; ++r) {
      unsigned long long top = 0;
      int at = 0;
      for (int e = tid; e < n; e += THREADS) if (list[e] > top) { top = list[e]; at = e; }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, top, o);
        const int other_at = __shfl_xor_sync(0xffffffffu, at, o);
        if (other > top) { top = other; at = other_at; }
      }
      if ((tid & 31) == 0) { best[2 * (tid >> 5)] = top; best[2 * (tid >> 5) + 1] = (unsigned long long)at; }
      __syncthreads();
      if (tid == 0) {
        int w = 0;
        for (int i = 1; i < WARPS; ++i) if (best[2 * i] > best[2 * w]) w = i;
        best[2 * WARPS + r] = best[2 * w];
        list[best[2 * w + 1]] = 0;
      }
      __syncthreads();
    }
    if (tid < kept) list[tid] = best[2 * WARPS + tid];
  }
  __syncthreads();
  return kept;
}

// A warp's 32 values in descending order.
__device__ __forceinline__ float sorted(float g) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
    for (int o = size >> 1; o > 0; o >>= 1) {
      const float other = __shfl_xor_sync(0xffffffffu, g, o);
      g = ((lane & size) == 0) == ((lane & o) == 0) ? fmaxf(g, other) : fminf(g, other);
    }
  return g;
}

// The k-th largest of the threads' values: each warp's in order, a value's place among the other warps' by search.  All threads.
__device__ __forceinline__ float kth_top(float top, int k, float (*tops)[32], float* result) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const float g = sorted(top);
  tops[warp][lane] = g;
  __syncthreads();
  int rank = lane;
#pragma unroll 2
  for (int w = 0; w < WARPS; ++w) {
    int before = 0;                                 // how many of the 32 come before this one
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) {
      const float other = tops[w][before + step - 1];
      if (other > g || (other == g && w < warp)) before += step;
    }
    const float other = tops[w][31];
    if (before == 31 && (other > g || (other == g && w < warp))) ++before;
    if (w != warp) rank += before;
  }
  if (rank == k - 1) *result = g;
  __syncthreads();
  return *result;
}

template <bool FP32, bool ALIGNED>
__global__ void __launch_bounds__(THREADS, BLOCKS_SM)
beam_scan_kernel(const __grid_constant__ Select a) {
  constexpr int SIZE = FP32 ? 4 : 2, VEC = 16 / SIZE, SLOTS = EACH / VEC;
  extern __shared__ unsigned long long list[];      // [LIST] keys
  __shared__ int added_s[3];                        // keys that a chunk adds, in turn
  __shared__ float group_top[32], thread_top[WARPS][32];
  __shared__ unsigned long long best[2 * WARPS + K_MAX];
  __shared__ Sum reduce[WARPS];
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
  auto all_inside = [&](int at) { return at - shift >= 0 && at - shift + CHUNK + (ALIGNED ? 0 : VEC) <= a.vocab; };
  auto load = [&](int at, uint32_t (&raw)[SLOTS][WORDS]) {
    auto vectors = [&](uint32_t (&w)[WORDS], const unsigned char* p) {
#pragma unroll
      for (int i = 0; i < WORDS; i += 4)
        asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "l"(p + 4 * i));
    };
    if (all_inside(at)) {                           // all chunks but a row's last one, and its first where it is not aligned
      const unsigned char* const p = src + (ptrdiff_t)(at + place(0) - shift) * SIZE;
#pragma unroll
      for (int j = 0; j < SLOTS; ++j) vectors(raw[j], p + j * (THREADS * 16));
      return;
    }
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      const int e0 = at + place(j);
      if (inside(e0)) vectors(raw[j], src + (ptrdiff_t)(e0 - shift) * SIZE);
      else {
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
  if (tid < 3) added_s[tid] = 0;
  __syncthreads();
  Sum sum{0.f, 0.f, 0.};
  float limit = -INFINITY, bar = -INFINITY;         // bar: what a logit has to reach or, behind the first chunk, to pass
  int n = 0, turn = 0;
  bool begun = false;
  for (int at = first; at < last; at += CHUNK) {
    float x[EACH];
#pragma unroll
    for (int j = 0; j < SLOTS; ++j) {
      if (!ALIGNED && inside(at + place(j))) cut(raw[j]);
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        x[j * VEC + v] = __uint_as_float(FP32 ? raw[j][v & 3] : v & 1 ? raw[j][v / 2] & 0xffff0000u : raw[j][v / 2] << 16);
    }
    if (at + CHUNK < last) load(at + CHUNK, raw);   // on its way while this chunk is looked at
    float top4[EACH / 4], top;
#pragma unroll
    for (int i = 0; i < EACH; i += 4) top4[i / 4] = max3(fmaxf(x[i], x[i + 1]), x[i + 2], x[i + 3]);
    top = max3(fmaxf(top4[0], top4[1]), top4[2], top4[3]);
    if (top > limit) {
      const Sum old = sum;
      const bool large = !(fabsf(top) < LARGE_LOGIT);
      sum.from = large ? top : 0.f;
      sum.lift = large ? LIFT : LIFT - rintf(top * LOG2E);
      if (sum.from == 0.f && old.from == 0.f) sum.total *= power((int)(sum.lift - old.lift));
      else if (old.total != 0.) sum.total = scaled(old.total, place_of(old) - place_of(sum));
      limit = top + LEEWAY;
    }
    const unsigned long long minus_from = pair(-sum.from, -sum.from), lift = pair(sum.lift, sum.lift), log2e = pair(LOG2E, LOG2E);
    auto terms = [&](int i) {                       // two of them
      float e0, e1;
      unpair(fma2(add2(pair(x[i], x[i + 1]), minus_from), log2e, lift), e0, e1);
      return pair(exp2_fast(e0), exp2_fast(e1));
    };
    unsigned long long four[EACH / 4];
#pragma unroll
    for (int i = 0; i < EACH; i += 4) four[i / 4] = add2(terms(i), terms(i + 2));
    float s0, s1;
    unpair(add2(add2(four[0], four[1]), add2(four[2], four[3])), s0, s1);
    sum.total += (double)(s0 + s1);
    if (!begun) {
      if (a.k <= FEW) {
        // the k-th largest of the maxima of 32 groups of eight threads
        float g = top;
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) g = fmaxf(g, __shfl_xor_sync(0xffffffffu, g, o));
        if (lane % 8 == 0) group_top[warp * 4 + lane / 8] = g;
        __syncthreads();
        bar = __shfl_sync(0xffffffffu, sorted(group_top[lane]), a.k - 1);
      } else {
        // in each warp as many threads' maxima as its share of k; the least of these
        const float g = __shfl_sync(0xffffffffu, sorted(top), (a.k + WARPS - 1) / WARPS - 1);
        if (lane == 0) group_top[warp] = g;
        __syncthreads();
        bar = group_top[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) bar = fminf(bar, group_top[w]);
      }
      // Too few groups or warps have logits, of a short vocabulary: all that there are would pass (the best 32 of 721 tokens 43 us, so 17).
      if (bar == -INFINITY) bar = kth_top(top, a.k, thread_top, group_top);
    }
    int* const added = added_s + turn;
    if (begun ? top > bar : top >= bar)
#pragma unroll
      for (int i = 0; i < EACH; i += 4)
        if (begun ? top4[i / 4] > bar : top4[i / 4] >= bar)
#pragma unroll
          for (int e = i; e < i + 4; ++e)
            if ((begun ? x[e] > bar : x[e] >= bar) && x[e] > -INFINITY)
              list[n + atomicAdd(added, 1)] = key_of(x[e], at + place(e / VEC) + e % VEC);
    // Counters go round three: this one is read behind the barrier, when the next chunk may be adding to the next one already, which was
    // read before the last barrier.
    if (tid == 0) added_s[turn == 2 ? 0 : turn + 1] = 0;
    __syncthreads();
    n += *added;
    turn = turn == 2 ? 0 : turn + 1;
    if (!begun || n > longest(a.k)) {
      n = cut_back(list, n, a.k, best);
      bar = n == a.k ? entry_of(list[a.k - 1]).value : -INFINITY;
      begun = true;
      __syncthreads();                              // the list is read before the next chunk adds to it
    }
  }
  n = cut_back(list, n, a.k, best);
  unsigned char* const out = segment_of(a, row, segment);
  if (tid < a.k) reinterpret_cast<Entry*>(out)[tid] = tid < n ? entry_of(list[tid]) : Entry{-INFINITY, -1};
  add_lanes<32>(sum);
  if (lane == 0) reduce[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    sum = lane < WARPS ? reduce[lane] : Sum{0.f, 0.f, 0.};
    add_lanes<WARPS>(sum);
    if (lane == 0) *reinterpret_cast<Sum*>(out + 8 * (size_t)a.k) = sum;
  }
}

// The best 32 EACH keys of a row's lists, in order, key lane + 32 j in best[j]; the first k are put out.  Returns how many there are.
template <int EACH, class Put>
__device__ __forceinline__ int merge_lists(const Select& a, int row, Put put) {
  const int lane = threadIdx.x & 31;
  auto load = [&](int segment, float2 (&v)[EACH]) {
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int e = lane + 32 * j;
      v[j] = make_float2(-INFINITY, 0.f);
      if (e < a.k && segment < a.segments) v[j] = __ldcg(reinterpret_cast<const float2*>(segment_of(a, row, segment)) + e);
    }
  };
  auto key = [](const float2& v) { return v.x > -INFINITY ? key_of(v.x, __float_as_int(v.y)) : 0ull; };
  unsigned long long best[EACH];
  float2 first[EACH], next[EACH], after[EACH];
  load(0, first);
  load(1, next);
#pragma unroll
  for (int j = 0; j < EACH; ++j) best[j] = key(first[j]);
  for (int segment = 1; segment < a.segments; ++segment) {
    load(segment + 1, after);                       // (as it is: its key is formed an iteration later, when it is there)
    // the first of the one list with the last of the other: the larger ones are the best of both, and go up and down at most once
    unsigned long long x[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) x[j] = __shfl_sync(0xffffffffu, key(next[EACH - 1 - j]), 31 - lane);
#pragma unroll
    for (int j = 0; j < EACH; ++j) if (x[j] > best[j]) best[j] = x[j];
    if (EACH == 2 && best[EACH - 1] > best[0]) { const unsigned long long y = best[0]; best[0] = best[EACH - 1]; best[EACH - 1] = y; }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const unsigned long long other = __shfl_xor_sync(0xffffffffu, best[j], o);
        if ((lane & o) == 0 ? other > best[j] : other < best[j]) best[j] = other;
      }
#pragma unroll
    for (int j = 0; j < EACH; ++j) next[j] = after[j];
  }
  int count = 0;
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int e = lane + 32 * j;
    if (e < a.k && best[j] != 0) put(e, best[j]);
    count += __popc(__ballot_sync(0xffffffffu, e < a.k && best[j] != 0));
  }
  return count;
}

// A block joins a request, a warp each beam: the best k of its segments' lists, in order, then where these stand among all beams'.
constexpr int NEAR = 64;                            // keys of a beam that may be among its best k: up to so many are ranked at once
__host__ __device__ constexpr size_t join_bytes(int beams, int k) { return (size_t)beams * (NEAR * 8 + 12 * (size_t)k); }
static_assert(join_bytes(BEAMS_MAX, K_MAX) <= 48 * 1024 - 256, "shared memory");
__global__ void __launch_bounds__(32 * BEAMS_MAX, 1)
beam_join_kernel(const __grid_constant__ Select a) {
  extern __shared__ unsigned long long join_smem[];                         // [beams][NEAR] keys, [beams][k] scores, [beams][k] tokens
  __shared__ int count_s[BEAMS_MAX];
  const int lane = threadIdx.x & 31, beam = threadIdx.x >> 5, request = blockIdx.x, row = request * a.beams + beam, k = a.k;
  unsigned long long* const near = join_smem + beam * NEAR;
  double* const scores = reinterpret_cast<double*>(join_smem + a.beams * NEAR);
  int* const tokens = reinterpret_cast<int*>(scores + a.beams * k);
  double* const mine = scores + beam * k;
  begin_after_previous();
  const float score = score_of(a, row);
  int count = 0;
  if (!finite(score)) {
  } else if (done_of(a, row)) {
    if (lane == 0) { mine[0] = score; tokens[beam * k] = a.eos; }
    count = 1;
  } else {
    // Two lists a lane, their maxima and sums; entries: all of them where they are few (lane + 32 i of the lists one behind the other),
    // else the first ones of the lane's lists.  All are on their way at once.
    constexpr int AHEAD = 4;
    const bool few = a.segments * k <= 64 * AHEAD;
    auto list_of = [&](int segment) { return reinterpret_cast<const float2*>(segment_of(a, row, segment)); };
    Sum part[2];
    float2 e[2][AHEAD];
    auto load = [&](int i, int first) {
#pragma unroll
      for (int p = 0; p < AHEAD; ++p)
        e[i][p] = lane + 32 * i < a.segments && first + p < k ? __ldcg(list_of(lane + 32 * i) + first + p) : make_float2(-INFINITY, 0.f);
    };
    // What at least k entries reach: if m of the first 32 lists have a j-th one that does, m j entries do.  From the first j on for which
    // there are enough lists, some j are tried; for the first entries alone one will do.  (Where all entries can be ranked none is needed,
    // which saves 0.6 to 1 us.)  The best 31 of 24 beams' 24 lists each: 25.0 us with the lists' second entries alone, 20.5.
    constexpr int TRIED = 4;
    const bool tried = a.segments * k > NEAR;
    const int lists = min(a.segments, 32), each = (k + lists - 1) / lists;
    float reach[TRIED];
#pragma unroll
    for (int t = 0; t < TRIED; ++t)
      reach[t] = tried && (t == 0 || each > 1) && lane < lists && each + t <= k ? __ldcg(list_of(lane) + each + t - 1).x : -INFINITY;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      part[i] = Sum{0.f, 0.f, 0.};
      if (lane + 32 * i < a.segments) {
        const float2 reference = __ldcg(list_of(lane + 32 * i) + k);
        part[i] = Sum{reference.x, reference.y, __ldcg(reinterpret_cast<const double*>(list_of(lane + 32 * i) + k + 1))};
      }
      if (!few) { load(i, 0); continue; }
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) {
        const int at = lane + 32 * (i * AHEAD + p), segment = at / k;
        e[i][p] = segment < a.segments ? __ldcg(list_of(segment) + at - segment * k) : make_float2(-INFINITY, 0.f);
      }
    }
    float bar = -INFINITY;
    if (tried) bar = __shfl_sync(0xffffffffu, sorted(reach[0]), (k + each - 1) / each - 1);
    if (tried && each > 1)
#pragma unroll
      for (int t = 1; t < TRIED; ++t) bar = fmaxf(bar, __shfl_sync(0xffffffffu, sorted(reach[t]), (k + each + t - 1) / (each + t) - 1));
    // One list is in order as it is, and k entries at least reach the bar.
    int n = a.segments == 1 || k >= NEAR ? NEAR + 1 : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bool more = n <= NEAR && (few || 32 * i < a.segments);
      for (int first = 0; more; first += AHEAD) {
        if (first > 0) load(i, first);
#pragma unroll
        for (int p = 0; p < AHEAD; ++p) {
          const bool take = e[i][p].x >= bar && e[i][p].x > -INFINITY;
          const unsigned who = __ballot_sync(0xffffffffu, take);
          const int at = n + __popc(who & ((1u << lane) - 1));
          if (take && at < NEAR) near[at] = key_of(e[i][p].x, __float_as_int(e[i][p].y));
          n += __popc(who);
          more = !few && who != 0 && n <= NEAR;
        }
      }
    }
    __syncwarp();
    add_lanes<32>(part[0]);
    if (a.segments > 32) {
      add_lanes<32>(part[1]);
      const double d = place_of(part[1]) - place_of(part[0]);
      if (d > 0.) part[0] = Sum{part[1].from, part[1].lift, part[1].total + scaled(part[0].total, -d)};
      else part[0].total += scaled(part[1].total, d);
    }
    const double base = (double)score - ((double)part[0].from + (log(part[0].total) - (double)part[0].lift * (1. / LOG2E)));
    auto put = [&](int rank, unsigned long long key) {
      const Entry e = entry_of(key);
      mine[rank] = base + (double)e.value;
      tokens[beam * k + rank] = e.token;
    };
    if (!(base >= -1.7e308 && base <= 1.7e308)) {       // no token, NaN or an infinity
    } else if (n <= NEAR) {
      for (int e = lane; e < n; e += 32) {
        const unsigned long long key = near[e];
        int rank = 0;
#pragma unroll 4
        for (int i = 0; i < n; ++i) rank += near[i] > key;
        if (rank < k) put(rank, key);
      }
      count = min(n, k);
    } else {
      // too many: list by list, of two lists in order the best of both and these in order again
      count = k <= 32 ? merge_lists<1>(a, row, put) : merge_lists<2>(a, row, put);
    }
  }
  if (lane == 0) count_s[beam] = count;
  __syncthreads();
  // a continuation's place: those of its beam before it, and those of the others that are better, or as good and of a lower beam
  for (int e = lane; e < count; e += 32) {
    const double x = mine[e];
    int rank = e;
    for (int b = 0; b < a.beams && rank < k; ++b) {
      if (b == beam) continue;
      const double* const of = scores + b * k;
      int lo = 0, n = count_s[b];                   // how many of the list's are before this one: it is in descending order
      while (n > 0) {
        const int half = n >> 1;
        if (of[lo + half] > x || (of[lo + half] == x && b < beam)) { lo += half + 1; n -= half + 1; } else n = half;
      }
      rank += lo;
    }
    if (rank < k) {
      const size_t at = (size_t)request * k + rank;
      const int token = tokens[beam * k + e];
      a.parent[at] = row;
      a.token[at] = token;
      a.new_scores[at] = (float)x;
      if (a.new_done) a.new_done[at] = token == a.eos;
    }
  }
  int all = 0;
  for (int b = 0; b < a.beams; ++b) all += count_s[b];
  for (int i = all + threadIdx.x; i < k; i += blockDim.x) {
    const size_t at = (size_t)request * k + i;
    a.parent[at] = a.token[at] = -1;
    a.new_scores[at] = -INFINITY;
    if (a.new_done) a.new_done[at] = 1;
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
  // as many segments as keep all blocks resident at once (32 x 8 beams over 152 064: half as many 55 us, half as many again 52, these
  // 43; 8 x 4 beams 17.2, 12.9, 14.5; 31 x 5 over 53 552: 30.5, 26.1, 21.8)
  constexpr int BLOCKS = 148 * BLOCKS_SM;
  int segments = rows < BLOCKS ? BLOCKS / rows : 1;
  if (segments > chunks) segments = chunks;
  if (segments > SEGMENTS_MAX) segments = SEGMENTS_MAX;
  const int each = cdiv(chunks, segments);
  segments = cdiv(chunks, each);
  const Select a{logits_dev, row_stride, scores_dev, done_dev, beams, vocab, k, eos, segments, each, (unsigned char*)workspace_dev,
                 parent_dev, token_dev, new_scores_dev, new_done_dev};
  cudaStream_t s = (cudaStream_t)cuda_stream;
  ET_COUNT_LAUNCH();
  Launch scan(dim3(segments, rows), THREADS, LIST * sizeof(unsigned long long), s);
  const bool aligned = aligned16(logits_dev) && (rows == 1 || row_stride % (logits_fp32 ? 4 : 8) == 0);
  auto* const kernel = logits_fp32 ? aligned ? beam_scan_kernel<true, true> : beam_scan_kernel<true, false>
                                   : aligned ? beam_scan_kernel<false, true> : beam_scan_kernel<false, false>;
  cudaError_t e = cudaLaunchKernelEx(&scan.cfg, kernel, a);
  if (e != cudaSuccess) return launched(e);
  ET_COUNT_LAUNCH();
  Launch join(n_req, 32 * beams, join_bytes(beams, k), s);
  return launched(cudaLaunchKernelEx(&join.cfg, beam_join_kernel, a));
}
