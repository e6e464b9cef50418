// The paged key / value cache: rows of a projection go in (turned and quantised on the way), rows come back.
//
// Device time in a chain of calls, B200, rows and cache not in L2 (of the measured copy bandwidth, bytes read + written): append of 21 124
// rows of 28 + 4 + 4 heads of 128, turned, bf16 66 us (0.91), e4m3 93 us (0.61: instructions, the rotation's among them); of 7 675
// rows of 4 + 4 heads, e4m3 8.9 us (0.41: launch and three loads that wait for one another); of one token 2.5 us, of 64 e4m3 3.7 us.
// Read of 63 435 rows of 16 + 16 heads of 64, bf16 86 us (0.93); of 7 675 rows, e4m3 8.9 us (0.41).
// 4 bits, heads of 128: append of 23 942 rows of 28 + 4 + 4 heads, turned, 102 us (0.61: keys turned and scaled in 64 bits), of 7 675 rows
// of 4 + 4 heads, not turned, 9.1 us (0.34), of one token 4.7 us; read of 23 942 rows 18.8 us (0.51), of 7 675 7.4 us (0.42), of one 2.4.
#include <cuda_fp8.h>

#include <type_traits>

#include "decode.cuh"

namespace et {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

// Finds the places of a warp's rows, which come in ascending order: the sequence is searched for only when a row leaves the
// last one's run, the page looked up only when a row leaves the last one's page, so most rows cost no load at all.
struct Places {
  int seq = -1, first = 0, behind = 0, start = 0;      // the current sequence's run of rows, its start position
  int page_of = -1, page = 0;                          // the table column that was looked up last, and the page there

  // page and place of a row; false: nothing is to be done for it
  __device__ __forceinline__ bool find(const PagedCache& c, const PagedRows& r, int row, int& page_out, int& place, long long& pos) {
    if (seq < 0 || row < first || row >= behind) {
      int s = row;
      first = row; behind = row + 1;
      if (r.offsets) {
        // the last sequence whose offset is not behind the row; outside its run the row is padding
        int lo = 0, hi = r.n_seq;
        while (hi - lo > 1) {
          const int mid = lo + ((hi - lo) >> 1);
          if (r.offsets[mid] <= row) lo = mid; else hi = mid;
        }
        s = lo;
        first = r.offsets[s];
        behind = r.offsets[s + 1];
      }
      seq = s;
      start = r.start[s];
      page_of = -1;
    }
    if (row < first || row >= behind || start < 0) return false;
    pos = (long long)start + row - first;                // 64 bits and not negative, whatever the offsets hold
    const int column = (int)(pos >> c.page_shift);
    if (column != page_of) {
      int unused;
      page_of = column;
      if (!paged_place(c, r.table, r.max_pages, seq, pos, r.status, page, unused)) page = -1;
    }
    page_out = page;
    place = (int)(pos & ((1 << c.page_shift) - 1));
    return page >= 0;
  }
};

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

// Lengths after the call: of the sequences' starts and rows.
__device__ __forceinline__ void advance_lengths(const PagedCache& c, const PagedRows& r, int* new_len) {
  for (unsigned s = threadIdx.x; s < (unsigned)r.n_seq; s += THREADS) {
    const int start = r.start[s];
    // rows that the call has: an offset that is none of theirs counts as the first or as the end
    auto row_at = [&](unsigned i) { return min(max(r.offsets[i], 0), r.rows); };
    const int n = r.offsets ? max(0, row_at(s + 1) - row_at(s)) : 1;
    const long long cap = (long long)r.max_pages << c.page_shift;
    new_len[s] = start < 0 ? start : (int)min((long long)start + n, cap);
  }
}

// x c - y s with two roundings (but for 2^-39 of x and y): x and y have 8 bits, c = c1 + c2 and s = s1 + s2 16 in their first parts,
// so that the products of those are exact.
__device__ __forceinline__ float turned_exactly(float x, float c1, float c2, float y, float s1, float s2) {
  return (x * c1 - y * s1) + fmaf(x, c2, -(y * s2));
}

// ---------------------------------------------------------------------------------------------
// Append.  A warp (or `parts` of them, where rows are few) takes a row, a lane elements i .. i+7 and i + d/2 .. i + d/2 + 7 of
// one head, the two halves that the rotation pairs; d/16 neighbouring lanes hold a head and find its maximum with shuffles, so
// a row is read once and written once.  The angle of position p and pair i is p * theta^(-2i/d): the host gives each frequency
// as a 64-bit fraction of a turn, so that p * f modulo 2^64 is the exact fraction of a turn however far p is.  A lane has the
// same pairs in every head: it keeps their (cos, sin) in registers for the row.  Keys on their way to e4m3 are turned more
// exactly: what fp32 products lose is small beside bf16's rounding, but takes one in 400 000 of them across a border between two
// e4m3 values, a sixteenth apart (now one in two million; 21 124 rows of 28 + 4 + 4 heads 87.6 -> 93.3 us).  Bound by memory, and with
// e4m3 and rotation by instructions.
// ---------------------------------------------------------------------------------------------
template <int DH, bool E4M3, bool ROTATE>
__global__ void __launch_bounds__(THREADS)
kv_append_kernel(const bf16* qkv, long long row_stride, int heads, PagedCache c, PagedRows r,
                 const __grid_constant__ RopeTurns turns, bf16* q_out, int* new_len, int rows_each, int parts) {
  constexpr int HALF = DH / 2, CHUNKS = DH / 16, UNROLL = 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int part = warp % parts, chunk = lane % CHUNKS, head_lane = lane / CHUNKS;
  constexpr int HEADS_ITER = 32 / CHUNKS;
  const int skip = ROTATE ? 0 : heads;                       // query heads that need nothing done
  const int all_heads = heads + 2 * c.kv_heads;

  begin_after_previous();
  // advance_lengths, written out: with the call the kernel for turned bf16 rows takes 94 registers in place of 80
  if (new_len && blockIdx.x == 0) {
    for (unsigned s = threadIdx.x; s < (unsigned)r.n_seq; s += THREADS) {
      const int start = r.start[s];
      // rows that the call has: an offset that is none of theirs counts as the first or as the end
      auto row_at = [&](unsigned i) { return min(max(r.offsets[i], 0), r.rows); };
      const int n = r.offsets ? max(0, row_at(s + 1) - row_at(s)) : 1;
      const long long cap = (long long)r.max_pages << c.page_shift;
      new_len[s] = start < 0 ? start : (int)min((long long)start + n, cap);
    }
  }

  Places places;
  // a block's rows are neighbours, dealt to its warps in turn: what one of them fetches of a page lies next to the others'
  const int step = WARPS / parts;
  const long long row0 = (long long)blockIdx.x * step * rows_each, row1 = min(row0 + step * rows_each, (long long)r.rows);
  for (long long row = row0 + warp / parts; row < row1; row += step) {
    const bf16* const src_row = qkv + row * row_stride + chunk * 8;
    uint4 va[UNROLL], vb[UNROLL];
    auto load = [&](int h0) {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int head = h0 + j * HEADS_ITER + head_lane;
        va[j] = vb[j] = make_uint4(0, 0, 0, 0);
        if (head < all_heads) {
          const bf16* src = src_row + (size_t)head * DH;
          va[j] = *reinterpret_cast<const uint4*>(src);
          vb[j] = *reinterpret_cast<const uint4*>(src + HALF);
        }
      }
    };
    int h0 = skip + part * HEADS_ITER * UNROLL;
    load(h0);                                                // on its way while the row's place is looked up
    int page, place;
    long long pos;
    if (!places.find(c, r, (int)row, page, place, pos)) continue;          // the same for all lanes
    constexpr bool EXACT = ROTATE && E4M3;
    float cs[8], sn[8], c1[8], s1[8];                        // EXACT: c1 + cs, s1 + sn
    if (ROTATE) {
      // HALF pairs, found by HALF lanes' worth of sincos and handed to the lanes that need them
      constexpr int EACH = HALF / 32 > 0 ? HALF / 32 : 1;
      float mc[EACH], ms[EACH], mc1[EACH], ms1[EACH];
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const unsigned long long turn = (unsigned long long)pos * turns.f[(lane * EACH + j) % HALF];
        if (EXACT) {
          double c, s;
          sincospi((double)(long long)turn * 0x1p-63, &s, &c);
          mc1[j] = __int_as_float(__float_as_int((float)c) & 0xffffff00);
          ms1[j] = __int_as_float(__float_as_int((float)s) & 0xffffff00);
          mc[j] = (float)(c - mc1[j]);
          ms[j] = (float)(s - ms1[j]);
        } else {
          sincospif(__ll2float_rn((long long)turn) * 0x1p-63f, &ms[j], &mc[j]);       // half turns in [-1, 1)
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int from = (chunk * 8 + k) / EACH;
        cs[k] = __shfl_sync(0xffffffffu, mc[k % EACH], from);
        sn[k] = __shfl_sync(0xffffffffu, ms[k % EACH], from);
        if (EXACT) {
          c1[k] = __shfl_sync(0xffffffffu, mc1[k % EACH], from);
          s1[k] = __shfl_sync(0xffffffffu, ms1[k % EACH], from);
        }
      }
    }
    for (;;) {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int head = h0 + j * HEADS_ITER + head_lane;
        float a[8], b[8];
        unpack8(va[j], a);
        unpack8(vb[j], b);
        if (EXACT && head >= heads && head < heads + c.kv_heads) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float x = a[k], y = b[k];
            a[k] = turned_exactly(x, c1[k], cs[k], y, s1[k], sn[k]);
            b[k] = turned_exactly(y, c1[k], cs[k], x, -s1[k], -sn[k]);
          }
        } else if (ROTATE && head < heads + c.kv_heads) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float x = a[k], y = b[k], co = EXACT ? c1[k] + cs[k] : cs[k], si = EXACT ? s1[k] + sn[k] : sn[k];
            a[k] = x * co - y * si;
            b[k] = y * co + x * si;
          }
        }
        if (ROTATE && head < heads) {
          uint4* dst = reinterpret_cast<uint4*>(q_out + ((size_t)row * heads + head) * DH + chunk * 8);
          dst[0] = pack8(a);
          dst[HALF / 8] = pack8(b);
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
        if (head >= heads && head < all_heads) {
          const int kvh = head - heads;
          const int plane = kvh >= c.kv_heads ? 1 : 0;
          const size_t at = cache_row(c, page, plane, kvh - plane * c.kv_heads, place);
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
      h0 += parts * HEADS_ITER * UNROLL;
      if (h0 >= all_heads) break;
      load(h0);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Append to a cache of 4 bits.  A block of 32 values has one bf16 scale s, the smallest that is not below max|x| / 7, and codes n + 8
// with n = x / s rounded to nearest, ties to even.  Both are what 64-bit arithmetic gives, turned keys' as well: with keys turned in
// fp32 one value in a few hundred thousand lies on the other side of a border between two codes, a seventh of the block's largest
// value away.
//
// A warp takes a row as above.  The queries come first, eight values of each half a lane, then keys and values, four of each half where
// keys are turned: sines, cosines and keys in 64 bits take twice the registers.
// ---------------------------------------------------------------------------------------------
// N bf16, four or eight
template <int N> struct Bf16s { uint32_t w[N / 2]; };
template <int N>
__device__ __forceinline__ Bf16s<N> load_bf16s(const bf16* p) {
  Bf16s<N> v;
  if constexpr (N == 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    v.w[0] = x.x; v.w[1] = x.y; v.w[N / 2 - 2] = x.z; v.w[N / 2 - 1] = x.w;
  } else {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v.w[0] = x.x; v.w[1] = x.y;
  }
  return v;
}
template <int N>
__device__ __forceinline__ void unpack(const Bf16s<N>& v, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) { x[2 * i] = __uint_as_float(v.w[i] << 16); x[2 * i + 1] = __uint_as_float(v.w[i] & 0xffff0000u); }
}
// The largest magnitude, infinite if one of them is not finite.
template <int N>
__device__ __forceinline__ float largest(const Bf16s<N>& v) {
  uint32_t m = v.w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < N / 2; ++i) m = __vmaxu2(m, v.w[i] & 0x7fff7fffu);
  const uint32_t top = max(m & 0xffffu, m >> 16);
  return top < 0x7f80u ? __uint_as_float(top << 16) : INFINITY;
}
// A row's queries, turned; a lane has the cosines and sines of HALF / 32 pairs.
template <int DH>
__device__ __forceinline__ void turn_queries(const bf16* src, int heads, bf16* dst, const double (&mc)[DH / 64], const double (&ms)[DH / 64],
                                             int part, int parts) {
  constexpr int HALF = DH / 2, CHUNKS = HALF / 8, HEADS_ITER = 32 / CHUNKS, UNROLL = 2, EACH = HALF / 32;
  const int lane = threadIdx.x & 31, chunk = lane % CHUNKS, head_lane = lane / CHUNKS;
  float co[8], si[8], mcf[EACH], msf[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) { mcf[j] = (float)mc[j]; msf[j] = (float)ms[j]; }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    co[k] = __shfl_sync(0xffffffffu, mcf[k % EACH], (chunk * 8 + k) / EACH);
    si[k] = __shfl_sync(0xffffffffu, msf[k % EACH], (chunk * 8 + k) / EACH);
  }
  for (int h0 = part * HEADS_ITER * UNROLL + head_lane; h0 < heads; h0 += parts * HEADS_ITER * UNROLL) {
    uint4 va[UNROLL], vb[UNROLL];
#pragma unroll
    for (int j = 0; j < UNROLL; ++j)
      if (h0 + j * HEADS_ITER < heads) {
        const bf16* const p = src + (size_t)(h0 + j * HEADS_ITER) * DH + chunk * 8;
        va[j] = *reinterpret_cast<const uint4*>(p);
        vb[j] = *reinterpret_cast<const uint4*>(p + HALF);
      }
#pragma unroll
    for (int j = 0; j < UNROLL; ++j)
      if (h0 + j * HEADS_ITER < heads) {
        float a[8], b[8];
        unpack8(va[j], a);
        unpack8(vb[j], b);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float x = a[k], y = b[k];
          a[k] = x * co[k] - y * si[k];
          b[k] = y * co[k] + x * si[k];
        }
        uint4* const q = reinterpret_cast<uint4*>(dst + (size_t)(h0 + j * HEADS_ITER) * DH + chunk * 8);
        q[0] = pack8(a);
        q[HALF / 8] = pack8(b);
      }
  }
}

constexpr float MAGIC = 12582912.f;                          // 1.5 * 2^23: adding it rounds to a whole number, ties to even

// The smallest bf16 s with 7 s >= top; top >= 0, finite.  7 s has eleven bits.
template <typename T>
__device__ __forceinline__ float int4_scale(T top) {
  // the quotient cut off to bf16 is the one below, or the one that is sought, or (the product is rounded) one further below
  float s = __int_as_float(__float_as_int((float)top * (1.f / 7)) & 0xffff0000);
#pragma unroll
  for (int i = 0; i < 2; ++i) if ((T)7 * s < top) s = __int_as_float(__float_as_int(s) + 0x10000);
  return s;
}
// The magnitude of a 64-bit number by its upper word, rounded up: enough to find the largest one and to compare it with numbers of up
// to 21 bits; as integers such words have the numbers' order.
__device__ __forceinline__ int upper_word(double x) { return (__double2hiint(x) & 0x7fffffff) + (__double2loint(x) != 0 ? 1 : 0); }
constexpr int UPPER_BEYOND = 0x47f00000;                     // of 2^128; what is below it, rounded up, fp32 holds

// Four or eight codes.  A quotient of two bf16 that is not half way between two whole numbers is 2^-12 or more away from that; one that
// is comes out exactly, since one step of Newton's takes its error below 2^-40: adding MAGIC then rounds it as it should be.  Of a
// number of 64 bits fp32 loses 2^-24, so a quotient next to the half is looked at in 64 bits.
template <typename T, int N>
__device__ __forceinline__ uint32_t int4_codes(const T (&x)[N], float s) {
  if (!(s > 0.f)) return 0x88888888u;                        // a block of zeros, or one whose scale is NaN
  const bool tiny = s < 0x1p-100f;                           // 1 / s could overflow
  const float up = tiny ? 0x1p64f : 1.f, su = s * up, inv = __fdividef(1.f, su);
  float n[N];
  bool near = false;
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float y = tiny ? (float)(x[k] * (T)up) : (float)x[k], q0 = y * inv, q = fmaf(fmaf(-q0, su, y), inv, q0);
    n[k] = (q + MAGIC) - MAGIC;
    if (sizeof(T) == 8) near |= fabsf(fabsf(q - n[k]) - 0.5f) < 0x1p-18f;
  }
  if (sizeof(T) == 8 && near) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const double r = fma((double)-n[k], (double)s, (double)x[k]), h = 0.5 * s;
      const bool odd = (int)n[k] & 1;
      if (r > h || (odd && r == h)) n[k] += 1.f;
      else if (r < -h || (odd && r == -h)) n[k] -= 1.f;
    }
  }
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < N; k += 4) {
    const float all = fmaf(n[k + 3], 4096.f, fmaf(n[k + 2], 256.f, fmaf(n[k + 1], 16.f, n[k]))) + (34952.f + 8388608.f);       // 34952 = 0x8888
    w |= (__float_as_uint(all) & 0xffffu) << (4 * k);
  }
  return w;
}

// 80 registers a thread where keys are turned, of which 116 bytes are spilled, else 64, which suffice for eight values of a lane.
template <int DH, bool ROTATE>
__global__ void __launch_bounds__(THREADS, ROTATE ? 3 : 4)
kv_append_int4_kernel(const bf16* qkv, long long row_stride, int heads, PagedCache c, PagedRows r,
                      const __grid_constant__ RopeTurns turns, bf16* q_out, int* new_len, int rows_each, int parts) {
  constexpr int HALF = DH / 2;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % parts;

  begin_after_previous();
  if (new_len && blockIdx.x == 0) advance_lengths(c, r, new_len);

  Places places;
  const int step = WARPS / parts;
  const long long row0 = (long long)blockIdx.x * step * rows_each, row1 = min(row0 + step * rows_each, (long long)r.rows);
  for (long long row = row0 + warp / parts; row < row1; row += step) {
    const bf16* const src_row = qkv + row * row_stride;
    // keys and values
    constexpr int E = ROTATE ? 4 : 8, CHUNKS = HALF / E, HEADS_ITER = 32 / CHUNKS, UNROLL = 2;
    using Codes = typename std::conditional<E == 8, uint32_t, uint16_t>::type;
    const int chunk = lane % CHUNKS, head_lane = lane / CHUNKS, all_heads = 2 * c.kv_heads;
    Bf16s<E> va[UNROLL], vb[UNROLL];
    auto load = [&](int h0) {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int head = h0 + j * HEADS_ITER + head_lane;
        va[j] = vb[j] = Bf16s<E>{};
        if (head < all_heads) {
          const bf16* src = src_row + (size_t)(heads + head) * DH + chunk * E;
          va[j] = load_bf16s<E>(src);
          vb[j] = load_bf16s<E>(src + HALF);
        }
      }
    };
    int h0 = part * HEADS_ITER * UNROLL;
    load(h0);                                                // on its way while the row's place is looked up
    int page, place;
    long long pos;
    if (!places.find(c, r, (int)row, page, place, pos)) continue;          // the same for all lanes
    double cd[ROTATE ? E : 1], sd[ROTATE ? E : 1];
    if constexpr (ROTATE) {
      constexpr int EACH = HALF / 32;
      double mc[EACH], ms[EACH];
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const unsigned long long turn = (unsigned long long)pos * turns.f[lane * EACH + j];
        sincospi((double)(long long)turn * 0x1p-63, &ms[j], &mc[j]);
      }
      turn_queries<DH>(src_row, heads, q_out + (size_t)row * heads * DH, mc, ms, part, parts);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        cd[k] = __shfl_sync(0xffffffffu, mc[k % EACH], (chunk * E + k) / EACH);
        sd[k] = __shfl_sync(0xffffffffu, ms[k % EACH], (chunk * E + k) / EACH);
      }
    }
    for (;;) {
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int head = h0 + j * HEADS_ITER + head_lane;
        if (h0 + j * HEADS_ITER >= all_heads) break;         // the same for all lanes
        const bool key = ROTATE && head < c.kv_heads;
        float a[E], b[E];
        unpack(va[j], a);
        unpack(vb[j], b);
        float sa, sb;
        uint32_t ca, cb;
        // keys among the warp's heads, values among them; where both are, every lane goes both ways
        if constexpr (ROTATE) if (__any_sync(0xffffffffu, key)) {
          double ad[E], bd[E];
          int ta = 0, tb = 0;
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const double x = a[k], y = b[k], co = cd[k], si = sd[k];
            ad[k] = x * co - y * si;
            bd[k] = y * co + x * si;
            ta = max(ta, upper_word(ad[k]));
            tb = max(tb, upper_word(bd[k]));
          }
#pragma unroll
          for (int o = 1; o < INT4_BLOCK / E; o <<= 1) {
            ta = max(ta, __shfl_xor_sync(0xffffffffu, ta, o));
            tb = max(tb, __shfl_xor_sync(0xffffffffu, tb, o));
          }
          sa = ta < UPPER_BEYOND ? int4_scale(__hiloint2double(ta, 0)) : NAN;
          sb = tb < UPPER_BEYOND ? int4_scale(__hiloint2double(tb, 0)) : NAN;
          ca = int4_codes(ad, sa);
          cb = int4_codes(bd, sb);
        }
        if (!ROTATE || __any_sync(0xffffffffu, !key)) {
          float ta = largest(va[j]), tb = largest(vb[j]);
#pragma unroll
          for (int o = 1; o < INT4_BLOCK / E; o <<= 1) {
            ta = fmaxf(ta, __shfl_xor_sync(0xffffffffu, ta, o));
            tb = fmaxf(tb, __shfl_xor_sync(0xffffffffu, tb, o));
          }
          if (!key) {
            sa = ta < INFINITY ? int4_scale(ta) : NAN;
            sb = tb < INFINITY ? int4_scale(tb) : NAN;
            ca = int4_codes(a, sa);
            cb = int4_codes(b, sb);
          }
        }
        if (head >= all_heads) continue;
        const int plane = head >= c.kv_heads ? 1 : 0;
        const size_t at = cache_row(c, page, plane, head - plane * c.kv_heads, place);
        Codes* const dst = reinterpret_cast<Codes*>(c.data + at * (DH / 2) + chunk * (E / 2));
        dst[0] = (Codes)ca;
        dst[HALF / E] = (Codes)cb;
        if (chunk % (INT4_BLOCK / E) == 0) {
          bf16* const scale = reinterpret_cast<bf16*>(c.scale) + at * (DH / INT4_BLOCK) + chunk / (INT4_BLOCK / E);
          scale[0] = __float2bfloat16_rn(sa);
          scale[HALF / INT4_BLOCK] = __float2bfloat16_rn(sb);
        }
      }
      h0 += parts * HEADS_ITER * UNROLL;
      if (h0 >= all_heads) break;
      load(h0);
    }
  }
}

// Eight codes as bf16 values, i and i + 4 together: a code's bits in a bf16 of 128 are 128 + c; less 136, times the scale (twice in s).
// The product has 12 bits and is rounded once.
__device__ __forceinline__ uint4 int4_row8(uint32_t w, uint32_t s) {
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = ((w >> (4 * i)) & 0x000f000fu) | 0x43004300u;
    asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(x[i]) : "r"(0x43084308u));
    asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"(x[i]) : "r"(s));
  }
  return make_uint4(__byte_perm(x[0], x[1], 0x5410), __byte_perm(x[2], x[3], 0x5410), __byte_perm(x[0], x[1], 0x7632), __byte_perm(x[2], x[3], 0x7632));
}

// ---------------------------------------------------------------------------------------------
// Read: a warp (or `parts` of them) takes a row, a lane 16 bytes of the cache at a time (8 bf16 or 16 e4m3 values), four of
// them on their way; of 4-bit values 4 bytes, so that what it writes stays 16 bytes next to its neighbours' (eight of them on
// their way: 22 us in place of 19 for 23 942 rows of 4 + 4 heads of 128, which have four a lane).  Bound by memory; of 4 bits its
// warps wait for their loads (8 cycles an instruction, 61 % of the issue slots used).
// ---------------------------------------------------------------------------------------------
template <int DH, int FMT>
__global__ void __launch_bounds__(THREADS)
kv_read_kernel(bf16* out, long long row_stride, PagedCache c, PagedRows r, int rows_each, int parts) {
  constexpr bool E4M3 = FMT == ET_KV_E4M3, INT4 = FMT == ET_KV_INT4;
  constexpr int VEC = E4M3 ? 16 : 8, CHUNKS = DH / VEC, UNROLL = 4;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, part = warp % parts;
  const int units = 2 * c.kv_heads * CHUNKS;
  begin_after_previous();
  Places places;
  // a block's rows are neighbours, dealt to its warps in turn: what one of them fetches of a page lies next to the others'
  const int step = WARPS / parts;
  const long long row0 = (long long)blockIdx.x * step * rows_each, row1 = min(row0 + step * rows_each, (long long)r.rows);
  for (long long row = row0 + warp / parts; row < row1; row += step) {
    int page, place;
    long long pos;
    if (!places.find(c, r, (int)row, page, place, pos)) continue;          // the same for all lanes
    bf16* const dst_row = out + row * row_stride;
    const unsigned base = ((unsigned)page * 2 * c.kv_heads << c.page_shift) + place;
    for (int u0 = part * 32 * UNROLL + lane; u0 < units; u0 += parts * 32 * UNROLL) {
      uint4 v[UNROLL];
      int b[UNROLL];
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int u = u0 + 32 * j, head = u / CHUNKS, chunk = u % CHUNKS;
        b[j] = 0;
        if (u < units) {
          const unsigned at = base + ((unsigned)head << c.page_shift);      // (plane 1 follows plane 0's heads; below 2^31)
          if (INT4) {
            v[j].x = *reinterpret_cast<const uint32_t*>(c.data + (size_t)at * (DH / 2) + chunk * 4);
            b[j] = (reinterpret_cast<const uint16_t*>(c.scale))[(size_t)at * (DH / INT4_BLOCK) + chunk / (INT4_BLOCK / 8)];
          } else v[j] = *reinterpret_cast<const uint4*>(c.data + (size_t)at * (DH * (E4M3 ? 1 : 2)) + chunk * 16);
          if (E4M3) b[j] = c.scale[at];
        }
      }
#pragma unroll
      for (int j = 0; j < UNROLL; ++j) {
        const int u = u0 + 32 * j;
        if (u >= units) continue;
        uint4* dst = reinterpret_cast<uint4*>(dst_row + (size_t)u * VEC);
        if (INT4) {
          *dst = int4_row8(v[j].x, (uint32_t)b[j] * 0x10001u);
        } else if (E4M3) {
          const float f = pow2(b[j] - 127);
          const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
          float lo[8], hi[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[k >> 1] >> (16 * (k & 1))), __NV_E4M3);
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&h));
            (k < 4 ? lo : hi)[(2 * k) % 8] = y.x * f;
            (k < 4 ? lo : hi)[(2 * k + 1) % 8] = y.y * f;
          }
          dst[0] = pack8(lo);
          dst[1] = pack8(hi);
        } else {
          *dst = v[j];
        }
      }
    }
  }
}

// How rows are dealt: several warps to a row where there are few, `each` rows to a warp where there are very many.  (96 warps
// an SM are two to three times what it holds; 24 and 48 measured 67 and 67 us on eight prompts of 2 000 to 4 000 rows, as 96
// does, but 8.3 and 7.4 us against 7.0 on one of 7 675.)
struct Deal { int blocks, each, parts; };
Deal deal_rows(int rows, int steps_row) {
  const int warps = 148 * 96;
  Deal d;
  d.parts = 1;
  while (d.parts < WARPS && d.parts < steps_row && (long long)rows * d.parts * 2 <= 148 * 24) d.parts *= 2;
  d.each = cdiv((long long)rows * d.parts, warps);
  d.blocks = cdiv(rows, (long long)d.each * (WARPS / d.parts));
  return d;
}

}  // namespace

cudaError_t launch_kv_append(const PagedCache& c, const PagedRows& r, const bf16* qkv, long long row_stride, int heads, bool rotate,
                             const RopeTurns& turns, bf16* q_out, int* new_len, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  const Deal d = deal_rows(r.rows, cdiv(((rotate ? heads : 0) + 2 * c.kv_heads) * (c.head_dim / 16), 64));
  Launch l(d.blocks, THREADS, 0, s);
#define ET_APPEND(D, E, R) return cudaLaunchKernelEx(&l.cfg, kv_append_kernel<D, E, R>, qkv, row_stride, heads, c, r, turns, q_out, new_len, d.each, d.parts)
#define ET_APPEND4(D, R) return cudaLaunchKernelEx(&l.cfg, kv_append_int4_kernel<D, R>, qkv, row_stride, heads, c, r, turns, q_out, new_len, d.each, d.parts)
#define ET_APPEND_D(D)                                                       \
  do {                                                                       \
    if (c.format == ET_KV_INT4) { if (rotate) ET_APPEND4(D, true); else ET_APPEND4(D, false); }      \
    else if (c.format == ET_KV_E4M3) { if (rotate) ET_APPEND(D, true, true); else ET_APPEND(D, true, false); }   \
    else { if (rotate) ET_APPEND(D, false, true); else ET_APPEND(D, false, false); }               \
  } while (0)
  if (c.head_dim == 64) ET_APPEND_D(64); else ET_APPEND_D(128);
#undef ET_APPEND_D
#undef ET_APPEND4
#undef ET_APPEND
}

cudaError_t launch_kv_read(const PagedCache& c, const PagedRows& r, bf16* out, long long row_stride, cudaStream_t s) {
  ET_COUNT_LAUNCH();
  const Deal d = deal_rows(r.rows, cdiv(2 * c.kv_heads * c.head_dim / (c.format == ET_KV_E4M3 ? 16 : 8), 128));
  Launch l(d.blocks, THREADS, 0, s);
#define ET_READ(D, E) return cudaLaunchKernelEx(&l.cfg, kv_read_kernel<D, E>, out, row_stride, c, r, d.each, d.parts)
#define ET_READ_D(D)                                                         \
  do {                                                                       \
    if (c.format == ET_KV_INT4) ET_READ(D, ET_KV_INT4);                      \
    else if (c.format == ET_KV_E4M3) ET_READ(D, ET_KV_E4M3);                 \
    else ET_READ(D, ET_KV_BF16);                                             \
  } while (0)
  if (c.head_dim == 64) ET_READ_D(64); else ET_READ_D(128);
#undef ET_READ_D
#undef ET_READ
}

}  // namespace et
