// Attention of one new token of each sequence over its paged key / value cache.
//
// Every cached byte is read once and used for `group` query heads (7 in a Qwen2-7B layer), about 7 multiply-adds a byte:
// the cache's bytes over the memory bandwidth bound it, and the work is arranged to keep copies in flight.
//
//   * A tile is 64 positions of one key / value head.  All tiles of the call, in the order (sequence, key / value head,
//     tile), are cut into one equal run per CTA (one CTA per SM), so a single long sequence and a ragged batch load every
//     SM alike.  Lengths are on the device, so each CTA works the cut out for itself; an item (a sequence's tiles of one head)
//     counts for some tiles more than it has, for what its beginning and end cost.
//   * Four warps copy: TMA boxes of a page's rows (hardware swizzle, so that ldmatrix meets no bank conflicts) into a ring
//     of stages.  Eight warps compute, two to a tile, 32 positions each, every warp with a running maximum, sum and
//     output of its own.  They meet only at the end of a piece (the part of an item that falls into the CTA's run), one piece
//     late, so that nobody waits; where a CTA has several short items, each goes to one pair of warps alone.
//   * The product is transposed, S^T = K Q^T and O^T = V^T P^T, so that the query heads are the narrow side (8) of
//     mma.sync's m16n8k16: up to 8 heads cost no padded rows.  (tcgen05 wants 64 or more rows a tile, and the tensor work
//     here is a few per cent of the time.)
//   * A piece that is a whole item is written out at once; the others leave (output, maximum, sum) in the workspace, and a
//     second, small kernel joins them in a fixed order.
//
// Scores, maxima, sums and outputs are fp32; a weight is rounded to 16 bits of mantissa for bf16 values (two bf16 added), to 11
// for e4m3 ones (a half), which the output's rounding to 8 covers.  A half has few exponents, and an e4m3 value's scale is part of
// its weight: the largest weight is kept at 2^15, so that 11 bits are there down to 2^-29 of it, and a tile with scales more than
// 2^8 below those of the values that the scores favour takes two bf16 a weight instead.  So a probability has its 11 bits down
// to 2^-21 of the largest one, whatever the scales, and is off by at most 2^-32 of that one below.
//
// Device time in a chain of calls, B200, cache not in L2 (of the measured copy bandwidth; a pure read can pass 1); a second figure is
// for calls repeated for a second, at the clock that the power limit leaves.  28 heads on 4 of 128, bf16, one sequence of 100 003 38.5 us
// (0.82), of 7 675 10.5 (0.23: start and joining kernel); e4m3, 64 ragged sequences up to 16 001 55 / 59 us (0.85 / 0.79); 16 heads
// of 128 on 16, one of 180 000, bf16 219 / 221 us (1.04), e4m3 116 / 121 us (0.99 / 0.95); 24 ragged up to 2 049, 16 heads of 64, bf16
// 22 / 21 us (0.51 / 0.54), e4m3 the same (0.27): short items; 16 heads to a key / value head, 64 ragged, bf16 105 / 110 us (0.88 /
// 0.85), e4m3 71 / 74 us (0.66 / 0.64: bound by conversions and exponentials).
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>
#include <type_traits>

#include "decode.cuh"
#include "tcgen05.cuh"

namespace et {

namespace {

using namespace tc;

constexpr int TILE = 64;                       // positions
constexpr int GROUP_WARPS = 2;                 // warps of one tile, BLOCKS blocks of 16 positions each
constexpr int BLOCKS = TILE / 16 / GROUP_WARPS;
constexpr int COMPUTE_WARPS = 8;
constexpr int GROUPS = COMPUTE_WARPS / GROUP_WARPS;   // tiles are dealt to the groups in turn
constexpr int COPY_WARPS = GROUPS;             // one for each group's tiles
constexpr int THREADS = 32 * (COMPUTE_WARPS + COPY_WARPS);
// With 16 heads (NT = 2) the computing warps take registers from the copying ones: of what a block is launched with, never more.
constexpr int LAUNCH_REGS = 168, COMPUTE_REGS = 208, COPY_REGS = 88;
static_assert(COMPUTE_WARPS % 4 == 0 && COPY_WARPS % 4 == 0, "whole warpgroups");
static_assert(COMPUTE_WARPS * COMPUTE_REGS + COPY_WARPS * COPY_REGS <= (COMPUTE_WARPS + COPY_WARPS) * LAUNCH_REGS, "register budget");
// A group takes an item of up to so many tiles alone, where a CTA has several: 72 sequences of 250, 16 heads of 128, e4m3:
// 29.8 -> 18.3 us, 56 of 320 29.9 -> 21.5 us; with 32 a batch of long and short ones gets slower (55.8 -> 60.2 us).
constexpr int ALONE_TILES = 8;
// The tensor core cuts off what does not fit an accumulator, which adds up over long sums (0.0016 of positive outputs after a
// million positions in a CTA).  So a piece has at most this many tiles, a quarter for each group; what is longer becomes several
// pieces, whose outputs are added in fp32.
constexpr int PIECE_TILES = 256 * GROUPS;
constexpr int MAX_CTAS = 148;
constexpr int PAD = 4;                         // floats between heads of the joining buffer: no bank conflicts
constexpr int SMEM_LIMIT = 232448 - 512;       // 227 KB, less the static part
constexpr int CONTROL_BYTES = 1024;            // barriers and the ring's flags

template <int DH, bool E4M3, int NT>
struct Cfg {
  static constexpr int ROW = DH * (E4M3 ? 1 : 2);                 // bytes of a row
  static constexpr int BOX_ROW = ROW > 128 ? 128 : ROW;           // bytes of a box row: the swizzle's width
  static constexpr int BOXES = ROW / BOX_ROW;
  static constexpr int PLANE = TILE * ROW;
  static constexpr int STAGE = 2 * PLANE;                         // keys, values
  // What an item costs beside its tiles, in tiles' worth of time (measured: 2.3 us beside 0.6 us a tile for bf16 rows of 128, 2.0
  // and 0.3 for e4m3 ones, 1.4 and 0.25 for bf16 rows of 64; with 16 heads 2.8 and 0.65, 3.7 and 0.4; e4m3 rows of 64 follow the
  // same formula unmeasured); an item that a group takes alone costs a good third of it.
  static constexpr int COST = (2 + 65536 / STAGE) * (NT + 1) / 2, COST_SHORT = NT == 1 ? 1 + 32768 / STAGE : COST;
  static constexpr int SCALES = E4M3 ? 2 * TILE : 0;
  static constexpr int HEADS = 8 * NT;
  static constexpr int JOIN = COMPUTE_WARPS * HEADS * (DH + PAD) * 4 + COMPUTE_WARPS * HEADS * 3 * 4;   // the warps' results of a piece
  static constexpr int JOINS = NT == 1 ? 2 : 1;                   // pieces whose results can wait to be joined
  static constexpr int Q_ROW = DH * 2 + 16;                       // a head's query; 16 bytes more: no bank conflicts
  static constexpr bool ALONE = NT == 1;                          // (with 16 heads there is no room for what it takes)
  static constexpr int PAIR = ALONE ? HEADS * (DH + PAD) * 4 + 3 * HEADS * 4 : 0;   // a group's own results
  static constexpr int EDGE = JOINS * JOIN + GROUPS * (HEADS * Q_ROW + PAIR);
  static constexpr int FIT = (SMEM_LIMIT - 1024 - CONTROL_BYTES - EDGE) / (STAGE + SCALES);
  // a multiple of the groups, so that a stage is always the same warps': they wait for its copies in turn, where warps that come to a
  // stage for the first time in its second round could take the barrier's state of the first for their own
  static constexpr int STAGES = (FIT > 16 ? 16 : FIT) / GROUPS * GROUPS;
  static constexpr int SMEM = 1024 + STAGES * (STAGE + SCALES) + EDGE + CONTROL_BYTES;
  static_assert(STAGES >= GROUPS, "ring");
  static_assert(COST <= PAGED_ITEM_COST_MAX, "units");
  static_assert(8 * (2 * STAGES + 2 * GROUPS + 4) + 4 * STAGES + 16 <= CONTROL_BYTES, "control area");
};

// An item is the work of one sequence, key / value head and head tile (8 or 16 of the query heads that read it).
// Workspace: one descriptor per CTA, then two slots of partial results per CTA.
struct alignas(16) Join { int seq, part, pieces, slot; };         // pieces == 0: nothing of this CTA is to be joined
constexpr int SLOT0 = 1024;                                       // floats
static_assert(MAX_CTAS * sizeof(Join) <= SLOT0 * 4, "descriptors");
template <int DH, int NT> struct Slot { static constexpr int FLOATS = 8 * NT * (DH + 2); };
static_assert((SLOT0 + 2 * MAX_CTAS * Slot<128, 2>::FLOATS) * 4 <= (int)ET_PAGED_WORKSPACE, "workspace");

struct Args {
  PagedCache c;
  PagedAttention a;
  int group, parts, whole;          // heads per key / value head; head tiles per key / value head; 1: items are not cut
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// two e4m3 values (the low 16 bits) as two halves, exactly
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t x) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)x, __NV_E4M3);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// 2^e for e in [-127, 127]
__device__ __forceinline__ float pow2(int e) { return __int_as_float(e > -127 ? (e + 127) << 23 : 1 << 22); }
// two halves as two bf16, exactly for e4m3 values (4 bits, 2^-9 .. 448)
__device__ __forceinline__ uint32_t f16x2_to_bf16x2(uint32_t x) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
  return pack_bf16(f.x, f.y);
}
constexpr float WEIGHT_SHIFT = 15.f;           // e4m3: the largest weight is 2^15, halves end at 65504
constexpr float SCALE_SPAN = 8.f;              // e4m3: binades that a tile's scales may lie low for halves to hold its weights
// A weight as the sum of two bf16: its upper half, which is cut off and not rounded, and the rest.  The rest is above zero
// wherever the weight is (by 2^-24 of the weight too large), since an infinite value is multiplied by both, and with a zero or a
// negative number it would become a NaN or the other infinity.
__device__ __forceinline__ uint32_t upper_halves(float a, float b) { return __byte_perm(__float_as_uint(a), __float_as_uint(b), 0x7632); }
__device__ __forceinline__ float lower_part(float x) {
  return fmaf(__uint_as_float(__float_as_uint(x) & 0xffff0000u), -(1.f - 0x1p-24f), x);
}
// Copies by a converged warp: all lanes execute the call, one elected lane issues.
__device__ __forceinline__ void arrive_expect_elect(uint32_t bar, uint32_t bytes) {
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
               "@q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tma_load_elect(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, uint64_t policy) {
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
               "@q cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%3, %4}], [%2], %5;\n\t}"
               ::"r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y), "l"(policy) : "memory");
}
__device__ __forceinline__ void bulk_load_elect(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
               "@q cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t}"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void group_sync(int group) { asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(32 * GROUP_WARPS) : "memory"); }
// 16 bytes by a lane's own asynchronous copy (zeros if not live); copies_arrive: an arrival once the lane's copies so far are there
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool live) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ int clamped_len(const Args& g, int s) {
  const long long cap = (long long)g.a.max_pages << g.c.page_shift;
  return (int)min((long long)max(g.a.len[s], 0), cap);
}
// An item's units: its tiles and, in front of them, units for what it costs beside them.  C: the kernel's Cfg
__device__ __forceinline__ int tiles_of(int len) { return (int)((unsigned)(len + (TILE - 1)) / TILE); }
template <class C> __device__ __forceinline__ int cost_of(int tiles) { return tiles <= ALONE_TILES ? C::COST_SHORT : C::COST; }
template <class C> __device__ __forceinline__ int units_of(const Args& g, int len) {
  const int tiles = tiles_of(len);
  return len <= 0 ? 0 : g.whole ? 1 : tiles + cost_of<C>(tiles);
}

// The run of units that falls to a CTA, walked piece by piece.
struct Walk {
  int left;                        // units still to do
  int s, part, unit;               // next unit: sequence, key / value head x head tile, unit of the item
  int len;                         // of the sequence
  bool opened;                     // a piece has been given out
  bool cut, cut_first, cut_opens;  // the last one was ended for its length; it was `first`, `opens`
};

struct Piece {
  int s, part, len, t0, t1;        // tiles t0 .. t1 - 1
  int units, units_end;            // the item's units, and those up to this piece's end
  bool first, last;                // contains the item's first, last tile (first: or goes on from a piece that does)
  bool opens;                      // is the first piece of its run (or goes on from it)
  bool goes_on, more;              // goes on from the piece before; the next piece goes on from it
};

// Which of a piece's tiles a group takes: every GROUPS-th one, or all or none of an item that is short next to the run (a
// piece that the groups share costs them all its queries, its result and a wait for one another, as much as several tiles).
// `turn` goes round the groups; copying and computing warps deal alike.
struct Deal { int t, step; bool alone; };
__device__ __forceinline__ Deal deal(const Piece& p, bool may, int chunk, int group, int& turn) {
  Deal d;
  const int n = p.t1 - p.t0;
  d.alone = may && n <= ALONE_TILES && p.units * GROUPS <= chunk && !p.goes_on;
  const int behind = (group - turn) & (GROUPS - 1);
  d.t = d.alone ? (behind == 0 ? p.t0 : p.t1) : p.t0 + behind;
  d.step = d.alone ? 1 : GROUPS;
  turn = (turn + (d.alone ? 1 : n)) & (GROUPS - 1);
  return d;
}

template <class C>
__device__ __forceinline__ bool next_piece(const Args& g, int parts_all, Walk& w, Piece& p) {
  while (w.left > 0) {
    const int units = units_of<C>(g, w.len);
    if (units > 0) {
      int end = w.unit + min(w.left, units - w.unit);
      p.s = w.s; p.part = w.part; p.len = w.len; p.units = units;
      const int tiles = tiles_of(w.len), cost = cost_of<C>(tiles);
      p.t0 = g.whole ? 0 : max(w.unit - cost, 0);
      p.t1 = g.whole ? tiles : max(end - cost, 0);
      p.more = p.t1 - p.t0 > PIECE_TILES;
      if (p.more) { p.t1 = p.t0 + PIECE_TILES; end = p.t1 + cost; }        // (an item that is not cut has no such length)
      p.goes_on = w.cut;
      p.first = w.cut ? w.cut_first : p.t0 == 0;
      p.last = end == units; p.units_end = end;
      w.left -= end - w.unit; w.unit = end;
      if (end == units) { w.unit = 0; ++w.part; }
    }
    if (units == 0 || w.part == parts_all) {                      // on to the next sequence
      w.part = 0;
      if (++w.s >= g.a.n_seq) w.left = 0; else if (w.left > 0) w.len = clamped_len(g, w.s);
    }
    if (units > 0 && p.t1 > p.t0) {                               // else the run ended in front of the item's first tile
      p.opens = w.cut ? w.cut_opens : !w.opened;
      w.opened = true; w.cut = p.more; w.cut_first = p.first; w.cut_opens = p.opens;
      return true;
    }
  }
  return false;
}

template <int DH, bool E4M3, int NT>
__global__ void __launch_bounds__(THREADS, 1)
attention_paged_kernel(const __grid_constant__ CUtensorMap map, const __grid_constant__ Args g) {
  using C = Cfg<DH, E4M3, NT>;
  constexpr int STAGES = C::STAGES, KS = DH / 16;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
  uint8_t* const gen = smem_raw + (base - raw);
  const uint32_t scales = base + STAGES * C::STAGE;
  uint8_t* const edge = gen + STAGES * (C::STAGE + C::SCALES);
  // results of a piece, each warp's: [COMPUTE_WARPS][HEADS][DH + PAD] outputs, then [3][COMPUTE_WARPS][HEADS]: maximum, output's
  // maximum, sum
  constexpr int JOIN_M = COMPUTE_WARPS * C::HEADS * (DH + PAD);
  auto join_of = [&](int i) { return reinterpret_cast<float*>(edge + i * C::JOIN); };
  auto query_of = [&](int i) { return edge + C::JOINS * C::JOIN + i * (C::HEADS * C::Q_ROW); };             // of a group
  auto pair_of = [&](int i) { return reinterpret_cast<float*>(edge + C::JOINS * C::JOIN + GROUPS * (C::HEADS * C::Q_ROW) + i * C::PAIR); };
  uint8_t* const ctl = edge + C::EDGE;
  const uint32_t bars = smem_u32(ctl);
  auto full = [&](int s) { return bars + 8u * (uint32_t)s; };
  auto empty = [&](int s) { return bars + 8u * (uint32_t)(STAGES + s); };
  auto q_full = [&](int i) { return bars + 8u * (uint32_t)(2 * STAGES + i); };
  auto q_empty = [&](int i) { return bars + 8u * (uint32_t)(2 * STAGES + GROUPS + i); };
  auto o_full = [&](int i) { return bars + 8u * (uint32_t)(2 * STAGES + 2 * GROUPS + i); };
  auto o_empty = [&](int i) { return bars + 8u * (uint32_t)(2 * STAGES + 2 * GROUPS + 2 + i); };
  volatile int* const absent = reinterpret_cast<volatile int*>(ctl + 8 * (2 * STAGES + 2 * GROUPS + 4));   // [STAGES]: bit i = slice i has no page
  volatile int* const abort_flag = absent + STAGES;

  __shared__ int warp_sum_s[THREADS / 32];
  __shared__ int walk_s[4];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x;
  const int kv_heads = g.c.kv_heads, parts_all = kv_heads * g.parts;
  if (tid == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");

  if (tid < STAGES) { mbar_init(full(tid), 1); mbar_init(empty(tid), GROUP_WARPS); }
  if (tid < GROUPS) { mbar_init(q_full(tid), 32); mbar_init(q_empty(tid), GROUP_WARPS); }
  if (tid < C::JOINS) { mbar_init(o_full(tid), COMPUTE_WARPS); mbar_init(o_empty(tid), COMPUTE_WARPS); }
  if (tid == 0) *abort_flag = 0;
  if (tid < 32) asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");

  begin_after_previous();
  // ---- this CTA's run: an exclusive prefix sum of the sequences' units over the threads
  Walk walk;
  int begin, chunk;                            // all units together are below 2^31 (checked on the host)
  {
    const int per = (g.a.n_seq + THREADS - 1) / THREADS, s0 = min(tid * per, g.a.n_seq), s1 = min(s0 + per, g.a.n_seq);
    int sum = 0;
    for (int s = s0; s < s1; ++s) sum += units_of<C>(g, clamped_len(g, s));
    sum *= parts_all;
    int inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int v = __shfl_up_sync(0xffffffffu, inc, o); if (lane >= o) inc += v; }
    if (lane == 31) warp_sum_s[warp] = inc;
    __syncthreads();
    int before = inc - sum, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) { const int v = warp_sum_s[w]; if (w < warp) before += v; total += v; }
    chunk = (int)(((unsigned)total + gridDim.x - 1) / gridDim.x);
    begin = min(chunk * b, total);
    if (begin >= before && begin < before + sum) {
      int r = begin - before;
      for (int s = s0; s < s1; ++s) {
        const int len = clamped_len(g, s), u = units_of<C>(g, len);
        if (r < u * parts_all) { walk_s[0] = s; walk_s[1] = r / u; walk_s[2] = r % u; walk_s[3] = len; break; }
        r -= u * parts_all;
      }
    }
    __syncthreads();
    walk.left = min(chunk, total - begin);
    walk.s = walk_s[0]; walk.part = walk_s[1]; walk.unit = walk_s[2]; walk.len = walk_s[3]; walk.opened = walk.cut = false;
  }

  bool ok = true;
  if constexpr (NT == 2) {
    if (warp >= COMPUTE_WARPS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(COPY_REGS));
    else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(COMPUTE_REGS));
  }
  if (warp >= COMPUTE_WARPS) {
    // ------------------------------------------------------------------ copies
    const int me = warp - COMPUTE_WARPS;
    const int box_shift = min(g.c.page_shift, 6), box_rows = 1 << box_shift, boxes_tile = TILE >> box_shift;
    const uint32_t box_bytes = (uint32_t)box_rows * (2 * C::ROW + (E4M3 ? 2 : 0));
    const int plane_rows = kv_heads << g.c.page_shift;
    // the cache is read once (several head tiles read it soon after one another): it need not push other things out of L2
    uint64_t policy;
    if (g.parts > 1) asm volatile("createpolicy.fractional.L2::evict_normal.b64 %0, 1.0;" : "=l"(policy));
    else asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    int stage = me;
    uint32_t phase = 0;
    long long issued = 0;
    int turn = 0;
    uint32_t q_phase = 0;
    Piece p;
    while (ok && next_piece<C>(g, parts_all, walk, p)) {
      const Deal dl = deal(p, C::ALONE, chunk, me, turn);
      if (dl.t >= p.t1) continue;
      // the piece's queries: rows of the heads, zeros for heads that the group does not have
      ok = mbar_wait_warp(q_empty(me), q_phase ^ 1u, abort_flag);
      if (!ok) break;
      q_phase ^= 1u;
      {
        const int h0 = (p.part % g.parts) * C::HEADS;
        const bf16* src = g.a.q + (size_t)p.s * g.a.q_stride + (size_t)((p.part / g.parts) * g.group + h0) * DH;
        const uint32_t dst = smem_u32(query_of(me));
#pragma unroll
        for (int i = 0; i < C::HEADS * (DH / 8) / 32; ++i) {
          const int e = i * 32 + lane, h = e / (DH / 8), d = e % (DH / 8);
          copy16(dst + h * C::Q_ROW + d * 16, src + (h0 + h < g.group ? h * DH + d * 8 : 0), h0 + h < g.group);
        }
        copies_arrive(q_full(me));
      }
      const int* table = g.a.table + (size_t)p.s * g.a.max_pages;
      const int kvh = p.part / g.parts;
      const int first_page = (int)(((long long)p.t0 * TILE) >> g.c.page_shift);
      const int last_page = (p.len - 1) >> g.c.page_shift;            // of the sequence
      // 32 entries of the table, one per lane, as the first rows of their keys in the cache (-1: not a page of the cache)
      auto load_ids = [&](int batch) {
        const long long i = (long long)first_page + batch * 32 + lane;
        return i <= last_page ? table[i] : 0;
      };
      auto rows_of = [&](int page) {
        const bool good = (unsigned)page < (unsigned)g.c.n_pages;
        if (!good && g.a.status) atomicMax(g.a.status, (int)ET_PAGED_BAD_PAGE);
        return good ? (page * 2 * kv_heads + kvh) << g.c.page_shift : -1;
      };
      int batch = 0, rows = rows_of(load_ids(0)), ids_next = load_ids(1);
      for (int t = dl.t; t < p.t1; t += dl.step) {
        const int pos = t * TILE;                                     // lengths are below 2^31
        const int page0 = (pos >> g.c.page_shift) - first_page;       // a multiple of the tile's pages: one batch has them all
        while ((page0 >> 5) > batch) { ++batch; rows = rows_of(ids_next); ids_next = load_ids(batch + 1); }
        const int in_page = pos & ((1 << g.c.page_shift) - 1);
        const int boxes = min(boxes_tile, (p.len - pos + box_rows - 1) >> box_shift);      // with positions
        int row[4], missing = 0;                                      // first row of each box's keys; negative: none
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          row[i] = __shfl_sync(0xffffffffu, rows, (page0 + i) & 31);
          if (i >= boxes) row[i] = -1;
          else if (row[i] < 0) missing |= 1 << i;
        }
        ok = mbar_wait_warp(empty(stage), phase ^ 1u, abort_flag);
        if (!ok) break;
        int gone = 0;
        if (missing)
          for (int i = 0; i < boxes; ++i) if (missing >> i & 1) gone |= ((1 << (box_rows / 16)) - 1) << (i * (box_rows / 16));
        if (lane == 0) absent[stage] = gone;
        __syncwarp();
        const uint32_t bar = full(stage), dst = base + stage * C::STAGE, sdst = scales + stage * C::SCALES;
        arrive_expect_elect(bar, (boxes - __popc(missing)) * box_bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (row[i] >= 0) {
            const int r0 = i << box_shift;
#pragma unroll
            for (int plane = 0; plane < 2; ++plane) {
              const int y = row[i] + in_page + plane * plane_rows;
#pragma unroll
              for (int half = 0; half < C::BOXES; ++half)
                tma_load_elect(dst + plane * C::PLANE + half * (TILE * C::BOX_ROW) + r0 * C::BOX_ROW, &map, bar,
                               half * (C::BOX_ROW / (E4M3 ? 1 : 2)), y, policy);
              if (E4M3) bulk_load_elect(sdst + plane * TILE + r0, g.c.scale + (unsigned)y, (uint32_t)box_rows, bar);
            }
          }
        }
        ++issued;
        if ((stage += GROUPS) >= STAGES) { stage = me; phase ^= 1u; }
      }
    }
    // copies have to land before this CTA's shared memory is given up, also if nobody waits for them any more
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (lane == 0) {
      for (int i = 0; i < STAGES / GROUPS && i < issued; ++i) {
        if ((stage -= GROUPS) < 0) { stage = STAGES - GROUPS + me; phase ^= 1u; }
        int given_up = 0;
        mbar_wait(full(stage), phase, &given_up);
      }
    }
  } else {
    // ------------------------------------------------------------------ the product
    const int my_group = warp / GROUP_WARPS, slice = (warp % GROUP_WARPS) * BLOCKS, r0 = slice * 16;    // first slice (of 16) and row
    const int gq = lane >> 2, tq = lane & 3;                         // mma's row group and column pair
    // this lane's row of the 16 and its 16-byte chunk (K: both halves of a k-step; V, transposed: see below)
    const int krow = r0 + (lane & 7) + ((lane >> 3) & 1) * 8, kchunk = lane >> 4;
    const int vrow = E4M3 ? krow : r0 + (lane & 7) + (lane >> 4) * 8, vchunk = E4M3 ? kchunk : (lane >> 3) & 1;
    auto swizzled = [&](int row, int chunk) -> uint32_t {            // 16-byte chunk of a row, as the copies place it
      if constexpr (C::BOX_ROW == 128)
        return (uint32_t)((chunk >> 3) * (TILE * 128) + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
      else
        return (uint32_t)(row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4));
    };
    const float softmax_scale = 1.4426950408889634f * (DH == 128 ? 0.08838834764831845f : 0.125f);   // log2(e) / sqrt(DH)

    // Four values of a head's output (not yet divided), its maximum and sum: to the output, or to the workspace if others follow.
    // A piece that goes on adds what the one before has left there; a head's lanes are the same ones of one warp then (`lanes`).
    auto put = [&](const Piece& p, int h, int d, float4 acc, float top, float sum, unsigned lanes) {
      if (p.goes_on) {
        const float* const part = g.a.workspace + SLOT0 + (size_t)(2 * b + (p.opens ? 0 : 1)) * Slot<DH, NT>::FLOATS;
        const float4 x = *reinterpret_cast<const float4*>(part + h * DH + d);
        const float top0 = part[C::HEADS * DH + 2 * h], sum0 = part[C::HEADS * DH + 2 * h + 1];
        __syncwarp(lanes);                                           // read by all before one of them writes
        const float now = fmaxf(top0, top), ref = now == -INFINITY ? 0.f : now, f0 = exp2_fast(top0 - ref), f = exp2_fast(top - ref);
        acc = make_float4(x.x * f0 + acc.x * f, x.y * f0 + acc.y * f, x.z * f0 + acc.z * f, x.w * f0 + acc.w * f);
        sum = sum0 * f0 + sum * f;
        top = now;
      }
      if (p.first && p.last) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;              // every page absent: zeros
        const size_t at = (size_t)p.s * g.a.heads + (p.part / g.parts) * g.group + (p.part % g.parts) * C::HEADS + h;
        *reinterpret_cast<uint2*>(g.a.out + at * DH + d) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        if (d == 0 && g.a.lse) g.a.lse[at] = sum == 0.f ? -INFINITY : (log2f(sum) + top) * 0.6931471805599453f;
      } else {
        float* const part = g.a.workspace + SLOT0 + (size_t)(2 * b + (p.opens ? 0 : 1)) * Slot<DH, NT>::FLOATS;
        *reinterpret_cast<float4*>(part + h * DH + d) = acc;
        if (d == 0) { part[C::HEADS * DH + 2 * h] = top; part[C::HEADS * DH + 2 * h + 1] = sum; }
      }
    };
    auto heads_of = [&](const Piece& p) { return min(C::HEADS, g.group - (p.part % g.parts) * C::HEADS); };
    // Joins the warps' results of the i-th piece that all groups share: every warp has left its own in a buffer and takes a
    // part of the heads' outputs.
    auto join_piece = [&](const Piece& p, int i) {
      const int buf = i % C::JOINS;
      if (ok) ok = mbar_wait_warp(o_full(buf), (uint32_t)(i / C::JOINS) & 1u, abort_flag);
      const float* const join = join_of(buf);
      const float* const join_m = join + JOIN_M;
      const int live = heads_of(p);
      for (int e = tid; ok && e < live * (DH / 4); e += 32 * COMPUTE_WARPS) {
        const int h = e / (DH / 4), d = (e % (DH / 4)) * 4;
        float top = -INFINITY, sum = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < COMPUTE_WARPS; ++w) top = fmaxf(top, join_m[w * C::HEADS + h]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int w = 0; w < COMPUTE_WARPS; ++w) {
          const float lw = join_m[(2 * COMPUTE_WARPS + w) * C::HEADS + h];
          if (lw != 0.f) {                                           // a warp without positions left no output (NaN is not zero)
            const float fl = exp2_fast(join_m[w * C::HEADS + h] - ref), fo = exp2_fast(join_m[(COMPUTE_WARPS + w) * C::HEADS + h] - ref);
            const float4 x = *reinterpret_cast<const float4*>(join + (w * C::HEADS + h) * (DH + PAD) + d);
            sum += lw * fl;
            acc.x += x.x * fo; acc.y += x.y * fo; acc.z += x.z * fo; acc.w += x.w * fo;
          }
        }
        put(p, h, d, acc, top, sum, live * (DH / 4) - (e - lane) >= 32 ? 0xffffffffu : 0xffffu);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(o_empty(buf));
    };

    Join mine{0, 0, 0, 0};
    int stage = my_group, shared = 0, turn = 0;                      // shared: pieces so far that all groups shared
    uint32_t phase = 0, q_phase = 0;
    Piece p, before;
    while (next_piece<C>(g, parts_all, walk, p)) {
      if (p.first && !p.last && !p.more) {
        // the item goes on in the CTAs behind this one, each of which finds it at the start of its run
        const int item0 = begin + chunk - p.units_end;               // this piece ends this CTA's run (whole items are not cut)
        mine = Join{p.s, p.part, (item0 + p.units - 1) / chunk - b + 1, 2 * b + (p.opens ? 0 : 1)};
      }
      const Deal dl = deal(p, C::ALONE, chunk, my_group, turn);
      const bool busy = dl.t < p.t1;                                 // this group has tiles of the piece
      if (dl.alone && !busy) continue;
      if (busy && ok) ok = mbar_wait_warp(q_full(my_group), q_phase, abort_flag);
      const uint8_t* const query = query_of(my_group);
      // ---- Q^T as the B operand: column gq = head, two rows (pairs of dimensions) a register
      uint32_t q[NT][KS][2];
      float qscale[NT][2];                                           // of heads 2 tq and 2 tq + 1
      if (busy) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const uint8_t* src = query + (n * 8 + gq) * C::Q_ROW;
          if constexpr (!E4M3) {
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              q[n][k][0] = *reinterpret_cast<const uint32_t*>(src + k * 32 + 4 * tq);
              q[n][k][1] = *reinterpret_cast<const uint32_t*>(src + k * 32 + 16 + 4 * tq);
            }
            qscale[n][0] = qscale[n][1] = softmax_scale;
          } else {
            // e4m3 keys are multiplied as halves, which hold them exactly.  A query row is scaled by a power of two that
            // brings its largest value to 2^14 .. 2^15: a value below 2^-29 of that loses bits, no other.  The dimensions of
            // a k-step are taken in the order that the keys' bytes come in: 4 tq, 4 tq + 1 | 4 tq + 2, 4 tq + 3.
            uint2 raw_q[KS];
            float top = 0.f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              raw_q[k] = *reinterpret_cast<const uint2*>(src + k * 32 + 8 * tq);
              const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw_q[k].x));
              const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw_q[k].y));
              top = fmaxf(top, fmaxf(fmaxf(fabsf(x.x), fabsf(x.y)), fmaxf(fabsf(y.x), fabsf(y.y))));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const int e = top > 0.f ? max((__float_as_int(top) >> 23) - 127 - 14, -127) : 0;
            const float f = pow2(-e);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw_q[k].x));
              const float2 y = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&raw_q[k].y));
              q[n][k][0] = pack_f16(x.x * f, x.y * f);
              q[n][k][1] = pack_f16(y.x * f, y.y * f);
            }
            const float back = pow2(e) * softmax_scale;
            qscale[n][0] = __shfl_sync(0xffffffffu, back, 8 * tq);
            qscale[n][1] = __shfl_sync(0xffffffffu, back, 8 * tq + 4);
          }
        }
      }
      if (busy) {
        q_phase ^= 1u;
        __syncwarp();
        if (lane == 0) mbar_arrive(q_empty(my_group));
      }
      // per head 2 tq + i: running maximum m of the scores (base 2), sum l of this lane's positions; mo: maximum of score +
      // log2(scale of the value), against which the output is kept (e4m3: a value's scale is part of its weight)
      float o[NT][KS][4], m[NT][2], mo[NT][2], l[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        m[n][0] = m[n][1] = mo[n][0] = mo[n][1] = -INFINITY;
        l[n][0] = l[n][1] = 0.f;
#pragma unroll
        for (int k = 0; k < KS; ++k) o[n][k][0] = o[n][k][1] = o[n][k][2] = o[n][k][3] = 0.f;
      }

      for (int t = dl.t; t < p.t1; t += dl.step) {
        const int st = stage;
        const uint32_t ph = phase;
        if ((stage += GROUPS) >= STAGES) { stage = my_group; phase ^= 1u; }
        if (ok) ok = mbar_wait_warp(full(st), ph, abort_flag);
        if (!ok) continue;
        // positions of each block that count: up to the length, none on an absent page (a page has whole slices)
        const int gone = absent[st] >> slice;
        int valid[BLOCKS], any = 0;
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
          const int room = p.len - t * TILE - r0 - 16 * j;
          valid[j] = (gone >> j & 1) ? 0 : max(0, min(16, room));
          any |= valid[j];
        }
        if (any) {
          const uint32_t kb = base + st * C::STAGE, vb = kb + C::PLANE;
          // ---- S^T = K Q^T: rows = positions gq, gq + 8 of a block, columns = heads 2 tq, 2 tq + 1
          float s[BLOCKS][NT][4];
#pragma unroll
          for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
            for (int n = 0; n < NT; ++n) s[j][n][0] = s[j][n][1] = s[j][n][2] = s[j][n][3] = 0.f;
          if constexpr (!E4M3) {
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
              for (int j = 0; j < BLOCKS; ++j) {
                uint32_t a[4];
                ldmatrix4(kb + swizzled(krow + 16 * j, 2 * k + kchunk), a);
#pragma unroll
                for (int n = 0; n < NT; ++n) mma16816<false>(s[j][n], a[0], a[1], a[2], a[3], q[n][k][0], q[n][k][1]);
              }
          } else {
#pragma unroll
            for (int k = 0; k < KS; k += 2)
#pragma unroll
              for (int j = 0; j < BLOCKS; ++j) {
                uint32_t a[4];                                        // positions gq / gq + 8 of k-step k, then of k + 1
                ldmatrix4(kb + swizzled(krow + 16 * j, k + kchunk), a);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                  const uint32_t a0 = e4m3x2_to_f16x2(a[2 * i] & 0xffffu), a2 = e4m3x2_to_f16x2(a[2 * i] >> 16);
                  const uint32_t a1 = e4m3x2_to_f16x2(a[2 * i + 1] & 0xffffu), a3 = e4m3x2_to_f16x2(a[2 * i + 1] >> 16);
#pragma unroll
                  for (int n = 0; n < NT; ++n) mma16816<true>(s[j][n], a0, a1, a2, a3, q[n][k + i][0], q[n][k + i][1]);
                }
              }
          }
          // scales of the block's two positions of this lane: keys' as factors, values' as exponents
          float ks[BLOCKS][2], ve[BLOCKS][2];
#pragma unroll
          for (int j = 0; j < BLOCKS; ++j) {
            if constexpr (E4M3) {
              const uint8_t* sc = gen + STAGES * C::STAGE + st * C::SCALES + r0 + 16 * j + gq;
              ks[j][0] = pow2((int)sc[0] - 127); ks[j][1] = pow2((int)sc[8] - 127);
              ve[j][0] = (float)((int)sc[TILE] - 127); ve[j][1] = (float)((int)sc[TILE + 8] - 127);
            } else {
              ks[j][0] = ks[j][1] = 1.f; ve[j][0] = ve[j][1] = 0.f;
            }
          }
          // e4m3: the smallest exponent of a live value, below which by how much the scores' favourites lie (mo - m)
          float lowest = INFINITY;
          if constexpr (E4M3) {
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j) {
              if (gq < valid[j]) lowest = fminf(lowest, ve[j][0]);
              if (gq + 8 < valid[j]) lowest = fminf(lowest, ve[j][1]);
            }
            lowest += SCALE_SPAN;
          }
          bool moved = false, spread = false;
          float alpha[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float top = -INFINITY, topo = -INFINITY;
#pragma unroll
              for (int j = 0; j < BLOCKS; ++j) {
                float& x = s[j][n][i];
                float& y = s[j][n][i + 2];
                x = gq < valid[j] ? x * qscale[n][i] * ks[j][0] : -INFINITY;
                y = gq + 8 < valid[j] ? y * qscale[n][i] * ks[j][1] : -INFINITY;
                top = fmaxf(top, fmaxf(x, y));
                if (E4M3) topo = fmaxf(topo, fmaxf(x + ve[j][0], y + ve[j][1]));
              }
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (E4M3) topo = fmaxf(topo, __shfl_xor_sync(0xffffffffu, topo, d));
              }
              const float mn = fmaxf(m[n][i], top), mu = mn == -INFINITY ? 0.f : mn;
              const float al = exp2_fast(m[n][i] - mu);
              float ou = 0.f, sum = 0.f;
              if (!E4M3) {
                moved |= mn != m[n][i];
                alpha[n][i] = al;
              } else {
                const float on = fmaxf(mo[n][i], topo);
                ou = on == -INFINITY ? 0.f : on;
                moved |= on != mo[n][i];
                alpha[n][i] = exp2_fast(mo[n][i] - ou);
                mo[n][i] = on;
                spread |= on - mn > lowest;
                ou -= WEIGHT_SHIFT;
              }
              // the scores become weights
#pragma unroll
              for (int j = 0; j < BLOCKS; ++j) {
                const float x = s[j][n][i], y = s[j][n][i + 2];
                const float e0 = exp2_fast(x - mu), e1 = exp2_fast(y - mu);
                sum += e0 + e1;
                s[j][n][i] = E4M3 ? exp2_fast(x + ve[j][0] - ou) : e0;
                s[j][n][i + 2] = E4M3 ? exp2_fast(y + ve[j][1] - ou) : e1;
              }
              l[n][i] = l[n][i] * al + sum;
              m[n][i] = mn;
            }
          // ---- O^T += V^T P^T.  P as the B operand: 8 x 8 transposes of the accumulator's pairs.  PAIR: a probability is split
          // into two bf16 (16 bits of it count); halves hold 11 bits of it.  Whatever stands behind the length must not meet a
          // zero probability (0 * NaN is NaN): the values there are cleared.
          auto add_values = [&](auto pair) {
            constexpr bool PAIR = decltype(pair)::value;
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j) {
              uint32_t ph0[NT], ph1[NT], pl0[NT], pl1[NT];
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                const float* x = s[j][n];
                if constexpr (!PAIR) {
                  ph0[n] = transpose8x8(pack_f16(x[0], x[1]));
                  ph1[n] = transpose8x8(pack_f16(x[2], x[3]));
                } else {
                  ph0[n] = transpose8x8(upper_halves(x[0], x[1]));
                  ph1[n] = transpose8x8(upper_halves(x[2], x[3]));
                  pl0[n] = transpose8x8(pack_bf16(lower_part(x[0]), lower_part(x[1])));
                  pl1[n] = transpose8x8(pack_bf16(lower_part(x[2]), lower_part(x[3])));
                }
              }
              const uint32_t keep0 = (2 * tq < valid[j] ? 0xffffu : 0u) | (2 * tq + 1 < valid[j] ? 0xffff0000u : 0u);
              const uint32_t keep1 = (2 * tq + 8 < valid[j] ? 0xffffu : 0u) | (2 * tq + 9 < valid[j] ? 0xffff0000u : 0u);
              if constexpr (!E4M3) {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  uint32_t a[4];                                      // rows d = 16 k + gq, + 8; columns = positions
                  ldmatrix4_trans(vb + swizzled(vrow + 16 * j, 2 * k + vchunk), a);
                  a[0] &= keep0; a[1] &= keep0; a[2] &= keep1; a[3] &= keep1;
#pragma unroll
                  for (int n = 0; n < NT; ++n) {
                    mma16816<false>(o[n][k], a[0], a[1], a[2], a[3], ph0[n], ph1[n]);
                    mma16816<false>(o[n][k], a[0], a[1], a[2], a[3], pl0[n], pl1[n]);
                  }
                }
              } else {
#pragma unroll
                for (int k = 0; k < KS; k += 2) {
                  // a transposed 8 x 8 of byte pairs: this lane has dimensions 2 gq, 2 gq + 1 of positions 2 tq, 2 tq + 1 (and + 8)
                  uint32_t a[4];
                  ldmatrix4_trans(vb + swizzled(vrow + 16 * j, k + vchunk), a);
#pragma unroll
                  for (int i = 0; i < 2; ++i) {
                    const uint32_t x = __byte_perm(a[2 * i] & keep0, 0, 0x3120), y = __byte_perm(a[2 * i + 1] & keep1, 0, 0x3120);
                    uint32_t a0 = e4m3x2_to_f16x2(x & 0xffffu), a1 = e4m3x2_to_f16x2(x >> 16);
                    uint32_t a2 = e4m3x2_to_f16x2(y & 0xffffu), a3 = e4m3x2_to_f16x2(y >> 16);
                    if constexpr (PAIR) {
                      a0 = f16x2_to_bf16x2(a0); a1 = f16x2_to_bf16x2(a1); a2 = f16x2_to_bf16x2(a2); a3 = f16x2_to_bf16x2(a3);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                      mma16816<!PAIR>(o[n][k + i], a0, a1, a2, a3, ph0[n], ph1[n]);
                      if constexpr (PAIR) mma16816<false>(o[n][k + i], a0, a1, a2, a3, pl0[n], pl1[n]);
                    }
                  }
                }
              }
            }
          };
          // one vote for both rare things: outputs to be scaled down, scales too far apart
          bool added = false;
          if (__any_sync(0xffffffffu, moved || spread)) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                o[n][k][0] *= alpha[n][0]; o[n][k][1] *= alpha[n][1]; o[n][k][2] *= alpha[n][0]; o[n][k][3] *= alpha[n][1];
              }
            if constexpr (E4M3)
              if (__any_sync(0xffffffffu, spread)) {
                add_values(std::true_type());
                added = true;
              }
          }
          if (!added) add_values(std::bool_constant<!E4M3>());
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
      }

      // ---- this warp's result
      if constexpr (E4M3) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < KS; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][k][i] *= 1.f / 32768.f;       // 2^-WEIGHT_SHIFT
      }
      const int live = heads_of(p);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], d);
      // dst: rows of heads' outputs
      auto leave_output = [&](float* dst) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int h = n * 8 + 2 * tq + i;
            if (h >= live) continue;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
              if (E4M3) *reinterpret_cast<float2*>(dst + h * (DH + PAD) + 16 * k + 2 * gq) = make_float2(o[n][k][i], o[n][k][i + 2]);
              else { dst[h * (DH + PAD) + 16 * k + gq] = o[n][k][i]; dst[h * (DH + PAD) + 16 * k + 8 + gq] = o[n][k][i + 2]; }
            }
          }
      };
      if (C::ALONE && dl.alone) {
        // the group's two warps: the first leaves its result, the second adds its own, both put the sum out
        float* const pair = pair_of(my_group);
        float* const pair_m = pair + C::HEADS * (DH + PAD);           // [3][HEADS]: maximum, output's maximum, sum
        group_sync(my_group);                                         // the memory is free
        if (warp % GROUP_WARPS == 0) {
          leave_output(pair);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int h = 2 * tq + i;
            if (gq == 0) { pair_m[h] = m[0][i]; pair_m[C::HEADS + h] = E4M3 ? mo[0][i] : m[0][i]; pair_m[2 * C::HEADS + h] = l[0][i]; }
          }
        }
        group_sync(my_group);
        if (warp % GROUP_WARPS == 1) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int h = 2 * tq + i;
            const float ma = pair_m[h], oa = pair_m[C::HEADS + h], la = pair_m[2 * C::HEADS + h];
            const float top = fmaxf(ma, m[0][i]), ref = top == -INFINITY ? 0.f : top;
            const float fa = exp2_fast(oa - ref), fb = exp2_fast((E4M3 ? mo[0][i] : m[0][i]) - ref);
            float* const dst = pair + h * (DH + PAD);
            if (h < live)
#pragma unroll
              for (int k = 0; k < KS; ++k) {
                float* const x = dst + 16 * k + (E4M3 ? 2 * gq : gq);
                float* const y = x + (E4M3 ? 1 : 8);
                *x = *x * fa + o[0][k][i] * fb;
                *y = *y * fa + o[0][k][i + 2] * fb;
              }
            __syncwarp();
            if (gq == 0) { pair_m[h] = top; pair_m[2 * C::HEADS + h] = la * exp2_fast(ma - ref) + l[0][i] * exp2_fast(m[0][i] - ref); }
          }
        }
        group_sync(my_group);
        for (int e = tid % (32 * GROUP_WARPS); ok && e < live * (DH / 4); e += 32 * GROUP_WARPS) {
          const int h = e / (DH / 4), d = (e % (DH / 4)) * 4;
          put(p, h, d, *reinterpret_cast<const float4*>(pair + h * (DH + PAD) + d), pair_m[h], pair_m[2 * C::HEADS + h], 0u);
        }
        continue;
      }
      // ---- the shared piece before is joined now, when its slowest warp is done; then this warp leaves its result of this one
      if (shared > 0) join_piece(before, shared - 1);
      const int buf = shared % C::JOINS;
      if (ok) ok = mbar_wait_warp(o_empty(buf), ((uint32_t)(shared / C::JOINS) & 1u) ^ 1u, abort_flag);
      if (ok) {
        float* const join = join_of(buf);
        float* const join_m = join + JOIN_M;
        if (gq == 0) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int h = n * 8 + 2 * tq + i;
              join_m[warp * C::HEADS + h] = m[n][i];
              join_m[(COMPUTE_WARPS + warp) * C::HEADS + h] = E4M3 ? mo[n][i] : m[n][i];
              join_m[(2 * COMPUTE_WARPS + warp) * C::HEADS + h] = l[n][i];
            }
        }
        if (busy) leave_output(join + warp * C::HEADS * (DH + PAD));
        __syncwarp();
        if (lane == 0) mbar_arrive(o_full(buf));
      }
      before = p;
      ++shared;
    }
    if (shared > 0) join_piece(before, shared - 1);

    // ---- sequences without positions, and lengths that the table cannot hold
    for (int s = b; s < g.a.n_seq; s += gridDim.x) {
      const int len = g.a.len[s];
      if (len <= 0) {
        for (int i = tid; i < g.a.heads * DH / 8; i += 32 * COMPUTE_WARPS)
          reinterpret_cast<uint4*>(g.a.out + (size_t)s * g.a.heads * DH)[i] = make_uint4(0, 0, 0, 0);
        if (g.a.lse) for (int i = tid; i < g.a.heads; i += 32 * COMPUTE_WARPS) g.a.lse[(size_t)s * g.a.heads + i] = -INFINITY;
      } else if (tid == 0 && g.a.status && len > (long long)g.a.max_pages << g.c.page_shift) {
        atomicMax(g.a.status, (int)ET_PAGED_CAPACITY);
      }
    }
    if (tid == 0) *reinterpret_cast<Join*>(g.a.workspace + b * 4) = mine;
  }
  __syncthreads();
  if (tid == 0 && *abort_flag && g.a.status) atomicMax(g.a.status, (int)DS_WAIT_EXPIRED);
}

// Joins the pieces of an item that was cut, one block per (first CTA of the item, head), in the order of the pieces.
constexpr int JOIN_THREADS = 128;
template <int DH, int NT>
__global__ void __launch_bounds__(JOIN_THREADS)
attention_join_kernel(const __grid_constant__ Args g) {
  begin_after_previous();
  constexpr int HEADS = 8 * NT, LANES = DH / 4, RUNS = JOIN_THREADS / LANES;
  const Join j = *reinterpret_cast<const Join*>(g.a.workspace + blockIdx.x * 4);
  const int h = blockIdx.y, kvh = j.part / g.parts, h0 = (j.part % g.parts) * HEADS;
  if (j.pieces == 0 || h0 + h >= g.group) return;
  const int next = 2 * blockIdx.x + 2;                               // slot of the second piece; the others follow two by two
  auto part = [&](int i) { return g.a.workspace + SLOT0 + (size_t)(i == 0 ? j.slot : next + 2 * (i - 1)) * Slot<DH, NT>::FLOATS; };
  constexpr int WARPS = JOIN_THREADS / 32, AHEAD = 8;
  __shared__ float weight[MAX_CTAS];
  __shared__ float tops[WARPS], sums[WARPS];
  __shared__ float4 accs[RUNS][LANES];
  const int tid = threadIdx.x, run = tid / LANES, d = (tid % LANES) * 4;
  // everything is on its way at once: the maxima and sums (a piece a thread), the outputs of the first pieces of each run
  float4 x[AHEAD];
#pragma unroll
  for (int k = 0; k < AHEAD; ++k)
    if (run + k * RUNS < j.pieces) x[k] = *reinterpret_cast<const float4*>(part(run + k * RUNS) + h * DH + d);
  static_assert(MAX_CTAS <= 2 * JOIN_THREADS, "two pieces a thread");
  float2 ml[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = tid + k * JOIN_THREADS;
    ml[k] = i < j.pieces ? *reinterpret_cast<const float2*>(part(i) + HEADS * DH + 2 * h) : make_float2(-INFINITY, 0.f);
  }
  float top = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
  if ((tid & 31) == 0) tops[tid >> 5] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WARPS; ++w) top = fmaxf(top, tops[w]);
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = tid + k * JOIN_THREADS;
    const float w = exp2_fast(ml[k].x - ref);
    if (i < j.pieces) weight[i] = w;
    sum += ml[k].y * w;
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
  if ((tid & 31) == 0) sums[tid >> 5] = sum;
  __syncthreads();
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) sum += sums[w];
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float4& v, float w) { acc.x += v.x * w; acc.y += v.y * w; acc.z += v.z * w; acc.w += v.w * w; };
#pragma unroll
  for (int k = 0; k < AHEAD; ++k) if (run + k * RUNS < j.pieces) add(x[k], weight[run + k * RUNS]);
#pragma unroll 4
  for (int i = run + AHEAD * RUNS; i < j.pieces; i += RUNS) add(*reinterpret_cast<const float4*>(part(i) + h * DH + d), weight[i]);
  accs[run][tid % LANES] = acc;
  __syncthreads();
  if (run == 0) {
    for (int r = 1; r < RUNS; ++r) add(accs[r][tid], 1.f);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const size_t at = (size_t)j.seq * g.a.heads + kvh * g.group + h0 + h;
    *reinterpret_cast<uint2*>(g.a.out + at * DH + d) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
    if (tid == 0 && g.a.lse) g.a.lse[at] = sum == 0.f ? -INFINITY : (log2f(sum) + top) * 0.6931471805599453f;
  }
}

bool make_cache_map(CUtensorMap* out, const PagedCache& c) {
  EncodeTiledFn fn = tensor_map_encoder();
  if (!fn) return false;
  const bool e4m3 = c.scale != nullptr;
  const int row = c.head_dim * (e4m3 ? 1 : 2), box_row = row > 128 ? 128 : row;
  const cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, ((cuuint64_t)c.n_pages * 2 * c.kv_heads) << c.page_shift};
  const cuuint64_t strides[1] = {(cuuint64_t)row};
  const cuuint32_t box[2] = {(cuuint32_t)(box_row / (e4m3 ? 1 : 2)), (cuuint32_t)(1 << (c.page_shift < 6 ? c.page_shift : 6))};
  const cuuint32_t estr[2] = {1, 1};
  return fn(out, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, c.data, dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, box_row == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DH, bool E4M3, int NT>
cudaError_t launch(const CUtensorMap& map, const Args& g, int ctas, cudaStream_t s) {
  using C = Cfg<DH, E4M3, NT>;
  static std::atomic<bool> ready[64];                                // per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64 || !ready[dev]) {
    if (NT == 2) {
      // setmaxnreg.inc waits for registers that only exist if the block was launched with LAUNCH_REGS of them a thread
      cudaFuncAttributes fa;
      e = cudaFuncGetAttributes(&fa, attention_paged_kernel<DH, E4M3, NT>);
      if (e != cudaSuccess) return e;
      if (fa.numRegs < LAUNCH_REGS) return cudaErrorLaunchOutOfResources;
    }
    e = cudaFuncSetAttribute(attention_paged_kernel<DH, E4M3, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
    if (e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64) ready[dev] = true;
  }
  ET_COUNT_LAUNCH();
  Launch l(ctas, THREADS, C::SMEM, s);
  e = cudaLaunchKernelEx(&l.cfg, attention_paged_kernel<DH, E4M3, NT>, map, g);
  if (e != cudaSuccess || g.whole) return e;
  ET_COUNT_LAUNCH();
  Launch join(dim3(ctas, g.group < C::HEADS ? g.group : C::HEADS), JOIN_THREADS, 0, s);
  return cudaLaunchKernelEx(&join.cfg, attention_join_kernel<DH, NT>, g);
}

}  // namespace

cudaError_t launch_attention_paged(const PagedCache& c, const PagedAttention& a, cudaStream_t s) {
  CUtensorMap map;
  if (!make_cache_map(&map, c)) return cudaErrorUnknown;
  Args g;
  g.c = c; g.a = a;
  g.group = a.heads / c.kv_heads;
  const int nt = g.group <= 8 ? 1 : 2;
  g.parts = (g.group + 8 * nt - 1) / (8 * nt);
  const long long tiles = (((long long)a.max_pages << c.page_shift) + TILE - 1) / TILE;      // of the longest sequence there can be
  // Where no sequence can have more than four tiles, items are not cut and nothing has to be joined.  The host knows the table's width
  // only: in one for 32 768 positions the same lengths take the other way, 1 x 61 6.7 us in place of 5.5, 16 x 200 8.7 of 6.5.
  g.whole = tiles <= 4;
  const long long most = (long long)a.n_seq * c.kv_heads * g.parts * (g.whole ? 1 : tiles + PAGED_ITEM_COST_MAX);
  if (most >= (1ll << 31) - MAX_CTAS) return cudaErrorInvalidValue;   // refused by the entry point already
  const int ctas = (int)(most < MAX_CTAS ? most : MAX_CTAS);
#define ET_PAGED(D, E) (nt == 1 ? launch<D, E, 1>(map, g, ctas, s) : launch<D, E, 2>(map, g, ctas, s))
  if (c.head_dim == 64) return c.scale ? ET_PAGED(64, true) : ET_PAGED(64, false);
  return c.scale ? ET_PAGED(128, true) : ET_PAGED(128, false);
#undef ET_PAGED
}

}  // namespace et
