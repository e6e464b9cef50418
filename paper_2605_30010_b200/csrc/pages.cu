// Pages of the cache, handed out and taken back on the device, and the beams' tables that follow a selection.
//
// What a step changes is little (a page for one sequence in page_size, a row of a table for each beam), so these calls are bound by
// latency: by launches, and by loads that wait for one another.
//
//   * The free pages are those whose count is 0, the i-th one the one with i smaller ones: there is no list to keep, so counts can be
//     changed by whoever likes, in any order, with the same result.  What it costs is a look at all counts (4 bytes a page).
//   * The parts of et_pages_update that depend on everything (which pages are free, how many pages and rows the sequences before
//     take) are done by one cluster of eight CTAs, sixteen for large tables, whose barrier costs a fraction of a launch: each CTA owns
//     its share of the sequences and of the counts, totals go round through distributed shared memory.
//   * Work of uneven sequences is dealt to threads entry by entry: a prefix sum over the sequences, and a search in it.
//
// Device time in a chain of calls, B200: et_pages_update, a few more positions for 64 sequences, 12 400 pages 8.3 us (a cluster's
// launch, four rounds of loads that wait for one another, three barriers); 700 prompts of up to 240 pages in place of others, 116 000
// pages, with their 2.1 million slots 30.6 (searches, and entries all over the tables; 25 where tables are in L2, without slots 16).
// The figures at the rules below are of tables in L2.  et_pages_fork, 4 rows of tables of 123 entries 6.6 us, 256 rows of 52 9.9.
// et_kv_copy, 2 half-filled pages of 4 + 4 heads of 128 1.7 us, 98 of them, bf16, 980 positions 3.0: a launch each.
#include <atomic>

#include "decode.cuh"
#include "earlytom_pages.h"

namespace et {

namespace {

constexpr int THREADS = 1024, WARPS = THREADS / 32;
constexpr int CLUSTER = 8, LARGE = 16;             // CTAs; kernels of either are written for a cluster of C

__device__ __forceinline__ int cluster_rank() {
  int r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// *p = v in the shared memory of CTA `cta` of the cluster
__device__ __forceinline__ void store_in(int* p, int cta, int v) {
  const uint32_t own = (uint32_t)__cvta_generic_to_shared(p);
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(own), "r"(cta));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(v) : "memory");
}
__device__ __forceinline__ void report(int* status, int code) { if (status) atomicMax(status, code); }

// Two sums side by side.  What is asked for in total may be more than a number holds (it then says any row); the takes, of entries that
// the tables have, never are, and nothing of the one sum reaches the other.
struct Two { int takes; unsigned rows; };
__device__ __forceinline__ Two operator+(Two a, Two b) { return Two{a.takes + b.takes, a.rows + b.rows}; }
__device__ __forceinline__ Two operator-(Two a, Two b) { return Two{a.takes - b.takes, a.rows - b.rows}; }
__device__ __forceinline__ int shfl_up(int v, int o) { return __shfl_up_sync(0xffffffffu, v, o); }
__device__ __forceinline__ int shfl(int v, int from) { return __shfl_sync(0xffffffffu, v, from); }
__device__ __forceinline__ Two shfl_up(Two v, int o) { return Two{__shfl_up_sync(0xffffffffu, v.takes, o), __shfl_up_sync(0xffffffffu, v.rows, o)}; }
__device__ __forceinline__ Two shfl(Two v, int from) { return Two{__shfl_sync(0xffffffffu, v.takes, from), __shfl_sync(0xffffffffu, v.rows, from)}; }

// Exclusive sums over the block's threads; `total`: all of them.  T: int or Two.
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* sums, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  T inc = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const T u = shfl_up(inc, o); if (lane >= o) inc = inc + u; }
  __syncthreads();                                 // sums is free
  if (lane == 31) sums[warp] = inc;
  __syncthreads();
  T w = sums[lane];                                // WARPS is 32
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) { const T u = shfl_up(w, o); if (lane >= o) w = w + u; }
  total = shfl(w, 31);
  const T before = shfl(w, warp ? warp - 1 : 0);
  return warp ? inc - v + before : inc - v;
}

// The last i of [0, n) with prefix[i] <= x (prefix ascending, prefix[0] <= x)
__device__ __forceinline__ int search(const int* prefix, int n, int x) {
  int lo = 0;
  while (n > 1) {
    const int half = n >> 1;
    if (prefix[lo + half] <= x) { lo += half; n -= half; } else n = half;
  }
  return lo;
}

// ---- free pages -------------------------------------------------------------------------------------------------------------------
// Each warp writes the free pages of its segment to the workspace, at the segment's own place; the segments' counts go to all CTAs.
template <int C> constexpr int SEGMENTS = C * WARPS;
// pages of a segment, a multiple of 32
template <int C> __device__ __forceinline__ int segment_size(int n_pages) { return ((n_pages + SEGMENTS<C> - 1) / SEGMENTS<C> + 31) & ~31; }

template <int C>
__device__ __forceinline__ void collect_free(const int* refs, int n_pages, int rank, int* list, int* counts) {
  const int lane = threadIdx.x & 31, segment = rank * WARPS + (threadIdx.x >> 5), size = segment_size<C>(n_pages);
  const int begin = min((long long)segment * size, (long long)n_pages), end = min((long long)begin + size, (long long)n_pages);
  constexpr int AHEAD = 8;
  int found = 0;
  for (int p0 = begin; p0 < end; p0 += 32 * AHEAD) {
    int r[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) r[j] = p0 + 32 * j + lane < end ? __ldcg(refs + p0 + 32 * j + lane) : 1;
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const unsigned free = __ballot_sync(0xffffffffu, r[j] == 0);
      if (r[j] == 0) list[begin + found + __popc(free & ((1u << lane) - 1))] = p0 + 32 * j + lane;
      found += __popc(free);
    }
  }
  if (lane < C) store_in(counts + segment, lane, found);
}
// Behind the cluster's barrier: counts become an exclusive sum; returns how many free pages there are.
template <int C>
__device__ __forceinline__ int sum_segments(int* counts, int* sums) {
  int total;
  const int v = threadIdx.x < SEGMENTS<C> ? counts[threadIdx.x] : 0, before = block_scan(v, sums, total);
  if (threadIdx.x < SEGMENTS<C>) counts[threadIdx.x] = before;
  __syncthreads();
  return total;
}
template <int C>
__device__ __forceinline__ int free_page(const int* list, const int* counts, int n_pages, int i) {
  const int segment = search(counts, SEGMENTS<C>, i);
  return __ldcg(list + (size_t)segment * segment_size<C>(n_pages) + i - counts[segment]);
}

// ---- et_pages_update --------------------------------------------------------------------------------------------------------------
struct Update {
  int* refs;
  int* table;
  const int* len;
  const int* keep;        // may be NULL
  const int* add;         // may be NULL
  int* new_len;
  int* offsets;           // may be NULL
  int* slots;             // may be NULL
  int* list;              // workspace: [n_pages] free pages,
  int* ends;              // [n_seq] the row behind the last one,
  int* start;             // [n_seq] position of the first row, -1: none was got
  int n_pages, page_shift, n_seq, max_pages, rows;
  int* status;
};

struct Turn { int kept, add, stay, drop, take; bool fits; };
__device__ __forceinline__ int entries_of(long long n, int shift) { return (int)((n + (1 << shift) - 1) >> shift); }
__device__ __forceinline__ Turn turn_of(const Update& u, int s) {
  const int cap = u.max_pages << u.page_shift;     // <= 2^30
  const int len = u.len[s], held = min(max(len, 0), cap);
  Turn t;
  t.kept = u.keep ? min(u.keep[s], held) : len < 0 ? -1 : held;
  if (t.kept < 0) t.kept = -1;
  t.add = t.kept < 0 ? 0 : u.add ? max(u.add[s], 0) : 1;
  t.stay = entries_of(max(t.kept, 0), u.page_shift);
  t.drop = entries_of(held, u.page_shift) - t.stay;
  t.fits = (long long)t.kept + t.add <= cap;
  t.take = t.fits ? entries_of(max(t.kept, 0) + t.add, u.page_shift) - t.stay : 0;
  return t;
}

// The slot of a position on the page that its table entry names, -1 if it is none (-2: there is no such entry)
__device__ __forceinline__ int slot_of(const Update& u, int page, int pos) {
  if ((unsigned)page < (unsigned)u.n_pages) return (page << u.page_shift) + (pos & ((1 << u.page_shift) - 1));
  if (page != -2) report(u.status, ET_PAGED_BAD_PAGE);
  return -1;
}
// The entry of a position of sequence s, -2 if the table has none
__device__ __forceinline__ int entry_at(const Update& u, int s, long long pos) {
  const long long column = pos >> u.page_shift;
  return pos >= 0 && column < u.max_pages ? __ldcg(u.table + (size_t)s * u.max_pages + column) : -2;
}

constexpr int AHEAD = 4;                           // entries of a thread that are on their way at once
__device__ __forceinline__ void give_back(const Update& u, int* const (&entry)[AHEAD]) {
  int page[AHEAD], old[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) if (entry[j]) { page[j] = *entry[j]; *entry[j] = -1; }
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) {
    old[j] = 1;
    if (!entry[j]) continue;
    if ((unsigned)page[j] >= (unsigned)u.n_pages) report(u.status, ET_PAGED_BAD_PAGE);
    else old[j] = atomicSub(u.refs + page[j], 1);
  }
#pragma unroll
  for (int j = 0; j < AHEAD; ++j)
    if (old[j] <= 0) {
      atomicAdd(u.refs + page[j], 1);
      report(u.status, ET_PAGED_BAD_COUNT);
    }
}

// Entries of large tables are given back by all SMs: a block takes a sequence's, or a slice of them.  (700 tables of 240 entries: 41 us
// with the entries given back by the eight SMs below, whose scattered atomics bound them, 30 with this kernel before them; 64 of 501
// 18.1 and 18.1; smaller ones up to 0.4 us more with it, and another launch of the host's.)
constexpr int GIVE_THREADS = 128;
constexpr long long GIVE_ENTRIES = 1 << 14;        // tables of more
// And twice as many CTAs do the rest for tables of more than this: 700 of 240 entries 25 us in place of 30, 3 000 of 63 24 of 26, 1 000 of
// 125 18.8 of 19.6; 64 of 501 16.4 of 15.9, 500 of 47, one position each, 9.8 of 9.3.
constexpr long long LARGE_ENTRIES = 1 << 16;
__global__ void __launch_bounds__(GIVE_THREADS)
pages_give_back_kernel(const __grid_constant__ Update u) {
  begin_after_previous();
  const int s = blockIdx.x;
  const Turn t = turn_of(u, s);
  int* const first = u.table + (size_t)s * u.max_pages + t.stay;
  for (int i0 = blockIdx.y * AHEAD * GIVE_THREADS + threadIdx.x; i0 < t.drop; i0 += gridDim.y * AHEAD * GIVE_THREADS) {
    int* entry[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) entry[j] = i0 + j * GIVE_THREADS < t.drop ? first + i0 + j * GIVE_THREADS : nullptr;
    give_back(u, entry);
  }
}

template <int C>
__global__ void __launch_bounds__(THREADS, 1)
pages_update_kernel(const __grid_constant__ Update u, bool slots_here, bool given_back) {
  __shared__ int counts[SEGMENTS<C>], taken_s[C], rows_s[C], sums[WARPS], prefix[THREADS], stay_s[THREADS], got_s[THREADS], row_s[THREADS], kept_s[THREADS];
  __shared__ Two sums2[WARPS];
  const int tid = threadIdx.x, rank = cluster_rank();
  const int per = (u.n_seq + C - 1) / C, s0 = min(rank * per, u.n_seq), s1 = min(s0 + per, u.n_seq);
  begin_after_previous();
  // ---- entries are given back; what is asked for is added up
  Two asked{0, 0};
  Turn t{};
  for (int b = s0; b < s1; b += THREADS) {
    const int s = b + tid;
    t = Turn{};
    if (s < s1) t = turn_of(u, s);
    asked = asked + Two{t.take, (unsigned)t.add};
    int dropped;
    const int before = block_scan(given_back ? 0 : t.drop, sums, dropped);
    if (dropped == 0) continue;
    prefix[tid] = before; stay_s[tid] = t.stay;
    __syncthreads();
    for (int i0 = tid; i0 < dropped; i0 += AHEAD * THREADS) {
      int* entry[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int i = i0 + j * THREADS;
        if (i >= dropped) { entry[j] = nullptr; continue; }
        const int k = search(prefix, min(THREADS, s1 - b), i);
        entry[j] = u.table + (size_t)(b + k) * u.max_pages + stay_s[k] + i - prefix[k];
      }
      give_back(u, entry);
    }
    __syncthreads();
  }
  Two cta;
  block_scan(asked, sums2, cta);
  cluster_sync();                                  // all counts have come down (and all CTAs have begun)
  if (tid < C) { store_in(taken_s + rank, tid, cta.takes); store_in(rows_s + rank, tid, (int)cta.rows); }
  collect_free<C>(u.refs, u.n_pages, rank, u.list, counts);
  cluster_sync();                                  // nobody writes into another's memory behind this
  const int n_free = sum_segments<C>(counts, sums);
  Two so_far{0, 0}, all{0, 0};                     // by the sequences before, by all
  for (int c = 0; c < C; ++c) {
    const Two of{taken_s[c], (unsigned)rows_s[c]};
    if (c < rank) so_far = so_far + of;
    all = all + of;
  }
  const int rows_all = (int)all.rows;
  // ---- entries are taken
  for (int b = s0; b < s1; b += THREADS) {
    const int s = b + tid;
    if (s1 - s0 > THREADS) { t = Turn{}; if (s < s1) t = turn_of(u, s); }          // else it is known
    Two batch;
    const Two ahead = block_scan(Two{t.take, (unsigned)t.add}, sums2, batch);
    const int taken = so_far.takes, row = (int)so_far.rows, before = ahead.takes, rows_before = (int)ahead.rows, take_all = batch.takes,
              rows_batch = (int)batch.rows;
    const bool got = t.fits && (t.take == 0 || taken + before + t.take <= n_free);
    if (s < s1) {
      if (!got) report(u.status, t.fits ? (int)ET_PAGED_NO_PAGE : (int)ET_PAGED_CAPACITY);
      u.new_len[s] = t.kept < 0 ? -1 : t.kept + (got ? t.add : 0);
      if (u.offsets) u.offsets[s] = (int)(so_far.rows + ahead.rows);
      if (u.slots && !slots_here) { u.ends[s] = (int)(so_far.rows + ahead.rows + t.add); u.start[s] = got ? t.kept : -1; }
    }
    prefix[tid] = before; stay_s[tid] = t.stay; got_s[tid] = got; row_s[tid] = rows_before; kept_s[tid] = t.kept;
    __syncthreads();
    for (int i0 = tid; i0 < take_all; i0 += AHEAD * THREADS) {
      int page[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int i = i0 + j * THREADS;
        page[j] = -1;
        if (i < take_all && (unsigned)(taken + i) < (unsigned)n_free) page[j] = free_page<C>(u.list, counts, u.n_pages, taken + i);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int i = i0 + j * THREADS;
        if (i >= take_all) continue;
        const int k = search(prefix, min(THREADS, s1 - b), i);
        if (!got_s[k]) page[j] = -1;
        u.table[(size_t)(b + k) * u.max_pages + stay_s[k] + i - prefix[k]] = page[j];
        if (page[j] >= 0) u.refs[page[j]] = 1;
      }
    }
    if (slots_here && u.slots) {
      __syncthreads();                             // the entries are there
      // (sums beyond 2^31 may say any row: none outside is written)
      const int rows = min(rows_batch, u.rows);
      for (int i0 = tid; i0 < rows; i0 += AHEAD * THREADS) {
        int page[AHEAD];
        long long pos[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          const int i = i0 + j * THREADS;
          page[j] = -2;
          pos[j] = 0;
          if (i >= rows) continue;
          const int k = search(row_s, min(THREADS, s1 - b), i);
          pos[j] = (long long)kept_s[k] + i - row_s[k];
          if (got_s[k]) page[j] = entry_at(u, b + k, pos[j]);
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
          const int i = i0 + j * THREADS, at = row + i;
          if (i < rows && (unsigned)at < (unsigned)u.rows) u.slots[at] = slot_of(u, page[j], (int)pos[j]);
        }
      }
    }
    so_far = so_far + batch;
    __syncthreads();
  }
  if (rank == 0) {
    if (tid == 0) {
      if (u.offsets) u.offsets[u.n_seq] = rows_all;
      if (u.slots && rows_all > u.rows) report(u.status, ET_PAGED_CAPACITY);
    }
    if (slots_here && u.slots) for (int r = max(rows_all, 0) + tid; r < u.rows; r += THREADS) u.slots[r] = -1;
  }
}

// Slots of many rows: a block takes neighbouring rows, a thread eight next to one another.  With few rows for each CTA of the cluster
// their threads write them, which saves a launch and its wait (32 sequences of 6 911 rows 8.6 us in place of 13.8, 200 of 21 710 11.6
// of 16.0; one of 16 000 12.6 of 9.5, 64 of 47 102 18.3 of 15.8): the host knows neither how the rows are dealt nor their number,
// which is `rows` at most.
constexpr int SLOT_THREADS = 256, SLOT_ROWS = 8, SLOT_SEQS = 8192, SLOTS_HERE = 4 * THREADS;      // a CTA
__global__ void __launch_bounds__(SLOT_THREADS)
slots_kernel(const __grid_constant__ Update u, int rows_each) {
  extern __shared__ int ends_s[];                  // [n_seq], where they fit
  begin_after_previous();
  const int* ends = u.ends;
  if (u.n_seq <= SLOT_SEQS) {
    for (int s = threadIdx.x; s < u.n_seq; s += SLOT_THREADS) ends_s[s] = __ldcg(u.ends + s);
    __syncthreads();
    ends = ends_s;
  }
  const int total = ends[u.n_seq - 1];
  const bool aligned = (reinterpret_cast<uintptr_t>(u.slots) & 15) == 0;
  const int first = blockIdx.x * rows_each, last = min(first + rows_each, u.rows);
  for (int r0 = first + threadIdx.x * SLOT_ROWS; r0 < last; r0 += SLOT_THREADS * SLOT_ROWS) {
    int slot[SLOT_ROWS], s = -1, behind = r0, start = -1, from = 0;
    auto look = [&](int r) {
      // the first sequence whose rows end behind this one
      int n = u.n_seq - s - 1;
      ++s;
      while (n > 0) {
        const int half = n >> 1;
        if (ends[s + half] <= r) { s += half + 1; n -= half + 1; } else n = half;
      }
      s = min(s, u.n_seq - 1);                     // (sums beyond 2^31 are in no order)
      from = s > 0 ? ends[s - 1] : 0; behind = ends[s];
    };
    if (r0 < total) { look(r0); start = __ldcg(u.start + s); }
    if (start >= 0 && r0 + SLOT_ROWS <= min(min(behind, total), last)) {
      // one sequence's, and so of one page or of two
      const long long pos = (long long)start + r0 - from;
      const int pa = entry_at(u, s, pos), pz = entry_at(u, s, pos + SLOT_ROWS - 1);
      const int a = slot_of(u, pa, (int)pos), z = slot_of(u, pz, (int)(pos + SLOT_ROWS - 1));
      const int left = (1 << u.page_shift) - (int)(pos & ((1 << u.page_shift) - 1));       // of the first page
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) slot[j] = j < left ? (a < 0 ? -1 : a + j) : z < 0 ? -1 : z + 1 + j - SLOT_ROWS;
    } else {
      // several sequences' rows: all starts on their way at once, then all pages
      int seq[SLOT_ROWS], pos[SLOT_ROWS];
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) {
        const int r = r0 + j;
        const bool live = r < total && r < last;
        if (live && r >= behind) look(r);
        seq[j] = live ? s : -1;
        pos[j] = r - from;
      }
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) {
        const int start_j = seq[j] >= 0 ? __ldcg(u.start + seq[j]) : -1;
        pos[j] = start_j < 0 ? -1 : (int)min((long long)start_j + pos[j], (long long)u.max_pages << u.page_shift);      // (<= 2^30)
      }
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) slot[j] = entry_at(u, seq[j], pos[j]);
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) slot[j] = slot_of(u, slot[j], pos[j]);
    }
    if (aligned && r0 + SLOT_ROWS <= last) {
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; j += 4) *reinterpret_cast<int4*>(u.slots + r0 + j) = make_int4(slot[j], slot[j + 1], slot[j + 2], slot[j + 3]);
    } else {
#pragma unroll
      for (int j = 0; j < SLOT_ROWS; ++j) if (r0 + j < last) u.slots[r0 + j] = slot[j];
    }
  }
}

// ---- et_pages_fork ----------------------------------------------------------------------------------------------------------------
struct Fork {
  int* refs;
  const int* table;
  const int* len;
  const int* parent;
  int* new_table;
  int* new_len;
  int* copies;
  int* list;              // workspace: [n_pages] free pages,
  int4* info;             // [n_new] how many rows the row's parent has, negative for the first of them; length; last page, if half-filled
  int n_pages, page_shift, n_old, n_new, max_pages;
  int* status;
};

// An old row's entries to its children's rows, by `threads` threads, of slices of it the slice-th; the counts of its pages go up by one
// less than it has children.
__device__ __forceinline__ void follow(const Fork& f, int p, const unsigned short* children, int n, int first, int tid, int threads, int slice,
                                       int slices) {
  const int length = max(f.len[p], -1), used = min(entries_of(max(length, 0), f.page_shift), f.max_pages);
  if (slice == 0 && n > 0) {
    const int column = length >> f.page_shift;
    const bool half = length > 0 && (length & ((1 << f.page_shift) - 1)) != 0 && column < f.max_pages;
    const int page = half ? f.table[(size_t)p * f.max_pages + column] : -1;
    for (int i = tid; i < n; i += threads) f.info[children[i]] = make_int4(children[i] == first ? -n : n, length, page, 0);
  }
  for (int c0 = slice * threads + tid; c0 < used; c0 += AHEAD * slices * threads) {
    int page[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) if (c0 + j * slices * threads < used) page[j] = f.table[(size_t)p * f.max_pages + c0 + j * slices * threads];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int c = c0 + j * slices * threads;
      if (c >= used) continue;
      if ((unsigned)page[j] >= (unsigned)f.n_pages) report(f.status, ET_PAGED_BAD_PAGE);
      else if (n > 1) atomicAdd(f.refs + page[j], n - 1);
      else if (n == 0 && atomicSub(f.refs + page[j], 1) <= 0) {
        atomicAdd(f.refs + page[j], 1);
        report(f.status, ET_PAGED_BAD_COUNT);
      }
      for (int i = 0; i < n; ++i) f.new_table[(size_t)children[i] * f.max_pages + c] = page[j];
    }
  }
}

// A block takes an old row, or a slice of it, to its children.
constexpr int FORK_THREADS = 256;
__global__ void __launch_bounds__(FORK_THREADS)
fork_rows_kernel(const __grid_constant__ Fork f) {
  extern __shared__ unsigned short children[];
  __shared__ int n_children, first;
  const int p = blockIdx.x, tid = threadIdx.x;
  begin_after_previous();
  if (tid == 0) { n_children = 0; first = f.n_new; }
  __syncthreads();
  for (int b = tid; b < f.n_new; b += FORK_THREADS)
    if (f.parent[b] == p) { children[atomicAdd(&n_children, 1)] = (unsigned short)b; atomicMin(&first, b); }
  __syncthreads();
  follow(f, p, children, n_children, first, tid, FORK_THREADS, blockIdx.y, gridDim.y);
}

// The same in the cluster below, a warp each old row, where rows are few and a row is one round of a warp's loads: a launch less, 2.6 us of
// the host's time a call, for up to 2 us of the device's (4 rows of 123 entries 6.8 us in place of 6.2, 64 of 52 8.4 of 7.1, 256 9.9 of 7.9);
// longer rows are left to the other kernel (16 of 481: 14.9 us here, 7.9 there).
constexpr int FORK_FEW = 256, FORK_COLUMNS = 32 * AHEAD;
__device__ __forceinline__ void fork_row(const Fork& f, int p, unsigned short* children) {
  const int lane = threadIdx.x & 31;
  int n = 0, first = f.n_new;
  for (int b0 = 0; b0 < f.n_new; b0 += 32) {
    const unsigned who = __ballot_sync(0xffffffffu, b0 + lane < f.n_new && f.parent[b0 + lane] == p);
    if (who >> lane & 1) children[n + __popc(who & ((1u << lane) - 1))] = (unsigned short)(b0 + lane);
    if (n == 0 && who != 0) first = b0 + __ffs(who) - 1;
    n += __popc(who);
  }
  __syncwarp();
  follow(f, p, children, n, first, lane, 32, 0, 1);
  __syncwarp();
}

// Half-filled last pages: which rows need one of their own, and which it is.
constexpr int FORK_EACH = 2, FORK_ROWS = 16384;
static_assert(CLUSTER * THREADS * FORK_EACH >= FORK_ROWS, "rows of a thread");
template <bool ALL>
__global__ void __launch_bounds__(THREADS, 1)
fork_last_pages_kernel(const __grid_constant__ Fork f) {
  __shared__ int counts[SEGMENTS<CLUSTER>], totals[CLUSTER], sums[WARPS];
  __shared__ unsigned short children[ALL ? WARPS : 1][FORK_FEW];
  const int tid = threadIdx.x, rank = cluster_rank();
  const int per = (f.n_new + CLUSTER - 1) / CLUSTER, b0 = rank * per, b1 = min(b0 + per, f.n_new);
  if (!ALL) cluster_sync();                        // all CTAs have begun
  begin_after_previous();
  if (ALL) {
    const int warp = tid >> 5;
    for (int p = rank * WARPS + warp; p < f.n_old; p += SEGMENTS<CLUSTER>) fork_row(f, p, children[ALL ? warp : 0]);
    cluster_sync();
  }
  int old[FORK_EACH], length[FORK_EACH];
  bool own[FORK_EACH];
  int wanted = 0;
#pragma unroll
  for (int j = 0; j < FORK_EACH; ++j) {
    const int b = b0 + tid * FORK_EACH + j;
    own[j] = false; old[j] = -1; length[j] = -1;
    if (b >= b1) continue;
    const int p = f.parent[b];
    const int4 info = __ldcg(f.info + b);            // (of a row whose parent is none whatever was there)
    if (p >= f.n_old) report(f.status, ET_PAGED_BAD_ROW);
    if ((unsigned)p >= (unsigned)f.n_old) continue;
    length[j] = info.y;
    old[j] = info.z;
    if ((unsigned)old[j] >= (unsigned)f.n_pages) continue;
    // A page that is named and has no count may be handed to another row below: nothing is copied from it, and its count stays.
    const int count = __ldcg(f.refs + old[j]);
    if (count <= 0) { report(f.status, ET_PAGED_BAD_COUNT); continue; }
    own[j] = !(info.x < 0 && count == -info.x);
    wanted += own[j];
  }
  int all;
  int i = block_scan(wanted, sums, all);
  if (tid < CLUSTER) store_in(totals + rank, tid, all);
  collect_free<CLUSTER>(f.refs, f.n_pages, rank, f.list, counts);
  cluster_sync();                                  // counts change from here on, and nobody writes into another's memory
  const int n_free = sum_segments<CLUSTER>(counts, sums);
  for (int c = 0; c < rank; ++c) i += totals[c];
  int left[FORK_EACH];
#pragma unroll
  for (int j = 0; j < FORK_EACH; ++j) {
    const int b = b0 + tid * FORK_EACH + j;
    left[j] = 1;
    if (b >= b1) continue;
    int from = -1, to = -1, n = 0;
    if (own[j]) {
      const int column = length[j] >> f.page_shift;
      left[j] = atomicSub(f.refs + old[j], 1);
      if (i < n_free) {
        from = old[j]; to = free_page<CLUSTER>(f.list, counts, f.n_pages, i); n = length[j] & ((1 << f.page_shift) - 1);
        f.refs[to] = 1;
      } else {
        report(f.status, ET_PAGED_NO_PAGE);
      }
      f.new_table[(size_t)b * f.max_pages + column] = to;
      ++i;
    }
    f.new_len[b] = length[j];
    f.copies[3 * b] = from; f.copies[3 * b + 1] = to; f.copies[3 * b + 2] = n;
  }
#pragma unroll
  for (int j = 0; j < FORK_EACH; ++j)
    if (left[j] <= 0) {                              // fewer counts than rows
      atomicAdd(f.refs + old[j], 1);
      report(f.status, ET_PAGED_BAD_COUNT);
    }
}

// ---- et_kv_copy: a page's rows of one plane and head are contiguous; a block takes some of these runs ------------------------------
constexpr int COPY_THREADS = 256;
__global__ void __launch_bounds__(COPY_THREADS)
kv_copy_kernel(PagedCache c, const int* copies, int* status, int runs_each) {
  begin_after_previous();
  const int from = copies[3 * blockIdx.x], to = copies[3 * blockIdx.x + 1];
  const int rows = min(copies[3 * blockIdx.x + 2], 1 << c.page_shift);
  if (from < 0 || to < 0 || rows <= 0) return;
  if (from >= c.n_pages || to >= c.n_pages) { if (threadIdx.x == 0) report(status, ET_PAGED_BAD_PAGE); return; }
  if (from == to) return;
  const int runs = 2 * c.kv_heads, run0 = blockIdx.y * runs_each, run1 = min(run0 + runs_each, runs);
  const int row_bytes = kv_row_bytes(c.format, c.head_dim), scale_bytes = kv_scale_bytes(c.format, c.head_dim);
  const int vectors = rows * row_bytes / 16;       // of a run
  constexpr int AHEAD = 4;
  for (int run = run0; run < run1; ++run) {
    const size_t a = ((size_t)from * runs + run) << c.page_shift, b = ((size_t)to * runs + run) << c.page_shift;     // rows
    const uint4* const src = reinterpret_cast<const uint4*>(c.data + a * row_bytes);
    uint4* const dst = reinterpret_cast<uint4*>(c.data + b * row_bytes);
    for (int i0 = threadIdx.x; i0 < vectors; i0 += AHEAD * COPY_THREADS) {
      uint4 v[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) if (i0 + j * COPY_THREADS < vectors) v[j] = src[i0 + j * COPY_THREADS];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) if (i0 + j * COPY_THREADS < vectors) dst[i0 + j * COPY_THREADS] = v[j];
    }
    for (int i = threadIdx.x; i < rows * scale_bytes; i += COPY_THREADS) c.scale[b * scale_bytes + i] = c.scale[a * scale_bytes + i];
  }
}

// Whether this device takes clusters of LARGE CTAs, more than every device has to.
bool large_clusters() {
  static std::atomic<int> known[64];               // per device; 0: not yet, 1: no, 2: yes
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
  if (known[dev] == 0) {
    int clusters = 0;
    Launch l(LARGE, THREADS, 0, nullptr, LARGE);
    const bool yes = cudaFuncSetAttribute(pages_update_kernel<LARGE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                     cudaOccupancyMaxActiveClusters(&clusters, pages_update_kernel<LARGE>, &l.cfg) == cudaSuccess && clusters > 0;
    if (!yes) (void)cudaGetLastError();
    known[dev] = yes ? 2 : 1;
  }
  return known[dev] == 2;
}

int shift_of(int page_size) {
  for (int s = 4; s <= 7; ++s) if (page_size == 1 << s) return s;
  return -1;
}

}  // namespace

}  // namespace et

using namespace et;

extern "C" {

et_status et_pages_update(int* refs_dev, int n_pages, int page_size, int* block_table_dev, int n_seq, int max_pages, const int* len_dev,
                          const int* keep_dev, const int* add_dev, int* new_len_dev, int* row_offsets_dev, int* slots_dev, int rows,
                          void* workspace_dev, size_t workspace_bytes, int* status_dev, void* cuda_stream) {
  if (!refs_dev || !block_table_dev || !len_dev || !new_len_dev || !workspace_dev || !aligned16(workspace_dev)) return ET_ERR_INVALID_ARG;
  if (new_len_dev == keep_dev || new_len_dev == add_dev) return ET_ERR_INVALID_ARG;
  const int shift = shift_of(page_size);
  if (shift < 0 || n_pages < 1 || n_seq < 1 || max_pages < 1 || rows < 0 || (rows > 0 && !slots_dev)) return ET_ERR_SHAPE;
  if ((long long)n_pages << shift >= 1ll << 31 || (long long)max_pages << shift > 1ll << 30 || n_seq > 65536 ||
      (long long)n_seq * max_pages >= 1ll << 31 || rows > 1 << 30) return ET_ERR_CAPACITY;
  if (workspace_bytes < ET_PAGES_WORKSPACE(n_pages, n_seq)) return ET_ERR_CAPACITY;
  int* const ws = (int*)workspace_dev;
  const Update u{refs_dev, block_table_dev, len_dev, keep_dev, add_dev, new_len_dev, row_offsets_dev, rows > 0 ? slots_dev : nullptr, ws,
                 ws + n_pages, ws + n_pages + n_seq, n_pages, shift, n_seq, max_pages, rows, status_dev};
  const bool here = rows <= SLOTS_HERE * (n_seq < CLUSTER ? n_seq : CLUSTER), many = (long long)n_seq * max_pages > GIVE_ENTRIES;
  if (many) {
    const int slices = cdiv(max_pages, AHEAD * GIVE_THREADS), most = 148 * 8 / n_seq + 1;
    ET_COUNT_LAUNCH();
    Launch give(dim3(n_seq, slices < most ? slices : most), GIVE_THREADS, 0, (cudaStream_t)cuda_stream);
    const cudaError_t e = cudaLaunchKernelEx(&give.cfg, pages_give_back_kernel, u);
    if (e != cudaSuccess) return launched(e);
  }
  const int cluster = (long long)n_seq * max_pages > LARGE_ENTRIES && large_clusters() ? LARGE : CLUSTER;
  ET_COUNT_LAUNCH();
  Launch l(cluster, THREADS, 0, (cudaStream_t)cuda_stream, cluster);
  const cudaError_t e = cudaLaunchKernelEx(&l.cfg, cluster == LARGE ? pages_update_kernel<LARGE> : pages_update_kernel<CLUSTER>, u, here, many);
  if (here || e != cudaSuccess) return launched(e);
  ET_COUNT_LAUNCH();
  const int tile = SLOT_THREADS * SLOT_ROWS, each = cdiv(cdiv(rows, 148 * 8), tile) * tile;
  Launch slots(cdiv(rows, each), SLOT_THREADS, n_seq <= SLOT_SEQS ? sizeof(int) * (size_t)n_seq : 0, (cudaStream_t)cuda_stream);
  return launched(cudaLaunchKernelEx(&slots.cfg, slots_kernel, u, each));
}

et_status et_pages_fork(int* refs_dev, int n_pages, int page_size, const int* block_table_dev, int n_old, int max_pages,
                        const int* len_dev, const int* parent_dev, int n_new, int* new_table_dev, int* new_len_dev, int* copies_dev,
                        void* workspace_dev, size_t workspace_bytes, int* status_dev, void* cuda_stream) {
  if (!refs_dev || !block_table_dev || !len_dev || !parent_dev || !new_table_dev || !new_len_dev || !copies_dev || !workspace_dev ||
      !aligned16(workspace_dev)) return ET_ERR_INVALID_ARG;
  if (new_table_dev == block_table_dev || new_len_dev == len_dev || new_len_dev == parent_dev) return ET_ERR_INVALID_ARG;
  const int shift = shift_of(page_size);
  if (shift < 0 || n_pages < 1 || n_old < 1 || n_new < 1 || max_pages < 1) return ET_ERR_SHAPE;
  if ((long long)n_pages << shift >= 1ll << 31 || (long long)max_pages << shift > 1ll << 30 || n_old > FORK_ROWS || n_new > FORK_ROWS ||
      (long long)(n_old > n_new ? n_old : n_new) * max_pages >= 1ll << 31) return ET_ERR_CAPACITY;
  if (workspace_bytes < ET_FORK_WORKSPACE(n_pages, n_new)) return ET_ERR_CAPACITY;
  int* const ws = (int*)workspace_dev;
  const Fork f{refs_dev, block_table_dev, len_dev, parent_dev, new_table_dev, new_len_dev, copies_dev, ws + 4 * n_new, (int4*)ws, n_pages, shift,
               n_old, n_new, max_pages, status_dev};
  const bool few = n_old <= FORK_FEW && n_new <= FORK_FEW && max_pages <= FORK_COLUMNS;
  if (few) {
    ET_COUNT_LAUNCH();
    Launch all(CLUSTER, THREADS, 0, (cudaStream_t)cuda_stream, CLUSTER);
    return launched(cudaLaunchKernelEx(&all.cfg, fork_last_pages_kernel<true>, f));
  }
  const int slices = max_pages / (AHEAD * FORK_THREADS) + 1, most = 148 * 4 / n_old + 1;
  ET_COUNT_LAUNCH();
  Launch rows(dim3(n_old, slices < most ? slices : most), FORK_THREADS, 2 * (size_t)n_new, (cudaStream_t)cuda_stream);
  cudaError_t e = cudaLaunchKernelEx(&rows.cfg, fork_rows_kernel, f);
  if (e != cudaSuccess) return launched(e);
  ET_COUNT_LAUNCH();
  Launch last(CLUSTER, THREADS, 0, (cudaStream_t)cuda_stream, CLUSTER);
  return launched(cudaLaunchKernelEx(&last.cfg, fork_last_pages_kernel<false>, f));
}

et_status et_kv_copy(const et_kv_cache* cache, const int* copies_dev, int n, int* status_dev, void* cuda_stream) {
  PagedCache c;
  const et_status st = check_cache(cache, &c);
  if (st != ET_OK) return st;
  if (!copies_dev) return ET_ERR_INVALID_ARG;
  if (n < 1) return ET_ERR_SHAPE;
  if (n > 1 << 24 || c.kv_heads > 1 << 15) return ET_ERR_CAPACITY;
  const int runs = 2 * c.kv_heads, split = cdiv(148 * 8, n) < runs ? cdiv(148 * 8, n) : runs, each = cdiv(runs, split);
  ET_COUNT_LAUNCH();
  Launch l(dim3(n, cdiv(runs, each)), COPY_THREADS, 0, (cudaStream_t)cuda_stream);
  return launched(cudaLaunchKernelEx(&l.cfg, kv_copy_kernel, c, copies_dev, status_dev, each));
}

}  // extern "C"
