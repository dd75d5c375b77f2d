// The batch of a step, from the sequences' lengths: offsets, block tables, positions and slots (esa_plan_paged).
//
// Three scans over the sequences (new rows, pages given back, pages taken), then work that is independent a row and a page: the page that
// entry e of a sequence's row gets is the (taken before it + e - held)-th of the queue "free pages of the ring, then pages given back", found from
// the offsets alone.  So no page's number passes through another one's, nothing is atomic, and the outcome does not depend on the order.
//
// What bounds it is latency: lengths, three scans of a few hundred cycles, a search in LDS, a table's or ring's entry.  So every workgroup makes the scans
// for itself (28 bytes a sequence in LDS) and no second launch has to wait for them: 200 sequences 4.8 us in a graph, of which 12000 pages move; two
// launches, the scans' results by way of memory, took 7.7, one workgroup 15.8.  One that goes on in place must not overwrite lengths that other workgroups
// have yet to read: they are left aside, and a launch of 2 us settles them.  More than 4096 sequences are one workgroup's and a second launch's: 4097 21 us,
// 16384 38, 65536 132.
#include "serve.h"

namespace esa {
namespace serve {
namespace {

// What rows and pages are filled from: [n_seq + 1] offsets (those of sequence b end at [b + 1]) and a sequence's numbers.  Sums that
// junk makes longer than 32 bits stop at INT32_MAX.
struct alignas(16) Of {
  int start, had, take, need;      // take: pages taken for the sequences before it
};
struct Queue {
  int first, count, given;         // the free pages, and what is given back and the ring has room for
};
struct Offsets {
  int32_t *row, *give, *take;
  Of* of;
};
__host__ __device__ inline size_t offsets_bytes(int n_seq) { return 16 + (size_t)n_seq * sizeof(Of) + 3 * ((size_t)n_seq + 1) * sizeof(int32_t); }
__host__ __device__ inline Offsets offsets_at(void* p, int n_seq) {
  Of* of = (Of*)((char*)p + 16);
  int32_t* ends = (int32_t*)(of + n_seq);
  const size_t n = (size_t)n_seq + 1;
  return Offsets{ends, ends + n, ends + 2 * n, of};
}

// Sums of numbers below 2^31 that stop at 2^32 - 1 (one instruction): what is beyond 2^31 is clamped to less in any case.
__device__ __forceinline__ uint32_t plus(uint32_t x, uint32_t y) { return __builtin_elementwise_add_sat(x, y); }
__device__ __forceinline__ int clamped(uint32_t x) { return (int)min(x, (uint32_t)INT32_MAX); }
__device__ __forceinline__ uint32_t wave_sums(uint32_t x) {      // of the lanes up to each
  x = plus(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false));      // row_shr 1, 2, 4, 8
  x = plus(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false));
  x = plus(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false));
  x = plus(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false));
  x = plus(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false));      // row_bcast 15, 31
  return plus(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false));
}
// Over N numbers a thread, of which its wave's j-th are behind its (j - 1)-th: what is in front of each, and all of the workgroup's.  part: [WAVES].  (Where
// a sum has stopped, what is left of it without a number below 2^31 is still 2^31 or more.)
template <int WAVES, int N> __device__ __forceinline__ uint32_t scan(const uint32_t (&x)[N], uint32_t (&before)[N], uint32_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = 0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const uint32_t upto = wave_sums(x[j]);
    before[j] = plus(sum, upto - x[j]);
    sum = plus(sum, paged::lane_value(upto, 63));
  }
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  const uint32_t sums = wave_sums(lane < WAVES ? part[lane] : 0);
  const uint32_t front = wave > 0 ? paged::lane_value(sums, wave - 1) : 0;
#pragma unroll
  for (int j = 0; j < N; ++j) before[j] = plus(front, before[j]);
  return paged::lane_value(sums, WAVES - 1);
}

// The sequences' lengths and offsets, by a workgroup of THREADS, EACH of them a thread at a time.  writes: whether it is the one that leaves the call's lengths.
// (A thread's sequences one behind the other, loads and LDS stores 16 bytes apart: 4000 of them 11.3 us for 9.3.)
template <int THREADS, int EACH> __device__ __forceinline__ Queue plan_offsets(const PlanArgs& a, const Offsets& o, bool writes) {
  constexpr int kWaves = THREADS / 64;
  __shared__ uint32_t part[3][kWaves];
  const int tid = threadIdx.x;
  const int at_in = a.ring_at_in[0], count_in = a.ring_at_in[1];
  uint32_t rows = 0, gives = 0, takes = 0;
  for (int r0 = 0; r0 < a.n_seq; r0 += THREADS * EACH) {
    const int b0 = r0 + (tid >> 6) * 64 * EACH + (tid & 63);      // the thread's sequences are 64 apart
    int start[EACH], had[EACH], grow[EACH], need[EACH];
    uint32_t fresh[EACH], before[EACH], x[EACH], y[EACH];
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int b = min(b0 + j * 64, a.n_seq - 1);
      start[j] = a.start_in[b];
      fresh[j] = max(a.fresh[b], 0);
      had[j] = a.held_in[b];
      grow[j] = a.grow ? a.grow[b] : 0;
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) fresh[j] = b0 + j * 64 < a.n_seq ? fresh[j] : 0;
    const uint32_t all = scan<kWaves, EACH>(fresh, before, part[0]);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const uint32_t at = plus(rows, before[j]);
      const int lo = (int)min(at, (uint32_t)a.n_tok), hi = (int)min(plus(at, fresh[j]), (uint32_t)a.n_tok);
      fresh[j] = hi;      // from here on the end of the sequence's rows
      had[j] = min(max(had[j], 0), a.max_pages);
      start[j] = (int)min(max((int64_t)start[j] + grow[j], (int64_t)0), (int64_t)(INT32_MAX - (hi - lo)));
      need[j] = (int)min(((uint32_t)start[j] + (uint32_t)(hi - lo) + (1u << a.page_log2) - 1) >> a.page_log2, (uint32_t)a.max_pages);
      const bool there = b0 + j * 64 < a.n_seq;
      x[j] = there ? max(had[j] - need[j], 0) : 0;
      y[j] = there ? max(need[j] - had[j], 0) : 0;
    }
    rows = plus(rows, all);
    uint32_t give[EACH], take[EACH];
    const uint32_t all_give = scan<kWaves, EACH>(x, give, part[1]), all_take = scan<kWaves, EACH>(y, take, part[2]);
#pragma unroll
    for (int j = 0; j < EACH; ++j) {
      const int b = b0 + j * 64;
      if (b >= a.n_seq) break;
      const uint32_t front = plus(takes, take[j]);
      o.of[b] = Of{start[j], had[j], clamped(front), need[j]};
      o.row[b + 1] = (int)fresh[j];
      o.give[b + 1] = clamped(plus(plus(gives, give[j]), x[j]));
      o.take[b + 1] = clamped(plus(front, y[j]));
      if (writes) {
        a.start[b] = start[j];
        a.cu[b + 1] = (int)fresh[j];
      }
    }
    gives = plus(gives, all_give);
    takes = plus(takes, all_take);
  }
  const int first = (int)((uint32_t)max(at_in, 0) % (uint32_t)a.n_pages), count = min(max(count_in, 0), a.n_pages);
  const int given = min(clamped(gives), a.n_pages - count), free = count + given, taken = min(clamped(takes), free);
  if (tid == 0) o.row[0] = o.give[0] = o.take[0] = 0;
  if (tid == 0 && writes) {
    a.cu[0] = 0;
    const uint32_t next = (uint32_t)first + taken;      // below 2 n_pages
    a.ring_at[0] = (int)(next >= (uint32_t)a.n_pages ? next - a.n_pages : next);
    a.ring_at[1] = free - taken;
    a.lack[0] = clamped(takes) - taken;
  }
  __syncthreads();
  for (int b = tid; writes && b < a.n_seq; b += THREADS) {
    const Of x = o.of[b];
    a.held[b] = x.need > x.had ? x.had + (int)min((uint32_t)x.take + (uint32_t)(x.need - x.had), (uint32_t)free) - min(x.take, free) : x.need;
  }
  return Queue{first, count, given};
}

// The sequence in which item i falls: the number of ends (end[1], end[2], ...) up to i.
__device__ __forceinline__ int sequence_of(const int32_t* end, int n_seq, int i) {
  int lo = 0, n = n_seq;
  while (n > 0) {
    const int half = n >> 1;
    const bool past = end[lo + half + 1] <= i;
    lo = past ? lo + half + 1 : lo;
    n = past ? n - half - 1 : half;
  }
  return lo;
}
// Place x < 3 n_pages round the ring.
__device__ __forceinline__ int64_t in_ring(const PlanArgs& a, int64_t x) {
  x -= x >= a.n_pages ? a.n_pages : 0;
  return x - (x >= a.n_pages ? a.n_pages : 0);
}
// The r-th page that is given back.
__device__ __forceinline__ int given_page(const PlanArgs& a, const Offsets& o, int r) {
  const int b = min(sequence_of(o.give, a.n_seq, r), a.n_seq - 1);
  return a.pages[(int64_t)b * a.pages_ld + min(o.of[b].need + (r - o.give[b]), a.max_pages - 1)];
}
// The t-th page of the queue, -1 behind its end.
__device__ __forceinline__ int taken_page(const PlanArgs& a, const Offsets& o, const Queue& q, int64_t t) {
  if (t < q.count) return a.ring[in_ring(a, q.first + t)];
  return t - q.count < q.given ? given_page(a, o, (int)(t - q.count)) : -1;
}

__device__ __forceinline__ void fill_row(const PlanArgs& a, const Offsets& o, const Queue& q, int i) {
  const int b = sequence_of(o.row, a.n_seq, i);
  int pos = -1, page = -1;
  if (b < a.n_seq) {
    const Of x = o.of[b];
    pos = x.start + (i - o.row[b]);
    const int e = pos >> a.page_log2;
    if (e < a.max_pages) page = e < x.had ? a.pages[(int64_t)b * a.pages_ld + e] : taken_page(a, o, q, (int64_t)x.take + (e - x.had));
  }
  a.pos[i] = pos;
  a.slot[i] = (uint32_t)page < (uint32_t)a.n_pages ? ((int64_t)page << a.page_log2) + (pos & ((1 << a.page_log2) - 1)) : -1;
}
// Pages that are given back, and those that are taken.
__device__ __forceinline__ void give_page(const PlanArgs& a, const Offsets& o, const Queue& q, int r) {
  a.ring[in_ring(a, (int64_t)q.first + q.count + r)] = given_page(a, o, r);
}
__device__ __forceinline__ void take_page(const PlanArgs& a, const Offsets& o, const Queue& q, int t) {
  const int b = min(sequence_of(o.take, a.n_seq, t), a.n_seq - 1);
  const Of x = o.of[b];
  a.pages[(int64_t)b * a.pages_ld + min(x.had + (t - x.take), a.max_pages - 1)] = taken_page(a, o, q, t);
}

// Item i of the rows, of the pages that are given back and of those that are taken.
__device__ __forceinline__ void fill(const PlanArgs& a, const Offsets& o, const Queue& q, int64_t i) {
  if (i < a.n_tok) return fill_row(a, o, q, (int)i);
  i -= a.n_tok;
  if (i < q.given) return give_page(a, o, q, (int)i);
  take_page(a, o, q, (int)(i - q.given));
}
__device__ __forceinline__ int64_t items_of(const PlanArgs& a, const Offsets& o, const Queue& q) { return (int64_t)a.n_tok + q.given + o.take[a.n_seq]; }

// One launch: every workgroup finds the offsets for itself and keeps them in LDS, the first one writes the lengths, which no other may be reading.
template <int THREADS, int EACH> __global__ __launch_bounds__(THREADS) void plan_whole(PlanArgs a) {
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const Offsets o = offsets_at(lds, a.n_seq);
  const Queue q = plan_offsets<THREADS, EACH>(a, o, blockIdx.x == 0);
  const int64_t n = items_of(a, o, q);
  for (int64_t i = blockIdx.x * THREADS + threadIdx.x; i < n; i += gridDim.x * THREADS) fill(a, o, q, i);
}

// The lengths that a launch has left aside go to their places: [n_seq] starts, [n_seq] numbers of pages, the ring's two.
__global__ __launch_bounds__(256) void plan_settle(PlanArgs a, const int32_t* aside) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= 2 * a.n_seq + 2) return;
  (i < a.n_seq ? a.start + i : i < 2 * a.n_seq ? a.held + (i - a.n_seq) : a.ring_at + (i - 2 * a.n_seq))[0] = aside[i];
}

// More sequences than LDS has room for: two launches, the offsets in the workspace.
constexpr int kThreads = 1024;
__global__ __launch_bounds__(kThreads) void plan_lengths(PlanArgs a) {
  const Queue q = plan_offsets<kThreads, 4>(a, offsets_at(a.ws, a.n_seq), true);
  if (threadIdx.x == 0) *(Queue*)a.ws = q;
}
__global__ __launch_bounds__(kThreads) void plan_fill(PlanArgs a) {
  const Offsets o = offsets_at(a.ws, a.n_seq);
  const Queue q = *(const Queue*)a.ws;
  const int64_t n = items_of(a, o, q);
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) fill(a, o, q, i);
}

constexpr int kLdsSeqs = 4096;          // sequences whose offsets a workgroup keeps in LDS

// A launch of `threads` for every row, but for 2^15 at least, as pages are many more than rows at times, and 2^18 at most; or of one workgroup.
template <int THREADS, int EACH> int launch_whole(const PlanArgs& a, bool alone, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.n_tok + THREADS - 1) / THREADS, fewest = (1 << 15) / THREADS, most = (1 << 18) / THREADS;
  plan_whole<THREADS, EACH><<<dim3((unsigned)(alone ? 1 : blocks < fewest ? fewest : blocks > most ? most : blocks)), THREADS, offsets_bytes(a.n_seq), st>>>(a);
  ESA_LAUNCH_CHECK("plan_whole");
  return ESA_OK;
}

}  // namespace

size_t plan_workspace(int n_seq, bool in_place) {
  return n_seq > kLdsSeqs ? align_up(offsets_bytes(n_seq), 256) : in_place ? align_up((2 * (size_t)n_seq + 2) * sizeof(int32_t), 256) : 0;
}

int launch_plan(const PlanArgs& a, hipStream_t st) {
  static OncePerDevice raised;
  if (a.n_seq > kLdsSeqs) {
    plan_lengths<<<dim3(1), kThreads, 0, st>>>(a);
    ESA_LAUNCH_CHECK("plan_lengths");
    plan_fill<<<dim3(256), kThreads, 0, st>>>(a);
    ESA_LAUNCH_CHECK("plan_fill");
    return ESA_OK;
  }
  // In place one workgroup does all where rows and entries of the table are few (how many pages move is not known on the host): sixteen sequences of
  // up to 1025 pages 3.3 us, as many workgroups take without being in place; of 1875 pages, with some sequences ended, 5.5 for 4.1 and a settling launch.
  const bool in_place = a.start == a.start_in || a.held == a.held_in || a.ring_at == a.ring_at_in;
  const bool alone = in_place && a.n_seq <= 256 && (int64_t)a.n_seq * a.max_pages <= 32768 && a.n_tok <= 2048;
  const bool aside = in_place && !alone;
  PlanArgs w = a;
  if (aside) {
    w.start = (int32_t*)a.ws;
    w.held = w.start + a.n_seq;
    w.ring_at = w.held + a.n_seq;
  }
  int rc = raise_lds_limit(raised, {(const void*)plan_whole<1024, 4>}, offsets_bytes(kLdsSeqs), "plan_whole");
  // About as many threads as there are sequences: with 1024 of them sixteen sequences took 4.0 us, 200 5.7, 32 prompts 5.2 for 4.4; with 256, each for
  // sixteen sequences in turn, 4000 took 15.1 us for 9.2; 600 by 1024, 512 or 256 threads 6.07, 5.87, 6.12; 1500 by two or four a thread 7.2 and 8.4.
  if (rc == ESA_OK) rc = a.n_seq <= 256 ? launch_whole<256, 1>(w, alone, st) : a.n_seq <= 1024 ? launch_whole<512, 2>(w, false, st) : a.n_seq <= 2048 ? launch_whole<1024, 2>(w, false, st) : launch_whole<1024, 4>(w, false, st);
  if (rc != ESA_OK || !aside) return rc;
  plan_settle<<<dim3((2 * a.n_seq + 2 + 255) / 256), 256, 0, st>>>(a, (const int32_t*)a.ws);
  ESA_LAUNCH_CHECK("plan_settle");
  return ESA_OK;
}

}  // namespace serve
}  // namespace esa
