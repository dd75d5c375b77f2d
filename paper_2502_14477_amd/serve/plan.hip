// The batch of a step, from the sequences' lengths: offsets, block tables, positions and slots (esa_plan_paged).
//
// Three scans over the sequences (new rows, pages given back, pages taken), then work that is independent a row and a page: the page that
// entry e of a sequence's row gets is the (taken before it + e - held)-th of the queue "free pages of the ring, then pages given back", found from
// the offsets alone.  So no page's number passes through another one's, nothing is atomic, and the outcome does not depend on the order.
#include "serve.h"

namespace esa {
namespace serve {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kWaves = kScanThreads / 64;

// What the rows and pages are filled from.  [n_seq + 1] offsets and [n_seq] numbers a sequence; sums that junk makes longer than 32
// bits stop at INT32_MAX.
struct Offsets {
  int32_t *row, *give, *take, *need, *had;
  int32_t* head;      // first free page's place, free pages, pages given back that the ring has room for
};
__host__ __device__ inline Offsets offsets_at(void* ws, int n_seq) {
  const size_t n = (size_t)n_seq + 1;
  int32_t* p = (int32_t*)ws;
  return Offsets{p + 4, p + 4 + n, p + 4 + 2 * n, p + 4 + 3 * n, p + 4 + 4 * n, p};
}

// Sums over the workgroup up to each thread, and of all.  part: [kWaves].
struct Scanned {
  int64_t before, all;
};
__device__ __forceinline__ Scanned scan(int64_t x, int64_t* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t upto = wave_scan_long(x);
  __syncthreads();
  if (lane == 63) part[wave] = upto;
  __syncthreads();
  int64_t before = upto - x, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int64_t v = part[w];
    before += w < wave ? v : 0;
    all += v;
  }
  return Scanned{before, all};
}
__device__ __forceinline__ int saturated(int64_t x) { return (int)min(x, (int64_t)INT32_MAX); }

// The sequences' lengths and offsets.  One workgroup.
__device__ void plan_offsets(const PlanArgs& a, const Offsets& o) {
  __shared__ int64_t part[kWaves];
  const int tid = threadIdx.x;
  const int first = (int)((uint32_t)max(a.ring_at_in[0], 0) % (uint32_t)a.n_pages), count = min(max(a.ring_at_in[1], 0), a.n_pages);
  int64_t rows = 0, gives = 0, takes = 0;
  for (int b0 = 0; b0 < a.n_seq; b0 += kScanThreads) {
    const int b = b0 + tid;
    const bool there = b < a.n_seq;
    const int at = there ? b : 0;
    int64_t start = (int64_t)a.start_in[at] + (a.grow ? a.grow[at] : 0);
    const int64_t fresh = there ? max(a.fresh[at], 0) : 0;
    const int had = min(max(a.held_in[at], 0), a.max_pages);
    const Scanned r = scan(fresh, part);
    const int lo = (int)min(rows + r.before, (int64_t)a.n_tok), hi = (int)min(rows + r.before + fresh, (int64_t)a.n_tok);
    rows += r.all;
    start = min(max(start, (int64_t)0), (int64_t)(INT32_MAX - (hi - lo)));
    const int need = (int)min((start + (hi - lo) + (1 << a.page_log2) - 1) >> a.page_log2, (int64_t)a.max_pages);
    const int64_t give = there ? max(had - need, 0) : 0, take = there ? max(need - had, 0) : 0;
    const Scanned g = scan(give, part), t = scan(take, part);
    if (there) {
      a.start[b] = (int)start;
      a.cu[b + 1] = hi;
      o.row[b + 1] = hi;
      o.give[b + 1] = saturated(gives + g.before + give);
      o.take[b + 1] = saturated(takes + t.before + take);
      o.need[b] = need;
      o.had[b] = had;
    }
    gives += g.all;
    takes += t.all;
  }
  const int given = (int)min(gives, (int64_t)(a.n_pages - count)), free = count + given, taken = (int)min(takes, (int64_t)free);
  __syncthreads();
  if (tid == 0) {
    a.cu[0] = o.row[0] = o.give[0] = o.take[0] = 0;
    o.head[0] = first;
    o.head[1] = count;
    o.head[2] = given;
    a.ring_at[0] = (int)(((int64_t)first + taken) % a.n_pages);
    a.ring_at[1] = free - taken;
    a.lack[0] = saturated(takes - taken);
  }
  __syncthreads();
  for (int b = tid; b < a.n_seq; b += kScanThreads) {
    const int need = o.need[b], had = o.had[b];
    a.held[b] = need > had ? had + min(o.take[b + 1], free) - min(o.take[b], free) : need;
  }
}

// The sequence in which item i falls, of those that end at end[1], end[2], ...: the number of ends up to i.
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

struct Queue {
  int first, count, given;
};
// The r-th page that is given back.
__device__ __forceinline__ int given_page(const PlanArgs& a, const Offsets& o, int r) {
  const int b = min(sequence_of(o.give, a.n_seq, r), a.n_seq - 1);
  return a.pages[(int64_t)b * a.pages_ld + min(o.need[b] + (r - o.give[b]), a.max_pages - 1)];
}
// The t-th page of the queue, -1 behind its end.
__device__ __forceinline__ int taken_page(const PlanArgs& a, const Offsets& o, const Queue& q, int64_t t) {
  if (t < q.count) return a.ring[(q.first + t) % a.n_pages];
  return t - q.count < q.given ? given_page(a, o, (int)(t - q.count)) : -1;
}

__device__ __forceinline__ void fill_row(const PlanArgs& a, const Offsets& o, const Queue& q, int i) {
  const int b = sequence_of(o.row, a.n_seq, i);
  int pos = -1, page = -1;
  if (b < a.n_seq) {
    pos = a.start[b] + (i - o.row[b]);
    const int e = pos >> a.page_log2, had = o.had[b];
    if (e < a.max_pages) page = e < had ? a.pages[(int64_t)b * a.pages_ld + e] : taken_page(a, o, q, (int64_t)o.take[b] + (e - had));
  }
  a.pos[i] = pos;
  a.slot[i] = (uint32_t)page < (uint32_t)a.n_pages ? ((int64_t)page << a.page_log2) + (pos & ((1 << a.page_log2) - 1)) : -1;
}
// Item m of the pages that are given back and then those that are taken.
__device__ __forceinline__ void move_page(const PlanArgs& a, const Offsets& o, const Queue& q, int64_t m) {
  if (m < q.given) {
    a.ring[(q.first + q.count + m) % a.n_pages] = given_page(a, o, (int)m);
    return;
  }
  const int t = (int)(m - q.given), b = min(sequence_of(o.take, a.n_seq, t), a.n_seq - 1);
  a.pages[(int64_t)b * a.pages_ld + min(o.had[b] + (t - o.take[b]), a.max_pages - 1)] = taken_page(a, o, q, t);
}

__global__ __launch_bounds__(kScanThreads) void plan_lengths(PlanArgs a) { plan_offsets(a, offsets_at(a.ws, a.n_seq)); }

__global__ __launch_bounds__(256) void plan_fill(PlanArgs a) {
  const Offsets o = offsets_at(a.ws, a.n_seq);
  const Queue q = {o.head[0], o.head[1], o.head[2]};
  const int64_t step = (int64_t)gridDim.x * 256, tid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = tid; i < a.n_tok; i += step) fill_row(a, o, q, (int)i);
  const int64_t moves = (int64_t)q.given + o.take[a.n_seq];
  for (int64_t m = tid; m < moves; m += step) move_page(a, o, q, m);
}

}  // namespace

size_t plan_workspace(int n_seq) { return align_up((4 + 5 * ((size_t)n_seq + 1)) * sizeof(int32_t), 256); }

int launch_plan(const PlanArgs& a, hipStream_t st) {
  plan_lengths<<<dim3(1), kScanThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("plan_lengths");
  const int64_t blocks = ((int64_t)a.n_tok + 255) / 256;
  plan_fill<<<dim3((unsigned)(blocks < 64 ? 64 : blocks > 1024 ? 1024 : blocks)), 256, 0, st>>>(a);
  ESA_LAUNCH_CHECK("plan_fill");
  return ESA_OK;
}

}  // namespace serve
}  // namespace esa
