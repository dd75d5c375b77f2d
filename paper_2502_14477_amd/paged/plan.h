// Which part of the attention a workgroup does.  The lengths lie on the device, so every workgroup finds its part from them: a scan over
// the sequences, a lane to each.
//
// A sequence's rows (new tokens x query heads of a KV head, numbered token by token) are cut into blocks, its keys into tiles, the tiles
// into slices of the same length for all sequences: long enough that the call has about as many (block, slice) units as the chip takes
// workgroups at a time, however the lengths are distributed.  A block whose keys are one slice writes its result; the others leave
// partial results that a second kernel merges.
#pragma once
#include "paged.h"

namespace esa {
namespace paged {

// Rows of a block, keys of a tile, workgroups at a time; a slice has least tiles or a multiple.
struct Shape {
  int rows, keys, target, least;
};
struct Cost {
  int blocks, tiles;
};
__device__ __forceinline__ Cost cost_of(const AttendArgs& a, const Shape& sh, int b) {
  const Seq s = sequence(a.batch, b);
  if (s.n == 0) return Cost{0, 0};
  return Cost{(s.n * a.group + sh.rows - 1) / sh.rows, (keys_of(a, s).n + sh.keys - 1) / sh.keys};
}
template <typename X> __device__ __forceinline__ X wave_total(X x) {
#pragma unroll
  for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d);
  return x;
}
struct Plan {
  Cost mine;      // of the lane's sequence among the first 64
  int slice;      // tiles of a slice
};
__device__ __forceinline__ Cost cost_in(const AttendArgs& a, const Shape& sh, const Cost& mine, int b0) {
  const int b = b0 + (int)(threadIdx.x & 63);
  return b0 == 0 ? mine : b < a.batch.n_seq ? cost_of(a, sh, b) : Cost{0, 0};
}
// Slices are as long as lets every workgroup have one unit if there are fewer blocks than that: sixteen sequences of 18 to 66 thousand
// tokens, cut by their mean, were 600 units for 512 places, and the second round took as long as the first.
__device__ __forceinline__ Plan plan_of(const AttendArgs& a, const Shape& sh) {
  const int lane = threadIdx.x & 63;
  Plan p;
  p.mine = lane < a.batch.n_seq ? cost_of(a, sh, lane) : Cost{0, 0};
  int64_t all = 0, blocks = 0;
  for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
    const Cost c = cost_in(a, sh, p.mine, b0);
    all += (int64_t)c.blocks * c.tiles;
    blocks += c.blocks;
  }
  all = wave_total(all) * a.cache.h_kv;
  blocks = wave_total(blocks) * a.cache.h_kv;
  const int64_t mean = max((all + sh.target - 1) / sh.target, (int64_t)1);
  p.slice = (int)((mean + sh.least - 1) / sh.least) * sh.least;
  if (blocks * 2 > sh.target) return p;
  for (int i = 0; i < 6; ++i) {
    int64_t units = 0;
    for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
      const Cost c = cost_in(a, sh, p.mine, b0);
      units += (int64_t)c.blocks * ((c.tiles + p.slice - 1) / p.slice);
    }
    units = wave_total(units) * a.cache.h_kv;
    if (units <= sh.target) break;
    // every sequence's last slice is half full in the mean: what is over target is spread over the others
    const int more = (int)((int64_t)p.slice * (units - sh.target) / (sh.target * 2));
    p.slice += (max(more, 1) + sh.least - 1) / sh.least * sh.least;
  }
  return p;
}
struct Part {
  int b, block, slice;      // b < 0: none
  int64_t slot;             // of the block's first slice among the partial results of a KV head (blocks next to each other), if it has several
  int blocks;
};
// The u-th unit.  A sequence's units are numbered slice by slice: neighbours read the same keys.
__device__ __forceinline__ Part part_of(const AttendArgs& a, const Shape& sh, const Plan& plan, int64_t u) {
  const int slice = plan.slice;
  int64_t slots = 0;
  for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
    const Cost c = cost_in(a, sh, plan.mine, b0);
    const int n = (c.tiles + slice - 1) / slice;
    const int64_t units = (int64_t)c.blocks * max(n, 1), parts = n > 1 ? units : 0, upto = wave_scan(units), parts_upto = wave_scan(parts);
    const uint64_t past = __ballot(upto > u);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      const int i = (int)(u - __shfl(upto - units, at)), blocks = __shfl(c.blocks, at);
      return Part{b0 + at, i % blocks, i / blocks, slots + __shfl(parts_upto - parts, at) + i % blocks, blocks};
    }
    u -= __shfl(upto, 63);
    slots += __shfl(parts_upto, 63);
  }
  return Part{-1, 0, 0, 0, 0};
}
// Partial results of a KV head in front of sequence b's.
__device__ __forceinline__ int64_t parts_before(const AttendArgs& a, const Shape& sh, const Plan& plan, int b) {
  int64_t parts = 0;
  for (int b0 = 0; b0 < b; b0 += 64) {
    const Cost c = cost_in(a, sh, plan.mine, b0);
    const int n = (c.tiles + plan.slice - 1) / plan.slice;
    if (n > 1 && b0 + (int)(threadIdx.x & 63) < b) parts += (int64_t)c.blocks * n;
  }
  return wave_total(parts);
}
// Keys that the rows up to `row` of a sequence see at most.
__device__ __forceinline__ int keys_until(const AttendArgs& a, const Seq& s, const Keys& k, int row) {
  const int width = a.batch.max_pages << a.batch.page_log2;
  return k.n - (min(s.t0 + s.n, width) - min(s.t0 + row / a.group + 1, width));
}
// Units of a KV head, and the partial results among them: a sequence of several slices has more than one slice's tiles, so at most
// twice as many slices as its tiles fill.
static inline int64_t most_units(const Shape& sh, int64_t n_tok, int n_seq, int group, int h_kv) {
  return sh.target / h_kv + 1 + n_tok * group / sh.rows + (n_seq < n_tok ? n_seq : n_tok);
}
static inline int64_t most_parts(const Shape& sh, int h_kv) { return 2 * ((int64_t)sh.target / h_kv + 1); }

}  // namespace paged
}  // namespace esa
