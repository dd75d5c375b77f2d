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

// Rows of a block, keys of a tile, workgroups at a time; a slice has a multiple of `least` tiles; a workgroup's beginning and end take
// as long as `overhead` tiles.  The kernel serves sequences of more than `above` rows, up to `upto`.
struct Shape {
  int rows, keys, target, least, overhead, above, upto;
};
struct Cost {
  int blocks, tiles;
};
__device__ __forceinline__ Cost cost_of(const AttendArgs& a, const Shape& sh, int b) {
  const Seq s = sequence(a.batch, b);
  const int rows = s.n * a.group;
  if (rows <= sh.above || rows > sh.upto) return Cost{0, 0};
  return Cost{(rows + sh.rows - 1) / sh.rows, (keys_of(a, s).n + sh.keys - 1) / sh.keys};
}
struct Plan {
  Cost mine;      // of the lane's sequence among the first 64
  int slice;      // tiles of a slice
};
__device__ __forceinline__ Cost cost_in(const AttendArgs& a, const Shape& sh, const Cost& mine, int b0) {
  const int b = b0 + (int)(threadIdx.x & 63);
  return b0 == 0 ? mine : b < a.batch.n_seq ? cost_of(a, sh, b) : Cost{0, 0};
}
// The length of a slice: what the call takes is estimated for slices of which every place of the chip gets one, two, three or four in the
// mean, and for longer ones of which no more than one round is needed.  (Sixteen sequences of 18 to 66 thousand tokens, cut by their mean,
// were 600 units for 512 places, and the second round took as long as the first: 497 us, 342 in one.)  Counts are fp32: exact where they
// decide, and every workgroup comes to the same ones.
__device__ __forceinline__ Plan plan_of(const AttendArgs& a, const Shape& sh) {
  const int lane = threadIdx.x & 63;
  Plan p;
  p.mine = lane < a.batch.n_seq ? cost_of(a, sh, lane) : Cost{0, 0};
  float all = 0.f;
  for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
    const Cost c = cost_in(a, sh, p.mine, b0);
    all += (float)c.blocks * (float)c.tiles;
  }
  all = wave_sum(all) * (float)a.cache.h_kv;
  const float places = (float)sh.target;
  const float mean = fmaxf(all / places, 1.f);
  auto rounded = [&](float x) { return (int)fminf(ceilf(x / (float)sh.least), 1e7f) * sh.least; };
  auto units_of = [&](int slice) {
    float units = 0.f;
    for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
      const Cost c = cost_in(a, sh, p.mine, b0);
      units += (float)c.blocks * (float)((c.tiles + slice - 1) / slice);
    }
    return wave_sum(units) * (float)a.cache.h_kv;
  };
  float best = INFINITY;
  p.slice = 0;
  auto consider = [&](int slice) {
    const float units = units_of(slice);
    const float took = units <= places ? (float)(slice + sh.overhead) : (all + units * (float)sh.overhead) / places + 0.5f * (float)slice;
    if (took < best) {
      best = took;
      p.slice = slice;
    }
    return units;
  };
  int slice = rounded(mean);
  for (int i = 0; i < 4; ++i) {
    const float units = consider(slice);
    if (units <= places) break;
    // every sequence's last slice is half full in the mean: what is over one round is spread over the others
    slice += rounded(fmaxf((float)slice * (units - places) / (2.f * places), 1.f));
  }
  if (mean > 4.f * (float)sh.overhead) {
    consider(rounded(mean * 0.5f));
    consider(rounded(mean * (1.f / 3.f)));
    consider(rounded(mean * 0.25f));
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
// The u-th row of a KV head among the sequences of several slices.
struct SplitRow {
  int b, row;               // b < 0: none
  int64_t slot;             // of the sequence's first partial result
};
__device__ __forceinline__ SplitRow split_row(const AttendArgs& a, const Shape& sh, const Plan& plan, int64_t u) {
  const int lane = threadIdx.x & 63;
  int64_t slots = 0;
  for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
    const Cost c = cost_in(a, sh, plan.mine, b0);
    const int n = (c.tiles + plan.slice - 1) / plan.slice;
    const int64_t rows = n > 1 ? (int64_t)sequence(a.batch, b0 + lane).n * a.group : 0, parts = n > 1 ? (int64_t)c.blocks * n : 0;
    const int64_t upto = wave_scan(rows), parts_upto = wave_scan(parts);
    const uint64_t past = __ballot(upto > u);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      return SplitRow{b0 + at, (int)(u - __shfl(upto - rows, at)), slots + __shfl(parts_upto - parts, at)};
    }
    u -= __shfl(upto, 63);
    slots += __shfl(parts_upto, 63);
  }
  return SplitRow{-1, 0, 0};
}
// Keys that the rows up to `row` of a sequence see at most.
__device__ __forceinline__ int keys_until(const AttendArgs& a, const Seq& s, const Keys& k, int row) {
  const int width = a.batch.max_pages << a.batch.page_log2;
  return k.n - (min(s.t0 + s.n, width) - min(s.t0 + row / a.group + 1, width));
}
// Units of a KV head at most (a slice is a quarter of the mean at least), and partial results among them: a sequence of several slices
// has more than one slice's tiles, so at most twice as many slices as its tiles fill.
static inline int64_t most_units(const Shape& sh, int64_t n_tok, int n_seq, int group, int h_kv) {
  return 4 * ((int64_t)sh.target / h_kv + 1) + n_tok * group / sh.rows + (n_seq < n_tok ? n_seq : n_tok);
}
static inline int64_t most_parts(const Shape& sh, int h_kv) { return 8 * ((int64_t)sh.target / h_kv + 1); }

}  // namespace paged
}  // namespace esa
