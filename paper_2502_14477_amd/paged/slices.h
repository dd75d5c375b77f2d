// Which part of the attention a workgroup of the kernel for few rows does.  The lengths lie on the device, so every workgroup finds its part from them: a scan over
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

// Rows of a block, keys of a tile, workgroups at a time; a slice has a multiple of `least` tiles.  The kernel serves sequences of up to `upto`
// rows.
struct SliceShape {
  static constexpr int rows = 32, keys = 32;
  int target, least, upto;
  bool uncut;      // no sequence can have more than `least` tiles
};
struct Cost {
  int blocks, tiles;
};
__device__ __forceinline__ Cost cost_of(const AttendArgs& a, const SliceShape& sh, int b) {
  const Seq s = sequence(a.batch, b);
  const int rows = s.n * a.group;
  if (rows > sh.upto) return Cost{0, 0};
  return Cost{(rows + sh.rows - 1) / sh.rows, (keys_of(a, s).n + sh.keys - 1) / sh.keys};
}
// The length of a slice: so long that no more than one round of units is needed.  (Sixteen sequences of 18 to 66 thousand tokens, cut by their
// mean, were 600 units for 512 places, and the second round took as long as the first: 497 us, 342 in one.  Shorter slices and several
// rounds were slower, as were shares of the same length that cut sequences anywhere, by what finding them takes in both kernels.)  Counts
// are fp32, rounded from 2^24 on, and both kernels have to come to the same slice: nothing is contracted, so that every operation is rounded as it
// stands wherever it is compiled.  total(of): the sum of of(cost) over all sequences.
template <typename F> __device__ __forceinline__ int slice_of(const SliceShape& sh, int h_kv, F&& total) {
#pragma clang fp contract(off)
  if (sh.uncut) return sh.least;
  const float all = total([](const Cost& c) {
#pragma clang fp contract(off)
    return (float)c.blocks * (float)c.tiles;
  }) * (float)h_kv;
  const float places = (float)sh.target, mean = fmaxf(all / places, 1.f);
  auto rounded = [&](float x) { return (int)fminf(ceilf(x / (float)sh.least), 1e7f) * sh.least; };
  auto units_of = [&](int slice) {
#pragma clang fp contract(off)
    return total([&](const Cost& c) {
#pragma clang fp contract(off)
      return (float)c.blocks * (float)((c.tiles + slice - 1) / slice);
    }) * (float)h_kv;
  };
  int slice = rounded(mean);
  float units = units_of(slice);
  for (int i = 0; i < 4 && units > places; ++i) {
    // every sequence's last slice is half full in the mean: what is over one round is spread over the others
    slice += rounded(fmaxf((float)slice * (units - places) / (2.f * places), 1.f));
    units = units_of(slice);
  }
  return slice;
}
// What a lane's sequence comes to: units, partial results (of several slices only), rows of which some are to be joined.
struct Counts {
  uint32_t units, parts, rows;
};
__device__ __forceinline__ Counts counts_of(const AttendArgs& a, const Cost& c, int slice, int b) {
  const int n = (c.tiles + slice - 1) / slice;
  Counts x;
  x.units = countable((int64_t)c.blocks * max(n, 1));
  x.parts = n > 1 ? x.units : 0;
  x.rows = n > 1 ? countable((int64_t)sequence(a.batch, b).n * a.group) : 0;
  return x;
}
// Up to 64 sequences: every workgroup finds the plan by itself, a lane to a sequence.  More: a workgroup has made it for all (1024 sequences of
// 512 keys, two heads: 154 us with it, 355 without; 256 sequences: 35, 38), with sums over 64 sequences each.
struct Upto {
  int64_t units, parts, rows;      // of 64 sequences and all in front of them
};
struct Plan {
  Cost mine;      // of the lane's sequence among up to 64; of the only one in every lane
  int slice;      // tiles of a slice
};
struct Made {
  int* slice;
  Upto* upto;     // [(n_seq + 63) / 64]
};
constexpr int kPlanBytes = 256;      // in front of upto
__device__ __forceinline__ Plan plan_of(const AttendArgs& a, const SliceShape& sh, const Made& made) {
  Plan p{Cost{0, 0}, 0};
  if (a.batch.n_seq > 64) {
    p.slice = uniform(*made.slice);
    return p;
  }
  const int lane = threadIdx.x & 63;
  const bool one = a.batch.n_seq == 1;
  if (lane < a.batch.n_seq || one) p.mine = cost_of(a, sh, one ? 0 : lane);
  p.slice = uniform(slice_of(sh, a.cache.h_kv, [&](auto&& of) { return one ? of(p.mine) : wave_sum(of(p.mine)); }));
  return p;
}
// The 64 sequences in which the u-th item falls, and what lies in front of them.
struct Group {
  int b0;         // -1: none
  Upto before;
};
template <typename F> __device__ __forceinline__ Group group_of(const AttendArgs& a, const Made& made, int64_t u, F&& items) {
  if (a.batch.n_seq <= 64) return Group{0, Upto{0, 0, 0}};
  const int groups = (a.batch.n_seq + 63) / 64;
  for (int c0 = 0; c0 < groups; c0 += 64) {
    const int c = c0 + (int)(threadIdx.x & 63);
    const uint64_t past = __ballot(c < groups && items(made.upto[min(c, groups - 1)]) > u);
    if (!past) continue;
    const int at = c0 + __ffsll((unsigned long long)past) - 1;
    return Group{at * 64, at > 0 ? made.upto[at - 1] : Upto{0, 0, 0}};
  }
  return Group{-1, Upto{0, 0, 0}};
}
__device__ __forceinline__ Cost cost_in(const AttendArgs& a, const SliceShape& sh, const Plan& plan, int b0) {
  const int b = b0 + (int)(threadIdx.x & 63);
  return a.batch.n_seq <= 64 ? plan.mine : b < a.batch.n_seq ? cost_of(a, sh, b) : Cost{0, 0};
}
struct Part {
  int b, block, slice;      // b < 0: none
  int64_t slot;             // of the block's first slice among the partial results of a KV head (blocks next to each other), if it has several
  int blocks;
};
__device__ __forceinline__ Part uniform(const Part& p) { return Part{uniform(p.b), uniform(p.block), uniform(p.slice), uniform(p.slot), uniform(p.blocks)}; }
// The u-th unit.  A sequence's units are numbered slice by slice: neighbours read the same keys.
__device__ __forceinline__ Part part_of(const AttendArgs& a, const SliceShape& sh, const Plan& plan, const Made& made, int64_t u) {
  if (a.batch.n_seq == 1) {
    const int blocks = uniform(plan.mine.blocks), n = max((uniform(plan.mine.tiles) + plan.slice - 1) / plan.slice, 1);
    if (u >= (int64_t)blocks * n) return Part{-1, 0, 0, 0, 0};
    return Part{0, (int)u % blocks, (int)u / blocks, (int)u % blocks, blocks};
  }
  const Group in = group_of(a, made, u, [](const Upto& x) { return x.units; });
  if (in.b0 < 0) return Part{-1, 0, 0, 0, 0};
  const int b = in.b0 + (int)(threadIdx.x & 63);
  const Cost c = cost_in(a, sh, plan, in.b0);
  const Counts x = b < a.batch.n_seq ? counts_of(a, c, plan.slice, b) : Counts{0, 0, 0};
  const uint32_t upto = wave_scan(x.units), parts_upto = wave_scan(x.parts);
  u -= in.before.units;
  const uint64_t past = __ballot(upto > u);
  if (!past) return Part{-1, 0, 0, 0, 0};
  const int at = __ffsll((unsigned long long)past) - 1;
  const int i = (int)(u - lane_value(upto - x.units, at)), blocks = (int)lane_value(c.blocks, at);
  return Part{in.b0 + at, i % blocks, i / blocks, in.before.parts + lane_value(parts_upto - x.parts, at) + i % blocks, blocks};
}
// The u-th row of the sequences of several slices.
struct Split {
  int b, i;                 // b < 0: none
  int64_t slot;             // of the sequence's first partial result
};
__device__ __forceinline__ Split uniform(const Split& s) { return Split{uniform(s.b), uniform(s.i), uniform(s.slot)}; }
__device__ __forceinline__ Split split_of(const AttendArgs& a, const SliceShape& sh, const Plan& plan, const Made& made, int64_t u) {
  if (a.batch.n_seq == 1) {
    const bool split = uniform(plan.mine.tiles) > plan.slice && u < (int64_t)sequence(a.batch, 0).n * a.group;
    return Split{split ? 0 : -1, (int)u, 0};
  }
  const Group in = group_of(a, made, u, [](const Upto& x) { return x.rows; });
  if (in.b0 < 0) return Split{-1, 0, 0};
  const int b = in.b0 + (int)(threadIdx.x & 63);
  const Counts x = b < a.batch.n_seq ? counts_of(a, cost_in(a, sh, plan, in.b0), plan.slice, b) : Counts{0, 0, 0};
  const uint32_t upto = wave_scan(x.rows), parts_upto = wave_scan(x.parts);
  u -= in.before.rows;
  const uint64_t past = __ballot(upto > u);
  if (!past) return Split{-1, 0, 0};
  const int at = __ffsll((unsigned long long)past) - 1;
  return Split{in.b0 + at, (int)(u - lane_value(upto - x.rows, at)), in.before.parts + lane_value(parts_upto - x.parts, at)};
}
// Blocks, units and partial results of a KV head at most.  A slice is the mean at least; a sequence of several slices has more than one
// slice's tiles, so at most twice as many slices as its tiles fill.
static inline int64_t most_blocks(const SliceShape& sh, int64_t n_tok, int n_seq, int group) {
  const int64_t by_rows = n_tok * group / sh.rows + (n_seq < n_tok ? n_seq : n_tok), by_limit = (int64_t)n_seq * ((sh.upto - 1) / sh.rows + 1);
  return by_rows < by_limit ? by_rows : by_limit;
}
static inline int64_t most_units(const SliceShape& sh, int64_t n_tok, int n_seq, int group, int h_kv) {
  return (int64_t)sh.target / h_kv + 1 + most_blocks(sh, n_tok, n_seq, group);
}
static inline int64_t most_parts(const SliceShape& sh, int h_kv) { return 2 * ((int64_t)sh.target / h_kv + 1); }

}  // namespace paged
}  // namespace esa
