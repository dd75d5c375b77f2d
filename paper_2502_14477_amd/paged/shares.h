// Which part of the attention a workgroup of the kernel for many rows does.  The lengths lie on the device, so every workgroup finds its part
// from them: a scan over the sequences, a lane to each.
//
// A sequence's rows (new tokens x query heads of a KV head, numbered token by token) are cut into blocks, its keys into tiles.  A block
// weighs about as much as its last row sees keys.  All blocks of a KV head, one behind the other, are shared out evenly among as many
// workgroups as the chip has places for (fewer where there is little to do), wherever that cuts a block: a workgroup goes through the end of
// one block, some whole ones, and the beginning of another.  What it has of a cut block it leaves as a partial result, at most two of them; a
// second kernel joins these.  Small blocks are not cut.  Where there are three workgroups to a block and more, or little to do, each block is
// shared out by itself among as many as its weight is worth, evenly: no workgroup has parts of two.  (512 tokens over 128, 2048 selected and
// 2048 local ones, 8 heads of eight blocks: 61.0 us, 66.4 with cuts wherever they fall; 1024 tokens from the beginning, two heads of 32 blocks
// that grow: 38.7 and 48.3.)
// (Slices of one length for all, so long that the units were about one round: with sequences of 18 to 66 thousand keys the last round was
// often a few units; chunks of prompts took 1.2 to 1.5 times what their tiles did.)
#pragma once
#include "paged.h"

namespace esa {
namespace paged {

// Rows of a block, keys of a tile, workgroups at a time; a share is worth its beginning and end from `least` keys on, and a block as much besides.
// Blocks are shared out by themselves where there are three workgroups to each, or one and no more than `little` keys to a workgroup (248 and
// 100 tokens from the beginning, two heads, capped: 40 us otherwise, now 30).  Blocks of up to `whole` keys are not cut; others, where they are not
// shared out by themselves, not within a quarter of a share (`near` keys at least, three times as many and half a share at most) of their begin
// and end.  (Five tiles for `whole`: with eight and no half a share, 64 tokens behind 300 to 2500, 8 heads, took 27 to 37 us, now 21 to 28; 512
// behind as many 39 to 54, now 31 to 52.)  The kernel serves sequences of more than `above` rows.
struct ShareShape {
  static constexpr int rows = 256, keys = 64, places = 256, least = 2 * keys, whole = 5 * keys, near = 6 * keys, little = 8 * keys;
  int above;
  int step, last;           // tokens from a block's first row to the next one's, about, and to its last row's
};

// A sequence's blocks: block r weighs first + r * step.
struct Weights {
  int blocks;
  int64_t first;
  int step;
  __device__ __forceinline__ int64_t upto(int r) const { return r * first + (int64_t)step * ((int64_t)r * (r - 1) / 2); }      // of r blocks
  __device__ __forceinline__ int64_t all() const { return upto(blocks); }
  __device__ __forceinline__ int64_t of(int r) const { return first + (int64_t)r * step; }
  // The block in which weight x < all() falls.
  __device__ __forceinline__ int block_at(int64_t x) const {
    int lo = 0, hi = blocks - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (upto(mid) <= x)
        lo = mid;
      else
        hi = mid - 1;
    }
    return lo;
  }
};
__device__ __forceinline__ Weights weights_of(const AttendArgs& a, const ShareShape& sh, const Seq& s) {
  const int rows = s.n * a.group;
  if (rows <= sh.above) return Weights{0, 0, 0};
  return Weights{(rows + sh.rows - 1) / sh.rows, max(keys_up_to(a, s, keys_of(a, s), min(sh.last, s.n - 1)), 1), sh.step};
}

// The call's blocks of a KV head, and their shares.
class Shares {
 public:
  __device__ __forceinline__ Shares(const AttendArgs& args, const ShareShape& shape) : a(args), sh(shape) {
    const int lane = threadIdx.x & 63;
    int64_t blocks;
    int my_blocks = 0;
    if (a.batch.n_seq == 1) {
      const Weights w = weights_of(a, sh, uniform(sequence(a.batch, 0)));
      total = w.all();
      blocks = w.blocks;
    } else {
      total = blocks = 0;
      for (int b0 = 0; b0 < a.batch.n_seq; b0 += 64) {
        const Weights w = b0 + lane < a.batch.n_seq ? weights(b0 + lane) : Weights{0, 0, 0};
        const int64_t weight = weight_of(w);
        if (b0 == 0) {
          mine = weight;
          my_blocks = w.blocks;
        }
        total += lane_long(wave_scan_long(weight), 63);
        blocks += lane_value(wave_scan((uint32_t)w.blocks), 63);
      }
    }
    total = uniform(total);
    const int64_t worth = (total + sh.least - 1) / sh.least + blocks;
    workers = uniform((int)min(max(worth, (int64_t)1), (int64_t)max(sh.places / a.cache.h_kv, 1)));
    if (total == 0) workers = 0;
    by_block = uniform((int)(3 * blocks <= workers || (blocks <= workers && total <= (int64_t)sh.little * workers)));
    if (by_block) {
      extra = uniform((int64_t)((double)total * __builtin_amdgcn_rcp((double)(2 * workers - (int)blocks))));
      total = uniform(total + blocks * extra);
      mine += my_blocks * extra;
    }
    share = (double)total * __builtin_amdgcn_rcp((double)max(workers, 1));      // (reciprocals: what is found here in front of all work counts)
    per_weight = (double)workers * __builtin_amdgcn_rcp((double)max(total, (int64_t)1));
    near = (int)fmin(fmin(fmax(share * 0.25, (double)sh.near), 3.0 * (double)sh.near), share * 0.5);
  }

  // The block in which weight x < total falls, from where the last one was found.
  struct Block {
    int b, r;               // sequence, block
    int64_t begin;          // weight in front of it
    Weights w;
  };
  __device__ __forceinline__ Block block_at(int64_t x) {
    int b = 0;
    int64_t base = 0;
    if (a.batch.n_seq > 1) {
      if (x < seen) go_to(0, 0);
      for (;;) {
        const int64_t upto = wave_scan_long(mine) + seen;
        const uint64_t past = __ballot(upto > x);
        if (past) {
          const int at = __ffsll((unsigned long long)past) - 1;
          b = b0 + at;
          base = lane_long(upto - mine, at);
          break;
        }
        if (b0 + 64 >= a.batch.n_seq) return Block{-1, 0, 0, Weights{0, 0, 0}};      // (not with x < total)
        go_to(b0 + 64, lane_long(upto, 63));
      }
    }
    b = uniform(b);
    Weights w = weights_of(a, sh, uniform(sequence(a.batch, b)));
    w = Weights{uniform(w.blocks), uniform(w.first) + extra, uniform(w.step)};
    const int r = uniform(w.block_at(x - base));
    return Block{b, r, uniform(base + w.upto(r)), w};
  }
  // Where share w begins.  (Doubles: the same ones wherever it is asked.)
  __device__ __forceinline__ int64_t begin_of(int w) {
    if (w <= 0) return 0;
    if (w >= workers) return total;
    const int64_t x = by_block ? middle_of(w) : min((int64_t)(share * (double)w), total);
    if (x <= 0 || x >= total) return x;
    const Block k = block_at(x);
    if (k.b < 0) return x;
    const int64_t all = k.w.of(k.r);
    if (by_block) {
      const int first = first_in(k.begin), n = first_in(k.begin + all) - first, i = w - first;
      if (i <= 0) return k.begin;
      return i >= n || all - extra <= sh.whole ? k.begin + all : k.begin + (int64_t)((double)all * (double)((float)i * __builtin_amdgcn_rcpf((float)n)));
    }
    // A cut in a small block, or near a block's begin or end, is made there instead: a further part of a block costs a workgroup as much as
    // some tiles.
    if (all <= sh.whole || x - k.begin <= near) return k.begin;
    return k.begin + all - x <= near ? k.begin + all : x;
  }
  // The tile of a block of `tiles` at which weight x of its `all` cuts it; each: tiles / all.
  static __device__ __forceinline__ int tile_at(int64_t x, int64_t all, int tiles, double each) {
    return x <= 0 ? 0 : x >= all ? tiles : min((int)((double)x * each), tiles);
  }

  const AttendArgs& a;
  const ShareShape& sh;
  int64_t total;
  int workers, near, by_block;
  double share, per_weight;

 private:
  __device__ __forceinline__ void go_to(int first, int64_t in_front) {
    if (first != b0) mine = first + (int)(threadIdx.x & 63) < a.batch.n_seq ? weight(first + (int)(threadIdx.x & 63)) : 0;
    b0 = first;
    seen = uniform(in_front);
  }
  __device__ __forceinline__ Weights weights(int b) const { return weights_of(a, sh, sequence(a.batch, b)); }
  static __device__ __forceinline__ int64_t weight_of(const Weights& w) { return min(w.all(), ((int64_t)1 << 46) - 1); }
  __device__ __forceinline__ int64_t weight(int b) const {
    Weights w = weights(b);
    w.first += extra;
    return weight_of(w);
  }
  // Where blocks are shared out one by one, each weighs half a share more, so that small ones have one for themselves as well.  A share belongs
  // to the block that has its middle.  The first share whose middle is not in front of x (or one beside it, by a rounding: the same one wherever
  // it is asked, and cuts stay in order).
  __device__ __forceinline__ int64_t middle_of(int w) const { return min((int64_t)(share * ((double)w + 0.5)), total - 1); }
  __device__ __forceinline__ int first_in(int64_t x) const {
    return min(max((int)ceil((double)x * per_weight - 0.5), 0), workers);
  }
  int b0 = 0;               // the sequences that the lanes hold, and what weighs in front of them
  int64_t mine = 0, seen = 0, extra = 0;
};

// A part of a block's work: keys of tiles [from, end) for its rows.
struct Part {
  Seq s;
  Keys keys;
  int b, row0, rows, n_vis, from, end;
  bool ends, alone;         // the block's last tile; all of its tiles
  int slot;                 // else: where the partial result goes
};
__device__ __forceinline__ Part part_of(const AttendArgs& a, const ShareShape& sh, const Shares::Block& k, int64_t from, int64_t upto) {
  Part p;
  p.b = k.b;
  p.s = uniform(sequence(a.batch, k.b));
  const Keys q = keys_of(a, p.s);
  p.keys = Keys{uniform(q.t0), uniform(q.i_end), uniform(q.n_sel), uniform(q.late), uniform(q.l_start), uniform(q.n)};
  p.row0 = k.r * sh.rows;
  p.rows = min(p.s.n * a.group - p.row0, sh.rows);
  p.n_vis = uniform(keys_until(a, p.s, p.keys, p.row0 + p.rows - 1));
  const int tiles = (p.n_vis + sh.keys - 1) / sh.keys;
  const int64_t all = k.w.of(k.r);
  const double each = (double)tiles * __builtin_amdgcn_rcp((double)all);
  p.from = uniform(Shares::tile_at(from, all, tiles, each));
  p.end = uniform(Shares::tile_at(upto, all, tiles, each));
  p.ends = p.end == tiles;
  p.alone = p.from == 0 && p.ends;
  return p;
}
// What a slot's partial result is of, for the kernel that joins them.  (Found from the lengths there too, that kernel took 5 us more.)
struct Record {
  int rows;                 // of the block; 0: the slot holds nothing
  int b, row0, tok0;        // sequence, the block's first row, the sequence's first token
  int begins, ends;         // the part has the block's first tile, its last one
  int pad[2];
};
// Every part of the workgroup's share: work(Part).  Parts of no tiles are another one's (or, of a block without keys, its whole).
template <typename F> __device__ __forceinline__ void for_parts(const AttendArgs& a, const ShareShape& sh, Record* records, F&& work) {
  if (threadIdx.x == 0) records[2 * blockIdx.x].rows = records[2 * blockIdx.x + 1].rows = 0;
  Shares shares(a, sh);
  const int w = uniform((int)blockIdx.x / a.cache.h_kv);
  if (w >= shares.workers) return;
  int64_t ends[2];          // of the share: its begin and its end
#pragma unroll 1            // (code that runs once: its instructions come from memory)
  for (int i = 0; i < 2; ++i) {
    const int64_t y = shares.begin_of(w + i);
    ends[0] = i == 0 ? uniform(y) : ends[0];
    ends[1] = uniform(y);
  }
  const int64_t begin = ends[0], end = ends[1];
#pragma unroll 1
  for (int64_t at = begin; at < end;) {
    const Shares::Block k = shares.block_at(at);
    if (k.b < 0) return;
    const int64_t all = k.w.of(k.r), from = at - k.begin, upto = min(all, end - k.begin);
    Part p = part_of(a, sh, k, from, upto);
    p.slot = 2 * blockIdx.x + (at == begin ? 0 : 1);
    if (p.from < p.end || (p.alone && from == 0)) {
      if (!p.alone && threadIdx.x == 0) records[p.slot] = Record{p.rows, p.b, p.row0, p.s.row0, p.from == 0, p.ends, {0, 0}};
      work(p);
    }
    at = k.begin + upto;
  }
}

// On the host: workgroups, their partial results, and whether there are any.
static inline int grid_of(int h_kv) { return (ShareShape::places / h_kv > 1 ? ShareShape::places / h_kv : 1) * h_kv; }

}  // namespace paged
}  // namespace esa
