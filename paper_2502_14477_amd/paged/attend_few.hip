// Attention of few rows over a paged cache (decode, drafts; fp32 of any length): 32 rows (new tokens x query heads of a KV head) and a
// slice of the keys to a workgroup, rows of up to 512 bytes.
//
// What counts is that many requests are in flight: a decode step reads every key and value once.  A wave takes tiles of 32 keys by
// itself, with staging space of its own and no barrier in the loop: a tile's rows arrive in registers, 16 bytes a lane and whole rows
// to neighbouring lanes, are brought to the arithmetic's type (8-bit pages: times the block's scale, a power of two, so exactly) on
// their way into LDS, and the next tile is requested before the products.  So from LDS on there is one kernel for all cache types.
//   S^T = K Q^T, O^T += V^T P^T: a lane stands for a row, softmax stays in the lane and its opposite in the other half of the wave, and
// the layout of S^T's accumulator is the second product's operand layout when key 16 s + 8 (j / 4) + 4 half + j % 4 is operand j of step s.
// bf16: v_mfma_f32_32x32x16_bf16.  A probability enters as two bf16 terms (16 bits), so that outputs are as near the exact ones as rounding them
// to bf16 leaves them: 1.66e-3 rms, 2.5e-3 of them are not the nearest number.  One term: 2.3e-3 and 0.42, which over 8-bit rows takes 272 us
// for 290 with two (sixteen sequences of 18 to 66 thousand keys) and 104 for 112 (one of 262144); behind bf16 rows two cost nothing.
// fp32: v_mfma_f32_32x32x2_f32.
//   HBM bounds, over 8-bit rows beside a wave's instructions: a token over 262144 8-bit keys of 8 heads of 128 elements 105 us, 537 MB at 5.4 TB/s but for
// the join's 5.5 us; sixteen over 18 to 66 thousand 292 us, 1500 MB.  Eight over 8 thousand take 26 us and 5.2 (95 MB): some 8 us of it start and end.
#include <algorithm>

#include "attend_common.h"
#include "slices.h"

namespace esa {
namespace paged {
namespace {

constexpr int kRows = SliceShape::rows, kKeys = SliceShape::keys, kWaves = 4;
struct FewArgs : SplitArgs<SliceShape> {
  Made made;
  int first;                // the launch's first unit
};
// The plan of a call of more than 64 sequences, by one workgroup.
__global__ __launch_bounds__(1024) void plan_few(FewArgs f) {
  __shared__ float sums[16];
  const AttendArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n_seq = a.batch.n_seq, groups = (n_seq + 63) / 64;
  const int slice = slice_of(f.shape, a.cache.h_kv, [&](auto&& of) {
    float sum = 0.f;
    for (int b = tid; b < n_seq; b += 1024) sum += of(cost_of(a, f.shape, b));
    sum = wave_sum(sum);
    __syncthreads();
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = 0.f;
    for (int w = 0; w < 16; ++w) sum += sums[w];
    return sum;
  });
  if (tid == 0) *f.made.slice = slice;
  for (int c = wave; c < groups; c += 16) {
    const int b = c * 64 + lane;
    const Counts x = b < n_seq ? counts_of(a, cost_of(a, f.shape, b), slice, b) : Counts{0, 0, 0};
    const uint32_t units = wave_scan(x.units), parts = wave_scan(x.parts), rows = wave_scan(x.rows);
    if (lane == 63) f.made.upto[c] = Upto{units, parts, rows};
  }
  __threadfence_block();
  __syncthreads();
  if (wave != 0) return;
  Upto before{0, 0, 0};
  for (int c0 = 0; c0 < groups; c0 += 64) {
    const Upto x = c0 + lane < groups ? f.made.upto[c0 + lane] : Upto{0, 0, 0};
    const Upto upto{before.units + wave_scan_long(x.units), before.parts + wave_scan_long(x.parts), before.rows + wave_scan_long(x.rows)};
    if (c0 + lane < groups) f.made.upto[c0 + lane] = upto;
    before = Upto{lane_long(upto.units, 63), lane_long(upto.parts, 63), lane_long(upto.rows, 63)};
  }
}
template <typename T, bool F8, int D, bool CAP>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(D * sizeof(T) > 256 ? 1 : F8 && D * sizeof(T) < 256 ? 3 : 2))) void attend_few(FewArgs f) {
  constexpr bool kBf16 = sizeof(T) == 2;
  constexpr bool kLags = kBf16 && F8;                           // the softmax's reference
  constexpr int kRowBytes = D * (int)sizeof(T);                 // of a staged row
  constexpr int kHeldBytes = F8 ? D : kRowBytes;                // of a row in the pool
  constexpr int kPieces = kHeldBytes / 16;                      // lanes that fetch a row
  constexpr int kLoadRows = 64 / kPieces, kLoads = kKeys / kLoadRows;
  constexpr int kKS = kRowBytes / 32;                           // 16-byte fragments of a half-wave's part of a row
  constexpr int kMD = D / 32;
  constexpr int kTileBytes = kKeys * kRowBytes;
  __shared__ __attribute__((aligned(16))) unsigned char stage[kWaves][2][kTileBytes];
  __shared__ float ml[kWaves][kRows][2];
  const AttendArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = f.first + (int)blockIdx.x, g = unit % a.cache.h_kv;
  const Plan plan = plan_of(a, f.shape, f.made);
  const int slice = plan.slice;
  const Part at = uniform(part_of(a, f.shape, plan, f.made, unit / a.cache.h_kv));
  if (at.b < 0) return;
  const Seq s = uniform(sequence(a.batch, at.b));
  const Keys keys = keys_of(a, s);
  const int n_rows = s.n * a.group, row0 = at.block * kRows, rows = min(n_rows - row0, kRows);
  const int n_vis = uniform(keys_until(a, s, keys, row0 + rows - 1)), tiles = (n_vis + kKeys - 1) / kKeys;
  const int first = at.slice * slice, end = min(first + slice, tiles);
  if (at.slice > 0 && first >= end) return;
  const bool alone = tiles <= slice;

  // a lane's row: both halves of the wave have it; rows behind the last repeat it
  const int row = row0 + min(r, rows - 1), c = row / a.group, head = g * a.group + row - c * a.group, own = s.t0 + c;
  const int own_first = s.t0 + row0 / a.group;                  // position of the block's first row
  u32x4 qf[kKS];
  {
    const char* q = a.q + (int64_t)(s.row0 + c) * a.ldq + (int64_t)head * kRowBytes + hi * 16;
#pragma unroll
    for (int i = 0; i < kKS; ++i) qf[i] = *(const u32x4*)(q + i * 32);
  }

  // Lane r stands for key r of a tile: its position (INT32_MAX: not seen), its row's place in the pool, its scales.  Entries of the index list
  // are requested three tiles ahead, of the page table two, rows one.  A tile that lies in one page, its rows within 32 bits of each other, is
  // found once for the whole wave.
  struct Meta {
    int pos0, pos, entry;                                       // pos0: of the tile's first key where it lies in one page, else -1
  };
  const int slot_mask = (1 << a.batch.page_log2) - 1;
  const uint32_t tok_bytes = a.cache.tok_bytes;
  auto request_entry = [&](int t) { return keys.n_sel && t < end ? entry_of(a, keys, at.b, t * kKeys + r) : 0; };
  auto request_page = [&](int t, int entry) __attribute__((always_inline)) {
    const int j0 = t * kKeys, late = j0 - keys.i_end - keys.late;
    Meta m;
    m.pos0 = j0 + kKeys <= keys.i_end ? j0 : late >= 0 ? late + keys.l_start : -1;
    if (j0 + kKeys > n_vis || (m.pos0 & (kKeys - 1)) != 0 || a.cache.close < kKeys) m.pos0 = -1;
    m.pos = -1;
    if (m.pos0 >= 0) {
      m.entry = page_entry(a.batch, at.b, m.pos0);
    } else {
      if (j0 + r < n_vis) m.pos = position(keys, j0 + r, entry);
      m.entry = page_entry(a.batch, at.b, m.pos);
    }
    return m;
  };
  u32x4 kr[kLoads], vr[kLoads];
  int kb = 127, vb = 127, now_pos = INT32_MAX;                  // of the lane's key: exponents of its scales, position
  int64_t place = 0;                                            // its row; where the tile lies in one page, that of the tile's first
  bool whole = false;
  auto find_rows = [&](const Meta& m) __attribute__((always_inline)) {
    whole = m.pos0 >= 0;
    if (whole) {
      const int entry = uniform(m.entry);
      const bool there = is_page(a.batch, a.cache.n_pages, m.pos0, entry);
      const int page = there ? entry : 0;
      now_pos = there ? m.pos0 + r : INT32_MAX;
      place = place_of(a.cache, page, g, m.pos0 & slot_mask);
      if constexpr (F8) {
        kb = a.cache.k_scale[block_of(a.cache, page, g)];
        vb = a.cache.v_scale[block_of(a.cache, page, g)];
      }
    } else {
      const bool there = is_page(a.batch, a.cache.n_pages, m.pos, m.entry);
      const int page = there ? m.entry : 0;
      now_pos = there ? m.pos : INT32_MAX;
      place = place_of(a.cache, page, g, there ? m.pos & slot_mask : 0);
      if constexpr (F8) {
        kb = a.cache.k_scale[block_of(a.cache, page, g)];
        vb = a.cache.v_scale[block_of(a.cache, page, g)];
      }
    }
  };
  // Keys are requested as soon as those before have left their registers, then values.
  auto load_whole = [&](u32x4 (&x)[kLoads], const char* cache) __attribute__((always_inline)) {
    const char* const from = cache + uniform(place);
    const uint32_t mine = (uint32_t)(lane / kPieces) * tok_bytes + lane % kPieces * 16;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = *(const u32x4*)(from + (uint32_t)(i * kLoadRows) * tok_bytes + mine);
  };
  auto load_apart = [&](u32x4 (&x)[kLoads], const char* cache) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) x[i] = *(const u32x4*)(cache + __shfl(place, i * kLoadRows + lane / kPieces) + lane % kPieces * 16);
  };
  auto load = [&](u32x4 (&x)[kLoads], const char* cache) __attribute__((always_inline)) {
    if (whole)
      load_whole(x, cache);
    else
      load_apart(x, cache);
  };
  // Staged rows are swizzled: 16-byte piece p of a key row lies in place p ^ (row mod 16), of a value row the 64-byte chunks by
  // row mod 4 (of rows of 128 or 64 bytes two or four share the 256 bytes that the banks cover, and take a half or a quarter of the row's number).
  auto k_swizzle = [](int key) { return kRowBytes >= 256 ? key & 15 : kRowBytes == 128 ? (key >> 1) & 7 : (key >> 2) & 3; };
  auto v_swizzle = [](int key) { return kRowBytes >= 256 ? (key & 3) << 2 : kRowBytes == 128 ? ((key >> 1) & 1) << 2 : 0; };
  unsigned char* const k_st = stage[wave][0];
  unsigned char* const v_st = stage[wave][1];
  auto put = [&](unsigned char* st, const u32x4& x, float scale, int key, int swizzle) {
    const int piece = lane % kPieces;
    unsigned char* to = st + key * kRowBytes;
    if constexpr (!F8) {
      *(u32x4*)(to + ((piece ^ swizzle) << 4)) = x;
    } else if constexpr (kBf16) {
      u32x4 y[2];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[i / 2][i % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, false));
        y[i / 2][i % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[i], scale, true));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) *(u32x4*)(to + (((piece * 2 + i) ^ swizzle) << 4)) = y[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float y[4];
        f8_unpack(x[i], y);
        *(f32x4*)(to + (((piece * 4 + i) ^ swizzle) << 4)) = f32x4{y[0] * scale, y[1] * scale, y[2] * scale, y[3] * scale};
      }
    }
  };

  f32x16 o[kMD];
#pragma unroll
  for (int md = 0; md < kMD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[md][v] = 0.f;
  float m_run = kNoReference, l_run = 0.f;

  int t = first + wave;
  Meta next{-1, -1, 0};
  int entry = 0;
  if (t < end) {
    const int mine = request_entry(t), after = request_entry(t + kWaves);
    entry = request_entry(t + 2 * kWaves);
    const Meta m = request_page(t, mine);
    next = request_page(t + kWaves, after);
    find_rows(m);
    load(kr, a.cache.k);
    load(vr, a.cache.v);
  }
  for (; t < end; t += kWaves) {
    const int pos = now_pos;
    const bool one_page = whole, more = t + kWaves < end;
    const uint64_t unseen = __ballot(pos == INT32_MAX);
    float ks = 1.f, vs = 1.f;
    if constexpr (F8) {
      // a page that nobody has may hold an infinite scale; whatever its rows hold: 0 times a NaN is one (scores of such keys are masked)
      const int k_byte = pos != INT32_MAX ? kb : 127, v_byte = pos != INT32_MAX ? vb : 127;
      ks = kBf16 ? scale_of(k_byte) : power_of(k_byte);
      vs = kBf16 ? scale_of(v_byte) : power_of(v_byte);
    }
    if (unseen) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if ((unseen >> (i * kLoadRows + lane / kPieces)) & 1) vr[i] = u32x4{0, 0, 0, 0};
    }
    auto put_rows = [&](unsigned char* st, const u32x4 (&x)[kLoads], float scale, auto swizzle) __attribute__((always_inline)) {
      float of_row[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) of_row[i] = scale;
      if (F8 && !one_page) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) of_row[i] = __shfl(scale, i * kLoadRows + lane / kPieces);
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int key = i * kLoadRows + lane / kPieces;
        put(st, x[i], of_row[i], key, swizzle(key));
      }
    };
    put_rows(k_st, kr, ks, k_swizzle);
    if (more) {
      find_rows(next);
      load(kr, a.cache.k);
    }
    if (t + 2 * kWaves < end) next = request_page(t + 2 * kWaves, entry);      // in front of the values: the next tile's keys do not wait for them
    entry = request_entry(t + 3 * kWaves);
    put_rows(v_st, vr, vs, v_swizzle);
    if (more) load(vr, a.cache.v);
    wave_fence();

    f32x16 x;
#pragma unroll
    for (int v = 0; v < 16; ++v) x[v] = 0.f;
#pragma unroll
    for (int i = 0; i < kKS; ++i) {
      const u32x4 kf = *(const u32x4*)(k_st + r * kRowBytes + (((2 * i + hi) ^ k_swizzle(r)) << 4));
      if constexpr (kBf16) {
        x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]), x, 0, 0, 0);
      } else {
        const f32x4 k4 = __builtin_bit_cast(f32x4, kf), q4 = __builtin_bit_cast(f32x4, qf[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(k4[e], q4[e], x, 0, 0, 0);
      }
    }
    const bool masked = __ballot(pos > own_first);
    if (masked) {                                               // some key is not for all rows
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (__shfl(pos, 8 * (v / 4) + 4 * hi + v % 4) > own) x[v] = -INFINITY;
    }
    f32x16 e;
    auto to_reference = [&](float to) __attribute__((always_inline)) {       // what the sums so far are relative to
      const float less = exp_of<T>(m_run - to);
      m_run = to;
      l_run *= less;
      if (__ballot(less != 1.f)) {
#pragma unroll
        for (int md = 0; md < kMD; ++md)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[md][v] *= less;
      }
    };
    auto largest = [&]() __attribute__((always_inline)) {
      float top = x[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) top = fmaxf(top, x[v]);
      top = halves_max(top);
      return top == -INFINITY ? kNoReference : score_of<T, CAP>(top, f.scale, f.cap);
    };
    auto exponentials = [&]() __attribute__((always_inline)) {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        e[v] = exp_of<T>(score_of<T, CAP>(x[v], f.scale, f.cap) - m_run);
        if (CAP && x[v] == -INFINITY) e[v] = 0.f;               // (a capped -inf is none)
        sum += e[v];
      }
      return sum;
    };
    if constexpr (kLags) {
      // Against the reference as it stands.  Where a row's exceed it by far (and at first) it moves to its largest logit, and they are taken again.
      float sum = exponentials();
      if (__ballot(sum > 256.f)) {
        to_reference(fmaxf(m_run, largest()));
        sum = exponentials();
      }
      l_run += sum;
    } else {
      // (two sets of sixteen registers for them are more than rows of 256 bytes and more on their way leave)
      to_reference(fmaxf(m_run, largest()));
      l_run += exponentials();
    }
    if constexpr (kBf16) {
      const int tr_key = 4 * hi + ((lane & 15) >> 2), tr_dim = ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
#pragma unroll
      for (int kp = 0; kp < 2; ++kp) {
        __builtin_amdgcn_sched_barrier(0);                      // (fragments of both at once cost registers that rows on their way need)
        bf16x8 p, rest;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = (__bf16)e[8 * kp + i];
          rest[i] = (__bf16)(e[8 * kp + i] - (float)p[i]);
        }
#pragma unroll
        for (int md = 0; md < kMD; ++md) {
          // lane i of sixteen receives element i % 4 of the 8 bytes that lanes 4 e + i / 4 address: dimension i of keys e = 0 .. 3
          auto part = [&](int key) {
            const int piece = (md * 32 + tr_dim) / 8;
            return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(v_st + key * kRowBytes + ((piece ^ v_swizzle(key)) << 4) + (tr_dim & 4) * 2));
          };
          const i16x4 lo = part(16 * kp + tr_key), up = part(16 * kp + 8 + tr_key);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
          o[md] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p, o[md], 0, 0, 0);
          o[md] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, rest, o[md], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        const int key = 8 * (v / 4) + 4 * hi + v % 4;
#pragma unroll
        for (int md = 0; md < kMD; ++md) {
          const int dim = md * 32 + r;
          const float vf = *(const float*)(v_st + key * kRowBytes + (((dim / 4) ^ v_swizzle(key)) << 4) + (dim & 3) * 4);
          o[md] = __builtin_amdgcn_mfma_f32_32x32x2f32(vf, e[v], o[md], 0, 0, 0);
        }
      }
    }
    wave_fence();
  }

  // ---- the waves' results meet in LDS: a wave's sums of row r, dimensions 4 n ..., at (n * 32 + (r ^ n)) * 16 of its staging space
  __syncthreads();
  l_run = nan_if(holds_nan<T>(qf), halves_sum(l_run));
  if (hi == 0) {
    ml[wave][r][0] = m_run;
    ml[wave][r][1] = l_run;
  }
  constexpr int kWaveFloats = 2 * kTileBytes / 4;
  static_assert(kWaveFloats >= kRows * D, "a wave's staging space holds its sums");
  float* const sums = (float*)&stage[0][0][0];
#pragma unroll
  for (int md = 0; md < kMD; ++md)
#pragma unroll
    for (int v = 0; v < 16; v += 4) {
      const int n = md * 8 + v / 4 * 2 + hi;
      *(f32x4*)(sums + wave * kWaveFloats + (n * kRows + (r ^ (n & 31))) * 4) = f32x4{o[md][v], o[md][v + 1], o[md][v + 2], o[md][v + 3]};
    }
  __syncthreads();
  for (int e = tid; e < rows * (D / 4); e += 64 * kWaves) {
    const int n = e % (D / 4), row_in = e / (D / 4);
    float m = ml[0][row_in][0], l = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, ml[w][row_in][0]);
    const float ref = m == -INFINITY ? 0.f : m;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = exp_of<T>(ml[w][row_in][0] - ref);
      l = __builtin_fmaf(ml[w][row_in][1], by, l);
      const f32x4 x = *(const f32x4*)(sums + w * kWaveFloats + (n * kRows + (row_in ^ (n & 31))) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(x[i], by, sum[i]);
    }
    if (alone) {
      const int rg = row0 + row_in, tok = rg / a.group, hd = g * a.group + rg - tok * a.group;
      const bool nothing = nothing_seen(l);
      const float inv = nothing ? 0.f : 1.f / l;
      char* to = a.out + (int64_t)(s.row0 + tok) * a.ldo + (int64_t)hd * kRowBytes;
      if constexpr (kBf16) {
        const bf16x2 lo = __builtin_convertvector((f32x2{sum[0] * inv, sum[1] * inv}), bf16x2), up = __builtin_convertvector((f32x2{sum[2] * inv, sum[3] * inv}), bf16x2);
        *(uint2*)(to + n * 8) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, up));
      } else {
        *(f32x4*)(to + n * 16) = nothing ? f32x4{0.f, 0.f, 0.f, 0.f} : sum / l;
      }
      if (a.lse && n == 0) a.lse[(int64_t)(s.row0 + tok) * a.h + hd] = nothing ? -INFINITY : lse_of<T>(m, l);
    } else {
      const int64_t part = ((at.slot + (int64_t)at.slice * at.blocks) * a.cache.h_kv + g) * kRows + row_in;
      *(f32x4*)(f.part_o + part * D + n * 4) = sum;
      if (n == 0) *(float2*)(f.part_ml + part * 2) = make_float2(m, l);
    }
  }
}

// Slices of a row joined: a workgroup takes a row, its four waves share the slices.  Only rows of sequences of several slices are gone
// through, by as many workgroups as the chip holds at most.
template <typename T, int D> __global__ __launch_bounds__(256) void join_few(FewArgs f) {
  constexpr int kMine = D > 64 ? D / 64 : 1, kLanes = D / kMine;      // a lane's dimensions; lanes that have some
  typedef __attribute__((ext_vector_type(kMine))) float vec;
  __shared__ vec sums[4][64];
  __shared__ float2 ml[4];
  const AttendArgs& a = f.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Plan plan = plan_of(a, f.shape, f.made);
  for (int64_t u = blockIdx.x;; u += gridDim.x) {
    const int g = (int)(u % a.cache.h_kv);
    const Split at = uniform(split_of(a, f.shape, plan, f.made, u / a.cache.h_kv));
    if (at.b < 0) return;
    const Seq s = uniform(sequence(a.batch, at.b));
    const Keys keys = keys_of(a, s);
    const int n_rows = s.n * a.group, block = at.i / kRows, blocks = (n_rows + kRows - 1) / kRows;
    const int n_vis = keys_until(a, s, keys, min(block * kRows + kRows, n_rows) - 1), tiles = (n_vis + kKeys - 1) / kKeys;
    const int n = (tiles + plan.slice - 1) / plan.slice;
    if (n <= 1) continue;
    auto place = [&](int i) { return ((at.slot + block + (int64_t)i * blocks) * a.cache.h_kv + g) * kRows + at.i - block * kRows; };
    float m = -INFINITY, l = 0.f;
    vec sum = 0.f;
    for (int i0 = wave; i0 < n; i0 += 256) {                    // a lane has the i0 + 4 lane-th slice's weight
      float mine = -INFINITY, part_l = 0.f;
      if (i0 + lane * 4 < n) {
        const float2 x = *(const float2*)(f.part_ml + place(i0 + lane * 4) * 2);
        mine = x.x;
        part_l = x.y;
      }
      const float top = fmaxf(m, wave_max(mine)), ref = top == -INFINITY ? 0.f : top, less = exp_of<T>(m - ref);
      m = top;
      const float by = exp_of<T>(mine - ref);
      l = l * less + wave_sum(part_l * by);
      sum *= less;
      const int here = min((n - i0 + 3) / 4, 64);
      for (int i = 0; i < here; i += 8) {
        vec x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = *(const vec*)(f.part_o + place(i0 + min(i + k, here - 1) * 4) * D + lane % kLanes * kMine);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k] * (i + k < here ? __shfl(by, min(i + k, 63)) : 0.f);
      }
    }
    __syncthreads();
    sums[wave][lane] = sum;
    if (lane == 0) ml[wave] = make_float2(m, l);
    __syncthreads();
    if (wave != 0) continue;
    m = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
    const float ref = m == -INFINITY ? 0.f : m;
    l = 0.f;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float by = exp_of<T>(ml[w].x - ref);
      l = __builtin_fmaf(ml[w].y, by, l);
      sum += sums[w][lane] * by;
    }
    const int tok = s.row0 + at.i / a.group, head = g * a.group + at.i % a.group;
    T* out = (T*)(a.out + (int64_t)tok * a.ldo) + (int64_t)head * D + lane * kMine;
    if (lane >= kLanes) continue;
#pragma unroll
    for (int i = 0; i < kMine; ++i) store_f32<T>(out + i, nothing_seen(l) ? 0.f : sum[i] / l);
    if (a.lse && lane == 0) a.lse[(int64_t)tok * a.h + head] = nothing_seen(l) ? -INFINITY : lse_of<T>(m, l);
  }
}

// Workgroups that the chip holds: staging space in LDS and registers leave a compute unit one of fp32 rows of 512 bytes, three of 8-bit rows
// of 64 elements brought to bf16, two of the others.  (1024 for rows of 64 elements, whatever their registers: eight sequences of 64 thousand
// keys, 8 bits, 138 us, 1.3 rounds.)  A slice has a tile for every wave; where no sequence can have more than 512 keys, four, so that none is
// cut and nothing is left to join (301 keys: 11.2 us cut and joined, 9.6 so).  Not so fp32, whose products take 3.4 us a tile, where there are few blocks (four
// sequences of 455 keys, 8 heads: 33 us uncut, 18.6 cut; two of 468 tokens 34 and 40).
SliceShape shape_of(int d, int es, bool f8, int most_rows, bool shorts) {
  return SliceShape{d * es > 256 ? 256 : f8 && d * es < 256 ? 768 : 512, shorts ? 4 * kWaves : kWaves, most_rows, shorts};
}

template <typename T, bool F8, int D> int launch(FewArgs f, int64_t units, dim3 join, hipStream_t st) {
  // (more units than a row of workgroups, one launch behind the other: looking at a second dimension cost sixteen sequences of 18 to 66 thousand
  // 8-bit keys 284 -> 293 us)
  for (f.first = 0; f.first < units; f.first += kGridRow) {
    const dim3 grid((unsigned)std::min<int64_t>(units - f.first, kGridRow));
    if (f.a.cap > 0.f)
      attend_few<T, F8, D, true><<<grid, 64 * kWaves, 0, st>>>(f);
    else
      attend_few<T, F8, D, false><<<grid, 64 * kWaves, 0, st>>>(f);
    ESA_LAUNCH_CHECK("attend_few");
  }
  if (join.x == 0) return ESA_OK;
  join_few<T, D><<<join, 256, 0, st>>>(f);
  ESA_LAUNCH_CHECK("join_few");
  return ESA_OK;
}
template <typename T> int launch_all(const AttendArgs& a, bool f8, int most_rows, void* ws, hipStream_t st) {
  const int d = a.cache.d;
  const int64_t most_keys = most_keys_of(a);
  const bool shorts = most_keys <= 4 * kWaves * kKeys && (sizeof(T) == 2 || a.batch.n_tok * a.h >= 128 * kRows);
  const SliceShape shape = shape_of(d, sizeof(T), f8, most_rows, shorts);
  const int64_t parts = most_parts(shape, a.cache.h_kv) * a.cache.h_kv;
  const SplitArgs<SliceShape> split = split_args<T>(a, shape, parts, ws);
  char* const made = (char*)ws + (split_workspace(parts, kRows, d) + kPlanBytes - 1) / kPlanBytes * kPlanBytes;
  const FewArgs f{split, Made{(int*)made, (Upto*)(made + kPlanBytes)}, 0};
  const int64_t units = most_units(f.shape, a.batch.n_tok, a.batch.n_seq, a.group, a.cache.h_kv) * a.cache.h_kv;
  if (a.batch.n_seq > 64) {
    plan_few<<<1, 1024, 0, st>>>(f);
    ESA_LAUNCH_CHECK("plan_few");
  }
  const int64_t by_blocks = most_blocks(f.shape, a.batch.n_tok, a.batch.n_seq, a.group) * kRows * a.cache.h_kv, by_tokens = a.batch.n_tok * a.h;
  const bool none_cut = most_keys <= (int64_t)shape.least * kKeys;
  const dim3 join(none_cut ? 0 : (unsigned)std::min<int64_t>(std::min(by_blocks, by_tokens), 2048));
  if (d == 32) return f8 ? launch<T, true, 32>(f, units, join, st) : launch<T, false, 32>(f, units, join, st);
  if (d == 64) return f8 ? launch<T, true, 64>(f, units, join, st) : launch<T, false, 64>(f, units, join, st);
  if constexpr (sizeof(T) == 2) {
    if (d == 256) return f8 ? launch<T, true, 256>(f, units, join, st) : launch<T, false, 256>(f, units, join, st);
  }
  return f8 ? launch<T, true, 128>(f, units, join, st) : launch<T, false, 128>(f, units, join, st);
}

}  // namespace

size_t few_workspace(int n_seq, int h_kv, int d, int dtype) {
  const int64_t parts = most_parts(shape_of(d, dtype == ESA_F32 ? 4 : 2, true, INT32_MAX, false), h_kv) * h_kv;
  return split_workspace(parts, kRows, d) + 2 * kPlanBytes + ((size_t)n_seq + 63) / 64 * sizeof(Upto);
}

int launch_few(const AttendArgs& a, bool f8, int dtype, int most_rows, void* ws, hipStream_t st) {
  return dtype == ESA_F32 ? launch_all<float>(a, f8, most_rows, ws, st) : launch_all<bf16_t>(a, f8, most_rows, ws, st);
}

}  // namespace paged
}  // namespace esa
