// Attention of many rows over a paged cache (chunks, prompts): bf16, head sizes 64 and 128.
//
// A workgroup has 256 rows (new tokens x query heads of a KV head), 32 to each of its eight waves, and a slice of the keys, in tiles of 64
// that the waves share: every thread fetches its part of a tile into registers ahead, brings it to bf16 (8-bit pages: times the block's
// scale, exactly) and writes it to LDS.  The products are those of the kernel for few rows: S^T = K Q^T, O^T += V^T P^T, a lane stands for a
// row; a probability is one bf16 term (its rounding is as large as the output's), and the reference of the softmax stays where it is until a
// logit exceeds it by 2^8, which spares the sums' rescaling.
//   Here the matrix cores bound: 32 instructions a wave and tile, 2048 cycles of a compute unit's four for all waves, and as many for the LDS
// reads; the softmax and the staging are about as many cycles of vector instructions, which ran one behind the other when the
// two waves of a SIMD (w and w + 4) went through a tile together (5600 cycles a tile).  So they take turns: in one phase waves 0 - 3 multiply
// (scores of tile j, sums of tile j - 1) while waves 4 - 7 do the softmax of tile j - 1 and stage their part of tile j + 1, in the
// next they change places.  Tile j's keys are read in phases 2 j and 2 j + 1, its values in 2 j + 2 and 2 j + 3, and it is written in
// 2 j - 2 (by waves 4 - 7) and 2 j - 1: two buffers of keys, three of values and positions.
#include "attend_sliced.h"

namespace esa {
namespace paged {
namespace {

constexpr int kRows = 256, kKeys = 64, kWaves = 8;

template <bool F8, int D, bool CAP>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void attend_many(SlicedArgs f) {
  constexpr int kRowBytes = D * 2;                              // of a staged row
  constexpr int kHeldBytes = F8 ? D : kRowBytes;
  constexpr int kPieces = kHeldBytes / 16;                      // threads that fetch a row
  constexpr int kPass = 64 * kWaves / kPieces;                  // rows that the workgroup fetches at a time, of the tile's keys and values
  constexpr int kLoads = 2 * kKeys / kPass;
  constexpr int kMine = kPass < kKeys ? kKeys / kPass : 1;      // keys of a thread
  constexpr int kKS = D / 16, kMD = D / 32;
  constexpr int kTileBytes = kKeys * kRowBytes;
  __shared__ __attribute__((aligned(16))) unsigned char k_stage[2][kTileBytes], v_stage[3][kTileBytes];
  __shared__ __attribute__((aligned(16))) int seen[3][kKeys];                         // positions, INT32_MAX: not seen
  const AttendArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % a.cache.h_kv;
  const Plan plan = plan_of(a, f.shape);
  const int slice = plan.slice;
  const Part at = part_of(a, f.shape, plan, blockIdx.x / a.cache.h_kv);
  if (at.b < 0) return;
  const Seq s = sequence(a.batch, at.b);
  const Keys keys = keys_of(a, s);
  const int n_rows = s.n * a.group, row0 = at.block * kRows, rows = min(n_rows - row0, kRows);
  const int n_vis = keys_until(a, s, keys, row0 + rows - 1), tiles = (n_vis + kKeys - 1) / kKeys;
  const int first = at.slice * slice, end = min(first + slice, tiles);
  if (at.slice > 0 && first >= end) return;
  const bool alone = tiles <= slice;

  // a lane's row; rows behind the last repeat it
  const int row = row0 + min(wave * 32 + r, rows - 1), c = row / a.group, head = g * a.group + row - c * a.group, own = s.t0 + c;
  const int own_first = s.t0 + (row0 + min(wave * 32, rows - 1)) / a.group;      // position of the wave's first row
  u32x4 qf[kKS];
  {
    const char* q = a.q + (int64_t)(s.row0 + c) * a.ldq + (int64_t)head * kRowBytes + hi * 16;
#pragma unroll
    for (int i = 0; i < kKS; ++i) qf[i] = *(const u32x4*)(q + i * 32);
  }

  // ---- staging: a thread has piece tid % kPieces of rows tid / kPieces + i kPass of the tile's keys, then values
  // Entries of the index list are requested three tiles ahead, of the page table two, rows one.
  struct Meta {
    int pos[kMine], entry[kMine];
  };
  struct Entries {
    int x[kMine];
  };
  const int piece = tid % kPieces, my_row = tid / kPieces;
  auto key_of = [&](int i) { return (my_row + i * kPass) % kKeys; };
  auto request_entries = [&](int t) {
    Entries e;
#pragma unroll
    for (int i = 0; i < kMine; ++i) e.x[i] = keys.n_sel && t < end ? entry_of(a, keys, at.b, t * kKeys + key_of(i)) : 0;
    return e;
  };
  auto request_pages = [&](int t, const Entries& e) {
    Meta m;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int j = t * kKeys + key_of(i);
      m.pos[i] = j < n_vis ? position(keys, j, e.x[i]) : -1;
      m.entry[i] = page_entry(a.batch, at.b, m.pos[i]);
    }
    return m;
  };
  const int slot_mask = (1 << a.batch.page_log2) - 1;
  struct Held {
    u32x4 x[kLoads];
    int scale[kLoads], pos[kMine];                              // position: INT32_MAX where nothing is seen
  };
  auto load = [&](Held& h, const Meta& m) {
    int64_t place[kMine], block[kMine];
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const bool there = is_page(a.batch, a.cache.n_pages, m.pos[n], m.entry[n]);
      const int page = there ? m.entry[n] : 0;
      h.pos[n] = there ? m.pos[n] : INT32_MAX;
      place[n] = page * a.cache.page_bytes + g * a.cache.head_bytes + (there ? m.pos[n] & slot_mask : 0) * a.cache.tok_bytes + piece * 16;
      block[n] = (int64_t)page * a.cache.h_kv + g;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool values = i * kPass + my_row >= kKeys;
      h.x[i] = *(const u32x4*)((values ? a.cache.v : a.cache.k) + place[kMine == 1 ? 0 : i % kMine]);
      if constexpr (F8) h.scale[i] = (values ? a.cache.v_scale : a.cache.k_scale)[block[kMine == 1 ? 0 : i % kMine]];
    }
  };
  auto k_swizzle = [](int key) { return kRowBytes >= 256 ? key & 15 : (key >> 1) & 7; };
  auto v_swizzle = [](int key) { return kRowBytes >= 256 ? (key & 3) << 2 : ((key >> 1) & 1) << 2; };
  auto put = [&](const Held& h, int j) {
    const int third = j % 3;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool values = i * kPass + my_row >= kKeys;
      const int n = kMine == 1 ? 0 : i % kMine, key = key_of(i);
      const bool there = h.pos[n] != INT32_MAX;
      unsigned char* to = (values ? v_stage[third] : k_stage[j & 1]) + key * kRowBytes;
      const int swizzle = values ? v_swizzle(key) : k_swizzle(key);
      u32x4 x = h.x[i];
      if (!there) x = u32x4{0, 0, 0, 0};                        // whatever lies there: 0 times a NaN is one
      if constexpr (F8) {
        const float by = scale_of(there ? h.scale[i] : 127);
        u32x4 y[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e / 2][e % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], by, false));
          y[e / 2][e % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x[e], by, true));
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) *(u32x4*)(to + (((piece * 2 + e) ^ swizzle) << 4)) = y[e];
      } else {
        *(u32x4*)(to + ((piece ^ swizzle) << 4)) = x;
      }
      if (piece == 0 && (kLoads == 1 ? !values : i < kMine)) seen[third][key] = h.pos[n];
    }
  };

  f32x16 o[kMD], x[2];
#pragma unroll
  for (int md = 0; md < kMD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[md][v] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  bf16x8 p[4];

  // First product of tile j.
  auto scores = [&](int j) __attribute__((always_inline)) {
    const unsigned char* const k_st = k_stage[j & 1];
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int v = 0; v < 16; ++v) x[n][v] = 0.f;
#pragma unroll
    for (int i = 0; i < kKS; ++i)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const u32x4 kf = *(const u32x4*)(k_st + (n * 32 + r) * kRowBytes + (((2 * i + hi) ^ k_swizzle(r)) << 4));
        x[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[i]), x[n], 0, 0, 0);
      }
  };
  // Second product of tile j.
  auto sums = [&](int buffer) __attribute__((always_inline)) {
    unsigned char* const v_st = v_stage[buffer];
    const int tr_key = 4 * hi + ((lane & 15) >> 2), tr_dim = ((lane >> 4) & 1) * 16 + 4 * (lane & 3);
#pragma unroll
    for (int kp = 0; kp < 4; ++kp)
#pragma unroll
      for (int md = 0; md < kMD; ++md) {
        // lane i of sixteen receives element i % 4 of the 8 bytes that lanes 4 e + i / 4 address: dimension i of keys e = 0 .. 3
        auto part = [&](int key) {
          const int at_piece = (md * 32 + tr_dim) / 8;
          return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(v_st + key * kRowBytes + ((at_piece ^ v_swizzle(key)) << 4) + (tr_dim & 4) * 2));
        };
        const i16x4 lo = part(16 * kp + tr_key), up = part(16 * kp + 8 + tr_key);
        o[md] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7)), p[kp], o[md], 0, 0, 0);
      }
  };
  // Tile j's probabilities from its scores.
  auto softmax = [&](int buffer) __attribute__((always_inline)) {
    if constexpr (CAP) {
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v) x[n][v] = score_of<bf16_t, CAP>(x[n][v], f.scale, f.cap);
    }
    const float scale = CAP ? 1.f : f.scale;
    if (__ballot(seen[buffer][lane] > own_first)) {             // some key is not for all rows of the wave
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int v = 0; v < 16; ++v)
          if (seen[buffer][n * 32 + 8 * (v / 4) + 4 * hi + v % 4] > own) x[n][v] = -INFINITY;
    }
    float top = fmaxf(x[0][0], x[1][0]);
#pragma unroll
    for (int v = 1; v < 16; ++v) top = fmaxf(fmaxf(top, x[0][v]), x[1][v]);
    top = halves_max(top) * scale;
    if (__ballot(top > m_run + 8.f)) {
      const float to = fmaxf(m_run, top), less = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - to);
      m_run = to;
      l_run *= less;
#pragma unroll
      for (int md = 0; md < kMD; ++md)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[md][v] *= less;
    }
    const float ref = m_run == -INFINITY ? 0.f : m_run;
    float sum[2] = {0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 16; ++v)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float e = __builtin_amdgcn_exp2f(CAP ? x[n][v] - ref : __builtin_fmaf(x[n][v], scale, -ref));
        sum[n] += e;
        p[2 * n + v / 8][v % 8] = (__bf16)e;
      }
    l_run += sum[0] + sum[1];
  };
  // Phases end together: LDS is settled, loads from memory stay on their way.
  auto phase_end = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  const int n_tiles = max(end - first, 0);
  Held held;
  Meta next;
  Entries entries;
  {
    const Entries e0 = request_entries(first), e1 = request_entries(first + 1);
    entries = request_entries(first + 2);
    const Meta m = request_pages(first, e0);
    next = request_pages(first + 1, e1);
    load(held, m);
  }
  // Part of tile j into LDS, the next ones' requested.
  auto stage = [&](int j) __attribute__((always_inline)) {
    if (j >= n_tiles) return;
    put(held, j);
    if (j + 1 < n_tiles) load(held, next);
    if (j + 2 < n_tiles) next = request_pages(first + j + 2, entries);
    entries = request_entries(first + j + 3);
  };
  stage(0);
  phase_end();
  const bool second = wave >= kWaves / 2;
  if (second) {
    stage(1);
    phase_end();
  }
  int vb = 2;                                                   // buffer of the tile before
  for (int j = 0; j < n_tiles; ++j) {
    const int vn = vb == 2 ? 0 : vb + 1;                        // j % 3
    __builtin_amdgcn_s_setprio(1);
    scores(j);
    if (j > 0) sums(vb);
    __builtin_amdgcn_s_setprio(0);
    phase_end();
    softmax(vn);
    stage(second ? j + 2 : j + 1);
    vb = vn;
    phase_end();
  }
  if (n_tiles > 0) sums(vb);
  if (!second) phase_end();

  l_run = halves_sum(l_run);
  if (wave * 32 + r >= rows) return;
  const int hd = head;
  if (alone) {
    const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
    char* to = a.out + (int64_t)(s.row0 + c) * a.ldo + (int64_t)hd * kRowBytes;
#pragma unroll
    for (int md = 0; md < kMD; ++md)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const bf16x2 lo = __builtin_convertvector((f32x2{o[md][v] * inv, o[md][v + 1] * inv}), bf16x2);
        const bf16x2 up = __builtin_convertvector((f32x2{o[md][v + 2] * inv, o[md][v + 3] * inv}), bf16x2);
        *(uint2*)(to + (md * 32 + v * 2 + 4 * hi) * 2) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, up));
      }
    if (a.lse && hi == 0) a.lse[(int64_t)(s.row0 + c) * a.h + hd] = l_run > 0.f ? lse_of<bf16_t>(m_run, l_run) : -INFINITY;
  } else {
    const int64_t part = ((at.slot + (int64_t)at.slice * at.blocks) * a.cache.h_kv + g) * kRows + wave * 32 + r;
#pragma unroll
    for (int md = 0; md < kMD; ++md)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *(f32x4*)(f.part_o + part * D + md * 32 + v * 2 + 4 * hi) = f32x4{o[md][v], o[md][v + 1], o[md][v + 2], o[md][v + 3]};
    if (hi == 0) *(float2*)(f.part_ml + part * 2) = make_float2(m_run, l_run);
  }
}

Shape shape_of(int above) { return Shape{kRows, kKeys, 256, 1, 4, above, INT32_MAX}; }

template <bool F8, int D> int launch(const SlicedArgs& f, dim3 grid, hipStream_t st) {
  if (f.a.cap > 0.f)
    attend_many<F8, D, true><<<grid, 64 * kWaves, 0, st>>>(f);
  else
    attend_many<F8, D, false><<<grid, 64 * kWaves, 0, st>>>(f);
  ESA_LAUNCH_CHECK("attend_many");
  return ESA_OK;
}

}  // namespace

size_t many_workspace(int h_kv, int d) { return sliced_workspace(shape_of(0), h_kv, d); }

int launch_many(const AttendArgs& a, bool f8, int above, void* ws, hipStream_t st) {
  SlicedArgs f;
  set_sliced<bf16_t>(f, a, shape_of(above), ws);
  const int64_t units = most_units(f.shape, a.batch.n_tok, a.batch.n_seq, a.group, a.cache.h_kv) * a.cache.h_kv;
  if (units > INT32_MAX) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: %lld workgroups", (long long)units);
  const dim3 grid((unsigned)units);
  int rc;
  if (a.cache.d == 64)
    rc = f8 ? launch<true, 64>(f, grid, st) : launch<false, 64>(f, grid, st);
  else
    rc = f8 ? launch<true, 128>(f, grid, st) : launch<false, 128>(f, grid, st);
  return rc != ESA_OK ? rc : launch_join<bf16_t, false>(f, st);
}

}  // namespace paged
}  // namespace esa
