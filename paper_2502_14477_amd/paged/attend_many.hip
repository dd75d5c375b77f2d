// Attention of many rows over a paged cache (chunks, prompts): bf16, head sizes 64 and 128.
//
// A workgroup has 256 rows (new tokens x query heads of a KV head), 32 to each of its eight waves, and a slice of the keys, in tiles of 64
// that the waves share: every thread fetches its part of a tile into registers ahead, brings it to bf16 (8-bit pages: times the block's
// scale, exactly) and writes it to LDS.  The products are those of the kernel for few rows: S^T = K Q^T, O^T += V^T P^T, a lane stands for a
// row; the reference of the softmax stays where it is until probabilities sum up to over 2^8, which spares the maxima and the sums'
// rescaling.  A probability enters as one bf16 term at head size 128, whose rounding is as large as the output's, and as two at 64 (16 bits), as
// contiguous chunks take one at 128 and more at 64: outputs are 2.3e-3 and 1.66e-3 from the exact ones.  The second term is half more matrix
// instructions and a third more vector ones: prompts of up to 1024 tokens behind 16 thousand 428 us at 64 (bf16 pages; 325 with one term), 673 at
// 128 (8-bit ones; 490).
//   Here the matrix cores bound: 32 instructions a wave and tile (24 with 64 elements a row), 2048 cycles of a compute unit's four for all waves, and as many for the LDS
// reads.  What else a wave has to do is 250 instructions a tile, so they have to run beside its own matrix instructions: in a step of 32 keys
// the scores of the next 32 and the sums of the 32 before are multiplied while the probabilities of these are made and a part of the tile
// after next is staged, slot by slot (one instruction of each product and its share of the rest), in an order that the compiler keeps.
// (Without that order, products and softmax one behind the other in a wave: 5600 cycles a tile.  Two groups of waves that took turns with
// products and softmax, a barrier between: the same, as a wave by itself issues a vector instruction every five cycles or so.)
//   In iteration j keys of tiles j and j + 1 and values of j - 1 and j are read and tile j + 2 is written: four buffers, one barrier.
//   A tile takes 1.8 us with 8-bit pages, 2.0 with bf16 ones, 2.4 with a cap, 1.65 with 64 elements a row; four chunks of up to 1024 tokens behind 16
// thousand, 32 and 8 heads, 8-bit pages, 480 to 504 us or 0.93 to 0.97 PFLOP/s.  A workgroup's way to its first tile and its partial sums take 14 to 20 us more.
#include <algorithm>

#include "attend_common.h"
#include "shares.h"

namespace esa {
namespace paged {
namespace {

constexpr int kRows = ShareShape::rows, kKeys = ShareShape::keys, kWaves = kRows / 32;
constexpr int terms_of(int d) { return d == 64 ? 2 : 1; }      // bf16 terms of a probability
// What the lower or the upper one of a pair of bf16 numbers leaves of x, exactly, in one instruction (capped chunks of 333 and 117 tokens over 5000 keys:
// 68 us with the number brought to fp32 and taken away, 63.5 so).  The factors are registers that the compiler does not see through: as constants
// they came out wrong.
struct Leaves {
  uint32_t minus_lower = 0x0000BF80u, minus_upper = 0xBF800000u;
  __device__ __forceinline__ Leaves() { asm("" : "+s"(minus_lower), "+s"(minus_upper)); }
  __device__ __forceinline__ float lower(bf16x2 p, float x) const { return __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2, minus_lower), x, false); }
  __device__ __forceinline__ float upper(bf16x2 p, float x) const { return __builtin_amdgcn_fdot2_f32_bf16(p, __builtin_bit_cast(bf16x2, minus_upper), x, false); }
};
struct ManyArgs : SplitArgs<ShareShape> {
  Record* records;          // [slot]
  int units;                // workgroups that share the work
};

template <bool F8, int D, bool CAP>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2))) void attend_many(ManyArgs f) {
  constexpr int kRowBytes = D * 2;                              // of a staged row
  constexpr int kHeldBytes = F8 ? D : kRowBytes;
  constexpr int kPieces = kHeldBytes / 16;                      // threads that fetch a row
  constexpr int kPass = 64 * kWaves / kPieces;                  // rows that the workgroup fetches at a time, of the tile's keys and values
  constexpr int kLoads = 2 * kKeys / kPass;
  constexpr int kMine = kPass < kKeys ? kKeys / kPass : 1;      // keys of a thread
  constexpr int kKS = D / 16, kMD = D / 32;
  // Rows in LDS are padded so that what lanes read together lies in different banks and every fragment's place is a constant from a lane's
  // first: 16 bytes behind a key row (eight lanes read 16 bytes of eight rows), 64 behind a value row (64 bytes of four).
  constexpr int kBuffers = 4, kKeyStride = kRowBytes + 16, kValueStride = kRowBytes + 64;
  static_assert(kKeyStride % 128 == 16 && (kValueStride % 256 == 64 || kValueStride % 256 == 192), "bank groups");
  __shared__ __attribute__((aligned(16))) unsigned char k_stage[kBuffers][kKeys * kKeyStride], v_stage[kBuffers][kKeys * kValueStride];
  __shared__ __attribute__((aligned(16))) int seen[kBuffers][kKeys];                  // positions, INT32_MAX: not seen
  const AttendArgs& a = f.a;
  const int tid = threadIdx.x, lane = tid & 63, r = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = uniform((int)blockIdx.x % a.cache.h_kv);
  for_parts(a, f.shape, f.records, [&](const Part& at) __attribute__((always_inline)) {
  const Seq& s = at.s;
  const Keys& keys = at.keys;
  const int row0 = at.row0, rows = at.rows, n_vis = at.n_vis, first = at.from, end = at.end;

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
  // Entries of the index list are requested three tiles ahead, of the page table two, rows one; behind the slice's last tile something is
  // fetched that nobody reads.  A tile that lies in one page, its rows within 32 bits of each other, is found once for the whole workgroup.
  const int piece = tid % kPieces, my_row = tid / kPieces;
  auto key_of = [&](int i) { return kPass <= kKeys ? my_row + i * kPass % kKeys : my_row % kKeys; };
  auto is_value = [&](int i) { return kPass <= kKeys ? i >= kKeys / kPass : my_row >= kKeys; };
  const int32_t* const list = keys.n_sel ? a.idx + (int64_t)at.b * a.idx_ld : a.batch.pages;
  const int list_last = max(keys.n_sel - 1, 0);
  const int slot_mask = (1 << a.batch.page_log2) - 1;
  const uint32_t tok_bytes = a.cache.tok_bytes;
  struct Entries {
    int x[kMine];
  };
  auto request_entries = [&](int t) {
    Entries e;
#pragma unroll
    for (int i = 0; i < kMine; ++i) e.x[i] = list[min(max(t * kKeys + key_of(i) - keys.i_end, 0), list_last)];
    return e;
  };
  struct Meta {
    int pos0;                                                   // of the tile's first key where it lies in one page, else -1
    int pos[kMine], entry[kMine];
  };
  auto request_pages = [&](int t, const Entries& e) {
    Meta m;
    const int j0 = t * kKeys, late = j0 - keys.i_end - keys.late;
    m.pos0 = j0 + kKeys <= keys.i_end ? j0 : late >= 0 ? late + keys.l_start : -1;
    if (j0 + kKeys > n_vis || (m.pos0 & (kKeys - 1)) != 0 || a.cache.close < kKeys) m.pos0 = -1;
    if (m.pos0 >= 0) {
      m.entry[0] = page_entry(a.batch, at.b, m.pos0);
    } else {
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int j = j0 + key_of(i), p = position(keys, j, e.x[i]);
        m.pos[i] = j < n_vis ? p : -1;
        m.entry[i] = page_entry(a.batch, at.b, m.pos[i]);
      }
    }
    return m;
  };
  struct Held {
    u32x4 x[kLoads];
    int scale[kLoads], pos[kMine];                              // position: INT32_MAX where nothing is seen
    bool whole;                                                 // a tile in one page
  };
  auto load = [&](Held& h, const Meta& m) {
    if (m.pos0 >= 0) {
      const int entry = __builtin_amdgcn_readfirstlane(m.entry[0]);
      const bool there = is_page(a.batch, a.cache.n_pages, m.pos0, entry);
      const int page = there ? entry : 0;
      const int64_t place = place_of(a.cache, page, g, m.pos0 & slot_mask);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        h.x[i] = *(const u32x4*)((is_value(i) ? a.cache.v : a.cache.k) + place + ((uint32_t)key_of(i) * tok_bytes + piece * 16));
      if constexpr (F8) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) h.scale[i] = (is_value(i) ? a.cache.v_scale : a.cache.k_scale)[block_of(a.cache, page, g)];
      }
#pragma unroll
      for (int n = 0; n < kMine; ++n) h.pos[n] = there ? m.pos0 + key_of(n) : INT32_MAX;
      h.whole = there;
      return;
    }
    h.whole = false;
    int64_t place[kMine];
    uint32_t block[kMine];
#pragma unroll
    for (int n = 0; n < kMine; ++n) {
      const bool there = is_page(a.batch, a.cache.n_pages, m.pos[n], m.entry[n]);
      const int page = there ? m.entry[n] : 0;
      h.pos[n] = there ? m.pos[n] : INT32_MAX;
      place[n] = place_of(a.cache, page, g, there ? m.pos[n] & slot_mask : 0) + piece * 16;
      block[n] = block_of(a.cache, page, g);
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      h.x[i] = *(const u32x4*)((is_value(i) ? a.cache.v : a.cache.k) + place[kMine == 1 ? 0 : i % kMine]);
      if constexpr (F8) h.scale[i] = (is_value(i) ? a.cache.v_scale : a.cache.k_scale)[block[kMine == 1 ? 0 : i % kMine]];
    }
  };
  // Values that are not there count as 0, whatever lies in their place and its scale: 0 times a NaN is one.  (Such keys' scores are masked.)
  auto without_unseen = [&](Held& h) __attribute__((always_inline)) {
    if (h.whole) return;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool there = h.pos[kMine == 1 ? 0 : i % kMine] != INT32_MAX;
#pragma unroll
      for (int w = 0; w < 4; ++w) h.x[i][w] = there ? h.x[i][w] : 0;
      if constexpr (F8) h.scale[i] = there ? h.scale[i] : 127;
    }
  };
  // Writing tile j is cut into kParts: 8-bit pages go four bytes of every 16 at a time, others a load at a time.
  constexpr int kParts = F8 ? 4 * kLoads : kLoads;
  u32x4 made[2];
  auto put = [&](const Held& h, int j, int part) __attribute__((always_inline)) {
    const int i = F8 ? part / 4 : part, e = part % 4;
    const bool values = is_value(i);
    const int n = kMine == 1 ? 0 : i % kMine, key = key_of(i);
    unsigned char* const to = (values ? v_stage[j & 3] + key * kValueStride : k_stage[j & 3] + key * kKeyStride) + piece * (F8 ? 32 : 16);
    if constexpr (F8) {
      const float by = scale_of(h.scale[i]);
      made[e / 2][e % 2 * 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(h.x[i][e], by, false));
      made[e / 2][e % 2 * 2 + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(h.x[i][e], by, true));
      if (e % 2) *(u32x4*)(to + e / 2 * 16) = made[e / 2];
    } else {
      *(u32x4*)to = h.x[i];
    }
    // (several threads write a key's position: the same one)
    if (part % (kParts / kLoads) == 0 && i < kMine) seen[j & 3][key] = h.pos[n];
  };

  constexpr int kSlots = kKS;                                   // of a step: as many instructions has each product
  static_assert(kSlots == 2 * kMD, "the products' instructions go in pairs");
  constexpr int kValues = 16 / kSlots;                          // probabilities of a slot
  constexpr int kTerms = terms_of(D);
  struct Probabilities {                                        // of 32 keys
    bf16x8 x[2][kTerms];
    // Sets a pair of them and adds it to the sum: the sum of what the second product sees (but for a second term's last bits).
    __device__ __forceinline__ void set(const Leaves& leaves, int v, float e0, float e1, float& sum) {
      const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
      if constexpr (kTerms > 1) sum += e0 + e1;
#pragma unroll
      for (int n = 0; n < kTerms; ++n) {
        const bf16x2 t = {(__bf16)e0, (__bf16)e1};
        x[v / 8][n][v % 8] = t[0];
        x[v / 8][n][v % 8 + 1] = t[1];
        if constexpr (kTerms == 1) sum = __builtin_amdgcn_fdot2_f32_bf16(t, ones, sum, false);
        e0 = leaves.lower(t, e0);
        e1 = leaves.upper(t, e1);
      }
    }
  };
  f32x16 o[kMD], x;
#pragma unroll
  for (int md = 0; md < kMD; ++md)
#pragma unroll
    for (int v = 0; v < 16; ++v) o[md][v] = 0.f;
  float m_run = kNoReference, l_run = 0.f;
  const Leaves leaves;
  Probabilities p;                                              // of the 32 keys before
#pragma unroll
  for (int v = 0; v < 16; v += 2) p.set(leaves, v, 0.f, 0.f, l_run);

  const int k_at = r * kKeyStride + hi * 16;
  auto key_part = [&](const unsigned char* from, int i) __attribute__((always_inline)) { return *(const u32x4*)(from + k_at + i * 32); };
  // Keys 16 kp + 8 upper + 4 hi + 0 .. 3 of dimension md * 32 + r: lane i of sixteen receives element i % 4 of the 8 bytes that lanes
  // 4 e + i / 4 address, which is dimension i of keys e = 0 .. 3.
  const int v_at = (4 * hi + ((lane & 15) >> 2)) * kValueStride + (((lane >> 4) & 1) * 16 + 4 * (lane & 3)) * 2;
  auto value_part = [&](unsigned char* from, int kp, int md, int upper) __attribute__((always_inline)) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(from + v_at + (16 * kp + 8 * upper) * kValueStride + md * 64));
  };
  auto joined = [](const i16x4& lo, const i16x4& up) __attribute__((always_inline)) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

  Held held;
  Meta next;
  Entries entries;
  {
    const Entries e0 = request_entries(first), e1 = request_entries(first + 1), e2 = request_entries(first + 2);
    entries = request_entries(first + 3);
    const Meta m0 = request_pages(first, e0), m1 = request_pages(first + 1, e1);
    next = request_pages(first + 2, e2);
    Held h0;
    load(h0, m0);
    load(held, m1);
    without_unseen(h0);
    without_unseen(held);
#pragma unroll
    for (int i = 0; i < kParts; ++i) put(h0, 0, i);
#pragma unroll
    for (int i = 0; i < kParts; ++i) put(held, 1, i);
    load(held, next);
    next = request_pages(first + 3, entries);
    entries = request_entries(first + 4);
    // the "32 keys before" of the first step: probabilities of 0 times values that are none
    for (int e = tid; e < 32 * kValueStride / 16; e += 64 * kWaves) *(u32x4*)(v_stage[3] + 32 * kValueStride + e * 16) = u32x4{0, 0, 0, 0};
  }
  // What the waves have written to LDS is there; the newest reads, which are behind the writes, and loads from memory stay on their way.
  auto meet = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(8)\n\ts_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  __syncthreads();
  x = zero;
#pragma unroll
  for (int i = 0; i < kKS; ++i)
    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, key_part(k_stage[0], i)), __builtin_bit_cast(bf16x8, qf[i]), x, 0, 0, 0);

  // Fragments are requested kAhead slots ahead, across the steps too.  Step (j, n), half n of tile j, multiplies keys 32 behind and values 32
  // in front of its own.
  constexpr int kAhead = 4;
  u32x4 kf[kAhead];
  i16x4 vf[kAhead][2];
  auto keys_from = [&](int j, int n) { return (const unsigned char*)k_stage[(j + n) & 3] + (1 - n) * 32 * kKeyStride; };
  auto values_from = [&](int j, int n) { return (unsigned char*)v_stage[(j - 1 + n) & 3] + (1 - n) * 32 * kValueStride; };
  auto request = [&](const unsigned char* k_from, unsigned char* v_from, int s) __attribute__((always_inline)) {
    kf[s % kAhead] = key_part(k_from, s);
    vf[s % kAhead][0] = value_part(v_from, s / kMD, s % kMD, 0);
    vf[s % kAhead][1] = value_part(v_from, s / kMD, s % kMD, 1);
  };
  int positions = seen[0][r];                                   // of the step's keys
#pragma unroll
  for (int s = 0; s < kAhead; ++s) request(keys_from(0, 0), values_from(0, 0), s);

  // Half `n` of tile j, whose scores are in x: leaves the next 32 keys' scores there, and the probabilities in p.
  auto step = [&](int j, auto half) __attribute__((always_inline)) {
    constexpr int n = decltype(half)::value;
    const unsigned char *const k_from = keys_from(j, n), *const k_after = keys_from(j + n, 1 - n);
    unsigned char *const v_from = values_from(j, n), *const v_after = values_from(j + n, 1 - n);
    if (n == 0) without_unseen(held);
    const bool masked = __ballot(positions > own_first);
    if (masked) {                                               // some key is not for all rows of the wave
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (seen[j & 3][n * 32 + 8 * (v / 4) + 4 * hi + v % 4] > own) x[v] = -INFINITY;
    }
    f32x16 x_next;
    Probabilities p_next;
    float sum[2] = {0.f, 0.f};
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const bf16x8 v_now = joined(vf[s % kAhead][0], vf[s % kAhead][1]);
      float e[kValues];
      x_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[s % kAhead]), __builtin_bit_cast(bf16x8, qf[s]), s ? x_next : zero, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < kValues; ++i) {
        const int v = s * kValues + i;
        if constexpr (CAP)
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(-2.f * f.cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[v] * f.scale)), f.cap - m_run));      // score_of(x) - m_run
        else
          e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[v], f.scale, -m_run));
        if (i & 1) p_next.set(leaves, v - 1, e[i - 1], e[i], sum[i / 2 & 1]);
      }
#pragma unroll
      for (int u = 0; u < kTerms; ++u) o[s % kMD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_now, p.x[s / kMD][u], o[s % kMD], 0, 0, 0);
      if (s + kAhead < kSlots)
        request(k_from, v_from, s + kAhead);
      else
        request(k_after, v_after, s + kAhead - kSlots);
      if (s == 0) positions = seen[(j + n) & 3][(1 - n) * 32 + r];
      if constexpr (n == 0) {
        if (kParts >= kSlots || s % (kSlots / kParts) == 0) {
#pragma unroll
          for (int i = 0; i < (kParts + kSlots - 1) / kSlots; ++i) put(held, j + 2, kParts >= kSlots ? s * (kParts / kSlots) + i : s * kParts / kSlots);
        }
      } else {
        if (s == 0) load(held, next);
        if (s == kSlots / 2) next = request_pages(first + j + 4, entries);
        if (s == kSlots - 1 && keys.n_sel) entries = request_entries(first + j + 5);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // The exponentials were taken against the reference as it stands.  Where a row's exceed it by far (and at first) it moves to its largest
    // logit and they are taken again; the sums so far, those of the 32 keys before among them, come to the new one.  (A capped -inf is none:
    // with masked keys capped scores are taken again too.)
    if ((CAP && masked) || __ballot(sum[0] + sum[1] > 256.f)) {
      float top = x[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) top = fmaxf(top, x[v]);
      top = halves_max(top);
      if (top != -INFINITY) top = score_of<bf16_t, CAP>(top, f.scale, f.cap);
      const float to = fmaxf(m_run, top), less = __builtin_amdgcn_exp2f(m_run - to);
      m_run = to;
      l_run *= less;
#pragma unroll
      for (int md = 0; md < kMD; ++md)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[md][v] *= less;
      sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int v = 0; v < 16; v += 2) {
        float e[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) e[u] = x[v + u] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(score_of<bf16_t, CAP>(x[v + u], f.scale, f.cap) - to);
        p_next.set(leaves, v, e[0], e[1], sum[0]);
      }
    }
    l_run += sum[0] + sum[1];
    x = x_next;
    p = p_next;
  };
  const int n_tiles = max(end - first, 0);
  for (int j = 0; j < n_tiles; ++j) {
    step(j, std::integral_constant<int, 0>{});
    step(j, std::integral_constant<int, 1>{});
    meet();
  }
  {
    unsigned char* const v_from = v_stage[(n_tiles - 1) & 3] + 32 * kValueStride;
#pragma unroll
    for (int s = 0; s < kSlots; ++s) {
      const bf16x8 v_now = joined(value_part(v_from, s / kMD, s % kMD, 0), value_part(v_from, s / kMD, s % kMD, 1));
#pragma unroll
      for (int u = 0; u < kTerms; ++u) o[s % kMD] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_now, p.x[s / kMD][u], o[s % kMD], 0, 0, 0);
    }
  }

  l_run = nan_if(holds_nan<bf16_t>(qf), halves_sum(l_run));
  if (!at.alone) {
    // as the lanes have it: 16 bytes a lane, 1 KB an instruction
    const int64_t part = (int64_t)at.slot * kWaves + wave;
#pragma unroll
    for (int md = 0; md < kMD; ++md)
#pragma unroll
      for (int v = 0; v < 16; v += 4)
        *((f32x4*)f.part_o + (part * (D / 8) + md * 4 + v / 4) * 64 + lane) = f32x4{o[md][v], o[md][v + 1], o[md][v + 2], o[md][v + 3]};
    if (hi == 0) *(float2*)(f.part_ml + (part * 32 + r) * 2) = make_float2(m_run, l_run);
  } else if (wave * 32 + r < rows) {
    const float inv = nothing_seen(l_run) ? 0.f : 1.f / l_run;
    char* to = a.out + (int64_t)(s.row0 + c) * a.ldo + (int64_t)head * kRowBytes;
#pragma unroll
    for (int md = 0; md < kMD; ++md)
#pragma unroll
      for (int v = 0; v < 16; v += 4) {
        const bf16x2 lo = __builtin_convertvector((f32x2{o[md][v] * inv, o[md][v + 1] * inv}), bf16x2);
        const bf16x2 up = __builtin_convertvector((f32x2{o[md][v + 2] * inv, o[md][v + 3] * inv}), bf16x2);
        *(uint2*)(to + (md * 32 + v * 2 + 4 * hi) * 2) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, up));
      }
    if (a.lse && hi == 0) a.lse[(int64_t)(s.row0 + c) * a.h + head] = nothing_seen(l_run) ? -INFINITY : lse_of<bf16_t>(m_run, l_run);
  }
  __syncthreads();                                              // (the next part's tiles go where this one's are)
  });
}

// Cut blocks joined: a workgroup takes 32 rows of a block as a wave has left them, its waves a quarter of the dimensions each.  A block's first
// part is the last thing that a share leaves, the others are the first that the shares behind it leave.
// Workgroups b and b + 8 n share an L2: what one of eight shares has left is read where it was written (33 MB in 9.7 us, 11.3 the other way round).
template <int D> __global__ __launch_bounds__(256) void join_many(ManyArgs f) {
  constexpr int kChunks = D / 8, kMine = kChunks / 4;           // 16 bytes a lane: of 32 rows, and of them a wave's
  constexpr int kGroups = kRows / 32;
  const AttendArgs& a = f.a;
  const int lane = threadIdx.x & 63, r = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = blockIdx.x / 8 % kGroups, unit = blockIdx.x / (8 * kGroups) * 8 + blockIdx.x % 8, h_kv = a.cache.h_kv, g = unit % h_kv;
  const int units = f.units;
  if (unit >= units) return;
  const bool second = f.records[2 * unit + 1].rows > 0;
  const int slot0 = 2 * unit + (second ? 1 : 0);
  const Record block = f.records[slot0];
  if (!block.begins || group * 32 >= block.rows) return;
  struct Partial {
    float2 ml;
    f32x4 x[kMine];
  };
  auto load = [&](int slot) {
    const int64_t part = (int64_t)slot * kGroups + group;
    Partial p;
    p.ml = *(const float2*)(f.part_ml + (part * 32 + r) * 2);
#pragma unroll
    for (int k = 0; k < kMine; ++k) p.x[k] = ((const f32x4*)f.part_o)[(part * kChunks + wave * kMine + k) * 64 + lane];
    return p;
  };
  Partial sum = load(slot0);
  constexpr int kAtOnce = 4;                                    // parts on their way together
  for (int u0 = unit + h_kv; u0 < units; u0 += 64 * h_kv) {     // shares behind this one, a lane to each
    const int u = u0 + lane * h_kv, slot = 2 * min(u, units - 1);
    const Record mine = f.records[slot];
    const bool same = u < units && mine.rows > 0 && mine.b == block.b && mine.row0 == block.row0 && !mine.begins;
    uint64_t there = __ballot(same);
    const bool done = __ballot(same && mine.ends) != 0;
    auto next = [&] {
      const int slot = 2 * (u0 + (__ffsll((unsigned long long)there) - 1) * h_kv);
      there &= there - 1;
      return slot;
    };
    while (there) {
      Partial p[kAtOnce];
      bool has[kAtOnce];
      float top = sum.ml.x;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        has[i] = there != 0;
        p[i] = load(has[i] ? next() : slot0);
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (has[i]) top = fmaxf(top, p[i].ml.x);
      const float less = __builtin_amdgcn_exp2f(sum.ml.x - top);
      sum.ml = make_float2(top, sum.ml.y * less);
#pragma unroll
      for (int k = 0; k < kMine; ++k) sum.x[k] *= less;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (!has[i]) break;
        const float by = __builtin_amdgcn_exp2f(p[i].ml.x - top);
        sum.ml.y = __builtin_fmaf(p[i].ml.y, by, sum.ml.y);
#pragma unroll
        for (int k = 0; k < kMine; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum.x[k][e] = __builtin_fmaf(p[i].x[k][e], by, sum.x[k][e]);
      }
    }
    if (done) break;
  }
  const int in = group * 32 + r, row = block.row0 + in;
  if (in >= block.rows) return;
  const float m = sum.ml.x, l = sum.ml.y;
  const int tok = block.tok0 + row / a.group, head = g * a.group + row % a.group;
  const float inv = nothing_seen(l) ? 0.f : 1.f / l;
  char* to = a.out + (int64_t)tok * a.ldo + (int64_t)head * D * 2;
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const bf16x2 lo = __builtin_convertvector((f32x2{sum.x[k][0] * inv, sum.x[k][1] * inv}), bf16x2), up = __builtin_convertvector((f32x2{sum.x[k][2] * inv, sum.x[k][3] * inv}), bf16x2);
    *(uint2*)(to + ((wave * kMine + k) * 8 + 4 * hi) * 2) = make_uint2(__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, up));
  }
  if (a.lse && wave == 0 && hi == 0) a.lse[(int64_t)tok * a.h + head] = nothing_seen(l) ? -INFINITY : lse_of<bf16_t>(m, l);
}


template <bool F8, int D> int launch(const ManyArgs& f, dim3 grid, hipStream_t st) {
  if (f.a.cap > 0.f)
    attend_many<F8, D, true><<<grid, 64 * kWaves, 0, st>>>(f);
  else
    attend_many<F8, D, false><<<grid, 64 * kWaves, 0, st>>>(f);
  ESA_LAUNCH_CHECK("attend_many");
  return ESA_OK;
}

}  // namespace

size_t many_workspace(int h_kv, int d) {
  const int64_t slots = 2 * (int64_t)grid_of(h_kv);
  return split_workspace(slots, kRows, d) + slots * sizeof(Record);
}

int launch_many(const AttendArgs& a, bool f8, int above, void* ws, hipStream_t st) {
  const ShareShape shape{above, std::max(kRows / a.group, 1), (kRows - 1) / a.group};
  const int64_t slots = 2 * (int64_t)grid_of(a.cache.h_kv);
  const SplitArgs<ShareShape> split = split_args<bf16_t>(a, shape, slots, ws);
  const ManyArgs f{split, (Record*)(split.part_ml + slots * kRows * 2), grid_of(a.cache.h_kv)};
  const dim3 grid((unsigned)f.units);
  int rc;
  if (a.cache.d == 64)
    rc = f8 ? launch<true, 64>(f, grid, st) : launch<false, 64>(f, grid, st);
  else
    rc = f8 ? launch<true, 128>(f, grid, st) : launch<false, 128>(f, grid, st);
  // (the longest sequence that the table has room for may be too short to be cut; a block weighs up to a block's tokens more than it sees)
  if (rc != ESA_OK || most_keys_of(a) + kRows <= shape.whole) return rc;
  const dim3 join((unsigned)((f.units + 7) / 8 * 8 * (kRows / 32)));
  if (a.cache.d == 64)
    join_many<64><<<join, 256, 0, st>>>(f);
  else
    join_many<128><<<join, 256, 0, st>>>(f);
  ESA_LAUNCH_CHECK("join_many");
  return ESA_OK;
}

}  // namespace paged
}  // namespace esa
