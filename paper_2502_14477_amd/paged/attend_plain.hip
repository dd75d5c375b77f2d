// Attention over a paged cache, plainly: fp32 rows of 256 elements, which leave the matrix-core kernels neither registers nor LDS for a tile.
// A workgroup has one token and query head, its four waves 64 keys at a time each: a lane finds a key's row, then the wave takes the rows
// eight at a time, a lane to four dimensions.  Keys and values are read once for every query head and token, out of L2 in the main: that bounds
// chunks (512 tokens of 32 heads over 4608 keys 16 ms, 5.2 from 8-bit pages); one wave's path through its keys bounds single tokens (one over 32
// thousand keys 1.6 ms, sixteen over 8 thousand 1.2 ms or 1.7 TB/s, 0.57 from 8-bit pages).  (A thread to a key, for its whole row: 15 ms and 4.1.)
#include "paged.h"

namespace esa {
namespace paged {
namespace {

constexpr int kWaves = 4, kD = 256, kAtOnce = 8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

template <bool F8> __device__ __forceinline__ f32x4 four(const char* row, int lane) {
  if constexpr (!F8) return ((const f32x4*)row)[lane];
  float x[4];
  f8_unpack(((const uint32_t*)row)[lane], x);
  return f32x4{x[0], x[1], x[2], x[3]};
}

template <bool F8> __global__ __launch_bounds__(64 * kWaves) void attend_plain(AttendArgs a) {
  __shared__ f32x4 sums[kWaves][64];
  __shared__ float2 ml[kWaves];
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), block = block_index(), head = block % a.h, tok = block / a.h, g = head / a.group;
  const int b = sequence_with(a.batch, tok);
  if (b < 0) return;
  const Seq s = sequence(a.batch, b);
  const Keys keys = keys_of(a, s);
  const int own = s.t0 + tok - s.row0;
  const f32x4 q = ((const f32x4*)(a.q + tok * a.ldq))[head * (kD / 4) + lane];
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = wave * 64; j0 < keys.n; j0 += 64 * kWaves) {
    int64_t at = 0;
    float k_by = 1.f, v_by = 1.f;
    bool seen = false;
    if (j0 + lane < keys.n) {
      const int p = position(keys, j0 + lane, entry_of(a, keys, b, j0 + lane));
      const int page = p >= 0 && p <= own ? page_of(a.batch, a.cache.n_pages, b, p) : -1;
      seen = page >= 0;
      if (seen) {
        at = place_of(a.cache, page, g, p & ((1 << a.batch.page_log2) - 1));
        if (F8) {
          k_by = power_of(a.cache.k_scale[block_of(a.cache, page, g)]);
          v_by = power_of(a.cache.v_scale[block_of(a.cache, page, g)]);
        }
      }
    }
    const uint64_t all = __ballot(seen);
    for (int k0 = 0; k0 < 64; k0 += kAtOnce) {
      if (((all >> k0) & ((1u << kAtOnce) - 1)) == 0) continue;
      f32x4 k[kAtOnce], v[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {                       // (of a key that is not seen: row 0 of the pool, left out below)
        const int64_t row = lane_long(at, k0 + i);
        k[i] = four<F8>(a.cache.k + row, lane);
        v[i] = four<F8>(a.cache.v + row, lane);
      }
      float x[kAtOnce], top = m;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const float dot = wave_sum(__builtin_fmaf(k[i][0], q[0], __builtin_fmaf(k[i][1], q[1], __builtin_fmaf(k[i][2], q[2], k[i][3] * q[3]))));
        x[i] = dot * (F8 ? __shfl(k_by, k0 + i) : 1.f) * a.scale;
        if (a.cap > 0.f) x[i] = a.cap * tanhf(x[i] / a.cap);
        if (!((all >> (k0 + i)) & 1)) x[i] = -INFINITY;
        top = fmaxf(top, x[i]);
      }
      const float less = m == -INFINITY ? 0.f : expf(m - top);
      m = top;
      l *= less;
      o *= less;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (!((all >> (k0 + i)) & 1)) continue;                 // whatever its row holds
        const float p = expf(x[i] - top), by = F8 ? __shfl(v_by, k0 + i) : 1.f;      // (of the value: beside a small scale p would be subnormal)
        l += p;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(p, v[i][e] * by, o[e]);
      }
    }
  }
  sums[wave][lane] = o;
  if (lane == 0) ml[wave] = make_float2(m, l);
  __syncthreads();
  if (wave != 0) return;
  m = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
  l = 0.f;
  o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float by = ml[w].x == -INFINITY ? 0.f : expf(ml[w].x - m);
    l = __builtin_fmaf(ml[w].y, by, l);
    o += sums[w][lane] * by;
  }
  ((f32x4*)(a.out + tok * a.ldo))[head * (kD / 4) + lane] = nothing_seen(l) ? f32x4{0.f, 0.f, 0.f, 0.f} : o / l;
  if (a.lse && lane == 0) a.lse[(int64_t)tok * a.h + head] = nothing_seen(l) ? -INFINITY : m + logf(l);
}

}  // namespace

int launch_plain(const AttendArgs& a, bool f8, hipStream_t st) {
  const dim3 grid = grid_for((int64_t)a.batch.n_tok * a.h);
  if (f8)
    attend_plain<true><<<grid, 64 * kWaves, 0, st>>>(a);
  else
    attend_plain<false><<<grid, 64 * kWaves, 0, st>>>(a);
  ESA_LAUNCH_CHECK("attend_plain");
  return ESA_OK;
}

}  // namespace paged
}  // namespace esa
