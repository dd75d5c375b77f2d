// What the matrix-core attention kernels of the paged cache share: arithmetic, arguments, and the kernel that joins slices.
#pragma once
#include <type_traits>

#include "plan.h"

namespace esa {
namespace paged {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Softmax in base 2 on the hardware's exponential for bf16, in base e and full precision for fp32.
template <typename T> __device__ __forceinline__ float exp_of(float x) { return sizeof(T) == 2 ? __builtin_amdgcn_exp2f(x) : expf(x); }
template <typename T> __device__ __forceinline__ float lse_of(float m, float l) { return sizeof(T) == 2 ? __builtin_fmaf(m, kLn2, logf(l)) : m + logf(l); }

__device__ __forceinline__ float halves_max(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float halves_sum(float v) {
  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}
__device__ __forceinline__ void wave_fence() {      // LDS operations of a wave are in order: only the compiler has to keep it
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct SlicedArgs {
  AttendArgs a;
  Shape shape;
  float* part_o;          // [slot][h_kv][shape.rows][D], relative to the slice's largest logit
  float* part_ml;         // [slot][h_kv][shape.rows][2]: the largest logit, the sum of exponentials
  float scale;            // bf16: includes log2(e); with a cap: 1 / cap
  float cap;              // bf16: includes log2(e)
};

// Scores as the softmax takes them.
template <typename T, bool CAP> __device__ __forceinline__ float score_of(float dot, float scale, float cap) {
  const float x = dot * scale;
  if constexpr (!CAP) return x;
  if constexpr (sizeof(T) == 4) return cap * tanhf(x);
  // tanh x = 1 - 2 / (1 + e^(2x)): some 2^-22 of the cap off where x is small, two roundings of a probability to 16 bits less than those
  const float e = __builtin_amdgcn_exp2f(x * (2.f * kLog2e));
  return __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + e), cap);
}

namespace {
// Slices of a row joined.  A wave takes a row, or (WIDE: rows of many slices) the four waves of a workgroup share one.  Only rows of
// sequences of several slices are gone through, by as many workgroups as the chip holds at most.
template <typename T, int D, bool WIDE> __global__ __launch_bounds__(256) void attend_join(SlicedArgs f) {
  constexpr int kMine = D / 64, kStep = WIDE ? 4 : 1;
  typedef __attribute__((ext_vector_type(kMine))) float vec;
  __shared__ vec sums[WIDE ? 4 : 1][64];
  __shared__ float2 ml[4];
  const AttendArgs& a = f.a;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Plan plan = plan_of(a, f.shape);
  for (int64_t u = WIDE ? blockIdx.x : blockIdx.x * 4 + wave;; u += WIDE ? gridDim.x : gridDim.x * 4) {
    const int g = (int)(u % a.cache.h_kv);
    const SplitRow at = split_row(a, f.shape, plan, u / a.cache.h_kv);
    if (at.b < 0) return;                                       // (of the whole workgroup if it shares the row)
    const Seq s = sequence(a.batch, at.b);
    const Keys keys = keys_of(a, s);
    const int n_rows = s.n * a.group, rows = f.shape.rows, block = at.row / rows, blocks = (n_rows + rows - 1) / rows;
    const int n_vis = keys_until(a, s, keys, min(block * rows + rows, n_rows) - 1), tiles = (n_vis + f.shape.keys - 1) / f.shape.keys;
    const int n = (tiles + plan.slice - 1) / plan.slice;
    if (n <= 1) continue;
    auto place = [&](int i) { return ((at.slot + block + (int64_t)i * blocks) * a.cache.h_kv + g) * rows + at.row - block * rows; };
    const int first = WIDE ? wave : 0;
    float m = -INFINITY, l = 0.f;
    vec sum = 0.f;
    for (int i0 = first; i0 < n; i0 += 64 * kStep) {            // a lane has the i0 + lane kStep-th slice's weight
      float mine = -INFINITY, part_l = 0.f;
      if (i0 + lane * kStep < n) {
        const float2 x = *(const float2*)(f.part_ml + place(i0 + lane * kStep) * 2);
        mine = x.x;
        part_l = x.y;
      }
      const float top = fmaxf(m, wave_max(mine)), ref = top == -INFINITY ? 0.f : top, less = exp_of<T>(m - ref);
      m = top;
      const float by = exp_of<T>(mine - ref);
      l = l * less + wave_sum(part_l * by);
      sum *= less;
      const int here = min((n - i0 + kStep - 1) / kStep, 64);
      for (int i = 0; i < here; i += 8) {
        vec x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = *(const vec*)(f.part_o + place(i0 + min(i + k, here - 1) * kStep) * D + lane * kMine);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k] * (i + k < here ? __shfl(by, min(i + k, 63)) : 0.f);
      }
    }
    if constexpr (WIDE) {
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
    }
    const int tok = s.row0 + at.row / a.group, head = g * a.group + at.row % a.group;
    T* out = (T*)(a.out + (int64_t)tok * a.ldo) + (int64_t)head * D + lane * kMine;
#pragma unroll
    for (int i = 0; i < kMine; ++i) store_f32<T>(out + i, l > 0.f ? sum[i] / l : 0.f);
    if (a.lse && lane == 0) a.lse[(int64_t)tok * a.h + head] = l > 0.f ? lse_of<T>(m, l) : -INFINITY;
  }
}
}  // namespace

// Arguments but for the shape's workspace; the slices' join, where the table has room for sequences of several.
template <typename T> static void set_sliced(SlicedArgs& f, const AttendArgs& a, const Shape& shape, void* ws) {
  f.a = a;
  f.shape = shape;
  f.part_o = (float*)ws;
  f.part_ml = f.part_o + most_parts(shape, a.cache.h_kv) * a.cache.h_kv * shape.rows * a.cache.d;
  const float base = sizeof(T) == 2 ? kLog2e : 1.f;
  f.scale = a.cap > 0.f ? a.scale / a.cap : a.scale * base;
  f.cap = a.cap * base;
}
static inline size_t sliced_workspace(const Shape& shape, int h_kv, int d) {
  return (size_t)(most_parts(shape, h_kv) * h_kv * shape.rows) * (d + 2) * sizeof(float);
}
template <typename T, bool WIDE> static int launch_join(const SlicedArgs& f, hipStream_t st) {
  const AttendArgs& a = f.a;
  if (((int64_t)a.batch.max_pages << a.batch.page_log2) + a.n_sel <= (int64_t)f.shape.least * f.shape.keys) return ESA_OK;
  const int64_t rows = a.batch.n_tok * (int64_t)a.h, groups = WIDE ? rows : (rows + 3) / 4;
  const dim3 join((unsigned)(groups < 2048 ? groups : 2048));
  if (a.cache.d == 64)
    attend_join<T, 64, WIDE><<<join, 256, 0, st>>>(f);
  else
    attend_join<T, 128, WIDE><<<join, 256, 0, st>>>(f);
  ESA_LAUNCH_CHECK("attend_join");
  return ESA_OK;
}

}  // namespace paged
}  // namespace esa
