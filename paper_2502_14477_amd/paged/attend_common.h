// What the matrix-core attention kernels of the paged cache share: arithmetic and arguments.
#pragma once
#include <type_traits>

#include "paged.h"

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

// Whether a lane's row of queries, of which it and its opposite have 16 bytes in turn, holds a NaN.  By their bits: the kernels are compiled without
// heed of NaN, and comparisons, maxima and selections may take one for anything.  The row's sum of exponentials is made NaN at its end, which the
// arithmetic behind it passes on.
template <typename T, int N> __device__ __forceinline__ bool holds_nan(const u32x4 (&q)[N]) {
  constexpr uint32_t kMagnitude = sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu, kToSign = sizeof(T) == 2 ? 0x007F007Fu : 0x007FFFFFu;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) any |= (q[i][w] & kMagnitude) + kToSign;      // past infinity: over into the sign
  const auto both = __builtin_amdgcn_permlane32_swap(any, any, false, false);
  return ((both[0] | both[1]) & ~kMagnitude) != 0;
}
__device__ __forceinline__ float nan_if(bool is, float x) {
  uint32_t bits = is ? 0x7FC00000u : __float_as_uint(x);
  asm("" : "+v"(bits));                     // (a NaN that the compiler sees it leaves out)
  return __uint_as_float(bits);
}

constexpr float kNoReference = -1e30f;      // of a softmax that has seen nothing: so low that the first logit exceeds it

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

// Arguments of a kernel whose blocks' keys are shared among workgroups as SHAPE says.
template <typename SHAPE> struct SplitArgs {
  AttendArgs a;
  SHAPE shape;
  float* part_o;          // [slot][shape.rows * D] (in a kernel's own order), relative to the part's reference
  float* part_ml;         // [slot][shape.rows][2]: the reference, the sum of exponentials
  float scale;            // bf16: includes log2(e); with a cap: 1 / cap, and bf16: 2 log2(e)
  float cap;              // bf16: includes log2(e)
};

// Scores as the softmax takes them.
template <typename T, bool CAP> __device__ __forceinline__ float score_of(float dot, float scale, float cap) {
  const float x = dot * scale;
  if constexpr (!CAP) return x;
  if constexpr (sizeof(T) == 4) return cap * tanhf(x);
  // tanh x = 1 - 2 / (1 + e^(2x)): some 2^-22 of the cap off where x is small, two roundings of a probability to 16 bits less than those
  return __builtin_fmaf(-2.f * cap, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x)), cap);
}

// slots: partial results that the workspace has room for.
template <typename T, typename SHAPE> static SplitArgs<SHAPE> split_args(const AttendArgs& a, const SHAPE& shape, int64_t slots, void* ws) {
  const float base = sizeof(T) == 2 ? kLog2e : 1.f;
  SplitArgs<SHAPE> f;
  f.a = a;
  f.shape = shape;
  f.part_o = (float*)ws;
  f.part_ml = f.part_o + slots * shape.rows * a.cache.d;
  f.scale = a.cap > 0.f ? a.scale / a.cap * (sizeof(T) == 2 ? 2.f * kLog2e : 1.f) : a.scale * base;
  f.cap = a.cap * base;
  return f;
}
static inline size_t split_workspace(int64_t slots, int rows, int d) { return (size_t)slots * rows * (d + 2) * sizeof(float); }

}  // namespace paged
}  // namespace esa
