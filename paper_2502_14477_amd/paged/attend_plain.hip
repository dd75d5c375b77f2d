// Attention over a paged cache, plainly: a workgroup has one token and query head and goes through the keys 256 at a time, a thread to a
// key for the logits, a thread to a dimension for the values.  Any head size, type and shape; reads keys and values once for every
// query head and token.
#include "paged.h"

namespace esa {
namespace paged {
namespace {

constexpr int kThreads = 256;

template <typename T, bool F8> __device__ __forceinline__ void load16_f32(const char* p, float (&x)[16]) {
  if constexpr (F8) {
    const u32x4 w = *(const u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float f[4];
      f8_unpack(w[i], f);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[4 * i + j] = f[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = load_f32<T>((const T*)p + i);
  }
}

__device__ __forceinline__ float block_max(float v, float* part) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
  __syncthreads();
  return v;
}
__device__ __forceinline__ float block_sum(float v, float* part) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = (part[0] + part[1]) + (part[2] + part[3]);
  __syncthreads();
  return v;
}

template <typename T, bool F8> __global__ __launch_bounds__(kThreads) void attend_plain(AttendArgs a) {
  __shared__ float q[256], part[4], weight[kThreads], sums[kThreads];
  __shared__ int64_t place[kThreads];
  const int tid = threadIdx.x, head = blockIdx.x % a.h, tok = blockIdx.x / a.h, d = a.cache.d, g = head / a.group;
  const int b = sequence_with(a.batch, tok);
  if (b < 0) return;
  const Seq s = sequence(a.batch, b);
  const Keys keys = keys_of(a, s);
  const int own = s.t0 + tok - s.row0;
  if (tid < d) q[tid] = load_f32<T>((const T*)(a.q + tok * a.ldq) + head * d + tid);
  __syncthreads();
  const int dim = tid % d, lane_group = tid / d, groups = kThreads / d;
  float m = -INFINITY, l = 0.f, o = 0.f;
  for (int j0 = 0; j0 < keys.n; j0 += kThreads) {
    float x = -INFINITY, by = 1.f;
    int64_t at = 0;
    if (j0 + tid < keys.n) {
      const int p = position(keys, j0 + tid, entry_of(a, keys, b, j0 + tid));
      const int page = p >= 0 && p <= own ? page_of(a.batch, a.cache.n_pages, b, p) : -1;
      if (page >= 0) {
        at = place_of(a.cache, page, g, p & ((1 << a.batch.page_log2) - 1));
        float dot = 0.f, k[16];
        for (int i = 0; i < d; i += 16) {
          load16_f32<T, F8>(a.cache.k + at + i * (F8 ? 1 : (int)sizeof(T)), k);
#pragma unroll
          for (int e = 0; e < 16; ++e) dot = __builtin_fmaf(q[i + e], k[e], dot);
        }
        if (F8) {
          dot *= scale_of(a.cache.k_scale[block_of(a.cache, page, g)]);
          by = scale_of(a.cache.v_scale[block_of(a.cache, page, g)]);
        }
        x = dot * a.scale;
        if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
      }
    }
    const float top = fmaxf(m, block_max(x, part));
    if (top == -INFINITY) continue;
    const float w = x == -INFINITY ? 0.f : expf(x - top), less = m == -INFINITY ? 0.f : expf(m - top);
    l = l * less + block_sum(w, part);
    m = top;
    weight[tid] = w == 0.f ? 0.f : w * by;
    place[tid] = at;
    __syncthreads();
    o *= less;
    for (int j = lane_group; j < min(kThreads, keys.n - j0); j += groups) {
      const float p = weight[j];
      if (p == 0.f) continue;
      const char* v = a.cache.v + place[j];
      float x1;
      if constexpr (F8)
        x1 = __builtin_amdgcn_cvt_f32_fp8((int)(uint8_t)v[dim], 0);
      else
        x1 = load_f32<T>((const T*)v + dim);
      o = __builtin_fmaf(p, x1, o);
    }
    __syncthreads();
  }
  sums[tid] = o;
  __syncthreads();
  if (tid < d) {
    for (int i = 1; i < groups; ++i) o += sums[tid + i * d];
    store_f32<T>((T*)(a.out + tok * a.ldo) + head * d + tid, l > 0.f ? o / l : 0.f);
    if (a.lse && tid == 0) a.lse[(int64_t)tok * a.h + head] = l > 0.f ? m + logf(l) : -INFINITY;
  }
}

}  // namespace

int launch_plain(const AttendArgs& a, bool f8, int dtype, hipStream_t st) {
  const dim3 grid((unsigned)(a.batch.n_tok * a.h));
  if (dtype == ESA_BF16) {
    if (f8)
      attend_plain<bf16_t, true><<<grid, kThreads, 0, st>>>(a);
    else
      attend_plain<bf16_t, false><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (f8)
      attend_plain<float, true><<<grid, kThreads, 0, st>>>(a);
    else
      attend_plain<float, false><<<grid, kThreads, 0, st>>>(a);
  }
  ESA_LAUNCH_CHECK("attend_plain");
  return ESA_OK;
}

}  // namespace paged
}  // namespace esa
