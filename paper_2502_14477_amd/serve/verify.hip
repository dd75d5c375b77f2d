// Verification of drafted tokens against the target's probabilities, from given random numbers (esa_verify_drafts).
//
// Row i of a sequence stands while u_i q_i(x_i) < p_{i-1}(x_i): two numbers a draft.  What has to be read is one row of the target and
// one of the draft a sequence, behind the last row that stands: the token is drawn from w = max(p - q, 0) by the sums of w up to each
// token.  Everything is fp64 (a product of two fp32 numbers is exact in it, a row's sum of a hundred thousand probabilities is off by 1e-16 or so), so the
// outcome is that of the definition but for random numbers that lie within 1e-15 of a border.
//
// A row is cut into chunks, a workgroup to each, which finds its sequence's last standing row by itself and leaves the chunk's sums of w and of p;
// then a workgroup a sequence finds the chunk in which the sums pass the drawn number, and in it the token.
#include "serve.h"

namespace esa {
namespace serve {
namespace {

constexpr int kThreads = 256;
constexpr int kEach = 16;                     // numbers of a chunk a thread
constexpr int kChunk = kThreads * kEach;

template <typename T> __device__ __forceinline__ double probability(T v);
template <> __device__ __forceinline__ double probability<float>(float v) { return v > 0.f && v < __builtin_huge_valf() ? (double)v : 0.0; }
template <> __device__ __forceinline__ double probability<bf16_t>(bf16_t v) { return probability<float>(bf16_to_f32(v)); }

// A sequence's rows, clamped.
struct Rows {
  int row0, n;
};
__device__ __forceinline__ Rows rows_of(const VerifyArgs& a, int b) {
  const int lo = min(max(a.cu[b], 0), a.n_tok), hi = min(max(a.cu[b + 1], lo), a.n_tok);
  return Rows{lo, hi - lo};
}

// Drafts that stand, of a sequence with n >= 1 rows.  The whole wave takes part, a lane to a draft.
template <typename T> __device__ int standing(const VerifyArgs& a, const Rows& s) {
  const int lane = threadIdx.x & 63;
  for (int i0 = 1; i0 < s.n; i0 += 64) {
    const int i = i0 + lane;
    const int64_t row = s.row0 + min(i, s.n - 1);
    const int x = a.tokens[row];
    const float u = a.u[row];
    const bool token = (uint32_t)x < (uint32_t)a.vocab;
    const int at = token ? x : 0;
    const double p = probability<T>(((const T*)(a.target + (row - 1) * a.ldt))[at]);
    const double q = a.draft ? probability<T>(((const T*)(a.draft + row * a.ldd))[at]) : 1.0;
    const uint64_t down = __ballot(i < s.n && !(token && (double)u * q < p));
    if (down) return i0 - 1 + __ffsll((unsigned long long)down) - 1;
  }
  return s.n - 1;
}

// What a sequence draws from.
struct Drawn {
  int row, mode;      // of the target; 0: p, 1: p - q with the draft's next row, 2: p without the token of the next row
  int token;
};
__device__ __forceinline__ Drawn drawn_of(const VerifyArgs& a, const Rows& s, int kept) {
  const bool all = kept == s.n - 1;
  return Drawn{s.row0 + kept, all ? 0 : a.draft ? 1 : 2, all ? -1 : a.tokens[s.row0 + kept + 1]};
}

// Weight of token t, and the target's probability of it.
template <typename T> struct Weight {
  double w, p;
};
template <typename T> __device__ __forceinline__ Weight<T> weight(const Drawn& d, T pv, T qv, int t) {
  const double p = probability<T>(pv);
  if (d.mode == 1) return {fmax(p - probability<T>(qv), 0.0), p};
  return {d.mode == 2 && t == d.token ? fmax(p - 1.0, 0.0) : p, p};
}

struct Work {
  double* sums;      // [n_seq][chunks][2]: of w, of p
  int32_t* kept;     // [n_seq]
};
__host__ __device__ inline int chunks_of(int vocab) { return (int)(((int64_t)vocab + kChunk - 1) / kChunk); }
__host__ __device__ inline Work work_at(void* ws, int n_seq, int vocab) {
  double* sums = (double*)ws;
  return Work{sums, (int32_t*)(sums + (size_t)n_seq * chunks_of(vocab) * 2)};
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// grid (chunks, sequences)
template <typename T> __global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a) {
  __shared__ double part[kThreads / 64][2];
  const int tid = threadIdx.x, chunk = blockIdx.x;
  for (int b = blockIdx.y; b < a.n_seq; b += gridDim.y) {
    const Rows s = rows_of(a, b);
    const Work k = work_at(a.ws, a.n_seq, a.vocab);
    if (s.n == 0) continue;
    const int kept = standing<T>(a, s);
    const Drawn d = drawn_of(a, s, kept);
    if (chunk == 0 && tid == 0) k.kept[b] = kept;
    const T* p = (const T*)(a.target + (int64_t)d.row * a.ldt);
    const T* q = d.mode == 1 ? (const T*)(a.draft + (int64_t)(d.row + 1) * a.ldd) : p;
    double w = 0.0, all = 0.0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      const int64_t t = (int64_t)chunk * kChunk + j * kThreads + tid;
      if (t < a.vocab) {
        const Weight<T> x = weight<T>(d, p[t], q[t], (int)t);
        w += x.w;
        all += x.p;
      }
    }
    w = wave_sum(w);
    all = wave_sum(all);
    __syncthreads();
    if ((tid & 63) == 0) {
      part[tid >> 6][0] = w;
      part[tid >> 6][1] = all;
    }
    __syncthreads();
    if (tid < 2) {
      double v = 0.0;
#pragma unroll
      for (int i = 0; i < kThreads / 64; ++i) v += part[i][tid];
      k.sums[((int64_t)b * gridDim.x + chunk) * 2 + tid] = v;
    }
  }
}

// Sums over the workgroup in front of each thread, and of all.
struct Scanned {
  double before, all;
};
__device__ __forceinline__ Scanned scan(double x, double* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const double v = __shfl_up(x, m);
    x += lane >= m ? v : 0.0;
  }
  const double left = __shfl_up(x, 1);
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  double all = 0.0, before = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w == wave) before = all;
    all += part[w];
  }
  return Scanned{before + (lane ? left : 0.0), all};
}

// A workgroup a sequence.
template <typename T> __global__ __launch_bounds__(kThreads) void verify_draw(VerifyArgs a) {
  __shared__ double part[kThreads / 64];
  __shared__ int found, last;
  __shared__ double before;
  const int tid = threadIdx.x, b = blockIdx.x;
  const Rows s = rows_of(a, b);
  if (s.n == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }
  const Work k = work_at(a.ws, a.n_seq, a.vocab);
  const int kept = k.kept[b], chunks = chunks_of(a.vocab);
  Drawn d = drawn_of(a, s, kept);
  for (int i = tid; i < s.n; i += kThreads)
    if (i != kept) a.out[s.row0 + i] = i < kept ? a.tokens[s.row0 + i + 1] : -1;
  if (tid == 0) a.count[b] = kept + 1;
  const float u = a.u[s.row0];
  const double* sums = k.sums + (int64_t)b * chunks * 2;
  // the sum of all, of w or else of p
  double w = 0.0, p = 0.0;
  for (int c = tid; c < chunks; c += kThreads) {
    w += sums[2 * c];
    p += sums[2 * c + 1];
  }
  double total = scan(w, part).all;
  int which = 0;
  if (!(total > 0.0)) {
    total = scan(p, part).all;
    which = 1;
    d.mode = 0;
  }
  if (!(total > 0.0)) {
    if (tid == 0) a.out[d.row] = -1;
    return;
  }
  const double target = u >= 1.f ? __builtin_huge_val() : u > 0.f ? u * total : 0.0;
  // the first chunk whose sums pass it, or the last with any
  if (tid == 0) {
    found = INT32_MAX;
    last = -1;
    before = 0.0;
  }
  double base = 0.0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + tid;
    const double x = c < chunks ? sums[2 * c + which] : 0.0;
    const Scanned y = scan(x, part);
    if (x > 0.0) {
      atomicMax(&last, c);
      if (base + y.before + x > target) atomicMin(&found, c);
    }
    __syncthreads();
    if (found == c || (found == INT32_MAX && last == c)) before = base + y.before;
    __syncthreads();
    if (found != INT32_MAX) break;
    base += y.all;
  }
  const int chunk = found != INT32_MAX ? found : last;
  const double start = before;
  __syncthreads();
  if (tid == 0) {
    found = INT32_MAX;
    last = -1;
  }
  const T* pr = (const T*)(a.target + (int64_t)d.row * a.ldt);
  const T* qr = d.mode == 1 ? (const T*)(a.draft + (int64_t)(d.row + 1) * a.ldd) : pr;
  double x[kEach], mine = 0.0;
  const int64_t t0 = (int64_t)chunk * kChunk + tid * kEach;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    x[j] = t0 + j < a.vocab ? weight<T>(d, pr[t0 + j], qr[t0 + j], (int)(t0 + j)).w : 0.0;
    mine += x[j];
  }
  double sum = start + scan(mine, part).before;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    sum += x[j];
    if (x[j] > 0.0) {
      atomicMax(&last, (int)(t0 + j));
      if (sum > target) atomicMin(&found, (int)(t0 + j));
    }
  }
  __syncthreads();
  if (tid == 0) a.out[d.row] = found != INT32_MAX ? found : last;
}

template <typename T> int launch_of(const VerifyArgs& a, hipStream_t st) {
  verify_sums<T><<<dim3((unsigned)chunks_of(a.vocab), (unsigned)(a.n_seq < 65535 ? a.n_seq : 65535)), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_sums");
  verify_draw<T><<<dim3((unsigned)a.n_seq), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_draw");
  return ESA_OK;
}

}  // namespace

size_t verify_workspace(int n_seq, int vocab) {
  return align_up((size_t)n_seq * (chunks_of(vocab) * 2 * sizeof(double) + sizeof(int32_t)), 256);
}

int launch_verify(const VerifyArgs& a, int dtype, hipStream_t st) { return dtype == ESA_F32 ? launch_of<float>(a, st) : launch_of<bf16_t>(a, st); }

}  // namespace serve
}  // namespace esa
