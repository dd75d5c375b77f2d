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
constexpr int kWaves = kThreads / 64;
constexpr int kEach = 16;                     // numbers of a chunk a thread
constexpr int kChunk = kThreads * kEach;

// Negative numbers, NaN (the maximum's other operand is taken) and infinities count as 0.
template <typename T> __device__ __forceinline__ float probability(T v);
template <> __device__ __forceinline__ float probability<float>(float v) {
  v = fmaxf(v, 0.f);
  return v < __builtin_huge_valf() ? v : 0.f;
}
template <> __device__ __forceinline__ float probability<bf16_t>(bf16_t v) { return probability<float>(bf16_to_f32(v)); }

// N numbers of a row, wherever it begins.
template <typename T, int N> struct Piece {
  T x[N];
};
template <typename T, int N> __device__ __forceinline__ Piece<T, N> load(const T* p) {
  Piece<T, N> v;
  __builtin_memcpy(&v, p, sizeof(v));
  return v;
}
// The largest pieces of a row of that many.
template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);

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

// Weights of M pieces of N tokens, `step` apart from `first` on: take(number, token, weight); those beyond the vocabulary are 0.  A piece
// that would reach over a row's end is read as the row's last N numbers, of which those that belong to other pieces do not count (the vocabulary has N or
// more).  All are requested in front of their first use.
template <typename T, int N, int M, typename F>
__device__ __forceinline__ void weights(const VerifyArgs& a, const Drawn& d, int64_t first, int step, F&& take) {
  const T* pr = (const T*)(a.target + (int64_t)d.row * a.ldt);
  const int64_t end = (int64_t)a.vocab - N;
  auto all = [&](auto&& of) {
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const int64_t want = first + m * step, at = min(want, end);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const double w = of(m, j, (int)at + j);
        take(m * N + j, (int)at + j, at + j >= want ? w : 0.0);
      }
    }
  };
  Piece<T, N> p[M];
#pragma unroll
  for (int m = 0; m < M; ++m) p[m] = load<T, N>(pr + min(first + m * step, end));
  if (d.mode == 1) {
    const T* qr = (const T*)(a.draft + (int64_t)(d.row + 1) * a.ldd);
    Piece<T, N> q[M];
#pragma unroll
    for (int m = 0; m < M; ++m) q[m] = load<T, N>(qr + min(first + m * step, end));
    all([&](int m, int j, int) { return fmax((double)probability<T>(p[m].x[j]) - (double)probability<T>(q[m].x[j]), 0.0); });
  } else {
    const int without = d.mode == 2 ? d.token : -1;      // the token that was looked up, with a probability of 1
    all([&](int m, int j, int t) {
      const double x = probability<T>(p[m].x[j]);
      return t == without ? fmax(x - 1.0, 0.0) : x;
    });
  }
}

struct Work {
  double* sums;      // [n_seq][chunks]
  int32_t* kept;     // [n_seq]
};
__host__ __device__ inline int chunks_of(int vocab) { return (int)(((int64_t)vocab + kChunk - 1) / kChunk); }
__host__ __device__ inline Work work_at(void* ws, int n_seq, int vocab) {
  double* sums = (double*)ws;
  return Work{sums, (int32_t*)(sums + (size_t)n_seq * chunks_of(vocab))};
}

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
// Of the workgroup, in every thread.
__device__ __forceinline__ double group_sum(double v, double* part) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) v += part[i];
  return v;
}

// grid (chunks, sequences)
template <typename T, int N> __global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a) {
  __shared__ double part[kWaves];
  const int tid = threadIdx.x, chunk = blockIdx.x;
  const Work k = work_at(a.ws, a.n_seq, a.vocab);
  for (int b = blockIdx.y; b < a.n_seq; b += gridDim.y) {
    const Rows s = rows_of(a, b);
    if (s.n == 0) continue;
    const int kept = standing<T>(a, s);
    const Drawn d = drawn_of(a, s, kept);
    double w = 0.0;
    weights<T, N, kEach / N>(a, d, (int64_t)chunk * kChunk + tid * N, kThreads * N, [&](int, int, double x) { w += x; });
    w = group_sum(w, part);
    if (tid == 0) {
      k.sums[(int64_t)b * gridDim.x + chunk] = w;
      if (chunk == 0) k.kept[b] = kept;
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
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = all;
    all += part[w];
  }
  return Scanned{before + (lane ? left : 0.0), all};
}

// The first item of which a thread says so (the threads' items ascend), and the last one with any weight: INT32_MAX, -1 where there is none.
struct Found {
  int first, last;
};
__device__ __forceinline__ Found find(int first, int last, Found* part) {
  const int wave = threadIdx.x >> 6;
  const uint64_t f = __ballot(first != INT32_MAX), l = __ballot(last >= 0);
  const Found mine = {f ? __shfl(first, __ffsll((unsigned long long)f) - 1) : INT32_MAX, l ? __shfl(last, 63 - __clzll((long long)l)) : -1};
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[wave] = mine;
  __syncthreads();
  Found r = {INT32_MAX, -1};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    r.first = min(r.first, part[w].first);
    r.last = max(r.last, part[w].last);
  }
  return r;
}

// A workgroup a sequence.
template <typename T, int N> __global__ __launch_bounds__(kThreads) void verify_draw(VerifyArgs a) {
  __shared__ double part[kWaves];
  __shared__ Found found[kWaves];
  __shared__ double at_chunk;
  const int tid = threadIdx.x, b = paged::block_index();
  if (b >= a.n_seq) return;
  const Rows s = rows_of(a, b);
  if (s.n == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }
  const Work k = work_at(a.ws, a.n_seq, a.vocab);
  const int kept = k.kept[b], chunks = chunks_of(a.vocab);
  const double* sums = k.sums + (int64_t)b * chunks;
  double mine = sums[min(tid, chunks - 1)];      // of the chunk that the thread's number is, in the first round of them
  mine = tid < chunks ? mine : 0.0;
  const float u = a.u[s.row0];
  Drawn d = drawn_of(a, s, kept);
  for (int i = tid; i < s.n; i += kThreads)
    if (i != kept) a.out[s.row0 + i] = i < kept ? a.tokens[s.row0 + i + 1] : -1;
  if (tid == 0) a.count[b] = kept + 1;
  // sums in front of the thread's chunk
  Scanned y = scan(mine, part);
  double total = y.all;
  for (int c = tid + kThreads; c - tid < chunks; c += kThreads) total += group_sum(c < chunks ? sums[c] : 0.0, part);
  bool again = false;                            // whether the chunks' sums are those of p
  if (!(total > 0.0)) {
    if (d.mode == 0) {
      if (tid == 0) a.out[d.row] = -1;
      return;
    }
    // p itself, of which there are no sums yet: one workgroup reads it all
    d.mode = 0;
    again = true;
    for (int c = 0; c < chunks; ++c) {
      double w = 0.0;
      weights<T, N, kEach / N>(a, d, (int64_t)c * kChunk + tid * N, kThreads * N, [&](int, int, double x) { w += x; });
      w = group_sum(w, part);
      if (tid == 0) k.sums[(int64_t)b * chunks + c] = w;
      total += w;
    }
    if (!(total > 0.0)) {
      if (tid == 0) a.out[d.row] = -1;
      return;
    }
    __syncthreads();
  }
  const double target = u >= 1.f ? __builtin_huge_val() : u > 0.f ? u * total : 0.0;
  // the first chunk whose sums pass it, or else the last with any
  int chunk = -1;
  double base = 0.0;
  for (int c0 = 0; c0 < chunks; c0 += kThreads) {
    const int c = c0 + tid;
    if (c0 > 0 || again) {
      mine = c < chunks ? sums[c] : 0.0;
      y = scan(mine, part);
    }
    const double before = base + y.before;
    const Found f = find(mine > 0.0 && before + mine > target ? c : INT32_MAX, mine > 0.0 ? c : -1, found);
    if (f.first != INT32_MAX) chunk = f.first;
    else if (f.last >= 0) chunk = f.last;
    if (chunk == c) at_chunk = before;
    if (f.first != INT32_MAX) break;
    base += y.all;
  }
  __syncthreads();
  double x[kEach], sum = 0.0;
  int t[kEach];
  weights<T, N, kEach / N>(a, d, (int64_t)chunk * kChunk + tid * kEach, N, [&](int j, int at, double w) {
    x[j] = w;
    t[j] = at;
    sum += w;
  });
  const double start = at_chunk;
  sum = start + scan(sum, part).before;
  int first = INT32_MAX, last = -1;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    sum += x[j];
    if (x[j] > 0.0) {
      last = t[j];
      if (sum > target && first == INT32_MAX) first = t[j];
    }
  }
  const Found f = find(first, last, found);
  if (tid == 0) a.out[d.row] = f.first != INT32_MAX ? f.first : f.last;
}

template <typename T, int N> int launch_of(const VerifyArgs& a, hipStream_t st) {
  verify_sums<T, N><<<dim3((unsigned)chunks_of(a.vocab), (unsigned)(a.n_seq < 65535 ? a.n_seq : 65535)), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_sums");
  verify_draw<T, N><<<paged::grid_for(a.n_seq), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_draw");
  return ESA_OK;
}

}  // namespace

size_t verify_workspace(int n_seq, int vocab) {
  return align_up((size_t)n_seq * (chunks_of(vocab) * sizeof(double) + sizeof(int32_t)), 256);
}

// Vocabularies shorter than a piece are read number by number.
int launch_verify(const VerifyArgs& a, int dtype, hipStream_t st) {
  if (dtype == ESA_F32) return a.vocab >= kPiece<float> ? launch_of<float, kPiece<float>>(a, st) : launch_of<float, 1>(a, st);
  return a.vocab >= kPiece<bf16_t> ? launch_of<bf16_t, kPiece<bf16_t>>(a, st) : launch_of<bf16_t, 1>(a, st);
}

}  // namespace serve
}  // namespace esa
