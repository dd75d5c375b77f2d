// Rotary encoding of queries and keys at positions that lie on the device (esa_rope_at).
//
// Pair j of a token at position p turns by a = p freq[j] in every head: x' = g (x cos a - y sin a), y' = g (y cos a + x sin a).  Angles,
// their sines and cosines and the products are fp64 with one rounding into the storage type, as esa_rope's are, by a shorter evaluation of the same
// precision.
//
// It is a copy with arithmetic, and runs as one: 19787 tokens of 32 and 8 heads of 128 bf16 elements 72 us, 406 MB at 5.65 TB/s, where a copy moves 5.4.
// A workgroup takes a token (or a few) with all its heads, which share the sines and cosines by way of LDS; a thread turns one piece of 16 bytes of
// either half, requested in front of the sines.  Four heads to a thread, as many fewer waves, were slower below 16 thousand tokens (1024: 7.3 us
// for 5.8, sixteen 4.6 for 2.9 in a graph); pieces of 8 bytes are quicker for sixteen tokens (2.7), the same for 250, and slower from 500 on (1024: 7.2,
// 16384: 100 for 64).  As it is 16, 250, 1024 and 16384 tokens take 2.9, 3.6, 6.0 and 52 us.  The frequencies lie on the device: as 1 KB of arguments they cost the host 0.5 to 1.2 us a launch.
#include <type_traits>

#include "serve.h"

namespace esa {
namespace serve {
namespace {

typedef __attribute__((ext_vector_type(2))) double f64x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256, kMostThreads = 512;      // of a workgroup: about the former where a token's heads take no more, else up to the latter

// Cosine and sine of an angle below 2^38 in magnitude.  Reduced to [-pi/4, pi/4] by a multiple of pi/2 that is held in two parts
// (the first product is exact in the fma, the second's error is 2^38 2^-107), then the Taylor series: x^17/17! is below 5e-17 of the sine, x^18/18!
// below 3e-18.
__device__ __forceinline__ f64x2 turn_of(double angle) {
  constexpr double kTwoOverPi = 0.63661977236758134308, kPio2 = 1.5707963267948965580, kPio2Low = 6.1232339957367660359e-17;
  const double k = __builtin_rint(angle * kTwoOverPi);
  const double x = __builtin_fma(-k, kPio2Low, __builtin_fma(-k, kPio2, angle)), z = x * x;
  double s = -1.0 / 1307674368000.0;      // 15!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, x, x);
  double c = 1.0 / 20922789888000.0;      // 16!
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int quarter = (int)(k - 4.0 * __builtin_floor(k * 0.25));
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return f64x2{quarter == 1 || quarter == 2 ? -a : a, quarter >= 2 ? -b : b};
}

template <typename T> __device__ __forceinline__ double to_f64(T v);
template <> __device__ __forceinline__ double to_f64<float>(float v) { return (double)v; }
template <> __device__ __forceinline__ double to_f64<bf16_t>(bf16_t v) { return (double)bf16_to_f32(v); }

// Rounded into storage, N at a time.
template <int N> __device__ __forceinline__ void to_storage(const double (&v)[N], float (&o)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = (float)v[i];
}
template <int N> __device__ __forceinline__ void to_storage(const double (&v)[N], bf16_t (&o)[N]) {
  float f[N];
  narrow_for_bf16(v, f);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const uint32_t w = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[i], f[i + 1]}), bf16x2));
    o[i] = (bf16_t)w;
    o[i + 1] = (bf16_t)(w >> 16);
  }
}

template <typename T, int N> struct alignas(N * sizeof(T)) Piece {
  T x[N];
};

// Where head hh of all sets' lies.
struct Place {
  const char* x;
  char* out;
};
__device__ __forceinline__ Place place_of(const RopeArgs& a, int64_t tok, int hh) {
  const RowSet &f = a.set[0], &g = a.set[1];
  const bool second = hh >= f.heads;
  const int64_t h = second ? hh - f.heads : hh;
  return Place{(second ? g.x : f.x) + tok * (second ? g.x_tok : f.x_tok) + h * (second ? g.x_head : f.x_head),
               (second ? g.out : f.out) + tok * (second ? g.out_tok : f.out_tok) + h * (second ? g.out_head : f.out_head)};
}

// What a thread takes of a head at a time: N pairs, which are two pieces of N elements, one in each half or one behind the other.  N = 1 takes
// elements one by one, whatever their alignment.  Behind the pairs' come two pieces at a time of what does not turn.
template <typename T, int N, bool HALVES, bool STREAM> struct Pieces {
  Piece<T, N> a, b;
  __device__ __forceinline__ void load(const char* p, int at, int gap) {
    a = *(const Piece<T, N>*)(p + at);
    b = *(const Piece<T, N>*)(p + at + gap);
  }
  __device__ __forceinline__ void store(char* p, int at, int gap) const {
    if constexpr (STREAM) {
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, a), (u32x4*)(p + at));
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, b), (u32x4*)(p + at + gap));
    } else {
      *(Piece<T, N>*)(p + at) = a;
      *(Piece<T, N>*)(p + at + gap) = b;
    }
  }
  __device__ __forceinline__ T& x(int j) {
    if constexpr (HALVES || N == 1) return a.x[j];
    return j < N / 2 ? a.x[2 * j] : b.x[2 * j - N];
  }
  __device__ __forceinline__ T& y(int j) {
    if constexpr (HALVES || N == 1) return b.x[j];
    return j < N / 2 ? a.x[2 * j + 1] : b.x[2 * j + 1 - N];
  }
  __device__ __forceinline__ void turn(const f64x2 (&cs)[N]) {
    constexpr int kTogether = N < 4 ? N : 4;      // pairs whose roundings share a branch
#pragma unroll
    for (int j0 = 0; j0 < N; j0 += kTogether) {
      double v[2 * kTogether];
      T o[2 * kTogether];
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        const double p = to_f64<T>(x(j0 + j)), q = to_f64<T>(y(j0 + j));
        v[j] = p * cs[j0 + j][0] - q * cs[j0 + j][1];
        v[kTogether + j] = q * cs[j0 + j][0] + p * cs[j0 + j][1];
      }
      to_storage(v, o);
#pragma unroll
      for (int j = 0; j < kTogether; ++j) {
        x(j0 + j) = o[j];
        y(j0 + j) = o[kTogether + j];
      }
    }
  }
};

// How a launch shares out its rows: a workgroup takes `toks` tokens and hs heads of each, a thread one of a head's `lanes` parts.
struct Split {
  int toks, hs, lanes, parts;      // parts of a head: those that turn, then those that do not
};

template <typename T, int N, bool HALVES, bool STREAM>
__global__ __launch_bounds__(kMostThreads) void rope_at(RopeArgs a, Split s) {
  extern __shared__ __attribute__((aligned(16))) f64x2 cs[];      // [toks][half]
  constexpr int kSize = N * (int)sizeof(T);
  const int tid = threadIdx.x;
  const int64_t tok0 = ((int64_t)blockIdx.y * paged::kGridRow + blockIdx.x) * s.toks;
  if (tok0 >= a.n_tok) return;
  const int n = (int)min((int64_t)s.toks, a.n_tok - tok0);
  const int turning = a.half / N;
  const int lane = tid % s.lanes, rest = tid / s.lanes, h = blockIdx.z * s.hs + rest % s.hs, r = rest / s.hs;
  const bool mine = r < n && h < a.heads;
  const int64_t tok = tok0 + (mine ? r : 0);
  const int p = a.pos[tok];
  const Place to = place_of(a, tok, mine ? h : 0);
  Pieces<T, N, HALVES, STREAM> v;
  int at = 0, gap = 0;
  auto request = [&](int i) {                     // part i of the thread's head
    if (i < turning) {
      at = i * (HALVES ? kSize : 2 * kSize);
      gap = HALVES ? a.half * (int)sizeof(T) : kSize;
    } else {
      at = 2 * a.half * (int)sizeof(T) + (i - turning) * 2 * kSize;
      gap = at + kSize < (2 * a.half + a.rest) * (int)sizeof(T) ? kSize : 0;      // a single piece is taken twice
    }
    v.load(to.x, at, gap);
  };
  request(lane);
  for (int e = tid; e < n * a.half; e += blockDim.x) {
    f64x2 t = turn_of((double)a.pos[tok0 + e / a.half] * a.freq[e % a.half]);
    t *= a.gain;
    if (a.transposed) t[1] = -t[1];
    cs[e] = t;
  }
  __syncthreads();
  if (!mine || p < 0) return;
  for (int i = lane; i < s.parts; i += s.lanes) {
    if (i != lane) request(i);
    if (i < turning) {
      f64x2 t[N];
#pragma unroll
      for (int j = 0; j < N; ++j) t[j] = cs[r * a.half + i * N + j];
      v.turn(t);
    }
    v.store(to.out, at, gap);
  }
}

template <typename T, int N> int launch_of(const RopeArgs& a, hipStream_t st) {
  Split s;
  s.parts = a.half / N + (a.rest / N + 1) / 2;
  s.lanes = s.parts < kThreads ? s.parts : kThreads;
  const int most = kMostThreads / s.lanes;             // heads' places of a workgroup
  const int rounds = (a.heads + most - 1) / most;      // workgroups that share a token's heads
  s.hs = (a.heads + rounds - 1) / rounds;
  s.toks = kThreads / (s.lanes * s.hs);
  if (s.toks < 1) s.toks = 1;
  dim3 grid = paged::grid_for(((int64_t)a.n_tok + s.toks - 1) / s.toks);
  grid.z = rounds;
  const unsigned threads = (unsigned)(s.toks * s.hs * s.lanes + 63) / 64 * 64;
  const size_t lds = (size_t)s.toks * a.half * sizeof(f64x2);
  // Results that, with what they are made of, are more than the last-level cache holds go past it: what reads them next finds none of them there
  // in any case.  Projection, rotation and a reader, 32 and 8 heads of 128, less the two others: 40000 tokens 153.3 -> 148.0 us, 16384 65.0 ->
  // 62.4; but 8192 25.2 -> 28.4, 4096 16.2 -> 19.1.  In place, where rows are half of what is counted here, either store takes the same time (a fill,
  // the rotation and a reader of 132, 160, 195, 244 MB: 93.1, 106.3, 131.0, 177.0 past the cache, 93.7, 106.7, 131.4, 177.4 not).
  constexpr int64_t kCache = (int64_t)256 << 20;
  const bool stream = N * sizeof(T) == 16 && (int64_t)a.n_tok * a.heads * (2 * a.half + a.rest) * (int64_t)sizeof(T) * 2 > kCache;
  auto run = [&](auto halves, auto streams) {
    rope_at<T, N, decltype(halves)::value, decltype(streams)::value && N * sizeof(T) == 16><<<grid, threads, lds, st>>>(a, s);
  };
  using yes = std::true_type;
  using no = std::false_type;
  if (a.pairs == ESA_PAIRS_HALVES)
    stream ? run(yes(), yes()) : run(yes(), no());
  else
    stream ? run(no(), yes()) : run(no(), no());
  ESA_LAUNCH_CHECK("rope_at");
  return ESA_OK;
}

constexpr int64_t kFewPieces = 65536;      // (of 16 bytes, two to a thread)

}  // namespace

int launch_rope_at(const RopeArgs& a, int dtype, hipStream_t st) {
  const int es = dtype == ESA_F32 ? 4 : 2;
  // Pieces of 16 or 8 bytes where every row, the pairs and what is behind them allow it.
  int64_t all = (int64_t)a.half * es | (int64_t)a.rest * es;
  for (const RowSet& s : a.set) {
    if (s.heads == 0) continue;
    all |= (int64_t)(uintptr_t)s.x | (int64_t)(uintptr_t)s.out | s.x_tok | s.x_head | s.out_tok | s.out_head;
  }
  int piece = all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : es;
  // Few rows leave compute units without work: half the instructions to a thread are quicker there.
  if (piece == 16 && (int64_t)a.n_tok * a.heads * (2 * a.half + a.rest) * es < 32 * kFewPieces) piece = 8;
  if (dtype == ESA_F32) return piece == 16 ? launch_of<float, 4>(a, st) : piece == 8 ? launch_of<float, 2>(a, st) : launch_of<float, 1>(a, st);
  return piece == 16 ? launch_of<bf16_t, 8>(a, st) : piece == 8 ? launch_of<bf16_t, 4>(a, st) : launch_of<bf16_t, 1>(a, st);
}

}  // namespace serve
}  // namespace esa
