// Verification of drafted tokens against the target's probabilities, from given random numbers (esa_verify_drafts).
//
// Row i of a sequence stands while u_i q_i(x_i) < p_{i-1}(x_i): two numbers a draft.  What has to be read is one row of the target and
// one of the draft a sequence, behind the last row that stands: the token is drawn from w = max(p - q, 0) by the sums of w up to each
// token.  Everything is fp64 (a product of two fp32 numbers is exact in it, a row's sum of a hundred thousand probabilities is off by 1e-16 or so), so the
// outcome is that of the definition but for random numbers that lie within 1e-15 of a border.
//
// What bounds it is latency (a draft's test is four dependent loads: offsets, token, probabilities, row) and, where sequences are many, HBM.  Rows of
// up to 16384 tokens are one workgroup's, in one launch (3.6 us and more).  Longer ones are cut into chunks, a workgroup to each, which finds
// its sequence's last standing row by itself and leaves its waves' sums; a second launch finds the block in which the sums pass the drawn number, and
// in it the token.  Rows are read in pieces of 16 bytes wherever they begin.  In a graph: one sequence of 32000 tokens and four drafts 6.3 us, sixteen of
// 131072 7.1, 128 21.5 (103 MB, half of them out of the last-level cache).  With loads behind bounds checks and the token found by LDS atomics these
// were 55, 83 and 117.  A wave that reads 1024 tokens of either row issues 216 vector instructions, its SIMD one in 38 % of its cycles; in bf16 242 and
// 60 %: there instructions bound it, not bytes (128 sequences 17.7).
#include "serve.h"

namespace esa {
namespace serve {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

template <typename T> __device__ __forceinline__ float number(T v);
template <> __device__ __forceinline__ float number<float>(float v) { return v; }
template <> __device__ __forceinline__ float number<bf16_t>(bf16_t v) { return bf16_to_f32(v); }
// Negative numbers, infinities and NaN count as 0: by their bits, one comparison.
template <typename T> __device__ __forceinline__ float probability(T v) {
  const float x = number<T>(v);
  return __float_as_uint(x) < 0x7F800000u ? x : 0.f;
}

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

// Drafts that stand, of a sequence with n >= 1 rows, and the one that does not (any token where all do).  The whole wave takes part, a lane to a draft.
struct Standing {
  int kept, token;
};
template <typename T> __device__ __forceinline__ Standing standing(const VerifyArgs& a, const Rows& s) {
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
    if (down) {
      const int l = __ffsll((unsigned long long)down) - 1;
      return Standing{i0 - 1 + l, (int)paged::lane_value((uint32_t)x, l)};
    }
  }
  return Standing{s.n - 1, -1};
}

// What a sequence draws from.
struct Drawn {
  int row, mode;      // of the target; 0: p, 1: p - q with the draft's next row, 2: p without the token of the next row
  int token;
};
__device__ __forceinline__ Drawn drawn_of(const VerifyArgs& a, const Rows& s, const Standing& x) {
  return Drawn{s.row0 + x.kept, x.kept == s.n - 1 ? 0 : a.draft ? 1 : 2, x.token};
}

// A piece of a row, and of the draft's: the N numbers from a token on, or, where these would reach over the row's end, the row's last N, of which `skip`
// belong to the piece in front or to nobody (the vocabulary has N or more).
template <typename T, int N> struct Pieces {
  Piece<T, N> p, q;
  int at, skip;
};
// M of them, `step` tokens apart from `first` on, all requested in front of their first use.  WITHIN: none reaches over the row's end.
template <typename T, int N, int M, bool WITHIN>
__device__ __forceinline__ void request(const VerifyArgs& a, const Drawn& d, int64_t first, int step, Pieces<T, N> (&x)[M]) {
  const T* pr = (const T*)(a.target + (int64_t)d.row * a.ldt);
  const T* qr = (const T*)(a.draft + (int64_t)(d.row + 1) * a.ldd);
  const int64_t end = (int64_t)a.vocab - N;
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const int64_t want = first + m * step, at = WITHIN ? want : min(want, end);
    x[m].at = (int)at;
    x[m].skip = WITHIN ? 0 : (int)(want - at);
    x[m].p = load<T, N>(pr + at);
  }
  if (d.mode == 1) {
#pragma unroll
    for (int m = 0; m < M; ++m) x[m].q = load<T, N>(qr + (WITHIN ? first + m * step : (int64_t)x[m].at));
  }
}
// The larger one, y not being negative: as whole numbers, by which negative ones are less and NaN (of positive sign) stays.
__device__ __forceinline__ float larger(float x, float y) { return __int_as_float(max(__float_as_int(x), __float_as_int(y))); }
// Its weights: take(number, token, weight).  All lanes of the wave take part.  STRICT: as they are defined.  Otherwise, two instructions a number fewer,
// where the target's probability is infinite or NaN the weight may be too, and the sum is.
template <bool STRICT, typename T, int N, typename F>
__device__ __forceinline__ void weigh(const Drawn& d, Pieces<T, N> x, F&& take) {
  if (__any(x.skip > 0)) {
#pragma unroll
    for (int j = 0; j < N; ++j) x.p.x[j] = j < x.skip ? (T)0 : x.p.x[j];
  }
  auto of = [](T v) { return STRICT ? probability<T>(v) : number<T>(v); };
  // the token that was looked up, with a probability of 1, is in few waves
  const int without = (int)((uint32_t)d.token - (uint32_t)x.at);
  if (d.mode == 1 || (d.mode == 2 && __any((uint32_t)without < (uint32_t)N))) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float q = d.mode == 1 ? probability<T>(x.q.x[j]) : j == without ? 1.f : 0.f;
      take(j, x.at + j, (double)larger(of(x.p.x[j]), q) - (double)q);
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) take(j, x.at + j, (double)larger(of(x.p.x[j]), 0.f));
  }
}

// A row is cut into chunks of EACH numbers a thread; its sums are kept by blocks, a wave's part of a chunk each.
template <int EACH> constexpr int kBlock = 64 * EACH;
template <int EACH> constexpr int kChunk = kThreads * EACH;
template <int EACH> __host__ __device__ inline int chunks_of(int vocab) { return (int)(((int64_t)vocab + kChunk<EACH> - 1) / kChunk<EACH>); }
template <int EACH> __host__ __device__ inline int blocks_of(int vocab) { return chunks_of<EACH>(vocab) * kWaves; }
struct Work {
  double* sums;      // [n_seq][blocks]
  int32_t* kept;     // [n_seq]
};
__host__ __device__ inline Work work_at(void* ws, int n_seq, int blocks) {
  double* sums = (double*)ws;
  return Work{sums, (int32_t*)(sums + (size_t)n_seq * blocks)};
}

// Sums over the lanes up to each, in the vector unit: shifts within rows of sixteen lanes, then the rows' last lanes passed on.
template <int CTRL, int ROWS> __device__ __forceinline__ double passed_on(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)u, CTRL, ROWS, 0xF, false), hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
  return __builtin_bit_cast(double, (uint64_t)lo | (uint64_t)hi << 32);
}
__device__ __forceinline__ double wave_sums(double x) {
  x += passed_on<0x111, 0xF>(x);      // row_shr 1, 2, 4, 8
  x += passed_on<0x112, 0xF>(x);
  x += passed_on<0x114, 0xF>(x);
  x += passed_on<0x118, 0xF>(x);
  x += passed_on<0x142, 0xA>(x);      // row_bcast 15, 31
  return x + passed_on<0x143, 0xC>(x);
}
__device__ __forceinline__ double lane_double(double x, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  return __builtin_bit_cast(double, (uint64_t)paged::lane_value((uint32_t)u, lane) | (uint64_t)paged::lane_value((uint32_t)(u >> 32), lane) << 32);
}

// A chunk's blocks' sums, by a workgroup.
template <bool STRICT, bool WITHIN, int EACH, typename T, int N> __device__ __forceinline__ void chunk_sums(const VerifyArgs& a, const Drawn& d, int chunk, double* sums) {
  constexpr int M = EACH / N;
  const int block = chunk * kWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  Pieces<T, N> x[M];
  request<T, N, M, WITHIN>(a, d, (int64_t)block * kBlock<EACH> + lane * N, 64 * N, x);
  double w = 0.0;
#pragma unroll
  for (int m = 0; m < M; ++m) weigh<STRICT>(d, x[m], [&](int, int, double y) { w += y; });
  w = wave_sums(w);
  if (lane == 63) sums[block] = w;
}

// grid (chunks, sequences)
template <typename T, int N, int EACH> __global__ __launch_bounds__(kThreads) void verify_sums(VerifyArgs a) {
  const int chunk = blockIdx.x, blocks = blocks_of<EACH>(a.vocab);
  const Work k = work_at(a.ws, a.n_seq, blocks);
  for (int b = blockIdx.y; b < a.n_seq; b += gridDim.y) {
    const Rows s = rows_of(a, b);
    if (s.n == 0) continue;
    const Standing x = standing<T>(a, s);
    const Drawn d = drawn_of(a, s, x);
    double* sums = k.sums + (int64_t)b * blocks;
    if ((int64_t)(chunk + 1) * kChunk<EACH> <= a.vocab)
      chunk_sums<false, true, EACH, T, N>(a, d, chunk, sums);
    else
      chunk_sums<false, false, EACH, T, N>(a, d, chunk, sums);
    if (chunk == 0 && threadIdx.x == 0) k.kept[b] = x.kept;
  }
}

// Sums over the workgroup in front of each thread, and of all.
struct Scanned {
  double before, all;
};
__device__ __forceinline__ Scanned scan(double x, double* part) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  x = wave_sums(x);
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

// The first item that passes, and the last one with any weight: INT32_MAX, -1 where there is none.  The threads' items ascend.
struct Found {
  int first, last;
};
__device__ __forceinline__ Found in_wave(const Found& x) {
  const uint64_t f = __ballot(x.first != INT32_MAX), l = __ballot(x.last >= 0);
  return {f ? (int)paged::lane_value((uint32_t)x.first, __ffsll((unsigned long long)f) - 1) : INT32_MAX,
          l ? (int)paged::lane_value((uint32_t)x.last, 63 - __clzll((long long)l)) : -1};
}
__device__ __forceinline__ Found find(const Found& x, Found* part) {
  const int wave = threadIdx.x >> 6;
  const Found mine = in_wave(x);
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

// The first of a thread's N tokens where sums pass the target, `sum` being what is in front of them, and the last one with any weight.
template <int N> __device__ __forceinline__ Found look(const double (&w)[N], int at, double sum, double target) {
  Found r = {INT32_MAX, -1};
#pragma unroll
  for (int j = 0; j < N; ++j) {
    sum += w[j];
    if (w[j] > 0.0) {
      r.last = at + j;
      if (sum > target && r.first == INT32_MAX) r.first = r.last;
    }
  }
  return r;
}
__device__ __forceinline__ double target_of(float u, double total) { return u >= 1.f ? __builtin_huge_val() : u > 0.f ? u * total : 0.0; }

// A workgroup a sequence.
constexpr int kBlocks = 4;      // blocks' sums a thread in a round
constexpr int kRound = kThreads * kBlocks;
template <typename T, int N, int EACH> __global__ __launch_bounds__(kThreads) void verify_draw(VerifyArgs a) {
  __shared__ double part[kWaves];
  __shared__ Found found[kWaves];
  __shared__ double at_block;
  const int tid = threadIdx.x, b = paged::block_index();
  if (b >= a.n_seq) return;
  const int blocks = blocks_of<EACH>(a.vocab);
  const Work k = work_at(a.ws, a.n_seq, blocks);
  double* const sums = k.sums + (int64_t)b * blocks;
  double x[kBlocks];
  Scanned y;
  auto fetch = [&](int r0) {
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) x[j] = sums[min(r0 + tid * kBlocks + j, blocks - 1)];
  };
  auto add_up = [&](int r0) {
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      x[j] = r0 + tid * kBlocks + j < blocks ? x[j] : 0.0;
      sum += x[j];
    }
    y = scan(sum, part);
  };
  fetch(0);
  const Rows s = rows_of(a, b);
  if (s.n == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }
  const int kept = k.kept[b];
  const float u = a.u[s.row0];
  Drawn d = drawn_of(a, s, Standing{kept, a.tokens[s.row0 + min(kept + 1, s.n - 1)]});
  for (int i = tid; i < s.n; i += kThreads)
    if (i != kept) a.out[s.row0 + i] = i < kept ? a.tokens[s.row0 + i + 1] : -1;
  if (tid == 0) a.count[b] = kept + 1;
  double total = 0.0;
  bool at_hand = blocks <= kRound;               // whether the first round's sums are those that are looked through
  for (int r0 = 0; r0 < blocks; r0 += kRound) {
    if (r0) fetch(r0);
    add_up(r0);
    total += y.all;
  }
  // Infinities or NaN among the target's probabilities, or nothing left and p itself wanted, of which there are no sums: one workgroup reads it all again.
  for (bool bad = !(total < __builtin_huge_val()); bad || (!(total > 0.0) && d.mode != 0); bad = false) {
    if (!bad) d.mode = 0;
    at_hand = false;
    __syncthreads();
    for (int c = 0; c < chunks_of<EACH>(a.vocab); ++c) chunk_sums<true, false, EACH, T, N>(a, d, c, sums);
    __syncthreads();
    total = 0.0;
    for (int r0 = 0; r0 < blocks; r0 += kRound) {
      fetch(r0);
      add_up(r0);
      total += y.all;
    }
  }
  if (!(total > 0.0)) {
    if (tid == 0) a.out[d.row] = -1;
    return;
  }
  const double target = target_of(u, total);
  // the first block whose sums pass it, or else the last with any
  int block = -1;
  double base = 0.0;
  for (int r0 = 0; r0 < blocks; r0 += kRound) {
    if (!at_hand) {
      fetch(r0);
      add_up(r0);
    }
    const Found f = find(look<kBlocks>(x, r0 + tid * kBlocks, base + y.before, target), found);
    if (f.first != INT32_MAX) block = f.first;
    else if (f.last >= 0) block = f.last;
    double before = base + y.before;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      if (block == r0 + tid * kBlocks + j) at_block = before;
      before += x[j];
    }
    if (f.first != INT32_MAX) break;
    base += y.all;
  }
  __syncthreads();
  Pieces<T, N> piece[1];
  const bool mine = tid < kBlock<EACH> / N;
  request<T, N, 1, false>(a, d, (int64_t)block * kBlock<EACH> + (mine ? tid : 0) * N, 0, piece);
  double w[N], sum = 0.0;
  weigh<true>(d, piece[0], [&](int j, int, double v) {
    w[j] = mine ? v : 0.0;
    sum += w[j];
  });
  sum = at_block + scan(sum, part).before;
  const Found f = find(look<N>(w, piece[0].at, sum, target), found);
  if (tid == 0) a.out[d.row] = f.first != INT32_MAX ? f.first : f.last;
}

// A short row is one workgroup's: a launch does all, M pieces a thread.  Its instructions are then one compute unit's, so that longer rows are quicker in
// two launches.  us a call in a graph, 1 / 16 / 128 / 512 sequences of four drafts, in one launch and in two:
//    fp32   2000 tokens  3.7 / 3.9 / 4.0 / 4.4 (256 threads)                        6.2 / 7.2 / 7.4 / 7.9
//           4000         3.6 / 4.1 / 4.3 / 4.9 (512)                                6.2 / 7.1 / 7.3 / 8.3
//           8000         3.9 / 4.5 / 4.8 / 6.8 (1024)                               6.0 / 7.0 / 7.3 / 10.5
//          16000         5.4 / 5.7 / 5.9 / 15.4 (1024, sixteen numbers each)        6.4 / 7.0 / 7.8 / 16.7
//          32000         9.4 / 10.1 / 10.6 / 25.7 (a trial of 32 numbers each)      6.0 / 7.0 / 9.5 / 23.8
//    bf16   2000         3.8 / 4.2 / 4.2 / 4.7                                      6.3 / 7.4 / 7.5 / 8.2
//           4000         3.6 / 4.3 / 4.4 / 5.2                                      5.8 / 7.2 / 7.4 / 8.4
//           8000         3.9 / 4.9 / 5.1 / 6.8                                      6.1 / 7.1 / 7.5 / 9.6
//          16000         5.3 / 5.7 / 6.0 / 10.5                                     6.6 / 7.1 / 7.9 / 12.9
// (2000 tokens by 1024 threads, fp32: 4.2 / 4.5 / 4.8 / 6.8.)
template <typename T, int N, int M, int THREADS> __global__ __launch_bounds__(THREADS) void verify_whole(VerifyArgs a) {
  constexpr int kWaves = THREADS / 64;
  constexpr int kSums = M * kWaves;      // sums of a wave's pieces in the tokens' order, a lane to each
  static_assert(kSums <= 64, "a lane to each sum");
  __shared__ double sums[64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = paged::block_index();
  if (b >= a.n_seq) return;
  const Rows s = rows_of(a, b);
  if (s.n == 0) {
    if (tid == 0) a.count[b] = 0;
    return;
  }
  const Standing st = standing<T>(a, s);
  const int kept = st.kept;
  Drawn d = drawn_of(a, s, st);
  const float u = a.u[s.row0];
  for (int i = tid; i < s.n; i += THREADS)
    if (i != kept) a.out[s.row0 + i] = i < kept ? a.tokens[s.row0 + i + 1] : -1;
  if (tid == 0) a.count[b] = kept + 1;
  if (tid >= kSums && tid < 64) sums[tid] = 0.0;
  double mine, upto, total;
  for (bool strict = false;;) {
    Pieces<T, N> x[M];
    request<T, N, M, false>(a, d, tid * N, THREADS * N, x);
#pragma unroll
    for (int m = 0; m < M; ++m) {
      double w = 0.0;
      if (strict)
        weigh<true>(d, x[m], [&](int, int, double y) { w += y; });
      else
        weigh<false>(d, x[m], [&](int, int, double y) { w += y; });
      w = wave_sums(w);
      if (lane == 63) sums[m * kWaves + wave] = w;
      __builtin_amdgcn_sched_barrier(0);      // (all pieces' numbers in 64 bits at once do not fit the registers)
    }
    __syncthreads();
    // every wave adds them up for itself
    mine = sums[lane];
    upto = wave_sums(mine);
    total = lane_double(upto, 63);
    if (!(total < __builtin_huge_val()))
      strict = true;
    else if (total > 0.0 || d.mode == 0)
      break;
    else
      d.mode = 0;      // nothing is left: p itself
    __syncthreads();
  }
  if (!(total > 0.0)) {
    if (tid == 0) a.out[d.row] = -1;
    return;
  }
  const double target = target_of(u, total);
  // the first sum that passes it, or else the last with any
  const uint64_t past = __ballot(mine > 0.0 && upto > target), any = __ballot(mine > 0.0);
  const int at = past ? __ffsll((unsigned long long)past) - 1 : 63 - __clzll((long long)any);
  const double base = at > 0 ? lane_double(upto, at - 1) : 0.0;
  if (wave != at % kWaves) return;
  Pieces<T, N> piece[1];
  request<T, N, 1, false>(a, d, tid * N + at / kWaves * (THREADS * N), 0, piece);
  double w[N], sum = 0.0;
  weigh<true>(d, piece[0], [&](int j, int, double v) {
    w[j] = v;
    sum += v;
  });
  const double front = __shfl_up(wave_sums(sum), 1);
  const Found f = in_wave(look<N>(w, piece[0].at, base + (lane ? front : 0.0), target));
  if (lane == 0) a.out[d.row] = f.first != INT32_MAX ? f.first : f.last;
}

template <typename T, int N, int M, int THREADS> int launch_whole(const VerifyArgs& a, hipStream_t st) {
  verify_whole<T, N, M, THREADS><<<paged::grid_for(a.n_seq), THREADS, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_whole");
  return ESA_OK;
}
template <typename T, int N, int EACH> int launch_two(const VerifyArgs& a, hipStream_t st) {
  verify_sums<T, N, EACH><<<dim3((unsigned)chunks_of<EACH>(a.vocab), (unsigned)(a.n_seq < 65535 ? a.n_seq : 65535)), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_sums");
  verify_draw<T, N, EACH><<<paged::grid_for(a.n_seq), kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("verify_draw");
  return ESA_OK;
}
constexpr int kWhole = 16384;      // tokens of a row that one workgroup takes
template <typename T> int launch_of(const VerifyArgs& a, hipStream_t st) {
  constexpr int N = kPiece<T>;
  if (a.vocab < N) return launch_whole<T, 1, 1, 64>(a, st);
  if (a.vocab <= 2048) return launch_whole<T, N, 8 / N, 256>(a, st);
  if (a.vocab <= 4096) return launch_whole<T, N, 8 / N, 512>(a, st);
  if (a.vocab <= 8192) return launch_whole<T, N, 8 / N, 1024>(a, st);
  if (a.vocab <= kWhole) return launch_whole<T, N, 16 / N, 1024>(a, st);
  // Sixteen numbers a thread where that makes more than four workgroups a compute unit, else eight: 16 / 32 / 64 / 128 / 200 sequences of 131072 tokens 7.9 /
  // 10.5 / 16.6 / 23.3 / 31.4 us in a graph with sixteen, 7.4 / 10.2 / 16.4 / 23.6 / 32.6 with eight; in bf16 8.2 / 8.9 / 11.7 / 17.8 / 22.3 and 7.6 / 8.9 /
  // 12.6 / 19.7 / 25.9.
  return (int64_t)chunks_of<16>(a.vocab) * a.n_seq > 1024 ? launch_two<T, N, 16>(a, st) : launch_two<T, N, 8>(a, st);
}

}  // namespace

size_t verify_workspace(int n_seq, int vocab) {
  return vocab <= kWhole ? 0 : align_up((size_t)n_seq * (blocks_of<8>(vocab) * sizeof(double) + sizeof(int32_t)), 256);
}

int launch_verify(const VerifyArgs& a, int dtype, hipStream_t st) { return dtype == ESA_F32 ? launch_of<float>(a, st) : launch_of<bf16_t>(a, st); }

}  // namespace serve
}  // namespace esa
