// Appending keys and values to a paged cache, the rotary encoding on the way (esa_append_paged).
//
// Row i of sequence b goes to position p = start[b] + i: pairs (j, j + d/2) of queries and keys turn by p base^(-2j/d), in fp64 with one
// rounding into the storage type, as esa_rope's do.  It is a copy with arithmetic: (2 h + 2 h_kv) d storage elements and 2 h_kv d cache
// elements a token.
//
// Pages in the storage type: a workgroup takes one to four tokens with all their heads, which share the tokens' sines and cosines.
// 8-bit pages: a scale belongs to a page and a head, so a workgroup takes the part of a page that a sequence writes to, for one head's
// keys or values: it turns the rows, keeps them in registers rounded to the storage type, takes their largest magnitude, and
// writes them by the block's scale.  No two workgroups touch one block, so nothing is atomic and the result does not depend on their order.
//   A step of sixteen sequences takes 5.5 us, a chain of dependent loads; eight prompts of up to 4096 tokens of 32 and 8 heads 101.7 us, 449 MB
// at 4.4 TB/s, where a copy moves 5.2.
#include <cmath>

#include "paged.h"

namespace esa {
namespace paged {
namespace {

typedef __attribute__((ext_vector_type(2))) double f64x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

constexpr int kThreads = 256;
constexpr int kMaxHalf = 128;
// Angle per position of every frequency, and its cosine and sine.
struct Turns {
  double freq[kMaxHalf], c[kMaxHalf], s[kMaxHalf];
};

struct AppendArgs {
  Batch batch;
  Cache cache;
  const char *k, *v, *q;
  char* out_q;
  int64_t ldk, ldv, ldq, ldoq;              // bytes
  int h, rotate;
  int row_tokens, row_blocks;               // tokens of a workgroup of append_rows, and such workgroups in front of the blocks'
  Turns turns;
};

// 16 bytes of a row.
template <typename T> struct Vec {
  static constexpr int n = 16 / (int)sizeof(T);
  T x[n] __attribute__((aligned(16)));
};
template <typename T> __device__ __forceinline__ Vec<T> load_vec(const char* p) {
  Vec<T> v;
  *(u32x4*)v.x = *(const u32x4*)p;
  return v;
}
template <typename T> __device__ __forceinline__ void store_vec(char* p, const Vec<T>& v) { *(u32x4*)p = *(const u32x4*)v.x; }

// Pairs of a row's two halves turned by the angles whose cosine and sine cs holds.
__device__ __forceinline__ void turn(Vec<float>& a, Vec<float>& b, const f64x2* cs) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f64x2 t = cs[i];
    const double x = a.x[i], y = b.x[i];
    a.x[i] = (float)(x * t[0] - y * t[1]);
    b.x[i] = (float)(y * t[0] + x * t[1]);
  }
}
__device__ __forceinline__ void turn(Vec<bf16_t>& a, Vec<bf16_t>& b, const f64x2* cs) {
#pragma unroll
  for (int i0 = 0; i0 < 8; i0 += 4) {       // the roundings of four pairs share a branch
    double v[8];
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f64x2 t = cs[i0 + i];
      const double x = bf16_to_f32(a.x[i0 + i]), y = bf16_to_f32(b.x[i0 + i]);
      v[i] = x * t[0] - y * t[1];
      v[4 + i] = y * t[0] + x * t[1];
    }
    narrow_for_bf16(v, f);
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      *(uint32_t*)(a.x + i0 + i) = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[i], f[i + 1]}), bf16x2));
      *(uint32_t*)(b.x + i0 + i) = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{f[4 + i], f[5 + i]}), bf16x2));
    }
  }
}

__device__ __forceinline__ f64x2 turn_of(double angle) {
  double s, c;
  sincos(angle, &s, &c);
  return f64x2{c, s};
}

// The tokens of workgroup `block`: queries, and, in the storage type, keys and values.
constexpr int kRowTokens = 4;
template <typename T> __device__ void append_rows(const AppendArgs& a, int block, bool paged, f64x2* cs) {
  __shared__ int pos[kRowTokens];
  __shared__ int64_t at[kRowTokens];        // a token's place in the pool for head 0, -1: none
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int tok0 = block * a.row_tokens, n = min(a.row_tokens, a.batch.n_tok - tok0);
  if (wave < n) {
    const int tok = tok0 + wave;
    const int b = sequence_with(a.batch, tok);
    if (lane == 0) {
      int p = -1;
      int64_t to = -1;
      if (b >= 0) {
        const Seq s = sequence(a.batch, b);
        p = s.t0 + tok - s.row0;
        const int page = paged ? page_of(a.batch, a.cache.n_pages, b, p) : -1;
        if (page >= 0) to = place_of(a.cache, page, 0, p & ((1 << a.batch.page_log2) - 1));
      }
      pos[wave] = p;
      at[wave] = to;
    }
  }
  __syncthreads();
  const int half = a.cache.d >> 1, vecs = half / Vec<T>::n, half_bytes = half * (int)sizeof(T);
  if (a.rotate) {
    for (int e = tid; e < n * half; e += kThreads) cs[e] = turn_of((double)max(pos[e / half], 0) * a.turns.freq[e % half]);
    __syncthreads();
  }
  const int heads = a.h + (paged ? 2 * a.cache.h_kv : 0), items = n * heads * vecs;
  constexpr int kAhead = 4;
  for (int e0 = tid; e0 < items; e0 += kThreads * kAhead) {
    Vec<T> x[kAhead], y[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int e = e0 + u * kThreads < items ? e0 + u * kThreads : e0;
      const int i = e % vecs, hh = e / vecs % heads;
      const int64_t tok = tok0 + e / (vecs * heads);
      const int g = hh - a.h, kv = g - a.cache.h_kv;
      const char* from = g < 0 ? a.q + tok * a.ldq + (int64_t)hh * 2 * half_bytes
                               : kv < 0 ? a.k + tok * a.ldk + (int64_t)g * 2 * half_bytes : a.v + tok * a.ldv + (int64_t)kv * 2 * half_bytes;
      x[u] = load_vec<T>(from + i * 16);
      y[u] = load_vec<T>(from + half_bytes + i * 16);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int e = e0 + u * kThreads;
      if (e >= items) break;
      const int i = e % vecs, hh = e / vecs % heads, r = e / (vecs * heads);
      const int g = hh - a.h, kv = g - a.cache.h_kv;
      if (pos[r] < 0) continue;             // behind the last sequence
      if (a.rotate && kv < 0) turn(x[u], y[u], cs + r * half + i * Vec<T>::n);
      char* to;
      if (g < 0) {
        to = a.out_q + (int64_t)(tok0 + r) * a.ldoq + (int64_t)hh * 2 * half_bytes;
      } else {
        if (at[r] < 0) continue;
        to = (kv < 0 ? a.cache.k : a.cache.v) + at[r] + (int64_t)(kv < 0 ? g : kv) * a.cache.head_bytes;
      }
      store_vec(to + i * 16, x[u]);
      store_vec(to + half_bytes + i * 16, y[u]);
    }
  }
}

template <typename T> __global__ __launch_bounds__(kThreads) void append_same(AppendArgs a) {
  extern __shared__ f64x2 table[];          // [kRowTokens][d / 2]
  append_rows<T>(a, block_index(), true, table);
}

template <typename T> __device__ __forceinline__ float largest(const Vec<T>& v) {
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < Vec<T>::n; ++i) m = fmaxf(m, fabsf(load_f32<T>(v.x + i)));
  return m;
}
template <typename T> __device__ __forceinline__ void store_f8(char* p, const Vec<T>& v, float by) {
#pragma unroll
  for (int i = 0; i < Vec<T>::n; i += 4)
    *(uint32_t*)(p + i) = f8_pack(load_f32<T>(v.x + i) * by, load_f32<T>(v.x + i + 1) * by, load_f32<T>(v.x + i + 2) * by, load_f32<T>(v.x + i + 3) * by);
}

// A block: keys or values of one head in the part of a page that a sequence writes to.  A thread has a 16-byte piece of both halves of
// every kThreads / (d / 2 / Vec)-th row of the page, J rows in all.
template <typename T, int J> __global__ __launch_bounds__(kThreads) void append_blocks(AppendArgs a) {
  constexpr int V = Vec<T>::n;
  __shared__ f64x2 cs[kThreads * V];        // a round's rows' turns: [rows][d / 2]
  __shared__ float most[kThreads / 64];
  const int block = block_index();
  if (block < a.row_blocks) {
    append_rows<T>(a, block, false, cs);
    return;
  }
  const int unit = block - a.row_blocks, tid = threadIdx.x;
  const bool keys = (unit & 1) == 0;
  const int g = (unit >> 1) % a.cache.h_kv, log2 = a.batch.page_log2, page_size = 1 << log2;
  const Found f = find(a.batch.n_seq, (unit >> 1) / a.cache.h_kv, [&](int b) -> int64_t {
    const Seq s = sequence(a.batch, b);
    return s.n > 0 ? ((s.t0 + s.n - 1) >> log2) - (s.t0 >> log2) + 1 : 0;
  });
  if (f.b < 0) return;
  const Seq s = sequence(a.batch, f.b);
  const int n_page = (s.t0 >> log2) + (int)f.i, pos0 = n_page << log2;      // the page's first position
  const int lo = max(s.t0 - pos0, 0), hi = min(s.t0 + s.n - pos0, page_size);
  const int page = page_of(a.batch, a.cache.n_pages, f.b, pos0);
  if (page < 0) return;
  uint8_t* scale = (keys ? a.cache.k_scale : a.cache.v_scale) + block_of(a.cache, page, g);
  const int held = lo > 0 ? *scale : kNoScale, old = held == kNoScale ? 0 : held;
  const int d = a.cache.d, half = d >> 1, vecs = half / V, rows = kThreads / vecs, i = tid % vecs, r0 = tid / vecs;
  const int64_t ld = keys ? a.ldk : a.ldv;
  const char* from = (keys ? a.k : a.v) + ((int64_t)s.row0 + pos0 - s.t0) * ld + ((int64_t)g * d + i * V) * (int)sizeof(T);
  Vec<T> x[J], y[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int r = min(max(j * rows + r0, lo), hi - 1);
    x[j] = load_vec<T>(from + r * ld);
    y[j] = load_vec<T>(from + r * ld + half * (int)sizeof(T));
  }
  float m = 0.f;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int first = max(j * rows, lo), end = min((j + 1) * rows, hi);     // the round's rows
    if (first >= end) continue;
    if (keys && a.rotate) {
      if (j) __syncthreads();
      const int groups = kThreads / half, per = rows / groups, c = tid % half, at = j * rows + tid / half * per;
      const int from_row = max(at, first), to_row = min(at + per, end);     // consecutive rows of a thread: the turn of the first, then by one position
      if (from_row < to_row) {
        f64x2 t = turn_of((double)(pos0 + from_row) * a.turns.freq[c]);
        const double dc = a.turns.c[c], ds = a.turns.s[c];
        for (int r = from_row; r < to_row; ++r) {
          cs[(r - j * rows) * half + c] = t;
          t = f64x2{t[0] * dc - t[1] * ds, t[1] * dc + t[0] * ds};
        }
      }
      __syncthreads();
    }
    const int r = j * rows + r0;
    if (r >= first && r < end) {
      if (keys && a.rotate) turn(x[j], y[j], cs + r0 * half + i * V);
      m = fmaxf(m, fmaxf(largest<T>(x[j]), largest<T>(y[j])));
    }
  }
  m = wave_max(m);
  if ((tid & 63) == 0) most[tid >> 6] = m;
  __syncthreads();
  m = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
  const int byte = max(scale_byte(m), old);
  char* to = (keys ? a.cache.k : a.cache.v) + place_of(a.cache, page, g, 0);
  const float by = power_of(254 - byte);
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int r = j * rows + r0;
    if (r >= lo && r < hi) {
      char* const row = to + row_at(a.cache, r);
      store_f8<T>(row + i * V, x[j], by);
      store_f8<T>(row + half + i * V, y[j], by);
    }
  }
  if (held != kNoScale && byte > old) {     // the sequence's earlier rows come to the larger scale
    const float less = scale_of(max(127 - (byte - old), 1));
    const int pieces = d / 16;
    for (int e = tid; e < lo * pieces; e += kThreads) {
      u32x4* p = (u32x4*)(to + row_at(a.cache, e / pieces) + e % pieces * 16);
      u32x4 w = *p;
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float v[4];
        f8_unpack(w[n], v);
        w[n] = f8_pack(v[0] * less, v[1] * less, v[2] * less, v[3] * less);
      }
      *p = w;
    }
  }
  if (tid == 0) *scale = (uint8_t)byte;
}

const Turns& turns_for(double base, int d) {
  struct Kept {
    double base = 0.0;
    int d = 0;
    Turns t;
  };
  static thread_local Kept k;
  if (k.base != base || k.d != d) {
    k.base = base;
    k.d = d;
    for (int i = 0; i < d / 2; ++i) {
      k.t.freq[i] = std::pow(base, -2.0 * (double)i / (double)d);
      k.t.c[i] = std::cos(k.t.freq[i]);
      k.t.s[i] = std::sin(k.t.freq[i]);
    }
  }
  return k.t;
}

template <typename T> int launch(AppendArgs& a, bool f8, hipStream_t st) {
  a.row_tokens = a.batch.n_tok <= 512 ? 1 : kRowTokens;
  const int row_blocks = (a.batch.n_tok + a.row_tokens - 1) / a.row_tokens;
  if (!f8) {
    append_same<T><<<grid_for(row_blocks), kThreads, kRowTokens * (a.cache.d / 2) * sizeof(f64x2), st>>>(a);
    ESA_LAUNCH_CHECK("append_same");
    return ESA_OK;
  }
  a.row_blocks = a.q ? row_blocks : 0;
  // parts of pages: a sequence of n tokens touches (n - 1) / page_size + 2 pages at most
  const int page_size = 1 << a.batch.page_log2, used = a.batch.n_seq < a.batch.n_tok ? a.batch.n_seq : a.batch.n_tok;
  int64_t parts = a.batch.n_tok / page_size + 2 * (int64_t)used;
  if (parts > a.batch.n_tok) parts = a.batch.n_tok;
  const int64_t grid = a.row_blocks + parts * 2 * a.cache.h_kv;
  const int rows = kThreads / (a.cache.d / 2 / Vec<T>::n), j = (page_size + rows - 1) / rows;
  const dim3 g = grid_for(grid);
  if (j <= 1)
    append_blocks<T, 1><<<g, kThreads, 0, st>>>(a);
  else if (j == 2)
    append_blocks<T, 2><<<g, kThreads, 0, st>>>(a);
  else if (j <= 4)
    append_blocks<T, 4><<<g, kThreads, 0, st>>>(a);
  else if (j <= 8)
    append_blocks<T, 8><<<g, kThreads, 0, st>>>(a);
  else
    append_blocks<T, 16><<<g, kThreads, 0, st>>>(a);
  ESA_LAUNCH_CHECK("append_blocks");
  return ESA_OK;
}

}  // namespace

int launch_append(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, int h, void* out_q, int64_t ldoq,
                  const Batch& b, const Cache& c, bool f8, double base, int dtype, hipStream_t st) {
  const int64_t es = dtype == ESA_F32 ? 4 : 2;
  AppendArgs a;
  a.batch = b;
  a.cache = c;
  a.k = (const char*)k;
  a.v = (const char*)v;
  a.q = (const char*)q;
  a.out_q = (char*)out_q;
  a.ldk = ldk * es;
  a.ldv = ldv * es;
  a.ldq = ldq * es;
  a.ldoq = ldoq * es;
  a.h = q ? h : 0;
  a.rotate = base > 0.0;
  a.row_blocks = 0;
  if (a.rotate) a.turns = turns_for(base, c.d);
  return dtype == ESA_F32 ? launch<float>(a, f8, st) : launch<bf16_t>(a, f8, st);
}

}  // namespace paged
}  // namespace esa
