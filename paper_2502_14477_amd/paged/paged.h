// What the kernels of the paged cache share: a call's sequences, the way from a position to its row, 8-bit blocks.
#pragma once
#include "esa_common.h"
#include "esa_paged.h"

namespace esa {
namespace paged {

// ---------------------------------------------------------------- the call as the kernels take it
struct Batch {
  const int32_t *cu, *start, *pages;
  int64_t pages_ld;
  int n_tok, n_seq, max_pages, page_log2;
};
struct Cache {
  char *k, *v;
  uint8_t *k_scale, *v_scale;               // [n_pages][h_kv]
  uint32_t page_bytes, head_bytes, tok_bytes;
  int n_pages, h_kv, d;
  int close;                                // positions of a page whose rows lie within 2^32 bytes: all of them, or 0 where they span more
};
// A row's place in the pool, and a block's number (the host keeps strides and the number of blocks within 32 bits; one instruction each).
__device__ __forceinline__ int64_t place_of(const Cache& c, int page, int g, int slot) {
  return (int64_t)((uint64_t)(uint32_t)page * c.page_bytes + (uint64_t)(uint32_t)g * c.head_bytes + (uint64_t)(uint32_t)slot * c.tok_bytes);
}
// What a row lies behind its block's first.
__device__ __forceinline__ int64_t row_at(const Cache& c, int slot) { return (int64_t)((uint64_t)(uint32_t)slot * c.tok_bytes); }
__device__ __forceinline__ uint32_t block_of(const Cache& c, int page, int g) { return (uint32_t)page * (uint32_t)c.h_kv + (uint32_t)g; }

// A sequence's rows, clamped so that no content of the arrays leads out of the buffers.
struct Seq {
  int row0, n, t0;                          // first row, new tokens, position of the first
};
__device__ __forceinline__ Seq sequence(const Batch& a, int b) {
  const int lo = min(max(a.cu[b], 0), a.n_tok), hi = min(max(a.cu[b + 1], lo), a.n_tok);
  Seq s;
  s.row0 = lo;
  s.n = hi - lo;
  s.t0 = min(max(a.start[b], 0), INT32_MAX - s.n);
  return s;
}

// The sequence that has row `tok`, -1: none.  The whole wave takes part with one tok.
__device__ __forceinline__ int sequence_with(const Batch& a, int tok) {
  const int lane = threadIdx.x & 63;
  int b = 0;                                // sequences that end in front of the row
  for (int b0 = 0; b0 < a.n_seq; b0 += 64) b += __popcll(__ballot(b0 + lane < a.n_seq && a.cu[b0 + lane + 1] <= tok));
  if (b == a.n_seq) return -1;
  const Seq s = sequence(a, b);
  return tok >= s.row0 && tok < s.row0 + s.n ? b : -1;
}

// The page of a position, -1 where there is none.
__device__ __forceinline__ int page_of(const Batch& a, int n_pages, int b, int pos) {
  const int n = pos >> a.page_log2;
  const int p = a.pages[(int64_t)b * a.pages_ld + min(n, a.max_pages - 1)];
  return n < a.max_pages && (uint32_t)p < (uint32_t)n_pages ? p : -1;
}

// ---------------------------------------------------------------- workgroups
// A launch has fewer than 2^32 threads a dimension: more workgroups than that leaves room for, of up to 1024 threads, lie in rows of 2^21.  The last
// row's may have nothing to do.
constexpr int kGridRow = 1 << 21;
static_assert((int64_t)kGridRow * 1024 < (int64_t)1 << 32, "threads of a row of workgroups");
inline dim3 grid_for(int64_t blocks) {
  return blocks <= kGridRow ? dim3((unsigned)blocks) : dim3(kGridRow, (unsigned)((blocks + kGridRow - 1) / kGridRow));
}
__device__ __forceinline__ int block_index() { return (int)(blockIdx.y * kGridRow + blockIdx.x); }

// ---------------------------------------------------------------- scans over the sequences, a lane to each, 64 at a time
// Sums over the lanes up to each (in the vector unit: DPP shifts within rows of sixteen, then the rows' last lanes passed on).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);      // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);      // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}
__device__ __forceinline__ uint32_t lane_value(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane(x, lane); }
// Sums over the lanes up to each, of numbers below 2^52: two halves of 26 bits, of which 64 fit into 32.
__device__ __forceinline__ int64_t wave_scan_long(int64_t x) {
  return (int64_t)wave_scan((uint32_t)x & 0x3FFFFFFu) + ((int64_t)wave_scan((uint32_t)(x >> 26)) << 26);
}
__device__ __forceinline__ int64_t lane_long(int64_t x, int lane) { return (int64_t)lane_value((uint32_t)x, lane) | (int64_t)(int)lane_value((uint32_t)(x >> 32), lane) << 32; }
// What a lane may count, so that 64 of them stay within 32 bits (more than any call has).
__device__ __forceinline__ uint32_t countable(int64_t n) { return (uint32_t)min(n, (int64_t)1 << 24); }
struct Found {
  int b;              // the sequence, -1: beyond the last
  int64_t i;          // what is left within it
};
// The sequence in which the u-th of count(b) items each falls.  The whole wave takes part with one u.
template <typename F> __device__ __forceinline__ Found find(int n_seq, int64_t u, F&& count) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < n_seq; b0 += 64) {
    const int b = b0 + lane;
    const uint32_t c = b < n_seq ? countable(count(b)) : 0, upto = wave_scan(c);
    const uint64_t past = __ballot(upto > u);
    if (past) {
      const int at = __ffsll((unsigned long long)past) - 1;
      return Found{b0 + at, u - (int64_t)(uint32_t)__builtin_amdgcn_readlane(upto - c, at)};
    }
    u -= (uint32_t)__builtin_amdgcn_readlane(upto, 63);
  }
  return Found{-1, 0};
}

// ---------------------------------------------------------------- 8-bit blocks
constexpr float kF8Max = 448.f;
constexpr int kScaleLow = 27, kScaleHigh = 239;      // 2^-100, 2^112
constexpr int kNoScale = 255;                        // a block that holds nothing
// 2^(byte - 127) as the conversions take it: by its exponent's bits alone; and as a number, 2^-127 a subnormal one.
__device__ __forceinline__ float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ __forceinline__ float power_of(int byte) { return byte > 0 ? scale_of(byte) : __uint_as_float(0x400000u); }
// The byte of the smallest power of two s with amax <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int byte = (int)(u >> 23) - 8 + ((u & 0x7FFFFFu) > 0x600000u);
  return min(max(byte, kScaleLow), kScaleHigh);
}
__device__ __forceinline__ float f8_clamped(float x) { return x > kF8Max ? kF8Max : x < -kF8Max ? -kF8Max : x; }      // NaN stays
// Four numbers, rounded to nearest even.
__device__ __forceinline__ uint32_t f8_pack(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(f8_clamped(a), f8_clamped(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f8_clamped(c), f8_clamped(d), r, true);
}
typedef __attribute__((ext_vector_type(2))) float f32x2;
__device__ __forceinline__ void f8_unpack(uint32_t x, float (&f)[4]) {
  const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  f[0] = lo[0];
  f[1] = lo[1];
  f[2] = hi[0];
  f[3] = hi[1];
}

// ---------------------------------------------------------------- attention
struct AttendArgs {
  Batch batch;
  Cache cache;
  const char* q;
  char* out;
  float* lse;
  const int32_t* idx;
  int64_t ldq, ldo, idx_ld;                 // q, out in bytes
  int h, group, n_sel, l_i, l_l;
  float scale, cap;
};

// A sequence's keys, numbered through [0, i_end), the selected entries, [l_start, t0 + n); in front of the last a gap of numbers that are no
// keys, so that a multiple of 64 of them is one of the positions too and tiles lie in one page there (sixteen tokens over 128 and 4097 8-bit
// ones: 35.5 us without, 32.5).
struct Keys {
  int t0, i_end, n_sel, late, l_start, n;      // late: the list's and the gap's
};
__device__ __forceinline__ Keys keys_of(const AttendArgs& a, const Seq& s) {
  const int width = a.batch.max_pages << a.batch.page_log2;      // positions from there on have no page
  Keys k;
  k.t0 = s.t0;
  k.i_end = min(min(a.l_i, s.t0), width);
  k.l_start = min(max(s.t0 - a.l_l, k.i_end), width);
  k.n_sel = k.l_start > k.i_end ? a.n_sel : 0;
  k.late = k.n_sel + ((k.l_start - k.i_end - k.n_sel) & 63);
  k.n = k.i_end + k.late + (min(s.t0 + s.n, width) - k.l_start);
  return k;
}
// Numbers that a sequence has at most.
inline int64_t most_keys_of(const AttendArgs& a) { return ((int64_t)a.batch.max_pages << a.batch.page_log2) + (a.n_sel ? a.n_sel + 63 : 0); }
// The position of key j < k.n, -1 for an entry that is not seen.  In two steps where a kernel requests ahead: a request's result is only
// looked at when it is needed, so that nothing waits for it in between.
__device__ __forceinline__ int entry_of(const AttendArgs& a, const Keys& k, int b, int j) {      // as it lies in the list
  const int i = j - k.i_end;
  return (uint32_t)i < (uint32_t)k.n_sel ? a.idx[(int64_t)b * a.idx_ld + i] : 0;
}
__device__ __forceinline__ int position(const Keys& k, int j, int entry) {
  if (j < k.i_end) return j;
  j -= k.i_end;
  if (j < k.n_sel) return entry >= k.i_end && entry < k.l_start ? entry : -1;
  return j < k.late ? -1 : j - k.late + k.l_start;
}
// The table's entry for a position (any: for -1, or one behind the table, some entry), and whether it is a page.
__device__ __forceinline__ int page_entry(const Batch& a, int b, int pos) {
  return a.pages[(int64_t)b * a.pages_ld + min(max(pos, 0) >> a.page_log2, a.max_pages - 1)];
}
__device__ __forceinline__ bool is_page(const Batch& a, int n_pages, int pos, int entry) {
  return pos >= 0 && pos >> a.page_log2 < a.max_pages && (uint32_t)entry < (uint32_t)n_pages;
}

// Keys that the tokens up to `token`, or the rows up to `row`, of a sequence see at most.
__device__ __forceinline__ int keys_up_to(const AttendArgs& a, const Seq& s, const Keys& k, int token) {
  const int width = a.batch.max_pages << a.batch.page_log2;
  return k.n - (min(s.t0 + s.n, width) - min(s.t0 + token + 1, width));
}
__device__ __forceinline__ int keys_until(const AttendArgs& a, const Seq& s, const Keys& k, int row) { return keys_up_to(a, s, k, row / a.group); }

// Whether a row whose exponentials sum up to l has seen nothing: the largest of what it sees is one or nearly so.  By its bits: l is NaN where the
// query is.
__device__ __forceinline__ bool nothing_seen(float l) { return __float_as_uint(l) == 0; }

// A value that is the same in every lane, where the compiler does not see it.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) { return (int64_t)(uint32_t)uniform((int)x) | (int64_t)uniform((int)(x >> 32)) << 32; }
__device__ __forceinline__ Seq uniform(const Seq& s) { return Seq{uniform(s.row0), uniform(s.n), uniform(s.t0)}; }

int launch_append(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, int h, void* out_q, int64_t ldoq,
                  const Batch& b, const Cache& c, bool f8, double base, int dtype, hipStream_t st);
int launch_plain(const AttendArgs& a, bool f8, hipStream_t st);                                // fp32
// Sequences of at most most_rows rows (new tokens x query heads of a KV head), rows of up to 512 bytes; bf16 ones of more than above, head sizes 64 and 128.
size_t few_workspace(int n_seq, int h_kv, int d, int dtype);
int launch_few(const AttendArgs& a, bool f8, int dtype, int most_rows, void* ws, hipStream_t st);
size_t many_workspace(int h_kv, int d);
int launch_many(const AttendArgs& a, bool f8, int above, void* ws, hipStream_t st);

}  // namespace paged
}  // namespace esa
