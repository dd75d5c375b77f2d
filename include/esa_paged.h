/*
 * libesa — a paged key/value cache beside esa.h's contiguous one: sequences of different lengths over one pool of pages, in the
 * storage type or in 8 bits, appended to with the rotary encoding on the way (esa_append_paged) and attended to (esa_attend_paged).
 * Conventions, error codes and error texts are those of esa.h: device pointers owned by the caller, strides in ELEMENTS, nothing
 * allocated, kept or enqueued on an error, every call returns without synchronising and may be captured into a graph.
 *
 * A call's lengths lie on the device, so that a captured call serves the lengths that it finds when it is replayed.  Nothing that
 * these arrays hold makes a kernel leave its buffers: what is out of range is clamped or left out as stated below.
 */
#ifndef ESA_PAGED_H
#define ESA_PAGED_H

#include "esa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache's element type beside ESA_F32 and ESA_BF16: 8-bit e4m3 (OCP, no infinities) with a scale for each page and KV head. */
#define ESA_E4M3 2

/*
 * The pool.  Page p holds page_size consecutive positions of one sequence; KV head g of its position s lies at
 *   k + p * page_stride + g * head_stride + s * tok_stride       (v likewise, same strides), d contiguous elements.
 *   page_size  16, 32, 64 or 128
 *   k_scale, v_scale  ESA_E4M3: [n_pages, h_kv] bytes (E8M0): a block's values are its e4m3 numbers times 2^(byte - 127).
 *                     Powers of two, so that a block grows to a larger scale without its numbers being rounded again (but for
 *                     e4m3's subnormals) and its values are bf16 numbers (those below 2^-126, of bytes 0 to 9, may count as 0 where
 *                     rows are bf16).  255: the block holds nothing.  NULL for other types.
 * Rows start on 16-byte boundaries (k, v, and every stride in bytes).  Strides may be in any order ([n_pages, page_size, h_kv, d]
 * is as good); two different elements must not overlap.  max_pages * page_size stays below 2^31 - 2^16, the tokens times the heads
 * below 2^28 - 2^16; offsets into the pool have 64 bits, a stride is below 2^31 bytes, n_pages * h_kv below 2^31.
 */
typedef struct {
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t page_stride, head_stride, tok_stride;
  int n_pages, page_size, h_kv, d;
  int dtype;                  /* the call's dtype, or ESA_E4M3 */
} esa_paged_cache;

/*
 * The call's sequences.  The new tokens of all of them lie one behind the other in n_tok rows: sequence b has rows
 * [cu[b], cu[b+1]) (none is allowed), which are its positions start[b], start[b] + 1, ...; rows behind cu[n_seq] belong to nobody.
 * Position p of sequence b is in page pages[b * pages_ld + p / page_size].  Entries of the table behind a sequence's last position
 * are not read.  A position without a page (beyond max_pages * page_size, or whose entry lies outside [0, n_pages)) is not written
 * and not seen.
 *   cu [n_seq + 1], start [n_seq], pages [n_seq][max_pages]: int32 on the device.  cu ascends from 0 to at most n_tok, start is not
 *   negative and no position reaches 2^31 (values that break this are clamped, the results are then unspecified)
 */
typedef struct {
  const int32_t* cu;
  const int32_t* start;
  const int32_t* pages;
  int64_t pages_ld;
  int64_t n_tok;
  int n_seq, max_pages;
} esa_paged_batch;

/*
 * Appends the new tokens' keys and values, the keys turned to their positions on the way, and turns the step's queries.
 *   k, v      [n_tok][h_kv, d], row strides ldk, ldv
 *   q, out_q  [n_tok][h, d] row strides ldq, ldoq; out_q may equal q when the strides are equal (in place).  q = NULL: keys and values only
 *   rope_base the encoding's base, as in esa_rope (pairs (i, i + d/2) turn by position * base^(-2i/d), fp64, rounded once into
 *             `dtype`); 0: rows are stored as they are and q must be NULL
 *   dtype     of k, v, q: ESA_F32 or ESA_BF16
 * ESA_E4M3: a block's scale is the smallest power of two with which 448, e4m3's largest number, covers the rows appended to it
 * (within 2^-100 ... 2^112; what is larger is held as the largest number, NaN as NaN).  A block whose earlier rows belong to the
 * sequence keeps its scale if that is larger and is brought to the new one otherwise; a block that begins with the first appended
 * row, or whose byte is 255, takes no heed of what the page held before.  Rows in `dtype` are rounded to the nearest e4m3 number, ties to even.
 * A page that is written to belongs to one sequence of the call and is listed once (pages that are only read may be shared): rows [start[b],
 * start[b] + new) of it are written, earlier ones only where the scale grows, later ones never.
 * The cache's k and v are two places, as are its scales (esa_attend_paged reads one place as both as well).
 * n_tok == 0 or n_seq == 0 is a no-op.  d: 32, 64, 128 or 256.  Rows of k, v, q and out_q start on 16-byte boundaries.
 */
ESA_API int esa_append_paged(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, int h, void* out_q,
               int64_t ldoq, const esa_paged_batch* batch, const esa_paged_cache* cache, double rope_base, int dtype, void* stream);

/*
 * Softmax attention of the new tokens over their sequence's pages, themselves included (their keys and values are in the cache):
 *   out[c,i] = sum_j softmax_j( f(scale * q[c,i].k[j,g]) ) v[j,g],   g = i / (h / h_kv),   f(x) = x, or cap * tanh(x / cap)
 * The token at position p = start[b] + c sees, of the positions up to its own,
 *   l_i >= start[b]        all of them (pass INT64_MAX for all sequences)
 *   otherwise              [0, i_end), the selected ones and [l_start, p], with i_end and l_start of esa_segments for t0 = start[b]
 *   idx  [n_seq][n_sel] int32, row stride idx_ld: the selected positions; an entry outside [i_end, l_start) is not seen (rows of
 *        different lengths end in -1), one that is listed twice counts twice.  NULL with n_sel = 0.
 *   cap  0: scores as they are; positive: capped (ESA_BF16: at most 4096, as a capped score is off by up to 2^-21 cap)
 *   q, out  [n_tok][h, d], row strides ldq, ldo; rows start on 16-byte boundaries; out does not overlap q
 *   lse  [n_tok][h] fp32 natural-log normaliser, or NULL
 *   workspace esa_attend_paged_workspace_bytes(n_tok, n_seq, h, h_kv, d, dtype) bytes, 256-byte aligned
 * A token that sees nothing (its pages are missing) has out = 0 and lse = -inf.  Rows of out and lse behind cu[n_seq] are left as
 * they were.  Keys and values that are seen must be finite, everything else in the pool may hold anything.  So must queries be, but that
 * one which holds a NaN makes its own row NaN, out and lse, if it sees anything, and no other.
 * Scores scale * q.k stay below 2^90 in magnitude, values below 2^90.
 * ESA_BF16: probabilities keep 16 bits, but 8 with d = 128 in a batch of more than 64 rows (tokens x h / h_kv) and more than 32 a sequence
 * in the mean, where only sequences of up to 64 may keep 16: outputs are then 2.3e-3 from the exact ones (relative, rms) instead of 1.66e-3,
 * as those of esa_attend's chunks with d = 128 are.
 * n_tok == 0 or n_seq == 0 is a no-op.  d: 32, 64, 128 or 256 (ESA_F32 with 256 by a plain kernel, far slower than the others).
 */
ESA_API size_t esa_attend_paged_workspace_bytes(int64_t n_tok, int n_seq, int h, int h_kv, int d, int dtype);
ESA_API int esa_attend_paged(const void* q, int64_t ldq, int h, const esa_paged_batch* batch, const esa_paged_cache* cache, int64_t l_i,
               int64_t l_l, const int32_t* idx, int n_sel, int64_t idx_ld, float scale, float cap, void* out, int64_t ldo, float* lse,
               int dtype, void* workspace, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ESA_PAGED_H */
