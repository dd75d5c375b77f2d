/*
 * libesa — what a serving step does around the paged cache of esa_paged.h: rotary positions of any layout and scaling, at positions that
 * lie on the device (esa_rope_at); the batch's offsets, block tables and slots, made from the sequences' lengths (esa_plan_paged);
 * and the verification of drafted tokens (esa_verify_drafts), whose counts are what the next plan grows the sequences by.
 * Conventions, error codes and error texts are those of esa.h: device pointers owned by the caller unless said otherwise, strides in
 * ELEMENTS, nothing allocated, kept or enqueued on an error, every call returns without synchronising and may be captured into a graph.
 * Lengths and positions lie on the device, so that a captured step serves those that it finds when it is replayed; nothing that these
 * arrays hold makes a kernel leave its buffers.
 */
#ifndef ESA_SERVE_H
#define ESA_SERVE_H

#include "esa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Which elements of a head turn together, of the first `rot`. */
#define ESA_PAIRS_HALVES 0      /* j and j + rot/2 */
#define ESA_PAIRS_NEIGHBOURS 1  /* 2j and 2j + 1 */

/* How the angle a position of pair j, f_j = base^(-2j/rot), is changed for contexts `factor` times as long. */
#define ESA_SCALE_NONE 0
#define ESA_SCALE_LINEAR 1 /* f_j / factor: positions are interpolated */
#define ESA_SCALE_NTK 2    /* the base becomes base * factor^(rot/(rot-2)): the slowest pair is divided by factor, the fastest stays */
#define ESA_SCALE_YARN 3   /* by parts: with r = length * f_j / (2 pi) turns in the original length and g = (r - slow) / (fast - slow), clamped
                              to [0, 1]: g f_j + (1 - g) f_j / factor */

/*
 * Host arithmetic (no GPU work): writes the rot/2 angles a position into the HOST array freq, which a program copies to the GPU once.
 *   base >= 1, rot even, 2 to 256; factor positive (not used by ESA_SCALE_NONE); length, fast > slow: ESA_SCALE_YARN only
 */
ESA_API int esa_rope_frequencies(double base, int rot, int scaling, double factor, double length, double fast, double slow, double* freq);

/* Rows of one tensor [n_tok][heads][d]: strides of tokens and heads in elements; out may equal x where their strides are equal (in place). */
typedef struct {
  const void* x;
  void* out;
  int64_t x_tok, x_head, out_tok, out_head;
  int heads;
} esa_rope_rows;

/*
 * Rotary encoding at given positions.  Token t's pair j turns by the angle a = pos[t] * freq[j], the same in every head of every tensor:
 *   x' = gain * (x cos a - y sin a),  y' = gain * (y cos a + x sin a)
 *   transposed != 0: by -a, which takes gradients of the encoded rows back to the rows (and, with a gain of 1, undoes the encoding)
 * Elements rot .. d of a head are copied.  A token of negative position belongs to nobody: its rows of out are left as they were.
 *   rows     n_rows of them, 1 or 2 (queries and keys); rows of one may be far apart or interleaved with another's, outputs
 *            must not overlap one another or another's input
 *   pos      [n_tok] int32
 *   d        2 <= rot <= d <= 1024, rot even, at most 256
 *   freq     [rot/2] float64 on the device, of magnitude 64 at most (angles beyond 2^38 lose their meaning, not more); gain finite
 * Angles, sines, cosines and products are fp64, rounded once into `dtype`.  n_tok == 0 is a no-op.  n_tok below 2^31 - 2^16.
 */
ESA_API int esa_rope_at(const esa_rope_rows* rows, int n_rows, const int32_t* pos, int64_t n_tok, int d, int rot, const double* freq, int pairs,
               double gain, int transposed, int dtype, void* stream);

/*
 * The pages of a pool (esa_paged.h) that sequences hold, and the ring of those that nobody holds.
 *   start [n_seq]    tokens that sequence b has in the cache          } read from *_in and written to the others, which may be the same
 *   held  [n_seq]    pages that it holds: entries [0, held[b])        } arrays (each call goes on from the last) or not (a call may then be
 *   ring_at [2]      place of the first free page, number of them     } repeated with the same outcome)
 *   pages [n_seq][max_pages], row stride pages_ld; ring [n_pages]: free pages, from ring[first] on, round the end
 *   page_size        16, 32, 64 or 128; max_pages * page_size below 2^31 - 2^16
 * A page is held once, by one sequence: one that several held (esa_attend_paged reads such tables) would come into the ring as often as it is given
 * back, and be handed out twice.
 * int32 on the device throughout.  A fresh pool: start = held = 0, ring = 0, 1, ... n_pages - 1, ring_at = {0, n_pages}.
 */
typedef struct {
  const int32_t *start_in, *held_in, *ring_at_in;
  int32_t *start, *held, *ring_at;
  int32_t* pages;
  int64_t pages_ld;
  int32_t* ring;
  int n_seq, max_pages, n_pages, page_size;
} esa_page_state;

/*
 * Begins a step of fresh[b] new tokens of sequence b: what esa_append_paged and esa_attend_paged read as cu, start and pages.
 *   start[b] = max(start_in[b] + grow[b], 0), but no position reaches 2^31 - 1; grow [n_seq] or NULL: what the step before has left in the cache (esa_verify_drafts'
 *           count, and rows that were not verified; minus what the sequence has ends it).  Tokens of one step that are not kept are written over by
 *           the next.
 *   cu [n_seq + 1]  cu[0] = 0, cu[b + 1] = min(cu[b] + max(fresh[b], 0), n_tok)
 *   With need = min(ceil((start[b] + cu[b + 1] - cu[b]) / page_size), max_pages): entries [need, held_in[b]) are given back, behind
 *   the free pages of the ring, sequence by sequence and in the order of the entries; then pages are taken from the front of the ring
 *   for entries [held_in[b], need), in the same order.  Those for which none is left become -1 and are not held; the next
 *   call tries again.  lack[0]: how many they are.  Other entries are left as they were.
 *   A sequence has all of its step where held[b] * page_size >= start[b] + cu[b + 1] - cu[b].  Where it has not (pages are lacking, or max_pages are too
 *   few), rows without a slot are stored nowhere, and the step must not count: the next call's grow[b] is 0 and the same tokens come again, or it ends.
 *   Grown all the same, the sequence would have positions that nothing was written for, and esa_attend_paged reads whatever lies there.
 *   pos [n_tok]   position of a row, -1 for rows behind cu[n_seq]
 *   slot [n_tok]  int64: page * page_size + pos % page_size, a row's place in an array of one entry a position of the pool; -1 for
 *                 rows behind cu[n_seq] and where there is no page (beyond max_pages, or an entry outside [0, n_pages))
 *   workspace     esa_plan_paged_workspace_bytes(state) bytes, 256-byte aligned; NULL where that is 0 (up to 4096 sequences, not in place)
 * What arrays hold that no sequence of calls leads to (a number of pages above max_pages or n_pages, say) is clamped, the outcome is then
 * unspecified.  n_seq == 0 is a no-op but for cu, lack, pos, slot and ring_at.
 * n_seq at most 2^24, n_tok below 2^31 - 2^16.  What is written overlaps nothing else (such a call is refused), but that start, held and ring_at
 * may be their *_in.
 */
ESA_API size_t esa_plan_paged_workspace_bytes(const esa_page_state* state);
ESA_API int esa_plan_paged(const esa_page_state* state, const int32_t* grow, const int32_t* fresh, int64_t n_tok, int32_t* cu, int32_t* pos,
               int64_t* slot, int32_t* lack, void* workspace, size_t ws_bytes, void* stream);

/*
 * Speculative sampling's verification.  Sequence b has rows [cu[b], cu[b + 1]) of a step: the last token that stands, then drafted ones.
 *   tokens  [n_tok] int32, the rows' tokens
 *   target  [n_tok][vocab] probabilities of the token that follows a row, as the target model has them (row stride ldt)
 *   draft   [n_tok][vocab] probabilities that the row's own token was drawn from (row stride ldd; a sequence's first row is not read), or
 *           NULL: tokens were not drawn but looked up, their probability is 1
 *   u       [n_tok] fp32 random numbers in [0, 1): a drafted row's decides whether it stands, that of the sequence's first row draws
 * With p and q for rows of target and draft: row i > cu[b] stands if all before it do and u[i] q_i(tokens[i]) < p_{i-1}(tokens[i]) (a
 * token outside [0, vocab) does not).  Behind the last row a that stands a token is drawn from w = max(p_a - q_{a+1}, 0), the draft
 * having been turned down, or, where there is none, from w = p_a: the lowest t with w_0 + ... + w_t > u[cu[b]] * (w_0 + ... + w_{vocab-1}).
 * Differences, products and sums are fp64; w need not sum to 1.  Probabilities that are negative, infinite or NaN count as 0; where all of
 * w is 0, w = p_a; where that is 0 too the token is -1.  A u that is negative or NaN draws as 0 does, one of
 * 1 or more the last token of positive weight; a draft does not stand by a u that is NaN.
 *   out     [n_tok] int32: the token that follows a row: tokens[i + 1] of rows before a, the drawn one of row a, -1 behind it
 *   count   [n_seq] int32: rows that stand, cu[b] among them, which is the number of new tokens too (a -1 that was drawn is counted); 0 for a sequence
 *           without rows
 * Every row behind a sequence's first one is taken for a draft.  A prompt's tokens are none: of a prompt the last row alone is verified, of one that
 * goes on in the next step nothing.  In a step that holds prompts cu, target, draft, tokens and u are those of the verified rows, one behind the other,
 * not the plan's, and a sequence grows by count and its rows that were not verified.
 * Rows behind cu[n_seq] are left as they were.  cu ascends from 0 to at most n_tok (other values are clamped, the results are then
 * unspecified).  dtype is that of target and draft: ESA_F32 or ESA_BF16.
 *   workspace esa_verify_drafts_workspace_bytes(n_seq, vocab) bytes, 256-byte aligned; NULL where that is 0 (vocabularies of up to 16384)
 * n_tok == 0: counts are 0.  n_seq == 0 is a no-op.  n_tok and vocab below 2^31 - 2^16, n_seq at most 2^24.  Rows may start at any element; those on 16-byte
 * boundaries are read fastest.  What is written overlaps nothing else (such a call is refused).
 */
ESA_API size_t esa_verify_drafts_workspace_bytes(int n_seq, int64_t vocab);
ESA_API int esa_verify_drafts(const void* target, int64_t ldt, const void* draft, int64_t ldd, const int32_t* tokens, const float* u, const int32_t* cu,
               int64_t n_tok, int n_seq, int64_t vocab, int32_t* out, int32_t* count, int dtype, void* workspace, size_t ws_bytes,
               void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ESA_SERVE_H */
