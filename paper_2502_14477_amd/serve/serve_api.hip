// The C ABI of the calls around the paged cache: argument validation and dispatch.
#include <cmath>

#include "serve.h"

using namespace esa;

namespace {

bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
constexpr int64_t kMost = INT32_MAX - 65535;      // rows and tokens: counters may run past them by a workgroup's stride
constexpr int kMostSeqs = 1 << 24;

// Rows [n_tok][heads][d] of which no two elements share a place, or, for inputs, any whose offsets stay within 64 bits.
bool strides_ok(int64_t n_tok, int64_t tok, int64_t heads, int64_t head, int64_t d, bool apart) {
  if (tok < 0 || head < 0 || tok > INT64_MAX / 16 / n_tok || head > INT64_MAX / 16 / heads) return false;
  if (!apart) return true;
  const bool tokens_inside = n_tok > 1 && (heads == 1 || tok < head);
  const int64_t inner = tokens_inside ? tok : head, inner_n = tokens_inside ? n_tok : heads;
  const int64_t outer = tokens_inside ? head : tok, outer_n = tokens_inside ? heads : n_tok;
  int64_t span = d;
  if (inner_n > 1) {
    if (inner < span) return false;
    span = inner * inner_n;
  }
  return outer_n == 1 || outer >= span - (inner_n > 1 ? inner - d : 0);
}

// Places of an array, and whether two share one; rows `ld` bytes apart, of `width` bytes each.
struct Span {
  uintptr_t lo, hi;
};
Span span(const void* p, int64_t n, size_t size) { return Span{(uintptr_t)p, (uintptr_t)p + (p ? (size_t)n * size : 0)}; }
bool meet(const Span& a, const Span& b) { return (a.lo < b.hi) & (b.lo < a.hi) & (a.lo < a.hi) & (b.lo < b.hi); }
bool meets_rows(const Span& a, const void* rows, int64_t n, int64_t ld, int64_t width) {
  if (n == 0 || !meet(a, span(rows, (n - 1) * ld + width, 1))) return false;
  if (a.lo <= (uintptr_t)rows) return true;
  const uintptr_t at = (a.lo - (uintptr_t)rows) % ld;
  return at < (uintptr_t)width || at + (a.hi - a.lo) > (uintptr_t)ld;
}

}  // namespace

extern "C" {

int esa_rope_frequencies(double base, int rot, int scaling, double factor, double length, double fast, double slow, double* freq) {
  const char* name = "esa_rope_frequencies";
  if (rot < 2 || rot > 2 * serve::kMaxHalf || rot % 2 != 0) ESA_FAIL(ESA_EINVAL, "%s: %d elements turn (even, 2 to %d)", name, rot, 2 * serve::kMaxHalf);
  if (!(base >= 1.0) || !std::isfinite(base) || !freq) ESA_FAIL(ESA_EINVAL, "%s: null array, or a base of %g (1 or more)", name, base);
  if (scaling < ESA_SCALE_NONE || scaling > ESA_SCALE_YARN) ESA_FAIL(ESA_EUNSUPPORTED, "%s: scaling %d", name, scaling);
  if (scaling != ESA_SCALE_NONE && (!(factor > 0.0) || !std::isfinite(factor))) ESA_FAIL(ESA_EINVAL, "%s: a factor of %g", name, factor);
  if (scaling == ESA_SCALE_YARN && (!(length > 0.0) || !std::isfinite(length) || !(fast > slow) || !std::isfinite(fast) || !std::isfinite(slow)))
    ESA_FAIL(ESA_EINVAL, "%s: a length of %g, turns from %g to %g", name, length, slow, fast);
  for (int j = 0; j < rot / 2; ++j) {
    double f = std::pow(base, -2.0 * j / rot);
    if (scaling == ESA_SCALE_LINEAR) f /= factor;
    if (scaling == ESA_SCALE_NTK && j > 0) f *= std::pow(factor, -2.0 * j / (rot - 2));      // (base factor^(rot/(rot-2)))^(-2j/rot)
    if (scaling == ESA_SCALE_YARN) {
      const double r = length * f / 6.283185307179586477, g = std::fmin(std::fmax((r - slow) / (fast - slow), 0.0), 1.0);
      f = g * f + (1.0 - g) * f / factor;
    }
    freq[j] = f;
  }
  return ESA_OK;
}

int esa_rope_at(const esa_rope_rows* rows, int n_rows, const int32_t* pos, int64_t n_tok, int d, int rot, const double* freq, int pairs,
                double gain, int transposed, int dtype, void* stream) {
  const char* name = "esa_rope_at";
  if (dtype != ESA_F32 && dtype != ESA_BF16) ESA_FAIL(ESA_EUNSUPPORTED, "%s: dtype %d", name, dtype);
  if (pairs != ESA_PAIRS_HALVES && pairs != ESA_PAIRS_NEIGHBOURS) ESA_FAIL(ESA_EUNSUPPORTED, "%s: pairs %d", name, pairs);
  if (d < 2 || d > 1024 || rot < 2 || rot > d || rot > 2 * serve::kMaxHalf || rot % 2 != 0)
    ESA_FAIL(ESA_EUNSUPPORTED, "%s: %d of %d elements of a head (even, at most %d, heads of 1024 at most)", name, rot, d, 2 * serve::kMaxHalf);
  if (!rows || n_rows < 1 || n_rows > serve::kMaxRowSets || n_tok < 0 || n_tok > kMost)
    ESA_FAIL(ESA_EINVAL, "%s: bad argument (n_rows=%d n_tok=%lld), or no rows", name, n_rows, (long long)n_tok);
  if (!std::isfinite(gain)) ESA_FAIL(ESA_EINVAL, "%s: a gain of %g", name, gain);
  const int64_t es = dtype == ESA_F32 ? 4 : 2;
  serve::RopeArgs a = {};
  bool copies = false;
  for (int k = 0; k < n_rows; ++k) {
    const esa_rope_rows& r = rows[k];
    if (r.heads <= 0 || r.heads > 65535) ESA_FAIL(ESA_EINVAL, "%s: %d heads", name, r.heads);
    if (n_tok == 0) continue;
    if (!r.x || !r.out || !aligned(r.x, (size_t)es) || !aligned(r.out, (size_t)es)) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned rows", name);
    if (!strides_ok(n_tok, r.x_tok, r.heads, r.x_head, d, false) || !strides_ok(n_tok, r.out_tok, r.heads, r.out_head, d, true))
      ESA_FAIL(ESA_EINVAL, "%s: strides of tokens %lld -> %lld, of heads %lld -> %lld: negative, or outputs overlap", name, (long long)r.x_tok,
               (long long)r.out_tok, (long long)r.x_head, (long long)r.out_head);
    if (r.x == r.out && ((n_tok > 1 && r.x_tok != r.out_tok) || (r.heads > 1 && r.x_head != r.out_head)))
      ESA_FAIL(ESA_EINVAL, "%s: in place needs equal strides", name);
    // a stride that nobody takes is no reason for smaller pieces
    const bool tok = n_tok > 1, head = r.heads > 1;
    a.set[k] = serve::RowSet{(const char*)r.x, (char*)r.out, tok ? r.x_tok * es : 0, head ? r.x_head * es : 0, tok ? r.out_tok * es : 0, head ? r.out_head * es : 0, r.heads};
    a.heads += r.heads;
    copies = copies || r.x != r.out;
  }
  if (n_tok == 0) return ESA_OK;
  if (n_rows == 2 && (rows[0].out == rows[1].out || rows[0].out == rows[1].x || rows[1].out == rows[0].x))
    ESA_FAIL(ESA_EINVAL, "%s: an output over the other's rows", name);
  if (!pos || !aligned(pos, 4) || !freq || !aligned(freq, 8)) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned positions or frequencies", name);
  a.pos = pos;
  a.freq = freq;
  a.gain = gain;
  a.n_tok = (int)n_tok;
  a.half = rot / 2;
  a.rest = copies ? d - rot : 0;
  a.pairs = pairs;
  a.transposed = transposed != 0;
  return serve::launch_rope_at(a, dtype, (hipStream_t)stream);
}

size_t esa_plan_paged_workspace_bytes(const esa_page_state* s) {
  if (!s || s->n_seq < 0 || s->n_seq > kMostSeqs) return 0;
  return serve::plan_workspace(s->n_seq, s->start == s->start_in || s->held == s->held_in || s->ring_at == s->ring_at_in);
}

int esa_plan_paged(const esa_page_state* state, const int32_t* grow, const int32_t* fresh, int64_t n_tok, int32_t* cu, int32_t* pos, int64_t* slot,
                   int32_t* lack, void* workspace, size_t ws_bytes, void* stream) {
  const char* name = "esa_plan_paged";
  if (!state) ESA_FAIL(ESA_EINVAL, "%s: null state", name);
  const esa_page_state& s = *state;
  if (s.page_size != 16 && s.page_size != 32 && s.page_size != 64 && s.page_size != 128)
    ESA_FAIL(ESA_EUNSUPPORTED, "%s: page_size %d (16, 32, 64 or 128)", name, s.page_size);
  if (s.n_seq < 0 || s.n_seq > kMostSeqs || s.max_pages <= 0 || s.pages_ld < s.max_pages || s.n_pages <= 0 || n_tok < 0 || n_tok > kMost)
    ESA_FAIL(ESA_EINVAL, "%s: bad size (n_seq=%d max_pages=%d pages_ld=%lld n_pages=%d n_tok=%lld)", name, s.n_seq, s.max_pages, (long long)s.pages_ld,
             s.n_pages, (long long)n_tok);
  if ((int64_t)s.max_pages * s.page_size > kMost || s.pages_ld > (INT64_MAX >> 28)) ESA_FAIL(ESA_EINVAL, "%s: more than 2^31-2^16 positions, or rows of the table too far apart", name);
  const void* always[] = {s.ring_at_in, s.ring_at, s.ring, cu, lack};
  const void* sequences[] = {s.start_in, s.held_in, s.start, s.held, s.pages, fresh};
  for (const void* p : always)
    if (!p || !aligned(p, 4)) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned pointer", name);
  for (const void* p : sequences)
    if (s.n_seq > 0 && (!p || !aligned(p, 4))) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned pointer", name);
  if (!aligned(grow, 4) || (n_tok > 0 && (!pos || !slot || !aligned(pos, 4) || !aligned(slot, 8)))) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned pointer", name);
  const size_t need = esa_plan_paged_workspace_bytes(state);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || ws_bytes < need))
    ESA_FAIL(ESA_EWORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned", name, need);
  // What is written lies apart from everything else: workgroups read while others write.  The first three may be what they are made from.
  const Span made_from[] = {span(s.start_in, s.n_seq, 4), span(s.held_in, s.n_seq, 4), span(s.ring_at_in, 2, 4), span(fresh, s.n_seq, 4), span(grow, s.n_seq, 4)};
  const Span written[] = {span(s.start, s.n_seq, 4), span(s.held, s.n_seq, 4), span(s.ring_at, 2, 4), span(s.ring, s.n_pages, 4), span(cu, (int64_t)s.n_seq + 1, 4),
                          span(lack, 1, 4), span(pos, n_tok, 4), span(slot, n_tok, 8), span(workspace, (int64_t)need, 1)};
  bool over = false;
  for (int i = 0; i < 9; ++i) {
    for (int j = 0; j < 5; ++j) over |= meet(written[i], made_from[j]) & !(i < 3 && i == j && written[i].lo == made_from[j].lo);
    for (int j = 0; j < i; ++j) over |= meet(written[i], written[j]);
    over |= meets_rows(written[i], s.pages, s.n_seq, s.pages_ld * 4, (int64_t)s.max_pages * 4);
  }
  for (const Span& x : made_from) over |= meets_rows(x, s.pages, s.n_seq, s.pages_ld * 4, (int64_t)s.max_pages * 4);
  if (over) ESA_FAIL(ESA_EINVAL, "%s: an array that is written overlaps another one", name);
  serve::PlanArgs a;
  a.start_in = s.start_in;
  a.held_in = s.held_in;
  a.ring_at_in = s.ring_at_in;
  a.grow = grow;
  a.fresh = fresh;
  a.start = s.start;
  a.held = s.held;
  a.ring_at = s.ring_at;
  a.pages = s.pages;
  a.ring = s.ring;
  a.cu = cu;
  a.pos = pos;
  a.lack = lack;
  a.slot = slot;
  a.pages_ld = s.pages_ld;
  a.n_seq = s.n_seq;
  a.max_pages = s.max_pages;
  a.n_pages = s.n_pages;
  a.page_log2 = __builtin_ctz((unsigned)s.page_size);
  a.n_tok = (int)n_tok;
  a.ws = workspace;
  return serve::launch_plan(a, (hipStream_t)stream);
}

size_t esa_verify_drafts_workspace_bytes(int n_seq, int64_t vocab) {
  return n_seq <= 0 || n_seq > kMostSeqs || vocab <= 0 || vocab > kMost ? 0 : serve::verify_workspace(n_seq, (int)vocab);
}

int esa_verify_drafts(const void* target, int64_t ldt, const void* draft, int64_t ldd, const int32_t* tokens, const float* u, const int32_t* cu,
                      int64_t n_tok, int n_seq, int64_t vocab, int32_t* out, int32_t* count, int dtype, void* workspace, size_t ws_bytes,
                      void* stream) {
  const char* name = "esa_verify_drafts";
  if (dtype != ESA_F32 && dtype != ESA_BF16) ESA_FAIL(ESA_EUNSUPPORTED, "%s: dtype %d", name, dtype);
  if (n_tok < 0 || n_tok > kMost || n_seq < 0 || n_seq > kMostSeqs || vocab <= 0 || vocab > kMost)
    ESA_FAIL(ESA_EINVAL, "%s: bad size (n_tok=%lld n_seq=%d vocab=%lld)", name, (long long)n_tok, n_seq, (long long)vocab);
  if (n_seq == 0) return ESA_OK;
  if (!cu || !count || !aligned(cu, 4) || !aligned(count, 4)) ESA_FAIL(ESA_EINVAL, "%s: null or misaligned pointer", name);
  const size_t es = dtype == ESA_F32 ? 4 : 2;
  if (n_tok > 0) {
    if (!target || !tokens || !u || !out || !aligned(target, es) || !aligned(draft, es) || !aligned(tokens, 4) || !aligned(u, 4) || !aligned(out, 4))
      ESA_FAIL(ESA_EINVAL, "%s: null or misaligned pointer", name);
    for (int64_t ld : {ldt, draft ? ldd : ldt})
      if (ld < vocab || ld > INT64_MAX / 16 / n_tok) ESA_FAIL(ESA_EINVAL, "%s: rows of %lld elements, %lld apart", name, (long long)vocab, (long long)ld);
  }
  const size_t need = esa_verify_drafts_workspace_bytes(n_seq, vocab);
  if (need > 0 && (!workspace || !aligned(workspace, 256) || ws_bytes < need))
    ESA_FAIL(ESA_EWORKSPACE, "%s: workspace needs %zu bytes, 256-byte aligned", name, need);
  // What is written lies apart from everything else: a sequence's workgroups read while another's write.
  const Span read[] = {span(tokens, n_tok, 4), span(u, n_tok, 4), span(cu, (int64_t)n_seq + 1, 4)};
  const Span written[] = {span(out, n_tok, 4), span(count, n_seq, 4), span(workspace, (int64_t)need, 1)};
  const int64_t width = vocab * (int64_t)es;
  bool over = false;
  for (int i = 0; i < 3; ++i) {
    for (const Span& x : read) over |= meet(written[i], x);
    for (int j = 0; j < i; ++j) over |= meet(written[i], written[j]);
    if (n_tok > 0) over |= meets_rows(written[i], target, n_tok, ldt * (int64_t)es, width) || (draft && meets_rows(written[i], draft, n_tok, ldd * (int64_t)es, width));
  }
  if (over) ESA_FAIL(ESA_EINVAL, "%s: an array that is written overlaps another one", name);
  serve::VerifyArgs a;
  a.target = (const char*)target;
  a.draft = (const char*)draft;
  a.ldt = ldt * (int64_t)es;
  a.ldd = ldd * (int64_t)es;
  a.tokens = tokens;
  a.cu = cu;
  a.u = u;
  a.out = out;
  a.count = count;
  a.n_tok = (int)n_tok;
  a.n_seq = n_seq;
  a.vocab = (int)vocab;
  a.ws = workspace;
  return serve::launch_verify(a, dtype, (hipStream_t)stream);
}

}  // extern "C"
