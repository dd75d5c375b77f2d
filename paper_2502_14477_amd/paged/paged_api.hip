// The C ABI of the paged cache: argument validation and dispatch.
#include <algorithm>

#include "paged.h"

using namespace esa;

namespace {

bool aligned(const void* p, size_t a) { return (uintptr_t)p % a == 0; }
bool head_size_ok(int d) { return d == 32 || d == 64 || d == 128 || d == 256; }

// Rows of `row` elements of es bytes, `ld` elements apart: on 16-byte boundaries, one behind the other.
bool rows_ok(const void* p, int64_t ld, int64_t row, int64_t es) { return aligned(p, 16) && ld >= row && ld * es % 16 == 0; }

constexpr int kFewRows = 64;      // of a sequence, new tokens x query heads of a KV head: up to two workgroups' share in the kernel for few rows
bool served_plainly(int d, int dtype) { return dtype == ESA_F32 && d == 256; }
bool in_many(int d, int dtype) { return dtype == ESA_BF16 && (d == 64 || d == 128); }      // whether the kernel for many rows takes it
constexpr int64_t kMostKeys = INT32_MAX - 65535;      // counters may run past them by a workgroup's stride
constexpr int64_t kMostRows = (1 << 28) - 65536;      // tokens x heads: what scans over the sequences count stays below 2^24 each

// Whether the pool's three dimensions, in any order, lie behind one another.
bool apart(const esa_paged_cache& c) {
  struct Dim {
    int64_t n, stride;
  } dims[3] = {{c.n_pages, c.page_stride}, {c.h_kv, c.head_stride}, {c.page_size, c.tok_stride}};
  std::sort(dims, dims + 3, [](const Dim& x, const Dim& y) { return x.stride < y.stride; });
  int64_t span = c.d;
  for (const Dim& x : dims) {
    if (x.n == 1) continue;
    if (x.stride < span || x.stride > INT64_MAX / 16 / x.n) return false;
    span = x.stride * x.n;
  }
  return true;
}

// What both calls ask of the batch and of the pool.
int common_ok(const char* name, const esa_paged_batch* b, const esa_paged_cache* c, int h, bool queries, int n_sel, int dtype) {
  if (!b || !c) ESA_FAIL(ESA_EINVAL, "%s: null batch or cache", name);
  if (dtype != ESA_F32 && dtype != ESA_BF16) ESA_FAIL(ESA_EUNSUPPORTED, "%s: dtype %d", name, dtype);
  if (c->dtype != dtype && c->dtype != ESA_E4M3) ESA_FAIL(ESA_EUNSUPPORTED, "%s: cache dtype %d beside dtype %d", name, c->dtype, dtype);
  if (b->n_tok < 0 || b->n_seq < 0 || b->max_pages <= 0 || b->pages_ld < b->max_pages || c->n_pages <= 0 || c->h_kv <= 0 || c->h_kv > 65535)
    ESA_FAIL(ESA_EINVAL, "%s: bad size (n_tok=%lld n_seq=%d max_pages=%d pages_ld=%lld n_pages=%d h_kv=%d)", name, (long long)b->n_tok, b->n_seq,
             b->max_pages, (long long)b->pages_ld, c->n_pages, c->h_kv);
  if (!head_size_ok(c->d)) ESA_FAIL(ESA_EUNSUPPORTED, "%s: head size %d (32, 64, 128 or 256)", name, c->d);
  if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128)
    ESA_FAIL(ESA_EUNSUPPORTED, "%s: page_size %d (16, 32, 64 or 128)", name, c->page_size);
  if (queries && (h <= 0 || h > 65535 || h % c->h_kv != 0)) ESA_FAIL(ESA_EINVAL, "%s: h=%d is not a multiple of h_kv=%d", name, h, c->h_kv);
  if ((int64_t)b->max_pages * c->page_size + n_sel > kMostKeys || b->n_tok > kMostRows / (queries && h > c->h_kv ? h : c->h_kv))
    ESA_FAIL(ESA_EINVAL, "%s: more than 2^31-2^16 positions, or 2^28-2^16 tokens times heads", name);
  if (b->n_tok == 0 || b->n_seq == 0) return ESA_OK;
  if (!b->cu || !b->start || !b->pages || !c->k || !c->v) ESA_FAIL(ESA_EINVAL, "%s: null pointer", name);
  if (!aligned(b->cu, 4) || !aligned(b->start, 4) || !aligned(b->pages, 4)) ESA_FAIL(ESA_EINVAL, "%s: misaligned pointer", name);
  const int64_t es = c->dtype == ESA_F32 ? 4 : c->dtype == ESA_BF16 ? 2 : 1;
  for (int64_t s : {c->page_stride, c->head_stride, c->tok_stride})
    if (s < c->d || s > INT64_MAX / 8 || s * es % 16 != 0) ESA_FAIL(ESA_EINVAL, "%s: a cache stride of %lld elements (at least d, whole 16 bytes)", name, (long long)s);
  for (int64_t s : {c->page_stride, c->head_stride, c->tok_stride})
    if (s * es > INT32_MAX) ESA_FAIL(ESA_EINVAL, "%s: a cache stride of %lld elements (below 2^31 bytes)", name, (long long)s);
  if ((int64_t)c->n_pages * c->h_kv > INT32_MAX) ESA_FAIL(ESA_EINVAL, "%s: more than 2^31 blocks", name);
  if (!apart(*c)) ESA_FAIL(ESA_EINVAL, "%s: elements of the cache overlap", name);
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) ESA_FAIL(ESA_EINVAL, "%s: misaligned cache", name);
  if (c->dtype == ESA_E4M3 && (!c->k_scale || !c->v_scale)) ESA_FAIL(ESA_EINVAL, "%s: an 8-bit cache needs its scales", name);
  return ESA_OK;
}

paged::Batch batch_of(const esa_paged_batch& b, int page_size) {
  paged::Batch x;
  x.cu = b.cu;
  x.start = b.start;
  x.pages = b.pages;
  x.pages_ld = b.pages_ld;
  x.n_tok = (int)b.n_tok;
  x.n_seq = b.n_seq;
  x.max_pages = b.max_pages;
  x.page_log2 = __builtin_ctz((unsigned)page_size);
  return x;
}
paged::Cache cache_of(const esa_paged_cache& c) {
  const int64_t es = c.dtype == ESA_F32 ? 4 : c.dtype == ESA_BF16 ? 2 : 1;
  paged::Cache x;
  x.k = (char*)c.k;
  x.v = (char*)c.v;
  x.k_scale = c.k_scale;
  x.v_scale = c.v_scale;
  x.page_bytes = (uint32_t)(c.page_stride * es);
  x.head_bytes = (uint32_t)(c.head_stride * es);
  x.tok_bytes = (uint32_t)(c.tok_stride * es);
  x.close = c.tok_stride * es * c.page_size <= (int64_t)UINT32_MAX ? c.page_size : 0;
  x.n_pages = c.n_pages;
  x.h_kv = c.h_kv;
  x.d = c.d;
  return x;
}

}  // namespace

extern "C" {

int esa_append_paged(const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, int h, void* out_q, int64_t ldoq,
                     const esa_paged_batch* batch, const esa_paged_cache* cache, double rope_base, int dtype, void* stream) {
  const int rc = common_ok("esa_append_paged", batch, cache, h, q != nullptr, 0, dtype);
  if (rc != ESA_OK) return rc;
  if (!(rope_base >= 0.0)) ESA_FAIL(ESA_EINVAL, "esa_append_paged: base must be positive, or 0 for rows as they are");
  if (q && rope_base == 0.0) ESA_FAIL(ESA_EINVAL, "esa_append_paged: queries without an encoding");
  if (batch->n_tok == 0 || batch->n_seq == 0) return ESA_OK;
  if (!k || !v || (q && !out_q)) ESA_FAIL(ESA_EINVAL, "esa_append_paged: null pointer");
  const int64_t es = dtype == ESA_F32 ? 4 : 2, row = (int64_t)cache->h_kv * cache->d;
  if (!rows_ok(k, ldk, row, es) || !rows_ok(v, ldv, row, es))
    ESA_FAIL(ESA_EINVAL, "esa_append_paged: rows of keys and values start on 16-byte boundaries and do not overlap");
  if (q && (!rows_ok(q, ldq, (int64_t)h * cache->d, es) || !rows_ok(out_q, ldoq, (int64_t)h * cache->d, es)))
    ESA_FAIL(ESA_EINVAL, "esa_append_paged: rows of queries start on 16-byte boundaries and do not overlap");
  if (q && q == out_q && ldq != ldoq) ESA_FAIL(ESA_EINVAL, "esa_append_paged: in place needs equal strides");
  if (cache->k == cache->v || (cache->dtype == ESA_E4M3 && cache->k_scale == cache->v_scale))
    ESA_FAIL(ESA_EINVAL, "esa_append_paged: keys and values in one place");
  return paged::launch_append(k, ldk, v, ldv, q, ldq, h, out_q, ldoq, batch_of(*batch, cache->page_size), cache_of(*cache),
                              cache->dtype == ESA_E4M3, rope_base, dtype, (hipStream_t)stream);
}

size_t esa_attend_paged_workspace_bytes(int64_t n_tok, int n_seq, int h, int h_kv, int d, int dtype) {
  if (n_tok <= 0 || n_seq <= 0 || h <= 0 || h_kv <= 0 || d <= 0 || h % h_kv != 0) return 256;
  if (served_plainly(d, dtype)) return 256;
  return std::max(paged::few_workspace(n_seq, h_kv, d, dtype), in_many(d, dtype) ? paged::many_workspace(h_kv, d) : 0);
}

int esa_attend_paged(const void* q, int64_t ldq, int h, const esa_paged_batch* batch, const esa_paged_cache* cache, int64_t l_i, int64_t l_l,
                     const int32_t* idx, int n_sel, int64_t idx_ld, float scale, float cap, void* out, int64_t ldo, float* lse, int dtype,
                     void* workspace, size_t ws_bytes, void* stream) {
  if (n_sel < 0 || l_i < 0 || l_l < 0) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: negative argument");
  const int rc = common_ok("esa_attend_paged", batch, cache, h, true, n_sel, dtype);
  if (rc != ESA_OK) return rc;
  // (times log2(e), and divided by a cap, it has to stay finite; the capped scores of bf16 are 2^-22 of the cap off)
  if (!(scale > 0.f) || !(scale < 1.0e38f)) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: scale must be positive and finite");
  if (!(cap >= 0.f) || !(cap < 3.0e38f)) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: cap must be finite and not negative");
  if (cap > 0.f && !(scale / cap < 1.0e38f)) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: a cap of %g with a scale of %g", (double)cap, (double)scale);
  if (cap > 4096.f && dtype == ESA_BF16) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: a cap of %g (bf16: at most 4096)", (double)cap);
  if (batch->n_tok == 0 || batch->n_seq == 0) return ESA_OK;
  if (!q || !out || q == out || (n_sel > 0 && !idx)) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: null pointer, or out over q");
  if (n_sel > 0 && (!aligned(idx, 4) || idx_ld < n_sel)) ESA_FAIL(ESA_EINVAL, "esa_attend_paged: misaligned index list, or rows that overlap");
  const int64_t es = dtype == ESA_F32 ? 4 : 2, row = (int64_t)h * cache->d;
  if (!rows_ok(q, ldq, row, es) || !rows_ok(out, ldo, row, es) || !aligned(lse, 4))
    ESA_FAIL(ESA_EINVAL, "esa_attend_paged: rows of q and out start on 16-byte boundaries and do not overlap");
  const size_t need = esa_attend_paged_workspace_bytes(batch->n_tok, batch->n_seq, h, cache->h_kv, cache->d, dtype);
  if (!workspace || !aligned(workspace, 256) || ws_bytes < need)
    ESA_FAIL(ESA_EWORKSPACE, "esa_attend_paged: workspace needs %zu bytes, 256-byte aligned", need);
  paged::AttendArgs a;
  a.batch = batch_of(*batch, cache->page_size);
  a.cache = cache_of(*cache);
  a.q = (const char*)q;
  a.out = (char*)out;
  a.lse = lse;
  a.idx = idx;
  a.ldq = ldq * es;
  a.ldo = ldo * es;
  a.idx_ld = idx_ld;
  a.h = h;
  a.group = h / cache->h_kv;
  a.n_sel = n_sel;
  a.l_i = (int)(l_i < INT32_MAX ? l_i : INT32_MAX);
  a.l_l = (int)(l_l < INT32_MAX ? l_l : INT32_MAX);
  a.scale = scale;
  a.cap = cap;
  const bool f8 = cache->dtype == ESA_E4M3;
  if (served_plainly(cache->d, dtype)) return paged::launch_plain(a, f8, (hipStream_t)stream);
  // The lengths are on the device, the mean is known.  A batch of few rows a sequence in the mean is served by the kernel for few rows, whatever
  // else is in it; other batches by both, one after the other in the same workspace, each of which finds the sequences that are its own.  One that
  // finds none takes 5 us and its join 5 more, while short sequences in the kernel for many rows cost no more than twice their time: where the
  // table has no room for more than 2^17 keys over all heads (8 tiles of 64 a workgroup, 15 us), that one serves them all.  (Chunks of 333 and 117
  // tokens over 5000 keys, 8 heads: 71 us by both, 63 by one.  Sixteen tokens of 16 thousand keys beside a long prompt: twice 270 us.)
  // Few rows in the mean with a chunk among them, 8-bit pages, 32 and 8 heads of 128 elements: 127 single tokens of 4000 keys beside a chunk of 896
  // 330 us by the kernel for few rows, 294 by both; 159 of 1000 beside a prompt of 1024 118 and 135, 255 of 500 beside a chunk of 100 79 and 101, 31
  // of 16 thousand beside a chunk of 220 264 and 261, eight of 4 tokens beside eight of 12 60 and 65.
  hipStream_t st = (hipStream_t)stream;
  const int64_t rows = batch->n_tok * a.group;
  if (!in_many(cache->d, dtype) || rows <= (int64_t)kFewRows || rows <= (int64_t)32 * batch->n_seq)
    return paged::launch_few(a, f8, dtype, INT32_MAX, workspace, st);
  const bool both = batch->n_seq > 1 && paged::most_keys_of(a) > (1 << 17) / ((int64_t)batch->n_seq * cache->h_kv);
  if (both) {
    const int few = paged::launch_few(a, f8, dtype, kFewRows, workspace, st);
    if (few != ESA_OK) return few;
  }
  return paged::launch_many(a, f8, both ? kFewRows : 0, workspace, st);
}

}  // extern "C"
