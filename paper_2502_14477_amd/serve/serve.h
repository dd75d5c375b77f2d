// What the kernels around the paged cache share.
#pragma once
#include "../paged/paged.h"
#include "esa_serve.h"

namespace esa {
namespace serve {

// ---------------------------------------------------------------- rotary positions
constexpr int kMaxRowSets = 2;
constexpr int kMaxHalf = 128;
struct RowSet {
  const char* x;
  char* out;
  int64_t x_tok, x_head, out_tok, out_head;      // bytes
  int heads;
};
struct RopeArgs {
  RowSet set[kMaxRowSets];
  const int32_t* pos;
  const double* freq;         // angle a position
  double gain;
  int n_tok, heads;           // heads: of all sets
  int half;                   // pairs
  int rest;                   // elements behind the pairs that have to be copied
  int pairs, transposed;
};
int launch_rope_at(const RopeArgs& a, int dtype, hipStream_t st);

// ---------------------------------------------------------------- plans
struct PlanArgs {
  const int32_t *start_in, *held_in, *ring_at_in, *grow, *fresh;
  int32_t *start, *held, *ring_at, *pages, *ring, *cu, *pos, *lack;
  int64_t* slot;
  int64_t pages_ld;
  int n_seq, max_pages, n_pages, page_log2, n_tok;
  void* ws;                   // null where plan_workspace is 0
};
size_t plan_workspace(int n_seq, bool in_place);
int launch_plan(const PlanArgs& a, hipStream_t st);

// ---------------------------------------------------------------- drafts
struct VerifyArgs {
  const char *target, *draft;      // draft null: looked up
  int64_t ldt, ldd;                // bytes
  const int32_t *tokens, *cu;
  const float* u;
  int32_t *out, *count;
  int n_tok, n_seq, vocab;
  void* ws;                        // null where verify_workspace is 0
};
size_t verify_workspace(int n_seq, int vocab);
int launch_verify(const VerifyArgs& a, int dtype, hipStream_t st);

}  // namespace serve
}  // namespace esa
