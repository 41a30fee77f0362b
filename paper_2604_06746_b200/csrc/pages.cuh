// A paged cache in 8 bits as the kernels see it.
#pragma once

#include "rope.cuh"

namespace skv {

constexpr int kBlockShift = 4, kBlockSlots = STRUCTKV_SCALE_BLOCK;   // slots that share a scale
constexpr int kLowExponent = -40;                                   // of a scale; 448 2^-40 is 4e-10

// Strides in bytes, s_page below 2^32.
struct PagesView {
  char *k, *v;
  unsigned char *k_scales, *v_scales;
  long long s_page, s_head, s_table;
  int s_token;
  const int* table;
  const int* lengths;
  int batch, n_kv, pages, page_shift, slots;                    // slots: of a sequence, columns of the table times slots of a page
  int* status;
};

struct AppendPagesArgs {
  PagesView c;
  Div by_splits, by_blocks, by_new;                             // blocks of slots that a sequence's rows may touch; n_new
  const char *k, *v;
  long long s_batch, s_token, s_head;
  int tokens, n_new, blocks, splits;                            // splits: CTAs that share a block's heads
  const int *counts, *index, *positions;
  long long s_index, s_positions;
  bool rotated;
  const char* q;
  long long q_batch, q_token, q_head;
  char* q_out;
  int heads, q_rows, head_step;                                 // q_rows: batch * n_new; head_step: heads that a lane takes
  int append_ctas;
};

struct RotateArgs {
  const char* x;
  char* out;
  long long x_batch, x_token, x_head, o_batch, o_token, o_head, s_positions;
  const int* positions;
  Div by_tokens;
  int rows, tokens, heads, head_step;                           // rows: batch * tokens
  bool inverse;
};

cudaError_t launch_rotate(const Ctx& ctx, const RopeArgs& r, const RotateArgs& a, cudaStream_t st);
int append_splits(long long blocks, int n_kv, int sms);
cudaError_t launch_append_pages(const Ctx& ctx, const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st);

// Heads that a lane takes one after another with the same angles: up to eight, as long as every SM has 1024 lanes at work.
inline int heads_at_once(long long rows, int lanes, int heads, int sms) {
  int n = 1;
  while (n < 8 && n < heads && rows * lanes * ((heads + 2 * n - 1) / (2 * n)) >= 1024ll * sms) n *= 2;
  return n;
}

#ifdef __CUDACC__

// New rows of sequence b that there is room for; n: its tokens.  -1: neither read nor written (the caller says so to the status word).
__device__ __forceinline__ int rows_of_sequence(const PagesView& c, const int* counts, int b, int n_new, int& n) {
  n = c.lengths[b];
  const int count = counts ? counts[b] : n_new;
  return n < 0 || count < 0 || count > n_new || n > c.slots - count ? -1 : count;
}
__device__ __forceinline__ void tell_invalid(const PagesView& c) { atomicCAS(c.status, 0, (int)STRUCTKV_ERR_INVALID_ARG); }

#endif  // __CUDACC__
}  // namespace skv
