// Attention of new tokens over a paged cache in 8 bits, what its kernels share: how the work is cut and partial results.
//
// An item is (sequence b, KV head g, block of up to RB rows) over the sequence's keys, lengths[b] old ones and count[b] new ones; row r =
// i G + h is new token i and head h of the group.  Items follow one another, sequence after sequence; their tiles of 64 keys, behind `over`
// places for what an item costs beside them, form one sequence of W places, of which C CTAs take runs that differ by one place at
// most.  What a CTA has of an item it leaves as a partial, in slot item + CTA (no other pair has it); a second launch merges an
// item's in order: results do not depend on timing.
#pragma once

#include "pages.cuh"

namespace skv {

struct AttendPagesArgs {
  PagesView c;
  Div by_blocks, by_group, by_ctas, by_rows, by_kv;
  const char* q;
  long long q_batch, q_token, q_head;
  const int* counts;
  int n_new, group, rows, blocks;                               // rows = n_new group; blocks of rows
  float scale2, cap2, inv_cap;                                  // as in AttendArgs
  char* out;
  float* lse;
  int2* item_parts;                                             // [item] its first partial's slot, and how many it has
  float2* part_stat;                                            // [slot][RB] reference (bits) and sum
  float* part_out;                                              // [slot][RB][d]
  int ctas, over;
};

// Rows of a block, CTAs that run at once, places of an item's own cost.
struct PagesPlan { int rb, ctas, over; };

cudaError_t launch_attend_pages(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st);
cudaError_t launch_attend_pages_tc(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st);
cudaError_t launch_attend_pages_finish(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st);

#ifdef __CUDACC__

constexpr float kRaise = 7.f;          // weights are up to 2^(kRaise + kSlack), the largest above 2^(kRaise - 1): fp16 keeps 11 bits of those down to 2^-20 of it, some down to 2^-30
constexpr float kNothing = -3.4e38f;   // reference of a row that has seen nothing

// Codes of a word's lower and upper half as two fp16 each.
__device__ __forceinline__ uint32_t half_lo(uint32_t w) {
  uint32_t x;
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %1;\ncvt.rn.f16x2.e4m3x2 %0, a;\n}" : "=r"(x) : "r"(w));
  return x;
}
__device__ __forceinline__ uint32_t half_hi(uint32_t w) {
  uint32_t x;
  asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %1;\ncvt.rn.f16x2.e4m3x2 %0, b;\n}" : "=r"(x) : "r"(w));
  return x;
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// A word's bytes that are NaN codes, as 0x80 of each.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ float exp2i(int e) { return __int_as_float(min(max(127 + e, 1), 254) << 23); }   // within fp32's normal numbers

// Keys of sequence b, old ones (n) and new ones; 0: nothing of it is looked at.
__device__ __forceinline__ int page_keys(const AttendPagesArgs& a, int b, int& n) {
  const int count = rows_of_sequence(a.c, a.counts, b, a.n_new, n);
  if (count < 0) tell_invalid(a.c);
  return count <= 0 ? 0 : n + count;
}
__device__ __forceinline__ int page_tiles(int keys) { return (keys + 63) >> 6; }

// A CTA's run of places and where it begins: sequence, its keys, places of one item before it.
struct PageRun { int lo, hi, b, before, keys, n; Shares all; };
__device__ __forceinline__ PageRun find_run(const AttendPagesArgs& a) {
  const int lane = threadIdx.x & 31, items = a.c.n_kv * a.blocks;
  int total = 0, keys = 0, n = 0, places = 0, incl = 0;
  auto sweep = [&](int b0) {
    keys = b0 + lane < a.c.batch ? page_keys(a, b0 + lane, n) : 0;
    places = incl = keys == 0 ? 0 : page_tiles(keys) + a.over;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
  };
#pragma unroll 1
  for (int b0 = 0; b0 < a.c.batch; b0 += 32) {
    sweep(b0);
    total += __shfl_sync(0xffffffffu, incl, 31);
  }
  PageRun w{};
  w.all = shares_of(total * items, a.ctas, a.by_ctas, 0);
  w.lo = first_of(w.all, blockIdx.x);
  w.hi = first_of(w.all, blockIdx.x + 1);
  if (w.lo >= w.hi) return w;
  int before = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < a.c.batch; b0 += 32) {
    if (a.c.batch > 32) sweep(b0);
    const unsigned mine = __ballot_sync(0xffffffffu, (before + incl) * items > w.lo);
    if (mine) {
      const int from = __ffs(mine) - 1;
      w.b = b0 + from;
      w.before = before + __shfl_sync(0xffffffffu, incl - places, from);
      w.keys = __shfl_sync(0xffffffffu, keys, from);
      w.n = __shfl_sync(0xffffffffu, n, from);
      break;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return w;
}

// A CTA's run item by item: tiles [t0, t1) of item `nth` of sequence b (none left: t1 = 0).
struct PageSegment { int b, nth, t0, t1, keys, n, tiles, at, hi; };
__device__ __forceinline__ void next_segment(PageSegment& s, const AttendPagesArgs& a) {
  s.at += s.tiles + a.over;
  s.t0 = s.t1 = 0;
  if (s.at + a.over >= s.hi) return;
  if (++s.nth == a.c.n_kv * a.blocks) {
    s.nth = 0;
    do ++s.b;
    while ((s.keys = page_keys(a, s.b, s.n)) == 0 && s.b < a.c.batch - 1);
    s.tiles = page_tiles(s.keys);
  }
  s.t1 = min(s.tiles, s.hi - s.at - a.over);
}
__device__ __forceinline__ PageSegment first_segment(const AttendPagesArgs& a, const PageRun& w) {
  const int items = a.c.n_kv * a.blocks;
  PageSegment s{w.b, 0, 0, 0, w.keys, w.n, page_tiles(w.keys), w.before * items, w.hi};
  if (w.lo >= w.hi) return s;
  const int each = s.tiles + a.over;
  s.nth = (w.lo - s.at) / each;
  s.at += s.nth * each;
  s.t0 = max(0, w.lo - s.at - a.over);
  s.t1 = max(0, min(s.tiles, w.hi - s.at - a.over));
  if (s.t1 <= s.t0) next_segment(s, a);
  return s;
}

#endif  // __CUDACC__
}  // namespace skv
