// Attention of new tokens over a compacted cache, what its kernels share: how the work is cut, partial results, options.
//
// A unit is (sequence, KV head) u = b H_kv + g, with lengths[u] + n_new keys (the new tokens are the last ones) and rows
// r = i G + h, new token i and head h of the group.  An item is a unit's block of up to RB rows over all of its keys; items
// follow one another unit after unit, and their key tiles, behind the places of 512 keys for what an item costs beside them, form one sequence of
// W places.  C CTAs take runs of it whose lengths differ by one place at most: every CTA has equally much to do whatever the lengths,
// which only the device knows.  (Without the places for the items' own cost a CTA that gets eight KV heads of one token is busy twice as
// long as the others: figures at kOverKeys.)  What a CTA has of an item it leaves as a partial (row references, sums, unscaled output) in slot item + CTA, which no other pair has, so that an
// item's partials lie side by side; attend_finish() merges them in that order: results do not depend on timing.  (Merged by the CTA
// that leaves an item's last partial, which spares the launch, 1 x 1024 keys took 16.8 us when that version's two launches took 13.4,
// which are down to 9.1 now: all of the merging stands in one row behind the last tile, on one SM.)
#pragma once

#include <atomic>

#include "common.cuh"
#include "score_tc.cuh"

namespace skv {

// Keys whose places are an item's own cost: a launch's AttendArgs::over is that in tiles.  (us, bf16, 32 heads over 8, with 0 / 256 / 512 keys
// in attend_mma, whose tiles have 64: 16 sequences of 1 to 5003 keys 56.0 / 32.9 / 28.6, 3 tokens over 4 x 4096 keys 20.1 / 18.0 /
// 16.9; in attend_tc, 128, with 0 / 512 / 1024: 8 tokens over the 16 sequences 51.4 / 35.4 / 38.7, 64 over 8 x 8192 keys 94.5 / 91.2 /
// 94.9; a speculative step over 4 x 4096 keys whose weighing has 0 / 256 / 512: 43.8 / 43.4 / 47.3.)
constexpr int kOverKeys = 512, kWeighOverKeys = 256;
constexpr int kMaxNew = STRUCTKV_MAX_NEW;   // new tokens of a sequence: a tree's masks are words of 64 bits

// The cache as the kernels see it; strides in bytes, words [batch, H_kv, capacity], lengths [batch, H_kv].
struct CacheView {
  char *k, *v;
  long long s_batch, s_head, s_token;
  int* positions;
  float* weights;
  int* lengths;
  int units, n_kv, capacity, row_bytes;
  int* status;
};
inline __host__ __device__ size_t unit_offset(const CacheView& c, int u) {
  return (size_t)(u / c.n_kv) * c.s_batch + (size_t)(u % c.n_kv) * c.s_head;
}

struct NewRows { const char *k, *v; long long s_batch, s_token, s_head; const int* positions; };

// Division by a number that the launch knows, of n < 2^31.
struct Div { unsigned mul, shift; };
inline Div div_by(unsigned d) {
  unsigned s = 0;
  while (1ull << s < d) ++s;
  return {(unsigned)((((1ull << s) - d) << 32) / d + 1), s};
}

struct AttendArgs {
  CacheView c;
  Div by_kv, by_group, by_rows, by_ctas;   // H_kv, group, rows, ctas
  const char* q;                       // element strides in bytes
  long long q_batch, q_token, q_head;
  int n_new, group, rows;              // rows = n_new * group
  float scale2;                        // scale log2(e)
  float cap2, inv_cap;                 // softcap log2(e) and scale / softcap; cap2 = 0: none
  const float* slopes;                 // [H] or NULL
  const unsigned long long* tree;      // [batch, n_new] or NULL
  float decay;
  char* out;                           // [batch, n_new, H, d]
  float* lse;                          // [batch, n_new, H] or NULL
  bool accumulate;                     // (n_new = 1)
  NewRows fresh;                       // the new tokens' rows, where the kernel appends them; k NULL: they are in the cache
  // workspace
  int* unit_start;                     // [units + 1] places before a unit, of one block of rows
  float2* part_stat;                   // [slot][RB] reference (bits) and sum
  float* part_out;                     // [slot][RB][d]
  float* logits;                       // [units][capacity][group] in bits (accumulate)
  int ctas, least, over;               // CTAs; log2 of the tiles that one of them has at least; places before an item's tiles
};

// Rows of a block, keys of a tile, CTAs that run at once, partials a CTA leaves of an item, log2 of the tiles it takes at least.
struct AttendPlan { int rb, tile, ctas, parts, least; };

cudaError_t launch_append(const CacheView& c, const NewRows& r, int n_new, cudaStream_t st);
cudaError_t launch_commit(const CacheView& c, int n_new, const int* counts, const int* path, cudaStream_t st);
cudaError_t launch_evict(const CacheView& c, int budget, int recent, cudaStream_t st);
// The kernels: fp32 storage on the CUDA cores; bf16 storage.
cudaError_t launch_attend_simt(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
cudaError_t launch_attend_mma(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
cudaError_t launch_attend_tc(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
cudaError_t launch_attend_finish(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
// weights[j] = decay weights[j] + the sum of exp(x - lse) over the rows of the accepted new tokens.
cudaError_t launch_weigh_fp32(const Ctx& ctx, const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st);
cudaError_t launch_weigh_bf16(const Ctx& ctx, const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st);

#ifdef __CUDACC__

// Raises a kernel's limit of dynamic shared memory, once a device.
template <auto Kernel>
inline cudaError_t allow_smem(int bytes) {
  static std::atomic<unsigned long long> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (ready.load(std::memory_order_acquire) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) ready.fetch_or(bit, std::memory_order_release);
  return e;
}

// Keys of a unit of length n, 0 where that is none: the caller is told, nothing of the unit is read or written.
__device__ __forceinline__ int keys_of(const CacheView& c, int n, int n_new) {
  if (n < 0 || n > c.capacity - n_new) {
    atomicCAS(c.status, 0, (int)STRUCTKV_ERR_INVALID_ARG);
    return 0;
  }
  return n + n_new;
}
__device__ __forceinline__ int unit_keys(const CacheView& c, int u, int n_new) { return keys_of(c, c.lengths[u], n_new); }

// Rows, positions and weight 0 of a unit's new tokens, by a warp: to slots n and up.
__device__ __forceinline__ void append_rows(const CacheView& c, const NewRows& r, int n_new, int u, int b, int g, int n, int lane) {
  const size_t off = unit_offset(c, u);
  const int per_row = c.row_bytes / 16;
  for (int tok = 0; tok < n_new; ++tok) {
    const size_t from = (size_t)b * r.s_batch + (size_t)tok * r.s_token + (size_t)g * r.s_head, to = off + (size_t)(n + tok) * c.s_token;
    for (int i = lane; i < 2 * per_row; i += 32) {
      const int ch = i < per_row ? i : i - per_row;
      *(uint4*)((i < per_row ? c.k : c.v) + to + ch * 16) = *(const uint4*)((i < per_row ? r.k : r.v) + from + ch * 16);
    }
  }
  const size_t w = (size_t)u * c.capacity + n;
  for (int i = lane; i < n_new; i += 32) {
    c.positions[w + i] = r.positions[(size_t)b * n_new + i];
    if (c.weights) c.weights[w + i] = 0.f;
  }
}

__device__ __forceinline__ int quotient(int n, Div d) { return (int)((__umulhi((unsigned)n, d.mul) + (unsigned)n) >> d.shift); }

// How W places are shared out: CTA c has [first(c), first(c + 1)), at least 2^least of them if there are as many.
struct Shares { int W, C, each, more; };
__device__ __forceinline__ Shares shares_of(int W, int ctas, Div by_ctas, int least) {
  if (W >> least >= ctas) {
    const int each = quotient(W, by_ctas);
    return {W, ctas, each, W - each * ctas};
  }
  // (W = C 2^least + r, r below 2^least, at most 3)
  const int C = max(1, W >> least), r = W >= 1 << least ? W & ((1 << least) - 1) : 0;
  const int each = W >= 1 << least ? (1 << least) + (r >= C) + (r >= 2 * C) + (r >= 3 * C) : W;
  return {W, C, each, W - each * C};
}
__device__ __forceinline__ int first_of(const Shares& s, int c) { return c >= s.C ? s.W : c * s.each + min(c, s.more); }
__device__ __forceinline__ int cta_of(const Shares& s, int x) {
  const int line = s.more * (s.each + 1);
  const bool low = x < line;
  const int n = low ? x : x - line, d = low ? s.each + 1 : s.each;
  int q = (int)__fdividef((float)n, (float)d);                   // below 2^10: off by one at most
  q -= q * d > n;
  q += (q + 1) * d <= n;
  return (low ? 0 : s.more) + q;
}

__device__ __forceinline__ int tiles_of(int keys, int tile_shift) { return (keys + (1 << tile_shift) - 1) >> tile_shift; }
__device__ __forceinline__ int places_of(int keys, int tile_shift, int over) { return keys == 0 ? 0 : tiles_of(keys, tile_shift) + over; }

// First partial of an item and how many it has; each: partials a CTA leaves of an item.
struct Parts { int first, count; };
__device__ __forceinline__ Parts parts_of(const Shares& s, int item, int start, int places, int each, int over) {
  const int c0 = cta_of(s, start + over), c1 = cta_of(s, start + places - 1);
  return {(item + c0) * each, (c1 - c0 + 1) * each};
}

// A CTA's run of places, and the unit that its first one is in: keys, places of one block of rows before it.
struct WorkStart { int lo, hi, unit, before, keys; };

// By the whole block, every warp for itself; a lane has `kLaneUnits` neighbouring units of a sweep.  save: unit_start.
constexpr int kLaneUnits = 4;
__device__ __forceinline__ WorkStart find_work(const AttendArgs& a, int tile_shift, int blocks, int* save) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  int keys[kLaneUnits], incl = 0, total = 0, sum = 0;
  auto sweep = [&](int u0) {
    sum = 0;
#pragma unroll
    for (int e = 0; e < kLaneUnits; ++e) keys[e] = c.lengths[min(u0 + lane * kLaneUnits + e, c.units - 1)];   // (all loads, then the checks)
#pragma unroll
    for (int e = 0; e < kLaneUnits; ++e) keys[e] = u0 + lane * kLaneUnits + e < c.units ? keys_of(c, keys[e], a.n_new) : 0;
#pragma unroll
    for (int e = 0; e < kLaneUnits; ++e) sum += places_of(keys[e], tile_shift, a.over);
    incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int t = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += t;
    }
  };
  // (one sweep where it holds all units; the sum of all is known only after all of them, so that else a second pass follows)
  constexpr int kSweep = 32 * kLaneUnits;
#pragma unroll 1
  for (int u0 = 0; u0 < c.units; u0 += kSweep) {
    sweep(u0);
    if (save && threadIdx.x < 32) {
      int at = total + incl - sum;
#pragma unroll
      for (int e = 0; e < kLaneUnits; ++e) {
        const int u = u0 + lane * kLaneUnits + e;
        if (u < c.units) save[u] = at;
        at += places_of(keys[e], tile_shift, a.over);
      }
    }
    total += __shfl_sync(0xffffffffu, incl, 31);
  }
  if (save && threadIdx.x == 0) save[c.units] = total;
  WorkStart w{};
  const Shares all = shares_of(total * blocks, a.ctas, a.by_ctas, a.least);
  w.lo = first_of(all, blockIdx.x);
  w.hi = first_of(all, blockIdx.x + 1);
  if (w.lo >= w.hi) return w;
  int before = 0;
#pragma unroll 1
  for (int u0 = 0; u0 < c.units; u0 += kSweep) {
    if (c.units > kSweep) sweep(u0);
    const unsigned mine = __ballot_sync(0xffffffffu, (before + incl) * blocks > w.lo);
    if (mine) {
      const int from = __ffs(mine) - 1;
      int at = before + __shfl_sync(0xffffffffu, incl - sum, from);
#pragma unroll
      for (int e = 0; e < kLaneUnits; ++e) {
        const int k = __shfl_sync(0xffffffffu, keys[e], from), t = places_of(k, tile_shift, a.over);
        if (at * blocks <= w.lo && w.lo < (at + t) * blocks) {
          w.unit = u0 + from * kLaneUnits + e;
          w.before = at;
          w.keys = k;
        }
        at += t;
      }
      break;
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return w;
}

// A CTA's run, item by item: tiles [t0, t1) of an item's.  (None left: t1 = 0.)
struct Segments {
  int u, rb, t0, t1, keys, tiles;
  int at, hi;                                                    // place where the item begins, where the run ends
};
__device__ __forceinline__ void next_segment(Segments& s, const AttendArgs& a, int tile_shift, int blocks) {
  s.at += s.tiles + a.over;
  s.t0 = s.t1 = 0;
  if (s.at + a.over >= s.hi) return;
  if (++s.rb == blocks) {
    s.rb = 0;
    do ++s.u;
    while ((s.keys = unit_keys(a.c, s.u, a.n_new)) == 0 && s.u < a.c.units - 1);
    s.tiles = tiles_of(s.keys, tile_shift);
  }
  s.t1 = min(s.tiles, s.hi - s.at - a.over);
}
__device__ __forceinline__ Segments first_segment(const AttendArgs& a, const WorkStart& w, int tile_shift, int blocks) {
  Segments s{w.unit, 0, 0, 0, w.keys, tiles_of(w.keys, tile_shift), w.before * blocks, w.hi};
  if (w.lo >= w.hi) return s;
  while (w.lo >= s.at + s.tiles + a.over) {
    s.at += s.tiles + a.over;
    ++s.rb;
  }
  s.t0 = max(0, w.lo - s.at - a.over);
  s.t1 = max(0, min(s.tiles, w.hi - s.at - a.over));
  if (s.t1 <= s.t0) next_segment(s, a, tile_shift, blocks);
  return s;
}

// cap tanh(y) in bits of two scores, y = scale s / cap: tanh(y) = y P(y^2) / Q(y^2), relatively exact down to zero (cap - 2 cap / (e^2y + 1)
// cancels there: off by 2^-22 cap whatever the score).  P and Q of degree four approximate tanh(y) / y on |y| <= 8.7, where tanh is 1 to 24
// bits, with the least largest relative error (1.5e-8; least squares of P - Q tanh(y) / y, reweighted by the error until it is level:
// Lawson's method); in fp32 tanh is off by 2^-21.4 at most, and by 2^-23 more for the reciprocal.  Infinite y give cap, NaN stays NaN.
// Packed instructions: one score at a time a tree of 16 over eight ragged sequences takes 44 us, so 30, and with e^2y 31.
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float within(float y, float end) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(y) : "f"(end));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(y) : "f"(-end));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void capped2(float& a, float& b, uint64_t cap2, uint64_t inv_cap) {
  const float P[5] = {1.3962095e-8f, 2.104377e-5f, 3.5219393e-3f, 1.3403216e-1f, 1.f};
  const float Q[5] = {8.0239e-7f, 3.328758e-4f, 2.5977228e-2f, 4.673654e-1f, 1.f};
  constexpr float kEnd = 8.7f;
  float y0, y1, q0, q1;
  unpack2(mul2(pack2(a, b), inv_cap), y0, y1);
  const uint64_t y = pack2(within(y0, kEnd), within(y1, kEnd)), z = mul2(y, y);
  uint64_t p = pack2(P[0], P[0]), q = pack2(Q[0], Q[0]);
#pragma unroll
  for (int i = 1; i < 5; ++i) {
    p = fma2(p, z, pack2(P[i], P[i]));
    q = fma2(q, z, pack2(Q[i], Q[i]));
  }
  unpack2(q, q0, q1);
  unpack2(mul2(cap2, mul2(mul2(y, p), pack2(reciprocal(q0), reciprocal(q1)))), a, b);
}

// The new tokens that row r of a unit sees, as bits.
__device__ __forceinline__ unsigned long long row_seen(const AttendArgs& a, int u, int r) {
  const int i = quotient(r, a.by_group);
  return a.tree ? a.tree[(size_t)quotient(u, a.by_kv) * a.n_new + i] : (i == 63 ? ~0ull : (1ull << (i + 1)) - 1);
}
// A row's option values.
struct RowOptions { unsigned long long seen; float slope2; int position; };
__device__ __forceinline__ RowOptions row_options(const AttendArgs& a, int u, int r) {
  RowOptions o;
  o.seen = row_seen(a, u, r);
  o.slope2 = 0.f;
  o.position = 0;
  if (a.slopes) {
    const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, i = quotient(r, a.by_group), h = r - i * a.group;
    o.slope2 = a.slopes[g * a.group + h] * kLog2e;
    o.position = a.fresh.k ? a.fresh.positions[(size_t)b * a.n_new + i] : a.c.positions[(size_t)u * a.c.capacity + a.c.lengths[u] + i];
  }
  return o;
}
// Whether key j of a unit whose first n tokens are old is seen.
__device__ __forceinline__ bool sees(unsigned long long mask, int j, int n) { return j < n || (mask >> ((j - n) & 63) & 1); }

// x in bits from the products of rows and keys, two at a time, but for the bias; and with it.
__device__ __forceinline__ void in_bits2(const AttendArgs& a, float& s0, float& s1) {
  if (a.cap2 != 0.f) capped2(s0, s1, pack2(a.cap2, a.cap2), pack2(a.inv_cap, a.inv_cap));
  else {
    s0 *= a.scale2;
    s1 *= a.scale2;
  }
}
__device__ __forceinline__ float biased(const AttendArgs& a, float x, const RowOptions& o, int key_position) {
  return a.slopes ? fmaf(-o.slope2, (float)(o.position - key_position), x) : x;
}

// Maps of a cache's K and V, and a copy of a tile's slots: 64 columns after 64 columns, rows of 128 bytes, 128-byte swizzle.
struct CacheMaps { CUtensorMap k, v; };
inline bool cache_maps(const Ctx& ctx, const AttendArgs& a, int tile, CacheMaps* m) {
  const CacheView& c = a.c;
  const int batch = c.units / c.n_kv;
  return tc_encode_cache(ctx, &m->k, c.k, c.capacity, c.n_kv, batch, c.s_token, c.s_head, c.s_batch, tile) &&
         tc_encode_cache(ctx, &m->v, c.v, c.capacity, c.n_kv, batch, c.s_token, c.s_head, c.s_batch, tile);
}
__device__ __forceinline__ void tma_load_slots(uint32_t dst, const CUtensorMap* map, uint32_t bar, int slot, int head, int seq, uint64_t policy) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
      "[%0], [%1, {%3, %4, %3, %5, %6}], [%2], %7;"
      ::"r"(dst), "l"((uint64_t)map), "r"(bar), "r"(0), "r"(slot), "r"(head), "r"(seq), "l"(policy) : "memory");
}
// Where 16-byte chunk `chunk` of a row lies in a tile of ROWS rows.
template <int ROWS>
__device__ __forceinline__ uint32_t tile_at(int row, int chunk) { return (chunk >> 3) * (ROWS * 128) + row * 128 + (((chunk ^ row) & 7) << 4); }
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Whether one of two bf16 is infinite or NaN.
__device__ __forceinline__ bool not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
// A row's reference follows its maximum only where that outgrows it by 2^kSlack.
constexpr float kSlack = 8.f;

// A segment's end, by NT threads: the outputs of `sets` warps (a multiple of four) in shared memory, [set][RB][ROW] each against its own
// reference, with references and sums [RB][SETS], become a partial.  sync: a barrier of the NT threads; none at the end.
template <int D, int NT, int RB, int ROW, int SETS, typename Sync>
__device__ __forceinline__ void leave_partial(const AttendArgs& a, int slot, int rows, const float* out, const float* refs, const float* sums,
                                              int sets, int t, Sync sync) {
  sync();
#pragma unroll 1
  for (int i = t; i < rows * (D / 4); i += NT) {
    const int row = i / (D / 4), c4 = i % (D / 4);
    float ref[SETS], top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < SETS; w += 4) {
      const float4 x = *(const float4*)(refs + row * SETS + w);
      ref[w] = x.x; ref[w + 1] = x.y; ref[w + 2] = x.z; ref[w + 3] = x.w;
      if (w < sets) top = fmaxf(fmaxf(fmaxf(top, x.x), fmaxf(x.y, x.z)), x.w);
    }
    const float base = top == -INFINITY ? 0.f : top;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* from = out + row * ROW + c4 * 4;
#pragma unroll
    for (int w = 0; w < SETS; w += 4)
      if (w < sets) {
        const float4 l = *(const float4*)(sums + row * SETS + w);
        const float f[4] = {fast_exp2(ref[w] - base), fast_exp2(ref[w + 1] - base), fast_exp2(ref[w + 2] - base), fast_exp2(ref[w + 3] - base)};
        sum += fmaf(f[0], l.x, f[1] * l.y) + fmaf(f[2], l.z, f[3] * l.w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 x = *(const float4*)(from + (w + e) * RB * ROW);
          v.x = fmaf(f[e], x.x, v.x); v.y = fmaf(f[e], x.y, v.y); v.z = fmaf(f[e], x.z, v.z); v.w = fmaf(f[e], x.w, v.w);
        }
      }
    *(float4*)(a.part_out + ((size_t)slot * RB + row) * D + c4 * 4) = v;
    if (c4 == 0) a.part_stat[(size_t)slot * RB + row] = make_float2(top, sum);
  }
}

#endif  // __CUDACC__
}  // namespace skv
