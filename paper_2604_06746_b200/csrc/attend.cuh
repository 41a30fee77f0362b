// Attention of new tokens over a compacted cache, what its kernels share: how the work is cut, partial results, options.
//
// A unit is (sequence, KV head) u = b H_kv + g, with lengths[u] + n_new keys (the new tokens are the last ones) and rows
// r = i G + h, new token i and head h of the group.  An item is a unit's block of up to RB rows over all of its keys; items
// follow one another unit after unit, and their key tiles form one sequence of W tiles.  C CTAs take runs of it whose lengths
// differ by one tile at most: every CTA reads equally much whatever the lengths, which only the device knows.  What a CTA has of
// an item it leaves as a partial (row references, sums, unscaled output) in slot item + CTA, which no other pair has, so that an
// item's partials lie side by side; attend_finish() merges them in that order: results do not depend on timing.
#pragma once

#include <atomic>

#include "common.cuh"

namespace skv {

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
  Div by_kv, by_group, by_rows;        // H_kv, group, rows
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
  int* unit_start;                     // [units + 1] tiles before a unit, of one block of rows
  float2* part_stat;                   // [slot][RB] reference (bits) and sum
  float* part_out;                     // [slot][RB][d]
  float* logits;                       // [units][capacity][group] in bits (accumulate)
  int ctas, least;                     // CTAs, tiles one of them has at least
};

// Rows of a block, keys of a tile, CTAs that run at once, partials a CTA leaves of an item, tiles it takes at least.
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

// Keys of a unit, 0 where its length is not one: the caller is told, nothing of the unit is read or written.
__device__ __forceinline__ int unit_keys(const CacheView& c, int u, int n_new) {
  const int n = c.lengths[u];
  if (n < 0 || n > c.capacity - n_new) {
    atomicCAS(c.status, 0, (int)STRUCTKV_ERR_INVALID_ARG);
    return 0;
  }
  return n + n_new;
}

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

// How W tiles are shared out: CTA c has tiles [first(c), first(c + 1)), at least `least` of them if there are as many.
struct Shares { int W, C, each, more; };
__device__ __forceinline__ Shares shares_of(int W, int ctas, int least) {
  const int C = max(1, min(W / least, ctas)), each = W / C;
  return {W, C, each, W - each * C};
}
__device__ __forceinline__ int first_of(const Shares& s, int c) { return c >= s.C ? s.W : c * s.each + min(c, s.more); }
__device__ __forceinline__ int cta_of(const Shares& s, int x) {
  const int line = s.more * (s.each + 1);
  return x < line ? x / (s.each + 1) : s.more + (x - line) / s.each;
}

// A CTA's run of tiles, and the unit that its first tile is in: keys, tiles of one block of rows before it.
struct WorkStart { int lo, hi, unit, before, keys; };

// By the whole block.  Units are scanned THREADS at a time.  save: unit_start.
template <int THREADS>
__device__ __forceinline__ WorkStart find_work(const CacheView& c, int n_new, int tile, int blocks, int ctas, int least, int* save) {
  constexpr int WARPS = THREADS / 32;
  __shared__ int warp_tiles[WARPS], hit[3];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // (one round where the units fit the block; the sum of all is known only after all of them, so that a second sweep follows)
  int total = 0, mine = 0, incl = 0, keys = 0, lo = 0, hi = 0;
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    int before = 0;
#pragma unroll 1
    for (int u0 = 0; u0 < c.units; u0 += THREADS) {
      if (round == 0 || c.units > THREADS) {
        const int u = u0 + tid;
        keys = u < c.units ? unit_keys(c, u, n_new) : 0;
        mine = (keys + tile - 1) / tile;
        incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += t;
        }
        __syncthreads();
        if (lane == 31) warp_tiles[warp] = incl;
        __syncthreads();
        const int w = lane < WARPS ? warp_tiles[lane] : 0;
        incl += before + (int)__reduce_add_sync(0xffffffffu, lane < warp ? w : 0);
        before += (int)__reduce_add_sync(0xffffffffu, w);
        if (round == 0 && save && u < c.units) save[u] = incl - mine;
      }
      if (round == 1 && (incl - mine) * blocks <= lo && lo < incl * blocks) {
        hit[0] = u0 + tid;
        hit[1] = incl - mine;
        hit[2] = keys;
      }
    }
    if (round == 0) {
      total = before;
      const Shares s = shares_of(total * blocks, ctas, least);
      lo = first_of(s, blockIdx.x);
      hi = first_of(s, blockIdx.x + 1);
    }
  }
  if (save && tid == 0) save[c.units] = total;
  __syncthreads();
  return {lo, hi, hit[0], hit[1], hit[2]};
}

// cap tanh(scale s / cap) in bits: for small arguments the odd series, else 1 - 2 / (e^2y + 1), both to fp32's last bits.
__device__ __forceinline__ float capped(float s, float cap2, float inv_cap) {
  const float y = s * inv_cap, a = fabsf(y), y2 = y * y;
  if (a < 0.25f) {
    // Taylor series of tanh about 0; the first term left out is below 9e-9 relative
    float p = fmaf(y2, 62.f / 2835.f, -17.f / 315.f);
    p = fmaf(y2, p, 2.f / 15.f);
    p = fmaf(y2, p, -1.f / 3.f);
    return cap2 * fmaf(y * y2, p, y);
  }
  if (!(a < 20.f)) return a == a ? copysignf(cap2, y) : y;        // (1 in fp32 from 10 on; a NaN stays one)
  const float e = fast_exp2(a * (2.f * kLog2e));
  return copysignf(cap2 * (1.f - __fdividef(2.f, e + 1.f)), y);
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

// x in bits from the product of a row and a key.
__device__ __forceinline__ float biased(const AttendArgs& a, float s, const RowOptions& o, int key_position) {
  float x = a.cap2 != 0.f ? capped(s, a.cap2, a.inv_cap) : s * a.scale2;
  if (a.slopes) x = fmaf(-o.slope2, (float)(o.position - key_position), x);
  return x;
}

#endif  // __CUDACC__
}  // namespace skv
