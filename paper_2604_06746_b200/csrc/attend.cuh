// Attention of new tokens over a compacted cache, what its kernels share: how the work is cut, partial results, options.
//
// A unit is (sequence, KV head) u = b H_kv + g, with lengths[u] + n_new keys (the new tokens are the last ones) and rows
// r = i G + h, new token i and head h of the group.  An item is a unit's block of up to RB rows over all of its keys; items
// follow one another unit after unit, and their key tiles form one sequence of W tiles.  CTA c of C takes tiles
// [c W / C, (c + 1) W / C): every CTA reads equally much whatever the lengths, which only the device knows.  An item that
// lies in one CTA is finished there; of the others each CTA leaves a partial (row maximum, sum, unscaled output), which
// attend_finish() merges in the order of the CTAs: results do not depend on timing.
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

struct AttendArgs {
  CacheView c;
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
  // workspace
  int* unit_start;                     // [units + 1] tiles before a unit
  float2* part_stat;                   // [2 ctas][RB] maximum and sum
  float* part_out;                     // [2 ctas][RB][d]
  float* row_lse;                      // [units][rows] in bits (accumulate)
  float* logits;                       // [units][capacity][group] in bits (accumulate)
  int ctas;
};

// Rows of a block, keys of a tile, CTAs that run at once.
struct AttendPlan { int rb, tile, ctas; };

cudaError_t launch_append(const CacheView& c, const NewRows& r, int n_new, cudaStream_t st);
cudaError_t launch_commit(const CacheView& c, int n_new, const int* counts, const int* path, cudaStream_t st);
cudaError_t launch_evict(const CacheView& c, int budget, int recent, cudaStream_t st);
// The kernels: fp32 storage on the CUDA cores; bf16 storage.
cudaError_t launch_attend_simt(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
cudaError_t launch_attend_mma(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st);
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

// First tile of CTA c of C, and the CTA that has tile x.  C is at most W, so that no CTA in between is without a tile; those from
// C on have none.
__device__ __forceinline__ int sharers(long long W, int ctas) { return (int)min(W, (long long)ctas); }
__device__ __forceinline__ long long cut(int c, long long W, int C) { return c >= C ? W : c * W / C; }
__device__ __forceinline__ int cta_of(long long x, long long W, int C) { return (int)(((x + 1) * C - 1) / W); }

struct WorkStart { int unit, before; long long total; };   // unit that holds a tile, tiles before the unit, tiles of all units

// By the whole block: tiles of all units, and the unit that holds tile number want(total).  Units are scanned THREADS at a time.
// save: unit_start.
template <int THREADS, typename Want>
__device__ __forceinline__ WorkStart find_work(const CacheView& c, int n_new, int tile, int blocks, Want want, int* save) {
  constexpr int WARPS = THREADS / 32;
  __shared__ int warp_tiles[WARPS], hit[2];
  __shared__ long long sum;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // (one round where the units fit the block; total is known only after all rounds, so a second sweep looks for the tile)
  long long total = 0;
  int mine = 0, incl = 0;
  for (int round = 0; round < 2; ++round) {
    long long before = 0;
    const long long at = round ? want(total) : 0;
    for (int u0 = 0; u0 < c.units; u0 += THREADS) {
      if (round == 0 || c.units > THREADS) {
        const int u = u0 + tid;
        mine = u < c.units ? (unit_keys(c, u, n_new) + tile - 1) / tile * blocks : 0;
        incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int t = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += t;
        }
        __syncthreads();
        if (lane == 31) warp_tiles[warp] = incl;
        __syncthreads();
        int earlier = 0, all = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
          earlier += w < warp ? warp_tiles[w] : 0;
          all += warp_tiles[w];
        }
        incl += earlier;
        if (round == 0 && save && u < c.units) save[u] = (int)(before + incl - mine);
        if (tid == 0) sum = all;
      }
      if (round == 1 && before + incl - mine <= at && at < before + incl) {
        hit[0] = u0 + tid;
        hit[1] = (int)(before + incl - mine);
      }
      __syncthreads();
      before += sum;
    }
    total = before;
  }
  if (save && tid == 0) save[c.units] = (int)total;
  __syncthreads();
  return {hit[0], hit[1], total};
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
  const int i = r / a.group;
  return a.tree ? a.tree[(size_t)(u / a.c.n_kv) * a.n_new + i] : (i == 63 ? ~0ull : (1ull << (i + 1)) - 1);
}
// A row's option values.
struct RowOptions { unsigned long long seen; float slope2; int position; };
__device__ __forceinline__ RowOptions row_options(const AttendArgs& a, int u, int r) {
  RowOptions o;
  const int g = u % a.c.n_kv, i = r / a.group, h = r % a.group;
  o.seen = row_seen(a, u, r);
  o.slope2 = a.slopes ? a.slopes[g * a.group + h] * kLog2e : 0.f;
  o.position = a.slopes ? a.c.positions[(size_t)u * a.c.capacity + a.c.lengths[u] + i] : 0;
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
