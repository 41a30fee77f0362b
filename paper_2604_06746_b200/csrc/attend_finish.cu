// What follows the attention kernels: items that several CTAs took are merged, and for single tokens every key's attention
// weight is added to what it has gathered.
//
// Merging: a warp per row; with the CTAs' maxima m_c and sums l_c, M = max m_c, out = sum 2^(m_c - M) O_c / sum 2^(m_c - M) l_c,
// c ascending.  Weights: the attention kernel left every logit (4 bytes a head and key beside the 4 d bytes of K and V that it
// read; the second reading of K that would spare them is 2 d); block c takes the keys of run c of C of all tiles.
#include "attend.cuh"

namespace skv {
namespace {

constexpr int kThreads = 256;

// CTAs that took an item, and the slot of CTA c.
struct Cover { int first, last; };
__device__ __forceinline__ Cover cover_of(long long start, int tiles, long long W, int C) {
  return {cta_of(start, W, C), cta_of(start + tiles - 1, W, C)};
}
__device__ __forceinline__ int slot_of(const Cover& v, int c) { return 2 * c + (c == v.first); }   // it begins there, or goes on

// Maximum and sum of a row over its CTAs, by a warp (the same in every lane).
__device__ __forceinline__ float2 merged_stat(const AttendArgs& a, const Cover& v, int rb_rows, int row, int lane) {
  float M = -INFINITY;
  for (int c = v.first + lane; c <= v.last; c += 32) M = fmaxf(M, a.part_stat[(size_t)slot_of(v, c) * rb_rows + row].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (M == -INFINITY) return make_float2(M, 0.f);
  float L = 0.f;
  for (int c = v.first + lane; c <= v.last; c += 32) {
    const float2 p = a.part_stat[(size_t)slot_of(v, c) * rb_rows + row];
    L += p.y * fast_exp2(p.x - M);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  return make_float2(M, L);
}
__device__ __forceinline__ float bits_of(float2 st) { return st.x == -INFINITY ? st.x : st.x + log2f(st.y); }

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads) attend_finish(const __grid_constant__ AttendArgs a, int rb_rows, int tile) {
  constexpr int DL = D / 32;
  __shared__ int hit;
  __shared__ float lse[kThreads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int blocks = (a.rows + rb_rows - 1) / rb_rows;
  pdl_trigger();
  pdl_wait();
  const long long W = a.unit_start[a.c.units];
  if (W == 0) return;
  const int C = sharers(W, a.ctas);
  const int all_rows = a.c.units * a.rows;
  for (int i = blockIdx.x * (kThreads / 32) + warp; i < all_rows; i += gridDim.x * (kThreads / 32)) {
    const int u = i / a.rows, r = i % a.rows, rb = r / rb_rows, row = r % rb_rows;
    const int start = a.unit_start[u], tiles = (a.unit_start[u + 1] - start) / blocks;
    if (tiles == 0) continue;
    const Cover v = cover_of((long long)start + (long long)rb * tiles, tiles, W, C);
    if (v.first == v.last) continue;                              // finished there
    const float2 st = merged_stat(a, v, rb_rows, row, lane);
    float acc[DL] = {};
    if (st.x != -INFINITY) {
#pragma unroll 4
      for (int c = v.first; c <= v.last; ++c) {
        const size_t at = (size_t)slot_of(v, c) * rb_rows + row;
        const float f = fast_exp2(a.part_stat[at].x - st.x);
#pragma unroll
        for (int e = 0; e < DL; ++e) acc[e] = fmaf(f, a.part_out[at * D + e * 32 + lane], acc[e]);
      }
    }
    const float inv = st.x == -INFINITY ? 0.f : 1.f / st.y;
    const int b = u / a.c.n_kv, g = u % a.c.n_kv, tok = r / a.group, h = r % a.group;
    const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
#pragma unroll
    for (int e = 0; e < DL; ++e) {
      if (BF16) ((__nv_bfloat16*)a.out)[q * D + e * 32 + lane] = __float2bfloat16(acc[e] * inv);
      else ((float*)a.out)[q * D + e * 32 + lane] = acc[e] * inv;
    }
    if (lane == 0 && a.lse) a.lse[q] = bits_of(st) * kLn2;
  }
  if (!a.accumulate) return;

  // tiles of all units, one block of rows each
  const long long W1 = W / blocks, lo = cut(blockIdx.x, W1, sharers(W1, gridDim.x)), hi = cut(blockIdx.x + 1, W1, sharers(W1, gridDim.x));
  if (lo >= hi) return;
  for (int u = tid; u < a.c.units; u += kThreads)
    if (a.unit_start[u] / blocks <= lo && lo < a.unit_start[u + 1] / blocks) hit = u;
  __syncthreads();
  int u = hit;
#pragma unroll 1
  for (long long at = lo; at < hi; ++u) {
    const int start = a.unit_start[u], tiles = (a.unit_start[u + 1] - start) / blocks;
    if (tiles == 0) continue;
    const int t0 = (int)(at - start / blocks), t1 = (int)min((long long)tiles, t0 + (hi - at));
    const int keys = unit_keys(a.c, u, a.n_new);
    float* const w = a.c.weights + (size_t)u * a.c.capacity;
#pragma unroll 1
    for (int h0 = 0; h0 < a.group; h0 += kThreads) {              // (one round, but for groups of more than 256 heads)
      const int heads = min(kThreads, a.group - h0);
      __syncthreads();
      for (int h = warp; h < heads; h += kThreads / 32) {
        const int r = h0 + h, rb = r / rb_rows;
        const Cover v = cover_of((long long)start + (long long)rb * tiles, tiles, W, C);
        const float x = v.first == v.last ? a.row_lse[(size_t)u * a.rows + r] : bits_of(merged_stat(a, v, rb_rows, r % rb_rows, lane));
        if (lane == 0) lse[h] = x == -INFINITY ? INFINITY : x;
      }
      __syncthreads();
      const bool fours = a.group % 4 == 0;
      for (int j = t0 * tile + tid; j < min(keys, t1 * tile); j += kThreads) {
        const float* const x = a.logits + ((size_t)u * a.c.capacity + j) * a.group + h0;
        float sum = 0.f;
        if (fours) {
          for (int h = 0; h < heads; h += 4) {
            const float4 v = *(const float4*)(x + h);
            sum += (fast_exp2(v.x - lse[h]) + fast_exp2(v.y - lse[h + 1])) + (fast_exp2(v.z - lse[h + 2]) + fast_exp2(v.w - lse[h + 3]));
          }
        } else {
          for (int h = 0; h < heads; ++h) sum += fast_exp2(x[h] - lse[h]);
        }
        w[j] = (h0 == 0 ? a.decay * w[j] : w[j]) + sum;
      }
    }
    at += t1 - t0;
  }
}

template <int D, bool BF16>
cudaError_t launch(const AttendArgs& a, const AttendPlan& p, int ctas, cudaStream_t st) {
  return launch_pdl(attend_finish<D, BF16>, dim3(ctas), dim3(kThreads), 0, st, a, p.rb, p.tile);
}

}  // namespace

cudaError_t launch_attend_finish(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  const int ctas = 2 * ctx.sm_count;
  if (ctx.cfg.dtype == STRUCTKV_BF16)
    return ctx.cfg.head_dim == 128 ? launch<128, true>(a, p, ctas, st) : launch<64, true>(a, p, ctas, st);
  return ctx.cfg.head_dim == 128 ? launch<128, false>(a, p, ctas, st) : launch<64, false>(a, p, ctas, st);
}

}  // namespace skv
