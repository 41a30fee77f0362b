// What follows the attention kernels: an item's partials are merged, and for single tokens every key's attention weight is
// added to what it has gathered.
//
// Merging: a warp per row; with the partials' references m_c and sums l_c, M = max m_c, out = sum 2^(m_c - M) O_c / sum 2^(m_c - M)
// l_c, c ascending.  Weights: the attention kernel left every logit (4 bytes a head and key beside the 4 d bytes of K and V that
// it read; the second reading of K that would spare them is 2 d); block c takes the keys of run c of all tiles.
// Bound by the chain of loads: where the partials lie follows from unit_start, their weights from their references.  With
// 64-bit divisions for the former the code alone (51 KB, fetched once a launch) took 10 us.
#include "attend.cuh"

namespace skv {
namespace {

constexpr int kThreads = 128;

// Reference and sum of a row over its partials, by a warp (the same in every lane).  mine: the lane's own partial, of the first 32.
__device__ __forceinline__ float2 merged(const float2* __restrict__ stat, Parts p, int rb_rows, int row, int lane, float2& mine) {
  mine = lane < p.count ? stat[(size_t)(p.first + lane) * rb_rows + row] : make_float2(-INFINITY, 0.f);
  float2 all = mine;
#pragma unroll 1
  for (int c = lane + 32; c < p.count; c += 32) {
    const float2 x = stat[(size_t)(p.first + c) * rb_rows + row];
    const float top = fmaxf(all.x, x.x), ref = top == -INFINITY ? 0.f : top;
    all = make_float2(top, all.y * fast_exp2(all.x - ref) + x.y * fast_exp2(x.x - ref));
  }
  float M = all.x;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  float L = all.y * fast_exp2(all.x - (M == -INFINITY ? 0.f : M));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
  return make_float2(M, L);
}
__device__ __forceinline__ float bits_of(float2 st) { return st.x == -INFINITY && st.y == 0.f ? st.x : st.x == -INFINITY ? st.y : st.x + log2f(st.y); }

template <int DL>
struct alignas(4 * DL) Cols { float v[DL]; };

// Blocks of 128 threads, which find room beside an attention CTA and so are there when it ends.
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 6) attend_finish(const __grid_constant__ AttendArgs a, int rb_shift, int tile_shift, int each, Div by_grid) {
  constexpr int DL = D / 32, kAhead = 8;
  __shared__ int hit[4];
  __shared__ float lse[kThreads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rb_rows = 1 << rb_shift;
  const int blocks = (a.rows + rb_rows - 1) >> rb_shift, all_rows = a.c.units * a.rows;
  // (rows from the last block on, weights from the first one on: where both are few they are beside one another)
  int i = (gridDim.x - 1 - blockIdx.x) * (kThreads / 32) + warp;
  const int u_row = quotient(min(i, all_rows - 1), a.by_rows), u_mine = min(tid, a.c.units - 1);
  pdl_trigger();
  pdl_wait();
  // (loads that depend on nothing go together: the total, the first row's unit, the units among which this block's run begins)
  const int W1 = a.unit_start[a.c.units];                         // places of one block of rows each
  int start = a.unit_start[u_row], places = a.unit_start[u_row + 1];
  const int start0 = a.unit_start[u_mine], end0 = a.unit_start[u_mine + 1], keys0 = a.c.lengths[u_mine] + a.n_new;
  places -= start;
  if (W1 == 0) return;
  const Shares sh = shares_of(W1 * blocks, a.ctas, a.by_ctas, a.least);
#pragma unroll 1
  for (int at = i; i < all_rows; i += gridDim.x * (kThreads / 32)) {
    const int u = quotient(i, a.by_rows), r = i - u * a.rows, rb = r >> rb_shift, row = r & (rb_rows - 1);
    if (i != at) {
      start = a.unit_start[u];
      places = a.unit_start[u + 1] - start;
    }
    if (places == 0) continue;
    const Parts p = parts_of(sh, u * blocks + rb, start * blocks + rb * places, places, each);
    const float* from = a.part_out + ((size_t)p.first * rb_rows + row) * D + lane * DL;
    Cols<DL> x[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) x[e] = e < p.count ? *(const Cols<DL>*)(from + (size_t)e * rb_rows * D) : Cols<DL>{};
    float2 mine;
    const float2 st = merged(a.part_stat, p, rb_rows, row, lane, mine);
    const float ref = st.x == -INFINITY ? 0.f : st.x;
    Cols<DL> acc{};
#pragma unroll 1
    for (int c0 = 0; c0 < p.count; c0 += 32) {
      if (c0 > 0) mine = c0 + lane < p.count ? a.part_stat[(size_t)(p.first + c0 + lane) * rb_rows + row] : make_float2(-INFINITY, 0.f);
      // (a partial that has nothing was not written)
      const float f = mine.x == -INFINITY && mine.y == 0.f ? -1.f : fast_exp2(mine.x - ref);
      const int n = min(32, p.count - c0);
#pragma unroll 1
      for (int c = 0; c < n; c += kAhead) {
        if (c0 + c > 0)
#pragma unroll
          for (int e = 0; e < kAhead; ++e) x[e] = c + e < n ? *(const Cols<DL>*)(from + (size_t)e * rb_rows * D) : Cols<DL>{};
        from += (size_t)kAhead * rb_rows * D;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const float w = __shfl_sync(0xffffffffu, f, (c + e) & 31);
          if (c + e < n && w != -1.f)
#pragma unroll
            for (int d = 0; d < DL; ++d) acc.v[d] = fmaf(w, x[e].v[d], acc.v[d]);
        }
      }
    }
    const float inv = st.x == -INFINITY ? 0.f : 1.f / st.y;       // (a NaN row stays one)
    const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, tok = quotient(r, a.by_group), h = r - tok * a.group;
    const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
    if (BF16) {
      __nv_bfloat162 y[DL / 2];
#pragma unroll
      for (int e = 0; e < DL / 2; ++e) y[e] = __floats2bfloat162_rn(acc.v[2 * e] * inv, acc.v[2 * e + 1] * inv);
      if constexpr (DL == 4) *(uint2*)(a.out + (q * D + lane * DL) * 2) = *(uint2*)y;
      else *(__nv_bfloat162*)(a.out + (q * D + lane * DL) * 2) = y[0];
    } else {
#pragma unroll
      for (int e = 0; e < DL; ++e) acc.v[e] *= inv;
      *(Cols<DL>*)(a.out + (q * D + lane * DL) * 4) = acc;
    }
    if (lane == 0 && a.lse) a.lse[q] = bits_of(st) * kLn2;
  }
  if (!a.accumulate) return;

  const Shares runs = shares_of(W1, gridDim.x, by_grid, 0);
  const int lo = first_of(runs, blockIdx.x), hi = first_of(runs, blockIdx.x + 1);
  if (lo >= hi) return;
  auto found = [&](int u, int start, int end, int keys) {
    if (start <= lo && lo < end) { hit[0] = u; hit[1] = start; hit[2] = end - start; hit[3] = keys; }
  };
  found(u_mine, start0, end0, keys0);
#pragma unroll 1
  for (int u = tid + kThreads; u < a.c.units; u += kThreads) found(u, a.unit_start[u], a.unit_start[u + 1], a.c.lengths[u] + a.n_new);
  __syncthreads();
  int u = hit[0], keys = hit[3];
  start = hit[1];
  places = hit[2];
#pragma unroll 1
  for (int at = lo; at < hi;) {
    const int next = min(hi, start + places), t0 = max(0, at - start - kOver), t1 = max(0, next - start - kOver);
    const int end = min(keys, t1 << tile_shift);
    float* const w = a.c.weights + (size_t)u * a.c.capacity;
#pragma unroll 1
    for (int h0 = 0; t0 < t1 && h0 < a.group; h0 += kThreads) {              // (one round, but for groups of more than 128 heads)
      const int heads = min(kThreads, a.group - h0);
      // the commonest group: four keys' loads in flight, the first ones while the references are on their way
      float4 x[4];
      float old[4];
      int j = (t0 << tile_shift) + tid;
      auto load = [&]() {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int k = j + e * kThreads;
          x[e] = k < end ? *(const float4*)(a.logits + ((size_t)u * a.c.capacity + k) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
          old[e] = k < end ? w[k] : 0.f;
        }
      };
      if (heads == 4) load();
      __syncthreads();
#pragma unroll 1
      for (int h = warp; h < heads; h += kThreads / 32) {
        const int r = h0 + h, rb = r >> rb_shift;
        const Parts p = parts_of(sh, u * blocks + rb, start * blocks + rb * places, places, each);
        float2 mine;
        const float x = bits_of(merged(a.part_stat, p, rb_rows, r & (rb_rows - 1), lane, mine));
        if (lane == 0) lse[h] = x == -INFINITY ? INFINITY : x;
      }
      __syncthreads();
      if (heads == 4) {
#pragma unroll 1
        while (j < end) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int k = j + e * kThreads;
            const float sum = (fast_exp2(x[e].x - lse[0]) + fast_exp2(x[e].y - lse[1])) + (fast_exp2(x[e].z - lse[2]) + fast_exp2(x[e].w - lse[3]));
            if (k < end) w[k] = fmaf(a.decay, old[e], sum);
          }
          j += 4 * kThreads;
          load();
        }
      } else {
#pragma unroll 1
        for (; j < end; j += kThreads) {
          const float* const x = a.logits + ((size_t)u * a.c.capacity + j) * a.group + h0;
          float sum = 0.f;
#pragma unroll 4
          for (int h = 0; h < heads; ++h) sum += fast_exp2(x[h] - lse[h]);
          w[j] = (h0 == 0 ? a.decay * w[j] : w[j]) + sum;
        }
      }
    }
    at = next;
    if (at < hi) {
      do {
        ++u;
        start = a.unit_start[u];
        places = a.unit_start[u + 1] - start;
      } while (places == 0);
      keys = a.c.lengths[u] + a.n_new;
    }
  }
}

// The same where rows are many (attend_tc.cu): a block takes 32 rows, a lane each, and 16 columns; its warps share an item's partials
// out, four in flight each, and add up in order.  Partials lie column of four after column, [slot][d / 4][RB].
template <int D>
__global__ void __launch_bounds__(kThreads, 6) attend_finish_rows(const __grid_constant__ AttendArgs a, int rb_shift, int each) {
  constexpr int CG = D / 16, WARPS = kThreads / 32, kAhead = 4;
  __shared__ float2 stat[WARPS][32];
  __shared__ float4 sums[WARPS][4][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, RB = 1 << rb_shift, blocks = (a.rows + RB - 1) >> rb_shift;
  const int per_item = (min(a.rows, RB) + 31) / 32 * CG, all = a.c.units * blocks * per_item;
  pdl_trigger();
  pdl_wait();
  const int W1 = a.unit_start[a.c.units];
  if (W1 == 0) return;
  const Shares sh = shares_of(W1 * blocks, a.ctas, a.by_ctas, a.least);
#pragma unroll 1
  for (int i = blockIdx.x; i < all; i += gridDim.x) {
    const int item = i / per_item, part = i - item * per_item, row0 = part / CG * 32, col0 = part % CG * 4;   // (columns of four)
    const int u = blocks > 1 ? item / blocks : item, rb = item - u * blocks, row = row0 + lane, r = rb * RB + row;
    const int start = a.unit_start[u], places = a.unit_start[u + 1] - start;
    if (places == 0 || rb * RB + row0 >= a.rows) continue;
    const Parts p = parts_of(sh, item, start * blocks + rb * places, places, each);
    const float2* const st = a.part_stat + ((size_t)p.first << rb_shift) + row;
    const float4* const from = (const float4*)a.part_out + (((size_t)p.first * (D / 4) + col0) << rb_shift) + row;
    float M = -INFINITY, L = 0.f;
    float4 acc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int c0 = warp; c0 < p.count; c0 += WARPS * kAhead) {
      float2 s[kAhead];
      float4 x[kAhead][4];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int c = min(c0 + k * WARPS, p.count - 1);
        s[k] = st[(size_t)c << rb_shift];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[k][e] = from[((size_t)c * (D / 4) + e) << rb_shift];
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (r >= a.rows || c0 + k * WARPS >= p.count || (s[k].x == -INFINITY && s[k].y == 0.f)) continue;   // (the last: not written)
        const float top = fmaxf(M, s[k].x), ref = top == -INFINITY ? 0.f : top, f = fast_exp2(M - ref), w = fast_exp2(s[k].x - ref);
        M = top;
        L = fmaf(L, f, s[k].y * w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[e].x = fmaf(acc[e].x, f, w * x[k][e].x); acc[e].y = fmaf(acc[e].y, f, w * x[k][e].y);
          acc[e].z = fmaf(acc[e].z, f, w * x[k][e].z); acc[e].w = fmaf(acc[e].w, f, w * x[k][e].w);
        }
      }
    }
    stat[warp][lane] = make_float2(M, L);
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][e][lane] = acc[e];
    __syncthreads();
    // warp w: column w of the four, all lanes' rows
    float top = -INFINITY, sum = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, stat[w][lane].x);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      const float2 s = stat[w][lane];
      const float f = fast_exp2(s.x - ref);
      const float4 x = sums[w][warp][lane];
      sum = fmaf(f, s.y, sum);
      v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
    }
    if (r < a.rows) {
      const float inv = top == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;   // (a NaN row stays one)
      const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, tok = quotient(r, a.by_group), h = r - tok * a.group;
      const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x * inv, v.y * inv), hi = __floats2bfloat162_rn(v.z * inv, v.w * inv);
      *(uint2*)(a.out + (q * D + (col0 + warp) * 4) * 2) = make_uint2(*(const uint32_t*)&lo, *(const uint32_t*)&hi);
      if (col0 == 0 && warp == 0 && a.lse) a.lse[q] = bits_of(make_float2(top, sum)) * kLn2;
    }
    __syncthreads();
  }
}

int log2_of(int x) {
  int s = 0;
  while (1 << s < x) ++s;
  return s;
}
template <int D, bool BF16>
cudaError_t launch(const AttendArgs& a, const AttendPlan& p, int ctas, cudaStream_t st) {
  return launch_pdl(attend_finish<D, BF16>, dim3(ctas), dim3(kThreads), 0, st, a, log2_of(p.rb), log2_of(p.tile), p.parts, div_by(ctas));
}

}  // namespace

cudaError_t launch_attend_finish(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  const int ctas = 4 * ctx.sm_count;
  if (p.rb >= 128)
    return launch_pdl(ctx.cfg.head_dim == 128 ? attend_finish_rows<128> : attend_finish_rows<64>, dim3(ctas), dim3(kThreads), 0, st, a, log2_of(p.rb), p.parts);
  if (ctx.cfg.dtype == STRUCTKV_BF16)
    return ctx.cfg.head_dim == 128 ? launch<128, true>(a, p, ctas, st) : launch<64, true>(a, p, ctas, st);
  return ctx.cfg.head_dim == 128 ? launch<128, false>(a, p, ctas, st) : launch<64, false>(a, p, ctas, st);
}

}  // namespace skv
