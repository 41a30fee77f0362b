// What follows the attention kernels: an item's partials are merged, and for single tokens every key's attention weight is
// added to what it has gathered.
//
// Merging: a warp per row; with the partials' references m_c and sums l_c, M = max m_c, out = sum 2^(m_c - M) O_c / sum 2^(m_c - M)
// l_c, c ascending.  Weights: the attention kernel left every logit (4 bytes a head and key beside the 4 d bytes of K and V that
// it read; the second reading of K that would spare them is 2 d); block c takes the keys of run c of all tiles.
// Bound by the chain of loads: where the partials lie follows from unit_start, their weights from their references.  With
// 64-bit divisions for the former the code alone (51 KB, fetched once a launch) took 10 us.
#include <algorithm>

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

// Blocks of 128 threads, which find room beside an attention CTA and so are there when it ends: the last `row_blocks` merge, the
// others weigh.  (All blocks doing both, one after the other: 16 sequences of 1 to 5003 tokens 33.9 us, so 32.4; with the merging
// blocks first, which the launch places first, 1 x 1024 keys take 10.0 us instead of 9.3.)
template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 6) attend_finish(const __grid_constant__ AttendArgs a, int rb_shift, int tile_shift, int each, int row_blocks, Div by_grid) {
  constexpr int DL = D / 32, kAhead = 8;
  __shared__ int hit[4];
  __shared__ float lse[kThreads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rb_rows = 1 << rb_shift;
  const int blocks = (a.rows + rb_rows - 1) >> rb_shift, all_rows = a.c.units * a.rows;
  const int run = blockIdx.x, runs_of = gridDim.x - row_blocks;   // (the weighing ones first)
  int i = run < runs_of ? all_rows : (run - runs_of) * (kThreads / 32) + warp;
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
  for (int at = i; i < all_rows; i += row_blocks * (kThreads / 32)) {
    const int u = quotient(i, a.by_rows), r = i - u * a.rows, rb = r >> rb_shift, row = r & (rb_rows - 1);
    if (i != at) {
      start = a.unit_start[u];
      places = a.unit_start[u + 1] - start;
    }
    if (places == 0) continue;
    const Parts p = parts_of(sh, u * blocks + rb, start * blocks + rb * places, places, each, a.over);
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
  if (run >= runs_of) return;

  const Shares runs = shares_of(W1, runs_of, by_grid, 0);
  const int lo = first_of(runs, run), hi = first_of(runs, run + 1);
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
    const int next = min(hi, start + places), t0 = max(0, at - start - a.over), t1 = max(0, next - start - a.over);
    const int end = min(keys, t1 << tile_shift);
    float* const w = a.c.weights + (size_t)u * a.c.capacity;
#pragma unroll 1
    for (int h0 = 0; t0 < t1 && h0 < a.group; h0 += kThreads) {              // (one round, but for groups of more than 128 heads)
      const int heads = min(kThreads, a.group - h0);
      // the commonest group, not the last four heads of a larger one: four keys' loads in flight, the first ones while the references
      // are on their way
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
      if (a.group == 4) load();
      __syncthreads();
#pragma unroll 1
      for (int h = warp; h < heads; h += kThreads / 32) {
        const int r = h0 + h, rb = r >> rb_shift;
        const Parts p = parts_of(sh, u * blocks + rb, start * blocks + rb * places, places, each, a.over);
        float2 mine;
        const float x = bits_of(merged(a.part_stat, p, rb_rows, r & (rb_rows - 1), lane, mine));
        if (lane == 0) lse[h] = x == -INFINITY ? INFINITY : x;
      }
      __syncthreads();
      if (a.group == 4) {
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

// The same where rows are many (attend_tc.cu): a task is 32 rows, a lane each, and four columns, which lie side by side in a
// partial ([slot][d / 4][RB]). 2^by of a block's warps share a task's partials, eight of them in flight for each, and the
// first joins what they found.
constexpr int kRowWarps = 8;

template <int D>
__global__ void __launch_bounds__(kRowWarps * 32, 3) attend_finish_rows(const __grid_constant__ AttendArgs a, int rb_shift, int each, int by, Div by_groups, Div by_blocks) {
  constexpr int C4 = D / 4, kAhead = 8;
  __shared__ float4 s_acc[kRowWarps][32];
  __shared__ float2 s_stat[kRowWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, RB = 1 << rb_shift, blocks = (a.rows + RB - 1) >> rb_shift;
  const int groups = (min(a.rows, RB) + 31) / 32;
  const int i = (blockIdx.x * kRowWarps + warp) >> by, mine = warp & ((1 << by) - 1);
  const int c4 = i % C4, rest = i / C4, item = quotient(rest, by_groups), row0 = (rest - item * groups) * 32;
  const int u = quotient(item, by_blocks), rb = item - u * blocks, row = row0 + lane, r = rb * RB + row;
  bool live = u < a.c.units && rb * RB + row0 < a.rows;
  pdl_trigger();
  pdl_wait();
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  auto join = [&](float2 s, float4 x, float ref) {
    if (s.x == -INFINITY && s.y == 0.f) return;                   // (was not written)
    const float w = fast_exp2(s.x - ref);
    L = fmaf(w, s.y, L);
    acc.x = fmaf(w, x.x, acc.x); acc.y = fmaf(w, x.y, acc.y); acc.z = fmaf(w, x.z, acc.z); acc.w = fmaf(w, x.w, acc.w);
  };
  if (live) {
    const int W1 = a.unit_start[a.c.units], start = a.unit_start[u], places = a.unit_start[u + 1] - start;
    live = places != 0;
    if (live) {
      const Shares sh = shares_of(W1 * blocks, a.ctas, a.by_ctas, a.least);
      const Parts p = parts_of(sh, item, start * blocks + rb * places, places, each, a.over);
      const int share = (p.count + (1 << by) - 1) >> by, begin = p.first + mine * share;
      const int left = min(share, p.count - mine * share);
      const float2* st = a.part_stat + ((size_t)begin << rb_shift) + row;
      const float4* from = (const float4*)a.part_out + (((size_t)begin * C4 + c4) << rb_shift) + row;
#pragma unroll 1
      for (int c = 0; c < left; c += kAhead) {
        float2 s[kAhead];
        float4 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (c + k < left) {
            s[k] = st[(size_t)k << rb_shift];
            x[k] = from[(size_t)(k * C4) << rb_shift];
          }
        st += (size_t)kAhead << rb_shift;
        from += (size_t)(kAhead * C4) << rb_shift;
        float top = M;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (c + k >= left || r >= a.rows) s[k] = make_float2(-INFINITY, 0.f);
          top = fmaxf(top, s[k].x);
        }
        const float ref = top == -INFINITY ? 0.f : top, f = fast_exp2(M - ref);
        M = top;
        L *= f;
        acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
        for (int k = 0; k < kAhead; ++k) join(s[k], x[k], ref);
      }
    }
  }
  if (by) {
    if (mine) {
      s_acc[warp][lane] = acc;
      s_stat[warp][lane] = make_float2(M, L);
    }
    __syncthreads();
    if (mine) return;
    float top = M;
    for (int k = 1; k < 1 << by; ++k) top = fmaxf(top, s_stat[warp + k][lane].x);
    const float ref = top == -INFINITY ? 0.f : top, f = fast_exp2(M - ref);
    M = top;
    L *= f;
    acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
    for (int k = 1; k < 1 << by; ++k) join(s_stat[warp + k][lane], s_acc[warp + k][lane], ref);
  }
  if (!live || r >= a.rows) return;
  const float inv = M == -INFINITY && L == 0.f ? 0.f : 1.f / L;   // (a NaN row stays one)
  const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, tok = quotient(r, a.by_group), h = r - tok * a.group;
  const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
  const __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), hi = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
  *(uint2*)(a.out + (q * D + c4 * 4) * 2) = make_uint2(*(const uint32_t*)&lo, *(const uint32_t*)&hi);
  if (c4 == 0 && a.lse) a.lse[q] = bits_of(make_float2(M, L)) * kLn2;
}

int log2_of(int x) {
  int s = 0;
  while (1 << s < x) ++s;
  return s;
}
template <int D, bool BF16>
cudaError_t launch(const AttendArgs& a, const AttendPlan& p, int sms, cudaStream_t st) {
  const int tasks = a.c.units * a.rows, rows = std::min((tasks - 1) / (kThreads / 32) + 1, (a.accumulate ? 2 : 4) * sms), weigh = a.accumulate ? 4 * sms : 0;
  return launch_pdl(attend_finish<D, BF16>, dim3(rows + weigh), dim3(kThreads), 0, st, a, log2_of(p.rb), log2_of(p.tile), p.parts, rows, div_by(std::max(1, weigh)));
}

}  // namespace

cudaError_t launch_attend_finish(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  const int sms = ctx.sm_count;
  if (p.rb >= 128) {
    const int blocks = (a.rows + p.rb - 1) / p.rb, groups = (std::min(a.rows, p.rb) + 31) / 32;
    const long long tasks = (long long)a.c.units * blocks * groups * (ctx.cfg.head_dim / 4);
    int by = 0;                                                   // (as many warps as the SMs hold, up to a block a task)
    while (by < 3 && tasks << by < 16 * sms) ++by;
    return launch_pdl(ctx.cfg.head_dim == 128 ? attend_finish_rows<128> : attend_finish_rows<64>, dim3((unsigned)((((tasks << by)) + kRowWarps - 1) / kRowWarps)),
                      dim3(kRowWarps * 32), 0, st, a, log2_of(p.rb), p.parts, by, div_by(groups), div_by(blocks));
  }
  if (ctx.cfg.dtype == STRUCTKV_BF16)
    return ctx.cfg.head_dim == 128 ? launch<128, true>(a, p, sms, st) : launch<64, true>(a, p, sms, st);
  return ctx.cfg.head_dim == 128 ? launch<128, false>(a, p, sms, st) : launch<64, false>(a, p, sms, st);
}

}  // namespace skv
