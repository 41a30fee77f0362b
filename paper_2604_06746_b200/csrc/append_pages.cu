// New tokens' rows go to pages: gathered, K rotated, quantised to e4m3 with a scale for 16 slots of a head.
//
// A CTA has one block of 16 slots of a sequence (or a share of its heads): cosines and sines of its tokens go to shared memory once, then
// a warp takes K or V of one head at a time, all 16 rows in registers: the largest magnitude is known before anything is
// written, and every element is read once.  Further CTAs rotate the queries that came along.
#include <algorithm>

#include "pages.cuh"

namespace skv {
namespace {

constexpr int kWarps = 8;

// The smallest e with which `top` stays within 448 2^e, from the bits of the finite top = m 2^x, 1 <= m < 2 (448 = 1.75 2^8).
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t w = __float_as_uint(top);
  return max((int)(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u), kLowExponent);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | (uint32_t)hi << 16;
}
// Two codes times a power of two (as two fp16), rounded anew.  (In fp16 the product is exact down to 2^-24, far below half of e4m3's
// smallest number, 2^-10.)
__device__ __forceinline__ uint32_t scaled2(uint32_t codes, uint32_t by) {
  uint32_t x;
  uint16_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((uint16_t)codes));
  asm("mul.f16x2 %0, %0, %1;" : "+r"(x) : "r"(by));
  asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(y) : "r"(x));
  return y;
}

template <typename T, int D>
__global__ void __launch_bounds__(kWarps * 32) append_pages(const __grid_constant__ RopeArgs r, const __grid_constant__ AppendPagesArgs a) {
  constexpr int N = Chunk<T>::N, LANES = D / (2 * N), ROWS = 32 / LANES, IT = kBlockSlots / ROWS;
  __shared__ float2 turns[kBlockSlots][D / 2 + 1];
  __shared__ int source[kBlockSlots];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  pdl_wait();
  if (blockIdx.x >= a.append_ctas) {
    // queries: a group of lanes a token
    const int per = kWarps * 32 / LANES, groups = (a.heads + a.head_step - 1) / a.head_step;
    const long long at = (long long)(blockIdx.x - a.append_ctas) * per + tid / LANES;
    const int row = (int)(at / groups), h0 = (int)(at % groups) * a.head_step;
    if (at >= (long long)a.q_rows * groups) return;
    const int b = quotient(row, a.by_new), i = row - b * a.n_new;
    rotate_heads<T>(r, false, (const T*)(a.q + b * a.q_batch + i * a.q_token), a.q_head / (int)sizeof(T),
                    (T*)a.q_out + (long long)row * a.heads * D, D, a.positions[b * a.s_positions + i], (tid % LANES) * N, h0,
                    min(h0 + a.head_step, a.heads));
    return;
  }
  const int job0 = blockIdx.x % a.splits, task = blockIdx.x / a.splits, b = quotient(task, a.by_blocks), nth = task - b * a.blocks;
  int n;
  const int count = rows_of_sequence(a.c, a.counts, b, a.n_new, n);
  if (count < 0) {
    if (nth == 0 && tid == 0) tell_invalid(a.c);
    return;
  }
  const int slot0 = ((n >> kBlockShift) + nth) << kBlockShift, lo = max(slot0, n), hi = min(slot0 + kBlockSlots, n + count);
  if (lo >= hi) return;
  const int page = *(const int*)((const char*)a.c.table + b * a.c.s_table + (long long)(slot0 >> a.c.page_shift) * 4);
  if (page < 0 || page >= a.c.pages) {
    if (tid == 0) tell_invalid(a.c);
    return;
  }
  if (tid < kBlockSlots) {
    const int j = slot0 + tid;
    int t = -1;
    if (j >= lo && j < hi) {
      t = a.index ? a.index[b * a.s_index + j - n] : j - n;
      if (t < 0 || t >= a.tokens) {
        tell_invalid(a.c);
        t = -1;
      }
    }
    source[tid] = t;
  }
  __syncthreads();
  if (a.rotated) {
    for (int i = tid; i < kBlockSlots * (r.dim / 2); i += kWarps * 32) {
      const int row = i / (r.dim / 2), p = i - row * (r.dim / 2), t = source[row];
      if (t >= 0) turns[row][p] = cos_sin<T>(turn_of(r.step[p], a.positions[b * a.s_positions + t]), r.amplitude);
    }
    __syncthreads();
  }
  const int in_page = slot0 & ((1 << a.c.page_shift) - 1), p0 = (lane % LANES) * N, row0 = lane / LANES;
#pragma unroll 1
  for (int job = job0 * kWarps + warp; job < 2 * a.c.n_kv; job += a.splits * kWarps) {
    const int g = job >> 1;
    const bool is_v = job & 1;
    const PairPlace<T> at(!is_v && a.rotated ? r.dim : 0, r.interleaved, p0);
    const char* const from = (is_v ? a.v : a.k) + b * a.s_batch + g * a.s_head;
    float u[IT][N], v[IT][N];
#pragma unroll
    for (int k = 0; k < IT; ++k) {
      const int t = source[k * ROWS + row0];
      if (t >= 0) load_pairs<T>(at, (const T*)(from + t * a.s_token), u[k], v[k]);
      else
#pragma unroll
        for (int i = 0; i < N; ++i) u[k][i] = v[k][i] = 0.f;
    }
    float top = 0.f;
#pragma unroll
    for (int k = 0; k < IT; ++k) {
      if (!is_v && a.rotated && source[k * ROWS + row0] >= 0)
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (at.turns(i)) turn(u[k][i], v[k][i], turns[k * ROWS + row0][p0 + i]);
#pragma unroll
      for (int i = 0; i < N; ++i) top = fmaxf(top, fmaxf(fabsf(u[k][i]), fabsf(v[k][i])));   // (NaN has no part in it)
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top == INFINITY) {
      // infinities are stored as NaN
      top = 0.f;
      auto no_infinity = [&](float& x) {
        if (fabsf(x) == INFINITY) x = __int_as_float(0x7fffffff);
        top = fmaxf(top, fabsf(x));
      };
#pragma unroll
      for (int k = 0; k < IT; ++k)
#pragma unroll
        for (int i = 0; i < N; ++i) { no_infinity(u[k][i]); no_infinity(v[k][i]); }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    int e = exponent_of(top);
    unsigned char* const scale = (is_v ? a.c.v_scales : a.c.k_scales) + (((size_t)page * a.c.n_kv + g) << (a.c.page_shift - kBlockShift)) + (in_page >> kBlockShift);
    char* const to = (is_v ? a.c.v : a.c.k) + page * a.c.s_page + g * a.c.s_head + in_page * a.c.s_token;
    if (slot0 < n) {
      // older tokens: their codes by the larger of the scales
      const int had = (int)*scale - 127;
      if (e > had) {
        const int down = min(e - had, 24);
        const uint32_t half = down > 14 ? 1u << (24 - down) : (uint32_t)(15 - down) << 10, by = half | half << 16;
        for (int i = lane; i < (n - slot0) * (D / 4); i += 32) {
          uint32_t* const w = (uint32_t*)(to + (i / (D / 4)) * a.c.s_token + (i % (D / 4)) * 4);
          const uint32_t x = *w;
          *w = scaled2(x & 0xffffu, by) | scaled2(x >> 16, by) << 16;
        }
      } else {
        e = had;
      }
      __syncwarp();
    }
    if (lane == 0) *scale = (unsigned char)(e + 127);
    const float by = __int_as_float((127 - e) << 23);
#pragma unroll
    for (int k = 0; k < IT; ++k) {
      const int row = k * ROWS + row0;
      if (slot0 + row < lo || slot0 + row >= hi) continue;
      char* const out = to + row * a.c.s_token;
#pragma unroll
      for (int i = 0; i < N; ++i) { u[k][i] *= by; v[k][i] *= by; }
      if (at.whole) {
        float x[N], y[N];
        join<T>(at, u[k], v[k], x, y);
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          *(uint32_t*)(out + at.a + i) = codes4(x[i], x[i + 1], x[i + 2], x[i + 3]);
          *(uint32_t*)(out + at.b + i) = codes4(y[i], y[i + 1], y[i + 2], y[i + 3]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int2 el = at.pair(i);
          const uint32_t w = codes4(u[k][i], v[k][i], 0.f, 0.f);
          out[el.x] = (char)w;
          out[el.y] = (char)(w >> 8);
        }
      }
    }
  }
}

template <typename T, int D>
cudaError_t launch(const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st) {
  constexpr int PER = kWarps * 32 / (D / (2 * Chunk<T>::N));
  const long long q = a.q ? (long long)a.q_rows * ((a.heads + a.head_step - 1) / a.head_step) : 0, ctas = a.append_ctas + (q + PER - 1) / PER;
  return launch_pdl(append_pages<T, D>, dim3((unsigned)ctas), dim3(kWarps * 32), 0, st, r, a);
}

}  // namespace

cudaError_t launch_append_pages(const Ctx& ctx, const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st) {
  if (ctx.cfg.dtype == STRUCTKV_BF16) return ctx.cfg.head_dim == 128 ? launch<__nv_bfloat16, 128>(r, a, st) : launch<__nv_bfloat16, 64>(r, a, st);
  return ctx.cfg.head_dim == 128 ? launch<float, 128>(r, a, st) : launch<float, 64>(r, a, st);
}

}  // namespace skv
