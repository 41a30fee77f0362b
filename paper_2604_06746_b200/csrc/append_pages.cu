// New tokens' rows go to pages: gathered, K rotated, quantised to e4m3 with a scale for 16 slots of a head.
//
// A CTA has one block of 16 slots of a sequence and K and V of one head or of four.  A lane has two chunks of 16 bytes of one row, of all those
// heads: their angles are worked out once, and all of a lane's loads are in flight together (of four heads to places of its own in shared
// memory, which leaves registers for six CTAs an SM: 16384 rows 26.7 to 23.4 us).  The blocks' largest magnitudes meet in shared memory; then
// every row goes through the rotation once more and becomes codes, so that nothing but the rows as they came is held meanwhile and every
// element is read once.  Further CTAs rotate the queries that came along.
//
// Codes of K are those of the rotated values rounded once to fp32, which work in fp32 cannot always tell: what a pair may be off by goes with |a| + |b|, not
// with what is left of them.  The largest and the smallest value that there may be are coded, and where these codes differ (of normal numbers one in 17
// thousand, a lane of 1100, a warp's head of 35), the lane's pairs are rotated in fp64, as they are for the scale of a block whose largest value is as
// close to a border between two scales.  All that takes 0.8 us of the 25.9 below: where pairs come to fp64 from global memory, not from the rows'
// place in shared memory, 0.4 more; with |a| + |b| of the pair as it came, which would send a third fewer there, 1.0 more; at the end of the CTA, not where
// a value is found, 3 more.
//
// 16384 rows of 131072 (8 heads, d 128, bf16, gathered): 25.9 us, 3.9 TB/s, 59 % of a measured copy; issue slots are the next bound (13
// instructions an element: angles 2, rotation twice, maximum, scale, codes), then the chain counts -> index -> rows -> scale -> codes, which six CTAs
// an SM hide.  One token of 16 sequences with its queries: 3.7 to 4.4 us, a launch's latency.
// A part of the head that is no whole number of chunks goes element by element; bf16 then spills 40 bytes of 128 registers.
#include <algorithm>

#include "pages.cuh"

namespace skv {
namespace {

constexpr int kManyHeads = 4;                                     // of a CTA, where there are many blocks; else one  (16384 rows by two heads: 6 % more)
constexpr float kEnd = 0x1.fffp127f;                              // from here on work in fp32 does not tell numbers from infinities
template <typename T>
constexpr int kPairs = 16 / sizeof(T);                            // a lane's of a row: two chunks of 16 bytes

// The smallest e with which `top` stays within 448 2^e, from the bits of the finite top = m 2^x, 1 <= m < 2 (448 = 1.75 2^8).
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t w = __float_as_uint(top);
  return max((int)(w >> 23) - 127 - 8 + ((w & 0x7fffffu) > 0x600000u), kLowExponent);
}
// Whether `top` lies within 2^-19.8 of a 448 2^e, where that changes.
__device__ __forceinline__ bool border_near(float top) { return (__float_as_uint(top) & 0x7fffffu) - (0x600000u - 16u) <= 32u; }
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

// The largest magnitude of a lane's bf16, NaN aside.
template <int N>
__device__ __forceinline__ float largest(const RawPairs<__nv_bfloat16, N>& r) {
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.x[i] & 0x7fff7fffu));
    asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.y[i] & 0x7fff7fffu));
  }
  return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
}
template <int N>
__device__ __forceinline__ float largest(const RawPairs<float, N>&) { return 0.f; }
// (nothing there: zeros, and nothing is read)
__device__ __forceinline__ void copy16(uint4* to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// A pair turned in 64 bits and rounded to fp32 (`turns` not: as it is); what is not finite then is NaN.
__device__ __forceinline__ float2 exact_pair(double u, double v, bool turns, unsigned long long step, int position, double amplitude) {
  if (turns) {
    const double2 cs = cos_sin64(step, position);
    const double c = cs.x * amplitude, s = cs.y * amplitude, y = fma(u, c, v * -s);
    v = fma(v, c, u * s);
    u = y;
  }
  const float x = (float)u, y = (float)v;
  return make_float2(fabsf(x) == INFINITY ? __int_as_float(0x7fffffff) : x, fabsf(y) == INFINITY ? __int_as_float(0x7fffffff) : y);
}

// A CTA for K and V of HEADS heads.  Of many heads a lane's rows wait in shared memory, in places of its own, and registers are left for more CTAs.
template <typename T, int D, Pairing P, int HEADS>
struct AppendShape {
  static constexpr int N = kPairs<T>, kJobs = 2 * HEADS, kLanes = D / (2 * N), kThreads = kBlockSlots * kLanes;
  static constexpr bool kStaged = HEADS > 1 && P != SINGLE;
  static constexpr int kUnroll = kStaged ? 1 : 2 * HEADS;         // (of heads; registers have no index)
  static constexpr int kSmem = kStaged ? kJobs * 2 * kThreads * 16 : 0, kPer = (kStaged ? 768 : 512) / kThreads;
};

template <typename T, int D, Pairing P, int HEADS>
__global__ void __launch_bounds__(AppendShape<T, D, P, HEADS>::kThreads, AppendShape<T, D, P, HEADS>::kPer) append_pages(const __grid_constant__ RopeArgs r, const __grid_constant__ AppendPagesArgs a) {
  using S = AppendShape<T, D, P, HEADS>;
  constexpr int N = S::N, JOBS = S::kJobs, LANES = S::kLanes, WARPS = S::kThreads / 32;
  extern __shared__ __align__(16) uint4 staged[];                 // [job][chunk][lane]
  using Place = PairPlace<T, D, P, N>;
  __shared__ float tops[JOBS][WARPS], exact_tops[JOBS][WARPS];
  __shared__ __align__(16) unsigned long long steps[D / 2];       // (lanes read different ones: from the arguments one after another)
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, p0 = (tid % LANES) * N;
  pdl_trigger();
  if (a.rotated && tid < D / 2) steps[tid] = r.step[tid];
  __syncthreads();
  pdl_wait();
  if (blockIdx.x >= a.append_ctas) {
    // queries: a group of lanes a token
    const int groups = (a.heads + a.head_step - 1) / a.head_step;
    const long long at = (long long)(blockIdx.x - a.append_ctas) * kBlockSlots + tid / LANES;
    const int row = (int)(at / groups), h0 = (int)(at % groups) * a.head_step;
    if (at >= (long long)a.q_rows * groups) return;
    const int b = quotient(row, a.by_new), i = row - b * a.n_new;
    rotate_heads<T, D, P, N>(r, steps, false, (const T*)(a.q + b * a.q_batch + i * a.q_token), a.q_head / (int)sizeof(T),
                                  (T*)a.q_out + (long long)row * a.heads * D, D, a.positions[b * a.s_positions + i], p0, h0,
                                  min(h0 + a.head_step, a.heads));
    return;
  }
  const int task = quotient(blockIdx.x, a.by_splits), g0 = (blockIdx.x - task * a.splits) * HEADS;
  const int b = quotient(task, a.by_blocks), nth = task - b * a.blocks, heads = min(HEADS, a.c.n_kv - g0);
  int n;
  const int count = rows_of_sequence(a.c, a.counts, b, a.n_new, n);
  if (count < 0) {
    if (nth == 0 && tid == 0) tell_invalid(a.c);
    return;
  }
  const int slot0 = ((n >> kBlockShift) + nth) << kBlockShift, slot = slot0 + tid / LANES;
  if (max(slot0, n) >= min(slot0 + kBlockSlots, n + count)) return;
  const bool mine = slot >= n && slot < n + count;
  int t = -1;                                                     // the slot's source token
  if (mine) t = a.index ? a.index[b * a.s_index + slot - n] : slot - n;
  const int page = *(const int*)((const char*)a.c.table + b * a.c.s_table + (long long)(slot0 >> a.c.page_shift) * 4);
  const bool is = t >= 0 && t < a.tokens, no_page = page < 0 || page >= a.c.pages;
  if ((mine && !is) || no_page) tell_invalid(a.c);
  if (no_page) return;
  const Place at(r, p0);
  typename Place::Raw raw[S::kStaged ? 1 : JOBS] = {};
  const char *const k_from = a.k + b * a.s_batch + t * a.s_token + g0 * a.s_head, *const v_from = a.v + (k_from - a.k);
  auto place = [&](int j, int chunk) { return staged + (2 * j + chunk) * S::kThreads + tid; };
  const bool any = __any_sync(0xffffffffu, mine);                 // (a decoding step's blocks have one new row)
  if (any)
#pragma unroll
  for (int j = 0; j < JOBS; ++j) {
    const bool there = is && j / 2 < heads;
    const T* const from = (const T*)((j & 1 ? v_from : k_from) + (j / 2) * a.s_head);
    if constexpr (!S::kStaged) {
      if (there) raw[j] = at.load(from);
    } else {
      copy16(place(j, 0), there ? from + at.a : (const T*)a.k, there);
      copy16(place(j, 1), there ? from + at.b : (const T*)a.k, there);
    }
  }
  uint64_t cos[N / 2], sin[N / 2];
  const int position = a.rotated && is ? a.positions[b * a.s_positions + t] : 0;
  if (any && a.rotated) at.angles(r, steps, position, false, cos, sin);
  if constexpr (S::kStaged) copies_landed();
  auto raw_of = [&](int j) {
    if constexpr (S::kStaged) return typename Place::Raw{*place(j, 0), *place(j, 1)};
    else return raw[j];
  };
  auto row_of = [&](int j, float (&u)[N], float (&v)[N]) {
    Place::pairs(raw_of(j), u, v);
    if (!(j & 1) && a.rotated) at.turn(u, v, cos, sin);
  };
  // (positive numbers are ordered as their bits are; NaN has no part in a maximum)
  auto across = [](float x) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x))); };
  // lane j of every warp: the scale of job j, where the block holds tokens already
  const int in_page = slot0 & ((1 << a.c.page_shift) - 1);
  const bool job = lane < JOBS && lane / 2 < heads;
  unsigned char* const scale = (lane & 1 ? a.c.v_scales : a.c.k_scales) +
                               (((size_t)page * a.c.n_kv + g0 + (job ? lane / 2 : 0)) << (a.c.page_shift - kBlockShift)) + (in_page >> kBlockShift);
  const int had = job && slot0 < n ? (int)*scale - 127 : -127;
  bool end = false;                                               // infinities, and numbers that in fp32 may become such or not
  if (!any && lane < JOBS) tops[lane][warp] = exact_tops[lane][warp] = 0.f;
  if (any)
#pragma unroll (S::kUnroll)
  for (int h = 0; h < HEADS; ++h)
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int j = 2 * h + s;
    float top = 0.f;
    if (sizeof(T) == 2 && (s || !a.rotated)) {
      top = largest(raw_of(j));
    } else {
      float u[N], v[N];
      row_of(j, u, v);
#pragma unroll
      for (int i = 0; i < N; ++i) top = max3(top, fabsf(u[i]), fabsf(v[i]));
    }
    top = across(top);
    end |= top >= kEnd;
    if (lane == 0) tops[j][warp] = top;
  }
  end = __syncthreads_or(end);
  auto of_warps = [&](const float (&x)[JOBS][WARPS]) {
    float top = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) top = fmaxf(top, x[lane][w]);
    return top;
  };
  float top = job ? of_warps(tops) : 0.f;
  // A pair's |a| + |b| is at most twice its larger result, so that the largest of K is off by a part of 2^-21.4 of it, with an amplitude 2^-20.6: where that is
  // too close to a border between two scales to tell, 64 bits decide.  Infinities are stored as NaN, and the others' largest is what counts.
  const bool unsure = a.rotated && job && !(lane & 1) && border_near(top);
  if (end || __any_sync(0xffffffffu, unsure)) {                   // (all warps have the same answer)
    if (any)
#pragma unroll 1
    for (int j = 0; j < 2 * heads; ++j) {
      const T* const from = (const T*)((j & 1 ? v_from : k_from) + (j / 2) * a.s_head);
      float largest = 0.f;
      if (is)
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const int2 el = at.pair(i);
        const float2 x = exact_pair((double)(float)from[el.x], (double)(float)from[el.y], !(j & 1) && a.rotated && at.turns(i),
                                    steps[min(p0 + i, D / 2 - 1)], position, r.amplitude64);
        largest = fmaxf(largest, fmaxf(fabsf(x.x), fabsf(x.y)));
      }
      largest = across(largest);
      if (lane == 0) exact_tops[j][warp] = largest;
    }
    __syncthreads();
    if (job) top = of_warps(exact_tops);
  }
  int e = 0, down = 0;                                            // how far older codes go down
  if (job) {
    e = exponent_of(top);
    if (slot0 < n) {
      down = max(0, min(e - had, 24));
      e = max(e, had);
    }
    if (warp == 0) *scale = (unsigned char)(e + 127);
  }
  char *const k = a.c.k + page * a.c.s_page + g0 * a.c.s_head + (in_page + tid / LANES) * a.c.s_token, *const v = a.c.v + (k - a.c.k);
#pragma unroll (S::kUnroll)
  for (int h = 0; h < HEADS; ++h)
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const int j = 2 * h + s;
    const int ej = __shfl_sync(0xffffffffu, e, j), dj = __shfl_sync(0xffffffffu, down, j);
    if (h >= heads) break;
    char* const out = (s ? v : k) + h * a.c.s_head;
    uint32_t differ = 0u;
    if (mine) {
      const float by = __int_as_float((127 - ej) << 23);
      float u[N], w[N];
      const bool turns = !s && a.rotated && (P == SINGLE || at.turns(0));
      row_of(j, u, w);
      if (end) {
        float largest = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          largest = max3(largest, fabsf(u[i]), fabsf(w[i]));
          if (fabsf(u[i]) == INFINITY) u[i] = __int_as_float(0x7fffffff);
          if (fabsf(w[i]) == INFINITY) w[i] = __int_as_float(0x7fffffff);
        }
        if (turns && largest >= kEnd) differ = 1u;                // (what overflowed on the way may be a number)
      }
      uint32_t cx[N / 4], cy[N / 4];
      uint64_t off[N / 2];                                        // what pairs may be off by in fp32, in codes' units: below a quarter of the smallest code
      if (turns) {
        const float part = r.off * by;
        auto of = [&](int i) { return P != SINGLE || at.turns(i) ? fmaf(fabsf(u[i]), part, fabsf(w[i]) * part) : 0.f; };
#pragma unroll
        for (int i = 0; i < N; i += 2) off[i / 2] = pack2(of(i), of(i + 1));
      }
      // codes of the row times f; near: with what it may be off by added
      auto codes_of = [&](float f, bool near, uint32_t (&cx)[N / 4], uint32_t (&cy)[N / 4]) {
        const uint64_t f2 = pack2(f, f);
        float p[N], q[N], x[N], y[N];
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const uint64_t pu = pack2(u[i], u[i + 1]), pw = pack2(w[i], w[i + 1]);
          unpack2(near ? fma2(pu, f2, off[i / 2]) : mul2(pu, f2), p[i], p[i + 1]);
          unpack2(near ? fma2(pw, f2, off[i / 2]) : mul2(pw, f2), q[i], q[i + 1]);
        }
        Place::chunks(p, q, x, y);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
          cx[i] = codes4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
          cy[i] = codes4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        }
      };
      if (turns) {
        // The largest value that there may be and, with its sign turned, the smallest have the same code, or 64 bits decide.  (Their signs differ
        // where both are zeros.)
        uint32_t lx[N / 4], ly[N / 4];
        codes_of(by, true, cx, cy);
        codes_of(-by, true, lx, ly);
#pragma unroll
        for (int i = 0; i < N / 4; ++i) differ |= ((cx[i] ^ lx[i]) | (cy[i] ^ ly[i])) & 0x7f7f7f7fu;
      } else {
        codes_of(by, false, cx, cy);
      }
      if constexpr (P == SINGLE) {
#pragma unroll
        for (int i = 0; i < N; ++i) {                             // (pairs of neighbours in cx, cy)
          const int2 el = at.pair(i);
          const uint32_t c = (i < N / 2 ? cx[i / 2 % (N / 4)] : cy[i / 2 % (N / 4)]) >> (16 * (i % 2));
          out[el.x] = (char)c;
          out[el.y] = (char)(c >> 8);
        }
      } else if constexpr (N == 8) {
        *(uint2*)(out + at.a) = make_uint2(cx[0], cx[1]);
        *(uint2*)(out + at.b) = make_uint2(cy[0], cy[1]);
      } else {
        *(uint32_t*)(out + at.a) = cx[0];
        *(uint32_t*)(out + at.b) = cy[0];
      }
    } else if (dj > 0 && slot < n) {
      // an older token: its codes by the larger scale
      const uint32_t half = dj > 14 ? 1u << (24 - dj) : (uint32_t)(15 - dj) << 10, f = half | half << 16;
      uint2* const at8 = (uint2*)(out + 2 * p0);
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        uint2 c = at8[i];
        c.x = scaled2(c.x & 0xffffu, f) | scaled2(c.x >> 16, f) << 16;
        c.y = scaled2(c.y & 0xffffu, f) | scaled2(c.y >> 16, f) << 16;
        at8[i] = c;
      }
    }
    if (!s && a.rotated) {
      // a lane with a value too close to a border to tell: all that it has of this head, a pair a lane
#pragma unroll 1
      for (unsigned left = __ballot_sync(0xffffffffu, differ != 0u); left; left &= left - 1) {
        const int who = __ffs(left) - 1, its = warp * 32 + who;
        const int source = __shfl_sync(0xffffffffu, t, who), where = __shfl_sync(0xffffffffu, position, who);
        __syncwarp();                                             // (its codes are written)
        if (lane >= N) continue;
        const Place there(r, its % LANES * N);
        const int2 el = there.pair(lane);
        double u, w;
        if constexpr (S::kStaged) {
          const T* const from = (const T*)(staged + (2 * j + (P == NEIGHBOURS && lane >= N / 2)) * S::kThreads + its);
          u = (double)(float)from[P == HALVES ? lane : 2 * lane % N];
          w = (double)(float)from[P == HALVES ? S::kThreads * N + lane : 2 * lane % N + 1];
        } else {
          const T* const from = (const T*)(a.k + b * a.s_batch + source * a.s_token + (g0 + h) * a.s_head);
          u = (double)(float)from[el.x];
          w = (double)(float)from[el.y];
        }
        const float by = __int_as_float((127 - ej) << 23);
        const float2 z = exact_pair(u, w, there.turns(lane), steps[min(there.p0 + lane, D / 2 - 1)], where, r.amplitude64);
        const uint32_t codes = codes4(z.x * by, z.y * by, 0.f, 0.f);
        char* const to = out + (its / LANES - tid / LANES) * a.c.s_token;
        to[el.x] = (char)codes;
        to[el.y] = (char)(codes >> 8);
      }
    }
  }
}

template <typename T, int D, Pairing P, int HEADS>
cudaError_t launch_one(const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st) {
  using S = AppendShape<T, D, P, HEADS>;
  const long long q = a.q ? (long long)a.q_rows * ((a.heads + a.head_step - 1) / a.head_step) : 0, ctas = a.append_ctas + (q + kBlockSlots - 1) / kBlockSlots;
  const cudaError_t e = allow_smem<append_pages<T, D, P, HEADS>>(S::kSmem);
  return e != cudaSuccess ? e : launch_pdl(append_pages<T, D, P, HEADS>, dim3((unsigned)ctas), dim3(S::kThreads), S::kSmem, st, r, a);
}
template <typename T, int D, Pairing P>
struct Launch {
  static cudaError_t run(const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st) {
    return a.splits == a.c.n_kv ? launch_one<T, D, P, 1>(r, a, st) : launch_one<T, D, P, kManyHeads>(r, a, st);
  }
};

}  // namespace

// One head a CTA as long as there are few: 2 x 1000 tokens (1008 CTAs) 6.6 us, four heads a CTA 7.9; 4 x 1000 (2016 CTAs) 10.8, four heads 10.4;
// 64 x 64 (2560) 13.1 and 10.4.
int append_splits(long long blocks, int n_kv, int sms) { return blocks * n_kv <= 8ll * sms || n_kv == 1 ? n_kv : (n_kv + kManyHeads - 1) / kManyHeads; }

cudaError_t launch_append_pages(const Ctx& ctx, const RopeArgs& r, const AppendPagesArgs& a, cudaStream_t st) {
  return by_pairing<Launch>(ctx, pairing_of(r, ctx.cfg.dtype == STRUCTKV_BF16 ? kPairs<__nv_bfloat16> : kPairs<float>), r, a, st);
}

}  // namespace skv
