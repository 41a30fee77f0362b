// Attention of new tokens over a paged cache in 8 bits.
//
// One pass: per row a reference m, sum l and unscaled output O over the keys seen so far.  16 keys at a time, which share a scale of K
// and one of V, give S = K Q^T, y = x + e_v (x in bits, 2^e_v the scale of V), w = 2^(y - m), l += 2^-e_v sum w, O^T += V^T w.  V's scale
// goes with the weights, and references follow what a key weighs in O: codes are exact operands of fp16 products, whose weights keep 11
// bits as long as they matter to O, whatever the scales.  Queries become fp16 as well, times a power of two that brings the
// row's largest element to 2^13 .. 2^14: bf16 queries lose nothing within 2^-28 of it; fp32 ones go in two pieces, as their weights do.
//
// Reading K and V is the bound, so a warp's loads go straight into the operands' registers: keys are the long side of the m16n8k16
// products, and neither the order of a row's elements within QK^T nor that of V's columns matters as long as both sides have the
// same, so that 16 bytes of a row are four products' share of a lane.  A warp takes every NW-th 16 keys of the CTA's run, with
// statistics of its own; nothing is waited for but loads, and a segment's end merges the warps.  References follow a row's maximum only
// where that outgrows it by 2^kSlack.
//
// Single tokens, 32 heads over 8, d 128: 16 x 16384 keys 91 to 97 us, 5.6 to 5.9 TB/s, 85 to 90 % of a measured copy; 16 sequences of 1 to 5003 keys
// 20.6 us, 3 TB/s; 1 x 1024 keys 8.9 to 9.1 us, which is two launches and their chains of loads (lengths, table, codes; partials).
// Four CTAs of four warps an SM (two with 16 rows or fp32): one begins or ends a segment while others stream.  16 x 16384 / 16 ragged, in one sitting:
// one of 14 warps 103 / 25 us, one of 16 98 / 25, two of 7 100 / 22.5, two of 8 92 / 21.6, three of 5 94 / 21.9, four of 4 92 / 21.3.  That leaves 128
// registers, of which d 128 spills 172 bytes (180 with caps; the merging launch 16 of 64).
// Weights of bf16 storage in one piece of 11 bits: a second piece, as fp32 storage has, takes 102.4 us where one takes 95.8 (16 ragged 21.5, 20.6; four
// capped tokens of eight sequences 22.1, 20.1; a step of 32 x 2048 38.4, 36.6).  The results, bf16 themselves, are off by 1.655e-3 to 1.707e-3 of their norm
// with two, which is their own rounding, and by 1.668e-3 to 1.715e-3 with one: 8 % of them are rounded to the other side.
// Codes through shared memory (cp.async, a ring for each warp) took 116 us where loads to registers took 101; e4m3 products (m16n8k32) for
// the scores, whose queries then need three pieces, 115 against 104.
#include <algorithm>

#include "attend_pages.cuh"

namespace skv {
namespace {

constexpr int kTileBlocks = 4;         // blocks of 16 keys of a place

__device__ __forceinline__ uint4 load16(const char* p) {
  uint4 x;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
  return x;
}
__device__ __forceinline__ uint2 load8(const char* p) {
  uint2 x;
  asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "l"(p));
  return x;
}
// What two values lose as fp16, as fp16.
__device__ __forceinline__ uint32_t rest2(float lo, float hi, uint32_t of) {
  float a, b;
  asm("{\n.reg .b16 x, y;\nmov.b32 {x, y}, %2;\ncvt.f32.f16 %0, x;\ncvt.f32.f16 %1, y;\n}" : "=f"(a), "=f"(b) : "r"(of));
  return f16x2(lo - a, hi - b);
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// NR blocks of 8 rows, NW warps.
template <int D, int NR, int NW>
struct PagesShape {
  static constexpr int RB = 8 * NR, kRow = D + 4, kSet = RB * kRow + 16;   // of a warp's output: neighbouring warps' are in other banks
  static constexpr int kRefs = NW <= 8 ? 8 : 16;                // a row's references that are read together
  static constexpr int kSmem = (NW * kSet + 2 * RB * kRefs) * 4;
  static_assert(NW <= 16 && kRefs - NW <= 8, "references of warps that there are not");
};

// F32: fp32 storage; CAP: capped scores.
template <int D, int NR, bool F32, bool CAP, int NW, int PER>
__global__ void __launch_bounds__(NW * 32, PER) attend_pages(const __grid_constant__ AttendPagesArgs a) {
  using S = PagesShape<D, NR, NW>;
  constexpr int RB = S::RB, KK = D / 16, KH = D / 64, PIECES = F32 ? 2 : 1, VW = D / 32, RW = S::kRefs;   // VW: words of V a lane has of a key
  extern __shared__ __align__(16) float smem[];
  float* const outs = smem;                                      // [warp] [RB][kRow]
  float* const refs = outs + NW * S::kSet;                       // [RB][kRefs], by warps
  float* const sums = refs + RB * RW;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g8 = lane >> 2, t4 = lane & 3;
  pdl_trigger();
  pdl_wait();
  const PageRun run = find_run(a);
  PageSegment sg = first_segment(a, run);
  const int sh4 = a.c.page_shift - kBlockShift, per_page = 1 << sh4, token = a.c.s_token;

  // A warp has every NW-th 16 keys of a segment.  Lane i knows the page and the scales of the i-th of 32 that it has, and in good time of the
  // 32 behind them; K's scale is 256 where the page is none: its slots are not seen (and its loads go to page 0).
  int b, g, rb, n_old, s, s_end, page, ks, vs, page_after = 0, ks_after = 0, vs_after = 0;
  const char *k0, *v0;
  const int* table;
  auto look = [&](int step, int& k, int& v) {                    // (nothing is made of the scales here: they may be on their way)
    int p = 0;
    k = 256;
    v = 127;
    if (step < s_end) {
      p = table[step >> sh4];
      if ((unsigned)p >= (unsigned)a.c.pages) {
        p = 0;
      } else {
        const unsigned at = (((unsigned)p * a.c.n_kv + g) << sh4) + (step & (per_page - 1));
        k = a.c.k_scales[at];
        v = a.c.v_scales[at];
      }
    }
    return p;
  };
  // this lane's rows of K (keys g8 and g8 + 8) and of V (keys 2 t4, + 1, + 8, + 9)
  uint4 kb[2][KH];
  uint32_t vb[4][VW];
  auto bytes_of = [&](int step, int p) { return (long long)((unsigned long long)(unsigned)p * (unsigned)a.c.s_page) + (step & (per_page - 1)) * (token << kBlockShift); };
  auto load_k = [&](long long at) {
    const char* const from = k0 + at;
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int h = 0; h < KH; ++h) kb[y][h] = load16(from + y * 8 * token + h * 64);
  };
  auto load_v = [&](long long at) {
    const char* const from = v0 + at;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const char* const at = from + ((e & 1) + 8 * (e >> 1)) * token;
      if constexpr (VW == 4) {
        const uint4 w = load16(at);
        vb[e][0] = w.x; vb[e][1] = w.y; vb[e][2] = w.z; vb[e][3] = w.w;
      } else {
        const uint2 w = load8(at);
        vb[e][0] = w.x; vb[e][1] = w.y;
      }
    }
  };
  // A lane's elements of row g8 (+ 8) as they lie in memory: 16 of each 64.
  constexpr int QW = F32 ? 4 : 2;                                // words of four
  uint32_t xq[NR][KK][QW];
  // A segment begins: its rows and its first keys are on their way.
  auto begin = [&]() {
    b = sg.b;
    g = quotient(sg.nth, a.by_blocks);
    rb = sg.nth - g * a.blocks;
    n_old = sg.n;
    s = sg.t0 * kTileBlocks + warp;
    s_end = min(sg.t1 * kTileBlocks, (sg.keys + 15) / 16);
    table = (const int*)((const char*)a.c.table + b * a.c.s_table);
    k0 = a.c.k + g * a.c.s_head + (long long)g8 * token + t4 * 16;
    v0 = a.c.v + g * a.c.s_head + 2ll * t4 * token + g8 * (VW * 4);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = min(rb * RB + 8 * i + g8, a.rows - 1), tok = quotient(r, a.by_group), h = r - tok * a.group;   // (rows behind the last: it again)
      const char* const q = a.q + b * a.q_batch + tok * a.q_token + (g * a.group + h) * a.q_head + t4 * (F32 ? 64 : 32);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int w = 0; w < QW; w += 2) {
          const uint2 x = *(const uint2*)(q + kk / 4 * (F32 ? 256 : 128) + kk % 4 * (QW * 4) + w * 4);
          xq[i][kk][w] = x.x;
          xq[i][kk][w + 1] = x.y;
        }
    }
    page = look(s + lane * NW, ks, vs);
    const long long at = bytes_of(s, __shfl_sync(0xffffffffu, page, 0));
    if (s < s_end) {
      load_k(at);
      load_v(at);
    }
  };
  if (sg.t1) begin();
#pragma unroll 1
  while (sg.t1) {
    const int first_row = rb * RB + 2 * t4, s0 = sg.t0 * (kTileBlocks);
    // the rows
    uint32_t qf[PIECES][NR][KK][2];
    float qs[NR][2];                                             // a row's factor: scale in bits (capped scores: 1), times 2^-the raise of its queries
    float o[NR][KK][4], m[NR][2], l[NR][2];                      // o[.][t]: columns 16 g8 (8 g8) + 2 t and + 1 of rows 2 t4 and + 1
    int last[NR][2];                                             // the last slot that a row sees
    bool far = false;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      float x[KK][4], top = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t w = xq[i][kk][F32 ? e % QW : e / 2];
          x[kk][e] = __uint_as_float(F32 ? w : e % 2 ? w & 0xffff0000u : w << 16);
          top = fmaxf(top, fabsf(x[kk][e]));
        }
      }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // raise: top's exponent becomes 13  (rows of zeros, tiny or infinite ones: as far as fp32's exponents go)
      const int raise = min(max(13 - ((int)(__float_as_uint(top) >> 23) - 127), -113), 126);
      const float up = exp2i(raise);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float lo = x[kk][2 * y] * up, hi = x[kk][2 * y + 1] * up;
          qf[0][i][kk][y] = f16x2(lo, hi);
          if (F32) qf[PIECES - 1][i][kk][y] = rest2(lo, hi, qf[0][i][kk][y]);
        }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int down = __shfl_sync(0xffffffffu, raise, (2 * t4 + e) * 4);
        qs[i][e] = exp2i(-down) * (CAP ? 1.f : a.scale2);
        last[i][e] = n_old + quotient(min(first_row + 8 * i + e, a.rows - 1), a.by_group);
        m[i][e] = kNothing;
        l[i][e] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < KK; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.f;
    }

#pragma unroll 1
    for (int nth = 0; s < s_end; ++nth, s += NW) {
      const int ahead = s + NW, j0 = s << kBlockShift, i32 = nth & 31;
      if (i32 == 0 && nth > 0) {
        page = page_after;
        ks = ks_after;
        vs = vs_after;
      }
      if (i32 == 8 && s + 24 * NW < s_end) page_after = look(s + (24 + lane) * NW, ks_after, vs_after);
      const int ke = __shfl_sync(0xffffffffu, ks, i32), ve = __shfl_sync(0xffffffffu, vs, i32);
      const int page_ahead = __shfl_sync(0xffffffffu, i32 < 31 ? page : page_after, (i32 + 1) & 31);
      const bool bad = ke == 256;
      const long long at_ahead = bytes_of(ahead, page_ahead);
      // products: two chains where a warp has one block of rows
      constexpr int CHAINS = NR == 1 ? 2 : 1;
      float acc[CHAINS][NR][4];
#pragma unroll
      for (int c = 0; c < CHAINS; ++c)
#pragma unroll
        for (int i = 0; i < NR; ++i) acc[c][i][0] = acc[c][i][1] = acc[c][i][2] = acc[c][i][3] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        const uint32_t* const w0 = (const uint32_t*)&kb[0][kk / 4];
        const uint32_t* const w1 = (const uint32_t*)&kb[1][kk / 4];
        const uint32_t x0 = half_lo(w0[kk % 4]), x1 = half_lo(w1[kk % 4]), x2 = half_hi(w0[kk % 4]), x3 = half_hi(w1[kk % 4]);
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
          for (int i = 0; i < NR; ++i) mma(acc[kk % CHAINS][i], x0, x1, x2, x3, qf[p][i][kk][0], qf[p][i][kk][1]);
      }
      const float kf = __int_as_float(ke << 23), vl = __int_as_float((254 - ve) << 23), vx = __int_as_float(0x4b000000 | ve) - (0x1p23f + 127.f);
      // y, element 2 z + x: key g8 + 8 z, row x; less the reference, or without.  References are whole numbers, so that vx - m is exact.  So far
      // from zero that an unrounded product and a rounded reference are off by a part of a bit, products are rounded as references are.
      float y[NR][4];
      auto scores = [&](int i, bool bare) {
        float z[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = CHAINS == 2 ? acc[0][i][e] + acc[CHAINS - 1][i][e] : acc[0][i][e];
        const float f[2] = {qs[i][0] * kf, qs[i][1] * kf};
        if (CAP) {
#pragma unroll
          for (int e = 0; e < 4; ++e) z[e] *= f[e & 1];
          capped2(z[0], z[1], pack2(a.cap2, a.cap2), pack2(a.inv_cap, a.inv_cap));
          capped2(z[2], z[3], pack2(a.cap2, a.cap2), pack2(a.inv_cap, a.inv_cap));
        }
        if (bare || far) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[i][e] = __fadd_rn(CAP ? z[e] : __fmul_rn(z[e], f[e & 1]), vx);
            if (!bare) y[i][e] = __fadd_rn(y[i][e], -m[i][e & 1]);
          }
        } else {
          const float c[2] = {vx - m[i][0], vx - m[i][1]};
#pragma unroll
          for (int e = 0; e < 4; ++e) y[i][e] = CAP ? z[e] + c[e & 1] : fmaf(z[e], f[e & 1], c[e & 1]);
        }
      };
      if (ahead < s_end) load_k(at_ahead);
      const bool tail = j0 + 16 > n_old + 1 || bad;
      auto hide = [&](int i) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (bad || j0 + g8 + 8 * (e >> 1) > last[i][e & 1]) y[i][e] = -INFINITY;
      };
      // references: those that are outgrown follow, and the scores are worked out again
#pragma unroll 1
      for (bool again = false;; again = true) {
        bool grown = false;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          scores(i, false);
          if (tail) hide(i);
          grown |= fmaxf(fmaxf(y[i][0], y[i][1]), fmaxf(y[i][2], y[i][3])) > kRaise + kSlack;
        }
        if (!__any_sync(0xffffffffu, grown) || again) break;
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          scores(i, true);
          if (tail) hide(i);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = fmaxf(y[i][e], y[i][2 + e]);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            t = fmaxf(ceilf(t) - kRaise, m[i][e]);
            const float f = fast_exp2(m[i][e] - t);
            m[i][e] = t;
            if (t != kNothing) top = fmaxf(top, fabsf(t));
            l[i][e] *= f;
#pragma unroll
            for (int k = 0; k < KK; ++k) { o[i][k][e] *= f; o[i][k][2 + e] *= f; }
          }
        }
        far = __any_sync(0xffffffffu, top > 0x1p20f);
      }
      uint32_t odd[4] = {0u, 0u, 0u, 0u};                        // columns of the lane's four keys whose V is NaN, as bits
      bool any_odd = false;
      if (tail) {
        if (bad && lane == 0) tell_invalid(a.c);
        // What holds NaN here reaches only rows that see it (0 x NaN): it is taken out, and put to those at the end.
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            const uint32_t is = nan_bytes(vb[e][w]);
            vb[e][w] &= ~((is >> 7) * 0xffu);
            odd[e] |= ((is >> 7 & 1) | (is >> 14 & 2) | (is >> 21 & 4) | (is >> 28 & 8)) << (4 * w);
          }
        any_odd = __any_sync(0xffffffffu, (odd[0] | odd[1] | odd[2] | odd[3]) != 0) && !bad;
      }
      uint32_t pf[PIECES][NR][2];                                // keys 2 t4 and + 1 (+ 8), row g8
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = fast_exp2(y[i][e]);
        l[i][0] = fmaf(p[0] + p[2], vl, l[i][0]);
        l[i][1] = fmaf(p[1] + p[3], vl, l[i][1]);
        // weights keep 11 bits for the product (22 for fp32 storage); the sum is of the unrounded ones
        const uint32_t w0 = f16x2(p[0], p[1]), w1 = f16x2(p[2], p[3]);
        pf[0][i][0] = transposed(w0);
        pf[0][i][1] = transposed(w1);
        if (F32) {
          pf[PIECES - 1][i][0] = transposed(rest2(p[0], p[1], w0));
          pf[PIECES - 1][i][1] = transposed(rest2(p[2], p[3], w1));
        }
      }
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        const uint32_t a0 = __byte_perm(vb[0][w], vb[1][w], 0x5140), a1 = __byte_perm(vb[0][w], vb[1][w], 0x7362);
        const uint32_t b0 = __byte_perm(vb[2][w], vb[3][w], 0x5140), b1 = __byte_perm(vb[2][w], vb[3][w], 0x7362);
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const uint32_t x = z ? a1 : a0, x2 = z ? b1 : b0, f0 = half_lo(x), f1 = half_hi(x), f2 = half_lo(x2), f3 = half_hi(x2);
#pragma unroll
          for (int q = 0; q < PIECES; ++q)
#pragma unroll
            for (int i = 0; i < NR; ++i) mma(o[i][2 * w + z], f0, f1, f2, f3, pf[q][i][0], pf[q][i][1]);
        }
      }
      if (ahead < s_end) load_v(at_ahead);
      if (any_odd) {
#pragma unroll 1
        for (int c = 0; c < 16; ++c) {                           // lane c / 4 of the four has key 2 (c / 4) + (c & 1) + 8 (c / 2 & 1)
          const uint32_t mine = c & 2 ? (c & 1 ? odd[3] : odd[2]) : (c & 1 ? odd[1] : odd[0]);
          const uint32_t cols = __shfl_sync(0xffffffffu, mine, (lane & 28) | c >> 2);
          const int j = j0 + 2 * (c >> 2) + (c & 1) + 8 * (c >> 1 & 1);
#pragma unroll
          for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if ((cols >> (2 * k + (e >> 1)) & 1) && j <= last[i][e & 1]) o[i][k][e] = __int_as_float(0x7fffffff);
        }
      }
    }

    // the segment ends: its warps' outputs, each against its own reference, then their sum against a common one
    const int sets = min(NW, s_end - s0), rows = min(RB, a.rows - rb * RB);
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) l[i][e] += __shfl_xor_sync(0xffffffffu, l[i][e], d);
        const int row = 8 * i + 2 * t4 + e;
        if (row >= rows) continue;
        if (g8 == 0) {
          refs[row * RW + warp] = m[i][e] == kNothing ? -INFINITY : m[i][e];
          sums[row * RW + warp] = l[i][e];
        }
        if (warp == 0 && NW + g8 < RW) refs[row * RW + NW + g8] = -INFINITY;
        if (warp < sets) {
          float* const to = outs + warp * S::kSet + row * S::kRow + g8 * (2 * KK);
#pragma unroll
          for (int k = 0; k < KK; k += 2) *(float4*)(to + 2 * k) = make_float4(o[i][k][e], o[i][k][2 + e], o[i][k + 1][e], o[i][k + 1][2 + e]);
        }
      }
    __syncthreads();
    const int item = b * a.c.n_kv * a.blocks + sg.nth, slot = item + blockIdx.x;
    if (tid == 0 && sg.t0 == 0) {
      // who merges this item: where its partials lie, and how many they are
      const int end = sg.at + a.over + sg.tiles - 1;
      a.item_parts[item] = make_int2(slot, cta_of(run.all, end) - (int)blockIdx.x + 1);
    }
    next_segment(sg, a);
    if (sg.t1) begin();
    // two neighbouring threads have four columns of a row, of every other warp
#pragma unroll 1
    for (int i = tid / 2; i < rows * (D / 4); i += NW * 16) {
      const int row = i / (D / 4), c4 = i % (D / 4), odd = tid & 1;
      float ref[RW], top = -INFINITY;
#pragma unroll
      for (int w = 0; w < RW; w += 4) {
        const float4 x = *(const float4*)(refs + row * RW + w);
        ref[w] = x.x; ref[w + 1] = x.y; ref[w + 2] = x.z; ref[w + 3] = x.w;
        top = fmaxf(fmaxf(fmaxf(top, x.x), fmaxf(x.y, x.z)), x.w);
      }
      const float base = top == -INFINITY ? 0.f : top;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      float sum = 0.f;
      const float* const from = outs + row * S::kRow + c4 * 4;
#pragma unroll
      for (int w = 0; w < NW; w += 2) {
        const int my = w + odd;
        if (my < sets) {
          const float f = fast_exp2((odd ? ref[(w + 1) % RW] : ref[w]) - base);
          const float4 x = *(const float4*)(from + my * S::kSet);
          sum = fmaf(f, sums[row * RW + my], sum);
          v.x = fmaf(f, x.x, v.x); v.y = fmaf(f, x.y, v.y); v.z = fmaf(f, x.z, v.z); v.w = fmaf(f, x.w, v.w);
        }
      }
      // (a warp has sixteen neighbouring pieces, and there are a multiple of as many: it is whole here)
      auto add = [&](float& x) { x += __shfl_xor_sync(0xffffffffu, x, 1); };
      add(v.x); add(v.y); add(v.z); add(v.w); add(sum);
      if (odd) continue;
      *(float4*)(a.part_out + ((size_t)slot * RB + row) * D + c4 * 4) = v;
      if (c4 == 0) a.part_stat[(size_t)slot * RB + row] = make_float2(top, sum);
    }
    __syncthreads();
  }
}

// Merges an item's partials: M = max m_c, out = sum 2^(m_c - M) O_c / sum 2^(m_c - M) l_c.  2^by warps of a block share a row's; each takes them in
// order, and their results are joined in order.  Blocks of 128 threads find room beside an attention CTA and so are there when it ends.
// About 3 us behind the attention at every listed size: launch, where the partials are, partials (eight on their way at once).
constexpr int kFinishThreads = 128;

template <int D, bool F32>
__global__ void __launch_bounds__(kFinishThreads, 8) attend_pages_finish(const __grid_constant__ AttendPagesArgs a, int rb_shift, int by) {
  constexpr int DL = D / 32, kAhead = 8, kWarps = kFinishThreads / 32;
  __shared__ float s_out[kWarps][D];
  __shared__ float2 s_stat[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, mine = warp & ((1 << by) - 1);
  const int at = blockIdx.x * (kWarps >> by) + (warp >> by);
  const bool is = at < a.c.batch * a.c.n_kv * a.rows;
  const int u = quotient(is ? at : 0, a.by_rows), r = is ? at - u * a.rows : 0, rb = r >> rb_shift;
  const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, tok = quotient(r, a.by_group), h = r - tok * a.group;
  pdl_trigger();
  pdl_wait();
  int n;
  const int2 where = a.item_parts[u * a.blocks + rb];
  const int count = rows_of_sequence(a.c, a.counts, b, a.n_new, n), parts = is && tok < count ? where.y : 0;
  float M = -INFINITY, L = 0.f, acc[DL];
#pragma unroll
  for (int e = 0; e < DL; ++e) acc[e] = 0.f;
  auto join = [&](float2 st, const float (&x)[DL], float ref) {
    if (st.x == -INFINITY && st.y == 0.f) return;                  // (may not have been written)
    const float w = fast_exp2(st.x - ref);
    L = fmaf(w, st.y, L);
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[d] = fmaf(w, x[d], acc[d]);
  };
  auto rescale = [&](float top) {
    const float ref = top == -INFINITY ? 0.f : top, f = fast_exp2(M - ref);
    M = top;
    L *= f;
#pragma unroll
    for (int d = 0; d < DL; ++d) acc[d] *= f;
    return ref;
  };
  // (this warp's are neighbours)
  const int share = (parts + (1 << by) - 1) >> by, first = where.x + mine * share, left = min(share, parts - mine * share);
  const int row = r & ((1 << rb_shift) - 1);
  const float2* const stat = a.part_stat + ((size_t)first << rb_shift) + row;
  const float* const from = a.part_out + (((size_t)first << rb_shift) + row) * D + lane * DL;
#pragma unroll 1
  for (int c = 0; c < left; c += kAhead) {
    float2 st[kAhead];
    float x[kAhead][DL];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const size_t k = (size_t)min(c + e, left - 1) << rb_shift;
      st[e] = stat[k];
      if constexpr (DL == 4) {
        const float4 v = *(const float4*)(from + k * D);
        x[e][0] = v.x; x[e][1] = v.y; x[e][2] = v.z; x[e][3] = v.w;
      } else {
        const float2 v = *(const float2*)(from + k * D);
        x[e][0] = v.x; x[e][1] = v.y;
      }
    }
    float top = M;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) top = fmaxf(top, st[e].x);
    const float ref = rescale(top);
#pragma unroll
    for (int e = 0; e < kAhead; ++e)
      if (c + e < left) join(st[e], x[e], ref);
  }
  if (by) {
    if (mine) {
#pragma unroll
      for (int d = 0; d < DL; ++d) s_out[warp][lane * DL + d] = acc[d];
      if (lane == 0) s_stat[warp] = make_float2(M, L);
    }
    __syncthreads();
    if (mine) return;
    float top = M;
    for (int k = 1; k < 1 << by; ++k) top = fmaxf(top, s_stat[warp + k].x);
    const float ref = rescale(top);
    for (int k = 1; k < 1 << by; ++k) {
      float x[DL];
#pragma unroll
      for (int d = 0; d < DL; ++d) x[d] = s_out[warp + k][lane * DL + d];
      join(s_stat[warp + k], x, ref);
    }
  }
  if (!is) return;
  const bool nothing = M == -INFINITY && L == 0.f;
  const float inv = nothing ? 0.f : 1.f / L;
  const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
#pragma unroll
  for (int d = 0; d < DL; ++d) acc[d] = nothing ? 0.f : acc[d] * inv;
  if constexpr (F32) {
    if constexpr (DL == 4) *(float4*)((float*)a.out + q * D + lane * DL) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    else *(float2*)((float*)a.out + q * D + lane * DL) = make_float2(acc[0], acc[1]);
  } else {
    if constexpr (DL == 4) *(uint2*)(a.out + (q * D + lane * DL) * 2) = make_uint2(bf16x2(acc[0], acc[1]), bf16x2(acc[2], acc[3]));
    else *(uint32_t*)(a.out + (q * D + lane * DL) * 2) = bf16x2(acc[0], acc[1]);
  }
  if (lane == 0 && a.lse) a.lse[q] = nothing ? -INFINITY : (M + log2f(L)) * kLn2;
}

template <int D, int NR, bool F32, bool CAP, int NW, int PER>
cudaError_t launch_one(const AttendPagesArgs& a, cudaStream_t st) {
  using S = PagesShape<D, NR, NW>;
  const cudaError_t e = allow_smem<attend_pages<D, NR, F32, CAP, NW, PER>>(S::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_pages<D, NR, F32, CAP, NW, PER>, dim3(a.ctas), dim3(NW * 32), S::kSmem, st, a);
}
template <int D, bool CAP>
cudaError_t launch_rows(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st) {
  if (ctx.cfg.dtype == STRUCTKV_FP32) return launch_one<D, 1, true, CAP, 4, 2>(a, st);
  return p.rb == 8 ? launch_one<D, 1, false, CAP, 4, 4>(a, st) : launch_one<D, 2, false, CAP, 4, 2>(a, st);
}

}  // namespace

cudaError_t launch_attend_pages(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st) {
  if (ctx.cfg.head_dim == 128) return a.cap2 != 0.f ? launch_rows<128, true>(ctx, a, p, st) : launch_rows<128, false>(ctx, a, p, st);
  return a.cap2 != 0.f ? launch_rows<64, true>(ctx, a, p, st) : launch_rows<64, false>(ctx, a, p, st);
}

cudaError_t launch_attend_pages_finish(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st) {
  const long long rows = (long long)a.c.batch * a.c.n_kv * a.rows;
  int by = 0, rb_shift = 3;                                       // (as many warps as the SMs hold beside an attention CTA)
  while (by < 2 && rows << by < 4 * ctx.sm_count) ++by;
  while (1 << rb_shift < p.rb) ++rb_shift;
  const dim3 grid((unsigned)(((rows << by) + 3) / 4));
  const bool f32 = ctx.cfg.dtype == STRUCTKV_FP32;
  auto* const kernel = ctx.cfg.head_dim == 128 ? (f32 ? attend_pages_finish<128, true> : attend_pages_finish<128, false>)
                                               : (f32 ? attend_pages_finish<64, true> : attend_pages_finish<64, false>);
  return launch_pdl(kernel, grid, dim3(kFinishThreads), 0, st, a, rb_shift, by);
}

}  // namespace skv
