// Attention of new tokens over a paged cache in 8 bits where a KV head has more than 16 rows.
//
// S = K Q^T's rows and O += P V on the tensor cores (tcgen05): tiles of 128 rows x 128 keys, lane = row.  Two streams, the even and the odd
// tiles of a segment, alternate, so that one's products run beside the other's exponentials; each leaves a partial.  K and V come as codes:
// a stream's four producing warps copy them lane by lane (cp.async, two units ahead), widen them to fp16, which is exact, and lay
// them out as the products' operands; a code is widened once for all rows.  Scales stay out of the operands: in bits, a score is
// s f 2^e_k and its weight in O 2^(s f 2^e_k + e_v - m), one multiply-add with two numbers for each 16 keys.  References, weights and queries
// as in attend_pages.cu.
//
// Warps: 0-3 and 4-7 bring a segment's rows (0-3) and are the streams' softmax; 8-11 and 12-15 produce; 16 and 17 issue the streams' products.
// A tile's scores are read twice, for their maximum and for the exponentials: 18 warps have 112 registers.
#include <algorithm>

#include "attend_pages.cuh"
#include "attend_tc.cuh"

namespace skv {
namespace {

constexpr int kThreads = 576, kBlocks = kTile / kBlockSlots;     // blocks of slots of a tile

__device__ __forceinline__ void copy16(uint32_t to, const char* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_landed() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ uint4 shared16(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ void put16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ float greatest16(const float* v) {
  float a = max3(v[0], v[1], v[2]), b = max3(v[3], v[4], v[5]);
#pragma unroll
  for (int e = 6; e < 14; e += 4) {
    a = max3(a, v[e], v[e + 1]);
    b = max3(b, v[e + 2], v[e + 3]);
  }
  return fmaxf(max3(a, v[14], v[15]), b);
}

template <int D>
struct PagesTc {
  static constexpr int kUnit = kTile * D * 2, kRaw = kTile * D;   // K or V of a tile, as operands and as codes
  static constexpr int kOps = kUnit, kRaws = kOps + 4 * kUnit, kInfo = kRaws + 4 * kRaw, kQs = kInfo + 4 * kBlocks * 16, kBars = kQs + kTile * 4;
  static constexpr int kSmem = kBars + 256 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

template <int D, bool CAP>
__global__ void __launch_bounds__(kThreads, 1) attend_pages_tc(const __grid_constant__ AttendPagesArgs a) {
  using S = PagesTc<D>;
  constexpr int RB = kTile;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  // (stream s, K or V: operands, codes; a job's numbers for every 16 keys: K's scale, exponent of V's, its inverse)
  auto operand = [&](int s, int v) { return (uint32_t)(S::kOps + (2 * s + v) * S::kUnit); };
  float4* const info = (float4*)(sm + S::kInfo);                 // [stream][job mod 2][block]
  float* const qs = (float*)(sm + S::kQs);                       // a row's factor: scale in bits (capped scores: 1) times 2^-the raise of its queries
  const uint32_t bars = base + S::kBars;
  auto full = [&](int s, int v) { return bars + 8 * (2 * s + v); };
  auto empty = [&](int s, int v) { return bars + 32 + 8 * (2 * s + v); };
  auto s_full = [&](int s) { return bars + 64 + 8 * s; };
  auto p_ready = [&](int s) { return bars + 80 + 8 * s; };
  auto o_done = [&](int s) { return bars + 96 + 8 * s; };
  auto o_free = [&](int s) { return bars + 112 + 8 * s; };
  auto drained = [&](int s) { return bars + 128 + 8 * s; };
  const uint32_t q_full = bars + 144, q_empty = bars + 152;
  volatile int* const words = (volatile int*)(sm + S::kBars + 160);
  volatile int *const abort_flag = words, *const odd_v = words + 2;   // odd_v[s]: in a tile of stream s some new token's V was NaN
  volatile uint32_t* const tmem_at = (volatile uint32_t*)words + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, token = a.c.s_token;
  pdl_trigger();
  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      for (int v = 0; v < 2; ++v) { mbar_init(full(s, v), 128); mbar_init(empty(s, v), 1); }
      mbar_init(s_full(s), 1); mbar_init(p_ready(s), 4); mbar_init(o_done(s), 1); mbar_init(o_free(s), 4); mbar_init(drained(s), 1);
    }
    mbar_init(q_full, 128);
    mbar_init(q_empty, 10);                                        // softmax's warps, products' warps
    *abort_flag = 0;
    odd_v[0] = odd_v[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 16) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_at)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  __syncthreads();
  pdl_wait();
  const PageRun run = find_run(a);
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  PageSegment sg = first_segment(a, run);
  const bool work = sg.t1 > 0;
  // (one answer for the warp: what follows is for all of its lanes)
  auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };
  auto wait_long = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait_producer(bar, parity, abort_flag, kWaitCycles)); };
  auto jobs_of = [](const PageSegment& x, int s) { return (x.t1 - x.t0 + 1 - s) / 2; };
  const int sh4 = a.c.page_shift - kBlockShift, per_page = 1 << sh4;

  if (work && warp >= 16) {
    // Products of stream s, each job's scores made after the outputs of the job before.
    const int s = warp - 16;
    const uint32_t lead = lane == 0;
    constexpr uint32_t kF16 = 1u << 4;                             // fp16 operands, fp32 results
    const uint32_t idesc_s = kF16 | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kTile >> 4) << 24 | (a.scale2 < 0.f ? 1u << 13 : 0u);
    constexpr uint32_t idesc_o = kF16 | (uint32_t)(D >> 3) << 17 | (uint32_t)(kTile >> 4) << 24 | kTransposeB;
    const uint64_t q_desc = smem_desc(base), k_desc = smem_desc(base + operand(s, 0)), v_desc = smem_desc_n(base + operand(s, 1));
    const uint32_t q_lo = (uint32_t)q_desc, k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc, hi_k = (uint32_t)(q_desc >> 32), hi_v = (uint32_t)(v_desc >> 32);
    const uint32_t s_at = tmem + s * 128, o_at = tmem + 256 + s * 128;
    int seg = 0, done = 0, used = 0;                               // segments, jobs, segments with jobs
    bool ok = true;
    do {
      const int jobs = jobs_of(sg, s);
      auto scores = [&](int job) {
        if (!(ok = wait(full(s, 0), job & 1))) return;
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          mma_ss(s_at, q_lo + (((kk / 4) * RB * 128 + (kk % 4) * 32) >> 4), k_lo + (((kk / 4) * kTile * 128 + (kk % 4) * 32) >> 4), hi_k, idesc_s, kk > 0, lead);
        commit_by(lead, s_full(s));
        commit_by(lead, empty(s, 0));
      };
      // (a stream without a tile in the segment says as well that it came by: else its wait might be for a phase that is gone)
      if ((ok = wait(q_full, seg & 1)) && lead) mbar_arrive(q_empty);
      if (ok && jobs > 0) scores(done);
#pragma unroll 1
      for (int k = 0; k < jobs && ok; ++k) {
        if (!(ok = wait(full(s, 1), done & 1))) break;
        if (k == 0 && used++ > 0 && !(ok = wait(o_free(s), used & 1))) break;
        if (!(ok = wait(p_ready(s), done & 1))) break;
        tc_fence_after();
#pragma unroll
        for (int kk = 0; kk < kTile / 16; ++kk) mma_ts(o_at, s_at + kk * 8, v_lo + ((kk * 16 * 128) >> 4), hi_v, idesc_o, k > 0 || kk > 0, lead);
        commit_by(lead, o_done(s));
        commit_by(lead, empty(s, 1));
        ++done;
        if (k + 1 < jobs) scores(done);
      }
      ++seg;
      next_segment(sg, a);
    } while (ok && sg.t1);
    commit_by(lead, drained(s));
    if (!mbar_drain(drained(s), 0, abort_flag)) *abort_flag = 2;
  } else if (work && warp >= 8) {
    // Producers of stream s: a warp has two blocks of 16 keys of every tile.  Lane i knows page and scales of block i mod 2 of the (i / 2)-th of
    // the next 16 jobs, and of the 16 behind them: bytes of K's and V's scale, and above them whether there is nothing (a block behind
    // the last key, or a page that is none).
    constexpr int NI = D / 32;                                     // 16-byte pieces of a block that a lane has
    const int s = (warp - 8) / 4, pw = warp & 3;
    const int c = D == 128 ? (lane & 3) | (lane & 8) >> 1 : lane & 3, row = D == 128 ? (lane >> 2 & 1) | lane >> 4 << 1 : lane >> 2;   // of piece 0
    constexpr int kRows = 16 / NI;                                 // rows from piece to piece
    const uint32_t raw = base + S::kRaws + s * 2 * S::kRaw + pw * (2 * NI * 512) + lane * 16;
    int j = 0, jobs = 0, page = 0, page_after = 0;
    unsigned about = 0, about_after = 0;
    const int* table = nullptr;
    const char *k0 = nullptr, *v0 = nullptr;
    int g = 0, n_old = 0;
    auto look = [&](int job, unsigned& what) {
      const int t = sg.t0 + s + 2 * job, step = t * kBlocks + 2 * pw + (lane & 1);
      int p = 0;
      what = 1u << 16;
      if (t < sg.t1 && step * 16 < sg.keys) {
        p = table[step >> sh4];
        if ((unsigned)p >= (unsigned)a.c.pages) {
          p = 0;
          tell_invalid(a.c);
        } else {
          const unsigned at = (((unsigned)p * a.c.n_kv + g) << sh4) + (step & (per_page - 1));
          what = a.c.k_scales[at] | (unsigned)a.c.v_scales[at] << 8;
        }
      }
      return p;
    };
    // A job: its tile, its sequence's keys and old ones among them, pages and scales of this warp's blocks.
    struct Job { int t, keys, n_old, page[2]; unsigned what[2]; const char *k, *v; bool live; };
    auto here = [&]() {
      Job x{sg.t0 + s + 2 * j, sg.keys, n_old, {}, {}, k0, v0, sg.t1 > 0};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        x.page[e] = __shfl_sync(0xffffffffu, page, 2 * (j & 15) + e);
        x.what[e] = __shfl_sync(0xffffffffu, about, 2 * (j & 15) + e);
      }
      return x;
    };
    auto enter = [&]() {                                           // the first segment from here on that has a job for this stream
      while (sg.t1 && jobs_of(sg, s) == 0) next_segment(sg, a);
      j = 0;
      if (sg.t1 == 0) return;
      jobs = jobs_of(sg, s);
      g = quotient(sg.nth, a.by_blocks);
      n_old = a.c.lengths[sg.b];
      table = (const int*)((const char*)a.c.table + sg.b * a.c.s_table);
      k0 = a.c.k + g * a.c.s_head + (long long)row * token + c * 16;
      v0 = a.c.v + g * a.c.s_head + (long long)row * token + c * 16;
      page = look(lane >> 1, about);
      page_after = look(16 + (lane >> 1), about_after);
    };
    auto next = [&]() {
      if (++j == jobs) {
        next_segment(sg, a);
        enter();
      } else if ((j & 15) == 0) {
        page = page_after;
        about = about_after;
        page_after = look(j + 16 + (lane >> 1), about_after);
      }
    };
    auto copy = [&](const Job& x, int v) {
      if (x.live)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (x.what[e] >> 16) continue;
          const int block = (x.t * kBlocks + 2 * pw + e) & (per_page - 1);
          const char* const from = (v ? x.v : x.k) + (long long)((unsigned long long)(unsigned)x.page[e] * (unsigned)a.c.s_page) + block * (token << kBlockShift);
#pragma unroll
          for (int i = 0; i < NI; ++i) copy16(raw + v * S::kRaw + (e * NI + i) * 512, from + i * kRows * token);
        }
      copies_end();
    };
    enter();
    Job now = here();
    copy(now, 0);
    copy(now, 1);
    bool ok = true;
#pragma unroll 1
    for (int done = 0; now.live && ok; ++done) {
      next();
      const Job then = here();
      const int key0 = now.t * kTile + pw * 32 + row;
      const bool tail = (now.t + 1) * kTile > now.n_old;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        copies_landed<1>();
        if (done > 0 && !(ok = wait_long(empty(s, v), (done - 1) & 1))) break;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (!(now.what[e] >> 16)) w = shared16(raw + v * S::kRaw + (e * NI + i) * 512);
            if (v == 1 && tail) {
              // What the slots behind the last key hold reaches nobody; NaN of a new token is added, at the end, to the rows that see it.
              const int key = key0 + e * 16 + i * kRows;
              if (key >= now.keys) w = make_uint4(0u, 0u, 0u, 0u);
              if (key >= now.n_old && (nan_bytes(w.x) | nan_bytes(w.y) | nan_bytes(w.z) | nan_bytes(w.w))) {
                odd_v[s] = 1;
                w.x &= ~((nan_bytes(w.x) >> 7) * 0xffu); w.y &= ~((nan_bytes(w.y) >> 7) * 0xffu);
                w.z &= ~((nan_bytes(w.z) >> 7) * 0xffu); w.w &= ~((nan_bytes(w.w) >> 7) * 0xffu);
              }
            }
            const uint32_t to = base + operand(s, v);
            const int r = pw * 32 + e * 16 + row + i * kRows;
            put16(to + tile_at<kTile>(r, 2 * c), half_lo(w.x), half_hi(w.x), half_lo(w.y), half_hi(w.y));
            put16(to + tile_at<kTile>(r, 2 * c + 1), half_lo(w.z), half_hi(w.z), half_lo(w.w), half_hi(w.w));
          }
        if (v == 0 && lane < 2) {
          // (this job's softmax is behind the one that had these numbers' place: its scores were made after that one's outputs)
          const unsigned what = lane ? now.what[1] : now.what[0];
          const int ke = what & 0xff, ve = what >> 8 & 0xff;
          info[(s * 2 + (done & 1)) * kBlocks + 2 * pw + lane] = what >> 16 ? make_float4(1.f, -INFINITY, 0.f, 0.f) : make_float4(exp2i(ke - 127), (float)(ve - 127), exp2i(127 - ve), 0.f);
        }
        copy(then, v);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(full(s, v));
      }
      now = then;
    }
    copies_landed<0>();
  } else if (work) {
    const int s = warp / 4, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at = tmem + s * 128 + lanes, o_at = tmem + 256 + s * 128 + lanes;
    const uint64_t cap2 = pack2(a.cap2, a.cap2), inv2 = pack2(fabsf(a.inv_cap), fabsf(a.inv_cap));
    const int row = quarter * 32 + lane;
    int done = 0, seg = 0;
    bool ok = true;
    do {
      const int g = quotient(sg.nth, a.by_blocks), rb = sg.nth - g * a.blocks, n_old = a.c.lengths[sg.b];
      const int r = rb * RB + row, tok = quotient(min(r, a.rows - 1), a.by_group), h = min(r, a.rows - 1) - tok * a.group;
      const bool is = r < a.rows, idle = r - lane >= a.rows;       // idle: no row of this warp, which only keeps step
      if (s == 0) {
        // the segment's rows, once the products of the segment before have read theirs
        if (seg > 0 && !(ok = wait(q_empty, (seg - 1) & 1))) break;
        const char* const q = a.q + sg.b * a.q_batch + tok * a.q_token + (g * a.group + h) * a.q_head;
        float top = 0.f;
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          const uint4 w = is ? *(const uint4*)(q + i * 16) : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) top = max3(top, fabsf(__uint_as_float(x[e] << 16)), fabsf(__uint_as_float(x[e] & 0xffff0000u)));
        }
        const int raise = min(max(13 - ((int)(__float_as_uint(top) >> 23) - 127), -113), 126);
        const float up = exp2i(raise);
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
          const uint4 w = is ? *(const uint4*)(q + i * 16) : make_uint4(0u, 0u, 0u, 0u);
          const uint32_t x[4] = {w.x, w.y, w.z, w.w};
          uint32_t y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = f16x2(__uint_as_float(x[e] << 16) * up, __uint_as_float(x[e] & 0xffff0000u) * up);
          put16(base + tile_at<RB>(row, i), y[0], y[1], y[2], y[3]);
        }
        qs[row] = exp2i(-raise) * (CAP ? 1.f : fabsf(a.scale2));   // (a negative scale negates the product)
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(q_full);
      }
      if (!(ok = wait(q_full, seg & 1))) break;
      ++seg;
      const float f = qs[row];
      const int jobs = jobs_of(sg, s), last = n_old + tok;
      float m = kNothing, l = 0.f;
      bool far = false;
#pragma unroll 1
      for (int k = 0; k < jobs; ++k, ++done) {
        const int j0 = (sg.t0 + s + 2 * k) * kTile;
        if (!(ok = wait(s_full(s), done & 1))) break;
        tc_fence_after();
        if (!idle) {
          const float4* const in = info + (s * 2 + (done & 1)) * kBlocks;
          const bool tail = j0 + kTile > n_old + 1;
          // y of 16 scores, in bits and with V's exponent, less c's; hidden ones minus infinity
          auto weigh = [&](const float* v, int col, float fk, float c, float (&y)[16]) {
            if (CAP) {
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                y[e] = v[e] * fk;
                y[e + 1] = v[e + 1] * fk;
                capped2(y[e], y[e + 1], cap2, inv2);
                y[e] += c;
                y[e + 1] += c;
              }
            } else {
              const uint64_t f2 = pack2(fk, fk), c2 = pack2(c, c);
#pragma unroll
              for (int e = 0; e < 16; e += 2) unpack2(fma2(pack2(v[e], v[e + 1]), f2, c2), y[e], y[e + 1]);
            }
            if (tail) {
              const int sees = last - j0 - col;                    // the columns up to this one
#pragma unroll
              for (int e = 0; e < 16; ++e) y[e] = e <= sees ? y[e] : -INFINITY;
            }
          };
          float v[2][32], top = -INFINITY;
          tmem_ld32(s_at, v[0]);
#pragma unroll
          for (int c = 0; c < kTile; c += 32) {
            float* const x = v[c / 32 & 1];
            tmem_landed(x);
            if (c + 32 < kTile) tmem_ld32(s_at + c + 32, v[(c / 32 + 1) & 1]);
#pragma unroll
            for (int b = 0; b < 32; b += 16) {
              const float4 n = in[(c + b) / 16];
              if (tail) {
                float y[16];
                weigh(x + b, c + b, f * n.x, n.y, y);
                top = fmaxf(top, greatest16(y));
              } else {
                float t = greatest16(x + b) * (f * n.x), u = t;    // (rises with the score)
                if (CAP) capped2(t, u, cap2, inv2);
                top = fmaxf(top, t + n.y);
              }
            }
          }
          // the first of the scores again, while the reference is looked at
          tmem_ld32(s_at, v[0]);
          const bool grown = top > m + (kRaise + kSlack);
          if (__any_sync(0xffffffffu, grown)) {
            const float to = grown ? fmaxf(ceilf(top) - kRaise, m) : m, by = fast_exp2(m - to);
            m = to;
            l *= by;
            far = __any_sync(0xffffffffu, is && m != kNothing && fabsf(m) > 0x1p20f);
            tmem_landed(v[0]);
            if (k > 0) {
              if (!(ok = wait(o_done(s), (done - 1) & 1))) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                float x[16];
                uint32_t y[16];
                tmem_ld_issue<16>(o_at + c, x);
                tmem_ld_wait(x);
#pragma unroll
                for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(x[e] * by);
                tmem_st16(o_at + c, y);
              }
              tmem_st_wait();
            }
          }
#pragma unroll
          for (int c = 0; c < kTile; c += 32) {
            float* const x = v[c / 32 & 1];
            uint32_t p[16];
            tmem_landed(x);
            if (c + 32 < kTile) tmem_ld32(s_at + c + 32, v[(c / 32 + 1) & 1]);
#pragma unroll
            for (int b = 0; b < 32; b += 16) {
              const float4 n = in[(c + b) / 16];
              float y[16];
              weigh(x + b, c + b, f * n.x, n.y - m, y);
              if (far)
#pragma unroll
                for (int e = 0; e < 16; ++e)
                  if (y[e] > kRaise + kSlack) y[e] = kRaise + kSlack;
              uint64_t sum = pack2(0.f, 0.f);
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                const uint64_t w = exp2_sfu2(pack2(y[e], y[e + 1]));
                float p0, p1;
                unpack2(w, p0, p1);
                sum = add2(sum, w);
                p[(b + e) / 2] = f16x2(p0, p1);
              }
              float s0, s1;
              unpack2(sum, s0, s1);
              l = fmaf(s0 + s1, n.z, l);
            }
            tmem_st16(s_at + c / 2, p);                            // (over scores that have been read)
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(s));
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(q_empty);                         // (this stream's scores are all there)
      const int item = sg.b * a.c.n_kv * a.blocks + sg.nth, slot = 2 * (item + blockIdx.x) + s;
      if (tid == 0 && sg.t0 == 0) {
        const int end = sg.at + a.over + sg.tiles - 1;
        a.item_parts[item] = make_int2(slot, 2 * (cta_of(run.all, end) - (int)blockIdx.x + 1));
      }
      const size_t at = (size_t)slot * RB + row;
      if (is) a.part_stat[at] = make_float2(m == kNothing ? -INFINITY : m, l);
      if (jobs > 0) {
        if (!(ok = wait(o_done(s), (done - 1) & 1))) break;
        tc_fence_after();
        if (!idle) {
          const bool odd = odd_v[s] && sg.t1 * kTile > n_old;
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float v[32];
            tmem_ld(o_at + c, v);
            if (odd && is) {
#pragma unroll 1
              for (int i = n_old; i <= last && i < sg.keys; ++i) {
                const int p = ((const int*)((const char*)a.c.table + sg.b * a.c.s_table))[i >> a.c.page_shift];
                if ((unsigned)p >= (unsigned)a.c.pages) continue;
                const uint32_t* const from = (const uint32_t*)(a.c.v + p * a.c.s_page + g * a.c.s_head + (long long)(i & ((1 << a.c.page_shift) - 1)) * token + c);
#pragma unroll
                for (int e = 0; e < 32; ++e)
                  if ((from[e / 4] >> (8 * (e % 4)) & 0x7f) == 0x7f) v[e] = __int_as_float(0x7fffffff);
              }
            }
            if (is) {
              float4* const to = (float4*)(a.part_out + at * D + c);
#pragma unroll
              for (int e = 0; e < 8; ++e) to[e] = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(o_free(s));
      }
      next_segment(sg, a);
    } while (sg.t1);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    tc_fence_after();
    if (*abort_flag != 2) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  if (tid == 0 && *abort_flag) atomicCAS(a.c.status, 0, (int)STRUCTKV_ERR_TIMEOUT);
}

template <int D, bool CAP>
cudaError_t launch_one(const AttendPagesArgs& a, cudaStream_t st) {
  const cudaError_t e = allow_smem<attend_pages_tc<D, CAP>>(PagesTc<D>::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_pages_tc<D, CAP>, dim3(a.ctas), dim3(kThreads), PagesTc<D>::kSmem, st, a);
}

}  // namespace

cudaError_t launch_attend_pages_tc(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan&, cudaStream_t st) {
  if (ctx.cfg.head_dim == 128) return a.cap2 != 0.f ? launch_one<128, true>(a, st) : launch_one<128, false>(a, st);
  return a.cap2 != 0.f ? launch_one<64, true>(a, st) : launch_one<64, false>(a, st);
}

}  // namespace skv
