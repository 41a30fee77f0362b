// Attention of new tokens over a paged cache in 8 bits where a KV head has more than 16 rows (with caps 32).
//
// S = Q K^T and O += P V on the tensor cores (tcgen05): tiles of 128 rows x 64 keys, lane = row.  Two streams, the even and the odd
// tiles of a segment, alternate; each has two places for scores, so that the next tile's are there when a tile's exponentials are done.
// K and V come as codes: a stream's four producing warps copy them lane by lane (cp.async, two tiles ahead: pages and strides as they
// come), widen them to fp16, which is exact, and lay them out as the products' operands; a code is widened once for all rows.  Scales stay
// out of the operands: in bits, a score is s f 2^e_k and its weight in O 2^(s f 2^e_k + e_v - m), one multiply-add with two numbers for each 16
// keys.  References, weights and queries as in attend_pages.cu; a segment's first tile finds its reference first, later tiles are weighed against
// the reference as it is, and again where that is outgrown.
//
// Up to 64 rows stand twice in a tile, and each copy weighs half of its keys (its weights of the others are zero): all eight softmax warps
// have work and a tile's exponentials take half as long, where half of the tensor cores' rows would be idle anyway.  At a segment's end streams and
// copies become one partial, through the rows' place in shared memory, which writes whole lines.
//
// Warps: 0-3 and 4-7 bring a segment's rows and are the streams' softmax; 8-11 and 12-15 produce; 16 and 17 issue the streams' products.
//
// 16 tokens over 4 x 8192 keys (64 rows, 67 MB of codes): 34.7 us, 1.9 TB/s and 250 TFLOP/s.  A steady tile takes 1150 clocks of an SM, for
// which the chain is the bound, not a unit: scores (1000) -> weights (1700) -> outputs (700) -> the next scores in that place, of four in
// flight, and the producers' steps (2200 for a tile, two streams); tensor pipe 25 %, issue slots 45 %.  The rest is the first tile (5 us: lengths,
// table, codes, cold instructions), the segment's end (2 us) and the second launch (3 us).  Without the copies 44 us; one partial for each stream and
// copy 45; tiles of 128 keys have no room for two places; one fence for K and V 36; e4m3 operands would need e4m3 weights.
// 576 threads have 96 registers: blocks of 128 rows at d 128 spill 80 bytes of them, with caps 116.
#include <algorithm>

#include "attend_pages.cuh"
#include "attend_tc.cuh"

namespace skv {
namespace {

constexpr int kThreads = 576, kRows = kTile, kKeys = 64, kBlocks = kKeys / kBlockSlots;   // of a tile: rows, keys, blocks of slots

// An N-major operand of 64-element blocks of 128-byte rows (128-byte swizzle): blocks kKeys rows apart, 8-row groups 1024 bytes.
__device__ __forceinline__ uint64_t keys_desc_n(uint32_t addr) { return smem_desc(addr) & ~(0x3fffull << 16) | (uint64_t)((kKeys * 128) >> 4) << 16; }

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

// Two words of a row.
__device__ __forceinline__ void tmem_st2(uint32_t at, float a, float b) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x2.b32 [%0], {%1, %2};\ntcgen05.wait::st.sync.aligned;" ::"r"(at), "f"(a), "f"(b) : "memory");
}
__device__ __forceinline__ void tmem_ld2(uint32_t at, float& a, float& b) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0, %1}, [%2];\ntcgen05.wait::ld.sync.aligned;" : "=f"(a), "=f"(b) : "r"(at) : "memory");
}

template <int D>
struct PagesTc {
  static constexpr int kUnit = kKeys * D * 2, kRaw = kKeys * D;   // K or V of a tile, as operands and as codes
  // the rows, then for each stream two tiles as operands, two as codes; a tile's numbers for every 16 keys, four tiles a stream
  static constexpr int kOps = kRows * D * 2, kRaws = kOps + 8 * kUnit, kInfo = kRaws + 8 * kRaw, kQs = kInfo + 8 * kBlocks * 16, kBars = kQs + kRows * 8;
  static constexpr int kSmem = kBars + 304 + 1024;
  static_assert(kSmem <= 227 * 1024, "shared memory");
};

template <int D, int COPIES, bool CAP>
__global__ void __launch_bounds__(kThreads, 1) attend_pages_tc(const __grid_constant__ AttendPagesArgs a) {
  using S = PagesTc<D>;
  constexpr int RB = kRows, NR = RB / COPIES, W = kKeys / COPIES;   // rows of a block, columns of a tile that a copy of them sees
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  // stream s, K or V, job mod 2
  auto operand = [&](int s, int v, int p) { return (uint32_t)(S::kOps + (4 * s + 2 * v + p) * S::kUnit); };
  float4* const info = (float4*)(sm + S::kInfo);                 // [stream][job mod 4][block]: K's scale, exponent of V's, its inverse
  float* const qs = (float*)(sm + S::kQs);                       // a row's factor: scale in bits (capped scores: 1) times 2^-the raise of its queries
  float2* const stats = (float2*)qs;                             // at a segment's end: a row's reference and sum
  const uint32_t bars = base + S::kBars;
  auto full = [&](int s, int v, int p) { return bars + 8 * (4 * s + 2 * v + p); };
  auto empty = [&](int s, int v, int p) { return bars + 64 + 8 * (4 * s + 2 * v + p); };
  auto s_full = [&](int s, int p) { return bars + 128 + 8 * (2 * s + p); };
  auto p_ready = [&](int s, int p) { return bars + 160 + 8 * (2 * s + p); };
  auto o_done = [&](int s, int p) { return bars + 192 + 8 * (2 * s + p); };
  auto drained = [&](int s) { return bars + 224 + 8 * s; };
  const uint32_t q_full = bars + 240, q_empty = bars + 248, met = bars + 256, sent = bars + 264;
  volatile int* const words = (volatile int*)(sm + S::kBars + 272);
  volatile int *const abort_flag = words, *const odd_v = words + 2;   // odd_v: some new token's V was NaN
  volatile uint32_t* const tmem_at = (volatile uint32_t*)words + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, token = a.c.s_token;
  pdl_trigger();
  if (tid == 0) {
    for (int s = 0; s < 2; ++s) {
      for (int p = 0; p < 2; ++p) {
        for (int v = 0; v < 2; ++v) { mbar_init(full(s, v, p), 128); mbar_init(empty(s, v, p), 1); }
        mbar_init(s_full(s, p), 1); mbar_init(p_ready(s, p), 4); mbar_init(o_done(s, p), 1);
      }
      mbar_init(drained(s), 1);
    }
    mbar_init(q_full, 256);
    mbar_init(q_empty, 10);                                        // softmax's warps, products' warps
    mbar_init(met, 8); mbar_init(sent, 8);
    *abort_flag = 0;
    *odd_v = 0;
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
    // Products of stream s: a job's outputs, then the scores of the job after next, which take its place.
    const int s = warp - 16;
    const uint32_t lead = lane == 0;
    constexpr uint32_t kF16 = 1u << 4;                             // fp16 operands, fp32 results
    const uint32_t idesc_s = kF16 | (uint32_t)(kKeys >> 3) << 17 | (uint32_t)(kRows >> 4) << 24 | (a.scale2 < 0.f ? 1u << 13 : 0u);
    constexpr uint32_t idesc_o = kF16 | (uint32_t)(D >> 3) << 17 | (uint32_t)(kRows >> 4) << 24 | kTransposeB;
    const uint64_t q_desc = smem_desc(base), k_desc = smem_desc(base + operand(s, 0, 0)), v_desc = keys_desc_n(base + operand(s, 1, 0));
    const uint32_t q_lo = (uint32_t)q_desc, k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc, hi_k = (uint32_t)(q_desc >> 32), hi_v = (uint32_t)(v_desc >> 32);
    const uint32_t s_at = tmem + s * 128, o_at = tmem + 256 + s * 128;
    int seg = 0, done = 0;                                         // segments, jobs
    bool ok = true;
    do {
      const int jobs = jobs_of(sg, s);
      // (a stream without a tile in the segment says as well that it came by: else its wait might be for a phase that is gone)
      if ((ok = wait(q_full, seg & 1)) && lead) mbar_arrive(q_empty);
      // (from two jobs before the first on, so that this code is there once: what a launch fetches of it is most of its way to the first tile)
#pragma unroll 1
      for (int k = -2; k < jobs && ok; ++k) {
        const int job = done + k, p = job & 1;
        if (k >= 0) {
          if (!(ok = wait(full(s, 1, p), job >> 1 & 1))) break;
          if (!(ok = wait(p_ready(s, p), job >> 1 & 1))) break;
          tc_fence_after();
          const uint32_t vd = v_lo + (p * S::kUnit >> 4);
#pragma unroll
          for (int kk = 0; kk < kKeys / 16; ++kk) mma_ts(o_at, s_at + p * 64 + kk * 8, vd + ((kk * 16 * 128) >> 4), hi_v, idesc_o, k > 0 || kk > 0, lead);
          commit_by(lead, o_done(s, p));
          commit_by(lead, empty(s, 1, p));
        }
        if (k + 2 < jobs) {
          // the scores of the job after next
          if (!(ok = wait(full(s, 0, p), (job + 2) >> 1 & 1))) break;
          tc_fence_after();
          const uint32_t kd = k_lo + (p * S::kUnit >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_ss(s_at + p * 64, q_lo + (((kk / 4) * RB * 128 + (kk % 4) * 32) >> 4), kd + (((kk / 4) * kKeys * 128 + (kk % 4) * 32) >> 4), hi_k, idesc_s, kk > 0, lead);
          commit_by(lead, s_full(s, p));
          commit_by(lead, empty(s, 0, p));
        }
      }
      done += max(jobs, 0);
      ++seg;
      next_segment(sg, a);
    } while (ok && sg.t1);
    commit_by(lead, drained(s));
    if (!mbar_drain(drained(s), 0, abort_flag)) *abort_flag = 2;
  } else if (work && warp >= 8) {
    // Producers of stream s: a warp has 16 keys of every tile.  Lane i knows page and scales of the i-th of 32 jobs, and in good time of
    // the 32 behind them: page -1: nothing there (behind the last key, or a page that is none); bytes of K's and V's scale.
    constexpr int NI = D / 32;                                     // 16-byte pieces that a lane has of 16 keys
    const int s = (warp - 8) / 4, pw = warp & 3;
    const int c = D == 128 ? (lane & 3) | (lane & 8) >> 1 : lane & 3, row = D == 128 ? (lane >> 2 & 1) | lane >> 4 << 1 : lane >> 2;   // of piece 0
    constexpr int kStep = 16 / NI;                                 // rows from piece to piece
    const uint32_t raw = base + S::kRaws + s * 4 * S::kRaw + pw * (NI * 512) + lane * 16;
    int j = -1, jobs = 0, page = -1, page_after = -1, g = 0, n_old = 0;
    uint8_t ks = 0, vs = 0, ks_after = 0, vs_after = 0;
    const int* table = nullptr;
    const char *k0 = nullptr, *v0 = nullptr;
    auto look = [&](int job, uint8_t& ks, uint8_t& vs) {
      const int t = sg.t0 + s + 2 * job, step = t * kBlocks + pw;
      int p = -1;
      if (t < sg.t1 && step * 16 < sg.keys) {
        p = table[step >> sh4];
        if ((unsigned)p >= (unsigned)a.c.pages) {
          p = -1;
          tell_invalid(a.c);
        }
        const unsigned at = (((unsigned)max(p, 0) * a.c.n_kv + g) << sh4) + (step & (per_page - 1));
        ks = a.c.k_scales[at];
        vs = a.c.v_scales[at];
      }
      return p;
    };
    // A job: its tile (-1: there is none), its sequence's keys and old ones among them, page and scales of this warp's part (the scales one
    // call later: copies need not wait for them).
    struct Job { int t, keys, n_old, page, scales; };
    auto next = [&](Job& last) {
      last.scales = __shfl_sync(0xffffffffu, ks | vs << 8, j & 31);
      if (sg.t1 && ++j == jobs) {
        if (j > 0) next_segment(sg, a);
        while (sg.t1 && jobs_of(sg, s) == 0) next_segment(sg, a);
        if (sg.t1) {
          j = 0;
          jobs = jobs_of(sg, s);
          g = quotient(sg.nth, a.by_blocks);
          n_old = sg.n;
          table = (const int*)((const char*)a.c.table + sg.b * a.c.s_table);
          k0 = a.c.k + g * a.c.s_head + (long long)row * token + c * 16;
          v0 = a.c.v + g * a.c.s_head + (long long)row * token + c * 16;
          page = look(lane, ks, vs);
        }
      } else if ((j & 31) == 0) {
        page = page_after;
        ks = ks_after;
        vs = vs_after;
      } else if ((j & 31) == 4 && jobs > (j | 31)) {
        page_after = look((j | 31) + 1 + lane, ks_after, vs_after);
      }
      const int p = __shfl_sync(0xffffffffu, page, j & 31);
      return sg.t1 ? Job{sg.t0 + s + 2 * j, sg.keys, n_old, p, 0} : Job{-1, 0, 0, -1, 0};
    };
    auto widen = [&](uint32_t to, const uint4 (&w)[NI]) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int r = pw * 16 + row + i * kStep;
        put16(to + tile_at<kKeys>(r, 2 * c), half_lo(w[i].x), half_hi(w[i].x), half_lo(w[i].y), half_hi(w[i].y));
        put16(to + tile_at<kKeys>(r, 2 * c + 1), half_lo(w[i].z), half_hi(w[i].z), half_lo(w[i].w), half_hi(w[i].w));
      }
    };
    // (from two jobs before the first on, so that this code is there once)
    Job now{-1, 0, 0, -1, 0}, then = now;
#pragma unroll 1
    for (int done = -2;; ++done) {
      const int p = done & 1;
      const Job later = next(then);
      const uint32_t codes = raw + 2 * p * S::kRaw;
      uint4 kw[NI], vw[NI];
      if (done >= 0) {
        if (now.t < 0) break;
        copies_landed<1>();
        const bool is = now.page >= 0;
#pragma unroll
        for (int i = 0; i < NI; ++i) vw[i] = is ? shared16(codes + S::kRaw + i * 512) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < NI; ++i) kw[i] = is ? shared16(codes + i * 512) : make_uint4(0u, 0u, 0u, 0u);
        if (done > 1 && !wait_long(empty(s, 0, p), (done >> 1) - 1 & 1)) break;
        widen(base + operand(s, 0, p), kw);
        if (lane == 0) {
          // (the job four before, which had this place, is done: the scores of the one two before were made behind its outputs)
          const int ke = now.scales & 0xff, ve = now.scales >> 8;
          info[(s * 4 + (done & 3)) * kBlocks + pw] = is ? make_float4(exp2i(ke - 127), (float)(ve - 127), exp2i(127 - ve), 0.f) : make_float4(1.f, -INFINITY, 0.f, 0.f);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(full(s, 0, p));
      }
      if (later.page >= 0) {
        // (k0 and v0 are the newest job's; the codes that were here are in registers: K's, read last, have been used)
        const long long off = (long long)((unsigned long long)(unsigned)later.page * (unsigned)a.c.s_page) + ((later.t * kBlocks + pw) & (per_page - 1)) * (token << kBlockShift);
        const char *const k = k0 + off, *const v = v0 + off;
#pragma unroll
        for (int i = 0; i < NI; ++i) copy16(codes + i * 512, k + i * kStep * token);
#pragma unroll
        for (int i = 0; i < NI; ++i) copy16(codes + S::kRaw + i * 512, v + i * kStep * token);
      }
      copies_end();
      if (done >= 0) {
        if ((now.t + 1) * kKeys > now.n_old) {
          // What the slots behind the last key hold reaches nobody; NaN of a new token is added, at the end, to the rows that see it.
#pragma unroll
          for (int i = 0; i < NI; ++i) {
            const int key = now.t * kKeys + pw * 16 + row + i * kStep;
            uint4& w = vw[i];
            if (key >= now.keys) w = make_uint4(0u, 0u, 0u, 0u);
            if (key >= now.n_old && (nan_bytes(w.x) | nan_bytes(w.y) | nan_bytes(w.z) | nan_bytes(w.w))) {
              *odd_v = 1;
              w.x &= ~((nan_bytes(w.x) >> 7) * 0xffu); w.y &= ~((nan_bytes(w.y) >> 7) * 0xffu);
              w.z &= ~((nan_bytes(w.z) >> 7) * 0xffu); w.w &= ~((nan_bytes(w.w) >> 7) * 0xffu);
            }
          }
        }
        if (done > 1 && !wait_long(empty(s, 1, p), (done >> 1) - 1 & 1)) break;
        widen(base + operand(s, 1, p), vw);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(full(s, 1, p));
      }
      now = then;
      then = later;
    }
    copies_landed<0>();
  } else if (work) {
    const int s = warp / 4, quarter = warp & 3;
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at0 = tmem + s * 128 + lanes, o_at = tmem + 256 + s * 128 + lanes;
    const uint64_t cap2 = pack2(a.cap2, a.cap2), inv2 = pack2(fabsf(a.inv_cap), fabsf(a.inv_cap));
    const int row = quarter * 32 + lane, copy = row / NR, c_from = copy * W;
    int done = 0, seg = 0;
    bool ok = true;
    do {
      const int g = quotient(sg.nth, a.by_blocks), rb = sg.nth - g * a.blocks, n_old = sg.n;
      const int r = rb * NR + row % NR, tok = quotient(min(r, a.rows - 1), a.by_group), h = min(r, a.rows - 1) - tok * a.group;
      const bool is = r < a.rows, idle = r - lane >= a.rows;       // idle: no row of this warp, which only keeps step
      // The segment's rows, once the products of the segment before have read theirs: D / 8 lanes a row.
      if (seg > 0 && !(ok = wait(q_empty, (seg - 1) & 1))) break;
      {
        constexpr int LANES = D / 8, ROWS = 32 / LANES;
        const int c = lane % LANES, end = min(NR, a.rows - rb * NR);
        const char* const q = a.q + sg.b * a.q_batch + (g * a.group) * a.q_head + c * 16;
        constexpr int BATCH = 4, STEP = 8 * ROWS;                  // rows that are on their way together, rows of all warps
#pragma unroll 1
        for (int i0 = warp * ROWS + lane / LANES; i0 - lane / LANES < end; i0 += BATCH * STEP) {
          uint4 w[BATCH];
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            const int x = rb * NR + min(i0 + b * STEP, end - 1), t = quotient(x, a.by_group);
            w[b] = *(const uint4*)(q + t * a.q_token + (x - t * a.group) * a.q_head);
          }
#pragma unroll
          for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * STEP;
            const uint32_t x[4] = {w[b].x, w[b].y, w[b].z, w[b].w};
            uint32_t top = 0u;                                     // of two elements' magnitudes, as bf16
#pragma unroll
            for (int e = 0; e < 4; ++e) asm("max.bf16x2 %0, %0, %1;" : "+r"(top) : "r"(x[e] & 0x7fff7fffu));
#pragma unroll
            for (int o = 1; o < LANES; o *= 2) asm("max.bf16x2 %0, %0, %1;" : "+r"(top) : "r"(__shfl_xor_sync(0xffffffffu, top, o)));
            const int exponent = (int)(max(top << 16, top & 0xffff0000u) >> 23);
            const int raise = min(max(13 - (exponent - 127), -113), 126);
            const float up = exp2i(raise);
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = f16x2(__uint_as_float(x[e] << 16) * up, __uint_as_float(x[e] & 0xffff0000u) * up);
            if (i < NR) {
#pragma unroll
              for (int k = 0; k < COPIES; ++k) put16(base + tile_at<RB>(k * NR + i, c), y[0], y[1], y[2], y[3]);
              if (c == 0) qs[i] = exp2i(-raise) * (CAP ? 1.f : fabsf(a.scale2));   // (a negative scale negates the product)
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(q_full);
      }
      if (!(ok = wait(q_full, seg & 1))) break;
      ++seg;
      const float f = qs[row % NR];                                     // (rows behind the last have anything, which stays with them)
      const int jobs = jobs_of(sg, s), last = n_old + tok;
      float m = kNothing, l = 0.f;
      bool far = false;
#pragma unroll 1
      for (int k = 0; k < jobs; ++k, ++done) {
        const int j0 = (sg.t0 + s + 2 * k) * kKeys;
        const uint32_t s_at = s_at0 + (done & 1) * 64;
        if (!(ok = wait(s_full(s, done & 1), done >> 1 & 1))) break;
        tc_fence_after();
        if (!idle) {
          const float4* const in = info + (s * 4 + (done & 3)) * kBlocks;
          const bool tail = j0 + kKeys > n_old + 1;
          const int sees = last - j0;                              // the last column that is seen
          // y of 16 scores from column col on, in bits and with V's exponent, less the reference or without; hidden ones minus infinity
          auto weigh = [&](const float* v, int col, const float4& n, bool bare, float (&y)[16]) {
            const float fk = f * n.x;
            if (CAP) {
#pragma unroll
              for (int e = 0; e < 16; e += 2) {
                y[e] = v[e] * fk;
                y[e + 1] = v[e + 1] * fk;
                capped2(y[e], y[e + 1], cap2, inv2);
              }
            }
            if (bare || far) {                                     // (as in attend_pages.cu)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                y[e] = __fadd_rn(CAP ? y[e] : __fmul_rn(v[e], fk), n.y);
                if (!bare) y[e] = __fadd_rn(y[e], -m);
              }
            } else {
              const uint64_t f2 = pack2(fk, fk), c2 = pack2(n.y - m, n.y - m);
#pragma unroll
              for (int e = 0; e < 16; e += 2) unpack2(CAP ? add2(pack2(y[e], y[e + 1]), c2) : fma2(pack2(v[e], v[e + 1]), f2, c2), y[e], y[e + 1]);
            }
            if (tail)
#pragma unroll
              for (int e = 0; e < 16; ++e) y[e] = col + e <= sees ? y[e] : -INFINITY;
          };
          uint32_t p[W / 2];
          float sum = 0.f;
          bool grown = true, settle = k == 0;                      // (a segment's first tile finds its reference before it is weighed)
#pragma unroll 1
          for (;;) {
            if (settle) {
              // the reference follows: the largest score, without the one as it was
              float top = -INFINITY;
#pragma unroll 1
              for (int c = c_from; c < c_from + W; c += 16) {
                float x[16], y[16];
                tmem_ld_issue<16>(s_at + c, x);
                tmem_ld_wait(x);
                const float4 n = in[c / 16];
                weigh(x, c, n, true, y);
                top = fmaxf(top, greatest16(y));
              }
              const float to = grown ? fmaxf(ceilf(top) - kRaise, m) : m, by = fast_exp2(m - to);
              m = to;
              l *= by;
              far = __any_sync(0xffffffffu, is && m != kNothing && fabsf(m) > 0x1p20f);
              if (k > 0) {
                if (!(ok = wait(o_done(s, (done - 1) & 1), (done - 1) >> 1 & 1))) break;
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
            float top = -INFINITY;
            sum = 0.f;
            constexpr int PART = W < 32 ? W : 32;
#pragma unroll
            for (int c = 0; c < W; c += PART) {
              float x[PART];
              if constexpr (PART == 32) {
                tmem_ld(s_at + c_from + c, x);
              } else {
                tmem_ld_issue<16>(s_at + c_from + c, x);
                tmem_ld_wait(x);
              }
#pragma unroll
              for (int b = 0; b < PART; b += 16) {
                const float4 n = in[(c_from + c + b) / 16];
                float y[16];
                weigh(x + b, c_from + c + b, n, false, y);
                top = fmaxf(top, greatest16(y));
                uint64_t part = pack2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                  const uint64_t w = exp2_sfu2(pack2(y[e], y[e + 1]));
                  float p0, p1;
                  unpack2(w, p0, p1);
                  part = add2(part, w);
                  p[(c + b + e) / 2] = f16x2(p0, p1);
                }
                float s0, s1;
                unpack2(part, s0, s1);
                sum = fmaf(s0 + s1, n.z, sum);
              }
            }
            grown = top > kRaise + kSlack;
            if (settle || !__any_sync(0xffffffffu, grown)) break;
            settle = true;
          }
          if (!ok) break;
          l += sum;
          // (over the scores; a copy's weights of other columns are zero)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t w[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) w[e] = COPIES == 1 || (16 * h + e) / (W / 2) == copy ? p[(16 * h + e) % (W / 2)] : 0u;
            tmem_st16(s_at + 16 * h, w);
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_ready(s, done & 1));
      }
      if (!ok) break;
      // The segment ends: its streams' results become one, and its copies'.  Rows' operands are read no more: their place takes what a copy
      // hands to the other.
      if (jobs > 0 && !(ok = wait(o_done(s, (done - 1) & 1), (done - 1) >> 1 & 1))) break;
      tc_fence_after();
      if (!idle) tmem_st2(s_at0, m, l);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(met);
      if (!(ok = wait(met, (seg - 1) & 1))) break;
      tc_fence_after();
      const int item = sg.b * a.c.n_kv * a.blocks + sg.nth, slot = item + blockIdx.x;
      if (tid == 0 && sg.t0 == 0) {
        const int end = sg.at + a.over + sg.tiles - 1;
        a.item_parts[item] = make_int2(slot, cta_of(run.all, end) - (int)blockIdx.x + 1);
      }
      constexpr int COLS = D / (2 * COPIES);                       // that a warp finishes
      const int c_mine = copy * (D / COPIES) + s * COLS;
      float w0 = 0.f, w1 = 0.f;
      // 16 columns of a row's two streams, from column c on
      auto joined = [&](int c, float (&x)[16]) {
        float y[16];
        tmem_ld_issue<16>(tmem + 256 + lanes + c, x);
        tmem_ld_issue<16>(tmem + 384 + lanes + c, y);
        tmem_ld_wait(x);
        tmem_ld_wait(y);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = (w0 < 0.f ? 0.f : x[e] * w0) + (w1 < 0.f ? 0.f : y[e] * w1);
      };
      // weights of two results of a row, -1: it has seen nothing, whatever its outputs are; and what they are together
      auto meet = [](float ma, float la, float mb, float lb, float& wa, float& wb) {
        const float top = fmaxf(ma, mb);
        wa = ma == kNothing && la == 0.f ? -1.f : fast_exp2(ma - top);
        wb = mb == kNothing && lb == 0.f ? -1.f : fast_exp2(mb - top);
        return make_float2(top, (wa < 0.f ? 0.f : wa * la) + (wb < 0.f ? 0.f : wb * lb));
      };
      float2 all;
      if (!idle) {
        float m2, l2;
        tmem_ld2(tmem + (1 - s) * 128 + lanes, m2, l2);
        all = s ? meet(m2, l2, m, l, w0, w1) : meet(m, l, m2, l2, w0, w1);
      }
      const int rr = row % NR;
      // Where 4 columns from c on of lane i's row pass through the rows' place: of all rows and columns for what a copy hands to the other, of
      // the warp's 32 rows and PIECE columns otherwise; 16 bytes each, in an order that differs from row to row, so that lanes meet no bank twice.
      constexpr int PIECE = D / 4;
      auto passing = [&](int i, int c) {
        if (COPIES == 2) return base + (quarter * 32 + i) % NR * (D * 4) + ((c >> 2 ^ i & 7) << 4);
        return base + (warp * 32 + i) * (PIECE * 4) + (((c & PIECE - 1) >> 2 ^ (D == 128 ? i & 7 : i >> 1 & 3)) << 4);
      };
      static_assert(8 * 32 * PIECE * 4 <= S::kOps && kRows / 2 * D * 4 <= S::kOps && COLS % PIECE == 0, "within the rows' place");
      float w_mine = 1.f, w_other = -1.f;
      if constexpr (COPIES == 2) {
        if (!idle) {
          const int c_other = (1 - copy) * (D / 2) + s * COLS;
#pragma unroll 1
          for (int c = c_other; c < c_other + COLS; c += 16) {
            float x[16];
            joined(c, x);
#pragma unroll
            for (int e = 0; e < 16; e += 4)
              put16(passing(lane, c + e), __float_as_uint(x[e]), __float_as_uint(x[e + 1]), __float_as_uint(x[e + 2]), __float_as_uint(x[e + 3]));
          }
          if (s == 0) stats[row] = all;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(sent);
        if (!(ok = wait(sent, (seg - 1) & 1))) break;
        if (!idle) {
          const float2 other = stats[(1 - copy) * NR + rr];
          all = meet(all.x, all.y, other.x, other.y, w_mine, w_other);
        }
      }
      if (!idle) {
        w0 = w0 < 0.f || w_mine < 0.f ? -1.f : w0 * w_mine;
        w1 = w1 < 0.f || w_mine < 0.f ? -1.f : w1 * w_mine;
        const bool odd = *odd_v && sg.t1 * kKeys > n_old;
        const size_t at = (size_t)slot * NR + rr;
        if (is && s == 0 && copy == 0) a.part_stat[at] = make_float2(all.x == kNothing ? -INFINITY : all.x, all.y);
#pragma unroll 1
        for (int c = c_mine; c < c_mine + COLS; c += 16) {
          float v[16];
          joined(c, v);
          if constexpr (COPIES == 2) {
            if (!(w_other < 0.f))
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const uint4 x = shared16(passing(lane, c + e));
                v[e] = fmaf(__uint_as_float(x.x), w_other, v[e]);
                v[e + 1] = fmaf(__uint_as_float(x.y), w_other, v[e + 1]);
                v[e + 2] = fmaf(__uint_as_float(x.z), w_other, v[e + 2]);
                v[e + 3] = fmaf(__uint_as_float(x.w), w_other, v[e + 3]);
              }
          }
          if (odd && is) {
#pragma unroll 1
            for (int i = n_old; i <= last && i < sg.keys; ++i) {
              const int pg = ((const int*)((const char*)a.c.table + sg.b * a.c.s_table))[i >> a.c.page_shift];
              if ((unsigned)pg >= (unsigned)a.c.pages) continue;
              const uint32_t* const from = (const uint32_t*)(a.c.v + pg * a.c.s_page + g * a.c.s_head + (long long)(i & ((1 << a.c.page_shift) - 1)) * token + c);
#pragma unroll
              for (int e = 0; e < 16; ++e)
                if ((from[e / 4] >> (8 * (e % 4)) & 0x7f) == 0x7f) v[e] = __int_as_float(0x7fffffff);
            }
          }
#pragma unroll
          for (int e = 0; e < 16; e += 4)
            put16(passing(lane, c + e), __float_as_uint(v[e]), __float_as_uint(v[e + 1]), __float_as_uint(v[e + 2]), __float_as_uint(v[e + 3]));
          // (lane by lane a row would be a line of its own each time; side by side, LANES lanes write one)
          constexpr int LANES = PIECE / 4;
          const int from = c + 16 - PIECE;
          if (from % PIECE == 0) {
            __syncwarp();
#pragma unroll
            for (int i0 = 0; i0 < 32; i0 += 32 / LANES) {
              const int i = i0 + lane / LANES, col = from + lane % LANES * 4;
              const uint4 x = shared16(passing(i, col));
              if (r - lane + i < min(a.rows, (rb + 1) * NR)) *(uint4*)(a.part_out + ((size_t)slot * NR + rr - lane + i) * D + col) = x;
            }
            __syncwarp();
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(q_empty);
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

template <int D, int COPIES, bool CAP>
cudaError_t launch_one(const AttendPagesArgs& a, cudaStream_t st) {
  const cudaError_t e = allow_smem<attend_pages_tc<D, COPIES, CAP>>(PagesTc<D>::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_pages_tc<D, COPIES, CAP>, dim3(a.ctas), dim3(kThreads), PagesTc<D>::kSmem, st, a);
}
template <int D, bool CAP>
cudaError_t launch_rows(const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st) {
  return p.rb == 64 ? launch_one<D, 2, CAP>(a, st) : launch_one<D, 1, CAP>(a, st);
}

}  // namespace

cudaError_t launch_attend_pages_tc(const Ctx& ctx, const AttendPagesArgs& a, const PagesPlan& p, cudaStream_t st) {
  if (ctx.cfg.head_dim == 128) return a.cap2 != 0.f ? launch_rows<128, true>(a, p, st) : launch_rows<128, false>(a, p, st);
  return a.cap2 != 0.f ? launch_rows<64, true>(a, p, st) : launch_rows<64, false>(a, p, st);
}

}  // namespace skv
