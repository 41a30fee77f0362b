// Attention of new tokens over a bf16 cache where a KV head has more than 16 rows: drafted trees, pieces of a prompt.
//
// S = Q K^T and O += P V on the tensor cores (tcgen05): a tile of 128 rows x 128 keys, lane = row, so that a row's maximum and sum
// stay inside one thread; P goes back to tensor memory, over S, as the A operand of the second product; V, whose rows are
// keys, is its B operand as it lies (N-major).  Two streams of such tiles alternate, so that one's products run beside the other's
// exponentials: the two halves of up to 256 rows over the same keys, or, with up to 128 rows, the even and the odd key tiles (the
// streams then leave a partial each).  Work is cut as everywhere (attend.cuh).
//
// Warps: 0 fills the ring of K and V tiles by TMA; 1 and 2 issue the streams' products (issuing eight takes up to 900 clocks: by one
// warp for both a key tile of 256 rows took 5850); 3 looks through V tiles that hold new tokens (what is not
// finite there is taken out and added, at the end, to the rows that see it: 0 x infinity); 4-7 and 8-11 bring a segment's rows
// and are the streams' softmax.  The reference of a row follows its maximum only where that outgrows it by 2^kSlack
// (64 tokens over 8 x 8192 keys 91 us, 105 where it follows at once).
//
// Bound by reading K and V up to about 128 rows, where there are many keys (4 sequences of 4096 keys, 32 rows: 67 MB in 20 us), by the way
// from launch to first tile to partial where there are few (2048 keys: 10 us).  256 rows over 4 x 16384 keys take 76 us, 0.90 PFLOP/s, and are
// bound by the chain of one half's tile, 4250 clocks: scores loaded 290, maximum 145, reference 330, exponentials 1220, the
// other quarters' 430, outputs 640, scores of the next tile 1050; products and exponentials alone would be 2048 each.  The
// chain is not shortened by a quarter of the exponentials on the FMA pipe (their NaN need a maximum that keeps one: 88 us became
// 92).  Not built: P takes half of the 128 columns that its scores had; half of the next tile's scores could be made in the other half
// meanwhile.
#include <algorithm>

#include "attend.cuh"

namespace skv {
namespace {

constexpr int kTile = 128, kThreads = 384;

// An N-major operand of 64-element blocks of 128-byte rows (128-byte swizzle): blocks kTile rows apart, 8-row groups 1024 bytes.
__device__ __forceinline__ uint64_t smem_desc_n(uint32_t addr) {
  return smem_desc(addr) & ~(0x3fffull << 16) | (uint64_t)((kTile * 128) >> 4) << 16;
}
constexpr uint32_t kTransposeB = 1u << 16;
// Products that a whole warp comes by and one lane (lead) issues: without a branch for it the operands can stay uniform.  Descriptors
// by their lower words; hi: the upper word, the same for all of an operand's.
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 da, db;\nsetp.ne.b32 q, %6, 0;\nsetp.ne.b32 p, %5, 0;\nmov.b64 da, {%1, %3};\nmov.b64 db, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n}"
      ::"r"(d_tmem), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}
// a in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t hi, uint32_t idesc, uint32_t accumulate, uint32_t lead) {
  asm volatile(
      "{\n.reg .pred p, q;\n.reg .b64 db;\nsetp.ne.b32 q, %6, 0;\nsetp.ne.b32 p, %5, 0;\nmov.b64 db, {%2, %3};\n"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n}"
      ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(hi), "r"(idesc), "r"(accumulate), "r"(lead) : "memory");
}
__device__ __forceinline__ void commit_by(uint32_t lead, uint32_t bar) {
  asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %1, 0;\n@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}"
               ::"r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
               ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
                 "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// The load of 32 columns and its wait apart: several loads travel together.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                 "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                 "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]),
                 "=f"(v[23]), "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]),
                 "=f"(v[30]), "=f"(v[31])
               : "r"(taddr) : "memory");
}
// (registers that a load in flight writes are operands of a wait, so that no use of them comes before it)
__device__ __forceinline__ void tmem_landed(float* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                 "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]),
                 "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]),
                 "+f"(v[30]), "+f"(v[31])
               :: "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const float (&f)[32]) {
  uint32_t lo[16], hi[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) { lo[i] = __float_as_uint(f[i]); hi[i] = __float_as_uint(f[16 + i]); }
  tmem_st16(taddr, lo);
  tmem_st16(taddr + 16, hi);
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// MT: halves of 128 rows in a block.
template <int D, int MT, bool OPT>
struct TcAttend {
  static constexpr int RB = 128 * MT, kUnit = kTile * D * 2, kQ = RB * D * 2, kPos = OPT ? kTile * 4 : 0;
  static constexpr int kFixed = kQ + 1024 + 512;
  // Places for tiles of K and of V; with two streams over different tiles each has a ring of its own: a wait by parity holds only for
  // who follows a barrier from phase to phase.
  static constexpr int kUnits = std::min(8, (227 * 1024 - 512 - kFixed) / (kUnit + kPos)) / (MT == 2 ? 1 : 2) * (MT == 2 ? 1 : 2);
  static constexpr int kRingUnits = MT == 2 ? kUnits : kUnits / 2;
  static constexpr int kSmem = kUnits * (kUnit + kPos) + kFixed;
  static_assert(kUnits >= 4, "a ring");
};

template <int D, int MT, bool OPT>
__global__ void __launch_bounds__(kThreads, 1) attend_tc(const __grid_constant__ AttendArgs a, const __grid_constant__ CacheMaps maps) {
  using S = TcAttend<D, MT, OPT>;
  constexpr int RB = S::RB, NU = S::kUnits, CH = D / 8;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kRing = S::kQ, kPosAt = kRing + NU * S::kUnit, kBars = kPosAt + NU * S::kPos;
  const uint32_t bars = base + kBars, more = bars + 16 * NU;
  // where unit u (K and V of a tile after one another) of the ring of stream s lies, and its phase there
  constexpr int NR = S::kRingUnits;
  auto place_of = [](int s, int u) { return (MT == 2 ? 0 : s * NR) + u % NR; };
  auto phase_of = [](int u) { return (u / NR) & 1; };
  auto full = [&](int u) { return bars + 8 * u; };
  auto empty = [&](int u) { return bars + 8 * (NU + u); };
  auto s_full = [&](int s) { return more + 8 * s; };
  auto p_ready = [&](int s) { return more + 16 + 8 * s; };
  auto o_done = [&](int s) { return more + 32 + 8 * s; };
  auto o_free = [&](int s) { return more + 48 + 8 * s; };
  auto v_look = [&](int s) { return more + 64 + 8 * s; };
  auto v_ready = [&](int s) { return more + 80 + 8 * s; };
  auto drained = [&](int s) { return more + 96 + 8 * s; };
  auto turn = [&](int s) { return more + 112 + 8 * s; };
  auto p_half = [&](int s) { return more + 160 + 8 * s; };       // (behind the words)
  const uint32_t q_full = more + 128, q_empty = more + 136;
  volatile int* const words = (volatile int*)(sm + kBars + 16 * NU + 144);
  volatile int *const abort_flag = words, *const odd_v = words + 2;   // odd_v[s]: in a tile of stream s some new token's V was not finite
  volatile uint32_t* const tmem_at = (volatile uint32_t*)words + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int blocks = (a.rows + RB - 1) / RB;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < NU; ++i) { mbar_init(full(i), S::kPos ? 33 : 1); mbar_init(empty(i), MT); }
    for (int s = 0; s < 2; ++s) {
      mbar_init(s_full(s), 1); mbar_init(p_half(s), 4); mbar_init(p_ready(s), 4); mbar_init(o_done(s), 1); mbar_init(o_free(s), 4);
      mbar_init(v_look(s), 1); mbar_init(v_ready(s), 32); mbar_init(drained(s), 1); mbar_init(turn(s), 4);
    }
    mbar_init(q_full, 256);
    mbar_init(q_empty, 10);                                        // softmax's warps, products' warps
    *abort_flag = 0;
    odd_v[0] = odd_v[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&maps.k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&maps.v) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_at)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    tc_fence_before();
  }
  __syncthreads();
  pdl_wait();
  const WorkStart ws = find_work(a, 7, blocks, blockIdx.x == 0 ? a.unit_start : nullptr);
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  Segments sg = first_segment(a, ws, 7, blocks);
  const bool work = sg.t1 > 0;
  // (one answer for the warp: what follows is for all of its lanes)
  auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag)); };
  bool clean = true;                                             // every MMA of this CTA has retired

  // 128 x 88 + 256 x 200 registers of the 384 x 168 that the block was launched with
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (work && warp == 0) {
      const uint64_t hint = blocks == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
      int made[2] = {0, 0};                                        // units of the rings
      bool ok = true;
      do {
        const int b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv;
#pragma unroll 1
        for (int t = sg.t0; t < sg.t1 && ok; ++t)
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv) {
            const int s = MT == 2 ? 0 : (t - sg.t0) & 1, n = s ? made[1]++ : made[0]++, st = place_of(s, n);
            if (n >= NR && !(ok = mbar_wait_producer(empty(st), phase_of(n) ^ 1, abort_flag, kWaitCycles))) {
              --(s ? made[1] : made[0]);
              break;
            }
            if (lane == 0) {
              mbar_expect_tx(full(st), S::kUnit);
              tma_load_slots(base + kRing + st * S::kUnit, kv ? &maps.v : &maps.k, full(st), t * kTile, g, b, hint);
            }
            if (S::kPos) {
              // positions go with V: its place is held until the softmax has read them
              if (a.slopes && kv == 1)
#pragma unroll
                for (int i = lane; i < kTile; i += 32) {
                  const int j = t * kTile + i;
                  ((int*)(sm + kPosAt + st * S::kPos))[i] = j < sg.keys ? a.c.positions[(size_t)sg.u * a.c.capacity + j] : 0;
                }
              mbar_arrive(full(st));
            }
          }
        next_segment(sg, a, 7, blocks);
      } while (ok && sg.t1);
      // copies in flight end before the block does
      if (!ok)
        for (int s = 0; s < 2; ++s)
          for (int n = s ? made[1] : made[0], i = max(0, n - NR); i < n; ++i) mbar_drain(full(place_of(s, i)), phase_of(i), abort_flag);
    } else if (work && warp < 3) {
      // Products of stream s, each job's scores made after the outputs of the job before.
      const int s = warp - 1;
      const uint32_t lead = lane == 0;
      const uint32_t idesc_s = instr_desc(128, kTile) | (a.scale2 < 0.f || a.inv_cap < 0.f ? 1u << 13 : 0u);
      constexpr uint32_t idesc_o = instr_desc(128, D) | kTransposeB;
      const uint64_t q_desc = smem_desc(base + (MT == 2 ? s * 128 * 128 : 0)), k_desc = smem_desc(base + kRing), v_desc = smem_desc_n(base + kRing);
      const uint32_t q_lo = (uint32_t)q_desc, k_lo = (uint32_t)k_desc, v_lo = (uint32_t)v_desc, hi_k = (uint32_t)(q_desc >> 32), hi_v = (uint32_t)(v_desc >> 32);
      const uint32_t s_at = tmem + s * 128, o_at = tmem + 256 + s * 128;
      int n = 0, seg = 0, tails = 0, done = 0, used = 0;           // jobs before the segment; segments; tails, jobs, segments with jobs
      bool ok = true;
      do {
        const int tiles = sg.t1 - sg.t0, jobs = MT == 2 ? tiles : (tiles + 1 - s) / 2, n_old = sg.keys - a.n_new;
        auto scores = [&](int k) {
          const int unit = 2 * (n + k), st = place_of(s, unit);
          if (!(ok = wait(full(st), phase_of(unit)))) return;
          tc_fence_after();
          const uint32_t kd = k_lo + ((st * S::kUnit) >> 4);
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk)
            mma_ss(s_at, q_lo + (((kk / 4) * RB * 128 + (kk % 4) * 32) >> 4), kd + (((kk / 4) * kTile * 128 + (kk % 4) * 32) >> 4), hi_k, idesc_s, kk > 0, lead);
          commit_by(lead, s_full(s));
          commit_by(lead, empty(st));
        };
        // (a stream without a tile in the segment says as well that it came by: else its wait might be for a phase that is gone)
        if ((ok = wait(q_full, seg & 1)) && lead) mbar_arrive(q_empty);
        if (ok && jobs > 0) scores(0);
#pragma unroll 1
        for (int k = 0; k < jobs && ok; ++k) {
          const int t = MT == 2 ? k : 2 * k + s, unit = 2 * (n + k) + 1, st = place_of(s, unit);
          if (!(ok = wait(full(st), phase_of(unit)))) break;
          // A tile with new tokens is handed to the warp that looks through it, and taken back: by barriers of their own, as a wait by
          // parity holds only for who follows a barrier from phase to phase.
          const bool tail = (sg.t0 + t + 1) * kTile > n_old;
          if (tail && lead) mbar_arrive(v_look(s));
          if (k == 0 && used++ > 0 && !(ok = wait(o_free(s), used & 1))) break;
          if (tail && !(ok = wait(v_ready(s), tails++ & 1))) break;
          const uint32_t vd = v_lo + ((st * S::kUnit) >> 4);
          // the first half of the keys beside the exponentials of the second
          if (!(ok = wait(p_half(s), done & 1))) break;
          tc_fence_after();
#pragma unroll
          for (int kk = 0; kk < kTile / 32; ++kk) mma_ts(o_at, s_at + kk * 8, vd + ((kk * 16 * 128) >> 4), hi_v, idesc_o, k > 0 || kk > 0, lead);
          if (!(ok = wait(p_ready(s), done & 1))) break;
          tc_fence_after();
#pragma unroll
          for (int kk = kTile / 32; kk < kTile / 16; ++kk) mma_ts(o_at, s_at + kk * 8, vd + ((kk * 16 * 128) >> 4), hi_v, idesc_o, 1, lead);
          commit_by(lead, o_done(s));
          commit_by(lead, empty(st));
          ++done;
          if (k + 1 < jobs) scores(k + 1);
        }
        n += jobs;
        ++seg;
        next_segment(sg, a, 7, blocks);
      } while (ok && sg.t1);
      commit_by(lead, drained(s));
      clean = mbar_drain(drained(s), 0, abort_flag);
      if (!clean) *abort_flag = 2;
    } else if (work) {
      // V tiles with new tokens
      int n[2] = {0, 0}, tails[2] = {0, 0};                        // jobs of the streams before the segment
      bool ok = true;
      do {
        const int n_old = sg.keys - a.n_new;
        for (int t = max(sg.t0, n_old / kTile); t < sg.t1 && ok; ++t) {
          const int of = MT == 2 ? 0 : (t - sg.t0) & 1, k = MT == 2 ? t - sg.t0 : (t - sg.t0) / 2, st = place_of(of, 2 * ((of ? n[1] : n[0]) + k) + 1);
          const int row0 = max(0, n_old - t * kTile), row1 = min(kTile, sg.keys - t * kTile);
          for (int s = 0; s < 2 && ok; ++s)
            if (MT == 2 || ((t - sg.t0) & 1) == s) ok = mbar_wait_producer(v_look(s), tails[s]++ & 1, abort_flag, kWaitCycles);
          if (!ok) break;
          // (rows behind the last key hold what the cache held there)
#pragma unroll 8
          for (int i = row1 * CH + lane; i < kTile * CH; i += 32) *(uint4*)(sm + kRing + st * S::kUnit + tile_at<kTile>(i / CH, i % CH)) = make_uint4(0, 0, 0, 0);
          constexpr int kGo = 8;
#pragma unroll 1
          for (int i0 = row0 * CH + lane; i0 < row1 * CH; i0 += 32 * kGo) {
            uint4 x[kGo];
#pragma unroll
            for (int e = 0; e < kGo; ++e) {
              const int i = min(i0 + 32 * e, row1 * CH - 1);
              x[e] = *(const uint4*)(sm + kRing + st * S::kUnit + tile_at<kTile>(i / CH, i % CH));
            }
            bool bad = false;
#pragma unroll
            for (int e = 0; e < kGo; ++e) bad |= not_finite(x[e].x) || not_finite(x[e].y) || not_finite(x[e].z) || not_finite(x[e].w);
            if (bad) {
              if (MT == 2) odd_v[0] = odd_v[1] = 1;
              else odd_v[of] = 1;
#pragma unroll
              for (int e = 0; e < kGo; ++e) {
                const int i = min(i0 + 32 * e, row1 * CH - 1);
                uint32_t w[4] = {x[e].x, x[e].y, x[e].z, x[e].w};
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                  if ((w[f] & 0x7f80u) == 0x7f80u) w[f] &= 0xffff0000u;
                  if ((w[f] & 0x7f800000u) == 0x7f800000u) w[f] &= 0xffffu;
                }
                *(uint4*)(sm + kRing + st * S::kUnit + tile_at<kTile>(i / CH, i % CH)) = make_uint4(w[0], w[1], w[2], w[3]);
              }
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          for (int s = 0; s < 2; ++s)
            if (MT == 2 || ((t - sg.t0) & 1) == s) mbar_arrive(v_ready(s));
        }
        const int tiles = sg.t1 - sg.t0;
        n[0] += MT == 2 ? tiles : (tiles + 1) / 2;
        n[1] += MT == 2 ? tiles : tiles / 2;
        next_segment(sg, a, 7, blocks);
      } while (ok && sg.t1);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    if (work) {
      const int s = (warp - 4) / 4, quarter = warp % 4;
      const uint32_t lanes = (uint32_t)(quarter * 32) << 16, s_at = tmem + s * 128 + lanes, o_at = tmem + 256 + s * 128 + lanes;
      const float scale2 = fabsf(a.scale2);                       // (a negative scale negates the product)
      const uint64_t cap2 = pack2(a.cap2, a.cap2), inv2 = pack2(fabsf(a.inv_cap), fabsf(a.inv_cap));
      int done = 0, seg = 0;
      bool ok = true;
      do {
        {
          // the segment's rows, once the products of the segment before have read theirs  (rows beyond the last do not reach these)
          if (seg > 0 && !(ok = wait(q_empty, (seg - 1) & 1))) break;
          const int b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv;
          const char* const q0 = a.q + (size_t)b * a.q_batch + (size_t)(g * a.group) * a.q_head;
#pragma unroll 4
          for (int i = tid - 128; i < min(RB, a.rows - sg.rb * RB) * CH; i += 256) {
            const int row = i / CH, ch = i % CH, r = sg.rb * RB + row, tok = quotient(r, a.by_group), h = r - tok * a.group;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                         ::"r"(base + (ch >> 3) * (RB * 128) + row * 128 + (((ch ^ row) & 7) << 4)),
                           "l"(q0 + (size_t)tok * a.q_token + (size_t)h * a.q_head + ch * 16) : "memory");
          }
          asm volatile("cp.async.wait_all;" ::: "memory");
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(q_full);
          ++seg;
        }
        const int tiles = sg.t1 - sg.t0, jobs = MT == 2 ? tiles : (tiles + 1 - s) / 2, n_old = sg.keys - a.n_new;
        const int row = (MT == 2 ? s * 128 : 0) + quarter * 32 + lane, r = sg.rb * RB + row;
        const bool idle = r - lane >= a.rows;                      // no row of this warp: it only keeps step
        const RowOptions ro = row_options(a, sg.u, min(r, a.rows - 1));
        float m = -INFINITY, l = 0.f;
        // A reference is a rounded product of a score and the scale, the products in the exponents are not rounded: 2^-24 |m| apart.  Where
        // that is more than 1/16 they are rounded as well (`far`).
#pragma unroll 1
        for (int k = 0; k < jobs; ++k, ++done) {
          const int t = MT == 2 ? k : 2 * k + s, j0 = (sg.t0 + t) * kTile;
          if (!(ok = wait(s_full(s), done & 1))) break;
          const int* kp = nullptr;
          if (OPT && a.slopes) {
            // (these scores were made after the outputs of the tile before, so that the place's previous tile has come and gone)
            const int unit = 2 * done + 1, st = place_of(s, unit);
            if (!(ok = wait(full(st), phase_of(unit)))) break;
            kp = (const int*)(sm + kPosAt + st * S::kPos);
          }
          tc_fence_after();
          if (!idle) {
            if (OPT) {
              // x in bits, back to its place (a loop: this code 128 times over would not stay in the instruction cache)
#pragma unroll 1
              for (int c = 0; c < kTile; c += 32) {
                float x[32];
                tmem_ld(s_at + c, x);
                if (a.cap2 != 0.f) {
#pragma unroll
                  for (int e = 0; e < 32; e += 2) capped2(x[e], x[e + 1], cap2, inv2);
                } else {
#pragma unroll
                  for (int e = 0; e < 32; ++e) x[e] *= scale2;
                }
                if (a.slopes) {
#pragma unroll
                  for (int e = 0; e < 32; ++e) x[e] = fmaf(-ro.slope2, (float)(ro.position - kp[c + e]), x[e]);
                }
                tmem_st32(s_at + c, x);
              }
              tmem_st_wait();
            }
            float v[kTile], top = -INFINITY;
#pragma unroll
            for (int c = 0; c < kTile; c += 32) tmem_ld32(s_at + c, v + c);
#pragma unroll
            for (int c = 0; c < kTile; c += 32) tmem_landed(v + c);
            if (j0 + kTile > n_old) {
              // the tile has new tokens: bit e of a word says whether column c + e is seen
#pragma unroll
              for (int c = 0; c < kTile; c += 32) {
                const int first = j0 + c - n_old, keys = sg.keys - j0 - c;     // of the new tokens; keys from here on
                uint32_t see = first >= 64 ? 0u : first >= 0 ? (uint32_t)(ro.seen >> first)
                               : first > -32 ? (uint32_t)(ro.seen << -first) | ((1u << -first) - 1u) : 0xffffffffu;
                see = keys >= 32 ? see : keys <= 0 ? 0u : see & ((1u << keys) - 1u);
#pragma unroll
                for (int e = 0; e < 32; ++e) v[c + e] = see >> e & 1 ? v[c + e] : -INFINITY;
              }
            }
            {
              float t0 = v[0], t1 = v[1];
#pragma unroll
              for (int e = 2; e + 3 < kTile; e += 4) {
                t0 = max3(t0, v[e], v[e + 1]);
                t1 = max3(t1, v[e + 2], v[e + 3]);
              }
              top = fmaxf(max3(t0, t1, v[kTile - 2]), v[kTile - 1]);
            }
            const float mul = OPT ? 1.f : scale2;
            float times = mul;
            top *= mul;
            auto far = [&] { return !OPT && r < a.rows && fabsf(m) > 0x1p20f; };   // (rows behind the last hold anything)
            const bool grown = top > m + kSlack;
            if (__any_sync(0xffffffffu, grown || far())) {
              const float to = grown ? top : m, f = m == -INFINITY ? 0.f : fast_exp2(m - to);
              m = to;
              l *= f;
              if (!OPT && __any_sync(0xffffffffu, far())) {
#pragma unroll
                for (int e = 0; e < kTile; ++e) v[e] *= mul;
                times = 1.f;
              }
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
                  for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(x[e] * f);
                  tmem_st16(o_at + c, y);
                }
                tmem_st_wait();
              }
            }
            // The halves of the rows take turns with the exponentials, so that one's run beside the other's products: left alone they fall
            // into step, and exponentials and products wait for one another (a key tile of 256 rows 5200 clocks).
            if (MT == 2 && done >= 1 - s && !(ok = wait(turn(s), (done - 1 + s) & 1))) break;
            const float ref = m == -INFINITY ? 0.f : m;
            const uint64_t mul2 = pack2(times, times), ref2 = pack2(-ref, -ref);
            uint64_t sum = pack2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < kTile; c += 32) {
              uint32_t p[16];
#pragma unroll
              for (int e = 0; e < 32; e += 2) {
                const uint64_t x = exp2_sfu2(fma2(pack2(v[c + e], v[c + e + 1]), mul2, ref2));
                float p0, p1;
                unpack2(x, p0, p1);
                sum = add2(sum, x);
                // p keeps 8 bits for the product, as V does; the sum l is of the unrounded values  (attend_mma.cu has the errors)
                p[e / 2] = bf16x2(p0, p1);
              }
              tmem_st16(s_at + c / 2, p);                          // (over scores, which are in registers)
              if (c == kTile / 2 - 32) {
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_half(s));
              }
            }
            float s0, s1;
            unpack2(sum, s0, s1);
            l += s0 + s1;
            tmem_st_wait();
          } else {
            if (MT == 2 && done >= 1 - s && !(ok = wait(turn(s), (done - 1 + s) & 1))) break;
            if (lane == 0) mbar_arrive(p_half(s));
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(p_ready(s));
            if (MT == 2) mbar_arrive(turn(1 - s));
          }
        }
        if (!ok) break;
        if (lane == 0) mbar_arrive(q_empty);                       // (this stream's scores are all there)
        const int slot = sg.u * blocks + sg.rb + blockIdx.x;
        const size_t at = MT == 2 ? (size_t)slot * RB + row : ((size_t)slot * 2 + s) * RB + row;
        if (r < a.rows) a.part_stat[at] = make_float2(m, l);
        if (jobs > 0) {
          if (!(ok = wait(o_done(s), (done - 1) & 1))) break;
          tc_fence_after();
          if (!idle) {
            // (this stream's own flag: o_done(s) comes behind the look through its tiles alone.  Tokens across two tiles may be added by both
            // streams: infinity and NaN stay what they are.)
            const bool odd = odd_v[s] && sg.t1 * kTile > n_old;
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float v[32];
              tmem_ld(o_at + c, v);
              if (odd && r < a.rows) {
                // V of new tokens that is not finite was left out of the product: it makes what sees it so
                unsigned long long rest = ro.seen & (a.n_new == 64 ? ~0ull : (1ull << a.n_new) - 1);
#pragma unroll 1
                for (; rest; rest &= rest - 1) {
                  const int i = __ffsll((long long)rest) - 1;
                  const uint32_t* const from = (const uint32_t*)(a.c.v + unit_offset(a.c, sg.u) + (size_t)(n_old + i) * a.c.s_token + c * 2);
#pragma unroll
                  for (int e = 0; e < 16; ++e) {
                    const uint32_t w = from[e];
                    if ((w & 0x7f80u) == 0x7f80u) v[2 * e] += __uint_as_float(w << 16);
                    if ((w & 0x7f800000u) == 0x7f800000u) v[2 * e + 1] += __uint_as_float(w & 0xffff0000u);
                  }
                }
              }
              if (r < a.rows) {
                // (column after column of four: neighbouring rows, the lanes, side by side)
                float4* const to = (float4*)a.part_out + ((at - row) / RB * (D / 4) + c / 4) * RB + row;
#pragma unroll
                for (int e = 0; e < 8; ++e) to[e * RB] = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(o_free(s));
        }
        next_segment(sg, a, 7, blocks);
      } while (sg.t1);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    clean = *abort_flag != 2;
    if (clean) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
  if (tid == 0 && *abort_flag) atomicCAS(a.c.status, 0, (int)STRUCTKV_ERR_TIMEOUT);
}

template <int D, int MT, bool OPT>
cudaError_t launch_one(const AttendArgs& a, const CacheMaps& m, cudaStream_t st) {
  using S = TcAttend<D, MT, OPT>;
  const cudaError_t e = allow_smem<attend_tc<D, MT, OPT>>(S::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_tc<D, MT, OPT>, dim3(a.ctas), dim3(kThreads), S::kSmem, st, a, m);
}
template <int D>
cudaError_t launch_d(const AttendArgs& a, const AttendPlan& p, const CacheMaps& m, cudaStream_t st) {
  // (without options what is masked is minus infinity before it is scaled: not for a scale of zero)
  const bool opt = a.cap2 != 0.f || a.slopes || a.scale2 == 0.f;
  if (p.rb == 256) return opt ? launch_one<D, 2, true>(a, m, st) : launch_one<D, 2, false>(a, m, st);
  return opt ? launch_one<D, 1, true>(a, m, st) : launch_one<D, 1, false>(a, m, st);
}

}  // namespace

cudaError_t launch_attend_tc(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  CacheMaps m;
  if (!cache_maps(ctx, a, kTile, &m)) return cudaErrorInvalidValue;
  return ctx.cfg.head_dim == 128 ? launch_d<128>(a, p, m, st) : launch_d<64>(a, p, m, st);
}

}  // namespace skv
