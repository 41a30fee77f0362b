// Attention of new tokens over a bf16 cache, up to 16 rows of a KV head at a time, and the weight of accepted tokens.
//
// One pass: per row a reference m, sum l and unscaled output O over the keys seen so far; a tile of 64 keys gives
// S = K Q^T, p = 2^(x - m), l += sum p, O^T += V^T p.  Rows are few and reading K and V is the bound, so keys are the long side of
// the m16n8k16 products (16 keys x 8 rows, then 16 columns of V x 8 rows): four rows of a single token fill half a product, in
// the other orientation a quarter.  A warp takes 16 keys of a tile and all rows; tiles come by TMA (128-byte swizzle)
// through a ring that one warp fills; NG groups of warps take tiles in turn, each warp with statistics of its own, so that
// nothing but the ring is waited for, and a segment's end merges the warps.  The reference follows a row's maximum only where
// that outgrows it by 2^kSlack: p then stays below 2^kSlack, far from overflow, and most tiles need neither shuffles nor scaling.
#include <algorithm>

#include "attend.cuh"

namespace skv {
namespace {

constexpr int kTileKeys = 64;

__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
// Arrives once this thread's cp.async copies so far are there (one of the barrier's expected arrivals).
__device__ __forceinline__ void cp_arrive(uint32_t bar) { asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void ldsm(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
// Transposes an 8 x 8 matrix of 16-bit values that a warp holds.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// Rows of D bf16 in shared memory: 16-byte chunk c of row r lies at chunk c ^ (r mod 8), so that eight rows' equal chunks are
// in different banks.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) { return row * (D * 2) + ((chunk ^ (row & 7)) << 4); }

// NR blocks of 8 rows; four warps along a tile's keys, NG groups of these.
template <int D, int NR, int NG>
struct AttendShape {
  static constexpr int RB = 8 * NR, kWarps = 4 * NG, THREADS = 64 + kWarps * 32, kSets = 4 * NG;
  static constexpr int kTileBytes = kTileKeys * D * 2;
  static constexpr int kPosOff = 2 * kTileBytes, kStage = kPosOff + 1024;
  static constexpr int kRow = D + 4;                             // of a set's output: rows two apart are eight banks apart
  static constexpr int kFixed = kSets * RB * (kRow + 2) * 4 + 256 + 1024;
  // (a place of the ring always serves the same group: a wait by parity holds only for who follows a barrier from phase to phase)
  static constexpr int kStages = std::min(8, (226 * 1024 - kFixed) / kStage) / NG * NG;
  static constexpr int kSmem = kStages * kStage + kFixed;
  static_assert(kStages >= 4 && kStage % 1024 == 0, "a ring");
};

template <int D, int NR, int NG, bool OPT>
__global__ void __launch_bounds__(64 + 128 * NG, 1) attend_mma(const __grid_constant__ AttendArgs a, const __grid_constant__ CacheMaps maps) {
  using S = AttendShape<D, NR, NG>;
  constexpr int RB = S::RB, CH = D / 8, ST = S::kStages, KK = D / 16;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  float* const outs = (float*)(sm + ST * S::kStage);            // [set][RB][kRow]
  float* const stat = outs + S::kSets * RB * S::kRow;           // [2][RB][set]
  const uint32_t bars = smem_u32(stat + 2 * S::kSets * RB);     // full [ST], empty [ST]
  volatile int* const abort_flag = (volatile int*)(stat + 2 * S::kSets * RB) + 4 * ST;
  auto full = [&](int st) { return bars + 8 * st; };
  auto empty = [&](int st) { return bars + 8 * (ST + st); };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int blocks = (a.rows + RB - 1) / RB;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(full(i), OPT ? 33 : 1);                         // the copies by TMA, and 32 lanes' own
      mbar_init(empty(i), 4);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&maps.k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&maps.v) : "memory");
  }
  __syncthreads();
  pdl_wait();
  const WorkStart ws = find_work(a, 6, blocks, blockIdx.x == 0 ? a.unit_start : nullptr);
  Segments sg = first_segment(a, ws, 6, blocks);
  if (sg.t1 == 0) return;

  if (warp == 0) {
    // the ring's producer
    const uint64_t hint = blocks == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
    int st = 0, n = 0;
    bool ok = true;
#pragma unroll 1
    for (; sg.t1 && ok; next_segment(sg, a, 6, blocks)) {
      const int b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv;
#pragma unroll 1
      for (int t = sg.t0; t < sg.t1; ++t, ++n) {
        const uint32_t to = base + st * S::kStage;
        if (n >= ST && !(ok = mbar_wait_producer(empty(st), (n / ST - 1) & 1, abort_flag, kWaitCycles))) break;
        if (lane == 0) {
          mbar_expect_tx(full(st), 2 * S::kTileBytes);
          tma_load_slots(to, &maps.k, full(st), t * kTileKeys, g, b, hint);
          tma_load_slots(to + S::kTileBytes, &maps.v, full(st), t * kTileKeys, g, b, hint);
        }
        if (OPT) {
          if (a.slopes) {
            const int* const pos = a.c.positions + (size_t)sg.u * a.c.capacity;
            const int n_old = sg.keys - a.n_new;
#pragma unroll
            for (int i = lane; i < kTileKeys; i += 32) {
              const int j = t * kTileKeys + i;
              const bool is_new = a.fresh.k && j >= n_old && j < sg.keys;      // (their places in the cache are being written)
              cp4(to + S::kPosOff + i * 4, is_new ? a.fresh.positions + (size_t)b * a.n_new + j - n_old : pos + (j < sg.keys ? j : 0), j < sg.keys);
            }
          }
          cp_arrive(full(st));
        }
        if (++st == ST) st = 0;
      }
    }
    if (*abort_flag) {
      // copies in flight end before the block does
      for (int i = max(0, n - ST); i < n; ++i) mbar_drain(full(i % ST), (i / ST) & 1, abort_flag);
      if (lane == 0) atomicCAS(a.c.status, 0, (int)STRUCTKV_ERR_TIMEOUT);
    }
    return;
  }
  if (warp == 1) {
    // New rows go into the cache; nobody here waits for that (patch() below).  Row blocks of a unit in other CTAs write the same bytes.
    if (!a.fresh.k) return;
#pragma unroll 1
    for (; sg.t1; next_segment(sg, a, 6, blocks)) {
      if (sg.t1 * kTileKeys <= sg.keys - a.n_new) continue;
      const int b = quotient(sg.u, a.by_kv);
      append_rows(a.c, a.fresh, a.n_new, sg.u, b, sg.u - b * a.c.n_kv, sg.keys - a.n_new, lane);
    }
    return;
  }

  const int cw = warp - 2, grp = cw / 4, kw = cw % 4, g8 = lane >> 2, t4 = lane & 3;
  auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(S::kWarps * 32) : "memory"); };
  uint32_t qf[NR][KK][2];
  float o[NR][KK][4];                                           // column g8 (+ 8) of 16, rows 2 t4 and + 1 of the block
  float m[NR][2], l[NR][2];
  float slope2[NR][2];
  int place[NR][2];
  bool fresh = true;                                            // nothing of this segment yet
  int n = 0, st = 0;
#pragma unroll 1
  for (; sg.t1; next_segment(sg, a, 6, blocks)) {
    const int first_row = sg.rb * RB + 2 * t4;                  // row of (block i, x): first_row + 8 i + x
    const int b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv, n_old = sg.keys - a.n_new, seg = n;
#pragma unroll 1
    for (int t = sg.t0; t < sg.t1; ++t, ++n, st = st + 1 == ST ? 0 : st + 1) {
      if (n % NG != grp) continue;
      const uint32_t from = base + st * S::kStage;
      const unsigned char* const here = sm + st * S::kStage;
      if (fresh) {
        // a segment begins: its rows, while the tile is on its way
        fresh = false;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
#pragma unroll
          for (int x = 0; x < 2; ++x) { m[i][x] = -INFINITY; l[i][x] = 0.f; }
#pragma unroll
          for (int k = 0; k < KK; ++k) o[i][k][0] = o[i][k][1] = o[i][k][2] = o[i][k][3] = 0.f;
          const int r = sg.rb * RB + 8 * i + g8;
          const bool is = r < a.rows;
          const int tok = is ? quotient(r, a.by_group) : 0, h = is ? r - tok * a.group : 0;
          const char* const q = a.q + (size_t)b * a.q_batch + (size_t)tok * a.q_token + (size_t)(g * a.group + h) * a.q_head + t4 * 4;
#pragma unroll
          for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int y = 0; y < 2; ++y) qf[i][kk][y] = is ? *(const uint32_t*)(q + kk * 32 + y * 16) : 0u;
        }
        if (OPT && a.slopes)
#pragma unroll
          for (int i = 0; i < NR; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const RowOptions ro = row_options(a, sg.u, min(first_row + 8 * i + x, a.rows - 1));
              slope2[i][x] = ro.slope2;
              place[i][x] = ro.position;
            }
      }
      const int j0 = t * kTileKeys + kw * 16;
      const bool tail = j0 + 16 > n_old;
      mbar_wait(full(st), (n / ST) & 1, abort_flag);            // (on expiry the numbers are void, the control flow goes on)
      if (tail && a.fresh.k) {
        // patch: new tokens among this warp's 16 keys, whose rows TMA did not find in the cache
#pragma unroll 1
        for (int i = max(0, j0 - n_old); i < min(a.n_new, j0 + 16 - n_old); ++i) {
          const size_t from = (size_t)b * a.fresh.s_batch + (size_t)i * a.fresh.s_token + (size_t)g * a.fresh.s_head;
          const int row = n_old + i - t * kTileKeys;
          for (int e = lane; e < 2 * CH; e += 32) {
            const bool is_v = e >= CH;
            const int ch = is_v ? e - CH : e;
            *(uint4*)(sm + st * S::kStage + (is_v ? S::kTileBytes : 0) + tile_at<kTileKeys>(row, ch)) = *(const uint4*)((is_v ? a.fresh.v : a.fresh.k) + from + ch * 16);
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // (the place's next tile comes by TMA)
        __syncwarp();
      }
      // products: two chains where a warp has one block of rows
      constexpr int CHAINS = NR == 1 ? 2 : 1;
      float acc[CHAINS][NR][4];
#pragma unroll
      for (int c = 0; c < CHAINS; ++c)
#pragma unroll
        for (int i = 0; i < NR; ++i) acc[c][i][0] = acc[c][i][1] = acc[c][i][2] = acc[c][i][3] = 0.f;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        uint32_t kf[4];
        ldsm(from + tile_at<kTileKeys>(kw * 16 + (lane & 15), kk * 2 + (lane >> 4)), kf);
#pragma unroll
        for (int i = 0; i < NR; ++i) mma_16x8x16(acc[kk % CHAINS][i], kf[0], kf[1], kf[2], kf[3], qf[i][kk][0], qf[i][kk][1]);
      }
      float s[NR][4];                                           // element 2 y + x: key g8 + 8 y, row x
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[i][e] = CHAINS == 2 ? acc[0][i][e] + acc[CHAINS - 1][i][e] : acc[0][i][e];
      // x in bits
      if (OPT) {
        int kp[2] = {0, 0};
        if (a.slopes) { kp[0] = ((const int*)(here + S::kPosOff))[kw * 16 + g8]; kp[1] = ((const int*)(here + S::kPosOff))[kw * 16 + g8 + 8]; }
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            in_bits2(a, s[i][e], s[i][e + 1]);
            if (a.slopes)
#pragma unroll
              for (int x = 0; x < 2; ++x) s[i][e + x] = fmaf(-slope2[i][x], (float)(place[i][x] - kp[e >> 1]), s[i][e + x]);
          }
      } else {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][e] *= a.scale2;
      }
      if (tail) {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const unsigned long long seen = row_seen(a, sg.u, min(first_row + 8 * i + x, a.rows - 1));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int j = j0 + g8 + 8 * y;
              if (j >= sg.keys || !sees(seen, j, n_old)) s[i][2 * y + x] = -INFINITY;
            }
          }
      }
      if (a.accumulate) {
        float* const to = a.logits + ((size_t)sg.u * a.c.capacity + j0 + g8) * a.group;
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int r = first_row + 8 * i + (e & 1);
            if (r < a.rows && j0 + g8 + 8 * (e >> 1) < sg.keys) to[8 * (e >> 1) * a.group + r] = s[i][e];
          }
      }
      // references
      bool grown = false;
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) grown |= fmaxf(s[i][x], s[i][2 + x]) > m[i][x] + kSlack;
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            float t = fmaxf(s[i][x], s[i][2 + x]);
#pragma unroll
            for (int d = 4; d < 32; d *= 2) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            t = fmaxf(t, m[i][x]);
            const float f = m[i][x] == -INFINITY ? 0.f : fast_exp2(m[i][x] - t);
            m[i][x] = t;
            l[i][x] *= f;
#pragma unroll
            for (int k = 0; k < KK; ++k) { o[i][k][x] *= f; o[i][k][2 + x] *= f; }
          }
      }
      uint32_t pf[NR][2];                                       // keys 2 t4 and + 1 (+ 8), row g8
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = fast_exp2(s[i][e] - (m[i][e & 1] == -INFINITY ? 0.f : m[i][e & 1]));
        l[i][0] += p[0] + p[2];
        l[i][1] += p[1] + p[3];
        // p keeps 8 bits for the product, as V does; the sum l is of the unrounded values.  (Outputs over 16 x 16384 keys are off by 2.0e-3,
        // relative, against 64 bits; with p in fp32 by 1.7e-3, which is the result's own rounding.)
        pf[i][0] = transposed(bf16x2(p[0], p[1]));
        pf[i][1] = transposed(bf16x2(p[2], p[3]));
      }
      // Where V of a new token, or of a slot behind them, is not finite, rows that do not see it must not meet it: 0 x infinity.  Those that
      // see it meet it, whatever is left of its probability.
      bool plain = true;
      if (tail) {
        bool bad = false;
#pragma unroll 2
        for (int i = lane; i < 16 * CH; i += 32) {
          const uint4 w = *(const uint4*)(here + S::kTileBytes + tile_at<kTileKeys>(kw * 16 + i / CH, i % CH));
          bad |= not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w);
        }
        plain = !__any_sync(0xffffffffu, bad);
      }
      if (plain) {
#pragma unroll
        for (int k = 0; k < KK; ++k) {
          uint32_t vf[4];
          ldsm_t(from + S::kTileBytes + tile_at<kTileKeys>(kw * 16 + (lane & 7) + (lane >> 4) * 8, k * 2 + ((lane >> 3) & 1)), vf);
#pragma unroll
          for (int i = 0; i < NR; ++i) mma_16x8x16(o[i][k], vf[0], vf[1], vf[2], vf[3], pf[i][0], pf[i][1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          unsigned see[2];                                      // keys of this warp's 16 that row 2 t4 + x sees
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const unsigned long long seen = row_seen(a, sg.u, min(first_row + 8 * i + x, a.rows - 1));
            see[x] = 0;
#pragma unroll 1
            for (int j = 0; j < 16; ++j) see[x] |= (unsigned)(j0 + j < sg.keys && sees(seen, j0 + j, n_old)) << j;
          }
#pragma unroll 1
          for (int j = 0; j < 16; ++j) {
            float p[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {                       // key j of row 2 t4 + x: lane (row, j / 2 mod 4)
              const uint32_t w0 = __shfl_sync(0xffffffffu, pf[i][0], (2 * t4 + x) * 4 + ((j & 7) >> 1));
              const uint32_t w1 = __shfl_sync(0xffffffffu, pf[i][1], (2 * t4 + x) * 4 + ((j & 7) >> 1));
              const uint32_t w = j < 8 ? w0 : w1;
              p[x] = __uint_as_float(j & 1 ? w & 0xffff0000u : w << 16);
            }
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
              for (int y = 0; y < 2; ++y) {
                const unsigned short h = *(const unsigned short*)(here + S::kTileBytes + tile_at<kTileKeys>(kw * 16 + j, k * 2 + y) + g8 * 2);
                const float v = __uint_as_float((uint32_t)h << 16);
#pragma unroll
                for (int x = 0; x < 2; ++x)
                  if (see[x] >> j & 1) o[i][k][2 * y + x] = fmaf(p[x], v, o[i][k][2 * y + x]);
              }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty(st));
    }

    {
      // the segment ends: its warps' outputs, each against its own reference, then their sum against a common one.  Sets (a group's
      // quarter of the keys) are counted from the group that took the segment's first tile.
      const int sets = min(S::kSets, (n - seg) * 4), my = ((grp + NG - seg % NG) % NG) * 4 + kw;
      if (my < sets) {
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) l[i][x] += __shfl_xor_sync(0xffffffffu, l[i][x], d);
            const int row = 8 * i + 2 * t4 + x;
            if (g8 == 0) {
              stat[row * S::kSets + my] = m[i][x];
              stat[(RB + row) * S::kSets + my] = l[i][x];
            }
            float* const to = outs + (my * RB + row) * S::kRow + g8;
#pragma unroll
            for (int k = 0; k < KK; ++k) { to[k * 16] = o[i][k][x]; to[k * 16 + 8] = o[i][k][2 + x]; }
          }
      }
      leave_partial<D, S::kWarps * 32, RB, S::kRow, S::kSets>(a, sg.u * blocks + sg.rb + blockIdx.x, min(RB, a.rows - sg.rb * RB), outs, stat,
                                                              stat + RB * S::kSets, sets, tid - 64, sync);
      sync();
      fresh = true;
    }
  }
}

// ---- weights of accepted tokens ------------------------------------------------------------------
// weights[j] = decay weights[j] + sum over accepted rows of 2^(x - lse): K tiles stream past the accepted tokens' rows
// (kWeighRows at a time in shared memory; a weight is rounded once for every kWeighRows of them); a warp has 16 keys of a tile in
// registers and adds up their rows.  4 x 16384 keys, 28 rows: K at 4.6 TB/s in 29.4 us; two groups of warps 40.8, twelve places
// instead of eight 29.6: what is left is a tile's way through load, products and sum, and the launch.
constexpr int kWeighRows = 64, kWeighStages = 8, kWeighGroups = 4, kWeighWarps = 4 * kWeighGroups;
static_assert(kWeighStages % kWeighGroups == 0, "a place of the ring serves one group");

template <int D>
constexpr int weigh_smem() {
  return kWeighStages * (kTileKeys * D * 2 + 1024) + kWeighRows * (D * 2 + 4 + sizeof(RowOptions)) + 256 + 1024;
}

template <int D, bool OPT>
__global__ void __launch_bounds__(32 + kWeighWarps * 32, 1)
weigh_mma(const __grid_constant__ AttendArgs a, const __grid_constant__ CacheMaps maps, const unsigned long long* __restrict__ accepted) {
  constexpr int CH = D / 8, KK = D / 16, ST = kWeighStages, kTileBytes = kTileKeys * D * 2, kStage = kTileBytes + 1024;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kQ = ST * kStage;
  RowOptions* const opts = (RowOptions*)(sm + kQ + kWeighRows * D * 2);
  float* const lse = (float*)(opts + kWeighRows);                 // in bits, +inf: no row
  const uint32_t bars = smem_u32(lse + kWeighRows);
  volatile int* const abort_flag = (volatile int*)(lse + kWeighRows) + 4 * ST;
  auto full = [&](int st) { return bars + 8 * st; };
  auto empty = [&](int st) { return bars + 8 * (ST + st); };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  if (tid == 0) {
    for (int i = 0; i < ST; ++i) {
      mbar_init(full(i), 33);
      mbar_init(empty(i), 4);
    }
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  const WorkStart ws = find_work(a, 6, 1, nullptr);
  Segments sg = first_segment(a, ws, 6, 1);
  if (sg.t1 == 0) return;
  // rows of the accepted tokens of a unit, and how often its tiles are gone through
  auto taken_of = [&](int u) { return accepted[quotient(u, a.by_kv)] & (a.n_new == 64 ? ~0ull : (1ull << a.n_new) - 1); };
  auto rounds_of = [&](int rows) { return rows <= kWeighRows ? 1 : (rows + kWeighRows - 1) / kWeighRows; };

  if (warp == 0) {
    const uint64_t policy = l2_policy_evict_first(), again = l2_policy_evict_normal();
    int n = 0;
    bool ok = true;
#pragma unroll 1
    for (; sg.t1 && ok; next_segment(sg, a, 6, 1)) {
      const int t0 = sg.t0, t1 = sg.t1, b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv;
      const int rounds = rounds_of(__popcll(taken_of(sg.u)) * a.group);
      for (int i = 0; i < rounds * (t1 - t0); ++i, ++n) {
        const int st = n % ST, t = t0 + i % (t1 - t0);
        const uint32_t to = base + st * kStage;
        if (n >= ST && !(ok = mbar_wait_producer(empty(st), (n / ST - 1) & 1, abort_flag, kWaitCycles))) break;
        if (lane == 0) {
          mbar_expect_tx(full(st), kTileBytes);
          tma_load_slots(to, &maps.k, full(st), t * kTileKeys, g, b, rounds == 1 ? policy : again);
        }
        if (OPT && a.slopes) {
          const int* const pos = a.c.positions + (size_t)sg.u * a.c.capacity;
#pragma unroll
          for (int e = lane; e < kTileKeys; e += 32) {
            const int j = t * kTileKeys + e;
            cp4(to + kTileBytes + e * 4, pos + (j < sg.keys ? j : 0), j < sg.keys);
          }
        }
        cp_arrive(full(st));
      }
    }
    if (*abort_flag) {
      for (int i = max(0, n - ST); i < n; ++i) mbar_drain(full(i % ST), (i / ST) & 1, abort_flag);
      if (lane == 0) atomicCAS(a.c.status, 0, (int)STRUCTKV_ERR_TIMEOUT);
    }
    return;
  }

  const int cw = warp - 1, grp = cw / 4, kw = cw % 4, g8 = lane >> 2, t4 = lane & 3;
  auto sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kWeighWarps * 32) : "memory"); };
  int n = 0;
#pragma unroll 1
  for (; sg.t1; next_segment(sg, a, 6, 1)) {                      // a unit's tiles of this CTA
    const int t0 = sg.t0, t1 = sg.t1;
    const int b = quotient(sg.u, a.by_kv), g = sg.u - b * a.c.n_kv, n_old = sg.keys - a.n_new;
    const unsigned long long taken = taken_of(sg.u);
    const int rows = __popcll(taken) * a.group, rounds = rounds_of(rows);
    float* const w = a.c.weights + (size_t)sg.u * a.c.capacity;
#pragma unroll 1
    for (int round = 0; round < rounds; ++round) {
      const int r0 = round * kWeighRows, n_rows = min(kWeighRows, rows - r0), n_blocks = (n_rows + 7) / 8;
      sync();
      for (int i = tid - 32; i < n_blocks * 8 * CH; i += kWeighWarps * 32) {
        const int row = i / CH, ch = i % CH;
        uint4 x = make_uint4(0, 0, 0, 0);
        float ref = INFINITY;
        RowOptions ro{0, 0.f, 0};
        if (row < n_rows) {
          unsigned long long rest = taken;                        // token of row r0 + row: the bit of that rank
          const int rank = quotient(r0 + row, a.by_group), h = r0 + row - rank * a.group;
          for (int skip = rank; skip > 0; --skip) rest &= rest - 1;
          const int tok = __ffsll((long long)rest) - 1;
          x = *(const uint4*)(a.q + (size_t)b * a.q_batch + (size_t)tok * a.q_token + (size_t)(g * a.group + h) * a.q_head + ch * 16);
          if (ch == 0) {
            ref = a.lse[((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h] * kLog2e;
            if (ref == -INFINITY) ref = INFINITY;                 // a row that saw nothing gave nothing
            ro = row_options(a, sg.u, tok * a.group + h);
          }
        }
        *(uint4*)(sm + kQ + chunk_at<D>(row, ch)) = x;
        if (ch == 0) { lse[row] = ref; opts[row] = ro; }
      }
      sync();
#pragma unroll 1
      for (int t = t0; t < t1; ++t, ++n) {
        if (n % kWeighGroups != grp) continue;
        const int st = n % ST;
        const uint32_t from = base + st * kStage;
        const int j_mine = t * kTileKeys + kw * 16 + g8 + 8 * t4;   // lane t4 = y of the four has key g8 + 8 y
        const float before = t4 < 2 && j_mine < sg.keys ? w[j_mine] : 0.f;
        mbar_wait(full(st), (n / ST) & 1, abort_flag);
        const int* const kp = (const int*)(sm + st * kStage + kTileBytes) + kw * 16;
        int pos[2] = {0, 0};
        if (OPT && a.slopes) { pos[0] = kp[g8]; pos[1] = kp[g8 + 8]; }
        uint32_t kf[KK][4];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) ldsm(from + tile_at<kTileKeys>(kw * 16 + (lane & 15), kk * 2 + (lane >> 4)), kf[kk]);
        __syncwarp();
        if (lane == 0) mbar_arrive(empty(st));
        const int j0 = t * kTileKeys + kw * 16;
        const bool tail = j0 + 16 > n_old;
        float sum[2] = {0.f, 0.f};                                // of keys g8 and g8 + 8, this thread's rows
#pragma unroll 1
        for (int rb = 0; rb < n_blocks; ++rb) {
          float s[2][4] = {};
#pragma unroll
          for (int kk = 0; kk < KK; kk += 2) {
            uint32_t qf[4];
            ldsm(base + kQ + chunk_at<D>(rb * 8 + (lane & 7), kk * 2 + (lane >> 3)), qf);
            mma_16x8x16(s[0], kf[kk][0], kf[kk][1], kf[kk][2], kf[kk][3], qf[0], qf[1]);
            mma_16x8x16(s[1], kf[kk + 1][0], kf[kk + 1][1], kf[kk + 1][2], kf[kk + 1][3], qf[2], qf[3]);
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int row = rb * 8 + 2 * t4 + x;
            const float ref = lse[row];
            RowOptions ro{};
            if (OPT || tail) ro = opts[row];
            float dot[2] = {s[0][x] + s[1][x], s[0][2 + x] + s[1][2 + x]};
            if (OPT) in_bits2(a, dot[0], dot[1]);
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int j = j0 + g8 + 8 * y;
              float v = OPT ? biased(a, dot[y], ro, pos[y]) : dot[y] * a.scale2;
              if (tail && (j >= sg.keys || !sees(ro.seen, j, n_old))) v = -INFINITY;
              sum[y] += ref == INFINITY ? 0.f : fast_exp2(v - ref);
            }
          }
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 1);
          sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 2);
        }
        if (t4 < 2 && j_mine < sg.keys) w[j_mine] = (round == 0 ? a.decay * before : before) + (t4 ? sum[1] : sum[0]);
      }
      if (rounds > 1) __threadfence_block();                      // (another warp may have the key in the next round)
    }
  }
}

bool options(const AttendArgs& a) { return a.cap2 != 0.f || a.slopes; }

template <int D, int NR, int NG, bool OPT>
cudaError_t launch_one(const AttendArgs& a, const CacheMaps& m, cudaStream_t st) {
  using S = AttendShape<D, NR, NG>;
  const cudaError_t e = allow_smem<attend_mma<D, NR, NG, OPT>>(S::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_mma<D, NR, NG, OPT>, dim3(a.ctas), dim3(S::THREADS), S::kSmem, st, a, m);
}
template <int D, bool OPT>
cudaError_t launch_rows(const AttendArgs& a, const AttendPlan& p, const CacheMaps& m, cudaStream_t st) {
  return p.rb == 8 ? launch_one<D, 1, 4, OPT>(a, m, st) : launch_one<D, 2, 2, OPT>(a, m, st);
}
template <int D, bool OPT>
cudaError_t launch_weigh(const AttendArgs& a, const CacheMaps& m, const unsigned long long* accepted, cudaStream_t st) {
  const cudaError_t e = allow_smem<weigh_mma<D, OPT>>(weigh_smem<D>());
  return e != cudaSuccess ? e : launch_pdl(weigh_mma<D, OPT>, dim3(a.ctas), dim3(32 + kWeighWarps * 32), weigh_smem<D>(), st, a, m, accepted);
}

}  // namespace

cudaError_t launch_attend_mma(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  CacheMaps m;
  if (!cache_maps(ctx, a, kTileKeys, &m)) return cudaErrorInvalidValue;
  if (ctx.cfg.head_dim == 128) return options(a) ? launch_rows<128, true>(a, p, m, st) : launch_rows<128, false>(a, p, m, st);
  return options(a) ? launch_rows<64, true>(a, p, m, st) : launch_rows<64, false>(a, p, m, st);
}

cudaError_t launch_weigh_bf16(const Ctx& ctx, const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st) {
  CacheMaps m;
  if (!cache_maps(ctx, a, kTileKeys, &m)) return cudaErrorInvalidValue;
  if (ctx.cfg.head_dim == 128) return options(a) ? launch_weigh<128, true>(a, m, accepted, st) : launch_weigh<128, false>(a, m, accepted, st);
  return options(a) ? launch_weigh<64, true>(a, m, accepted, st) : launch_weigh<64, false>(a, m, accepted, st);
}

}  // namespace skv
