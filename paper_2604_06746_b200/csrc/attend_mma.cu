// Attention of new tokens over a bf16 cache, up to 64 rows of a KV head at a time, and the weight of accepted tokens.
//
// Flash form: per row a running maximum m, sum l and unscaled output O over the keys seen so far; a key tile of 64 gives
// S = Q K^T, p = 2^(x - m), l += sum p, O += p V.  WK warps share a tile's keys (16 or 32 each), WR warps the rows (16 each);
// every warp has statistics of its own, so that nothing but the ring of tiles is waited for, and a segment's end merges
// them.  Products are m16n8k16: rows are few, and reading K and V is the bound.
#include <algorithm>

#include "attend.cuh"
#include "score_tc.cuh"

namespace skv {
namespace {

constexpr int kTileKeys = 64;

__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldsm(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t at, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// Whether one of two bf16 is infinite or NaN.
__device__ __forceinline__ bool not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
// Rows of D bf16 in shared memory: 16-byte chunk c of row r lies at chunk c ^ (r mod 8), so that eight rows' equal chunks are
// in different banks.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) { return row * (D * 2) + ((chunk ^ (row & 7)) << 4); }

// Where a CTA is in its run of tiles.
struct Cursor {
  int u, rb, t, tiles, keys;
  const char *k, *v;
};
__device__ __forceinline__ void enter(Cursor& c, const CacheView& cache, int n_new, int tile) {
  c.keys = c.u < cache.units ? unit_keys(cache, c.u, n_new) : 0;
  while (c.keys == 0 && c.u < cache.units - 1) c.keys = unit_keys(cache, ++c.u, n_new);
  c.tiles = (c.keys + tile - 1) / tile;
  const size_t off = unit_offset(cache, min(c.u, cache.units - 1));
  c.k = cache.k + off;
  c.v = cache.v + off;
}
__device__ __forceinline__ void advance(Cursor& c, const CacheView& cache, int n_new, int tile, int blocks) {
  if (++c.t < c.tiles) return;
  c.t = 0;
  if (++c.rb < blocks) return;
  c.rb = 0;
  ++c.u;
  enter(c, cache, n_new, tile);
}

template <int D, int WR, int WK>
struct AttendShape {
  static constexpr int RB = 16 * WR, THREADS = WR * WK * 32, KW = kTileKeys / WK;
  static constexpr int kTileBytes = kTileKeys * D * 2, kQBytes = RB * D * 2;
  static constexpr int kStage = 2 * kTileBytes + kQBytes + kTileKeys * 4;
  static constexpr int kStages = WR == 1 ? 3 : WR == 2 ? 4 : 3;
  static constexpr int kMergeRow = D + 4;
  static constexpr int kSmem = kStages * kStage + RB * kMergeRow * 4 + 2 * WK * RB * 4 + 128;
};

template <int D, int WR, int WK, bool OPT>
__global__ void __launch_bounds__(WR * WK * 32, WR == 1 ? 2 : 1) attend_mma(const __grid_constant__ AttendArgs a) {
  using S = AttendShape<D, WR, WK>;
  constexpr int RB = S::RB, KW = S::KW, NT = S::THREADS, CH = D / 8, NB = KW / 8;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  float* const merge = (float*)(sm + S::kStages * S::kStage);
  float* const stat = merge + RB * S::kMergeRow;                // [2][WK][RB]
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wr = warp / WK, wk = warp % WK;
  const int cta = blockIdx.x, blocks = (a.rows + RB - 1) / RB;
  pdl_trigger();
  pdl_wait();
  const WorkStart ws = find_work<NT>(a.c, a.n_new, kTileKeys, blocks, [&](long long W) { return cut(cta, W, sharers(W, gridDim.x)); },
                                     cta == 0 ? a.unit_start : nullptr);
  const int C = sharers(ws.total, gridDim.x);
  const long long lo = cut(cta, ws.total, C), hi = cut(cta + 1, ws.total, C);
  if (lo >= hi) return;
  Cursor cur;
  cur.u = ws.unit;
  enter(cur, a.c, a.n_new, kTileKeys);
  {
    const int rest = (int)(lo - ws.before);
    cur.rb = rest / cur.tiles;
    cur.t = rest - cur.rb * cur.tiles;
  }
  Cursor ld = cur;
  long long at = lo, ld_at = lo;

  auto load = [&]() {
    const int stage = (int)((ld_at - lo) % S::kStages);
    const uint32_t to = base + stage * S::kStage;
    const int j0 = ld.t * kTileKeys;
#pragma unroll 4
    for (int i = tid; i < kTileKeys * CH; i += NT) {
      const int row = i / CH, ch = i % CH, j = j0 + row;
      const bool there = j < ld.keys;
      const size_t off = there ? (size_t)j * a.c.s_token + ch * 16 : 0;
      cp16(to + chunk_at<D>(row, ch), ld.k + off, there);
      cp16(to + S::kTileBytes + chunk_at<D>(row, ch), ld.v + off, there);
    }
    if (OPT && a.slopes)
      for (int i = tid; i < kTileKeys; i += NT) {
        const bool there = j0 + i < ld.keys;
        cp4(to + 2 * S::kTileBytes + S::kQBytes + i * 4, a.c.positions + (size_t)ld.u * a.c.capacity + (there ? j0 + i : 0), there);
      }
    if (ld.t == 0 || ld_at == lo) {                             // a segment begins: its rows come along
      const int b = ld.u / a.c.n_kv, g = ld.u % a.c.n_kv;
      for (int i = tid; i < RB * CH; i += NT) {
        const int row = i / CH, ch = i % CH, r = ld.rb * RB + row;
        const bool there = r < a.rows;
        const int tok = there ? r / a.group : 0, h = there ? r - tok * a.group : 0;
        cp16(to + 2 * S::kTileBytes + chunk_at<D>(row, ch),
             a.q + (size_t)b * a.q_batch + (size_t)tok * a.q_token + (size_t)(g * a.group + h) * a.q_head + ch * 16, there);
      }
    }
    ++ld_at;
    if (ld_at < hi) advance(ld, a.c, a.n_new, kTileKeys, blocks);
  };
#pragma unroll 1
  for (int s = 0; s < S::kStages - 1; ++s) {
    if (ld_at < hi) load();
    cp_commit();
  }

  uint32_t qf[D / 16][4];
  float o[D / 8][4];
  float m[2], l[2];
  RowOptions ro[2];
  int seg_first = 0;                                            // 1: the segment begins the item
  const int rowa = wr * 16 + (lane >> 2);                       // this thread's rows of the block: rowa, rowa + 8
#pragma unroll 1
  for (; at < hi; ++at) {
    const int stage = (int)((at - lo) % S::kStages);
    const uint32_t from = base + stage * S::kStage;
    unsigned char* const here = sm + stage * S::kStage;
    cp_wait<S::kStages - 2>();
    __syncthreads();
    if (ld_at < hi) load();
    cp_commit();
    if (cur.t == 0 || at == lo) {
      seg_first = cur.t == 0;
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk)
        ldsm(from + 2 * S::kTileBytes + chunk_at<D>(wr * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), kk * 2 + (lane >> 4)), qf[kk]);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
      m[0] = m[1] = -INFINITY;
      l[0] = l[1] = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x) ro[x] = row_options(a, cur.u, min(cur.rb * RB + rowa + 8 * x, a.rows - 1));
    }
    const int n_old = cur.keys - a.n_new, j0 = cur.t * kTileKeys + wk * KW;
    // products
    float s[NB][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
      for (int nb = 0; nb < NB; nb += 2) {
        uint32_t kf[4];
        ldsm(from + chunk_at<D>(wk * KW + nb * 8 + (lane >> 4) * 8 + (lane & 7), kk * 2 + ((lane >> 3) & 1)), kf);
        mma_16x8x16(s[nb], qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3], kf[0], kf[1]);
        mma_16x8x16(s[nb + 1], qf[kk][0], qf[kk][1], qf[kk][2], qf[kk][3], kf[2], kf[3]);
      }
    // x in bits
    const int* const kp = (const int*)(here + 2 * S::kTileBytes + S::kQBytes) + wk * KW;
    const bool tail = j0 + KW > n_old;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int jj = nb * 8 + (lane & 3) * 2 + (e & 1);
        float x = OPT ? biased(a, s[nb][e], ro[e >> 1], a.slopes ? kp[jj] : 0) : s[nb][e] * a.scale2;
        if (tail && (j0 + jj >= cur.keys || !sees(ro[e >> 1].seen, j0 + jj, n_old))) x = -INFINITY;
        s[nb][e] = x;
      }
    if (a.accumulate) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + nb * 8 + (lane & 3) * 2 + (e & 1), r = cur.rb * RB + rowa + 8 * (e >> 1);
          if (j < cur.keys && r < a.rows) a.logits[((size_t)cur.u * a.group + r) * a.c.capacity + j] = s[nb][e];
        }
    }
    // running maximum
    bool grown = false;
    float ref[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float t = -INFINITY;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) t = fmaxf(t, fmaxf(s[nb][2 * x], s[nb][2 * x + 1]));
      t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
      t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
      ref[x] = fmaxf(t, m[x]);
      grown |= ref[x] > m[x];
    }
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float f = m[x] == -INFINITY ? 0.f : fast_exp2(m[x] - ref[x]);
        l[x] *= f;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) { o[i][2 * x] *= f; o[i][2 * x + 1] *= f; }
        m[x] = ref[x];
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) ref[x] = m[x] == -INFINITY ? 0.f : m[x];
    uint32_t pf[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = fast_exp2(s[nb][e] - ref[e >> 1]);
      l[0] += p[0] + p[1];
      l[1] += p[2] + p[3];
      // p keeps 8 bits for the product, as V does; the sum l is of the unrounded values
      pf[nb][0] = bf16x2(p[0], p[1]);
      pf[nb][1] = bf16x2(p[2], p[3]);
    }
    // Where a new token's V is not finite, rows that do not see it must not meet it: 0 x infinity.
    bool plain = true;
    if (tail) {
      bool bad = false;
#pragma unroll 2
      for (int i = lane; i < KW * CH; i += 32) {
        const uint4 w = *(const uint4*)(here + S::kTileBytes + (wk * KW + i / CH) * (D * 2) + (i % CH) * 16);
        bad |= not_finite(w.x) || not_finite(w.y) || not_finite(w.z) || not_finite(w.w);
      }
      plain = !__any_sync(0xffffffffu, bad);
    }
    if (plain) {
#pragma unroll
      for (int nb = 0; nb < NB; nb += 2)
#pragma unroll
        for (int dn = 0; dn < D / 16; ++dn) {
          uint32_t vf[4];
          ldsm_t(from + S::kTileBytes + chunk_at<D>(wk * KW + nb * 8 + ((lane >> 3) & 1) * 8 + (lane & 7), dn * 2 + (lane >> 4)), vf);
          mma_16x8x16(o[2 * dn], pf[nb][0], pf[nb][1], pf[nb + 1][0], pf[nb + 1][1], vf[0], vf[1]);
          mma_16x8x16(o[2 * dn + 1], pf[nb][0], pf[nb][1], pf[nb + 1][0], pf[nb + 1][1], vf[2], vf[3]);
        }
    } else {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll 1
        for (int kk = 0; kk < 8; ++kk) {
          const int key = wk * KW + nb * 8 + kk;
          float p[2];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t w = __shfl_sync(0xffffffffu, pf[nb][x], (lane & ~3) | (kk >> 1));
            p[x] = __uint_as_float(kk & 1 ? w & 0xffff0000u : w << 16);
          }
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const uint32_t w = *(const uint32_t*)(here + S::kTileBytes + chunk_at<D>(key, i) + (lane & 3) * 4);
#pragma unroll
            for (int x = 0; x < 2; ++x)
              if (p[x] != 0.f) {
                o[i][2 * x] = fmaf(p[x], __uint_as_float(w << 16), o[i][2 * x]);
                o[i][2 * x + 1] = fmaf(p[x], __uint_as_float(w & 0xffff0000u), o[i][2 * x + 1]);
              }
          }
        }
    }

    const bool item_ends = cur.t + 1 == cur.tiles;
    if (item_ends || at + 1 == hi) {
      // the warps that share the keys: common maximum, then their outputs one after the other
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
        if ((lane & 3) == 0) {
          stat[wk * RB + rowa + 8 * x] = m[x];
          stat[(WK + wk) * RB + rowa + 8 * x] = l[x];
        }
      }
      __syncthreads();
      float f[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, stat[w * RB + rowa + 8 * x]);
        f[x] = m[x] == -INFINITY ? 0.f : fast_exp2(m[x] - M);
      }
#pragma unroll 1
      for (int w = 0; w < WK; ++w) {
        if (wk == w) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              float2* const to = (float2*)(merge + (rowa + 8 * x) * S::kMergeRow + i * 8 + (lane & 3) * 2);
              float2 v = make_float2(o[i][2 * x] * f[x], o[i][2 * x + 1] * f[x]);
              if (w > 0) { const float2 e = *to; v.x += e.x; v.y += e.y; }
              *to = v;
            }
        }
        __syncthreads();
      }
      const bool whole = seg_first && item_ends;
      const int slot = 2 * cta + seg_first;
      const int b = cur.u / a.c.n_kv, g = cur.u % a.c.n_kv;
      for (int i = tid; i < RB * (D / 4); i += NT) {
        const int row = i / (D / 4), c4 = i % (D / 4), r = cur.rb * RB + row;
        if (r >= a.rows) break;
        float M = -INFINITY, L = 0.f;
#pragma unroll
        for (int w = 0; w < WK; ++w) M = fmaxf(M, stat[w * RB + row]);
        if (M != -INFINITY)
#pragma unroll
          for (int w = 0; w < WK; ++w) L += stat[(WK + w) * RB + row] * fast_exp2(stat[w * RB + row] - M);
        const float4 v = *(const float4*)(merge + row * S::kMergeRow + c4 * 4);
        if (!whole) {
          *(float4*)(a.part_out + ((size_t)slot * RB + row) * D + c4 * 4) = v;
          if (c4 == 0) a.part_stat[(size_t)slot * RB + row] = make_float2(M, L);
          continue;
        }
        const int tok = r / a.group, h = r - tok * a.group;
        const size_t q = ((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h;
        const float inv = M == -INFINITY ? 0.f : 1.f / L;          // (a NaN row stays one)
        *(uint2*)(a.out + (q * D + c4 * 4) * 2) = make_uint2(bf16x2(v.x * inv, v.y * inv), bf16x2(v.z * inv, v.w * inv));
        if (c4 == 0) {
          const float bits = M == -INFINITY ? M : M + log2f(L);
          if (a.lse) a.lse[q] = bits * kLn2;
          if (a.accumulate) a.row_lse[(size_t)cur.u * a.rows + r] = bits;
        }
      }
      __syncthreads();
    }
    advance(cur, a.c, a.n_new, kTileKeys, blocks);
  }
}

// ---- weights of accepted tokens ------------------------------------------------------------------
// weights[j] = decay weights[j] + sum over accepted rows of 2^(x - lse): the accepted tokens' rows are the operand that stays
// (kWeighRows at a time), K tiles stream past them; a key belongs to one warp, which adds up its rows.
constexpr int kWeighRows = 64, kWeighStages = 4, kWeighWarps = 4;

template <int D>
constexpr int weigh_smem() { return kWeighStages * (kTileKeys * D * 2 + kTileKeys * 4) + kWeighRows * (D * 2 + 4 + sizeof(RowOptions)) + 128; }

template <int D, bool OPT>
__global__ void __launch_bounds__(kWeighWarps * 32, 2) weigh_mma(const __grid_constant__ AttendArgs a, const unsigned long long* __restrict__ accepted) {
  constexpr int NT = kWeighWarps * 32, CH = D / 8, kStage = kTileKeys * D * 2 + kTileKeys * 4;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 127u) & ~127u;
  unsigned char* const sm = smem_raw + (base - smem_u32(smem_raw));
  constexpr uint32_t kQ = kWeighStages * kStage;
  float* const lse = (float*)(sm + kQ + kWeighRows * D * 2);      // in bits, +inf: no row
  RowOptions* const opts = (RowOptions*)(lse + kWeighRows);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = blockIdx.x;
  pdl_trigger();
  pdl_wait();
  const WorkStart ws = find_work<NT>(a.c, a.n_new, kTileKeys, 1, [&](long long W) { return cut(cta, W, sharers(W, gridDim.x)); }, nullptr);
  const int C = sharers(ws.total, gridDim.x);
  const long long lo = cut(cta, ws.total, C), hi = cut(cta + 1, ws.total, C);
  if (lo >= hi) return;
  long long at = lo;
  Cursor cur;
  cur.u = ws.unit;
  enter(cur, a.c, a.n_new, kTileKeys);
  cur.rb = 0;
  cur.t = (int)(lo - ws.before);
#pragma unroll 1
  while (at < hi) {                                               // a unit's tiles of this CTA
    const int t0 = cur.t, t1 = (int)min((long long)cur.tiles, cur.t + (hi - at));
    const int b = cur.u / a.c.n_kv, g = cur.u % a.c.n_kv, n_old = cur.keys - a.n_new;
    const unsigned long long taken = accepted[b] & (a.n_new == 64 ? ~0ull : (1ull << a.n_new) - 1);
    const int rows = __popcll(taken) * a.group;
    float* const w = a.c.weights + (size_t)cur.u * a.c.capacity;
#pragma unroll 1
    for (int r0 = 0; r0 == 0 || r0 < rows; r0 += kWeighRows) {
      const int n_rows = min(kWeighRows, rows - r0), n_blocks = (n_rows + 15) / 16;
      __syncthreads();
      for (int i = tid; i < kWeighRows; i += NT) {
        float x = INFINITY;
        if (i < n_rows) {
          unsigned long long rest = taken;                        // token of row r0 + i: the bit of that rank
          for (int skip = (r0 + i) / a.group; skip > 0; --skip) rest &= rest - 1;
          const int tok = __ffsll((long long)rest) - 1, h = (r0 + i) % a.group;
          x = a.lse[((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h] * kLog2e;
          if (x == -INFINITY) x = INFINITY;                       // a row that saw nothing gave nothing
          opts[i] = row_options(a, cur.u, tok * a.group + h);
          const char* const src = a.q + (size_t)b * a.q_batch + (size_t)tok * a.q_token + (size_t)(g * a.group + h) * a.q_head;
#pragma unroll 4
          for (int ch = 0; ch < CH; ++ch) *(uint4*)(sm + kQ + chunk_at<D>(i, ch)) = *(const uint4*)(src + ch * 16);
        } else {
          for (int ch = 0; ch < CH; ++ch) *(uint4*)(sm + kQ + chunk_at<D>(i, ch)) = make_uint4(0, 0, 0, 0);
          opts[i] = RowOptions{0, 0.f, 0};
        }
        lse[i] = x;
      }
      auto load = [&](int t) {
        const uint32_t to = base + (t - t0) % kWeighStages * kStage;
        for (int i = tid; i < kTileKeys * CH; i += NT) {
          const int row = i / CH, ch = i % CH, j = t * kTileKeys + row;
          cp16(to + chunk_at<D>(row, ch), cur.k + (j < cur.keys ? (size_t)j * a.c.s_token + ch * 16 : 0), j < cur.keys);
        }
        if (OPT && a.slopes)
          for (int i = tid; i < kTileKeys; i += NT) {
            const int j = t * kTileKeys + i;
            cp4(to + kTileKeys * D * 2 + i * 4, a.c.positions + (size_t)cur.u * a.c.capacity + (j < cur.keys ? j : 0), j < cur.keys);
          }
      };
#pragma unroll 1
      for (int s = 0; s < kWeighStages - 1; ++s) {
        if (t0 + s < t1) load(t0 + s);
        cp_commit();
      }
#pragma unroll 1
      for (int t = t0; t < t1; ++t) {
        cp_wait<kWeighStages - 2>();
        __syncthreads();
        if (t + kWeighStages - 1 < t1) load(t + kWeighStages - 1);
        cp_commit();
        const int stage = (t - t0) % kWeighStages;
        const uint32_t from = base + stage * kStage;
        const int* const kp = (const int*)(sm + stage * kStage + kTileKeys * D * 2) + warp * 16;
        const int j0 = t * kTileKeys + warp * 16;
        const bool tail = j0 + 16 > n_old;
        float sum[2][2] = {{0.f, 0.f}, {0.f, 0.f}};               // of keys 8 nb + 2 (lane % 4) + e
#pragma unroll 1
        for (int rb = 0; rb < n_blocks; ++rb) {
          float s[2][4] = {};
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            uint32_t qf[4], kf[4];
            ldsm(base + kQ + chunk_at<D>(rb * 16 + ((lane >> 3) & 1) * 8 + (lane & 7), kk * 2 + (lane >> 4)), qf);
            ldsm(from + chunk_at<D>(warp * 16 + (lane >> 4) * 8 + (lane & 7), kk * 2 + ((lane >> 3) & 1)), kf);
            mma_16x8x16(s[0], qf[0], qf[1], qf[2], qf[3], kf[0], kf[1]);
            mma_16x8x16(s[1], qf[0], qf[1], qf[2], qf[3], kf[2], kf[3]);
          }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const int row = rb * 16 + (lane >> 2) + 8 * x;
            const float ref = lse[row];
            RowOptions ro{};
            if (OPT || tail) ro = opts[row];
#pragma unroll
            for (int nb = 0; nb < 2; ++nb)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const int jj = nb * 8 + (lane & 3) * 2 + e;
                float v = OPT ? biased(a, s[nb][2 * x + e], ro, a.slopes ? kp[jj] : 0) : s[nb][2 * x + e] * a.scale2;
                if (tail && (j0 + jj >= cur.keys || !sees(ro.seen, j0 + jj, n_old))) v = -INFINITY;
                sum[nb][e] += ref == INFINITY ? 0.f : fast_exp2(v - ref);
              }
          }
        }
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d *= 2) sum[nb][e] += __shfl_xor_sync(0xffffffffu, sum[nb][e], d);
          }
        // lane l < 16 has key l: nb = l / 8, l % 8 = 2 (source lane) + e
        float mine = 0.f;
#pragma unroll
        for (int nb = 0; nb < 2; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float v = __shfl_sync(0xffffffffu, sum[nb][e], (lane & 7) >> 1);
            if ((lane >> 3 & 1) == nb && (lane & 1) == e) mine = v;
          }
        if (lane < 16 && j0 + lane < cur.keys) {
          const float old = w[j0 + lane];
          w[j0 + lane] = (r0 == 0 ? a.decay * old : old) + mine;
        }
      }
    }
    at += t1 - t0;
    cur.t = t1 - 1;
    if (at < hi) advance(cur, a.c, a.n_new, kTileKeys, 1);
  }
}

template <int D, int WR, int WK, bool OPT>
cudaError_t launch_one(const AttendArgs& a, cudaStream_t st) {
  using S = AttendShape<D, WR, WK>;
  const cudaError_t e = allow_smem<attend_mma<D, WR, WK, OPT>>(S::kSmem);
  return e != cudaSuccess ? e : launch_pdl(attend_mma<D, WR, WK, OPT>, dim3(a.ctas), dim3(S::THREADS), S::kSmem, st, a);
}
template <int D, bool OPT>
cudaError_t launch_rows(const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  return p.rb == 16 ? launch_one<D, 1, 4, OPT>(a, st) : p.rb == 32 ? launch_one<D, 2, 4, OPT>(a, st) : launch_one<D, 4, 2, OPT>(a, st);
}
bool options(const AttendArgs& a) { return a.cap2 != 0.f || a.slopes; }

template <int D, bool OPT>
cudaError_t launch_weigh(const AttendArgs& a, const unsigned long long* accepted, int ctas, cudaStream_t st) {
  const cudaError_t e = allow_smem<weigh_mma<D, OPT>>(weigh_smem<D>());
  return e != cudaSuccess ? e : launch_pdl(weigh_mma<D, OPT>, dim3(ctas), dim3(kWeighWarps * 32), weigh_smem<D>(), st, a, accepted);
}

}  // namespace

cudaError_t launch_attend_mma(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  if (ctx.cfg.head_dim == 128) return options(a) ? launch_rows<128, true>(a, p, st) : launch_rows<128, false>(a, p, st);
  return options(a) ? launch_rows<64, true>(a, p, st) : launch_rows<64, false>(a, p, st);
}

cudaError_t launch_weigh_bf16(const Ctx& ctx, const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st) {
  const int ctas = 2 * ctx.sm_count;
  if (ctx.cfg.head_dim == 128) return options(a) ? launch_weigh<128, true>(a, accepted, ctas, st) : launch_weigh<128, false>(a, accepted, ctas, st);
  return options(a) ? launch_weigh<64, true>(a, accepted, ctas, st) : launch_weigh<64, false>(a, accepted, ctas, st);
}

}  // namespace skv
