// Attention of new tokens over an fp32 cache on the CUDA cores, and the weight of accepted tokens.
//
// The one pass of attend_mma.cu in fp32: eight warps share a tile of 64 keys, eight each, and every warp takes all of the
// block's R rows (4 or 8).  Products: lane = (key, quarter of the head dimension), the quarters added by two shuffles; output:
// lane = D / 32 columns, the probabilities by shuffle.  K and V are read from shared memory once a block of rows.
// us, 32 heads over 8, d 128 (floor of the bytes): single tokens over 16 x 16384 keys 452 (335), over 4 x 4096 41 (21); 8 tokens over 4 x 4096
// 207 (21; four blocks of rows, each of which goes through K and V), 64 tokens 1450 (23; 32 blocks; at the fp32 rate of 148 SMs, 74
// TFLOP/s, the arithmetic is 236).  8 tokens: bound by waiting, with two warps a scheduler that issue in 44 % of the clocks; shared memory's
// pipe is busy half of the time (every warp reads all of the block's rows of Q for every eight keys), FMA a fifth, DRAM 15 %.
#include <algorithm>

#include "attend.cuh"

namespace skv {
namespace {

constexpr int kTileKeys = 64, kWarps = 8, kThreads = kWarps * 32;

__device__ __forceinline__ void cp16(float* dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Rows of K are padded so that the eight lanes of a 16-byte access phase, two keys of four quarters each, are in different banks.
template <int D>
struct Shape {
  static constexpr int kRow = D + 16, kStages = D == 128 ? 2 : 4;
  static constexpr int kStage = kTileKeys * kRow + kTileKeys * D;     // floats
  template <int R>
  static constexpr int kSmem = (kStages * kStage + R * D + kWarps * R * (D + 2)) * 4;
};

template <int D>
__device__ __forceinline__ void load_tile(float* to, const char* k, const char* v, long long s_token, int j0, int keys) {
  constexpr int CH = D / 4;
  for (int i = threadIdx.x; i < kTileKeys * CH; i += kThreads) {
    const int row = i / CH, ch = i % CH;
    const bool there = j0 + row < keys;
    const size_t off = there ? (size_t)(j0 + row) * s_token + ch * 16 : 0;
    cp16(to + row * Shape<D>::kRow + ch * 4, k + off, there);
    if (v) cp16(to + kTileKeys * Shape<D>::kRow + row * D + ch * 4, v + off, there);
  }
}
// s[r] = q[r] . k for this lane's key (lane / 4), in all four lanes of the key.
template <int D, int R>
__device__ __forceinline__ void products(const float* q, const float* k, int lane, float (&s)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r) s[r] = 0.f;
  const float* const kr = k + (lane >> 2) * Shape<D>::kRow + (lane & 3) * 4;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) {
    const float4 kv = *(const float4*)(kr + i * 16);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const float4 qv = *(const float4*)(q + r * D + i * 16 + (lane & 3) * 4);
      s[r] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, s[r]))));
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    s[r] += __shfl_xor_sync(0xffffffffu, s[r], 1);
    s[r] += __shfl_xor_sync(0xffffffffu, s[r], 2);
  }
}

template <int D, int R>
__global__ void __launch_bounds__(kThreads, 1) attend_simt(const __grid_constant__ AttendArgs a) {
  using S = Shape<D>;
  constexpr int DL = D / 32;                                          // output columns of a lane
  extern __shared__ __align__(16) float sm[];
  float* const qs = sm + S::kStages * S::kStage;
  float* const part = qs + R * D;                                     // [warp][R][D], then [warp][R] maxima and sums
  float* const stat = part + kWarps * R * D;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, blocks = (a.rows + R - 1) / R;
  pdl_trigger();
  pdl_wait();
  const WorkStart ws = find_work(a, 6, blocks, blockIdx.x == 0 ? a.unit_start : nullptr);
#pragma unroll 1
  for (Segments sg = first_segment(a, ws, 6, blocks); sg.t1; next_segment(sg, a, 6, blocks)) {   // the tiles of an item in this CTA
    const int u = sg.u, rb = sg.rb, keys = sg.keys, t0 = sg.t0, t1 = sg.t1;
    const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, n_old = keys - a.n_new;
    const char *const k = a.c.k + unit_offset(a.c, u), *const v = a.c.v + unit_offset(a.c, u);
    __syncthreads();
#pragma unroll 1
    for (int s = 0; s < S::kStages - 1; ++s) {
      if (t0 + s < t1) load_tile<D>(sm + s * S::kStage, k, v, a.c.s_token, (t0 + s) * kTileKeys, keys);
      cp_commit();
    }
    for (int i = tid; i < R * D; i += kThreads) {
      const int r = rb * R + i / D;
      float x = 0.f;
      if (r < a.rows) x = *(const float*)(a.q + (size_t)b * a.q_batch + (size_t)(r / a.group) * a.q_token +
                                          (size_t)(g * a.group + r % a.group) * a.q_head + (i % D) * 4);
      qs[i] = x;
    }
    RowOptions ro[R];
    float m[R], l[R], o[R][DL];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      ro[r] = row_options(a, u, min(rb * R + r, a.rows - 1));
      m[r] = -INFINITY;
      l[r] = 0.f;
#pragma unroll
      for (int c = 0; c < DL; ++c) o[r][c] = 0.f;
    }
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      cp_wait<S::kStages - 2>();
      __syncthreads();
      if (t + S::kStages - 1 < t1)
        load_tile<D>(sm + (t + S::kStages - 1 - t0) % S::kStages * S::kStage, k, v, a.c.s_token, (t + S::kStages - 1) * kTileKeys, keys);
      cp_commit();
      const float* const ks = sm + (t - t0) % S::kStages * S::kStage + warp * 8 * S::kRow;
      const float* const vs = sm + (t - t0) % S::kStages * S::kStage + kTileKeys * S::kRow + warp * 8 * D;
      float s[R];
      products<D, R>(qs, ks, lane, s);
      const int j = t * kTileKeys + warp * 8 + (lane >> 2);
      const int kp = a.slopes && j < keys ? a.c.positions[(size_t)u * a.c.capacity + j] : 0;
#pragma unroll
      for (int r = 0; r < R; r += 2) in_bits2(a, s[r], s[r + 1]);
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float x = biased(a, s[r], ro[r], kp);
        if (j >= keys || !sees(ro[r].seen, j, n_old)) x = -INFINITY;
        if (a.accumulate && (lane & 3) == 0 && j < keys && rb * R + r < a.rows)
          a.logits[((size_t)u * a.c.capacity + j) * a.group + rb * R + r] = x;
        float top = x;
#pragma unroll
        for (int d = 4; d < 32; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        if (top > m[r]) {                                             // (the same in every lane)
          const float f = m[r] == -INFINITY ? 0.f : fast_exp2(m[r] - top);
          l[r] *= f;
#pragma unroll
          for (int c = 0; c < DL; ++c) o[r][c] *= f;
          m[r] = top;
        }
        s[r] = fast_exp2(x - (m[r] == -INFINITY ? 0.f : m[r]));
        l[r] += s[r];                                                 // (each key in four lanes)
        // nothing that is seen weighs zero: V that is not finite reaches the row, however small its probability
        float least = x == -INFINITY ? 0.f : 1e-45f;
        asm("max.NaN.f32 %0, %0, %1;" : "+f"(s[r]) : "f"(least));
      }
#pragma unroll
      for (int jj = 0; jj < 8; ++jj) {
        float vv[DL];
#pragma unroll
        for (int c = 0; c < DL; ++c) vv[c] = vs[jj * D + c * 32 + lane];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float p = __shfl_sync(0xffffffffu, s[r], jj * 4);
          if (p != 0.f)                                               // (0 x infinity: a row must not meet what it does not see)
#pragma unroll
            for (int c = 0; c < DL; ++c) o[r][c] = fmaf(p, vv[c], o[r][c]);
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
      for (int d = 4; d < 32; d *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
      if (lane == 0) { stat[r * kWarps + warp] = m[r]; stat[(R + r) * kWarps + warp] = l[r]; }
#pragma unroll
      for (int c = 0; c < DL; ++c) part[(warp * R + r) * D + c * 32 + lane] = o[r][c];
    }
    leave_partial<D, kThreads, R, D, kWarps>(a, u * blocks + rb + blockIdx.x, min(R, a.rows - rb * R), part, stat, stat + kWarps * R, kWarps,
                                             tid, [] { __syncthreads(); });
  }
}

// weights[j] = decay weights[j] + sum over accepted rows of 2^(x - lse), eight rows at a time over the same keys (a weight is
// rounded once for every eight: its rows' sum is not kept anywhere else).  A tile is waited for as soon as it is asked for: 4 of 8
// tokens over 4 x 4096 keys, 32 heads over 8, take 92 us (10.6 for the bytes), 8 of 64 176.
template <int D>
__global__ void __launch_bounds__(kThreads, 1) weigh_simt(const __grid_constant__ AttendArgs a, const unsigned long long* __restrict__ accepted) {
  using S = Shape<D>;
  constexpr int R = 8;
  extern __shared__ __align__(16) float sm[];
  float* const qs = sm + kTileKeys * S::kRow;
  __shared__ float lse[R];
  __shared__ int row_of[R];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  pdl_trigger();
  pdl_wait();
  const WorkStart ws = find_work(a, 6, 1, nullptr);
#pragma unroll 1
  for (Segments sg = first_segment(a, ws, 6, 1); sg.t1; next_segment(sg, a, 6, 1)) {
    const int u = sg.u, keys = sg.keys, t0 = sg.t0, t1 = sg.t1;
    const int b = quotient(u, a.by_kv), g = u - b * a.c.n_kv, n_old = keys - a.n_new;
    const unsigned long long taken = accepted[b] & (a.n_new == 64 ? ~0ull : (1ull << a.n_new) - 1);
    const int rows = __popcll(taken) * a.group;
    float* const w = a.c.weights + (size_t)u * a.c.capacity;
#pragma unroll 1
    for (int r0 = 0; r0 == 0 || r0 < rows; r0 += R) {
      __syncthreads();
      if (tid < R) {
        int r = -1;
        float x = INFINITY;                                           // no row
        if (r0 + tid < rows) {
          unsigned long long rest = taken;
          const int rank = quotient(r0 + tid, a.by_group), h = r0 + tid - rank * a.group;
          for (int skip = rank; skip > 0; --skip) rest &= rest - 1;
          const int tok = __ffsll((long long)rest) - 1;
          r = tok * a.group + h;
          x = a.lse[((size_t)b * a.n_new + tok) * (a.group * a.c.n_kv) + g * a.group + h] * kLog2e;
          if (x == -INFINITY) x = INFINITY;                           // a row that saw nothing gave nothing
        }
        row_of[tid] = r;
        lse[tid] = x;
      }
      __syncthreads();
      for (int i = tid; i < R * D; i += kThreads) {
        const int r = row_of[i / D];
        qs[i] = r < 0 ? 0.f : *(const float*)(a.q + (size_t)b * a.q_batch + (size_t)(r / a.group) * a.q_token +
                                              (size_t)(g * a.group + r % a.group) * a.q_head + (i % D) * 4);
      }
      RowOptions ro[R];
#pragma unroll
      for (int r = 0; r < R; ++r) ro[r] = row_options(a, u, max(row_of[r], 0));
#pragma unroll 1
      for (int t = t0; t < t1; ++t) {
        __syncthreads();
        load_tile<D>(sm, a.c.k + unit_offset(a.c, u), nullptr, a.c.s_token, t * kTileKeys, keys);
        cp_commit();
        cp_wait<0>();
        __syncthreads();
        float s[R], sum = 0.f;
        products<D, R>(qs, sm + warp * 8 * S::kRow, lane, s);
        const int j = t * kTileKeys + warp * 8 + (lane >> 2);
        const int kp = a.slopes && j < keys ? a.c.positions[(size_t)u * a.c.capacity + j] : 0;
#pragma unroll
        for (int r = 0; r < R; r += 2) in_bits2(a, s[r], s[r + 1]);
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (lse[r] != INFINITY && sees(ro[r].seen, j, n_old)) sum += fast_exp2(biased(a, s[r], ro[r], kp) - lse[r]);
        if ((lane & 3) == 0 && j < keys) w[j] = (r0 == 0 ? a.decay * w[j] : w[j]) + sum;
      }
    }
  }
}

template <int D, int R>
cudaError_t launch_one(const AttendArgs& a, cudaStream_t st) {
  const cudaError_t e = allow_smem<attend_simt<D, R>>(Shape<D>::template kSmem<R>);
  return e != cudaSuccess ? e : launch_pdl(attend_simt<D, R>, dim3(a.ctas), dim3(kThreads), Shape<D>::template kSmem<R>, st, a);
}
template <int D>
cudaError_t launch_weigh(const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st) {
  constexpr int smem = (kTileKeys * Shape<D>::kRow + 8 * D) * 4;
  static_assert(smem <= 48 * 1024, "no limit to raise");
  return launch_pdl(weigh_simt<D>, dim3(a.ctas), dim3(kThreads), smem, st, a, accepted);
}

}  // namespace

cudaError_t launch_attend_simt(const Ctx& ctx, const AttendArgs& a, const AttendPlan& p, cudaStream_t st) {
  if (ctx.cfg.head_dim == 128) return p.rb == 4 ? launch_one<128, 4>(a, st) : launch_one<128, 8>(a, st);
  return p.rb == 4 ? launch_one<64, 4>(a, st) : launch_one<64, 8>(a, st);
}
cudaError_t launch_weigh_fp32(const Ctx& ctx, const AttendArgs& a, const unsigned long long* accepted, cudaStream_t st) {
  return ctx.cfg.head_dim == 128 ? launch_weigh<128>(a, accepted, st) : launch_weigh<64>(a, accepted, st);
}

}  // namespace skv
