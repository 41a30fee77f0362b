// Rotary positions applied to heads that stay in memory.
//
// A lane has the pairs of 16-byte chunks of a token's heads: their angles are worked out once for all heads that it takes, up to eight where there
// are enough lanes.  Reading and writing is the bound: 131072 tokens of 8 heads (537 MB both ways) 84 to 86 us, 6.3 TB/s, 96 to 98 % of a measured copy; 64
// tokens of 32 heads 3.1 to 3.6 us, a launch's latency.
#include "pages.cuh"

namespace skv {
namespace {

constexpr int kThreads = 256;

template <typename T, int D, Pairing P>
__global__ void __launch_bounds__(kThreads, 3) rotate(const __grid_constant__ RopeArgs r, const __grid_constant__ RotateArgs a) {
  constexpr int N = 16 / sizeof(T), LANES = D / (2 * N);
  __shared__ __align__(16) unsigned long long steps[D / 2];       // (lanes read different ones: from the arguments one after another)
  pdl_trigger();
  if (threadIdx.x < D / 2) steps[threadIdx.x] = r.step[threadIdx.x];
  __syncthreads();
  pdl_wait();
  const long long row = (long long)blockIdx.x * (kThreads / LANES) + threadIdx.x / LANES;
  const int h0 = blockIdx.y * a.head_step;
  if (row >= a.rows) return;
  const int b = quotient((int)row, a.by_tokens), i = (int)row - b * a.tokens;
  rotate_heads<T, D, P, N>(r, steps, a.inverse, (const T*)(a.x + b * a.x_batch + i * a.x_token), a.x_head / (int)sizeof(T),
                  (T*)(a.out + b * a.o_batch + i * a.o_token), a.o_head / (int)sizeof(T), a.positions[b * a.s_positions + i],
                  (threadIdx.x % LANES) * N, h0, min(h0 + a.head_step, a.heads));
}

template <typename T, int D, Pairing P>
struct Launch {
  static cudaError_t run(const RopeArgs& r, const RotateArgs& a, cudaStream_t st) {
    constexpr int PER = kThreads / (D * (int)sizeof(T) / 32);
    return launch_pdl(rotate<T, D, P>, dim3((unsigned)(((long long)a.rows + PER - 1) / PER), (a.heads + a.head_step - 1) / a.head_step), dim3(kThreads),
                      0, st, r, a);
  }
};

}  // namespace

cudaError_t launch_rotate(const Ctx& ctx, const RopeArgs& r, const RotateArgs& a, cudaStream_t st) {
  return by_pairing<Launch>(ctx, pairing_of(r, ctx.cfg.dtype == STRUCTKV_BF16 ? 8 : 4), r, a, st);
}

}  // namespace skv
