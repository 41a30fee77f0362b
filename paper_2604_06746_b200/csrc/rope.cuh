// Rotary positions on the device: angles, and 16-byte chunks of a head as pairs.
#pragma once

#include "attend.cuh"

namespace skv {

struct RopeArgs {
  int dim, interleaved;
  float amplitude;
  float off;                                                    // what a turned pair (a', b') is off by in fp32 at most, of |a'| + |b'|
  double amplitude64;
  unsigned long long step[STRUCTKV_ROPE_MAX_DIM / 2];
};

#ifdef __CUDACC__

// position * step modulo one turn, in 2^-32 of it (signed: half a turn either way).
__device__ __forceinline__ int turn_of(unsigned long long step, int position) {
  const unsigned lo = (unsigned)step, p = (unsigned)position;
  return (int)(__umulhi(lo, p) + (unsigned)(step >> 32) * p - (position < 0 ? lo : 0u));
}
// Cosine and sine of a turn, times the amplitude.  The nearest quarter goes first, in integers, so that what is left, r within an eighth of a turn,
// is exact to 24 bits; sin(2 pi r) = r S(r^2) and cos(2 pi r) = C(r^2) with polynomials fitted for the least largest error there (2^-28,
// relative, and 2^-34; least squares reweighted by the error until it is level: Lawson's method).  In fp32 both are off by 2^-23 at most.
// The special-function unit is off by 2^-21: that rounds one of some thousand bf16 queries to the other side.
__device__ __forceinline__ float2 cos_sin(int turn, float amplitude) {
  const unsigned quarter = ((unsigned)turn + 0x20000000u) >> 30;
  const float r = (float)(int)((unsigned)turn - (quarter << 30)) * 2.3283064365386963e-10f, z = r * r;   // 2^-32
  float s = fmaf(fmaf(fmaf(-75.39356f, z, 81.592354f), z, -41.34166145f), z, 6.283185287f) * (r * amplitude);
  float c = fmaf(fmaf(fmaf(fmaf(59.220406f, z, -85.44285f), z, 64.939316f), z, -19.73920865f), z, 1.f) * amplitude;
  const float x = quarter & 1 ? s : c;
  s = quarter & 1 ? c : s;
  c = __uint_as_float(__float_as_uint(x) ^ (quarter + 1 & 2) << 30);
  return make_float2(c, __uint_as_float(__float_as_uint(s) ^ (quarter & 2) << 30));
}

__device__ __forceinline__ void put(__nv_bfloat16* at, float x) { *at = __float2bfloat16(x); }
__device__ __forceinline__ void put(float* at, float x) { *at = x; }

// The same in 64 bits (Taylor's polynomials within an eighth of a turn, 2^-41).
__device__ __forceinline__ double2 cos_sin64(unsigned long long step, int position) {
  const double turn = (double)(long long)(step * (unsigned long long)(long long)position) * 0x1p-64, quarter = rint(4.0 * turn);
  const double x = fma(quarter, -0.25, turn) * 6.283185307179586, z = x * x;
  double s = 1.0 / 6227020800.0, c = 1.0 / 479001600.0;
  s = fma(s, z, -1.0 / 39916800.0); s = fma(s, z, 1.0 / 362880.0); s = fma(s, z, -1.0 / 5040.0); s = fma(s, z, 1.0 / 120.0); s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, -1.0 / 3628800.0); c = fma(c, z, 1.0 / 40320.0); c = fma(c, z, -1.0 / 720.0); c = fma(c, z, 1.0 / 24.0); c = fma(c, z, -0.5);
  s = fma(s * z, x, x);
  c = fma(c, z, 1.0);
  const int k = (int)quarter & 3;
  const double a = k & 1 ? s : c, b = k & 1 ? c : s;
  return make_double2(k + 1 & 2 ? -a : a, k & 2 ? -b : b);
}

// How a head's D elements form pairs for a lane that has N of them from pair p0 on, as two chunks of N elements at `a` and `b`:
// HALVES: element i of one with element i of the other, the pairs (c, c + dim / 2), and behind them, not turned, (c, c + (D - dim) / 2);
// NEIGHBOURS: pairs within a chunk; both where whole chunks are turned or are not (dim a multiple of 2 N).  SINGLE: element by element.
enum Pairing { HALVES, NEIGHBOURS, SINGLE };
inline __host__ __device__ Pairing pairing_of(const RopeArgs& r, int n) { return r.dim % (2 * n) ? SINGLE : r.interleaved ? NEIGHBOURS : HALVES; }

// A lane's chunks as they lie in memory (SINGLE: as whole pairs of neighbours would).
template <typename T, int N>
struct RawPairs {
  uint32_t x[N * sizeof(T) / 4], y[N * sizeof(T) / 4];
  RawPairs() = default;
  __device__ __forceinline__ RawPairs(const uint4& a, const uint4& b) : x{a.x, a.y, a.z, a.w}, y{b.x, b.y, b.z, b.w} {}
};

template <typename T, int D, Pairing P, int N>
struct PairPlace {
  using Raw = RawPairs<T, N>;
  static constexpr int W = N * sizeof(T) / 4;                   // words of a chunk
  int p0, a, b, half;
  bool apart;
  __device__ __forceinline__ PairPlace(const RopeArgs& r, int p) {
    p0 = p;
    half = r.dim / 2;
    apart = !r.interleaved;
    a = P == HALVES ? (p < half ? p : p + half) : 2 * p;
    b = P == HALVES ? (p < half ? p + half : p + D / 2) : 2 * p + N;
  }
  // SINGLE: elements of pair p0 + i
  __device__ __forceinline__ int2 pair(int i) const {
    const int p = p0 + i;
    return apart && p < half ? make_int2(p, p + half) : make_int2(2 * p, 2 * p + 1);
  }
  __device__ __forceinline__ bool turns(int i) const { return P == SINGLE ? p0 + i < half : p0 < half; }

  static __device__ __forceinline__ void load_chunk(const T* p, uint32_t (&w)[W]) {
    if constexpr (W == 4) {
      const uint4 v = *(const uint4*)p;
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint2 v = *(const uint2*)p;
      w[0] = v.x; w[1] = v.y;
    }
  }
  __device__ __forceinline__ Raw load(const T* row) const {
    Raw r;
    if constexpr (P != SINGLE) {
      load_chunk(row + a, r.x);
      load_chunk(row + b, r.y);
    } else {
      T x[N], y[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int2 e = pair(i);
        (i < N / 2 ? x : y)[(2 * i) % N] = row[e.x];
        (i < N / 2 ? x : y)[(2 * i + 1) % N] = row[e.y];
      }
      memcpy(r.x, x, sizeof(r.x));
      memcpy(r.y, y, sizeof(r.y));
    }
    return r;
  }
  static __device__ __forceinline__ float element(const uint32_t (&w)[W], int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
  static __device__ __forceinline__ void pairs(const Raw& r, float (&u)[N], float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      u[i] = P == HALVES ? element(r.x, i) : i < N / 2 ? element(r.x, 2 * i) : element(r.y, 2 * i - N);
      v[i] = P == HALVES ? element(r.y, i) : i < N / 2 ? element(r.x, 2 * i + 1) : element(r.y, 2 * i + 1 - N);
    }
  }
  // Pairs as chunks.
  static __device__ __forceinline__ void chunks(const float (&u)[N], const float (&v)[N], float (&x)[N], float (&y)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = P == HALVES ? u[i] : i % 2 ? v[i / 2] : u[i / 2];
      y[i] = P == HALVES ? v[i] : i % 2 ? v[N / 2 + i / 2] : u[N / 2 + i / 2];
    }
  }
  static __device__ __forceinline__ void store_chunk(T* p, const float (&x)[N]) {
    uint32_t w[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
      else w[i] = bf16x2(x[2 * i], x[2 * i + 1]);
    }
    if constexpr (W == 4) *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
    else *(uint2*)p = make_uint2(w[0], w[1]);
  }
  __device__ __forceinline__ void store(T* row, const float (&u)[N], const float (&v)[N]) const {
    if constexpr (P != SINGLE) {
      float x[N], y[N];
      chunks(u, v, x, y);
      store_chunk(row + a, x);
      store_chunk(row + b, y);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int2 e = pair(i);
        put(row + e.x, u[i]);
        put(row + e.y, v[i]);
      }
    }
  }
  // Cosines and sines of a position, two pairs to a word pair for the packed products; (1, 0) where nothing turns.  `step`: the rope's.
  __device__ __forceinline__ void angles(const RopeArgs& r, const unsigned long long* step, int position, bool inverse, uint64_t (&cos)[N / 2], uint64_t (&sin)[N / 2]) const {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float2 cs[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        cs[e] = turns(i + e) ? cos_sin(turn_of(step[min(p0 + i + e, D / 2 - 1)], position), r.amplitude) : make_float2(1.f, 0.f);
        if (inverse) cs[e].y = -cs[e].y;
      }
      cos[i / 2] = pack2(cs[0].x, cs[1].x);
      sin[i / 2] = pack2(cs[0].y, cs[1].y);
    }
  }
  // Turns the pairs (those that do not turn stay as they are, infinities and NaN among them).
  __device__ __forceinline__ void turn(float (&u)[N], float (&v)[N], const uint64_t (&cos)[N / 2], const uint64_t (&sin)[N / 2]) const {
    if (P != SINGLE && !turns(0)) return;
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const uint64_t x = pack2(u[i], u[i + 1]), y = pack2(v[i], v[i + 1]);
      float a0, a1, b0, b1;
      unpack2(fma2(x, cos[i / 2], mul2(y, sin[i / 2] ^ 0x8000000080000000ull)), a0, a1);
      unpack2(fma2(y, cos[i / 2], mul2(x, sin[i / 2])), b0, b1);
      if (turns(i)) { u[i] = a0; v[i] = b0; }
      if (turns(i + 1)) { u[i + 1] = a1; v[i + 1] = b1; }
    }
  }
};

// Heads [h0, h1) of one token: this lane's N pairs of each, from pair p0 on.  `step`: the rope's.
template <typename T, int D, Pairing P, int N>
__device__ __forceinline__ void rotate_heads(const RopeArgs& r, const unsigned long long* step, bool inverse, const T* x, long long x_head, T* y, long long y_head, int position,
                                             int p0, int h0, int h1) {
  constexpr int U = 2;
  using Place = PairPlace<T, D, P, N>;
  const Place at(r, p0);
  typename Place::Raw raw[U];
  auto load = [&](int h) {
#pragma unroll
    for (int e = 0; e < U; ++e) raw[e] = at.load(x + (long long)min(h + e, h1 - 1) * x_head);
  };
  load(h0);
  uint64_t cos[N / 2], sin[N / 2];
  at.angles(r, step, position, inverse, cos, sin);
#pragma unroll 1
  for (int h = h0; h < h1; h += U) {
#pragma unroll
    for (int e = 0; e < U; ++e) {
      float u[N], v[N];
      at.pairs(raw[e], u, v);
      at.turn(u, v, cos, sin);
      if (h + e < h1) at.store(y + (long long)(h + e) * y_head, u, v);
    }
    if (h + U < h1) load(h + U);
  }
}

// Runs L<storage type, elements of a head, pairing of a lane's n pairs>::run(args).
template <template <typename, int, Pairing> class L, typename T, int D, typename... Args>
inline cudaError_t by_dim(Pairing p, const Args&... args) {
  return p == SINGLE ? L<T, D, SINGLE>::run(args...) : p == HALVES ? L<T, D, HALVES>::run(args...) : L<T, D, NEIGHBOURS>::run(args...);
}
template <template <typename, int, Pairing> class L, typename... Args>
inline cudaError_t by_pairing(const Ctx& ctx, Pairing p, const Args&... args) {
  const bool bf16 = ctx.cfg.dtype == STRUCTKV_BF16, wide = ctx.cfg.head_dim == 128;
  if (bf16) return wide ? by_dim<L, __nv_bfloat16, 128>(p, args...) : by_dim<L, __nv_bfloat16, 64>(p, args...);
  return wide ? by_dim<L, float, 128>(p, args...) : by_dim<L, float, 64>(p, args...);
}

#endif  // __CUDACC__
}  // namespace skv
