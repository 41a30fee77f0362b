// Rotary positions on the device: angles, and 16-byte chunks of a head as pairs.
#pragma once

#include <cuda_fp8.h>

#include "attend.cuh"

namespace skv {

struct RopeArgs {
  int dim, interleaved;
  float amplitude;
  unsigned long long step[STRUCTKV_ROPE_MAX_DIM / 2];
};

#ifdef __CUDACC__

// position * step modulo one turn, in 2^-32 of it (signed: half a turn either way).
__device__ __forceinline__ int turn_of(unsigned long long step, int position) {
  const unsigned lo = (unsigned)step, p = (unsigned)position;
  return (int)(__umulhi(lo, p) + (unsigned)(step >> 32) * p - (position < 0 ? lo : 0u));
}
// Cosine and sine times the amplitude.  For bf16 by the special-function unit, whose 2^-21 is far below the 2^-9 of a rounding.
template <typename T>
__device__ __forceinline__ float2 cos_sin(int turn, float amplitude) {
  float s, c;
  if constexpr (sizeof(T) == 2) __sincosf((float)turn * 1.4629180792671596e-9f, &s, &c);   // 2 pi 2^-32
  else sincospif((float)turn * 4.656612873077393e-10f, &s, &c);                            // 2^-31
  return make_float2(c * amplitude, s * amplitude);
}

template <typename T>
struct Chunk {
  static constexpr int N = 16 / sizeof(T);                      // elements of 16 bytes, and pairs that a lane has of a row
};
__device__ __forceinline__ void widen(uint4 x, float (&f)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void widen(uint4 x, float (&f)[4]) {
  f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
}
__device__ __forceinline__ uint4 narrow(const float (&f)[8]) { return make_uint4(bf16x2(f[0], f[1]), bf16x2(f[2], f[3]), bf16x2(f[4], f[5]), bf16x2(f[6], f[7])); }
__device__ __forceinline__ uint4 narrow(const float (&f)[4]) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ void put(__nv_bfloat16* at, float x) { *at = __float2bfloat16(x); }
__device__ __forceinline__ void put(float* at, float x) { *at = x; }

// Where a row's N pairs from pair p0 on lie: two chunks of N elements at `a` and `b`, element i of one paired with element i of the other
// (apart), or pairs of neighbours.  Whole chunks of pairs are rotated or are not where dim is a multiple of 2 N; else element by element.
template <typename T>
struct PairPlace {
  static constexpr int N = Chunk<T>::N;
  int p0, a, b, half;
  bool apart, turned, whole;
  __device__ __forceinline__ PairPlace(int dim, bool interleaved, int p) {
    p0 = p;
    half = dim / 2;
    whole = dim % (2 * N) == 0;
    turned = p < half;
    apart = turned && !interleaved;
    a = apart ? p : 2 * p;
    b = apart ? p + half : 2 * p + N;
  }
  // elements of pair p0 + i
  __device__ __forceinline__ int2 pair(int i) const {
    const int p = p0 + i;
    return apart && p < half ? make_int2(p, p + half) : make_int2(2 * p, 2 * p + 1);
  }
  __device__ __forceinline__ bool turns(int i) const { return whole ? turned : p0 + i < half; }
};
// x: pairs as (u[i], v[i])
template <typename T>
__device__ __forceinline__ void split(const PairPlace<T>& at, const float (&x)[Chunk<T>::N], const float (&y)[Chunk<T>::N], float (&u)[Chunk<T>::N],
                                      float (&v)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    u[i] = at.apart ? x[i] : i < N / 2 ? x[(2 * i) % N] : y[(2 * i) % N];
    v[i] = at.apart ? y[i] : i < N / 2 ? x[(2 * i + 1) % N] : y[(2 * i + 1) % N];
  }
}
template <typename T>
__device__ __forceinline__ void join(const PairPlace<T>& at, const float (&u)[Chunk<T>::N], const float (&v)[Chunk<T>::N], float (&x)[Chunk<T>::N],
                                     float (&y)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = at.apart ? u[i] : i % 2 ? v[i / 2] : u[i / 2];
    y[i] = at.apart ? v[i] : i % 2 ? v[N / 2 + i / 2] : u[N / 2 + i / 2];
  }
}
template <typename T>
__device__ __forceinline__ void load_pairs(const PairPlace<T>& at, const T* row, float (&u)[Chunk<T>::N], float (&v)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
  if (at.whole) {
    float x[N], y[N];
    widen(*(const uint4*)(row + at.a), x);
    widen(*(const uint4*)(row + at.b), y);
    split<T>(at, x, y, u, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int2 e = at.pair(i);
      u[i] = value(row[e.x]);
      v[i] = value(row[e.y]);
    }
  }
}
template <typename T>
__device__ __forceinline__ void store_pairs(const PairPlace<T>& at, T* row, const float (&u)[Chunk<T>::N], const float (&v)[Chunk<T>::N]) {
  constexpr int N = Chunk<T>::N;
  if (at.whole) {
    float x[N], y[N];
    join<T>(at, u, v, x, y);
    *(uint4*)(row + at.a) = narrow(x);
    *(uint4*)(row + at.b) = narrow(y);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int2 e = at.pair(i);
      put(row + e.x, u[i]);
      put(row + e.y, v[i]);
    }
  }
}
__device__ __forceinline__ void turn(float& u, float& v, float2 cs) {
  const float x = u;
  u = fmaf(x, cs.x, -(v * cs.y));
  v = fmaf(v, cs.x, x * cs.y);
}

// Heads [h0, h1) of one token: this lane's N pairs of each, from pair p0 on.
template <typename T>
__device__ __forceinline__ void rotate_heads(const RopeArgs& r, bool inverse, const T* x, long long x_head, T* y, long long y_head, int position,
                                             int p0, int h0, int h1) {
  constexpr int N = Chunk<T>::N, U = 4;
  const PairPlace<T> at(r.dim, r.interleaved, p0);
  float2 cs[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    cs[i] = at.turns(i) ? cos_sin<T>(turn_of(r.step[min(p0 + i, STRUCTKV_ROPE_MAX_DIM / 2 - 1)], position), r.amplitude) : make_float2(1.f, 0.f);
    if (inverse) cs[i].y = -cs[i].y;
  }
#pragma unroll 1
  for (int h = h0; h < h1; h += U) {
    float u[U][N], v[U][N];
#pragma unroll
    for (int e = 0; e < U; ++e) load_pairs<T>(at, x + (long long)min(h + e, h1 - 1) * x_head, u[e], v[e]);
#pragma unroll
    for (int e = 0; e < U; ++e) {
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (at.turns(i)) turn(u[e][i], v[e][i], cs[i]);
      if (h + e < h1) store_pairs<T>(at, y + (long long)(h + e) * y_head, u[e], v[e]);
    }
  }
}

#endif  // __CUDACC__
}  // namespace skv
