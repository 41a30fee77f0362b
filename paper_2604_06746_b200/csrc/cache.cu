// Rows that come into a compacted cache, are moved in it, and go: append, commit, evict.
#include <algorithm>

#include "attend.cuh"
#include "radix.cuh"

namespace skv {
namespace {

// Rows of the new tokens to slots lengths[u] and up, with their positions and weight 0: gridDim.y blocks a unit take kAppend
// tokens each, in turn.  (One block a unit took 12 us for 128 units of 128 tokens.)
constexpr int kAppend = 16;
__global__ void __launch_bounds__(256) append(const __grid_constant__ CacheView c, const __grid_constant__ NewRows r, int n_new) {
  pdl_trigger();
  pdl_wait();
  const int u = blockIdx.x, n = unit_keys(c, u, n_new) - n_new, b = u / c.n_kv, g = u - b * c.n_kv;
  if (n < 0) return;
  const int per_row = c.row_bytes / 16, shift = per_row == 8 ? 3 : per_row == 16 ? 4 : 5;      // (64 or 128 elements of 2 or 4 bytes)
  const size_t off = unit_offset(c, u) + (size_t)n * c.s_token, from = (size_t)b * r.s_batch + (size_t)g * r.s_head;
  const size_t w = (size_t)u * c.capacity + n;
  for (int t0 = blockIdx.y * kAppend; t0 < n_new; t0 += gridDim.y * kAppend) {
    const int count = min(kAppend, n_new - t0);
#pragma unroll 4
    for (int i = threadIdx.x; i < count << (shift + 1); i += blockDim.x) {
      const int tok = t0 + (i >> (shift + 1)), ch = i & (per_row - 1);
      const bool is_v = i >> shift & 1;
      *(uint4*)((is_v ? c.v : c.k) + off + (size_t)tok * c.s_token + ch * 16) = *(const uint4*)((is_v ? r.v : r.k) + from + (size_t)tok * r.s_token + ch * 16);
    }
    if (threadIdx.x < count) {
      c.positions[w + t0 + threadIdx.x] = r.positions[(size_t)b * n_new + t0 + threadIdx.x];
      if (c.weights) c.weights[w + t0 + threadIdx.x] = 0.f;
    }
  }
}

// A block per unit: the accepted new tokens, path[0] < path[1] < ..., move to the first slots behind the old ones.  A thread has
// one 16-byte column of K or V (or the words) and goes through the rows in order, several at a time: path[i] >= i, so that a row
// that is still to be read is never written before.
__global__ void __launch_bounds__(256) commit(const __grid_constant__ CacheView c, int n_new, const int* __restrict__ counts,
                                              const int* __restrict__ path) {
  __shared__ int from[kMaxNew];
  __shared__ int bad;
  const int u = blockIdx.x, b = u / c.n_kv, tid = threadIdx.x;
  if (tid == 0) bad = 0;
  pdl_trigger();
  pdl_wait();
  const int n = unit_keys(c, u, n_new) - n_new, m = counts ? counts[b] : n_new;
  __syncthreads();
  if (path && tid < n_new && tid < m) {
    const int p = path[(size_t)b * n_new + tid];
    if (p < 0 || p >= n_new || (tid > 0 && p <= path[(size_t)b * n_new + tid - 1])) bad = 1;
    from[tid] = p;
  }
  if (tid == 0 && (m < 0 || m > n_new)) bad = 1;
  __syncthreads();
  if (n < 0) return;
  if (bad) {
    if (tid == 0) atomicCAS(c.status, 0, (int)STRUCTKV_ERR_INVALID_ARG);
    return;
  }
  if (path) {
    const size_t off = unit_offset(c, u) + (size_t)n * c.s_token, w = (size_t)u * c.capacity + n;
    const int per_row = c.row_bytes / 16;
    constexpr int kGo = 8;
    for (int i = tid; i < 2 * per_row; i += blockDim.x) {
      char* const col = (i < per_row ? c.k : c.v) + off + (size_t)(i % per_row) * 16;
      for (int r0 = 0; r0 < m; r0 += kGo) {
        uint4 x[kGo];
#pragma unroll
        for (int e = 0; e < kGo; ++e)
          if (r0 + e < m) x[e] = *(const uint4*)(col + (size_t)from[r0 + e] * c.s_token);
#pragma unroll
        for (int e = 0; e < kGo; ++e)
          if (r0 + e < m && from[r0 + e] != r0 + e) *(uint4*)(col + (size_t)(r0 + e) * c.s_token) = x[e];
      }
    }
    if (tid >= 192) {                                              // two warps: positions, weights; read before written
      int* const words = tid < 224 ? c.positions + w : (int*)c.weights + w;
      if (tid < 224 || c.weights) {
        const int lane = tid & 31;
        int x[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (lane + 32 * e < m) x[e] = words[from[lane + 32 * e]];
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (lane + 32 * e < m) words[lane + 32 * e] = x[e];
      }
    }
  }
  if (tid == 0) c.lengths[u] = n + m;
}

// A block per unit with more than `budget` tokens.  Kept are the budget first by (recent or not, weight, lower slot), recent:
// position above the newest less `recent`.  The kept tokens in slots from budget on move, in order, into the slots below it
// whose tokens go.  The two sets are disjoint, so that nothing is read after it was written, and a step that brought E tokens
// moves at most E rows, where a compaction in order would move up to `budget`.
//
// The threshold is found as in select.cu (radix.cuh); lists of both sets are taken kList entries at a time.
//
// Where one token goes, which is what a step of decoding asks for, there is no rank to search: it is the last of the lowest.
// A thread holds kItems tokens of a chunk: 8 where the capacity fits them or holds more than a chunk of 16, with two blocks an SM,
// else 16 with one.  (A unit of 8320 tokens was read anew for each level with 8.)  The code runs once a block, so that fetching it counts:
// the forms for one chunk and for many are compiled apart.
//
// A block goes through its steps once, each waiting for the one before: 128 units of 8320 tokens, 128 of which go, take 9.5 us (8.5 MB
// read, 8.4 MB moved: 3 at the copy bandwidth): words there 1.3, keys 1.2, rank 1.7, lists 2.0, rows 1.5, their words and the
// end 1.8; 256 units of 2049, one of which goes, 3.5.  A block a unit is a choice: a cluster of CTAs a unit, as select.cu has it, is not
// built.  Beyond 16384 tokens the words are read again for every level and for the lists: append, commit and eviction of 128 of 32896 for
// 128 units take 57 us (10.5 for the bytes), of 1 of 32769 for 64 units 14 (2.6).
constexpr int kList = 4096;
struct EvictShared {
  RadixShared<1> radix;
  unsigned counts[2][32];
  unsigned kept[16 * kRxThreads / 32];   // bits of a chunk's tokens
  int newest[32];
  unsigned low[2][32];
};

template <int kItems, bool kMany>
__global__ void __launch_bounds__(kRxThreads, kItems == 8 ? 2 : 1) evict(const __grid_constant__ CacheView c, int budget, int recent) {
  extern __shared__ __align__(16) unsigned char smem[];
  EvictShared& s = *reinterpret_cast<EvictShared*>(smem);
  int* const lists = reinterpret_cast<int*>(&s.radix);                // [2][kList], once the threshold is known
  static_assert(sizeof(RadixShared<1>) >= 2 * kList * sizeof(int), "the lists take the histograms' place");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, u = blockIdx.x;
  pdl_trigger();
  radix_clear(s.radix);
  pdl_wait();
  const int n = unit_keys(c, u, 0);
  if (n <= budget) return;
  const int* const pos = c.positions + (size_t)u * c.capacity;
  const float* const wt = c.weights + (size_t)u * c.capacity;
  constexpr int kChunk = kRxThreads * kItems;
  const int chunks = kMany ? (n + kChunk - 1) / kChunk : 1;           // more than one: the unit does not fit the registers
  unsigned key[kItems];
  int mine = 0, items = 0;
  // a warp's tokens are consecutive, as many for every warp; item e of this thread: first + 32 e
  auto token_of = [&](int ch) {
    items = min(kItems, (n - ch * kChunk + kRxThreads - 1) / kRxThreads);
    return ch * kChunk + warp * (32 * items) + lane;
  };
  int p[kItems];
  auto fetch = [&](int ch) {
    const int first = token_of(ch);
    mine = min(items, (n - first + 31) >> 5);
#pragma unroll
    for (int e = 0; e < kItems; ++e) {
      key[e] = e < mine ? __float_as_uint(wt[first + 32 * e]) : 0u;
      p[e] = e < mine ? pos[first + 32 * e] : -1;
    }
  };
  int newest = -1;
  for (int ch = 0; ch < chunks; ++ch) {
    fetch(ch);
#pragma unroll
    for (int e = 0; e < kItems; ++e) newest = max(newest, p[e]);
  }
  newest = __reduce_max_sync(0xffffffffu, newest);
  if (lane == 0) s.newest[warp] = newest;
  __syncthreads();
  newest = __reduce_max_sync(0xffffffffu, s.newest[lane]);
  const int line = newest - recent;                                   // (newest is -1 at least)
  // (a NaN weight, all bits set, comes below the recent ones)
  auto keys = [&] {
#pragma unroll
    for (int e = 0; e < kItems; ++e) key[e] = p[e] > line ? 0xffffffffu : min(order_key(__uint_as_float(key[e])), 0xfffffffeu);
  };
  auto load = [&](int ch) {
    fetch(ch);
    keys();
  };
  const size_t off = unit_offset(c, u);
  const int per_row = c.row_bytes / 16, row_shift = per_row == 8 ? 3 : per_row == 16 ? 4 : 5;
  if (chunks == 1) keys();
  if (n - budget == 1) {
    unsigned low = 0xffffffffu;
    int at = -1;
    for (int ch = 0; ch < chunks; ++ch) {
      if (chunks > 1) load(ch);
      const int first = token_of(ch);
#pragma unroll
      for (int e = 0; e < kItems; ++e)
        if (e < mine && key[e] <= low) {
          low = key[e];
          at = first + 32 * e;
        }
    }
    const unsigned low_warp = __reduce_min_sync(0xffffffffu, low);
    at = __reduce_max_sync(0xffffffffu, low == low_warp ? at : -1);
    if (lane == 0) {
      s.low[0][warp] = low_warp;
      s.low[1][warp] = (unsigned)at;
    }
    __syncthreads();
    if (warp != 0) return;
    low = s.low[0][lane];
    const unsigned lowest = __reduce_min_sync(0xffffffffu, low);
    at = __reduce_max_sync(0xffffffffu, low == lowest ? (int)s.low[1][lane] : -1);
    if (at != budget) {
      for (int i = lane; i < 2 << row_shift; i += 32) {
        char* const col = (i >> row_shift ? c.v : c.k) + off + (i & (per_row - 1)) * 16;
        *(uint4*)(col + (size_t)at * c.s_token) = *(const uint4*)(col + (size_t)budget * c.s_token);
      }
      if (lane == 0) {
        c.positions[(size_t)u * c.capacity + at] = pos[budget];
        c.weights[(size_t)u * c.capacity + at] = wt[budget];
      }
    }
    if (lane == 0) c.lengths[u] = budget;
    return;
  }
  unsigned thr = 0, remaining = (unsigned)budget, above = 0, need_eq = 0;
  int level = 0;
#pragma unroll 1
  for (; level < kRxLevels; ++level) {
    const unsigned mask = level == 0 ? 0u : 0xffffffffu << radix_shift(level - 1);
    for (int ch = 0; ch < chunks; ++ch) {
      if (chunks > 1) load(ch);
#pragma unroll
      for (int e = 0; e < kItems; ++e)
        if (e < items) radix_count(s.radix, level, radix_digit(key[e], level), e < mine && (key[e] & mask) == thr);
    }
    unsigned digit, in;
    radix_pick(s.radix, level, remaining, digit, in);
    thr |= digit << radix_shift(level);
    if (in == remaining) break;
  }
  above = level < kRxLevels ? thr - 1 : thr;
  need_eq = level < kRxLevels ? 0 : remaining;
  const unsigned below = (1u << lane) - 1u;

  // Entries [lo, lo + kList) of both lists, then their tokens.  Where the lists are longer, the last entries come first: the
  // tokens moved then lie above all that is still to be listed, and the copies that moved count as kept, equal ones before
  // the kept ones that remain, as many as were kept behind them.
  bool sized = false;
  for (int lo = 0; lo >= 0;) {
    __syncthreads();
    unsigned run_eq = 0, run_free = 0, run_move = 0;
    for (int ch = 0; ch < chunks; ++ch) {
      if (chunks > 1) load(ch);
      // this warp's tokens equal to the threshold, which decide by rank
      unsigned eq = 0;
      if (need_eq) {
#pragma unroll
        for (int e = 0; e < kItems; ++e)
          if (e < items) eq += __popc(__ballot_sync(0xffffffffu, e < mine && key[e] == thr));
        if (lane == 0) s.counts[0][warp] = eq;
        __syncthreads();
        const unsigned incl = warp_scan(s.counts[0][lane], lane);
        eq = run_eq + __shfl_sync(0xffffffffu, incl - s.counts[0][lane], warp);
        run_eq += __shfl_sync(0xffffffffu, incl, 31);
      }
      // a word for 32 tokens, by the warp that has them; then a thread a word
      // (this code runs once a launch: what bounds it is that it is fetched)
      token_of(ch);
#pragma unroll
      for (int e = 0; e < kItems; ++e) {
        if (e >= items) break;
        const unsigned bits = __ballot_sync(0xffffffffu, e < mine && key[e] > above);
        if (lane == 0) s.kept[warp * items + e] = bits;
      }
      if (need_eq) {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < kItems; ++e) {
          if (e >= items) break;
          const bool equal = e < mine && key[e] == thr;
          const unsigned be = __ballot_sync(0xffffffffu, equal), bits = __ballot_sync(0xffffffffu, equal && eq + __popc(be & below) < need_eq);
          eq += __popc(be);
          if (lane == 0) s.kept[warp * items + e] |= bits;
        }
      }
      __syncthreads();
      const int j0 = ch * kChunk + 32 * tid;
      auto under = [&](int line) { return line <= j0 ? 0u : line - j0 >= 32 ? 0xffffffffu : (1u << (line - j0)) - 1u; };
      unsigned fr = 0, mv = 0;
      if (tid < 32 * items) {
        const unsigned kept = s.kept[tid], low = under(budget);
        fr = under(n) & ~kept & low;
        mv = kept & ~low;
      }
      const unsigned both = __popc(fr) | __popc(mv) << 16, incl = warp_scan(both, lane);      // (a chunk has at most 2^14)
      if (lane == 31) s.counts[1][warp] = incl;
      __syncthreads();
      const unsigned of_warp = s.counts[1][lane], upto = warp_scan(of_warp, lane), all = __shfl_sync(0xffffffffu, upto, 31);
      const unsigned at = __shfl_sync(0xffffffffu, upto - of_warp, warp) + incl - both;
      unsigned fa = run_free + (at & 0xffffu) - lo, ma = run_move + (at >> 16) - lo;
      run_free += all & 0xffffu;
      run_move += all >> 16;
      for (; fr; fr &= fr - 1, ++fa)
        if (fa < (unsigned)kList) lists[fa] = j0 + __ffs(fr) - 1;
      for (; mv; mv &= mv - 1, ++ma)
        if (ma < (unsigned)kList) lists[kList + ma] = j0 + __ffs(mv) - 1;
      __syncthreads();
    }
    const int moves = (int)run_move;                                  // as many free slots as tokens to move
    if (!sized && moves > kList) {
      sized = true;
      lo = (moves - 1) / kList * kList;
      continue;
    }
    sized = true;
    const int here = min(kList, moves - lo);
    int* const to_pos = c.positions + (size_t)u * c.capacity;
    float* const to_wt = c.weights + (size_t)u * c.capacity;
    int p0 = 0;
    float w0 = 0.f;
    if (tid < here) {
      p0 = pos[lists[kList + tid]];
      w0 = wt[lists[kList + tid]];
    }
    constexpr int kGo = 4;
    for (int i0 = tid; i0 < here << (row_shift + 1); i0 += kGo * kRxThreads) {
      uint4 x[kGo];
      char* col[kGo];
#pragma unroll
      for (int e = 0; e < kGo; ++e) {
        const int i = i0 + e * kRxThreads, row = i >> (row_shift + 1);
        if (row < here) {
          col[e] = (i >> row_shift & 1 ? c.v : c.k) + off + (i & (per_row - 1)) * 16;
          x[e] = *(const uint4*)(col[e] + (size_t)lists[kList + row] * c.s_token);
          col[e] += (size_t)lists[row] * c.s_token;
        }
      }
#pragma unroll
      for (int e = 0; e < kGo; ++e)
        if ((i0 + e * kRxThreads) >> (row_shift + 1) < here) *(uint4*)col[e] = x[e];
    }
    if (tid < here) {
      to_pos[lists[tid]] = p0;
      to_wt[lists[tid]] = w0;
    }
    for (int i = tid + kRxThreads; i < here; i += kRxThreads) {
      to_pos[lists[i]] = pos[lists[kList + i]];
      to_wt[lists[i]] = wt[lists[kList + i]];
    }
    lo -= kList;
  }
  if (tid == 0) c.lengths[u] = budget;
}

}  // namespace

cudaError_t launch_append(const CacheView& c, const NewRows& r, int n_new, cudaStream_t st) {
  return launch_pdl(append, dim3(c.units, std::min((n_new + kAppend - 1) / kAppend, 64)), dim3(256), 0, st, c, r, n_new);
}
cudaError_t launch_commit(const CacheView& c, int n_new, const int* counts, const int* path, cudaStream_t st) {
  return launch_pdl(commit, dim3(c.units), dim3(256), 0, st, c, n_new, counts, path);
}
cudaError_t launch_evict(const CacheView& c, int budget, int recent, cudaStream_t st) {
  auto go = [&](auto kernel, cudaError_t e) {
    return e != cudaSuccess ? e : launch_pdl(kernel, dim3(c.units), dim3(kRxThreads), sizeof(EvictShared), st, c, budget, recent);
  };
  constexpr int kBytes = (int)sizeof(EvictShared);
  if (c.capacity <= 8 * kRxThreads) return go(evict<8, false>, allow_smem<evict<8, false>>(kBytes));
  if (c.capacity <= 16 * kRxThreads) return go(evict<16, false>, allow_smem<evict<16, false>>(kBytes));
  return go(evict<8, true>, allow_smem<evict<8, true>>(kBytes));
}

}  // namespace skv
