// C ABI of decoding over a compacted cache: argument validation and dispatch.
#include <algorithm>
#include <cmath>

#include "attend.cuh"

using namespace skv;

namespace skv {
namespace {

// tcgen05's tiles have 128 rows, attend_mma's 16 at most: from 17 rows on the former takes them (single tokens of 17 heads and more stay,
// 16 at a time, with the kernel that leaves the logits).  us, attend_mma / attend_tc over 1 x 2048, 4 x 4096 and 8 x 8192 keys:
//   32 heads over 8, d 128: 16 rows 12.2 / 12.7, 17.0 / 23.3, 45.4 / 53.5; 20 rows 13.1 / 12.9, 23.7 / 23.4, 71 / 54; 32 rows 13.5 / 13.0,
//   26.3 / 22.9, 73 / 54.  16 over 8: 16 rows 13.2 / 12.7, 17.9 / 23.8, 45.3 / 53.2; 18 rows 14.1 / 13.0, 25.7 / 24.2, 71 / 54.
//   28 over 4, d 128: 14 rows 12.9 / 12.2, 14.0 / 17.6, 27.2 / 34.4; 21 rows 11.8 / 12.3, 16.7 / 17.6, 39.8 / 35.6.
//   32 over 8, d 64: 16 rows 9.4 / 11.3, 12.0 / 20.5, 26.4 / 45.4; 20 rows 9.5 / 11.3, 16.3 / 20.0, 43.9 / 45.6; 32 rows 10.1 / 11.2,
//   17.6 / 20.1, 45.8 / 45.5: d 64 loses by the rule from 17 to 32 rows, by up to a fifth over few keys.
bool by_tensor_cores(const structkv_config& cfg, int n_new) {
  return cfg.dtype == STRUCTKV_BF16 && n_new > 1 && cfg.n_q_heads / cfg.n_kv_heads * n_new > 16;
}
AttendPlan attend_plan(const structkv_config& cfg, int n_new, int sms) {
  const int rows = cfg.n_q_heads / cfg.n_kv_heads * n_new;
  if (cfg.dtype == STRUCTKV_FP32) return {rows <= 4 ? 4 : 8, 64, sms, 1, 1};
  if (by_tensor_cores(cfg, n_new)) return rows <= 128 ? AttendPlan{128, 128, sms, 2, 1} : AttendPlan{256, 128, sms, 1, 0};
  return {rows <= 8 ? 8 : 16, 64, sms, 1, rows <= 8 ? 1 : 0};
}

struct AttendWs { int* unit_start; float2* part_stat; float *part_out, *logits; size_t bytes; };
AttendWs carve_attend(const structkv_config& cfg, const AttendPlan& p, int batch, int n_new, int capacity, void* base) {
  AttendWs w{};
  char* at = (char*)base;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    void* r = at ? (void*)(at + off) : nullptr;
    off += align_up(bytes, 256);
    return r;
  };
  const size_t units = (size_t)batch * cfg.n_kv_heads, group = cfg.n_q_heads / cfg.n_kv_heads;
  w.unit_start = (int*)take((units + 1) * sizeof(int));
  const size_t slots = (units * ((group * n_new + p.rb - 1) / p.rb) + p.ctas) * p.parts;
  w.part_stat = (float2*)take(slots * p.rb * sizeof(float2));
  w.part_out = (float*)take(slots * p.rb * cfg.head_dim * sizeof(float));
  if (n_new == 1) w.logits = (float*)take(units * group * capacity * sizeof(float));
  w.bytes = off;
  return w;
}

// (units are counted in 31 bits)
bool sizes_ok(const structkv_config& cfg, int batch, int n_new, int capacity) {
  return batch >= 1 && capacity >= 1 && capacity <= 1 << 30 && n_new >= 0 && n_new <= capacity && (long long)batch * cfg.n_kv_heads <= 0x3fffffffll;
}
// What lays out tiles of new tokens' rows, attend and weigh: these and the tiles of all units are counted in 31 bits as well.
bool tiles_ok(const structkv_config& cfg, int batch, int n_new, int capacity) {
  const long long units = (long long)batch * cfg.n_kv_heads, rows = (long long)cfg.n_q_heads / cfg.n_kv_heads * n_new;
  return units * rows <= 0x3fffffffll && units * ((rows + 3) / 4) <= 0x7fffffffll / (capacity / 64 + 1 + kOverKeys / 64);
}
bool strides_ok(int elem, long long a, long long b, long long c) { return (a * elem) % 16 == 0 && (b * elem) % 16 == 0 && (c * elem) % 16 == 0; }

// False: not a cache of this context's shape.
bool view_of(const structkv_ctx* ctx, const structkv_cache* cache, int n_new, CacheView* v) {
  if (!ctx || !cache || !cache->k || !cache->v || !cache->positions || !cache->lengths) return false;
  const structkv_config& cfg = ctx->c.cfg;
  const int elem = cfg.dtype == STRUCTKV_BF16 ? 2 : 4;
  if (!sizes_ok(cfg, cache->batch, n_new, cache->capacity)) return false;
  if (((uintptr_t)cache->k | (uintptr_t)cache->v) % 16 || ((uintptr_t)cache->positions | (uintptr_t)cache->weights | (uintptr_t)cache->lengths) % 4)
    return false;
  if (!strides_ok(elem, cache->stride_batch, cache->stride_head, cache->stride_token)) return false;
  if (std::max({cache->stride_batch, cache->stride_head, cache->stride_token}) >= 1ll << 37) return false;   // (a tensor map's limit: 2^40 bytes)
  if ((cache->capacity > 1 && cache->stride_token < cfg.head_dim) || (cfg.n_kv_heads > 1 && cache->stride_head < cfg.head_dim) ||
      (cache->batch > 1 && cache->stride_batch < cfg.head_dim))
    return false;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev != ctx->c.device) return false;
  *v = CacheView{(char*)cache->k, (char*)cache->v, cache->stride_batch * elem, cache->stride_head * elem, cache->stride_token * elem,
                 cache->positions, cache->weights, cache->lengths, cache->batch * cfg.n_kv_heads, cfg.n_kv_heads, cache->capacity,
                 cfg.head_dim * elem, ctx->c.ws.status};
  return true;
}
bool rows_of(const structkv_ctx* ctx, const structkv_new_rows* r, NewRows* out) {
  const int elem = ctx->c.cfg.dtype == STRUCTKV_BF16 ? 2 : 4;
  if (!r || !r->k || !r->v || !r->positions || ((uintptr_t)r->k | (uintptr_t)r->v) % 16 || (uintptr_t)r->positions % 4) return false;
  if (!strides_ok(elem, r->stride_batch, r->stride_token, r->stride_head)) return false;
  *out = NewRows{(const char*)r->k, (const char*)r->v, r->stride_batch * elem, r->stride_token * elem, r->stride_head * elem, r->positions};
  return true;
}
// What attend and weigh have in common.
bool args_of(const structkv_ctx* ctx, const structkv_cache* cache, const structkv_attend_args* x, AttendArgs* a) {
  const structkv_config& cfg = ctx->c.cfg;
  const int elem = cfg.dtype == STRUCTKV_BF16 ? 2 : 4;
  if (x->n_new < 1 || x->n_new > kMaxNew || !tiles_ok(cfg, cache->batch, x->n_new, cache->capacity)) return false;
  if (!x->q || (uintptr_t)x->q % 16 || !strides_ok(elem, x->q_stride_batch, x->q_stride_token, x->q_stride_head)) return false;
  if (!std::isfinite(x->scale) || !std::isfinite(x->softcap) || x->softcap < 0.f || !std::isfinite(x->decay)) return false;
  if ((uintptr_t)x->slopes % 4 || (uintptr_t)x->tree % 8 || (uintptr_t)x->lse % 4) return false;
  // A cap beyond 2^100 |scale| caps nothing: tanh(y) is y to 24 bits for products of q and k below 2^88, and scale / softcap, or y, would lose
  // bits below the smallest normal number.
  const float softcap = x->softcap > 0x1p100f * std::fabs(x->scale) ? 0.f : x->softcap;
  const float inv = softcap > 0.f ? x->scale / softcap : 0.f, cap2 = softcap * kLog2e;
  if (!std::isfinite(inv) || !std::isfinite(cap2) || !std::isfinite(x->scale * kLog2e)) return false;
  a->q = (const char*)x->q;
  a->q_batch = x->q_stride_batch * elem;
  a->q_token = x->q_stride_token * elem;
  a->q_head = x->q_stride_head * elem;
  a->n_new = x->n_new;
  a->group = cfg.n_q_heads / cfg.n_kv_heads;
  a->rows = a->group * x->n_new;
  a->by_kv = div_by(cfg.n_kv_heads);
  a->by_group = div_by(a->group);
  a->by_rows = div_by(a->rows);
  a->scale2 = x->scale * kLog2e;
  a->cap2 = cap2;
  a->inv_cap = inv;
  a->slopes = x->slopes;
  a->tree = x->tree;
  a->decay = x->decay;
  a->lse = x->lse;
  return true;
}
structkv_status told(cudaError_t e) { return e == cudaSuccess ? STRUCTKV_OK : STRUCTKV_ERR_CUDA; }

}  // namespace
}  // namespace skv

extern "C" {

structkv_status structkv_append(structkv_ctx* ctx, const structkv_cache* cache, const structkv_new_rows* rows, int n_new, void* stream) {
  CacheView v;
  NewRows r;
  if (n_new < 1 || !view_of(ctx, cache, n_new, &v) || !rows_of(ctx, rows, &r)) return STRUCTKV_ERR_INVALID_ARG;
  return told(launch_append(v, r, n_new, (cudaStream_t)stream));
}

size_t structkv_attend_workspace_bytes(const structkv_config* cfg, int batch, int n_new, int capacity) {
  if (structkv_workspace_bytes(cfg) == 0 || n_new < 1 || n_new > kMaxNew || !sizes_ok(*cfg, batch, n_new, capacity) ||
      !tiles_ok(*cfg, batch, n_new, capacity))
    return 0;
  return carve_attend(*cfg, attend_plan(*cfg, n_new, kMaxSms), batch, n_new, capacity, nullptr).bytes;
}

structkv_status structkv_attend(structkv_ctx* ctx, const structkv_cache* cache, const structkv_attend_args* args, void* stream) {
  AttendArgs a{};
  NewRows r;
  if (!args || !view_of(ctx, cache, args->n_new, &a.c) || !args_of(ctx, cache, args, &a)) return STRUCTKV_ERR_INVALID_ARG;
  if (!args->out || (uintptr_t)args->out % 16 || (args->rows && !rows_of(ctx, args->rows, &r))) return STRUCTKV_ERR_INVALID_ARG;
  if (args->accumulate && !cache->weights) return STRUCTKV_ERR_INVALID_ARG;
  if (args->accumulate && args->n_new > 1) return STRUCTKV_ERR_UNSUPPORTED;
  const Ctx& c = ctx->c;
  const AttendPlan plan = attend_plan(c.cfg, args->n_new, std::min(c.sm_count, kMaxSms));
  const AttendWs w = carve_attend(c.cfg, plan, cache->batch, args->n_new, cache->capacity, args->workspace);
  if (!args->workspace || args->workspace_bytes < w.bytes || (uintptr_t)args->workspace % 256) return STRUCTKV_ERR_WORKSPACE;
  const bool tc = by_tensor_cores(c.cfg, args->n_new);
  a.out = (char*)args->out;
  a.accumulate = args->accumulate != 0;
  a.unit_start = w.unit_start;
  a.part_stat = w.part_stat;
  a.part_out = w.part_out;
  a.logits = w.logits;
  a.ctas = plan.ctas;
  a.by_ctas = div_by(plan.ctas);
  a.least = plan.least;
  a.over = kOverKeys / plan.tile;
  cudaStream_t st = (cudaStream_t)stream;
  // A few rows are appended by the kernel itself (a launch of its own takes 0.9 to 1.3 us more, whatever the keys); a warp that copies
  // more of them holds its tiles up.
  cudaError_t e = cudaSuccess;
  if (args->rows && c.cfg.dtype == STRUCTKV_BF16 && !tc && args->n_new <= 8) a.fresh = r;
  else if (args->rows) e = launch_append(a.c, r, args->n_new, st);
  if (e == cudaSuccess)
    e = (c.cfg.dtype != STRUCTKV_BF16 ? launch_attend_simt : tc ? launch_attend_tc : launch_attend_mma)(c, a, plan, st);
  if (e == cudaSuccess) e = launch_attend_finish(c, a, plan, st);
  return told(e);
}

structkv_status structkv_weigh(structkv_ctx* ctx, const structkv_cache* cache, const structkv_attend_args* args,
                               const unsigned long long* accepted, void* stream) {
  AttendArgs a{};
  if (!args || !accepted || (uintptr_t)accepted % 8 || !args->lse) return STRUCTKV_ERR_INVALID_ARG;
  if (!view_of(ctx, cache, args->n_new, &a.c) || !cache->weights || !args_of(ctx, cache, args, &a)) return STRUCTKV_ERR_INVALID_ARG;
  a.ctas = ctx->c.cfg.dtype == STRUCTKV_BF16 ? ctx->c.sm_count : 4 * ctx->c.sm_count;   // (CTAs that run at once)
  a.by_ctas = div_by(a.ctas);
  a.over = kWeighOverKeys / 64;
  return told((ctx->c.cfg.dtype == STRUCTKV_BF16 ? launch_weigh_bf16 : launch_weigh_fp32)(ctx->c, a, accepted, (cudaStream_t)stream));
}

structkv_status structkv_commit(structkv_ctx* ctx, const structkv_cache* cache, int n_new, const int* counts, const int* path,
                                void* stream) {
  CacheView v;
  if (n_new < 1 || (path && (!counts || n_new > kMaxNew)) || ((uintptr_t)path | (uintptr_t)counts) % 4 || !view_of(ctx, cache, n_new, &v))
    return STRUCTKV_ERR_INVALID_ARG;
  return told(launch_commit(v, n_new, counts, path, (cudaStream_t)stream));
}

structkv_status structkv_evict(structkv_ctx* ctx, const structkv_cache* cache, int budget, int recent, void* stream) {
  CacheView v;
  if (budget < 1 || recent < 0 || !view_of(ctx, cache, 0, &v) || !cache->weights) return STRUCTKV_ERR_INVALID_ARG;
  return told(launch_evict(v, budget, recent, (cudaStream_t)stream));
}

}  // extern "C"
