// C ABI of rotary positions and of the paged cache: argument validation and dispatch.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <cstring>

#include "attend_pages.cuh"

using namespace skv;

namespace skv {
namespace {

// Places of an item's own cost, in tiles of 64 keys.  16 sequences of 1 to 5003 keys 20.8 us; 1 place 23.0, 12 places 22.0.  On tcgen05 16 tokens over
// 4 x 8192 keys 35.3 us; 2 places 37.0, 24 places 37.6.
constexpr int kOver = 4, kOverTc = 8;

structkv_status told(cudaError_t e) { return e == cudaSuccess ? STRUCTKV_OK : STRUCTKV_ERR_CUDA; }
int elem_of(const structkv_ctx* ctx) { return ctx->c.cfg.dtype == STRUCTKV_BF16 ? 2 : 4; }
bool on_device(const structkv_ctx* ctx) {
  int dev = -1;
  return cudaGetDevice(&dev) == cudaSuccess && dev == ctx->c.device;
}
bool steps_16(int elem, long long a, long long b, long long c) { return (a * elem) % 16 == 0 && (b * elem) % 16 == 0 && (c * elem) % 16 == 0; }
bool rope_ok(const structkv_ctx* ctx, const structkv_rope* r) {
  return r && r->dim >= 2 && r->dim % 2 == 0 && r->dim <= ctx->c.cfg.head_dim && std::isfinite((float)r->amplitude);
}
RopeArgs rope_args(const structkv_rope* r) {
  RopeArgs a{};
  if (!r) return a;
  a.dim = r->dim;
  a.interleaved = r->interleaved != 0;
  a.amplitude = (float)r->amplitude;
  a.amplitude64 = r->amplitude;
  // In units of 2^-24 of amplitude (|a| + |b|): cosine or sine and its product's rounding are off by 2.53 at most (all angles were tried), by 1 more
  // where an amplitude is multiplied in, which rounds, and by what that is off itself.  amplitude (|a| + |b|) is at most sqrt(2) (|a'| + |b'|), and the
  // sum is rounded.
  int exponent;
  const double size = std::fabs(r->amplitude), itself = size > 0.0 ? std::fabs(a.amplitude - r->amplitude) / size * 0x1p24 : 0.0;
  a.off = (float)((std::sqrt(2.0) * (2.54 + (std::frexp(size, &exponent) == 0.5 ? 0.0 : 1.0 + itself)) + 1.0) * 0x1p-24);
  std::memcpy(a.step, r->step, sizeof(a.step));
  return a;
}

bool view_of(const structkv_ctx* ctx, const structkv_pages* p, PagesView* v) {
  if (!ctx || !p || !p->k || !p->v || !p->k_scales || !p->v_scales || !p->table || !p->lengths) return false;
  const structkv_config& cfg = ctx->c.cfg;
  if (p->batch < 1 || p->pages < 1 || p->table_columns < 1 || p->table_stride < 0) return false;
  if (p->page_size < 16 || p->page_size > 256 || (p->page_size & (p->page_size - 1))) return false;
  if ((long long)p->table_columns * p->page_size > 1 << 30) return false;
  if (((uintptr_t)p->k | (uintptr_t)p->v) % 16 || ((uintptr_t)p->table | (uintptr_t)p->lengths) % 4) return false;
  if (!steps_16(1, p->stride_page, p->stride_head, p->stride_token)) return false;
  if (p->stride_token < cfg.head_dim || (cfg.n_kv_heads > 1 && p->stride_head < cfg.head_dim) || (p->pages > 1 && p->stride_page < cfg.head_dim))
    return false;
  // (a step within a page is counted in 31 bits, one between pages in 32, blocks of slots in 31)
  if (p->stride_token >= 1ll << 22 || p->stride_page >= 1ll << 32 || (long long)p->pages * cfg.n_kv_heads * (p->page_size / 16) > 0x7fffffffll) return false;
  int shift = 4;
  while (1 << shift < p->page_size) ++shift;
  *v = PagesView{(char*)p->k, (char*)p->v, p->k_scales, p->v_scales, p->stride_page, p->stride_head, p->table_stride * 4,
                 (int)p->stride_token, p->table, p->lengths, p->batch, cfg.n_kv_heads, p->pages, shift, p->table_columns << shift, ctx->c.ws.status};
  return true;
}

// More than 16 rows of a KV head go to tcgen05, with caps more than 32 (each score's hyperbolic tangent is worked out by 8 warps an SM there, by
// 8 or 16 here).  Up to 16 rows mma.sync has one pass over the codes, from 17 on two or more.  20 rows over 32 x 4096 keys: 129 us on mma.sync, 100 on
// tcgen05; over 4 x 8192 39.6, 34.0; over 1 x 4096 14.5, 15.2 (how many keys there are is known on the device only).  With caps 20 rows over
// 4 x 8192 43 us and 47, 40 rows 58 and 48.
PagesPlan plan_of(const structkv_config& cfg, int n_new, int sms, bool capped) {
  const int rows = cfg.n_q_heads / cfg.n_kv_heads * n_new;
  if (cfg.dtype == STRUCTKV_BF16 && rows > (capped ? 32 : 16)) return {rows <= 64 ? 64 : 128, sms, kOverTc};
  // (several CTAs an SM: one begins or ends a segment while others stream)
  return cfg.dtype == STRUCTKV_FP32 ? PagesPlan{8, 2 * sms, kOver} : rows <= 8 ? PagesPlan{8, 4 * sms, kOver} : PagesPlan{16, 2 * sms, kOver};
}
// Items, rows and places are counted in 31 bits.
bool sizes_ok(const structkv_config& cfg, int batch, int n_new, long long slots) {
  if (batch < 1 || n_new < 1 || n_new > kMaxNew || slots < 1 || slots > 1 << 30) return false;
  const long long units = (long long)batch * cfg.n_kv_heads, rows = (long long)cfg.n_q_heads / cfg.n_kv_heads * n_new;
  return units <= 0x3fffffffll && units * rows <= 0x3fffffffll && units * ((rows + 7) / 8) <= 0x7fffffffll / (slots / 64 + 1 + kOverTc);
}
struct PagesWs { int2* item_parts; float2* part_stat; float* part_out; size_t bytes; };
PagesWs carve(const structkv_config& cfg, const PagesPlan& p, int batch, int n_new, void* base) {
  PagesWs w{};
  char* at = (char*)base;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    void* r = at ? (void*)(at + off) : nullptr;
    off += align_up(bytes, 256);
    return r;
  };
  const size_t group = cfg.n_q_heads / cfg.n_kv_heads, items = (size_t)batch * cfg.n_kv_heads * ((group * n_new + p.rb - 1) / p.rb), slots = items + p.ctas;
  w.item_parts = (int2*)take(items * sizeof(int2));
  w.part_stat = (float2*)take(slots * p.rb * sizeof(float2));
  w.part_out = (float*)take(slots * p.rb * cfg.head_dim * sizeof(float));
  w.bytes = off;
  return w;
}

}  // namespace
}  // namespace skv

extern "C" {

structkv_status structkv_rope_init(structkv_rope* rope, int dim, int interleaved, double base, int scaling, double factor, double original,
                                   double slow, double fast) {
  if (!rope || dim < 2 || dim % 2 || dim > STRUCTKV_ROPE_MAX_DIM || !(base > 1.0) || !std::isfinite(base)) return STRUCTKV_ERR_INVALID_ARG;
  if (scaling < STRUCTKV_ROPE_PLAIN || scaling > STRUCTKV_ROPE_RAMP) return STRUCTKV_ERR_INVALID_ARG;
  auto positive = [](double x) { return x > 0.0 && std::isfinite(x); };
  const bool parts = scaling == STRUCTKV_ROPE_BANDS || scaling == STRUCTKV_ROPE_RAMP;
  if (scaling != STRUCTKV_ROPE_PLAIN && !positive(factor)) return STRUCTKV_ERR_INVALID_ARG;
  if (parts && !(positive(original) && positive(slow) && positive(fast) && slow < fast)) return STRUCTKV_ERR_INVALID_ARG;
  if (scaling == STRUCTKV_ROPE_BASE && dim == 2) return STRUCTKV_ERR_INVALID_ARG;
  const long double two_pi = 6.283185307179586476925286766559005768L, by = (long double)factor;
  long double b = base;
  if (scaling == STRUCTKV_ROPE_BASE) b *= powl(by, (long double)dim / (dim - 2));
  if (!std::isfinite((double)b) || b <= 1.0L) return STRUCTKV_ERR_INVALID_ARG;
  long double lo = 0, hi = 0;
  if (scaling == STRUCTKV_ROPE_RAMP) {
    auto pair = [&](long double turns) { return dim * logl((long double)original / (turns * two_pi)) / (2 * logl(b)); };
    lo = std::max(0.0L, floorl(pair(fast)));
    hi = std::min((long double)(dim - 1), ceill(pair(slow)));
  }
  structkv_rope r{};
  r.dim = dim;
  r.interleaved = interleaved != 0;
  r.amplitude = scaling == STRUCTKV_ROPE_RAMP && factor > 1.0 ? (double)(0.1L * logl(by) + 1.0L) : 1.0;
  for (int c = 0; c < dim / 2; ++c) {
    long double f = powl(b, -2.0L * c / dim);
    if (scaling == STRUCTKV_ROPE_LINEAR) f /= by;
    if (parts) {
      long double part = scaling == STRUCTKV_ROPE_BANDS ? ((long double)original * f / two_pi - slow) / ((long double)fast - slow)
                                                         : 1.0L - (c - lo) / std::max(hi - lo, 0.001L);
      part = std::min(1.0L, std::max(0.0L, part));
      f = part * f + (1.0L - part) * f / by;
    }
    long double turns = f / two_pi;
    turns -= floorl(turns);
    const long double units = roundl(turns * 18446744073709551616.0L);
    r.step[c] = units >= 18446744073709551616.0L ? 0ull : (unsigned long long)units;
  }
  *rope = r;
  return STRUCTKV_OK;
}

structkv_status structkv_rotate(structkv_ctx* ctx, const structkv_rope* rope, const structkv_rotate_args* x, void* stream) {
  if (!ctx || !x || !rope_ok(ctx, rope) || x->batch < 0 || x->tokens < 0 || x->heads < 0 || x->positions_stride < 0) return STRUCTKV_ERR_INVALID_ARG;
  const long long rows = (long long)x->batch * x->tokens;
  if (rows > 0x7fffffffll) return STRUCTKV_ERR_INVALID_ARG;
  if (rows == 0 || x->heads == 0) return STRUCTKV_OK;
  const int elem = elem_of(ctx), d = ctx->c.cfg.head_dim;
  if (!x->x || !x->out || !x->positions || ((uintptr_t)x->x | (uintptr_t)x->out) % 16 || (uintptr_t)x->positions % 4) return STRUCTKV_ERR_INVALID_ARG;
  if (!steps_16(elem, x->x_stride_batch, x->x_stride_token, x->x_stride_head) || !steps_16(elem, x->out_stride_batch, x->out_stride_token, x->out_stride_head))
    return STRUCTKV_ERR_INVALID_ARG;
  auto apart = [&](int n, long long stride) { return n == 1 || std::llabs(stride) >= d; };
  if (!apart(x->batch, x->out_stride_batch) || !apart(x->tokens, x->out_stride_token) || !apart(x->heads, x->out_stride_head)) return STRUCTKV_ERR_INVALID_ARG;
  auto same = [](int n, long long a, long long b) { return n == 1 || a == b; };
  if (x->x == x->out && !(same(x->batch, x->x_stride_batch, x->out_stride_batch) && same(x->tokens, x->x_stride_token, x->out_stride_token) &&
                          same(x->heads, x->x_stride_head, x->out_stride_head)))
    return STRUCTKV_ERR_INVALID_ARG;
  if (!on_device(ctx)) return STRUCTKV_ERR_INVALID_ARG;
  RotateArgs a{(const char*)x->x, (char*)x->out, x->x_stride_batch * elem, x->x_stride_token * elem, x->x_stride_head * elem,
               x->out_stride_batch * elem, x->out_stride_token * elem, x->out_stride_head * elem, x->positions_stride, x->positions,
               div_by(x->tokens), (int)rows, x->tokens, x->heads, 1, x->inverse != 0};
  a.head_step = heads_at_once(rows, d * elem / 32, x->heads, ctx->c.sm_count);
  if ((x->heads + a.head_step - 1) / a.head_step > 65535) a.head_step = (x->heads + 65534) / 65535;
  return told(launch_rotate(ctx->c, rope_args(rope), a, (cudaStream_t)stream));
}

structkv_status structkv_append_pages(structkv_ctx* ctx, const structkv_pages* pages, const structkv_append_pages_args* x, void* stream) {
  AppendPagesArgs a{};
  if (!x || !view_of(ctx, pages, &a.c) || !x->k || !x->v || ((uintptr_t)x->k | (uintptr_t)x->v) % 16) return STRUCTKV_ERR_INVALID_ARG;
  const int elem = elem_of(ctx), d = ctx->c.cfg.head_dim;
  if (!steps_16(elem, x->stride_batch, x->stride_token, x->stride_head)) return STRUCTKV_ERR_INVALID_ARG;
  if (x->n_new < 1 || x->n_new > a.c.slots || x->tokens < 1 || (!x->index && x->n_new > x->tokens)) return STRUCTKV_ERR_INVALID_ARG;
  if (((uintptr_t)x->counts | (uintptr_t)x->index | (uintptr_t)x->positions) % 4 || x->index_stride < 0 || x->positions_stride < 0) return STRUCTKV_ERR_INVALID_ARG;
  if ((x->rope && !rope_ok(ctx, x->rope)) || (x->rope != nullptr) != (x->positions != nullptr)) return STRUCTKV_ERR_INVALID_ARG;
  if ((x->q != nullptr) != (x->q_out != nullptr) || (x->q && (x->index || !x->rope))) return STRUCTKV_ERR_INVALID_ARG;
  const int heads = ctx->c.cfg.n_q_heads;
  if (x->q) {
    if (((uintptr_t)x->q | (uintptr_t)x->q_out) % 16 || !steps_16(elem, x->q_stride_batch, x->q_stride_token, x->q_stride_head)) return STRUCTKV_ERR_INVALID_ARG;
    auto whole = [](int n, long long stride, long long want) { return n == 1 || stride == want; };
    if (x->q == x->q_out && !(whole(heads, x->q_stride_head, d) && whole(x->n_new, x->q_stride_token, (long long)heads * d) &&
                              whole(a.c.batch, x->q_stride_batch, (long long)x->n_new * heads * d)))
      return STRUCTKV_ERR_INVALID_ARG;
  }
  const long long blocks = ((long long)x->n_new + 2 * kBlockSlots - 2) / kBlockSlots, rows = (long long)a.c.batch * x->n_new;
  // (CTAs of both kinds are counted in 31 bits)
  if (rows * (heads + 1) > 0x3fffffffll || a.c.batch * blocks * a.c.n_kv > 0x3fffffffll) return STRUCTKV_ERR_INVALID_ARG;
  if (!on_device(ctx)) return STRUCTKV_ERR_INVALID_ARG;
  a.by_blocks = div_by((unsigned)blocks);
  a.by_new = div_by(x->n_new);
  a.k = (const char*)x->k;
  a.v = (const char*)x->v;
  a.s_batch = x->stride_batch * elem;
  a.s_token = x->stride_token * elem;
  a.s_head = x->stride_head * elem;
  a.tokens = x->tokens;
  a.n_new = x->n_new;
  a.blocks = (int)blocks;
  a.counts = x->counts;
  a.index = x->index;
  a.positions = x->positions;
  a.s_index = x->index_stride;
  a.s_positions = x->positions_stride;
  a.rotated = x->rope != nullptr;
  a.q = (const char*)x->q;
  a.q_batch = x->q_stride_batch * elem;
  a.q_token = x->q_stride_token * elem;
  a.q_head = x->q_stride_head * elem;
  a.q_out = (char*)x->q_out;
  a.heads = heads;
  a.q_rows = (int)rows;
  a.head_step = heads_at_once(rows, d * elem / 32, heads, ctx->c.sm_count);
  a.splits = append_splits(a.c.batch * blocks, a.c.n_kv, ctx->c.sm_count);
  a.by_splits = div_by(a.splits);
  a.append_ctas = (int)(a.c.batch * blocks * a.splits);
  return told(launch_append_pages(ctx->c, rope_args(x->rope), a, (cudaStream_t)stream));
}

size_t structkv_attend_pages_workspace_bytes(const structkv_config* cfg, int batch, int n_new, long long slots) {
  if (structkv_workspace_bytes(cfg) == 0 || !sizes_ok(*cfg, batch, n_new, slots)) return 0;
  return std::max(carve(*cfg, plan_of(*cfg, n_new, kMaxSms, false), batch, n_new, nullptr).bytes, carve(*cfg, plan_of(*cfg, n_new, kMaxSms, true), batch, n_new, nullptr).bytes);
}

structkv_status structkv_attend_pages(structkv_ctx* ctx, const structkv_pages* pages, const structkv_attend_pages_args* x, void* stream) {
  AttendPagesArgs a{};
  if (!x || !view_of(ctx, pages, &a.c)) return STRUCTKV_ERR_INVALID_ARG;
  const structkv_config& cfg = ctx->c.cfg;
  const int elem = elem_of(ctx);
  if (!sizes_ok(cfg, a.c.batch, x->n_new, a.c.slots)) return STRUCTKV_ERR_INVALID_ARG;
  if (!x->q || !x->out || ((uintptr_t)x->q | (uintptr_t)x->out) % 16 || ((uintptr_t)x->counts | (uintptr_t)x->lse) % 4) return STRUCTKV_ERR_INVALID_ARG;
  if (!steps_16(elem, x->q_stride_batch, x->q_stride_token, x->q_stride_head)) return STRUCTKV_ERR_INVALID_ARG;
  if (!std::isfinite(x->scale) || !std::isfinite(x->softcap) || x->softcap < 0.f) return STRUCTKV_ERR_INVALID_ARG;
  // (a cap beyond 2^100 |scale| caps nothing, as in structkv_attend)
  const float softcap = x->softcap > 0x1p100f * std::fabs(x->scale) ? 0.f : x->softcap;
  a.scale2 = x->scale * kLog2e;
  a.cap2 = softcap * kLog2e;
  a.inv_cap = softcap > 0.f ? x->scale / softcap : 0.f;
  if (!std::isfinite(a.scale2) || !std::isfinite(a.cap2) || !std::isfinite(a.inv_cap)) return STRUCTKV_ERR_INVALID_ARG;
  if (!on_device(ctx)) return STRUCTKV_ERR_INVALID_ARG;
  const PagesPlan plan = plan_of(cfg, x->n_new, std::min(ctx->c.sm_count, kMaxSms), a.cap2 != 0.f);
  const PagesWs w = carve(cfg, plan, a.c.batch, x->n_new, x->workspace);
  if (!x->workspace || x->workspace_bytes < w.bytes || (uintptr_t)x->workspace % 256) return STRUCTKV_ERR_WORKSPACE;
  a.q = (const char*)x->q;
  a.q_batch = x->q_stride_batch * elem;
  a.q_token = x->q_stride_token * elem;
  a.q_head = x->q_stride_head * elem;
  a.counts = x->counts;
  a.n_new = x->n_new;
  a.group = cfg.n_q_heads / cfg.n_kv_heads;
  a.rows = a.group * x->n_new;
  a.blocks = (a.rows + plan.rb - 1) / plan.rb;
  a.by_blocks = div_by(a.blocks);
  a.by_group = div_by(a.group);
  a.by_rows = div_by(a.rows);
  a.by_kv = div_by(cfg.n_kv_heads);
  a.by_ctas = div_by(plan.ctas);
  a.out = (char*)x->out;
  a.lse = x->lse;
  a.item_parts = w.item_parts;
  a.part_stat = w.part_stat;
  a.part_out = w.part_out;
  a.ctas = plan.ctas;
  a.over = plan.over;
  cudaError_t e = (plan.rb > 16 ? launch_attend_pages_tc : launch_attend_pages)(ctx->c, a, plan, (cudaStream_t)stream);
  if (e == cudaSuccess) e = launch_attend_pages_finish(ctx->c, a, plan, (cudaStream_t)stream);
  return told(e);
}

}  // extern "C"
