// Host side of the paged K/V cache and the attention over it: configuration
// checks, the layout of the state, argument validation and launches. The
// kernels are in pages.hip and attend.hip.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <new>

#include "serve_internal.h"

namespace ldr {

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

static bool make_pages_shape(const ldr_pages_config* c, PagesShape* s) {
  if (!c) return false;
  if (c->n_layers < 1 || c->n_layers > 1024 || c->n_kv_heads < 1 || c->n_kv_heads > 1024)
    return false;
  if (c->n_layers * c->n_kv_heads > 65535) return false;   // a grid's second dimension
  if (c->head_dim != 64 && c->head_dim != 128) return false;
  if (c->page != 32 && c->page != 64 && c->page != 128 && c->page != 256) return false;
  if (c->n_pages < 1 || c->n_pages > (1 << 28)) return false;
  if (c->batch < 1 || c->batch > kMaxSeqs) return false;
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page >= (1 << 30)) return false;
  if (c->dtype != LDR_F32 && c->dtype != LDR_BF16 && c->dtype != LDR_MXFP4 &&
      c->dtype != LDR_MXFP8)
    return false;
  s->layers = c->n_layers; s->hkv = c->n_kv_heads; s->d = c->head_dim; s->page = c->page;
  s->n_pages = c->n_pages; s->batch = c->batch; s->max_pages = c->max_pages; s->dtype = c->dtype;
  s->bits = c->dtype == LDR_MXFP4 ? 4 : c->dtype == LDR_MXFP8 ? 8 : 0;
  s->el = c->dtype == LDR_F32 ? 4 : 2;
  s->head_bytes = (size_t)s->page * (s->bits ? s->d * s->bits / 8 + s->d / kMxBlock : s->d * s->el);
  s->page_bytes = s->hkv * s->head_bytes;
  // regions start on 256 bytes
  auto words = [](size_t n) { return align_up(n * 4) / 4; };
  size_t off = kPagesHeader;
  s->rows = off; off += words(s->batch);
  s->open = off; off += words(s->batch);
  s->table = off; off += words((size_t)s->batch * s->max_pages);
  s->refs = off; off += words(s->n_pages);
  s->list = off; off += words(s->n_pages);
  const size_t pairs = (size_t)s->n_pages / 2 + 1;
  s->pairs = off; off += words(2 * (pairs > (size_t)s->batch ? pairs : (size_t)s->batch));
  s->words = off;
  return true;
}

static bool attend_sizes_ok(const PagesShape& s, int32_t hq, int32_t max_new) {
  return hq > 0 && hq % s.hkv == 0 && max_new > 0 &&
         (int64_t)s.batch * max_new < (1 << 27) / (int64_t)hq;
}

}  // namespace ldr

using namespace ldr;

struct ldr_pages {
  PagesShape s;
  PagesPtrs p;
};

static int done(hipError_t e) { return e == hipSuccess ? LDR_OK : LDR_EHIP; }

extern "C" {

size_t ldr_pages_pool_bytes(const ldr_pages_config* cfg) {
  PagesShape s;
  if (!make_pages_shape(cfg, &s)) return 0;
  return (size_t)2 * s.layers * s.n_pages * s.page_bytes;
}

size_t ldr_pages_state_bytes(const ldr_pages_config* cfg) {
  PagesShape s;
  if (!make_pages_shape(cfg, &s)) return 0;
  return s.words * 4;
}

int ldr_pages_layout(const ldr_pages_config* cfg, size_t offsets[4]) {
  PagesShape s;
  if (!offsets || !make_pages_shape(cfg, &s)) return LDR_EINVAL;
  offsets[0] = s.rows * 4; offsets[1] = s.open * 4; offsets[2] = s.table * 4;
  offsets[3] = s.refs * 4;
  return LDR_OK;
}

int ldr_pages_init(ldr_pages** out, const ldr_pages_config* cfg, void* pool, void* state,
                   void* stream) {
  if (!out) return LDR_EINVAL;
  *out = nullptr;
  PagesShape s;
  if (!make_pages_shape(cfg, &s) || !pool || !state || !aligned(pool, kAlign) ||
      !aligned(state, kAlign))
    return LDR_EINVAL;
  ldr_pages* p = new (std::nothrow) ldr_pages;
  if (!p) return LDR_ENOMEM;
  p->s = s;
  static std::atomic<int32_t> handles{0};
  p->p = PagesPtrs{static_cast<uint8_t*>(pool), static_cast<int32_t*>(state), ++handles};
  if (launch_pages_reset(s, p->p, static_cast<hipStream_t>(stream)) != hipSuccess) {
    delete p;
    return LDR_EHIP;
  }
  *out = p;
  return LDR_OK;
}

int ldr_pages_reserve(ldr_pages* p, const int32_t* n_new, int32_t max_new, void* stream) {
  if (!p || !n_new || !aligned(n_new, 4) || max_new < 0) return LDR_EINVAL;
  return done(launch_pages_reserve(p->s, p->p, n_new, max_new, static_cast<hipStream_t>(stream)));
}

int ldr_pages_write(ldr_pages* p, int32_t layer, int32_t n_layers, const void* K, const void* V,
                    int32_t max_new, void* stream) {
  if (!p || layer < 0 || n_layers < 1 || layer >= p->s.layers || n_layers > p->s.layers - layer)
    return LDR_EINVAL;
  if (max_new < 1 || max_new > (1 << 28) || !K || !V || !aligned(K, 16) || !aligned(V, 16))
    return LDR_EINVAL;
  return done(launch_pages_write(p->s, p->p, layer, n_layers, K, V, max_new,
                                 static_cast<hipStream_t>(stream)));
}

int ldr_pages_read(const ldr_pages* p, int32_t layer, int32_t n_layers, const int32_t* first,
                   const int32_t* n, void* K, void* V, int32_t max_rows, void* stream) {
  if (!p || layer < 0 || n_layers < 1 || layer >= p->s.layers || n_layers > p->s.layers - layer)
    return LDR_EINVAL;
  if (!first || !n || !aligned(first, 4) || !aligned(n, 4)) return LDR_EINVAL;
  if (max_rows < 1 || max_rows > (1 << 28) || !K || !V || !aligned(K, 16) || !aligned(V, 16))
    return LDR_EINVAL;
  // every workgroup reads the counts, the tables and the pool while others write
  const PagesShape& s = p->s;
  const size_t counts = (size_t)s.batch * 4;
  const size_t rows = (size_t)s.batch * max_rows * n_layers * s.hkv * s.d * s.el;
  const Range k{K, rows}, v{V, rows};
  for (const Range& o : {Range{first, counts}, Range{n, counts}, Range{p->p.state, s.words * 4},
                         Range{p->p.pool, (size_t)2 * s.layers * s.n_pages * s.page_bytes}})
    if (overlap(k, o) || overlap(v, o)) return LDR_EINVAL;
  if (overlap(k, v)) return LDR_EINVAL;
  return done(launch_pages_read(s, p->p, layer, n_layers, first, n, K, V, max_rows,
                                static_cast<hipStream_t>(stream)));
}

int ldr_pages_keep(ldr_pages* p, const int32_t* kept, void* stream) {
  if (!p || !kept || !aligned(kept, 4)) return LDR_EINVAL;
  return done(launch_pages_keep(p->s, p->p, kept, static_cast<hipStream_t>(stream)));
}

int ldr_pages_fork(ldr_pages* p, const int32_t* src, void* stream) {
  if (!p || !src || !aligned(src, 4)) return LDR_EINVAL;
  return done(launch_pages_fork(p->s, p->p, src, static_cast<hipStream_t>(stream)));
}

int ldr_pages_compact(ldr_pages* p, void* stream) {
  if (!p) return LDR_EINVAL;
  return done(launch_pages_compact(p->s, p->p, static_cast<hipStream_t>(stream)));
}

int ldr_pages_status(ldr_pages* p, int clear, void* stream) {
  if (!p) return LDR_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int32_t flags = 0;
  if (hipMemcpyAsync(&flags, p->p.state + kPagesFlags, sizeof(flags), hipMemcpyDeviceToHost, st) !=
          hipSuccess ||
      hipStreamSynchronize(st) != hipSuccess)
    return LDR_EHIP;
  if (clear && flags &&
      (launch_pages_clear_flags(p->p, st) != hipSuccess || hipStreamSynchronize(st) != hipSuccess))
    return LDR_EHIP;
  if (flags & kFlagRange) return LDR_ERANGE;
  if (flags & kFlagPages) return LDR_EPAGES;
  return flags & kFlagPlan ? LDR_EINVAL : LDR_OK;
}

void ldr_pages_destroy(ldr_pages* p) { delete p; }

size_t ldr_attend_workspace_bytes(const ldr_pages_config* cfg, int32_t n_q_heads,
                                  int32_t max_new) {
  PagesShape s;
  if (!make_pages_shape(cfg, &s) || !attend_sizes_ok(s, n_q_heads, max_new)) return 0;
  return attend_workspace_bytes(s, n_q_heads, max_new);
}

int ldr_attend_plan(const ldr_pages* p, int32_t n_q_heads, int32_t max_new,
                    const int32_t* groups, void* workspace, size_t workspace_bytes,
                    void* stream) {
  if (!p || !attend_sizes_ok(p->s, n_q_heads, max_new) || !aligned(groups, 4)) return LDR_EINVAL;
  if (!workspace || !aligned(workspace, kAlign) ||
      workspace_bytes < attend_workspace_bytes(p->s, n_q_heads, max_new))
    return LDR_EINVAL;
  return done(launch_attend_plan(p->s, p->p, n_q_heads, max_new, groups, workspace,
                                 static_cast<hipStream_t>(stream)));
}

int ldr_attend(const ldr_pages* p, int32_t layer, const void* q, int64_t q_stride,
               int32_t n_q_heads, int32_t max_new, float scale, void* o, float* lse,
               void* workspace, size_t workspace_bytes, void* stream) {
  if (!p || layer < 0 || layer >= p->s.layers || !attend_sizes_ok(p->s, n_q_heads, max_new))
    return LDR_EINVAL;
  if (!q || !o || !aligned(q, 16) || !aligned(o, 16) || !aligned(lse, 4)) return LDR_EINVAL;
  if (q_stride < (int64_t)n_q_heads * p->s.d || q_stride % (16 / (int64_t)p->s.el))
    return LDR_EINVAL;
  if (!std::isnormal(scale) || scale < 0.f) return LDR_EINVAL;
  if (!std::isfinite(scale * kLog2e)) return LDR_EINVAL;   // the kernels' exponents are of base 2
  if (!workspace || !aligned(workspace, kAlign) ||
      workspace_bytes < attend_workspace_bytes(p->s, n_q_heads, max_new))
    return LDR_EINVAL;
  return done(launch_attend(p->s, p->p, layer, q, (long)q_stride, n_q_heads, max_new, scale, o, lse,
                            workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
