// Host side of the operators that serve a batch of requests from one shared prefix: page
// plans, paged appends and attention over prefix and tails.  Arguments are validated here,
// before any device work; lengths, tables and maps are device data that the host never reads,
// so the kernels bound every index that they take from them.
#include <algorithm>
#include <cmath>

#include "host_util.h"
#include "jolt_internal.h"
#include "kernels.h"

namespace {

bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int log2_exact(int x) {
  int s = 0;
  while ((1 << s) < x) ++s;
  return s;
}

// what jolt_page_plan uses of a descriptor
int validate_page_count(const jolt_page_desc *p) {
  if (!p) return jolt_fail(JOLT_E_INVAL, "page descriptor is null");
  if (p->page_size < 1 || p->page_size > SERVE_PAGE_MAX || (p->page_size & (p->page_size - 1)))
    return jolt_fail(JOLT_E_INVAL, "page_size must be a power of two in 1..%d (got %d)", SERVE_PAGE_MAX, p->page_size);
  if (p->n_pages < 1 || (int64_t)p->n_pages * p->page_size >= ((int64_t)1 << 31))
    return jolt_fail(JOLT_E_INVAL, "n_pages must be >= 1 with n_pages * page_size < 2^31");
  return JOLT_OK;
}

int validate_pages(const jolt_page_desc *p) {
  int rc = validate_page_count(p);
  if (rc) return rc;
  if (p->dtype != JOLT_F32 && p->dtype != JOLT_BF16)
    return jolt_fail(JOLT_E_INVAL, "dtype must be JOLT_F32 or JOLT_BF16");
  if (p->d != 32 && p->d != 64 && p->d != 128)
    return jolt_fail(JOLT_E_UNSUPPORTED, "d must be 32, 64 or 128 (got %d)", p->d);
  if (p->n_heads < 1 || p->n_heads > 1024) return jolt_fail(JOLT_E_INVAL, "n_heads must be in 1..1024");
  struct Dim { int64_t stride, count; } dim[3] = {
      {p->stride_page, p->n_pages}, {p->stride_head, p->n_heads}, {p->stride_token, p->page_size}};
  int64_t extent = p->d;   // of everything placed so far: each stride, in rising order, clears it
  std::sort(dim, dim + 3, [](const Dim &a, const Dim &b) { return a.stride < b.stride; });
  for (const Dim &x : dim) {
    if (x.stride < 0 || (x.stride % 8)) return jolt_fail(JOLT_E_INVAL, "page strides must be multiples of 8 elements, >= 0");
    if (x.count == 1) continue;
    if (x.stride < extent) return jolt_fail(JOLT_E_INVAL, "page strides let rows overlap");
    if (x.stride > ((int64_t)1 << 60) / x.count) return jolt_fail(JOLT_E_INVAL, "page strides too large");
    extent += (x.count - 1) * x.stride;
  }
  return JOLT_OK;
}

int validate_rows(const char *what, const void *base, const jolt_row_strides *s) {
  if (!base || !s) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: %s or its strides are null", what);
  if (misaligned(base, 16)) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: %s must be 16-byte aligned", what);
  if (s->stride_token < 0 || s->stride_head < 0 || (s->stride_token % 8) || (s->stride_head % 8))
    return jolt_fail(JOLT_E_INVAL, "jolt_page_append: strides of %s must be multiples of 8 elements, >= 0", what);
  return JOLT_OK;
}

// Validates a call's shapes and fills what the kernels and the workspace size depend on.
int resolve_prefix_attend(const jolt_cell_desc *prefix, const jolt_page_desc *pages, const jolt_attend_batch *b,
                          PrefixAttendArgs *a, int *d, int *dtype) {
  if (!b) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: batch is null");
  if (!prefix && !pages) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: neither a prefix nor pages");
  int rc;
  if (prefix && (rc = validate_desc(prefix))) return rc;
  if (pages && (rc = validate_pages(pages))) return rc;
  if (prefix && prefix->T >= (1 << 20)) return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_prefix_attend: T must be below 2^20");
  const int H = pages ? pages->n_heads : prefix->n_heads;
  *d = pages ? pages->d : prefix->d;
  *dtype = pages ? pages->dtype : prefix->dtype;
  if (prefix && (prefix->n_heads != H || prefix->d != *d || prefix->dtype != *dtype))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: prefix and pages differ in heads, d or dtype");
  if (H > 1024) return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_prefix_attend: at most 1024 key-value heads");
  if (b->n_req < 1 || b->n_tok < 1 || b->n_q < 1) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: empty call");
  if (b->n_req > SERVE_REQ_MAX)
    return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_prefix_attend: at most %d requests", SERVE_REQ_MAX);
  if (b->n_q % H)
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: n_q = %d is not a multiple of the %d key-value heads", b->n_q, H);
  if (b->n_q / H > SERVE_REP_MAX)
    return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_prefix_attend: at most %d query heads per key-value head", SERVE_REP_MAX);
  if ((int64_t)b->n_tok * b->n_q >= ((int64_t)1 << 28))
    return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_prefix_attend: n_tok * n_q must be below 2^28");
  if (b->max_new < 0) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: max_new must be >= 0");
  const int64_t row = (int64_t)b->n_q * *d;
  if (b->q_stride < row || b->o_stride < row || (b->q_stride % 8) || (b->o_stride % 8) ||
      std::max(b->q_stride, b->o_stride) > ((int64_t)1 << 40))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: strides of Q and O must be multiples of 8 elements, >= n_q * d");
  if (pages && (b->max_pages < 1 || (int64_t)b->max_pages * pages->page_size >= ((int64_t)1 << 30)))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: max_pages must be >= 1 with max_pages * page_size < 2^30");
  *a = PrefixAttendArgs{};
  a->n_req = b->n_req; a->n_tok = b->n_tok; a->n_q = b->n_q; a->heads = H; a->group = b->n_q / H;
  a->q_stride = b->q_stride; a->o_stride = b->o_stride;
  a->T = prefix ? prefix->T : 0;
  a->max_new = b->max_new == 0 ? b->n_tok : std::min(b->max_new, b->n_tok);
  if (prefix) a->prefix = PrefixSource{nullptr, nullptr, 0, prefix->stride_head, prefix->stride_token, 30, 1};
  if (pages) {
    a->max_pages = b->max_pages;
    a->tail = PrefixSource{nullptr, nullptr, pages->stride_page, pages->stride_head, pages->stride_token,
                           log2_exact(pages->page_size), pages->n_pages};
  }
  return JOLT_OK;
}

}  // namespace

extern "C" int jolt_page_plan(jolt_ctx *ctx, const jolt_page_desc *pages, int n_req, const int32_t *have,
                              const int32_t *add, const int32_t *free_pages, int free_cap, const int32_t *n_free,
                              int32_t *table, int max_pages, int n_tok, int32_t *kv_len, int32_t *q_start,
                              int32_t *slots, int32_t *positions, int32_t *n_free_out, int32_t *info,
                              jolt_stream stream) {
  int rc = validate_page_count(pages);
  if (rc) return rc;
  if (n_req < 1 || n_tok < 1 || max_pages < 1 || free_cap < 0)
    return jolt_fail(JOLT_E_INVAL, "jolt_page_plan: n_req, n_tok and max_pages must be >= 1, free_cap >= 0");
  if ((int64_t)max_pages * pages->page_size >= ((int64_t)1 << 30))
    return jolt_fail(JOLT_E_INVAL, "jolt_page_plan: max_pages * page_size must be below 2^30");
  if (n_req > SERVE_REQ_MAX) return jolt_fail(JOLT_E_UNSUPPORTED, "jolt_page_plan: at most %d requests", SERVE_REQ_MAX);
  if (!have || !add || (!free_pages && free_cap) || !n_free || !table || !kv_len || !q_start || !slots || !positions ||
      !n_free_out || !info)
    return jolt_fail(JOLT_E_INVAL, "jolt_page_plan: null argument");
  if (kv_len == have || kv_len == add || n_free_out == n_free)
    return jolt_fail(JOLT_E_INVAL, "jolt_page_plan: kv_len and n_free_out need memory of their own");
  if (!ctx) return jolt_fail(JOLT_E_INVAL, "jolt_page_plan: ctx is null");
  DeviceGuard dg;
  HIP_OK(dg.enter(ctx->device));
  hipStream_t st = (hipStream_t)stream;
  PagePlanArgs a{};
  a.have = have; a.add = add; a.free_pages = free_pages; a.n_free = n_free;
  a.table = table; a.kv_len = kv_len; a.q_start = q_start; a.slots = slots; a.positions = positions;
  a.n_free_out = n_free_out; a.info = info;
  a.n_req = n_req; a.free_cap = free_cap; a.max_pages = max_pages; a.n_tok = n_tok;
  a.n_pages = pages->n_pages; a.page_shift = log2_exact(pages->page_size);
  StageTimer t(ctx, st, JOLT_STAGE_PAGE_PLAN);
  HIP_OK(launch_page_plan(a, st));
  return JOLT_OK;
}

extern "C" int jolt_page_append(jolt_ctx *ctx, const jolt_page_desc *pages, int n_tok, const int32_t *slots,
                                const int32_t *positions, const jolt_rope *rope, const void *K,
                                const jolt_row_strides *k_strides, const void *V, const jolt_row_strides *v_strides,
                                void *K_pages, void *V_pages, jolt_stream stream) {
  int rc = validate_pages(pages);
  if (rc) return rc;
  if (n_tok < 1) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: n_tok must be >= 1");
  if (!slots || !K_pages || !V_pages || (rope && !positions)) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: null argument");
  if (misaligned(K_pages, 16) || misaligned(V_pages, 16))
    return jolt_fail(JOLT_E_INVAL, "jolt_page_append: the pools must be 16-byte aligned");
  if (K_pages == V_pages) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: keys and values need a pool each");
  if ((rc = validate_rows("K", K, k_strides)) || (rc = validate_rows("V", V, v_strides))) return rc;
  if (rope && (!(rope->base > 1.0) || !std::isfinite(rope->base) || rope->position_offset < 0))
    return jolt_fail(JOLT_E_INVAL, "jolt_page_append: rope needs a finite base > 1 and position_offset >= 0");
  if (!ctx) return jolt_fail(JOLT_E_INVAL, "jolt_page_append: ctx is null");
  DeviceGuard dg;
  HIP_OK(dg.enter(ctx->device));
  hipStream_t st = (hipStream_t)stream;
  PageAppendArgs a{};
  a.slots = slots; a.positions = positions; a.K = K; a.V = V; a.Kp = K_pages; a.Vp = V_pages;
  a.k_tok = k_strides->stride_token; a.k_head = k_strides->stride_head;
  a.v_tok = v_strides->stride_token; a.v_head = v_strides->stride_head;
  a.s_page = pages->stride_page; a.s_head = pages->stride_head; a.s_tok = pages->stride_token;
  a.n_tok = n_tok; a.n_heads = pages->n_heads; a.page_shift = log2_exact(pages->page_size);
  a.n_slots = pages->n_pages * pages->page_size;
  if (rope) {
    a.rope = 1;
    a.offset = rope->position_offset;
    for (int j = 0; j < pages->d / 2; ++j)
      a.turns[j] = std::pow(rope->base, -2.0 * j / pages->d) / (2.0 * M_PI);
  }
  StageTimer t(ctx, st, JOLT_STAGE_PAGE_APPEND);
  HIP_OK(launch_page_append(a, pages->d, pages->dtype, st));
  return JOLT_OK;
}

extern "C" int jolt_prefix_attend_workspace_size(const jolt_cell_desc *prefix, const jolt_page_desc *pages,
                                                 const jolt_attend_batch *batch, size_t *bytes) {
  PrefixAttendArgs a;
  int d, dtype;
  int rc = resolve_prefix_attend(prefix, pages, batch, &a, &d, &dtype);
  if (rc) return rc;
  if (!bytes) return jolt_fail(JOLT_E_INVAL, "bytes is null");
  *bytes = prefix_attend_cut(a, d, dtype).ws_bytes;
  return JOLT_OK;
}

extern "C" int jolt_debug_prefix_cut(const jolt_cell_desc *prefix, const jolt_page_desc *pages,
                                     const jolt_attend_batch *batch, int64_t *out) {
  PrefixAttendArgs a;
  int d, dtype;
  int rc = resolve_prefix_attend(prefix, pages, batch, &a, &d, &dtype);
  if (rc) return rc;
  if (!out) return jolt_fail(JOLT_E_INVAL, "jolt_debug_prefix_cut: out is null");
  const PrefixCut c = prefix_attend_cut(a, d, dtype);
  const bool pre = a.T > 0 && !c.whole, tails = a.max_pages > 0 && !c.whole;
  out[0] = c.whole;
  out[1] = !pre ? 0 : (c.prefix_few ? 16 : 64) * c.prefix_nq;
  out[2] = c.n_prefix;
  out[3] = pre && !c.prefix_few ? c.prefix_tiles : 0;
  out[4] = pre && !c.prefix_few ? c.kv_tiles : 0;
  out[5] = pre && !c.prefix_few ? c.share : 0;
  out[6] = tails || c.whole ? 16 * c.few_nq : 0;
  out[7] = tails && c.tails_many ? 64 * c.many_nq : 0;
  out[8] = c.n_many;
  out[9] = c.join_lanes;
  return JOLT_OK;
}

extern "C" int jolt_prefix_attend(jolt_ctx *ctx, const jolt_cell_desc *prefix, const void *K, const void *V, int layer,
                                  const jolt_page_desc *pages, const void *K_pages, const void *V_pages,
                                  const int32_t *table, const jolt_attend_batch *batch, const int32_t *q_start,
                                  const int32_t *kv_len, const void *Q, float scale, void *O, float *lse, void *ws,
                                  size_t ws_bytes, jolt_stream stream) {
  PrefixAttendArgs a;
  int d, dtype;
  int rc = resolve_prefix_attend(prefix, pages, batch, &a, &d, &dtype);
  if (rc) return rc;
  if (!q_start || !Q || !O || !ws) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: null argument");
  if (prefix && (!K || !V)) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: a prefix without keys or values");
  if (prefix && (layer < 0 || layer >= prefix->n_layers))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: layer %d outside the cell's %d layers", layer, prefix->n_layers);
  if (pages && (!K_pages || !V_pages || !table || !kv_len))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: pages without pools, table or lengths");
  if (misaligned(Q, 16) || misaligned(O, 16) || (prefix && (misaligned(K, 16) || misaligned(V, 16))) ||
      (pages && (misaligned(K_pages, 16) || misaligned(V_pages, 16))))
    return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: Q, O, keys and values must be 16-byte aligned");
  if (misaligned(ws, 256)) return jolt_fail(JOLT_E_INVAL, "workspace must be 256-byte aligned");
  // the kernels form scores in units of log2: scale * log2(e) has to be finite too
  if (!(scale > 0.f) || !(scale < 0x1p127f)) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: scale must be > 0 and below 2^127");
  const PrefixCut cut = prefix_attend_cut(a, d, dtype);
  if (ws_bytes < cut.ws_bytes) return jolt_fail(JOLT_E_WORKSPACE, "workspace %zu < %zu bytes", ws_bytes, cut.ws_bytes);
  if (!ctx) return jolt_fail(JOLT_E_INVAL, "jolt_prefix_attend: ctx is null");
  DeviceGuard dg;
  HIP_OK(dg.enter(ctx->device));
  forget_spectra(ctx, ws, ws_bytes);
  hipStream_t st = (hipStream_t)stream;
  if (prefix) {
    const int64_t off = (int64_t)layer * prefix->stride_layer * (dtype == JOLT_BF16 ? 2 : 4);
    a.prefix.K = static_cast<const uint8_t *>(K) + off;
    a.prefix.V = static_cast<const uint8_t *>(V) + off;
  }
  if (pages) {
    a.tail.K = K_pages;
    a.tail.V = V_pages;
    a.table = table;
    a.kv_len = kv_len;
  }
  a.q_start = q_start; a.Q = Q; a.O = O; a.lse = lse; a.scale = scale;
  StageTimer t(ctx, st, JOLT_STAGE_PREFIX_ATTEND);
  HIP_OK(launch_prefix_attend(a, cut, d, dtype, ws, st));
  return JOLT_OK;
}
