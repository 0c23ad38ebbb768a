// C entries of the 8-bit cache: argument checks and launch plans.  Nothing is allocated or kept.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/osprey.h"
#include "kv8.h"

#define OSPREY_API extern "C" __attribute__((visibility("default")))

namespace {

using namespace osp;

int fail(int code, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return report_error(code, buf);
}

// (rows x heads fit a grid and an int)
constexpr long kMaxRowCount = 1L << 22, kMaxRowHeads = 1L << 28;

int check_cache(const osprey_kv8_cache* c) {
  if (!c) return fail(OSPREY_E_INVALID, "the cache is NULL");
  if (!c->page_table || !c->codes || !c->scales) return fail(OSPREY_E_INVALID, "page_table, codes and scales must be non-NULL");
  if (c->batch < 1 || c->batch > 4096) return fail(OSPREY_E_INVALID, "batch %d not in [1, 4096]", c->batch);
  if (c->max_pages < 1 || c->max_pages > 1 << 25) return fail(OSPREY_E_INVALID, "max_pages %d not in [1, 2^25]", c->max_pages);
  if (c->num_pages < 1) return fail(OSPREY_E_INVALID, "num_pages %d", c->num_pages);
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024) return fail(OSPREY_E_SHAPE, "n_kv_heads %d not in [1, 1024]", c->n_kv_heads);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(OSPREY_E_UNSUPPORTED, "head_dim %d (supported: 64, 128)", c->head_dim);
  if (((uintptr_t)c->codes & 15) || c->page_stride % 16)
    return fail(OSPREY_E_INVALID, "codes and page_stride must be multiples of 16 bytes");
  if (c->page_stride < 2L * c->n_kv_heads * kKv8Page * c->head_dim)
    return fail(OSPREY_E_SHAPE, "page_stride %ld < %ld", (long)c->page_stride, 2L * c->n_kv_heads * kKv8Page * c->head_dim);
  if ((uintptr_t)c->scales & 3) return fail(OSPREY_E_INVALID, "scales must be 4-byte aligned");
  if (c->scale_stride < 2L * c->n_kv_heads)
    return fail(OSPREY_E_SHAPE, "scale_stride %ld < %d", (long)c->scale_stride, 2 * c->n_kv_heads);
  return OSPREY_OK;
}

int check_rows(const osprey_kv8_cache* c, int rows, const int32_t* cu, const int32_t* cached) {
  if (!cached) return fail(OSPREY_E_INVALID, "cached is NULL");
  if (rows < 0 || rows > kMaxRowCount) return fail(OSPREY_E_INVALID, "rows %d not in [0, %ld]", rows, kMaxRowCount);
  if (!cu && rows != c->batch) return fail(OSPREY_E_SHAPE, "%d rows for %d sequences need cu_rows", rows, c->batch);
  return OSPREY_OK;
}

// Rows of `heads` heads, `stride` elements apart, on 16-byte boundaries.
int check_buffer(const char* name, const void* p, long stride, int heads, int hd, int dtype) {
  const int el = dtype == OSPREY_BF16 ? 2 : 4;
  if (!p) return fail(OSPREY_E_INVALID, "%s is NULL", name);
  if (((uintptr_t)p & 15) || stride * el % 16) return fail(OSPREY_E_INVALID, "%s: rows must lie on 16-byte boundaries", name);
  if (stride < (long)heads * hd) return fail(OSPREY_E_SHAPE, "%s: stride %ld < %ld", name, stride, (long)heads * hd);
  return OSPREY_OK;
}

int check_heads(const osprey_kv8_cache* c, int nq, int rows) {
  if ((long)rows * nq > kMaxRowHeads) return fail(OSPREY_E_UNSUPPORTED, "%d rows of %d heads: over 2^28", rows, nq);
  if (nq < 1 || nq > 4096 || nq % c->n_kv_heads)
    return fail(OSPREY_E_SHAPE, "n_q_heads %d must be a multiple of n_kv_heads %d, at most 4096", nq, c->n_kv_heads);
  return OSPREY_OK;
}

Kv8Pool pool_of(const osprey_kv8_cache* c) {
  Kv8Pool p{};
  p.table = c->page_table;
  p.max_pages = c->max_pages;
  p.num_pages = c->num_pages;
  p.codes = (uint8_t*)c->codes;
  p.page_stride = c->page_stride;
  p.scales = c->scales;
  p.scale_stride = c->scale_stride;
  p.nkv = c->n_kv_heads;
  return p;
}

int done() {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(OSPREY_E_DEVICE, "kernel launch: %s", hipGetErrorString(e));
  return report_error(OSPREY_OK, "");
}

// CUs of the current device, looked up once per device (0: none).
int compute_units() {
  constexpr int kMaxDev = 64;
  static int known[kMaxDev];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  if (dev < kMaxDev && __atomic_load_n(&known[dev], __ATOMIC_RELAXED) > 0) return __atomic_load_n(&known[dev], __ATOMIC_RELAXED);
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  if (dev < kMaxDev) __atomic_store_n(&known[dev], n, __ATOMIC_RELAXED);
  return n;
}

constexpr int kSplitQuantum = 128;
constexpr long kPartBytes = 256L << 20;

struct AttnPlan {
  int form, n_split, tiles, items, by_units;
  size_t ns_bytes, part_bytes;
};
AttnPlan attention_plan(int batch, int nkv, int hd, int rows, int nq, int x_bf16, int max_rows, int max_context, int max_pages,
                        int n_cu) {
  AttnPlan p{};
  p.form = kv8_attention_form(x_bf16, nq / nkv, max_rows, (long)batch * max_context, nkv);
  const int cols = kv8_form_cols(p.form, x_bf16);
  p.tiles = (int)((long)rows * (nq / nkv) / cols) + batch;
  // Eight wavefronts per CU: what registers leave resident with 128-wide heads.  (With 64-wide ones
  // twelve are, but more items make shorter splits: 4 sequences of 500 rows over 4000 positions take
  // 120 us unsplit and 162 in three blocks' worth.)
  p.items = std::max(1, ((p.form == kKv8Shared ? 1 : 2) * n_cu + nkv - 1) / nkv);
  p.n_split = (int)std::min<long>(kKv8MaxSplits, std::max(1L, ((long)max_context + kSplitQuantum - 1) / kSplitQuantum));
  // A pass that fills the chip with its tiles is not cut.  The partials of others take 256 MB at most,
  // or what twice the even deal needs: enough for one long context among many short ones.
  const long full = (long)rows * (nq / nkv) / cols;
  if (full >= p.items) {
    p.n_split = 1;
  } else if (rows > 0) {
    const long room = kPartBytes / ((long)rows * nq * (hd + 2) * 4);
    p.n_split = (int)std::min<long>(p.n_split, std::max(room, 2L * p.items / std::max(full, 1L) + 2));
  }
  // (splits by units may begin anywhere in a sequence: one more; their count fits an int)
  p.by_units = p.n_split > 1 && p.form != kKv8Prompt && (long)p.tiles * (max_pages / 8 + 1) < 1L << 30;
  if (p.by_units) p.n_split = std::min(p.n_split + 1, kKv8MaxSplits);
  if (p.n_split > 1) {
    p.ns_bytes = ((size_t)rows * nq * 4 + 255) & ~size_t(255);
    p.part_bytes = (size_t)rows * nq * p.n_split * (hd + 2) * 4;
  }
  return p;
}

}  // namespace

OSPREY_API int osprey_kv8_append(const osprey_kv8_cache* c, const osprey_kv8_append_args* a, void* hip_stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!a) return fail(OSPREY_E_INVALID, "the arguments are NULL");
  if ((rc = check_rows(c, a->rows, a->cu_rows, a->cached))) return rc;
  if (a->rows == 0) return report_error(OSPREY_OK, "");   // nothing to do
  if (a->dtype != OSPREY_F32 && a->dtype != OSPREY_BF16) return fail(OSPREY_E_INVALID, "dtype %d", a->dtype);
  if ((rc = check_buffer("k", a->k, a->k_stride, c->n_kv_heads, c->head_dim, a->dtype))) return rc;
  if ((rc = check_buffer("v", a->v, a->v_stride, c->n_kv_heads, c->head_dim, a->dtype))) return rc;
  if (a->q) {
    if (a->n_q_heads < 1 || a->n_q_heads > 4096) return fail(OSPREY_E_SHAPE, "n_q_heads %d not in [1, 4096]", a->n_q_heads);
    if ((long)a->rows * a->n_q_heads > kMaxRowHeads)
      return fail(OSPREY_E_UNSUPPORTED, "%d rows of %d heads: over 2^28", a->rows, a->n_q_heads);
    if ((rc = check_buffer("q", a->q, a->q_stride, a->n_q_heads, c->head_dim, a->dtype))) return rc;
    if ((rc = check_buffer("q_out", a->q_out, a->q_out_stride, a->n_q_heads, c->head_dim, a->dtype))) return rc;
    if (a->q_out == a->q && a->q_out_stride != a->q_stride)
      return fail(OSPREY_E_INVALID, "q_out in place of q needs its stride");
  }
  if ((a->q_norm || a->k_norm) && !(a->eps > 0.f && std::isfinite(a->eps))) return fail(OSPREY_E_INVALID, "eps must be > 0");
  if (!a->rope_cos != !a->rope_sin) return fail(OSPREY_E_INVALID, "rope_cos and rope_sin go together");
  if (a->rope_cos && a->rope_len < 1) return fail(OSPREY_E_INVALID, "rope_len %d", a->rope_len);
  Kv8AppendArgs k{};
  k.pool = pool_of(c);
  k.r = Kv8Rows{c->batch, a->rows, nullptr, a->cu_rows, a->cached, nullptr};
  k.rope_pos = a->rope_pos;
  k.x_bf16 = k.g_bf16 = a->dtype == OSPREY_BF16;
  k.q = a->q;
  k.k = a->k;
  k.v = a->v;
  k.ldq = a->q_stride;
  k.ldk = a->k_stride;
  k.ldv = a->v_stride;
  k.ks = 1;
  k.nq = a->q ? a->n_q_heads : 0;
  k.hd = c->head_dim;
  k.q_norm = a->q_norm;
  k.k_norm = a->k_norm;
  k.eps = a->eps;
  k.rope_cos = a->rope_cos;
  k.rope_sin = a->rope_sin;
  k.max_pos = a->rope_len;
  k.q_out = a->q_out;
  k.ldo = a->q_out_stride;
  k.q_scale = 1.f;
  k.err = a->err;
  if (!launch_kv8_append(k, (hipStream_t)hip_stream))
    return fail(OSPREY_E_UNSUPPORTED, "%d rows of %d kv heads and %d query heads: more than a grid holds", a->rows, c->n_kv_heads, k.nq);
  return done();
}

OSPREY_API size_t osprey_kv8_workspace_bytes(const osprey_kv8_cache* c, int32_t rows, int32_t n_q_heads, int32_t max_rows,
                                             int32_t max_context) {
  if (check_cache(c) || check_heads(c, n_q_heads, rows)) return 0;
  if (rows < 0 || rows > kMaxRowCount || max_rows < 1 || max_context < 1) {
    fail(OSPREY_E_INVALID, "rows %d, max_rows %d, max_context %d", rows, max_rows, max_context);
    return 0;
  }
  const int n_cu = compute_units();
  if (n_cu < 1) {
    fail(OSPREY_E_DEVICE, "no HIP device");
    return 0;
  }
  size_t need = 256;
  for (int bf16 = 0; bf16 < 2; ++bf16) {   // (of either type of rows)
    const AttnPlan p = attention_plan(c->batch, c->n_kv_heads, c->head_dim, rows, n_q_heads, bf16, max_rows, max_context, c->max_pages, n_cu);
    need = std::max(need, p.ns_bytes + p.part_bytes);
  }
  report_error(OSPREY_OK, "");
  return need;
}

OSPREY_API int osprey_kv8_attention(const osprey_kv8_cache* c, const osprey_kv8_attention_args* a, void* hip_stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!a) return fail(OSPREY_E_INVALID, "the arguments are NULL");
  if ((rc = check_rows(c, a->rows, a->cu_rows, a->cached))) return rc;
  if (a->rows == 0) return report_error(OSPREY_OK, "");   // nothing to do
  if ((rc = check_heads(c, a->n_q_heads, a->rows))) return rc;
  if (a->dtype != OSPREY_F32 && a->dtype != OSPREY_BF16) return fail(OSPREY_E_INVALID, "dtype %d", a->dtype);
  if (a->max_rows < 1 || a->max_context < 1)
    return fail(OSPREY_E_INVALID, "max_rows %d and max_context %d must be at least 1", a->max_rows, a->max_context);
  if (a->tree_mask && a->max_rows > 128) return fail(OSPREY_E_SHAPE, "a tree mask takes at most 128 rows a sequence, max_rows is %d", a->max_rows);
  if ((uintptr_t)a->tree_mask & 7) return fail(OSPREY_E_INVALID, "tree_mask must be 8-byte aligned");
  // (scores are taken to base 2)
  if (!(a->scale > 0.f && std::isfinite(a->scale * 1.4426950408889634f))) return fail(OSPREY_E_INVALID, "scale must be > 0 and finite over ln 2");
  if ((rc = check_buffer("q", a->q, a->q_stride, a->n_q_heads, c->head_dim, a->dtype))) return rc;
  if ((rc = check_buffer("out", a->out, a->out_stride, a->n_q_heads, c->head_dim, a->dtype))) return rc;
  const int n_cu = compute_units();
  if (n_cu < 1) return fail(OSPREY_E_DEVICE, "no HIP device");
  const AttnPlan p = attention_plan(c->batch, c->n_kv_heads, c->head_dim, a->rows, a->n_q_heads, a->dtype == OSPREY_BF16,
                                    a->max_rows, a->max_context, c->max_pages, n_cu);
  if (p.part_bytes > 0) {
    if (!a->workspace || ((uintptr_t)a->workspace & 15)) return fail(OSPREY_E_INVALID, "workspace must be non-NULL and 16-byte aligned");
    if (a->workspace_bytes < p.ns_bytes + p.part_bytes)
      return fail(OSPREY_E_CAPACITY, "workspace_bytes %zu < %zu", a->workspace_bytes, p.ns_bytes + p.part_bytes);
  }
  Kv8AttnArgs k{};
  k.pool = pool_of(c);
  k.r = Kv8Rows{c->batch, a->rows, nullptr, a->cu_rows, a->cached, nullptr};
  k.x_bf16 = a->dtype == OSPREY_BF16;
  k.q = a->q;
  k.ldq = a->q_stride;
  k.nq = a->n_q_heads;
  k.hd = c->head_dim;
  k.scale = a->scale;
  k.tree = a->tree_mask;
  k.form = p.form;
  k.n_split = p.n_split;
  k.items = p.items;
  k.by_units = p.by_units;
  k.tiles = p.tiles;
  // (a last-level cache of 256 MB: contexts beyond it are not read again soon)
  k.stream = (long)c->batch * a->max_context * c->n_kv_heads * c->head_dim * 2 > (160L << 20);
  k.out = a->out;
  k.ldo = a->out_stride;
  k.err = a->err;
  if (p.n_split > 1) {
    k.row_ns = (int32_t*)a->workspace;
    k.part = (float*)((char*)a->workspace + p.ns_bytes);
  }
  launch_kv8_attention(k, (hipStream_t)hip_stream);
  if (p.n_split > 1) launch_kv8_join(k, (hipStream_t)hip_stream);
  return done();
}

OSPREY_API int osprey_kv8_keep(const osprey_kv8_cache* c, const osprey_kv8_keep_args* a, void* hip_stream) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!a || !a->base || !a->path || !a->n) return fail(OSPREY_E_INVALID, "base, path and n must be non-NULL");
  if (a->path_stride < 1) return fail(OSPREY_E_SHAPE, "path_stride %d", a->path_stride);
  Kv8KeepArgs k{};
  k.pool = pool_of(c);
  k.B = c->batch;
  k.hd = c->head_dim;
  k.base = a->base;
  k.path = a->path;
  k.ld = a->path_stride;
  k.n = a->n;
  k.err = a->err;
  launch_kv8_keep(k, (hipStream_t)hip_stream);
  return done();
}
