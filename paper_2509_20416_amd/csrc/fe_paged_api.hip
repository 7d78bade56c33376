// fe_paged_api.hip -- C entry points of the paged cache and of tree attention
// (include/fe.h): argument checks, then one launcher call.
#include <math.h>
#include <stdio.h>

#include "fe_host.h"
#include "fe_paged.h"

using namespace fe;

namespace {

bool aligned4(const void *p) { return ((uintptr_t)p & 3u) == 0; }

int es_of(int dtype) { return dtype == FE_F32 ? 4 : dtype == FE_BF16 ? 2 : 1; }

fe_status check_cache(const fe_paged_kv *c) {
  if (!c) return fail(FE_E_INVALID, "cache is NULL");
  if (c->dtype != FE_F32 && c->dtype != FE_BF16 && c->dtype != FE_F8)
    return fail(FE_E_INVALID, "unknown cache dtype %d", c->dtype);
  if (c->n_pages <= 0 || c->page_rows <= 0 || c->n_kv_heads <= 0)
    return fail(FE_E_INVALID, "cache has a non-positive size");
  if (c->page_rows < 16 || c->page_rows > 65536 || (c->page_rows & (c->page_rows - 1)))
    return fail(FE_E_UNSUPPORTED, "page_rows must be a power of two, 16 .. 65536");
  if ((int64_t)c->n_pages * c->page_rows > INT32_MAX) return fail(FE_E_UNSUPPORTED, "the pool has more than 2^31 - 1 rows");
  if (c->n_kv_heads > 256) return fail(FE_E_UNSUPPORTED, "n_kv_heads > 256");
  if (c->head_dim != 64 && c->head_dim != 128) return fail(FE_E_UNSUPPORTED, "head_dim must be 64 or 128");
  if (!c->k || !c->v) return fail(FE_E_INVALID, "cache keys or values are NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(FE_E_ALIGN, "the cache must be 16-byte aligned");
  if (c->dtype == FE_F8) {
    if (!c->k_scale || !c->v_scale) return fail(FE_E_INVALID, "an 8-bit cache needs its scales");
    if (!aligned4(c->k_scale) || !aligned4(c->v_scale))
      return fail(FE_E_ALIGN, "the scales must be 4-byte aligned");
  }
  return FE_OK;
}

fe_status check_table(const fe_paged_kv *c, const fe_page_table *t) {
  if (!t) return fail(FE_E_INVALID, "page table is NULL");
  if (!t->pages) return fail(FE_E_INVALID, "page ids are NULL");
  if (!aligned4(t->pages)) return fail(FE_E_ALIGN, "page ids must be 4-byte aligned");
  if (t->max_pages < 1 || t->max_len < 1 || t->max_len > (int64_t)t->max_pages * c->page_rows)
    return fail(FE_E_INVALID, "max_len %d outside [1, max_pages * page_rows]", t->max_len);
  if (t->max_len > 1 << 30) return fail(FE_E_UNSUPPORTED, "max_len > 2^30");
  return FE_OK;
}

fe_status check_dtype(const fe_paged_kv *c, int32_t dtype) {
  if (dtype != FE_F32 && dtype != FE_BF16) return fail(FE_E_INVALID, "unknown dtype %d", dtype);
  if (c->dtype != dtype && c->dtype != FE_F8)
    return fail(FE_E_UNSUPPORTED, "a cache of dtype %d takes and serves rows of its own dtype", c->dtype);
  return FE_OK;
}

// Rows of `width` elements, `stride` apart.
fe_status check_rows(const char *name, const void *p, int64_t stride, int64_t width, int32_t dtype) {
  if (!p) return fail(FE_E_INVALID, "%s is NULL", name);
  if (!aligned16(p)) return fail(FE_E_ALIGN, "%s must be 16-byte aligned", name);
  if (stride < width || stride > (int64_t)1 << 31)
    return fail(FE_E_INVALID, "the row stride of %s is below a row or above 2^31", name);
  if (stride * es_of(dtype) % 16) return fail(FE_E_ALIGN, "the row stride of %s must be a multiple of 16 bytes", name);
  return FE_OK;
}

fe_status check_batch(int32_t batch, int32_t nodes) {
  if (batch < 0 || batch > 65535) return fail(FE_E_INVALID, "batch %d outside [0, 65535]", batch);
  if (nodes < 0 || (int64_t)batch * nodes > (1 << 30))
    return fail(FE_E_INVALID, "nodes %d is negative or batch * nodes exceeds 2^30", nodes);
  return FE_OK;
}

bool overlap(const void *a, int64_t na, const void *b, int64_t nb) {
  return (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

PagedView view(const fe_paged_kv *c, const fe_page_table *t) {
  PagedView v;
  v.k = c->k;
  v.v = c->v;
  v.ks = c->k_scale;
  v.vs = c->v_scale;
  v.pages = t->pages;
  v.n_pages = c->n_pages;
  v.shift = __builtin_ctz((unsigned)c->page_rows);
  v.max_pages = t->max_pages;
  v.max_len = t->max_len;
  v.Hkv = c->n_kv_heads;
  v.D = c->head_dim;
  v.dtype = c->dtype;
  return v;
}

#define FE_CHECK(x)                   \
  do {                                \
    const fe_status st_ = (x);        \
    if (st_ != FE_OK) return st_;     \
  } while (0)

// Checks that fe_tree_attention and its workspace size share.
fe_status check_attention(const fe_paged_kv *cache, const fe_page_table *table, int32_t batch, int32_t nodes,
                          int32_t n_q_heads, int32_t dtype) {
  FE_CHECK(check_cache(cache));
  FE_CHECK(check_table(cache, table));
  FE_CHECK(check_dtype(cache, dtype));
  FE_CHECK(check_batch(batch, nodes));
  if (n_q_heads < 1 || n_q_heads % cache->n_kv_heads)
    return fail(FE_E_INVALID, "n_q_heads must be a positive multiple of n_kv_heads");
  if (n_q_heads > 1024) return fail(FE_E_UNSUPPORTED, "n_q_heads > 1024");
  if ((int64_t)nodes * (n_q_heads / cache->n_kv_heads) > (1 << 20))
    return fail(FE_E_UNSUPPORTED, "nodes * n_q_heads / n_kv_heads > 2^20");
  if ((int64_t)cache->n_kv_heads * table->max_len > (int64_t)1 << 36)
    return fail(FE_E_UNSUPPORTED, "n_kv_heads * max_len > 2^36");
  return FE_OK;
}

}  // namespace

extern "C" fe_status fe_rope_frequencies(int32_t rotary_dim, double theta, int32_t scaling, double factor,
                                         double low, double high, double trained_len, double *freqs,
                                         float *magnitude) {
  if (!freqs || !magnitude) return fail(FE_E_INVALID, "frequency outputs are NULL");
  if (rotary_dim < 2 || rotary_dim % 2) return fail(FE_E_INVALID, "rotary_dim must be positive and even");
  if (!(theta > 1.0) || !isfinite(theta)) return fail(FE_E_INVALID, "theta must be finite and above 1");
  if (scaling < FE_SCALE_NONE || scaling > FE_SCALE_RAMP) return fail(FE_E_INVALID, "unknown scaling %d", scaling);
  if (scaling != FE_SCALE_NONE && (!(factor >= 1.0) || !isfinite(factor)))
    return fail(FE_E_INVALID, "factor must be finite and at least 1");
  const bool bands = scaling == FE_SCALE_BANDED || scaling == FE_SCALE_RAMP;
  if (bands && (!(low > 0.0) || !(high > low) || !isfinite(high)))
    return fail(FE_E_INVALID, "low must be positive and below high");
  if (bands && (!(trained_len >= 1.0) || !isfinite(trained_len)))
    return fail(FE_E_INVALID, "trained_len must be at least 1");
  const double kTwoPi = 6.283185307179586476925286766559;
  const int half = rotary_dim / 2;
  double a = 0.0, b = 1.0;
  *magnitude = 1.f;
  if (scaling == FE_SCALE_RAMP) {
    auto index = [&](double turns) {
      return rotary_dim * log(trained_len / (kTwoPi * turns)) / (2.0 * log(theta));
    };
    a = fmax(floor(index(high)), 0.0);
    b = fmin(ceil(index(low)), half - 1.0);
    if (!(b > a)) b = a + 0.001;
    *magnitude = (float)(0.1 * log(factor) + 1.0);
  }
  for (int m = 0; m < half; ++m) {
    const double w = pow(theta, -2.0 * m / rotary_dim);
    double f = w;
    if (scaling == FE_SCALE_LINEAR) f = w / factor;
    if (scaling == FE_SCALE_BANDED) {
      const double s = fmin(1.0, fmax(0.0, (trained_len * w / kTwoPi - low) / (high - low)));
      f = (1.0 - s) * w / factor + s * w;
    }
    if (scaling == FE_SCALE_RAMP) {
      const double r = fmin(1.0, fmax(0.0, (m - a) / (b - a)));
      f = w / factor * r + w * (1.0 - r);
    }
    freqs[m] = f;
  }
  return FE_OK;
}

extern "C" fe_status fe_cache_append(const fe_paged_kv *cache, const fe_page_table *table, int32_t batch,
                                     int32_t nodes, const int32_t *starts, const int32_t *counts,
                                     const int32_t *positions, const fe_rope *rope, int32_t dtype,
                                     const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                     const void *q, int64_t q_stride, int32_t n_q_heads, void *q_out,
                                     void *stream) {
  const Range range("fe_cache_append");
  FE_CHECK(check_cache(cache));
  FE_CHECK(check_table(cache, table));
  FE_CHECK(check_dtype(cache, dtype));
  FE_CHECK(check_batch(batch, nodes));
  if (batch == 0 || nodes == 0) return FE_OK;
  const int64_t kvw = (int64_t)cache->n_kv_heads * cache->head_dim;
  FE_CHECK(check_rows("k", k, k_stride, kvw, dtype));
  FE_CHECK(check_rows("v", v, v_stride, kvw, dtype));
  if (q) {
    if (n_q_heads < 1 || n_q_heads > 1024) return fail(FE_E_INVALID, "n_q_heads %d outside [1, 1024]", n_q_heads);
    const int64_t qw = (int64_t)n_q_heads * cache->head_dim, rows = (int64_t)batch * nodes;
    FE_CHECK(check_rows("q", q, q_stride, qw, dtype));
    FE_CHECK(check_rows("q_out", q_out, qw, qw, dtype));
    if (overlap(q, ((rows - 1) * q_stride + qw) * es_of(dtype), q_out, rows * qw * es_of(dtype)))
      return fail(FE_E_INVALID, "q_out overlaps q");
  }
  if (!starts) return fail(FE_E_INVALID, "starts is NULL");
  if (!aligned4(starts) || !aligned4(counts) || !aligned4(positions))
    return fail(FE_E_ALIGN, "starts, counts and positions must be 4-byte aligned");
  RopeArgs r{nullptr, 0, 0, 1.f};
  if (rope) {
    if (!rope->freqs) return fail(FE_E_INVALID, "rope->freqs is NULL");
    if ((uintptr_t)rope->freqs & 7u) return fail(FE_E_ALIGN, "rope->freqs must be 8-byte aligned");
    if (rope->rotary_dim < 1 || rope->rotary_dim > cache->head_dim)
      return fail(FE_E_INVALID, "rotary_dim %d outside [1, head_dim]", rope->rotary_dim);
    if (rope->rotary_dim % 16) return fail(FE_E_UNSUPPORTED, "rotary_dim must be a multiple of 16");
    if (rope->layout != FE_ROPE_HALF && rope->layout != FE_ROPE_INTERLEAVED)
      return fail(FE_E_INVALID, "unknown rope layout %d", rope->layout);
    if (!(rope->magnitude > 0.f) || !isfinite(rope->magnitude))
      return fail(FE_E_INVALID, "rope->magnitude must be positive and finite");
    r = RopeArgs{rope->freqs, rope->rotary_dim, rope->layout == FE_ROPE_INTERLEAVED, rope->magnitude};
  }
  FE_TRY(cache_append(view(cache, table), batch, nodes, starts, counts, positions, r, dtype, k, (long)k_stride, v,
                      (long)v_stride, q, (long)q_stride, n_q_heads, q_out, (hipStream_t)stream));
  return FE_OK;
}

extern "C" fe_status fe_cache_gather(const fe_paged_kv *cache, const fe_page_table *table, int32_t batch,
                                     const int32_t *starts, const int32_t *cu_rows, int32_t n_rows,
                                     int32_t dtype, void *k_out, void *v_out, void *stream) {
  const Range range("fe_cache_gather");
  FE_CHECK(check_cache(cache));
  FE_CHECK(check_table(cache, table));
  if (dtype != FE_F32 && dtype != FE_BF16) return fail(FE_E_INVALID, "unknown dtype %d", dtype);
  FE_CHECK(check_batch(batch, 1));
  if (n_rows < 0) return fail(FE_E_INVALID, "n_rows is negative");
  if (!k_out && !v_out) return fail(FE_E_INVALID, "k_out and v_out are both NULL");
  if (!aligned16(k_out) || !aligned16(v_out)) return fail(FE_E_ALIGN, "k_out and v_out must be 16-byte aligned");
  if (batch == 0 || n_rows == 0) return FE_OK;
  if (!cu_rows) return fail(FE_E_INVALID, "cu_rows is NULL");
  if (!aligned4(cu_rows) || !aligned4(starts)) return fail(FE_E_ALIGN, "cu_rows and starts must be 4-byte aligned");
  FE_TRY(cache_gather(view(cache, table), batch, starts, cu_rows, n_rows, dtype, k_out, v_out,
                      (hipStream_t)stream));
  return FE_OK;
}

extern "C" size_t fe_tree_attention_workspace_bytes(const fe_paged_kv *cache, const fe_page_table *table,
                                                    int32_t batch, int32_t nodes, int32_t n_q_heads,
                                                    int32_t dtype) {
  if (check_attention(cache, table, batch, nodes, n_q_heads, dtype) != FE_OK) return 0;
  return tree_attention_ws(view(cache, table), batch, nodes, n_q_heads, dtype);
}

extern "C" fe_status fe_tree_attention(const fe_paged_kv *cache, const fe_page_table *table, int32_t batch,
                                       int32_t nodes, int32_t n_q_heads, const int32_t *prefix_lens,
                                       const int32_t *counts, const uint8_t *mask, int32_t dtype,
                                       const void *q, int64_t q_stride, float scale, void *out,
                                       void *workspace, size_t ws_bytes, void *stream) {
  const Range range("fe_tree_attention");
  FE_CHECK(check_attention(cache, table, batch, nodes, n_q_heads, dtype));
  if (batch == 0 || nodes == 0) return FE_OK;
  const int64_t qw = (int64_t)n_q_heads * cache->head_dim, rows = (int64_t)batch * nodes;
  FE_CHECK(check_rows("q", q, q_stride, qw, dtype));
  FE_CHECK(check_rows("out", out, qw, qw, dtype));
  if (overlap(q, ((rows - 1) * q_stride + qw) * es_of(dtype), out, rows * qw * es_of(dtype)))
    return fail(FE_E_INVALID, "out overlaps q");
  if (!prefix_lens) return fail(FE_E_INVALID, "prefix_lens is NULL");
  if (!aligned4(prefix_lens) || !aligned4(counts))
    return fail(FE_E_ALIGN, "prefix_lens and counts must be 4-byte aligned");
  if (!(scale > 0.f) || !isfinite(scale)) return fail(FE_E_INVALID, "scale must be positive and finite");
  const PagedView c = view(cache, table);
  const size_t need = tree_attention_ws(c, batch, nodes, n_q_heads, dtype);
  if (!workspace || ws_bytes < need)
    return fail(FE_E_WORKSPACE, "workspace needs %zu bytes, got %zu", need, workspace ? ws_bytes : 0);
  if ((uintptr_t)workspace & 255u) return fail(FE_E_ALIGN, "workspace must be 256-byte aligned");
  const TreeArgs a{c, batch, nodes, n_q_heads, prefix_lens, counts, mask, q, (long)q_stride, scale, out,
                   (float *)workspace};
  FE_TRY(tree_attention(a, dtype, (hipStream_t)stream));
  return FE_OK;
}

extern "C" fe_status fe_cache_commit(const fe_paged_kv *caches, int32_t n_layers, const fe_page_table *table,
                                     int32_t batch, int32_t nodes, int32_t n_paths, int32_t depth,
                                     const int32_t *prefix_lens, const int32_t *retrieve,
                                     const int32_t *accept_path, const int32_t *accept_len,
                                     int32_t *new_lens, void *stream) {
  const Range range("fe_cache_commit");
  if (!caches) return fail(FE_E_INVALID, "caches is NULL");
  if (n_layers < 1 || n_layers > 1024) return fail(FE_E_INVALID, "n_layers %d outside [1, 1024]", n_layers);
  CommitPool pools[1024];
  for (int l = 0; l < n_layers; ++l) {
    const fe_paged_kv &c = caches[l];
    FE_CHECK(check_cache(&c));
    if (c.n_pages != caches[0].n_pages || c.page_rows != caches[0].page_rows || c.dtype != caches[0].dtype ||
        c.n_kv_heads != caches[0].n_kv_heads || c.head_dim != caches[0].head_dim)
      return fail(FE_E_INVALID, "layer %d's cache has another shape than layer 0's", l);
    pools[l] = CommitPool{(char *)c.k, (char *)c.v, c.k_scale, c.v_scale};
  }
  FE_CHECK(check_table(caches, table));
  FE_CHECK(check_batch(batch, nodes));
  if (nodes < 1 || n_paths < 1) return fail(FE_E_INVALID, "a tree has at least one node and one path");
  if (depth < 0) return fail(FE_E_INVALID, "depth is negative");
  if (depth > kCommitDepth) return fail(FE_E_UNSUPPORTED, "depth > %d", kCommitDepth);
  if (batch == 0) return FE_OK;
  if (!prefix_lens || !retrieve || !accept_path || !accept_len || !new_lens)
    return fail(FE_E_INVALID, "every commit input and output is required");
  const void *ptrs[] = {prefix_lens, retrieve, accept_path, accept_len, new_lens};
  for (const void *p : ptrs)
    if (!aligned4(p)) return fail(FE_E_ALIGN, "commit arrays must be 4-byte aligned");
  const void *in[] = {prefix_lens, accept_path, accept_len};
  for (const void *p : in)
    if (overlap(p, 4 * (int64_t)batch, new_lens, 4 * (int64_t)batch))
      return fail(FE_E_INVALID, "new_lens overlaps an input");
  for (int l = 1; l < n_layers; ++l)
    for (int m = 0; m < l; ++m)
      if (pools[l].k == pools[m].k || pools[l].v == pools[m].v)
        return fail(FE_E_INVALID, "layers %d and %d share a cache", m, l);
  FE_TRY(cache_commit(view(caches, table), pools, n_layers, batch, nodes, n_paths, depth, prefix_lens, retrieve,
                      accept_path, accept_len, new_lens, (hipStream_t)stream));
  return FE_OK;
}
