// C entries of the serving operators: argument checks, then one launcher each.  Stateless; nothing here touches device
// memory.
#include <math.h>
#include <string.h>

#include <new>

#include "pt_serving.h"

// Whether pt_sample and pt_sample_bytes take this many rows and tokens (a grid holds less than 2^32 threads, 1024 to a row).
static int check_logits(int32_t rows, int32_t vocab) {
  if (rows < 0 || rows > (1 << 21) || vocab < 1 || vocab > (1 << 24))
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "rows must be in 0..2^21 and vocab in 1..2^24");
  return PT_OK;
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

static int check_cache(const pt_paged_cache* c) {
  if (!c) return pt_set_error(PT_ERR_NULL_POINTER, "cache is NULL");
  if (!c->k || !c->v) return pt_set_error(PT_ERR_NULL_POINTER, "the cache's k or v is NULL");
  if (!aligned16(c->k) || !aligned16(c->v)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the cache's k and v must be 16-byte aligned");
  if (c->dtype != PT_F32 && c->dtype != PT_BF16) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "dtype must be PT_F32 or PT_BF16");
  if (c->n_layers < 1 || c->n_pages < 1 || c->n_kv_heads < 1)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "n_layers, n_pages and n_kv_heads must be >= 1");
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)))
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "page_size = %d, need a power of two in 16..4096", c->page_size);
  if (c->head_dim < 8 || c->head_dim % 8 || c->head_dim > 256)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "head_dim must be a multiple of 8 in 8..256");
  const int64_t vec = c->dtype == PT_F32 ? 4 : 8;
  if (c->layer_stride < 0 || c->page_stride < 0 || c->head_stride < 0 || c->token_stride < c->head_dim ||
      c->token_stride > (1 << 24) || (int64_t)c->page_size * c->token_stride >= (int64_t)1 << 31)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the cache's strides are out of range");
  if (c->layer_stride % vec || c->page_stride % vec || c->head_stride % vec || c->token_stride % vec)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the cache's strides must be multiples of 16 bytes");
  return PT_OK;
}

static int check_layer(const pt_paged_cache* c, int32_t layer) {
  if (layer < 0 || layer >= c->n_layers) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "layer %d out of range", layer);
  return PT_OK;
}

// Whether a batch has no row: buffers of none may have no address.
static bool no_rows(const pt_paged_batch* b) { return b->n_seqs == 0 || b->total_rows == 0; }

// Checks the batch and resolves its unknown bounds.  need_ptrs: false where only sizes are asked for.
static int check_batch(const pt_paged_cache* c, const pt_paged_batch* b, bool need_ptrs, pt_paged_rows* r) {
  if (!b) return pt_set_error(PT_ERR_NULL_POINTER, "batch is NULL");
  if (b->n_seqs < 0 || b->total_rows < 0 || b->pages_stride < 0 || b->max_q_len < 0 || b->max_kv_len < 0)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "a size of the batch is negative");
  if (b->total_rows > (1 << 23)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "total_rows = %d exceeds 2^23", b->total_rows);
  if (need_ptrs && !no_rows(b)) {
    if (!b->row_start || !b->kv_len || (!b->pages && b->pages_stride > 0))
      return pt_set_error(PT_ERR_NULL_POINTER, "row_start, kv_len or pages is NULL");
    if (((uintptr_t)b->row_start | (uintptr_t)b->kv_len | (uintptr_t)b->pages | (uintptr_t)b->status) & 3)
      return pt_set_error(PT_ERR_INVALID_ARGUMENT, "row_start, kv_len, pages and status must be 4-byte aligned");
  }
  int shift = 0;
  while ((1 << shift) < c->page_size) ++shift;
  const int64_t room = b->pages_stride > (0x7fffffff >> shift) ? 0x7fffffff : b->pages_stride << shift;
  if (b->max_kv_len > room)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "max_kv_len = %d exceeds the %lld positions of a row of the page table", b->max_kv_len, (long long)room);
  r->row_start = b->row_start;
  r->kv_len = b->kv_len;
  r->pages = b->pages;
  r->pages_stride = b->pages_stride;
  r->status = b->status;
  r->n_seqs = b->n_seqs;
  r->total_rows = b->total_rows;
  r->max_q_len = b->max_q_len == 0 || b->max_q_len > b->total_rows ? b->total_rows : b->max_q_len;
  // positions stay below 2^31 - 2^20, so that sums with tile sizes do not overflow
  const int64_t cap = 0x7fffffff - (1 << 20);
  int64_t kv = b->max_kv_len == 0 ? room : b->max_kv_len;
  r->max_kv_len = (int32_t)(kv < cap ? kv : cap);
  r->n_pages = c->n_pages;
  r->page_shift = shift;
  return PT_OK;
}

static int check_rows(const pt_head_rows* h, int32_t dtype, const pt_paged_batch* b, const char* name) {
  if (!h || (!h->data && !no_rows(b))) return pt_set_error(PT_ERR_NULL_POINTER, "%s is NULL", name);
  const int64_t vec = dtype == PT_F32 ? 4 : 8;
  if (!aligned16(h->data)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "%s is not 16-byte aligned", name);
  if (h->row_stride < 0 || h->head_stride < 0 || h->row_stride % vec || h->head_stride % vec)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the strides of %s must be multiples of 16 bytes and not negative", name);
  return PT_OK;
}

static void* layer_of(void* base, const pt_paged_cache* c, int32_t layer) {
  return (char*)base + (size_t)(layer * c->layer_stride) * (c->dtype == PT_F32 ? 4 : 2);
}

extern "C" int pt_rope_init(pt_rope* out, int32_t layout, int32_t rotary_dim, double theta, int32_t scaling, double factor,
                            double low, double high, int32_t original_len, double magnitude) {
  if (!out) return pt_set_error(PT_ERR_NULL_POINTER, "out is NULL");
  if (layout != PT_ROPE_HALF && layout != PT_ROPE_INTERLEAVED) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "unknown rotary layout %d", layout);
  if (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > 256) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "rotary_dim must be even and in 2..256");
  if (!(theta > 0.0) || !isfinite(theta) || !isfinite(magnitude)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "theta must be positive, theta and magnitude finite");
  if (scaling < PT_ROPE_UNSCALED || scaling > PT_ROPE_BY_PARTS) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "unknown rotary scaling %d", scaling);
  if (scaling != PT_ROPE_UNSCALED && (!(factor > 0.0) || !isfinite(factor))) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "factor must be positive and finite");
  if (scaling == PT_ROPE_BY_PARTS && (!(low >= 0.0) || !(high > low) || !isfinite(high) || original_len < 1))
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "need 0 <= low < high and original_len >= 1");
  memset(out, 0, sizeof(*out));
  out->layout = layout;
  out->rotary_dim = rotary_dim;
  out->magnitude = magnitude;
  for (int j = 0; j < rotary_dim / 2; ++j) {
    double f = pow(theta, -2.0 * j / rotary_dim);
    if (scaling == PT_ROPE_LINEAR) f /= factor;
    if (scaling == PT_ROPE_BY_PARTS) {
      double w = (original_len * f / (2.0 * M_PI) - low) / (high - low);
      w = w < 0.0 ? 0.0 : w > 1.0 ? 1.0 : w;
      f *= w + (1.0 - w) / factor;
    }
    out->turns[j] = f / (2.0 * M_PI);
  }
  return PT_OK;
}

extern "C" int pt_paged_append(const pt_paged_cache* cache, int32_t layer, const pt_paged_batch* batch, const pt_rope* rope,
                               const pt_head_rows* q, const pt_head_rows* q_out, int32_t n_heads, const pt_head_rows* k,
                               const pt_head_rows* v, void* hip_stream) {
  pt_append_args a;
  memset(&a, 0, sizeof(a));
  int rc = check_cache(cache);
  if (!rc) rc = check_layer(cache, layer);
  if (!rc) rc = check_batch(cache, batch, true, &a.b);
  if (!rc) rc = check_rows(k, cache->dtype, batch, "k");
  if (!rc) rc = check_rows(v, cache->dtype, batch, "v");
  if (!rc && (q != nullptr) != (q_out != nullptr)) rc = pt_set_error(PT_ERR_NULL_POINTER, "q and q_out must both be given or both be NULL");
  if (!rc && q) {
    rc = check_rows(q, cache->dtype, batch, "q");
    if (!rc) rc = check_rows(q_out, cache->dtype, batch, "q_out");
    if (!rc && n_heads < 1) rc = pt_set_error(PT_ERR_INVALID_ARGUMENT, "n_heads must be >= 1");
    if (!rc && q->data && q->data == q_out->data && (q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
      rc = pt_set_error(PT_ERR_INVALID_ARGUMENT, "q_out is q with other strides");
  }
  // head numbers and their sums with a workgroup's passes are 32-bit
  if (!rc && (int64_t)(q ? n_heads : 0) + cache->n_kv_heads > 1 << 30) rc = pt_set_error(PT_ERR_INVALID_ARGUMENT, "more than 2^30 heads of queries and keys");
  if (rc) return rc;
  if (rope) {
    if ((rope->layout != PT_ROPE_HALF && rope->layout != PT_ROPE_INTERLEAVED) || rope->rotary_dim < 2 || rope->rotary_dim % 2 ||
        rope->rotary_dim > cache->head_dim)
      return pt_set_error(PT_ERR_INVALID_ARGUMENT, "the rotary description is not one of pt_rope_init for heads of %d", cache->head_dim);
  }
  if (no_rows(batch)) return PT_OK;
  if (q) {
    a.q = q->data; a.q_rs = q->row_stride; a.q_hs = q->head_stride;
    a.q_out = q_out->data; a.qo_rs = q_out->row_stride; a.qo_hs = q_out->head_stride;
    a.H = n_heads;
  }
  a.k = k->data; a.k_rs = k->row_stride; a.k_hs = k->head_stride;
  a.v = v->data; a.v_rs = v->row_stride; a.v_hs = v->head_stride;
  a.kc = layer_of(cache->k, cache, layer);
  a.vc = layer_of(cache->v, cache, layer);
  a.page_stride = cache->page_stride; a.head_stride = cache->head_stride; a.token_stride = cache->token_stride;
  a.Hkv = cache->n_kv_heads; a.hd = cache->head_dim;
  return pt_launch_paged_append(a, rope, cache->dtype, (hipStream_t)hip_stream);
}

// Plan of an attention call; sizes only.
static int plan_attention(const pt_paged_cache* cache, const pt_paged_batch* batch, int32_t n_heads, bool need_ptrs,
                          pt_paged_rows* rows, pt_paged_plan* plan) {
  int rc = check_cache(cache);
  if (!rc) rc = check_batch(cache, batch, need_ptrs, rows);
  if (rc) return rc;
  if (n_heads < 1 || n_heads % cache->n_kv_heads)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "n_kv_heads (%d) must divide n_heads (%d)", cache->n_kv_heads, n_heads);
  memset(plan, 0, sizeof(*plan));
  if (no_rows(batch)) return PT_OK;
  return pt_plan_paged_attn(cache->dtype, cache->head_dim, n_heads, cache->n_kv_heads, *rows, plan);
}

extern "C" int pt_paged_attention_bytes(const pt_paged_cache* cache, const pt_paged_batch* batch, int32_t n_heads, size_t* bytes) {
  if (!bytes) return pt_set_error(PT_ERR_NULL_POINTER, "bytes is NULL");
  pt_paged_rows rows;
  pt_paged_plan plan;
  const int rc = plan_attention(cache, batch, n_heads, false, &rows, &plan);
  if (rc) return rc;
  *bytes = plan.bytes;
  return PT_OK;
}

extern "C" int pt_paged_attention(const pt_paged_cache* cache, int32_t layer, const pt_paged_batch* batch, const pt_head_rows* q,
                                  const pt_head_rows* out, int32_t n_heads, float scale, int32_t causal, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  pt_paged_attn_args a;
  memset(&a, 0, sizeof(a));
  pt_paged_plan plan;
  int rc = plan_attention(cache, batch, n_heads, true, &a.b, &plan);
  if (!rc) rc = check_layer(cache, layer);
  if (!rc) rc = check_rows(q, cache->dtype, batch, "q");
  if (!rc) rc = check_rows(out, cache->dtype, batch, "out");
  if (rc) return rc;
  if (!isfinite(scale)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "scale is not finite");
  if (q->data && q->data == out->data && (q->row_stride != out->row_stride || q->head_stride != out->head_stride))
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "out is q with other strides");
  if (plan.bytes > 0) {
    if (!workspace) return pt_set_error(PT_ERR_NULL_POINTER, "workspace is NULL, %zu bytes needed", plan.bytes);
    if (!aligned16(workspace)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "workspace is not 16-byte aligned");
    if (workspace_bytes < plan.bytes)
      return pt_set_error(PT_ERR_ARENA_TOO_SMALL, "workspace: %zu bytes given, %zu needed", workspace_bytes, plan.bytes);
  }
  if (no_rows(batch)) return PT_OK;
  a.q = q->data; a.q_rs = q->row_stride; a.q_hs = q->head_stride;
  a.o = out->data; a.o_rs = out->row_stride; a.o_hs = out->head_stride;
  a.kc = layer_of(cache->k, cache, layer);
  a.vc = layer_of(cache->v, cache, layer);
  a.page_stride = cache->page_stride; a.head_stride = cache->head_stride; a.token_stride = cache->token_stride;
  a.part = (float*)workspace;
  a.part_rows[0] = plan.part_rows[0]; a.part_rows[1] = plan.part_rows[1]; a.seq_rows = plan.seq_rows;
  a.scale_log2 = scale == 0.0f ? 1.0f : (float)(fabs((double)scale) * 1.4426950408889634);
  a.q_sign = scale == 0.0f ? 0.0f : scale < 0.0f ? -1.0f : 1.0f;
  a.causal = causal != 0;
  a.H = n_heads; a.Hkv = cache->n_kv_heads; a.hd = cache->head_dim;
  a.few = plan.few; a.cut[0] = plan.cut[0]; a.cut[1] = plan.cut[1];
  return pt_launch_paged_attn(a, cache->dtype, (hipStream_t)hip_stream);
}

extern "C" int pt_page_copy(const pt_paged_cache* cache, const int32_t* host_pairs, int32_t n_pairs, void* hip_stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (n_pairs < 0) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "n_pairs is negative");
  if (n_pairs == 0) return PT_OK;
  if (!host_pairs) return pt_set_error(PT_ERR_NULL_POINTER, "host_pairs is NULL");
  for (int64_t i = 0; i < 2 * (int64_t)n_pairs; ++i)
    if (host_pairs[i] < 0 || host_pairs[i] >= cache->n_pages)
      return pt_set_error(PT_ERR_INVALID_ARGUMENT, "pair %lld names page %d of %d", (long long)(i / 2), host_pairs[i], cache->n_pages);
  // one bit per page that is written
  const size_t words = ((size_t)cache->n_pages + 63) / 64;
  uint64_t few[64];
  uint64_t* written = words <= 64 ? few : new (std::nothrow) uint64_t[words];
  if (!written) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "out of host memory");
  memset(written, 0, words * 8);
  int32_t twice = -1, both = -1;
  for (int64_t i = 0; i < n_pairs; ++i) {
    const int32_t d = host_pairs[2 * i + 1];
    if (written[d >> 6] >> (d & 63) & 1) twice = d;
    written[d >> 6] |= (uint64_t)1 << (d & 63);
  }
  for (int64_t i = 0; i < n_pairs; ++i) {
    const int32_t s = host_pairs[2 * i];
    if (written[s >> 6] >> (s & 63) & 1) both = s;
  }
  if (written != few) delete[] written;
  if (twice >= 0) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "page %d would be written twice", twice);
  if (both >= 0) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "page %d would be both read and written", both);
  return pt_launch_page_copy(*cache, host_pairs, n_pairs, (hipStream_t)hip_stream);
}

extern "C" int pt_sample_bytes(int32_t rows, int32_t vocab, size_t* bytes) {
  if (!bytes) return pt_set_error(PT_ERR_NULL_POINTER, "bytes is NULL");
  const int rc = check_logits(rows, vocab);
  if (rc) return rc;
  *bytes = rows == 0 ? 0 : pt_sample_workspace(rows, vocab);
  return PT_OK;
}

extern "C" int pt_sample(const float* dev_logits, int64_t row_stride, int32_t rows, int32_t vocab, const float* dev_uniform,
                         const float* dev_temperature, const int32_t* dev_top_k, const float* dev_top_p, const float* dev_min_p,
                         int32_t* dev_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_logits(rows, vocab);
  if (rc) return rc;
  if (rows == 0) return PT_OK;
  if (!dev_logits || !dev_uniform || !dev_out) return pt_set_error(PT_ERR_NULL_POINTER, "logits, uniform or out is NULL");
  if (row_stride < 0 || (rows > 1 && row_stride < vocab)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "row_stride is below vocab");
  if (((uintptr_t)dev_logits | (uintptr_t)dev_uniform | (uintptr_t)dev_temperature | (uintptr_t)dev_top_k | (uintptr_t)dev_top_p |
       (uintptr_t)dev_min_p | (uintptr_t)dev_out) & 3)
    return pt_set_error(PT_ERR_INVALID_ARGUMENT, "a pointer is not aligned to its elements");
  const size_t need = pt_sample_workspace(rows, vocab);
  if (need > 0) {
    if (!workspace) return pt_set_error(PT_ERR_NULL_POINTER, "workspace is NULL, %zu bytes needed", need);
    if (!aligned16(workspace)) return pt_set_error(PT_ERR_INVALID_ARGUMENT, "workspace is not 16-byte aligned");
    if (workspace_bytes < need) return pt_set_error(PT_ERR_ARENA_TOO_SMALL, "workspace: %zu bytes given, %zu needed", workspace_bytes, need);
  }
  const pt_sample_args a = {dev_logits, row_stride, dev_uniform, dev_temperature, dev_top_k, dev_top_p, dev_min_p, dev_out, workspace, rows, vocab, 0, 0};
  return pt_launch_sample(a, (hipStream_t)hip_stream);
}
