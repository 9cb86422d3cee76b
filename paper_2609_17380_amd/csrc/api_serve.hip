// api_serve.hip - the C ABI of what a model answers with: products in int8 with a step per token, rotary positions, the paged
// cache in 8 bits and attention over it.  Argument checks and launches; no memory is allocated on the device.
#include <hip/hip_runtime.h>
#include <math.h>

#include <initializer_list>

#include "canon.h"
#include "canon_internal.h"

using namespace canon;

namespace {

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
canon_status dev(hipError_t e) { return e == hipSuccess ? CANON_OK : CANON_EDEVICE; }
bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool dtype_ok(int32_t t) { return t == CANON_F32 || t == CANON_BF16; }
int64_t dtype_size(int32_t t) { return t == CANON_F32 ? 4 : 2; }

constexpr int64_t kMaxElements = int64_t(1) << 40;

// a * b <= most, all >= 0
bool product_ok(int64_t a, int64_t b, int64_t most) { return a == 0 || b == 0 || a <= most / b; }

// A device range that a call reads or writes; of null pointers and empty ranges there is nothing to check.
struct Range {
  const void* p;
  int64_t bytes;
  bool out;
};
bool apart(std::initializer_list<Range> ranges) {
  for (const Range* a = ranges.begin(); a != ranges.end(); ++a)
    for (const Range* b = a + 1; b != ranges.end(); ++b) {
      if ((!a->out && !b->out) || !a->p || !b->p || a->bytes <= 0 || b->bytes <= 0) continue;
      const uintptr_t x = (uintptr_t)a->p, y = (uintptr_t)b->p;
      if (x < y + (uintptr_t)b->bytes && y < x + (uintptr_t)a->bytes) return false;
    }
  return true;
}

// bytes from a matrix's first element to its last: rows of `width`, `stride` apart
int64_t span(int64_t rows, int64_t width, int64_t stride, int64_t size) {
  return rows > 0 && width > 0 ? ((rows - 1) * stride + width) * size : 0;
}

// rows of `width` elements `stride` apart: a pointer that its type allows, a stride that holds a row
canon_status check_rows(const void* p, int64_t rows, int64_t width, int64_t stride, int64_t size) {
  if (stride < width) return CANON_EINVAL;
  if (rows > 0 && width > 0 && (!p || !aligned(p, size))) return CANON_EINVAL;
  if (!product_ok(rows, stride, kMaxElements * 16)) return CANON_EUNSUPPORTED;
  return CANON_OK;
}

canon_status check_turn(const canon_rotation* r, int64_t dim, Turn& t) {
  t = Turn{nullptr, nullptr, 0, 0, 0};
  if (!r) return CANON_OK;
  if (r->rot_dim < 0 || r->rot_dim % 2 || r->rot_dim > dim || r->positions < 0 || (r->interleaved != 0 && r->interleaved != 1))
    return CANON_EINVAL;
  if (r->rot_dim > 0 && r->positions > 0 && (!r->cos || !r->sin || !aligned(r->cos, 4) || !aligned(r->sin, 4)))
    return CANON_EINVAL;
  if (r->positions > (int64_t(1) << 31)) return CANON_EUNSUPPORTED;
  t = Turn{r->cos, r->sin, r->positions, r->rot_dim, r->interleaved};
  return CANON_OK;
}
int64_t table_bytes(const Turn& t) { return 4 * t.positions * (t.rot / 2); }

int page_log2(int64_t page) {
  switch (page) {
    case 16: return 4;
    case 32: return 5;
    case 64: return 6;
    case 128: return 7;
    case 256: return 8;
  }
  return 0;
}

canon_status check_cache(const canon_kv_cache* c, CacheView& v) {
  if (!c || c->n_pages < 0 || c->n_kv_heads < 1 || c->head_dim < 1 || c->batch < 0 || c->table_len < 0 || !page_log2(c->page))
    return CANON_EINVAL;
  if (c->head_dim % 32 || c->head_dim > 256 || c->n_kv_heads > 65535 || c->batch > 65535 || c->n_pages > 0x7FFFFFFF ||
      !product_ok(c->n_pages, c->n_kv_heads * c->page * c->head_dim, int64_t(1) << 44) || c->table_len > 0x7FFFFFFF)
    return CANON_EUNSUPPORTED;
  if (c->n_pages > 0 && (!c->k_codes || !c->v_codes || !c->k_steps || !c->v_steps)) return CANON_EINVAL;
  if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16) || !aligned(c->k_steps, 16) || !aligned(c->v_steps, 16) ||
      !aligned(c->table, 4))
    return CANON_EINVAL;
  if (c->batch > 0 && c->table_len > 0 && !c->table) return CANON_EINVAL;
  v = CacheView{c->k_codes, c->v_codes, c->k_steps, c->v_steps, c->table, c->n_pages, c->table_len, c->batch,
                page_log2(c->page), (int32_t)c->n_kv_heads, (int32_t)c->head_dim};
  return CANON_OK;
}
int64_t cache_codes(const canon_kv_cache* c) { return c->n_pages * c->n_kv_heads * c->page * c->head_dim; }
int64_t cache_steps(const canon_kv_cache* c) { return 4 * c->n_pages * c->n_kv_heads * c->page; }
int64_t cache_table(const canon_kv_cache* c) { return 4 * c->batch * c->table_len; }

canon_status check_new_rows(const canon_kv_cache* c, const canon_cache_rows* r, CacheRowsArgs& v) {
  if (!r || r->q_len < 0 || !aligned(r->q_starts, 4) || !aligned(r->q_lens, 4)) return CANON_EINVAL;
  if (r->q_start > (int64_t(1) << 30) || r->q_start < -(int64_t(1) << 30) || r->q_len > (int64_t(1) << 27) ||
      !product_ok(c->batch * c->n_kv_heads * c->head_dim, r->q_len, int64_t(1) << 33))
    return CANON_EUNSUPPORTED;
  v = CacheRowsArgs{r->q_len, r->q_start, r->q_starts, r->q_lens};
  return CANON_OK;
}

}  // namespace

// ---- products in int8 with a step per token --------------------------------------------------------------------------

canon_status canon_quant_tokens(int64_t rows, int64_t cols, int32_t in_dtype, const void* x, int8_t* codes, float* steps,
                                void* stream) {
  if (rows < 0 || cols < 0 || !dtype_ok(in_dtype)) return CANON_EINVAL;
  if (rows > (int64_t(1) << 31) || cols > 65536) return CANON_EUNSUPPORTED;
  if (rows == 0) return CANON_OK;
  if (!steps || !aligned(steps, 4) || (cols > 0 && (!x || !codes || !aligned(x, dtype_size(in_dtype))))) return CANON_EINVAL;
  const int64_t n = rows * cols;
  if (!apart({{x, n * dtype_size(in_dtype), false}, {codes, n, true}, {steps, 4 * rows, true}})) return CANON_EINVAL;
  return dev(quant_tokens_launch(rows, cols, in_dtype == CANON_BF16, x, codes, steps, as_stream(stream)));
}

canon_status canon_gemm_i8_tokens(int64_t m, int64_t n, int64_t k, const int8_t* a, int64_t lda, const float* sa,
                                  const int8_t* b, int64_t ldb, const float* sb, int32_t y_dtype, void* y, int64_t ldc,
                                  void* stream) {
  if (m < 0 || n < 0 || k < 0 || lda < k || ldb < k || ldc < n || !dtype_ok(y_dtype)) return CANON_EINVAL;
  if (k > 65536 || m > (int64_t(1) << 31) || n > (int64_t(1) << 31) || !product_ok(m, ldc, kMaxElements) ||
      !product_ok(m, lda, kMaxElements) || !product_ok(n, ldb, kMaxElements))
    return CANON_EUNSUPPORTED;
  // workgroups of a launch stay below 2^32 threads (at least 64 x 8 outputs each)
  if (!product_ok((m + 63) / 64, (n + 7) / 8, int64_t(1) << 23)) return CANON_EUNSUPPORTED;
  if (m == 0 || n == 0) return CANON_OK;
  if ((k > 0 && (!a || !b)) || !y || !sa || !sb || !aligned(y, dtype_size(y_dtype)) || !aligned(sa, 4) || !aligned(sb, 4))
    return CANON_EINVAL;
  if (!apart({{a, span(m, k, lda, 1), false}, {b, span(n, k, ldb, 1), false}, {sa, 4 * m, false}, {sb, 4 * n, false},
              {y, span(m, n, ldc, dtype_size(y_dtype)), true}}))
    return CANON_EINVAL;
  GemmI8Args g{};
  g.a = a; g.b = b; g.y = (float*)y; g.sa = sa; g.sb = sb;
  g.m = m; g.n = n; g.k = k; g.lda = lda; g.ldb = ldb; g.ldc = ldc;
  g.sa_rows = 1;
  g.y_bf16 = y_dtype == CANON_BF16;
  return dev(gemm_i8_launch(g, as_stream(stream)));
}

// ---- rotary positions -----------------------------------------------------------------------------------------------------

canon_status canon_rope_tables(int32_t rot_dim, double theta, const canon_rope_scaling* scaling, int64_t first,
                               int64_t positions, float* cos_out, float* sin_out) {
  if (rot_dim < 2 || rot_dim % 2 || rot_dim > 1024 || !(theta > 0.0) || !(theta < INFINITY) || first < 0 || positions < 0)
    return CANON_EINVAL;
  if (first > (int64_t(1) << 31) || positions > (int64_t(1) << 31) - first) return CANON_EUNSUPPORTED;
  if (positions > 0 && (!cos_out || !sin_out)) return CANON_EINVAL;
  canon_rope_scaling s{CANON_ROPE_PLAIN, 1.0, 0.0, 1.0, 1.0, 1.0};
  if (scaling) s = *scaling;
  if (s.amplitude == 0.0) s.amplitude = 1.0;
  if (s.kind < CANON_ROPE_PLAIN || s.kind > CANON_ROPE_BANDS || !(fabs(s.amplitude) < INFINITY)) return CANON_EINVAL;
  if (s.kind != CANON_ROPE_PLAIN && (!(s.factor >= 1.0) || !(s.factor < INFINITY))) return CANON_EINVAL;
  if (s.kind == CANON_ROPE_BASE && rot_dim == 2) return CANON_EINVAL;
  if (s.kind == CANON_ROPE_BANDS &&
      (!(s.low >= 0.0) || !(s.low < s.high) || !(s.high < INFINITY) || !(s.context > 0.0) || !(s.context < INFINITY)))
    return CANON_EINVAL;
  const int32_t half = rot_dim / 2;
  double w[512];
  for (int32_t i = 0; i < half; ++i) {
    double base = theta;
    if (s.kind == CANON_ROPE_BASE) base = theta * pow(s.factor, (double)rot_dim / (double)(rot_dim - 2));
    w[i] = pow(base, -2.0 * i / rot_dim);
    if (s.kind == CANON_ROPE_LINEAR) w[i] /= s.factor;
    if (s.kind == CANON_ROPE_BANDS) {
      const double turns = s.context * w[i] / (2.0 * 3.14159265358979323846);
      double g = (turns - s.low) / (s.high - s.low);
      g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
      w[i] *= g + (1.0 - g) / s.factor;
    }
  }
  for (int64_t p = 0; p < positions; ++p)
    for (int32_t i = 0; i < half; ++i) {
      const double angle = (double)(first + p) * w[i];
      cos_out[p * half + i] = (float)(s.amplitude * cos(angle));
      sin_out[p * half + i] = (float)(s.amplitude * sin(angle));
    }
  return CANON_OK;
}

canon_status canon_rope(int32_t backward, int64_t tokens, int64_t n_heads, int64_t head_dim, const canon_rotation* rotation,
                        const int32_t* positions, int32_t x_dtype, const void* x, int64_t x_stride, int32_t y_dtype, void* y,
                        int64_t y_stride, void* stream) {
  if ((backward != 0 && backward != 1) || tokens < 0 || n_heads < 0 || head_dim < 0 || !rotation || !dtype_ok(x_dtype) ||
      !dtype_ok(y_dtype) || !aligned(positions, 4))
    return CANON_EINVAL;
  if (head_dim > 1024 || n_heads > (1 << 20) || !product_ok(tokens, n_heads * head_dim, kMaxElements)) return CANON_EUNSUPPORTED;
  Turn t;
  canon_status st = check_turn(rotation, head_dim, t);
  const int64_t width = n_heads * head_dim, xs = dtype_size(x_dtype), ys = dtype_size(y_dtype);
  if (st == CANON_OK) st = check_rows(x, tokens, width, x_stride, xs);
  if (st == CANON_OK) st = check_rows(y, tokens, width, y_stride, ys);
  if (st != CANON_OK) return st;
  if (tokens == 0 || width == 0) return CANON_OK;
  const int64_t xb = span(tokens, width, x_stride, xs), yb = span(tokens, width, y_stride, ys), tb = table_bytes(t);
  const bool in_place = x == y && x_dtype == y_dtype && x_stride == y_stride;
  if (!apart({{in_place ? nullptr : x, xb, false}, {y, yb, true}, {t.cos, tb, false}, {t.sin, tb, false},
              {positions, 4 * tokens, false}}))
    return CANON_EINVAL;
  return dev(rope_launch(backward, tokens, n_heads, head_dim, t, positions, x_dtype == CANON_BF16, x, x_stride,
                         y_dtype == CANON_BF16, y, y_stride, as_stream(stream)));
}

// ---- the cache --------------------------------------------------------------------------------------------------------------

canon_status canon_cache_append(const canon_kv_cache* cache, const canon_cache_rows* rows, int32_t in_dtype, const void* k,
                                int64_t k_stride, const void* v, int64_t v_stride, const canon_rotation* rotation,
                                void* stream) {
  CacheView c;
  CacheRowsArgs r;
  Turn t;
  canon_status st = check_cache(cache, c);
  if (st == CANON_OK) st = check_new_rows(cache, rows, r);
  if (st == CANON_OK) st = check_turn(rotation, cache->head_dim, t);
  if (st != CANON_OK) return st;
  if (!dtype_ok(in_dtype)) return CANON_EINVAL;
  const int64_t n = cache->batch * rows->q_len, width = cache->n_kv_heads * cache->head_dim, size = dtype_size(in_dtype);
  st = check_rows(k, n, width, k_stride, size);
  if (st == CANON_OK) st = check_rows(v, n, width, v_stride, size);
  if (st != CANON_OK) return st;
  if (n == 0 || cache->n_pages == 0 || cache->table_len == 0) return CANON_OK;
  const int64_t codes = cache_codes(cache), steps = cache_steps(cache);
  if (!apart({{c.kc, codes, true}, {c.vc, codes, true}, {c.ks, steps, true}, {c.vs, steps, true},
              {c.table, cache_table(cache), false}, {k, span(n, width, k_stride, size), false},
              {v, span(n, width, v_stride, size), false}, {t.cos, table_bytes(t), false}, {t.sin, table_bytes(t), false},
              {r.q_starts, 4 * cache->batch, false}, {r.q_lens, 4 * cache->batch, false}}))
    return CANON_EINVAL;
  return dev(cache_append_launch(c, r, in_dtype == CANON_BF16, k, k_stride, v, v_stride, t, as_stream(stream)));
}

canon_status canon_cache_read(const canon_kv_cache* cache, const canon_cache_rows* rows, int32_t out_dtype, void* k, void* v,
                              void* stream) {
  CacheView c;
  CacheRowsArgs r;
  canon_status st = check_cache(cache, c);
  if (st == CANON_OK) st = check_new_rows(cache, rows, r);
  if (st != CANON_OK) return st;
  if (!dtype_ok(out_dtype) || !aligned(k, dtype_size(out_dtype)) || !aligned(v, dtype_size(out_dtype))) return CANON_EINVAL;
  const int64_t n = cache->batch * rows->q_len * cache->n_kv_heads * cache->head_dim * dtype_size(out_dtype);
  if (n == 0 || (!k && !v)) return CANON_OK;
  const int64_t codes = cache_codes(cache), steps = cache_steps(cache);
  if (!apart({{c.kc, codes, false}, {c.vc, codes, false}, {c.ks, steps, false}, {c.vs, steps, false},
              {c.table, cache_table(cache), false}, {k, n, true}, {v, n, true}, {r.q_starts, 4 * cache->batch, false},
              {r.q_lens, 4 * cache->batch, false}}))
    return CANON_EINVAL;
  return dev(cache_read_launch(c, r, out_dtype == CANON_BF16, k, v, as_stream(stream)));
}

// ---- attention over it --------------------------------------------------------------------------------------------------------

namespace {
canon_status check_attention(const canon_kv_cache* cache, const canon_attn_rows* rows, CacheAttnArgs& a) {
  canon_status st = check_cache(cache, a.c);
  if (st != CANON_OK) return st;
  if (!rows || rows->batch != cache->batch || rows->n_heads < 1 || rows->n_heads % cache->n_kv_heads || rows->q_len < 0 ||
      rows->k_len < 0 || rows->ld != 0 || rows->window < 0 || (rows->causal != 0 && rows->causal != 1) ||
      rows->k_len > cache->table_len * cache->page || (rows->k_len > 0 && cache->n_pages < 1) || !aligned(rows->q_starts, 4) || !aligned(rows->q_lens, 4) ||
      !aligned(rows->k_lens, 4))
    return CANON_EINVAL;
  if (rows->k_len > (int64_t(1) << 21) || rows->n_heads >= (1 << 24) ||
      !product_ok(rows->batch * rows->n_heads, rows->q_len, (int64_t(1) << 24) - 1) || rows->q_start > (int64_t(1) << 30) ||
      rows->q_start < -(int64_t(1) << 30))
    return CANON_EUNSUPPORTED;
  a.q_len = rows->q_len;
  a.k_len = rows->k_len;
  a.q_start = rows->q_start;
  a.window = rows->window < (int64_t(1) << 33) ? rows->window : int64_t(1) << 33;  // wider than any distance
  a.q_starts = rows->q_starts;
  a.q_lens = rows->q_lens;
  a.k_lens = rows->k_lens;
  a.heads = (int32_t)rows->n_heads;
  a.causal = rows->causal;
  a.scale = rows->scale;
  return CANON_OK;
}
}  // namespace

size_t canon_cache_attention_workspace_bytes(const canon_kv_cache* cache, const canon_attn_rows* rows) {
  CacheAttnArgs a{};
  if (check_attention(cache, rows, a) != CANON_OK) return 0;
  return cache_attention_workspace(a);
}

canon_status canon_cache_attention(const canon_order* order, const canon_kv_cache* cache, const canon_attn_rows* rows,
                                   int32_t q_dtype, const void* q, int64_t q_stride, uint16_t* out, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (!order) return CANON_EINVAL;
  if (order->version != 1 || order->chunk != 32 || order->tree != CANON_TREE_BINARY_CARRY || order->ftz != 1)
    return CANON_EUNSUPPORTED;
  CacheAttnArgs a{};
  canon_status st = check_attention(cache, rows, a);
  if (st != CANON_OK) return st;
  if (!dtype_ok(q_dtype)) return CANON_EINVAL;
  const int64_t n = cache->batch * rows->q_len, width = rows->n_heads * cache->head_dim, size = dtype_size(q_dtype);
  st = check_rows(q, n, width, q_stride, size);
  if (st != CANON_OK) return st;
  if (n == 0) return CANON_OK;
  if (!out || !aligned(out, 2)) return CANON_EINVAL;
  const size_t need = cache_attention_workspace(a);
  if (need > 0 && (!workspace || !aligned(workspace, 256))) return CANON_EINVAL;
  if (workspace_bytes < need) return CANON_EWORKSPACE;
  const int64_t codes = cache_codes(cache), steps = cache_steps(cache), lens = 4 * cache->batch;
  if (!apart({{a.c.kc, codes, false}, {a.c.vc, codes, false}, {a.c.ks, steps, false}, {a.c.vs, steps, false},
              {a.c.table, cache_table(cache), false}, {q, span(n, width, q_stride, size), false}, {out, 2 * n * width, true},
              {workspace, (int64_t)need, true}, {a.q_starts, lens, false}, {a.q_lens, lens, false}, {a.k_lens, lens, false}}))
    return CANON_EINVAL;
  a.q = q;
  a.q_bf16 = q_dtype == CANON_BF16;
  a.q_stride = q_stride;
  a.out = out;
  a.parts = (float*)workspace;
  return dev(cache_attention_launch(a, as_stream(stream)));
}
