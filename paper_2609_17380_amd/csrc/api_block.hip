// api_block.hip - the C ABI of the operators around a block: layer norm, activations kept in 8 bits, SwiGLU from them and
// attention rows with a relative position bias.  Argument checks and launches; no memory is allocated on the device.
#include <hip/hip_runtime.h>
#include <string.h>

#include <initializer_list>

#include "canon.h"
#include "canon_internal.h"

using namespace canon;

namespace {

hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }
canon_status dev(hipError_t e) { return e == hipSuccess ? CANON_OK : CANON_EDEVICE; }

canon_status check_order(const canon_order* o) {
  if (!o) return CANON_EINVAL;
  if (o->version != 1 || o->chunk != 32 || o->tree != CANON_TREE_BINARY_CARRY || o->ftz != 1)
    return CANON_EUNSUPPORTED;
  return CANON_OK;
}

constexpr int64_t kMaxElements = int64_t(1) << 40;
constexpr int64_t kMaxRows = int64_t(1) << 26;

// rows * cols within `most`, both >= 0
bool product_ok(int64_t rows, int64_t cols, int64_t most) { return rows == 0 || cols == 0 || rows <= most / cols; }

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

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
bool dtype_ok(int32_t t) { return t == CANON_F32 || t == CANON_BF16; }
int64_t dtype_size(int32_t t) { return t == CANON_F32 ? 4 : 2; }

// log2 of a group, 0 for none of the four
int group_log2(int32_t group) {
  switch (group) {
    case 32: return 5;
    case 64: return 6;
    case 128: return 7;
    case 256: return 8;
  }
  return 0;
}
int64_t groups_of(int64_t cols, int32_t group) { return cols / group + (cols % group != 0); }

canon_status check_kept(const canon_act8* k, int64_t elements) {
  if (!group_log2(k->group)) return CANON_EINVAL;
  if (elements > 0 && (!k->codes || !k->steps || !aligned(k->steps, 4))) return CANON_EINVAL;
  return CANON_OK;
}

// the input of a backward pass: x of a type, or what it was kept as
canon_status input_of(int32_t dtype, const void* x, const canon_act8* kept, int64_t elements, ActIn& in) {
  if (kept) {
    if (x) return CANON_EINVAL;
    canon_status st = check_kept(kept, elements);
    if (st != CANON_OK) return st;
    in = ActIn{kept->codes, kept->steps, ACT_Q8, group_log2(kept->group)};
    return CANON_OK;
  }
  if (!dtype_ok(dtype) || (elements > 0 && (!x || !aligned(x, dtype_size(dtype))))) return CANON_EINVAL;
  in = ActIn{x, nullptr, dtype == CANON_F32 ? ACT_F32 : ACT_BF16, 0};
  return CANON_OK;
}

ActKeep keep_of(const canon_act8* kept) {
  if (!kept) return ActKeep{nullptr, nullptr, 5};
  return ActKeep{kept->codes, kept->steps, group_log2(kept->group)};
}

int64_t step_bytes(int64_t rows, int64_t cols, const canon_act8* k) { return k ? 4 * rows * groups_of(cols, k->group) : 0; }

}  // namespace

// ---- activations kept in 8 bits -------------------------------------------------------------------------------------

int64_t canon_act8_groups(int64_t cols, int32_t group) {
  if (cols < 0 || !group_log2(group)) return 0;
  return groups_of(cols, group);
}

canon_status canon_act8_pack(int64_t rows, int64_t cols, int32_t in_dtype, const void* x, const canon_act8* kept,
                             void* stream) {
  if (rows < 0 || cols < 0 || !kept || !dtype_ok(in_dtype)) return CANON_EINVAL;
  if (!product_ok(rows, cols, kMaxElements)) return CANON_EUNSUPPORTED;
  const int64_t n = rows * cols;
  canon_status st = check_kept(kept, n);
  if (st != CANON_OK) return st;
  if (n == 0) return CANON_OK;
  ActIn in;
  st = input_of(in_dtype, x, nullptr, n, in);
  if (st != CANON_OK) return st;
  if (!apart({{x, n * dtype_size(in_dtype), false}, {kept->codes, n, true}, {kept->steps, step_bytes(rows, cols, kept), true}}))
    return CANON_EINVAL;
  return dev(act8_pack_launch(rows, cols, in, keep_of(kept), as_stream(stream)));
}

canon_status canon_act8_unpack(int64_t rows, int64_t cols, const canon_act8* kept, int32_t out_dtype, void* out,
                               void* stream) {
  if (rows < 0 || cols < 0 || !kept || !dtype_ok(out_dtype)) return CANON_EINVAL;
  if (!product_ok(rows, cols, kMaxElements)) return CANON_EUNSUPPORTED;
  const int64_t n = rows * cols;
  ActIn in;
  canon_status st = input_of(0, nullptr, kept, n, in);
  if (st != CANON_OK) return st;
  if (n == 0) return CANON_OK;
  if (!out || !aligned(out, dtype_size(out_dtype))) return CANON_EINVAL;
  if (!apart({{kept->codes, n, false}, {kept->steps, step_bytes(rows, cols, kept), false}, {out, n * dtype_size(out_dtype), true}}))
    return CANON_EINVAL;
  return dev(act8_unpack_launch(rows, cols, in, out_dtype == CANON_BF16, out, as_stream(stream)));
}

canon_status canon_swiglu(int64_t T, int64_t F, int32_t in_dtype, const void* gu, uint16_t* a, const canon_act8* kept,
                          void* stream) {
  if (T < 0 || F < 0 || !dtype_ok(in_dtype)) return CANON_EINVAL;
  if (!product_ok(T, F, kMaxElements / 2)) return CANON_EUNSUPPORTED;
  const int64_t n = T * F;
  ActIn in;
  canon_status st = input_of(in_dtype, gu, nullptr, n, in);
  if (st == CANON_OK && kept) st = check_kept(kept, n);
  if (st != CANON_OK) return st;
  if (n == 0) return CANON_OK;
  if (!a || !aligned(a, 2)) return CANON_EINVAL;
  if (!apart({{gu, 2 * n * dtype_size(in_dtype), false}, {a, 2 * n, true}, {kept ? kept->codes : nullptr, 2 * n, true},
              {kept ? kept->steps : nullptr, step_bytes(2 * T, F, kept), true}}))
    return CANON_EINVAL;
  return dev(swiglu_keep_launch(T, F, in, a, keep_of(kept), as_stream(stream)));
}

canon_status canon_swiglu_bwd(int64_t T, int64_t F, int32_t in_dtype, const void* gu, const canon_act8* kept,
                              const float* da, uint16_t* dgu, uint16_t* a, void* stream) {
  if (T < 0 || F < 0) return CANON_EINVAL;
  if (!product_ok(T, F, kMaxElements / 2)) return CANON_EUNSUPPORTED;
  const int64_t n = T * F;
  ActIn in;
  canon_status st = input_of(in_dtype, gu, kept, n, in);
  if (st != CANON_OK) return st;
  if (n == 0) return CANON_OK;
  if (!da || !dgu || !aligned(da, 4) || !aligned(dgu, 2) || !aligned(a, 2)) return CANON_EINVAL;
  if (!apart({{in.x, kept ? 2 * n : 2 * n * dtype_size(in_dtype), false}, {in.steps, step_bytes(2 * T, F, kept), false},
              {da, 4 * n, false}, {dgu, 4 * n, true}, {a, 2 * n, true}}))
    return CANON_EINVAL;
  return dev(swiglu_grad_launch(T, F, in, da, dgu, a, as_stream(stream)));
}

// ---- layer norm --------------------------------------------------------------------------------------------------------

canon_status canon_layernorm(const canon_order* order, int64_t rows, int64_t cols, int32_t x_dtype, const void* x,
                             const uint16_t* gain, const uint16_t* bias, float eps, int32_t y_dtype, void* y,
                             float* mean, float* rstd, const canon_act8* kept, void* stream) {
  canon_status st = check_order(order);
  if (st != CANON_OK) return st;
  if (rows < 0 || cols < 1 || !dtype_ok(x_dtype) || !dtype_ok(y_dtype)) return CANON_EINVAL;
  if (cols > 32768 || rows > kMaxRows) return CANON_EUNSUPPORTED;  // a workgroup holds 16 parts of 2048 columns
  const int64_t n = rows * cols;
  ActIn in;
  st = input_of(x_dtype, x, nullptr, n, in);
  if (st == CANON_OK && kept) st = check_kept(kept, n);
  if (st != CANON_OK) return st;
  if (rows == 0) return CANON_OK;
  if (!gain || !y || !mean || !rstd || !aligned(gain, 2) || !aligned(bias, 2) || !aligned(y, dtype_size(y_dtype)) ||
      !aligned(mean, 4) || !aligned(rstd, 4))
    return CANON_EINVAL;
  if (!apart({{x, n * dtype_size(x_dtype), false}, {gain, 2 * cols, false}, {bias, 2 * cols, false},
              {y, n * dtype_size(y_dtype), true}, {mean, 4 * rows, true}, {rstd, 4 * rows, true},
              {kept ? kept->codes : nullptr, n, true}, {kept ? kept->steps : nullptr, step_bytes(rows, cols, kept), true}}))
    return CANON_EINVAL;
  return dev(layernorm_fwd_launch(rows, cols, in, gain, bias, eps, y_dtype == CANON_BF16, y, mean, rstd, keep_of(kept),
                                  as_stream(stream)));
}

size_t canon_layernorm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 1 || cols > 32768 || rows > kMaxRows) return 0;
  return sizeof(float) * (size_t)layernorm_part_floats(rows, cols);
}

canon_status canon_layernorm_bwd(const canon_order* order, int64_t rows, int64_t cols, int32_t x_dtype, const void* x,
                                 const canon_act8* kept, const uint16_t* gain, const float* mean, const float* rstd,
                                 const float* dy, float* dx, float* dgain, float* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  canon_status st = check_order(order);
  if (st != CANON_OK) return st;
  if (rows < 0 || cols < 1) return CANON_EINVAL;
  if (cols > 32768 || rows > kMaxRows) return CANON_EUNSUPPORTED;
  const int64_t n = rows * cols;
  ActIn in;
  st = input_of(x_dtype, x, kept, n, in);
  if (st != CANON_OK) return st;
  if (!aligned(dgain, 4) || !aligned(dbias, 4)) return CANON_EINVAL;
  if (rows > 0 && (!gain || !mean || !rstd || !dy || !dx || !aligned(gain, 2) || !aligned(mean, 4) || !aligned(rstd, 4) ||
                   !aligned(dy, 4) || !aligned(dx, 4)))
    return CANON_EINVAL;
  const size_t need = dgain || dbias ? canon_layernorm_bwd_workspace_bytes(rows, cols) : 0;
  if (need > 0) {
    if (workspace_bytes < need) return CANON_EWORKSPACE;
    if (!workspace || !aligned(workspace, 256)) return CANON_EINVAL;
  }
  if (!apart({{in.x, kept ? n : n * dtype_size(x_dtype), false}, {in.steps, step_bytes(rows, cols, kept), false},
              {gain, 2 * cols, false}, {mean, 4 * rows, false}, {rstd, 4 * rows, false}, {dy, 4 * n, false},
              {dx, 4 * n, true}, {dgain, 4 * cols, true}, {dbias, 4 * cols, true}, {workspace, (int64_t)need, true}}))
    return CANON_EINVAL;
  return dev(layernorm_bwd_launch(rows, cols, in, gain, mean, rstd, dy, dx, dgain, dbias, (float*)workspace,
                                  as_stream(stream)));
}

// ---- attention rows with a relative position bias -------------------------------------------------------------------

namespace {

static_assert(CANON_RELBIAS_MAX_STARTS == kRelStarts, "the record holds what the kernels take");

// A whole number of up to 40 words of 32 bits, for the exact comparison of canon_relbias_log: at most 1024^64 64^64, 33
// words.
struct Whole {
  uint32_t w[40] = {1};
  int n = 1;
  Whole& power(uint32_t base, int times) {
    for (int t = 0; t < times; ++t) {
      uint64_t carry = 0;
      for (int i = 0; i < n; ++i) {
        carry += (uint64_t)w[i] * base;
        w[i] = (uint32_t)carry;
        carry >>= 32;
      }
      if (carry) w[n++] = (uint32_t)carry;
    }
    return *this;
  }
  bool at_least(const Whole& o) const {
    if (n != o.n) return n > o.n;
    for (int i = n; i-- > 0;)
      if (w[i] != o.w[i]) return w[i] > o.w[i];
    return true;
  }
};

bool bias_ok(const canon_relbias* r) {
  if (!r || r->n_starts < 1 || r->n_starts > CANON_RELBIAS_MAX_STARTS || (r->bidirectional != 0 && r->bidirectional != 1))
    return false;
  if (r->start[0] != 0) return false;
  for (int i = 1; i < r->n_starts; ++i)
    if (r->start[i] < r->start[i - 1]) return false;
  return true;
}

int64_t buckets_of(const canon_relbias* b) { return (int64_t)b->n_starts * (b->bidirectional ? 2 : 1); }

constexpr int64_t kMaxStart = int64_t(1) << 30;
constexpr int64_t kMaxAttnRows = int64_t(1) << 31;
constexpr int64_t kMaxLd = int64_t(1) << 31;
constexpr int64_t kMaxTable = int64_t(1) << 24;  // columns of the rows' sums: a launch folds 16 threads to each

canon_status check_rows(const canon_attn_rows* r, const canon_relbias* bias) {
  if (!r || r->batch < 0 || r->n_heads < 0 || r->q_len < 0 || r->k_len < 0 || r->window < 0 ||
      (r->causal != 0 && r->causal != 1) || (r->ld != 0 && r->ld < r->k_len) || r->q_start < -kMaxStart ||
      r->q_start > kMaxStart)
    return CANON_EINVAL;
  if (!bias_ok(bias)) return CANON_EINVAL;
  if (bias->start[bias->n_starts - 1] > kRelFar) return CANON_EUNSUPPORTED;
  if (r->k_len > 32768 || r->ld > kMaxLd) return CANON_EUNSUPPORTED;
  if (!product_ok(r->batch, r->n_heads, kMaxAttnRows) || !product_ok(r->batch * r->n_heads, r->q_len, kMaxAttnRows) ||
      r->batch > kMaxAttnRows || r->q_len > kMaxAttnRows || !product_ok(r->n_heads, buckets_of(bias), kMaxTable) ||
      !product_ok(r->batch * r->n_heads * r->q_len, r->ld ? r->ld : r->k_len, kMaxElements))
    return CANON_EUNSUPPORTED;
  if (!aligned(r->q_starts, 4) || !aligned(r->q_lens, 4) || !aligned(r->k_lens, 4)) return CANON_EINVAL;
  return CANON_OK;
}

RelBiasArgs args_of(const canon_attn_rows* r, const canon_relbias* bias, const uint16_t* table) {
  RelBiasArgs a;
  memset(&a, 0, sizeof(a));
  a.batch = r->batch; a.heads = r->n_heads; a.q_len = r->q_len; a.k_len = r->k_len;
  a.ld = r->ld ? r->ld : r->k_len;
  a.q_start = r->q_start;
  a.window = r->window < 4 * kMaxStart ? r->window : 4 * kMaxStart;  // no position is further from a key
  a.q_starts = r->q_starts; a.q_lens = r->q_lens; a.k_lens = r->k_lens;
  a.table = table; a.scale = r->scale; a.causal = r->causal;
  a.n_side = bias->n_starts; a.bidirectional = bias->bidirectional;
  memcpy(a.start, bias->start, sizeof(int32_t) * (size_t)bias->n_starts);
  for (int n = 0, d = 0; n < a.n_side; ++n)
    for (const int end = n + 1 < a.n_side ? a.start[n + 1] : a.start[n] + 1; d < end; ++d) a.bucket[d] = (uint8_t)n;
  const int far = a.start[a.n_side - 1];
  a.far_only = !a.bidirectional || far >= 32;  // 32: no chunk of 32 keys has keys of both last buckets
  for (int k = 0; k < a.n_side * (a.bidirectional ? 2 : 1); ++k) {
    const RelKeys keys = relbias_keys(a, k);
    if (keys.short_one()) {
      a.short_most = keys.hi - keys.lo > a.short_most ? keys.hi - keys.lo : a.short_most;
    } else {
      a.longs[a.n_long++] = (uint8_t)k;
      if (k % a.n_side != a.n_side - 1) a.far_only = 0;
    }
  }
  return a;
}

// bytes from the first to behind the last key of the rows
int64_t row_bytes(const canon_attn_rows* r, int64_t size) {
  const int64_t n = r->batch * r->n_heads * r->q_len;
  return n == 0 || r->k_len == 0 ? 0 : ((n - 1) * (r->ld ? r->ld : r->k_len) + r->k_len) * size;
}

}  // namespace

canon_status canon_relbias_log(int32_t n_buckets, int32_t bidirectional, int32_t max_distance, canon_relbias* bias) {
  if (!bias || (bidirectional != 0 && bidirectional != 1) || n_buckets < 1 || (bidirectional && n_buckets % 2))
    return CANON_EINVAL;
  const int n = bidirectional ? n_buckets / 2 : n_buckets, half = n / 2;
  if (n > CANON_RELBIAS_MAX_STARTS || max_distance > kRelFar) return CANON_EUNSUPPORTED;
  if (max_distance <= half || n < 2) return CANON_EINVAL;
  memset(bias, 0, sizeof(*bias));
  bias->n_starts = n;
  bias->bidirectional = bidirectional;
  for (int d = 0; d < half; ++d) bias->start[d] = d;
  int d = half;
  for (int i = 0; i < n - half; ++i) {  // the first d with d^(n-half) half^i >= max_distance^i half^(n-half)
    Whole bound;
    bound.power((uint32_t)max_distance, i).power((uint32_t)half, n - half);
    for (; d < max_distance; ++d) {
      Whole left;
      left.power((uint32_t)d, n - half).power((uint32_t)half, i);
      if (left.at_least(bound)) break;
    }
    bias->start[half + i] = d;
  }
  return CANON_OK;
}

size_t canon_softmax_relbias_bwd_workspace_bytes(const canon_attn_rows* rows, const canon_relbias* bias) {
  if (check_rows(rows, bias) != CANON_OK) return 0;
  return sizeof(float) * (size_t)relbias_scratch_floats(rows->batch * rows->q_len, rows->n_heads, buckets_of(bias));
}

canon_status canon_softmax_relbias(const canon_order* order, const canon_attn_rows* rows, const canon_relbias* bias,
                                   const uint16_t* table, const float* scores, uint16_t* probs, void* stream) {
  canon_status st = check_order(order);
  if (st == CANON_OK) st = check_rows(rows, bias);
  if (st != CANON_OK) return st;
  if (row_bytes(rows, 1) == 0) return CANON_OK;
  if (!table || !scores || !probs || !aligned(table, 2) || !aligned(scores, 4) || !aligned(probs, 2)) return CANON_EINVAL;
  if (!apart({{scores, row_bytes(rows, 4), false}, {table, 2 * buckets_of(bias) * rows->n_heads, false},
              {rows->q_starts, 4 * rows->batch, false}, {rows->q_lens, 4 * rows->batch, false},
              {rows->k_lens, 4 * rows->batch, false}, {probs, row_bytes(rows, 2), true}}))
    return CANON_EINVAL;
  return dev(relbias_fwd_launch(args_of(rows, bias, table), scores, probs, as_stream(stream)));
}

canon_status canon_softmax_relbias_bwd(const canon_order* order, const canon_attn_rows* rows, const canon_relbias* bias,
                                       const uint16_t* probs, const float* dprobs, uint16_t* dscores, float* dtable,
                                       void* workspace, size_t workspace_bytes, void* stream) {
  canon_status st = check_order(order);
  if (st == CANON_OK) st = check_rows(rows, bias);
  if (st != CANON_OK) return st;
  if (row_bytes(rows, 1) > 0 && (!probs || !dprobs || !dscores || !aligned(probs, 2) || !aligned(dprobs, 4) || !aligned(dscores, 2)))
    return CANON_EINVAL;
  if (!aligned(dtable, 4)) return CANON_EINVAL;
  const size_t need = dtable ? canon_softmax_relbias_bwd_workspace_bytes(rows, bias) : 0;
  if (need > 0) {
    if (workspace_bytes < need) return CANON_EWORKSPACE;
    if (!workspace || !aligned(workspace, 256)) return CANON_EINVAL;
  }
  if (!apart({{probs, row_bytes(rows, 2), false}, {dprobs, row_bytes(rows, 4), false},
              {rows->q_starts, 4 * rows->batch, false}, {rows->q_lens, 4 * rows->batch, false},
              {rows->k_lens, 4 * rows->batch, false}, {dscores, row_bytes(rows, 2), true},
              {dtable, 4 * buckets_of(bias) * rows->n_heads, true}, {workspace, (int64_t)need, true}}))
    return CANON_EINVAL;
  return dev(relbias_bwd_launch(args_of(rows, bias, nullptr), probs, dprobs, dscores, dtable, (float*)workspace,
                                as_stream(stream)));
}
