/*
 * block_ref.c - CPU oracle of the operators around a block: layer norm (R20), activations kept in 8 bits (R21) and
 * attention rows with a learned relative position bias (R22).
 *
 * TEST INFRASTRUCTURE, as canon_ref.c, whose R0 operations and R1 sums it uses.  Every operation is spelled out; a sum's
 * terms are written down in their order and handed to cref_rsum.
 */
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "canon_ref.h"

static float of_bits(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static uint32_t to_bits(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
static float wide16(uint16_t h) { return cref_mul(of_bits((uint32_t)h << 16), 1.0f); } /* a subnormal reads as zero */
static float inverse(int64_t n) { return (float)(1.0 / (double)n); }
static float* floats(int64_t n) { return (float*)malloc(sizeof(float) * (size_t)(n > 0 ? n : 1)); }

#define RN_1_127 0x3C010204u /* RN32(1/127) */

int cref_act8_pack(int64_t rows, int64_t cols, int32_t group, const float* x, int8_t* codes, float* steps) {
  if (rows < 0 || cols < 0 || group < 1) return -1;
  const int64_t groups = (cols + group - 1) / group;
#pragma omp parallel for schedule(static)
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t g = 0; g < groups; ++g) {
      const int64_t j0 = g * group, j1 = j0 + group < cols ? j0 + group : cols;
      uint32_t top = 0;
      for (int64_t j = j0; j < j1; ++j) {
        const uint32_t u = to_bits(x[r * cols + j]) & 0x7FFFFFFFu;
        if (u > top) top = u;
      }
      float step = cref_mul(of_bits(top), of_bits(RN_1_127));
      steps[r * groups + g] = step;
      cref_quantize(1, j1 - j0, 0, x + r * cols + j0, &step, 0, codes + r * cols + j0);
    }
  return 0;
}

int cref_act8_unpack(int64_t rows, int64_t cols, int32_t group, const int8_t* codes, const float* steps, float* out) {
  if (rows < 0 || cols < 0 || group < 1) return -1;
  const int64_t groups = (cols + group - 1) / group;
  for (int64_t r = 0; r < rows; ++r)
    for (int64_t j = 0; j < cols; ++j)
      out[r * cols + j] = cref_mul((float)codes[r * cols + j], steps[r * groups + j / group]);
  return 0;
}

int cref_layernorm_fwd(int64_t rows, int64_t cols, const float* x, const uint16_t* gain, const uint16_t* bias, float eps,
                       float* y, float* mean, float* rstd) {
  if (rows < 0 || cols < 1) return -1;
  const float inv = inverse(cols);
#pragma omp parallel for schedule(static)
  for (int64_t r = 0; r < rows; ++r) {
    const float* xr = x + r * cols;
    float* d = floats(cols);
    const float mu = cref_mul(cref_rsum(xr, cols, 1, 32), inv);
    for (int64_t k = 0; k < cols; ++k) d[k] = cref_sub(xr[k], mu);
    const float var = cref_mul(cref_rdot_f32(d, 1, d, 1, cols, 32), inv);
    const float rs = cref_div(1.0f, cref_sqrt(cref_add(var, eps)));
    mean[r] = mu;
    rstd[r] = rs;
    for (int64_t k = 0; k < cols; ++k) {
      const float v = cref_mul(cref_mul(d[k], rs), wide16(gain[k]));
      y[r * cols + k] = bias ? cref_add(v, wide16(bias[k])) : v;
    }
    free(d);
  }
  return 0;
}

int cref_layernorm_bwd(int64_t rows, int64_t cols, const float* x, const uint16_t* gain, const float* mean,
                       const float* rstd, const float* dy, float* dx, float* dgain, float* dbias) {
  if (rows < 0 || cols < 1) return -1;
  const float inv = inverse(cols);
#pragma omp parallel for schedule(static)
  for (int64_t r = 0; r < rows; ++r) {
    float *xh = floats(cols), *gy = floats(cols);
    for (int64_t k = 0; k < cols; ++k) {
      xh[k] = cref_mul(cref_sub(x[r * cols + k], mean[r]), rstd[r]);
      gy[k] = cref_mul(dy[r * cols + k], wide16(gain[k]));
    }
    const float m1 = cref_mul(cref_rsum(gy, cols, 1, 32), inv);
    const float m2 = cref_mul(cref_rdot_f32(gy, 1, xh, 1, cols, 32), inv);
    for (int64_t k = 0; k < cols; ++k)
      dx[r * cols + k] = cref_mul(rstd[r], cref_sub(cref_sub(gy[k], m1), cref_mul(xh[k], m2)));
    free(xh);
    free(gy);
  }
#pragma omp parallel for schedule(static)
  for (int64_t k = 0; k < cols; ++k) {
    float *g = floats(rows), *b = floats(rows);
    for (int64_t r = 0; r < rows; ++r) {
      b[r] = dy[r * cols + k];
      g[r] = cref_mul(b[r], cref_mul(cref_sub(x[r * cols + k], mean[r]), rstd[r]));
    }
    dgain[k] = cref_rsum(g, rows, 1, 32);
    dbias[k] = cref_rsum(b, rows, 1, 32);
    free(g);
    free(b);
  }
  return 0;
}

/* the bucket of key j for a query at position pos */
static int64_t bucket(int64_t n_starts, int32_t bidirectional, const int32_t* start, int64_t pos, int64_t j) {
  int64_t d = pos - j, at = 0;
  if (!bidirectional && d < 0) d = 0;
  for (int64_t i = 0; i < n_starts; ++i)
    if (start[i] <= (d < 0 ? -d : d)) at = i;
  return d < 0 ? n_starts + at : at;
}

/* whether query i of sequence b sees key j: cfg holds batch, heads, q_len, k_len, window, causal */
static int sees(const int64_t* cfg, const int32_t* q_starts, const int32_t* q_lens, const int32_t* k_lens, int64_t b,
                int64_t i, int64_t j) {
  const int64_t pos = q_starts[b] + i;
  if (j >= k_lens[b] || i >= q_lens[b]) return 0;
  if (cfg[5] && j > pos) return 0;
  return !cfg[4] || (pos - j < cfg[4] && j - pos < cfg[4]);
}

int cref_relbias_fwd(const int64_t* cfg, int64_t n_starts, int32_t bidirectional, const int32_t* start, float scale,
                     const int32_t* q_starts, const int32_t* q_lens, const int32_t* k_lens, const uint16_t* table,
                     const float* scores, uint16_t* probs) {
  const int64_t B = cfg[0], H = cfg[1], Q = cfg[2], K = cfg[3];
#pragma omp parallel for schedule(dynamic, 4)
  for (int64_t r = 0; r < B * H * Q; ++r) {
    const int64_t i = r % Q, h = r / Q % H, b = r / Q / H;
    float *z = floats(K), *e = floats(K);
    float m = -INFINITY;
    for (int64_t j = 0; j < K; ++j)
      if (sees(cfg, q_starts, q_lens, k_lens, b, i, j)) {
        const int64_t n = bucket(n_starts, bidirectional, start, q_starts[b] + i, j);
        z[j] = cref_add(cref_mul(scores[r * K + j], scale), wide16(table[n * H + h]));
        if (z[j] > m) m = z[j];
      }
    if (m == -INFINITY) m = 0.0f;
    for (int64_t j = 0; j < K; ++j)
      e[j] = sees(cfg, q_starts, q_lens, k_lens, b, i, j) ? cref_exp(cref_sub(z[j], m)) : 0.0f;
    const float S = cref_rsum(e, K, 1, 32);
    const float inv = S == 0.0f ? 0.0f : cref_div(1.0f, S);
    for (int64_t j = 0; j < K; ++j)
      probs[r * K + j] = sees(cfg, q_starts, q_lens, k_lens, b, i, j) ? cref_bf16(cref_mul(e[j], inv)) : 0;
    free(z);
    free(e);
  }
  return 0;
}

int cref_relbias_bwd(const int64_t* cfg, int64_t n_starts, int32_t bidirectional, const int32_t* start, float scale,
                     const int32_t* q_starts, const int32_t* q_lens, const int32_t* k_lens, const uint16_t* probs,
                     const float* dprobs, uint16_t* dscores, float* dtable) {
  const int64_t B = cfg[0], H = cfg[1], Q = cfg[2], K = cfg[3], N = n_starts * (bidirectional ? 2 : 1);
  float* row = floats(B * H * Q * N); /* [h][n][b][i] */
#pragma omp parallel for schedule(dynamic, 4)
  for (int64_t r = 0; r < B * H * Q; ++r) {
    const int64_t i = r % Q, h = r / Q % H, b = r / Q / H;
    float *t = floats(K), *ds = floats(K);
    for (int64_t j = 0; j < K; ++j)
      t[j] = sees(cfg, q_starts, q_lens, k_lens, b, i, j) ? cref_mul(wide16(probs[r * K + j]), dprobs[r * K + j]) : 0.0f;
    const float D = cref_rsum(t, K, 1, 32);
    for (int64_t j = 0; j < K; ++j) {
      ds[j] = sees(cfg, q_starts, q_lens, k_lens, b, i, j)
                  ? cref_mul(wide16(probs[r * K + j]), cref_sub(dprobs[r * K + j], D)) : 0.0f;
      dscores[r * K + j] = sees(cfg, q_starts, q_lens, k_lens, b, i, j) ? cref_bf16(cref_mul(ds[j], scale)) : 0;
    }
    for (int64_t n = 0; n < N; ++n) {
      for (int64_t j = 0; j < K; ++j)
        t[j] = bucket(n_starts, bidirectional, start, q_starts[b] + i, j) == n ? ds[j] : 0.0f;
      row[((h * N + n) * B + b) * Q + i] = cref_rsum(t, K, 1, 32);
    }
    free(t);
    free(ds);
  }
  for (int64_t h = 0; h < H; ++h)
    for (int64_t n = 0; n < N; ++n) dtable[n * H + h] = cref_rsum(row + (h * N + n) * B * Q, B * Q, 1, 32);
  free(row);
  return 0;
}
