/*
 * serve_ref.c - CPU oracle of what a model answers with: products of int8 codes with a step per token (R23), rotary
 * positions (R24), a paged cache of keys and values in 8 bits (R25) and attention over it (R26).
 *
 * TEST INFRASTRUCTURE, as canon_ref.c, whose R0 operations it uses.  Integer sums are written in 64 bits, one term at a time.
 */
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "canon_ref.h"

static float of_bits(uint32_t u) { float f; memcpy(&f, &u, 4); return f; }
static uint32_t to_bits(float f) { uint32_t u; memcpy(&u, &f, 4); return u; }
static float flushed(float x) { return cref_mul(x, 1.0f); }

int cref_gemm_i8_tokens(int64_t m, int64_t n, int64_t k, const int8_t* a, const float* sa, const int8_t* b, const float* sb,
                        float* y) {
#pragma omp parallel for schedule(static)
  for (int64_t i = 0; i < m; ++i)
    for (int64_t j = 0; j < n; ++j) {
      int64_t acc = 0;
      for (int64_t l = 0; l < k; ++l) acc += (int64_t)a[i * k + l] * b[j * k + l];
      y[i * n + j] = cref_mul(cref_mul((float)acc, sa[i]), sb[j]);
    }
  return 0;
}

/* one head, in and out of place */
static void turn(int64_t dim, int64_t rot, int32_t interleaved, int32_t backward, const float* c, const float* s,
                 const float* x, float* y) {
  for (int64_t d = rot; d < dim; ++d) y[d] = flushed(x[d]);
  for (int64_t i = 0; i < rot / 2; ++i) {
    const int64_t p = interleaved ? 2 * i : i, q = interleaved ? 2 * i + 1 : i + rot / 2;
    const float a = x[p], b = x[q];
    if (!c) {
      y[p] = y[q] = NAN;
    } else if (!backward) {
      y[p] = cref_sub(cref_mul(a, c[i]), cref_mul(b, s[i]));
      y[q] = cref_add(cref_mul(b, c[i]), cref_mul(a, s[i]));
    } else {
      y[p] = cref_add(cref_mul(a, c[i]), cref_mul(b, s[i]));
      y[q] = cref_sub(cref_mul(b, c[i]), cref_mul(a, s[i]));
    }
  }
}

int cref_rope(int32_t backward, int64_t tokens, int64_t heads, int64_t dim, int64_t rot, int32_t interleaved,
              int64_t positions, const float* c, const float* s, const int32_t* pos, const float* x, float* y) {
  for (int64_t t = 0; t < tokens; ++t)
    for (int64_t h = 0; h < heads; ++h) {
      const int64_t at = (t * heads + h) * dim;
      const int in = pos[t] >= 0 && pos[t] < positions;
      turn(dim, rot, interleaved, backward, in ? c + pos[t] * (rot / 2) : NULL, in ? s + pos[t] * (rot / 2) : NULL, x + at,
           y + at);
    }
  return 0;
}

/* cache: n_pages, page, kv heads, dim, batch, table_len */
static int64_t slot_of(const int64_t* cache, const int32_t* table, int64_t b, int64_t h, int64_t j) {
  if (j < 0 || j >= cache[5] * cache[1]) return -1;
  const int64_t p = table[b * cache[5] + j / cache[1]];
  return p < 0 || p >= cache[0] ? -1 : (p * cache[2] + h) * cache[1] + j % cache[1];
}
static int64_t v_at(const int64_t* cache, int64_t slot, int64_t d) {
  return slot / 16 * 16 * cache[3] + d * 16 + slot % 16;
}

int cref_cache_append(const int64_t* cache, const int32_t* table, int64_t q_len, const int32_t* q_starts,
                      const int32_t* q_lens, const float* k, const float* v, int64_t rot, int32_t interleaved,
                      int64_t positions, const float* c, const float* s, int8_t* kc, int8_t* vc, float* ks, float* vs) {
  const int64_t H = cache[2], D = cache[3];
  for (int64_t b = 0; b < cache[4]; ++b)
    for (int64_t i = 0; i < q_len && i < q_lens[b]; ++i)
      for (int64_t h = 0; h < H; ++h) {
        const int64_t pos = (int64_t)q_starts[b] + i, slot = slot_of(cache, table, b, h, pos);
        if (slot < 0) continue;
        const float *kr = k + ((b * q_len + i) * H + h) * D, *vr = v + ((b * q_len + i) * H + h) * D;
        float turned[256];
        int8_t code[256];
        if (rot) {
          const int in = pos >= 0 && pos < positions;
          turn(D, rot, interleaved, 0, in ? c + pos * (rot / 2) : NULL, in ? s + pos * (rot / 2) : NULL, kr, turned);
          kr = turned;
        }
        cref_act8_pack(1, D, (int32_t)D, kr, kc + slot * D, ks + slot);
        cref_act8_pack(1, D, (int32_t)D, vr, code, vs + slot);
        for (int64_t d = 0; d < D; ++d) vc[v_at(cache, slot, d)] = code[d];
      }
  return 0;
}

/* R26's exponential: 2^x of x in [-127, 0], 0 below 2^-126.  Without the last step: p 2^n. */
static float exp2_parts(float x, int* n) {
  *n = (int)nearbyint(x);
  const float t = x - (float)*n; /* exact */
  float p = of_bits(0x3AADED20u);
  p = cref_fma(p, t, of_bits(0x3C1E7456u));
  p = cref_fma(p, t, of_bits(0x3D635B6Cu));
  p = cref_fma(p, t, of_bits(0x3E75FCE1u));
  p = cref_fma(p, t, of_bits(0x3F317215u));
  return cref_fma(p, t, 1.0f);
}
static float exp2_neg(float x) {
  int n;
  const float p = exp2_parts(x, &n);
  return flushed(ldexpf(p, n));
}
int cref_exp2(int64_t n, const float* x, float* e) {
  for (int64_t i = 0; i < n; ++i) e[i] = exp2_neg(x[i]);
  return 0;
}
/* four times 2^(128 (y - 1)), y in [0, 1]: the same exponential, of a range whose ends are normal numbers */
int cref_exp2_unit(int64_t n, const float* y, float* e4) {
  for (int64_t i = 0; i < n; ++i) {
    int k;
    const double x = 128.0 * (double)y[i] - 128.0;
    const float p = exp2_parts((float)x, &k);
    e4[i] = ldexpf(p, k + 2);
  }
  return 0;
}
/* what is left of a whole number to the nearest multiple of 256, -128 .. 127 */
static int64_t low_digit(int64_t n) { return ((n + 128) % 256 + 256) % 256 - 128; }

/* the least s for which x 2^-s, rounded, fits three digits of -128 .. 127: 127 (65536 + 256 + 1); x finite, not negative */
static int step_of(float x) {
  int s = -200;
  while (rint(ldexp((double)x, -s)) > 8355711.0) ++s;
  return s;
}

/* x held to [-127, 0] */
static float held(float x) { return x > -127.0f ? (x < 0.0f ? x : 0.0f) : -127.0f; }

/* 2^(a - b) of whole a <= b */
static float shift(float a, float b) {
  if (a == -INFINITY) return 1.0f;
  const float x = cref_sub(a, b);
  return x != x ? x : x < -126.0f ? 0.0f : ldexpf(1.0f, (int)x);
}

/* cfg: heads, q_len, k_len, window, causal */
int cref_cache_attention(const int64_t* cache, const int64_t* cfg, float scale, const int32_t* table,
                         const int32_t* q_starts, const int32_t* q_lens, const int32_t* k_lens, const int8_t* kc,
                         const int8_t* vc, const float* ks, const float* vs, const float* q, uint16_t* out) {
  const int64_t B = cache[4], KV = cache[2], D = cache[3], H = cfg[0], QL = cfg[1], KL = cfg[2], W = cfg[3];
#pragma omp parallel for schedule(dynamic, 4)
  for (int64_t r = 0; r < B * QL * H; ++r) {
    const int64_t h = r % H, i = r / H % QL, b = r / H / QL, kvh = h / (H / KV);
    const int64_t pos = (int64_t)q_starts[b] + i;
    const float* x = q + r * D;
    int64_t Q[256];
    uint32_t amax = 0;
    for (int64_t d = 0; d < D; ++d) {
      const uint32_t u = to_bits(x[d]) & 0x7FFFFFFFu;
      if (u > amax) amax = u;
    }
    const int zero = amax < 0x00800000u, finite_q = !zero && amax < 0x7F800000u, qs = finite_q ? step_of(of_bits(amax)) : 0;
    for (int64_t d = 0; d < D; ++d)
      Q[d] = finite_q ? (int64_t)rint(ldexp((double)flushed(scale < 0.0f ? -x[d] : x[d]), -qs)) : 0;
    const double fs = ldexp((double)cref_mul(fabsf(scale), of_bits(0x3FB8AA3Bu)), qs); /* RN32(1 / ln 2) */
    const float f = zero ? 0.0f : !finite_q ? NAN : fs >= 0x1p128 ? INFINITY : fs < 0x1p-126 ? 0.0f : (float)fs;
    float R = -INFINITY, S = 0.0f, O[256]; /* a NaN among the scores makes R and S NaN */
    for (int64_t d = 0; d < D; ++d) O[d] = 0.0f;
    for (int64_t j0 = 0; j0 < KL; j0 += 256) {
      float t[256], e[256], m = -INFINITY;
      int8_t sees[256];
      int64_t slot[256], any = 0;
      for (int64_t j = 0; j < 256; ++j) {
        const int64_t key = j0 + j;
        sees[j] = key < KL && key < k_lens[b] && i < q_lens[b] && !(cfg[4] && key > pos) &&
                  !(W && (pos - key >= W || key - pos >= W));
        if (!sees[j]) continue;
        any = 1;
        slot[j] = slot_of(cache, table, b, kvh, key);
        int64_t hi = 0, lo = 0;
        for (int64_t d = 0; slot[j] >= 0 && d < D; ++d) {
          const int64_t l = low_digit(Q[d]);
          hi += (Q[d] - l) / 256 * kc[slot[j] * D + d];
          lo += l * kc[slot[j] * D + d];
        }
        t[j] = slot[j] < 0 ? NAN : cref_mul(cref_fma((float)hi, 256.0f, (float)lo), ks[slot[j]]);
        if (t[j] > m || t[j] != t[j] || m != m) m = t[j] != t[j] || m != m ? NAN : t[j];
      }
      if (!any) continue;
      const float rb = m == -INFINITY ? m : ceilf(cref_mul(m, f));
      const float ref = rb == -INFINITY ? 0.0f : rb;
      float p[256];
      uint32_t top = 0;
      for (int64_t j = 0; j < 256; ++j) {
        e[j] = p[j] = 0.0f;
        if (!sees[j]) continue;
        const float near = cref_fma(t[j], f, -ref), far = cref_sub(cref_mul(t[j], f), ref);
        e[j] = exp2_neg(held(fabsf(ref) <= 4194304.0f ? near : far));
        p[j] = cref_mul(e[j], slot[j] < 0 ? NAN : vs[slot[j]]);
        if ((to_bits(p[j]) & 0x7FFFFFFFu) > top) top = to_bits(p[j]) & 0x7FFFFFFFu;
      }
      float part[16];
      for (int c = 0; c < 16; ++c) {
        part[c] = 0.0f;
        for (int j = 0; j < 16; ++j) part[c] = cref_add(part[c], e[16 * c + j]);
      }
      for (int n = 16; n > 1; n /= 2)
        for (int c = 0; c < n / 2; ++c) part[c] = cref_add(part[2 * c], part[2 * c + 1]);
      const int finite = top < 0x7F800000u;
      int step = finite ? step_of(of_bits(top)) : 0;
      if (step < -126) step = -126;
      const float Rn = R != R || rb != rb ? NAN : R > rb ? R : rb, xo = shift(R, Rn), y = shift(rb, Rn);
      const float Sb = rb == -INFINITY ? 0.0f : rb < INFINITY ? part[0] : NAN;
      S = cref_fma(Sb, y, cref_mul(S, xo));
      for (int64_t d = 0; d < D; ++d) {
        int64_t hi = 0, lo = 0;
        for (int64_t j = 0; j < 256; ++j)
          if (sees[j] && finite && slot[j] >= 0) {
            const int64_t w = (int64_t)rint(ldexp((double)p[j], -step)), l = low_digit(w);
            hi += (w - l) / 256 * vc[v_at(cache, slot[j], d)];
            lo += l * vc[v_at(cache, slot[j], d)];
          }
        const float A = finite ? cref_fma((float)hi, 256.0f, (float)lo) : NAN;
        O[d] = cref_fma(cref_mul(A, y), ldexpf(1.0f, step), cref_mul(O[d], xo));
      }
      R = Rn;
    }
    const float is = S == 0.0f ? 0.0f : cref_div(1.0f, S);
    for (int64_t d = 0; d < D; ++d) out[r * D + d] = S == 0.0f ? 0 : cref_bf16(cref_mul(cref_add(O[d], 0.0f), is));
  }
  return 0;
}
