// act8_dev.h - activations kept in 8 bits (R21), four consecutive elements of a row per lane: the step and codes of the
// groups that a wavefront's 256 consecutive elements make up, and the values that codes stand for.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

constexpr uint32_t kInv127Bits = 0x3C010204u;  // RN32(1/127)

struct __attribute__((packed, aligned(1))) B4 {
  uint32_t x;
};

// Elements j .. j + 3 of a row of n (j a multiple of 4 whose lanes run through whole groups; v holds 0 beyond n) into
// codes and their group's step.  Every lane of the wavefront takes part.  The magnitudes are compared as bit patterns,
// so that a NaN ranks above every number.
template <int Q>
__device__ __forceinline__ void steps4(const float (&v)[Q][4], int lg, float (&s)[Q]) {  // of Q vectors
  uint32_t m[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    m[q] = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint32_t a = __float_as_uint(v[q][t]) & 0x7FFFFFFFu;
      m[q] = a > m[q] ? a : m[q];
    }
  }
  lanes_join(m, 1 << (lg - 2), [](uint32_t a, uint32_t b) { return a > b ? a : b; });
#pragma unroll
  for (int q = 0; q < Q; ++q) s[q] = __uint_as_float(m[q]) * __uint_as_float(kInv127Bits);
}
// The reciprocal of a step of keep4's (|v / s| <= 127 (1 + 2^-23)), for quant_pack's rule: v_rcp_f32 is within 2^-23 of 1/s,
// so t = RN(v rs) within 127 (2^-23 + 2^-24) (1 + 2^-22) < 2.28e-5 of v / s, and RN(v / s) within 2^-18: together below the
// 2^-15 that t has to be away from every half-integer.  The correctly rounded quotient took 12 instructions.
__device__ __forceinline__ float step_rcp(float s) { return recip_step_ok(s) ? __builtin_amdgcn_rcpf(s) : 0.0f; }
// vector v of elements j .. j + 3, whose group has step s
template <bool TAIL>
__device__ __forceinline__ void keep4(const float (&v)[4], float s, int64_t j, int64_t n, int lg, int8_t* codes,
                                      float* steps) {
  if (j >= n) return;
  uint32_t w[1];
  quant_pack<4>(v, s, step_rcp(s), recip_step_ok(s), w);
  if ((j & ((1 << lg) - 1)) == 0) steps[j >> lg] = s;
  if (!TAIL || j + 4 <= n) {
    reinterpret_cast<B4*>(codes + j)->x = w[0];
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (j + t < n) codes[j + t] = (int8_t)(w[0] >> (8 * t));
  }
}
// The same of a part of a row (part_load): v holds 0 beyond n.  Every code is taken through the reciprocal first; the few
// vectors with a value that it does not decide (quant_pack's rule) are remembered and done exactly behind the loop, in one
// branch instead of one per vector, whose masks spilled.
template <bool TAIL, int Q>
__device__ __forceinline__ void part_keep(const float (&v)[Q][4], int n, int lg, int8_t* codes, float* steps) {
  n = again(n);
  lg = again(lg);  // or the steps' places, the same for every row, are held from one to the next and spill: their reloads
                   // waited for the stores before them (4096 rows of 16384 kept 116 us, then 90)
  const int at = 4 * (threadIdx.x & 63);
  uint32_t w[Q], undecided = 0;
  float s[Q];
  steps4(v, lg, s);
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const float rs = step_rcp(s[q]);
    float off = 0.0f;  // how far the furthest is from its integer
    uint32_t x = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float y = v[q][t] * rs, k = __builtin_rintf(y);
      off = fmaxf(off, fabsf(y - k));
      x = __builtin_amdgcn_cvt_pk_u8_f32(k + 128.0f, t, x);
    }
    w[q] = x ^ 0x80808080u;
    undecided |= rs > 0.0f && off < 0.5f - 0x1p-15f ? 0u : 1u << q;
  }
  // of the vectors that the row has in this lane (groups behind its end have the step 0, which nothing is decided by)
  const int have = n > at ? (n - at + 255) >> 8 : 0;
  undecided &= (1u << (have < Q ? have : Q)) - 1;
  while (undecided) {  // one vector of each lane that has any
    const int k = __builtin_ctz(undecided);
    undecided &= undecided - 1;
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f}, sx = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
#pragma unroll
      for (int t = 0; t < 4; ++t) x[t] = q == k ? v[q][t] : x[t];
      sx = q == k ? s[q] : sx;
    }
    uint32_t c = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) c |= (uint32_t)(uint8_t)quant1(x[t], sx) << (8 * t);
#pragma unroll
    for (int q = 0; q < Q; ++q) w[q] = q == k ? c : w[q];
  }
  const int mine = TAIL && (n & 3) && n > 0 && at == (n & 252) ? n >> 8 : -1;
  uint32_t cut = 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (256 * q >= n) break;
    const int j = 256 * q + at;
    if (j < n && (j & ((1 << lg) - 1)) == 0) steps[j >> lg] = s[q];
    if (j + 4 <= n) reinterpret_cast<B4*>(codes + j)->x = w[q];
    cut = q == mine ? w[q] : cut;
  }
  if (mine >= 0) {
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (t < (n & 3)) codes[(n & ~3) + t] = (int8_t)(cut >> (8 * t));
  }
}

// results of arithmetic to bf16, elements j .. j + 3 of a row of n
template <bool TAIL>
__device__ __forceinline__ void stb4_arith(uint16_t* row, int64_t j, int64_t n, const float (&f)[4]) {
  if (!TAIL || j + 4 <= n) {
    stb_arith(row + j, f);
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (j + t < n) row[j + t] = bf16_arith(f[t]);
  }
}

// the values RN(step * code) of elements j .. j + 3 of a row of n, those beyond its end as 0
template <bool TAIL>
__device__ __forceinline__ void kept4(const int8_t* codes, const float* steps, int64_t j, int64_t n, int lg,
                                      float (&f)[4]) {
  const float s = steps[j >> lg];
  if (!TAIL || j + 4 <= n) {
    const uint32_t w = reinterpret_cast<const B4*>(codes + j)->x;
#pragma unroll
    for (int t = 0; t < 4; ++t) f[t] = (float)(int8_t)(w >> (8 * t)) * s;
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t) f[t] = j + t < n ? (float)codes[j + t] * s : 0.0f;
  }
}

// elements j .. j + 3 of row `row` of an activation (fp32, bf16 or kept in 8 bits), for arithmetic
template <int SRC, bool TAIL>
__device__ __forceinline__ void act4(const ActIn& a, int64_t row, int64_t j, int64_t n, float (&f)[4]) {
  if constexpr (SRC == ACT_F32) ldf4<TAIL>((const float*)a.x + row * n, j, n, f);
  else if constexpr (SRC == ACT_BF16) {
    const uint16_t* p = (const uint16_t*)a.x + row * n + j;
    if (!TAIL || j + 4 <= n) {
      ldb_wide(p, f);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = j + t < n ? bf16_wide(p[t]) : 0.0f;
    }
  }
  else kept4<TAIL>((const int8_t*)a.x + row * n, a.steps + row * ((n + (1 << a.lg) - 1) >> a.lg), j, n, a.lg, f);
}

// a part of a row of an activation, from element `seg` (a multiple of 256) on
template <int SRC>
struct PartIn {
  const void* p;
  const float* steps;
  int lg;
  __device__ __forceinline__ PartIn(const ActIn& a, int64_t row, int64_t cols, int seg) {
    const int64_t at = row * cols + seg;
    lg = a.lg;
    steps = nullptr;
    if constexpr (SRC == ACT_F32) p = (const float*)a.x + at;
    else if constexpr (SRC == ACT_BF16) p = (const uint16_t*)a.x + at;
    else {
      p = (const int8_t*)a.x + at;
      steps = a.steps + row * ((cols + (1 << lg) - 1) >> lg) + (seg >> lg);
    }
  }
  // four elements as they are stored, to be widened when they are needed, so that nothing waits for them before
  struct Raw {
    float f[SRC == ACT_F32 ? 4 : 1];  // fp32; in 8 bits the step
    uint32_t w[SRC == ACT_BF16 ? 2 : 1];
  };
  __device__ __forceinline__ void load4(int j, Raw& r) const { load4(j, j, r); }
  __device__ __forceinline__ void load4(int j, int group, Raw& r) const {  // with the step of element `group`
    if constexpr (SRC == ACT_F32) {
      ldf<4>((const float*)p + j, r.f);
    } else if constexpr (SRC == ACT_BF16) {
      const H4 h = *reinterpret_cast<const H4*>((const uint16_t*)p + j);
      r.w[0] = h.x; r.w[1] = h.y;
    } else {
      r.f[0] = steps[group >> lg];
      r.w[0] = reinterpret_cast<const B4*>((const int8_t*)p + j)->x;
    }
  }
  // bf16 or 8 bits: four elements of which the last n are wanted (n > 3: all) to the first n places, 0 behind them
  static __device__ __forceinline__ void ends(Raw& r, int n) {
    const int away = n > 0 && n < 4 ? 4 - n : 0;
    if constexpr (SRC == ACT_BF16) {
      const uint64_t w = (((uint64_t)r.w[1] << 32) | r.w[0]) >> (16 * away);
      r.w[0] = (uint32_t)w; r.w[1] = (uint32_t)(w >> 32);
    } else {
      r.w[0] >>= 8 * away;
    }
  }
  // element j + t into place t
  __device__ __forceinline__ void load1(int j, int t, Raw& r) const {
    if constexpr (SRC == ACT_F32) {
      r.f[t] = ((const float*)p)[j + t];
    } else if constexpr (SRC == ACT_BF16) {
      r.w[t >> 1] |= (uint32_t)((const uint16_t*)p)[j + t] << (16 * (t & 1));
    } else {
      r.f[0] = steps[j >> lg];
      r.w[0] |= (uint32_t)((const uint8_t*)p)[j + t] << (8 * t);
    }
  }
  static __device__ __forceinline__ void wide(const Raw& r, float (&f)[4]) {
    if constexpr (SRC == ACT_F32) {
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = r.f[t];
    } else if constexpr (SRC == ACT_BF16) {
      f[0] = __uint_as_float(r.w[0] << 16); f[1] = __uint_as_float(r.w[0] & 0xFFFF0000u);
      f[2] = __uint_as_float(r.w[1] << 16); f[3] = __uint_as_float(r.w[1] & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int t = 0; t < 4; ++t) f[t] = (float)(int8_t)(r.w[0] >> (8 * t)) * r.f[0];
    }
  }
  // the part's first n elements, as part_load; widened behind the last load (widened each in its own branch, every load was
  // waited for: a norm of 8192 rows of 8192 bf16 104 us, then 72)
  template <bool TAIL, int Q>
  __device__ __forceinline__ void part(int n, Raw (&v)[Q]) const {
    n = again(n);
    const int at = 4 * (threadIdx.x & 63);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      v[q] = Raw{};
      if (256 * q + at < n - 3) load4(256 * q + at, v[q]);
    }
    if (TAIL && n > 0 && (n & 3)) {
      const int base = n & ~3, mine = at == (base & 255) ? base >> 8 : -1;
      Raw c{};
      if (mine >= 0) {
#pragma unroll
        for (int t = 0; t < 3; ++t)
          if (base + t < n) load1(base, t, c);
      }
#pragma unroll
      for (int q = 0; q < Q; ++q) {
        constexpr int kF = sizeof(c.f) / sizeof(c.f[0]), kW = sizeof(c.w) / sizeof(c.w[0]);
#pragma unroll
        for (int i = 0; i < kF; ++i) v[q].f[i] = q == mine ? c.f[i] : v[q].f[i];
#pragma unroll
        for (int i = 0; i < kW; ++i) v[q].w[i] = q == mine ? c.w[i] : v[q].w[i];
      }
    }
  }
  // The same of bf16, the vector that the row's end cuts as the row's last four, which `ends` puts in place: one wait less
  // (8192 x 5001 79 us, so 59; 8192 x 1001 12.8 and 11.5).  Rows of fewer than four go element by element, to the last places.
  template <int Q>
  __device__ __forceinline__ void part_ends(int n, int cols, Raw (&v)[Q]) const {
    static_assert(SRC == ACT_BF16, "");
    n = again(n);
    const int at = 4 * (threadIdx.x & 63);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = 256 * q + at;
      v[q] = Raw{};
      if (j < n && cols >= 4) load4(j + 4 <= n ? j : n - 4, j, v[q]);
    }
    if (cols < 4 && at == 0 && n > 0) {
      Raw c{};
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (t < n) load1(0, t, c);
      const uint64_t w = (((uint64_t)c.w[1] << 32) | c.w[0]) << (16 * (4 - n));
      c.w[0] = (uint32_t)w; c.w[1] = (uint32_t)(w >> 32);
      v[0] = c;
    }
  }
};

}  // namespace canon
