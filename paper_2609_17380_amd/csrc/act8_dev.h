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

// the largest of m over each aligned set of `lanes` lanes (a power of two from 8 to 64)
__device__ __forceinline__ uint32_t lanes_max(uint32_t m, int lanes) {
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) {
    if (s >= lanes) break;
    const uint32_t o = __shfl_xor(m, s, 64);
    m = o > m ? o : m;
  }
  return m;
}

// Elements j .. j + 3 of a row of n (j a multiple of 4 whose lanes run through whole groups; v holds 0 beyond n) into
// codes and their group's step.  Every lane of the wavefront takes part.  The magnitudes are compared as bit patterns,
// so that a NaN ranks above every number.
template <bool TAIL>
__device__ __forceinline__ void keep4(const float (&v)[4], int64_t j, int64_t n, int lg, int8_t* codes, float* steps) {
  uint32_t m = 0;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const uint32_t a = __float_as_uint(v[t]) & 0x7FFFFFFFu;
    m = a > m ? a : m;
  }
  m = lanes_max(m, 1 << (lg - 2));
  const float s = __uint_as_float(m) * __uint_as_float(kInv127Bits);
  const bool recip = recip_step_ok(s);
  const float rs = recip ? 1.0f / s : 0.0f;
  uint32_t w[1];
  quant_pack<4>(v, s, rs, recip, w);
  if (j >= n) return;
  if ((j & ((1 << lg) - 1)) == 0) steps[j >> lg] = s;
  if (!TAIL || j + 4 <= n) {
    reinterpret_cast<B4*>(codes + j)->x = w[0];
  } else {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      if (j + t < n) codes[j + t] = (int8_t)(w[0] >> (8 * t));
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

// four elements of row `row` of an activation: fp32, bf16 or kept in 8 bits
template <int SRC, bool TAIL>
__device__ __forceinline__ void act4(const ActIn& a, int64_t row, int64_t j, int64_t n, float (&f)[4]) {
  if constexpr (SRC == ACT_F32) ldf4<TAIL>((const float*)a.x + row * n, j, n, f);
  else if constexpr (SRC == ACT_BF16) ldb4<TAIL>((const uint16_t*)a.x + row * n, j, n, f);
  else kept4<TAIL>((const int8_t*)a.x + row * n, a.steps + row * ((n + (1 << a.lg) - 1) >> a.lg), j, n, a.lg, f);
}

}  // namespace canon
