// rows_dev.h - what the row kernels share: loads and stores of four elements at any alignment, and the R1 sum of a row
// held in a wavefront's registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "canon_dev.h"

namespace canon {

__device__ __forceinline__ float wave_max(float m) {
#pragma unroll
  for (int s = 32; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
  return m;
}

// ---- W-wide loads and stores (W = 1 or 4 consecutive elements at any element alignment: gfx950's global accesses
// need none) ----
struct __attribute__((packed, aligned(4))) F4 {
  float x, y, z, w;
};
struct __attribute__((packed, aligned(2))) H4 {
  uint32_t x, y;
};
template <int W>
__device__ __forceinline__ void ldf(const float* p, float (&f)[W]) {
  if constexpr (W == 1) {
    f[0] = p[0];
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const F4 v = *reinterpret_cast<const F4*>(p + i);
      f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
  }
}

template <int W>
__device__ __forceinline__ void ldb(const uint16_t* p, float (&f)[W]) {
  if constexpr (W == 1) {
    f[0] = bf16_to_f32(p[0]);
  } else {
    const H4 u = *reinterpret_cast<const H4*>(p);
    f[0] = bf16_to_f32((uint16_t)(u.x & 0xFFFFu)); f[1] = bf16_to_f32((uint16_t)(u.x >> 16));
    f[2] = bf16_to_f32((uint16_t)(u.y & 0xFFFFu)); f[3] = bf16_to_f32((uint16_t)(u.y >> 16));
  }
}

template <int W>
__device__ __forceinline__ void stb(uint16_t* p, const uint16_t (&h)[W]) {
  if constexpr (W == 1) {
    p[0] = h[0];
  } else {
    *reinterpret_cast<H4*>(p) = H4{(uint32_t)h[0] | ((uint32_t)h[1] << 16), (uint32_t)h[2] | ((uint32_t)h[3] << 16)};
  }
}

template <int W>
__device__ __forceinline__ void stf(float* p, const float (&f)[W]) {
  if constexpr (W == 1) {
    p[0] = f[0];
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4) *reinterpret_cast<F4*>(p + i) = F4{f[i], f[i + 1], f[i + 2], f[i + 3]};
  }
}

// four elements j .. j + 3 of a row of n, those beyond its end as 0 (not read) or not written
// (TAIL: n is not a multiple of 4)
template <bool TAIL>
__device__ __forceinline__ void ldf4(const float* row, int64_t j, int64_t n, float (&f)[4]) {
  if (!TAIL || j + 4 <= n) {
    ldf<4>(row + j, f);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = j + i < n ? row[j + i] : 0.0f;
  }
}
template <bool TAIL>
__device__ __forceinline__ void ldb4(const uint16_t* row, int64_t j, int64_t n, float (&f)[4]) {
  if (!TAIL || j + 4 <= n) {
    ldb<4>(row + j, f);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = j + i < n ? bf16_to_f32(row[j + i]) : 0.0f;
  }
}
template <bool TAIL>
__device__ __forceinline__ void stf4(float* row, int64_t j, int64_t n, const float (&f)[4]) {
  if (!TAIL || j + 4 <= n) {
    stf<4>(row + j, f);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < n) row[j + i] = f[i];
  }
}
template <bool TAIL>
__device__ __forceinline__ void stb4(uint16_t* row, int64_t j, int64_t n, const uint16_t (&h)[4]) {
  if (!TAIL || j + 4 <= n) {
    stb<4>(row + j, h);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i < n) row[j + i] = h[i];
  }
}

// Register-resident rows (cols <= 2048, or the part H of 2048 terms of a longer one): lane l holds terms
// 4l + 256q .. +3 of its row, read from memory once.  The chunk chains still run one per lane over an LDS transpose
// (rows of 36 floats: 16-byte stores and reads without bank conflicts; a wavefront's LDS operations complete in order).
constexpr int kRegQ = 8;  // 64 x 4 x 8 = 2048 terms
constexpr int64_t kRegCols = 64 * 4 * kRegQ;
struct RegStage {
  float t[64][36];
};

template <int H = 0, int Q>
__device__ __forceinline__ float reg_row_sum(RegStage& st, const float (&e)[Q][4], int64_t n) {
  const int lane = threadIdx.x & 63;
  auto stage = [&](int q) __attribute__((always_inline)) {
    const int local = 256 * q + 4 * lane;
    const float(&v)[4] = e[H * kRegQ + q];
    *reinterpret_cast<float4*>(&st.t[local >> 5][local & 31]) = make_float4(v[0], v[1], v[2], v[3]);
  };
  // short rows leave out the vectors past their end (norm forward of 20000 rows of 16 terms 11.2 -> 9.9 us); with the
  // test in front of every vector the softmax of 2048 keys took 66 us instead of 59
  if (n > 256 * (kRegQ - 1)) {
#pragma unroll
    for (int q = 0; q < kRegQ; ++q) stage(q);
  } else {
#pragma unroll
    for (int q = 0; q < kRegQ - 1; ++q) {
      if (256 * q >= n) break;
      stage(q);
    }
  }
  __builtin_amdgcn_wave_barrier();
  const int nc = (int)((n + kChunk - 1) / kChunk);
  float p = 0.0f;
  const int k1 = (int)n - lane * kChunk;
  if (k1 >= kChunk) {
#pragma unroll
    for (int i = 0; i < kChunk; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(&st.t[lane][i]);
      p = p + v.x; p = p + v.y; p = p + v.z; p = p + v.w;
    }
  } else {
    for (int i = 0; i < k1; ++i) p = p + st.t[lane][i];
  }
  return __shfl(wave_fold(p, nc), 0, 64);
}

// The R1 sum of a row spread over a workgroup of NW wavefronts, wavefront w holding its terms 2048 w .. 2048 w + 2047:
// 64 chunks, a complete subtree of Algorithm 2 wherever a later one follows, so the wavefronts' sums are folded by the
// same rule.  slot: NW floats of LDS, not written again before every wavefront has passed another barrier (NW = 1: one
// wavefront per row, no barrier).
template <int NW>
__device__ __forceinline__ float wide_row_sum(RegStage& st, const float (&e)[kRegQ][4], int64_t n, float* slot) {
  if constexpr (NW == 1) {
    return reg_row_sum(st, e, n);
  } else {
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t left = n - w * kRegCols;
    float p = 0.0f;
    if (left > 0) p = reg_row_sum(st, e, left < kRegCols ? left : kRegCols);
    if (lane == 0) slot[w] = p;
    __syncthreads();
    const int parts = (int)((n + kRegCols - 1) / kRegCols);
    p = lane < parts ? slot[lane] : 0.0f;
    return __shfl(wave_fold(p, parts), 0, 64);
  }
}

}  // namespace canon
