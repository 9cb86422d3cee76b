// act8.hip - activations kept in 8 bits between the forward and the backward pass (R21), and SwiGLU that keeps its input
// so and reads it back (R4's rule).  One pass over the data each; bound: HBM.
#include <hip/hip_runtime.h>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

namespace {

// A wavefront takes kTileQ vectors of 256 consecutive elements of a row (all its loads in flight before the first group
// is reduced), then the tile a grid further on.
constexpr int kTileQ = 4;
constexpr int64_t kTile = 256 * kTileQ;
constexpr int64_t kMaxBlocks = 1 << 20;

unsigned tile_blocks(int64_t tiles) {
  const int64_t b = (tiles + 3) / 4;
  return (unsigned)(b < kMaxBlocks ? b : kMaxBlocks);
}

// Steps and codes: a group's largest magnitude is joined over the 8 to 64 lanes that hold it, the tile's four vectors a step
// at a time.  8192 x 8192 fp32 80 us: 337 MB moved, 4.2 TB/s; 33 x 2048 4.5 us, a launch and one load's latency.
template <int SRC, bool TAIL>
__global__ __launch_bounds__(256) void act8_pack_kernel(int64_t rows, int64_t cols, int64_t tiles, ActIn x, ActKeep k) {
  const int lane = threadIdx.x & 63;
  const int64_t per_row = (cols + kTile - 1) / kTile, groups = (cols + (1 << k.lg) - 1) >> k.lg;
  for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += (int64_t)gridDim.x * 4) {
    const int64_t row = tile / per_row, j0 = (tile - row * per_row) * kTile + 4 * lane;
    float v[kTileQ][4];
#pragma unroll
    for (int q = 0; q < kTileQ; ++q) {
      const int64_t j = j0 + 256 * q;
#pragma unroll
      for (int t = 0; t < 4; ++t) v[q][t] = 0.0f;
      if (j < cols) act4<SRC, TAIL>(x, row, j, cols, v[q]);
    }
    float s[kTileQ];
    steps4(v, k.lg, s);
#pragma unroll
    for (int q = 0; q < kTileQ; ++q)
      keep4<TAIL>(v[q], s[q], j0 + 256 * q, cols, k.lg, k.codes + row * cols, k.steps + row * groups);
  }
}

// The values again: 65 us for the same 337 MB, 5.2 TB/s.
template <bool BF16, bool TAIL>
__global__ __launch_bounds__(256) void act8_unpack_kernel(int64_t rows, int64_t cols, int64_t tiles, ActIn k,
                                                          void* __restrict__ out) {
  const int lane = threadIdx.x & 63;
  const int64_t per_row = (cols + kTile - 1) / kTile;
  for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += (int64_t)gridDim.x * 4) {
    const int64_t row = tile / per_row, j0 = (tile - row * per_row) * kTile + 4 * lane;
    float v[kTileQ][4];
#pragma unroll
    for (int q = 0; q < kTileQ; ++q)
      if (j0 + 256 * q < cols) act4<ACT_Q8, TAIL>(k, row, j0 + 256 * q, cols, v[q]);
#pragma unroll
    for (int q = 0; q < kTileQ; ++q) {
      const int64_t j = j0 + 256 * q;
      if (j >= cols) continue;
      if (BF16) {
        stb4_arith<TAIL>((uint16_t*)out + row * cols, j, cols, v[q]);
      } else {
        stf4<TAIL>((float*)out + row * cols, j, cols, v[q]);
      }
    }
  }
}

// SwiGLU of a tile of kGluQ vectors of gate and the same of up: a = bf16(RN(silu(g) u)); with keep, the tile's codes, gate
// and up as two rows of F.  8192 x 8192 from fp32, kept: 150 us for 809 MB, 5.4 TB/s.
constexpr int kGluQ = 2;
constexpr int64_t kGluTile = 256 * kGluQ;

template <int SRC, bool TAIL, bool KEEP>
__global__ __launch_bounds__(256) void swiglu_keep_kernel(int64_t T, int64_t F, int64_t tiles, ActIn gu,
                                                          uint16_t* __restrict__ a, ActKeep k) {
  const int lane = threadIdx.x & 63;
  const int64_t per_row = (F + kGluTile - 1) / kGluTile, groups = KEEP ? (F + (1 << k.lg) - 1) >> k.lg : 0;
  for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += (int64_t)gridDim.x * 4) {
    const int64_t t = tile / per_row, j0 = (tile - t * per_row) * kGluTile + 4 * lane;
    float g[kGluQ][4], u[kGluQ][4];
#pragma unroll
    for (int q = 0; q < kGluQ; ++q) {
      const int64_t j = j0 + 256 * q;
#pragma unroll
      for (int i = 0; i < 4; ++i) g[q][i] = u[q][i] = 0.0f;
      if (j < F) {
        act4<SRC, TAIL>(gu, 2 * t, j, F, g[q]);
        act4<SRC, TAIL>(gu, 2 * t + 1, j, F, u[q]);
      }
    }
    float sg[kGluQ], su[kGluQ];
    if (KEEP) {
      steps4(g, k.lg, sg);
      steps4(u, k.lg, su);
    }
#pragma unroll
    for (int q = 0; q < kGluQ; ++q) {
      const int64_t j = j0 + 256 * q;
      if (KEEP) {
        keep4<TAIL>(g[q], sg[q], j, F, k.lg, k.codes + 2 * t * F, k.steps + 2 * t * groups);
        keep4<TAIL>(u[q], su[q], j, F, k.lg, k.codes + (2 * t + 1) * F, k.steps + (2 * t + 1) * groups);
      }
      if (j >= F) continue;
      float h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sl = csilu(g[q][i]);
        h[i] = sl * u[q][i];
      }
      stb4_arith<TAIL>(a + t * F, j, F, h);
    }
  }
}

// its gradient: du = bf16(RN(da silu(g))), dg = bf16(RN(RN(da u) dsg)), dsg = RN(sig RN(1 + RN(g RN(1 - sig)))); with a
// the activation again (the same values' forward).  8192 x 8192 from 8 bits with the activation: 141 us for 809 MB, 5.7 TB/s.
template <int SRC, bool TAIL>
__global__ __launch_bounds__(256) void swiglu_grad_kernel(int64_t T, int64_t F, int64_t tiles, ActIn gu,
                                                          const float* __restrict__ da, uint16_t* __restrict__ dgu,
                                                          uint16_t* __restrict__ a) {
  const int lane = threadIdx.x & 63;
  const int64_t per_row = (F + kGluTile - 1) / kGluTile;
  for (int64_t tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); tile < tiles; tile += (int64_t)gridDim.x * 4) {
    const int64_t t = tile / per_row, j0 = (tile - t * per_row) * kGluTile + 4 * lane;
    float g[kGluQ][4], u[kGluQ][4], d[kGluQ][4];
#pragma unroll
    for (int q = 0; q < kGluQ; ++q) {
      const int64_t j = j0 + 256 * q;
      if (j >= F) continue;
      act4<SRC, TAIL>(gu, 2 * t, j, F, g[q]);
      act4<SRC, TAIL>(gu, 2 * t + 1, j, F, u[q]);
      ldf4<TAIL>(da + t * F, j, F, d[q]);
    }
#pragma unroll
    for (int q = 0; q < kGluQ; ++q) {
      const int64_t j = j0 + 256 * q;
      if (j >= F) continue;
      float hg[4], hu[4], ha[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float sig = csigmoid(g[q][i]);
        const float sl = g[q][i] * sig;
        const float oms = 1.0f - sig;
        const float gs = g[q][i] * oms;
        const float ops = 1.0f + gs;
        const float dsg = sig * ops;
        const float du = d[q][i] * u[q][i];
        hg[i] = du * dsg;
        hu[i] = d[q][i] * sl;
        ha[i] = sl * u[q][i];
      }
      stb4_arith<TAIL>(dgu + 2 * t * F, j, F, hg);
      stb4_arith<TAIL>(dgu + (2 * t + 1) * F, j, F, hu);
      if (a) stb4_arith<TAIL>(a + t * F, j, F, ha);
    }
  }
}

// Rows of whole groups follow each other without a gap in codes and steps alike: one long row.
void join_rows(int64_t& rows, int64_t& cols, int lg) {
  if ((cols & ((1 << lg) - 1)) == 0) {
    cols *= rows;
    rows = 1;
  }
}

}  // namespace

hipError_t act8_pack_launch(int64_t rows, int64_t cols, const ActIn& x, const ActKeep& k, hipStream_t s) {
  if (rows * cols == 0) return hipSuccess;
  join_rows(rows, cols, k.lg);
  const int64_t tiles = rows * ((cols + kTile - 1) / kTile);
  const dim3 grid(tile_blocks(tiles));
#define CANON_PACK(SRC, TAIL) \
  hipLaunchKernelGGL((act8_pack_kernel<SRC, TAIL>), grid, dim3(256), 0, s, rows, cols, tiles, x, k)
  if (x.src == ACT_F32) {
    if (cols % 4 == 0) CANON_PACK(ACT_F32, false);
    else CANON_PACK(ACT_F32, true);
  } else {
    if (cols % 4 == 0) CANON_PACK(ACT_BF16, false);
    else CANON_PACK(ACT_BF16, true);
  }
#undef CANON_PACK
  return hipGetLastError();
}

hipError_t act8_unpack_launch(int64_t rows, int64_t cols, const ActIn& k, int out_bf16, void* out, hipStream_t s) {
  if (rows * cols == 0) return hipSuccess;
  join_rows(rows, cols, k.lg);
  const int64_t tiles = rows * ((cols + kTile - 1) / kTile);
  const dim3 grid(tile_blocks(tiles));
#define CANON_UNPACK(BF16, TAIL) \
  hipLaunchKernelGGL((act8_unpack_kernel<BF16, TAIL>), grid, dim3(256), 0, s, rows, cols, tiles, k, out)
  if (out_bf16) {
    if (cols % 4 == 0) CANON_UNPACK(true, false);
    else CANON_UNPACK(true, true);
  } else {
    if (cols % 4 == 0) CANON_UNPACK(false, false);
    else CANON_UNPACK(false, true);
  }
#undef CANON_UNPACK
  return hipGetLastError();
}

hipError_t swiglu_keep_launch(int64_t T, int64_t F, const ActIn& gu, uint16_t* a, const ActKeep& k, hipStream_t s) {
  if (T * F == 0) return hipSuccess;
  const int64_t tiles = T * ((F + kGluTile - 1) / kGluTile);
  const dim3 grid(tile_blocks(tiles));
#define CANON_GLU(SRC, TAIL)                                                                                       \
  do {                                                                                                             \
    if (k.codes)                                                                                                   \
      hipLaunchKernelGGL((swiglu_keep_kernel<SRC, TAIL, true>), grid, dim3(256), 0, s, T, F, tiles, gu, a, k);     \
    else                                                                                                           \
      hipLaunchKernelGGL((swiglu_keep_kernel<SRC, TAIL, false>), grid, dim3(256), 0, s, T, F, tiles, gu, a, k);    \
  } while (0)
  if (gu.src == ACT_F32) {
    if (F % 4 == 0) CANON_GLU(ACT_F32, false);
    else CANON_GLU(ACT_F32, true);
  } else {
    if (F % 4 == 0) CANON_GLU(ACT_BF16, false);
    else CANON_GLU(ACT_BF16, true);
  }
#undef CANON_GLU
  return hipGetLastError();
}

hipError_t swiglu_grad_launch(int64_t T, int64_t F, const ActIn& gu, const float* da, uint16_t* dgu, uint16_t* a,
                              hipStream_t s) {
  if (T * F == 0) return hipSuccess;
  const int64_t tiles = T * ((F + kGluTile - 1) / kGluTile);
  const dim3 grid(tile_blocks(tiles));
#define CANON_GLU(SRC)                                                                                            \
  do {                                                                                                            \
    if (F % 4 == 0)                                                                                               \
      hipLaunchKernelGGL((swiglu_grad_kernel<SRC, false>), grid, dim3(256), 0, s, T, F, tiles, gu, da, dgu, a);   \
    else                                                                                                          \
      hipLaunchKernelGGL((swiglu_grad_kernel<SRC, true>), grid, dim3(256), 0, s, T, F, tiles, gu, da, dgu, a);    \
  } while (0)
  if (gu.src == ACT_F32) CANON_GLU(ACT_F32);
  else if (gu.src == ACT_BF16) CANON_GLU(ACT_BF16);
  else CANON_GLU(ACT_Q8);
#undef CANON_GLU
  return hipGetLastError();
}

}  // namespace canon
