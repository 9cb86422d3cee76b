// gemm_i8_split.hip - the exact int8 GEMM of gemm_i8.hip for outputs that are no whole 256 x 256 tiles, or too few of them.
//
// The sum over k is exact, so a workgroup's eight wavefronts take every eighth 128 bytes of k of the same TM x TN tile and join
// their int32 sums through LDS at the end.  Nothing is shared before: each wavefront brings its own rows into its own part of
// LDS (128 bytes of eight rows a load, whole cache lines, where loading the operands of the matrix instructions directly takes
// pieces of 64 bytes of 16 rows that fall on the same few channels), the next ones on their way in registers meanwhile, and no
// barrier is met in the loop.
#include <hip/hip_runtime.h>

#include "canon_dev.h"
#include "canon_internal.h"
#include "i8_dev.h"

namespace canon {

typedef int32_t i32x16 __attribute__((ext_vector_type(16)));
template <int TM, int TN>
__global__ __launch_bounds__(512) void gemm_i8_split_kernel(GemmI8Args g, int64_t tiles_m, int64_t tiles_n) {
  constexpr int NW = 8, KS = 128, LD = KS + 16;  // padded rows: 32 of them at one k offset fall on different banks
  constexpr int HB = TM / 32, WN = TN / 32, AV = TM / 8, BV = TN / 8;
  constexpr int PART = (TM + TN) * LD;
  static_assert(PART >= TM * TN * 4, "a wavefront's sums fit where its rows were");
  __shared__ __attribute__((aligned(16))) int8_t lds[NW * PART];

  // a contiguous run of tiles per XCD, walked in groups of 8 tile rows
  constexpr int64_t GM = 8;
  const int64_t tiles = tiles_m * tiles_n, per = (tiles + 7) >> 3;
  const int64_t tile = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
  if ((int64_t)(blockIdx.x >> 3) >= per || tile >= tiles) return;
  const int64_t group = tile / (GM * tiles_n), first_m = group * GM;
  const int64_t gsize = (tiles_m - first_m) < GM ? (tiles_m - first_m) : GM;
  const int64_t within = tile - group * GM * tiles_n;
  const int64_t row0 = (first_m + within % gsize) * TM, col0 = (within / gsize) * TN;

  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int8_t* const mine = lds + w * PART;
  // rows behind the last are read as the last: what they give is not stored
  const int lr = lane >> 3, ls = 16 * (lane & 7);
  const int8_t *ap[AV], *bp[BV];
#pragma unroll
  for (int i = 0; i < AV; ++i) {
    const int64_t r = row0 + 8 * i + lr;
    ap[i] = g.a + (r < g.m ? r : g.m - 1) * g.lda + ls;
  }
#pragma unroll
  for (int i = 0; i < BV; ++i) {
    const int64_t r = col0 + 8 * i + lr;
    bp[i] = g.b + (r < g.n ? r : g.n - 1) * g.ldb + ls;
  }
  i32x16 acc[HB][WN];
#pragma unroll
  for (int h = 0; h < HB; ++h)
#pragma unroll
    for (int v2 = 0; v2 < WN; ++v2)
#pragma unroll
      for (int v = 0; v < 16; ++v) acc[h][v2][v] = 0;

  i32x4 ra[AV], rb[BV];
  const bool longer = g.k >= 16;
  auto load = [&](int64_t st) {
    const int64_t k0 = st * KS;
    if (k0 + KS <= g.k) {
#pragma unroll
      for (int i = 0; i < AV; ++i) ra[i] = whole16(ap[i] + k0);
#pragma unroll
      for (int i = 0; i < BV; ++i) rb[i] = whole16(bp[i] + k0);
    } else {
      const int64_t valid = g.k - k0 - ls;
#pragma unroll
      for (int i = 0; i < AV; ++i) ra[i] = cut16(ap[i] + k0, valid, longer);
#pragma unroll
      for (int i = 0; i < BV; ++i) rb[i] = cut16(bp[i] + k0, valid, longer);
    }
  };
  // this wavefront's stages: w, w + 8, ...; workgroups begin at different ones, as rows a power of two apart come from the same
  // channels of the L2
  const int32_t stages = (int32_t)((g.k + KS - 1) / KS), count = (stages - w + NW - 1) / NW;
  const int32_t rot = count > 0 ? (int32_t)((blockIdx.x >> 3) % (uint32_t)count) : 0;
  auto at = [&](int32_t j) {
    j += rot;
    return (int64_t)(w + NW * (j < count ? j : j - count));
  };
  const int rl = lane & 31, kh = 16 * (lane >> 5);
  if (count > 0) load(at(0));
  for (int32_t j = 0; j < count; ++j) {
#pragma unroll
    for (int i = 0; i < AV; ++i) *reinterpret_cast<i32x4*>(mine + (8 * i + lr) * LD + ls) = ra[i];
#pragma unroll
    for (int i = 0; i < BV; ++i) *reinterpret_cast<i32x4*>(mine + (TM + 8 * i + lr) * LD + ls) = rb[i];
    in_order();
    if (j + 1 < count) load(at(j + 1));
#pragma unroll
    for (int ks = 0; ks < KS / 32; ++ks) {
      i32x4 a[HB], b[WN];
#pragma unroll
      for (int h = 0; h < HB; ++h) a[h] = *reinterpret_cast<const i32x4*>(mine + (32 * h + rl) * LD + 32 * ks + kh);
#pragma unroll
      for (int v2 = 0; v2 < WN; ++v2) b[v2] = *reinterpret_cast<const i32x4*>(mine + (TM + 32 * v2 + rl) * LD + 32 * ks + kh);
#pragma unroll
      for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int v2 = 0; v2 < WN; ++v2)
          acc[h][v2] = __builtin_amdgcn_mfma_i32_32x32x32_i8(a[h], b[v2], acc[h][v2], 0, 0, 0);
    }
    in_order();
  }

  // the sums: four registers of a lane are rows r .. r + 3 of column lane % 32 of a 32 x 32 block, r = 8 (v / 4) + 4 (lane / 32)
#pragma unroll
  for (int h = 0; h < HB; ++h)
#pragma unroll
    for (int v2 = 0; v2 < WN; ++v2)
#pragma unroll
      for (int v = 0; v < 4; ++v)
        *reinterpret_cast<i32x4*>(mine + 16 * (64 * (4 * (h * WN + v2) + v) + lane)) =
            i32x4{acc[h][v2][4 * v], acc[h][v2][4 * v + 1], acc[h][v2][4 * v + 2], acc[h][v2][4 * v + 3]};
  __syncthreads();
  // everything is finished before the first store: a wait between two stores is one for the first of them
  constexpr int VECS = TM * TN / 4, IT = VECS > 512 ? VECS / 512 : 1;
  if (VECS < 512 && threadIdx.x >= VECS) return;
  i32x4 sum[IT];
  float y[IT][4];
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int idx = (int)threadIdx.x + 512 * it, l = idx & 63, v = (idx >> 6) & 3, blk = idx >> 8;
    const int64_t j = col0 + 32 * (blk % WN) + (l & 31), i0 = row0 + 32 * (blk / WN) + 8 * v + 4 * (l >> 5);
    float sb = 0.0f, sa[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (g.y) {
      sb = g.sb[g.sb_scalar ? 0 : j < g.n ? j : g.n - 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) sa[e] = g.sa[!g.sa_rows ? 0 : i0 + e < g.m ? i0 + e : g.m - 1];
    }
    sum[it] = i32x4{0, 0, 0, 0};
#pragma unroll
    for (int o = 0; o < NW; ++o) sum[it] = sum[it] + *reinterpret_cast<const i32x4*>(lds + o * PART + 16 * idx);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float t = (float)sum[it][e] * sa[e];
      y[it][e] = t * sb;
      asm volatile("" : "+v"(y[it][e]));
    }
  }
#pragma unroll
  for (int it = 0; it < IT; ++it) {
    const int idx = (int)threadIdx.x + 512 * it, l = idx & 63, v = (idx >> 6) & 3, blk = idx >> 8;
    const int64_t j = col0 + 32 * (blk % WN) + (l & 31), i0 = row0 + 32 * (blk / WN) + 8 * v + 4 * (l >> 5);
    if (j >= g.n) continue;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t i = i0 + e;
      if (i >= g.m) break;
      if (g.acc) g.acc[i * g.ldc + j] = sum[it][e];
      if (g.y && g.y_bf16) reinterpret_cast<uint16_t*>(g.y)[i * g.ldc + j] = f32_to_bf16(y[it][e]);
      else if (g.y) g.y[i * g.ldc + j] = y[it][e];
    }
  }
}

template <int TM, int TN>
static hipError_t split_go(const GemmI8Args& g, hipStream_t s) {
  const int64_t tm = (g.m + TM - 1) / TM, tn = (g.n + TN - 1) / TN, tiles = tm * tn;
  hipLaunchKernelGGL((gemm_i8_split_kernel<TM, TN>), dim3((unsigned)(8 * ((tiles + 7) / 8))), dim3(512), 0, s, g, tm, tn);
  return hipGetLastError();
}

// the largest tile of which there are enough to keep six tenths of the CUs busy (128 x 2048 x 8192: 22, 16 and 11.5 us with 64, 128
// and 256 tiles; 33 x 16384 x 2048: 11, 13.5 and 14 us with 256, 512 and 1024)
hipError_t gemm_i8_split_launch(const GemmI8Args& g, int cus, hipStream_t s) {
  const int64_t m64 = (g.m + 63) / 64, enough = 6 * (int64_t)cus / 10;
  if (m64 * ((g.n + 63) / 64) >= enough) return split_go<64, 64>(g, s);
  if (m64 * ((g.n + 31) / 32) >= enough) return split_go<64, 32>(g, s);
  return split_go<32, 32>(g, s);
}

}  // namespace canon
