// gemm_i8_rows.hip - activations into 8 bits with a step per token (R23), and the int8 product of a few tokens with weights.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "i8_dev.h"
#include "rows_dev.h"

namespace canon {

// ---- a step per token -----------------------------------------------------------------------------------------------------
// A workgroup holds a row in registers, Q vectors of four elements a thread (Q = 0: longer rows, read a second time): one pass
// over memory, one join of the maximum between.  8192 x 2048 from bf16: 13.9 us; one row of 2048 2.5, a launch.
template <bool XB, int NT, int Q>
__global__ __launch_bounds__(NT) void quant_tokens_kernel(int64_t rows, int64_t cols, const void* __restrict__ x,
                                                          int8_t* __restrict__ codes, float* __restrict__ steps) {
  __shared__ uint32_t tops[NT / 64];
  const int64_t r = blockIdx.x;
  const int n = (int)cols;
  auto load = [&](int j, float (&v)[4]) {
    if constexpr (XB) {
      const uint16_t* p = (const uint16_t*)x + r * cols + j;
      if (j + 4 <= n) {
        ldb<4>(p, v);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = j + e < n ? bf16_to_f32(p[e]) : 0.0f;
      }
    } else {
      ldf4<true>((const float*)x + r * cols, j, cols, v);
    }
  };
  auto top_of = [](const float (&v)[4], uint32_t m) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t u = __float_as_uint(v[e]) & 0x7FFFFFFFu;
      m = u > m ? u : m;
    }
    return m;
  };
  float v[Q > 0 ? Q : 1][4];
  uint32_t m = 0;
  if constexpr (Q > 0) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = 4 * (threadIdx.x + NT * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[q][e] = 0.0f;
      if (j < n) load(j, v[q]);
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) m = top_of(v[q], m);
  } else {
    for (int j = 4 * threadIdx.x; j < n; j += 4 * NT) {
      load(j, v[0]);
      m = top_of(v[0], m);
    }
  }
  m = lanes_join(m, 64, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NT / 64; ++i) m = tops[i] > m ? tops[i] : m;
  }
  const float s = __uint_as_float(m) * __uint_as_float(kInv127Bits);
  if (threadIdx.x == 0) steps[r] = s;
  const float rs = step_rcp(s);
  const bool recip = recip_step_ok(s);
  int8_t* out = codes + r * cols;
  auto keep = [&](int j, const float (&f)[4]) {
    uint32_t w[1];
    quant_pack<4>(f, s, rs, recip, w);
    if (j + 4 <= n) {
      reinterpret_cast<B4*>(out + j)->x = w[0];
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (j + e < n) out[j + e] = (int8_t)(w[0] >> (8 * e));
    }
  };
  if constexpr (Q > 0) {
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int j = 4 * (threadIdx.x + NT * q);
      if (j < n) keep(j, v[q]);
    }
  } else {
    for (int j = 4 * threadIdx.x; j < n; j += 4 * NT) {
      load(j, v[0]);
      keep(j, v[0]);
    }
  }
}

template <bool XB>
static hipError_t quant_go(int64_t rows, int64_t cols, const void* x, int8_t* codes, float* steps, hipStream_t s) {
  // workgroups of a launch: below 2^32 threads
  const int64_t most = (int64_t)1 << 23;
  for (int64_t r0 = 0; r0 < rows; r0 += most) {
    const int64_t n = rows - r0 < most ? rows - r0 : most;
    const void* xr = (const char*)x + r0 * cols * (XB ? 2 : 4);
    int8_t* cr = codes + r0 * cols;
    float* sr = steps + r0;
    auto go = [&](auto nt, auto q) {
      hipLaunchKernelGGL((quant_tokens_kernel<XB, nt.value, q.value>), dim3((unsigned)n), dim3(nt.value), 0, s, n, cols, xr, cr,
                         sr);
    };
    using N64 = std::integral_constant<int, 64>;
    using N256 = std::integral_constant<int, 256>;
    using N1024 = std::integral_constant<int, 1024>;
    if (cols <= 256) go(N64{}, std::integral_constant<int, 1>{});
    else if (cols <= 512) go(N64{}, std::integral_constant<int, 2>{});
    else if (cols <= 1024) go(N256{}, std::integral_constant<int, 1>{});
    else if (cols <= 2048) go(N256{}, std::integral_constant<int, 2>{});
    else if (rows < 256 && cols <= 4096) go(N1024{}, std::integral_constant<int, 1>{});
    else if (rows < 256 && cols <= 8192) go(N1024{}, std::integral_constant<int, 2>{});
    else if (cols <= 4096) go(N256{}, std::integral_constant<int, 4>{});
    else if (cols <= 8192) go(N256{}, std::integral_constant<int, 8>{});
    else if (cols <= 16384) go(N256{}, std::integral_constant<int, 16>{});
    else go(N256{}, std::integral_constant<int, 0>{});
  }
  return hipGetLastError();
}

hipError_t quant_tokens_launch(int64_t rows, int64_t cols, int32_t bf16, const void* x, int8_t* codes, float* steps,
                               hipStream_t s) {
  return bf16 ? quant_go<true>(rows, cols, x, codes, steps, s) : quant_go<false>(rows, cols, x, codes, steps, s);
}

// ---- few tokens -----------------------------------------------------------------------------------------------------------
// What counts is the weights' stream.  A workgroup takes CW channels over all of k, its 8 wavefronts every eighth cache line of
// them, so that a channel's row is read in runs of 1024 bytes and the whole chip has loads in flight however few the channels
// are; the partial sums are whole numbers and are joined through LDS in any order.  Channels are the rows of
// v_mfma_i32_16x16x64_i8 and tokens its columns: lane (c, g) supplies bytes 16 g .. + 15 of channel c and of token c, and
// receives channels 4 g .. 4 g + 3 of token c, which it stores together.  With CW = 8 half of the rows stay empty.

template <int CW, int U>
__global__ __launch_bounds__(512) void gemm_i8_rows_kernel(GemmI8Args g) {
  constexpr int NW = 8;
  __shared__ __attribute__((aligned(16))) i32x4 part[NW][64];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, q = lane >> 4;
  const int64_t col0 = (int64_t)blockIdx.x * CW;
  const int64_t ch = col0 + c;
  const bool has = c < CW && ch < g.n;
  const int8_t* bp = g.b + (has ? ch : 0) * g.ldb + 16 * q;
  const bool tok = c < g.m;
  const int8_t* ap = g.a + (tok ? c : 0) * g.lda + 16 * q;
  i32x4 acc = {0, 0, 0, 0};
  // Whole steps: this wavefront has 2 w, 2 w + 1 (a cache line), 16 + 2 w, ...  Workgroups begin at different ones: tokens' rows a power of two apart come
  // from the same few channels of the L2, and all workgroups would ask for the same bytes at once.
  const int32_t steps = (int32_t)(g.k >> 6), rest = (steps & 15) - 2 * w;
  const int32_t mine = 2 * (steps >> 4) + (rest > 1 ? 2 : rest > 0 ? rest : 0);
  const int32_t rot = mine > 1 ? 2 * (int32_t)((blockIdx.x >> 3) % (uint32_t)(mine >> 1)) : 0;  // by 8: within an XCD
  for (int32_t j0 = 0; j0 < mine; j0 += U) {
    i32x4 b[U], a[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      int32_t j = (j0 + u < mine ? j0 + u : mine - 1) + rot;
      j = j < mine ? j : j - mine;
      at[u] = 64 * (int64_t)(16 * (j >> 1) + 2 * w + (j & 1));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) b[u] = i32x4{0, 0, 0, 0};
    if (has) {
#pragma unroll
      for (int u = 0; u < U; ++u) b[u] = whole16(bp + at[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) a[u] = i32x4{0, 0, 0, 0};
    if (tok) {
#pragma unroll
      for (int u = 0; u < U; ++u) a[u] = whole16(ap + at[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u >= mine) break;
      acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b[u], a[u], acc, 0, 0, 0);
    }
  }
  if ((g.k & 63) && w == (steps & (NW - 1))) {  // the cut step
    const int64_t valid = (g.k & 63) - 16 * q;
    const bool longer = g.k >= 16;
    const i32x4 b = cut16(bp + 64 * (int64_t)steps, has ? valid : 0, longer);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(b, cut16(ap + 64 * (int64_t)steps, tok ? valid : 0, longer), acc, 0, 0, 0);
  }
  part[w][lane] = acc;
  __syncthreads();
  if (w > 0) return;
  i32x4 sum = {0, 0, 0, 0};
#pragma unroll
  for (int o = 0; o < NW; ++o) sum = sum + part[o][lane];
  const int64_t i = c;
  if (i >= g.m || 4 * q >= CW) return;
  const float sa = g.sa[i];
  const int64_t j0 = col0 + 4 * q;
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = j0 + e < g.n ? ((float)sum[e] * sa) * g.sb[j0 + e] : 0.0f;
  if (g.y_bf16) {
    uint16_t* o = reinterpret_cast<uint16_t*>(g.y) + i * g.ldc + j0;
    if (j0 + 4 <= g.n) {
      *reinterpret_cast<H4*>(o) = H4{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (j0 + e < g.n) o[e] = f32_to_bf16(y[e]);
    }
  } else {
    float* o = g.y + i * g.ldc + j0;
    if (j0 + 4 <= g.n) {
      stf<4>(o, y);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (j0 + e < g.n) o[e] = y[e];
    }
  }
}

hipError_t gemm_i8_rows_launch(const GemmI8Args& g, hipStream_t s) {
  auto go = [&](auto cw, auto u) {
    hipLaunchKernelGGL((gemm_i8_rows_kernel<cw.value, u.value>), dim3((unsigned)((g.n + cw.value - 1) / cw.value)), dim3(512), 0,
                       s, g);
    return hipGetLastError();
  };
  auto depth = [&](auto cw) {  // as many steps on their way as a wavefront has, up to 8
    if (g.k < 64 * 8 * 8) return go(cw, std::integral_constant<int, 4>{});
    return go(cw, std::integral_constant<int, 8>{});
  };
  // half as many channels a workgroup where there would be fewer workgroups than CUs
  if (g.n <= 2048) return depth(std::integral_constant<int, 8>{});
  return depth(std::integral_constant<int, 16>{});
}

}  // namespace canon
