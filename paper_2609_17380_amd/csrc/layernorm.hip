// layernorm.hip - layer norm rows (R20): forward, which can keep its input in 8 bits (R21) in the same pass, and the
// gradients of input, gain and bias, whose input may be read back from those 8 bits.
//
// A row of up to 2048 terms is held by one wavefront, a longer one by a workgroup of up to 16 (wide_row_sum), so it is
// read from memory once however long it is.  Bound: HBM.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

namespace {

template <int SRC, int NW, bool TAIL, bool KEEP>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, NW == 1 ? 4 : 1) void layernorm_fwd_kernel(
    int64_t rows, int cols, ActIn x, const uint16_t* __restrict__ gain, const uint16_t* __restrict__ bias, float eps,
    float inv_d, int y_bf16, void* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, ActKeep k) {
  constexpr int kRows = NW == 1 ? 4 : 1;  // rows of a workgroup
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;  // this wavefront's part of the row
  const int n = cols - seg < (int)kRegCols ? cols - seg : (int)kRegCols;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? w : 0); row < rows; row += (int64_t)gridDim.x * kRows) {
    const PartIn<SRC> in(x, row, cols, seg);
    float xv[kRegQ][4];
    part_load<TAIL>(n, xv, [&](int j, float(&v)[4]) { in.load4(j, v); }, [&](int j) { return in.load1(j); });
    const float sum = wide_row_sum<NW>(st[w], xv, cols, slot[0]);
    const float mu = sum * inv_d;
    float sq[kRegQ][4];  // what lies behind the row's end is not read by the chains
#pragma unroll
    for (int q = 0; q < kRegQ; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float d = xv[q][t] - mu;
        sq[q][t] = d * d;
      }
    const float ss = wide_row_sum<NW>(st[w], sq, cols, slot[1]);
    const float var = ss * inv_d;
    const float v = var + eps;
    const float r = 1.0f / __builtin_sqrtf(v);
    if (lane == 0 && seg == 0) {
      mean[row] = mu;
      rstd[row] = r;
    }
    if (KEEP)
      part_keep<TAIL>(xv, n, k.lg, k.codes + row * cols + seg,
                      k.steps + row * ((cols + (1 << k.lg) - 1) >> k.lg) + (seg >> k.lg));
    uint16_t* yh = (uint16_t*)y + row * cols + seg;
    float* yf = (float*)y + row * cols + seg;
    part_store<TAIL>(n,
                     [&](int q, float(&o)[4]) {
#pragma unroll
                       for (int t = 0; t < 4; ++t) {
                         const float d = xv[q][t] - mu;
                         o[t] = d * r;
                       }
                     },
                     [&](int j, float(&o)[4]) {
                       float gv[4];
                       ldb_wide(gain + seg + j, gv);
#pragma unroll
                       for (int t = 0; t < 4; ++t) o[t] = o[t] * gv[t];
                       if (bias) {
                         ldb_wide(bias + seg + j, gv);
#pragma unroll
                         for (int t = 0; t < 4; ++t) o[t] = o[t] + gv[t];
                       }
                       if (y_bf16) stb_arith(yh + j, o);
                       else stf<4>(yf + j, o);
                     },
                     [&](int j, float xh) {
                       float o = xh * bf16_wide(gain[seg + j]);
                       if (bias) o = o + bf16_wide(bias[seg + j]);
                       if (y_bf16) yh[j] = bf16_arith(o);
                       else yf[j] = o;
                     });
  }
}

// dx = RN(r RN(RN(gy - m1) - RN(xh m2))): gy = RN(dy g), m1 and m2 the row's means of gy and of RN(gy xh)
template <int SRC, int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, NW == 1 ? 4 : 1) void layernorm_dx_kernel(
    int64_t rows, int cols, ActIn x, const uint16_t* __restrict__ gain, const float* __restrict__ mean,
    const float* __restrict__ rstd, const float* __restrict__ dy, float inv_d, float* __restrict__ dx) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  const int w = wave_id();
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;
  const int n = cols - seg < (int)kRegCols ? cols - seg : (int)kRegCols;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? w : 0); row < rows; row += (int64_t)gridDim.x * kRows) {
    const float mu = mean[row], r = rstd[row];
    const PartIn<SRC> in(x, row, cols, seg);
    const float* dr = dy + row * cols + seg;
    float xh[kRegQ][4], gy[kRegQ][4], tm[kRegQ][4];
    part_load<TAIL>(n, xh, [&](int j, float(&v)[4]) { in.load4(j, v); }, [&](int j) { return in.load1(j); });
    part_load<TAIL>(n, gy, [&](int j, float(&v)[4]) { ldf<4>(dr + j, v); }, [&](int j) { return dr[j]; });
    part_load<TAIL>(n, tm, [&](int j, float(&v)[4]) { ldb_wide(gain + seg + j, v); },
                    [&](int j) { return bf16_wide(gain[seg + j]); });
#pragma unroll
    for (int q = 0; q < kRegQ; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float d = xh[q][t] - mu;
        xh[q][t] = d * r;
        gy[q][t] = gy[q][t] * tm[q][t];
        tm[q][t] = gy[q][t] * xh[q][t];
      }
    const float s1 = wide_row_sum<NW>(st[w], gy, cols, slot[0]);
    const float s2 = wide_row_sum<NW>(st[w], tm, cols, slot[1]);
    const float m1 = s1 * inv_d, m2 = s2 * inv_d;
    float* out = dx + row * cols + seg;
    part_store<TAIL>(n,
                     [&](int q, float(&o)[4]) {
#pragma unroll
                       for (int t = 0; t < 4; ++t) {
                         const float a = gy[q][t] - m1;
                         const float b = xh[q][t] * m2;
                         const float c = a - b;
                         o[t] = r * c;
                       }
                     },
                     [&](int j, const float(&o)[4]) { stf<4>(out + j, o); }, [&](int j, float o) { out[j] = o; });
  }
}

// The chains of 32 rows of dgain[k] = R1 over rows of RN(dy xh) and dbias[k] = R1 over rows of dy: V columns per thread,
// B rows in flight.  part: [2][chunks][cols].
template <int SRC, int V, int B>
__global__ __launch_bounds__(256 / V) void layernorm_part_kernel(int64_t rows, int64_t cols, ActIn x,
                                                                 const float* __restrict__ mean,
                                                                 const float* __restrict__ rstd,
                                                                 const float* __restrict__ dy,
                                                                 float* __restrict__ part) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x * V;
  if (col >= cols) return;
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  for (int64_t c = blockIdx.y; c < nc; c += gridDim.y) {
    const int64_t t0 = c * kChunk, t1 = t0 + kChunk < rows ? t0 + kChunk : rows;
    float sg[V] = {}, sb[V] = {};
    auto steps = [&](int64_t t, auto n) __attribute__((always_inline)) {
      constexpr int N = decltype(n)::value;
      float xv[N][V], dv[N][V];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (V == 4) {
          act4<SRC, false>(x, t + i, col, cols, xv[i]);
        } else {
          const int64_t at = (t + i) * cols + col;
          if constexpr (SRC == ACT_F32) xv[i][0] = ((const float*)x.x)[at];
          else if constexpr (SRC == ACT_BF16) xv[i][0] = bf16_to_f32(((const uint16_t*)x.x)[at]);
          else xv[i][0] = (float)((const int8_t*)x.x)[at] *
                          x.steps[(t + i) * ((cols + (1 << x.lg) - 1) >> x.lg) + (col >> x.lg)];
        }
        ldf<V>(dy + (t + i) * cols + col, dv[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float mu = mean[t + i], r = rstd[t + i];
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float d = xv[i][k] - mu;
          const float xh = d * r;
          const float pr = dv[i][k] * xh;
          sg[k] = sg[k] + pr;
          sb[k] = sb[k] + dv[i][k];
        }
      }
    };
    int64_t t = t0;
    for (; t + B <= t1; t += B) steps(t, std::integral_constant<int, B>{});
    for (; t < t1; ++t) steps(t, std::integral_constant<int, 1>{});
    stf<V>(part + c * cols + col, sg);
    stf<V>(part + (nc + c) * cols + col, sb);
  }
}

// Algorithm 2 over the chunk partials of a column: 16 wavefronts take 64 columns, wavefront g folds the aligned
// power-of-two block of chunks [g G, g G + G), and the block results are folded with the pass-through rule.
constexpr int kFoldBlocks = 16;
__global__ __launch_bounds__(64 * kFoldBlocks) void column_fold_kernel(int64_t nc, int64_t cols, int64_t inner,
                                                                       const float* __restrict__ part,
                                                                       float* __restrict__ out0, float* __restrict__ out1) {
  __shared__ float res[kFoldBlocks][64];
  float* out = blockIdx.y ? out1 : out0;
  if (!out) return;
  part += blockIdx.y * nc * cols;
  const int lane = threadIdx.x & 63, g = threadIdx.x >> 6;
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  const int64_t G = block_chunks(nc, kFoldBlocks);
  const int64_t c0 = g * G, c1 = c0 + G < nc ? c0 + G : nc;
  LocalFoldN<22> f;
  if (col < cols) {
    int64_t c = c0;
    for (; c + 8 <= c1; c += 8) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = part[(c + i) * cols + col];
#pragma unroll
      for (int i = 0; i < 8; ++i) f.push(p[i]);
    }
    for (; c < c1; ++c) f.push(part[c * cols + col]);
  }
  res[g][lane] = f.result();
  __syncthreads();
  if (g == 0 && col < cols) {
    float v[kFoldBlocks];
#pragma unroll
    for (int q = 0; q < kFoldBlocks; ++q) v[q] = res[q][lane];
#pragma unroll
    for (int d = 1; d < kFoldBlocks; d <<= 1)
#pragma unroll
      for (int q = 0; q + d < kFoldBlocks; q += 2 * d)
        if ((q + d) * G < nc) v[q] = v[q] + v[q + d];
    out[inner > 0 ? (col % inner) * (cols / inner) + col / inner : col] = v[0];
  }
}

constexpr int64_t kMaxBlocks = 1 << 20;

// wavefronts that hold a row of cols terms
int row_waves(int64_t cols) {
  int nw = 1;
  while (nw * kRegCols < cols) nw <<= 1;
  return nw;
}

}  // namespace

hipError_t column_fold_launch(int64_t rows, int64_t cols, int64_t inner, const float* part, float* out, float* out1,
                              hipStream_t s) {
  if (cols == 0) return hipSuccess;
  hipLaunchKernelGGL(column_fold_kernel, dim3((unsigned)((cols + 63) / 64), out1 ? 2 : 1), dim3(64 * kFoldBlocks), 0, s,
                     (rows + kChunk - 1) / kChunk, cols, inner, part, out, out1);
  return hipGetLastError();
}

#define CANON_LN_WAVES(K, SRC)                \
  switch (row_waves(cols)) {                  \
    case 1: K(SRC, 1); break;                 \
    case 2: K(SRC, 2); break;                 \
    case 4: K(SRC, 4); break;                 \
    case 8: K(SRC, 8); break;                 \
    default: K(SRC, 16); break;               \
  }

hipError_t layernorm_fwd_launch(int64_t rows, int64_t cols, const ActIn& x, const uint16_t* gain, const uint16_t* bias,
                                float eps, int y_bf16, void* y, float* mean, float* rstd, const ActKeep& k,
                                hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const float inv_d = (float)(1.0 / (double)cols);  // RN32(1/cols), correctly rounded
  const int nw = row_waves(cols);
  const int64_t blocks = nw == 1 ? (rows + 3) / 4 : rows;
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks)), wg(nw == 1 ? 256 : 64 * nw);
#define CANON_LN_K(SRC, NW, TAIL, KEEP)                                                                                \
  hipLaunchKernelGGL((layernorm_fwd_kernel<SRC, NW, TAIL, KEEP>), grid, wg, 0, s, rows, (int)cols, x, gain, bias, eps, \
                     inv_d, y_bf16, y, mean, rstd, k)
#define CANON_LN(SRC, NW)                          \
  do {                                             \
    if (cols % 4 == 0) {                           \
      if (k.codes) CANON_LN_K(SRC, NW, false, true); \
      else CANON_LN_K(SRC, NW, false, false);      \
    } else {                                       \
      if (k.codes) CANON_LN_K(SRC, NW, true, true);  \
      else CANON_LN_K(SRC, NW, true, false);       \
    }                                              \
  } while (0)
  if (x.src == ACT_F32) {
    CANON_LN_WAVES(CANON_LN, ACT_F32)
  } else {
    CANON_LN_WAVES(CANON_LN, ACT_BF16)
  }
#undef CANON_LN
#undef CANON_LN_K
  return hipGetLastError();
}

int64_t layernorm_part_floats(int64_t rows, int64_t cols) { return 2 * ((rows + kChunk - 1) / kChunk) * cols; }

hipError_t layernorm_bwd_launch(int64_t rows, int64_t cols, const ActIn& x, const uint16_t* gain, const float* mean,
                                const float* rstd, const float* dy, float* dx, float* dgain, float* dbias, float* part,
                                hipStream_t s) {
  const float inv_d = (float)(1.0 / (double)cols);
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  if ((dgain || dbias) && rows > 0) {
    const dim3 grid((unsigned)((cols + 255) / 256), (unsigned)(nc < 65535 ? nc : 65535));
#define CANON_LN_PART(SRC)                                                                                            \
  do {                                                                                                                \
    if (cols % 4 == 0)                                                                                                \
      hipLaunchKernelGGL((layernorm_part_kernel<SRC, 4, 4>), grid, dim3(64), 0, s, rows, cols, x, mean, rstd, dy,     \
                         part);                                                                                       \
    else                                                                                                              \
      hipLaunchKernelGGL((layernorm_part_kernel<SRC, 1, 8>), grid, dim3(256), 0, s, rows, cols, x, mean, rstd, dy,    \
                         part);                                                                                       \
  } while (0)
    if (x.src == ACT_F32) CANON_LN_PART(ACT_F32);
    else if (x.src == ACT_BF16) CANON_LN_PART(ACT_BF16);
    else CANON_LN_PART(ACT_Q8);
#undef CANON_LN_PART
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (dgain || dbias) {
    hipError_t e = column_fold_launch(rows, cols, 0, part, dgain, dbias, s);
    if (e != hipSuccess) return e;
  }
  if (rows == 0) return hipSuccess;
  const int nw = row_waves(cols);
  const int64_t blocks = nw == 1 ? (rows + 3) / 4 : rows;
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks)), wg(nw == 1 ? 256 : 64 * nw);
#define CANON_LN(SRC, NW)                                                                                              \
  do {                                                                                                                 \
    if (cols % 4 == 0)                                                                                                 \
      hipLaunchKernelGGL((layernorm_dx_kernel<SRC, NW, false>), grid, wg, 0, s, rows, (int)cols, x, gain, mean, rstd,  \
                         dy, inv_d, dx);                                                                                   \
    else                                                                                                               \
      hipLaunchKernelGGL((layernorm_dx_kernel<SRC, NW, true>), grid, wg, 0, s, rows, (int)cols, x, gain, mean, rstd,   \
                         dy, inv_d, dx);                                                                                   \
  } while (0)
  if (x.src == ACT_F32) {
    CANON_LN_WAVES(CANON_LN, ACT_F32)
  } else if (x.src == ACT_BF16) {
    CANON_LN_WAVES(CANON_LN, ACT_BF16)
  } else {
    CANON_LN_WAVES(CANON_LN, ACT_Q8)
  }
#undef CANON_LN
  return hipGetLastError();
}

}  // namespace canon
