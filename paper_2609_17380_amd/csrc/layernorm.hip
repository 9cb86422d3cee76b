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

// Whether a wavefront loads its next row while it sums and writes one: rows of 1025 to 2048 columns that are not kept in 8
// bits (8192 x 2048 24.0 -> 22.1 us, 4096 x 2048 13.8 -> 13.7).  Of shorter rows and of those that several wavefronts share
// enough are on the chip at once (8192 x 1024 13.2 us ahead, 12.6 not; 8192 x 5001 91 and 68), and the codes take the
// registers.
constexpr bool layernorm_ahead(bool keep, int q, int waves) { return !keep && q == 8 && waves == 1; }

// Two sums to a row, the second over the squares of the differences from the first's mean: the row stays in registers.
// 8192 x 2048 fp32 22 us (100.7 MB: 21 at a large copy's rate), bf16 16.4 (14), bf16 kept as well 22 (18); one row of 2048
// 3.1.  Rows of 8192 bf16 take 72 us where a copy takes 50: the two sums, some 20 vector instructions to an element.
template <int SRC, int Q, int NW, bool TAIL, bool KEEP>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, Q == 8 ? 4 : 1) void layernorm_fwd_kernel(
    int64_t rows, int cols, ActIn x, const uint16_t* __restrict__ gain, const uint16_t* __restrict__ bias, float eps,
    float inv_d, int y_bf16, void* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, ActKeep k) {
  constexpr int kRows = NW == 1 ? 4 : 1;  // rows of a workgroup
  __shared__ __attribute__((aligned(16))) RowStage<Q> st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int seg = NW == 1 ? 0 : w * 256 * Q;  // this wavefront's part of the row
  const int n = cols - seg < 256 * Q ? cols - seg : 256 * Q;
  using In = PartIn<SRC>;
  // beside the codes of 8 vectors the places of the last four spill (8192 x 5001 kept 101 us, with them 123)
  constexpr bool kEnds = TAIL && SRC == ACT_BF16 && !(KEEP && Q == 8);
  auto load = [&](int64_t row, typename In::Raw(&v)[Q]) __attribute__((always_inline)) {
    const In in(x, row, cols, seg);
    if constexpr (kEnds) in.part_ends(row < rows ? n : 0, cols, v);
    else in.template part<TAIL>(row < rows ? n : 0, v);
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  // the next row is on its way while one is summed and written, where the registers allow it
  constexpr bool kAhead = layernorm_ahead(KEEP, Q, NW);
  typename In::Raw next[Q];
  // Gain and bias, all vectors at once: with a load and its wait per vector 1023 x 5116 took 10.5 us instead of 9.4, 4096 x
  // 16384 92 instead of 78, kept rows of 2048 27.8 instead of 26.6; beside a next row the registers spill (22.7, so 23.5).
  constexpr bool kEach = kAhead && !TAIL;
  uint32_t gw[Q][2], bw[Q][2];
  auto load_gain = [&]() __attribute__((always_inline)) {
    part_load_bf16<TAIL>(0, again(n), gw, gain + seg);
    part_load_bf16<TAIL>(0, again(bias ? n : 0), bw, bias + seg);
  };
  int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? w : 0);
  if (kAhead) load(row, next);
  for (; row < rows; row += step) {
    float xv[Q][4];
    if (!kAhead) load(row, next);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if constexpr (kEnds) In::ends(next[q], again(n) - (256 * q + 4 * (int)(threadIdx.x & 63)));
      In::wide(next[q], xv[q]);
    }
    if (kAhead) load(row + step, next);
    const float sum = wide_row_sum<NW>(st[w], xv, cols, slot[0]);
    const float mu = sum * inv_d;
    float sq[Q][4];  // what lies behind the row's end is not read by the chains
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float d = xv[q][t] - mu;
        sq[q][t] = d * d;
      }
    if (!KEEP && !kAhead) load_gain();  // on its way while the squares are summed, where the registers allow it
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
    if (KEEP || (kAhead && !kEach)) load_gain();
    uint16_t* yh = (uint16_t*)y + row * cols + seg;
    float* yf = (float*)y + row * cols + seg;
    part_store<TAIL, Q>(n,
                     [&](int q, float(&o)[4]) {
                       float gv[4], bv[4];
                       if constexpr (kEach) {
                         if (256 * q + 4 * lane < n) {
                           ldb_wide(gain + seg + 256 * q + 4 * lane, gv);
                           if (bias) ldb_wide(bias + seg + 256 * q + 4 * lane, bv);
                         }
                       } else {
                         wide4(gw[q], gv);
                         wide4(bw[q], bv);
                       }
#pragma unroll
                       for (int t = 0; t < 4; ++t) {
                         const float d = xv[q][t] - mu;
                         const float xh = d * r;
                         o[t] = xh * gv[t];
                         if (bias) o[t] = o[t] + bv[t];
                       }
                     },
                     [&](int j, const float(&o)[4]) {
                       if (y_bf16) stb_arith(yh + j, o);
                       else stf<4>(yf + j, o);
                     },
                     [&](int j, float o) {
                       if (y_bf16) yh[j] = bf16_arith(o);
                       else yf[j] = o;
                     });
  }
}

// dx = RN(r RN(RN(gy - m1) - RN(xh m2))): gy = RN(dy g), m1 and m2 the row's means of gy and of RN(gy xh).  1023 x 5001 from
// 8 bits 11 us: all its rows are on the chip at once, so that a row's latency (loads, two sums, stores) is the kernel's.
template <int SRC, int Q, int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, Q == 8 ? 4 : 1) void layernorm_dx_kernel(
    int64_t rows, int cols, ActIn x, const uint16_t* __restrict__ gain, const float* __restrict__ mean,
    const float* __restrict__ rstd, const float* __restrict__ dy, float inv_d, float* __restrict__ dx) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RowStage<Q> st[NW == 1 ? 4 : NW];
  using In = PartIn<SRC>;
  __shared__ float slot[2][NW];
  const int w = wave_id();
  const int seg = NW == 1 ? 0 : w * 256 * Q;
  const int n = cols - seg < 256 * Q ? cols - seg : 256 * Q;
  for (int64_t row = (int64_t)blockIdx.x * kRows + (NW == 1 ? w : 0); row < rows; row += (int64_t)gridDim.x * kRows) {
    const float mu = mean[row], r = rstd[row];
    const float* dr = dy + row * cols + seg;
    typename In::Raw xr[Q];
    uint32_t gw[Q][2];
    float xh[Q][4], gy[Q][4], tm[Q][4];
    In(x, row, cols, seg).template part<TAIL>(n, xr);
    part_load<TAIL>(0, n, gy, dr);
    part_load_bf16<TAIL>(0, again(n), gw, gain + seg);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      In::wide(xr[q], xh[q]);
      wide4(gw[q], tm[q]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float d = xh[q][t] - mu;
        xh[q][t] = d * r;
        gy[q][t] = gy[q][t] * tm[q][t];
        tm[q][t] = gy[q][t] * xh[q][t];
      }
    }
    const float s1 = wide_row_sum<NW>(st[w], gy, cols, slot[0]);
    const float s2 = wide_row_sum<NW>(st[w], tm, cols, slot[1]);
    const float m1 = s1 * inv_d, m2 = s2 * inv_d;
    float* out = dx + row * cols + seg;
    part_store<TAIL, Q>(n,
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

// Four columns of a row of 4 or more from column j on, n of them there (none: n <= 0), x as it is stored; +0 where there are
// none.  The vector that the row's end cuts is loaded element by element, or (ENDS, bf16 and 8 bits) as the row's last four,
// which `ends` puts in place when they are needed.
template <int SRC, bool TAIL, bool ENDS>
__device__ __forceinline__ void load_columns(const ActIn& x, const float* dy, int64_t rows, int64_t row, int cols, int j,
                                             int n, typename PartIn<SRC>::Raw& xr, float (&dv)[4]) {
  xr = typename PartIn<SRC>::Raw{};
#pragma unroll
  for (int t = 0; t < 4; ++t) dv[t] = 0.0f;
  if (row >= rows) return;
  const PartIn<SRC> in(x, row, cols, 0);
  const float* dr = dy + row * cols;
  if (ENDS && n > 0) in.load4(TAIL && n < 4 ? cols - 4 : j, j, xr);
  if (n == 4) {
    if (!ENDS) in.load4(j, xr);
    ldf<4>(dr + j, dv);
  } else if (TAIL) {
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (t < n) {
        if (!ENDS) in.load1(j, t, xr);
        dv[t] = dr[j + t];
      }
  }
}

// The chains of 32 rows of dgain[k] = R1 over rows of RN(dy xh) and dbias[k] = R1 over rows of dy, a column to a thread, B
// rows in flight.  part: [2][chunks][cols].  1023 x 5001 from 8 bits 10 us: a chain's 32 rows are four batches of loads, each
// waited for.  (Four columns to a thread are fewer, wider loads and were never faster: 8192 x 2048 with dx 69 us, so 64.5;
// 1023 x 5001 bf16 32 and 23.)
template <int SRC, int B>
__global__ __launch_bounds__(256) void layernorm_part_kernel(int64_t rows, int cols, ActIn x, const float* __restrict__ mean,
                                                             const float* __restrict__ rstd, const float* __restrict__ dy,
                                                             float* __restrict__ part) {
  const int j = blockIdx.x * 256 + threadIdx.x;
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  if (j >= cols) return;
  for (int64_t c = blockIdx.y; c < nc; c += gridDim.y) {
    float sg = 0.0f, sb = 0.0f;
    auto steps = [&](int64_t t, auto count) __attribute__((always_inline)) {  // all loads, then the chains' steps
      constexpr int N = decltype(count)::value;
      typename PartIn<SRC>::Raw xr[N];
      float dv[N];
#pragma unroll
      for (int r = 0; r < N; ++r) {
        xr[r] = typename PartIn<SRC>::Raw{};
        PartIn<SRC>(x, t + r, cols, 0).load1(j, 0, xr[r]);
        dv[r] = dy[(t + r) * cols + j];
      }
#pragma unroll
      for (int r = 0; r < N; ++r) {
        float xv[4];
        PartIn<SRC>::wide(xr[r], xv);
        const float d = xv[0] - mean[t + r];
        const float xh = d * rstd[t + r];
        const float pr = dv[r] * xh;
        sg = sg + pr;
        sb = sb + dv[r];
      }
    };
    const int64_t t1 = (c + 1) * kChunk < rows ? (c + 1) * kChunk : rows;
    int64_t t = c * kChunk;
    for (; t + B <= t1; t += B) steps(t, std::integral_constant<int, B>{});
    for (; t < t1; ++t) steps(t, std::integral_constant<int, 1>{});
    part[c * cols + j] = sg;
    part[(nc + c) * cols + j] = sb;
  }
}

// The whole backward in one pass over x and dy: a workgroup takes a chain of 32 rows, wavefront w the 256 VQ columns from
// 256 VQ w on, R = 4 / VQ rows at a time.  A lane's columns run through the 32 rows in order, so it holds their chains of
// dgain and dbias; a row's own sums, two to a row, are cut into 8 VQ chunks to a wavefront, 64 chains in all, a lane to a
// chain over an LDS transpose, folded over the wavefront's chunks and then over the wavefronts.  The next rows are loaded
// before the barrier that the sums wait at.  8192 x 2048 fp32 36 us behind the forward, which leaves part of x and dy in the
// last-level cache (201 MB: 42 from memory); from 8 bits 29.
template <int SRC, int VQ, int NW, bool TAIL>
__global__ __launch_bounds__(64 * NW) void layernorm_pass_kernel(int64_t rows, int cols, ActIn x,
                                                                 const uint16_t* __restrict__ gain,
                                                                 const float* __restrict__ mean,
                                                                 const float* __restrict__ rstd,
                                                                 const float* __restrict__ dy, float inv_d,
                                                                 float* __restrict__ dx, float* __restrict__ part) {
  constexpr int R = 4 / VQ, kSums = 2 * R, kLanes = 8 * VQ;  // lanes to a sum's chunks
  // bf16 and 8-bit elements one by one are waited for (4096 x 2047 bf16 38 us, so 27), but two vectors to a lane leave no
  // registers (4096 x 7001 from 8 bits 109 us, one by one 76), and fp32 ones need no wait
  constexpr bool kEnds = SRC != ACT_F32 && VQ == 1;
  using In = PartIn<SRC>;
  __shared__ __attribute__((aligned(16))) RegStage st[NW];
  __shared__ float slot[2][kSums][NW];
  const int w = wave_id(), lane = threadIdx.x & 63;
  int j[VQ], n[VQ];  // this lane's first columns, and how many of each four there are
#pragma unroll
  for (int v = 0; v < VQ; ++v) {
    j[v] = 256 * (VQ * w + v) + 4 * lane;
    n[v] = cols - j[v] < 4 ? cols - j[v] : 4;
  }
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  auto load = [&](int64_t row, typename In::Raw(&xr)[VQ], float(&dv)[VQ][4]) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < VQ; ++v) load_columns<SRC, TAIL, kEnds>(x, dy, rows, row, cols, j[v], n[v], xr[v], dv[v]);
  };
  auto add = [](uint32_t a, uint32_t b) {
    const float s = __uint_as_float(a) + __uint_as_float(b);
    return __float_as_uint(s);
  };
  float gv[VQ][4];  // kNoTerm where there is no column: times the dy of +0 there, kNoTerm again
#pragma unroll
  for (int v = 0; v < VQ; ++v)
#pragma unroll
    for (int t = 0; t < 4; ++t) gv[v][t] = t < n[v] ? bf16_wide(gain[j[v] + t]) : kNoTerm;
  for (int64_t c = blockIdx.x; c < nc; c += gridDim.x) {
    const int64_t t0 = c * kChunk;
    typename In::Raw xr[R][VQ];
    float dv[R][VQ][4], sg[VQ][4], sb[VQ][4];
#pragma unroll
    for (int v = 0; v < VQ; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i) sg[v][i] = sb[v][i] = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r) load(t0 + r, xr[r], dv[r]);
    for (int k = 0; k < kChunk / R; ++k) {
      const int64_t t = t0 + R * k;
      if (t >= rows) break;
      float xh[R][VQ][4], gy[R][VQ][4], rs[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int64_t row = t + r < rows ? t + r : rows - 1;
        const float mu = mean[row];
        rs[r] = rstd[row];
#pragma unroll
        for (int v = 0; v < VQ; ++v) {
          float tm[4], xv[4];
          if constexpr (kEnds && TAIL) In::ends(xr[r][v], n[v]);
          In::wide(xr[r][v], xv);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float d = xv[i] - mu;
            xh[r][v][i] = d * rs[r];
            gy[r][v][i] = dv[r][v][i] * gv[v][i];
            tm[i] = gy[r][v][i] * xh[r][v][i];
            if (i >= n[v]) tm[i] = gy[r][v][i];  // no column: both kNoTerm
            const float pr = dv[r][v][i] * xh[r][v][i];
            if (t + r < rows) {
              sg[v][i] = sg[v][i] + pr;
              sb[v][i] = sb[v][i] + dv[r][v][i];
            }
          }
          st[w].put((2 * r) * VQ + v, lane, gy[r][v]);
          st[w].put((2 * r + 1) * VQ + v, lane, tm);
        }
      }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int r = 0; r < R; ++r) load(t + R + r < t0 + kChunk ? t + R + r : rows, xr[r], dv[r]);
      // the chain of chunk lane % kLanes of sum lane / kLanes; of a chunk that the row does not have +0, and -c0 is kNoTerm
      const float c0 = st[w].chain(lane);
      const float c = kChunk * (kLanes * w + (lane & (kLanes - 1))) < cols ? c0 : -c0;
      const float p = __uint_as_float(lanes_join(__float_as_uint(c), kLanes, add));
      if ((lane & (kLanes - 1)) == 0) slot[k & 1][lane / kLanes][w] = p;
      __syncthreads();
      float m[kSums];
      constexpr int kWide = NW <= 8 ? 8 : 16, kOnce = 64 / kWide;  // lanes to a sum's wavefronts, and sums at a time
#pragma unroll
      for (int i0 = 0; i0 < kSums; i0 += kOnce) {
        const int sum = i0 + lane / kWide, of = lane & (kWide - 1);
        float s = sum < kSums && of < NW ? slot[k & 1][sum < kSums ? sum : 0][of < NW ? of : 0] : kNoTerm;
        s = __uint_as_float(lanes_join(__float_as_uint(s), kWide, add)) * inv_d;
#pragma unroll
        for (int i = 0; i < kOnce; ++i)
          if (i0 + i < kSums) m[i0 + i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(s), kWide * i));
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (t + r >= rows) break;
#pragma unroll
        for (int v = 0; v < VQ; ++v) {
          float o[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = gy[r][v][i] - m[2 * r];
            const float b = xh[r][v][i] * m[2 * r + 1];
            const float d = a - b;
            o[i] = rs[r] * d;
          }
          float* out = dx + (t + r) * cols + j[v];
          if (n[v] == 4) {
            stf<4>(out, o);
          } else if (TAIL) {
#pragma unroll
            for (int i = 0; i < 3; ++i)
              if (i < n[v]) out[i] = o[i];
          }
        }
      }
    }
#pragma unroll
    for (int v = 0; v < VQ; ++v)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n[v]) {
          part[c * cols + j[v] + i] = sg[v][i];
          part[(nc + c) * cols + j[v] + i] = sb[v][i];
        }
  }
}

// Algorithm 2 over the chunk partials of a column: 16 wavefronts take 64 columns, wavefront g folds the aligned
// power-of-two block of chunks [g G, g G + G), and the block results are folded with the pass-through rule.  Within a block
// 16 partials at a time are loaded and folded as a tree, those past the last chunk as kNoTerm (of no chunk at all the sum is
// +0); only blocks of more need Algorithm 2's stack (whose levels are indexed in scratch memory).  256 partials of 2048
// columns, twice, 4.6 us.
constexpr int kFoldBlocks = 16;
constexpr int kFoldUnit = 16;
__global__ __launch_bounds__(64 * kFoldBlocks) void column_fold_kernel(int64_t nc, int64_t cols, int64_t inner,
                                                                       const float* __restrict__ part,
                                                                       float* __restrict__ out0, float* __restrict__ out1) {
  __shared__ float res[kFoldBlocks][64];
  float* out = blockIdx.y ? out1 : out0;
  if (!out) return;
  part += blockIdx.y * nc * cols;
  const int lane = threadIdx.x & 63, g = wave_id();
  const int64_t col = (int64_t)blockIdx.x * 64 + lane;
  const int64_t G = block_chunks(nc, kFoldBlocks);
  const int64_t c0 = g * G, c1 = c0 + G < nc ? c0 + G : nc;
  auto unit = [&](int64_t c) __attribute__((always_inline)) {
    float p[kFoldUnit];
#pragma unroll
    for (int i = 0; i < kFoldUnit; ++i) p[i] = c + i < c1 ? part[(c + i) * cols + col] : kNoTerm;
#pragma unroll
    for (int d = 1; d < kFoldUnit; d <<= 1)
#pragma unroll
      for (int i = 0; i + d < kFoldUnit; i += 2 * d) p[i] = p[i] + p[i + d];
    return p[0];
  };
  float r = nc > 0 ? kNoTerm : 0.0f;
  if (col < cols && c0 < c1) {
    if (G <= kFoldUnit) {
      r = unit(c0);
    } else {
      LocalFoldN<20> f;
      for (int64_t c = c0; c < c1; c += kFoldUnit) f.push(unit(c));
      r = f.result();
    }
  }
  res[g][lane] = r;
  __syncthreads();
  if (g == 0 && col < cols) {
    float v[kFoldBlocks];
#pragma unroll
    for (int q = 0; q < kFoldBlocks; ++q) v[q] = res[q][lane];
#pragma unroll
    for (int d = 1; d < kFoldBlocks; d <<= 1)
#pragma unroll
      for (int q = 0; q + d < kFoldBlocks; q += 2 * d) v[q] = v[q] + v[q + d];
    out[inner > 0 ? (col % inner) * (cols / inner) + col / inner : col] = v[0];
  }
}

constexpr int64_t kMaxBlocks = 1 << 20;
constexpr int64_t kPassCols = 8192;  // 16 wavefronts of 512 columns

}  // namespace

hipError_t column_fold_launch(int64_t rows, int64_t cols, int64_t inner, const float* part, float* out, float* out1,
                              hipStream_t s) {
  if (cols == 0) return hipSuccess;
  hipLaunchKernelGGL(column_fold_kernel, dim3((unsigned)((cols + 63) / 64), out1 ? 2 : 1), dim3(64 * kFoldBlocks), 0, s,
                     (rows + kChunk - 1) / kChunk, cols, inner, part, out, out1);
  return hipGetLastError();
}

#define CANON_LN_ACT_F32(Q, NW) CANON_LN(ACT_F32, Q, NW)
#define CANON_LN_ACT_BF16(Q, NW) CANON_LN(ACT_BF16, Q, NW)
#define CANON_LN_ACT_Q8(Q, NW) CANON_LN(ACT_Q8, Q, NW)

hipError_t layernorm_fwd_launch(int64_t rows, int64_t cols, const ActIn& x, const uint16_t* gain, const uint16_t* bias,
                                float eps, int y_bf16, void* y, float* mean, float* rstd, const ActKeep& k,
                                hipStream_t s) {
  if (rows == 0) return hipSuccess;
  const float inv_d = (float)(1.0 / (double)cols);  // RN32(1/cols), correctly rounded
  const RowShape shape = row_shape(rows, cols, 8);
  const int64_t blocks = shape.groups(rows);
  // rows that are loaded ahead: no more workgroups than are on the chip at once
  const int64_t most = layernorm_ahead(k.codes, shape.q, shape.waves) ? device_cus() * 4 : kMaxBlocks;
  const dim3 grid((unsigned)(blocks < most ? blocks : most)), wg(shape.threads());
#define CANON_LN_K(SRC, Q, NW, TAIL, KEEP)                                                                               \
  hipLaunchKernelGGL((layernorm_fwd_kernel<SRC, Q, NW, TAIL, KEEP>), grid, wg, 0, s, rows, (int)cols, x, gain, bias, eps, \
                     inv_d, y_bf16, y, mean, rstd, k)
#define CANON_LN(SRC, Q, NW)                         \
  do {                                             \
    if (cols % 4 == 0) {                           \
      if (k.codes) CANON_LN_K(SRC, Q, NW, false, true); \
      else CANON_LN_K(SRC, Q, NW, false, false);      \
    } else {                                       \
      if (k.codes) CANON_LN_K(SRC, Q, NW, true, true);  \
      else CANON_LN_K(SRC, Q, NW, true, false);       \
    }                                              \
  } while (0)
  if (x.src == ACT_F32) {
    CANON_ROW_SHAPES(CANON_LN_ACT_F32, shape);
  } else {
    CANON_ROW_SHAPES(CANON_LN_ACT_BF16, shape);
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
  // One pass over x and dy where its workgroups, one to 32 rows, are half as many as the CUs or more, and its wavefronts four
  // to a CU (4096 x 8192 in 103 us, in two passes 128; 8192 x 2048 47 and 65; 4096 x 2048 30.5 and 32; 8192 x 1024 27 and 32; of
  // 2048 x 8192 86 and 63.5, 4096 x 1001 29 and 21, 8192 x 512 20 and 19.5).  fp32 rows of up to 1024 columns that four does not
  // divide lose by it, 8192 x 1001 39 and 34, 16384 x 511 44 and 41, which bf16 and 8 bits do not: 25 and 30, 29 and 36.
  const bool once = (dgain || dbias) && cols >= 4 && cols <= kPassCols && 2 * nc >= device_cus() &&
                    nc * ((cols + 255) / 256 < 16 ? (cols + 255) / 256 : 16) >= 4 * device_cus();
  if (once) {
    const dim3 grid((unsigned)(nc < kMaxBlocks ? nc : kMaxBlocks));
#define CANON_LN_PASS(SRC, VQ, NW)                                                                                         \
  do {                                                                                                                  \
    if (cols % 4 == 0)                                                                                                  \
      hipLaunchKernelGGL((layernorm_pass_kernel<SRC, VQ, NW, false>), grid, dim3(64 * NW), 0, s, rows, (int)cols, x, gain,  \
                         mean, rstd, dy, inv_d, dx, part);                                                              \
    else                                                                                                                \
      hipLaunchKernelGGL((layernorm_pass_kernel<SRC, VQ, NW, true>), grid, dim3(64 * NW), 0, s, rows, (int)cols, x, gain,   \
                         mean, rstd, dy, inv_d, dx, part);                                                              \
  } while (0)
#define CANON_LN_PASS_WAVES(SRC)                      \
  do {                                                \
    if (cols <= 512) CANON_LN_PASS(SRC, 1, 2);        \
    else if (cols <= 1024) CANON_LN_PASS(SRC, 1, 4);  \
    else if (cols <= 2048) CANON_LN_PASS(SRC, 1, 8);  \
    else if (cols <= 4096) CANON_LN_PASS(SRC, 1, 16); \
    else CANON_LN_PASS(SRC, 2, 16);                   \
  } while (0)
    if (x.src == ACT_F32) CANON_LN_PASS_WAVES(ACT_F32);
    else if (x.src == ACT_BF16) CANON_LN_PASS_WAVES(ACT_BF16);
    else CANON_LN_PASS_WAVES(ACT_Q8);
#undef CANON_LN_PASS_WAVES
#undef CANON_LN_PASS
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return column_fold_launch(rows, cols, 0, part, dgain, dbias, s);
  }
  if ((dgain || dbias) && rows > 0) {
    const dim3 grid((unsigned)((cols + 255) / 256), (unsigned)(nc < 65535 ? nc : 65535));
#define CANON_LN_PART(SRC) \
  hipLaunchKernelGGL((layernorm_part_kernel<SRC, 8>), grid, dim3(256), 0, s, rows, (int)cols, x, mean, rstd, dy, part)
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
  const RowShape shape = row_shape(rows, cols, 8);
  const int64_t blocks = shape.groups(rows);
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks)), wg(shape.threads());
#define CANON_LN(SRC, Q, NW)                                                                                             \
  do {                                                                                                                 \
    if (cols % 4 == 0)                                                                                                 \
      hipLaunchKernelGGL((layernorm_dx_kernel<SRC, Q, NW, false>), grid, wg, 0, s, rows, (int)cols, x, gain, mean, rstd,  \
                         dy, inv_d, dx);                                                                                   \
    else                                                                                                               \
      hipLaunchKernelGGL((layernorm_dx_kernel<SRC, Q, NW, true>), grid, wg, 0, s, rows, (int)cols, x, gain, mean, rstd,   \
                         dy, inv_d, dx);                                                                                   \
  } while (0)
  if (x.src == ACT_F32) {
    CANON_ROW_SHAPES(CANON_LN_ACT_F32, shape);
  } else if (x.src == ACT_BF16) {
    CANON_ROW_SHAPES(CANON_LN_ACT_BF16, shape);
  } else {
    CANON_ROW_SHAPES(CANON_LN_ACT_Q8, shape);
  }
#undef CANON_LN
  return hipGetLastError();
}

}  // namespace canon
