// relbias.hip - attention rows with a learned relative position bias (R22): raw scores to probabilities, and the gradient
// of the scores and of the bias table.
//
// A row of up to 2048 keys is held by one wavefront, a longer one by a workgroup of up to 16 (wide_row_sum): scores,
// probabilities and their gradient are read from memory once.  The keys that a query sees are one range j0 <= j < j1
// (lengths, causality and the window all cut it from an end), so no mask is read.  A head's biases, by distance up to
// the last bucket's first, are laid out in LDS once for the queries of a workgroup.  Bound: HBM.
#include <hip/hip_runtime.h>

#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

namespace {

constexpr int kQueries = 4;             // queries that a wavefront (or, of longer rows, a workgroup) takes in turn
constexpr int64_t kFarPos = 1 << 20;    // beyond every key's distance and the last bucket
constexpr int64_t kMaxBlocks = 1 << 20;

// bucket of a distance on one side: the last one that begins at or before it
__device__ __forceinline__ int bucket_of(const int32_t* start, int n, int d) {
  int lo = 0, hi = n;  // start[lo] <= d < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= d) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The keys j0 <= j < j1 that query i of sequence b sees, and its position (cut to +-kFarPos, which leaves every bucket as
// it is).
struct Query {
  int j0, j1, pos;
};
__device__ __forceinline__ Query query_of(const RelBiasArgs& a, int64_t b, int64_t i) {
  const int64_t pos = (a.q_starts ? (int64_t)a.q_starts[b] : a.q_start) + i;
  int64_t lo = 0, hi = a.k_len;
  if (a.k_lens) hi = a.k_lens[b] < hi ? a.k_lens[b] : hi;
  if (a.causal) hi = pos + 1 < hi ? pos + 1 : hi;
  if (a.window > 0) {
    lo = pos - a.window + 1 > lo ? pos - a.window + 1 : lo;
    hi = pos + a.window < hi ? pos + a.window : hi;
  }
  if (a.q_lens && i >= a.q_lens[b]) hi = 0;
  if (hi <= lo) lo = hi = 0;
  Query q;
  q.j0 = __builtin_amdgcn_readfirstlane((int)lo);
  q.j1 = __builtin_amdgcn_readfirstlane((int)hi);
  q.pos = __builtin_amdgcn_readfirstlane((int)(pos < -kFarPos ? -kFarPos : pos > kFarPos ? kFarPos : pos));
  return q;
}

template <int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void relbias_fwd_kernel(RelBiasArgs a, int64_t blocks,
                                                                              int64_t per_head,
                                                                              const float* __restrict__ scores,
                                                                              uint16_t* __restrict__ probs) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW], top[NW];
  extern __shared__ float near_[];  // bias by position: of the key less the query's, the near side of the last buckets
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int far = a.start[a.n_side - 1], right = a.bidirectional ? far : 0;
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;
  const int64_t ld = a.ld;
  int turn = 0;  // rows in turn take one of two slots, so that a barrier lies between a slot's reads and its next writes
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int64_t bh = blk / per_head, b = bh / a.heads, h = bh - b * a.heads;
    const int64_t i0 = (blk - bh * per_head) * (kRows * kQueries);
    __syncthreads();  // the last block's biases are read
    for (int e = threadIdx.x; e <= far + right; e += blockDim.x) {
      const int d = far - e;  // query less key: far .. -right
      const int n = d >= 0 ? bucket_of(a.start, a.n_side, d) : a.n_side + bucket_of(a.start, a.n_side, -d);
      near_[e] = bf16_to_f32(a.table[n * a.heads + h]);
    }
    __syncthreads();
    for (int it = 0; it < kQueries; ++it) {
      const int64_t i = i0 + it * kRows + (NW == 1 ? w : 0);
      if (i >= a.q_len) break;  // the same for every wavefront that shares the row
      const Query qy = query_of(a, b, i);
      const int j0 = qy.j0, j1 = qy.j1;
      const int64_t row = bh * a.q_len + i;
      const float* rr = scores + row * ld;
      auto any = [&](int q) { return seg + 256 * q < j1 && seg + 256 * q + 255 >= j0; };
      auto all = [&](int q) { return seg + 256 * q + 255 < j1 && seg + 256 * q >= j0; };
      float e[kRegQ][4];
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
#pragma unroll
        for (int t = 0; t < 4; ++t) e[q][t] = 0.0f;
        const int j = seg + 256 * q + 4 * lane;
        if (any(q) && j < j1 && j + 3 >= j0) ldf4<TAIL>(rr, j, a.k_len, e[q]);
      }
      float m = -__builtin_inff();
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        if (!any(q)) continue;
        const int j = seg + 256 * q + 4 * lane;
        // entry of key j: far + j - pos, cut to the table's ends
        const int at = far + j - qy.pos;
        if (far + seg + 256 * q + 255 - qy.pos <= 0 || far + seg + 256 * q - qy.pos >= far + right) {
          const float bias = near_[far + seg + 256 * q + 255 - qy.pos <= 0 ? 0 : far + right];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float x = e[q][t] * a.scale;
            e[q][t] = x + bias;
          }
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int k = at + t < 0 ? 0 : at + t > far + right ? far + right : at + t;
            const float x = e[q][t] * a.scale;
            e[q][t] = x + near_[k];
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
          if (all(q) || (j + t < j1 && j + t >= j0)) m = fmaxf(m, e[q][t]);
      }
#pragma unroll
      for (int s = 32; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
      if constexpr (NW > 1) {
        if (lane == 0) top[w] = m;
        __syncthreads();
        m = lane < NW ? top[lane] : -__builtin_inff();
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
      }
      // a row whose seen scores are all -inf has e = cexp(-inf) = +0, not cexp(-inf - -inf)
      m = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        if (!any(q)) continue;
        const int j = seg + 256 * q + 4 * lane;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = cexp_neg(e[q][t] - m);
          e[q][t] = all(q) || (j + t < j1 && j + t >= j0) ? x : 0.0f;  // masked keys enter the chain as +0 terms
        }
      }
      turn ^= 1;
      const float S = wide_row_sum<NW>(st[w], e, a.k_len, slot[turn]);
      const float rcp = S == 0.0f ? 0.0f : 1.0f / S;
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        const int j = seg + 256 * q + 4 * lane;
        if (j >= a.k_len) continue;
        uint16_t o[4] = {0, 0, 0, 0};
        if (any(q)) {  // a masked key's +0 rcp is a NaN where S is one: its zero is kept
#pragma unroll
          for (int t = 0; t < 4; ++t)
            if (all(q) || (j + t < j1 && j + t >= j0)) o[t] = f32_to_bf16(e[q][t] * rcp);
        }
        stb4<TAIL>(probs + row * ld, j, a.k_len, o);
      }
    }
  }
}

// ds = RN(P RN(dP - D)), D = R1 over the keys of RN(P dP); dS = bf16(RN(ds scale)).  rowsum [batch][q_len][heads][buckets]:
// for every bucket R1 over the keys of ds, those outside it as +0 terms.  A bucket of up to 32 distances touches at most
// two chunks, whose chains one lane runs and adds (their sum is the fold whatever lies between); a longer one is summed
// chunk by chunk, a lane to a chunk, like the row.
template <int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void relbias_bwd_kernel(RelBiasArgs a, int64_t blocks,
                                                                              int64_t per_head,
                                                                              const uint16_t* __restrict__ probs,
                                                                              const float* __restrict__ dprobs,
                                                                              uint16_t* __restrict__ dscores,
                                                                              float* __restrict__ rowsum) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  __shared__ float part[2][NW];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;
  const int nb = a.n_side * (a.bidirectional ? 2 : 1);
  const int64_t ld = a.ld;
  int turn = 0;  // as above
  // the keys of bucket n, less the query's position: lo <= j - pos < hi
  auto range = [&](int n, int& lo, int& hi) {
    const int m = n < a.n_side ? n : n - a.n_side;
    const int d0 = a.start[m], d1 = m + 1 < a.n_side ? a.start[m + 1] : 2 * (int)kFarPos;
    if (n < a.n_side) {
      lo = 1 - d1;
      hi = d0 == d1 ? lo : d0 == 0 && !a.bidirectional ? 2 * (int)kFarPos : 1 - d0;
    } else {
      lo = d0 > 0 ? d0 : 1;
      hi = d1;
    }
  };
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int64_t bh = blk / per_head, b = bh / a.heads, h = bh - b * a.heads;
    const int64_t i0 = (blk - bh * per_head) * (kRows * kQueries);
    for (int it = 0; it < kQueries; ++it) {
      const int64_t i = i0 + it * kRows + (NW == 1 ? w : 0);
      if (i >= a.q_len) break;
      const Query qy = query_of(a, b, i);
      const int j0 = qy.j0, j1 = qy.j1;
      const int64_t row = bh * a.q_len + i;
      auto any = [&](int q) { return seg + 256 * q < j1 && seg + 256 * q + 255 >= j0; };
      auto all = [&](int q) { return seg + 256 * q + 255 < j1 && seg + 256 * q >= j0; };
      float p[kRegQ][4], dp[kRegQ][4], e[kRegQ][4];
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
#pragma unroll
        for (int t = 0; t < 4; ++t) p[q][t] = dp[q][t] = 0.0f;
        const int j = seg + 256 * q + 4 * lane;
        if (any(q) && j < j1 && j + 3 >= j0) {
          ldb4<TAIL>(probs + row * ld, j, a.k_len, p[q]);
          ldf4<TAIL>(dprobs + row * ld, j, a.k_len, dp[q]);
        }
      }
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        const int j = seg + 256 * q + 4 * lane;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = p[q][t] * dp[q][t];
          e[q][t] = any(q) && (all(q) || (j + t < j1 && j + t >= j0)) ? x : 0.0f;
        }
      }
      turn ^= 1;
      const float D = wide_row_sum<NW>(st[w], e, a.k_len, slot[turn]);
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        const int j = seg + 256 * q + 4 * lane;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float d = dp[q][t] - D;
          const float x = p[q][t] * d;
          e[q][t] = any(q) && (all(q) || (j + t < j1 && j + t >= j0)) ? x : 0.0f;
        }
        if (j < a.k_len) {
          uint16_t o[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) o[t] = f32_to_bf16(e[q][t] * a.scale);
          stb4<TAIL>(dscores + row * ld, j, a.k_len, o);
        }
      }
      if (!rowsum) continue;
      float* out = rowsum + ((b * a.q_len + i) * a.heads + h) * nb;
      // the row's ds, a chunk to a row of LDS (a wavefront's own, its LDS operations in order)
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        const int local = 256 * q + 4 * lane;
        *reinterpret_cast<float4*>(&st[w].t[local >> 5][local & 31]) = make_float4(e[q][0], e[q][1], e[q][2], e[q][3]);
      }
      if constexpr (NW > 1) __syncthreads();
      else __builtin_amdgcn_wave_barrier();
      for (int n = NW == 1 ? lane : (int)threadIdx.x; n < nb; n += NW == 1 ? 64 : 64 * NW) {
        int lo, hi;
        range(n, lo, hi);
        if (hi - lo > kRelShort) continue;
        const int b0 = qy.pos + lo > j0 ? qy.pos + lo : j0, b1 = qy.pos + hi < j1 ? qy.pos + hi : j1;
        const int mid = (b0 | 31) + 1;  // the next chunk's first key
        float s0 = 0.0f, s1 = 0.0f;
        for (int j = b0; j < b1 && j < mid; ++j) s0 = s0 + st[NW == 1 ? w : j >> 11].t[(j >> 5) & 63][j & 31];
        for (int j = mid; j < b1; ++j) s1 = s1 + st[NW == 1 ? w : j >> 11].t[(j >> 5) & 63][j & 31];
        out[n] = s0 + s1;
      }
      for (int l = 0; l < a.n_long; ++l) {
        const int n = a.longs[l];
        int lo, hi;
        range(n, lo, hi);
        const int b0 = qy.pos + lo > j0 ? qy.pos + lo : j0, b1 = qy.pos + hi < j1 ? qy.pos + hi : j1;
        float sum = 0.0f;
        if (b0 < b1 && b0 < seg + (int)kRegCols && b1 > seg) {  // the same for the whole wavefront
          const int first = b0 - seg - 32 * lane, last = b1 - seg - 32 * lane;
#pragma unroll
          for (int k = 0; k < kChunk; k += 4) {
            const float4 v = *reinterpret_cast<const float4*>(&st[w].t[lane][k]);
            sum = sum + (k >= first && k < last ? v.x : 0.0f);
            sum = sum + (k + 1 >= first && k + 1 < last ? v.y : 0.0f);
            sum = sum + (k + 2 >= first && k + 2 < last ? v.z : 0.0f);
            sum = sum + (k + 3 >= first && k + 3 < last ? v.w : 0.0f);
          }
          const int64_t left = a.k_len - seg < kRegCols ? a.k_len - seg : kRegCols;
          sum = wave_fold(sum, (int)((left + kChunk - 1) / kChunk));
        }
        if constexpr (NW > 1) {
          if (lane == 0) part[l & 1][w] = sum;
          __syncthreads();
          const int parts = (int)((a.k_len + kRegCols - 1) / kRegCols);
          sum = wave_fold(lane < parts ? part[l & 1][lane] : 0.0f, parts);
        }
        if (lane == 0 && (NW == 1 || w == 0)) out[n] = sum;
      }
      if constexpr (NW > 1) __syncthreads();  // the row's ds are read
    }
  }
}

// chains of 32 rows of a [rows][cols] matrix's columns
__global__ __launch_bounds__(256) void column_chain_kernel(int64_t rows, int64_t cols, const float* __restrict__ x,
                                                           float* __restrict__ part) {
  const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (col >= cols) return;
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  for (int64_t c = blockIdx.y; c < nc; c += gridDim.y) {
    const int64_t t0 = c * kChunk;
    const int n = (int)(rows - t0 < kChunk ? rows - t0 : kChunk);
    float s = 0.0f;
    if (n == kChunk) {
#pragma unroll
      for (int k = 0; k < kChunk; k += 8) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = x[(t0 + k + i) * cols + col];
#pragma unroll
        for (int i = 0; i < 8; ++i) s = s + v[i];
      }
    } else {
      for (int k = 0; k < n; ++k) s = s + x[(t0 + k) * cols + col];
    }
    part[c * cols + col] = s;
  }
}

int key_waves(int64_t k_len) {
  int nw = 1;
  while (nw * kRegCols < k_len) nw <<= 1;
  return nw;
}

}  // namespace

#define CANON_REL_WAVES(K, nw)  \
  switch (nw) {                 \
    case 1: K(1); break;        \
    case 2: K(2); break;        \
    case 4: K(4); break;        \
    case 8: K(8); break;        \
    default: K(16); break;      \
  }

hipError_t relbias_fwd_launch(const RelBiasArgs& a, const float* scores, uint16_t* probs, hipStream_t s) {
  const int nw = key_waves(a.k_len);
  const int64_t per_head = (a.q_len + (nw == 1 ? 4 : 1) * kQueries - 1) / ((nw == 1 ? 4 : 1) * kQueries);
  const int64_t blocks = a.batch * a.heads * per_head;
  if (blocks == 0 || a.k_len == 0) return hipSuccess;
  const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks)), wg(nw == 1 ? 256 : 64 * nw);
  const bool tail = a.k_len % 4 != 0;
  const int far = a.start[a.n_side - 1];
  const size_t lds = sizeof(float) * (size_t)(far + 1 + (a.bidirectional ? far : 0));
#define CANON_REL(NW)                                                                                                   \
  do {                                                                                                                  \
    if (tail)                                                                                                           \
      hipLaunchKernelGGL((relbias_fwd_kernel<NW, true>), grid, wg, lds, s, a, blocks, per_head, scores, probs);         \
    else                                                                                                                \
      hipLaunchKernelGGL((relbias_fwd_kernel<NW, false>), grid, wg, lds, s, a, blocks, per_head, scores, probs);        \
  } while (0)
  CANON_REL_WAVES(CANON_REL, nw)
#undef CANON_REL
  return hipGetLastError();
}

int64_t relbias_scratch_floats(int64_t rows, int64_t heads, int64_t buckets) {
  return (rows + (rows + kChunk - 1) / kChunk) * heads * buckets;
}

hipError_t relbias_bwd_launch(const RelBiasArgs& a, const uint16_t* probs, const float* dprobs, uint16_t* dscores,
                              float* dtable, float* rowsum, hipStream_t s) {
  const int nw = key_waves(a.k_len);
  const int64_t per_head = (a.q_len + (nw == 1 ? 4 : 1) * kQueries - 1) / ((nw == 1 ? 4 : 1) * kQueries);
  const int64_t blocks = a.batch * a.heads * per_head;
  const bool empty = blocks == 0 || a.k_len == 0;
  if (!empty) {
    const dim3 grid((unsigned)(blocks < kMaxBlocks ? blocks : kMaxBlocks)), wg(nw == 1 ? 256 : 64 * nw);
    const bool tail = a.k_len % 4 != 0;
    float* rs = dtable ? rowsum : nullptr;
#define CANON_REL(NW)                                                                                                   \
  do {                                                                                                                  \
    if (tail)                                                                                                           \
      hipLaunchKernelGGL((relbias_bwd_kernel<NW, true>), grid, wg, 0, s, a, blocks, per_head, probs, dprobs, dscores,   \
                         rs);                                                                                           \
    else                                                                                                                \
      hipLaunchKernelGGL((relbias_bwd_kernel<NW, false>), grid, wg, 0, s, a, blocks, per_head, probs, dprobs, dscores,  \
                         rs);                                                                                           \
  } while (0)
    CANON_REL_WAVES(CANON_REL, nw)
#undef CANON_REL
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!dtable) return hipSuccess;
  const int64_t nb = a.n_side * (a.bidirectional ? 2 : 1), cols = a.heads * nb;
  const int64_t rows = empty ? 0 : a.batch * a.q_len, nc = (rows + kChunk - 1) / kChunk;
  float* part = rowsum + rows * cols;
  if (rows > 0) {
    hipLaunchKernelGGL(column_chain_kernel, dim3((unsigned)((cols + 255) / 256), (unsigned)(nc < 65535 ? nc : 65535)),
                       dim3(256), 0, s, rows, cols, rowsum, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return column_fold_launch(rows, cols, nb, part, dtable, s);
}

}  // namespace canon
