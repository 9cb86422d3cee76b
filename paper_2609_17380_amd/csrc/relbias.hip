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
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, NW == 1 ? 4 : 1) void relbias_fwd_kernel(
    RelBiasArgs a, int64_t blocks, int64_t per_head, const float* __restrict__ scores, uint16_t* __restrict__ probs) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW], top[NW];
  extern __shared__ float near_[];  // bias by position: of the key less the query's, the near side of the last buckets
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int far = a.start[a.n_side - 1], right = a.bidirectional ? far : 0;
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;  // this wavefront's part of the row
  const int n = (int)a.k_len - seg < (int)kRegCols ? (int)a.k_len - seg : (int)kRegCols;
  int turn = 0;  // rows in turn take one of two slots, so that a barrier lies between a slot's reads and its next writes
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int64_t bh = blk / per_head, b = bh / a.heads, h = bh - b * a.heads;
    const int64_t i0 = (blk - bh * per_head) * (kRows * kQueries);
    __syncthreads();  // the last block's biases are read
    for (int e = threadIdx.x; e <= far + right; e += blockDim.x) {
      const int d = far - e;  // query less key: far .. -right
      const int k = d >= 0 ? bucket_of(a.start, a.n_side, d) : a.n_side + bucket_of(a.start, a.n_side, -d);
      near_[e] = bf16_to_f32(a.table[k * a.heads + h]);
    }
    __syncthreads();
    for (int it = 0; it < kQueries; ++it) {
      const int64_t i = i0 + it * kRows + (NW == 1 ? w : 0);
      if (i >= a.q_len) break;  // the same for every wavefront that shares the row
      const Query qy = query_of(a, b, i);
      const int j0 = qy.j0 - seg, span = qy.j1 - qy.j0, first = far + seg - qy.pos;  // near_ entry of the part's first key
      const float* rr = scores + (bh * a.q_len + i) * a.ld + seg;
      auto any = [&](int q) { return 256 * q < j0 + span && 256 * q + 255 >= j0; };
      float e[kRegQ][4];
      part_load<TAIL>(n < j0 + span ? n : j0 + span + 3 < n ? j0 + span + 3 : n, e,
                      [&](int j, float(&v)[4]) {
                        if (j + 3 >= j0) ldf<4>(rr + j, v);
                        else v[0] = v[1] = v[2] = v[3] = 0.0f;
                      },
                      [&](int j) { return rr[j]; });
      float m = -__builtin_inff();
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
        if (!any(q)) {
#pragma unroll
          for (int t = 0; t < 4; ++t) e[q][t] = -__builtin_inff();
          continue;
        }
        const int j = 256 * q + 4 * lane;
        const bool left = first + 256 * q + 255 <= 0;
        float bias[4];
        if (left || first + 256 * q >= far + right) {
          bias[0] = bias[1] = bias[2] = bias[3] = near_[left ? 0 : far + right];
        } else {
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int k = first + j + t;
            bias[t] = near_[k < 0 ? 0 : k > far + right ? far + right : k];
          }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = e[q][t] * a.scale;
          const float z = x + bias[t];
          e[q][t] = (unsigned)(j + t - j0) < (unsigned)span ? z : -__builtin_inff();  // unseen: an e of +0
          m = fmaxf(m, e[q][t]);
        }
      }
      m = wave_most(m);
      if constexpr (NW > 1) {
        if (lane == 0) top[w] = m;
        __syncthreads();
        m = wave_most(lane < NW ? top[lane] : -__builtin_inff());
      }
      // a row whose seen scores are all -inf has e = cexp(-inf) = +0, not cexp(-inf - -inf)
      m = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
      for (int q = 0; q < kRegQ; ++q) {
#pragma unroll
        for (int t = 0; t < 4; ++t) e[q][t] = any(q) ? cexp_neg(e[q][t] - m) : 0.0f;
      }
      turn ^= 1;
      const float S = wide_row_sum<NW>(st[w], e, (int)a.k_len, slot[turn]);
      const float rcp = S == 0.0f ? 0.0f : 1.0f / S;
      uint16_t* pr = probs + (bh * a.q_len + i) * a.ld + seg;
      if (S == S) {
        part_store<TAIL>(n,
                         [&](int q, float(&o)[4]) {
#pragma unroll
                           for (int t = 0; t < 4; ++t) o[t] = e[q][t] * rcp;
                         },
                         [&](int j, const float(&o)[4]) { stb_arith(pr + j, o); },
                         [&](int j, float o) { pr[j] = bf16_arith(o); });
      } else {  // a NaN among the seen: every seen key's, and still +0 elsewhere
        for (int j = lane; j < n; j += 64) pr[j] = (unsigned)(j - j0) < (unsigned)span ? 0x7FC0 : 0;
      }
    }
  }
}

// ds = RN(P RN(dP - D)), D = R1 over the keys of RN(P dP); dS = bf16(RN(ds scale)).  rowsum [batch][q_len][heads][buckets]:
// for every bucket R1 over the keys of ds, those outside it as +0 terms.  A bucket of up to 32 distances touches at most
// two chunks, whose chains one lane runs and adds (their sum is the fold whatever lies between); a longer one is summed
// chunk by chunk, a lane to a chunk, like the row.
template <int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, NW == 1 ? 4 : 1) void relbias_bwd_kernel(
    RelBiasArgs a, int64_t blocks, int64_t per_head, const uint16_t* __restrict__ probs,
    const float* __restrict__ dprobs, uint16_t* __restrict__ dscores, float* __restrict__ rowsum) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RegStage st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  __shared__ float part[2][NW];
  __shared__ int lo_[2 * kRelStarts], hi_[2 * kRelStarts];  // the keys of a bucket, less the query's position: lo <= . < hi
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int seg = NW == 1 ? 0 : w * (int)kRegCols;
  const int n = (int)a.k_len - seg < (int)kRegCols ? (int)a.k_len - seg : (int)kRegCols;
  const int nb = a.n_side * (a.bidirectional ? 2 : 1);
  int turn = 0;  // as above
  if (rowsum) {
    for (int k = threadIdx.x; k < nb; k += blockDim.x) {
      const int side = k < a.n_side ? k : k - a.n_side;
      const int d0 = a.start[side], d1 = side + 1 < a.n_side ? a.start[side + 1] : 2 * (int)kFarPos;
      if (k < a.n_side) {
        lo_[k] = 1 - d1;
        hi_[k] = d0 == d1 ? 1 - d1 : d0 == 0 && !a.bidirectional ? 2 * (int)kFarPos : 1 - d0;
      } else {
        lo_[k] = d0 > 0 ? d0 : 1;
        hi_[k] = d1;
      }
    }
    __syncthreads();
  }
  for (int64_t blk = blockIdx.x; blk < blocks; blk += gridDim.x) {
    const int64_t bh = blk / per_head, b = bh / a.heads, h = bh - b * a.heads;
    const int64_t i0 = (blk - bh * per_head) * (kRows * kQueries);
    for (int it = 0; it < kQueries; ++it) {
      const int64_t i = i0 + it * kRows + (NW == 1 ? w : 0);
      if (i >= a.q_len) break;
      const Query qy = query_of(a, b, i);
      const int j0 = qy.j0 - seg, span = qy.j1 - qy.j0;
      const int64_t at = (bh * a.q_len + i) * a.ld + seg;
      const uint16_t* pr = probs + at;
      const float* dr = dprobs + at;
      const int upto = n < j0 + span ? n : j0 + span + 3 < n ? j0 + span + 3 : n;  // whole vectors of what is seen
      float p[kRegQ][4], dp[kRegQ][4], e[kRegQ][4];
      part_load<TAIL>(upto, p,
                      [&](int j, float(&v)[4]) {
                        if (j + 3 >= j0) ldb_wide(pr + j, v);
                        else v[0] = v[1] = v[2] = v[3] = 0.0f;
                      },
                      [&](int j) { return bf16_wide(pr[j]); });
      part_load<TAIL>(upto, dp,
                      [&](int j, float(&v)[4]) {
                        if (j + 3 >= j0) ldf<4>(dr + j, v);
                        else v[0] = v[1] = v[2] = v[3] = 0.0f;
                      },
                      [&](int j) { return dr[j]; });
      auto seen = [&](int q, int t, int first) { return (unsigned)(256 * q + 4 * lane + t - first) < (unsigned)span; };
#pragma unroll
      for (int q = 0; q < kRegQ; ++q)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float x = p[q][t] * dp[q][t];
          e[q][t] = seen(q, t, j0) ? x : 0.0f;
        }
      turn ^= 1;
      const float D = wide_row_sum<NW>(st[w], e, (int)a.k_len, slot[turn]);
      const int first = again(j0);
#pragma unroll
      for (int q = 0; q < kRegQ; ++q)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float d = dp[q][t] - D;
          const float x = p[q][t] * d;
          e[q][t] = seen(q, t, first) ? x : 0.0f;
        }
      uint16_t* sr = dscores + at;
      part_store<TAIL>(n,
                       [&](int q, float(&o)[4]) {
#pragma unroll
                         for (int t = 0; t < 4; ++t) o[t] = e[q][t] * a.scale;
                       },
                       [&](int j, const float(&o)[4]) { stb_arith(sr + j, o); },
                       [&](int j, float o) { sr[j] = bf16_arith(o); });
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
      for (int k = NW == 1 ? lane : (int)threadIdx.x; k < nb; k += NW == 1 ? 64 : 64 * NW) {
        const int lo = lo_[k], hi = hi_[k];
        if (hi - lo > kRelShort) continue;
        const int b0 = qy.pos + lo > qy.j0 ? qy.pos + lo : qy.j0, b1 = qy.pos + hi < qy.j1 ? qy.pos + hi : qy.j1;
        const int mid = (b0 | 31) + 1;  // the next chunk's first key
        float s0 = 0.0f, s1 = 0.0f;
        for (int j = b0; j < b1; j += 4) {
          float v[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const int u = j + t < b1 ? j + t : b0;
            v[t] = st[NW == 1 ? w : u >> 11].t[(u >> 5) & 63][u & 31];
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            s0 = s0 + (j + t < b1 && j + t < mid ? v[t] : 0.0f);
            s1 = s1 + (j + t < b1 && j + t >= mid ? v[t] : 0.0f);
          }
        }
        out[k] = s0 + s1;
      }
      for (int l = 0; l < a.n_long; ++l) {
        const int k = a.longs[l];
        const int lo = lo_[k], hi = hi_[k];
        const int b0 = (qy.pos + lo > qy.j0 ? qy.pos + lo : qy.j0) - seg, b1 = (qy.pos + hi < qy.j1 ? qy.pos + hi : qy.j1) - seg;
        float sum = 0.0f;
        if (b0 < b1 && b0 < (int)kRegCols && b1 > 0) {  // the same for the whole wavefront
          const int c0 = b0 - 32 * lane, len = b1 - b0;
#pragma unroll
          for (int t = 0; t < kChunk; t += 4) {
            const float4 v = *reinterpret_cast<const float4*>(&st[w].t[lane][t]);
            sum = sum + ((unsigned)(t - c0) < (unsigned)len ? v.x : 0.0f);
            sum = sum + ((unsigned)(t + 1 - c0) < (unsigned)len ? v.y : 0.0f);
            sum = sum + ((unsigned)(t + 2 - c0) < (unsigned)len ? v.z : 0.0f);
            sum = sum + ((unsigned)(t + 3 - c0) < (unsigned)len ? v.w : 0.0f);
          }
          sum = wave_total(sum);
        }
        if constexpr (NW > 1) {
          if (lane == 0) part[l & 1][w] = sum;
          __syncthreads();
          const int parts = ((int)a.k_len + (int)kRegCols - 1) / (int)kRegCols;
          sum = wave_total(lane < parts ? part[l & 1][lane] : 0.0f);
        }
        if (lane == 0 && (NW == 1 || w == 0)) out[k] = sum;
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
  return column_fold_launch(rows, cols, nb, part, dtable, nullptr, s);
}

}  // namespace canon
