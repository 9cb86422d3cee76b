// relbias.hip - attention rows with a learned relative position bias (R22): raw scores to probabilities, and the gradient
// of the scores and of the bias table.
//
// A row of up to 2048 keys is held by one wavefront, a longer one by a workgroup of up to 16 (wide_row_sum): scores,
// probabilities and their gradient are read from memory once.  The keys that a query sees are one range j0 <= j < j1
// (lengths, causality and the window all cut it from an end), so no mask is read.  A head's biases, by distance up to
// the last bucket's first, are laid out in LDS while the row is on its way.  Bound: HBM.
#include <hip/hip_runtime.h>

#include <atomic>

#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

namespace {

constexpr int64_t kMaxBlocks = 1 << 20;  // of up to 1024 threads: 2^30 of 2^32

// distances after the query that the bias table holds: up to the last bucket's, one at least
__host__ __device__ inline int relbias_right(const RelBiasArgs& a) {
  const int far = a.start[a.n_side - 1];
  return a.bidirectional ? (far > 0 ? far : 1) : 0;
}

// The keys j0 <= j < j1 that query i of sequence b sees (none behind the last query), and its position (cut to +-kRelFarPos,
// which leaves every bucket as it is).
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
  if (i >= a.q_len || (a.q_lens && i >= a.q_lens[b])) hi = 0;
  if (hi <= lo) lo = hi = 0;
  Query q;
  q.j0 = __builtin_amdgcn_readfirstlane((int)lo);
  q.j1 = __builtin_amdgcn_readfirstlane((int)hi);
  q.pos = __builtin_amdgcn_readfirstlane((int)(pos < -kRelFarPos ? -kRelFarPos : pos > kRelFarPos ? kRelFarPos : pos));
  return q;
}

// What a query sees of a wavefront's part of the row, n keys from `seg` on: its elements from .. end - 1, all of them in
// the vectors q0 .. q1 - 1; upto: the end of the vectors that hold them, within the part.
struct Part {
  int from, end, upto, q0, q1;
  __device__ __forceinline__ bool sees(int j) const { return (unsigned)(j - from) < (unsigned)(end - from); }
  __device__ __forceinline__ bool sees_all(int q) const { return from <= 256 * q && 256 * q + 256 <= end; }
};
__device__ __forceinline__ Part part_of(const Query& q, int seg, int n) {
  Part p;
  p.from = q.j0 - seg > 0 ? q.j0 - seg : 0;
  p.end = q.j1 - seg < n ? q.j1 - seg : n;
  if (p.end <= p.from) p.from = p.end = 0;
  p.upto = p.end + 3 < n ? (p.end + 3) & ~3 : n;
  if (p.end == 0) p.upto = 0;
  p.q0 = p.from >> 8;
  p.q1 = (p.end + 255) >> 8;
  return p;
}

// 16 x 2048 x 2048 causal 70 us (the 268 MB that it cannot do without take 56 at a large copy's rate), in both directions 92
// (85); a padded batch of 4 x 8 x 1001 x 1001 37.8 (26), where vector instructions, 26 of a canonical exponential among the
// 40 to a score, take 61% of the cycles: more than anything else, but no bound.  With the next row loaded ahead and a matrix's
// biases laid out once for many rows the padded batch took 40: fewer rows at a time.
template <int Q, int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, Q == 8 ? 4 : 1) void relbias_fwd_kernel(
    RelBiasArgs a, uint32_t heads, uint32_t matrices, uint32_t per_head, const float* __restrict__ scores,
    uint16_t* __restrict__ probs) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RowStage<Q> st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW], top[NW];
  extern __shared__ float near_[];  // bias by place: key less query, from -far to `right`
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int far = a.start[a.n_side - 1], right = relbias_right(a);
  const int seg = NW == 1 ? 0 : w * 256 * Q;  // this wavefront's part of the row
  const int n = (int)a.k_len - seg < 256 * Q ? (int)a.k_len - seg : 256 * Q;
  const int parts = ((int)a.k_len + 256 * Q - 1) / (256 * Q);
  int turn = 0;  // rows in turn take one of two slots, so that a barrier lies between a slot's reads and its next writes
  // a matrix's rows along x, the matrices (batch and head) along y; each further on by the grid where that ends first
  bool once = true;  // this workgroup's first rows
  for (uint32_t m = blockIdx.y; m < matrices; m += gridDim.y)
  for (uint32_t blk = blockIdx.x; blk < per_head; blk += gridDim.x) {
    const int64_t bh = m, b = m / heads, h = m % heads;
    const int64_t i = (int64_t)blk * kRows + (NW == 1 ? w : 0);
    const Query qy = query_of(a, b, i);
    const Part pt = part_of(qy, seg, n);
    const int64_t row = (bh * a.q_len + i) * a.ld + seg;
    const float* rr = scores + row;
    uint16_t* pr = probs + row;
    float e[Q][4];
    part_load<TAIL>(pt.from, pt.upto, e, rr);
    if (!once) __syncthreads();  // the last row's biases are read
    once = false;
    for (int k = threadIdx.x; k <= far + right; k += blockDim.x) {
      const int d = far - k;  // query less key
      near_[k] = bf16_to_f32(a.table[(d >= 0 ? a.bucket[d] : a.n_side + a.bucket[-d < far ? -d : far]) * a.heads + h]);
    }
    __syncthreads();
    if (i >= a.q_len) continue;  // NW = 1: a wavefront without a row
    const int first = far + seg - qy.pos;  // the part's first key in near_
    float most = -__builtin_inff();
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (q < pt.q0 || q >= pt.q1) continue;
      const int j = 256 * q + 4 * lane;
      float bias[4];
      if (first + 256 * q <= -255) {
        bias[0] = bias[1] = bias[2] = bias[3] = near_[0];
      } else if (first + 256 * q >= far + right) {
        bias[0] = bias[1] = bias[2] = bias[3] = near_[far + right];
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
        e[q][t] = x + bias[t];
      }
      if (!pt.sees_all(q)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) e[q][t] = pt.sees(j + t) ? e[q][t] : -__builtin_inff();  // unseen: an e of +0
      }
#pragma unroll
      for (int t = 0; t < 4; ++t) most = fmaxf(most, e[q][t]);
    }
    most = wave_most(most);
    if constexpr (NW > 1) {
      if (lane == 0) top[w] = most;
      __syncthreads();
      most = wave_most(lane < parts ? top[lane] : -__builtin_inff());
    }
    // a row whose seen scores are all -inf has e = cexp(-inf) = +0, not cexp(-inf - -inf)
    most = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (q < pt.q0 || q >= pt.q1) continue;
#pragma unroll
      for (int t = 0; t < 4; ++t) e[q][t] = cexp_neg(e[q][t] - most);
      st[w].put(q, lane, e[q]);
    }
    turn ^= 1;
    const float S = wide_join<NW>(st[w].span_sum(pt.q0, pt.q1), parts, slot[turn]);
    const float rcp = S == 0.0f ? 0.0f : 1.0f / S;
    if (S == S) {
      part_store<TAIL, Q>(n,
                       [&](int q, float(&o)[4]) {
                         if (q >= pt.q0 && q < pt.q1) {
#pragma unroll
                           for (int t = 0; t < 4; ++t) o[t] = e[q][t] * rcp;
                         } else {
                           o[0] = o[1] = o[2] = o[3] = 0.0f;
                         }
                       },
                       [&](int j, const float(&o)[4]) { stb_arith(pr + j, o); },
                       [&](int j, float o) { pr[j] = bf16_arith(o); });
    } else {  // a NaN among the seen: every seen key's, and still +0 elsewhere
      for (int j = lane; j < n; j += 64) pr[j] = pt.sees(j) ? 0x7FC0 : 0;
    }
  }
}

// ds = RN(P RN(dP - D)), D = R1 over the keys of RN(P dP); dS = bf16(RN(ds scale)).  rowsum [batch][q_len][heads][buckets]:
// for every bucket R1 over the keys of ds, those outside it as +0 terms.  A bucket of up to 32 keys touches at most two
// chunks, whose chains two lanes run and add (their sum is the fold whatever lies between); a longer one is summed chunk by
// chunk, a lane to a chunk, like the row: 16 x 2048 x 2048 causal with 32 buckets up to 256 85 us, up to 1024 115; in both
// directions (537 MB: 113) up to 128 113, 256 132, 1024 149.
// 16 x 2048 x 2048 causal 68 us, and 10 for the sums over the rows (336 MB: 70.5), without the table's gradient 70; 16 x 16 x
// 512 110 (71), without 75: there the buckets' sums, about 190 vector instructions to a row of at most 512 keys, take most of the
// difference (119 with seven workgroups to a CU, as the registers of a kernel without a bound let in, and eight launched).
template <int Q, int NW, bool TAIL>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW, Q == 8 ? 4 : Q == 2 ? 8 : 1) void relbias_bwd_kernel(
    RelBiasArgs a, uint32_t heads, uint32_t units, uint32_t per_head, const uint16_t* __restrict__ probs,
    const float* __restrict__ dprobs, uint16_t* __restrict__ dscores, float* __restrict__ rowsum) {
  constexpr int kRows = NW == 1 ? 4 : 1;
  __shared__ __attribute__((aligned(16))) RowStage<Q> st[NW == 1 ? 4 : NW];
  __shared__ float slot[2][NW];
  __shared__ float part[2][NW];
  __shared__ int lo_[2 * kRelStarts], hi_[2 * kRelStarts];  // the keys of a bucket, less the query's position: lo <= . < hi
  const int w = wave_id(), lane = threadIdx.x & 63;
  const int seg = NW == 1 ? 0 : w * 256 * Q;
  const int n = (int)a.k_len - seg < 256 * Q ? (int)a.k_len - seg : 256 * Q;
  const int parts = ((int)a.k_len + 256 * Q - 1) / (256 * Q);
  const int nb = a.n_side * (a.bidirectional ? 2 : 1);
  int turn = 0;  // as above
  // What is made of a size: held, or beside 8 vectors, which leave no register, made again where it is used (4096 rows of 4096
  // keys 354 us, held 387).
  auto use = [](int size) __attribute__((always_inline)) { return Q == 8 ? again(size) : size; };
  auto none = [&]() __attribute__((always_inline)) { return kChunk * lane < use(n) ? 0.0f : kNoTerm; };  // a chunk without a term
  uint32_t pw[Q][2];
  float dp[Q][4];
  // A unit is kRows queries of a matrix (batch and head); a wavefront loads its row of the next one before it sums this
  // one's buckets, when this one's values are no longer needed.
  struct At {
    Query qy;
    Part pt;
    int64_t i, b, h, row;
  };
  auto load = [&](uint32_t unit) __attribute__((always_inline)) {  // of no key behind the last one
    const uint32_t u = unit < units ? unit : units - 1, m = u / per_head;
    At t;
    t.b = m / heads;
    t.h = m % heads;
    t.i = unit < units ? (int64_t)(u - m * per_head) * kRows + (NW == 1 ? w : 0) : a.q_len;
    t.qy = query_of(a, t.b, t.i);
    t.pt = part_of(t.qy, seg, n);
    t.row = ((int64_t)m * a.q_len + t.i) * a.ld + seg;
    const uint16_t* pr = probs + t.row;
    const float* dr = dprobs + t.row;
    part_load_bf16<TAIL>(t.pt.from, t.pt.upto, pw, pr);
    part_load<TAIL>(t.pt.from, t.pt.upto, dp, dr);
    return t;
  };
  // Units are dealt out forth and back, so that a workgroup's causal rows are long and short in turn.
  auto dealt = [&](uint32_t round) {
    return round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
  };
  const uint32_t rounds = (units + gridDim.x - 1) / gridDim.x;
  At at = load(dealt(0));
  if (rowsum) {
    for (int k = threadIdx.x; k < nb; k += blockDim.x) {
      const RelKeys keys = relbias_keys(a, k);
      lo_[k] = keys.lo;
      hi_[k] = keys.hi;
    }
    __syncthreads();
  }
  for (uint32_t round = 0; round < rounds; ++round) {
    const At now = at;
    const Query qy = now.qy;
    const Part pt = now.pt;
    if (now.i >= a.q_len) {  // a wavefront, or in the last round a workgroup, without a row
      at = load(round + 1 < rounds ? dealt(round + 1) : units);
      continue;
    }
    uint16_t* sr = dscores + now.row;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      if (q < pt.q0 || q >= pt.q1) continue;
      float e[4];
      wide4(pw[q], e);
#pragma unroll
      for (int t = 0; t < 4; ++t) e[t] = e[t] * dp[q][t];
      if (!pt.sees_all(q)) {
#pragma unroll
        for (int t = 0; t < 4; ++t) e[t] = pt.sees(256 * q + 4 * lane + t) ? e[t] : 0.0f;
      }
      st[w].put(q, lane, e);
    }
    turn ^= 1;
    st[w].end(use(n));
    __builtin_amdgcn_wave_barrier();
    const float D = wide_join<NW>(wave_total(st[w].span_chain(pt.q0, pt.q1, use(n), none())), parts, slot[turn]);
    Part pu = pt;
    pu.from = again(pt.from);
    part_store<TAIL, Q>(n,
                     [&](int q, float(&o)[4]) {
                       if (q >= pt.q0 && q < pt.q1) {
                         float ds[4];
                         wide4(pw[q], ds);
#pragma unroll
                         for (int t = 0; t < 4; ++t) {
                           const float d = dp[q][t] - D;
                           ds[t] = ds[t] * d;
                         }
#pragma unroll
                         for (int t = 0; t < 4; ++t) o[t] = ds[t] * a.scale;
                         if (!pu.sees_all(q)) {
#pragma unroll
                           for (int t = 0; t < 4; ++t) {
                             const bool sees = pu.sees(256 * q + 4 * lane + t);
                             ds[t] = sees ? ds[t] : 0.0f;
                             o[t] = sees ? o[t] : 0.0f;  // +0 whatever the scale's sign
                           }
                         }
                         st[w].put(q, lane, ds);  // for the buckets' sums
                       } else {
                         o[0] = o[1] = o[2] = o[3] = 0.0f;
                       }
                     },
                     [&](int j, const float(&o)[4]) { stb_arith(sr + j, o); },
                     [&](int j, float o) { sr[j] = bf16_arith(o); });
    at = load(round + 1 < rounds ? dealt(round + 1) : units);
    if (!rowsum) continue;
    st[w].end(use(n));
    float* out = rowsum + ((now.b * a.q_len + now.i) * a.heads + now.h) * nb;
    if constexpr (NW > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    const int keys = use((int)a.k_len);
    for (int k2 = NW == 1 ? lane : (int)threadIdx.x; k2 < 2 * nb; k2 += NW == 1 ? 64 : (int)blockDim.x) {
      const int k = k2 >> 1, lo = lo_[k], hi = hi_[k];
      const bool pair = RelKeys{lo, hi}.short_one();
      const int b0 = qy.pos + lo > qy.j0 ? qy.pos + lo : qy.j0, b1 = qy.pos + hi < qy.j1 ? qy.pos + hi : qy.j1;
      const int mid = (b0 | 31) + 1;  // the next chunk's first key
      const int c0 = k2 & 1 ? mid : b0, c1 = k2 & 1 || b1 < mid ? b1 : mid;
      float sum = 0.0f;
      if (c0 < c1 && pair) {
        const float* t = &st[NW == 1 ? w : c0 / (256 * Q)].t[(c0 >> 5) & (8 * Q - 1)][c0 & 31];
        const uint32_t mine = 0xFFFFFFFFu >> (32 - (c1 - c0));  // a bit for each of its keys
        for (int j = 0; j < a.short_most && j < c1 - c0; j += 4) {  // up to three places behind the chunk's end: its row's padding
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const uint32_t take = (uint32_t)__builtin_amdgcn_sbfe((int)mine, j + u, 1);  // all ones or none
            sum = sum + __uint_as_float((__float_as_uint(t[j + u]) & take) | (__float_as_uint(kNoTerm) & ~take));
          }
        }
      }
      // The bucket's two chunks, of which a -0 is left as it is only where nothing is added to it: no term of +0 behind the
      // bucket in the chunk, no partial of +0 but theirs, and none after their sum.
      if (keys > 2 * kChunk) {
        sum = sum + 0.0f;
        sum = sum + __uint_as_float(lane_move<0xB1>(__float_as_uint(sum)));
        const float more = sum + 0.0f;
        sum = mid == kChunk << (31 - __builtin_clz((unsigned)(keys - 1) / kChunk)) ? sum : more;
      } else {
        if (c0 < c1 && (c1 & (kChunk - 1)) != 0 && c1 < keys) sum = sum + 0.0f;
        if (keys > kChunk) {
          sum = sum + __uint_as_float(lane_move<0xB1>(__float_as_uint(sum)));
          if (mid > kChunk) sum = sum + 0.0f;
        }
      }
      if (!(k2 & 1) && pair) out[k] = sum;
    }
    if (a.far_only) {
      // the last bucket(s) alone are long: the keys nearer than them give way to +0, and a lane's chunk is one bucket's
      if constexpr (NW > 1) __syncthreads();  // the short buckets' keys are read
      else __builtin_amdgcn_wave_barrier();
      const int far = a.start[a.n_side - 1];
      const int z0 = (qy.pos - far + 1 > qy.j0 ? qy.pos - far + 1 : qy.j0) - seg;
      const int z1 = (a.bidirectional && qy.pos + far < qy.j1 ? qy.pos + far : qy.j1) - seg;
      if (far > 0)  // one bucket alone: no key is nearer
        for (int z = (z0 > 0 ? z0 : 0) + lane; z < z1 && z < 256 * Q; z += 64) st[w].t[z >> 5][z & 31] = 0.0f;
      __builtin_amdgcn_wave_barrier();
      const float no = none(), c = st[w].span_chain(pt.q0, pt.q1, use(n), no);
      const bool before = !a.bidirectional || seg + 32 * lane <= qy.pos - far;
      float left = wave_total(before ? c : no);
      float right = a.bidirectional ? wave_total(before ? no : c) : 0.0f;
      if constexpr (NW > 1) {
        if (lane == 0) {
          part[0][w] = left;
          part[1][w] = right;
        }
        __syncthreads();
        left = wave_total(lane < parts ? part[0][lane] : kNoTerm);
        right = wave_total(lane < parts ? part[1][lane] : kNoTerm);
      }
      if (lane == 0 && (NW == 1 || w == 0)) {
        out[a.n_side - 1] = left;
        if (a.bidirectional) out[nb - 1] = right;
      }
    } else {
      for (int l = 0; l < a.n_long; ++l) {
        const int k = a.longs[l];
        const int lo = lo_[k], hi = hi_[k];
        const int b0 = (qy.pos + lo > qy.j0 ? qy.pos + lo : qy.j0) - seg, b1 = (qy.pos + hi < qy.j1 ? qy.pos + hi : qy.j1) - seg;
        float sum = 0.0f;
        if (b0 < b1 && b0 < 256 * Q && b1 > 0) {  // the same for the whole wavefront
          float p = 0.0f;
          if (32 * lane < n) {  // up to the row's end what ends it is added as well
            const int c0 = b0 - 32 * lane, len = (b1 < n ? b1 : 256 * Q) - b0;
#pragma unroll
            for (int t = 0; t < kChunk; t += 4) {
              const float4 v = st[w].vec(lane, t / 4);
              p = p + ((unsigned)(t - c0) < (unsigned)len ? v.x : 0.0f);
              p = p + ((unsigned)(t + 1 - c0) < (unsigned)len ? v.y : 0.0f);
              p = p + ((unsigned)(t + 2 - c0) < (unsigned)len ? v.z : 0.0f);
              p = p + ((unsigned)(t + 3 - c0) < (unsigned)len ? v.w : 0.0f);
            }
          } else {
            p = kNoTerm;
          }
          sum = wave_total(p);
        }
        if constexpr (NW > 1) {
          if (lane == 0) part[l & 1][w] = sum;
          __syncthreads();
          sum = wave_total(lane < parts ? part[l & 1][lane] : kNoTerm);
        }
        if (lane == 0 && (NW == 1 || w == 0)) out[k] = sum;
      }
    }
    if constexpr (NW > 1) __syncthreads();  // the row's ds are read
  }
}

// Chains of 32 rows of a [rows][cols] matrix's columns, a wavefront to 64 columns of one, 16 rows in flight: 2048 rows of
// 512 columns 5.3 us, bound by the latency of two batches of loads (4.2 MB).
__global__ __launch_bounds__(64) void column_chain_kernel(int64_t rows, int64_t cols, const float* __restrict__ x,
                                                          float* __restrict__ part) {
  const int64_t col = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (col >= cols) return;
  const int64_t nc = (rows + kChunk - 1) / kChunk;
  for (int64_t c = blockIdx.y; c < nc; c += gridDim.y) {
    const int64_t t0 = c * kChunk;
    const int n = (int)(rows - t0 < kChunk ? rows - t0 : kChunk);
    float s = 0.0f;
    if (n == kChunk) {
#pragma unroll
      for (int k = 0; k < kChunk; k += 16) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = x[(t0 + k + i) * cols + col];
#pragma unroll
        for (int i = 0; i < 16; ++i) s = s + v[i];
      }
    } else {
      for (int k = 0; k < n; ++k) s = s + x[(t0 + k) * cols + col];
    }
    part[c * cols + col] = s;
  }
}

}  // namespace

// Rows along x, matrices along y, within 2^32 threads of x and 65535 of y.
static dim3 relbias_grid(const RowShape& shape, int64_t matrices, int64_t per_head) {
  const int64_t x = per_head < kMaxBlocks ? per_head : kMaxBlocks;
  return dim3((unsigned)x, (unsigned)(matrices < 65535 ? matrices : 65535));
}

hipError_t relbias_fwd_launch(const RelBiasArgs& a, const float* scores, uint16_t* probs, hipStream_t s) {
  const RowShape shape = row_shape(a.batch * a.heads * a.q_len, a.k_len, 6);
  const int64_t matrices = a.batch * a.heads, per_head = shape.groups(a.q_len);
  if (matrices * per_head == 0 || a.k_len == 0) return hipSuccess;
  const dim3 grid = relbias_grid(shape, matrices, per_head), wg(shape.threads());
  const bool tail = a.k_len % 4 != 0;
  const size_t lds = sizeof(float) * (size_t)(a.start[a.n_side - 1] + 1 + relbias_right(a));
#define CANON_REL_K(Q, NW, TAIL)                                                                                    \
  hipLaunchKernelGGL((relbias_fwd_kernel<Q, NW, TAIL>), grid, wg, lds, s, a, (uint32_t)a.heads, (uint32_t)matrices, \
                     (uint32_t)per_head, scores, probs)
#define CANON_REL(Q, NW)                   \
  do {                                     \
    if (tail) CANON_REL_K(Q, NW, true);    \
    else CANON_REL_K(Q, NW, false);        \
  } while (0)
  CANON_ROW_SHAPES(CANON_REL, shape);
#undef CANON_REL
#undef CANON_REL_K
  return hipGetLastError();
}

// Workgroups of the backward that are on the chip at once.  Rows are dealt to all that are launched, so one that has to wait
// for another to end runs its share when the chip is nearly empty: with 8 to a CU where the LDS of two wavefronts' rows lets 7
// in, 16 x 4096 x 4096 took 354 us, so 288; 4 x 16 x 1000 x 1000 88 and 82; 16 x 512 x 10000 152 and 129.  Asked of the runtime
// once per kernel, workgroup size and device.
template <int Q, int NW, bool TAIL>
static hipError_t relbias_resident(int threads, int64_t& groups) {
  static std::atomic<int> known[64][17];
  int dev = 0, per_cu = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const bool keep = dev >= 0 && dev < 64;
  if (keep) per_cu = known[dev][threads / 64].load(std::memory_order_relaxed);
  if (per_cu == 0) {
    e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, relbias_bwd_kernel<Q, NW, TAIL>, threads, 0);
    if (e != hipSuccess) return e;
    if (per_cu < 1) per_cu = 1;
    if (keep) known[dev][threads / 64].store(per_cu, std::memory_order_relaxed);
  }
  groups = device_cus() * per_cu;
  return hipSuccess;
}

int64_t relbias_scratch_floats(int64_t rows, int64_t heads, int64_t buckets) {
  return (rows + (rows + kChunk - 1) / kChunk) * heads * buckets;
}

hipError_t relbias_bwd_launch(const RelBiasArgs& a, const uint16_t* probs, const float* dprobs, uint16_t* dscores,
                              float* dtable, float* rowsum, hipStream_t s) {
  const RowShape shape = row_shape(a.batch * a.heads * a.q_len, a.k_len, 6);
  const int64_t matrices = a.batch * a.heads, per_head = shape.groups(a.q_len);
  const bool empty = matrices * per_head == 0 || a.k_len == 0;
  if (!empty) {
    const int64_t units = matrices * per_head;
    const dim3 wg(shape.threads());
    int64_t most = 0;
    const bool tail = a.k_len % 4 != 0;
    float* rs = dtable ? rowsum : nullptr;
#define CANON_REL_K(Q, NW, TAIL)                                                                                        \
  do {                                                                                                                  \
    hipError_t e = relbias_resident<Q, NW, TAIL>(shape.threads(), most);                                                \
    if (e != hipSuccess) return e;                                                                                      \
    hipLaunchKernelGGL((relbias_bwd_kernel<Q, NW, TAIL>), dim3((unsigned)(units < most ? units : most)), wg, 0, s, a,   \
                       (uint32_t)a.heads, (uint32_t)units, (uint32_t)per_head, probs, dprobs, dscores, rs);             \
  } while (0)
#define CANON_REL(Q, NW)                   \
  do {                                     \
    if (tail) CANON_REL_K(Q, NW, true);    \
    else CANON_REL_K(Q, NW, false);        \
  } while (0)
    CANON_ROW_SHAPES(CANON_REL, shape);
#undef CANON_REL
#undef CANON_REL_K
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!dtable) return hipSuccess;
  const int64_t nb = a.n_side * (a.bidirectional ? 2 : 1), cols = a.heads * nb;
  const int64_t rows = empty ? 0 : a.batch * a.q_len, nc = (rows + kChunk - 1) / kChunk;
  float* part = rowsum + rows * cols;
  if (rows > 0) {
    hipLaunchKernelGGL(column_chain_kernel, dim3((unsigned)((cols + 63) / 64), (unsigned)(nc < 65535 ? nc : 65535)),
                       dim3(64), 0, s, rows, cols, rowsum, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return column_fold_launch(rows, cols, nb, part, dtable, nullptr, s);
}

}  // namespace canon
