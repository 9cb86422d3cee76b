// rows_dev.h - what the row kernels share: loads and stores of four elements at any alignment, and the R1 sum of a row
// held in a wavefront's registers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "canon_dev.h"
#include "canon_internal.h"

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

// A lane's value joined with that of its partner at distance 1, 2, 4, .. 32 in turn, so that every lane ends with the whole
// wavefront's (or, of fewer steps, its aligned set's).  The steps within 16 lanes are register moves between lanes (the
// partner at distance 4 and 8 may be any lane of the other half: those hold the same by then), the last two swap rows of
// 16 and halves; no LDS operation, whose latency a shuffle has each time.
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, true);
}
template <int N, class Join>
__device__ __forceinline__ void lanes_join(uint32_t (&x)[N], int lanes, Join join) {  // N values, a step of all at a time
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = join(x[i], lane_move<0xB1>(x[i]));   // lanes 1 0 3 2 of each four
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = join(x[i], lane_move<0x4E>(x[i]));   // lanes 2 3 0 1
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = join(x[i], lane_move<0x141>(x[i]));  // each eight mirrored
  if (lanes > 8) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = join(x[i], lane_move<0x140>(x[i]));  // each sixteen mirrored
  }
  if (lanes > 16) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const auto r = __builtin_amdgcn_permlane16_swap(x[i], x[i], false, false);
      x[i] = join(r[0], r[1]);
    }
  }
  if (lanes > 32) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const auto r = __builtin_amdgcn_permlane32_swap(x[i], x[i], false, false);
      x[i] = join(r[0], r[1]);
    }
  }
}
template <class Join>
__device__ __forceinline__ uint32_t lanes_join(uint32_t x, int lanes, Join join) {
  uint32_t v[1] = {x};
  lanes_join(v, lanes, join);
  return v[0];
}
// What a sum's padding adds: x + -0 is x for every x, +0 and -0 among them.  +0 would turn a -0 (a result below 2^-126 is
// flushed to the zero of its sign) into +0.
constexpr float kNoTerm = -0.0f;
// Algorithm 2 over 64 chunk partials, one per lane, of which those past the last chunk are kNoTerm: adding them is the
// pass-through rule.  The sum in every lane.
__device__ __forceinline__ float wave_total(float p) {
  return __uint_as_float(lanes_join(__float_as_uint(p), 64, [](uint32_t a, uint32_t b) {
    const float s = __uint_as_float(a) + __uint_as_float(b);
    return __float_as_uint(s);
  }));
}
__device__ __forceinline__ float wave_most(float m) {
  return __uint_as_float(lanes_join(__float_as_uint(m), 64, [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}

// Register-resident rows (cols <= 2048, or the part H of 2048 terms of a longer one): lane l holds terms
// 4l + 256q .. +3 of its row, read from memory once.  The chunk chains still run one per lane over an LDS transpose (rows
// of 36 floats: 16-byte stores and reads without bank conflicts; a wavefront's LDS operations complete in order).
constexpr int kRegQ = 8;  // 64 x 4 x 8 = 2048 terms
constexpr int64_t kRegCols = 64 * 4 * kRegQ;
template <int Q>
struct RowStage {  // of a row of up to 256 Q terms
  float t[8 * Q][36];
  __device__ __forceinline__ float4& vec(int chunk, int k) { return *reinterpret_cast<float4*>(&t[chunk][4 * k]); }
  __device__ __forceinline__ float chain(int chunk) {
    float p = 0.0f;
#pragma unroll
    for (int k = 0; k < kChunk / 4; ++k) {
      const float4 v = vec(chunk, k);
      p = p + v.x; p = p + v.y; p = p + v.z; p = p + v.w;
    }
    return p;
  }
  // vector `q` of lane `lane` of a part: terms 256 q + 4 lane .. +3
  __device__ __forceinline__ void put(int q, int lane, const float (&v)[4]) {
    vec(8 * q + (lane >> 3), lane & 7) = make_float4(v[0], v[1], v[2], v[3]);
  }
  // the places behind n terms in their last chunk hold no term (left out by a select in every step of the chain instead, a
  // norm of 20000 rows of 16 terms took 10.0 us, so 9.2; 8192 x 1001 kept 16.0 and 15.5)
  __device__ __forceinline__ void end(int n) {
    __builtin_amdgcn_wave_barrier();
    if ((n & (kChunk - 1)) != 0) {
      const int at = n + (threadIdx.x & 63);
      if (at < ((n + kChunk - 1) & ~(kChunk - 1))) t[at >> 5][at & 31] = kNoTerm;
    }
  }
  // the sum of the n terms put into it
  __device__ __forceinline__ float sum(int n) {
    const int lane = threadIdx.x & 63;
    end(n);
    __builtin_amdgcn_wave_barrier();
    return wave_total(lane * kChunk < n ? chain(lane) : kNoTerm);
  }
  // the sum of a row whose terms outside vectors q0 .. q1 - 1 are +0, like their chunks' partials, and have not been put;
  // of terms that are not below +0 (no sum of them is -0)
  __device__ __forceinline__ float span_sum(int q0, int q1) {
    const int lane = threadIdx.x & 63;
    __builtin_amdgcn_wave_barrier();
    return wave_total(lane >= 8 * q0 && lane < 8 * q1 ? chain(lane) : 0.0f);
  }
  // The partial of this lane's chunk of such a row of n terms of any sign, ended; none: +0, or kNoTerm behind the row's last
  // chunk.
  __device__ __forceinline__ float span_chain(int q0, int q1, int n, float none) {
    const int lane = threadIdx.x & 63, upto = (n + kChunk - 1) / kChunk;
    return lane >= 8 * q0 && lane < (8 * q1 < upto ? 8 * q1 : upto) ? chain(lane) : none;
  }
};
using RegStage = RowStage<kRegQ>;

template <int H = 0, int Q>
__device__ __forceinline__ float reg_row_sum(RegStage& st, const float (&e)[Q][4], int64_t n) {
  const int lane = threadIdx.x & 63;
  auto stage = [&](int q) __attribute__((always_inline)) { st.put(q, lane, e[H * kRegQ + q]); };
  // short rows leave out the vectors past their end (norm forward of 20000 rows of 16 terms 11.2 -> 9.9 us, now 9.2); with the
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
  return st.sum((int)n);
}

// a value that the compiler does not know to be the same as before: masks made from it are made again instead of being
// held in scalar registers from their first use to the next, which spills them
__device__ __forceinline__ int again(int x) {
  asm("" : "+s"(x));
  return x;
}

// ---- a part of a row in a wavefront's registers: up to 256 Q elements, lane l holding 256 q + 4 l .. +3 -----------------
// Elements from .. upto - 1 (and what shares a vector with the first of them) are loaded, +0 stands elsewhere.  Vectors that
// end at or before `upto` are moved whole; the one that it cuts (TAIL: it need not be a multiple of 4) belongs to one lane
// of one q and is moved by element beside the loop, so that the loop has a single condition per vector (with the cut
// vector's branches in every iteration the masks spilled: padded rows of 1001 keys 109 us, then 53).
template <bool TAIL, int Q>
__device__ __forceinline__ void part_load(int from, int upto, float (&v)[Q][4], const float* p) {
  const int at = 4 * (threadIdx.x & 63), first = from - 3;
  const unsigned whole = upto - 3 > first ? (unsigned)(upto - 3 - first) : 0u;  // places where a vector may begin
#pragma unroll
  for (int q = 0; q < Q; ++q) {
#pragma unroll
    for (int t = 0; t < 4; ++t) v[q][t] = 0.0f;
    if ((unsigned)(256 * q + at - first) < whole) ldf<4>(p + 256 * q + at, v[q]);
  }
  if (TAIL && upto > from && (upto & 3)) {
    const int base = upto & ~3;
    float c[3] = {0.0f, 0.0f, 0.0f};
    const int mine = at == (base & 255) ? base >> 8 : -1;  // the cut vector's q, in its lane
    if (mine >= 0) {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (base + t < upto) c[t] = p[base + t];
    }
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int t = 0; t < 3; ++t) v[q][t] = q == mine ? c[t] : v[q][t];
  }
}
// The same of bf16 elements, kept as they are stored, two to a word: half the registers while they wait.
template <bool TAIL, int Q>
__device__ __forceinline__ void part_load_bf16(int from, int upto, uint32_t (&v)[Q][2], const uint16_t* p) {
  const int at = 4 * (threadIdx.x & 63), first = from - 3;
  const unsigned whole = upto - 3 > first ? (unsigned)(upto - 3 - first) : 0u;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    v[q][0] = v[q][1] = 0u;
    if ((unsigned)(256 * q + at - first) < whole) {
      const H4 h = *reinterpret_cast<const H4*>(p + 256 * q + at);
      v[q][0] = h.x; v[q][1] = h.y;
    }
  }
  if (TAIL && upto > from && (upto & 3)) {
    const int base = upto & ~3;
    uint32_t c[2] = {0u, 0u};
    const int mine = at == (base & 255) ? base >> 8 : -1;
    if (mine >= 0) {
#pragma unroll
      for (int t = 0; t < 3; ++t)
        if (base + t < upto) c[t >> 1] |= (uint32_t)p[base + t] << (16 * (t & 1));
    }
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      v[q][0] = q == mine ? c[0] : v[q][0];
      v[q][1] = q == mine ? c[1] : v[q][1];
    }
  }
}
__device__ __forceinline__ void wide4(const uint32_t (&w)[2], float (&f)[4]) {
  f[0] = __uint_as_float(w[0] << 16); f[1] = __uint_as_float(w[0] & 0xFFFF0000u);
  f[2] = __uint_as_float(w[1] << 16); f[3] = __uint_as_float(w[1] & 0xFFFF0000u);
}
// value(q, o) makes vector q, store4(j, o) moves the one at element j, store1(j, o) an element
template <bool TAIL, int Q, class Value, class Store4, class Store1>
__device__ __forceinline__ void part_store(int n, Value value, Store4 store4, Store1 store1) {
  n = again(n);
  const int at = 4 * (threadIdx.x & 63);
  const int mine = TAIL && (n & 3) && n > 0 && at == (n & 252) ? n >> 8 : -1;
  float c[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (256 * q >= n) break;
    float o[4];
    value(q, o);
    if (256 * q + at + 4 <= n) store4(256 * q + at, o);
    if (TAIL) {
#pragma unroll
      for (int t = 0; t < 3; ++t) c[t] = q == mine ? o[t] : c[t];
    }
  }
  if (mine >= 0) {
#pragma unroll
    for (int t = 0; t < 3; ++t)
      if (t < (n & 3)) store1((n & ~3) + t, c[t]);
  }
}

// bf16 to fp32 where arithmetic follows at once, which reads a subnormal as zero by itself
__device__ __forceinline__ float bf16_wide(uint16_t h) { return __uint_as_float((uint32_t)h << 16); }
__device__ __forceinline__ void ldb_wide(const uint16_t* p, float (&f)[4]) {
  const H4 u = *reinterpret_cast<const H4*>(p);
  f[0] = __uint_as_float(u.x << 16); f[1] = __uint_as_float(u.x & 0xFFFF0000u);
  f[2] = __uint_as_float(u.y << 16); f[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
// results of arithmetic (never subnormal) to bf16
__device__ __forceinline__ void stb_arith(uint16_t* p, const float (&f)[4]) {
  *reinterpret_cast<H4*>(p) = H4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
}
__device__ __forceinline__ uint16_t bf16_arith(float f) { return (uint16_t)pack_bf16(f, 0.0f); }

// this wavefront's place in its workgroup, known to be the same for all its lanes
__device__ __forceinline__ int wave_id() { return __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)); }

// The R1 sum of a row of n terms spread over a workgroup of NW wavefronts, wavefront w holding its part from 2048 w on: 64
// chunks, a complete subtree of Algorithm 2 wherever a later part follows, so the parts' sums are folded by the same rule.
// slot: NW floats of LDS, not written again before every wavefront has passed another barrier (NW = 1: one wavefront per
// row, no barrier).
// join: every wavefront's own part's sum p into the row's
template <int NW>
__device__ __forceinline__ float wide_join(float p, int parts, float* slot) {
  if constexpr (NW == 1) {
    return p;
  } else {
    const int lane = threadIdx.x & 63;
    if (lane == 0) slot[wave_id()] = p;
    __syncthreads();
    return wave_total(lane < parts ? slot[lane] : kNoTerm);
  }
}
template <int NW, int Q>
__device__ __forceinline__ float wide_row_sum(RowStage<Q>& st, const float (&e)[Q][4], int n, float* slot) {
  const int lane = threadIdx.x & 63, left = again(NW == 1 ? n : n - wave_id() * 256 * Q);
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    if (256 * q >= left) break;
    st.put(q, lane, e[q]);
  }
  const float p = left > 0 ? st.sum(left < 256 * Q ? left : 256 * Q) : kNoTerm;
  return wide_join<NW>(p, (n + 256 * Q - 1) / (256 * Q), slot);
}

// How `rows` rows of n terms are held.  Rows of up to 512 and 1024 terms take fewer registers and less LDS, so that more
// of them are on the chip at once.  Where there are few rows, up to `per_cu` wavefronts of 8 vectors to a CU, a row of up to
// 8192 terms is spread over four times the wavefronts, each a quarter of the work: a norm of one row of 2048 takes 3.3 us
// instead of 5.6, of 1024 rows of 4096 8.8 instead of 10.9, 128 attention rows of 4096 keys 6.4 instead of 9.8; of 2048
// rows of 2048 a norm still 8.7 instead of 10.6, attention 13.5 instead of 11.6.
struct RowShape {
  int q, waves;  // vectors to a wavefront, and the wavefronts that a kernel is built for
  int used;      // wavefronts that a row needs
  int threads() const { return waves == 1 ? 256 : 64 * used; }
  int64_t groups(int64_t rows) const { return waves == 1 ? (rows + 3) / 4 : rows; }  // a wavefront's row or a workgroup's
};
inline RowShape row_shape(int64_t rows, int64_t n, int64_t per_cu) {
  auto parts = [&](int q) { return (int)((n + 256 * q - 1) / (256 * q)); };
  auto up = [](int x) {
    int p = 1;
    while (p < x) p <<= 1;
    return p;
  };
  if (n > 1024 && n <= 8192 && rows * parts(8) <= per_cu * device_cus()) return RowShape{2, up(parts(2)), parts(2)};
  if (n <= 1024) return RowShape{n <= 512 ? 2 : 4, 1, 1};
  return RowShape{8, up(parts(8)), parts(8)};
}
// K(q, waves) of a shape
#define CANON_ROW_SHAPES(K, shape)          \
  do {                                      \
    if ((shape).q == 2) {                   \
      switch ((shape).waves) {              \
        case 1: K(2, 1); break;             \
        case 4: K(2, 4); break;             \
        case 8: K(2, 8); break;             \
        default: K(2, 16); break;           \
      }                                     \
    } else if ((shape).q == 4) {            \
      K(4, 1);                              \
    } else {                                \
      switch ((shape).waves) {              \
        case 1: K(8, 1); break;             \
        case 2: K(8, 2); break;             \
        case 4: K(8, 4); break;             \
        case 8: K(8, 8); break;             \
        default: K(8, 16); break;           \
      }                                     \
    }                                       \
  } while (0)

}  // namespace canon
