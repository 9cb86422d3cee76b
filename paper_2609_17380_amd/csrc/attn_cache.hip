// attn_cache.hip - attention over the paged cache of keys and values in 8 bits (R26).
//
// Every long sum is a sum of products of whole numbers, so it runs on the int8 matrix instructions in any order: a query (and a
// weight times its value's step) is a whole number of 23 bits in three digits of 8, x = 256 (256 hi + mid) + lo, the sum over the
// first two of them exact in 32 bits and that over the third another.  Left to floating point are a maximum, a tile's 256
// exponentials and their tree, and one fused multiply-add per tile and element, with every change of reference a power of two.
//
// v_mfma_i32_16x16x64_i8 multiplies 16 rows by 16 columns over 64 k.  Lane (c, g) = (lane % 16, lane / 16) supplies bytes 16 g
// .. 16 g + 15 of row (column) c and receives rows 4 g .. 4 g + 3 of column c.  Keys are the rows of the score product, queries
// its columns: taking key 16 (row / 4) + 4 t + row % 4 of 64 for row `row` of instruction t, lane (c, g) receives the scores of
// keys 16 g + 4 t + i (t, i = 0 .. 3): the 16 consecutive keys that it has to supply, as weights, to the product with the values,
// whose rows are elements of a head (the cache keeps 16 tokens of an element together) and whose columns are the queries again.
// No lane ever needs another's weights, and a query's maxima and sums cross 4 lanes.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "dma_dev.h"
#include "rows_dev.h"

namespace canon {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int kTile = 256;                      // keys of a tile of the rule
constexpr float kNegInf = -__builtin_inff();

#define CANON_NAN4 __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")
__device__ const __attribute__((aligned(16))) float kNanSteps[16] = {CANON_NAN4, CANON_NAN4, CANON_NAN4, CANON_NAN4};
#undef CANON_NAN4

// 2^x, |x| <= 1/2: the polynomial of least relative error with the constant 1, its coefficients rounded: 9.4e-8, and 1.6e-7 with
// the roundings of its steps (with one term less 2.9e-6, which showed beside the rounding of the output).
constexpr uint32_t kExp2C[5] = {0x3F317215u, 0x3E75FCE1u, 0x3D635B6Cu, 0x3C1E7456u, 0x3AADED20u};

// The weight 2^x, x in [-127, 0].  n = rne(x) goes to the exponent by an integer addition; below 2^-126 a subnormal number comes
// of it, which everything that reads it takes for 0 (at -127, where all that is smaller is held, 0 itself).
constexpr float kExpShift = 12582912.0f;  // 1.5 2^23
__device__ __forceinline__ float weight(float x) {
  const float t = x + kExpShift, g = t - kExpShift;  // n in the low bits; n
  const float f = x - g;
  float p = __builtin_fmaf(__uint_as_float(kExp2C[4]), f, __uint_as_float(kExp2C[3]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[2]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[1]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[0]));
  p = __builtin_fmaf(p, f, 1.0f);
  return __uint_as_float(__float_as_uint(p) + (__float_as_uint(t) << 23));
}
// A tile's reference for one query: x = u f - r in one rounding.  Beyond 2^22 r's own rounding would show in it: the product is
// rounded as r's was there.
struct Ref {
  float r, f, ref;
  bool near;
  __device__ __forceinline__ Ref(float m, float f_) : f(f_) {
    const float mf = m * f;
    r = m == kNegInf ? m : __builtin_ceilf(mf);
    ref = r == kNegInf ? 0.0f : r;
    near = fabsf(ref) <= 4194304.0f;
  }
  static __device__ __forceinline__ float held(float x) { return __builtin_amdgcn_fmed3f(x, -127.0f, 0.0f); }
  __device__ __forceinline__ float x_near(float u) const { return held(__builtin_fmaf(u, f, -ref)); }
  __device__ __forceinline__ float x(float u) const {
    const float t = u * f, far = t - ref;
    return held(near ? __builtin_fmaf(u, f, -ref) : far);
  }
  // a tile's sum: 0 where no score is above -inf, NaN where one is NaN or +inf
  __device__ __forceinline__ float sum(float s) const {
    return r == kNegInf ? 0.0f : r < __builtin_inff() ? s : __builtin_nanf("");
  }
};

// Numbers are kept as multiples of 2^s, s the least that leaves the largest of them three digits, 127 (65536 + 256 + 1): its
// exponent less 22, or 21 where its significand is above theirs.  s + 149 for the largest number's bits:
__device__ __forceinline__ uint32_t three_digits(uint32_t top) { return (top + 65793u) >> 23; }
// What a tile's products of weight and value step are kept to (s >= -126: the smallest normal number).  A part of the largest
// *product*: of the largest value step alone, one key with a large value and no weight took the bits of all the others.
struct Whole {
  float up, down;  // 2^-s; 2^s, NaN where the largest is an infinity or a NaN
  __device__ __forceinline__ explicit Whole(uint32_t top) {
    const uint32_t at = three_digits(top), s149 = at > 23u ? at : 23u;
    up = __uint_as_float((276u - s149) << 23);
    down = top < 0x7F800000u ? __uint_as_float((s149 - 22u) << 23) : __builtin_nanf("");
  }
};

// 2^(a - b) of whole a <= b, 1 where a is -inf
__device__ __forceinline__ float shift2(float a, float b) {
  const float x = a - b;
  const float s = __uint_as_float((uint32_t)((int32_t)fmaxf(x, -127.0f) + 127) << 23);
  return a == kNegInf ? 1.0f : x == x ? (x < -126.0f ? 0.0f : s) : x;
}

__device__ __forceinline__ float max4(float m) {  // over the four lanes of a column
  m = __builtin_elementwise_maximum(m, __shfl_xor(m, 16, 64));
  return __builtin_elementwise_maximum(m, __shfl_xor(m, 32, 64));
}
__device__ __forceinline__ uint32_t umax4(uint32_t m) {
  uint32_t o = __shfl_xor(m, 16, 64);
  m = o > m ? o : m;
  o = __shfl_xor(m, 32, 64);
  return o > m ? o : m;
}
__device__ __forceinline__ float sum4(float s) {  // the tree over four chains
  s = s + __shfl_xor(s, 16, 64);
  return s + __shfl_xor(s, 32, 64);
}

__device__ __forceinline__ i32x4 mfma(const i32x4& a, const i32x4& b, const i32x4& c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// A query of the block's 16 columns: its row and the keys [lo, hi) that it sees.
struct Column {
  int64_t row;  // of q and out, in heads: (b q_len + i) heads + h
  int64_t tok, lo, hi;
  int32_t h;
  bool real;
};
__device__ __forceinline__ Column column_of(const CacheAttnArgs& a, int64_t b, int32_t kvh, int64_t idx) {
  Column c;
  const uint32_t G = (uint32_t)(a.heads / a.c.heads), iq = (uint32_t)idx / G;  // rows of a call: below 2^24
  const int64_t i = iq;
  c.h = kvh * (int32_t)G + (int32_t)((uint32_t)idx - iq * G);
  c.real = i < a.q_len;
  c.tok = b * a.q_len + i;
  c.row = c.tok * a.heads + c.h;
  const int64_t pos = (a.q_starts ? a.q_starts[b] : a.q_start) + i;
  int64_t hi = a.k_len, lo = 0;
  if (a.k_lens) hi = a.k_lens[b] < hi ? a.k_lens[b] : hi;
  if (a.causal) hi = pos + 1 < hi ? pos + 1 : hi;
  if (a.window) {
    hi = pos + a.window < hi ? pos + a.window : hi;
    lo = pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
  }
  if (!c.real || (a.q_lens && i >= a.q_lens[b]) || hi < lo) lo = hi = 0;
  c.lo = lo;
  c.hi = hi < 0 ? 0 : hi;
  if (c.lo >= c.hi) c.lo = c.hi = 0;
  return c;
}
// the first tile that one of a block of 16 columns sees, one behind all if none does
__device__ __forceinline__ int64_t first_tile(const CacheAttnArgs& a, int64_t b, int32_t kvh, int64_t block) {
  const Column c = column_of(a, b, kvh, block * 16 + (threadIdx.x & 15));
  int32_t lo = c.hi > c.lo ? (int32_t)c.lo : 0x7FFFFFFF;
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    const int32_t l = __shfl_xor(lo, s, 64);
    lo = l < lo ? l : lo;
  }
  return __builtin_amdgcn_readfirstlane(lo) / kTile;
}
// which of a tile's keys a column sees: those from lo on, n of them
struct Seen {
  int32_t lo, n;
  __device__ __forceinline__ bool key(int32_t at) const { return (uint32_t)(at - lo) < (uint32_t)n; }
};
__device__ __forceinline__ Seen seen_of(const Column& c, int64_t t0) {
  const int64_t lo = c.lo > t0 ? c.lo - t0 : 0, hi = c.hi - t0;
  const int32_t l = lo < kTile ? (int32_t)lo : kTile, h = hi < 0 ? 0 : hi < kTile ? (int32_t)hi : kTile;
  return Seen{l, h > l ? h - l : 0};
}

// the 16 keys from j on (a multiple of 16): their first slot in head kvh, or -1
__device__ __forceinline__ int64_t slot16(const CacheAttnArgs& a, int32_t kvh, int64_t j, int32_t page) {
  if (page < 0 || page >= a.c.n_pages) return -1;
  return (((int64_t)page * a.c.heads + kvh) << a.c.lg) + (j & ((1 << a.c.lg) - 1));
}
__device__ __forceinline__ int32_t page_of(const CacheAttnArgs& a, int64_t b, int64_t j) {
  return j < a.k_len ? a.c.table[b * a.c.table_len + (j >> a.c.lg)] : -1;
}

// a sum of products, from the sums over the first two digits and over the last
__device__ __forceinline__ float whole_sum(int32_t hi, int32_t lo) { return __builtin_fmaf((float)hi, 256.0f, (float)lo); }

__device__ __forceinline__ i32x4 load16(const int8_t* p) { return *reinterpret_cast<const i32x4*>(p); }

// The queries of a block: lane (c, g) has elements 64 s + 16 g .. + 15 of column c, first as they are stored (asked for early),
// then as digits with the column's f.
struct __attribute__((packed, aligned(2))) U16x8 {
  uint32_t w[4];
};
template <int HD>
struct RawQuery {
  static constexpr int NS = (HD + 63) / 64;
  uint32_t w[NS][16];
};
template <int HD>
struct Query {
  static constexpr int NS = (HD + 63) / 64;
  i32x4 hi[NS], mid[NS], lo[NS];
  float f;
};
template <int HD>
__device__ __forceinline__ void ask_query(const CacheAttnArgs& a, const Column& c, RawQuery<HD>& r) {
  const int g = (threadIdx.x & 63) >> 4;
  const int64_t at = c.real ? c.tok * a.q_stride + (int64_t)c.h * HD : 0;  // an unreal column: the first row, unused
#pragma unroll
  for (int s = 0; s < RawQuery<HD>::NS; ++s) {
    const int d = HD % 64 == 0 || 64 * s + 16 * g < HD ? 64 * s + 16 * g : 0;
    const char* p = (const char*)a.q + (at + d) * (a.q_bf16 ? 2 : 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= 2 && a.q_bf16) break;
      const U16x8 x = reinterpret_cast<const U16x8*>(p)[i];
#pragma unroll
      for (int e = 0; e < 4; ++e) r.w[s][4 * i + e] = x.w[e];
    }
  }
}
template <int HD>
__device__ __forceinline__ void make_query(const CacheAttnArgs& a, const Column& c, const RawQuery<HD>& r, Query<HD>& out) {
  constexpr int NS = Query<HD>::NS;
  const int g = (threadIdx.x & 63) >> 4;
  float v[NS][16];
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const bool has = c.real && (HD % 64 == 0 || 64 * s + 16 * g < HD);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t half = e & 1 ? r.w[s][e >> 1] & 0xFFFF0000u : r.w[s][e >> 1] << 16;
      v[s][e] = has ? __uint_as_float(a.q_bf16 ? half : r.w[s][e]) : 0.0f;
      const uint32_t u = __float_as_uint(v[s][e]) & 0x7FFFFFFFu;
      top = u > top ? u : top;
    }
  }
  top = umax4(top);
  // Whole numbers of three digits: bf16 elements down to 2^-14 of the largest come as they are (with 16 bits, a channel 1000
  // times the others left these six, and outputs off by 2%).  2^-s and 2^s in two factors each, as their exponents leave the
  // range of one; a product with them rounds at most to zero.
  const int s = (int)three_digits(top) - 149, h = s >> 1;
  const bool zero = top < 0x00800000u, finite = !zero && top < 0x7F800000u;
  auto pow2 = [](int e) { return __uint_as_float((uint32_t)(e + 127) << 23); };
  const float up = pow2(-h), up2 = a.scale < 0.0f ? -pow2(h - s) : pow2(h - s);
#pragma unroll
  for (int q = 0; q < NS; ++q)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t d0 = 0, d1 = 0, d2 = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = v[q][4 * w + e] * up;
        const int32_t n = (int32_t)__builtin_rintf(finite ? x * up2 : 0.0f);
        d0 |= (uint32_t)(n & 0xFF) << (8 * e);  // n = 65536 d2 + 256 d1 + d0, the last two in [-128, 127]
        d1 |= (uint32_t)(((n + 128) >> 8) & 0xFF) << (8 * e);
        d2 |= (uint32_t)(((n + 32896) >> 16) & 0xFF) << (8 * e);
      }
      out.hi[q][w] = (int32_t)d2;
      out.mid[q][w] = (int32_t)d1;
      out.lo[q][w] = (int32_t)d0;
    }
  const float sc = fabsf(a.scale) * kLog2e, part = sc * pow2(h), f = part * pow2(s - h);
  out.f = zero ? 0.0f : finite ? f : __builtin_nanf("");
}

// Four products as whole numbers of 2^s, 0 .. 8355711, into a dword of each digit.  Adding 2^23 + 32768 + 128 rounds to a whole
// number and leaves w + 32896 in the low bits: byte 2 is the high digit, bytes 1 and 0 the others with their sign bits inverted.
constexpr float kWhole = 8421504.0f;
__device__ __forceinline__ void digits4(const float (&p)[4], float up, int32_t& hi, int32_t& mid, int32_t& lo) {
  const uint32_t a = __float_as_uint(__builtin_fmaf(p[0], up, kWhole)), b = __float_as_uint(__builtin_fmaf(p[1], up, kWhole));
  const uint32_t c = __float_as_uint(__builtin_fmaf(p[2], up, kWhole)), d = __float_as_uint(__builtin_fmaf(p[3], up, kWhole));
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
  const uint32_t cd = __builtin_amdgcn_perm(d, c, 0x05010400u);
  lo = (int32_t)(__builtin_amdgcn_perm(cd, ab, 0x05040100u) ^ 0x80808080u);
  mid = (int32_t)(__builtin_amdgcn_perm(cd, ab, 0x07060302u) ^ 0x80808080u);
  const uint32_t ab2 = __builtin_amdgcn_perm(b, a, 0x0C0C0602u), cd2 = __builtin_amdgcn_perm(d, c, 0x06020C0Cu);  // a2 b2 0 0; 0 0 c2 d2
  hi = (int32_t)(ab2 | cd2);
}

__device__ __forceinline__ void store_out(const CacheAttnArgs& a, int64_t row, int d, float inv, const f32x4& o, int hd) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float x = o[i] + 0.0f;
    f[i] = x * inv;
  }
  *reinterpret_cast<H4*>(a.out + row * hd + d) = H4{pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3])};
}

}  // namespace

// ---- one tile of keys a workgroup: few queries, many keys ---------------------------------------------------------------
//
// Four wavefronts, each with 64 of the tile's 256 keys in the score product and a quarter of the head's elements in the product
// with the values (the weights cross through LDS, 12 KB): a workgroup has all of its 2 * 256 * head_dim bytes of the cache on
// their way at once and waits for them once.  What a tile gives goes to `parts`, a row's tiles one after the other, to be
// joined by attn_join_kernel; where there is one tile only, straight to the output.
// With a window, `span` workgroups (and places in `parts`) a block of queries, from the first tile that one of them sees on (of
// all tiles, 12 of 257 queries behind 2744 keys, most workgroups had nothing to do).
// Bound by memory where there is enough of it: 4 x 16 heads x 32768 keys of 128, 554 MB, 112 us, 4.9 TB/s; 8 x 2 heads of up to
// 4096 keys 8 us, the latencies of table entry, codes and join in a row.
template <int HD>
__global__ __launch_bounds__(256) void attn_tile_kernel(CacheAttnArgs a, int64_t tiles, int64_t blocks, int64_t span) {
  constexpr int NS = Query<HD>::NS, ND = HD / 16, NW = (ND + 3) / 4;  // 16-element parts of a head, of a wavefront
  __shared__ __attribute__((aligned(16))) i32x4 wts[3][4][64];
  __shared__ float ms[4][16], ss[4][16];
  __shared__ uint32_t vs[4][16];
  const uint32_t id = blockIdx.x, bt = id / (uint32_t)span, bk = bt / (uint32_t)blocks;
  const int64_t place = id - bt * (uint32_t)span;
  const int64_t cb = bt - bk * (uint32_t)blocks;
  const int64_t b = bk / (uint32_t)a.c.heads;
  const int32_t kvh = (int32_t)(bk - (uint32_t)b * (uint32_t)a.c.heads);
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cc = lane & 15, g = lane >> 4;
  const int at0 = 64 * w + 16 * g;  // of this lane's 16 keys in the tile
  const int64_t tile = place + (span < tiles ? first_tile(a, b, kvh, cb) : 0);
  if (tile >= tiles) return;
  const int64_t t0 = tile * kTile;
  // which pages, and the queries: asked for before anything is waited for
  const int32_t kpage = page_of(a, b, t0 + 64 * w + 16 * (cc >> 2));
  int32_t vpage[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) vpage[q] = page_of(a, b, t0 + 64 * q + 16 * g);
  const Column col = column_of(a, b, kvh, cb * 16 + cc);
  RawQuery<HD> raw;
  ask_query<HD>(a, col, raw);
  const Seen sees = seen_of(col, t0);
  if (tiles > 1 && !__any(sees.n > 0)) return;  // the join passes over tiles that a row does not see

  // The cache, all at once.  Slots that it does not have: any of its codes (their weights are 0, or their steps NaN).
  int64_t kslot = slot16(a, kvh, t0 + 64 * w + 16 * (cc >> 2), kpage), vslot[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) vslot[q] = slot16(a, kvh, t0 + 64 * q + 16 * g, vpage[q]);
  const int64_t gslot = w == 0 ? vslot[0] : w == 1 ? vslot[1] : w == 2 ? vslot[2] : vslot[3];
  kslot = kslot < 0 ? 0 : kslot;
  i32x4 kx[4][NS], vx[NW][4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int s = 0; s < NS; ++s)  // elements behind a head of 32 (mod 64): its first ones, which meet digits of 0
      kx[t][s] = load16(a.c.kc + (kslot + 4 * t + (cc & 3)) * HD + (HD % 64 == 0 || 64 * s + 16 * g < HD ? 64 * s + 16 * g : 0));
  typedef const __attribute__((address_space(1))) f32x4* GlobalVec;  // or the choice between the two arrays makes flat loads
  const GlobalVec kp = (GlobalVec)(uintptr_t)(gslot < 0 ? kNanSteps : a.c.ks + gslot);
  const GlobalVec vp = (GlobalVec)(uintptr_t)(gslot < 0 ? kNanSteps : a.c.vs + gslot);
  f32x4 kst[4], vst[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    kst[t] = kp[t];
    vst[t] = vp[t];
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int8_t* p = a.c.vc + (vslot[q] < 0 ? 0 : vslot[q]) * HD + 16 * cc;
#pragma unroll
    for (int n = 0; n < NW; ++n) vx[n][q] = load16(p + 256 * (ND % 4 == 0 || w + 4 * n < ND ? w + 4 * n : 0));
  }
  // the loads stay before the queries' divisions (left to itself, the compiler asked for keys and values when they were used)
  __builtin_amdgcn_sched_barrier(0);
  Query<HD> qd;
  make_query<HD>(a, col, raw, qd);

  float t[4][4];
  float m = kNegInf;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < NS; ++s) acc = mfma(kx[k][s], qd.hi[s], acc);
    acc = acc << 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) acc = mfma(kx[k][s], qd.mid[s], acc);
    i32x4 low = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < NS; ++s) low = mfma(kx[k][s], qd.lo[s], low);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool seen = sees.key(at0 + 4 * k + i);
      t[k][i] = seen ? whole_sum(acc[i], low[i]) * kst[k][i] : kNegInf;
      m = __builtin_elementwise_maximum(m, t[k][i]);
    }
  }
  m = max4(m);
  if (g == 0) ms[w][cc] = m;
  __syncthreads();
#pragma unroll
  for (int o = 0; o < 4; ++o) m = __builtin_elementwise_maximum(m, ms[o][cc]);
  const Ref rf(m, qd.f);
  float sum = 0.0f;
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool seen = sees.key(at0 + 4 * k + i);
      float e = weight(rf.x(t[k][i])), p = e * vst[k][i];
      e = seen ? e : 0.0f;
      p = seen ? p : 0.0f;
      sum = sum + e;
      t[k][i] = p;
      const uint32_t u = __float_as_uint(p);  // never negative
      top = u > top ? u : top;
    }
  top = umax4(top);
  sum = sum4(sum);
  if (g == 0) {
    vs[w][cc] = top;
    ss[w][cc] = sum;
  }
  __syncthreads();
#pragma unroll
  for (int o = 0; o < 4; ++o) top = vs[o][cc] > top ? vs[o][cc] : top;
  const Whole whole(top);
  i32x4 wh, wm, wl;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    int32_t h, d, l;
    digits4(t[k], whole.up, h, d, l);
    wh[k] = h;
    wm[k] = d;
    wl[k] = l;
  }
  wts[0][w][lane] = wh;
  wts[1][w][lane] = wm;
  wts[2][w][lane] = wl;
  __syncthreads();
  const float S = rf.sum((ss[0][cc] + ss[1][cc]) + (ss[2][cc] + ss[3][cc]));
  const float inv = S == 0.0f ? 0.0f : 1.0f / S;
  float* parts = a.parts + (col.row * span + place) * (HD + 4);
  if (tiles > 1 && col.real && w == 0 && g == 0)
    *reinterpret_cast<f32x4*>(parts + HD) = f32x4{rf.r, S, whole.down, 0.0f};
#pragma unroll
  for (int n = 0; n < NW; ++n) {
    const int part = w + 4 * n;
    if (ND % 4 != 0 && part >= ND) break;
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = mfma(vx[n][q], wts[0][q][lane], acc);
    acc = acc << 8;
#pragma unroll
    for (int q = 0; q < 4; ++q) acc = mfma(vx[n][q], wts[1][q][lane], acc);
    i32x4 low = {0, 0, 0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) low = mfma(vx[n][q], wts[2][q][lane], low);
    if (!col.real) continue;
    f32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = whole_sum(acc[i], low[i]);
    if (tiles > 1) {
      *reinterpret_cast<f32x4*>(parts + 16 * part + 4 * g) = o;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = S == 0.0f ? 0.0f : o[i] * whole.down;
      store_out(a, col.row, 16 * part + 4 * g, inv, o, HD);
    }
  }
}

// A row's tiles joined, ascending: one wavefront a row, E elements a lane.  What the references change by is worked out for 64
// tiles at once, a tile a lane (the largest reference up to a tile is a prefix maximum), so that the chain over the tiles is two
// operations an element; and 16 tiles' sums are on their way together.  (One tile after the other, each waited for: a row of 128
// tiles took 156 us, so 13; of 16 16, so 4.)
template <int HD>
__global__ __launch_bounds__(64) void attn_join_kernel(CacheAttnArgs a, int64_t tiles, int64_t span) {
  constexpr int E = HD > 128 ? 4 : 2, U = 16;
  typedef float Vec __attribute__((ext_vector_type(E)));
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x, at = lane * E < HD ? lane * E : 0;
  const int64_t tok = (uint32_t)row / (uint32_t)a.heads, b = (uint32_t)tok / (uint32_t)a.q_len;  // rows of a call: below 2^24
  const int32_t G = a.heads / a.c.heads, h = (int32_t)(row - tok * a.heads);
  const int64_t idx = (tok - b * a.q_len) * G + h % G, base = span < tiles ? first_tile(a, b, h / G, idx / 16) : 0;
  const Column col = column_of(a, b, h / G, idx);
  const float* parts = a.parts + row * span * (HD + 4);
  float R = kNegInf, S = 0.0f;
  Vec o;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  const int64_t first = col.lo / kTile, end = col.hi > col.lo ? (col.hi + kTile - 1) / kTile : first;
  for (int64_t c0 = first; c0 < end; c0 += 64) {
    const int n = end - c0 < 64 ? (int)(end - c0) : 64;
    const float* p = parts + (c0 - base) * (HD + 4);
    const f32x4 d = *reinterpret_cast<const f32x4*>(p + (lane < n ? lane : n - 1) * (HD + 4) + HD);
    // R of the rule before and after this lane's tile
    float up = d[0];
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
      const float x = __shfl_up(up, s, 64);
      up = lane >= s ? __builtin_elementwise_maximum(up, x) : up;
    }
    const float after = __builtin_elementwise_maximum(R, up), left = __shfl_up(after, 1, 64), before = lane == 0 ? R : left;
    const float x = shift2(before, after), y = shift2(d[0], after), sy = d[1], sc = d[2];
    Vec v[U], ahead[U];
    auto ask = [&](int t0) {
#pragma unroll
      for (int u = 0; u < U; ++u) ahead[u] = *reinterpret_cast<const Vec*>(p + (t0 + u < n ? t0 + u : n - 1) * (HD + 4) + at);
    };
    ask(0);
    for (int t0 = 0; t0 < n; t0 += U) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ahead[u];
      if (t0 + U < n) ask(t0 + U);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int t = t0 + u < n ? t0 + u : n - 1;
        if (t0 + u >= n) continue;
        auto of = [&](float f) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), t)); };
        const float xt = of(x), yt = of(y), st = of(sc);
        S = __builtin_fmaf(of(sy), yt, S * xt);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = __builtin_fmaf(v[u][e] * yt, st, o[e] * xt);
      }
    }
    R = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(after), n - 1));
  }
  if (lane * E >= HD) return;
  const float inv = S == 0.0f ? 0.0f : 1.0f / S;
#pragma unroll
  for (int e = 0; e < E; e += 2) {
    const float f0 = o[e] + 0.0f, f1 = o[e + 1] + 0.0f;
    struct __attribute__((packed, aligned(2))) H2 { uint32_t x; };
    reinterpret_cast<H2*>(a.out + row * HD + at + e)->x = S == 0.0f ? 0u : pack_bf16(f0 * inv, f1 * inv);
  }
}

// ---- all keys of a block of queries in one workgroup: prompts -------------------------------------------------------------
//
// Four wavefronts of 16 queries each go over the tiles together.  A tile's keys and values come straight into LDS in the order
// in which the matrix instructions take them (each 1 KB block is one instruction's operand, lane l's bytes at 16 l, so that
// reading has no bank conflicts and no address is computed per lane), a wavefront fetching its quarter of the tile: the next
// tile's keys while the present one's weights are computed, its values while the next scores are.  Two workgroups a CU (heads
// of up to 128) run out of step, one's products under the other's exponentials.
// Bound by its vector instructions: 16 heads x 4096 x 128 152 us in a graph, 32 of them for each 64 visible scores, 85% of a
// SIMD's cycles issuing one; the third digits of queries and weights and the exponential's last term are a fifth of them.
// Registers: heads of 128 leave 12 a lane in scratch, of 96 3, of 224 18 and of 256 26, addresses for the most part.
template <int HD>
struct RowsLds {
  static constexpr int NS = Query<HD>::NS, ND = HD / 16;
  i32x4 k[16 * NS][64];  // block (4 q + t) NS + s: 64 q keys on, instruction t, elements 64 s on
  i32x4 v[4 * ND][64];   // block q ND + n
  float ks[2][kTile], vs[2][kTile];
  int32_t span[4][2];     // tiles of the wavefronts
};

template <int HD>
__global__ __launch_bounds__(256, HD <= 128 ? 2 : 1) void attn_rows_kernel(CacheAttnArgs a, int64_t blocks) {
  constexpr int NS = Query<HD>::NS, ND = HD / 16;
  typedef const __attribute__((address_space(4))) int32_t* ConstInts;  // the table through the scalar cache
  __shared__ __attribute__((aligned(1024))) RowsLds<HD> L;
  // workgroups of one head of a sequence on one XCD where their number allows it, the longest causal rows first
  const uint32_t n_bh = (uint32_t)(a.c.heads * a.c.batch), turn = blockIdx.x / n_bh, bh = blockIdx.x - turn * n_bh;
  const int64_t cb = blocks - 1 - turn, b = bh / (uint32_t)a.c.heads;
  const int32_t kvh = (int32_t)(bh - (uint32_t)b * (uint32_t)a.c.heads);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), cc = lane & 15, g = lane >> 4;
  const Column col = column_of(a, b, kvh, (cb * 4 + w) * 16 + cc);
  // keys that some query of the wavefront sees, and that all of them see (k_len fits 32 bits)
  int32_t lo = col.hi > col.lo ? (int32_t)col.lo : 0x7FFFFFFF, hi = (int32_t)col.hi;
  int32_t in_lo = col.real ? (int32_t)col.lo : 0, in_hi = col.real ? (int32_t)col.hi : 0x7FFFFFFF;
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    const int32_t l = __shfl_xor(lo, s, 64), h = __shfl_xor(hi, s, 64), il = __shfl_xor(in_lo, s, 64), ih = __shfl_xor(in_hi, s, 64);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
    in_lo = il > in_lo ? il : in_lo;
    in_hi = ih < in_hi ? ih : in_hi;
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  hi = __builtin_amdgcn_readfirstlane(hi);
  in_lo = __builtin_amdgcn_readfirstlane(in_lo);
  in_hi = lo < hi ? __builtin_amdgcn_readfirstlane(in_hi) : 0;  // a wavefront without queries: no whole tiles
  if (lane == 0) {
    L.span[w][0] = lo;
    L.span[w][1] = hi;
  }
  Query<HD> qd;
  {
    RawQuery<HD> raw;
    ask_query<HD>(a, col, raw);
    make_query<HD>(a, col, raw, qd);
  }
  __syncthreads();
  int32_t all_lo = 0x7FFFFFFF, all_hi = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    all_lo = L.span[i][0] < all_lo ? L.span[i][0] : all_lo;
    all_hi = L.span[i][1] > all_hi ? L.span[i][1] : all_hi;
  }
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);

  const unsigned lk = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)&L.k[0][0];
  const unsigned lv = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)&L.v[0][0];
  const unsigned lks = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)&L.ks[0][0];
  const unsigned lvs = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)&L.vs[0][0];
  const ConstInts table = (ConstInts)(uintptr_t)(a.c.table + b * a.c.table_len);
  // the first slots of the four groups of 16 keys of this wavefront's quarter of a tile, -1 where there is none
  auto group_slots = [&](int32_t t0, int64_t (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int32_t j = t0 + 64 * w + 16 * i;
      s[i] = j < (int32_t)a.k_len ? slot16(a, kvh, j, table[j >> a.c.lg]) : -1;
      asm volatile("" : "+s"(s[i]));  // in scalar registers, for the picks below to be selections
    }
  };
  auto pick = [](const int64_t (&s)[4], int i) { return i == 0 ? s[0] : i == 1 ? s[1] : i == 2 ? s[2] : s[3]; };
  // Slots that the cache does not have: any of its codes (their weights are 0, or the step NaN), the step NaN.
  auto fetch_keys = [&](const int64_t (&s)[4], int par) {
    int64_t ks = pick(s, cc >> 2);
    const int64_t gs = pick(s, g);
    ks = ks < 0 ? 0 : ks;
    const int8_t* p = a.c.kc + (ks + (cc & 3)) * HD;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int e = 0; e < NS; ++e)  // elements behind a head of 32 (mod 64): its first ones, which meet digits of 0
        dma16(p + 4 * t * HD + (HD % 64 == 0 || 64 * e + 16 * g < HD ? 64 * e + 16 * g : 0), lk + 1024 * ((4 * w + t) * NS + e));
    dma4(gs < 0 ? kNanSteps : a.c.ks + gs + cc, lks + 1024 * par + 256 * w);
    dma4(gs < 0 ? kNanSteps : a.c.vs + gs + cc, lvs + 1024 * par + 256 * w);
  };
  auto fetch_values = [&](const int64_t (&s)[4]) {
    int64_t vs = pick(s, g);
    vs = vs < 0 ? 0 : vs;
    const int8_t* p = a.c.vc + vs * HD + 16 * cc;
#pragma unroll
    for (int n = 0; n < ND; ++n) dma16(p + 256 * n, lv + 1024 * (w * ND + n));
  };

  float R = kNegInf, S = 0.0f;
  f32x4 o[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  int64_t slots[4];
  int32_t t0 = all_lo < all_hi ? all_lo / kTile * kTile : all_hi;
  int par = 0;
  if (t0 < all_hi) {
    group_slots(t0, slots);
    fetch_keys(slots, 0);
  }
  // One tile.  FULL: every query of the wavefront sees all of it, so that nothing is masked.
  auto tile = [&](auto full, bool mine, const Seen& sees) {
    constexpr bool FULL = full.value;
    // quarters of the tile that some query of this wavefront sees
    const int q0 = FULL || lo <= t0 ? 0 : (lo - t0) >> 6;
    const int q1 = FULL ? 4 : !mine ? 0 : hi - t0 < kTile ? (hi - t0 + 63) >> 6 : 4;
    float u[4][4][4];
    float m = kNegInf;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (FULL || (q >= q0 && q < q1)) {
        i32x4 acc[4], low[4], kx[4][NS];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = low[t] = i32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int t = 0; t < 4; ++t) kx[t][s] = L.k[(4 * q + t) * NS + s][lane];
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[t] = mfma(kx[t][s], qd.hi[s], acc[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = acc[t] << 8;
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int t = 0; t < 4; ++t) low[t] = mfma(kx[t][s], qd.lo[s], low[t]);
#pragma unroll
        for (int s = 0; s < NS; ++s)
#pragma unroll
          for (int t = 0; t < 4; ++t) acc[t] = mfma(kx[t][s], qd.mid[s], acc[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f32x4 st = *reinterpret_cast<const f32x4*>(&L.ks[par][64 * q + 16 * g + 4 * t]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            u[q][t][i] = whole_sum(acc[t][i], low[t][i]) * st[i];
            if (!FULL) u[q][t][i] = sees.key(64 * q + 16 * g + 4 * t + i) ? u[q][t][i] : kNegInf;
            m = __builtin_elementwise_maximum(m, u[q][t][i]);
          }
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) u[q][t][i] = kNegInf;
      }
    }
    __builtin_amdgcn_s_setprio(0);
    // every wavefront is done with the keys: the next tile's
    __syncthreads();
    const bool more = t0 + kTile < all_hi;
    if (more) {
      group_slots(t0 + kTile, slots);
      fetch_keys(slots, par ^ 1);
    }
    m = max4(m);
    const Ref rf(m, qd.f);
    const float r = rf.r;
    // weights, and their products with the values' steps in the scores' places
    float sums[4];
    uint32_t top = 0;
    auto weigh = [&](auto is_near) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        sums[q] = 0.0f;
        if (!FULL && (q < q0 || q >= q1)) {
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) u[q][t][i] = 0.0f;
          continue;
        }
        float sum = 0.0f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f32x4 vst = *reinterpret_cast<const f32x4*>(&L.vs[par][64 * q + 16 * g + 4 * t]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const bool seen = FULL || sees.key(64 * q + 16 * g + 4 * t + i);
            float e = weight(is_near.value ? rf.x_near(u[q][t][i]) : rf.x(u[q][t][i])), p = e * vst[i];
            e = seen ? e : 0.0f;
            p = seen ? p : 0.0f;
            sum = sum + e;
            u[q][t][i] = p;
            const uint32_t x = __float_as_uint(p);  // never negative
            top = x > top ? x : top;
          }
        }
        sums[q] = sum4(sum);
        // one quarter's steps in registers at a time (all four's: 45 registers in scratch, 16 heads x 4096 160 us instead of 142, with queries of two digits)
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (__all(rf.near)) weigh(std::true_type{});
    else weigh(std::false_type{});
    const Whole whole(umax4(top));
    i32x4 wh[4], wm[4], wl[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        int32_t h, d, l;
        digits4(u[q][t], whole.up, h, d, l);
        wh[q][t] = h;
        wm[q][t] = d;
        wl[q][t] = l;
      }
    const float Sb = rf.sum((sums[0] + sums[1]) + (sums[2] + sums[3]));
    const float Rn = __builtin_elementwise_maximum(R, r), x = shift2(R, Rn), y = shift2(r, Rn);
    // A column that sees nothing of the tile has S_b = 0 and A = 0 and keeps R: the steps below leave its row as it is (but for
    // the sign of a zero, which the output's + 0 takes away).
    S = __builtin_fmaf(Sb, y, S * x);
    R = Rn;
    const bool still = __all(x == 1.0f);
    // the values have landed (what was asked for after them, the next keys, may not have)
    if (more) vm_left<4 * NS + 2>();
    else vm_left<0>();
    __syncthreads();
    if (!FULL && !mine) return;
    if (!still) {
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = o[n][i] * x;
    }
    __builtin_amdgcn_s_setprio(1);
    constexpr int C = 2;  // chains of products side by side
#pragma unroll
    for (int n = 0; n < ND; n += C) {
      i32x4 acc[C], low[C], vx[C][4];
#pragma unroll
      for (int d = 0; d < C; ++d) acc[d] = low[d] = i32x4{0, 0, 0, 0};
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int d = 0; d < C; ++d) vx[d][q] = L.v[q * ND + n + d][lane];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int d = 0; d < C; ++d) acc[d] = mfma(vx[d][q], wh[q], acc[d]);
#pragma unroll
      for (int d = 0; d < C; ++d) acc[d] = acc[d] << 8;
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int d = 0; d < C; ++d) low[d] = mfma(vx[d][q], wl[q], low[d]);
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int d = 0; d < C; ++d) acc[d] = mfma(vx[d][q], wm[q], acc[d]);
#pragma unroll
      for (int d = 0; d < C; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = whole_sum(acc[d][i], low[d][i]) * y;  // y 2^s may be subnormal where this times 2^s is not
          o[n + d][i] = __builtin_fmaf(s, whole.down, o[n + d][i]);
        }
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // runs of whole tiles and of others in loops of their own, which keep their registers where they are from tile to tile
  auto run = [&](auto full) {
    while (t0 < all_hi && (t0 >= in_lo && t0 + kTile <= in_hi) == full.value) {
      // this tile's keys have landed, and every wavefront is done with the last one's values
      vm_left<0>();
      __syncthreads();
      fetch_values(slots);
      tile(full, lo < t0 + kTile && hi > t0, seen_of(col, t0));
      t0 += kTile;
      par ^= 1;
    }
  };
  while (t0 < all_hi) {
    run(std::false_type{});
    run(std::true_type{});
  }
  if (!col.real) return;
  const float inv = S == 0.0f ? 0.0f : 1.0f / S;
#pragma unroll
  for (int n = 0; n < ND; ++n) {
    if (S == 0.0f) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    store_out(a, col.row, 16 * n + 4 * g, inv, o[n], HD);
  }
}

// ---- which of them --------------------------------------------------------------------------------------------------------

namespace {
struct Plan {
  int64_t tiles, span;  // of all keys; that the keys of a block's queries can lie in: those of one query, and the others' positions
  bool split;
};
Plan plan_of(const CacheAttnArgs& a) {
  const int64_t G = a.heads / a.c.heads, cols = a.q_len * G, tiles = (a.k_len + kTile - 1) / kTile;
  int64_t span = tiles;
  if (a.window > 0) {
    const int64_t keys = (a.causal ? a.window : 2 * a.window - 1) + 15 / G + 1;
    span = keys / kTile + 2 < tiles ? keys / kTile + 2 : tiles;
  }
  // A workgroup for every tile where those for 64 queries would be few (2 heads of 8 over 2048 keys: 64 of them 38 us, 55 in
  // whole rows; 128 of them 63 and 55; of one tile, 192 of them 12.8 and 14.1, 256 16.5 and 14.5), or would have at most two
  // wavefronts with queries (8 x 8 heads x 48 of 4000 50 and 102); launches stay below 2^32 threads.
  const int64_t groups = a.c.batch * a.c.heads, wgs = groups * ((cols + 63) / 64);
  const int64_t split_wgs = span * groups * ((cols + 15) / 16);
  // Without keys there may be no cache either (no pages, null pointers): whole rows, which load nothing of it then.
  return Plan{tiles, span, tiles > 0 && (cols <= 32 || wgs < (tiles <= 1 ? 200 : 96)) && split_wgs < (int64_t(1) << 24)};
}
}  // namespace

size_t cache_attention_workspace(const CacheAttnArgs& a) {
  const Plan p = plan_of(a);
  if (!p.split || p.tiles <= 1) return 0;
  return sizeof(float) * (size_t)(a.c.batch * a.q_len * a.heads * p.span) * (size_t)(a.c.dim + 4);
}

template <int HD>
static hipError_t attn_go(const CacheAttnArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  const int64_t cols = a.q_len * (a.heads / a.c.heads);
  if (!p.split) {
    const int64_t blocks = (cols + 63) / 64;
    const int64_t n = blocks * a.c.heads * a.c.batch;
    hipLaunchKernelGGL((attn_rows_kernel<HD>), dim3((unsigned)n), dim3(256), 0, s, a, blocks);
    return hipGetLastError();
  }
  const int64_t blocks = (cols + 15) / 16, tiles = p.tiles, span = p.span;
  hipLaunchKernelGGL((attn_tile_kernel<HD>), dim3((unsigned)(span * blocks * a.c.heads * a.c.batch)), dim3(256), 0, s, a,
                     tiles, blocks, span);
  if (tiles > 1)
    hipLaunchKernelGGL((attn_join_kernel<HD>), dim3((unsigned)(a.c.batch * a.q_len * a.heads)), dim3(64), 0, s, a, tiles, span);
  return hipGetLastError();
}

hipError_t cache_attention_launch(const CacheAttnArgs& a, hipStream_t s) {
  switch (a.c.dim) {
    case 32: return attn_go<32>(a, s);
    case 64: return attn_go<64>(a, s);
    case 96: return attn_go<96>(a, s);
    case 128: return attn_go<128>(a, s);
    case 160: return attn_go<160>(a, s);
    case 192: return attn_go<192>(a, s);
    case 224: return attn_go<224>(a, s);
    default: return attn_go<256>(a, s);
  }
}

}  // namespace canon
