// attn_cache.hip - attention over the paged cache of keys and values in 8 bits (R26).
//
// Every long sum is a sum of products of whole numbers, so it runs on the int8 matrix instructions in any order: a query (and
// a weight) is a whole number of 16 bits, split into two digits of 8, x = 256 hi + lo, and sum x k = 256 sum hi k + sum lo k.
// Left to floating point are a maximum, a tile's 256 exponentials and their tree, and one fused multiply-add per tile and
// element, with every change of reference a power of two.
//
// v_mfma_i32_16x16x64_i8 multiplies 16 rows by 16 columns over 64 k.  Lane (c, g) = (lane % 16, lane / 16) supplies bytes 16 g
// .. 16 g + 15 of row (column) c and receives rows 4 g .. 4 g + 3 of column c.  Keys are the rows of the score product, queries
// its columns: taking key 16 (row / 4) + 4 t + row % 4 of 64 for row `row` of instruction t, lane (c, g) receives the scores of
// keys 16 g + 4 t + i (t, i = 0 .. 3): the 16 consecutive keys that it has to supply, as weights, to the product with the values,
// whose rows are elements of a head (the cache keeps 16 tokens of an element together) and whose columns are the queries again.
// No lane ever needs another's weights, and a query's maxima and sums cross 4 lanes.
#include <hip/hip_runtime.h>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int kTile = 256;                      // keys of a tile of the rule
constexpr float kDigits = 32512.0f;             // largest whole number of a query or a weight: its high digit is 127
constexpr uint32_t kInvDigits = 0x38010204u;    // RN32(1 / 32512)
constexpr float kNegInf = -__builtin_inff();

// 2^x, |x| <= 1/2: the polynomial of least relative error with the constant 1 (its coefficients rounded; 1.6e-7 in all)
constexpr uint32_t kExp2C[5] = {0x3F317215u, 0x3E75FCDEu, 0x3D635BA9u, 0x3C1E7544u, 0x3AADDD09u};

// cexp2 of x <= 0 or NaN.  The clamp makes n = -127 of all that lies below, whose scale's bits are zero; it passes a NaN on.
__device__ __forceinline__ float cexp2(float x) {
  x = __builtin_elementwise_maximum(x, -127.0f);
  const float u = x + 0x1.8p23f;  // rne(x), also in the low bits
  const float f = x - (u - 0x1.8p23f);
  float p = __builtin_fmaf(__uint_as_float(kExp2C[4]), f, __uint_as_float(kExp2C[3]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[2]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[1]));
  p = __builtin_fmaf(p, f, __uint_as_float(kExp2C[0]));
  p = __builtin_fmaf(p, f, 1.0f);
  return p * __uint_as_float((__float_as_uint(u) << 23) + 0x3F800000u);
}

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
  const int32_t G = a.heads / a.c.heads;
  const int64_t i = idx / G;
  c.h = kvh * G + (int32_t)(idx - i * G);
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

// the 16 keys from j on (a multiple of 16): their first slot in head kvh, or -1
__device__ __forceinline__ int64_t slots16(const CacheAttnArgs& a, int64_t b, int32_t kvh, int64_t j) {
  if (j >= a.k_len) return -1;
  const int64_t p = a.c.table[b * a.c.table_len + (j >> a.c.lg)];
  if (p < 0 || p >= a.c.n_pages) return -1;
  return ((p * a.c.heads + kvh) << a.c.lg) + (j & ((1 << a.c.lg) - 1));
}

__device__ __forceinline__ i32x4 load16(const int8_t* p) { return *reinterpret_cast<const i32x4*>(p); }

// The queries of a block as digits: lane (c, g) holds elements 64 s + 16 g .. + 15 of column c, and the column's f.
template <int HD>
struct Query {
  static constexpr int NS = (HD + 63) / 64;
  i32x4 hi[NS], lo[NS];
  float f;
};
template <int HD>
__device__ __forceinline__ void load_query(const CacheAttnArgs& a, const Column& c, Query<HD>& out) {
  constexpr int NS = Query<HD>::NS;
  const int g = (threadIdx.x & 63) >> 4;
  float v[NS][16];
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 64 * s + 16 * g;
#pragma unroll
    for (int e = 0; e < 16; ++e) v[s][e] = 0.0f;
    if (c.real && d < HD) {
      const int64_t at = c.tok * a.q_stride + (int64_t)c.h * HD + d;
#pragma unroll
      for (int e = 0; e < 16; e += 4) {
        float t[4];
        if (a.q_bf16) ldb<4>((const uint16_t*)a.q + at + e, t);
        else ldf<4>((const float*)a.q + at + e, t);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[s][e + i] = t[i];
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t u = __float_as_uint(v[s][e]) & 0x7FFFFFFFu;
      top = u > top ? u : top;
    }
  }
  top = umax4(top);
  const float sq = __uint_as_float(top) * __uint_as_float(kInvDigits);
  const float rs = sq > 0.0f ? 1.0f / sq : 0.0f;
#pragma unroll
  for (int s = 0; s < NS; ++s)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      uint32_t h = 0, l = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = v[s][4 * w + e] * rs;
        x = sq > 0.0f && x == x ? fminf(fmaxf(x, -kDigits), kDigits) : 0.0f;
        const int32_t n = (int32_t)__builtin_rintf(x), d = (n + 128) >> 8;  // n = 256 d + (n - 256 d), the rest in [-128, 127]
        h |= (uint32_t)(d & 0xFF) << (8 * e);
        l |= (uint32_t)(n & 0xFF) << (8 * e);
      }
      out.hi[s][w] = (int32_t)h;
      out.lo[s][w] = (int32_t)l;
    }
  const float sc = sq * a.scale;
  out.f = sc * kLog2e;
}

// Four weights as whole numbers, 0 <= w <= 32512, into a dword of each digit.  Adding 1.5 2^23 + 128 rounds to a whole number
// and leaves w + 128 in the low bits: byte 1 is the high digit, byte 0 the low one with its sign bit inverted.
__device__ __forceinline__ void digits4(float w0, float w1, float w2, float w3, int32_t& hi, int32_t& lo) {
  const uint32_t a = __float_as_uint(w0 + 12583040.0f), b = __float_as_uint(w1 + 12583040.0f);
  const uint32_t c = __float_as_uint(w2 + 12583040.0f), d = __float_as_uint(w3 + 12583040.0f);
  const uint32_t ab = __builtin_amdgcn_perm(b, a, 0x05010400u);  // a0 b0 a1 b1
  const uint32_t cd = __builtin_amdgcn_perm(d, c, 0x05010400u);
  lo = (int32_t)(__builtin_amdgcn_perm(cd, ab, 0x05040100u) ^ 0x80808080u);
  hi = (int32_t)__builtin_amdgcn_perm(cd, ab, 0x07060302u);
}

// what a tile's values are scaled by: rv (0 where all weights are) and RN(V RN(1/32512))
__device__ __forceinline__ float value_recip(uint32_t vtop) {
  const float V = __uint_as_float(vtop);
  const float rv = V > 0.0f ? kDigits / V : 0.0f;
  return rv < __builtin_inff() ? rv : 0.0f;
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
// with the values (the weights cross through LDS, 8 KB): a workgroup has all of its 2 * 256 * head_dim bytes of the cache on
// their way at once and waits for them once.  What a tile gives goes to `parts`, a row's tiles one after the other, to be
// joined by attn_join_kernel; where there is one tile only, straight to the output.
template <int HD>
__global__ __launch_bounds__(256) void attn_tile_kernel(CacheAttnArgs a, int64_t tiles, int64_t blocks) {
  constexpr int NS = Query<HD>::NS, ND = HD / 16, NW = (ND + 3) / 4;  // 16-element parts of a head, of a wavefront
  __shared__ __attribute__((aligned(16))) i32x4 wts[2][4][64];
  __shared__ float ms[4][16], ss[4][16];
  __shared__ uint32_t vs[4][16];
  int64_t id = blockIdx.x;
  const int64_t tile = id % tiles;
  id /= tiles;
  const int64_t cb = id % blocks;
  id /= blocks;
  const int32_t kvh = (int32_t)(id % a.c.heads);
  const int64_t b = id / a.c.heads;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cc = lane & 15, g = lane >> 4;
  const Column col = column_of(a, b, kvh, cb * 16 + cc);
  const int64_t t0 = tile * kTile;
  const bool touched = col.lo < t0 + kTile && col.hi > t0;
  if (tiles > 1 && !__any(touched)) return;  // the join passes over tiles that a row does not see

  // everything from the cache first
  const int64_t j0 = t0 + 64 * w;
  const int64_t kslot = slots16(a, b, kvh, j0 + 16 * (cc >> 2)), gslot = slots16(a, b, kvh, j0 + 16 * g);
  i32x4 kx[4][NS];
#pragma unroll
  for (int t = 0; t < 4; ++t)
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      kx[t][s] = i32x4{0, 0, 0, 0};
      if (kslot >= 0 && (HD % 64 == 0 || 64 * s + 16 * g < HD))
        kx[t][s] = load16(a.c.kc + (kslot + 4 * t + (cc & 3)) * HD + 64 * s + 16 * g);
    }
  f32x4 kst[4], vst[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    kst[t] = vst[t] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
    if (gslot >= 0) {
      kst[t] = *reinterpret_cast<const f32x4*>(a.c.ks + gslot + 4 * t);
      vst[t] = *reinterpret_cast<const f32x4*>(a.c.vs + gslot + 4 * t);
    }
  }
  i32x4 vx[NW][4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t vslot = slots16(a, b, kvh, t0 + 64 * q + 16 * g);
#pragma unroll
    for (int n = 0; n < NW; ++n) {
      const int part = w + 4 * n;
      vx[n][q] = i32x4{0, 0, 0, 0};
      if (vslot >= 0 && (ND % 4 == 0 || part < ND)) vx[n][q] = load16(a.c.vc + vslot * HD + (16 * part + cc) * 16);
    }
  }
  Query<HD> qd;
  load_query<HD>(a, col, qd);

  float t[4][4];
  float m = kNegInf;
  uint32_t vtop = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < NS; ++s) acc = mfma(kx[k][s], qd.hi[s], acc);
    acc = acc << 8;
#pragma unroll
    for (int s = 0; s < NS; ++s) acc = mfma(kx[k][s], qd.lo[s], acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t j = j0 + 16 * g + 4 * k + i;
      const bool seen = j >= col.lo && j < col.hi;
      const float x = (float)acc[i] * qd.f;
      t[k][i] = seen ? x * kst[k][i] : kNegInf;
      m = __builtin_elementwise_maximum(m, t[k][i]);
      const uint32_t u = seen ? __float_as_uint(vst[k][i]) & 0x7FFFFFFFu : 0u;
      vtop = u > vtop ? u : vtop;
    }
  }
  m = max4(m);
  vtop = umax4(vtop);
  if (g == 0) {
    ms[w][cc] = m;
    vs[w][cc] = vtop;
  }
  __syncthreads();
#pragma unroll
  for (int o = 0; o < 4; ++o) {
    m = __builtin_elementwise_maximum(m, ms[o][cc]);
    vtop = vs[o][cc] > vtop ? vs[o][cc] : vtop;
  }
  const float r = __builtin_ceilf(m), ref = r == kNegInf ? 0.0f : r, rv = value_recip(vtop);
  float sum = 0.0f;
  i32x4 wh, wl;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = cexp2(t[k][i] - ref);
      sum = sum + e;
      const int64_t j = j0 + 16 * g + 4 * k + i;
      const float ratio = vst[k][i] * rv;
      x[i] = rv != 0.0f && j >= col.lo && j < col.hi ? e * ratio : 0.0f;
    }
    int32_t h, l;
    digits4(x[0], x[1], x[2], x[3], h, l);
    wh[k] = h;
    wl[k] = l;
  }
  wts[0][w][lane] = wh;
  wts[1][w][lane] = wl;
  sum = sum4(sum);
  if (g == 0) ss[w][cc] = sum;
  __syncthreads();
  const float S = (ss[0][cc] + ss[1][cc]) + (ss[2][cc] + ss[3][cc]);
  const float vsc = __uint_as_float(vtop) * __uint_as_float(kInvDigits);
  const float inv = S == 0.0f ? 0.0f : 1.0f / S;
  float* parts = a.parts + (col.row * tiles + tile) * (HD + 4);
  if (tiles > 1 && col.real && w == 0 && g == 0)
    *reinterpret_cast<f32x4*>(parts + HD) = f32x4{r, S, vsc, 0.0f};
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
    if (!col.real) continue;
    f32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (float)acc[i];
    if (tiles > 1) {
      *reinterpret_cast<f32x4*>(parts + 16 * part + 4 * g) = o;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = S == 0.0f ? 0.0f : o[i] * vsc;
      store_out(a, col.row, 16 * part + 4 * g, inv, o, HD);
    }
  }
}

// A row's tiles joined, ascending: one wavefront a row, HD / 64 (or fewer) elements a lane.
template <int HD>
__global__ __launch_bounds__(64) void attn_join_kernel(CacheAttnArgs a, int64_t tiles) {
  constexpr int E = (HD + 63) / 64;
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x;
  const int64_t tok = row / a.heads, b = tok / a.q_len;
  const int32_t G = a.heads / a.c.heads, h = (int32_t)(row - tok * a.heads);
  const Column col = column_of(a, b, h / G, (tok - b * a.q_len) * G + h % G);
  const float* parts = a.parts + row * tiles * (HD + 4);
  float R = kNegInf, S = 0.0f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.0f;
  if (col.hi > col.lo)
    for (int64_t t = col.lo / kTile; t <= (col.hi - 1) / kTile; ++t) {
      const float* p = parts + t * (HD + 4);
      const f32x4 d = *reinterpret_cast<const f32x4*>(p + HD);
      const float Rn = __builtin_elementwise_maximum(R, d[0]), x = shift2(R, Rn), y = shift2(d[0], Rn);
      S = __builtin_fmaf(d[1], y, S * x);
      const float sc = d[2] * y;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (lane + 64 * e < HD) o[e] = __builtin_fmaf(p[lane + 64 * e], sc, o[e] * x);
      R = Rn;
    }
  const float inv = S == 0.0f ? 0.0f : 1.0f / S;
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (lane + 64 * e < HD) {
      const float x = o[e] + 0.0f;
      a.out[row * HD + lane + 64 * e] = S == 0.0f ? 0 : f32_to_bf16(x * inv);
    }
}

// ---- all keys of a block of queries in one wavefront: prompts ------------------------------------------------------------
template <int HD>
__global__ __launch_bounds__(256, 1) void attn_rows_kernel(CacheAttnArgs a, int64_t blocks) {
  constexpr int NS = Query<HD>::NS, ND = HD / 16;
  int64_t id = blockIdx.x;
  const int64_t cb = blocks - 1 - id % blocks;  // the longest causal rows first
  id /= blocks;
  const int32_t kvh = (int32_t)(id % a.c.heads);
  const int64_t b = id / a.c.heads;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, cc = lane & 15, g = lane >> 4;
  const Column col = column_of(a, b, kvh, (cb * 4 + w) * 16 + cc);
  if (!__any(col.real)) return;
  int64_t lo = col.hi > col.lo ? col.lo : (int64_t)1 << 62, hi = col.hi;
#pragma unroll
  for (int s = 1; s < 16; s <<= 1) {
    const int64_t l = __shfl_xor(lo, s, 64), h = __shfl_xor(hi, s, 64);
    lo = l < lo ? l : lo;
    hi = h > hi ? h : hi;
  }
  Query<HD> qd;
  load_query<HD>(a, col, qd);
  float R = kNegInf, S = 0.0f;
  f32x4 o[ND];
#pragma unroll
  for (int n = 0; n < ND; ++n) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  for (int64_t t0 = hi > lo ? lo / kTile * kTile : hi; t0 < hi; t0 += kTile) {
    const bool all = __all(!col.real || (col.lo <= t0 && col.hi >= t0 + kTile));
    float t[4][4][4];
    float m = kNegInf;
    uint32_t vtop = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t j0 = t0 + 64 * q;
      const int64_t kslot = slots16(a, b, kvh, j0 + 16 * (cc >> 2)), gslot = slots16(a, b, kvh, j0 + 16 * g);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        i32x4 kx[NS];
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          kx[s] = i32x4{0, 0, 0, 0};
          if (kslot >= 0 && (HD % 64 == 0 || 64 * s + 16 * g < HD))
            kx[s] = load16(a.c.kc + (kslot + 4 * k + (cc & 3)) * HD + 64 * s + 16 * g);
        }
        f32x4 kst{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")}, vst = kst;
        if (gslot >= 0) {
          kst = *reinterpret_cast<const f32x4*>(a.c.ks + gslot + 4 * k);
          vst = *reinterpret_cast<const f32x4*>(a.c.vs + gslot + 4 * k);
        }
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < NS; ++s) acc = mfma(kx[s], qd.hi[s], acc);
        acc = acc << 8;
#pragma unroll
        for (int s = 0; s < NS; ++s) acc = mfma(kx[s], qd.lo[s], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int64_t j = j0 + 16 * g + 4 * k + i;
          const bool seen = all || (j >= col.lo && j < col.hi);
          const float x = (float)acc[i] * qd.f;
          t[q][k][i] = seen ? x * kst[i] : kNegInf;
          m = __builtin_elementwise_maximum(m, t[q][k][i]);
          const uint32_t u = seen ? __float_as_uint(vst[i]) & 0x7FFFFFFFu : 0u;
          vtop = u > vtop ? u : vtop;
        }
      }
    }
    m = max4(m);
    vtop = umax4(vtop);
    const float r = __builtin_ceilf(m), ref = r == kNegInf ? 0.0f : r, rv = value_recip(vtop);
    i32x4 wh[4], wl[4];
    float sums[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int64_t j0 = t0 + 64 * q, gslot = slots16(a, b, kvh, j0 + 16 * g);
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f32x4 vst{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
        if (gslot >= 0) vst = *reinterpret_cast<const f32x4*>(a.c.vs + gslot + 4 * k);
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = cexp2(t[q][k][i] - ref);
          sum = sum + e;
          const int64_t j = j0 + 16 * g + 4 * k + i;
          const float ratio = vst[i] * rv;
          x[i] = rv != 0.0f && (all || (j >= col.lo && j < col.hi)) ? e * ratio : 0.0f;
        }
        int32_t h, l;
        digits4(x[0], x[1], x[2], x[3], h, l);
        wh[q][k] = h;
        wl[q][k] = l;
      }
      sums[q] = sum4(sum);
    }
    const float Sb = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const float Rn = __builtin_elementwise_maximum(R, r), x = shift2(R, Rn), y = shift2(r, Rn);
    // A column that sees nothing of the tile has S_b = 0, A = 0 and V = 0 and keeps R: the steps below leave its row as it is
    // (but for the sign of a zero, which the output's + 0 takes away).
    S = __builtin_fmaf(Sb, y, S * x);
    R = Rn;
    const float sc = (__uint_as_float(vtop) * __uint_as_float(kInvDigits)) * y;
    int64_t vslot[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) vslot[q] = slots16(a, b, kvh, t0 + 64 * q + 16 * g);
#pragma unroll
    for (int n = 0; n < ND; ++n) {
      i32x4 vx[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        vx[q] = i32x4{0, 0, 0, 0};
        if (vslot[q] >= 0) vx[q] = load16(a.c.vc + vslot[q] * HD + (16 * n + cc) * 16);
      }
      i32x4 acc = {0, 0, 0, 0};
#pragma unroll
      for (int q = 0; q < 4; ++q) acc = mfma(vx[q], wh[q], acc);
      acc = acc << 8;
#pragma unroll
      for (int q = 0; q < 4; ++q) acc = mfma(vx[q], wl[q], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][i] = __builtin_fmaf((float)acc[i], sc, o[n][i] * x);
    }
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
  int64_t tiles;  // 1: the rows kernel, or one tile that the tile kernel finishes
  bool split;
};
Plan plan_of(const CacheAttnArgs& a) {
  const int64_t cols = a.q_len * (a.heads / a.c.heads), tiles = (a.k_len + kTile - 1) / kTile;
  const int64_t rows_wg = a.c.batch * a.c.heads * ((cols + 63) / 64);
  return Plan{tiles, tiles <= 1 || rows_wg < 256};
}
}  // namespace

size_t cache_attention_workspace(const CacheAttnArgs& a) {
  const Plan p = plan_of(a);
  if (!p.split || p.tiles <= 1) return 0;
  return sizeof(float) * (size_t)(a.c.batch * a.q_len * a.heads * p.tiles) * (size_t)(a.c.dim + 4);
}

template <int HD>
static hipError_t attn_go(const CacheAttnArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  const int64_t cols = a.q_len * (a.heads / a.c.heads);
  if (!p.split) {
    const int64_t blocks = (cols + 63) / 64;
    hipLaunchKernelGGL((attn_rows_kernel<HD>), dim3((unsigned)(blocks * a.c.heads * a.c.batch)), dim3(256), 0, s, a, blocks);
    return hipGetLastError();
  }
  const int64_t blocks = (cols + 15) / 16, tiles = p.tiles > 0 ? p.tiles : 1;
  hipLaunchKernelGGL((attn_tile_kernel<HD>), dim3((unsigned)(tiles * blocks * a.c.heads * a.c.batch)), dim3(256), 0, s, a,
                     tiles, blocks);
  if (tiles > 1)
    hipLaunchKernelGGL((attn_join_kernel<HD>), dim3((unsigned)(a.c.batch * a.q_len * a.heads)), dim3(64), 0, s, a, tiles);
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
