// rope.hip - rotary positions as a call (R24), and the paged cache of keys and values in 8 bits (R25): appending with the
// rotation on the way, and reading back.
//
// All of it moves bytes: an element is read once and written once, with a handful of operations between, so what counts is
// that every lane has a wide load of its own in flight and no lane waits for another's.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "act8_dev.h"
#include "canon_dev.h"
#include "canon_internal.h"
#include "rows_dev.h"

namespace canon {

// W elements of a row, fp32 or bf16, as arithmetic reads them (a subnormal as zero)
template <bool BF16, int W>
__device__ __forceinline__ void wide_in(const void* p, int64_t at, float (&f)[W]) {
  static_assert(W == 1 || W == 2 || W % 4 == 0, "");
  if constexpr (W < 4) {
#pragma unroll
    for (int i = 0; i < W; ++i) f[i] = BF16 ? bf16_to_f32(((const uint16_t*)p)[at + i]) : step_daz(((const float*)p)[at + i]);
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      float t[4];
      if constexpr (BF16) {
        ldb<4>((const uint16_t*)p + at + i, t);
      } else {
        ldf<4>((const float*)p + at + i, t);
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = step_daz(t[j]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) f[i + j] = t[j];
    }
  }
}
template <bool BF16, int W>
__device__ __forceinline__ void wide_out(void* p, int64_t at, const float (&f)[W]) {
  static_assert(W == 1 || W == 2 || W % 4 == 0, "");
  if constexpr (W < 4) {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (BF16) ((uint16_t*)p)[at + i] = f32_to_bf16(f[i]);
      else ((float*)p)[at + i] = f[i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const float t[4] = {f[i], f[i + 1], f[i + 2], f[i + 3]};
      if constexpr (BF16) *reinterpret_cast<H4*>((uint16_t*)p + at + i) = H4{pack_bf16(t[0], t[1]), pack_bf16(t[2], t[3])};
      else stf<4>((float*)p + at + i, t);
    }
  }
}

// A pair turned: forward (a c - b s, b c + a s), backward with the angle's sign the other way.  A product's sign passes
// through its rounding, so the backward is the forward with -s.
__device__ __forceinline__ void turn_pair(float a, float b, float c, float s, float& x, float& y) {
  x = a * c - b * s;
  y = b * c + a * s;
}

// One thread turns W pairs of a head (or keeps 2 W elements behind them): unit u < rot / (2 W) pairs, then the kept ones.
// Bound by memory: 8192 tokens of 16 heads of 128, fp32 in and bf16 out, 16.6 us a direction; 8 tokens 2.9, a launch.
template <bool XB, bool YB, int W, bool PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(int32_t backward, int64_t n, int32_t units, int32_t per_token, int32_t dim,
                                                   Turn t, const int32_t* __restrict__ positions, const void* x, int64_t xs,
                                                   void* y, int64_t ys) {
  const int64_t idx = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (idx >= n) return;
  int64_t tok;
  int32_t in;
  if (n <= 0x7FFFFFFF) {
    tok = (uint32_t)idx / (uint32_t)per_token;
    in = (uint32_t)idx % (uint32_t)per_token;
  } else {
    tok = idx / per_token;
    in = (int32_t)(idx % per_token);
  }
  const int32_t h = (uint32_t)in / (uint32_t)units, u = in - h * units;
  const int32_t half = t.rot >> 1, turning = half / W;
  const int64_t xr = tok * xs + (int64_t)h * dim, yr = tok * ys + (int64_t)h * dim;
  if (u >= turning) {
    const int32_t at = t.rot + 2 * W * (u - turning);
    float f[2 * W];
    if (at + 2 * W <= dim) {
      wide_in<XB, 2 * W>(x, xr + at, f);
      wide_out<YB, 2 * W>(y, yr + at, f);
    } else {  // W = 1: an odd head's last
      float g[1];
      wide_in<XB, 1>(x, xr + at, g);
      wide_out<YB, 1>(y, yr + at, g);
    }
    return;
  }
  const int64_t pos = positions ? positions[tok] : tok;
  const int32_t i = u * W;
  float c[W], s[W], f[2 * W], r[2 * W];
  const bool in_table = pos >= 0 && pos < t.positions;
  if (in_table) {
    ldf<W>(t.cos + pos * half + i, c);
    ldf<W>(t.sin + pos * half + i, s);
  } else {
#pragma unroll
    for (int k = 0; k < W; ++k) c[k] = s[k] = __builtin_nanf("");
  }
  if constexpr (PAIRS) {
    wide_in<XB, 2 * W>(x, xr + 2 * i, f);
  } else {
    float a[W], b[W];
    wide_in<XB, W>(x, xr + i, a);
    wide_in<XB, W>(x, xr + i + half, b);
#pragma unroll
    for (int k = 0; k < W; ++k) { f[2 * k] = a[k]; f[2 * k + 1] = b[k]; }
  }
#pragma unroll
  for (int k = 0; k < W; ++k) turn_pair(f[2 * k], f[2 * k + 1], c[k], backward ? -s[k] : s[k], r[2 * k], r[2 * k + 1]);
  if constexpr (PAIRS) {
    wide_out<YB, 2 * W>(y, yr + 2 * i, r);
  } else {
    float a[W], b[W];
#pragma unroll
    for (int k = 0; k < W; ++k) { a[k] = r[2 * k]; b[k] = r[2 * k + 1]; }
    wide_out<YB, W>(y, yr + i, a);
    wide_out<YB, W>(y, yr + i + half, b);
  }
}

hipError_t rope_launch(int32_t backward, int64_t tokens, int64_t heads, int64_t dim, const Turn& t, const int32_t* positions,
                       int32_t x_bf16, const void* x, int64_t xs, int32_t y_bf16, void* y, int64_t ys, hipStream_t s) {
  const bool wide = t.rot % 8 == 0 && dim % 8 == 0;
  const int w = wide ? 4 : 1;
  const int32_t units = (int32_t)(t.rot / 2 / w + (dim - t.rot + 2 * w - 1) / (2 * w));
  const int32_t per_token = (int32_t)(heads * units);
  auto go = [&](auto xb, auto yb, auto width, auto pairs) {
    // launches below 2^32 threads
    const int64_t most = ((int64_t)1 << 31) / per_token > 0 ? ((int64_t)1 << 31) / per_token : 1;
    for (int64_t t0 = 0; t0 < tokens; t0 += most) {
      const int64_t nt = tokens - t0 < most ? tokens - t0 : most, nn = nt * per_token;
      Turn tt = t;
      const int32_t* ps = positions ? positions + t0 : nullptr;
      if (!positions) {  // token t at position t
        tt.cos = t.cos + t0 * (t.rot / 2);
        tt.sin = t.sin + t0 * (t.rot / 2);
        tt.positions = t.positions > t0 ? t.positions - t0 : 0;
      }
      hipLaunchKernelGGL((rope_kernel<xb.value, yb.value, width.value, pairs.value>), dim3((unsigned)((nn + 255) / 256)),
                         dim3(256), 0, s, backward, nn, units, per_token, (int32_t)dim, tt, ps,
                         (const char*)x + t0 * xs * (xb.value ? 2 : 4), xs, (char*)y + t0 * ys * (yb.value ? 2 : 4), ys);
    }
    return hipGetLastError();
  };
  using T = std::true_type;
  using F = std::false_type;
  using W1 = std::integral_constant<int, 1>;
  using W4 = std::integral_constant<int, 4>;
  auto layout = [&](auto xb, auto yb) {
    if (wide) return t.interleaved ? go(xb, yb, W4{}, T{}) : go(xb, yb, W4{}, F{});
    return t.interleaved ? go(xb, yb, W1{}, T{}) : go(xb, yb, W1{}, F{});
  };
  if (x_bf16) return y_bf16 ? layout(T{}, T{}) : layout(T{}, F{});
  return y_bf16 ? layout(F{}, T{}) : layout(F{}, F{});
}

// ---- the cache ------------------------------------------------------------------------------------------------------

// the slot of position j of sequence b in head h's steps, -1 if the cache has none
__device__ __forceinline__ int64_t cache_slot(const CacheView& c, int64_t b, int32_t h, int64_t j) {
  if (j < 0 || (j >> c.lg) >= c.table_len) return -1;
  const int64_t p = c.table[b * c.table_len + (j >> c.lg)];
  if (p < 0 || p >= c.n_pages) return -1;
  return (((p * c.heads + h) << c.lg)) + (j & ((1 << c.lg) - 1));
}

// Workgroup: 16 positions that share a group of the value codes, of one head of one sequence.  LPT lanes hold a token, four
// consecutive elements each (those behind head_dim idle).  Keys go out as they are, four codes a lane; values through LDS,
// so that a whole group leaves as 16-byte stores; a group with tokens missing leaves byte by byte, the others untouched (they may
// be another sequence's of the same call; two tokens in one slot are not kept apart).
// Bound by memory: 5120 tokens of 4 sequences, 8 heads of 128 from fp32, 16.4 us; a token each of 16 sequences 4.2.
template <bool XB, int LPT>
__global__ __launch_bounds__(256) void cache_append_kernel(CacheView c, CacheRowsArgs r, const void* __restrict__ k,
                                                           int64_t k_stride, const void* __restrict__ v, int64_t v_stride,
                                                           Turn t) {
  constexpr int TPP = 256 / LPT < 16 ? 256 / LPT : 16;  // tokens at a time
  __shared__ __attribute__((aligned(16))) uint8_t vt[256 * 16];
  const int64_t b = blockIdx.z;
  const int32_t h = blockIdx.y, dim = c.dim;
  const int64_t first = r.q_starts ? r.q_starts[b] : r.q_start;
  int64_t count = r.q_len;
  if (r.q_lens) count = r.q_lens[b] < count ? r.q_lens[b] : count;
  if (count <= 0) return;
  const int64_t g0 = ((first >> 4) + blockIdx.x) << 4;  // the group's first position (first may be negative)
  if (g0 >= first + count) return;
  const int64_t base = cache_slot(c, b, h, g0);  // a group lies in one page
  if (base < 0) return;
  const int tl = threadIdx.x / LPT, at = 4 * (threadIdx.x % LPT), half = t.rot >> 1;
  for (int t0 = 0; t0 < 16; t0 += TPP) {
    const int in = t0 + tl;
    const int64_t pos = g0 + in, i = pos - first;
    const bool real = tl < TPP && i >= 0 && i < count;
    const bool mine = real && at < dim;
    float kv[1][4] = {{0.0f, 0.0f, 0.0f, 0.0f}}, vv[1][4] = {{0.0f, 0.0f, 0.0f, 0.0f}};
    if (mine) {
      const int64_t row = b * r.q_len + i;
      const int64_t ka = row * k_stride + (int64_t)h * dim, va = row * v_stride + (int64_t)h * dim;
      wide_in<XB, 4>(v, va + at, vv[0]);
      wide_in<XB, 4>(k, ka + at, kv[0]);
      if (at < t.rot) {
        const bool in_table = pos < t.positions;
        const float* cp = t.cos + pos * half;
        const float* sp = t.sin + pos * half;
        float o[4];
        if (t.interleaved) {  // elements at, at + 1 and at + 2, at + 3 together
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            if (at + e < t.rot) {
              const float cc = in_table ? cp[(at + e) / 2] : __builtin_nanf(""), ss = in_table ? sp[(at + e) / 2] : __builtin_nanf("");
              turn_pair(kv[0][e], kv[0][e + 1], cc, ss, o[e], o[e + 1]);
            } else {
              o[e] = kv[0][e];
              o[e + 1] = kv[0][e + 1];
            }
          }
        } else if (t.rot % 8 == 0) {  // four elements of one half, with the same four of the other
          const int p = at < half ? at : at - half;
          float other[4], cs[4], sn[4];
          wide_in<XB, 4>(k, ka + (at < half ? at + half : p), other);
          if (in_table) {
            ldf<4>(cp + p, cs);
            ldf<4>(sp + p, sn);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) cs[e] = sn[e] = __builtin_nanf("");
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x, y;
            turn_pair(at < half ? kv[0][e] : other[e], at < half ? other[e] : kv[0][e], cs[e], sn[e], x, y);
            o[e] = at < half ? x : y;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int d = at + e, p = d < half ? d : d - half;
            o[e] = kv[0][e];
            if (d < t.rot) {
              float other[1], x, y;
              wide_in<XB, 1>(k, ka + (d < half ? d + half : p), other);
              const float cc = in_table ? cp[p] : __builtin_nanf(""), ss = in_table ? sp[p] : __builtin_nanf("");
              turn_pair(d < half ? kv[0][e] : other[0], d < half ? other[0] : kv[0][e], cc, ss, x, y);
              o[e] = d < half ? x : y;
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) kv[0][e] = o[e];
      }
    }
    float ks[1], vs[1];
    constexpr int lg = LPT == 8 ? 5 : LPT == 16 ? 6 : LPT == 32 ? 7 : 8;
    steps4(kv, lg, ks);
    steps4(vv, lg, vs);
    if (mine) {
      const int64_t slot = base + in;
      uint32_t w[1];
      quant_pack<4>(kv[0], ks[0], step_rcp(ks[0]), recip_step_ok(ks[0]), w);
      *reinterpret_cast<uint32_t*>(c.kc + slot * dim + at) = w[0];
      quant_pack<4>(vv[0], vs[0], step_rcp(vs[0]), recip_step_ok(vs[0]), w);
#pragma unroll
      for (int e = 0; e < 4; ++e) vt[(at + e) * 16 + in] = (uint8_t)(w[0] >> (8 * e));
      if (at == 0) {
        c.ks[slot] = ks[0];
        c.vs[slot] = vs[0];
      }
    }
  }
  __syncthreads();
  int8_t* out = c.vc + base * dim;  // base is a multiple of 16: the group's [dim][16]
  const int lo = first > g0 ? (int)(first - g0) : 0, hi = first + count < g0 + 16 ? (int)(first + count - g0) : 16;
  if (lo == 0 && hi == 16) {
    for (int d = threadIdx.x; d < dim; d += 256) reinterpret_cast<uint4*>(out)[d] = reinterpret_cast<const uint4*>(vt)[d];
  } else {
    for (int d = threadIdx.x; d < dim; d += 256)
      for (int e = lo; e < hi; ++e) out[d * 16 + e] = (int8_t)vt[d * 16 + e];
  }
}

hipError_t cache_append_launch(const CacheView& c, const CacheRowsArgs& r, int32_t bf16, const void* k, int64_t k_stride,
                               const void* v, int64_t v_stride, const Turn& t, hipStream_t s) {
  const dim3 grid((unsigned)((r.q_len + 15) / 16 + 1), (unsigned)c.heads, (unsigned)c.batch);
  auto go = [&](auto xb, auto lpt) {
    hipLaunchKernelGGL((cache_append_kernel<xb.value, lpt.value>), grid, dim3(256), 0, s, c, r, k, k_stride, v, v_stride, t);
    return hipGetLastError();
  };
  auto lanes = [&](auto xb) {
    if (c.dim <= 32) return go(xb, std::integral_constant<int, 8>{});
    if (c.dim <= 64) return go(xb, std::integral_constant<int, 16>{});
    if (c.dim <= 128) return go(xb, std::integral_constant<int, 32>{});
    return go(xb, std::integral_constant<int, 64>{});
  };
  return bf16 ? lanes(std::true_type{}) : lanes(std::false_type{});
}

// One thread: four elements of a head of the 16 tokens that share a group of the value codes: four 16-byte vectors of values,
// turned over four by four bytes, and a row's four key codes at a time (one thread to four elements of one token gathered its
// value codes byte by byte: 4 x 2048 tokens of 8 heads of 128 22.5 us, so 16).
template <bool YB>
__global__ __launch_bounds__(256) void cache_read_kernel(CacheView c, CacheRowsArgs r, void* k, void* v) {
  const uint32_t per = (uint32_t)c.dim >> 2, idx = blockIdx.y * 256 + threadIdx.x;
  if (idx >= per * (uint32_t)c.heads) return;
  const int32_t h = (int32_t)(idx / per), at = 4 * (int32_t)(idx - (uint32_t)h * per);
  const int64_t b = blockIdx.z, first = r.q_starts ? r.q_starts[b] : r.q_start, g0 = ((first >> 4) + blockIdx.x) << 4;
  const int64_t count = r.q_lens && r.q_lens[b] < r.q_len ? r.q_lens[b] : r.q_len;  // rows that exist
  if (g0 >= first + r.q_len) return;
  const int64_t base = cache_slot(c, b, h, g0);  // of the group, in one page
  const int64_t i0 = g0 - first;
  const int lo = i0 < 0 ? (int)-i0 : 0, end = i0 + 16 > r.q_len ? (int)(r.q_len - i0) : 16;
  const int64_t out0 = ((b * r.q_len + i0) * c.heads + h) * c.dim + at, next = (int64_t)c.heads * c.dim;
  uint32_t w[16];
  auto put = [&](void* out, const float* steps) {
#pragma unroll
    for (int t = 0; t < 16; ++t) {
      if (t < lo || t >= end) continue;
      float f[4];
      if (i0 + t >= count) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = 0.0f;
      } else if (base < 0) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = __builtin_nanf("");
      } else {
        const float st = steps[base + t];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = (float)(int8_t)(w[t] >> (8 * e)) * st;
      }
      wide_out<YB, 4>(out, out0 + t * next, f);
    }
  };
  if (k) {
    if (base >= 0) {
#pragma unroll
      for (int t = 0; t < 16; ++t) w[t] = *reinterpret_cast<const uint32_t*>(c.kc + (base + t) * c.dim + at);
    }
    put(k, c.ks);
  }
  if (v) {
    if (base >= 0) {
      const uint4* p = reinterpret_cast<const uint4*>(c.vc + base * c.dim + 16 * at);
      uint4 d[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) d[e] = p[e];
#pragma unroll
      for (int q = 0; q < 4; ++q) {  // tokens 4 q .. 4 q + 3: byte t of the dword of element e becomes byte e of token t's
        uint32_t x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = q == 0 ? d[e].x : q == 1 ? d[e].y : q == 2 ? d[e].z : d[e].w;
        const uint32_t a01 = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u), b01 = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);
        const uint32_t a23 = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u), b23 = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
        w[4 * q] = __builtin_amdgcn_perm(a23, a01, 0x05040100u);
        w[4 * q + 1] = __builtin_amdgcn_perm(a23, a01, 0x07060302u);
        w[4 * q + 2] = __builtin_amdgcn_perm(b23, b01, 0x05040100u);
        w[4 * q + 3] = __builtin_amdgcn_perm(b23, b01, 0x07060302u);
      }
    }
    put(v, c.vs);
  }
}

hipError_t cache_read_launch(const CacheView& c, const CacheRowsArgs& r, int32_t bf16, void* k, void* v, hipStream_t s) {
  const dim3 grid((unsigned)((r.q_len + 15) / 16 + 1), (unsigned)((c.heads * (c.dim / 4) + 255) / 256), (unsigned)c.batch);
  if (bf16) hipLaunchKernelGGL(cache_read_kernel<true>, grid, dim3(256), 0, s, c, r, k, v);
  else hipLaunchKernelGGL(cache_read_kernel<false>, grid, dim3(256), 0, s, c, r, k, v);
  return hipGetLastError();
}

}  // namespace canon
