// i8_dev.h - what the int8 products share: 16 bytes of a row at any alignment, whole or cut by the row's end; order in LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace canon {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(1))) Bytes16 {
  uint32_t w[4];
};
// A wavefront's LDS operations complete in order; this holds the compiler to it where lanes read what others of the wavefront wrote,
// or write where they read.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }
// rows off 16-byte boundaries load as wide
__device__ __forceinline__ i32x4 whole16(const int8_t* p) {
  const Bytes16 v = *reinterpret_cast<const Bytes16*>(p);
  return i32x4{(int32_t)v.w[0], (int32_t)v.w[1], (int32_t)v.w[2], (int32_t)v.w[3]};
}
// 16 bytes of which the first `valid` exist, the others 0.  A cut vector is read as the row's last 16 and moved into place
// (`longer`: the row has 16); byte by byte, every byte's load was waited for: 1541 x 5001 x 2056 took 63 us, 2048 columns 50.
__device__ __forceinline__ i32x4 cut16(const int8_t* p, int64_t valid, bool longer) {
  if (valid >= 16) return whole16(p);
  i32x4 r = {0, 0, 0, 0};
  if (valid > 0) {
    if (longer) {
      const Bytes16 v = *reinterpret_cast<const Bytes16*>(p + valid - 16);
      unsigned __int128 x = ((unsigned __int128)v.w[3] << 96) | ((unsigned __int128)v.w[2] << 64) |
                            ((unsigned __int128)v.w[1] << 32) | v.w[0];
      x >>= 8 * (16 - (int)valid);
      r = i32x4{(int32_t)(uint32_t)x, (int32_t)(uint32_t)(x >> 32), (int32_t)(uint32_t)(x >> 64), (int32_t)(uint32_t)(x >> 96)};
    } else {  // a row of fewer than 16 bytes
      uint32_t w[4] = {0u, 0u, 0u, 0u};
      for (int e = 0; e < (int)valid; ++e) {
        const uint32_t b = (uint32_t)(uint8_t)p[e] << (8 * (e & 3));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] |= i == (e >> 2) ? b : 0u;
      }
      r = i32x4{(int32_t)w[0], (int32_t)w[1], (int32_t)w[2], (int32_t)w[3]};
    }
  }
  return r;
}

}  // namespace canon
