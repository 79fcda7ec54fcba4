// x of a product with 4-bit weights, eight columns at a time, as bf16 in the order in
// which a 32-bit word of codes yields its eight columns: 0 4 1 5 2 6 3 7.
#pragma once
#include <cuda_fp8.h>

#include "common.cuh"

namespace fovea {

// bf16 columns a row of x becomes: an fp32 row is the sum of three.
__host__ __device__ __forceinline__ int x_parts(int dtype) { return dtype == FOVEA_FP32 ? 3 : 1; }

// Whether every eight columns of every row can be read as vectors.
inline bool x_vectors(const void* x, long long ld, int dtype) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(x);
  if (dtype == FOVEA_BF16) return (p & 15u) == 0 && ld % 8 == 0;
  if (dtype == FOVEA_FP32) return (p & 15u) == 0 && ld % 4 == 0;
  return (p & 7u) == 0 && ld % 8 == 0;
}

// Eight columns as they lie in memory.
struct X8 {
  uint4 a, b;
  __device__ __forceinline__ void load(const void* x, long long at, int dtype, bool vec) {
    if (dtype == FOVEA_BF16) {
      const uint16_t* p = static_cast<const uint16_t*>(x) + at;
      if (vec) {
        a = *reinterpret_cast<const uint4*>(p);
      } else {
        a = make_uint4(p[0] | (uint32_t)p[1] << 16, p[2] | (uint32_t)p[3] << 16, p[4] | (uint32_t)p[5] << 16,
                       p[6] | (uint32_t)p[7] << 16);
      }
    } else if (dtype == FOVEA_FP32) {
      const uint32_t* p = static_cast<const uint32_t*>(x) + at;
      if (vec) {
        a = reinterpret_cast<const uint4*>(p)[0];
        b = reinterpret_cast<const uint4*>(p)[1];
      } else {
        a = make_uint4(p[0], p[1], p[2], p[3]);
        b = make_uint4(p[4], p[5], p[6], p[7]);
      }
    } else {
      const uint8_t* p = static_cast<const uint8_t*>(x) + at;
      if (vec) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        a.x = v.x;
        a.y = v.y;
      } else {
        a.x = p[0] | (uint32_t)p[1] << 8 | (uint32_t)p[2] << 16 | (uint32_t)p[3] << 24;
        a.y = p[4] | (uint32_t)p[5] << 8 | (uint32_t)p[6] << 16 | (uint32_t)p[7] << 24;
      }
    }
  }
  // The bf16 columns: one, or for fp32 the three truncations that add up to it (an
  // infinity or a NaN is the first alone).  e4m3 is exact in bf16.
  __device__ __forceinline__ void columns(int dtype, uint4 (&out)[3]) const {
    if (dtype == FOVEA_BF16) {
      out[0] = make_uint4(__byte_perm(a.x, a.z, 0x5410), __byte_perm(a.x, a.z, 0x7632),
                          __byte_perm(a.y, a.w, 0x5410), __byte_perm(a.y, a.w, 0x7632));
      return;
    }
    uint32_t v[3][8];
    if (dtype == FOVEA_FP32) {
      const uint32_t e[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if ((e[i] & 0x7F800000u) == 0x7F800000u) {
          v[0][i] = __bfloat16_as_ushort(__float2bfloat16_rn(__uint_as_float(e[i])));
          v[1][i] = v[2][i] = 0u;
        } else {
          v[0][i] = e[i] >> 16;
          const float r1 = __uint_as_float(e[i]) - __uint_as_float(v[0][i] << 16);
          v[1][i] = __float_as_uint(r1) >> 16;
          v[2][i] = __float_as_uint(r1 - __uint_as_float(v[1][i] << 16)) >> 16;
        }
      }
    } else {
      const uint32_t w[2] = {a.x, a.y};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const __half h = __half(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)(w[i / 4] >> (8 * (i % 4))), __NV_E4M3));
        v[0][i] = __bfloat16_as_ushort(__float2bfloat16_rn(__half2float(h)));
        v[1][i] = v[2][i] = 0u;
      }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p)
      out[p] = make_uint4(v[p][0] | v[p][4] << 16, v[p][1] | v[p][5] << 16, v[p][2] | v[p][6] << 16,
                          v[p][3] | v[p][7] << 16);
  }
};

}  // namespace fovea
