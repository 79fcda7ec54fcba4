// Residual addition, RMS norm and an 8-bit output (fovea_add_rms_norm):
//   s = x + r,  y = s * rsqrt(mean(s^2) + eps) * gamma,
//   q = e4m3(y / scale) with scale = max|y| / 448 over a row or over `group`
//   consecutive columns of it (q = 0 where scale is 0).
// s is rounded once, to the type it is stored in; the norm and q follow from
// the unrounded fp32 sum.
#include <cuda_fp8.h>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kChunk = 8;            // columns a thread handles together

// max of magnitudes that a NaN wins (fmaxf would drop it, and a row with a NaN
// would get a finite scale).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Columns [c0, c0 + 8) of a row as they lie in memory; columns from d on are 0.
template <class T>
struct Chunk {
  uint4 raw[sizeof(T) / 2];
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p, int c0, int d) {
    constexpr int kVecs = sizeof(T) / 2;
#pragma unroll
    for (int h = 0; h < kVecs; ++h) raw[h] = make_uint4(0u, 0u, 0u, 0u);
    if (VEC) {
      if (c0 < d) {
#pragma unroll
        for (int h = 0; h < kVecs; ++h) raw[h] = reinterpret_cast<const uint4*>(p + c0)[h];
      }
    } else {
      T* e = reinterpret_cast<T*>(raw);
#pragma unroll
      for (int i = 0; i < kChunk; ++i)
        if (c0 + i < d) e[i] = p[c0 + i];
    }
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(reinterpret_cast<const T*>(raw)[i]); }
};
template <class T, bool VEC>
__device__ __forceinline__ void store_chunk(T* p, int c0, int d, const float (&v)[kChunk]) {
  if (VEC) {
    if (c0 < d) {
      __align__(16) T e[kChunk];
#pragma unroll
      for (int i = 0; i < kChunk; ++i) e[i] = from_f32<T>(v[i]);
#pragma unroll
      for (int h = 0; h < (int)(kChunk * sizeof(T) / 16); ++h)
        reinterpret_cast<uint4*>(p + c0)[h] = reinterpret_cast<const uint4*>(e)[h];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
      if (c0 + i < d) p[c0 + i] = from_f32<T>(v[i]);
  }
}
// The chunk of y in e4m3 at the given scale.  y / scale is y times the
// scale's reciprocal where that is a normal number (one rounding more: the
// quotient is off by 2^-23 of itself at most, e4m3's step is 2^-4).
template <bool VEC>
__device__ __forceinline__ void store_q8(uint8_t* p, int c0, int d, const float (&y)[kChunk],
                                         float scale) {
  float v[kChunk];
  const bool normal = scale > 1e-30f;
  const float inv = 1.0f / scale;
#pragma unroll
  for (int i = 0; i < kChunk; ++i) v[i] = scale == 0.0f ? 0.0f : normal ? y[i] * inv : y[i] / scale;
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h], v[4 * h + 1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h + 2], v[4 * h + 3]), __NV_SATFINITE, __NV_E4M3);
    w[h] = lo | hi << 16;
  }
  if (VEC) {
    if (c0 < d) *reinterpret_cast<uint2*>(p + c0) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
      if (c0 + i < d) p[c0 + i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// One row at a time by all threads of the CTA; thread t holds the chunks t,
// t + blockDim, ... (C of them) in registers from the load to the last store, and
// the next row's are on their way meanwhile.  blockDim is a multiple of 32, so a group
// of 32, 64 or 128 columns lies in 4, 8 or 16 neighbouring lanes.
template <class T, int C, bool VEC, bool RESIDUAL>
__global__ void __launch_bounds__(512) add_rms_norm_kernel(const NormArgs a) {
  __shared__ float red[2][2][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int d = a.d;
  Chunk<T> x[C], r[C], g[C];
  auto fetch = [&](long long row) {
    if (row >= a.N) return;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int c0 = (c * blockDim.x + tid) * kChunk;
      x[c].template load<VEC>(static_cast<const T*>(a.x) + row * a.x_ld, c0, d);
      if (RESIDUAL) r[c].template load<VEC>(static_cast<const T*>(a.residual) + row * a.residual_ld, c0, d);
    }
  };
  pdl_wait();
  pdl_trigger();
  fetch(blockIdx.x);
#pragma unroll
  for (int c = 0; c < C; ++c)
    g[c].template load<VEC>(static_cast<const T*>(a.gamma), (c * blockDim.x + tid) * kChunk, d);
  const int groups = a.q8_group != 0 ? (d + a.q8_group - 1) / a.q8_group : 1;
  int buf = 0;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, buf ^= 1) {
    float s[C][kChunk];
    float ss = 0.0f, top = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < kChunk; ++i) {
        s[c][i] = RESIDUAL ? x[c].at(i) + r[c].at(i) : x[c].at(i);
        ss = fmaf(s[c][i], s[c][i], ss);
        top = max_nan(top, fabsf(s[c][i] * g[c].at(i)));
      }
    fetch(row + gridDim.x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(0xffffffffu, ss, o);
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    // two buffers: a warp may write the next row's while another still reads
    if (lane == 0) {
      red[buf][0][warp] = ss;
      red[buf][1][warp] = top;
    }
    if (RESIDUAL && a.sum != nullptr) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        store_chunk<T, VEC>(static_cast<T*>(a.sum) + row * d, (c * blockDim.x + tid) * kChunk, d, s[c]);
    }
    __syncthreads();
    const int w = lane & 15;                               // of at most 16 warps, in both halves
    ss = w < warps ? red[buf][0][w] : 0.0f;
    top = w < warps ? red[buf][1][w] : 0.0f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      ss += __shfl_xor_sync(0xffffffffu, ss, o);
      top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    }
    const float rstd = __frsqrt_rn(ss / (float)d + a.eps);
    // max |y| is max |s gamma| times rstd, so that a row's scale needs no
    // second pass over its threads
    const float row_scale = top * rstd / kE4m3Max;
    if (a.q8 != nullptr && a.q8_group == 0 && tid == 0) a.q8_scale[row] = row_scale;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int c0 = (c * blockDim.x + tid) * kChunk;
      if (!RESIDUAL && a.sum != nullptr) store_chunk<T, VEC>(static_cast<T*>(a.sum) + row * d, c0, d, s[c]);
      float y[kChunk];
#pragma unroll
      for (int i = 0; i < kChunk; ++i) y[i] = s[c][i] * rstd * g[c].at(i);
      if (a.out != nullptr) store_chunk<T, VEC>(static_cast<T*>(a.out) + row * d, c0, d, y);
      if (a.q8 == nullptr) continue;
      float scale = row_scale;
      if (a.q8_group != 0) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) m = max_nan(m, fabsf(y[i]));
        for (int o = a.q8_group / kChunk / 2; o > 0; o >>= 1)
          m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
        scale = m / kE4m3Max;
        if (c0 < d && (c0 & (a.q8_group - 1)) == 0) a.q8_scale[row * groups + c0 / a.q8_group] = scale;
      }
      store_q8<VEC>(a.q8 + row * d, c0, d, y, scale);
    }
  }
}

template <class T, int C, bool VEC, bool RESIDUAL>
cudaError_t launch(const NormArgs& a, int threads, cudaStream_t s) {
  auto kern = add_rms_norm_kernel<T, C, VEC, RESIDUAL>;
  int resident = 0;
  const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kern, threads, 0);
  if (e != cudaSuccess) return e;
  const long long most = 152ll * resident;
  return launch_pdl(kern, dim3((unsigned)(a.N < most ? a.N : most)), dim3(threads), 0, s, a);
}
template <class T>
cudaError_t launch(const NormArgs& a, int threads, int per, bool vec, cudaStream_t s) {
  if (a.residual != nullptr) {
    if (per == 1) return vec ? launch<T, 1, true, true>(a, threads, s) : launch<T, 1, false, true>(a, threads, s);
    return vec ? launch<T, 2, true, true>(a, threads, s) : launch<T, 2, false, true>(a, threads, s);
  }
  if (per == 1) return vec ? launch<T, 1, true, false>(a, threads, s) : launch<T, 1, false, false>(a, threads, s);
  return vec ? launch<T, 2, true, false>(a, threads, s) : launch<T, 2, false, false>(a, threads, s);
}

}  // namespace

cudaError_t launch_add_rms_norm(int dtype, const NormArgs& a, cudaStream_t s) {
  const size_t size = dtype == FOVEA_BF16 ? 2 : 4;
  auto aligned = [](const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  const bool vec = a.d % kChunk == 0 && aligned(a.x, 16) && aligned(a.residual, 16) &&
                   aligned(a.gamma, 16) && aligned(a.sum, 16) && aligned(a.out, 16) &&
                   aligned(a.q8, 8) && a.x_ld * size % 16 == 0 && a.residual_ld * size % 16 == 0;
  const int chunks = (a.d + kChunk - 1) / kChunk;
  const int per = chunks <= 128 ? 1 : 2;
  const int threads = (chunks + per * 32 - 1) / (per * 32) * 32;
  return dtype == FOVEA_BF16 ? launch<__nv_bfloat16>(a, threads, per, vec, s) : launch<float>(a, threads, per, vec, s);
}

}  // namespace fovea
