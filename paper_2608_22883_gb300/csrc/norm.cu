// Residual addition, RMS norm and an 8-bit output (fovea_add_rms_norm):
//   s = x + r,  y = s * rsqrt(mean(s^2) + eps) * gamma,
//   q = e4m3(y / scale) with scale = max|y| / 448 over a row or over `group`
//   consecutive columns of it (q = 0 where scale is 0).
// s is rounded once, to the type it is stored in; the norm and q follow from
// the unrounded fp32 sum.
#include <cuda_fp8.h>

#include <atomic>

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

// Columns [c0, c0 + 8) of a row as they lie in memory; columns from d on are 0.  Where
// the row is off the vectors' boundary, whole chunks are cut out of the aligned vectors
// around them, which lie within the row but for its first and last chunk; those go by
// element.
template <class T>
struct Chunk {
  static constexpr int kVecs = sizeof(T) / 2;
  uint4 raw[kVecs];
  __device__ __forceinline__ void load(const T* p, int c0, int d) {        // of an aligned row
#pragma unroll
    for (int h = 0; h < kVecs; ++h) raw[h] = make_uint4(0u, 0u, 0u, 0u);
    if (c0 < d) {
#pragma unroll
      for (int h = 0; h < kVecs; ++h) raw[h] = reinterpret_cast<const uint4*>(p + c0)[h];
    }
  }
  __device__ __forceinline__ void load_any(const T* p, int c0, int d) {
#pragma unroll
    for (int h = 0; h < kVecs; ++h) raw[h] = make_uint4(0u, 0u, 0u, 0u);
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 15u);     // one for the whole row
    const T* from = p + c0 - off / sizeof(T);
    if (from >= p && c0 + kChunk + 16 / (int)sizeof(T) <= d) {
      uint32_t w[4 * (kVecs + 1)], v[4 * kVecs];
#pragma unroll
      for (int h = 0; h <= kVecs; ++h) {
        const uint4 u = reinterpret_cast<const uint4*>(from)[h];
        w[4 * h] = u.x; w[4 * h + 1] = u.y; w[4 * h + 2] = u.z; w[4 * h + 3] = u.w;
      }
      const uint32_t bits = 8 * (off & 3);
      switch (off >> 2) {                                  // the same in the whole CTA
        case 0: cut<0>(w, bits, v); break;
        case 1: cut<1>(w, bits, v); break;
        case 2: cut<2>(w, bits, v); break;
        default: cut<3>(w, bits, v);
      }
#pragma unroll
      for (int h = 0; h < kVecs; ++h) raw[h] = make_uint4(v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]);
    } else {
      T* e = reinterpret_cast<T*>(raw);
#pragma unroll
      for (int i = 0; i < kChunk; ++i)
        if (c0 + i < d) e[i] = p[c0 + i];
    }
  }
  template <int Q>
  __device__ __forceinline__ static void cut(const uint32_t (&w)[4 * (kVecs + 1)], uint32_t bits, uint32_t (&v)[4 * kVecs]) {
#pragma unroll
    for (int i = 0; i < 4 * kVecs; ++i) v[i] = __funnelshift_r(w[i + Q], w[i + Q + 1 < 4 * (kVecs + 1) ? i + Q + 1 : i + Q], bits);
  }
  __device__ __forceinline__ float at(int i) const { return to_f32(reinterpret_cast<const T*>(raw)[i]); }
};
template <class T>
__device__ __forceinline__ void store_chunk(T* p, int c0, int d, const float (&v)[kChunk], bool vec) {
  if (vec) {
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
// The chunk of y in e4m3 at the given scale.  y / scale is y times the scale's
// reciprocal where both are normal numbers (off by 2^-21 of itself at most; e4m3's step
// is 2^-4).
__device__ __forceinline__ void store_q8(uint8_t* p, int c0, int d, const float (&y)[kChunk],
                                         float scale, bool vec) {
  float v[kChunk];
  if (scale > 1e-30f && scale < 1e30f) {
    const float inv = __fdividef(1.0f, scale);
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = y[i] * inv;
  } else {
#pragma unroll
    for (int i = 0; i < kChunk; ++i) v[i] = scale == 0.0f ? 0.0f : y[i] / scale;
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h], v[4 * h + 1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * h + 2], v[4 * h + 3]), __NV_SATFINITE, __NV_E4M3);
    w[h] = lo | hi << 16;
  }
  if (vec) {
    if (c0 < d) *reinterpret_cast<uint2*>(p + c0) = make_uint2(w[0], w[1]);
  } else {
#pragma unroll
    for (int i = 0; i < kChunk; ++i)
      if (c0 + i < d) p[c0 + i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
}

// One row at a time by all threads of the CTA; thread t holds the chunks t,
// t + blockDim, ... (C of them) in registers from the load to the last store.
// blockDim is a multiple of 32, so a group of 32, 64 or 128 columns lies in 4, 8 or 16
// neighbouring lanes.  VEC: every row of every tensor is aligned, and the next row is on
// its way meanwhile; otherwise (fewer registers, more CTAs an SM) rows that are not
// aligned are read through shifted vectors, and written by element.
//
// One pass: a row is read once, normalised and written from registers, so memory bounds
// a long run of rows.  8192 rows of 5120 bf16 with a residual, three outputs and 8 bits
// in groups of 128: 63.4 us, 5.97 TB/s (88 % of the measured copy); without the next
// row on its way 78 us.  One row of 4096: 1.8 us on the device, the call's own cost on
// the host is several times that.
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
      const T* xp = static_cast<const T*>(a.x) + row * a.x_ld;
      const T* rp = static_cast<const T*>(a.residual) + row * a.residual_ld;
      if (VEC) x[c].load(xp, c0, d);
      else x[c].load_any(xp, c0, d);
      if (RESIDUAL && VEC) r[c].load(rp, c0, d);
      else if (RESIDUAL) r[c].load_any(rp, c0, d);
    }
  };
  pdl_wait();
  pdl_trigger();
  if (VEC) fetch(blockIdx.x);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (VEC) g[c].load(static_cast<const T*>(a.gamma), (c * blockDim.x + tid) * kChunk, d);
    else g[c].load_any(static_cast<const T*>(a.gamma), (c * blockDim.x + tid) * kChunk, d);
  }
  const bool vec = VEC || a.out_vec;
  const int groups = a.q8_group != 0 ? (d + a.q8_group - 1) / a.q8_group : 1;
  int buf = 0;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, buf ^= 1) {
    if (!VEC) fetch(row);
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
    if (VEC) fetch(row + gridDim.x);
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
        store_chunk(static_cast<T*>(a.sum) + row * d, (c * blockDim.x + tid) * kChunk, d, s[c], vec);
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
    const float row_scale = top * rstd * (1.0f / kE4m3Max);
    if (a.q8 != nullptr && a.q8_group == 0 && tid == 0) a.q8_scale[row] = row_scale;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int c0 = (c * blockDim.x + tid) * kChunk;
      if (!RESIDUAL && a.sum != nullptr) store_chunk(static_cast<T*>(a.sum) + row * d, c0, d, s[c], vec);
      float y[kChunk];
#pragma unroll
      for (int i = 0; i < kChunk; ++i) y[i] = s[c][i] * rstd * g[c].at(i);
      if (a.out != nullptr) store_chunk(static_cast<T*>(a.out) + row * d, c0, d, y, vec);
      if (a.q8 == nullptr) continue;
      float scale = row_scale;
      if (a.q8_group != 0) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kChunk; ++i) m = max_nan(m, fabsf(y[i]));
        for (int o = a.q8_group / kChunk / 2; o > 0; o >>= 1)
          m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
        scale = m * (1.0f / kE4m3Max);
        if (c0 < d && (c0 & (a.q8_group - 1)) == 0) a.q8_scale[row * groups + c0 / a.q8_group] = scale;
      }
      store_q8(a.q8 + row * d, c0, d, y, scale, vec);
    }
  }
}

template <class T, int C, bool VEC, bool RESIDUAL>
cudaError_t launch(const NormArgs& a, int threads, cudaStream_t s) {
  auto kern = add_rms_norm_kernel<T, C, VEC, RESIDUAL>;
  static std::atomic<int> known[17];                       // CTAs an SM, by warps (asking takes a microsecond)
  int resident = known[threads / 32].load(std::memory_order_relaxed);
  if (resident == 0) {
    const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&resident, kern, threads, 0);
    if (e != cudaSuccess) return e;
    if (resident < 1) return cudaErrorInvalidConfiguration;
    known[threads / 32].store(resident, std::memory_order_relaxed);
  }
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

cudaError_t launch_add_rms_norm(int dtype, NormArgs a, cudaStream_t s) {
  const size_t size = dtype == FOVEA_BF16 ? 2 : 4;
  auto aligned = [](const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
  const bool whole = a.d % kChunk == 0;                    // and so are the dense rows
  a.out_vec = whole && aligned(a.sum, 16) && aligned(a.out, 16) && aligned(a.q8, 8);
  const bool vec = a.out_vec && aligned(a.gamma, 16) && aligned(a.x, 16) && a.x_ld * size % 16 == 0 &&
                   aligned(a.residual, 16) && a.residual_ld * size % 16 == 0;
  const int chunks = (a.d + kChunk - 1) / kChunk;
  // two chunks a thread halve the reductions' share of a long run of rows; a few rows are
  // done sooner with one (64 rows of 4096: 2.75 us against 3.22; 8192 rows 41.1 against 37.4)
  const int per = chunks <= 128 || (a.N <= 2 * 152 && chunks <= 512) ? 1 : 2;
  const int threads = (chunks + per * 32 - 1) / (per * 32) * 32;
  return dtype == FOVEA_BF16 ? launch<__nv_bfloat16>(a, threads, per, vec, s) : launch<float>(a, threads, per, vec, s);
}

}  // namespace fovea
