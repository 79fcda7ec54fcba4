// Residual addition, RMS norm and an 8-bit output (fovea_add_rms_norm):
//   s = x + r,  y = s * rsqrt(mean(s^2) + eps) * gamma,
//   q = e4m3(y / scale) with scale = max|y| / 448 over a row or over `group`
//   consecutive columns of it (q = 0 where scale is 0).
// s is rounded once, to the type it is stored in; the norm and q follow from
// the unrounded fp32 sum.
#include <cuda_fp8.h>

#include <atomic>

#include "common.cuh"
#include "packed.cuh"

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
  __device__ __forceinline__ uint64_t two(int i) const {                   // columns i and i + 1
    const T* e = reinterpret_cast<const T*>(raw);
    return pack2(to_f32(e[i]), to_f32(e[i + 1]));
  }
};

// The same of a row anywhere, in three steps, so that the loads of several rows are on
// their way together (a wait within a branch for each took 7500 clocks a row): the
// aligned vectors around the chunk that lie in the row whole; the chunk cut out of them;
// and the few chunks around which a vector sticks out of the row by element.
template <class T>
struct Around {
  static constexpr int kVecs = sizeof(T) / 2, kUnit = 16 / sizeof(T);
  uint4 v[kVecs + 1];
  __device__ __forceinline__ static int off(const T* p) {                  // one for the whole row
    return (int)(reinterpret_cast<uintptr_t>(p) & 15u) / (int)sizeof(T);
  }
  __device__ __forceinline__ void load(const T* p, int c0, int d) {
    const int at = c0 - off(p);
#pragma unroll
    for (int h = 0; h <= kVecs; ++h) {
      v[h] = make_uint4(0u, 0u, 0u, 0u);
      if (at + h * kUnit >= 0 && at + (h + 1) * kUnit <= d && (h < kVecs || at != c0))
        v[h] = *reinterpret_cast<const uint4*>(p + at + h * kUnit);
    }
  }
  template <int Q>
  __device__ __forceinline__ void cut(uint32_t bits, Chunk<T>& to) const {
    uint32_t w[4 * (kVecs + 1)];
#pragma unroll
    for (int h = 0; h <= kVecs; ++h) {
      w[4 * h] = v[h].x; w[4 * h + 1] = v[h].y; w[4 * h + 2] = v[h].z; w[4 * h + 3] = v[h].w;
    }
    uint32_t r[4 * kVecs];
#pragma unroll
    for (int i = 0; i < 4 * kVecs; ++i)
      r[i] = __funnelshift_r(w[i + Q], w[i + Q + 1 < 4 * (kVecs + 1) ? i + Q + 1 : i + Q], bits);
#pragma unroll
    for (int h = 0; h < kVecs; ++h) to.raw[h] = make_uint4(r[4 * h], r[4 * h + 1], r[4 * h + 2], r[4 * h + 3]);
  }
  __device__ __forceinline__ void chunk(const T* p, Chunk<T>& to) const {
    const uint32_t bytes = off(p) * sizeof(T);
    switch (bytes >> 2) {                                  // the same in the whole CTA
      case 0: cut<0>(8 * (bytes & 3), to); break;
      case 1: cut<1>(8 * (bytes & 3), to); break;
      case 2: cut<2>(8 * (bytes & 3), to); break;
      default: cut<3>(8 * (bytes & 3), to);
    }
  }
  __device__ __forceinline__ static bool ragged(const T* p, int c0, int d) {
    const int at = c0 - off(p);
    return c0 < d && (at < 0 || at + (kVecs + (at != c0)) * kUnit > d);
  }
  __device__ __forceinline__ static void elements(const T* p, int c0, int d, Chunk<T>& to) {
    T e[kChunk];
#pragma unroll
    for (int i = 0; i < kChunk; ++i) e[i] = c0 + i < d ? p[c0 + i] : from_f32<T>(0.0f);
#pragma unroll
    for (int i = 0; i < kChunk; ++i) reinterpret_cast<T*>(to.raw)[i] = e[i];
  }
};
// The W words of each lane's chunk to rows off the vectors' boundary: aligned vectors of
// V words, cut out of a lane's chunk and the next lane's; what no vector covers (the
// warp's first and last bytes, the row's end) goes by element.  p: the chunk's place, its
// first `left` elements in the row.  All lanes of the warp.
template <class E, int Q, int W, int V>
__device__ __forceinline__ void store_cut(const uint32_t (&both)[W + V], uint32_t bits, E* p, int head, int left,
                                          bool last) {
#pragma unroll
  for (int h = 0; h < W / V; ++h) {
    if (head + (h + 1) * (4 * V / (int)sizeof(E)) > left || (last && h == W / V - 1)) continue;
    uint32_t v[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
      v[i] = __funnelshift_r(both[h * V + i + Q], both[h * V + i + Q + 1 < W + V ? h * V + i + Q + 1 : W + V - 1], bits);
    E* to = p + head + h * (4 * V / (int)sizeof(E));
    if (V == 4) *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[V - 2], v[V - 1]);
    else *reinterpret_cast<uint2*>(to) = make_uint2(v[0], v[1]);
  }
}
template <class E, int W, int V>
__device__ __forceinline__ void store_shifted(E* p, int left, const uint32_t (&w)[W]) {
  constexpr int kUnit = 4 * V / (int)sizeof(E);            // elements of a vector
  const int lane = threadIdx.x & 31;
  const int off = (int)(reinterpret_cast<uintptr_t>(p) & (4 * V - 1)) / (int)sizeof(E);    // the same in the whole row
  uint32_t both[W + V];
#pragma unroll
  for (int i = 0; i < W; ++i) both[i] = w[i];
#pragma unroll
  for (int i = 0; i < V; ++i) both[W + i] = __shfl_down_sync(0xffffffffu, w[i], 1);
  const int head = off == 0 ? 0 : kUnit - off;             // elements before the first vector's
  const int bytes = head * (int)sizeof(E);
  const uint32_t bits = 8 * (bytes & 3);
  const bool last = lane == 31 && head != 0;               // the next lane's words are not here
  switch (bytes >> 2) {
    case 0: store_cut<E, 0, W, V>(both, bits, p, head, left, last); break;
    case 1: store_cut<E, 1, W, V>(both, bits, p, head, left, last); break;
    case 2: store_cut<E, V == 4 ? 2 : 0, W, V>(both, bits, p, head, left, last); break;
    default: store_cut<E, V == 4 ? 3 : 0, W, V>(both, bits, p, head, left, last);
  }
  if (lane == 0 || last || left < 2 * kChunk) {
    const bool before = lane > 0 && head <= left;          // the lane before has stored this one's head
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      const int h = (i - head) / kUnit;                    // of i >= head: its vector
      const bool stored = i < head ? before : head + (h + 1) * kUnit <= left && !(last && h == W / V - 1);
      if (i < left && !stored)
        p[i] = reinterpret_cast<const E*>(w)[i];
    }
  }
}
template <class T>
__device__ __forceinline__ void store_chunk(T* p, int c0, int d, const float (&v)[kChunk], bool vec) {
  constexpr int kWords = kChunk * sizeof(T) / 4;
  uint32_t w[kWords];
#pragma unroll
  for (int i = 0; i < kChunk; ++i) reinterpret_cast<T*>(w)[i] = from_f32<T>(v[i]);
  if (!vec) {
    store_shifted<T, kWords, 4>(p + c0, d - c0, w);
  } else if (c0 < d) {
#pragma unroll
    for (int h = 0; h < kWords / 4; ++h)
      reinterpret_cast<uint4*>(p + c0)[h] = make_uint4(w[4 * h], w[4 * h + 1], w[4 * h + 2], w[4 * h + 3]);
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
    for (int i = 0; i < kChunk; i += 2) {
      const uint64_t two = mul2(pack2(y[i], y[i + 1]), pack2(inv, inv));
      v[i] = lo2(two);
      v[i + 1] = hi2(two);
    }
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
  if (!vec) store_shifted<uint8_t, 2, 2>(p + c0, d - c0, w);
  else if (c0 < d) *reinterpret_cast<uint2*>(p + c0) = make_uint2(w[0], w[1]);
}

// One row at a time by all threads of the CTA; thread t holds the chunks t,
// t + blockDim, ... (C of them) in registers from the load to the last store.
// blockDim is a multiple of 32, so a group of 32, 64 or 128 columns lies in 4, 8 or 16
// neighbouring lanes.  VEC: every row of every tensor is aligned, and the next row is on
// its way meanwhile; otherwise rows that are not aligned are read and written through
// shifted vectors, in 64 registers, which leaves an SM more CTAs to wait with (4096 bf16
// rows of 5111 with 8 bits by 128: 97 us against 113 in 122 registers; 139 with element
// stores and a wait for each load).
//
// One pass: a row is read once, normalised and written from registers, so memory bounds
// a long run of rows, if instructions are few (pairs of columns in packed arithmetic).
// 8192 rows of 5120 bf16 with a residual, three outputs and 8 bits in groups of 128: 61.6
// us, 6.15 TB/s (91 % of the measured copy); 63.7 without the packed arithmetic, 78
// without the next row on its way either.  One row of 4096: 1.8 us on the device, the
// call's own cost on the host is several times that.
template <class T, int C, bool VEC, bool RESIDUAL>
__global__ void __launch_bounds__(512, (VEC ? 0 : 2)) add_rms_norm_kernel(const NormArgs a) {
  __shared__ float red[2][2][16];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int d = a.d;
  Chunk<T> x[C], r[C], g[C];
  auto fetch = [&](long long row) {
    if (row >= a.N) return;
    const T* xp = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* rp = static_cast<const T*>(a.residual) + row * a.residual_ld;
    if constexpr (VEC) {
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int c0 = (c * blockDim.x + tid) * kChunk;
        x[c].load(xp, c0, d);
        if (RESIDUAL) r[c].load(rp, c0, d);
      }
    } else {
      Around<T> ax[C], ar[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int c0 = (c * blockDim.x + tid) * kChunk;
        ax[c].load(xp, c0, d);
        if (RESIDUAL) ar[c].load(rp, c0, d);
      }
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const int c0 = (c * blockDim.x + tid) * kChunk;
        ax[c].chunk(xp, x[c]);
        if (RESIDUAL) ar[c].chunk(rp, r[c]);
        if (Around<T>::ragged(xp, c0, d) || (RESIDUAL && Around<T>::ragged(rp, c0, d))) {
          Around<T>::elements(xp, c0, d, x[c]);
          if (RESIDUAL) Around<T>::elements(rp, c0, d, r[c]);
        }
      }
    }
  };
  pdl_wait();
  pdl_trigger();
  if (VEC) fetch(blockIdx.x);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int c0 = (c * blockDim.x + tid) * kChunk;
    const T* gp = static_cast<const T*>(a.gamma);
    if (VEC) {
      g[c].load(gp, c0, d);
    } else {
      Around<T> ag;
      ag.load(gp, c0, d);
      ag.chunk(gp, g[c]);
      if (Around<T>::ragged(gp, c0, d)) Around<T>::elements(gp, c0, d, g[c]);
    }
  }
  const bool vec = VEC || a.out_vec;
  const int groups = a.q8_group != 0 ? (d + a.q8_group - 1) / a.q8_group : 1;
  int buf = 0;
  for (long long row = blockIdx.x; row < a.N; row += gridDim.x, buf ^= 1) {
    if (!VEC) fetch(row);
    float s[C][kChunk];
    uint64_t squares = 0;
    float top = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < kChunk; i += 2) {
        uint64_t v = x[c].two(i);
        if (RESIDUAL) v = add2(v, r[c].two(i));
        squares = fma2(v, v, squares);
        const uint64_t y = mul2(v, g[c].two(i));
        top = max_nan(max_nan(top, fabsf(lo2(y))), fabsf(hi2(y)));
        s[c][i] = lo2(v);
        s[c][i + 1] = hi2(v);
      }
    float ss = lo2(squares) + hi2(squares);
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
      for (int i = 0; i < kChunk; i += 2) {
        const uint64_t v = mul2(mul2(pack2(s[c][i], s[c][i + 1]), pack2(rstd, rstd)), g[c].two(i));
        y[i] = lo2(v);
        y[i + 1] = hi2(v);
      }
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
  // done sooner with one (64 rows of 4096: 2.75 us against 3.22; 8192 rows 41.1 against
  // 37.4), and so are rows that need shifting (4096 fp32 rows of 3001: 51 against 55)
  const int per = chunks <= 128 || ((a.N <= 2 * 152 || !vec) && chunks <= 512) ? 1 : 2;
  const int threads = (chunks + per * 32 - 1) / (per * 32) * 32;
  return dtype == FOVEA_BF16 ? launch<__nv_bfloat16>(a, threads, per, vec, s) : launch<float>(a, threads, per, vec, s);
}

}  // namespace fovea
