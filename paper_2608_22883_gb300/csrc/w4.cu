// Weights in 4 bits with a scale (and a zero point) per group of columns:
// their making (fovea_quantize_w4) and the product with a few rows
// (fovea_linear_w4).
//   w[o, k] = (code[o, k] - zero[o, k / group]) * scale[o, k / group]
#include <cuda_fp8.h>

#include "common.cuh"

namespace fovea {

namespace {

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// ---------------------------------------------------------------------------
// Codes, scales and zero points of a matrix
// ---------------------------------------------------------------------------

constexpr int kQuantThreads = 256;

// Eight columns a thread, so that a group of 32, 64 or 128 columns is 4, 8 or
// 16 neighbouring lanes; each row is laid out over a multiple of 16 lanes
// (`slots`), so that no group crosses a warp.  Scale and code use IEEE
// divisions: the codes are those of the definition, bit for bit.
template <class T, bool VEC>
__global__ void __launch_bounds__(kQuantThreads)
quantize_w4_kernel(const T* __restrict__ W, long long ld, int in, int slots, long long total, int group,
                   bool symmetric, uint8_t* __restrict__ codes, __nv_bfloat16* __restrict__ scales,
                   uint8_t* __restrict__ zeros) {
  pdl_wait();
  pdl_trigger();
  const int groups = (in + group - 1) / group;
  const long long step = (long long)gridDim.x * kQuantThreads;
  // every lane of a warp takes the same number of turns: total is a multiple of 16
  // and the tail's lanes run with nothing in hand
  for (long long base = (long long)blockIdx.x * kQuantThreads; base < total; base += step) {
    const long long i = base + threadIdx.x;
    const long long row = i / slots;
    const int c0 = (int)(i - row * slots) * 8;
    const bool live = i < total && c0 < in;
    float w[8];
    if (live) {
      const T* p = W + row * ld + c0;
      if (VEC) {
        uint4 raw[sizeof(T) / 2];
#pragma unroll
        for (int h = 0; h < (int)(sizeof(T) / 2); ++h) raw[h] = reinterpret_cast<const uint4*>(p)[h];
        const T* e = reinterpret_cast<const T*>(raw);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = to_f32(e[j]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = to_f32(p[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = 0.0f;
    }
    float hi = 0.0f, lo = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      hi = max_nan(hi, symmetric ? fabsf(w[j]) : w[j]);
      lo = symmetric ? 0.0f : min_nan(lo, w[j]);
    }
    for (int o = group / 16; o > 0; o >>= 1) {
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    }
    const __nv_bfloat16 stored = __float2bfloat16_rn(symmetric ? __fdiv_rn(hi, 7.0f) : __fdiv_rn(hi - lo, 15.0f));
    const float scale = __bfloat162float(stored);
    const bool some = scale > 0.0f;
    float zero = 8.0f;
    if (!symmetric && some) zero = fminf(fmaxf(rintf(__fdiv_rn(-lo, scale)), 0.0f), 15.0f);
    uint32_t word = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = some ? rintf(__fdiv_rn(w[j], scale)) : 0.0f;
      const float code = fminf(fmaxf(q, -zero), 15.0f - zero) + zero;
      word |= (uint32_t)code << (4 * j);
    }
    if (live) {
      *reinterpret_cast<uint32_t*>(codes + (row * in + c0) / 2) = word;
      if (c0 % group == 0) {
        const long long at = row * groups + c0 / group;
        scales[at] = stored;
        if (zeros != nullptr) zeros[at] = (uint8_t)zero;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Product with a few rows
// ---------------------------------------------------------------------------

constexpr int kWarps = 16, kThreads = kWarps * 32;
constexpr int kSpan = 128;             // columns a warp handles together
constexpr int kTileRows = 16;          // weight rows of a tile

// Offset within a span of the eight columns of word j of lane quarter t: the
// four quarters of a warp's lanes share the sum of one tensor-core product, so
// the columns of one product lie in one group.  A group of 128 columns lets a lane
// read 16 bytes in a row, 64 columns 8 and 32 columns 4.
template <int G>
__device__ __forceinline__ int word_column(int j, int t) {
  if (G == 128) return 32 * t + 8 * j;
  if (G == 64) return 64 * (j >> 1) + 16 * t + 8 * (j & 1);
  return 32 * j + 8 * t;
}

__device__ __forceinline__ uint32_t bf16_sub2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                            uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// One span of codes of weight rows g and g + 8 with their scales and zeros.
template <int G>
struct Span {
  uint32_t w[2][4];
  __nv_bfloat16 s[2][kSpan / G];
  uint8_t z[2][kSpan / G];
};

template <int G>
__device__ __forceinline__ void load_span(Span<G>& r, const W4& w, int groups, long long row0,
                                          int span, int lane) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // rows past the end repeat the last one (their results are not stored)
    const long long row = min(row0 + g + 8 * h, (long long)w.out - 1);
    const uint8_t* p = w.codes + row * (w.in / 2);
    constexpr int kWords = G / 32;               // words in a row of bytes
#pragma unroll
    for (int j = 0; j < 4; j += kWords) {
      const int k = span * kSpan + word_column<G>(j, t);
#pragma unroll
      for (int i = 0; i < kWords; ++i) r.w[h][j + i] = 0u;
      if (k + 8 * kWords <= w.in) {
        if (kWords == 4) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p + k / 2));
          r.w[h][0] = v.x; r.w[h][1] = v.y; r.w[h][2] = v.z; r.w[h][3] = v.w;
        } else if (kWords == 2) {
          const uint2 v = __ldg(reinterpret_cast<const uint2*>(p + k / 2));
          r.w[h][j] = v.x; r.w[h][j + 1] = v.y;
        } else {
          r.w[h][j] = __ldg(reinterpret_cast<const uint32_t*>(p + k / 2));
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kSpan / G; ++i) {
      const int gi = span * (kSpan / G) + i;
      const bool in = gi < groups;
      r.s[h][i] = in ? w.scales[row * groups + gi] : __nv_bfloat16(0.0f);
      r.z[h][i] = in && w.zeros != nullptr ? w.zeros[row * groups + gi] : 8;
    }
  }
}

// y of up to 8 NT columns (rows of x, an fp32 row as three) in one launch.
//
// A persistent CTA takes every gridDim.x-th tile of 16 weight rows.  Its warps
// split the tile's spans; each turns its codes into bf16 integers c - z (exact)
// and multiplies them on the tensor cores, weights as the 16-row operand, with
// x from shared memory; a group's fp32 sum is then taken times its scale.  The
// warps' partial tiles meet in shared memory in a fixed order.
//
// fp32 rows enter as three bf16 rows that add up to them exactly; e4m3 rows are
// exact in bf16 and their scales join the group's or the result.
template <int G, int NT>
__global__ void __launch_bounds__(kThreads) linear_w4_kernel(const LinearW4Args a, int n0, int n1) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int parts = a.x_dtype == FOVEA_FP32 ? 3 : 1;
  const int rows = n1 - n0, cols = rows * parts;
  const int spans = (a.w.in + kSpan - 1) / kSpan;
  const int groups = (a.w.in + G - 1) / G;
  // [span][word][quarter][column] units of eight x values; partial tiles
  // [warp][row][column]; scales of x [group][column]
  uint4* xs = reinterpret_cast<uint4*>(smem);
  float* part = reinterpret_cast<float*>(xs + (long long)spans * 16 * cols);
  float* xscale = part + kWarps * kTileRows * 8 * NT;
  const long long tiles = ((long long)a.w.out + kTileRows - 1) / kTileRows;

  pdl_wait();
  pdl_trigger();
  // x, eight columns at a time, in the order in which the codes of a word
  // come out of it: columns 0 4 1 5 2 6 3 7
  for (int u = tid; u < spans * 16 * rows; u += kThreads) {
    const int n = u / (spans * 16), unit = u - n * (spans * 16);
    const int span = unit >> 4, k8 = unit & 15;
    int j, q;                                  // word and quarter of these columns
    if (G == 128) { q = k8 >> 2; j = k8 & 3; }
    else if (G == 64) { j = 2 * (k8 >> 3) + (k8 & 1); q = (k8 & 7) >> 1; }
    else { j = k8 >> 2; q = k8 & 3; }
    const int k0 = unit * 8;
    const long long at = (long long)(n0 + n) * a.x_ld + k0;
    uint32_t pk[3][4] = {};
    if (k0 < a.w.in) {
      constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t b0 = 0, b1 = 0, b2 = 0;
        if (a.x_dtype == FOVEA_BF16) {
          b0 = static_cast<const uint16_t*>(a.x)[at + order[i]];
        } else if (a.x_dtype == FOVEA_FP32) {
          const float v = static_cast<const float*>(a.x)[at + order[i]];
          const uint32_t bits = __float_as_uint(v);
          if ((bits & 0x7F800000u) == 0x7F800000u) {       // infinity, NaN
            b0 = __bfloat16_as_ushort(__float2bfloat16_rn(v));
          } else {                                         // v is the sum of its three truncations
            b0 = bits >> 16;
            const float r1 = v - __uint_as_float(b0 << 16);
            b1 = __float_as_uint(r1) >> 16;
            b2 = __float_as_uint(r1 - __uint_as_float(b1 << 16)) >> 16;
          }
        } else {
          const __half h = __half(__nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(a.x)[at + order[i]], __NV_E4M3));
          b0 = __bfloat16_as_ushort(__float2bfloat16_rn(__half2float(h)));
        }
        pk[0][i / 2] |= b0 << (16 * (i & 1));
        pk[1][i / 2] |= b1 << (16 * (i & 1));
        pk[2][i / 2] |= b2 << (16 * (i & 1));
      }
    }
    for (int p = 0; p < parts; ++p)
      xs[((span * 4 + j) * 4 + q) * cols + n * parts + p] =
          p == 0 ? make_uint4(pk[0][0], pk[0][1], pk[0][2], pk[0][3])
                 : p == 1 ? make_uint4(pk[1][0], pk[1][1], pk[1][2], pk[1][3])
                          : make_uint4(pk[2][0], pk[2][1], pk[2][2], pk[2][3]);
  }
  const bool by_group = a.x_scale != nullptr && a.x_group != 0;
  if (by_group)
    for (int u = tid; u < groups * cols; u += kThreads)
      xscale[u] = a.x_scale[(long long)(n0 + u % cols) * groups + u / cols];
  __syncthreads();

  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    float acc[NT][4] = {};
    for (int span = warp; span < spans; span += kWarps) {
      Span<G> r;
      load_span<G>(r, a.w, groups, tile * kTileRows, span, lane);
#pragma unroll
      for (int i = 0; i < kSpan / G; ++i) {
        float sum[NT][4] = {};
        const uint32_t z0 = 0x43004300u | r.z[0][i] * 0x10001u, z1 = 0x43004300u | r.z[1][i] * 0x10001u;
#pragma unroll
        for (int jj = 0; jj < G / 32; ++jj) {
          const int j = i * (G / 32) + jj;
          uint32_t w0[4], w1[4];               // column pairs 0 4, 1 5, 2 6, 3 7
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            // 0x4300 | c is the bf16 number 128 + c
            w0[p] = bf16_sub2(((r.w[0][j] >> (4 * p)) & 0x000F000Fu) | 0x43004300u, z0);
            w1[p] = bf16_sub2(((r.w[1][j] >> (4 * p)) & 0x000F000Fu) | 0x43004300u, z1);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint4 b = make_uint4(0u, 0u, 0u, 0u);
            if (nt * 8 + g < cols) b = xs[((span * 4 + j) * 4 + t) * cols + nt * 8 + g];
            mma_16x8x16(sum[nt], w0[0], w1[0], w0[1], w1[1], b.x, b.y);
            mma_16x8x16(sum[nt], w0[2], w1[2], w0[3], w1[3], b.z, b.w);
          }
        }
        const float s0 = __bfloat162float(r.s[0][i]), s1 = __bfloat162float(r.s[1][i]);
        const int gi = span * (kSpan / G) + i;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float x0 = 1.0f, x1 = 1.0f;
          if (by_group && gi < groups) {
            const int n = nt * 8 + 2 * t;
            x0 = n < cols ? xscale[gi * cols + n] : 0.0f;
            x1 = n + 1 < cols ? xscale[gi * cols + n + 1] : 0.0f;
          }
          acc[nt][0] = fmaf(sum[nt][0], s0 * x0, acc[nt][0]);
          acc[nt][1] = fmaf(sum[nt][1], s0 * x1, acc[nt][1]);
          acc[nt][2] = fmaf(sum[nt][2], s1 * x0, acc[nt][2]);
          acc[nt][3] = fmaf(sum[nt][3], s1 * x1, acc[nt][3]);
        }
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[(warp * kTileRows + g + 8 * (e >> 1)) * 8 * NT + nt * 8 + 2 * t + (e & 1)] = acc[nt][e];
    __syncthreads();
    for (int u = tid; u < kTileRows * rows; u += kThreads) {
      const int r = u & (kTileRows - 1), n = u / kTileRows;
      const long long o = tile * kTileRows + r;
      float v = 0.0f;
      for (int w = 0; w < kWarps; ++w)
        for (int p = 0; p < parts; ++p) v += part[(w * kTileRows + r) * 8 * NT + n * parts + p];
      if (o < a.w.out) {
        if (a.x_scale != nullptr && a.x_group == 0) v *= a.x_scale[n0 + n];
        if (a.bias != nullptr) v += a.bias[o];
        const long long at = (long long)(n0 + n) * a.w.out + o;
        if (a.y_dtype == FOVEA_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.y)[at] = v;
      }
    }
    __syncthreads();
  }
}

template <int G, int NT>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, size_t smem, int grid, cudaStream_t s) {
  cudaError_t e = cudaFuncSetAttribute(linear_w4_kernel<G, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       227 * 1024);
  if (e != cudaSuccess) return e;
  return launch_pdl(linear_w4_kernel<G, NT>, dim3(grid), dim3(kThreads), smem, s, a, n0, n1);
}

}  // namespace

cudaError_t launch_quantize_w4(int dtype, const void* W, long long ld, int out, int in, int group,
                               uint8_t* codes, __nv_bfloat16* scales, uint8_t* zeros, cudaStream_t s) {
  const int slots = (in / 8 + 15) / 16 * 16;
  const long long total = (long long)slots * out;
  const long long blocks = (total + kQuantThreads - 1) / kQuantThreads;
  const int grid = (int)(blocks < 152 * 8 ? blocks : 152 * 8);
  const bool symmetric = zeros == nullptr;
  const size_t size = dtype == FOVEA_BF16 ? 2 : 4;
  const bool vec = (reinterpret_cast<uintptr_t>(W) & 15u) == 0 && ld * size % 16 == 0;
  auto go = [&](auto kern, auto* w) {
    return launch_pdl(kern, dim3(grid), dim3(kQuantThreads), 0, s, w, ld, in, slots, total, group, symmetric,
                      codes, scales, zeros);
  };
  if (dtype == FOVEA_BF16) {
    const __nv_bfloat16* w = static_cast<const __nv_bfloat16*>(W);
    return vec ? go(quantize_w4_kernel<__nv_bfloat16, true>, w) : go(quantize_w4_kernel<__nv_bfloat16, false>, w);
  }
  const float* w = static_cast<const float*>(W);
  return vec ? go(quantize_w4_kernel<float, true>, w) : go(quantize_w4_kernel<float, false>, w);
}

// Rows (an fp32 row counts three times) from which the codes go through tensor
// memory instead of each warp's registers.
constexpr int kFewCols = 16;
static bool few_rows(int N, int x_dtype) { return (long long)N * (x_dtype == FOVEA_FP32 ? 3 : 1) <= kFewCols; }

size_t linear_w4_workspace(int N, int in, int group, int x_dtype, bool by_group) {
  return few_rows(N, x_dtype) ? 0 : linear_w4_tc_workspace(N, in, group, x_dtype, by_group);
}

cudaError_t launch_linear_w4(const LinearW4Args& a, cudaStream_t s) {
  if (!few_rows(a.N, a.x_dtype)) return launch_linear_w4_tc(a, s);
  const int parts = a.x_dtype == FOVEA_FP32 ? 3 : 1;
  const long long spans = (a.w.in + kSpan - 1) / kSpan;
  const int groups = (a.w.in + a.w.group - 1) / a.w.group;
  // as many rows a launch as shared memory and 16 columns hold
  const long long col_bytes = spans * 16 * 16 + (a.x_group != 0 ? 4ll * groups : 0);
  const long long room = 227 * 1024 - kWarps * kTileRows * 16 * 4;
  long long rows = std::min<long long>(16 / parts, room / (col_bytes * parts));
  if (rows < 1) return cudaErrorInvalidValue;
  const long long tiles = ((long long)a.w.out + kTileRows - 1) / kTileRows;
  const int grid = (int)std::min<long long>(tiles, 152);
  for (int n0 = 0; n0 < a.N; n0 += (int)rows) {
    const int n1 = (int)std::min<long long>(a.N, n0 + rows);
    const int cols = (n1 - n0) * parts;
    const int nt = cols <= 8 ? 1 : 2;
    const size_t smem = cols * col_bytes + kWarps * kTileRows * 8 * nt * 4;
    cudaError_t e;
    if (a.w.group == 128) e = nt == 1 ? launch_few<128, 1>(a, n0, n1, smem, grid, s) : launch_few<128, 2>(a, n0, n1, smem, grid, s);
    else if (a.w.group == 64) e = nt == 1 ? launch_few<64, 1>(a, n0, n1, smem, grid, s) : launch_few<64, 2>(a, n0, n1, smem, grid, s);
    else e = nt == 1 ? launch_few<32, 1>(a, n0, n1, smem, grid, s) : launch_few<32, 2>(a, n0, n1, smem, grid, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
