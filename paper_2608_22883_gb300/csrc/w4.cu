// Weights in 4 bits with a scale (and a zero point) per group of columns:
// their making (fovea_quantize_w4) and the product with a few rows
// (fovea_linear_w4).
//   w[o, k] = (code[o, k] - zero[o, k / group]) * scale[o, k / group]
#include <cuda_fp8.h>

#include <algorithm>

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
constexpr int kDepth = 4;              // spans of codes a warp has on their way
constexpr int kRegScales = 4;          // scales of the next tile a thread has on their way

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
// N words of codes where `live`, in one predicated instruction into the registers
// they stay in (behind a branch the words would be merged with their old values, and
// so waited for, at once).  Codes are read once: they need not displace x and the
// scales in L1; runs shorter than a sector share it with the next.
template <int N>
__device__ __forceinline__ void load_words(uint32_t* r, const uint8_t* p, bool live) {
  if (N == 4)
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %5, 0;\n"
        " @q ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]) : "l"(p), "r"((uint32_t)live));
  else if (N == 2)
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %3, 0;\n @q ld.global.nc.v2.u32 {%0, %1}, [%2];\n}"
        : "+r"(r[0]), "+r"(r[1]) : "l"(p), "r"((uint32_t)live));
  else
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %2, 0;\n @q ld.global.nc.u32 %0, [%1];\n}"
        : "+r"(r[0]) : "l"(p), "r"((uint32_t)live));
}
// v as the sum of three bf16 numbers: its truncations (an infinity or a NaN is the first alone).
__device__ __forceinline__ void split3(float v, uint32_t& b0, uint32_t& b1, uint32_t& b2) {
  const uint32_t bits = __float_as_uint(v);
  if ((bits & 0x7F800000u) == 0x7F800000u) {
    b0 = __bfloat16_as_ushort(__float2bfloat16_rn(v));
    b1 = b2 = 0u;
  } else {
    b0 = bits >> 16;
    const float r1 = v - __uint_as_float(b0 << 16);
    b1 = __float_as_uint(r1) >> 16;
    b2 = __float_as_uint(r1 - __uint_as_float(b1 << 16)) >> 16;
  }
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                            uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The codes of one span of weight rows g and g + 8 that this lane holds.
struct Span {
  uint32_t w[2][4];
};

template <int G>
__device__ __forceinline__ void load_span(Span& r, const W4& w, long long row0, int span, int lane, bool live) {
  const int g = lane >> 2, t = lane & 3;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // rows past the end repeat the last one (their results are not stored)
    const long long row = min(row0 + g + 8 * h, (long long)w.out - 1);
    const uint8_t* p = w.codes + row * (w.in / 2) + span * (kSpan / 2);
    constexpr int kWords = G / 32;               // words in a row of bytes
#pragma unroll
    for (int j = 0; j < 4; j += kWords) {
      const int k = word_column<G>(j, t);
      // past the row's end (whole runs: both are multiples of theirs) the words keep
      // what they held, and x is 0
      load_words<kWords>(&r.w[h][j], p + k / 2, live && span * kSpan + k < w.in);
    }
  }
}

// Eight columns of a row of x, as the bf16 columns that add up to them, in the order
// in which the codes of a word come out of it: 0 4 1 5 2 6 3 7.
__device__ __forceinline__ void layout_x8(const void* x, long long at, int dtype, bool vec, uint4 (&out)[3]) {
  out[1] = out[2] = make_uint4(0u, 0u, 0u, 0u);
  if (dtype == FOVEA_BF16 && vec) {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + at);
    out[0] = make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632),
                        __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
    return;
  }
  uint32_t pk[3][4] = {};
  constexpr int order[8] = {0, 4, 1, 5, 2, 6, 3, 7};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t b0 = 0, b1 = 0, b2 = 0;
    if (dtype == FOVEA_BF16) {
      b0 = static_cast<const uint16_t*>(x)[at + order[i]];
    } else if (dtype == FOVEA_FP32) {
      split3(static_cast<const float*>(x)[at + order[i]], b0, b1, b2);
    } else {
      const __half h = __half(__nv_cvt_fp8_to_halfraw(static_cast<const uint8_t*>(x)[at + order[i]], __NV_E4M3));
      b0 = __bfloat16_as_ushort(__float2bfloat16_rn(__half2float(h)));
    }
    pk[0][i / 2] |= b0 << (16 * (i & 1));
    pk[1][i / 2] |= b1 << (16 * (i & 1));
    pk[2][i / 2] |= b2 << (16 * (i & 1));
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) out[p] = make_uint4(pk[p][0], pk[p][1], pk[p][2], pk[p][3]);
}

// y of up to 8 NT columns (rows of x, an fp32 row as three) in one launch.
//
// A persistent CTA takes every gridDim.x-th tile of 16 weight rows.  Its warps
// split the tile's spans; each turns its codes into bf16 integers c - z (exact)
// and multiplies them on the tensor cores, weights as the 16-row operand, with
// x from shared memory; a group's fp32 sum is then taken times its scale.  The
// warps' partial tiles meet in shared memory in a fixed order.  The codes of the next
// kDepth spans, across tiles, are on their way in registers meanwhile, and so are
// the scales of the next tile.
//
// fp32 rows enter as three bf16 rows that add up to them exactly; e4m3 rows are
// exact in bf16 and their scales join the group's or the result.
template <int G, int NT, bool ZEROS>
__global__ void __launch_bounds__(kThreads, 1) linear_w4_kernel(const LinearW4Args a, int n0, int n1, bool x_vec) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int parts = a.x_dtype == FOVEA_FP32 ? 3 : 1;
  const int rows = n1 - n0, cols = rows * parts;
  const int spans = (a.w.in + kSpan - 1) / kSpan;
  const int groups = (a.w.in + G - 1) / G;
  // [span][word][quarter][column] units of eight x values; two partial tiles
  // [warp][row][column]; scales of x [group][column]; scales and zeros of two
  // tiles [row][group]
  uint4* xs = reinterpret_cast<uint4*>(smem);
  float* part = reinterpret_cast<float*>(xs + (long long)spans * 16 * cols);
  float* xscale = part + 2 * kWarps * kTileRows * 8 * NT;
  const bool by_group = a.x_scale != nullptr && a.x_group != 0;
  __nv_bfloat16* ws = reinterpret_cast<__nv_bfloat16*>(xscale + (by_group ? groups * cols : 0));
  const int tile_scales = kTileRows * groups;
  uint8_t* wz = reinterpret_cast<uint8_t*>(ws + 2 * tile_scales);
  const int tiles = (a.w.out + kTileRows - 1) / kTileRows;
  const int per = (spans + kWarps - 1) / kWarps;         // spans a warp has of a tile
  const long long all_scales = (long long)a.w.out * groups;

  // scales of a tile: kRegScales a thread through registers, others at once
  auto scale_at = [&](int tile, int e) { return min((long long)tile * tile_scales + e, all_scales - 1); };

  pdl_wait();
  pdl_trigger();
  Span ring[kDepth] = {};
  int next_tile = blockIdx.x, next_i = 0;
  auto refill = [&](Span& r) {
    const int span = next_i * kWarps + warp;
    load_span<G>(r, a.w, (long long)next_tile * kTileRows, span, lane, next_tile < tiles && span < spans);
    if (++next_i == per) {
      next_i = 0;
      next_tile += gridDim.x;
    }
  };
#pragma unroll
  for (int q = 0; q < kDepth; ++q) refill(ring[q]);
  for (int e = tid; e < tile_scales; e += kThreads) {
    ws[e] = a.w.scales[scale_at(blockIdx.x, e)];
    if (ZEROS) wz[e] = a.w.zeros[scale_at(blockIdx.x, e)];
  }
  for (int u = tid; u < spans * 16 * rows; u += kThreads) {
    const int n = u / (spans * 16), unit = u - n * (spans * 16);
    const int span = unit >> 4, k8 = unit & 15;
    int j, q;                                  // word and quarter of these columns
    if (G == 128) { q = k8 >> 2; j = k8 & 3; }
    else if (G == 64) { j = 2 * (k8 >> 3) + (k8 & 1); q = (k8 & 7) >> 1; }
    else { j = k8 >> 2; q = k8 & 3; }
    uint4 v[3] = {};
    if (unit * 8 < a.w.in) layout_x8(a.x, (long long)(n0 + n) * a.x_ld + unit * 8, a.x_dtype, x_vec, v);
    uint4* dst = xs + ((span * 4 + j) * 4 + q) * cols + n * parts;
    dst[0] = v[0];
    if (parts == 3) {
      dst[1] = v[1];
      dst[2] = v[2];
    }
  }
  if (by_group)
    for (int u = tid; u < groups * cols; u += kThreads)
      xscale[u] = a.x_scale[(long long)(n0 + u % cols) * groups + u / cols];
  __syncthreads();

  float acc[NT][4] = {};
  int tile = blockIdx.x, i = 0, buf = 0;
  __nv_bfloat16 sreg[kRegScales];
  uint8_t zreg[kRegScales];
  while (tile < tiles) {
#pragma unroll
    for (int d = 0; d < kDepth; ++d) {
      if (tile >= tiles) break;
      const int span = i * kWarps + warp;
      if (i == 0 && tile + (int)gridDim.x < tiles) {       // the next tile's scales set out
#pragma unroll
        for (int q = 0; q < kRegScales; ++q) {
          const int e = tid + q * kThreads;
          if (e < tile_scales) {
            sreg[q] = a.w.scales[scale_at(tile + gridDim.x, e)];
            if (ZEROS) zreg[q] = a.w.zeros[scale_at(tile + gridDim.x, e)];
          }
        }
      }
      if (span < spans) {
        const Span& r = ring[d];
        const __nv_bfloat16* sp = ws + buf * tile_scales + g * groups;
        const uint8_t* zp = wz + buf * tile_scales + g * groups;
#pragma unroll
        for (int ii = 0; ii < kSpan / G; ++ii) {
          const int gi = span * (kSpan / G) + ii;
          const int gs = kSpan / G == 1 ? gi : min(gi, groups - 1);   // past the last group x is 0
          float sum[NT][4] = {};
          uint32_t z0 = 0x43084308u, z1 = 0x43084308u;
          if (ZEROS) {
            z0 = 0x43004300u | zp[gs] * 0x10001u;
            z1 = 0x43004300u | zp[8 * groups + gs] * 0x10001u;
          }
#pragma unroll
          for (int jj = 0; jj < G / 32; ++jj) {
            const int j = ii * (G / 32) + jj;
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
          const float s0 = __bfloat162float(sp[gs]), s1 = __bfloat162float(sp[8 * groups + gs]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float x0 = 1.0f, x1 = 1.0f;
            if (by_group) {
              const int n = nt * 8 + 2 * t;
              x0 = n < cols ? xscale[gs * cols + n] : 0.0f;
              x1 = n + 1 < cols ? xscale[gs * cols + n + 1] : 0.0f;
            }
            acc[nt][0] = fmaf(sum[nt][0], s0 * x0, acc[nt][0]);
            acc[nt][1] = fmaf(sum[nt][1], s0 * x1, acc[nt][1]);
            acc[nt][2] = fmaf(sum[nt][2], s1 * x0, acc[nt][2]);
            acc[nt][3] = fmaf(sum[nt][3], s1 * x1, acc[nt][3]);
          }
        }
      }
      refill(ring[d]);
      if (++i < per) continue;
      // the tile's end
      float* mine = part + buf * (kWarps * kTileRows * 8 * NT);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          *reinterpret_cast<float2*>(mine + (warp * kTileRows + g + 8 * h) * 8 * NT + nt * 8 + 2 * t) =
              make_float2(acc[nt][2 * h], acc[nt][2 * h + 1]);
          acc[nt][2 * h] = acc[nt][2 * h + 1] = 0.0f;
        }
      if (tile + (int)gridDim.x < tiles) {
        const int other = (buf ^ 1) * tile_scales;
#pragma unroll
        for (int q = 0; q < kRegScales; ++q) {
          const int e = tid + q * kThreads;
          if (e < tile_scales) {
            ws[other + e] = sreg[q];
            if (ZEROS) wz[other + e] = zreg[q];
          }
        }
        for (int e = tid + kRegScales * kThreads; e < tile_scales; e += kThreads) {
          ws[other + e] = a.w.scales[scale_at(tile + gridDim.x, e)];
          if (ZEROS) wz[other + e] = a.w.zeros[scale_at(tile + gridDim.x, e)];
        }
      }
      // one barrier a tile: the buffers written here were last read before the
      // previous tile's barrier
      __syncthreads();
      for (int u = tid; u < kTileRows * rows; u += kThreads) {
        const int r = u & (kTileRows - 1), n = u / kTileRows;
        const long long o = (long long)tile * kTileRows + r;
        float v = 0.0f;
        const float* from = mine + r * 8 * NT + n * parts;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += from[w * kTileRows * 8 * NT];
        for (int p = 1; p < parts; ++p)
#pragma unroll
          for (int w = 0; w < kWarps; ++w) v += from[w * kTileRows * 8 * NT + p];
        if (o < a.w.out) {
          if (a.x_scale != nullptr && !by_group) v *= a.x_scale[n0 + n];
          if (a.bias != nullptr) v += a.bias[o];
          const long long at = (long long)(n0 + n) * a.w.out + o;
          if (a.y_dtype == FOVEA_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
          else static_cast<float*>(a.y)[at] = v;
        }
      }
      i = 0;
      buf ^= 1;
      tile += gridDim.x;
    }
  }
}

template <int G, int NT, bool ZEROS>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, size_t smem, int grid, cudaStream_t s) {
  cudaError_t e = cudaFuncSetAttribute(linear_w4_kernel<G, NT, ZEROS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       227 * 1024);
  if (e != cudaSuccess) return e;
  const bool x_vec = a.x_dtype == FOVEA_BF16 && (reinterpret_cast<uintptr_t>(a.x) & 15u) == 0 && a.x_ld % 8 == 0;
  return launch_pdl(linear_w4_kernel<G, NT, ZEROS>, dim3(grid), dim3(kThreads), smem, s, a, n0, n1, x_vec);
}
template <int G>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, int nt, size_t smem, int grid, cudaStream_t s) {
  if (a.w.zeros != nullptr)
    return nt == 1 ? launch_few<G, 1, true>(a, n0, n1, smem, grid, s) : launch_few<G, 2, true>(a, n0, n1, smem, grid, s);
  return nt == 1 ? launch_few<G, 1, false>(a, n0, n1, smem, grid, s) : launch_few<G, 2, false>(a, n0, n1, smem, grid, s);
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

// Columns of x (an fp32 row counts three times) that the warps' registers take;
// beyond them the codes go through tensor memory.
constexpr int kFewCols = 16;
// Shared memory of the few-column product: of a column, and whatever their number
// (with zero points, so that the choice of path does not depend on them).
static long long col_bytes(int in, int group, bool by_group) {
  return (in + kSpan - 1) / kSpan * 256ll + (by_group ? 4ll * ((in + group - 1) / group) : 0);
}
static long long fixed_bytes(int in, int group) {
  return 2 * kWarps * kTileRows * 16 * 4 + 2ll * kTileRows * ((in + group - 1) / group) * 3;
}
static long long few_rows(int in, int group, int x_dtype, bool by_group) {    // of a launch
  const int parts = x_dtype == FOVEA_FP32 ? 3 : 1;
  return std::min<long long>(kFewCols / parts,
                             (227 * 1024 - fixed_bytes(in, group)) / (col_bytes(in, group, by_group) * parts));
}
static bool is_few(int N, int in, int group, int x_dtype, bool by_group) {
  return (long long)N * (x_dtype == FOVEA_FP32 ? 3 : 1) <= kFewCols && few_rows(in, group, x_dtype, by_group) > 0;
}

size_t linear_w4_workspace(int N, int in, int group, int x_dtype, bool by_group) {
  return N == 0 || is_few(N, in, group, x_dtype, by_group) ? 0
                                                           : linear_w4_tc_workspace(N, in, group, x_dtype, by_group);
}

cudaError_t launch_linear_w4(const LinearW4Args& a, cudaStream_t s) {
  const bool by_group = a.x_group != 0;
  if (!is_few(a.N, a.w.in, a.w.group, a.x_dtype, by_group)) return launch_linear_w4_tc(a, s);
  const int parts = a.x_dtype == FOVEA_FP32 ? 3 : 1;
  const int rows = (int)few_rows(a.w.in, a.w.group, a.x_dtype, by_group);
  const int tiles = (a.w.out + kTileRows - 1) / kTileRows;
  const int grid = std::min(tiles, 152);
  for (int n0 = 0; n0 < a.N; n0 += rows) {
    const int n1 = std::min(a.N, n0 + rows);
    const int cols = (n1 - n0) * parts, nt = cols <= 8 ? 1 : 2;
    const size_t smem = cols * col_bytes(a.w.in, a.w.group, by_group) + fixed_bytes(a.w.in, a.w.group);
    const cudaError_t e = a.w.group == 128 ? launch_few<128>(a, n0, n1, nt, smem, grid, s)
                          : a.w.group == 64 ? launch_few<64>(a, n0, n1, nt, smem, grid, s)
                                            : launch_few<32>(a, n0, n1, nt, smem, grid, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
