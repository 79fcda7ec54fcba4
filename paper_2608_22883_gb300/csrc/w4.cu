// Weights in 4 bits with a scale (and a zero point) per group of columns:
// their making (fovea_quantize_w4) and the product with a few rows
// (fovea_linear_w4).
//   w[o, k] = (code[o, k] - zero[o, k / group]) * scale[o, k / group]
#include <algorithm>

#include "common.cuh"
#include "w4_x.cuh"

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

constexpr int kMaxSmem = 227 * 1024;
constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kSpan = 128;             // columns a warp handles together
constexpr int kTileRows = 16;          // weight rows of a tile
constexpr int kQuad = 4;               // spans of codes a warp has on their way
// Columns of x (an fp32 row counts three times) that a tile takes: the tensor-core
// instruction's eight.  More go through tensor memory (w4_tc.cu): with two such
// instructions a word 16 rows by 4096 x 32000 took 44.8 us here against 27.3 there, 8
// rows 26.4.
constexpr int kFewCols = 8;
constexpr int kTilePart = kTileRows * kFewCols;

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
__device__ __forceinline__ void load_words(uint32_t* r, const uint8_t* p, uint32_t live) {
  if (N == 4)
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %5, 0;\n"
        " @q ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n}"
        : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]) : "l"(p), "r"(live));
  else if (N == 2)
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %3, 0;\n @q ld.global.nc.v2.u32 {%0, %1}, [%2];\n}"
        : "+r"(r[0]), "+r"(r[1]) : "l"(p), "r"(live));
  else
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.u32 q, %2, 0;\n @q ld.global.nc.u32 %0, [%1];\n}"
        : "+r"(r[0]) : "l"(p), "r"(live));
}
// A barrier of the `split` warps of a team (barriers 1 to 8).
__device__ __forceinline__ void team_sync(int team, int split) {
  asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(split * 32) : "memory");
}
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                            uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The first product of a sum.
__device__ __forceinline__ void mma_16x8x16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                                  uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
// x from shared memory, which nothing writes once it is laid out (so: not volatile).
__device__ __forceinline__ uint4 lds_x(uint32_t at) {
  uint4 v;
  asm("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}

// The codes of one span of weight rows g and g + 8 that this lane holds.
struct Span {
  uint32_t w[2][4];
};

// The scales (bf16 pairs) and zero points (bytes) of four spans of a weight row.
template <int G>
struct Quad {
  static constexpr int kGroups = kQuad * kSpan / G;      // 4, 8 or 16
  uint32_t s[kGroups / 2], z[kGroups / 4];
  // `vec`: every row's scales and zeros start at a multiple of kGroups, aligned
  template <bool ZEROS>
  __device__ __forceinline__ void load(const W4& w, long long row_at, int g0, int groups, bool vec) {
    if (vec) {
      const __nv_bfloat16* p = w.scales + row_at + g0;
      if (kGroups == 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
        s[0] = v.x; s[1] = v.y;
      } else {
#pragma unroll
        for (int i = 0; i < kGroups / 8; ++i) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
          s[4 * i] = v.x; s[4 * i + 1] = v.y; s[4 * i + 2] = v.z; s[4 * i + 3] = v.w;
        }
      }
      if (ZEROS) {
#pragma unroll
        for (int i = 0; i < kGroups / 4; ++i)
          z[i] = __ldg(reinterpret_cast<const uint32_t*>(w.zeros + row_at + g0) + i);
      }
    } else {                                             // past the last group x is 0
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const uint32_t v = g0 + i < groups ? __bfloat16_as_ushort(w.scales[row_at + g0 + i]) : 0u;
        s[i / 2] = i & 1 ? s[i / 2] | v << 16 : v;
        if (ZEROS) {
          const uint32_t b = g0 + i < groups ? w.zeros[row_at + g0 + i] : 8u;
          z[i / 4] = i & 3 ? z[i / 4] | b << (8 * (i & 3)) : b;
        }
      }
    }
  }
  __device__ __forceinline__ float scale(int i) const {
    return __uint_as_float(i & 1 ? s[i / 2] & 0xFFFF0000u : s[i / 2] << 16);
  }
  __device__ __forceinline__ uint32_t zero2(int i) const {     // 128 + z, twice
    return 0x43004300u | ((z[i / 4] >> (8 * (i & 3))) & 15u) * 0x10001u;
  }
};

// y of up to kFewCols columns (rows of x, an fp32 row as three) in one launch.
//
// `split` warps take a tile of 16 weight rows, each a range of its quads (four spans of
// 128 columns); a warp goes from tile to tile by itself, x in shared memory.  It
// turns the codes into bf16 integers c - z (exact) and multiplies them on the tensor
// cores, weights as the 16-row operand; a group's fp32 sum is then taken times its
// scale.  The codes of the next four spans are on their way in registers
// meanwhile, across tiles, and so are the next quad's scales.  Only the warps of a
// split tile meet, in shared memory, in a fixed order.
//
// fp32 rows enter as three bf16 rows that add up to them exactly; e4m3 rows are
// exact in bf16 and their scales join the group's or the result.
template <int G, bool ZEROS>
__global__ void __launch_bounds__(kThreads, 1)
linear_w4_kernel(const LinearW4Args a, int n0, int n1, int split, bool x_vec, bool scale_vec,
                 uint32_t k128) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int parts = x_parts(a.x_dtype);
  const int rows = n1 - n0, cols = rows * parts;
  const int spans = (a.w.in + kSpan - 1) / kSpan;
  const int groups = (a.w.in + G - 1) / G;
  // sixteen zero bytes; [span][word][quarter][column] units of eight x values; each
  // warp's partial tile [row][column]; scales of x [group][column]
  uint4* xs = reinterpret_cast<uint4*>(smem) + 1;
  float* part = reinterpret_cast<float*>(xs + (long long)spans * 16 * cols);
  float* xscale = part + kWarps * kTilePart;
  const bool by_group = a.x_scale != nullptr && a.x_group != 0;
  const int tiles = (a.w.out + kTileRows - 1) / kTileRows;
  const int quads = (spans + kQuad - 1) / kQuad;
  // tiles go round the CTAs first, so that every SM has work of a short list
  const int team = warp / split, rank = warp - team * split;
  const int first = team * (int)gridDim.x + (int)blockIdx.x, step = (int)gridDim.x * (kWarps / split);
  const int q_lo = quads * rank / split, q_hi = quads * (rank + 1) / split;

  pdl_wait();
  pdl_trigger();
  // The next quad's codes: this lane's first words of rows g and g + 8 (past the last
  // row, of that one again: the results are not stored), and how far they are into the
  // row.  A word past its row's end keeps what the register held: x is 0 there.
  const int row_bytes = a.w.in / 2;
  constexpr int kQuadBytes = kQuad * kSpan / 2;
  const int lane_byte = word_column<G>(0, t) / 2;
  const uint8_t *next0, *next1;
  int next_tile = first, next_quad = q_lo;
  auto enter = [&]() {                                     // a tile
    const long long row = (long long)next_tile * kTileRows + g, last = a.w.out - 1;
    next0 = a.w.codes + min(row, last) * row_bytes + q_lo * kQuadBytes + lane_byte;
    next1 = a.w.codes + min(row + 8, last) * row_bytes + q_lo * kQuadBytes + lane_byte;
  };
  auto refill = [&](Span& r, int d) {
    constexpr int kWords = G / 32;               // words in a row of bytes
#pragma unroll
    for (int j = 0; j < 4; j += kWords) {
      const int off = d * (kSpan / 2) + word_column<G>(j, 0) / 2;
      uint32_t in = next_tile < tiles;
      if (in && (next_quad + 1) * kQuadBytes > row_bytes)  // the row's last quad, cut short
        in = next_quad * kQuadBytes + lane_byte + off < row_bytes;
      load_words<kWords>(&r.w[0][j], next0 + off, in);
      load_words<kWords>(&r.w[1][j], next1 + off, in);
    }
  };
  auto turn = [&]() {                                      // after a quad
    next0 += kQuadBytes;
    next1 += kQuadBytes;
    if (++next_quad == q_hi) {
      next_quad = q_lo;
      next_tile += step;
      if (next_tile < tiles) enter();
    }
  };
  Span ring[kQuad] = {};
  if (first < tiles) {
    enter();
#pragma unroll
    for (int d = 0; d < kQuad; ++d) refill(ring[d], d);
    turn();
  }
  auto row_at = [&](int tile, int h) {                     // scales of row g + 8 h, the last row's past the end
    return min((long long)tile * kTileRows + g + 8 * h, (long long)a.w.out - 1) * groups;
  };
  Quad<G> n_0 = {}, n_1 = {};
  if (first < tiles) {
    n_0.template load<ZEROS>(a.w, row_at(first, 0), q_lo * Quad<G>::kGroups, groups, scale_vec);
    n_1.template load<ZEROS>(a.w, row_at(first, 1), q_lo * Quad<G>::kGroups, groups, scale_vec);
  }
  if (tid == 0) xs[-1] = make_uint4(0u, 0u, 0u, 0u);
  // x, a few units a thread on their way together
  constexpr int kBatch = 4;
  for (int u0 = tid; u0 < spans * 16 * rows; u0 += kBatch * kThreads) {
    X8 raw[kBatch] = {};
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + i * kThreads, n = u / (spans * 16), k0 = (u - n * (spans * 16)) * 8;
      if (n < rows && k0 < a.w.in) raw[i].load(a.x, (long long)(n0 + n) * a.x_ld + k0, a.x_dtype, x_vec);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int u = u0 + i * kThreads, n = u / (spans * 16), unit = u - n * (spans * 16);
      if (n >= rows) continue;
      const int span = unit >> 4, k8 = unit & 15;
      int j, q;                                // word and quarter of these columns
      if (G == 128) { q = k8 >> 2; j = k8 & 3; }
      else if (G == 64) { j = 2 * (k8 >> 3) + (k8 & 1); q = (k8 & 7) >> 1; }
      else { j = k8 >> 2; q = k8 & 3; }
      uint4 v[3];
      raw[i].columns(a.x_dtype, v);
      uint4* dst = xs + ((span * 4 + j) * 4 + q) * cols + n * parts;
      dst[0] = v[0];
      if (parts == 3) {
        dst[1] = v[1];
        dst[2] = v[2];
      }
    }
  }
  if (by_group)
    for (int u = tid; u < groups * cols; u += kThreads)
      xscale[u] = a.x_scale[(long long)(n0 + u % cols) * groups + u / cols];
  __syncthreads();

  // this lane's column of x: a column past the last reads the zeros
  const uint32_t x_step = g < cols ? 64u * cols : 0u;    // bytes from one word to the next
  const uint32_t x_first =
      (uint32_t)__cvta_generic_to_shared(g < cols ? xs + (q_lo * kQuad * 16 + t) * cols + g : xs - 1);
  float* mine = part + warp * kTilePart;
  const float* tile_part = part + team * split * kTilePart;
  for (int tile = first; tile < tiles; tile += step) {
    float acc[4] = {};
    uint32_t x_at = x_first;
    for (int quad = q_lo; quad < q_hi; ++quad) {
      const Quad<G> c_0 = n_0, c_1 = n_1;
      {
        const bool same = quad + 1 < q_hi;
        const int tt = same ? tile : tile + step, qq = same ? quad + 1 : q_lo;
        if (tt < tiles) {
          n_0.template load<ZEROS>(a.w, row_at(tt, 0), qq * Quad<G>::kGroups, groups, scale_vec);
          n_1.template load<ZEROS>(a.w, row_at(tt, 1), qq * Quad<G>::kGroups, groups, scale_vec);
        }
      }
#pragma unroll
      for (int d = 0; d < kQuad; ++d) {
        const int span = quad * kQuad + d;
        if (span < spans) {
          const Span& r = ring[d];
#pragma unroll
          for (int ii = 0; ii < kSpan / G; ++ii) {
            const int gq = d * (kSpan / G) + ii;           // of the quad's groups
            float sum[4];
            uint32_t z0 = 0x43084308u, z1 = 0x43084308u;
            if (ZEROS) {
              z0 = c_0.zero2(gq);
              z1 = c_1.zero2(gq);
            }
#pragma unroll
            for (int jj = 0; jj < G / 32; ++jj) {
              const int j = ii * (G / 32) + jj;
              uint32_t w0[4], w1[4];               // column pairs 0 4, 1 5, 2 6, 3 7
#pragma unroll
              for (int p = 0; p < 4; ++p) {
                w0[p] = bf16_sub2(w4_pair(r.w[0][j] >> (4 * p), k128), z0);
                w1[p] = bf16_sub2(w4_pair(r.w[1][j] >> (4 * p), k128), z1);
              }
              const uint4 b = lds_x(x_at);
              x_at += x_step;
              if (jj == 0) mma_16x8x16_first(sum, w0[0], w1[0], w0[1], w1[1], b.x, b.y);
              else mma_16x8x16(sum, w0[0], w1[0], w0[1], w1[1], b.x, b.y);
              mma_16x8x16(sum, w0[2], w1[2], w0[3], w1[3], b.z, b.w);
            }
            const float s0 = c_0.scale(gq), s1 = c_1.scale(gq);
            if (by_group) {
              const int n = 2 * t, gs = min(quad * Quad<G>::kGroups + gq, groups - 1);
              const float x0 = n < cols ? xscale[gs * cols + n] : 0.0f;
              const float x1 = n + 1 < cols ? xscale[gs * cols + n + 1] : 0.0f;
              acc[0] = fmaf(sum[0], s0 * x0, acc[0]);
              acc[1] = fmaf(sum[1], s0 * x1, acc[1]);
              acc[2] = fmaf(sum[2], s1 * x0, acc[2]);
              acc[3] = fmaf(sum[3], s1 * x1, acc[3]);
            } else {
              acc[0] = fmaf(sum[0], s0, acc[0]);
              acc[1] = fmaf(sum[1], s0, acc[1]);
              acc[2] = fmaf(sum[2], s1, acc[2]);
              acc[3] = fmaf(sum[3], s1, acc[3]);
            }
          }
        }
        refill(ring[d], d);
      }
      turn();
    }
    // the tile's end
    if (split > 1) team_sync(team, split);                 // the last tile has been read
    else __syncwarp();
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float2*>(mine + (g + 8 * h) * kFewCols + 2 * t) = make_float2(acc[2 * h], acc[2 * h + 1]);
    if (split > 1) team_sync(team, split);
    else __syncwarp();
    for (int u = rank * 32 + lane; u < kTileRows * rows; u += 32 * split) {
      const int r = u & (kTileRows - 1), n = u / kTileRows;
      const long long o = (long long)tile * kTileRows + r;
      float v = 0.0f;
      const float* from = tile_part + r * kFewCols + n * parts;
      for (int p = 0; p < parts; ++p)
        for (int w = 0; w < split; ++w) v += from[w * kTilePart + p];
      if (o < a.w.out) {
        if (a.x_scale != nullptr && !by_group) v *= a.x_scale[n0 + n];
        if (a.bias != nullptr) v += a.bias[o];
        const long long at = (long long)(n0 + n) * a.w.out + o;
        if (a.y_dtype == FOVEA_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
        else static_cast<float*>(a.y)[at] = v;
      }
    }
  }
}

template <int G, bool ZEROS>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, size_t smem, cudaStream_t s) {
  auto kern = linear_w4_kernel<G, ZEROS>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
  if (e != cudaSuccess) return e;
  const bool x_vec = x_vectors(a.x, a.x_ld, a.x_dtype);
  const int groups = (a.w.in + G - 1) / G;
  const bool scale_vec = groups % Quad<G>::kGroups == 0 && (reinterpret_cast<uintptr_t>(a.w.scales) & 15u) == 0 &&
                         (reinterpret_cast<uintptr_t>(a.w.zeros) & 3u) == 0;
  const int tiles = (a.w.out + kTileRows - 1) / kTileRows;
  const int quads = (a.w.in + kQuad * kSpan - 1) / (kQuad * kSpan);
  // warps a tile: few tiles are split until each warp of the device has work
  int split = 1;
  while (split < 8 && split * 2 <= quads && (long long)tiles * split * 2 <= 152 * kWarps) split *= 2;
  const long long work = (long long)tiles * split;
  const int grid = (int)std::min<long long>(152, std::max<long long>(1, split == 1 ? work : (work + split - 1) / split));
  return launch_pdl(kern, dim3(grid), dim3(kThreads), smem, s, a, n0, n1, split, x_vec, scale_vec,
                    kW4One28);
}
template <int G>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, size_t smem, cudaStream_t s) {
  return a.w.zeros != nullptr ? launch_few<G, true>(a, n0, n1, smem, s) : launch_few<G, false>(a, n0, n1, smem, s);
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

// Shared memory of the few-column product: of a column, and whatever their number.
static long long col_bytes(int in, int group, bool by_group) {
  return (in + kSpan - 1) / kSpan * 256ll + (by_group ? 4ll * ((in + group - 1) / group) : 0);
}
constexpr long long kFixedBytes = 16 + kWarps * kTilePart * 4;
static long long few_rows(int in, int group, int x_dtype, bool by_group) {    // of a launch
  const int parts = x_parts(x_dtype);
  return std::min<long long>(kFewCols / parts,
                             (kMaxSmem - kFixedBytes) / (col_bytes(in, group, by_group) * parts));
}
static bool is_few(int N, int in, int group, int x_dtype, bool by_group) {
  return (long long)N * x_parts(x_dtype) <= kFewCols && few_rows(in, group, x_dtype, by_group) > 0;
}

size_t linear_w4_workspace(int N, int in, int group, int x_dtype, bool by_group) {
  return N == 0 || is_few(N, in, group, x_dtype, by_group) ? 0
                                                           : linear_w4_tc_workspace(N, in, group, x_dtype, by_group);
}

cudaError_t launch_linear_w4(const LinearW4Args& a, cudaStream_t s) {
  const bool by_group = a.x_group != 0;
  if (!is_few(a.N, a.w.in, a.w.group, a.x_dtype, by_group)) return launch_linear_w4_tc(a, s);
  const int parts = x_parts(a.x_dtype);
  const int rows = (int)few_rows(a.w.in, a.w.group, a.x_dtype, by_group);
  for (int n0 = 0; n0 < a.N; n0 += rows) {
    const int n1 = std::min(a.N, n0 + rows);
    const int cols = (n1 - n0) * parts;
    const size_t smem = (size_t)(cols * col_bytes(a.w.in, a.w.group, by_group) + kFixedBytes);
    const cudaError_t e = a.w.group == 128 ? launch_few<128>(a, n0, n1, smem, s)
                          : a.w.group == 64 ? launch_few<64>(a, n0, n1, smem, s)
                                            : launch_few<32>(a, n0, n1, smem, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
