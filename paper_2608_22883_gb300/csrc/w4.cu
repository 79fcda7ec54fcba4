// Weights in 4 bits with a scale (and a zero point) per group of columns:
// their making (fovea_quantize_w4) and the product with a few rows
// (fovea_linear_w4).
//   w[o, k] = (code[o, k] - zero[o, k / group]) * scale[o, k / group]
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "packed.cuh"
#include "w4_x.cuh"

namespace fovea {

namespace {

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

__device__ __forceinline__ uint32_t min_bf16x2(uint32_t a, uint32_t b) {        // a NaN is dropped
  uint32_t r;
  asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// ---------------------------------------------------------------------------
// Codes, scales and zero points of a matrix
// ---------------------------------------------------------------------------

constexpr int kQuantThreads = 256;

// bf16 of the IEEE quotient a / n (a >= 0, n a small integer).  a times the reciprocal is
// off by less than four units of fp32's last place, which matters only that near a
// midpoint of two bf16 numbers.
static __device__ __noinline__ float quotient(float a, float b) { return __fdiv_rn(a, b); }
__device__ __forceinline__ __nv_bfloat16 bf16_quotient(float a, float n) {
  float v = a * (1.0f / n);
  const uint32_t below = __float_as_uint(v) & 0xFFFFu;
  if ((below > 0x7FF0u && below < 0x8010u) || !(v > 1e-30f)) v = quotient(a, n);
  return __float2bfloat16_rn(v);
}

// rint(w / scale) of the quotient rounded to fp32; twice_rcp is 2 / scale to 2^-21.
//
// The nearest half-integer h / 2 is wrong by one place at most, and the remainder w - h
// scale / 2 is exact (scale has 8 bits, h at most 6).  On a midpoint of two integers,
// where bf16 weights often lie, the remainder is 0 and the sum below the midpoint
// itself, which rounds to even; elsewhere the remainder's own quotient is so small that
// its error of 2^-21 stays far below the rounding of the sum.
__device__ __forceinline__ float rint_quotient(float w, float half_scale, float twice_rcp) {
  constexpr float kMagic = 12582912.0f;                  // 1.5 * 2^23: a sum with it is an integer
  const float h = fmaf(w, twice_rcp, kMagic) - kMagic;
  const float r = fmaf(-h, half_scale, w);
  return fmaf(fmaf(r, twice_rcp, h), 0.5f, kMagic) - kMagic;
}

// Two of them in packed instructions, the same operations.
__device__ __forceinline__ uint64_t rint_quotient2(uint64_t w, uint64_t minus_half_scale, uint64_t twice_rcp) {
  constexpr float kMagic = 12582912.0f;
  const uint64_t up = pack2(kMagic, kMagic), down = pack2(-kMagic, -kMagic), half = pack2(0.5f, 0.5f);
  const uint64_t h = add2(fma2(w, twice_rcp, up), down);
  const uint64_t r = fma2(h, minus_half_scale, w);
  return add2(fma2(fma2(r, twice_rcp, h), half, up), down);
}

// A warp takes strips of 256 columns of a row, eight columns a lane, so that a group
// of G columns is G / 8 neighbouring lanes; U strips are on their way together.  Scale
// and code are those of IEEE divisions, bit for bit.
//
// Reads W once and writes a seventh (fp32) or a quarter (bf16) of its bytes: bound by
// memory and by instruction issue about evenly, hence the packed arithmetic (fp32 108 us
// without).  W [32000, 4096]: fp32 in groups of 32 with zero points 101 us (6.0 TB/s, 88 %
// of the measured copy), bf16 the same 96, symmetric in groups of 128 81; W [4096, 4096]
// bf16 takes 13 us.  One strip and six CTAs an SM: 115, 122 and 86 us.
template <bool VEC>
struct QuantShape {                                      // strips on their way; CTAs an SM
  static constexpr int U = VEC ? 2 : 1, kCtas = VEC ? 4 : 6;
};
template <class T, int G, bool VEC, bool SYMMETRIC>
__global__ void __launch_bounds__(kQuantThreads, (QuantShape<VEC>::kCtas))
quantize_w4_kernel(const T* __restrict__ W, long long ld, int out, int in, uint8_t* __restrict__ codes,
                   __nv_bfloat16* __restrict__ scales, uint8_t* __restrict__ zeros) {
  constexpr int U = QuantShape<VEC>::U;
  constexpr int kVecs = sizeof(T) / 2;                   // 16-byte vectors of eight columns
  constexpr int kStrip = 256;
  const int lane = threadIdx.x & 31;
  const int groups = (in + G - 1) / G, strips = (in + kStrip - 1) / kStrip;
  const int warps = (int)gridDim.x * (kQuantThreads / 32);
  const int first = (int)blockIdx.x * (kQuantThreads / 32) + (int)(threadIdx.x >> 5);
  // the warp's next strip: row, first column, where this lane's weights, codes and
  // scale lie; and the steps to the one after it, without and with a carry to the next row
  const int row0 = first / strips, row_step = warps / strips;
  const int col_step = (warps - row_step * strips) * kStrip;
  int row = row0, col = (first - row0 * strips) * kStrip + lane * 8;
  const T* src = W + (long long)row * ld + col;
  long long code_at = (long long)row * in + col, scale_at = (long long)row * groups + col / G;
  const long long src_step = (long long)row_step * ld + col_step, src_carry = ld - strips * kStrip;
  const long long code_step = (long long)row_step * in + col_step, code_carry = in - strips * kStrip;
  const long long scale_step = (long long)row_step * groups + col_step / G, scale_carry = groups - strips * (kStrip / G);
  pdl_wait();
  pdl_trigger();
  while (row < out) {
    uint4 raw[U][kVecs];
    long long code_of[U], scale_of[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      live[u] = row < out && col < in;
      code_of[u] = code_at;
      scale_of[u] = scale_at;
#pragma unroll
      for (int h = 0; h < kVecs; ++h) raw[u][h] = make_uint4(0u, 0u, 0u, 0u);
      if (live[u]) {
        if (VEC) {
#pragma unroll
          for (int h = 0; h < kVecs; ++h) raw[u][h] = __ldg(reinterpret_cast<const uint4*>(src) + h);
        } else {
          T* e = reinterpret_cast<T*>(raw[u]);
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = src[j];
        }
      }
      row += row_step;
      col += col_step;
      src += src_step;
      code_at += code_step;
      scale_at += scale_step;
      if (col >= strips * kStrip) {
        ++row;
        col -= strips * kStrip;
        src += src_carry;
        code_at += code_carry;
        scale_at += scale_carry;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float w[8];
      const T* e = reinterpret_cast<const T*>(raw[u]);
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] = to_f32(e[j]);
      float hi = 0.0f, lo = 0.0f;
      if (sizeof(T) == 2) {
        // two at a time, a NaN the largest
        const uint32_t v[4] = {raw[u][0].x, raw[u][0].y, raw[u][0].z, raw[u][0].w};
        constexpr uint32_t kKeep = SYMMETRIC ? 0x7FFF7FFFu : ~0u;
        uint32_t m = v[0] & kKeep, least = v[0];
#pragma unroll
        for (int j = 1; j < 4; ++j) {
          m = max_nan_bf16x2(m, v[j] & kKeep);
          if (!SYMMETRIC) least = min_bf16x2(least, v[j]);
        }
        hi = max_nan(max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u)), 0.0f);
        if (!SYMMETRIC)
          lo = fminf(fminf(__uint_as_float(least << 16), __uint_as_float(least & 0xFFFF0000u)), 0.0f);
      } else {
        float odd = 0.0f;                                // w 0: NaN for a NaN, which fmaxf drops (and for an infinity)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          hi = fmaxf(hi, SYMMETRIC ? fabsf(w[j]) : w[j]);
          if (!SYMMETRIC) lo = fminf(lo, w[j]);
          odd = fmaf(w[j], 0.0f, odd);
        }
        if (odd != 0.0f) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (w[j] != w[j]) hi = w[j];
        }
      }
#pragma unroll
      for (int o = G / 16; o > 0; o >>= 1) {
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        if (!SYMMETRIC) lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      }
      const __nv_bfloat16 stored = SYMMETRIC ? bf16_quotient(hi, 7.0f) : bf16_quotient(hi - lo, 15.0f);
      const float scale = __bfloat162float(stored);
      const bool some = scale > 0.0f;                    // not 0, not NaN
      float zero = 8.0f;
      float q[8];
      if (scale > 1e-30f && scale < 1e30f) {
        const float half_scale = 0.5f * scale, twice_rcp = __fdividef(2.0f, scale);
        if (!SYMMETRIC) zero = fminf(fmaxf(rint_quotient(-lo, half_scale, twice_rcp), 0.0f), 15.0f);
        const uint64_t mh2 = pack2(-half_scale, -half_scale), tr2 = pack2(twice_rcp, twice_rcp);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const uint64_t v = rint_quotient2(pack2(w[j], w[j + 1]), mh2, tr2);
          q[j] = lo2(v);
          q[j + 1] = hi2(v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          // symmetric: max |w| / scale < 7.03, so no code leaves [-7, 7]
          if (!SYMMETRIC) q[j] = fminf(fmaxf(q[j], -zero), 15.0f - zero);
        }
      } else {                                           // 0, NaN, or no remainder to rely on
        if (!SYMMETRIC && some) zero = fminf(fmaxf(rintf(quotient(-lo, scale)), 0.0f), 15.0f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          q[j] = fminf(fmaxf(some ? rintf(quotient(w[j], scale)) : 0.0f, -zero), 15.0f - zero);
      }
      // four codes are one integer below 2^16, which the low bits of its sum with 2^23 hold
      const float base = fmaf(zero, 4369.0f, 8388608.0f);
      uint32_t half[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint64_t two = fma2(pack2(q[4 * h + 2], q[4 * h + 3]), pack2(256.0f, 256.0f), pack2(q[4 * h], q[4 * h + 1]));
        half[h] = __float_as_uint(fmaf(hi2(two), 16.0f, lo2(two)) + base);
      }
      if (live[u]) {
        *reinterpret_cast<uint32_t*>(codes + code_of[u] / 2) = __byte_perm(half[0], half[1], 0x5410);
        if ((lane & (G / 8 - 1)) == 0) {
          scales[scale_of[u]] = stored;
          if (!SYMMETRIC) zeros[scale_of[u]] = (uint8_t)zero;
        }
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
constexpr int kQuad = 2;               // spans of codes a warp has on their way
// Columns of x (an fp32 row counts three times) that a tile takes: the tensor-core
// instruction's eight.  More go through tensor memory (w4_tc.cu): with two such
// instructions a word 16 rows by 4096 x 32000 took 44.8 us here against 27.3 there, 8
// rows 22.4.  (Rows that do not fit shared memory together take a launch each few, which
// that path would do sooner: 8 rows by [4096, 14336] 32.4 us, 9 there 15.9; by [4096,
// 32768] 86.5 and 26.5.)
constexpr int kFewCols = 8;
// A tile is 8 * R weight rows, of which a lane holds the words of R: 16 rows are one
// operand, 32 two that share each read of x.  The registers for 32 are there with
// symmetric groups of 128 alone (64: spills, 23.2 against 22.1 us).  There 32 rows are
// faster once every SM has more than four tiles of 16 and rows are long enough to pay
// for fewer warps at work; one row of x, us with 16 and with 32 weight rows a tile:
// 128000 x 4096 67.1 and 57.2, 48000 33.3 and 27.8, 32000 20.2 and 19.1, 11000 10.9 and
// 10.2, 8192 7.6 and 8.4; 32000 x 1024 7.4 and 7.9.  Eight rows of x, 32000 x 4096: 26.2
// and 22.4.
template <int R> constexpr int kTileFloats = 8 * R * kFewCols;     // a warp's partial tile
template <int R> constexpr long long kFixedBytes = 16 + kWarps * kTileFloats<R> * 4;

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
// x from shared memory, which nothing writes once it is laid out: not volatile, so that
// the compiler may move it.  What keeps it behind the barrier is its address, which comes
// out of a volatile statement there.
__device__ __forceinline__ uint4 lds_x(uint32_t at) {
  uint4 v;
  asm("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}

// The codes of one span of weight rows g, g + 8, ... that this lane holds.
template <int R>
struct Span {
  uint32_t w[R][4];
};

// The scales (bf16 pairs) and zero points (bytes) of kQuad spans of a weight row.
template <int G>
struct Quad {
  static constexpr int kGroups = kQuad * kSpan / G;
  uint32_t s[kGroups / 2], z[(kGroups + 3) / 4];
  // `vec`: every row's scales and zeros start at a multiple of kGroups, aligned
  // p, pz: of the row's group g0
  template <bool ZEROS>
  __device__ __forceinline__ void load(const __nv_bfloat16* p, const uint8_t* pz, int g0, int groups, bool vec) {
    if (vec) {
      if (kGroups == 2) {
        s[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
      } else if (kGroups == 4) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
        s[0] = v.x; s[1] = v.y;
      } else {
#pragma unroll
        for (int i = 0; i < kGroups / 8; ++i) {
          const uint4 v = __ldg(reinterpret_cast<const uint4*>(p) + i);
          s[4 * i] = v.x; s[4 * i + 1] = v.y; s[4 * i + 2] = v.z; s[4 * i + 3] = v.w;
        }
      }
      if (ZEROS && kGroups == 2) {
        z[0] = __ldg(reinterpret_cast<const uint16_t*>(pz));
      } else if (ZEROS) {
#pragma unroll
        for (int i = 0; i < kGroups / 4; ++i)
          z[i] = __ldg(reinterpret_cast<const uint32_t*>(pz) + i);
      }
    } else {                                             // past the last group x is 0
#pragma unroll
      for (int i = 0; i < kGroups; ++i) {
        const uint32_t v = g0 + i < groups ? __bfloat16_as_ushort(p[i]) : 0u;
        s[i / 2] = i & 1 ? s[i / 2] | v << 16 : v;
        if (ZEROS) {
          const uint32_t b = g0 + i < groups ? pz[i] : 8u;
          z[i / 4] = i & 3 ? z[i / 4] | b << (8 * (i & 3)) : b;
        }
      }
    }
  }
  __device__ __forceinline__ float scale(int i) const {
    return __uint_as_float(i & 1 ? s[i / 2] & 0xFFFF0000u : s[i / 2] << 16);
  }
  __device__ __forceinline__ uint32_t zero2(int i) const {     // 128 + z, twice
    return 0x43004300u | ((z[i / 4] >> (8 * (i & 3))) & 127u) * 0x10001u;
  }
};

// y of up to kFewCols columns (rows of x, an fp32 row as three) in one launch.
//
// `split` warps take a tile of 8 * R weight rows, each a range of its quads (kQuad spans
// of 128 columns); a warp goes from tile to tile by itself, x in shared memory.  It
// turns the codes into bf16 integers c - z (exact) and multiplies them on the tensor
// cores, weights as the operands of 16 rows; a group's fp32 sum is then taken times its
// scale.  The codes of the next kQuad spans are on their way in registers
// meanwhile, across tiles, and so are the next quad's scales.  Only the warps of a
// split tile meet, in shared memory, in a fixed order.
//
// fp32 rows enter as three bf16 rows that add up to them exactly; e4m3 rows are
// exact in bf16 and their scales join the group's or the result.
//
// The weights' bytes are the floor; what it spends is instructions on the codes: a
// shift, a LOP3 and a subtraction for two of them, at most 4.75 cycles of a scheduler,
// besides the products.  A warp a tile without barriers and the operands' layout
// chosen so that a word needs no exchange between lanes keep the rest small.  One bf16
// row by [32000, 4096] in groups of 128: 19.3 us, 3.5 TB/s (52 % of the measured copy;
// tensor pipe 20 %); by [128000, 4096] 58.0 us (69 %); 7 rows by [3584, 3584] in groups of
// 64 with zero points 7.8 us, a tile's latency.
template <int G, bool ZEROS, int R>
__global__ void __launch_bounds__(kThreads, 1)
linear_w4_kernel(const LinearW4Args a, int n0, int n1, int split, bool x_vec, bool scale_vec,
                 uint32_t k128) {
  constexpr int kRows = 8 * R, kTilePart = kTileFloats<R>;
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
  const int tiles = (a.w.out + kRows - 1) / kRows;
  const int quads = (spans + kQuad - 1) / kQuad;
  // tiles go round the CTAs first, so that every SM has work of a short list
  const int team = warp / split, rank = warp - team * split;
  const int first = team * (int)gridDim.x + (int)blockIdx.x, step = (int)gridDim.x * (kWarps / split);
  const int q_lo = quads * rank / split, q_hi = quads * (rank + 1) / split;

  pdl_wait();
  pdl_trigger();
  // The next quad: this lane's first words of its rows (past the last row, of that one
  // again: the results are not stored) and their scales.  A word past its row's end keeps
  // what the register held: x is 0 there.
  const int row_bytes = a.w.in / 2;
  constexpr int kQuadBytes = kQuad * kSpan / 2;
  const int lane_byte = word_column<G>(0, t) / 2;
  const uint8_t* next[R];
  const __nv_bfloat16* next_scale[R];
  const uint8_t* next_zero[R];
  int next_tile = first, next_quad = q_lo;
  auto enter = [&]() {                                     // a tile
#pragma unroll
    for (int h = 0; h < R; ++h) {
      const long long row = min((long long)next_tile * kRows + g + 8 * h, (long long)a.w.out - 1);
      next[h] = a.w.codes + row * row_bytes + q_lo * kQuadBytes + lane_byte;
      next_scale[h] = a.w.scales + row * groups + q_lo * Quad<G>::kGroups;
      if (ZEROS) next_zero[h] = a.w.zeros + row * groups + q_lo * Quad<G>::kGroups;
    }
  };
  auto refill = [&](Span<R>& r, int d) {
    constexpr int kWords = G / 32;               // words in a row of bytes
#pragma unroll
    for (int j = 0; j < 4; j += kWords) {
      const int off = d * (kSpan / 2) + word_column<G>(j, 0) / 2;
      uint32_t in = next_tile < tiles;
      if (in && (next_quad + 1) * kQuadBytes > row_bytes)  // the row's last quad, cut short
        in = next_quad * kQuadBytes + lane_byte + off < row_bytes;
#pragma unroll
      for (int h = 0; h < R; ++h) load_words<kWords>(&r.w[h][j], next[h] + off, in);
    }
  };
  Quad<G> n[R] = {};
  auto refill_scales = [&]() {
    if (next_tile < tiles)
#pragma unroll
      for (int h = 0; h < R; ++h)
        n[h].template load<ZEROS>(next_scale[h], next_zero[h], next_quad * Quad<G>::kGroups, groups, scale_vec);
  };
  auto turn = [&]() {                                      // after a quad
#pragma unroll
    for (int h = 0; h < R; ++h) {
      next[h] += kQuadBytes;
      next_scale[h] += Quad<G>::kGroups;
      if (ZEROS) next_zero[h] += Quad<G>::kGroups;
    }
    if (++next_quad == q_hi) {
      next_quad = q_lo;
      next_tile += step;
      if (next_tile < tiles) enter();
    }
  };
  Span<R> ring[kQuad] = {};
  if (first < tiles) {
    enter();
#pragma unroll
    for (int d = 0; d < kQuad; ++d) refill(ring[d], d);
    refill_scales();
    turn();
  }
  if (tid == 0) {
    xs[-1] = make_uint4(0u, 0u, 0u, 0u);
    if (a.header != nullptr && blockIdx.x == 0) ensure_header(a.header);
  }
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
  uint32_t x_first =
      (uint32_t)__cvta_generic_to_shared(g < cols ? xs + (q_lo * kQuad * 16 + t) * cols + g : xs - 1);
  asm volatile("" : "+r"(x_first) : : "memory");           // no read of x (lds_x) passes the barrier
  float* mine = part + warp * kTilePart;
  const float* tile_part = part + team * split * kTilePart;
  for (int tile = first; tile < tiles; tile += step) {
    float acc[R / 2][4] = {};
    uint32_t x_at = x_first;
    for (int quad = q_lo; quad < q_hi; ++quad) {
      Quad<G> c[R];
#pragma unroll
      for (int h = 0; h < R; ++h) c[h] = n[h];
      refill_scales();
#pragma unroll
      for (int d = 0; d < kQuad; ++d) {
        const int span = quad * kQuad + d;
        if (span < spans) {
          const Span<R>& r = ring[d];
#pragma unroll
          for (int ii = 0; ii < kSpan / G; ++ii) {
            const int gq = d * (kSpan / G) + ii;           // of the quad's groups
            float sum[R / 2][4];
            uint32_t z[R];
#pragma unroll
            for (int h = 0; h < R; ++h) z[h] = ZEROS ? c[h].zero2(gq) : 0x43084308u;
#pragma unroll
            for (int jj = 0; jj < G / 32; ++jj) {
              const int j = ii * (G / 32) + jj;
              const uint4 b = lds_x(x_at);
              x_at += x_step;
#pragma unroll
              for (int m = 0; m < R / 2; ++m) {
                uint32_t w0[4], w1[4];             // column pairs 0 4, 1 5, 2 6, 3 7
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                  w0[p] = bf16_sub2(w4_pair(r.w[2 * m][j] >> (4 * p), k128), z[2 * m]);
                  w1[p] = bf16_sub2(w4_pair(r.w[2 * m + 1][j] >> (4 * p), k128), z[2 * m + 1]);
                }
                if (jj == 0) mma_16x8x16_first(sum[m], w0[0], w1[0], w0[1], w1[1], b.x, b.y);
                else mma_16x8x16(sum[m], w0[0], w1[0], w0[1], w1[1], b.x, b.y);
                mma_16x8x16(sum[m], w0[2], w1[2], w0[3], w1[3], b.z, b.w);
              }
            }
            float x0 = 1.0f, x1 = 1.0f;
            if (by_group) {
              const int col = 2 * t, gs = min(quad * Quad<G>::kGroups + gq, groups - 1);
              x0 = col < cols ? xscale[gs * cols + col] : 0.0f;
              x1 = col + 1 < cols ? xscale[gs * cols + col + 1] : 0.0f;
            }
#pragma unroll
            for (int m = 0; m < R / 2; ++m) {
              const float s0 = c[2 * m].scale(gq), s1 = c[2 * m + 1].scale(gq);
              acc[m][0] = fmaf(sum[m][0], s0 * x0, acc[m][0]);
              acc[m][1] = fmaf(sum[m][1], s0 * x1, acc[m][1]);
              acc[m][2] = fmaf(sum[m][2], s1 * x0, acc[m][2]);
              acc[m][3] = fmaf(sum[m][3], s1 * x1, acc[m][3]);
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
    for (int h = 0; h < R; ++h)
      *reinterpret_cast<float2*>(mine + (g + 8 * h) * kFewCols + 2 * t) =
          make_float2(acc[h / 2][2 * (h & 1)], acc[h / 2][2 * (h & 1) + 1]);
    if (split > 1) team_sync(team, split);
    else __syncwarp();
    for (int u = rank * 32 + lane; u < kRows * rows; u += 32 * split) {
      const int r = u & (kRows - 1), n = u / kRows;
      const long long o = (long long)tile * kRows + r;
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

template <int G, bool ZEROS, int R>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, long long x_bytes, cudaStream_t s) {
  auto kern = linear_w4_kernel<G, ZEROS, R>;
  static std::atomic<unsigned long long> done{0};          // devices whose limit is raised
  const cudaError_t e = raise_smem_limit(kern, kMaxSmem, done);
  if (e != cudaSuccess) return e;
  const bool x_vec = x_vectors(a.x, a.x_ld, a.x_dtype);
  const int groups = (a.w.in + G - 1) / G;
  const bool scale_vec = groups % Quad<G>::kGroups == 0 && (reinterpret_cast<uintptr_t>(a.w.scales) & 15u) == 0 &&
                         (reinterpret_cast<uintptr_t>(a.w.zeros) & 3u) == 0;
  const int tiles = (a.w.out + 8 * R - 1) / (8 * R);
  const int quads = (a.w.in + kQuad * kSpan - 1) / (kQuad * kSpan);
  // warps a tile: few tiles are split until each warp of the device has work (one row by
  // [4096, 4096]: one warp a tile 15.4 us, up to four 6.3, up to eight 5.5; [1024, 8192]:
  // 29.4, 9.0, 6.3)
  int split = 1;
  while (split < 8 && split * 2 <= quads && (long long)tiles * split * 2 <= 152 * kWarps) split *= 2;
  const long long work = (long long)tiles * split;
  const int grid = (int)std::min<long long>(152, std::max<long long>(1, split == 1 ? work : (work + split - 1) / split));
  return launch_pdl(kern, dim3(grid), dim3(kThreads), (size_t)(x_bytes + kFixedBytes<R>), s, a, n0, n1, split, x_vec, scale_vec,
                    kW4One28);
}
template <int G>
cudaError_t launch_few(const LinearW4Args& a, int n0, int n1, long long x_bytes, cudaStream_t s) {
  if (a.w.zeros != nullptr) return launch_few<G, true, 2>(a, n0, n1, x_bytes, s);
  if constexpr (G == 128)
    if (a.w.out > 4 * 152 * 16 && a.w.in >= 2048 && x_bytes + kFixedBytes<4> <= kMaxSmem)
      return launch_few<G, false, 4>(a, n0, n1, x_bytes, s);
  return launch_few<G, false, 2>(a, n0, n1, x_bytes, s);
}

}  // namespace

template <class T, int G, bool VEC>
static cudaError_t quantize(const T* W, long long ld, int out, int in, uint8_t* codes, __nv_bfloat16* scales,
                            uint8_t* zeros, cudaStream_t s) {
  const long long strips = (long long)out * ((in + 255) / 256);
  const long long ctas = (strips + kQuantThreads / 32 - 1) / (kQuantThreads / 32);
  const bool symmetric = zeros == nullptr;
  return launch_pdl(symmetric ? quantize_w4_kernel<T, G, VEC, true> : quantize_w4_kernel<T, G, VEC, false>,
                    dim3((int)std::min<long long>(ctas, 152 * QuantShape<VEC>::kCtas)), dim3(kQuantThreads), 0, s, W,
                    ld, out, in, codes, scales, zeros);
}
template <class T>
static cudaError_t quantize(const void* W, long long ld, int out, int in, int group, uint8_t* codes,
                            __nv_bfloat16* scales, uint8_t* zeros, cudaStream_t s) {
  const T* w = static_cast<const T*>(W);
  if ((reinterpret_cast<uintptr_t>(W) & 15u) == 0 && ld * sizeof(T) % 16 == 0)
    return group == 128 ? quantize<T, 128, true>(w, ld, out, in, codes, scales, zeros, s)
           : group == 64 ? quantize<T, 64, true>(w, ld, out, in, codes, scales, zeros, s)
                         : quantize<T, 32, true>(w, ld, out, in, codes, scales, zeros, s);
  return group == 128 ? quantize<T, 128, false>(w, ld, out, in, codes, scales, zeros, s)
         : group == 64 ? quantize<T, 64, false>(w, ld, out, in, codes, scales, zeros, s)
                       : quantize<T, 32, false>(w, ld, out, in, codes, scales, zeros, s);
}

cudaError_t launch_quantize_w4(int dtype, const void* W, long long ld, int out, int in, int group,
                               uint8_t* codes, __nv_bfloat16* scales, uint8_t* zeros, cudaStream_t s) {
  return dtype == FOVEA_BF16 ? quantize<__nv_bfloat16>(W, ld, out, in, group, codes, scales, zeros, s)
                             : quantize<float>(W, ld, out, in, group, codes, scales, zeros, s);
}

// Shared memory of the few-column product: of a column, and whatever their number.
static long long col_bytes(int in, int group, bool by_group) {
  return (in + kSpan - 1) / kSpan * 256ll + (by_group ? 4ll * ((in + group - 1) / group) : 0);
}
static long long few_rows(int in, int group, int x_dtype, bool by_group) {    // of a launch
  const int parts = x_parts(x_dtype);
  return std::min<long long>(kFewCols / parts,
                             (kMaxSmem - kFixedBytes<2>) / (col_bytes(in, group, by_group) * parts));
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
    const long long x_bytes = cols * col_bytes(a.w.in, a.w.group, by_group);
    const cudaError_t e = a.w.group == 128 ? launch_few<128>(a, n0, n1, x_bytes, s)
                          : a.w.group == 64 ? launch_few<64>(a, n0, n1, x_bytes, s)
                                            : launch_few<32>(a, n0, n1, x_bytes, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
