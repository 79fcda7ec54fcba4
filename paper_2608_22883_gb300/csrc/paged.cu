// Attention of the newest entries of sequences over a paged key-value cache
// (fovea_paged_attention): a few rows (one new token, or the nodes of a draft tree)
// against all entries of their sequence,
//   s = scale q.k,  p = e^(s - lse),  lse = log sum e^s,  out = sum p v
// over the entries a row sees.
//
// One pass over the cache with a running maximum and sum.  The rows of a key head (its
// query heads times the nodes) are the narrow side of the products, the entries the wide
// one: S^T = K Q^T and O^T = V^T P^T with mma.sync, 16 entries by 8 rows, so that eight
// rows waste nothing.  The work is bound by the cache's bytes, not by the tensor cores
// (8 rows: 16 operations a byte of bf16), and needs no shared memory: the order of a
// head's dims within a contraction is free, so a lane's 16-byte loads of keys are its
// fragments as they come (a lane of the quad takes every fourth chunk of a row), and
// those of values become fragments of V^T by pairing two entries' halves (one prmt a
// register).  P goes from S^T's layout to the other operand's by movmatrix.
//
// Measured: four sequences of 98304 to 131072 e4m3 entries, 32 heads over 8 of keys of 128:
// 156 us, 6.0 TB/s; 64 of 1536 to 2048 bf16 entries, 28 over 4: 46 us, 5.1 TB/s; 64 of 0 to
// 8192, pages of 16: 31 us, 4.0 TB/s (the loads' latency: 12 warps an SM hold 96 KB on their
// way; more warps, or more blocks a warp, cost registers that spill); one of 640 entries, 32
// heads: 7.4 us, latency throughout.
#include <atomic>
#include <cstddef>

#include "paged_core.cuh"
#include "tc_ptx.cuh"

namespace fovea {

namespace {

__device__ __forceinline__ float dsmem_f32(uint32_t at, uint32_t rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(tc::map_dsmem(at, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x as the sum of two tf32 values: hi its upper 11 bits, lo the other 13, of which the
// product reads 11 (an error of 2^-21 of x at most).  The product of two lower parts, 2^-20 at
// most, is left out: a product is right to 2^-19.  Upper parts that are rounded to nearest
// bring it to 2^-21, for two more instructions an element: 8 sequences of 2048 37 us instead
// of 34, heads of 256 79 instead of 69, 64 rows over 4 heads 132 instead of 115.
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t& hi, uint32_t& lo) {
  const bool finite = (x << 1) < 0xFF000000u;
  hi = finite ? x & 0xFFFFE000u : x;
  lo = finite ? __float_as_uint(__uint_as_float(x) - __uint_as_float(hi)) : 0u;
}
// How entries of a type are cut among the lanes.  g = lane / 4, t = lane % 4.
// Keys: lane (g, t) holds entries g and g + 8, of each the 16-byte chunks t, t + 4, ...
// Values: lane (g, t) holds, of its entries, `kSpan` dims from kSpan g of each part of
// 8 kSpan dims.  Entries: 2t, 2t + 1, 2t + 8, 2t + 9 (16 bits and less), t, t + 4, t + 8,
// t + 12 (32 bits).
template <class C, int D> struct Cut {
  static constexpr int kSize = sizeof(C);
  static constexpr int kUnit = 16 / kSize;                        // elements of a 16-byte chunk
  static constexpr int kKeyChunks = D / (4 * kUnit);              // chunks of a lane's entry
  static constexpr int kSpan = kUnit < D / 8 ? kUnit : D / 8;
  static constexpr int kParts = D / (8 * kSpan);
  static constexpr int kSpanWords = kSpan * kSize / 4;            // 32-bit words of a span: 4 or 2
  static constexpr int kTiles = D / 16;                           // 16-dim tiles of O^T
  static constexpr int kSteps = kSize == 4 ? D / 8 : D / 16;      // of the contraction over dims
};

// Blocks that a warp takes together.
template <class C, int D, int RT> constexpr int kTogether = sizeof(C) * D * RT <= 128 ? 2 : 1;

// Whether a step's pages are asked for a step ahead: with 8-bit entries (four sequences of
// 131072: 179 us without, 155 with) and bf16 of 256 dims (49.7 and 46.2); it costs the
// others (one sequence of 4096 10.3 and 11.5, fp32 of 128 dims 33 and 39, of 256 68.7 and 71.6).
template <class C, int D> constexpr bool kAsks = sizeof(C) == 1 || (sizeof(C) == 2 && D == 256);

// Whether a block's values are loaded when its scores are formed, and the next keys when its
// values are used, in the same registers: keys and values of fp32 entries of 256 dims take 128
// registers a lane each.  16 sequences of 2048: 68.7 us, with both on their way, which spills
// 1.5 KB, 98.9; one of 1000 15.6 and 22.3.  It costs those that fit: fp32 of 128 dims 33.6 to
// 34.8, bf16 of 256 45.8 to 47.7.
template <class C, int D> constexpr bool kTakesTurns = sizeof(C) * D > 512;

// FOLD: at most four rows, over 8-bit entries.  They stand twice among the eight of a
// product, the second time for p's lower halves: one product does for both (four sequences
// of 131072: 155 us; with two products 169, with p to 11 bits 157).
template <class C, class Q, int D, int RT, bool FOLD = false>
struct Attention {
  using G = Cut<C, D>;
  static_assert(!FOLD || (sizeof(C) == 1 && RT == 1), "one tile of rows");
  static constexpr bool kF32 = sizeof(C) == 4, kE4 = sizeof(C) == 1;
  static constexpr bool kWaits = false;
  static constexpr int kRows = 8 * RT, kBlock = 16, kLeast = kWarps;
  // 64 sequences of 0 to 8192 entries with 0 / 8 / 16 / 24 blocks in front of a segment: 85 /
  // 37 / 31 / 31 us
  static constexpr uint32_t kFront = RT == 1 ? 16 : 24;
  static constexpr int kSlot = kRows * (D + 2);                  // floats of a partial segment
  static constexpr uint32_t kBytes = kBlock * D * sizeof(C);     // of a block
  // p beside 8-bit values is held in fp16, times 2^15: its smallest step is then 2^-39
  static constexpr float kLift = kE4 ? 15.0f : 0.0f;

  struct Shared {
    uint2 q[RT][G::kSteps][32];      // Q^T's fragments
    float row_scale[kRows];          // of s, to powers of two
    int odd;                         // what the segment has met (Odd)
    uint32_t lost;                   // rows whose sum is no number, as bits
    float m[kWarps][kRows], l[kWarps][kRows];
    alignas(16) float o[kWarps][kRows][D + 4];
  };

  static constexpr int kSub = kTogether<C, D, RT>;
  static constexpr bool kAsk = kAsks<C, D>;
  static constexpr bool kInTurn = kTakesTurns<C, D>;
  // The keys and values of kSub blocks as a lane holds them.
  uint4 k[kSub][2][G::kKeyChunks];
  uint32_t v[kSub][4][G::kParts][G::kSpanWords];
  float o[RT][G::kTiles][4];
  float m[RT][2], l[RT][2];

  __device__ __forceinline__ static int row_in(int r) { return FOLD ? r & 3 : r; }   // of place r
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      m[r][0] = m[r][1] = -INFINITY;
      l[r][0] = l[r][1] = 0.0f;
#pragma unroll
      for (int i = 0; i < G::kTiles; ++i) o[r][i][0] = o[r][i][1] = o[r][i][2] = o[r][i][3] = 0.0f;
    }
  }
  __device__ __forceinline__ static int value_entry(int t, int e) {      // the lane's e-th entry of values
    return kF32 ? t + 4 * e : 2 * t + (e & 1) + 8 * (e >> 1);
  }
  // `at`: the lane's first byte of the block (keys_from and values_from behind its start).
  __device__ __forceinline__ static uint32_t keys_from() {
    const int lane = threadIdx.x & 31;
    return ((lane >> 2) * D + (lane & 3) * G::kUnit) * G::kSize;
  }
  __device__ __forceinline__ static uint32_t values_from() {
    const int lane = threadIdx.x & 31;
    return (value_entry(lane & 3, 0) * D + (lane >> 2) * G::kSpan) * G::kSize;
  }
  __device__ __forceinline__ void load_keys(int u, const uint8_t* at) {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int j = 0; j < G::kKeyChunks; ++j)
        k[u][e][j] = __ldg(reinterpret_cast<const uint4*>(at + 8 * e * D * G::kSize + 64 * j));
  }
  __device__ __forceinline__ void load_values(int u, const uint8_t* at) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int p = 0; p < G::kParts; ++p) {
        const uint8_t* q = at + (value_entry(0, e) * D + p * 8 * G::kSpan) * G::kSize;
        if constexpr (G::kSpanWords == 4) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(q));
          v[u][e][p][0] = x.x; v[u][e][p][1] = x.y; v[u][e][p][2] = x.z; v[u][e][p][3] = x.w;
        } else {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(q));
          v[u][e][p][0] = x.x; v[u][e][p][1] = x.y;
        }
      }
  }
  __device__ __forceinline__ static uint32_t word(const uint4& x, int i) {
    return i == 0 ? x.x : i == 1 ? x.y : i == 2 ? x.z : x.w;
  }

  // S^T of the block: s[r][0..3] = entries g, g, g + 8, g + 8 by rows 2t, 2t + 1, 2t, 2t + 1.
  __device__ __forceinline__ void scores(int u, const Shared& sh, float (&s)[RT][4]) const {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int r = 0; r < RT; ++r) s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.0f;
    if constexpr (kF32) {
      // The tensor cores truncate each addition to an accumulator; products of the high
      // parts go to a fresh one every four steps, and the small ones to one of their own.
      float small[RT][4];
#pragma unroll
      for (int r = 0; r < RT; ++r) small[r][0] = small[r][1] = small[r][2] = small[r][3] = 0.0f;
#pragma unroll
      for (int c = 0; c < G::kSteps; c += 4) {
        float part[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) part[r][0] = part[r][1] = part[r][2] = part[r][3] = 0.0f;
#pragma unroll
        for (int i = c; i < c + 4; ++i) {
          const int j = i >> 1, h = 2 * (i & 1);
          const uint32_t x[4] = {word(k[u][0][j], h), word(k[u][1][j], h), word(k[u][0][j], h + 1), word(k[u][1][j], h + 1)};
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) split_tf32(x[e], hi[e], lo[e]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const uint2 q = sh.q[r][i][lane];
            uint32_t h0, l0, h1, l1;
            split_tf32(q.x, h0, l0);
            split_tf32(q.y, h1, l1);
            mma_tf32(part[r], hi, h0, h1);
            mma_tf32(small[r], hi, l0, l1);
            mma_tf32(small[r], lo, h0, h1);
          }
        }
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[r][e] += part[r][e];
      }
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[r][e] += small[r][e];
    } else {
#pragma unroll
      for (int i = 0; i < G::kSteps; ++i) {
        uint32_t a[4];
        if constexpr (kE4) {
          const uint32_t x = word(k[u][0][i >> 2], i & 3), y = word(k[u][1][i >> 2], i & 3);
          a[0] = halves_of_e4m3(x & 0xFFFFu); a[1] = halves_of_e4m3(y & 0xFFFFu);
          a[2] = halves_of_e4m3(x >> 16);     a[3] = halves_of_e4m3(y >> 16);
        } else {
          const int j = i >> 1, h = 2 * (i & 1);
          a[0] = word(k[u][0][j], h); a[1] = word(k[u][1][j], h);
          a[2] = word(k[u][0][j], h + 1); a[3] = word(k[u][1][j], h + 1);
        }
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const uint2 q = sh.q[r][i][lane];
          mma16<kE4>(s[r], a, q.x, q.y);
        }
      }
    }
  }

  // The values' fragment of a tile of 16 dims (dims 2i and 2i + 1 of the spans, i = tile
  // within the part): f[0..3] of the entries 2t, 2t + 1 and 2t + 8, 2t + 9.
  __device__ __forceinline__ void value_tile(int u, int tile, uint32_t (&f)[4]) const {
    constexpr int kPer = G::kSpan / 2;                     // tiles of a part
    const int p = tile / kPer, i = tile % kPer;
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      if constexpr (kE4) {                                 // bytes of two entries side by side, then to fp16
        const uint32_t x = __byte_perm(v[u][e][p][i >> 1], v[u][e + 1][p][i >> 1], i & 1 ? 0x7362 : 0x5140);
        f[e] = halves_of_e4m3(x & 0xFFFFu);
        f[e + 1] = halves_of_e4m3(x >> 16);
      } else {
        f[e] = low_halves(v[u][e][p][i], v[u][e + 1][p][i]);
        f[e + 1] = high_halves(v[u][e][p][i], v[u][e + 1][p][i]);
      }
    }
  }

  // O^T += V^T P^T; p in S^T's layout.
  __device__ __forceinline__ void add_values(int u, const float (&p)[RT][4]) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    if constexpr (kF32) {
      uint32_t bh[RT][4], bl[RT][4];                       // entries t, t + 4, t + 8, t + 12 of row g
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int from = (t + 4 * (e & 1)) * 4 + (g >> 1);
          const float x = __shfl_sync(0xffffffffu, p[r][2 * (e >> 1)], from);
          const float y = __shfl_sync(0xffffffffu, p[r][2 * (e >> 1) + 1], from);
          split_tf32(__float_as_uint(g & 1 ? y : x), bh[r][e], bl[r][e]);
        }
#pragma unroll
      for (int i = 0; i < G::kTiles; ++i) {
        const int part = i / 2, w = 2 * (i & 1);
        float sum[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r) sum[r][0] = sum[r][1] = sum[r][2] = sum[r][3] = 0.0f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t hi[4], lo[4];
          split_tf32(v[u][2 * c][part][w], hi[0], lo[0]);
          split_tf32(v[u][2 * c][part][w + 1], hi[1], lo[1]);
          split_tf32(v[u][2 * c + 1][part][w], hi[2], lo[2]);
          split_tf32(v[u][2 * c + 1][part][w + 1], hi[3], lo[3]);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            mma_tf32(sum[r], lo, bh[r][2 * c], bh[r][2 * c + 1]);
            mma_tf32(sum[r], hi, bl[r][2 * c], bl[r][2 * c + 1]);
            mma_tf32(sum[r], hi, bh[r][2 * c], bh[r][2 * c + 1]);
          }
        }
        // fresh sums of a block, added in fp32 (the tensor cores would truncate)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[r][i][e] += sum[r][e];
      }
    } else {
      // p as two bf16 values that add up to 16 bits of it (one alone would add an error of
      // the output's own rounding), beside 8-bit values as two of fp16: 22 bits (p times
      // 2^kLift is 2^15 at most, the smallest step 2^-24)
      uint32_t bh[RT][2], bl[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = p[r][2 * e], y = p[r][2 * e + 1];
          if constexpr (kE4) {
            uint32_t hi, lo;
            split_halves(x, y, hi, lo);
            bh[r][e] = transpose8(FOLD && t >= 2 ? lo : hi);      // rows 2t, 2t + 1
            if constexpr (!FOLD) bl[r][e] = transpose8(lo);
          } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
            const float2 f = __bfloat1622float2(h);
            const __nv_bfloat162 d = __floats2bfloat162_rn(x - f.x, y - f.y);
            bh[r][e] = transpose8(*reinterpret_cast<const uint32_t*>(&h));
            bl[r][e] = transpose8(*reinterpret_cast<const uint32_t*>(&d));
          }
        }
#pragma unroll
      for (int i = 0; i < G::kTiles; ++i) {
        uint32_t f[4];
        value_tile(u, i, f);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          mma16<kE4>(o[r][i], f, bh[r][0], bh[r][1]);
          if constexpr (!FOLD) mma16<kE4>(o[r][i], f, bl[r][0], bl[r][1]);
        }
      }
    }
  }

  // Values of entries from `left` on are cleared: what stands there is not used.
  __device__ __forceinline__ void clear_values(int u, int left) {
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (value_entry(t, e) >= left)
#pragma unroll
        for (int p = 0; p < G::kParts; ++p)
#pragma unroll
          for (int w = 0; w < G::kSpanWords; ++w) v[u][e][p][w] = 0;
  }

  // Odd values of the block's entries from `from` on cleared (add_odd_values): true where there was one.
  __device__ __forceinline__ bool clear_odd_values(int u, int from) {
    const int t = threadIdx.x & 3;
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (value_entry(t, e) >= from)
#pragma unroll
        for (int p = 0; p < G::kParts; ++p)
#pragma unroll
          for (int w = 0; w < G::kSpanWords; ++w) {
            const uint32_t odd = odd_in<C>(v[u][e][p][w]);
            v[u][e][p][w] &= ~odd;
            any |= odd;
          }
    return any != 0;
  }

  // Q^T's fragments of the rows from row0 on.  All threads; between barriers of the caller.
  __device__ __forceinline__ static void stage_rows(const PagedArgs& a, Shared& sh, int b, int h, int row0) {
    const int tid = threadIdx.x, lane = tid & 31;
    const int rows = a.nodes * a.group;
    auto row_at = [&](int r) { return row_of<Q>(a, b, h, r); };
    if (tid == 0) sh.odd = 0;
    if constexpr (kE4) {
      for (int r = tid >> 5; r < kRows; r += kWarps) {
        float top = 0.0f;
        if (row0 + row_in(r) < rows) {
          const Q* p = row_at(row0 + row_in(r));
          for (int d = lane; d < D; d += 32) top = fmaxf(top, fabsf(to_f32(p[d])));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) sh.row_scale[r] = row_power(top);
      }
      __syncthreads();
    }
    for (int i = tid; i < RT * G::kSteps * 32; i += kThreads) {
      const int lane_of = i & 31, step = (i >> 5) % G::kSteps, r = (i >> 5) / G::kSteps;
      const int row = row0 + row_in(8 * r + (lane_of >> 2)), t = lane_of & 3;
      uint2 f = make_uint2(0u, 0u);
      if (row < rows) {
        const Q* p = row_at(row);
        if constexpr (kF32) {
          p += (4 * (step >> 1) + t) * G::kUnit + 2 * (step & 1);
          f = make_uint2(__float_as_uint(p[0]), __float_as_uint(p[1]));
        } else if constexpr (kE4) {
          p += (4 * (step >> 2) + t) * G::kUnit + 4 * (step & 3);
          const float k = 1.0f / sh.row_scale[8 * r + (lane_of >> 2)];
          const __half2 x = __floats2half2_rn(to_f32(p[0]) * k, to_f32(p[1]) * k);
          const __half2 y = __floats2half2_rn(to_f32(p[2]) * k, to_f32(p[3]) * k);
          f = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        } else {
          p += (4 * (step >> 1) + t) * G::kUnit + 4 * (step & 1);
          const uint16_t* w = reinterpret_cast<const uint16_t*>(p);
          f = make_uint2((uint32_t)w[0] | ((uint32_t)w[1] << 16), (uint32_t)w[2] | ((uint32_t)w[3] << 16));
        }
      }
      sh.q[r][step][lane_of] = f;
    }
  }

  // Blocks [lo, hi) of one segment, kSub by each warp in turn.
  __device__ __forceinline__ void blocks(const PagedArgs& a, Shared& sh, int b, int h, int row0, int n,
                                         uint32_t lo, uint32_t hi) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t* tree = tree_of(a, b);
    const int32_t* table = a.table + (size_t)b * a.width;
    const uint32_t per_page = a.page / kBlock, stride = a.kv_heads * per_page;
    const uint8_t* keys = static_cast<const uint8_t*>(a.k_pages) + (size_t)h * per_page * kBytes + keys_from();
    const uint8_t* values = static_cast<const uint8_t*>(a.v_pages) + (size_t)h * per_page * kBytes + values_from();
    const float factor = a.scale * kLog2e * (kE4 && a.k_scale != nullptr ? a.k_scale[h] : 1.0f);
    float f[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) f[r][e] = kE4 ? factor * sh.row_scale[8 * r + 2 * t + e] : factor;
    clear();
    uint32_t at = lo + warp * kSub;
    if (at >= hi) return;
    // Pages are looked up a step ahead; with kAsk two, and the next step's keys and values are
    // asked for from memory, into L2, a step before their loads: registers hold one step's alone.
    int id[kSub];
    uint32_t in_page[kSub];
    auto look_up = [&](uint32_t first) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const uint32_t block = min(first + u, hi - 1), p = page_of(a, block);
        id[u] = table[p];
        in_page[u] = block - p * per_page;
      }
    };
    unsigned long long off[kSub], next_off[kSub];          // bytes from the pools' lane pointers
    bool bad = false, next_bad = false;                    // a page is not in the pool
    auto place = [&]() {
      next_bad = false;
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const bool out = (unsigned)id[u] >= (unsigned)a.n_pages;
        next_bad |= out;
        next_off[u] = ((unsigned long long)(out ? 0u : (uint32_t)id[u]) * stride + in_page[u]) * kBytes;
      }
    };
    auto ask = [&]() {
      constexpr uint32_t kLines = kBytes / 128;
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (uint32_t i = 0; i < kLines; i += 32)
          if (kLines >= 32 || lane < (int)kLines) {
            const size_t line = next_off[u] + (i + lane) * 128;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(keys - keys_from() + line));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(values - values_from() + line));
          }
    };
    look_up(at);
    place();
#pragma unroll
    for (int u = 0; u < kSub; ++u) {
      off[u] = next_off[u];
      if constexpr (!kInTurn) load_keys(u, keys + off[u]);
    }
    bad = next_bad;
    if (kAsk && at + kWarps * kSub < hi) look_up(at + kWarps * kSub);
    const int end = min(n, (int)(hi * kBlock));            // the run's last entry
    const int plain = min(end, plain_end(a, n));
    while (true) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        if constexpr (kInTurn) load_keys(u, keys + off[u]);
        else load_values(u, values + off[u]);
      }
      const uint32_t next = at + kWarps * kSub, after = next + kWarps * kSub;
      const bool more = next < hi;
      if (more) {
        if constexpr (kAsk) {
          place();
          ask();
          if (after < hi) look_up(after);
        } else {
          look_up(next);
        }
      }
      float s[kSub][RT][4];
#pragma unroll
      for (int u = 0; u < kSub; ++u) scores(u, sh, s[u]);
      if constexpr (kInTurn) {
#pragma unroll
        for (int u = 0; u < kSub; ++u) load_values(u, values + off[u]);
      }
      const bool was_bad = bad;
      if (more) {
        if constexpr (!kAsk) place();
        bad = next_bad;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          off[u] = next_off[u];
          if constexpr (!kInTurn) load_keys(u, keys + off[u]);
        }
      }
      const int first = (int)at * kBlock;
#pragma unroll
      for (int u = 0; u < kSub; ++u)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[u][r][e] *= f[r][e & 1];
      if (was_bad || first + kSub * kBlock > plain) {
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
          const int start = first + u * kBlock;
          // which of the block's pages: looked up again, this is rare
          const bool out = was_bad && start < end && (unsigned)table[page_of(a, at + u)] >= (unsigned)a.n_pages;
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int node = min((row0 + row_in(8 * r + 2 * t + e)) / a.group, a.nodes - 1);
              const uint32_t bits = seen_bits(a, tree, n, node, start, end);
#pragma unroll
              for (int x = e; x < 4; x += 2) s[u][r][x] = bits >> (g + 4 * (x - e)) & 1u ? s[u][r][x] : -INFINITY;
              if (out && (bits & 0xFFFFu) != 0) l[r][e] = NAN;   // a page that is not there
            }
          clear_values(u, out ? 0 : end - start);
          if ((a.nodes > 1 || tree != nullptr) && clear_odd_values(u, n - a.nodes - start)) sh.odd = kOddCleared;
        }
      }
      // running maxima and sums
      bool moved = false;
      float top[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(s[0][r][e], s[0][r][e + 2]);
#pragma unroll
          for (int u = 1; u < kSub; ++u) x = fmaxf(x, fmaxf(s[u][r][e], s[u][r][e + 2]));
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
          top[r][e] = fmaxf(m[r][e], x);
          moved |= top[r][e] != m[r][e];
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          float c[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            c[e] = top[r][e] == m[r][e] ? 1.0f : exp2_(m[r][e] - top[r][e]);
            m[r][e] = top[r][e];
            l[r][e] *= c[e];
          }
#pragma unroll
          for (int i = 0; i < G::kTiles; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][i][e] *= c[e & 1];
        }
      }
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        float p[RT][4];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float base = m[r][e & 1] == -INFINITY ? 0.0f : m[r][e & 1] - kLift;
            p[r][e] = exp2_(s[u][r][e] - base);
            l[r][e & 1] += p[r][e];
          }
        add_values(u, p);
      }
      if (!more) break;
      at = next;
    }
  }

  // The warps' sums to shared memory, and of all warps together (dims d .. d + 3 of row r).
  __device__ __forceinline__ void stage_sums(Shared& sh) const {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[r][e];
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
        if (g == 0) {
          sh.m[warp][8 * r + 2 * t + e] = m[r][e];
          sh.l[warp][8 * r + 2 * t + e] = x;
        }
      }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int i = 0; i < G::kTiles; ++i) {
        constexpr int kPer = G::kSpan / 2;
        const int d = (i / kPer) * 8 * G::kSpan + g * G::kSpan + 2 * (i % kPer);
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *reinterpret_cast<float2*>(&sh.o[warp][8 * r + 2 * t + e][d]) = make_float2(o[r][i][e], o[r][i][2 + e]);
      }
  }
  __device__ __forceinline__ static float4 warps_sum(const Shared& sh, int r, int d, float& top, float& sum) {
    top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.m[w][r]);
    sum = 0.0f;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float mw = sh.m[w][r], c = mw == top ? 1.0f : exp2_(mw - top);
      float4 y = *reinterpret_cast<const float4*>(&sh.o[w][r][d]);
      if constexpr (FOLD) {
        const float4 z = *reinterpret_cast<const float4*>(&sh.o[w][r + 4][d]);
        y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
      }
      sum += c * sh.l[w][r];
      x.x += c * y.x; x.y += c * y.y; x.z += c * y.z; x.w += c * y.w;
    }
    return x;
  }

  // A segment's sums to the output when it is whole, else to a partial slot.
  __device__ __forceinline__ void finish(const PagedArgs& a, Shared& sh, int b, int h, int row0, int n, uint32_t lo,
                                         uint32_t hi, bool whole, float* slot) {
    const int tid = threadIdx.x;
    stage_sums(sh);
    __syncthreads();
    const int rows = min(a.nodes * a.group - row0, kRows);
    const float v_scale = kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    const bool poison = too_long(a, b);
#pragma unroll 1
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i % (D / 4)) * 4;
      float top, sum;
      const float4 x = warps_sum(sh, r, d, top, sum);
      if (poison) sum = NAN;
      if (odd_sums(x)) atomicOr(&sh.odd, kOddSums);
      if (!whole) {
        *reinterpret_cast<float4*>(slot + r * D + d) = x;
        if (d == 0) {
          slot[kRows * D + 2 * r] = top;
          slot[kRows * D + 2 * r + 1] = sum;
        }
      } else {
        const int row = row0 + r, node = row / a.group;
        const int head = h * a.group + row - node * a.group;
        write_row<Q>(a, (long long)b * a.nodes + node, head, d, D, x, top, sum, v_scale, kLift);
      }
    }
    __syncthreads();
    if (sh.odd != 0) {
      if (tid < 32) {
        float top, sum = 0.0f;
        if (tid < rows) warps_sum(sh, tid, 0, top, sum);
        const uint32_t lost = __ballot_sync(0xffffffffu, poison || !(sum > 0.0f));
        if (tid == 0) sh.lost = lost;
      }
      add_odd_values<C, Q, D>(a, b, h, row0, rows, n, (int)lo * kBlock, (int)hi * kBlock, whole ? nullptr : slot, sh.odd,
                              &sh.o[0][0][0], &sh.lost);
    }
  }
};

// CTAs an SM, by registers.
template <class C, int D, int RT> constexpr int per_sm() {
  return sizeof(C) == 4 || RT * D >= 256 ? 2 : sizeof(C) == 2 && RT * D == 64 ? 4 : 3;
}

template <class C, class Q, int D, int RT, bool FOLD>
__global__ void __launch_bounds__(kThreads, per_sm<C, D, RT>()) paged_attention_kernel(const __grid_constant__ PagedArgs a) {
  using A = Attention<C, Q, D, RT, FOLD>;
  extern __shared__ __align__(16) uint8_t raw[];
  typename A::Shared& sh = *reinterpret_cast<typename A::Shared*>(raw);
  static_assert(offsetof(typename A::Shared, o) % 16 == 0 && sizeof(typename A::Shared) % 16 == 0, "16-byte loads");
  uint32_t* before = reinterpret_cast<uint32_t*>(raw + sizeof(typename A::Shared));
  __shared__ uint32_t scratch[kWarps];
  pdl_wait();
  pdl_trigger();                     // the joining kernel makes the same plan meanwhile
  const Plan plan = make_plan<A>(a, before, scratch, (int)gridDim.x);
  const Run run = make_run(a, plan, before);
  A at;
  each_segment<A>(a, run, before, [&](int b, int h, int row0, uint32_t lo, uint32_t hi, bool whole, float* slot) {
    A::stage_rows(a, sh, b, h, row0);
    __syncthreads();
    const int n = length_of(a, b);
    at.blocks(a, sh, b, h, row0, n, lo, hi);
    at.finish(a, sh, b, h, row0, n, lo, hi, whole, slot);
    __syncthreads();
  });
}

constexpr int kMostCtas = 8;

// Small tables: a cluster of CTAs a segment, each an equal share of its blocks, which join
// their sums through distributed shared memory: one launch, no partial sums in memory.
template <class C, class Q, int D, int RT, bool FOLD>
__global__ void __launch_bounds__(kThreads, per_sm<C, D, RT>()) paged_cluster_kernel(const __grid_constant__ PagedArgs a,
                                                                                     int ctas) {
  using A = Attention<C, Q, D, RT, FOLD>;
  extern __shared__ __align__(16) uint8_t raw[];
  typename A::Shared& sh = *reinterpret_cast<typename A::Shared*>(raw);
  // a CTA's maxima and sums of its rows, what it has met of odd values; of all CTAs
  __shared__ float mine_of[2 * A::kRows + 1], all[kMostCtas][2 * A::kRows + 1];
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, rank = (int)blockIdx.x % ctas, seg = (int)blockIdx.x / ctas;
  const int segments = a.kv_heads * a.row_blocks, b = seg / segments, h = (seg - b * segments) / a.row_blocks;
  const int row0 = (seg - b * segments - h * a.row_blocks) * A::kRows, rows = min(a.nodes * a.group - row0, A::kRows);
  const int n = length_of(a, b);
  if (blockIdx.x == 0 && tid == 0) ensure_header(a.header);
  int* met = reinterpret_cast<int*>(&mine_of[2 * A::kRows]);
  if (tid == 0) *met = 0;
  A::stage_rows(a, sh, b, h, row0);
  __syncthreads();
  const uint32_t blocks = (uint32_t)(n + A::kBlock - 1) / A::kBlock;
  const uint32_t each = (blocks + ctas - 1) / ctas, lo = min(rank * each, blocks), hi = min(lo + each, blocks);
  A at;
  at.blocks(a, sh, b, h, row0, n, lo, hi);
  at.stage_sums(sh);
  __syncthreads();
#pragma unroll 1
  for (int i = tid; i < rows * (D / 4); i += kThreads) {         // the CTA's sums, in the first warp's place
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
    float m, l;
    const float4 x = A::warps_sum(sh, r, d, m, l);
    *reinterpret_cast<float4*>(&sh.o[0][r][d]) = x;
    if (odd_sums(x)) atomicOr(met, kOddSums);
    if (d == 0) {
      mine_of[r] = m;
      mine_of[A::kRows + r] = l;
    }
  }
  if (tid == 0) atomicOr(met, sh.odd);
  tc::cluster_sync();
  // every value of the others is asked for at once: a load through the cluster takes as long
  // as a pass over the rows
  const float v_scale = A::kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
  const uint32_t theirs = tc::smem_u32(mine_of), sums_at = tc::smem_u32(&sh.o[0][0][0]);
  const int i0 = tid * ctas + rank, most = rows * (D / 4);
  float4 y[kMostCtas];
  auto fetch = [&](int i) {
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
#pragma unroll
    for (int q = 0; q < kMostCtas; ++q)
      if (q < ctas) y[q] = tc::ld_dsmem_f4(tc::map_dsmem(sums_at + (r * (D + 4) + d) * 4, q));
  };
  if (i0 < most) fetch(i0);
#pragma unroll 1
  for (int i = tid; i < ctas * (2 * A::kRows + 1); i += kThreads) {
    const int q = i / (2 * A::kRows + 1), e = i - q * (2 * A::kRows + 1);
    all[q][e] = dsmem_f32(theirs + 4 * e, q);
  }
  __syncthreads();
#pragma unroll 1
  for (int i = i0; i < most; i += kThreads * ctas) {
    const int r = i / (D / 4), d = (i % (D / 4)) * 4;
    if (i != i0) fetch(i);
    float m = -INFINITY, l = 0.0f;
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int q = 0; q < kMostCtas; ++q)
      if (q < ctas) m = fmaxf(m, all[q][r]);
#pragma unroll
    for (int q = 0; q < kMostCtas; ++q)
      if (q < ctas) {
        const float mq = all[q][r], c = mq == m ? 1.0f : exp2_(mq - m);
        l += c * all[q][A::kRows + r];
        x.x += c * y[q].x; x.y += c * y[q].y; x.z += c * y[q].z; x.w += c * y[q].w;
      }
    if (too_long(a, b)) l = NAN;
    const int row = row0 + r, node = row / a.group;
    write_row<Q>(a, (long long)b * a.nodes + node, h * a.group + row - node * a.group, d, D, x, m, l, v_scale, A::kLift);
  }
  int odd = 0;                       // of any of the cluster's CTAs: the first adds them
#pragma unroll 1
  for (int q = 0; rank == 0 && q < ctas; ++q) odd |= __float_as_int(all[q][2 * A::kRows]);
  tc::cluster_sync();
  if (odd == 0) return;
  if (tid < 32) {                    // the rows' sums again
    float m = -INFINITY, l = 0.0f;
#pragma unroll 1
    for (int q = 0; tid < rows && q < ctas; ++q) m = fmaxf(m, all[q][tid]);
#pragma unroll 1
    for (int q = 0; tid < rows && q < ctas; ++q) {
      const float mq = all[q][tid];
      l += (mq == m ? 1.0f : exp2_(mq - m)) * all[q][A::kRows + tid];
    }
    const uint32_t lost = __ballot_sync(0xffffffffu, too_long(a, b) || !(l > 0.0f));
    if (tid == 0) sh.lost = lost;
  }
  add_odd_values<C, Q, D>(a, b, h, row0, rows, n, 0, n, nullptr, odd, &sh.o[0][0][0], &sh.lost);
}

// More rows of a key head than kManyRows go to the kernels of many rows: that on tcgen05
// where the dims and the types allow it, 8-bit entries, which it has to widen on the way,
// only from more than kWideRows rows on.  us, here / mma.sync on staged tiles / tcgen05:
// bf16, 8 trees of 14 rows 12.7 / 23.5 / 17.7, of 28 rows 24.7 on the second and 19.2 on the
// third, of 32 rows and 32 key heads 46.4 and 39.5; e4m3, 24 rows 40.4 and 50.3, 64 rows 52.1
// and 58.6, 100 rows 85.8 and 77.0.
constexpr int kManyRows = 16, kWideRows = 64;
// Whether a warp takes 9 to 16 rows together: where its registers hold them.
template <class C, int D> constexpr bool kTwoTiles = sizeof(C) < 4 && D < 256;

// CTAs a segment for a cluster of them each, or 0: few segments, of a table that leaves a
// warp few steps, since a cluster whose sequence is shorter than its table idles.  One
// sequence of 640 entries, 32 heads: 7.4 us and one launch (7.4 us on the host), 9.5 and
// two (9.7) in runs; 4096 entries, 8 key heads: 12.2 and 15.3.  16 sequences of 1 to 4096
// entries: 25 and 17; 8 of 2048, 32 key heads: 55 and 44.
template <class A> int cluster_ctas(const PagedArgs& a, int resident) {
  const long long segments = (long long)a.B * a.kv_heads * ((a.nodes * a.group + A::kRows - 1) / A::kRows);
  int ctas = 1;
  while (ctas < kMostCtas && segments * ctas * 2 <= 152 * resident) ctas *= 2;
  const long long steps = ((long long)a.width * a.page + A::kBlock * kWarps * ctas - 1) / (A::kBlock * kWarps * ctas);
  return segments <= 152 * resident && steps <= (a.B == 1 ? 16 : 4) ? ctas : 0;
}

template <class C, class Q, int D, int RT, bool FOLD>
cudaError_t launch_cluster(PagedArgs a, int ctas, cudaStream_t s) {
  using A = Attention<C, Q, D, RT, FOLD>;
  static std::atomic<unsigned long long> raised{0};
  set_up<A>(a);
  cudaError_t e = raise_smem_limit(paged_cluster_kernel<C, Q, D, RT, FOLD>, 64 * 1024, raised);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((long long)a.B * a.kv_heads * a.row_blocks * ctas));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(typename A::Shared);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, paged_cluster_kernel<C, Q, D, RT, FOLD>, a, ctas);
}

template <class C, class Q, int D, int RT, bool FOLD = false>
cudaError_t launch_as(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  using A = Attention<C, Q, D, RT, FOLD>;
  static std::atomic<unsigned long long> raised{0};
  if (workspace == nullptr) {
    const int ctas = cluster_ctas<A>(a, per_sm<C, D, RT>());
    if (ctas > 0) return launch_cluster<C, Q, D, RT, FOLD>(a, ctas, s);
  }
  return launch_runs<A, C, Q, D>(a, paged_attention_kernel<C, Q, D, RT, FOLD>, kThreads, sizeof(typename A::Shared),
                                 152 * per_sm<C, D, RT>(), s, workspace, raised);
}

template <class C, class Q, int D>
cudaError_t launch_dim(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  const int rows = a.nodes * a.group;
  if (sizeof(C) < 4 && D < 256 && rows > (sizeof(C) == 2 ? kManyRows : kWideRows)) return launch_paged_tree(a, s, workspace);
  if (sizeof(C) < 4 && rows > kManyRows) return launch_paged_rows(a, s, workspace);
  if constexpr (kTwoTiles<C, D>)
    if (rows > 8) return launch_as<C, Q, D, 2>(a, s, workspace);
  if constexpr (sizeof(C) == 1)
    if (rows <= 4) return launch_as<C, Q, D, 1, true>(a, s, workspace);
  return launch_as<C, Q, D, 1>(a, s, workspace);
}
template <class C, class Q>
cudaError_t launch_type(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  return a.dim == 64 ? launch_dim<C, Q, 64>(a, s, workspace)
       : a.dim == 128 ? launch_dim<C, Q, 128>(a, s, workspace) : launch_dim<C, Q, 256>(a, s, workspace);
}
cudaError_t launch_any(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  return a.cache_dtype == FOVEA_BF16 ? launch_type<__nv_bfloat16, __nv_bfloat16>(a, s, workspace)
       : a.cache_dtype == FOVEA_E4M3 ? launch_type<__nv_fp8_e4m3, __nv_bfloat16>(a, s, workspace)
                                     : launch_type<float, float>(a, s, workspace);
}

}  // namespace

size_t paged_attention_workspace(const PagedArgs& a) {
  size_t n = 0;
  launch_any(a, nullptr, &n);
  return n;
}
cudaError_t launch_paged_attention(const PagedArgs& a, cudaStream_t s) { return launch_any(a, s, nullptr); }

}  // namespace fovea
