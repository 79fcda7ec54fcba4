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
// The entries of all sequences and key heads are one list of blocks of 16, cut into equal
// runs, one a CTA; a run covers parts of one or several (sequence, head, rows) segments.
// A segment within one run is finished there; the others leave partial sums, which a
// second kernel joins in the order of the runs (results do not vary from run to run).
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>
#include <cstddef>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kBlock = 16;           // entries of a block
constexpr int kLeast = kWarps;       // blocks of a run, at least
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x5410); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __byte_perm(a, b, 0x7632); }

template <bool HALF>                 // HALF: fp16 operands, else bf16
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (HALF)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x as the sum of two tf32 values: hi its upper 11 bits, lo the other 13, of which the
// product reads 11 (an error of 2^-21 of x at most).
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t& hi, uint32_t& lo) {
  const bool finite = (x << 1) < 0xFF000000u;
  hi = finite ? x & 0xFFFFE000u : x;
  lo = finite ? __float_as_uint(__uint_as_float(x) - __uint_as_float(hi)) : 0u;
}
__device__ __forceinline__ uint32_t halves_of_e4m3(uint32_t two) {   // the low 16 bits: two values
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return (uint32_t)h.x | ((uint32_t)h.y << 16);
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

// A segment's rows are staged and its sums put together, which takes a CTA as long as some
// blocks: the runs are cut as if each segment had so many empty ones in front.  (The batch
// of 64 sequences of 0 to 8192 entries, us, with 0 / 4 / 8 / 16 / 24: 85 / 49 / 38 / 36 / 37;
// eight trees of 32 nodes 204 / 85 / 63 / 46 / 44.)
template <int RT> constexpr uint32_t kFront = RT == 1 ? 16 : 24;

// The blocks of all segments as one list: sequence by sequence, key head by key head, rows
// by rows.
struct Plan {
  uint64_t total;      // blocks
  uint32_t runs;       // that have any
  __device__ __forceinline__ uint64_t start(uint32_t run) const { return total * run / runs; }
  __device__ __forceinline__ uint32_t run_of(uint64_t block) const {     // start(run) <= block < start(run + 1)
    return (uint32_t)(((block + 1) * runs + total - 1) / total - 1);
  }
};

__device__ __forceinline__ int length_of(const PagedArgs& a, int b) {
  const int n = a.lens[b];
  const long long most = (long long)a.width * a.page;
  return n < 0 ? 0 : n > most ? (int)most : n;
}
__device__ __forceinline__ bool too_long(const PagedArgs& a, int b) { return a.lens[b] > (long long)a.width * a.page; }
__device__ __forceinline__ uint32_t blocks_of(int len, uint32_t front) {
  return len > 0 ? (uint32_t)(len + kBlock - 1) / kBlock + front : 0;
}

// Sums of the sequences' blocks before each (before[0 .. B], in shared memory) and the
// cut into runs.  All threads of the CTA.
__device__ Plan make_plan(const PagedArgs& a, uint32_t* before, uint32_t* scratch, int max_runs, uint32_t front) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.B + nt - 1) / nt, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  uint32_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += blocks_of(length_of(a, b), front);
  uint32_t sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 31) scratch[warp] = sum;
  __syncthreads();
  uint32_t base = sum - mine;
  for (int w = 0; w < warp; ++w) base += scratch[w];
  for (int b = b0; b < b1; ++b) {
    before[b] = base;
    base += blocks_of(length_of(a, b), front);
  }
  if (b1 == a.B && b0 < b1) before[a.B] = base;
  __syncthreads();
  Plan p;
  p.total = (uint64_t)before[a.B] * (uint32_t)(a.kv_heads * a.row_blocks);
  const uint64_t most = (p.total + kLeast - 1) / kLeast;
  p.runs = most < (uint64_t)max_runs ? (uint32_t)most : (uint32_t)max_runs;
  return p;
}

__device__ __forceinline__ const uint32_t* tree_of(const PagedArgs& a, int b) {
  return a.tree != nullptr ? a.tree + (size_t)(a.tree_rows == 1 ? 0 : b) * a.nodes * a.words : nullptr;
}
__device__ __forceinline__ float to_f32_any(float x) { return x; }
__device__ __forceinline__ float to_f32_any(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32_any(__nv_fp8_e4m3 x) { return float(x); }
// Whether row `node` sees entry `at` of a sequence of n entries.
__device__ __forceinline__ bool sees(const PagedArgs& a, const uint32_t* tree, int n, int node, int at) {
  if (at >= n) return false;
  const int j = at - (n - a.nodes);
  if (j < 0) return true;
  if (tree == nullptr) return j <= node;
  return (tree[(size_t)node * a.words + (j >> 5)] >> (j & 31)) & 1u;
}

// Blocks that a warp takes together.
template <class C, int D, int RT> constexpr int kTogether = sizeof(C) * D * RT <= 128 ? 2 : 1;

template <class C, class Q, int D, int RT>
struct Attention {
  using G = Cut<C, D>;
  static constexpr bool kF32 = sizeof(C) == 4, kE4 = sizeof(C) == 1;
  static constexpr int kRows = 8 * RT;
  static constexpr uint32_t kBytes = kBlock * D * sizeof(C);     // of a block
  // p of 8-bit values is held in fp16, times 2^15: its smallest step is then 2^-39
  static constexpr float kLift = kE4 ? 15.0f : 0.0f;

  struct Shared {
    uint2 q[RT][G::kSteps][32];      // Q^T's fragments
    float row_scale[kRows];          // of s, to powers of two
    int odd;                         // a masked block had infinite values or NaN
    float m[kWarps][kRows], l[kWarps][kRows];
    alignas(16) float o[kWarps][kRows][D + 4];
  };

  static constexpr int kSub = kTogether<C, D, RT>;
  // The keys and values of kSub blocks as a lane holds them.
  uint4 k[kSub][2][G::kKeyChunks];
  uint32_t v[kSub][4][G::kParts][G::kSpanWords];
  float o[RT][G::kTiles][4];
  float m[RT][2], l[RT][2];

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
      // the output's own rounding); 11 bits of fp16 beside values of four
      uint32_t bh[RT][2], bl[RT][2];
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float x = p[r][2 * e], y = p[r][2 * e + 1];
          if constexpr (kE4) {
            const __half2 h = __floats2half2_rn(x, y);
            bh[r][e] = transpose8(*reinterpret_cast<const uint32_t*>(&h));
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
          if constexpr (!kE4) mma16<kE4>(o[r][i], f, bl[r][0], bl[r][1]);
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

  // Values that are infinite or NaN, where only some rows see an entry: a product with a
  // p of 0 would give NaN to the others.  They are cleared here, and the rows that see one
  // take it when the segment is finished.  True where there was one.
  __device__ __forceinline__ bool clear_odd_values(int u) {
    uint32_t any = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int p = 0; p < G::kParts; ++p)
#pragma unroll
        for (int w = 0; w < G::kSpanWords; ++w) {
          uint32_t& x = v[u][e][p][w];
          uint32_t odd;
          if constexpr (kF32) odd = (x & 0x7F800000u) == 0x7F800000u ? 0xFFFFFFFFu : 0u;
          else if constexpr (kE4) odd = __vcmpeq4(x & 0x7F7F7F7Fu, 0x7F7F7F7Fu);
          else odd = __vcmpeq2(x & 0x7F807F80u, 0x7F807F80u);
          x &= ~odd;
          any |= odd;
        }
    return any != 0;
  }
  // Dims d .. d + 3 of such values of the entries from `from` to `to` that the row sees, added to x.
  __device__ __noinline__ static float4 odd_values(const PagedArgs& a, int b, int h, int node, int n, int from, int to,
                                                   int d, float4 x) {
    const uint32_t* tree = tree_of(a, b);
    for (int at = max(from, n - a.nodes); at < min(to, n); ++at) {
      const int page = a.table[(size_t)b * a.width + at / a.page];
      if (!sees(a, tree, n, node, at) || (unsigned)page >= (unsigned)a.n_pages) continue;
      const C* p = static_cast<const C*>(a.v_pages) + (((size_t)page * a.kv_heads + h) * a.page + at % a.page) * D + d;
      float* y = &x.x;
      for (int e = 0; e < 4; ++e) {
        const float value = to_f32_any(p[e]);
        if (!isfinite(value)) y[e] += value;
      }
    }
    return x;
  }

  // Q^T's fragments of the rows from row0 on.  All threads; between barriers of the caller.
  __device__ __forceinline__ static void stage_rows(const PagedArgs& a, Shared& sh, int b, int h, int row0) {
    const int tid = threadIdx.x, lane = tid & 31;
    const Q* q = static_cast<const Q*>(a.q);
    const int rows = a.nodes * a.group;
    auto row_at = [&](int r) -> const Q* {
      const int node = r / a.group;
      return q + ((long long)b * a.nodes + node) * a.q_ld + (long long)(h * a.group + (r - node * a.group)) * a.q_hs;
    };
    if (tid == 0) sh.odd = 0;
    if constexpr (kE4) {
      // rows to a largest magnitude in [1, 2), by a power of two, for fp16
      for (int r = tid >> 5; r < kRows; r += kWarps) {
        float top = 0.0f;
        if (row0 + r < rows) {
          const Q* p = row_at(row0 + r);
          for (int d = lane; d < D; d += 32) top = fmaxf(top, fabsf(to_f32(p[d])));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const uint32_t e = __float_as_uint(top) >> 23;
        // 2^(e - 127); 1 for rows of zeros, subnormals and infinities
        if (lane == 0) sh.row_scale[r] = e > 0 && e < 254 ? __uint_as_float(e << 23) : 1.0f;
      }
      __syncthreads();
    }
    for (int i = tid; i < RT * G::kSteps * 32; i += kThreads) {
      const int lane_of = i & 31, step = (i >> 5) % G::kSteps, r = (i >> 5) / G::kSteps;
      const int row = row0 + 8 * r + (lane_of >> 2), t = lane_of & 3;
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
    // Where a block's page stands in the table and where the block in its page: a page has
    // 1 to 64 blocks and a sequence fewer than 2^26, for which the product is exact.
    auto page_of = [&](uint32_t block) { return a.page_magic == 0 ? block : __umulhi(block, a.page_magic); };
    int id[kSub];
    uint32_t in_page[kSub];
    auto look_up = [&](uint32_t first) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const uint32_t block = u == 0 ? first : min(first + u, hi - 1), p = page_of(block);
        id[u] = table[p];
        in_page[u] = block - p * per_page;
      }
    };
    unsigned long long off[kSub];                          // bytes from the pools' lane pointers
    bool bad = false;                                      // a page is not in the pool
    auto place = [&]() {
      bad = false;
#pragma unroll
      for (int u = 0; u < kSub; ++u) {
        const bool out = (unsigned)id[u] >= (unsigned)a.n_pages;
        bad |= out;
        off[u] = ((unsigned long long)(out ? 0u : (uint32_t)id[u]) * stride + in_page[u]) * kBytes;
      }
    };
    look_up(at);
    place();
#pragma unroll
    for (int u = 0; u < kSub; ++u) load_keys(u, keys + off[u]);
    const int end = min(n, (int)(hi * kBlock));            // the run's last entry
    const int plain = min(end, n - a.nodes + (a.nodes == 1 && tree == nullptr));   // up to here all rows see all
    while (true) {
#pragma unroll
      for (int u = 0; u < kSub; ++u) load_values(u, values + off[u]);
      const uint32_t next = at + kWarps * kSub;
      const bool more = next < hi;
      if (more) look_up(next);
      float s[kSub][RT][4];
#pragma unroll
      for (int u = 0; u < kSub; ++u) scores(u, sh, s[u]);
      const bool was_bad = bad;
      if (more) {
        place();
#pragma unroll
        for (int u = 0; u < kSub; ++u) load_keys(u, keys + off[u]);
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
          const bool out = was_bad && start < end && (unsigned)table[page_of(at + u)] >= (unsigned)a.n_pages;
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int node = min((row0 + 8 * r + 2 * t + (e & 1)) / a.group, a.nodes - 1);
              const int entry = start + g + 8 * (e >> 1);
              const bool yes = entry < end && sees(a, tree, n, node, entry);
              s[u][r][e] = yes ? (out ? NAN : s[u][r][e]) : -INFINITY;
            }
          clear_values(u, out ? 0 : end - start);
          if ((a.nodes > 1 || tree != nullptr) && clear_odd_values(u)) sh.odd = 1;
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

  // The warps' sums of a segment together; written to the output when the segment is
  // whole, else to a partial slot.
  __device__ __forceinline__ void finish(const PagedArgs& a, Shared& sh, int b, int h, int row0, int n, uint32_t lo,
                                         uint32_t hi, bool whole, float* slot) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
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
    __syncthreads();
    const int rows = min(a.nodes * a.group - row0, kRows);
    const float v_scale = kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    const bool poison = too_long(a, b);
    for (int i = tid; i < rows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), d = (i % (D / 4)) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sh.m[w][r]);
      float sum = 0.0f;
      float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float mw = sh.m[w][r], c = mw == top ? 1.0f : exp2_(mw - top);
        const float4 y = *reinterpret_cast<const float4*>(&sh.o[w][r][d]);
        sum += c * sh.l[w][r];
        x.x += c * y.x; x.y += c * y.y; x.z += c * y.z; x.w += c * y.w;
      }
      if (poison) sum = NAN;
      if (sh.odd) x = odd_values(a, b, h, (row0 + r) / a.group, n, (int)lo * kBlock, (int)hi * kBlock, d, x);
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
  }

  template <class T>
  __device__ __forceinline__ static void write_row(const PagedArgs& a, long long n, int head, int d, int dim, float4 x,
                                                   float top, float sum, float v_scale, float lift) {
    const float k = sum == 0.0f ? 0.0f : v_scale / sum;    // nothing seen: 0 (an infinite value stays NaN)
    T* out = static_cast<T*>(a.out) + (n * a.heads + head) * dim + d;
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4*>(out) = make_float4(x.x * k, x.y * k, x.z * k, x.w * k);
    } else {
      const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x * k, x.y * k), hi = __floats2bfloat162_rn(x.z * k, x.w * k);
      *reinterpret_cast<uint2*>(out) =
          make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
    if (d == 0 && a.lse != nullptr)
      a.lse[n * a.heads + head] = sum == 0.0f ? -INFINITY : (top - lift + log2f(sum)) * kLn2;
  }
};

// CTAs an SM, by registers.
template <class C, int D, int RT> constexpr int per_sm() {
  return sizeof(C) == 4 || RT * D >= 256 ? 2 : 3;
}

template <class C, class Q, int D, int RT>
__global__ void __launch_bounds__(kThreads, per_sm<C, D, RT>()) paged_attention_kernel(const __grid_constant__ PagedArgs a) {
  using A = Attention<C, Q, D, RT>;
  extern __shared__ __align__(16) uint8_t raw[];
  typename A::Shared& sh = *reinterpret_cast<typename A::Shared*>(raw);
  uint32_t* before = reinterpret_cast<uint32_t*>(raw + sizeof(typename A::Shared));
  static_assert(offsetof(typename A::Shared, o) % 16 == 0 && sizeof(typename A::Shared) % 16 == 0, "16-byte loads");
  __shared__ uint32_t scratch[kWarps];
  constexpr uint32_t front = kFront<RT>;
  pdl_wait();
  pdl_trigger();                     // the joining kernel makes the same plan meanwhile
  const Plan plan = make_plan(a, before, scratch, (int)gridDim.x, front);
  if (blockIdx.x >= plan.runs) return;
  const uint64_t from = plan.start(blockIdx.x), to = plan.start(blockIdx.x + 1);
  const uint32_t segments = a.kv_heads * a.row_blocks;    // of a sequence
  float* slots = static_cast<float*>(a.workspace) + (size_t)blockIdx.x * 2 * A::kRows * (D + 2);
  int b = 0;
  {
    int hi = a.B - 1;                // the last b with before[b] * segments <= from
    while (b < hi) {
      const int mid = (b + hi + 1) >> 1;
      if ((uint64_t)before[mid] * segments <= from) b = mid; else hi = mid - 1;
    }
  }
  A at;
  for (uint64_t u = from; u < to;) {
    while ((uint64_t)before[b + 1] * segments <= u) ++b;
    const uint32_t count = before[b + 1] - before[b];
    const uint64_t within = u - (uint64_t)before[b] * segments;
    const uint32_t seg = (uint32_t)(within / count), first = (uint32_t)(within % count);
    const uint32_t end = (uint32_t)min((uint64_t)count, first + (to - u));
    // a segment that begins before or with this run goes to its first slot, a later one to its second
    const bool begun = u - first <= from;
    u += end - first;
    if (end <= front) continue;
    const uint32_t lo = max(first, front) - front, hi = end - front;
    const int h = seg / a.row_blocks, row0 = (seg % a.row_blocks) * A::kRows;
    A::stage_rows(a, sh, b, h, row0);
    __syncthreads();
    const int n = length_of(a, b);
    at.blocks(a, sh, b, h, row0, n, lo, hi);
    at.finish(a, sh, b, h, row0, n, lo, hi, lo == 0 && hi == count - front, slots + (begun ? 0 : A::kRows * (D + 2)));
    __syncthreads();
  }
}

// A row whose segment is cut between runs, joined in their order; rows of sequences
// without entries get 0.  A warp a row.
template <class C, class Q, int D, int RT>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const __grid_constant__ PagedArgs a, int runs) {
  using A = Attention<C, Q, D, RT>;
  extern __shared__ __align__(16) uint8_t raw[];
  uint32_t* before = reinterpret_cast<uint32_t*>(raw);
  __shared__ uint32_t scratch[kWarps];
  constexpr uint32_t front = kFront<RT>;
  const int lane = threadIdx.x & 31;
  const Plan plan = make_plan(a, before, scratch, runs, front);
  pdl_wait();
  const long long rows = (long long)a.B * a.nodes * a.heads;
  for (long long i = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); i < rows; i += (long long)gridDim.x * kWarps) {
    const long long n = i / a.heads;
    const int head = (int)(i - n * a.heads), b = (int)(n / a.nodes), node = (int)(n - (long long)b * a.nodes);
    const int h = head / a.group, row = node * a.group + head - h * a.group;
    const uint32_t segments = a.kv_heads * a.row_blocks, count = before[b + 1] - before[b];
    const float v_scale = A::kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    if (count == 0) {
      for (int d = 4 * lane; d < D; d += 128)
        A::template write_row<Q>(a, n, head, d, D, make_float4(0.0f, 0.0f, 0.0f, 0.0f), -INFINITY, 0.0f, 1.0f, 0.0f);
      continue;
    }
    const uint64_t s0 = (uint64_t)before[b] * segments + (uint64_t)(h * a.row_blocks + row / A::kRows) * count;
    const uint32_t first = plan.run_of(s0 + front), last = plan.run_of(s0 + count - 1);
    if (first == last) continue;     // written already
    const float* base = static_cast<const float*>(a.workspace);
    const int r = row % A::kRows;
    auto slot = [&](uint32_t run) {
      return base + ((size_t)run * 2 + (run == first && plan.start(run) < s0)) * A::kRows * (D + 2);
    };
    float top = -INFINITY;
    for (uint32_t run = first + lane; run <= last; run += 32) top = fmaxf(top, __ldcg(slot(run) + A::kRows * D + 2 * r));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float sum = 0.0f;
    constexpr int kVecs = (D + 127) / 128;
    float4 x[kVecs];
#pragma unroll
    for (int c = 0; c < kVecs; ++c) x[c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (uint32_t run = first; run <= last; ++run) {
      const float* p = slot(run);
      const float2 ml = __ldcg(reinterpret_cast<const float2*>(p + A::kRows * D + 2 * r));
      const float c = ml.x == top ? 1.0f : exp2_(ml.x - top);
      sum += c * ml.y;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int d = 128 * v + 4 * lane;
        if (d < D) {
          const float4 y = __ldcg(reinterpret_cast<const float4*>(p + r * D + d));
          x[v].x += c * y.x; x[v].y += c * y.y; x[v].z += c * y.z; x[v].w += c * y.w;
        }
      }
    }
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
      const int d = 128 * v + 4 * lane;
      if (d < D) A::template write_row<Q>(a, n, head, d, D, x[v], top, sum, v_scale, A::kLift);
    }
  }
}

// Rows that a warp takes together, by 8: as many as there are, up to what its registers hold.
template <class C, int D> constexpr int most_tiles() {
  return sizeof(C) == 4 || D == 256 ? 1 : D == 128 ? 2 : 4;
}

template <class C, class Q, int D, int RT>
cudaError_t launch_as(PagedArgs a, cudaStream_t s, size_t* workspace) {
  using A = Attention<C, Q, D, RT>;
  const uint32_t per_page = a.page / kBlock;
  a.page_magic = per_page <= 1 ? 0 : (uint32_t)((1ull << 32) / per_page + 1);
  a.row_blocks = (a.nodes * a.group + A::kRows - 1) / A::kRows;
  const size_t plan_bytes = ((size_t)a.B + 1) * 4;
  const size_t smem = sizeof(typename A::Shared) + plan_bytes;
  static std::atomic<unsigned long long> raised{0};
  const int grid = 152 * per_sm<C, D, RT>();
  if (workspace != nullptr) {
    *workspace = (size_t)grid * 2 * A::kRows * (D + 2) * 4;
    return cudaSuccess;
  }
  cudaError_t e = raise_smem_limit(paged_attention_kernel<C, Q, D, RT>, 227 * 1024 - 1024, raised);
  if (e != cudaSuccess) return e;
  e = launch_pdl(paged_attention_kernel<C, Q, D, RT>, dim3(grid), dim3(kThreads), smem, s, a);
  if (e != cudaSuccess) return e;
  const long long rows = (long long)a.B * a.nodes * a.heads;
  const int join = (int)((rows + kWarps - 1) / kWarps < 152 * 8 ? (rows + kWarps - 1) / kWarps : 152 * 8);
  return launch_pdl(paged_join_kernel<C, Q, D, RT>, dim3(join), dim3(kThreads), plan_bytes, s, a, grid);
}

template <class C, class Q, int D>
cudaError_t launch_dim(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  const int rows = a.nodes * a.group;
  if constexpr (most_tiles<C, D>() >= 4)
    if (rows > 16) return launch_as<C, Q, D, 4>(a, s, workspace);
  if constexpr (most_tiles<C, D>() >= 2)
    if (rows > 8) return launch_as<C, Q, D, 2>(a, s, workspace);
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
