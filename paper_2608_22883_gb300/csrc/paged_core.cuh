// What the kernels of fovea_paged_attention share: the cut of the work into runs, which
// entries a row sees, the rows' results, and the joining of runs.
//
// The entries of all sequences and key heads are one list of blocks, cut into equal runs,
// one a CTA; a run covers parts of one or several (sequence, head, rows) segments.  A
// segment within one run is finished there; the others leave partial sums, which a second
// kernel joins in the order of the runs (results do not vary from run to run).
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
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
__device__ __forceinline__ uint32_t halves_of_e4m3(uint32_t two) {   // the low 16 bits: two values
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
  return (uint32_t)h.x | ((uint32_t)h.y << 16);
}
__device__ __forceinline__ uint32_t bits_of(__half2 x) { return *reinterpret_cast<const uint32_t*>(&x); }
__device__ __forceinline__ uint32_t bits_of(__nv_bfloat162 x) { return *reinterpret_cast<const uint32_t*>(&x); }

// x and y (below 2^16) as sums of two fp16 values each: 22 bits, or down to 2^-25.
__device__ __forceinline__ void split_halves(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __half2 h = __floats2half2_rn(x, y);
  const float2 back = __half22float2(h);
  hi = bits_of(h);
  lo = bits_of(__floats2half2_rn(x - back.x, y - back.y));
}

// The kernels' code is fetched by every SM when it is first run, which small calls wait
// for; divisions of 64 bits, a kilobyte each, stay out of line or are replaced here.
__device__ __noinline__ uint64_t divide_long(uint64_t x, uint32_t d) { return x / d; }

struct Plan {
  uint64_t total;      // blocks
  uint32_t runs;       // that have any
  uint64_t each;       // total / runs
  uint32_t rest;       // the first runs, which have one block more
  float runs_a_block;
  __device__ __forceinline__ uint64_t start(uint32_t run) const { return each * run + min(run, rest); }
  // The run of a block: start(run) <= block < start(run + 1), from an estimate near it.
  __device__ __forceinline__ uint32_t run_of(uint64_t block) const {
    uint32_t run = min((uint32_t)(__ull2float_rn(block) * runs_a_block), runs - 1);
#pragma unroll 1
    while (start(run) > block) --run;
#pragma unroll 1
    while (start(run + 1) <= block) ++run;
    return run;
  }
};

__device__ __forceinline__ int length_of(const PagedArgs& a, int b) { return max(0, min(a.lens[b], a.room)); }
__device__ __forceinline__ bool too_long(const PagedArgs& a, int b) { return a.lens[b] > a.room; }

// K, of a kernel: kWaits: its waits may give up; kBlock entries a block; kLeast blocks of a run, at least; kFront: the
// staging of a segment's rows and the end of its sums take a CTA as long as some blocks,
// and the runs are cut as if each segment had so many empty ones in front.
template <class K> __device__ __forceinline__ uint32_t blocks_of(int len) {
  return len > 0 ? (uint32_t)(len + K::kBlock - 1) / K::kBlock + K::kFront : 0;
}
// Sums of the sequences' blocks before each (before[0 .. B], in shared memory) and the
// cut into runs.  All threads of the CTA.
template <class K> __device__ __forceinline__ Plan make_plan(const PagedArgs& a, uint32_t* before, uint32_t* scratch,
                                                             int max_runs) {
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.B + nt - 1) / nt, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  uint32_t mine = 0;
#pragma unroll 1
  for (int b = b0; b < b1; ++b) mine += blocks_of<K>(length_of(a, b));
  uint32_t sum = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  if (lane == 31) scratch[warp] = sum;
  __syncthreads();
  uint32_t base = sum - mine;
#pragma unroll 1
  for (int w = 0; w < warp; ++w) base += scratch[w];
#pragma unroll 1
  for (int b = b0; b < b1; ++b) {
    before[b] = base;
    base += blocks_of<K>(length_of(a, b));
  }
  if (b1 == a.B && b0 < b1) before[a.B] = base;
  __syncthreads();
  Plan p;
  p.total = (uint64_t)before[a.B] * (uint32_t)(a.kv_heads * a.row_blocks);
  const uint64_t most = p.total < (uint64_t)max_runs * K::kLeast ? ((uint32_t)p.total + K::kLeast - 1) / K::kLeast : max_runs;
  p.runs = (uint32_t)most;
  const uint32_t d = max(p.runs, 1u);
  p.each = p.total >> 32 == 0 ? (uint32_t)p.total / d : divide_long(p.total, d);
  p.rest = (uint32_t)(p.total - p.each * d);
  p.runs_a_block = __fdividef((float)p.runs, __ull2float_rn(max(p.total, (uint64_t)1)));
  return p;
}

// Where a CTA's run begins, found once; each_segment goes on from there.
struct Run {
  uint64_t from, to;
  int b;               // sequence
  uint32_t seg, first; // its segment, the block within it
};
__device__ __forceinline__ Run make_run(const PagedArgs& a, const Plan& plan, const uint32_t* before) {
  Run r{};
  if (blockIdx.x >= plan.runs) return r;
  r.from = plan.start(blockIdx.x);
  r.to = plan.start(blockIdx.x + 1);
  const uint32_t segments = a.kv_heads * a.row_blocks;    // of a sequence, < 2^16
  int hi = a.B - 1;                  // the last b with before[b] * segments <= from
#pragma unroll 1
  while (r.b < hi) {
    const int mid = (r.b + hi + 1) >> 1;
    if ((uint64_t)before[mid] * segments <= r.from) r.b = mid; else hi = mid - 1;
  }
  const uint32_t count = before[r.b + 1] - before[r.b];   // not 0: `from` lies in it
  const uint64_t within = r.from - (uint64_t)before[r.b] * segments;
  r.seg = min((uint32_t)__fdividef(__ull2float_rn(within), (float)count), segments - 1);   // near it
#pragma unroll 1
  while ((uint64_t)r.seg * count > within) --r.seg;
#pragma unroll 1
  while ((uint64_t)(r.seg + 1) * count <= within) ++r.seg;
  r.first = (uint32_t)(within - (uint64_t)r.seg * count);
  return r;
}
// The segments of a CTA's run: body(sequence, key head, first row, first block, end, whether
// the segment is whole, its partial slot).
template <class K, class F>
__device__ __forceinline__ void each_segment(const PagedArgs& a, const Run& run, const uint32_t* before, F body) {
  float* slots = a.slots + (size_t)blockIdx.x * 2 * K::kSlot;
  const uint32_t segments = a.kv_heads * a.row_blocks;
  int b = run.b;
  uint32_t seg = run.seg, first = run.first;
#pragma unroll 1
  for (uint64_t u = run.from; u < run.to;) {
    const uint32_t count = before[b + 1] - before[b];
    if (seg == segments || count == 0) {                  // the next sequence
      ++b;
      seg = 0;
      continue;
    }
    const uint32_t end = (uint32_t)min((uint64_t)count, first + (run.to - u));
    // a segment that begins before or with this run goes to its first slot, a later one to its second
    const bool begun = u - first <= run.from;
    u += end - first;
    if (end > K::kFront) {
      const uint32_t lo = max(first, K::kFront) - K::kFront, hi = end - K::kFront;
      const int h = (int)(seg / (uint32_t)a.row_blocks);
      body(b, h, (int)(seg - h * a.row_blocks) * K::kRows, lo, hi, lo == 0 && hi == count - K::kFront,
           slots + (begun ? 0 : K::kSlot));
    }
    first = 0;
    ++seg;
  }
}

__device__ __forceinline__ const uint32_t* tree_of(const PagedArgs& a, int b) {
  return a.tree != nullptr ? a.tree + (size_t)(a.tree_rows == 1 ? 0 : b) * a.nodes * a.words : nullptr;
}
// Whether row `node` sees entry `at` of a sequence of n entries.
__device__ __forceinline__ bool sees(const PagedArgs& a, const uint32_t* tree, int n, int node, int at) {
  if (at >= n) return false;
  const int j = at - (n - a.nodes);
  if (j < 0) return true;
  if (tree == nullptr) return j <= node;
  return (tree[(size_t)node * a.words + (j >> 5)] >> (j & 31)) & 1u;
}
// The word of bits that tells which of the newest entries 32 w, 32 w + 1, ... row `node` sees
// (all before the newest, w < 0).
__device__ __forceinline__ uint32_t seen_word(const PagedArgs& a, const uint32_t* tree, int node, int w) {
  if (w < 0) return 0xFFFFFFFFu;
  if (tree != nullptr) return w < a.words ? tree[(size_t)node * a.words + w] : 0u;
  return node >= 32 * w + 31 ? 0xFFFFFFFFu : node < 32 * w ? 0u : (2u << (node - 32 * w)) - 1u;
}
__device__ __forceinline__ uint32_t below(int left) {      // the lowest `left` bits
  return left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
}
// Which of the entries first .. first + 31 (those from `end` on not) row `node` sees.
__device__ __forceinline__ uint32_t seen_bits(const PagedArgs& a, const uint32_t* tree, int n, int node, int first, int end) {
  const int j0 = first - (n - a.nodes), w0 = j0 >> 5;      // the first one's number among the newest
  return __funnelshift_r(seen_word(a, tree, node, w0), seen_word(a, tree, node, w0 + 1), j0 & 31) & below(end - first);
}
// The same of 64 entries.
__device__ __forceinline__ void seen_bits(const PagedArgs& a, const uint32_t* tree, int n, int node, int first, int end,
                                          uint32_t (&bits)[2]) {
  const int j0 = first - (n - a.nodes), w0 = j0 >> 5;
  const uint32_t middle = seen_word(a, tree, node, w0 + 1);
  bits[0] = __funnelshift_r(seen_word(a, tree, node, w0), middle, j0 & 31) & below(end - first);
  bits[1] = __funnelshift_r(middle, seen_word(a, tree, node, w0 + 2), j0 & 31) & below(end - first - 32);
}
// 16 bytes to shared memory, zeros when not `there` (nothing is read then).
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// Entries up to here are seen by all rows.
__device__ __forceinline__ int plain_end(const PagedArgs& a, int n) {
  return n - a.nodes + (a.nodes == 1 && a.tree == nullptr);
}

__device__ __forceinline__ float to_f32_any(float x) { return x; }
__device__ __forceinline__ float to_f32_any(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32_any(__nv_fp8_e4m3 x) { return float(x); }

// The odd halves, bytes or words of x as all ones: the exponent (of 8 bits: all seven) is
// ones where one more carries out of it.
template <class C> __device__ __forceinline__ uint32_t odd_in(uint32_t x) {
  if constexpr (sizeof(C) == 4) return (x & 0x7F800000u) == 0x7F800000u ? 0xFFFFFFFFu : 0u;
  else if constexpr (sizeof(C) == 1) return (((x & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0xFFu;
  else return (((x & 0x7F807F80u) + 0x00800080u) >> 15 & 0x00010001u) * 0xFFFFu;
}

// Values that are infinite or NaN ("odd"), which no product with p gets right: with a p of 0,
// of a row that does not see them, it is NaN, and p's upper and lower parts may differ in
// sign.  Among the newest entries, of which rows see different ones, they are cleared before
// the products; in front of them the sums lose their numbers (odd_sums).  When a segment's
// rows have been written (to out, or to a partial slot), every element with odd values among
// the entries from `from` to `to` that its row sees becomes their sum: infinite, or NaN.
enum Odd { kOddCleared = 1, kOddSums = 2 };                // what a segment has met
__device__ __forceinline__ bool odd_sums(const float4& x) {
  return fmaf(x.x, 0.0f, fmaf(x.y, 0.0f, fmaf(x.z, 0.0f, x.w * 0.0f))) != 0.0f;
}
__device__ __forceinline__ void bar_rows() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// By the CTA's first kThreads threads; front: D floats of theirs; lost: rows whose sum of p
// is 0 or no number, as bits, which stay as they are.
template <class C, class Q, int D>
__device__ __noinline__ void add_odd_values(const PagedArgs& a, int b, int h, int row0, int rows, int n, int from, int to,
                                            float* slot, int met, float* front, const uint32_t* lost) {
  const int tid = threadIdx.x;
  constexpr int kUnit = 16 / sizeof(C), kChunks = D / kUnit;
  const uint32_t* tree = tree_of(a, b);
  const int32_t* table = a.table + (size_t)b * a.width;
  const C* pool = static_cast<const C*>(a.v_pages);
  const int newest = max(n - a.nodes, 0);
  auto place = [&](int at) -> const C* {                   // null: not in the pool
    const int page = table[at / a.page];
    return (unsigned)page < (unsigned)a.n_pages ? pool + (((size_t)page * a.kv_heads + h) * a.page + at % a.page) * D : nullptr;
  };
  bar_rows();
#pragma unroll 1
  for (int d = tid; d < D; d += kThreads) front[d] = 0.0f;
  bar_rows();
  if (met & kOddSums) {              // of the entries that all rows see, one sum a dim
    float mine[kUnit] = {};
#pragma unroll 1
    for (int at = from + tid / kChunks; at < min(to, newest); at += kThreads / kChunks) {
      const C* p = place(at);
      if (p == nullptr) continue;
      const uint4 x = *reinterpret_cast<const uint4*>(p + tid % kChunks * kUnit);
      if ((odd_in<C>(x.x) | odd_in<C>(x.y) | odd_in<C>(x.z) | odd_in<C>(x.w)) == 0) continue;
#pragma unroll
      for (int i = 0; i < kUnit; ++i) {
        const float v = to_f32_any(reinterpret_cast<const C*>(&x)[i]);
        if (!isfinite(v)) mine[i] += v;
      }
    }
#pragma unroll
    for (int i = 0; i < kUnit; ++i)
      if (mine[i] != 0.0f) atomicAdd(&front[tid % kChunks * kUnit + i], mine[i]);   // the same in any order
  }
  bar_rows();
#pragma unroll 1
  for (int i = tid; i < rows * D; i += kThreads) {
    const int r = i / D, d = i % D, row = row0 + r, node = row / a.group;
    if (lost[r >> 5] >> (r & 31) & 1u) continue;
    float odd = front[d];
#pragma unroll 1
    for (int at = max(from, newest); at < min(to, n); ++at) {
      const C* p = sees(a, tree, n, node, at) ? place(at) : nullptr;
      const float v = p != nullptr ? to_f32_any(p[d]) : 0.0f;
      if (!isfinite(v)) odd += v;
    }
    if (odd == 0.0f) continue;
    if (slot != nullptr) slot[i] = odd;
    else static_cast<Q*>(a.out)[(((long long)b * a.nodes + node) * a.heads + h * a.group + row - node * a.group) * D + d] = from_f32<Q>(odd);
  }
}
// Dims d .. d + 3 of a row's result, from the sums of p v and of p (p times 2^lift).
template <class T>
__device__ __forceinline__ void write_row(const PagedArgs& a, long long n, int head, int d, int dim, float4 x, float top,
                                          float sum, float v_scale, float lift) {
  const float k = sum == 0.0f ? 0.0f : v_scale * __frcp_rn(sum);   // nothing seen: 0 (an infinite value stays NaN)
  T* out = static_cast<T*>(a.out) + (n * a.heads + head) * dim + d;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(x.x * k, x.y * k, x.z * k, x.w * k);
  } else {
    *reinterpret_cast<uint2*>(out) = make_uint2(bits_of(__floats2bfloat162_rn(x.x * k, x.y * k)),
                                                bits_of(__floats2bfloat162_rn(x.z * k, x.w * k)));
  }
  if (d == 0 && a.lse != nullptr)
    a.lse[n * a.heads + head] = sum == 0.0f ? -INFINITY : (top - lift + log2f(sum)) * kLn2;
}

// A power of two, with a reciprocal, that takes a row's largest magnitude, `top`, to [1, 2), for
// fp16; that of the very largest to [2, 4), subnormal ones (at least 2^-133) below 1.  1 for
// infinities.
__device__ __forceinline__ float row_power(float top) {
  const uint32_t e = __float_as_uint(top) >> 23;
  return e == 255 ? 1.0f : __uint_as_float(min(max(e, 1u), 253u) << 23);
}

// Where row r of a key head's rows stands in q.
template <class Q> __device__ __forceinline__ const Q* row_of(const PagedArgs& a, int b, int h, int r) {
  const int node = r / a.group;
  return static_cast<const Q*>(a.q) + ((long long)b * a.nodes + node) * a.q_ld +
         (long long)(h * a.group + (r - node * a.group)) * a.q_hs;
}

// Rows whose segment is cut between runs, joined in their order; rows of sequences without
// entries get 0.  A warp takes `chunk` rows of a key head together (a divisor of kRows), as
// a segment that one run has written is passed over whole.
template <class K, class C, class Q, int D>
__global__ void __launch_bounds__(kThreads) paged_join_kernel(const __grid_constant__ PagedArgs a, int runs, int chunk) {
  extern __shared__ __align__(16) uint8_t raw[];
  uint32_t* before = reinterpret_cast<uint32_t*>(raw);
  __shared__ uint32_t scratch[kWarps];
  const int lane = threadIdx.x & 31;
  const Plan plan = make_plan<K>(a, before, scratch, runs);
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x < 32) {               // the header, and the waits that gave up
    if (lane == 0) ensure_header(a.header);
    if constexpr (K::kWaits) {
      bool any = false;
#pragma unroll 1
      for (uint32_t run = lane; run < plan.runs; run += 32) any |= __ldcg(a.gave_up + run) != 0;
      if (__any_sync(0xffffffffu, any) && lane == 0) atomicOr(a.header, kErrTimeout);
    }
  }
  const uint32_t rows = a.nodes * a.group, chunks = (rows + chunk - 1) / chunk;
  const uint32_t items = (uint32_t)a.B * a.kv_heads * chunks;    // < 2^30
#pragma unroll 1
  for (uint32_t i = blockIdx.x * kWarps + (threadIdx.x >> 5); i < items; i += gridDim.x * kWarps) {
    const uint32_t head_of = i / chunks, row_from = (i - head_of * chunks) * chunk;
    const int b = (int)(head_of / a.kv_heads), h = (int)(head_of - b * a.kv_heads);
    const uint32_t segments = a.kv_heads * a.row_blocks, count = before[b + 1] - before[b];
    const float v_scale = sizeof(C) == 1 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    constexpr int kVecs = (D + 127) / 128, kAhead = 4;
    uint32_t first = 1, last = 0;    // runs; none
    bool second = false;             // the first run's second slot
    if (count != 0) {
      const uint64_t s0 = (uint64_t)before[b] * segments + (uint64_t)(h * a.row_blocks + row_from / K::kRows) * count;
      first = plan.run_of(s0 + K::kFront);
      last = plan.run_of(s0 + count - 1);
      if (first == last) continue;   // written already
      second = plan.start(first) < s0;
    }
    const uint32_t row_to = min(row_from + chunk, rows);
#pragma unroll 1
    for (uint32_t row = row_from; row < row_to; ++row) {
      float top = -INFINITY, sum = 0.0f;
      float4 x[kVecs];
#pragma unroll
      for (int c = 0; c < kVecs; ++c) x[c] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      const float* slot = a.slots + (size_t)(2 * first + second) * K::kSlot;   // of `run`
      const int r = row % K::kRows;
      // maxima and sums a lane a run, 32 runs at a time, with the first runs' sums of p v on
      // their way beside them
#pragma unroll 1
      for (uint32_t run0 = first; run0 <= last; run0 += 32) {
        const int left = (int)min(32u, last - run0 + 1);
        float2 ml = make_float2(-INFINITY, 0.0f);
        float c = 0.0f;              // of this lane's run
        if (lane < left)
          ml = __ldcg(reinterpret_cast<const float2*>(a.slots + (size_t)(2 * (run0 + lane) + (run0 + lane == first && second)) * K::kSlot +
                                                      K::kRows * D + 2 * r));
#pragma unroll 1
        for (int j0 = 0; j0 < left; j0 += kAhead) {
          float4 y[kAhead][kVecs];
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
              const int d = 128 * v + 4 * lane;
              y[j][v] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
              if (j0 + j < left && d < D) y[j][v] = __ldcg(reinterpret_cast<const float4*>(slot + r * D + d));
            }
            slot += run0 + j0 + j == first && second ? K::kSlot : 2 * K::kSlot;
          }
          if (j0 == 0) {
            float high = ml.x;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
            high = fmaxf(high, top);
            float keep = top == high ? 1.0f : exp2_(top - high);
            top = high;
            c = ml.x == top ? 1.0f : exp2_(ml.x - top);
            float mine = lane < left ? c * ml.y : 0.0f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
            sum = sum * keep + mine;
            // the weights of p v are not 0, so that an infinite sum stays one
            keep = fmaxf(keep, 0x1p-149f);
            c = fmaxf(c, 0x1p-149f);
#pragma unroll
            for (int v = 0; v < kVecs; ++v) {
              x[v].x *= keep; x[v].y *= keep; x[v].z *= keep; x[v].w *= keep;
            }
          }
#pragma unroll
          for (int j = 0; j < kAhead; ++j) {
            const float cj = __shfl_sync(0xffffffffu, c, (j0 + j) & 31);
            if (j0 + j < left) {
#pragma unroll
              for (int v = 0; v < kVecs; ++v) {
                x[v].x += cj * y[j][v].x; x[v].y += cj * y[j][v].y; x[v].z += cj * y[j][v].z; x[v].w += cj * y[j][v].w;
              }
            }
          }
        }
      }
      const int node = (int)(row / a.group), head = h * a.group + (int)row - node * a.group;
#pragma unroll
      for (int v = 0; v < kVecs; ++v) {
        const int d = 128 * v + 4 * lane;
        if (d < D) write_row<Q>(a, (long long)b * a.nodes + node, head, d, D, x[v], top, sum, v_scale, K::kLift);
      }
    }
  }
}

// What the kernels are told beside the call's arguments.
template <class K> void set_up(PagedArgs& a) {
  uint8_t* ws = static_cast<uint8_t*>(a.workspace);
  a.header = reinterpret_cast<int*>(ws);
  a.slots = reinterpret_cast<float*>(ws + kWsHeaderBytes);
  a.wait_ns = wait_limit_ns();
  const uint32_t per_page = a.page / 16;
  a.page_magic = per_page <= 1 ? 0 : (uint32_t)((1ull << 32) / per_page + 1);
  a.q_words = (reinterpret_cast<uintptr_t>(a.q) & 3) == 0 && a.q_ld % 2 == 0 && a.q_hs % 2 == 0;
  a.q_chunks = (reinterpret_cast<uintptr_t>(a.q) & 15) == 0 && a.q_ld % 8 == 0 && a.q_hs % 8 == 0;
  a.room = a.width * a.page;
  a.row_blocks = (a.nodes * a.group + K::kRows - 1) / K::kRows;
}

// Launches a kernel of `grid` CTAs and the joining one, or tells the workspace's bytes.
template <class K, class C, class Q, int D, class Kernel>
cudaError_t launch_runs(PagedArgs a, Kernel kernel, int threads, size_t shared, int grid, cudaStream_t s,
                        size_t* workspace, std::atomic<unsigned long long>& raised) {
  const size_t slots = (size_t)grid * 2 * K::kSlot * 4;
  if (workspace != nullptr) {
    *workspace = kWsHeaderBytes + slots + (size_t)grid * 4;
    return cudaSuccess;
  }
  set_up<K>(a);
  a.gave_up = reinterpret_cast<int*>(static_cast<uint8_t*>(a.workspace) + kWsHeaderBytes + slots);
  const size_t plan_bytes = ((size_t)a.B + 1) * 4;
  cudaError_t e = raise_smem_limit(kernel, 227 * 1024 - 1024, raised);
  if (e != cudaSuccess) return e;
  e = launch_pdl(kernel, dim3(grid), dim3(threads), shared + plan_bytes, s, a);
  if (e != cudaSuccess) return e;
  // rows a warp: few enough to leave every SM its warps
  int chunk = 4;
  const long long rows = (long long)a.nodes * a.group, heads = (long long)a.B * a.kv_heads;
  while (chunk > 1 && heads * ((rows + chunk - 1) / chunk) < 152 * 32) chunk /= 2;
  const long long ctas = (heads * ((rows + chunk - 1) / chunk) + kWarps - 1) / kWarps;
  return launch_pdl(paged_join_kernel<K, C, Q, D>, dim3((unsigned)(ctas < 152 * 8 ? ctas : 152 * 8)), dim3(kThreads),
                    plan_bytes, s, a, grid, chunk);
}

// The number of a block of 16 entries' page in the table: a page has 1 to 64 blocks and a
// sequence fewer than 2^26, for which the product is exact.
__device__ __forceinline__ uint32_t page_of(const PagedArgs& a, uint32_t block) {
  return a.page_magic == 0 ? block : __umulhi(block, a.page_magic);
}

}  // namespace

}  // namespace fovea
