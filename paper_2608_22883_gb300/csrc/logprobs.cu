// Log probabilities of given tokens with entropy and the best alternatives
// (fovea_token_logprobs), and their gradient (fovea_token_logprobs_grad).
// With z_i = logit_i * row_scale over a row's allowed tokens (z = -inf for the
// others):
//   lse = log sum_i e^{z_i},  logp_i = z_i - lse,  H = -sum_i p_i logp_i
//   dz_i = [gradients of the tokens equal to i] - p_i G - g_H p_i (logp_i + H) + g_lse p_i
// with G the sum of the counted tokens' gradients.
#include "common.cuh"
#include "packed.cuh"
#include "rowmath.cuh"
#include "tc_ptx.cuh"

namespace fovea {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kGroups = kThreads / 4;   // four neighbouring lanes' tokens are one group of the selection
constexpr int kCands = 512;             // candidate keys a CTA collects
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float ex2(float x) {       // 2^x, subnormal results as 0
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// e^x for a gradient that is stored in fp32.  It is 2^t with t = x log2 e; the rounding of t
// (u |t|, ten times u and more for most tokens' log probabilities) is put back with the
// remainder r = x - t ln 2 as 2^t (1 + r).  A gradient in bf16 does without: its own
// rounding is 2^15 u (and with it 4096 rows of 32000 took 91.2 us for 81.7; 2048 fp32 rows
// 84.1 both ways).
template <class T>
__device__ __forceinline__ uint64_t exp_for(uint64_t x) {  // two of them
  constexpr float kLn2 = 0.6931471805599453f, kLn2Lo = (float)(0.6931471805599453 - (double)kLn2);
  const uint64_t t = mul2(x, pack2(kLog2e, kLog2e));
  const uint64_t e = pack2(ex2(lo2(t)), ex2(hi2(t)));
  if (sizeof(T) == 2) return e;
  const uint64_t r = fma2(t, pack2(-kLn2Lo, -kLn2Lo), fma2(t, pack2(-kLn2, -kLn2), x));
  return fma2(e, r, e);
}

// z of a logit: the product rounded once, also where a difference follows that the compiler
// would fuse with it (z - max of the largest is 0 then, and no log probability above 0).
__device__ __forceinline__ float z_of(float x, float scale) { return __fmul_rn(x, scale); }
template <bool SCALED>
__device__ __forceinline__ uint64_t z_of2(float x0, float x1, float scale) {
  const uint64_t x = pack2(x0, x1);
  return SCALED ? product2(x, pack2(scale, scale)) : x;
}

// Order of logits as signed integers: every NaN above +inf (and not the largest integer:
// no key below is ~0), both zeros equal.
__device__ __forceinline__ int32_t order_of(float x) {
  if (x != x) return 0x7FFFFFFE;
  const int32_t b = __float_as_int(x + 0.0f);
  return b < 0 ? b ^ 0x7FFFFFFF : b;
}
__device__ __forceinline__ float value_of(int32_t o) { return __int_as_float(o < 0 ? o ^ 0x7FFFFFFF : o); }
constexpr int32_t kOrderNegInf = (int32_t)0x807FFFFF;     // order_of(-inf)

// A token's key: larger logits first, then the lower token; neither 0 nor ~0.
__device__ __forceinline__ unsigned long long key_of(int32_t order, int token) {
  return (unsigned long long)((uint32_t)order ^ 0x80000000u) << 32 | (uint32_t)~token;
}
__device__ __forceinline__ int token_of(unsigned long long key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ int32_t order_in(unsigned long long key) {
  return (int32_t)((uint32_t)(key >> 32) ^ 0x80000000u);
}

// One row's logits in 16-byte chunks of the address space: chunk c holds the
// tokens c * NV - shift ... of the row, those outside [0, V) as -inf.  Only
// chunks that lie in the row whole are read as vectors.
template <class T>
struct Row {
  static constexpr int NV = VecOf<T>::N;
  const T* p;
  int V, shift, chunks;
  const uint32_t* allowed;

  __device__ __forceinline__ Row(const void* base, long long ld, long long row, int V_,
                                 const uint32_t* allowed_, long long allowed_ld)
      : p(static_cast<const T*>(base) + row * ld), V(V_) {
    shift = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    chunks = (int)(((long long)V + shift + NV - 1) / NV);
    allowed = allowed_ != nullptr ? allowed_ + row * allowed_ld : nullptr;
  }
  __device__ __forceinline__ int first(int c) const { return c * NV - shift; }
  __device__ __forceinline__ bool whole(int c) const { return first(c) >= 0 && first(c) + NV <= V; }
  // The first and last chunk of the row that are whole.
  __device__ __forceinline__ int whole_lo() const { return shift != 0 ? 1 : 0; }
  __device__ __forceinline__ int whole_hi() const { return (V + shift) / NV; }
  // Bits of the tokens of a chunk (those outside the row: any).
  __device__ __forceinline__ uint32_t bits(int c) const {
    const int i0 = first(c), last = (V - 1) >> 5;
    const uint32_t lo = allowed[max(i0, 0) >> 5], hi = allowed[min((i0 + NV - 1) >> 5, last)];
    return i0 < 0 ? lo << -i0 : __funnelshift_r(lo, hi, i0 & 31);
  }
  __device__ __forceinline__ uint4 raw(int c) const {            // of a whole chunk
    return *reinterpret_cast<const uint4*>(p + first(c));        // (which the gradient may overwrite)
  }
  __device__ __forceinline__ void mask(uint32_t m, float (&v)[NV]) const {
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (!(m >> i & 1u)) v[i] = -INFINITY;
  }
  __device__ __forceinline__ void load(int c, float (&v)[NV]) const {
    const int i0 = first(c);
    if (whole(c)) {
      ln_unpack<T>(raw(c), v);
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) v[i] = i0 + i >= 0 && i0 + i < V ? to_f32(p[i0 + i]) : -INFINITY;
    }
    if (allowed != nullptr) mask(bits(c), v);
  }
  // One token's logit: -inf where it is not allowed.
  __device__ __forceinline__ float at(int k) const {
    if (allowed != nullptr && !((allowed[k >> 5] >> (k & 31)) & 1u)) return -INFINITY;
    return to_f32(p[k]);
  }
};

// Running softmax sums about a reference m (one of the row's z, which the largest seen
// passes by 2 at most):
// S = sum e^{z - m}, W = sum e^{z - m} (z - m).
struct Sums {
  float m, S, W;
};
// The same sums about m2 >= m (or about the first m, when nothing was summed).
__device__ __forceinline__ void rebase(Sums& a, float m2) {
  // e^{-200} is 0 in fp32; without the bound S dm can overflow (a reference near
  // the type's lowest value) and leave 0 * inf
  const float dm = max_nan(a.m - m2, -200.0f);
  const float f = a.m == -INFINITY ? 0.0f : ex2(dm * kLog2e);
  a.W = a.m == -INFINITY ? 0.0f : f * fmaf(a.S, dm, a.W);
  a.S *= f;
  a.m = m2;
}
// The sums of both about the larger reference; the smaller one's are rescaled.
__device__ __forceinline__ void join(Sums& a, Sums b) {
  const bool up = !(b.m <= a.m);                           // (a NaN goes through d)
  const Sums hi = up ? b : a, lo = up ? a : b;
  const float m = max_nan(a.m, b.m);
  const float d = lo.m == -INFINITY ? 0.0f : max_nan(lo.m - m, -200.0f);   // nothing summed: S, W are 0
  const float f = ex2(d * kLog2e);
  a.S = fmaf(f, lo.S, hi.S);
  a.W = fmaf(f, fmaf(lo.S, d, lo.W), hi.W);
  a.m = m;
}

// A thread's sums over the tokens it has seen (even and odd ones apart), and the
// largest logit with its chunk.
struct Seen {
  float m = -INFINITY;
  uint64_t S = 0, W = 0;
  float top = -INFINITY;
  int chunk = 0;

  __device__ __forceinline__ Sums sums() const { return Sums{m, lo2(S) + hi2(S), lo2(W) + hi2(W)}; }
  // Before the first chunk, by a whole warp: the largest logit of its lanes' chunks as the
  // reference, which few later ones pass by 2.
  template <int NV>
  __device__ __forceinline__ void seed(const float (&v)[NV], float scale) {
    float cm = v[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) cm = max_nan(cm, v[i]);
    const float z = z_of(value_of(__reduce_max_sync(0xffffffffu, order_of(cm))), scale);
    if (fabsf(z) < INFINITY) m = z;
  }
  // One chunk's logits; a NaN among them makes the sums NaN.  ASCENDING: no later chunk
  // was taken before this one (of equal logits the lowest chunk's is kept).
  template <bool SCALED, bool ASCENDING = true, int NV>
  __device__ __forceinline__ void take(const float (&v)[NV], int c, float scale) {
    float cm = v[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) cm = max_nan(cm, v[i]);
    const float zm = z_of(cm, scale);
    if (zm == -INFINITY) return;
    if (cm > top || (!ASCENDING && cm == top && c < chunk)) {
      top = cm;
      chunk = c;
    }
    if (!(zm <= m + 2.0f)) {
      Sums a = {m, lo2(S), lo2(W)}, b = {m, hi2(S), hi2(W)};
      rebase(a, zm);
      rebase(b, zm);
      m = zm;
      S = pack2(a.S, b.S);
      W = pack2(a.W, b.W);
    }
    const uint64_t m2 = pack2(-m, -m), log2e2 = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int i = 0; i < NV; i += 2) {
      const uint64_t d = add2(z_of2<SCALED>(v[i], v[i + 1], scale), m2);
      // -inf: e^{-200} is 0 and so is its term of W
      const uint64_t dz = pack2(max_nan(lo2(d), -200.0f), max_nan(hi2(d), -200.0f));
      const uint64_t x = mul2(dz, log2e2);
      const uint64_t e = pack2(ex2(lo2(x)), ex2(hi2(x)));
      S = add2(S, e);
      W = fma2(e, dz, W);
    }
  }
};

struct Shared {
  float m[kWarps], S[kWarps], W[kWarps];
  unsigned long long upper[kGroups];   // no key of the group is above it
  unsigned long long lower[kGroups];   // some key of the group is at least this
  unsigned long long threshold;
  unsigned long long cand[kCands];
  unsigned long long best[FOVEA_MAX_KC];
  unsigned long long red[kWarps];
  int count;
  // of the whole row (leading CTA): what the others left
  Sums total;
  unsigned long long all[kMaxCluster * FOVEA_MAX_KC];
};

// A cluster of CTAs takes one row, each a range of its chunks.  One pass
// over the logits keeps the softmax sums and, per group of four lanes, the
// largest logit.  The k-th largest of the groups' bounds is a threshold that at
// least k tokens reach, so only groups that reach it (k of them, and ties) are
// read again, from L2, for the tokens above it: a few more than k.
//
// Instructions bound the pass (two fp32 operations in one where there is such a form)
// and latency the search.  4096 rows of 32000 bf16: 49 us without alternatives (78 % of
// the measured copy's bandwidth), 69.5 us with six (56 %), 98 with 32, 72.4 with six under
// temperatures; 2048 masked 49.2 (42 %); 2048 fp32 rows 55 (70 %); one fp32 row of 32000
// 7.1 us, where the cluster's two meetings and the search's steps follow one another.
// 256 threads: 128 and 512 measured no better.
//
// Six CTAs an SM are worth 40 registers to unmasked bf16 rows (72.6 to 69.6 us) and not to
// the others (masked bf16 a fifth slower, fp32 2 %).
template <class T, bool MASKED, bool SCALED>
__global__ void __launch_bounds__(kThreads, (sizeof(T) == 2 && !MASKED ? 6 : 0))
token_logprobs_kernel(const ScoreArgs a) {
  constexpr int NV = Row<T>::NV;
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, rank = blockIdx.x;       // the cluster spans the grid's x
  const long long n = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  const Row<T> row(a.logits, a.ld, n, a.V, a.allowed, a.allowed_ld);
  const float scale = SCALED ? a.row_scale[n] : 1.0f;
  const int per = (row.chunks + ctas - 1) / ctas;
  const int c_lo = min(rank * per, row.chunks), c_hi = min(c_lo + per, row.chunks);

  // whole chunks lo + tid, + kThreads, ... of this CTA; and the row's ragged ends, the
  // first one thread 0's, the last one thread 1's
  const int lo = max(c_lo, row.whole_lo()), hi = min(c_hi, row.whole_hi());
  auto ragged = [&](int i) {                               // chunk of end i, or -1
    const int e = i == 0 ? 0 : row.chunks - 1;
    return e >= c_lo && e < c_hi && !row.whole(e) && (i == 0 || e != 0) ? e : -1;
  };
  Seen seen;
  {
    // chunks on their way together (4096 rows of 32000 bf16, 4, 3 and 5: 69.6, 70.5 and 71.5
    // us; 64 masked fp32 rows 3 and 4: 10.5 and 10.9; 64 unmasked 6 and 4: 9.2 and 9.7)
    constexpr int U = MASKED ? 3 : sizeof(T) == 4 ? 6 : 4;
    int c = lo + tid;
    bool seeded = lo + (tid | 31) + (U - 1) * kThreads >= hi;      // no round of a whole warp
    for (; c + (U - 1) * kThreads < hi; c += U * kThreads) {
      uint4 raw[U];
      uint32_t keep[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        raw[u] = row.raw(c + u * kThreads);
        if (MASKED) keep[u] = row.bits(c + u * kThreads);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[NV];
        ln_unpack<T>(raw[u], v);
        if (MASKED) row.mask(keep[u], v);
        if (u == 0 && !seeded) {
          seen.seed(v, scale);
          seeded = true;
        }
        seen.take<SCALED>(v, c + u * kThreads, scale);
      }
    }
    if (c < hi) {                                          // the last round, cut short
      uint4 raw[U - 1];
      uint32_t keep[U - 1];
#pragma unroll
      for (int u = 0; u < U - 1; ++u) {
        const int at = min(c + u * kThreads, hi - 1);
        raw[u] = row.raw(at);
        if (MASKED) keep[u] = row.bits(at);
      }
#pragma unroll
      for (int u = 0; u < U - 1; ++u) {
        if (c + u * kThreads >= hi) break;
        float v[NV];
        ln_unpack<T>(raw[u], v);
        if (MASKED) row.mask(keep[u], v);
        seen.take<SCALED>(v, c + u * kThreads, scale);
      }
    }
    if (tid < 2 && ragged(tid) >= 0) {
      float v[NV];
      row.load(ragged(tid), v);
      seen.take<SCALED, false>(v, ragged(tid), scale);             // thread 0's comes before its whole ones
    }
  }
  Sums s = seen.sums();
  int32_t top = order_of(seen.top);
  const int top_chunk = seen.chunk;
  // the largest z itself (the reference is one of the row's)
  if (top != kOrderNegInf && z_of(seen.top, scale) > s.m) rebase(s, z_of(seen.top, scale));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Sums b;
    b.m = __shfl_xor_sync(0xffffffffu, s.m, o);
    b.S = __shfl_xor_sync(0xffffffffu, s.S, o);
    b.W = __shfl_xor_sync(0xffffffffu, s.W, o);
    join(s, b);
  }
  if (lane == 0) {
    sh.m[warp] = s.m;
    sh.S[warp] = s.S;
    sh.W[warp] = s.W;
  }
  if (tid == 0) sh.count = 0;
  if (a.k > 0) {
    // tokens of the chunk lie in [first, first + NV): bounds of the group's best key
    unsigned long long up = 0, low = 0;
    if (top != kOrderNegInf) {
      up = key_of(top, max(row.first(top_chunk), 0));
      low = key_of(top, row.first(top_chunk) + NV - 1);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const unsigned long long u2 = __shfl_xor_sync(0xffffffffu, up, o), l2 = __shfl_xor_sync(0xffffffffu, low, o);
      up = u2 > up ? u2 : up;
      low = l2 > low ? l2 : low;
    }
    if ((lane & 3) == 0) {
      sh.upper[tid >> 2] = up;
      sh.lower[tid >> 2] = low;
    }
    if (tid == 0) sh.threshold = 1ull;                 // fewer than k groups with a token: every token
  }
  __syncthreads();
  if (tid == kThreads - 32) {                              // not of a warp that ranks below
    Sums t = {sh.m[0], sh.S[0], sh.W[0]};
    for (int w = 1; w < kWarps; ++w) join(t, Sums{sh.m[w], sh.S[w], sh.W[w]});
    sh.total = t;
  }
  if (a.k > 0) {
    if (tid < kGroups && sh.lower[tid] != 0ull) {
      const unsigned long long mine = sh.lower[tid];
      int above = 0;
#pragma unroll 8
      for (int i = 0; i < kGroups; ++i) above += sh.lower[i] > mine;
      if (above == a.k - 1) sh.threshold = mine;       // keys are distinct
    }
    if (tid < a.k) sh.best[tid] = 0ull;
    __syncthreads();
    // a NaN (or +inf) is in no bound: then every token is looked at
    const bool odd = sh.total.S != sh.total.S;
    const unsigned long long threshold = odd ? 1ull : sh.threshold;
    // no key at or above the threshold has a logit below this (a NaN lets all pass)
    const float least = value_of(order_in(threshold));
    auto each_key = [&](int gr, auto&& f) {                // of a group's tokens, by a warp
      constexpr int U = 2;                                 // chunks on their way together
      for (int c = lo + gr * 4 + (lane >> 2) * kThreads + (lane & 3); c < hi; c += U * 8 * kThreads) {
        uint4 raw[U];
        uint32_t keep[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = min(c + u * 8 * kThreads, hi - 1);
          raw[u] = row.raw(at);
          if (MASKED) keep[u] = row.bits(at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          if (u > 0 && c + u * 8 * kThreads >= hi) break;
          float v[NV];
          ln_unpack<T>(raw[u], v);
          if (MASKED) row.mask(keep[u], v);
          const int first = row.first(c + u * 8 * kThreads);
#pragma unroll
          for (int i = 0; i < NV; ++i)
            if (!(v[i] < least) && z_of(v[i], scale) != -INFINITY) f(key_of(order_of(v[i]), first + i));
        }
      }
      if (gr == 0 && lane < 2 && ragged(lane) >= 0) {
        float v[NV];
        row.load(ragged(lane), v);
        for (int i = 0; i < NV; ++i)
          if (z_of(v[i], scale) != -INFINITY) f(key_of(order_of(v[i]), row.first(ragged(lane)) + i));
      }
    };
    uint32_t mine = 0;                                     // of this warp's groups, those to search
#pragma unroll
    for (int q = 0; q < kGroups / kWarps; ++q) mine |= (uint32_t)(sh.upper[q * kWarps + warp] >= threshold) << q;
    if (!odd)
      for (; mine != 0; mine &= mine - 1) {
        each_key((__ffs(mine) - 1) * kWarps + warp, [&](unsigned long long key) {
          if (key < threshold) return;
          const int at = atomicAdd(&sh.count, 1);
          if (at < kCands) sh.cand[at] = key;
        });
      }
    __syncthreads();
    const int count = sh.count;
    if (!odd && count <= kCands) {
      for (int i = tid; i < count; i += kThreads) {
        const unsigned long long mine = sh.cand[i];
        int above = 0;
        for (int j = 0; j < count; ++j) above += sh.cand[j] > mine;
        if (above < a.k) sh.best[above] = mine;
      }
    } else {
      // more candidates than fit (many large logits in a few groups): the
      // largest key below the last one, k times
      unsigned long long last = ~0ull;
      for (int r = 0; r < a.k; ++r) {
        unsigned long long mine = 0ull;
        for (int gr = warp; gr < kGroups; gr += kWarps) {
          if (!odd && sh.upper[gr] < threshold) continue;
          each_key(gr, [&](unsigned long long key) {
            if (key < last && key > mine) mine = key;
          });
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
          const unsigned long long t = __shfl_xor_sync(0xffffffffu, mine, o);
          mine = t > mine ? t : mine;
        }
        if (lane == 0) sh.red[warp] = mine;
        __syncthreads();
        mine = 0ull;
        for (int w = 0; w < kWarps; ++w) mine = sh.red[w] > mine ? sh.red[w] : mine;
        if (tid == 0) sh.best[r] = mine;
        last = mine;
        __syncthreads();
      }
    }
  }
  __syncthreads();

  // the CTAs' sums and keys meet in the first one, in the CTAs' order
  Sums total = sh.total;
  const unsigned long long* best = sh.best;
  if (ctas > 1) {
    tc::cluster_sync();
    if (rank == 0) {
      for (int i = tid; i < ctas * a.k; i += kThreads) {
        const uint32_t at = tc::map_dsmem(tc::smem_u32(&sh.best[i % a.k]), i / a.k);
        unsigned long long v;
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
        sh.all[i] = v;
      }
      for (int r = 1; r < ctas; ++r) {
        const uint32_t at = tc::map_dsmem(tc::smem_u32(&sh.total), r);
        Sums b;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(b.m) : "r"(at) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(b.S) : "r"(at + 4) : "memory");
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(b.W) : "r"(at + 8) : "memory");
        join(total, b);
      }
    }
    tc::cluster_sync();
    if (rank != 0) return;
    for (int i = tid; i < a.k; i += kThreads) sh.cand[i] = 0ull;
    __syncthreads();
    for (int i = tid; i < ctas * a.k; i += kThreads) {
      const unsigned long long mine = sh.all[i];
      int above = 0;
      for (int j = 0; j < ctas * a.k; ++j) above += sh.all[j] > mine;
      if (mine != 0ull && above < a.k) sh.cand[above] = mine;
    }
    __syncthreads();
    best = sh.cand;
  }
  const float log_S = logf(total.S);
  const bool empty = total.m == -INFINITY;
  // logp = (z - max) - log S: the difference is exact for the large ones, and stays so
  // where |max| is so large that max + log S would lose log S
  const float m = empty ? 0.0f : total.m, log_sum = empty ? 0.0f : log_S;
  if (tid == 0) {
    a.lse[n] = total.m + log_S;
    a.stats[2 * n] = total.m;
    a.stats[2 * n + 1] = log_S;
    a.entropy[n] = empty ? 0.0f : log_S - total.W / total.S;
  }
  for (int j = tid; j < a.T; j += kThreads) {
    const int tok = a.tokens[n * a.T + j];
    float lp = 0.0f;
    if (tok >= 0) lp = tok < a.V ? (z_of(row.at(tok), scale) - m) - log_sum : __int_as_float(0x7FC00000);
    a.logprobs[n * a.T + j] = lp;
  }
  for (int j = tid; j < a.k; j += kThreads) {
    const unsigned long long key = best[j];
    a.top_idx[n * a.k + j] = key != 0ull ? token_of(key) : -1;
    a.top_logprobs[n * a.k + j] = key != 0ull ? (z_of(value_of(order_in(key)), scale) - m) - log_sum : -INFINITY;
  }
}

// The gradient of one row's range of chunks.  Every token's term is p (A - g_H
// logp) with A of the row; the few tokens with a gradient of their own are
// written again after it, by the CTA whose range they lie in.  Bound by memory: 4096
// rows of 32000 bf16 82 us, 6.4 TB/s (94 % of the measured copy); 2048 masked 51.3 (78 %);
// 40 masked fp32 rows 7.1 us.
template <class T, bool MASKED, bool SCALED>
__global__ void __launch_bounds__(kThreads) token_logprobs_grad_kernel(const ScoreGradArgs a) {
  constexpr int NV = Row<T>::NV;
  extern __shared__ __align__(16) uint8_t smem[];
  const int tid = threadIdx.x;
  const int E = a.T + a.k;                     // entries: tokens, then alternatives
  int* tok = reinterpret_cast<int*>(smem);
  float* grad = reinterpret_cast<float*>(tok + E);
  float* logit = grad + E;
  const long long n = blockIdx.y;
  pdl_wait();
  pdl_trigger();
  const Row<T> row(a.logits, a.ld, n, a.V, a.allowed, a.allowed_ld);
  T* out = static_cast<T*>(a.dlogits) + n * a.V;
  const bool out_vec = ((reinterpret_cast<uintptr_t>(out) & 15u) / sizeof(T)) == (unsigned)row.shift;
  const float scale = SCALED ? a.row_scale[n] : 1.0f;
  const bool empty = a.stats[2 * n] == -INFINITY;
  const float m = empty ? 0.0f : a.stats[2 * n], log_sum = empty ? 0.0f : a.stats[2 * n + 1];
  for (int j = tid; j < E; j += kThreads) {
    int k = j < a.T ? a.tokens[n * a.T + j] : a.top_idx[n * a.k + j - a.T];
    float g = j < a.T ? a.grad_logprobs[n * a.T + j] : a.grad_top[n * a.k + j - a.T];
    float x = 0.0f;
    if (k >= a.V) {                            // no such token: the row's gradient shows it
      g = __int_as_float(0x7FC00000);
      k = -1;
    } else if (k < 0) {
      g = 0.0f;
    } else {
      x = row.at(k);
      if (z_of(x, scale) == -INFINITY) {                // no probability, no gradient
        k = -1;
        g = 0.0f;
      }
    }
    tok[j] = k;
    grad[j] = g;
    logit[j] = x;
  }
  __syncthreads();
  float G = 0.0f;
  for (int j = 0; j < E; ++j) G += grad[j];
  // a row without tokens has lse -inf: an infinity may come back, and counts for nothing
  const float gH = a.grad_entropy != nullptr && !empty ? a.grad_entropy[n] : 0.0f;
  const float gl = a.grad_lse != nullptr && !empty ? a.grad_lse[n] : 0.0f;
  const float A = gl - G - gH * a.entropy[n];

  const int per = (row.chunks + gridDim.x - 1) / gridDim.x;
  const int c_lo = min((int)blockIdx.x * per, row.chunks), c_hi = min(c_lo + per, row.chunks);
  auto gradient = [&](float (&v)[NV]) {
    const uint64_t scale2 = pack2(scale, scale), m2 = pack2(-m, -m), s2 = pack2(-log_sum, -log_sum),
                   gH2 = pack2(-gH, -gH), A2 = pack2(A, A);
#pragma unroll
    for (int i = 0; i < NV; i += 2) {
      const uint64_t d = add2(add2(z_of2<SCALED>(v[i], v[i + 1], scale), m2), s2);
      // -inf: p is 0, and so is p logp
      const uint64_t lp = pack2(max_nan(lo2(d), -1e4f), max_nan(hi2(d), -1e4f));
      uint64_t g = mul2(exp_for<T>(lp), fma2(gH2, lp, A2));
      if (SCALED) g = mul2(g, scale2);
      v[i] = lo2(g);
      v[i + 1] = hi2(g);
    }
  };
  auto store = [&](int c, const float (&v)[NV]) {          // one value at a time
    const int i0 = row.first(c);
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i0 + i >= 0 && i0 + i < a.V) out[i0 + i] = from_f32<T>(v[i]);
  };
  auto store_whole = [&](int c, const float (&v)[NV]) {
    if (out_vec) {
      __align__(16) T e[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) e[i] = from_f32<T>(v[i]);
      *reinterpret_cast<uint4*>(out + row.first(c)) = *reinterpret_cast<const uint4*>(e);
    } else {
      store(c, v);
    }
  };
  {
    constexpr int U = 4;                                   // chunks on their way together
    const int lo = max(c_lo, row.whole_lo()), hi = min(c_hi, row.whole_hi());
    int c = lo + tid;
    for (; c + (U - 1) * kThreads < hi; c += U * kThreads) {
      uint4 raw[U];
      uint32_t keep[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        raw[u] = row.raw(c + u * kThreads);
        if (MASKED) keep[u] = row.bits(c + u * kThreads);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float v[NV];
        ln_unpack<T>(raw[u], v);
        if (MASKED) row.mask(keep[u], v);
        gradient(v);
        store_whole(c + u * kThreads, v);
      }
    }
    if (c < hi) {                                          // the last round, cut short
      uint4 raw[U - 1];
      uint32_t keep[U - 1];
#pragma unroll
      for (int u = 0; u < U - 1; ++u)
        if (c + u * kThreads < hi) {
          raw[u] = row.raw(c + u * kThreads);
          if (MASKED) keep[u] = row.bits(c + u * kThreads);
        }
#pragma unroll
      for (int u = 0; u < U - 1; ++u) {
        if (c + u * kThreads >= hi) break;
        float v[NV];
        ln_unpack<T>(raw[u], v);
        if (MASKED) row.mask(keep[u], v);
        gradient(v);
        store_whole(c + u * kThreads, v);
      }
    }
    const int e = tid == 0 ? 0 : row.chunks - 1;           // the ragged ends
    if (tid < 2 && e >= c_lo && e < c_hi && !row.whole(e) && (tid == 0 || e != 0)) {
      float v[NV];
      row.load(e, v);
      gradient(v);
      store(e, v);
    }
  }
  __syncthreads();
  // where any of these is not finite, p = 0 times it was no 0 for the tokens that are not
  // allowed (a select for each in the loops above: 58.5 us for 51.7, 2048 masked bf16 rows)
  if (MASKED && !(fabsf(A) < INFINITY && fabsf(gH) < INFINITY && fabsf(m) < INFINITY && fabsf(log_sum) < INFINITY))
    for (int c = c_lo + tid; c < c_hi; c += kThreads) {
      const int i0 = row.first(c);
      const uint32_t keep = row.bits(c);
      for (int i = 0; i < NV; ++i)
        if (i0 + i >= 0 && i0 + i < a.V && !(keep >> i & 1u)) out[i0 + i] = from_f32<T>(0.0f);
    }
  for (int j = tid; j < E; j += kThreads) {
    const int k = tok[j];
    if (k < max(row.first(c_lo), 0) || k >= min(row.first(c_hi), a.V)) continue;
    // a token given more than once: its first entry takes the sum, in order
    bool again = false;
    float g = 0.0f;
    for (int i = 0; i < E; ++i)
      if (tok[i] == k) {
        again |= i < j;
        g += grad[i];
      }
    if (again) continue;
    const float lp = max_nan((z_of(logit[j], scale) - m) - log_sum, -1e4f);
    out[k] = from_f32<T>(fmaf(lo2(exp_for<T>(pack2(lp, lp))), fmaf(-gH, lp, A), g) * scale);
  }
}

template <class... KArgs, class... Args>
cudaError_t launch_cluster(void (*kern)(KArgs...), dim3 grid, int cluster, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, static_cast<KArgs>(args)...);
}

// CTAs of a row's log probabilities.  Each CTA has a search for the largest logits of
// its own, so the row is cut in two while that leaves a thread six chunks or more,
// and as many more as there are CTAs for an SM already.  us, one CTA and this: 1 x 151000
// bf16 21.6 and 9.4, 40 x 32000 fp32 11.6 and 8.8, 64 masked 16.2 and 10.5 (eight CTAs a
// row 12.5), 250 x 32000 bf16 11.6, not cut (four CTAs a row 19.1).
int score_split(long long N, int V, int size) {
  const long long chunks = (long long)V * size / (16 * kThreads);          // a thread's of a whole row
  int c = 1;
  while (c < kMaxCluster && chunks * 152 >= 12 * c * std::max(152ll, N * c)) c *= 2;
  return c;
}

// CTAs of a row's gradient: enough that the rows fill the device four times over, as
// long as each has at least two chunks a thread (us, one CTA a row and this: 1 x 151000
// bf16 12.9 and 3.8, 40 x 32000 fp32 11.2 and 6.7, 200 x 151000 bf16 30.1 and 24.3).
int grad_split(long long N, int V, int size) {
  int c = 1;
  while (c < kMaxCluster && N * c < 4 * 152 && (long long)V * size / (16 * kThreads) >= 4 * c) c *= 2;
  return c;
}

// The kernels of a call: a mask and temperatures each have code of their own (a
// multiplication by 1 of every logit: 72.6 us for 69.4 in training).
template <class T>
auto scores_of(const ScoreArgs& a) {
  if (a.allowed != nullptr)
    return a.row_scale != nullptr ? token_logprobs_kernel<T, true, true> : token_logprobs_kernel<T, true, false>;
  return a.row_scale != nullptr ? token_logprobs_kernel<T, false, true> : token_logprobs_kernel<T, false, false>;
}
template <class T>
auto grad_of(const ScoreGradArgs& a) {
  if (a.allowed != nullptr)
    return a.row_scale != nullptr ? token_logprobs_grad_kernel<T, true, true> : token_logprobs_grad_kernel<T, true, false>;
  return a.row_scale != nullptr ? token_logprobs_grad_kernel<T, false, true> : token_logprobs_grad_kernel<T, false, false>;
}

constexpr long long kRowsPerLaunch = 65535;        // the grid's y

}  // namespace

cudaError_t launch_token_logprobs(int dtype, const ScoreArgs& all, cudaStream_t s) {
  const int size = dtype == FOVEA_BF16 ? 2 : 4;
  for (long long n0 = 0; n0 < all.N; n0 += kRowsPerLaunch) {
    ScoreArgs a = all;
    a.N = std::min(kRowsPerLaunch, all.N - n0);
    a.logits = static_cast<const uint8_t*>(all.logits) + n0 * all.ld * size;
    if (a.row_scale != nullptr) a.row_scale += n0;
    if (a.allowed != nullptr) a.allowed += n0 * all.allowed_ld;
    if (a.T > 0) { a.tokens += n0 * all.T; a.logprobs += n0 * all.T; }
    if (a.k > 0) { a.top_idx += n0 * all.k; a.top_logprobs += n0 * all.k; }
    a.lse += n0;
    a.stats += 2 * n0;
    a.entropy += n0;
    const int split = score_split(a.N, a.V, size);
    const dim3 grid(split, (unsigned)a.N);
    const cudaError_t e = launch_cluster(dtype == FOVEA_BF16 ? scores_of<__nv_bfloat16>(a) : scores_of<float>(a),
                                         grid, split, s, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_token_logprobs_grad(int dtype, const ScoreGradArgs& all, cudaStream_t s) {
  const int size = dtype == FOVEA_BF16 ? 2 : 4;
  for (long long n0 = 0; n0 < all.N; n0 += kRowsPerLaunch) {
    ScoreGradArgs a = all;
    a.N = std::min(kRowsPerLaunch, all.N - n0);
    a.logits = static_cast<const uint8_t*>(all.logits) + n0 * all.ld * size;
    a.dlogits = static_cast<uint8_t*>(all.dlogits) + n0 * all.V * size;
    if (a.row_scale != nullptr) a.row_scale += n0;
    if (a.allowed != nullptr) a.allowed += n0 * all.allowed_ld;
    if (a.T > 0) { a.tokens += n0 * all.T; a.grad_logprobs += n0 * all.T; }
    if (a.k > 0) { a.top_idx += n0 * all.k; a.grad_top += n0 * all.k; }
    if (a.grad_entropy != nullptr) a.grad_entropy += n0;
    if (a.grad_lse != nullptr) a.grad_lse += n0;
    a.stats += 2 * n0;
    a.entropy += n0;
    // in place, a CTA may not overwrite logits that another CTA of the row still
    // has to read for its tokens' entries
    const int split = a.dlogits == a.logits ? 1 : grad_split(a.N, a.V, size);
    const dim3 grid(split, (unsigned)a.N);
    const size_t smem = (size_t)(a.T + a.k) * 12;
    const cudaError_t e = launch_pdl(dtype == FOVEA_BF16 ? grad_of<__nv_bfloat16>(a) : grad_of<float>(a), grid,
                                     dim3(kThreads), smem, s, a);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
