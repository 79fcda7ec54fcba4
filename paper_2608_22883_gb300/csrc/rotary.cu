// Rotary positions with several axes (fovea_rotary_axes) and new entries of a paged cache
// (fovea_cache_append), which rotates on the way.
//
// Pair j of a token's head is turned by phi_j = positions[axis_j] f_j:
//   a' = a cos phi - b sin phi,  b' = a sin phi + b cos phi   (inverse: -phi, the gradient).
// Angles of far positions lose their bits in fp32 (position 10^6 by 1 radian: 0.06), and in
// fp64 they cost the few fp64 units.  A turn is therefore held in fixed point: f / 2 pi, as
// the sum of two fp64 values, is taken to 64 fractional bits, and its product with an integer
// position modulo 2^64 is exact in integers: the angle is right to 7e-10 (of frequencies up to
// 2^40, whose lower value is below a turn) before it is rounded to 24 bits of what it has over
// the nearest quarter turn.
//
// Bound by memory: each element is read and written once.  A thread keeps the sines of
// eight pairs of a token and applies them to up to sixteen heads, so that their cost is
// shared; its two chunks of eight elements of a head are the pairs' two halves.  Measured:
// image prompts (23040 bf16 tokens, 28 + 4 heads of 128, three axes) 62 us, 6.1 TB/s; the
// gradient of 9216 fp32 tokens of 80 heads 121 us, 6.2 TB/s; prompts into an 8-bit cache
// (32768 rows, 20480 of them stored, 32 + 8 heads) 119 us, 5.6 TB/s.  Rows off 16 bytes, and
// heads or rotated dims that are no multiples of 16, go one element a thread: heads of 72 take
// 176 us (floor 31), 24 rotated dims of 128 198 (56).
#include <cuda_fp8.h>

#include <atomic>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kMaxThreads = 256;

// CTAs an SM and heads on their way together in a thread: of 16-bit rows many threads with
// one, of 32-bit rows (whose angles and values take twice the registers) fewer with two.
// 23040 bf16 tokens of 32 heads with 1 head and 4 / 3 / 5 CTAs: 62 / 72 / 68 us, 2 heads
// and 3 CTAs 67, 4 and 2 68; 9216 fp32 tokens of 80 heads with 2 heads and 2 CTAs 120, 1
// and 4 128.
template <class T> constexpr int kResident = sizeof(T) == 2 ? 4 : 2;
template <class T> constexpr int kAhead = sizeof(T) == 2 ? 1 : 2;
constexpr int kChunk = 8;            // elements of a thread's chunk

// Turns per position of a frequency in radians, modulo 1, times 2^64.  1 / (2 pi) is the sum of
// its fp64 value and what that leaves out; the product's rounding is got back exactly.
__device__ __forceinline__ unsigned long long turns_of(double f) {
  constexpr double kUpper = 0.15915494309189535, kLower = -9.839338337591243e-18;
  const double upper = f * kUpper;
  double lower = fma(f, kLower, fma(f, kUpper, -upper));
  lower -= rint(lower);
  const double frac = upper - rint(upper);                        // within half a turn, exactly
  return (unsigned long long)__double2ll_rn(frac * 18446744073709551616.0) +
         (unsigned long long)__double2ll_rn(lower * 18446744073709551616.0);
}

struct Work {
  HeadRows q, k, v;                  // v: entries alone
  int N, dim;
  RotaryArgs r;
  void* q_out; void* k_out;
  CachePages c;                      // paged: where k and v go
  const int32_t* sequence; const int32_t* entry;
  int slots, turned;                 // slots of a head (two chunks each), of them rotated
  int blocks;                        // threads that share a token's heads: head h is taken by thread h % blocks
  int tokens;                        // of a CTA at a time
};

// E elements of a row of T.  Plain loads: the outputs may be the inputs' own memory, which the
// read-only path is not for.
template <class T, int E>
struct Chunk {
  uint4 raw[E == 1 ? 1 : E * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (E == 1) {
      *reinterpret_cast<T*>(raw) = *p;
    } else {
#pragma unroll
      for (int i = 0; i < (int)(E * sizeof(T) / 16); ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
    }
  }
  template <class C> __device__ __forceinline__ void copy(C* p) const {
    if constexpr (E == 1) {
      *p = *reinterpret_cast<const C*>(raw);
    } else {
#pragma unroll
      for (int i = 0; i < (int)(E * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(p)[i] = raw[i];
    }
  }
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(raw)[i]); }
};

// x / scale for 8-bit entries, rounded once: a product with the reciprocal rounds twice, and
// is wrong where that is no number.  The product's remainder, exact in one fused operation,
// corrects it (Markstein, IBM J. Res. Dev. 34, 1990).  x and a scale near an end of fp32's
// range go by 2^80 together; quotients beyond 2^20, which the type saturates, are cut first,
// so that infinities stay.  Prompts into 8 bits: 119 us; divided 124, by products alone 116;
// two elements an operation 126, for want of registers.
struct Divisor {
  float power, scale, inverse;
  __device__ __forceinline__ explicit Divisor(float s) {
    power = fabsf(s) < 0x1p-40f ? 0x1p80f : fabsf(s) > 0x1p40f ? 0x1p-80f : 1.0f;
    scale = isinf(s) ? copysignf(0x1p120f, s) : s * power;
    inverse = 1.0f / scale;
  }
  __device__ __forceinline__ float quotient(float x) const {
    x *= power;
    const float q = fminf(fmaxf(x * inverse, -0x1p20f), 0x1p20f);
    return fmaf(fmaf(q, scale, -x), -inverse, q);        // so that zeros keep their sign
  }
};

// E values in the cache's type; those of 8-bit entries over their scale.
template <class C, int E>
__device__ __forceinline__ void store(C* p, const float (&x)[E], const Divisor& by) {
  if constexpr (sizeof(C) == 1) {
    uint32_t w[(E + 3) / 4] = {};
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float2 two = make_float2(by.quotient(x[i]), i + 1 < E ? by.quotient(x[i + 1 < E ? i + 1 : i]) : 0.0f);
      w[i / 4] |= (uint32_t)__nv_cvt_float2_to_fp8x2(two, __NV_SATFINITE, __NV_E4M3) << (8 * (i & 3));
    }
    if constexpr (E == 1) *reinterpret_cast<uint8_t*>(p) = (uint8_t)w[0];
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else if constexpr (E == 1) {
    *p = from_f32<C>(x[0]);
  } else if constexpr (sizeof(C) == 2) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
#pragma unroll
    for (int i = 0; i < E; i += 4) reinterpret_cast<float4*>(p)[i / 4] = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
  }
}

// cos and sin of an angle in 2^-64 turns.  It is taken to the nearest quarter turn, the
// rest (at most pi / 4) goes through the Taylor series: up to x^9 and x^8, whose next terms
// are below 2e-9 and 2.5e-8.  The lower 32 bits count in small angles, whose sine would
// otherwise keep few bits (1e-6 radians are 683 steps of the upper ones).
__device__ __forceinline__ void cos_sin(unsigned long long angle, float& c, float& s) {
  const uint32_t turn = (uint32_t)(angle >> 32), quarter = (turn + 0x20000000u) >> 30;
  const float rest = fmaf((float)(uint32_t)angle, 0x1p-32f, (float)(int)(turn - (quarter << 30)));
  const float x = rest * 1.4629180792671596e-9f;         // 2 pi / 2^32
  const float y = x * x;
  const float sine = fmaf(x * y, fmaf(y, fmaf(y, fmaf(y, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), x);
  const float cosine = fmaf(y, fmaf(y, fmaf(y, fmaf(y, 2.4801587e-5f, -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.0f);
  c = quarter & 1 ? sine : cosine;
  s = quarter & 1 ? cosine : sine;
  if ((quarter + 1) & 2) c = -c;
  if (quarter & 2) s = -s;
}

// Where a thread's chunks lie in a head, and its angles.
template <int E> struct Turn {
  int at, apart;                     // the first chunk's first element, the second's behind it
  bool turns, second;                // rotated dims; there is a second chunk
  float c[E], s[E];
};

// The heads block, block + blocks, ... of a token: from `in`, `step` elements from one to the
// next, to `out`.  TURN: they are rotated where the thread's dims are; ADJ: in adjacent pairs.
template <class T, class C, int E, bool ADJ, bool TURN, int kHeads>
__device__ __forceinline__ void run_heads(const Turn<E>& w, const T* in, long long step, C* out, long long out_step,
                                          int block, int blocks, int heads, const float* scales) {
  for (int h = block; h < heads; h += kHeads * blocks) {
    Chunk<T, E> x[kHeads][2];
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (h + i * blocks < heads) {
        x[i][0].load(in);
        if (w.second) x[i][1].load(in + w.apart);
      }
      in += step;
    }
#pragma unroll
    for (int i = 0; i < kHeads; ++i) {
      if (h + i * blocks >= heads) break;
      C* p = out;
      out += out_step;
      if (sizeof(T) == sizeof(C) && !(TURN && w.turns)) {            // as they are
        x[i][0].copy(p);
        if (w.second) x[i][1].copy(p + w.apart);
      } else {
        float y[2][E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          y[0][e] = x[i][0].get(e);
          y[1][e] = w.second ? x[i][1].get(e) : 0.0f;
        }
        if (TURN && w.turns) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            // pair e: elements 2e, 2e + 1 of both chunks together, or e of each
            float& a = ADJ ? y[2 * e / E][2 * e % E] : y[0][e];
            float& b = ADJ ? y[(2 * e + 1) / E][(2 * e + 1) % E] : y[1][e];
            const float a0 = a, b0 = b;
            a = a0 * w.c[e] - b0 * w.s[e];
            b = a0 * w.s[e] + b0 * w.c[e];
          }
        }
        const Divisor by(sizeof(C) == 1 && scales != nullptr ? scales[h + i * blocks] : 1.0f);
        store<C, E>(p, y[0], by);
        if (w.second) store<C, E>(p + w.apart, y[1], by);
      }
    }
  }
}

// MODE: rotated rows to dense outputs, to pages, or rows as they are to pages (with two heads
// on their way: 16 trees of 64 entries of 40 heads stored and kept, 13.1 us; one 14.6, four
// and two CTAs an SM 16.2).
enum Mode { kDense, kTurned, kPlain };

template <class T, class C, int E, bool ADJ, int MODE>
__global__ void __launch_bounds__(kMaxThreads, MODE == kPlain ? 4 : kResident<T>) rotary_kernel(const __grid_constant__ Work w) {
  constexpr bool PAGED = MODE != kDense, ROTARY = MODE != kPlain;
  constexpr int kHeads = MODE == kPlain && sizeof(T) == 2 ? 2 : kAhead<T>;
  __shared__ unsigned long long phase[ROTARY ? kRotaryPairs : 1];     // turns per position, times 2^64
  __shared__ int axis_of[ROTARY ? kRotaryPairs : 1];                  // -1: no number
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  if constexpr (ROTARY) {
    for (int j = tid; j < w.r.rot / 2; j += blockDim.x) {
      const double f = w.r.frequencies[j];
      const int axis = w.r.axis != nullptr ? w.r.axis[j] : 0;
      axis_of[j] = (unsigned)axis < (unsigned)w.r.axes && isfinite(f) ? axis : -1;
      phase[j] = turns_of(f);
    }
    __syncthreads();
  }
  const int per_token = w.blocks * w.slots;
  const int local = tid / per_token, rest = tid - local * per_token;
  const int block = rest / w.slots, slot = rest - block * w.slots;
  if (local >= w.tokens) return;
  Turn<E> t;
  t.turns = slot < w.turned;
  t.at = t.turns ? (ADJ ? 2 * E * slot : E * slot) : w.r.rot + 2 * E * (slot - w.turned);
  t.apart = t.turns && !ADJ ? w.r.rot / 2 : E;
  t.second = t.at + t.apart < w.dim;                     // not the last element of an odd rest
  for (long long n = (long long)blockIdx.x * w.tokens + local; n < w.N; n += (long long)gridDim.x * w.tokens) {
    long long place = -1;                                // of the entry: (page kv_heads) page + offset in it
    if constexpr (PAGED) {
      const int b = w.sequence[n], e = w.entry[n];
      if ((unsigned)b < (unsigned)w.c.B && e >= 0 && e < (long long)w.c.width * w.c.page) {
        const int id = w.c.table[(long long)b * w.c.width + e / w.c.page];
        if ((unsigned)id < (unsigned)w.c.n_pages) place = (long long)id * w.c.kv_heads * w.c.page + e % w.c.page;
      }
      if (place < 0 && w.q.heads == 0) continue;
    }
    if (ROTARY && t.turns) {
      int axis = -2, p = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int j = E * slot + i, next = axis_of[j];
        if (next != axis) {
          axis = next;
          p = axis < 0 ? 0 : w.r.positions[axis * w.r.pos_ld + n];
        }
        cos_sin((unsigned long long)(long long)p * phase[j], t.c[i], t.s[i]);
        if (w.r.inverse) t.s[i] = -t.s[i];
        if (axis < 0) t.c[i] = t.s[i] = NAN;
      }
    }
    const long long out_step = (long long)w.blocks * w.dim;
    if (ROTARY && w.q.heads > 0)
      run_heads<T, T, E, ADJ, true, kHeads>(t, static_cast<const T*>(w.q.x) + n * w.q.ld + block * w.q.hs + t.at, w.blocks * w.q.hs,
                               static_cast<T*>(w.q_out) + (n * w.q.heads + block) * w.dim + t.at, out_step, block,
                               w.blocks, w.q.heads, nullptr);
    const T* k = static_cast<const T*>(w.k.x) + n * w.k.ld + block * w.k.hs + t.at;
    if constexpr (PAGED) {
      if (place < 0) continue;
      const long long to = (place + (long long)block * w.c.page) * w.dim + t.at, page_step = out_step * w.c.page;
      run_heads<T, C, E, ADJ, MODE == kTurned, kHeads>(t, k, w.blocks * w.k.hs, static_cast<C*>(w.c.k) + to, page_step, block, w.blocks,
                               w.k.heads, w.c.k_scale);
      run_heads<T, C, E, ADJ, false, kHeads>(t, static_cast<const T*>(w.v.x) + n * w.v.ld + block * w.v.hs + t.at,
                                w.blocks * w.v.hs, static_cast<C*>(w.c.v) + to, page_step, block, w.blocks, w.v.heads,
                                w.c.v_scale);
    } else if (w.k.heads > 0) {
      run_heads<T, T, E, ADJ, true, kHeads>(t, k, w.blocks * w.k.hs, static_cast<T*>(w.k_out) + (n * w.k.heads + block) * w.dim + t.at,
                               out_step, block, w.blocks, w.k.heads, nullptr);
    }
  }
}

template <class T, class C, int E, bool ADJ, int MODE>
cudaError_t launch_as(Work w, cudaStream_t s) {
  const int rot = w.r.rot, heads = w.q.heads + w.k.heads + w.v.heads;
  w.turned = rot / 2 / E;
  w.slots = w.turned + (w.dim - rot + 2 * E - 1) / (2 * E);
  // Threads that share a token's heads, a power of two (so that q, k and v, often of 4, 8 or
  // 32 heads, go even): the fewest that leave a thread's sines to fewer than 16 heads, more
  // where that leaves SMs without work.
  w.blocks = 1;
  while (w.blocks * 16 <= heads || (w.blocks < heads && (long long)w.N * w.blocks * w.slots < 152 * 1024)) w.blocks *= 2;
  while (w.blocks > 1 && w.blocks * w.slots > kMaxThreads) w.blocks /= 2;
  const int per_token = w.blocks * w.slots;
  w.tokens = per_token >= 256 ? 1 : 256 / per_token;
  const int threads = (w.tokens * per_token + 31) / 32 * 32;
  const long long ctas = ((long long)w.N + w.tokens - 1) / w.tokens;
  // CTAs go on to further tokens: each makes the table of turns, which a CTA for every few
  // tokens would pay for (image prompts 66 us instead of 62)
  const int grid = (int)(ctas < 152 * 4 ? ctas : 152 * 4);
  return launch_pdl(rotary_kernel<T, C, E, ADJ, MODE>, dim3(grid), dim3(threads), 0, s, w);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool vectors(const HeadRows& r, size_t size) {
  return r.heads == 0 || (aligned(r.x, 16) && r.ld * size % 16 == 0 && r.hs * size % 16 == 0);
}

template <class T, class C, int MODE>
cudaError_t launch_type(const Work& w, cudaStream_t s) {
  constexpr int E = kChunk;
  const bool whole = w.dim % (2 * E) == 0 && w.r.rot % (2 * E) == 0 && vectors(w.q, sizeof(T)) && vectors(w.k, sizeof(T)) &&
                     vectors(w.v, sizeof(T)) && aligned(w.q_out, 16) && aligned(w.k_out, 16);
  if constexpr (MODE != kPlain) {
    if (w.r.adjacent)
      return whole ? launch_as<T, C, E, true, MODE>(w, s) : launch_as<T, C, 1, true, MODE>(w, s);
  }
  return whole ? launch_as<T, C, E, false, MODE>(w, s) : launch_as<T, C, 1, false, MODE>(w, s);
}

}  // namespace

cudaError_t launch_rotary(int dtype, const HeadRows& q, const HeadRows& k, int N, int dim, const RotaryArgs& r,
                          void* q_out, void* k_out, cudaStream_t s) {
  Work w{};
  w.q = q; w.k = k; w.N = N; w.dim = dim; w.r = r;
  w.q_out = q_out; w.k_out = k_out;
  return dtype == FOVEA_BF16 ? launch_type<__nv_bfloat16, __nv_bfloat16, kDense>(w, s)
                             : launch_type<float, float, kDense>(w, s);
}

cudaError_t launch_cache_append(int dtype, const HeadRows& q, const HeadRows& k, const HeadRows& v, int N,
                                const RotaryArgs& r, const CachePages& c, const int32_t* sequence,
                                const int32_t* entry, void* q_out, cudaStream_t s) {
  Work w{};
  w.q = q; w.k = k; w.v = v; w.N = N; w.dim = c.dim; w.r = r;
  w.q_out = q_out;
  w.c = c; w.sequence = sequence; w.entry = entry;
  if (r.rot == 0)
    return dtype == FOVEA_FP32     ? launch_type<float, float, kPlain>(w, s)
           : c.dtype == FOVEA_E4M3 ? launch_type<__nv_bfloat16, __nv_fp8_e4m3, kPlain>(w, s)
                                   : launch_type<__nv_bfloat16, __nv_bfloat16, kPlain>(w, s);
  return dtype == FOVEA_FP32     ? launch_type<float, float, kTurned>(w, s)
         : c.dtype == FOVEA_E4M3 ? launch_type<__nv_bfloat16, __nv_fp8_e4m3, kTurned>(w, s)
                                 : launch_type<__nv_bfloat16, __nv_bfloat16, kTurned>(w, s);
}

}  // namespace fovea
