// Rotary positions with several axes (fovea_rotary_axes) and new entries of a paged cache
// (fovea_cache_append), which rotates on the way.
//
// Pair j of a token's head is turned by phi_j = positions[axis_j] f_j:
//   a' = a cos phi - b sin phi,  b' = a sin phi + b cos phi   (inverse: -phi, the gradient).
// Angles of far positions lose their bits in fp32 (position 10^6 by 1 radian: 0.06), and in
// fp64 they cost the few fp64 units.  A turn is therefore held in fixed point: f / 2 pi is
// rounded once to 64 fractional bits, and its product with an integer position modulo
// 2^64 is exact in integers; the upper 32 bits are the angle to 1.5e-9.
//
// Bound by memory: each element is read and written once.  A thread keeps the sines of
// eight pairs of a token and applies them to up to eight heads, so that their cost is
// shared; its two 16-byte chunks of a head are the pairs' two halves.
#include <cuda_fp8.h>

#include <atomic>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kMaxThreads = 512;

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

// E elements of a row of T.
template <class T, int E>
struct Chunk {
  uint4 raw[E == 1 ? 1 : E * sizeof(T) / 16];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (E == 1) {
      *reinterpret_cast<T*>(raw) = *p;
    } else {
#pragma unroll
      for (int i = 0; i < (int)(E * sizeof(T) / 16); ++i) raw[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
    }
  }
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(raw)[i]); }
};

// E values in the cache's type; `scale` is of 8-bit entries.
template <class C, int E>
__device__ __forceinline__ void store(C* p, const float (&x)[E], float scale) {
  if constexpr (sizeof(C) == 1) {
    uint32_t w[(E + 3) / 4] = {};
#pragma unroll
    for (int i = 0; i < E; i += 2) {
      const float2 two = make_float2(__fdiv_rn(x[i], scale), i + 1 < E ? __fdiv_rn(x[i + 1 < E ? i + 1 : i], scale) : 0.0f);
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
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

template <class T, class C, int E, bool PAGED>
__global__ void __launch_bounds__(kMaxThreads) rotary_kernel(const __grid_constant__ Work w) {
  __shared__ unsigned long long phase[kRotaryPairs];     // turns per position, times 2^64
  __shared__ int axis_of[kRotaryPairs];                  // -1: no number
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  for (int j = tid; j < w.r.rot / 2; j += blockDim.x) {
    double f = w.r.frequencies[j] * 0.15915494309189533577;       // 1 / (2 pi)
    const int axis = w.r.axis != nullptr ? w.r.axis[j] : 0;
    axis_of[j] = (unsigned)axis < (unsigned)w.r.axes && isfinite(f) ? axis : -1;
    f -= rint(f);                                                 // within half a turn
    phase[j] = (unsigned long long)__double2ll_rn(f * 18446744073709551616.0);
  }
  __syncthreads();
  const int per_token = w.blocks * w.slots;
  const int local = tid / per_token, rest = tid - local * per_token;
  const int block = rest / w.slots, slot = rest - block * w.slots;
  if (local >= w.tokens) return;
  const bool turns = slot < w.turned;
  int at[2];                                             // the chunks' first elements
  if (turns) {
    at[0] = w.r.adjacent ? 2 * E * slot : E * slot;
    at[1] = w.r.adjacent ? at[0] + E : w.r.rot / 2 + E * slot;
  } else {
    at[0] = w.r.rot + 2 * E * (slot - w.turned);
    at[1] = at[0] + E;
  }
  const bool second = at[1] < w.dim;                     // not the last element of an odd rest
  const int heads = w.q.heads + w.k.heads + w.v.heads;
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;         // heads on their way together

  for (long long n = (long long)blockIdx.x * w.tokens + local; n < w.N; n += (long long)gridDim.x * w.tokens) {
    float c[E], s[E];
    if (turns) {
      int axis = -2, p = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int j = E * slot + i, next = axis_of[j];
        if (next != axis) {
          axis = next;
          p = axis < 0 ? 0 : w.r.positions[axis * w.r.pos_ld + n];
        }
        const unsigned long long turn = (unsigned long long)(long long)p * phase[j];
        const int hi = (int)(turn >> 32);                // in 2^-32 turns, signed
        sincospif((float)hi * 4.656612873077393e-10f, &s[i], &c[i]);   // 2^-31
        if (w.r.inverse) s[i] = -s[i];
        if (axis < 0) c[i] = s[i] = NAN;
      }
    }
    long long place = -1;                                // of the entry: (page kv_heads) page + offset in it
    if constexpr (PAGED) {
      const int b = w.sequence[n], e = w.entry[n];
      if ((unsigned)b < (unsigned)w.c.B && e >= 0 && e < (long long)w.c.width * w.c.page) {
        const int id = w.c.table[(long long)b * w.c.width + e / w.c.page];
        if ((unsigned)id < (unsigned)w.c.n_pages) place = (long long)id * w.c.kv_heads * w.c.page + e % w.c.page;
      }
    }
    for (int h0 = block; h0 < heads; h0 += kAhead * w.blocks) {
      Chunk<T, E> x[kAhead][2];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + i * w.blocks;
        if (h < heads) {
          const bool is_q = h < w.q.heads, is_k = h < w.q.heads + w.k.heads;
          const HeadRows& r = is_q ? w.q : is_k ? w.k : w.v;
          const int head = is_q ? h : is_k ? h - w.q.heads : h - w.q.heads - w.k.heads;
          const T* p = static_cast<const T*>(r.x) + n * r.ld + head * r.hs;
          x[i][0].load(p + at[0]);
          if (second) x[i][1].load(p + at[1]);
        }
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int h = h0 + i * w.blocks;
        if (h >= heads) break;
        const bool is_q = h < w.q.heads, is_k = h < w.q.heads + w.k.heads;
        float y[2][E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          y[0][e] = x[i][0].get(e);
          y[1][e] = second ? x[i][1].get(e) : 0.0f;
        }
        if (turns && is_k) {
          if (w.r.adjacent && E > 1) {
#pragma unroll
            for (int e = 0; e < E; ++e) {                // pair e: elements 2e, 2e + 1 of both chunks
              float& a = y[2 * e / E][2 * e % E];
              float& b = y[2 * e / E][(2 * e + 1) % E];
              const float a0 = a, b0 = b;
              a = a0 * c[e] - b0 * s[e];
              b = a0 * s[e] + b0 * c[e];
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float a0 = y[0][e], b0 = y[1][e];
              y[0][e] = a0 * c[e] - b0 * s[e];
              y[1][e] = a0 * s[e] + b0 * c[e];
            }
          }
        }
        if (is_q) {
          T* p = static_cast<T*>(w.q_out) + (n * w.q.heads + h) * w.dim;
          store<T, E>(p + at[0], y[0], 1.0f);
          if (second) store<T, E>(p + at[1], y[1], 1.0f);
        } else if constexpr (PAGED) {
          if (place >= 0) {
            const int head = is_k ? h - w.q.heads : h - w.q.heads - w.k.heads;
            C* p = static_cast<C*>(is_k ? w.c.k : w.c.v) + (place + (long long)head * w.c.page) * w.dim;
            const float* scales = is_k ? w.c.k_scale : w.c.v_scale;
            const float scale = sizeof(C) == 1 && scales != nullptr ? scales[head] : 1.0f;
            store<C, E>(p + at[0], y[0], scale);
            if (second) store<C, E>(p + at[1], y[1], scale);
          }
        } else {
          T* p = static_cast<T*>(w.k_out) + (n * w.k.heads + h - w.q.heads) * w.dim;
          store<T, E>(p + at[0], y[0], 1.0f);
          if (second) store<T, E>(p + at[1], y[1], 1.0f);
        }
      }
    }
  }
}

template <class T, class C, int E, bool PAGED>
cudaError_t launch_as(Work w, cudaStream_t s) {
  const int rot = w.r.rot, heads = w.q.heads + w.k.heads + w.v.heads;
  w.turned = rot / 2 / E;
  w.slots = w.turned + (w.dim - rot + 2 * E - 1) / (2 * E);
  // heads a thread: up to eight share its sines, fewer where that leaves SMs without work
  int per = 8;
  while (per > 1 && (long long)w.N * ((heads + per - 1) / per) * w.slots < 152 * 1024) per /= 2;
  while ((heads + per - 1) / per * w.slots > kMaxThreads) per *= 2;
  w.blocks = (heads + per - 1) / per;
  const int per_token = w.blocks * w.slots;
  w.tokens = per_token >= 256 ? 1 : 256 / per_token;
  const int threads = (w.tokens * per_token + 31) / 32 * 32;
  const long long ctas = ((long long)w.N + w.tokens - 1) / w.tokens;
  const int grid = (int)(ctas < 152 * 8 ? ctas : 152 * 8);
  return launch_pdl(rotary_kernel<T, C, E, PAGED>, dim3(grid), dim3(threads), 0, s, w);
}

bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool vectors(const HeadRows& r, size_t size) {
  return r.heads == 0 || (aligned(r.x, 16) && r.ld * size % 16 == 0 && r.hs * size % 16 == 0);
}

template <class T, class C, bool PAGED>
cudaError_t launch_type(const Work& w, cudaStream_t s) {
  const bool whole = w.dim % 16 == 0 && w.r.rot % 16 == 0 && vectors(w.q, sizeof(T)) && vectors(w.k, sizeof(T)) &&
                     vectors(w.v, sizeof(T)) && aligned(w.q_out, 16) && aligned(w.k_out, 16);
  return whole ? launch_as<T, C, 8, PAGED>(w, s) : launch_as<T, C, 1, PAGED>(w, s);
}

}  // namespace

cudaError_t launch_rotary(int dtype, const HeadRows& q, const HeadRows& k, int N, int dim, const RotaryArgs& r,
                          void* q_out, void* k_out, cudaStream_t s) {
  Work w{};
  w.q = q; w.k = k; w.N = N; w.dim = dim; w.r = r;
  w.q_out = q_out; w.k_out = k_out;
  return dtype == FOVEA_BF16 ? launch_type<__nv_bfloat16, __nv_bfloat16, false>(w, s)
                             : launch_type<float, float, false>(w, s);
}

cudaError_t launch_cache_append(int dtype, const HeadRows& q, const HeadRows& k, const HeadRows& v, int N,
                                const RotaryArgs& r, const CachePages& c, const int32_t* sequence,
                                const int32_t* entry, void* q_out, cudaStream_t s) {
  Work w{};
  w.q = q; w.k = k; w.v = v; w.N = N; w.dim = c.dim; w.r = r;
  w.q_out = q_out;
  w.c = c; w.sequence = sequence; w.entry = entry;
  return dtype == FOVEA_FP32         ? launch_type<float, float, true>(w, s)
         : c.dtype == FOVEA_E4M3 ? launch_type<__nv_bfloat16, __nv_fp8_e4m3, true>(w, s)
                                 : launch_type<__nv_bfloat16, __nv_bfloat16, true>(w, s);
}

}  // namespace fovea
