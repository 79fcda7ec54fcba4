// fovea_paged_attention with many rows a key head (draft trees): paged.cu has the formulas.
//
// Heads of 256 dims, and 17 to 64 rows over 8-bit entries (paged_tree.cu takes the others).
// With 64 rows a block's keys and values serve enough products that the tensor cores' feed
// counts, not the cache's bytes: a CTA takes 64 rows, 16 a warp, and all of them the same
// tiles of keys and values, staged in shared memory two deep by asynchronous copies (16-byte
// chunks, swizzled by row, so that ldmatrix reads without conflicts).  A warp keeps its rows
// of Q and of O in registers; S = Q K^T of a tile stays there too and becomes the operand of
// P V in place.  A warp has all entries of its rows: nothing is joined within the CTA.
// Eight trees of 6 nodes over 3000 e4m3 entries, 24 rows a key head: 40 us (floor 6.4), bound
// by the latencies of a run's few tiles; 16 sequences of 4096 bf16 entries of 256 dims, 16
// heads over 4: 46 us (floor 34).
#include <atomic>
#include <cstddef>

#include "paged_core.cuh"

namespace fovea {

namespace {

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
template <class C, int D> struct Rows {
  static constexpr bool kE4 = sizeof(C) == 1, kWaits = false;
  static constexpr float kLift = kE4 ? 15.0f : 0.0f;             // as in paged.cu
  static constexpr int kRows = 16 * kWarps, kTile = D == 256 ? 32 : 64, kBlock = kTile, kLeast = 1;
  static constexpr uint32_t kFront = 2;                          // tiles: 1 / 2 / 4 / 8: 40 / 40 / 44 / 43 us (24 rows)
  static constexpr int kSlot = kRows * (D + 2);
  static constexpr int kRowBytes = D * sizeof(C), kChunks = kRowBytes / 16;
  static constexpr int kTileBytes = kTile * kRowBytes;
  static constexpr int kParts = kTile / 16;                      // blocks of 16 entries of a tile
  static constexpr int kSteps = D / 16;                          // of the contraction over dims
  static constexpr int kCopies = kTile * kChunks / kThreads;     // chunks of keys a thread copies

  struct Shared {
    alignas(128) uint8_t kv[2][2][kTileBytes];                   // stage; keys, values
    float front[D];                                              // of add_odd_values
    uint32_t lost[kRows / 32];
    int odd;
  };
  // A chunk's place in a tile: rows of 128 bytes and more put it at chunk ^ (row % 8), two
  // rows of 64 bytes share 128.
  __device__ __forceinline__ static uint32_t place(int row, int chunk) {
    const int swizzle = kChunks >= 8 ? row & 7 : (row >> 1) & 3;
    return (uint32_t)(row * kRowBytes + ((chunk ^ swizzle) << 4));
  }

  uint32_t q[kSteps][4];
  float o[D / 8][4];
  float m[2], l[2], f[2];

  // This warp's rows of Q as fragments (rows g and g + 8; a step's dims in the order in
  // which the keys' fragments have them: 2t, 2t + 1, 2t + 8, 2t + 9, of 8 bits 4t to 4t + 3).
  __device__ __forceinline__ void load_rows(const PagedArgs& a, int b, int h, int row0) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int rows = a.nodes * a.group;
    const float factor = a.scale * kLog2e * (kE4 && a.k_scale != nullptr ? a.k_scale[h] : 1.0f);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int row = row0 + g + 8 * e;
      const bool there = row < rows;
      const __nv_bfloat16* p = row_of<__nv_bfloat16>(a, b, h, there ? row : 0);
      float top = 0.0f;
      if constexpr (kE4) {
#pragma unroll
        for (int i = 0; i < kSteps; ++i)
#pragma unroll
          for (int x = 0; x < 4; ++x) top = fmaxf(top, there ? fabsf(to_f32(p[16 * i + 4 * t + x])) : 0.0f);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      }
      const float power = kE4 ? row_power(top) : 1.0f, k = 1.0f / power;
      f[e] = factor * power;
#pragma unroll
      for (int i = 0; i < kSteps; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) {                            // a[0], a[1]: rows g, g + 8; a[2], a[3]
          const __nv_bfloat16* d = p + 16 * i + (kE4 ? 4 * t + 2 * x : 2 * t + 8 * x);
          uint32_t v = 0;
          if (there) {
            if constexpr (kE4) {
              v = bits_of(__floats2half2_rn(to_f32(d[0]) * k, to_f32(d[1]) * k));
            } else {
              if (a.q_words) {
                v = *reinterpret_cast<const uint32_t*>(d);
              } else {
                const uint16_t* w = reinterpret_cast<const uint16_t*>(d);
                v = (uint32_t)w[0] | ((uint32_t)w[1] << 16);
              }
            }
          }
          q[i][2 * x + e] = v;
        }
    }
  }

  // Tiles [lo, hi) of one segment.
  __device__ __forceinline__ void tiles(const PagedArgs& a, Shared& sh, int b, int h, int row0, int n, uint32_t lo,
                                        uint32_t hi) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int warp_row = row0 + 16 * warp;
    const bool works = warp_row < a.nodes * a.group;             // a warp past the last row copies only
    load_rows(a, b, h, warp_row);
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.0f;
    const uint32_t* tree = tree_of(a, b);
    const int32_t* table = a.table + (size_t)b * a.width;
    const uint32_t per_page = a.page / 16, stride = a.kv_heads * per_page;
    const uint8_t* keys = static_cast<const uint8_t*>(a.k_pages) + (size_t)h * per_page * 16 * kRowBytes;
    const uint8_t* values = static_cast<const uint8_t*>(a.v_pages) + (size_t)h * per_page * 16 * kRowBytes;
    const int end = min(n, (int)(hi * kTile)), plain = min(end, plain_end(a, n));
    const uint32_t last_block = (uint32_t)(end - 1) / 16;
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(&sh.kv[0][0][0]);

    int id[kParts];
    auto look_up = [&](uint32_t tile) {
#pragma unroll
      for (int u = 0; u < kParts; ++u) id[u] = table[page_of(a, min(tile * kParts + u, last_block))];
    };
    // Copies of a tile whose pages are in id[]; entries from `end` on, and those of pages
    // outside the pool, become zeros.  Which parts lie in such pages, as bits.
    auto copy = [&](uint32_t tile, int stage) {
      uint32_t outside = 0;
      unsigned long long off[kParts];
#pragma unroll
      for (int u = 0; u < kParts; ++u) {
        const uint32_t block = min(tile * kParts + u, last_block);
        const bool out = (unsigned)id[u] >= (unsigned)a.n_pages;
        outside |= (uint32_t)out << u;
        off[u] = ((unsigned long long)(out ? 0u : (uint32_t)id[u]) * stride + (block - page_of(a, block) * per_page)) *
                 (16 * kRowBytes);
      }
      const uint32_t to = base + stage * 2 * kTileBytes;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        constexpr int kPass = kThreads / kChunks;                // rows of one pass of the threads
        const int chunk = tid % kChunks, row = tid / kChunks + i * kPass;
        const int u0 = i * kPass / 16;                           // the row's part, known but for rows of 64 bytes
        unsigned long long from = off[u0];
        uint32_t out = outside >> u0 & 1u;
        if constexpr (kPass > 16) {
          if (tid / kChunks >= 16) {
            from = off[u0 + 1];
            out = outside >> (u0 + 1) & 1u;
          }
        }
        from += (uint32_t)(row & 15) * kRowBytes + (uint32_t)chunk * 16;
        const bool there = !out && (int)(tile * kTile) + row < end;
        copy16(to + place(row, chunk), keys + from, there);
        copy16(to + kTileBytes + place(row, chunk), values + from, there);
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
      return outside;
    };
    look_up(lo);
    uint32_t outside = copy(lo, 0), next_outside = 0;
    if (lo + 1 < hi) look_up(lo + 1);
    for (uint32_t tile = lo; tile < hi; ++tile) {
      const int stage = (tile - lo) & 1;
      if (tile + 1 < hi) {
        next_outside = copy(tile + 1, stage ^ 1);
        if (tile + 2 < hi) look_up(tile + 2);
        asm volatile("cp.async.wait_group 1;" ::: "memory");
      } else {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
      }
      const int first = (int)tile * kTile;
      const bool masked = outside != 0 || first + kTile > plain;
      const uint32_t ks = base + stage * 2 * kTileBytes, vs = ks + kTileBytes;
      if (masked && (a.nodes > 1 || tree != nullptr)) {
        // odd values of the newest entries, of this thread's own copies, which have arrived
        uint32_t any = 0;
#pragma unroll 1
        for (int i = 0; i < kCopies; ++i) {
          constexpr int kPass = kThreads / kChunks;
          if (first + tid / kChunks + i * kPass < n - a.nodes) continue;
          uint4* p = reinterpret_cast<uint4*>(&sh.kv[stage][1][place(tid / kChunks + i * kPass, tid % kChunks)]);
          uint4 x = *p;
          const uint4 odd = make_uint4(odd_in<C>(x.x), odd_in<C>(x.y), odd_in<C>(x.z), odd_in<C>(x.w));
          const uint32_t here = odd.x | odd.y | odd.z | odd.w;
          if (here != 0) *p = make_uint4(x.x & ~odd.x, x.y & ~odd.y, x.z & ~odd.z, x.w & ~odd.w);
          any |= here;
        }
        if (any != 0) sh.odd = 1;
      }
      __syncthreads();
      if (works) {
        // S: kTile / 8 tiles of 8 entries; s[j][0..3] = rows g, g, g + 8, g + 8 by entries 8j + 2t, + 1
        float s[kTile / 8][4];
#pragma unroll
        for (int j = 0; j < kTile / 8; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.0f;
        // a step of the dims for all entries, then the next: products in a row have
        // accumulators of their own
        if constexpr (kE4) {
          // matrices (entries 0-7, 8-15) of chunk i, of chunk i + 1
#pragma unroll
          for (int i = 0; i < kSteps; i += 2)
#pragma unroll
            for (int j = 0; j < kTile / 16; ++j) {
              uint32_t r[4];
              ldmatrix4(r, ks + place(16 * j + (lane & 15), i + (lane >> 4)));
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                  mma16<kE4>(s[2 * j + x], q[i + c], halves_of_e4m3(r[2 * c + x] & 0xFFFFu),
                             halves_of_e4m3(r[2 * c + x] >> 16));
            }
        } else {
          // matrices (entries 0-7) of chunks 2i and 2i + 1, (entries 8-15) of the same
#pragma unroll
          for (int i = 0; i < kSteps; ++i)
#pragma unroll
            for (int j = 0; j < kTile / 16; ++j) {
              uint32_t r[4];
              ldmatrix4(r, ks + place(16 * j + (lane & 7) + (lane >> 4) * 8, 2 * i + (lane >> 3 & 1)));
              mma16<kE4>(s[2 * j], q[i], r[0], r[1]);
              mma16<kE4>(s[2 * j + 1], q[i], r[2], r[3]);
            }
        }
#pragma unroll
        for (int j = 0; j < kTile / 8; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[j][e] *= f[e >> 1];
        if (masked) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int node = min((warp_row + g + 8 * e) / a.group, a.nodes - 1);
            uint32_t bits[2];                                    // entries 0-31, 32-63 of the tile
            seen_bits(a, tree, n, node, first, end, bits);
            bits[0] >>= 2 * t;
            bits[1] >>= 2 * t;
#pragma unroll
            for (int j = 0; j < kTile / 8; ++j)
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                float& y = s[j][2 * e + x];
                y = bits[j / 4] >> (8 * (j & 3) + x) & 1u ? y : -INFINITY;
              }
            // a row that sees an entry of a page outside the pool is NaN
            const uint32_t out0 = (outside & 1u ? 0xFFFFu : 0u) | (outside & 2u ? 0xFFFF0000u : 0u);
            const uint32_t out1 = (outside & 4u ? 0xFFFFu : 0u) | (outside & 8u ? 0xFFFF0000u : 0u);
            if (((bits[0] << 2 * t & out0) | (bits[1] << 2 * t & out1)) != 0) l[e] = NAN;
          }
        }
        float c[2];
        bool moved = false;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = -INFINITY;
#pragma unroll
          for (int j = 0; j < kTile / 8; ++j) x = fmaxf(x, fmaxf(s[j][2 * e], s[j][2 * e + 1]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          x = fmaxf(x, m[e]);
          c[e] = x == m[e] ? 1.0f : exp2_(m[e] - x);
          moved |= x != m[e];
          m[e] = x;
        }
        if (__any_sync(0xffffffffu, moved)) {
          l[0] *= c[0];
          l[1] *= c[1];
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            o[i][0] *= c[0]; o[i][1] *= c[0];
            o[i][2] *= c[1]; o[i][3] *= c[1];
          }
        }
        const float below[2] = {m[0] == -INFINITY ? 0.0f : m[0] - kLift, m[1] == -INFINITY ? 0.0f : m[1] - kLift};
#pragma unroll
        for (int j = 0; j < kTile / 16; ++j) {
          // p of 16 entries as the fragment of a step: two bf16 values that add up to 16 bits
          // of it, or two of fp16 beside 8-bit values (22 bits, paged.cu)
          uint32_t hi_[4], lo_[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int e = x & 1;                                 // rows g, g + 8
            const float* y = &s[2 * j + (x >> 1)][2 * e];
            const float p0 = exp2_(y[0] - below[e]), p1 = exp2_(y[1] - below[e]);
            l[e] += p0 + p1;
            if constexpr (kE4) {
              split_halves(p0, p1, hi_[x], lo_[x]);
            } else {
              const __nv_bfloat162 two = __floats2bfloat162_rn(p0, p1);
              const float2 back = __bfloat1622float2(two);
              hi_[x] = bits_of(two);
              lo_[x] = bits_of(__floats2bfloat162_rn(p0 - back.x, p1 - back.y));
            }
          }
          if constexpr (kE4) {
            // matrices (entries 0-7, 8-15) of chunk i, of chunk i + 1: a chunk's even dims are
            // one tile of 8, its odd dims the next
#pragma unroll
            for (int i = 0; i < kChunks; i += 2) {
              uint32_t r[4];
              ldmatrix4_trans(r, vs + place(16 * j + (lane & 15), i + (lane >> 4)));
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const uint32_t u = __byte_perm(r[2 * x], 0, 0x3120), w = __byte_perm(r[2 * x + 1], 0, 0x3120);
                const uint32_t u0 = halves_of_e4m3(u & 0xFFFFu), w0 = halves_of_e4m3(w & 0xFFFFu);
                const uint32_t u1 = halves_of_e4m3(u >> 16), w1 = halves_of_e4m3(w >> 16);
                mma16<kE4>(o[2 * (i + x)], hi_, u0, w0);
                mma16<kE4>(o[2 * (i + x) + 1], hi_, u1, w1);
                mma16<kE4>(o[2 * (i + x)], lo_, u0, w0);
                mma16<kE4>(o[2 * (i + x) + 1], lo_, u1, w1);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < kChunks; i += 4) {
              uint32_t r[2][4];
              ldmatrix4_trans(r[0], vs + place(16 * j + (lane & 15), i + (lane >> 4)));
              ldmatrix4_trans(r[1], vs + place(16 * j + (lane & 15), i + 2 + (lane >> 4)));
#pragma unroll
              for (int x = 0; x < 4; ++x) mma16<kE4>(o[i + x], hi_, r[x >> 1][2 * (x & 1)], r[x >> 1][2 * (x & 1) + 1]);
#pragma unroll
              for (int x = 0; x < 4; ++x) mma16<kE4>(o[i + x], lo_, r[x >> 1][2 * (x & 1)], r[x >> 1][2 * (x & 1) + 1]);
            }
          }
        }
      }
      __syncthreads();
      outside = next_outside;
    }
  }

  // Each warp's rows to the output, or to a partial slot.
  __device__ __forceinline__ void finish(const PagedArgs& a, Shared& sh, int b, int h, int row0, int n, uint32_t lo,
                                         uint32_t hi, bool whole, float* slot) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int rows = a.nodes * a.group;
    const float v_scale = kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    const bool poison = too_long(a, b);
    bool any_odd = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float sum = l[e];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (poison) sum = NAN;
      const int r = 16 * warp + g + 8 * e, row = row0 + r;
      const int node = min(row, rows - 1) / a.group, head = h * a.group + row - node * a.group;
      if (t == 0 && !(sum > 0.0f)) atomicOr(&sh.lost[r >> 5], 1u << (r & 31));
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        // four dims side by side: 8-bit values have them (even and odd tiles); else the lanes
        // of a pair exchange two, and take a tile each
        float4 x;
        int d;
        if constexpr (kE4) {
          x = make_float4(o[2 * i][2 * e], o[2 * i + 1][2 * e], o[2 * i][2 * e + 1], o[2 * i + 1][2 * e + 1]);
          d = 16 * i + 4 * t;
        } else {
          const bool odd = t & 1;
          const float g0 = odd ? o[2 * i][2 * e] : o[2 * i + 1][2 * e], g1 = odd ? o[2 * i][2 * e + 1] : o[2 * i + 1][2 * e + 1];
          const float y0 = __shfl_xor_sync(0xffffffffu, g0, 1), y1 = __shfl_xor_sync(0xffffffffu, g1, 1);
          x = odd ? make_float4(y0, y1, o[2 * i + 1][2 * e], o[2 * i + 1][2 * e + 1])
                  : make_float4(o[2 * i][2 * e], o[2 * i][2 * e + 1], y0, y1);
          d = 16 * i + (odd ? 8 : 0) + 4 * (t >> 1);
        }
        if (row >= rows) continue;
        any_odd |= odd_sums(x);
        if (whole) {
          write_row<__nv_bfloat16>(a, (long long)b * a.nodes + node, head, d, D, x, m[e], sum, v_scale, kLift);
        } else {
          *reinterpret_cast<float4*>(slot + r * D + d) = x;
          if (d == 0) {
            slot[kRows * D + 2 * r] = m[e];
            slot[kRows * D + 2 * r + 1] = sum;
          }
        }
      }
    }
    any_odd = __syncthreads_or(any_odd);
    if (any_odd || sh.odd)
      add_odd_values<C, __nv_bfloat16, D>(a, b, h, row0, min(rows - row0, kRows), n, (int)(lo * kTile), (int)(hi * kTile),
                                          whole ? nullptr : slot, any_odd ? kOddCleared | kOddSums : kOddCleared, sh.front,
                                          sh.lost);
  }
};

template <class C, int D> constexpr int rows_per_sm = D == 256 ? 2 : 3;

template <class C, int D>
__global__ void __launch_bounds__(kThreads, rows_per_sm<C, D>) paged_rows_kernel(const __grid_constant__ PagedArgs a) {
  using A = Rows<C, D>;
  extern __shared__ __align__(128) uint8_t tiles_raw[];
  typename A::Shared& sh = *reinterpret_cast<typename A::Shared*>(tiles_raw);
  uint32_t* before = reinterpret_cast<uint32_t*>(tiles_raw + sizeof(typename A::Shared));
  __shared__ uint32_t scratch[kWarps];
  pdl_wait();
  pdl_trigger();                     // the joining kernel makes the same plan meanwhile
  const Plan plan = make_plan<A>(a, before, scratch, (int)gridDim.x);
  const Run run = make_run(a, plan, before);
  A at;
  each_segment<A>(a, run, before, [&](int b, int h, int row0, uint32_t lo, uint32_t hi, bool whole, float* slot) {
    if (threadIdx.x == 0) sh.odd = 0;
    if (threadIdx.x < A::kRows / 32) sh.lost[threadIdx.x] = 0;
    __syncthreads();
    const int n = length_of(a, b);
    at.tiles(a, sh, b, h, row0, n, lo, hi);
    at.finish(a, sh, b, h, row0, n, lo, hi, whole, slot);
    __syncthreads();
  });
}

template <class C, int D> cudaError_t launch_as(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  using A = Rows<C, D>;
  static std::atomic<unsigned long long> raised{0};
  return launch_runs<A, C, __nv_bfloat16, D>(a, paged_rows_kernel<C, D>, kThreads, sizeof(typename A::Shared),
                                             152 * rows_per_sm<C, D>, s, workspace, raised);
}

}  // namespace

cudaError_t launch_paged_rows(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  if (a.cache_dtype == FOVEA_BF16) return launch_as<__nv_bfloat16, 256>(a, s, workspace);
  return a.dim == 64    ? launch_as<__nv_fp8_e4m3, 64>(a, s, workspace)
         : a.dim == 128 ? launch_as<__nv_fp8_e4m3, 128>(a, s, workspace)
                        : launch_as<__nv_fp8_e4m3, 256>(a, s, workspace);
}

}  // namespace fovea
