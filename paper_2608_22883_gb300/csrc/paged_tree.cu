// fovea_paged_attention with many rows a key head (draft trees) on tcgen05: paged.cu has
// the formulas, paged_rows.cu the form for other sizes.
//
// A CTA takes 128 rows and tiles of 64 entries.  S = Q K^T goes to tensor memory, a row a
// lane, so that a thread has a row's scores of a tile and no maximum or sum crosses lanes.
// It writes p back over the scores, as the first operand of O += P V (two bf16 values that
// add up to 16 bits of p, or two of fp16 beside 8-bit values: 22 bits, lifted so that the
// largest fit).  V lies as it is cached, entries by dims, and is read along its rows (MN-major).
// The roles, joined by mbarriers with bounded waits: four warps turn S into P; two copy
// keys and two values of the pages (asynchronous copies, or through registers where 8 bits
// become fp16) into the 128-byte-swizzled layout; one issues the products.  S of a tile is
// formed while P of the one before is made (two places in tensor memory), and two CTAs an
// SM fill one another's waits.
//
// Measured: eight trees of 32 nodes over 32 to 2912 entries, 28 heads over 4: 26 us; 16 of 64 nodes, 40 key heads, 480 to 640 entries: 86 us (floor
// 30).  What bounds it is a tile's chain, most of it the 64 exponentials and twice as many
// conversions of a row in one thread (1 to 2 us by time stamps, 27 % of the issue slots used),
// and per run the first tile's and the last products' latencies (about 3 us each).
//
// O stays in tensor memory.  A row's reference moves only when its maximum has grown by
// 2^8, so that O is seldom read back and rescaled; until then p is up to 2^8.
#include <atomic>

#include "packed.cuh"
#include "paged_core.cuh"
#include "tc_ptx.cuh"

namespace fovea {

namespace {

using namespace tc;

constexpr int kTreeThreads = 9 * 32;
constexpr uint32_t kTmemCols = 256;
constexpr float kSlack = 8.0f;       // growth of a maximum that a row's reference bears

__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// mbar_wait of a converged warp (the same answer in every lane), its first try in line; a
// wait that gives up tells the other roles.
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, int* abort, uint64_t limit_ns) {
  if (__all_sync(0xffffffffu, mbar_test_wait(bar, parity))) return true;
  if (__all_sync(0xffffffffu, mbar_wait(bar, parity, abort, limit_ns))) return true;
  *static_cast<volatile int*>(abort) = 1;
  return false;
}
// 32 bytes, a whole sector (two stores of 16 each would write half of one).
__device__ __forceinline__ void store32(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f,
                                        uint32_t g, uint32_t h) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d),
               "r"(e), "r"(f), "r"(g), "r"(h)
               : "memory");
}
// A barrier of the four warps that hold the rows, and whether any thread of theirs has x.
__device__ __forceinline__ bool any_row(bool x) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, 1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n}\n" : "=r"(any) : "r"((uint32_t)x) : "memory");
  return any != 0;
}
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

template <class C, int D> struct Tree {
  static constexpr bool kE4 = sizeof(C) == 1, kWaits = true;
  static constexpr float kLift = kE4 ? 7.0f : 0.0f;              // p 2^7 2^8 fits fp16
  // runs of three tiles at least: one tree of 64 nodes over 704 entries 17 us, with one 23
  static constexpr int kRows = 128, kBlock = 64, kLeast = 3;
  static constexpr uint32_t kFront = 2;
  static constexpr int kSlot = kRows * (D + 2);                  // a multiple of 8 floats
  static constexpr int kStages = 2, kParts = kBlock / 16;
  static constexpr int kHalves = D / 64;                         // blocks of 64 dims, 128 bytes a row
  static constexpr int kTileBytes = kHalves * kBlock * 128;      // keys or values of a tile, 16 bits each
  static constexpr int kRowBytes = D * sizeof(C), kChunks = kRowBytes / 16;
  static constexpr uint32_t kFormat = kE4 ? 0u : 1u;
  // D fp32, A and B of the format, M = 128; S: N = 64 entries, K-major; O: N = D dims, MN-major
  static constexpr uint32_t kIdesc = (1u << 4) | (kFormat << 7) | (kFormat << 10) | ((uint32_t)(kRows >> 4) << 24);
  static constexpr uint32_t kIdescS = kIdesc | ((uint32_t)(kBlock >> 3) << 17);
  static constexpr uint32_t kIdescO = kIdesc | ((uint32_t)(D >> 3) << 17) | (1u << 16);
  static constexpr uint32_t kColS = 128;                         // two places of 64 columns behind O

  // A wait by parity tells of a phase only while its barrier is neither a phase behind it nor
  // ahead.  Every barrier serves every second tile (q_empty: every segment), and the wait for
  // a tile comes when the one two tiles before is known to have ended and the one two tiles
  // behind cannot have: tile c's S is formed when O has tile c - 2, O gets tile c when the
  // softmax has given its P, and the products end in the order in which they are issued.
  struct Shared {
    uint8_t q[kHalves * kRows * 128];
    uint8_t k[kStages][kTileBytes], v[kStages][kTileBytes];
    // of the last segments begun, four at most before one is done: rows' powers (8 bits),
    // and whether a masked tile had odd values
    float power[4][kRows];
    int odd[4];
    uint32_t lost[kRows / 32];       // rows whose sum is no number, as bits
    float front[D];                  // of add_odd_values
    uint32_t outside[4];             // of the last tiles: parts whose page is not in the pool, as bits
    uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
    uint64_t q_empty, s_full[2], p_full[2], o_done[2], drain;
    uint32_t tmem;
    int abort;
    uint32_t scratch[kTreeThreads / 32];
  };
  // A chunk of 16 bytes in a tile of rows of 128 bytes with the 128-byte swizzle.
  __device__ __forceinline__ static uint32_t place(int row, int chunk, int rows) {
    return (uint32_t)((chunk >> 3) * rows * 128 + row * 128 + (((chunk & 7) ^ (row & 7)) << 4));
  }
};

// Sixteen 8-bit values as two chunks of fp16.
__device__ __forceinline__ void widen(const uint4& x, uint4& lo, uint4& hi) {
  lo = make_uint4(halves_of_e4m3(x.x & 0xFFFFu), halves_of_e4m3(x.x >> 16), halves_of_e4m3(x.y & 0xFFFFu),
                  halves_of_e4m3(x.y >> 16));
  hi = make_uint4(halves_of_e4m3(x.z & 0xFFFFu), halves_of_e4m3(x.z >> 16), halves_of_e4m3(x.w & 0xFFFFu),
                  halves_of_e4m3(x.w >> 16));
}
template <class C> __device__ __forceinline__ uint32_t clear_odd(uint4& x) {
  const uint4 odd = make_uint4(odd_in<C>(x.x), odd_in<C>(x.y), odd_in<C>(x.z), odd_in<C>(x.w));
  x = make_uint4(x.x & ~odd.x, x.y & ~odd.y, x.z & ~odd.z, x.w & ~odd.w);
  return odd.x | odd.y | odd.z | odd.w;
}

// Copies of the pages: keys (behind the queries of each segment) by warps 4 and 5, values by
// warps 6 and 7.
template <class C, int D, bool KEYS> struct Copier {
  using T = Tree<C, D>;
  using S = typename T::Shared;
  static constexpr int kThreads2 = 64, kPass = kThreads2 / T::kChunks, kCopies = T::kBlock / kPass;
  const PagedArgs& a;
  S& sh;
  int tid;                           // 0 .. 63
  uint32_t begun = 0, segments = 0;  // tiles, segments
  bool go = true;

  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    return go = warp_wait(bar, parity, &sh.abort, a.wait_ns);
  }
  __device__ __forceinline__ void queries(int b, int h, int row0) {
    const int rows = a.nodes * a.group;
#pragma unroll 1
    for (int r = tid; r < T::kRows; r += kThreads2) {
      const int row = row0 + r;
      const bool there = row < rows;
      const __nv_bfloat16* p = row_of<__nv_bfloat16>(a, b, h, there ? row : 0);
      if (!T::kE4 && a.q_chunks) {   // with the copies of the first keys
        const uint32_t q = smem_u32(sh.q);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) copy16(q + T::place(r, c, T::kRows), p + 8 * c, there);
        continue;
      }
      float power = 1.0f;
      if constexpr (T::kE4) {
        float top = 0.0f;
#pragma unroll 16
        for (int d = 0; d < D; ++d) top = fmaxf(top, there ? fabsf(to_f32(p[d])) : 0.0f);
        power = row_power(top);
        sh.power[segments & 3][r] = power;
      }
      const float k = 1.0f / power;
#pragma unroll 4
      for (int c = 0; c < D / 8; ++c) {
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (there) {
          if (a.q_chunks) {
            x = *reinterpret_cast<const uint4*>(p + 8 * c);
          } else {
            const uint16_t* w = reinterpret_cast<const uint16_t*>(p + 8 * c);
            x = make_uint4(w[0] | (uint32_t)w[1] << 16, w[2] | (uint32_t)w[3] << 16, w[4] | (uint32_t)w[5] << 16,
                           w[6] | (uint32_t)w[7] << 16);
          }
          if constexpr (T::kE4) {
            uint32_t* w = &x.x;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[i] = bits_of(__floats2half2_rn(__uint_as_float(w[i] << 16) * k, __uint_as_float(w[i] & 0xFFFF0000u) * k));
          }
        }
        *reinterpret_cast<uint4*>(sh.q + T::place(r, c, T::kRows)) = x;
      }
    }
  }

  __device__ __forceinline__ void segment(int b, int h, int row0, uint32_t lo, uint32_t hi) {
    if (!go) return;
    const int n = length_of(a, b);
    const int end = min(n, (int)(hi * T::kBlock));
    const uint32_t last_block = (uint32_t)(end - 1) / 16;
    const int32_t* table = a.table + (size_t)b * a.width;
    const uint32_t per_page = a.page / 16, stride = a.kv_heads * per_page;
    const bool mixed = a.nodes > 1 || a.tree != nullptr;         // rows may differ in what they see
    const int chunk = tid % T::kChunks, row = tid / T::kChunks;  // this thread's of the first pass
    const uint8_t* mine = static_cast<const uint8_t*>(KEYS ? a.k_pages : a.v_pages) +
                          (size_t)h * per_page * 16 * T::kRowBytes + row * T::kRowBytes + chunk * 16;
    // The blocks of a tile in the pool (below 2^32 of them) and the parts that are not in it.
    int id[T::kParts];
    uint32_t block[T::kParts], outside = 0;
    auto look_up = [&](uint32_t tile) {
#pragma unroll
      for (int u = 0; u < T::kParts; ++u) id[u] = table[page_of(a, min(tile * T::kParts + u, last_block))];
    };
    auto find = [&](uint32_t tile) {
      outside = 0;
#pragma unroll
      for (int u = 0; u < T::kParts; ++u) {
        const uint32_t at = min(tile * T::kParts + u, last_block);
        const bool out = (unsigned)id[u] >= (unsigned)a.n_pages;
        outside |= (uint32_t)out << u;
        block[u] = (out ? 0u : (uint32_t)id[u]) * stride + (at - page_of(a, at) * per_page);
      }
    };
    // pass i: rows row + i kPass of the tile, of part i kPass / 16 (rows of 64 bytes: 16 rows
    // a pass, one part)
    auto source = [&](int i) {
      constexpr int kRow = T::kRowBytes;
      return mine + (unsigned long long)block[i * kPass / 16] * (16 * kRow) + (i * kPass % 16) * kRow;
    };
    auto there = [&](uint32_t tile, int i) {
      return !(outside >> (i * kPass / 16) & 1u) && (int)(tile * T::kBlock) + row + i * kPass < end;
    };
    // pass i's row is one of the newest entries, whose odd values are cleared
    auto newest = [&](uint32_t tile, int i) { return (int)(tile * T::kBlock) + row + i * kPass >= n - a.nodes; };
    auto masked = [&](uint32_t tile) { return mixed && (int)(tile + 1) * T::kBlock > n - a.nodes; };
    uint64_t* empty = KEYS ? sh.k_empty : sh.v_empty;
    uint8_t (*places)[T::kTileBytes] = KEYS ? sh.k : sh.v;
    look_up(lo);
    if constexpr (KEYS) {
      if (segments > 0 && !wait(&sh.q_empty, (segments - 1) & 1)) return;
      queries(b, h, row0);
    }
    if constexpr (T::kE4) {
      uint4 x[kCopies];                                          // the next tile's, on their way
      auto load = [&](uint32_t tile) {
        find(tile);
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          x[i] = make_uint4(0u, 0u, 0u, 0u);
          if (there(tile, i)) x[i] = __ldg(reinterpret_cast<const uint4*>(source(i)));
        }
        if (tile + 1 < hi) look_up(tile + 1);
      };
      load(lo);
#pragma unroll 1
      for (uint32_t tile = lo; tile < hi; ++tile, ++begun) {
        const int st = begun % T::kStages;
        if (begun >= T::kStages && !wait(&empty[st], (begun / T::kStages - 1) & 1)) return;
        uint32_t any = 0;
        if (!KEYS && masked(tile)) {
#pragma unroll
          for (int i = 0; i < kCopies; ++i)
            if (newest(tile, i)) any |= clear_odd<C>(x[i]);
        }
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
          uint4 y, z;
          widen(x[i], y, z);
          *reinterpret_cast<uint4*>(places[st] + T::place(row + i * kPass, 2 * chunk, T::kBlock)) = y;
          *reinterpret_cast<uint4*>(places[st] + T::place(row + i * kPass, 2 * chunk + 1, T::kBlock)) = z;
        }
        landed(begun, outside, any);
        if (tile + 1 < hi) load(tile + 1);
      }
    } else {
      // As many tiles on their way as there are places; the oldest is waited for when the
      // next has none.
      uint32_t tile = lo, oldest = lo, outsides = 0;             // of the tiles on their way, 4 bits a place
#pragma unroll 1
      while (oldest < hi) {
        const int st = begun % T::kStages;
        bool is_free = tile < hi && tile - oldest < T::kStages;
        if (is_free && begun >= T::kStages) {
          const uint32_t parity = (begun / T::kStages - 1) & 1;
          is_free = __all_sync(0xffffffffu, mbar_test_wait(&empty[st], parity));
          if (!is_free && tile == oldest) {                      // nothing on its way
            if (!wait(&empty[st], parity)) return;
            is_free = true;
          }
        }
        if (is_free) {
          find(tile);
          const uint32_t to = smem_u32(places[st]);
          const bool all = outside == 0 && (int)(tile + 1) * T::kBlock <= end;
#pragma unroll
          for (int i = 0; i < kCopies; ++i)
            copy16(to + T::place(row + i * kPass, chunk, T::kBlock), source(i), all || there(tile, i));
          asm volatile("cp.async.commit_group;" ::: "memory");
          outsides = (outsides & ~(15u << 4 * st)) | outside << 4 * st;
          ++tile;
          ++begun;
          if (tile < hi) look_up(tile);
          continue;
        }
        if (tile - oldest == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        const uint32_t done = begun - (tile - oldest), out = outsides >> 4 * (done % T::kStages) & 15u;
        uint32_t any = 0;
        if (!KEYS && masked(oldest)) {
#pragma unroll 1
          for (int i = 0; i < kCopies; ++i) {
            if (!newest(oldest, i)) continue;
            uint4* p = reinterpret_cast<uint4*>(places[done % T::kStages] + T::place(row + i * kPass, chunk, T::kBlock));
            uint4 x = *p;
            const uint32_t here = clear_odd<C>(x);
            if (here != 0) *p = x;
            any |= here;
          }
        }
        landed(done, out, any);
        ++oldest;
      }
    }
    ++segments;
  }
  // A tile is in its place: seen by the tensor cores after the fence, by all with the arrival.
  __device__ __forceinline__ void landed(uint32_t tile, uint32_t outside, uint32_t any) {
    if (KEYS && tid == 0) sh.outside[tile & 3] = outside;
    if (any != 0) sh.odd[segments & 3] = 1;
    fence_async();
    __syncwarp();
    if ((tid & 31) == 0) arrive(&(KEYS ? sh.k_full : sh.v_full)[tile % T::kStages]);
  }
};

// The products, by warp 8: S of a tile before O of the one in front of it.
template <class C, int D> struct Issuer {
  using T = Tree<C, D>;
  using S = typename T::Shared;
  const PagedArgs& a;
  S& sh;
  uint32_t tmem;
  uint32_t formed = 0, added = 0;    // tiles of S, of O
  bool go = true;

  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    return go = warp_wait(bar, parity, &sh.abort, a.wait_ns);
  }
  __device__ __forceinline__ void form(bool last) {
    const int st = formed % T::kStages, buf = formed & 1;
    if (!wait(&sh.k_full[st], formed / T::kStages & 1)) return;
    // the place of S held P of two tiles before
    if (formed >= 2 && !wait(&sh.o_done[buf], (formed - 2) / 2 & 1)) return;
    tc_fence_after();
    if (elect_one()) {
      const uint64_t q = sw128_desc(smem_u32(sh.q)), k = sw128_desc(smem_u32(sh.k[st]));
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        umma_bf16(tmem + T::kColS + buf * 64, q + (uint64_t)(((i >> 2) * T::kRows * 128 >> 4) + 2 * (i & 3)),
                  k + (uint64_t)(((i >> 2) * T::kBlock * 128 >> 4) + 2 * (i & 3)), T::kIdescS, i > 0);
      umma_commit(&sh.s_full[buf]);
      umma_commit(&sh.k_empty[st]);
      if (last) umma_commit(&sh.q_empty);
    }
    __syncwarp();
    ++formed;
  }
  __device__ __forceinline__ void add(bool first) {
    const int st = added % T::kStages, buf = added & 1;
    if (!wait(&sh.v_full[st], added / T::kStages & 1) || !wait(&sh.p_full[buf], added / 2 & 1)) return;
    tc_fence_after();
    if (elect_one()) {
      // 64 dims of V, 16 entries a step: 1 KB from 8 entries to the next, a block of dims
      // behind the other
      const uint64_t v = sw128_desc(smem_u32(sh.v[st])) + ((uint64_t)((T::kBlock * 128 >> 4) - 1) << 16);
      const uint32_t p = tmem + T::kColS + buf * 64;
#pragma unroll
      for (int part = 0; part < 2; ++part)                       // p's upper and lower bits
#pragma unroll
        for (int i = 0; i < T::kBlock / 16; ++i)
          umma_ts(tmem, p + part * 32 + i * 8, v + (uint64_t)(i * (16 * 128 >> 4)), T::kIdescO,
                  !first || part > 0 || i > 0);
      umma_commit(&sh.v_empty[st]);
      umma_commit(&sh.o_done[buf]);
    }
    __syncwarp();
    ++added;
  }
  __device__ __forceinline__ void segment(uint32_t lo, uint32_t hi) {
    if (go) form(lo + 1 == hi);
    for (uint32_t tile = lo; go && tile < hi; ++tile) {
      if (tile + 1 < hi) form(tile + 2 == hi);
      if (go) add(tile == lo);
    }
  }
};

// Scores to p, and the rows' results: warps 0 to 3, a row a thread.
template <class C, int D> struct Softmax {
  using T = Tree<C, D>;
  using S = typename T::Shared;
  const PagedArgs& a;
  S& sh;
  uint32_t tmem;                     // with the warp's first lane
  uint32_t tiles = 0, segments = 0;
  bool go = true;

  __device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity) {
    return go = warp_wait(bar, parity, &sh.abort, a.wait_ns);
  }
  __device__ __forceinline__ void segment(int b, int h, int row0, uint32_t lo, uint32_t hi, bool whole, float* slot) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = threadIdx.x;
    const int rows = a.nodes * a.group, row = row0 + r;
    const int n = length_of(a, b);
    const int end = min(n, (int)(hi * T::kBlock)), plain = min(end, plain_end(a, n));
    const uint32_t* tree = tree_of(a, b);
    const bool works = row0 + 32 * warp < rows;                  // else its rows are none
    const int node = min(row, rows - 1) / a.group;
    float f = a.scale * kLog2e * (T::kE4 && a.k_scale != nullptr ? a.k_scale[h] : 1.0f);
    const bool long_one = too_long(a, b);
    float m = -INFINITY, l = 0.0f;
    for (uint32_t tile = lo; go && tile < hi; ++tile, ++tiles) {
      const int buf = tiles & 1;
      const int first = (int)tile * T::kBlock;
      // the words of the tree, while the scores are on their way
      uint32_t bits[2] = {0xFFFFFFFFu, 0xFFFFFFFFu};
      if (works && first + T::kBlock > plain) seen_bits(a, tree, n, node, first, end, bits);
      if (!wait(&sh.s_full[buf], tiles / 2 & 1)) break;
      tc_fence_after();
      if (works) {
        if (T::kE4 && tile == lo) f *= sh.power[segments & 3][r];
        const uint32_t at = tmem + T::kColS + buf * 64;
        float s[64];
        {
          float (&x)[32] = *reinterpret_cast<float (*)[32]>(&s[0]);
          float (&y)[32] = *reinterpret_cast<float (*)[32]>(&s[32]);
          tmem_ld32(at, x);
          tmem_ld32(at + 32, y);
        }
#pragma unroll
        for (int i = 0; i < 64; ++i) s[i] *= f;
        const uint32_t outside = *static_cast<volatile uint32_t*>(&sh.outside[tiles & 3]);
        if (outside != 0 || first + T::kBlock > plain) {
#pragma unroll
          for (int i = 0; i < 64; ++i) {
            s[i] = bits[i / 32] >> (i & 31) & 1u ? s[i] : -INFINITY;
          }
          // a row that sees an entry of a page outside the pool is NaN
          const uint32_t out0 = (outside & 1u ? 0xFFFFu : 0u) | (outside & 2u ? 0xFFFF0000u : 0u);
          const uint32_t out1 = (outside & 4u ? 0xFFFFu : 0u) | (outside & 8u ? 0xFFFF0000u : 0u);
          if (((bits[0] & out0) | (bits[1] & out1)) != 0) l = NAN;
        }
        __syncwarp();
        float tops[4] = {s[0], s[1], s[2], s[3]};                // four chains
#pragma unroll
        for (int i = 4; i < 64; ++i) tops[i & 3] = fmaxf(tops[i & 3], s[i]);
        const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
        const bool grows = top > m + kSlack || (m == -INFINITY && top > -INFINITY);
        const float c = grows ? exp2_(m - top) : 1.0f;
        if (grows) m = top;
        l *= c;
        if (tile > lo && __any_sync(0xffffffffu, grows)) {       // O of the tiles before, rescaled
          if (!wait(&sh.o_done[(tiles - 1) & 1], (tiles - 1) / 2 & 1)) break;
          tc_fence_after();
#pragma unroll 1
          for (int d = 0; d < D; d += 8) {
            float x[8];
            tmem_ld8(tmem + d, x);
            uint32_t y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = __float_as_uint(x[i] * c);
            tmem_st8(tmem + d, y);
          }
        }
        const float below = m == -INFINITY ? 0.0f : m - T::kLift;
        float sums[4] = {l, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 64; i += 16) {
          uint32_t hi_[8], lo_[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float p0 = exp2_(s[i + 2 * j] - below), p1 = exp2_(s[i + 2 * j + 1] - below);
            sums[2 * (j & 1)] += p0;
            sums[2 * (j & 1) + 1] += p1;
            if constexpr (T::kE4) {
              split_halves(p0, p1, hi_[j], lo_[j]);
            } else {
              const __nv_bfloat162 two = __floats2bfloat162_rn(p0, p1);
              const float2 back = __bfloat1622float2(two);
              hi_[j] = bits_of(two);
              lo_[j] = bits_of(__floats2bfloat162_rn(p0 - back.x, p1 - back.y));
            }
          }
          tmem_st8(at + i / 2, hi_);
          tmem_st8(at + 32 + i / 2, lo_);
        }
        l = (sums[0] + sums[1]) + (sums[2] + sums[3]);
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive(&sh.p_full[buf]);
    }
    if (go) wait(&sh.o_done[(tiles - 1) & 1], (tiles - 1) / 2 & 1);
    tc_fence_after();
    const bool there = row < rows, poison = !go || long_one;
    const bool odd = *static_cast<volatile int*>(&sh.odd[segments & 3]) != 0;
    const float v_scale = T::kE4 && a.v_scale != nullptr ? a.v_scale[h] : 1.0f;
    const int head = h * a.group + row - node * a.group;
    const float sum = poison ? NAN : l;
    const float k = sum == 0.0f ? 0.0f : v_scale * __frcp_rn(sum);   // as in write_row; NaN when given up
    uint64_t check[2] = {0, 0};      // stay 0 beside finite sums
    if (works) {
      const long long at = ((long long)b * a.nodes + node) * a.heads + head;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + at * D;
      const bool sectors = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
#pragma unroll 1
      for (int d = 0; d < D; d += 32) {
        float x[32];
        tmem_ld32(tmem + d, x);
        if (there) {
#pragma unroll
          for (int i = 0; i < 32; i += 2) check[i / 2 & 1] = fma2(pack2(x[i], x[i + 1]), 0, check[i / 2 & 1]);
          if (whole) {
            uint32_t y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = bits_of(__floats2bfloat162_rn(x[2 * i] * k, x[2 * i + 1] * k));
            if (sectors) {
#pragma unroll
              for (int i = 0; i < 16; i += 8)
                store32(out + d + 2 * i, y[i], y[i + 1], y[i + 2], y[i + 3], y[i + 4], y[i + 5], y[i + 6], y[i + 7]);
            } else {
#pragma unroll
              for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<uint4*>(out + d + 2 * i) = make_uint4(y[i], y[i + 1], y[i + 2], y[i + 3]);
            }
          } else {
            const uint32_t* y = reinterpret_cast<const uint32_t*>(x);
#pragma unroll
            for (int i = 0; i < 32; i += 8)
              store32(slot + r * D + d + i, y[i], y[i + 1], y[i + 2], y[i + 3], y[i + 4], y[i + 5], y[i + 6], y[i + 7]);
          }
        }
        __syncwarp();
      }
      if (there && !whole) *reinterpret_cast<float2*>(slot + T::kRows * D + 2 * r) = make_float2(m, sum);
      if (there && whole && a.lse != nullptr)
        a.lse[at] = sum == 0.0f ? -INFINITY : (m - T::kLift + log2f(sum)) * kLn2;
    }
    tc_fence_before();
    const uint32_t none = __ballot_sync(0xffffffffu, !(sum > 0.0f));
    if (lane == 0) sh.lost[warp] = none;
    const uint64_t checked = add2(check[0], check[1]);
    const bool odd_sum = any_row(lo2(checked) != 0.0f || hi2(checked) != 0.0f);   // all four warps have written, and read the segment's word
    if (odd || odd_sum)
      add_odd_values<C, __nv_bfloat16, D>(a, b, h, row0, min(rows - row0, T::kRows), n, (int)(lo * T::kBlock),
                                          (int)(hi * T::kBlock), whole ? nullptr : slot,
                                          odd_sum ? kOddCleared | kOddSums : kOddCleared, sh.front, sh.lost);
    if (threadIdx.x == 0) *static_cast<volatile int*>(&sh.odd[segments & 3]) = 0;
    ++segments;
  }
};

template <class C, int D>
__global__ void __launch_bounds__(kTreeThreads, 2) paged_tree_kernel(const __grid_constant__ PagedArgs a) {
  using T = Tree<C, D>;
  using S = typename T::Shared;
  extern __shared__ uint8_t tree_raw[];
  uint8_t* base = tree_raw + ((1024u - (smem_u32(tree_raw) & 1023u)) & 1023u);
  S& sh = *reinterpret_cast<S*>(base);
  uint32_t* before = reinterpret_cast<uint32_t*>(base + sizeof(S));
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < T::kStages; ++i) {
      mbar_init(&sh.k_full[i], 2);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], 2);
      mbar_init(&sh.v_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_full[i], 4);
      mbar_init(&sh.o_done[i], 1);
    }
    mbar_init(&sh.q_empty, 1);
    mbar_init(&sh.drain, 1);
    for (int i = 0; i < 4; ++i) sh.odd[i] = 0;
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    tmem_alloc(&sh.tmem, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  pdl_wait();
  pdl_trigger();                     // the joining kernel makes the same plan meanwhile
  const Plan plan = make_plan<T>(a, before, sh.scratch, (int)gridDim.x);
  const Run run = make_run(a, plan, before);
  if (warp < 4) {
    Softmax<C, D> w{a, sh, tmem + ((uint32_t)(32 * warp) << 16)};
    each_segment<T>(a, run, before, [&](int b, int h, int row0, uint32_t lo, uint32_t hi, bool whole, float* slot) {
      w.segment(b, h, row0, lo, hi, whole, slot);
    });
  } else if (warp < 8) {
    auto copy = [&](auto w) {
      each_segment<T>(a, run, before, [&](int b, int h, int row0, uint32_t lo, uint32_t hi, bool, float*) {
        w.segment(b, h, row0, lo, hi);
      });
    };
    if (warp < 6) copy(Copier<C, D, true>{a, sh, (int)threadIdx.x - 128});
    else copy(Copier<C, D, false>{a, sh, (int)threadIdx.x - 192});
    if constexpr (!T::kE4) asm volatile("cp.async.wait_all;" ::: "memory");
  } else {
    Issuer<C, D> w{a, sh, tmem};
    each_segment<T>(a, run, before, [&](int, int, int, uint32_t lo, uint32_t hi, bool, float*) { w.segment(lo, hi); });
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const bool gave_up = *static_cast<volatile int*>(&sh.abort) != 0;
  if (gave_up && warp == 8) {        // the products issued end before tensor memory goes
    if (elect_one()) umma_commit(&sh.drain);
    __syncwarp();
    mbar_wait(&sh.drain, 0, nullptr, kDefaultWaitLimitNs);
  }
  if (threadIdx.x == 0 && blockIdx.x < plan.runs) a.gave_up[blockIdx.x] = gave_up;
  __syncwarp();
  if (warp == 8) tmem_dealloc(tmem, kTmemCols);
}

template <class C, int D> cudaError_t launch_as(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  using T = Tree<C, D>;
  static std::atomic<unsigned long long> raised{0};
  return launch_runs<T, C, __nv_bfloat16, D>(a, paged_tree_kernel<C, D>, kTreeThreads, 1024 + sizeof(typename T::Shared),
                                             152 * 2, s, workspace, raised);
}

}  // namespace

cudaError_t launch_paged_tree(const PagedArgs& a, cudaStream_t s, size_t* workspace) {
  if (a.cache_dtype == FOVEA_BF16)
    return a.dim == 64 ? launch_as<__nv_bfloat16, 64>(a, s, workspace) : launch_as<__nv_bfloat16, 128>(a, s, workspace);
  return a.dim == 64 ? launch_as<__nv_fp8_e4m3, 64>(a, s, workspace) : launch_as<__nv_fp8_e4m3, 128>(a, s, workspace);
}

}  // namespace fovea
