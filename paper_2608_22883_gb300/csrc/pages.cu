// Pages of a cache: the accepted path of a verified draft tree moved to the front of its
// entries (fovea_cache_keep), and sequences continued, forked and dropped
// (fovea_cache_fork).
#include <atomic>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kKeepThreads = 128;
// Staged entries: what is left of the 48 KB of a launch without a raised limit, beside the
// kernel's places of the entries and their number.
constexpr int kKeepBytes = 48 * 1024 - 2 * FOVEA_MAX_TREE * 8 - 64;

// Entry base + i <- entry base + nodes[i], base = lens - size: all sources are read, into
// shared memory, before an entry is written, so that any list of nodes is right.  A CTA
// takes `cols` 16-byte columns of a head of a sequence's keys or values.  Bound by latency:
// a path's entries are a few KB a head, behind the loads of a length and of a page.  With
// the storing of the tree in front: one sequence 6.7 us, 16 of 40 heads 13 (floor 6.4).
__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(const __grid_constant__ CachePages c,
                                                                  const int32_t* lens, const int32_t* nodes, int path,
                                                                  int size, int cols, int row_vecs, int32_t* new_lens) {
  extern __shared__ uint4 staged[];
  // each entry's first vector where it is and where it goes; no move: -1
  __shared__ long long from[FOVEA_MAX_TREE], to[FOVEA_MAX_TREE];
  __shared__ int count;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, b = blockIdx.y;
  const int parts = (row_vecs + cols - 1) / cols, h = blockIdx.x / parts, col0 = blockIdx.x % parts * cols;
  if (tid == 0) count = path;
  const int n = lens[b], base = n >= size ? n - size : -1;     // the lowest lengths would wrap
  __syncthreads();
  const long long room = (long long)c.width * c.page;
  auto place = [&](int e) -> long long {                 // of an entry's first vector, -1: none
    if (e >= room) return -1;
    const int id = c.table[(long long)b * c.width + e / c.page];
    if ((unsigned)id >= (unsigned)c.n_pages) return -1;
    return (((long long)id * c.kv_heads + h) * c.page + e % c.page) * row_vecs + col0;
  };
  for (int i = tid; i < path; i += kKeepThreads) {
    const int x = nodes[(long long)b * path + i];
    const bool valid = (unsigned)x < (unsigned)size;
    if (!valid) atomicMin(&count, i);                    // the path ends before it
    const bool moves = valid && x != i && base >= 0;     // a shorter (idle) sequence stays as it is
    const long long p = moves ? place(base + x) : -1, q = moves ? place(base + i) : -1;
    from[i] = q < 0 ? -1 : p;
    to[i] = q;
  }
  __syncthreads();
  if (blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) new_lens[b] = base >= 0 ? base + count : n;
  uint4* pool = static_cast<uint4*>(blockIdx.z == 0 ? c.k : c.v);
  const int most = min(cols, row_vecs - col0), total = count * most;
  for (int i = tid; i < total; i += kKeepThreads) {
    const long long p = from[i / most];
    if (p >= 0) staged[i] = pool[p + i % most];
  }
  __syncthreads();
  for (int i = tid; i < total; i += kKeepThreads)
    if (from[i / most] >= 0) pool[to[i / most] + i % most] = staged[i];
}

// ---------------------------------------------------------------------------
// Fork
// ---------------------------------------------------------------------------

constexpr int kPlanThreads = 1024;

// What a continuation keeps: its first `n` entries, `whole` full pages and `rest` entries
// of one more, and the pages it shall have.
struct Kept { int parent, n, whole, rest, need; };
__device__ __forceinline__ Kept kept_of(const CachePages& c, const ForkArgs& f, int child) {
  Kept k;
  k.parent = f.parents[child];
  long long held = 0;
  if ((unsigned)k.parent < (unsigned)c.B) {
    held = f.lens[k.parent];
    const int width = c.width < f.new_width ? c.width : f.new_width;
    held = max(0ll, min(held, (long long)width * c.page));
    if (f.keep != nullptr) held = max(0ll, min(held, (long long)f.keep[child]));
  } else {
    k.parent = -1;
  }
  k.n = (int)held;
  k.whole = k.n / c.page;
  k.rest = k.n - k.whole * c.page;
  const long long room = f.room != nullptr ? max(0, f.room[child]) : 0;
  const long long need = (held + room + c.page - 1) / c.page;
  k.need = (int)min(need, (long long)f.new_width);
  return k;
}

// Exclusive sum over the CTA's threads, and the total.
__device__ __forceinline__ int block_scan(int x, int* scratch, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += up;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = sum;
  __syncthreads();
  int before = sum - x;
  total = 0;
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  return before;
}

// Shared memory of the plan, in words: the marks, a bit a page; of each continuation; the
// table of last pages.
struct PlanLayout {
  int words, C, slots;               // slots: of the table, a power of two
  __host__ __device__ PlanLayout(int n_pages, int C_) : words((n_pages + 31) / 32), C(C_), slots(32) {
    while (slots < 2 * C) slots *= 2;
  }
  __host__ __device__ size_t total() const { return (size_t)words + 6 * (size_t)C + 1 + 2 * (size_t)slots; }
};
__device__ __forceinline__ uint32_t slot_of(int page, int slots) { return ((uint32_t)page * 2654435761u >> 8) & (slots - 1); }

// Which pages are held, which last pages stay, and the fresh pages of every continuation,
// the lowest free pages first.  One CTA, bound by latency: the marks are a bit a page in
// shared memory, and the steps depend on one another.  With the copies: one sequence as six
// 7.2 us, 128 sequences of up to 8192 entries 10.2 (15.8 with the children's lengths worked
// out in each step, last pages compared in pairs and nothing read ahead).  Writes the fresh
// entries of the new table, the entry of each partly filled page and the number of pages
// left; the rest is the copies' kernel's.
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const __grid_constant__ CachePages c,
                                                                 const __grid_constant__ ForkArgs f) {
  extern __shared__ uint32_t marks[];
  const PlanLayout y(c.n_pages, f.C);
  int* last = reinterpret_cast<int*>(marks + y.words);   // partly filled page of a child, -1: none
  int* parent = last + f.C;
  int* whole = parent + f.C;                             // full pages
  int* need = whole + f.C;                               // pages that it shall have
  int* have = need + f.C;                                // pages that it has without fresh ones
  int* begin = have + f.C;                               // fresh pages of the children before it
  int* keys = begin + f.C + 1;                           // last pages, -1: an empty slot
  int* first = keys + y.slots;                           // the first child that holds each
  __shared__ int scratch[kPlanThreads / 32];
  __shared__ int chunk_free[kPlanThreads];               // free pages before each thread's words
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int child = tid; child < f.C; child += kPlanThreads) {
    const Kept k = kept_of(c, f, child);
    parent[child] = k.parent;
    whole[child] = k.whole;
    need[child] = k.need;
    last[child] = k.rest > 0 ? 0 : -1;
  }
  for (int i = tid; i < y.words; i += kPlanThreads) marks[i] = 0;
  for (int i = tid; i < y.slots; i += kPlanThreads) {
    keys[i] = -1;
    first[i] = f.C;
  }
  __syncthreads();
  for (int child = warp; child < f.C; child += kPlanThreads / 32) {
    const int n = whole[child];
    const bool part = last[child] >= 0;
    const int32_t* row = c.table + (long long)max(parent[child], 0) * c.width;
    for (int i = lane; i < n + part; i += 32) {
      const int id = row[i];
      const bool there = (unsigned)id < (unsigned)c.n_pages;
      if (i < n) {
        if (there) atomicOr(&marks[id >> 5], 1u << (id & 31));
      } else {
        // its place in the table of last pages (at most half full: the search ends)
        last[child] = there ? id : -2;                   // -2: a partly filled page outside the pool
        if (there) {
          uint32_t at = slot_of(id, y.slots);
          while (true) {
            const int key = atomicCAS(&keys[at], -1, id);
            if (key == -1 || key == id) break;
            at = (at + 1) & (y.slots - 1);
          }
          atomicMin(&first[at], child);
        }
      }
    }
  }
  __syncthreads();
  // a last page stays with the first of its holders, unless some child holds it whole
  int sum = 0;
  const int per = (f.C + kPlanThreads - 1) / kPlanThreads;
  const int c0 = min(tid * per, f.C), c1 = min(c0 + per, f.C);
  for (int child = c0; child < c1; ++child) {
    const int id = last[child], w = whole[child];
    bool stays = id == -2;
    if (id >= 0) {
      uint32_t at = slot_of(id, y.slots);
      while (keys[at] != id) at = (at + 1) & (y.slots - 1);
      stays = first[at] == child && (marks[id >> 5] >> (id & 31) & 1u) == 0;
    }
    if (stays)
      f.new_table[(long long)child * f.new_width + w] = id >= 0 ? id : c.table[(long long)parent[child] * c.width + w];
    have[child] = w + stays;
    sum += need[child] - have[child];
  }
  int fresh;
  int at = block_scan(sum, scratch, fresh);              // a barrier: the marks have been read
  for (int child = c0; child < c1; ++child) {
    begin[child] = at;
    at += need[child] - have[child];
    const int id = last[child];
    if (id >= 0) atomicOr(&marks[id >> 5], 1u << (id & 31));
  }
  if (tid == 0) begin[f.C] = fresh;
  __syncthreads();
  // free pages: those without a mark
  auto free_in = [&](int word) -> uint32_t {
    const int left = c.n_pages - 32 * word;
    return ~marks[word] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
  };
  const int span = (y.words + kPlanThreads - 1) / kPlanThreads;
  const int w0 = min(tid * span, y.words), w1 = min(w0 + span, y.words);
  sum = 0;
  for (int i = w0; i < w1; ++i) sum += __popc(free_in(i));
  int available;
  chunk_free[tid] = block_scan(sum, scratch, available);
  if (tid == 0) *f.free = available - fresh;
  __syncthreads();
  for (int r = tid; r < fresh; r += kPlanThreads) {
    int lo = 0, hi = f.C - 1;                            // the last child with begin <= r
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (begin[mid] <= r) lo = mid; else hi = mid - 1;
    }
    int id = -1;
    if (r < available) {
      int t0 = 0, t1 = kPlanThreads - 1;                 // the last chunk with chunk_free <= r
      while (t0 < t1) {
        const int mid = (t0 + t1 + 1) >> 1;
        if (chunk_free[mid] <= r) t0 = mid; else t1 = mid - 1;
      }
      int skip = r - chunk_free[t0], word = t0 * span;
      while (true) {                                     // ends: the chunk has more than `skip` free pages
        const int here = __popc(free_in(word));
        if (skip < here) break;
        skip -= here;
        ++word;
      }
      uint32_t bits = free_in(word);
      for (; skip > 0; --skip) bits &= bits - 1;
      id = 32 * word + __ffs(bits) - 1;
    }
    f.new_table[(long long)lo * f.new_width + have[lo] + (r - begin[lo])] = id;
  }
}

// The new tables' other entries and lengths, and the copies of last pages: a CTA a child,
// head and kind.  What does not depend on the plan, the entries to copy among it (no page is
// both copied from and to), is read while that is made.
__global__ void __launch_bounds__(256) fork_copy_kernel(const __grid_constant__ CachePages c,
                                                        const __grid_constant__ ForkArgs f, int row_vecs) {
  constexpr int kAhead = 4;
  const int tid = threadIdx.x, child = blockIdx.x, h = blockIdx.y >> 1;
  const Kept k = kept_of(c, f, child);
  const int32_t* row = c.table + (long long)max(k.parent, 0) * c.width;
  int32_t* to = f.new_table + (long long)child * f.new_width;
  if (blockIdx.y == 0) {
    for (int i = tid; i < f.new_width; i += 256) {
      if (i < k.whole) to[i] = row[i];
      else if (i >= k.need) to[i] = -1;
    }
    if (tid == 0) f.new_lens[child] = k.n;
  }
  const int src = k.rest > 0 ? row[k.whole] : -1, n = k.rest * row_vecs;
  const bool there = (unsigned)src < (unsigned)c.n_pages;
  uint4* pool = static_cast<uint4*>(blockIdx.y & 1 ? c.v : c.k);
  const uint4* p = pool + ((long long)(there ? src : 0) * c.kv_heads + h) * c.page * row_vecs;
  uint4 x[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j)
    if (there && tid + 256 * j < n) x[j] = p[tid + 256 * j];
  pdl_wait();
  pdl_trigger();
  if (!there || *f.free < 0) return;
  const int dst = to[k.whole];
  if (src == dst || (unsigned)dst >= (unsigned)c.n_pages) return;
  uint4* q = pool + ((long long)dst * c.kv_heads + h) * c.page * row_vecs;
  for (int i = tid; i < n; i += kAhead * 256) {
    if (i != tid) {
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + 256 * j < n) x[j] = p[i + 256 * j];
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i + 256 * j < n) q[i + 256 * j] = x[j];
  }
}

int vecs_of_row(const CachePages& c) {
  return c.dim * (c.dtype == FOVEA_BF16 ? 2 : c.dtype == FOVEA_FP32 ? 4 : 1) / 16;
}

}  // namespace

cudaError_t launch_cache_keep(const CachePages& c, const int32_t* lens, const int32_t* nodes, int path, int size,
                              int32_t* new_lens, cudaStream_t s) {
  const int row_vecs = vecs_of_row(c);
  int cols = row_vecs;
  while (cols * path * 16 > kKeepBytes) cols = (cols + 1) / 2;
  const int parts = (row_vecs + cols - 1) / cols;
  return launch_pdl(cache_keep_kernel, dim3(c.kv_heads * parts, c.B, 2), dim3(kKeepThreads), (size_t)cols * path * 16, s,
                    c, lens, nodes, path, size, cols, row_vecs, new_lens);
}

cudaError_t launch_cache_fork(const CachePages& c, const ForkArgs& f, cudaStream_t s) {
  static std::atomic<unsigned long long> raised{0};
  const size_t smem = PlanLayout(c.n_pages, f.C).total() * 4;
  cudaError_t e = raise_smem_limit(fork_plan_kernel, 220 * 1024, raised);
  if (e != cudaSuccess) return e;
  e = launch_pdl(fork_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, c, f);
  if (e != cudaSuccess || f.C == 0) return e;
  return launch_pdl(fork_copy_kernel, dim3(f.C, 2 * c.kv_heads), dim3(256), 0, s, c, f, vecs_of_row(c));
}

}  // namespace fovea
