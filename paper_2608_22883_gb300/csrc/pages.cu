// Pages of a cache: the accepted path of a verified draft tree moved to the front of its
// entries (fovea_cache_keep), and sequences continued, forked and dropped
// (fovea_cache_fork).
#include <atomic>

#include "common.cuh"

namespace fovea {

namespace {

constexpr int kKeepThreads = 256, kKeepBytes = 48 * 1024;

// Entry base + i <- entry base + nodes[i], base = lens - size: all sources are read, into
// shared memory, before an entry is written, so that any list of nodes is right.  A CTA
// takes `cols` 16-byte columns of a head of a sequence's keys or values.  Bound by latency:
// a path's entries are a few KB a head.
__global__ void __launch_bounds__(kKeepThreads) cache_keep_kernel(const __grid_constant__ CachePages c,
                                                                  const int32_t* lens, const int32_t* nodes, int path,
                                                                  int size, int cols, int row_vecs, int32_t* new_lens) {
  extern __shared__ uint4 staged[];
  __shared__ int node_of[FOVEA_MAX_TREE];
  __shared__ int count;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, b = blockIdx.y;
  const int parts = (row_vecs + cols - 1) / cols, h = blockIdx.x / parts, col0 = blockIdx.x % parts * cols;
  if (tid == 0) count = path;
  __syncthreads();
  const int n = lens[b];
  for (int i = tid; i < path; i += kKeepThreads) {
    const int x = nodes[(long long)b * path + i];
    node_of[i] = x;
    if ((unsigned)x >= (unsigned)size) atomicMin(&count, i);       // the path ends before it
  }
  __syncthreads();
  const bool there = n >= size;      // else (an idle sequence) nothing moves
  if (blockIdx.x == 0 && blockIdx.z == 0 && tid == 0) new_lens[b] = there ? n - size + count : n;
  if (!there) return;
  uint4* pool = static_cast<uint4*>(blockIdx.z == 0 ? c.k : c.v);
  const int base = n - size, most = min(cols, row_vecs - col0);
  const long long room = (long long)c.width * c.page;
  auto place = [&](int e) -> long long {                           // of an entry's first vector, -1: none
    if (e >= room) return -1;
    const int id = c.table[(long long)b * c.width + e / c.page];
    if ((unsigned)id >= (unsigned)c.n_pages) return -1;
    return (((long long)id * c.kv_heads + h) * c.page + e % c.page) * row_vecs + col0;
  };
  for (int i = tid; i < count * most; i += kKeepThreads) {
    const int p = i / most;
    if (node_of[p] == p) continue;
    const long long from = place(base + node_of[p]);
    if (from >= 0) staged[i] = pool[from + i % most];
  }
  __syncthreads();
  for (int i = tid; i < count * most; i += kKeepThreads) {
    const int p = i / most;
    if (node_of[p] == p || place(base + node_of[p]) < 0) continue;
    const long long to = place(base + p);
    if (to >= 0) pool[to + i % most] = staged[i];
  }
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

// Which pages are held, which last pages stay, and the fresh pages of every continuation,
// the lowest free pages first.  One CTA: the marks are a bit a page in shared memory, and
// the steps depend on one another.  Writes the fresh entries of the new table, the entry
// of each partly filled page and the number of pages left; the rest is the copies' kernel's.
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(const __grid_constant__ CachePages c,
                                                                 const __grid_constant__ ForkArgs f) {
  extern __shared__ uint32_t marks[];                    // a bit a page, then the children's arrays
  const int words = (c.n_pages + 31) / 32;
  int* last = reinterpret_cast<int*>(marks + words);     // partly filled page of a child, -1: none
  int* begin = last + f.C;                               // fresh pages of the children before it
  int* have = begin + f.C + 1;                           // pages that it has without fresh ones
  __shared__ int scratch[kPlanThreads / 32];
  __shared__ int chunk_free[kPlanThreads];               // free pages before each thread's words
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < words; i += kPlanThreads) marks[i] = 0;
  __syncthreads();
  for (int child = warp; child < f.C; child += kPlanThreads / 32) {
    const Kept k = kept_of(c, f, child);
    const int32_t* row = c.table + (long long)max(k.parent, 0) * c.width;
    for (int i = lane; i < k.whole; i += 32) {
      const int id = row[i];
      if ((unsigned)id < (unsigned)c.n_pages) atomicOr(&marks[id >> 5], 1u << (id & 31));
    }
    if (lane == 0) {
      const int id = k.rest > 0 ? row[k.whole] : -1;
      last[child] = (unsigned)id < (unsigned)c.n_pages ? id : -1;
    }
  }
  __syncthreads();
  // a last page stays with the first of its holders, unless some child holds it whole
  int sum = 0;
  const int per = (f.C + kPlanThreads - 1) / kPlanThreads;
  const int c0 = min(tid * per, f.C), c1 = min(c0 + per, f.C);
  for (int child = c0; child < c1; ++child) {
    const Kept k = kept_of(c, f, child);
    const int id = last[child];
    bool stays = k.rest > 0;
    if (id >= 0) {
      stays = (marks[id >> 5] >> (id & 31) & 1u) == 0;
      for (int other = 0; stays && other < child; ++other) stays = last[other] != id;
    }
    if (stays) f.new_table[(long long)child * f.new_width + k.whole] =
        id >= 0 ? id : c.table[(long long)k.parent * c.width + k.whole];
    have[child] = k.whole + stays;
    sum += k.need - have[child];
  }
  int fresh;
  int at = block_scan(sum, scratch, fresh);
  for (int child = c0; child < c1; ++child) {
    begin[child] = at;
    at += kept_of(c, f, child).need - have[child];
  }
  if (tid == 0) begin[f.C] = fresh;
  __syncthreads();
  for (int child = tid; child < f.C; child += kPlanThreads)
    if (last[child] >= 0) atomicOr(&marks[last[child] >> 5], 1u << (last[child] & 31));
  __syncthreads();
  // free pages: those without a mark
  auto free_in = [&](int word) -> uint32_t {
    const int left = c.n_pages - 32 * word;
    return ~marks[word] & (left >= 32 ? 0xffffffffu : (1u << left) - 1u);
  };
  const int span = (words + kPlanThreads - 1) / kPlanThreads;
  const int w0 = min(tid * span, words), w1 = min(w0 + span, words);
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
      id = 32 * word + __fns(free_in(word), 0, skip + 1);
    }
    f.new_table[(long long)lo * f.new_width + have[lo] + (r - begin[lo])] = id;
  }
}

// The new tables' other entries and lengths, and the copies of last pages: a CTA a child,
// head and kind.
__global__ void __launch_bounds__(256) fork_copy_kernel(const __grid_constant__ CachePages c,
                                                        const __grid_constant__ ForkArgs f, int row_vecs) {
  pdl_wait();
  pdl_trigger();
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
  if (k.rest == 0 || *f.free < 0) return;
  const int src = row[k.whole], dst = to[k.whole];
  if (src == dst || (unsigned)src >= (unsigned)c.n_pages || (unsigned)dst >= (unsigned)c.n_pages) return;
  uint4* pool = static_cast<uint4*>(blockIdx.y & 1 ? c.v : c.k);
  const uint4* p = pool + ((long long)src * c.kv_heads + h) * c.page * row_vecs;
  uint4* q = pool + ((long long)dst * c.kv_heads + h) * c.page * row_vecs;
  const int n = k.rest * row_vecs;
  for (int i = tid; i < n; i += 4 * 256) {               // four on their way together
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + 256 * j < n) x[j] = p[i + 256 * j];
#pragma unroll
    for (int j = 0; j < 4; ++j)
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
  const size_t smem = ((size_t)(c.n_pages + 31) / 32 + 3 * (size_t)f.C + 1) * 4;
  cudaError_t e = raise_smem_limit(fork_plan_kernel, 200 * 1024, raised);
  if (e != cudaSuccess) return e;
  e = launch_pdl(fork_plan_kernel, dim3(1), dim3(kPlanThreads), smem, s, c, f);
  if (e != cudaSuccess || f.C == 0) return e;
  return launch_pdl(fork_copy_kernel, dim3(f.C, 2 * c.kv_heads), dim3(256), 0, s, c, f, vecs_of_row(c));
}

}  // namespace fovea
