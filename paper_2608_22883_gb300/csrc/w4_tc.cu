// fovea_linear_w4 for more rows than fit one warp's tensor-core tile: the
// weights' codes become bf16 integers in tensor memory, where tcgen05 takes them
// as its 128-row operand.
//
//   y[n, o] = sum over groups g of scale[o, g] sum_{k in g} x[n, k] (code[o, k] - zero[o, g])
//
// A first kernel lays x out as the other operand: bf16 columns (an fp32 row as
// three that add up to it), each run of eight k in the order in which a 32-bit word
// of codes yields them, zero-padded.  The product's CTAs then stream 128 weight
// rows x 256 k of codes a stage (16 KB, TMA) with the stage's x; eight warps turn
// codes into integers, one weight row a thread, and write them to tensor memory; one
// lane of each of two warps issues the MMAs, each group's sum into an accumulator of its
// own; four or eight warps read the accumulators, a weight row a thread, and add them
// times their scales in fp32.
//
// The weights' bytes are the floor, and the tensor pipe is busy a quarter of the time.
// What bounds it are the instructions that make integers of the codes (a shift, a LOP3
// and a subtraction for two), the trips of each group's sum through tensor memory, and
// the last round of tiles: 250 tiles of [32000, 4096] give 98 SMs two and 54 one.  By
// that matrix in symmetric groups of 128: 16 bf16 rows 24.3 us, 40 27.6, 64 29.5 (2.6
// TB/s, 38 % of the measured copy); 64 e4m3 rows with scales by row 32.0, by group 36.6,
// whose every sum takes a product of two scales; 40 bf16 rows in groups of 64 37.0, of 32
// 62.0 (with zero points 40.0 and 66.8).  Each 64 columns of x are a launch that makes the
// integers again: 128 bf16 rows 55.2, 1024 418; 64 fp32 rows 108.
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "packed.cuh"
#include "tc_ptx.cuh"
#include "w4_x.cuh"

namespace fovea {
namespace w4tc {

using namespace tc;

constexpr int kRows = 128;                 // weight rows of a tile
constexpr int kStageK = 256;               // columns of a stage: 128 bytes of codes a row
constexpr int kCodeBytes = kRows * 128;
constexpr int kUnitK = 128;                // columns of an operand buffer in tensor memory
constexpr int kMaxCols = 64;               // columns of x a launch takes
constexpr int kBufs = 4;                   // operand buffers
constexpr int kMaxStages = 6;
constexpr int kMaxSumWarps = 8;
constexpr int kIntWarps = 8;               // two teams of four, taking turns by unit
constexpr int kMmaWarps = 2;               // taking turns by unit
// Summing warps for NC columns: one team of four, or two that take half of the
// columns each.
// us with one and with two, 4096 x 32000 in groups of 128: 16 rows 24.4 and 26.3, 32
// 25.6 and 26.5; in two teams 64 took less than in one.
template <int NC> constexpr int kSums = NC <= 32 ? 4 : kMaxSumWarps;
template <int NC> constexpr int kThreads = 32 * (kSums<NC> + kIntWarps + kMmaWarps + 1);
constexpr int kBarBytes = 1024;
constexpr int kScaleBytes = 4 * 4 * kMaxCols * 4;   // x's scales of four groups, a copy per warp
constexpr int kSmemBudget = 224 * 1024;
constexpr uint32_t kTmemCols = 512;
constexpr int kSlots = 4;                  // accumulator slots
constexpr uint32_t kAccCol = 256;          // they follow the operand buffers (64 columns each)

struct Args {
  W4 w;
  int groups;
  int cols, cols_pad;                // columns of x (rows times parts); padded to 16, 32, 48 or 64
  int parts;                         // columns a row of x is the sum of
  int n0, rows;                      // rows of y
  const float* x_scale;              // by_group: [groups, kMaxCols]; else [kMaxCols] or null
  bool by_group;
  const float* bias;
  void* y; int y_dtype;
  long long ldy;
  int stages, ksteps, tiles, split;  // ring depth; stages of the contraction; tiles; CTAs a tile
  uint32_t k128;                     // kW4One28
  unsigned long long wait_ns;
  int* err;
};

__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(tmem_d),
      "r"(tmem_a), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
      "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]),
      "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]),
      "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Consecutive accumulator columns of this thread's lane, of one group or of two that
// lie kPair columns apart, with their wait (several reads: early outputs, that none
// takes the place of a later read's address).
constexpr uint32_t kPair = 32;
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[1][16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0][0]), "=r"(r[0][1]), "=r"(r[0][2]), "=r"(r[0][3]), "=r"(r[0][4]), "=r"(r[0][5]),
        "=r"(r[0][6]), "=r"(r[0][7]), "=r"(r[0][8]), "=r"(r[0][9]), "=r"(r[0][10]), "=r"(r[0][11]),
        "=r"(r[0][12]), "=r"(r[0][13]), "=r"(r[0][14]), "=r"(r[0][15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[1][24]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7}, [%24];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {"
      "%8, %9, %10, %11, %12, %13, %14, %15}, [%25];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {"
      "%16, %17, %18, %19, %20, %21, %22, %23}, [%26];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r[0][0]), "=&r"(r[0][1]), "=&r"(r[0][2]), "=&r"(r[0][3]), "=&r"(r[0][4]), "=&r"(r[0][5]),
        "=&r"(r[0][6]), "=&r"(r[0][7]), "=&r"(r[0][8]), "=&r"(r[0][9]), "=&r"(r[0][10]), "=&r"(r[0][11]),
        "=&r"(r[0][12]), "=&r"(r[0][13]), "=&r"(r[0][14]), "=&r"(r[0][15]), "=&r"(r[0][16]),
        "=&r"(r[0][17]), "=&r"(r[0][18]), "=&r"(r[0][19]), "=&r"(r[0][20]), "=&r"(r[0][21]),
        "=&r"(r[0][22]), "=&r"(r[0][23])
      : "r"(taddr), "r"(taddr + 8u), "r"(taddr + 16u)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[1][32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0][0]), "=r"(r[0][1]), "=r"(r[0][2]), "=r"(r[0][3]), "=r"(r[0][4]), "=r"(r[0][5]),
        "=r"(r[0][6]), "=r"(r[0][7]), "=r"(r[0][8]), "=r"(r[0][9]), "=r"(r[0][10]), "=r"(r[0][11]),
        "=r"(r[0][12]), "=r"(r[0][13]), "=r"(r[0][14]), "=r"(r[0][15]), "=r"(r[0][16]), "=r"(r[0][17]),
        "=r"(r[0][18]), "=r"(r[0][19]), "=r"(r[0][20]), "=r"(r[0][21]), "=r"(r[0][22]), "=r"(r[0][23]),
        "=r"(r[0][24]), "=r"(r[0][25]), "=r"(r[0][26]), "=r"(r[0][27]), "=r"(r[0][28]), "=r"(r[0][29]),
        "=r"(r[0][30]), "=r"(r[0][31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[2][16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%32];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%33];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r[0][0]), "=&r"(r[0][1]), "=&r"(r[0][2]), "=&r"(r[0][3]), "=&r"(r[0][4]), "=&r"(r[0][5]),
        "=&r"(r[0][6]), "=&r"(r[0][7]), "=&r"(r[0][8]), "=&r"(r[0][9]), "=&r"(r[0][10]), "=&r"(r[0][11]),
        "=&r"(r[0][12]), "=&r"(r[0][13]), "=&r"(r[0][14]), "=&r"(r[0][15]), "=&r"(r[1][0]), "=&r"(r[1][1]),
        "=&r"(r[1][2]), "=&r"(r[1][3]), "=&r"(r[1][4]), "=&r"(r[1][5]), "=&r"(r[1][6]), "=&r"(r[1][7]),
        "=&r"(r[1][8]), "=&r"(r[1][9]), "=&r"(r[1][10]), "=&r"(r[1][11]), "=&r"(r[1][12]), "=&r"(r[1][13]),
        "=&r"(r[1][14]), "=&r"(r[1][15])
      : "r"(taddr), "r"(taddr + kPair)
      : "memory");
}
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[2][32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
      "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%64];\n\t"
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
      "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, %48, "
      "%49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%65];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=&r"(r[0][0]), "=&r"(r[0][1]), "=&r"(r[0][2]), "=&r"(r[0][3]), "=&r"(r[0][4]), "=&r"(r[0][5]),
        "=&r"(r[0][6]), "=&r"(r[0][7]), "=&r"(r[0][8]), "=&r"(r[0][9]), "=&r"(r[0][10]), "=&r"(r[0][11]),
        "=&r"(r[0][12]), "=&r"(r[0][13]), "=&r"(r[0][14]), "=&r"(r[0][15]), "=&r"(r[0][16]),
        "=&r"(r[0][17]), "=&r"(r[0][18]), "=&r"(r[0][19]), "=&r"(r[0][20]), "=&r"(r[0][21]),
        "=&r"(r[0][22]), "=&r"(r[0][23]), "=&r"(r[0][24]), "=&r"(r[0][25]), "=&r"(r[0][26]),
        "=&r"(r[0][27]), "=&r"(r[0][28]), "=&r"(r[0][29]), "=&r"(r[0][30]), "=&r"(r[0][31]), "=&r"(r[1][0]),
        "=&r"(r[1][1]), "=&r"(r[1][2]), "=&r"(r[1][3]), "=&r"(r[1][4]), "=&r"(r[1][5]), "=&r"(r[1][6]),
        "=&r"(r[1][7]), "=&r"(r[1][8]), "=&r"(r[1][9]), "=&r"(r[1][10]), "=&r"(r[1][11]), "=&r"(r[1][12]),
        "=&r"(r[1][13]), "=&r"(r[1][14]), "=&r"(r[1][15]), "=&r"(r[1][16]), "=&r"(r[1][17]),
        "=&r"(r[1][18]), "=&r"(r[1][19]), "=&r"(r[1][20]), "=&r"(r[1][21]), "=&r"(r[1][22]),
        "=&r"(r[1][23]), "=&r"(r[1][24]), "=&r"(r[1][25]), "=&r"(r[1][26]), "=&r"(r[1][27]),
        "=&r"(r[1][28]), "=&r"(r[1][29]), "=&r"(r[1][30]), "=&r"(r[1][31])
      : "r"(taddr), "r"(taddr + kPair)
      : "memory");
}
__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* map, uint64_t* bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y)
      : "memory");
}
// mbar_wait of a converged warp (the same answer in every lane).  The first try
// is in line: a call makes the caller's loads in flight arrive first, and the
// clock behind the limit costs more than most of the waits here last (a satisfied
// wait: 25 clocks so, 119 with the limit's loop in line).
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort_flag,
                                          uint64_t limit_ns) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit_ns));
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ float ld_dsmem_f32(uint32_t caddr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(caddr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_dsmem_u32(uint32_t caddr) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(caddr) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t bf16_sub2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&a), *reinterpret_cast<__nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// y of row n of the block and weight row o.
__device__ __forceinline__ void store_y(const Args& a, long long o, int n, float v) {
  if (!a.by_group && a.x_scale != nullptr) v *= a.x_scale[n * a.parts];
  if (a.bias != nullptr) v += __ldg(a.bias + o);
  const long long at = (long long)(a.n0 + n) * a.ldy + o;
  if (a.y_dtype == FOVEA_BF16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
  else static_cast<float*>(a.y)[at] = v;
}
// y of weight row o from the sums of the columns col0, col0 + 1, ...
template <class T, int C>
__device__ __forceinline__ void store_rows(const Args& a, long long o, int col0, const float (&acc)[C]) {
  const float b = a.bias != nullptr ? __ldg(a.bias + o) : 0.0f;
  T* y = static_cast<T*>(a.y) + (long long)(a.n0 + col0) * a.ldy + o;
  const float* scale = a.by_group ? nullptr : a.x_scale;
#pragma unroll
  for (int j = 0; j < C; ++j) {
    if (col0 + j < a.cols) *y = from_f32<T>(fmaf(acc[j], scale != nullptr ? scale[col0 + j] : 1.0f, b));
    y += a.ldy;
  }
}
// A barrier of the summing warps alone.
template <int WARPS>
__device__ __forceinline__ void sum_teams_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory");
}

// A place in a ring of barriers and the parity of its round (no division in the
// loops: one costs as much as the wait it serves).
struct Turn {
  int i = 0;
  uint32_t parity = 0;
  __device__ __forceinline__ void next(int size) {
    if (++i == size) {
      i = 0;
      parity ^= 1u;
    }
  }
  // `by` places on; true when the ring's end was passed
  __device__ __forceinline__ bool skip(int by, int size) {
    i += by;
    if (i < size) return false;
    i -= size;
    parity ^= 1u;
    return true;
  }
};

// NC: accumulator columns (cols_pad), in the instruction's steps of 16: the summing
// warps' work goes with them (40 rows by 4096 x 32000, 48 columns against 64: 27.3 and
// 28.8 us, in groups of 64 with zero points 40.1 and 44.0).  G: the group.  A tile's contraction may
// be split over the CTAs of a cluster, which then has one tile.
template <int NC, int G>
__global__ void __launch_bounds__(kThreads<NC>, 1)
linear_w4_tc_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmX,
                    const __grid_constant__ Args a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  constexpr int kSumWarps = kSums<NC>;
  constexpr int kXBlock = NC * 128;                        // 64 k of every column
  constexpr int kStageBytes = kCodeBytes + 4 * kXBlock;
  float* xs_ring = reinterpret_cast<float*>(smem + a.stages * kStageBytes);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + a.stages * kStageBytes + kScaleBytes);
  float* parts_tile = reinterpret_cast<float*>(smem + a.stages * kStageBytes + kScaleBytes + kBarBytes);
  uint64_t* empty = full + kMaxStages;
  uint64_t* afull = empty + kMaxStages;
  uint64_t* aempty = afull + kBufs;
  uint64_t* dfull = aempty + kBufs;
  uint64_t* dempty = dfull + kSlots;
  uint64_t* drain = dempty + kSlots;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int split = a.split;
  const int rank = split > 1 ? (int)cluster_rank() : 0;
  const int first = (int)blockIdx.x / split, step = (int)gridDim.x / split;
  const int k_lo = a.ksteps * rank / split, k_hi = a.ksteps * (rank + 1) / split;
  constexpr int kPerUnit = kUnitK / G;                     // groups in a unit: 1, 2 or 4
  // accumulators, 64 columns a slot: of one group, or of two of up to 32 columns, which
  // then share its waits (with zero points, 16 rows by 4096 x 32000 in groups of 32: 48.3 us,
  // one by one 60.0; with more columns there were only two slots, 40 rows: 68.5 us and 67.3)
  constexpr int kSlotGroups = NC <= 32 && kPerUnit > 1 ? 2 : 1, kSlotsUnit = kPerUnit / kSlotGroups;
  // issuing warps: as many as leave each slot to one of them (a barrier's parity tells
  // a warp only of the round before its own)
  constexpr int kMmas = kSlots >= kMmaWarps * kSlotsUnit ? kMmaWarps : 1;
  constexpr int kPart = NC / (kSumWarps / 4);              // columns of a summing team
  if (threadIdx.x == 0) {
    for (int i = 0; i < kMaxStages; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], kMmas);
    }
    for (int i = 0; i < kBufs; ++i) {
      mbar_init(&afull[i], kIntWarps / 2);
      mbar_init(&aempty[i], 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&dfull[i], 1);
      mbar_init(&dempty[i], kSumWarps);
    }
    mbar_init(drain, kMmaWarps);
    *abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&tmW);
    prefetch_tmap(&tmX);
  }
  if (warp == 0) {
    tmem_alloc(tmem_slot, kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  pdl_trigger();

  if (warp == kSumWarps + kIntWarps + kMmaWarps) {
    // ---- copies.  The codes may be read before the wait: the kernel in front
    // (the one that lays x out) had waited for whatever came before it when it let
    // this one start.
    if (lane == 0) {
      bool waited = false, go = true;
      int i = 0;
      Turn st;
      for (int t = first; go && t < a.tiles; t += step) {
        for (int k = k_lo; k < k_hi; ++k, ++i, st.next(a.stages)) {
          if (i >= a.stages && !mbar_wait(&empty[st.i], st.parity ^ 1u, abort_flag, a.wait_ns)) {
            *abort_flag = 1;
            go = false;
            break;
          }
          uint8_t* dst = smem + st.i * kStageBytes;
          mbar_expect_tx(&full[st.i], (uint32_t)kStageBytes);
          tma_load_2d(dst, &tmW, &full[st.i], k * (kStageK / 2), t * kRows);
          if (waited) {
            tma_load_3d(dst + kCodeBytes, &tmX, &full[st.i], 0, 0, k * 4);
          } else if (i + 1 == a.stages || (t + step >= a.tiles && k + 1 == k_hi)) {
            // the ring is full of codes: now x of the same stages
            pdl_wait();
            waited = true;
            for (int j = 0; j <= i; ++j)
              tma_load_3d(smem + j * kStageBytes + kCodeBytes, &tmX, &full[j], 0, 0,
                          (k_lo + j % (k_hi - k_lo)) * 4);
          }
        }
      }
      if (!waited) pdl_wait();
    }
  } else if (warp >= kSumWarps + kIntWarps) {
    // ---- MMAs: a warp runs its units converged, with addresses and descriptors
    // in uniform registers; one elected lane issues.  That a unit's integers are
    // there also says that its stage has landed.
    constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NC >> 3) << 17) |
                                ((uint32_t)(kRows >> 4) << 24);
    const uint64_t desc0 = sw128_desc(smem_u32(smem) + kCodeBytes);
    const int w = warp - kSumWarps - kIntWarps;
    Turn st, ab, db;
    ab.i = w;
    db.i = w * kSlotsUnit;                                 // the unit's first slot
    bool go = w < kMmas, reused = false;                   // its slots for the second time
    for (int t = first; go && t < a.tiles; t += step) {
      for (int k = k_lo; go && k < k_hi; ++k, st.next(a.stages)) {
        const uint64_t bdesc = desc0 + (uint64_t)((st.i * kStageBytes) >> 4);
#pragma unroll
        for (int hh = 0; hh < 2; hh += kMmas) {
          const int h = kMmas == 1 ? hh : w;
          go = go && warp_wait(&afull[ab.i], ab.parity, abort_flag, a.wait_ns);
          const uint32_t ta = tmem_base + (uint32_t)(ab.i * 64);
#pragma unroll
          for (int s = 0; s < kSlotsUnit; ++s) {
            if (reused)
              go = go && warp_wait(&dempty[db.i + s], db.parity ^ 1u, abort_flag, a.wait_ns);
            if (go) {
              tc_fence_after();
              const uint32_t td = tmem_base + kAccCol + (uint32_t)((db.i + s) * 64);
              const uint64_t bh = bdesc + (uint64_t)(h * (2 * kXBlock >> 4));
              if (elect_one()) {
                constexpr int kSteps = 8 / kPerUnit;       // of 16 columns, a group
#pragma unroll
                for (int q = 0; q < kSlotGroups * kSteps; ++q) {
                  const int k16 = s * kSlotGroups * kSteps + q;      // of the unit's eight
                  umma_ts(td + (uint32_t)(q / kSteps) * kPair, ta + (uint32_t)(k16 * 8),
                          bh + (uint64_t)(((k16 >> 2) * kXBlock >> 4) + 2 * (k16 & 3)), kIdesc,
                          q % kSteps > 0 ? 1u : 0u);
                }
                umma_commit(&dfull[db.i + s]);
                if (s == kSlotsUnit - 1) {
                  umma_commit(&aempty[ab.i]);
                  if (kMmas == 2 || h == 1) umma_commit(&empty[st.i]);
                }
              }
              __syncwarp();
            }
          }
          ab.skip(kMmas, kBufs);
          reused |= db.skip(kMmas * kSlotsUnit, kSlots);
        }
      }
    }
    if (!go && w < kMmas) *abort_flag = 1;
  } else if (warp >= kSumWarps) {
    // ---- codes to integers: thread = weight row, a team's warps every other unit
    const int quarter = warp & 3, team = (warp - kSumWarps) >> 2;
    const int r = quarter * 32 + lane;
    const uint32_t dst = tmem_base + ((uint32_t)(quarter * 32) << 16);
    Turn st, ab;
    ab.i = team;                                           // units 2 i + team
    bool go = true, reused = false;
    const uint32_t k128 = a.k128;
    for (int t = first; go && t < a.tiles; t += step) {
      const long long row = min((long long)t * kRows + r, (long long)a.w.out - 1);
      const uint8_t* zeros = a.w.zeros != nullptr ? a.w.zeros + row * a.groups : nullptr;
      for (int k = k_lo; k < k_hi; ++k) {
        uint32_t z[4] = {0x43084308u, 0x43084308u, 0x43084308u, 0x43084308u};   // of the unit's runs of 32 columns
        if (zeros != nullptr) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int g = (k * kStageK + team * kUnitK + q * 32) / G;
            if (g < a.groups) z[q] = 0x43004300u | (__ldg(zeros + g) & 127u) * 0x10001u;
          }
        }
        if (!warp_wait(&full[st.i], st.parity, abort_flag, a.wait_ns)) {
          go = false;
          break;
        }
        const uint8_t* src = smem + st.i * kStageBytes + r * 128;
        uint4 w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w[q] = *reinterpret_cast<const uint4*>(src + (((team * 4 + q) ^ (r & 7)) << 4));
        if (reused && !warp_wait(&aempty[ab.i], ab.parity ^ 1u, abort_flag, a.wait_ns)) {
          go = false;
          break;
        }
        tc_fence_after();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t v[32];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint4 c = w[2 * half + q];
            const uint32_t ww[4] = {c.x, c.y, c.z, c.w};
            const uint32_t zq = z[2 * half + q];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
              for (int p = 0; p < 4; ++p)
                v[16 * q + 4 * j + p] = bf16_sub2(w4_pair(ww[j] >> (4 * p), k128), zq);
          }
          tmem_st32(dst + (uint32_t)(ab.i * 64 + half * 32), v);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&afull[ab.i]);
        st.next(a.stages);
        reused |= ab.skip(2, kBufs);
      }
    }
    if (!go) *abort_flag = 1;
  } else {
    // ---- sums: thread = weight row, a team's warps half of the columns
    const int quarter = warp & 3, col0 = (warp >> 2) * kPart;
    const int r = quarter * 32 + lane;
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16) + kAccCol + (uint32_t)col0;
    const int slots = (k_hi - k_lo) * 2 * kPerUnit, g0 = k_lo * 2 * kPerUnit;
    float* xs = xs_ring + warp * 4 * kPart;
    Turn db;
    bool go = true;
    pdl_wait();                                            // x's scales come from the kernel in front
    for (int t = first; t < a.tiles; t += step) {
      const long long o = (long long)t * kRows + r;
      const __nv_bfloat16* scales = a.w.scales + min(o, (long long)a.w.out - 1) * a.groups;
      uint64_t acc[kPart / 2];                             // pairs of columns
#pragma unroll
      for (int j = 0; j < kPart / 2; ++j) acc[j] = 0;
      // scales are loaded a round of four groups before their sums arrive: the
      // weight row's own, and with x's in groups a column a lane, which the warp
      // then shares
      constexpr int kAhead = 4;
      float s[kAhead], xq[kAhead];
      const bool quads = a.groups % kAhead == 0 && g0 % kAhead == 0 && slots % kAhead == 0 &&
                         (reinterpret_cast<uintptr_t>(a.w.scales) & 7u) == 0;
      auto fetch = [&](int i0) {
        const int left = min(slots - i0, a.groups - g0 - i0);
        if (quads) {
          uint2 raw = make_uint2(0u, 0u);
          if (left > 0) raw = __ldg(reinterpret_cast<const uint2*>(scales + g0 + i0));
          s[0] = __uint_as_float(raw.x << 16);
          s[1] = __uint_as_float(raw.x & 0xFFFF0000u);
          s[2] = __uint_as_float(raw.y << 16);
          s[3] = __uint_as_float(raw.y & 0xFFFF0000u);
        } else {
#pragma unroll
          for (int q = 0; q < kAhead; ++q) s[q] = q < left ? __bfloat162float(scales[g0 + i0 + q]) : 0.0f;
        }
        if (a.by_group) {
          const float* x = a.x_scale + (long long)(g0 + i0) * kMaxCols + col0 + min(lane, kPart - 1);
#pragma unroll
          for (int q = 0; q < kAhead; ++q) xq[q] = q < left ? x[q * kMaxCols] : 0.0f;
        }
      };
      fetch(0);
      for (int i0 = 0; go && i0 < slots; i0 += kAhead) {
        float sc[kAhead];
        if (a.by_group) {
          __syncwarp();                                    // the last round's have been read
#pragma unroll
          for (int q = 0; q < kAhead; ++q)
            if (lane < kPart) xs[q * kPart + lane] = xq[q];
          __syncwarp();
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) sc[q] = s[q];
        if (i0 + kAhead < slots) fetch(i0 + kAhead);
#pragma unroll
        for (int q = 0; q < kAhead; q += kSlotGroups) {
          if (i0 + q >= slots) break;
          if (!warp_wait(&dfull[db.i], db.parity, abort_flag, a.wait_ns)) {
            go = false;
            break;
          }
          tc_fence_after();
          uint32_t v[kSlotGroups][kPart];
          tmem_ld_cols(lanes + (uint32_t)(db.i * 64), v);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&dempty[db.i]);
#pragma unroll
          for (int u = 0; u < kSlotGroups; ++u) {
            const uint32_t sq = __float_as_uint(sc[q + u]);
            const uint64_t s2 = pack2(sq, sq);
            if (a.by_group) {
#pragma unroll
              for (int j = 0; j < kPart; j += 4) {
                const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(xs + (q + u) * kPart + j);
                acc[j / 2] = fma2(pack2(v[u][j], v[u][j + 1]), mul2(s2, f.x), acc[j / 2]);
                acc[j / 2 + 1] = fma2(pack2(v[u][j + 2], v[u][j + 3]), mul2(s2, f.y), acc[j / 2 + 1]);
              }
            } else {
#pragma unroll
              for (int j = 0; j < kPart; j += 2) acc[j / 2] = fma2(pack2(v[u][j], v[u][j + 1]), s2, acc[j / 2]);
            }
          }
          db.next(kSlots);
        }
      }
      if (!go) {                                           // a result that shows it
        *abort_flag = 1;
#pragma unroll
        for (int j = 0; j < kPart / 2; ++j) acc[j] = 0x7FC000007FC00000ull;
      }
      float sum[kPart];
#pragma unroll
      for (int j = 0; j < kPart; ++j) sum[j] = __uint_as_float((uint32_t)(acc[j / 2] >> (32 * (j & 1))));
      if (split > 1 || a.parts > 1) {
        // the partial tile, [column][row]: over the ring when its tile is the CTA's
        // only one (every stage has been consumed), else behind it
        float* part = split > 1 ? reinterpret_cast<float*>(smem) : parts_tile;
        if (split == 1) sum_teams_sync<kSumWarps>();                  // the last tile's readers are done
#pragma unroll
        for (int j = 0; j < kPart; ++j) part[(col0 + j) * kRows + r] = sum[j];
        if (split == 1) {
          sum_teams_sync<kSumWarps>();
          if (o < a.w.out)
            for (int n = warp >> 2; n < a.rows; n += kSumWarps / 4)
              store_y(a, o, n, part[3 * n * kRows + r] + part[(3 * n + 1) * kRows + r] + part[(3 * n + 2) * kRows + r]);
        }
      } else if (o < a.w.out) {
        if (a.y_dtype == FOVEA_BF16) store_rows<__nv_bfloat16, kPart>(a, o, col0, sum);
        else store_rows<float, kPart>(a, o, col0, sum);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (*abort_flag != 0) {
    if (threadIdx.x == 0) atomicOr(a.err, kErrTimeout);
    if (warp >= kSumWarps + kIntWarps && warp < kSumWarps + kIntWarps + kMmaWarps && elect_one())
      umma_commit(drain);                                  // each issuing warp's MMAs
    if (lane == 0) {
      mbar_wait(drain, 0, nullptr, kDefaultWaitLimitNs);
      const uint64_t t0 = globaltimer_ns();                // copies in flight land
      while (globaltimer_ns() - t0 < 2000000ull) {}
    }
    __syncwarp();
    __syncthreads();
  }
  if (split > 1) {
    // the CTAs' partial tiles meet: CTA `rank` sums every split-th row of y over
    // them in rank order
    cluster_sync();
    const int r = threadIdx.x & (kRows - 1);
    const long long o = (long long)first * kRows + r;
    const uint32_t part = smem_u32(smem), aborted = smem_u32(const_cast<int*>(abort_flag));
    constexpr int kLanes = kThreads<NC> / kRows;
    if (threadIdx.x < kLanes * kRows && o < a.w.out) {
      bool whole = true;                                   // no CTA of the tile gave up
      for (int q = 0; q < split; ++q) whole &= ld_dsmem_u32(map_dsmem(aborted, (uint32_t)q)) == 0u;
      for (int n = rank + split * (int)(threadIdx.x / kRows); n < a.rows; n += split * kLanes) {
        float v = 0.0f;
        for (int p = 0; p < a.parts; ++p)
          for (int q = 0; q < split; ++q)
            v += ld_dsmem_f32(map_dsmem(part + (uint32_t)(((n * a.parts + p) * kRows + r) * 4), (uint32_t)q));
        store_y(a, o, n, whole ? v : __int_as_float(0x7FC00000));
      }
    }
    cluster_sync();
  }
  if (warp == 0) tmem_dealloc(tmem_base, kTmemCols);
}

// x as the product's second operand: out[c, k] bf16, c = block * kMaxCols + the
// block's column, k padded to whole stages; every eight k in the order 0 4 1 5 2
// 6 3 7; and its scales as [groups or 1, kMaxCols] per block.
struct LayoutArgs {
  const void* x; long long ld; int dtype; bool vec;
  const float* x_scale; int x_groups;      // 0: none; 1: one a row; else per group
  int N, in, k_pad;
  int rows_block, blocks, parts;
  __nv_bfloat16* out;
  float* scale_out;
  int* err;
};
constexpr int kLayoutThreads = 256;

__global__ void __launch_bounds__(kLayoutThreads) layout_x_kernel(const LayoutArgs a) {
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x == 0 && threadIdx.x == 0) ensure_header(a.err);
  const int units = a.k_pad / 8;
  const int slots = kMaxCols / a.parts;                    // rows of a block, padding among them
  const long long row_items = (long long)a.blocks * slots * units;
  const long long total = row_items + (long long)a.x_groups * a.blocks * kMaxCols;
  for (long long it = blockIdx.x * kLayoutThreads + threadIdx.x; it < total; it += gridDim.x * kLayoutThreads) {
    if (it >= row_items) {                                 // [block][group][column]
      const long long j = it - row_items;
      const int c = (int)(j % kMaxCols), g = (int)(j / kMaxCols % a.x_groups), b = (int)(j / (kMaxCols * a.x_groups));
      const int n = b * a.rows_block + c;
      a.scale_out[j] = c < a.rows_block && n < a.N ? a.x_scale[(long long)n * a.x_groups + g] : 0.0f;
      continue;
    }
    const int unit = (int)(it % units), slot = (int)(it / units % slots), b = (int)(it / ((long long)units * slots));
    const int n = b * a.rows_block + slot, k0 = unit * 8;
    X8 raw = {};
    if (slot < a.rows_block && n < a.N && k0 < a.in) raw.load(a.x, (long long)n * a.ld + k0, a.dtype, a.vec);
    uint4 v[3];
    raw.columns(a.dtype, v);
#pragma unroll
    for (int p = 0; p < 3; ++p)
      if (p < a.parts)
        *reinterpret_cast<uint4*>(a.out + ((long long)b * kMaxCols + slot * a.parts + p) * a.k_pad + k0) = v[p];
  }
}

struct Plan {
  int parts, rows_block, blocks, k_pad;
  size_t scale_at, bytes;
};
static Plan plan(int N, int in, int group, int x_dtype, bool by_group) {
  Plan p;
  p.parts = x_parts(x_dtype);
  p.rows_block = kMaxCols / p.parts;
  p.blocks = (N + p.rows_block - 1) / p.rows_block;
  p.k_pad = (in + kStageK - 1) / kStageK * kStageK;
  p.scale_at = kWsHeaderBytes + (size_t)p.blocks * kMaxCols * p.k_pad * 2;
  const int groups = x_dtype != FOVEA_E4M3 ? 0 : by_group ? (in + group - 1) / group : 1;
  p.bytes = p.scale_at + (size_t)p.blocks * kMaxCols * groups * 4;
  return p;
}

template <int NC, int G>
static cudaError_t launch(const CUtensorMap& tmW, const CUtensorMap& tmX, Args& a, cudaStream_t s) {
  auto kern = linear_w4_tc_kernel<NC, G>;
  constexpr int stage = kCodeBytes + 4 * NC * 128;
  const int tile = a.parts > 1 && a.split == 1 ? NC * kRows * 4 : 0;
  const int rest = 1024 + kScaleBytes + kBarBytes + tile;
  a.stages = std::min(kMaxStages, (kSmemBudget - rest) / stage);
  const size_t smem = (size_t)a.stages * stage + rest;
  static std::atomic<unsigned long long> done{0};          // devices whose limit is raised
  const cudaError_t e = raise_smem_limit(kern, 227 * 1024, done);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  const int groups = a.split > 1 ? a.tiles : std::min(a.tiles, 152);
  cfg.gridDim = dim3(groups * a.split);
  cfg.blockDim = dim3(kThreads<NC>);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, tmW, tmX, a);
}

template <int G>
static cudaError_t launch(const CUtensorMap& tmW, const CUtensorMap& tmX, Args& a, cudaStream_t s) {
  return a.cols_pad == 16   ? launch<16, G>(tmW, tmX, a, s)
         : a.cols_pad == 32 ? launch<32, G>(tmW, tmX, a, s)
         : a.cols_pad == 48 ? launch<48, G>(tmW, tmX, a, s)
                            : launch<64, G>(tmW, tmX, a, s);
}

}  // namespace w4tc

size_t linear_w4_tc_workspace(int N, int in, int group, int x_dtype, bool by_group) {
  return w4tc::plan(N, in, group, x_dtype, by_group).bytes;
}

cudaError_t launch_linear_w4_tc(const LinearW4Args& l, cudaStream_t s) {
  using namespace w4tc;
  const bool by_group = l.x_group != 0;
  const Plan p = plan(l.N, l.w.in, l.w.group, l.x_dtype, by_group);
  uint8_t* ws = static_cast<uint8_t*>(l.workspace);
  const int groups = (l.w.in + l.w.group - 1) / l.w.group;
  LayoutArgs x{};
  x.x = l.x; x.ld = l.x_ld; x.dtype = l.x_dtype; x.vec = x_vectors(l.x, l.x_ld, l.x_dtype);
  x.x_scale = l.x_scale; x.x_groups = l.x_scale == nullptr ? 0 : by_group ? groups : 1;
  x.N = l.N; x.in = l.w.in; x.k_pad = p.k_pad;
  x.rows_block = p.rows_block; x.blocks = p.blocks; x.parts = p.parts;
  x.out = reinterpret_cast<__nv_bfloat16*>(ws + kWsHeaderBytes);
  x.scale_out = reinterpret_cast<float*>(ws + p.scale_at);
  x.err = reinterpret_cast<int*>(ws);
  const long long items = (long long)p.blocks * kMaxCols * (p.k_pad / 8 + x.x_groups);
  const int grid = (int)std::min<long long>((items + kLayoutThreads - 1) / kLayoutThreads, 152 * 8);
  cudaError_t e = launch_pdl(layout_x_kernel, dim3(grid), dim3(kLayoutThreads), 0, s, x);
  if (e != cudaSuccess) return e;

  CUtensorMap tmW, tmX;
  if (!encode_byte_map(&tmW, l.w.codes, l.w.out, l.w.in / 2, kRows)) return cudaErrorInvalidValue;
  for (int b = 0; b < p.blocks; ++b) {
    Args a{};
    a.w = l.w;
    a.groups = groups;
    a.n0 = b * p.rows_block;
    a.rows = std::min(p.rows_block, l.N - a.n0);
    a.parts = p.parts;
    a.cols = a.rows * p.parts;
    a.cols_pad = (a.cols + 15) / 16 * 16;                  // the instruction's step
    a.by_group = by_group;
    a.x_scale = x.x_groups == 0 ? nullptr : x.scale_out + (size_t)b * kMaxCols * x.x_groups;
    a.bias = l.bias;
    a.y = l.y; a.y_dtype = l.y_dtype; a.ldy = l.w.out;
    a.ksteps = p.k_pad / kStageK;
    a.tiles = (l.w.out + kRows - 1) / kRows;
    // one tile's contraction over a cluster while the tiles leave SMs idle (us, whole and
    // split: 16 rows by [4096, 4096] 14.1 and 9.2, 64 rows by [4096, 14336] 43.8 and 20.2)
    a.split = 1;
    while (a.split < 8 && a.tiles * a.split * 2 <= 152 && a.split * 2 <= a.ksteps) a.split *= 2;
    a.k128 = kW4One28;
    a.wait_ns = wait_limit_ns();
    a.err = x.err;
    const TmaOperand xop{x.out + (size_t)b * kMaxCols * p.k_pad, a.cols_pad, p.k_pad, p.k_pad};
    if (!encode_kblock_map(&tmX, xop, a.cols_pad, kStageK / 64)) return cudaErrorInvalidValue;
    e = l.w.group == 128 ? launch<128>(tmW, tmX, a, s)
        : l.w.group == 64 ? launch<64>(tmW, tmX, a, s) : launch<32>(tmW, tmX, a, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace fovea
