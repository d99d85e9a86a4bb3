// moe_scaled_product / moe_scaled_swiglu: sorted e4m3 rows with a scale per 128 columns times the experts' e4m3 matrices with a scale per 128 x 128.
//
//   product   out[p, n] = sum_b sx[p, b] sw[e, n / 128, b] sum_{k in block b} x[p, k] w[e, n, k]        (rounded once)
//   swiglu    g, u = products with rows n and I + n of w[e];  a = g / (1 + exp(-g)) u in fp32, quantised per 128 columns to codes and a scale
//
// tcgen05.mma.kind::f8f6f4 knows no scales, so the 128 products of a block are added up in the tensor core, each block in a fresh buffer in TMEM (a partial), and eight
// epilogue warps read every partial and multiply-add it with its two scales into fp32 registers: one multiply-add and four bytes out of TMEM for 128 products.
//
// Forms.  Few rows an expert: weight rows are the M of the instruction, twice 128 TMEM lanes, up to 64 rows its N in steps of 16; one CTA a tile, four partials.  Where such tiles
// are few, four CTAs, a cluster, share a tile's blocks and add up a part of its rows each.  More rows (tall): 128 rows are the M of a CTA and 256 weight rows its N (64 where
// tiles are few; for swiglu the four CTAs that have a block of 128 outputs are a cluster and tell one another their rows' largest magnitudes), or 256 rows that of a pair of CTAs (cta_group::2), each of which holds 128 of either.  A thread then has a row: one multiplier for all of its columns.  The columns are two halves of 128, each
// with buffers and epilogue warps of its own, so that what one half loads and the other adds alternates.
//
// Roles: warps 0-7 epilogue, 8 TMA (one thread; a stage is a block of 128 columns: 128-byte rows, swizzled), 9 MMA (one thread), 10 and 11 bring the products of the two scales, four
// blocks at a time, into a ring in shared memory.
// What bounds them: few rows, the weight stream (100 tokens on 128 experts: gate/up 302 us, 6.2 TB/s; one CTA streams 97 GB/s); many, power and the way of a partial from the tensor core to
// the epilogue and back: 8192 x 4096 x 4096 by itself 130-135 us (2.0-2.1 PFLOP/s, tensor pipe 55 % of the cycles), over and over 143-147 (1.9), 65 536 rows of 64 experts, K 4096, 3584 gate/up rows
// 1 070-1 190 us, K 1792, 4096 columns 580-590, at 1 000 W and 1.46 GHz.  Without loads from TMEM and additions the same launch takes 0.81 of that, without the additions alone 0.84.
// Every wait is bounded (2 s); where one runs out the launch ends, after another such limit for its copies in flight, and what it has not computed is NaN (a scale of NaN).  A warp that gave
// up hands nothing back, so that what others still read stays as it is.
#include <cuda_fp16.h>

#include <type_traits>

#include "moe_dev.cuh"
#include "moe_grouped.cuh"
#include "moe_ptx.cuh"
#include "moe_scaled.cuh"

namespace moe {
namespace {

constexpr int kThreads = 384;
constexpr int kTmaWarp = 8, kMmaWarp = 9, kScaleWarp = 10, kScaleThreads = 64;
constexpr int kBlock = kScaledBlock;
constexpr int kSplit = 4, kSplitRows = 8;       // CTAs that share a tile's blocks, and its most rows
constexpr int kQuad = 4;                        // blocks whose scales are handed over together
constexpr int kQuads = 4;                       // ... of them in the ring
constexpr int kTurnBytes = 32 * 128;            // outputs on their way out: 128 bytes of 32 rows of a warp, swizzled as TMA does

struct Shared : Segments {
  unsigned long long full[8], empty[8], part_full[8], part_empty[8], scales_full[kQuads], scales_empty[kQuads], drained;
  unsigned tmem;
  volatile int dead;             // a wait ran out
  unsigned tops[4][2][128];      // swiglu: largest magnitudes on their way from warp to warp (narrow tiles: from CTA to CTA)
};

enum Form { kFew, kNarrow, kTile, kTilePair };
template <Form kForm, bool kSwiglu>
struct Shape {
  static constexpr bool kTall = kForm != kFew;
  static constexpr int kCtas = kForm == kTilePair ? 2 : 1;
  static constexpr int kRows = kTall ? 128 * kCtas : 64;            // of a tile
  static constexpr int kCols = kForm == kNarrow ? 64 : 256;         // weight rows of a tile; narrow ones for swiglu: of one of the four CTAs that have a block of outputs
  static constexpr bool kQuarter = kForm == kNarrow && kSwiglu;
  // Tall: a half of the columns has 64 of the first 128 weight rows and 64 of the second; where one CTA has them all, and their order is free, its share of them in a row
  static constexpr bool kMixed = kForm == kTilePair || kSwiglu;
  // weight rows and parts (gate, up) of a TMA box, boxes of a stage
  static constexpr int kBoxWeights = kForm == kTilePair ? 128 : !kSwiglu ? kCols : kTall ? kCols / 4 : 128, kBoxParts = kSwiglu && kForm != kTilePair ? 2 : 1;
  static constexpr int kBoxes = (kForm == kTile || kForm == kNarrow) && kSwiglu ? 2 : 1;
  static constexpr int kMine = kRows / kCtas;                       // ... in this CTA
  static constexpr int kWBytes = kCols / kCtas * kBlock, kXBytes = kMine * kBlock, kStageBytes = kWBytes + kXBytes;
  static constexpr int kBoxRows = kTall ? 64 : 32;                  // of a TMA box of rows
  // A partial.  Tall: half of the columns of a block's products, which four of the epilogue's warps read, two or four for each half; else all of them, four.
  static constexpr int kHalves = kTall ? 2 : 1, kHalfCols = kCols / 2;
  static constexpr int kPartCols = kTall ? kHalfCols : 2 * kRows;   // TMEM columns
  static constexpr int kParts = kForm == kNarrow || !kTall ? 4 : 2; // of a half
  static constexpr int kScaleFloats = kQuad * 2 * kMine;            // of a place in the ring: [block][half][row]
  static constexpr int kScaleBytes = kQuads * kScaleFloats * 4;
  static constexpr int kTurns = kForm == kTilePair ? 2 : 1;         // ... of a warp (pairs: four stages are left; one, and five: 588 -> 598 us)
  static constexpr int kOutBytes = kTall && !kSwiglu ? 8 * kTurns * kTurnBytes : 0;
  static constexpr int kStages = (227 * 1024 - 1024 - (int)sizeof(Shared) - kScaleBytes - kOutBytes) / kStageBytes;
  static constexpr int kSmem = 1024 + kStages * kStageBytes + kScaleBytes + kOutBytes + (int)sizeof(Shared);
  static_assert(kStages >= 3 && kStages <= 8 && kHalves * kParts <= 8 && kHalves * kParts * kPartCols <= 512, "barriers, TMEM");
};

struct Args {
  CUtensorMap tm_w;              // [E][parts][rows][K], parts: gate and up for swiglu, else 1
  CUtensorMap tm_x;              // [R][K]
  CUtensorMap tm_out;            // [R][N] as bytes
  const float* x_scales;         // [R, blocks]
  const float* w_scales;         // [E, row_blocks, blocks]
  const int* offsets;            // [E + 1], or NULL: one matrix for all rows
  void* out;                     // [R, N], or codes [R, I]
  float* out_scales;             // swiglu: [R, I / 128]
  int R, E, N, I;                // N: weight rows; I: N / 2 for swiglu
  int blocks, row_blocks;
  int dtype, wide;               // of out; its rows are 16-byte aligned
  int by_tma;                    // tm_out is there
  int wide_scales;               // four scales of a row can be loaded at once
  int split;                     // kSplit: so many CTAs, a cluster, share the blocks of a tile; else 1
};

// e4m3 operands, fp32 sums, both K-major, M rows, N columns
__device__ __forceinline__ unsigned idesc_of(unsigned m, unsigned n) { return 1u << 4 | (n >> 3) << 17 | (m >> 4) << 24; }
// one block: four products of 32 columns into fresh sums
template <bool kPair>
__device__ __forceinline__ void mma_block(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc) {
  if (kPair)
    asm volatile(
        "{\n\t.reg .pred p0, p1;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "setp.ne.b32 p0, 0, 0;\n\tsetp.eq.b32 p1, 0, 0;\n\t"
        "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a1, b1, %3, p1;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a2, b2, %3, p1;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a3, b3, %3, p1;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p0, p1;\n\t.reg .b64 a1, a2, a3, b1, b2, b3;\n\t"
        "setp.ne.b32 p0, 0, 0;\n\tsetp.eq.b32 p1, 0, 0;\n\t"
        "add.u64 a1, %1, 2;\n\tadd.u64 a2, %1, 4;\n\tadd.u64 a3, %1, 6;\n\t"
        "add.u64 b1, %2, 2;\n\tadd.u64 b2, %2, 4;\n\tadd.u64 b3, %2, 6;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a1, b1, %3, p1;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a2, b2, %3, p1;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a3, b3, %3, p1;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc)
        : "memory");
}
template <bool kPair>
__device__ __forceinline__ void tma_4d(unsigned dst, const CUtensorMap* m, int x, int y, int z, int w, unsigned bar, unsigned long long policy) {
  if (kPair)
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
        "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "l"(policy)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(dst),
        "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar), "l"(policy)
        : "memory");
}
__device__ __forceinline__ float4 ld_shared_f4(unsigned saddr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(saddr) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_shared16(unsigned saddr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(saddr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared16(unsigned saddr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(saddr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ float ld_shared_f(unsigned saddr) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(saddr) : "memory");
  return v;
}
__device__ __forceinline__ void st_shared_f(unsigned saddr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(saddr), "f"(v) : "memory"); }
// the same place of shared memory in another CTA of the cluster
__device__ __forceinline__ unsigned map_address(unsigned saddr, unsigned rank) {
  unsigned r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
// all threads of a cluster; a warp's together
__device__ __forceinline__ void meet() {
  __syncwarp();
  cluster_sync_all();
}
__device__ __forceinline__ void st_cluster_f(unsigned cluster_addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u(unsigned cluster_addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ bool try_at(unsigned saddr, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(saddr), "r"(parity)
      : "memory");
  return ok != 0;
}
// whether the phase is over; the answer is not waited for before it is used
__device__ __forceinline__ bool test_at(unsigned saddr, unsigned parity) {
  unsigned ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(saddr), "r"(parity)
      : "memory");
  return ok != 0;
}
// 128 bytes of 32 rows out of shared memory; the thread that asks is the one that waits
__device__ __forceinline__ void tma_store(const CUtensorMap* m, int x, int y, unsigned from) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(from)
               : "memory");
  asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// all but the last kLeft of this thread's have been read from shared memory
template <int kLeft>
__device__ __forceinline__ void tma_stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(kLeft) : "memory"); }
__device__ __forceinline__ void tma_stores_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// what a wait was for cannot be used before it
__device__ __forceinline__ void loaded(unsigned (&r)[16]) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]),
               "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
}
__device__ __forceinline__ void loaded(unsigned (&r)[32]) {
  loaded(reinterpret_cast<unsigned(&)[16]>(r[0]));
  loaded(reinterpret_cast<unsigned(&)[16]>(r[16]));
}
// The same wait for a whole warp, of which all lanes get the same answer; short where the barrier's phase is over.
__device__ __noinline__ bool wait_longer(unsigned saddr, unsigned parity, volatile int* dead) {
  const unsigned long long start = gtime_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (__all_sync(0xffffffffu, try_at(saddr, parity))) return true;
    if (__any_sync(0xffffffffu, *dead)) return false;
    if (__any_sync(0xffffffffu, gtime_ns() - start > kWaitNs)) {
      *dead = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool warp_wait(unsigned saddr, unsigned parity, volatile int* dead) {
  return __all_sync(0xffffffffu, try_at(saddr, parity)) || wait_longer(saddr, parity, dead);
}
__device__ __forceinline__ void bar_sync(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

template <class E> __device__ __forceinline__ E rounded(float v);
template <> __device__ __forceinline__ float rounded(float v) { return v; }
template <> __device__ __forceinline__ __half rounded(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rounded(float v) { return __float2bfloat16_rn(v); }
// f with a pointer of the outputs' type
template <class F>
__device__ __forceinline__ void with_type(int dtype, void* out, F f) {
  if (dtype == MOE_DTYPE_BF16) f(static_cast<__nv_bfloat16*>(out));
  else if (dtype == MOE_DTYPE_FP16) f(static_cast<__half*>(out));
  else f(static_cast<float*>(out));
}

template <Form kForm, bool kSwiglu>
__global__ void __launch_bounds__(kThreads, 1) scaled_product_kernel(const __grid_constant__ Args a) {
  using S = Shape<kForm, kSwiglu>;
  constexpr bool kTall = S::kTall, kPair = kForm == kTilePair;
  extern __shared__ unsigned char raw[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  float* ring = reinterpret_cast<float*>(stages + S::kStages * S::kStageBytes);
  unsigned char* turned = reinterpret_cast<unsigned char*>(ring) + S::kScaleBytes;
  Shared& s = *reinterpret_cast<Shared*>(turned + S::kOutBytes);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  constexpr int kStep = kSwiglu ? 128 : S::kCols;                  // output columns of a tile
  const unsigned rank = kPair ? cluster_ctarank() : 0u;
  // Few tiles of a few rows: the CTAs of a cluster have a part of the blocks each (b_first to b_last), and at the end a part of the rows, which they add up.  A cluster
  // has one tile at most.
  const int split = kForm == kFew ? a.split : 1, part_of = S::kQuarter || (kForm == kFew && split > 1) ? (int)cluster_ctarank() : 0;
  const int b_first = S::kQuarter ? 0 : part_of * a.blocks / split, b_last = S::kQuarter ? a.blocks : (part_of + 1) * a.blocks / split;
  const bool meets = S::kQuarter || (kForm == kFew && split > 1);      // twice, at the end of the tile
  const int ctas = S::kQuarter ? kSplit : kForm == kFew ? split : S::kCtas, unit = (int)blockIdx.x / ctas, n_units = (int)gridDim.x / ctas;
  const int n_blocks = ((kSwiglu ? a.I : a.N) + kStep - 1) / kStep;

  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&s.full[i], S::kCtas);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < S::kHalves * S::kParts; ++i) {
      mbar_init(&s.part_full[i], 1);
      mbar_init(&s.part_empty[i], 8 / S::kHalves * S::kCtas);
    }
    for (int i = 0; i < kQuads; ++i) {
      mbar_init(&s.scales_full[i], kScaleThreads / 32);
      mbar_init(&s.scales_empty[i], 8);
    }
    mbar_init(&s.drained, 1);
    s.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_proxy_smem();
  }
  if (warp == kMmaWarp) {
    if (kPair) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s.tmem)) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  grid_dep_wait();
#pragma unroll 1
  for (int e = tid; e <= a.E; e += kThreads) s.first_row[e] = a.offsets ? min(max(a.offsets[e], 0), a.R) : e ? a.R : 0;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) list_tiles<S::kRows>(s, a.E, n_blocks, lane);
  __syncthreads();
  if (kPair) cluster_sync_all();          // the other CTA's barriers exist before anything arrives on them
  const unsigned tmem = s.tmem;
  const int n_tiles = uniform(s.first_tile[a.E]);

  if (warp < kTmaWarp) {
    if (kTall) asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    const int quarter = warp & 3, half = warp >> 2;
    const unsigned lanes = tmem + ((unsigned)quarter << 21);       // this warp's 32 TMEM lanes
    const unsigned first = kTall ? S::kParts * half : 0;            // buffer of this warp's partials
    const unsigned full0 = smem_u32(&s.part_full[first]), empty0 = kPair ? map_to_cta(&s.part_empty[first], 0) : smem_u32(&s.part_empty[first]);
    const unsigned ring0 = smem_u32(ring), ring_full = smem_u32(&s.scales_full[0]);
    unsigned part = 0, place = 0;  // partials, places in the ring so far
    unsigned turn = 0;             // exchanges of maxima so far
    bool met = false;              // the cluster has had its two meetings
    bool ok = true;
    const auto next_partial = [&] {                                 // -> its address
      const unsigned buf = part % S::kParts;
      if (ok) ok = warp_wait(full0 + 8 * buf, (part / S::kParts) & 1, &s.dead);
      tc_fence_after();
      return lanes + (first + buf) * S::kPartCols;
    };
    // What a warp waited for in vain it does not give back: others may still read it.
    const auto hand_back = [&] {                                    // the warp has what it loads of the partial
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_relaxed(empty0 + 8 * (part % S::kParts));
      ++part;
    };
    const auto next_scales = [&] {                                  // -> address of four blocks' scales: [block][half][row]
      const unsigned at = place % kQuads;
      if (ok) ok = warp_wait(ring_full + 8 * at, (place / kQuads) & 1, &s.dead);
      return ring0 + at * (S::kScaleFloats * 4);
    };
    const auto scales_read = [&] {
      __syncwarp();
      if (lane == 0) mbar_arrive(&s.scales_empty[place % kQuads]);
      ++place;
    };
    for (int t = unit; t < n_tiles; t += n_units) {
      const Tile at = uniform(tile_at<S::kRows>(s, a.E, t, kStep));
      if constexpr (kTall) {
        const int mine = 32 * quarter + lane, row = 128 * (int)rank + mine;
        const bool used = uniform(128 * (int)rank + 32 * quarter) < at.rows, valid = row < at.rows;
        // Pairs of neighbouring columns, of this half.  kMixed: 0-63 are of the first 128 weight rows (swiglu: gate rows), 64-127 of the second (up rows)
        unsigned long long sum[S::kHalfCols / 2];
#pragma unroll
        for (int i = 0; i < S::kHalfCols / 2; ++i) sum[i] = 0ull;
        if (!used) {               // (no row of the tile: the hand-overs alone)
#pragma unroll 1
          for (int b = 0; b < a.blocks && ok; ++b) {
            if (b % kQuad == 0) {
              next_scales();
              if (ok) scales_read();
            }
            next_partial();
            if (ok) hand_back();
          }
          if (S::kQuarter) {
            meet();
            meet();
            met = true;
          } else if (kSwiglu) {
            ++turn;
            bar_sync(1 + quarter, 64);
          }
          continue;
        }
        if constexpr (S::kHalfCols == 32) {
          // the next block's columns are on their way while one's are added
          unsigned v[2][32];
          unsigned sc = next_scales() + 4 * mine, from = next_partial();
          if (ok) tc_ld32(from, v[0]);
#pragma unroll 1
          for (int b0 = 0; b0 < a.blocks && ok; b0 += 2)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              const int b = b0 + u;
              if (b >= a.blocks) break;
              const float m0 = ld_shared_f(sc), m1 = kSwiglu ? ld_shared_f(sc + 4 * S::kMine) : m0;
              sc += 8 * S::kMine;
              const bool more = b < a.blocks - 1;
              tc_wait_ld();
              loaded(v[u]);
              hand_back();
              if (b % kQuad == kQuad - 1 || !more) {
                scales_read();
                if (more) sc = next_scales() + 4 * mine;
              }
              if (more) {
                from = next_partial();
                if (!ok) break;
                tc_ld32(from, v[u ^ 1]);
              }
              const unsigned long long s0 = f32x2(m0, m0), s1 = f32x2(m1, m1);
#pragma unroll
              for (int j = 0; j < 16; ++j) sum[j] = fma_f32x2(f32x2(__uint_as_float(v[u][2 * j]), __uint_as_float(v[u][2 * j + 1])), j < 8 ? s0 : s1, sum[j]);
            }
        } else {
          // 64 columns are on their way or being added at any time: a wait is for all loads before it, so there are two a block, and the next block's first
          // loads go out between this one's last additions.  (Five waits a block, 16 and 32 columns at a time: gate/up of 65 536 rows 2 490 us for 2 120.)
          unsigned v[2][32];
          const auto add = [&](int c, unsigned long long m) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              sum[16 * c + j] = fma_f32x2(f32x2(__uint_as_float(v[c & 1][2 * j]), __uint_as_float(v[c & 1][2 * j + 1])), m, sum[16 * c + j]);
          };
          unsigned sc = next_scales() + 4 * mine, from = next_partial();
          if (ok) {
            tc_ld32(from, v[0]);
            tc_ld32(from + 32, v[1]);
          }
#pragma unroll 1
          for (int b = 0; b < a.blocks && ok; ++b) {
            const float m0 = ld_shared_f(sc + (S::kMixed ? 0 : half * 4 * S::kMine)), m1 = S::kMixed ? ld_shared_f(sc + 4 * S::kMine) : m0;
            sc += 8 * S::kMine;
            const unsigned long long s0 = f32x2(m0, m0), s1 = f32x2(m1, m1);
            const bool more = b < a.blocks - 1;
            tc_wait_ld();
            loaded(v[0]);
            loaded(v[1]);
            add(0, s0);
            tc_ld32(from + 64, v[0]);
            add(1, s0);
            tc_ld32(from + 96, v[1]);
            if (b % kQuad == kQuad - 1 || !more) {
              scales_read();
              if (more) sc = next_scales() + 4 * mine;
            }
            tc_wait_ld();
            loaded(v[0]);
            loaded(v[1]);
            hand_back();
            add(2, s1);
            if (more) {
              from = next_partial();
              if (!ok) break;
              tc_ld32(from, v[0]);
            }
            add(3, s1);
            if (more) tc_ld32(from + 32, v[1]);
          }
        }
        const size_t p = (size_t)at.row0 + row;
        float acc[S::kHalfCols];
#pragma unroll
        for (int i = 0; i < S::kHalfCols / 2; ++i) {
          const float2 two = f32x2_parts(sum[i]);
          acc[2 * i] = two.x;
          acc[2 * i + 1] = two.y;
        }
        if constexpr (kSwiglu) {
          constexpr int kOuts = S::kHalfCols / 2;
          unsigned top = 0u;
#pragma unroll
          for (int i = 0; i < kOuts; ++i) {
            acc[i] = silu_times(acc[i], acc[kOuts + i]);
            top = max(top, __float_as_uint(acc[i]) & 0x7fffffffu);
          }
          if (!ok) top = 0x7fffffffu;        // (of the whole block, whoever else has its sums: its scale is NaN)
          if constexpr (S::kQuarter) {       // the row's other outputs are with the other half, and with three other CTAs, which are known to run once they have met
            meet();
#pragma unroll
            for (int to = 0; to < kSplit; ++to) st_cluster_u(map_address(smem_u32(&s.tops[part_of][half][mine]), to), top);
            meet();
            met = true;
#pragma unroll
            for (int i = 0; i < 2 * kSplit; ++i) top = max(top, s.tops[i / 2][i % 2][mine]);
          } else {
            s.tops[turn & 1][half][mine] = top;
            bar_sync(1 + quarter, 64);
            top = max(top, s.tops[turn++ & 1][half ^ 1][mine]);
          }
          const float scale = scaled_scale(top), inv = __fdividef(1.f, scale);
          if (valid) {
            uint4* to = reinterpret_cast<uint4*>(static_cast<unsigned char*>(a.out) + p * a.I + at.n0 + (S::kQuarter ? 32 * part_of : 0) + kOuts * half);
#pragma unroll
            for (int i = 0; i < kOuts; ++i) acc[i] *= inv;
#pragma unroll
            for (int i = 0; i < kOuts / 16; ++i)
              to[i] = make_uint4(e4m3_codes4(acc + 16 * i), e4m3_codes4(acc + 16 * i + 4), e4m3_codes4(acc + 16 * i + 8), e4m3_codes4(acc + 16 * i + 12));
            if (half == 0 && (!S::kQuarter || part_of == 0)) a.out_scales[p * (a.I / kBlock) + at.n0 / kBlock] = scale;
          }
        } else {
          if (!ok) {
#pragma unroll
            for (int i = 0; i < S::kHalfCols; ++i) acc[i] = __uint_as_float(0x7fffffffu);
          }
          // A warp turns its 32 rows round in shared memory, 128 bytes of each at a time.  Where all 32 are the tile's, TMA takes them from there while the next tile's
          // sums begin (down product of 65 536 rows, K 1792, over and over 587 us; all stored by the warps 615); else the warp stores 128 bytes of four rows at a time.
          const unsigned own = smem_u32(turned + warp * S::kTurns * kTurnBytes);
          const int row_out = at.row0 + 128 * (int)rank + 32 * quarter, rows = min(32, at.rows - 128 * (int)rank - 32 * quarter);
          const bool by_tma = kForm != kNarrow && a.by_tma && rows == 32;
          with_type(a.dtype, a.out, [&](auto* out) {
            using E = typename std::remove_pointer<decltype(out)>::type;
            constexpr int kIn = 16 / (int)sizeof(E), kCols = S::kHalfCols < 128 / (int)sizeof(E) ? S::kHalfCols : 128 / (int)sizeof(E);
            constexpr int kPieces = kCols / kIn;           // 16-byte pieces of a row at a time
            out += (size_t)row_out * a.N;
#pragma unroll
            for (int c = 0; c < S::kHalfCols / kCols; ++c) {
              const int col0 = at.n0 + (S::kMixed ? 128 * (c * kCols / 64) + 64 * half + c * kCols % 64 : S::kHalfCols * half + c * kCols), cols = min(kCols, a.N - col0);
              if (cols <= 0) break;                        // (so that every pass so far has had its store, which the waits count)
              const unsigned turn_at = own + c % S::kTurns * kTurnBytes;
              const auto piece = [&](int r, int i) { return turn_at + 128 * r + 16 * (i ^ (r & 7)); };
              // Nothing of an earlier store is read from there any more: of the tile before all of them, which frees every place; then the one whose place comes again.
              if (kForm != kNarrow && (c == 0 || c >= S::kTurns)) {
                if (lane == 0) {
                  if (c == 0) tma_stores_read<0>();
                  else tma_stores_read<S::kTurns - 1>();
                }
                __syncwarp();
              }
#pragma unroll
              for (int i = 0; i < kPieces; ++i) {
                uint4 v;
#pragma unroll
                for (int j = 0; j < kIn; ++j) reinterpret_cast<E*>(&v)[j] = rounded<E>(acc[c * kCols + i * kIn + j]);
                st_shared16(piece(lane, i), v);
              }
              if (by_tma) {
                fence_async_proxy_smem();
                __syncwarp();
                if (lane == 0) tma_store(&a.tm_out, col0 * (int)sizeof(E), row_out, turn_at);
                continue;
              }
              __syncwarp();
              if (a.wide) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                  const int r = 32 / kPieces * i + lane / kPieces, at_col = lane % kPieces * kIn;
                  const uint4 v = ld_shared16(piece(r, lane % kPieces));
                  if (r < rows && at_col < cols) *reinterpret_cast<uint4*>(out + (size_t)r * a.N + col0 + at_col) = v;
                }
              } else {
                // an element a lane, eight rows' at once on their way
                const unsigned char* from = turned + (turn_at - smem_u32(turned));
                constexpr int kLanePieces = 32 / kIn;      // piece (lane / kIn + kLanePieces h) ^ r % 8
                int own_at[kLanePieces];
#pragma unroll
                for (int j = 0; j < kLanePieces; ++j) own_at[j] = 16 * ((lane / kIn) ^ j) + (lane % kIn) * (int)sizeof(E);
                E* to = out + col0 + lane;
#pragma unroll 1
                for (int r = 0; r < rows; r += 8, from += 8 * 128, to += 8 * (size_t)a.N) {
                  E v[8][kCols / 32];
#pragma unroll
                  for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int h = 0; h < kCols / 32; ++h)
                      v[i][h] = *reinterpret_cast<const E*>(from + 128 * i + own_at[i % kLanePieces] + 16 * kLanePieces * (h ^ i / kLanePieces));
#pragma unroll
                  for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int h = 0; h < kCols / 32; ++h)
                      if (r + i < rows && lane + 32 * h < cols) to[(size_t)i * a.N + 32 * h] = v[i][h];
                }
              }
              __syncwarp();
            }
          });
        }
      } else {
        // groups of 16 rows; plain: all of them, of the 128 weight rows of this half; swiglu: every other, gate and up
        const int groups = uniform((at.rows + 15) / 16);
        constexpr int kGroups = kSwiglu ? 2 : 4;
        const auto group = [&](int i) { return kSwiglu ? half + 2 * i : i; };
        float acc[kGroups][kSwiglu ? 2 : 1][16];
#pragma unroll
        for (int i = 0; i < kGroups; ++i)
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            acc[i][0][j] = 0.f;
            if (kSwiglu) acc[i][kSwiglu ? 1 : 0][j] = 0.f;
          }
#pragma unroll 1
        for (int b0 = b_first; b0 < b_last && ok; b0 += kQuad) {
          unsigned sc = next_scales();
#pragma unroll 1
          for (int b = b0; b < min(b0 + kQuad, b_last); ++b, sc += 8 * S::kMine) {
            const unsigned from = next_partial();
            if (!ok) break;
            unsigned p[kGroups][kSwiglu ? 2 : 1][16];
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
              if (group(i) < groups) {
                tc_ld16(from + (kSwiglu ? 0 : half * S::kRows) + 16 * group(i), p[i][0]);
                if (kSwiglu) tc_ld16(from + S::kRows + 16 * group(i), p[i][kSwiglu ? 1 : 0]);
              }
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
              loaded(p[i][0]);
              if (kSwiglu) loaded(p[i][kSwiglu ? 1 : 0]);
            }
            hand_back();
#pragma unroll
            for (int i = 0; i < kGroups; ++i)
              if (group(i) < groups) {
#pragma unroll
                for (int h = 0; h < (kSwiglu ? 2 : 1); ++h)
#pragma unroll
                  for (int j = 0; j < 16; j += 4) {
                    const float4 m = ld_shared_f4(sc + 4 * ((kSwiglu ? h : half) * S::kMine + 16 * group(i) + j));
                    acc[i][h][j] = fmaf(__uint_as_float(p[i][h][j]), m.x, acc[i][h][j]);
                    acc[i][h][j + 1] = fmaf(__uint_as_float(p[i][h][j + 1]), m.y, acc[i][h][j + 1]);
                    acc[i][h][j + 2] = fmaf(__uint_as_float(p[i][h][j + 2]), m.z, acc[i][h][j + 2]);
                    acc[i][h][j + 3] = fmaf(__uint_as_float(p[i][h][j + 3]), m.w, acc[i][h][j + 3]);
                  }
              }
          }
          if (ok) scales_read();
        }
        const int n = at.n0 + (kSwiglu ? 0 : 128 * half) + 32 * quarter + lane;
        // row r of the tile is this CTA's: the one of the cluster whose turn it is
        const auto is_mine = [&](int r) { return r < at.rows && (r & (split - 1)) == part_of; };
        if (split > 1) {
          // Sums of the others' rows to their shared memory, [from][row / kSplit][256 weight rows], over the stages, which nobody uses any more; then added in order.
          meet();
          const unsigned at_lane = smem_u32(stages) + 4 * (32 * quarter + lane);
          constexpr int kEach = kSplitRows / kSplit;
          const auto all = [&](auto f) {
            if (group(0) != 0) return;
#pragma unroll
            for (int r = 0; r < kSplitRows; ++r)
              if (r < at.rows)
#pragma unroll
                for (int h = 0; h < (kSwiglu ? 2 : 1); ++h) f(r, kSwiglu ? h : half, acc[0][h][r]);
          };
          all([&](int r, int h, float& v) {
            if (!ok) v = __uint_as_float(0x7fffffffu);
            if (!is_mine(r)) st_cluster_f(map_address(at_lane + 4 * ((part_of * kEach + r / kSplit) * 256 + 128 * h), r % kSplit), v);
          });
          meet();
          all([&](int r, int h, float& v) {
            if (is_mine(r)) {
              const float own = v;
              v = 0.f;
#pragma unroll
              for (int from = 0; from < kSplit; ++from)
                v += from == part_of ? own : ld_shared_f(at_lane + 4 * ((from * kEach + r / kSplit) * 256 + 128 * h));
            }
          });
          met = true;
        }
        if constexpr (kSwiglu) {
#pragma unroll
          for (int i = 0; i < kGroups; ++i) {
            if (group(i) >= groups) break;
            unsigned mine = 0u;    // lane j < 16: of row j of the group
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              acc[i][0][j] = silu_times(acc[i][0][j], acc[i][kSwiglu ? 1 : 0][j]);
              const unsigned top = __reduce_max_sync(0xffffffffu, __float_as_uint(acc[i][0][j]) & 0x7fffffffu);
              if (lane == j) mine = top;
            }
            if (!ok) mine = 0x7fffffffu;
            unsigned* tops = s.tops[turn++ & 1][half];
            if (lane < 16) tops[16 * quarter + lane] = mine;
            bar_sync(1 + half, 128);
#pragma unroll
            for (int q = 0; q < 4; ++q) mine = max(mine, tops[16 * q + (lane & 15)]);
            const float scale = scaled_scale(mine), inv = __fdividef(1.f, scale);
            const int row = 16 * group(i);
            if (quarter == 0 && lane < 16 && is_mine(row + lane))
              a.out_scales[((size_t)at.row0 + row + lane) * (a.I / kBlock) + at.n0 / kBlock] = scale;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const unsigned code = e4m3_codes2(acc[i][0][j] * __shfl_sync(0xffffffffu, inv, j), 0.f) & 0xffu;
              if (is_mine(row + j)) static_cast<unsigned char*>(a.out)[((size_t)at.row0 + row + j) * a.I + n] = (unsigned char)code;
            }
          }
        } else {
          with_type(a.dtype, a.out, [&](auto* out) {
            using E = typename std::remove_pointer<decltype(out)>::type;
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
              if (i >= groups) break;
#pragma unroll
              for (int j = 0; j < 16; ++j)
                if (is_mine(16 * i + j) && n < a.N)
                  out[((size_t)at.row0 + 16 * i + j) * a.N + n] = rounded<E>(ok ? acc[i][0][j] : __uint_as_float(0x7fffffffu));
            }
          });
        }
      }
    }
    if (kTall && !kSwiglu && kForm != kNarrow && lane == 0) tma_stores_done();
    if (meets && !met) {             // (no tile)
      meet();
      meet();
    }
    // rows that belong to no expert: zeros (scales 1), by the epilogue warps of the whole grid
    const int lo = s.first_row[0], hi = s.first_row[a.E], none = lo + (a.R - hi);
    for (int i = blockIdx.x; i < none; i += gridDim.x) {
      const size_t p = (size_t)(i < lo ? i : hi + (i - lo));
      if (kSwiglu) {
#pragma unroll 1
        for (int c = tid; c < a.I; c += 256) {
          static_cast<unsigned char*>(a.out)[p * a.I + c] = 0;
          if (c < a.I / kBlock) a.out_scales[p * (a.I / kBlock) + c] = 1.f;
        }
      } else {
        with_type(a.dtype, a.out, [&](auto* out) {
          using E = typename std::remove_pointer<decltype(out)>::type;
#pragma unroll 1
          for (int c = tid; c < a.N; c += 256) out[p * a.N + c] = rounded<E>(0.f);
        });
      }
    }
  } else {
    if (kTall) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == kTmaWarp) {
      if (elect_one()) {
        unsigned n = 0;            // stages so far
        for (int t = unit; t < n_tiles && !s.dead; t += n_units) {
          const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
          const int row0 = at.row0 + (int)rank * S::kMine, mine = min(S::kMine, at.rows - (int)rank * S::kMine);
          const int boxes = mine > 0 ? (mine + S::kBoxRows - 1) / S::kBoxRows : 0;
          const unsigned long long policy = at.alone ? l2_evict_first() : l2_evict_normal();
          const int n0 = at.n0 + (S::kQuarter ? 32 * part_of : kSwiglu ? 0 : 128 * (int)rank), which = kSwiglu ? (int)rank : 0;      // (rank is 0 where there is no pair)
#pragma unroll 1
          for (int i = b_first; i < b_last; ++i, ++n) {
            const unsigned slot = n % S::kStages, round = n / S::kStages;
            if (round && !wait(&s.empty[slot], (round - 1) & 1, &s.dead)) break;
            const unsigned to = smem_u32(stages + slot * S::kStageBytes);
            const unsigned bar = kPair ? map_to_cta(&s.full[slot], 0) : smem_u32(&s.full[slot]);
            expect_tx(bar, S::kWBytes + boxes * S::kBoxRows * kBlock);
#pragma unroll
            for (int x = 0; x < S::kBoxes; ++x)
              tma_4d<kPair>(to + x * (S::kWBytes / S::kBoxes), &a.tm_w, i * kBlock, n0 + x * S::kBoxWeights, which, at.expert, bar, policy);
#pragma unroll 1
            for (int x = 0; x < boxes; ++x)
              tma_2d<kPair>(to + S::kWBytes + x * S::kBoxRows * kBlock, &a.tm_x, i * kBlock, row0 + x * S::kBoxRows, bar);
          }
        }
        // The block's shared memory belongs to its copies until they have landed, and where another role has given up nobody else waits for the last ones.
        // The second CTA of a pair, whose copies count on the leader's barriers, sees its own by the stages that the MMAs are done with (or runs into the limit).
        const unsigned long long start = gtime_ns();
#pragma unroll 1
        for (unsigned m = n > S::kStages ? n - S::kStages : 0; m < n; ++m) {
          unsigned long long* bar = rank ? &s.empty[m % S::kStages] : &s.full[m % S::kStages];
          while (!mbar_try(bar, (m / S::kStages) & 1) && gtime_ns() - start < kWaitNs) {}
        }
      }
      __syncwarp();
    } else if (warp == kMmaWarp) {
      if (rank == 0 && elect_one()) {
        const auto commit = [](unsigned long long* bar) {
          if (kPair) tc_commit_pair(bar);
          else tc_commit(bar);
        };
        // Small tiles: the barriers of the next block are asked while this one's products are issued, and the answers read when their turn has come; waiting for each in its place takes
        // some hundred clocks a barrier (16 rows of 4096 x 4096 14.7 us for 11.5).  Where the next buffer is never back that early, asking costs 2-3 %.  (Single CTAs alone.)
        // (A pair's hand-backs are relaxed arrivals: what they order, the tcgen05 fences on both sides do.)
        const auto hand_back_of = [&](unsigned n, int h) { return smem_u32(&s.part_empty[n % S::kParts + S::kParts * h]); };
        constexpr bool kAsk = kForm == kNarrow;
        unsigned slot = 0, parity = 0;                   // of the stage
        bool full = false, empty[S::kHalves] = {}, ok = true;      // known to have come
        unsigned n = 0;            // blocks so far
        for (int t = unit; t < n_tiles && ok; t += n_units) {
          const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
          const unsigned idesc = kTall ? idesc_of(128 * S::kCtas, S::kHalfCols) : idesc_of(128, (unsigned)(at.rows + 15) & ~15u);
#pragma unroll 1
          for (int i = b_first; i < b_last; ++i, ++n) {
            const unsigned st = smem_u32(stages + slot * S::kStageBytes), buf = n % S::kParts;
            const unsigned next_slot = slot + 1 == S::kStages ? 0u : slot + 1, next_parity = parity ^ (next_slot == 0);
#pragma unroll
            for (int h = 0; h < S::kHalves; ++h) {
              if (n >= S::kParts && !empty[h])
                ok = ok && wait<kPair ? mbar_try_relaxed : mbar_try>(&s.part_empty[buf + S::kParts * h], (n / S::kParts - 1) & 1, &s.dead);
              if (h == 0 && !full) ok = ok && wait(&s.full[slot], parity, &s.dead);
              if (!ok) break;
              tc_fence_after();
              if (kAsk && h == 0) full = test_at(smem_u32(&s.full[next_slot]), next_parity);
              if (kAsk) empty[h] = n + 1 >= S::kParts && test_at(hand_back_of(n + 1, h), ((n + 1) / S::kParts - 1) & 1);
              const unsigned d = tmem + (buf + S::kParts * h) * S::kPartCols;
              if (kTall) {
                mma_block<kPair>(d, umma_desc(st + S::kWBytes, 128), umma_desc(st + h * (S::kWBytes / 2), 128), idesc);
              } else {
                mma_block<kPair>(d, umma_desc(st, 128), umma_desc(st + S::kWBytes, 128), idesc);
                mma_block<kPair>(d + S::kRows, umma_desc(st + 128 * kBlock, 128), umma_desc(st + S::kWBytes, 128), idesc);
              }
              if (h == S::kHalves - 1) commit(&s.empty[slot]);
              commit(&s.part_full[buf + S::kParts * h]);
            }
            if (!ok) break;
            slot = next_slot;
            parity = next_parity;
          }
        }
        commit(&s.drained);     // nothing of this block's is left in the tensor core when it frees its TMEM
        const unsigned long long start = gtime_ns();
        while (!mbar_try(&s.drained, 0) && gtime_ns() - start < kWaitNs) {}
      }
      __syncwarp();
    } else {
      // A thread has one row of the tile (few rows) or two: it loads four blocks' scales and those of both halves' weights, and stores the products.
      constexpr int kOwn = S::kMine / kScaleThreads;
      const int r0 = tid - 32 * kScaleWarp;
      unsigned place = 0;
      const auto four = [&](const float* p, int left, float (&v)[4]) {
        if (a.wide_scales) {
          const float4 q = __ldg(reinterpret_cast<const float4*>(p));
          v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = i < left ? __ldg(p + i) : 0.f;
        }
      };
      bool ok = true;
      for (int t = unit; t < n_tiles && ok; t += n_units) {
        const Tile at = uniform(tile_at<S::kRows>(s, a.E, t, kStep));
        const float* w0 = a.w_scales + ((size_t)at.expert * a.row_blocks + at.n0 / kBlock) * a.blocks;
        const int second = kSwiglu ? a.I / kBlock : S::kCols > kBlock && at.n0 / kBlock + 1 < a.row_blocks ? 1 : 0;      // (a half behind the last row: any scale, nothing of it is stored)
        const float* w1 = w0 + (size_t)second * a.blocks;
        const float* x[kOwn];
#pragma unroll
        for (int q = 0; q < kOwn; ++q)
          x[q] = a.x_scales + ((size_t)at.row0 + min((int)rank * S::kMine + r0 + q * kScaleThreads, at.rows - 1)) * a.blocks;
#pragma unroll 1
        for (int b = b_first; b < b_last; b += kQuad, ++place) {
          float u[kOwn][4], v0[4], v1[4];
          four(w0 + b, b_last - b, v0);
          four(w1 + b, b_last - b, v1);
#pragma unroll
          for (int q = 0; q < kOwn; ++q) four(x[q] + b, b_last - b, u[q]);
          const unsigned slot = place % kQuads, round = place / kQuads;
          if (round) ok = __all_sync(0xffffffffu, wait(&s.scales_empty[slot], (round - 1) & 1, &s.dead));
          if (!ok) break;
          const unsigned to = smem_u32(ring + slot * S::kScaleFloats + r0);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < kOwn; ++q) {
              st_shared_f(to + 4 * (2 * i * S::kMine + q * kScaleThreads), u[q][i] * v0[i]);
              st_shared_f(to + 4 * ((2 * i + 1) * S::kMine + q * kScaleThreads), u[q][i] * v1[i]);
            }
          __syncwarp();
          if (lane == 0) mbar_arrive(&s.scales_full[slot]);
        }
      }
    }
    if (meets) {
      meet();
      meet();
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (kPair) cluster_sync_all();          // no CTA leaves while the other may still signal its barriers, or read its shared memory
  if (warp == kMmaWarp) {
    tc_fence_after();
    if (kPair) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

// codes as bytes [e][parts][rows][cols], boxes of 128 bytes x box_rows rows x box_parts
bool encode(CUtensorMap* out, const void* base, long long cols, int rows, int parts, int e, int box_rows, int box_parts) {
  const EncodeFn fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)parts, (cuuint64_t)e};
  const cuuint64_t strides[3] = {(cuuint64_t)cols, (cuuint64_t)cols * rows, (cuuint64_t)cols * rows * parts};
  const cuuint32_t box[4] = {128u, (cuuint32_t)box_rows, (cuuint32_t)box_parts, 1u}, one[4] = {1u, 1u, 1u, 1u};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, parts ? 4 : 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// most tiles that the rows can make
long long most_tiles(const Args& a, int rows, int cols, int step) {
  return (a.R + (long long)(a.R < a.E ? a.R : a.E) * (rows - 1)) / rows * (((long long)cols + step - 1) / step);
}

template <Form kForm, bool kSwiglu>
cudaError_t product_launch(Args& a, const void* codes, const void* w_codes, int K, int sms, cudaStream_t stream) {
  using S = Shape<kForm, kSwiglu>;
  static_assert(S::kSmem <= 227 * 1024, "shared memory");
  const int parts = kSwiglu ? 2 : 1;
  if (!encode(&a.tm_w, w_codes, K, a.N / parts, parts, a.E, S::kBoxWeights, S::kBoxParts) ||
      !encode(&a.tm_x, codes, K, a.R, 0, 0, S::kBoxRows, 0))
    return cudaErrorInvalidValue;
  const long long row_bytes = (long long)a.N * (a.dtype == MOE_DTYPE_FP32 ? 4 : 2);
  a.by_tma = !kSwiglu && (kForm == kTile || kForm == kTilePair) && a.wide && row_bytes < 1ll << 31 && encode(&a.tm_out, a.out, row_bytes, a.R, 0, 0, 32, 0);
  auto* kernel = scaled_product_kernel<kForm, kSwiglu>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
  if (e != cudaSuccess) return e;
  const long long tiles = most_tiles(a, S::kRows, kSwiglu ? a.I : a.N, kSwiglu ? 128 : S::kCols);
  if (tiles > 0x3fffffffll) return cudaErrorInvalidValue;
  int ctas = S::kQuarter ? kSplit : S::kCtas;
  a.split = 1;
  if (kForm == kFew) {
    // Clusters of four share the blocks as long as all of them fit (32 do; 36 take a second round).  us, one row, alone / shared, by weight rows: K 4096: 2048 13.7 / 6.9,
    // 4096 14.3 / 7.9, 6144 14.4 / 8.7, 8192 14.6 / 10.0, 9216 14.6 / 16.5; K 2048: 4096 8.7 / 5.8; K 1024: 4096 5.9 / 5.0; K 512: 2048 4.4 / 4.5.  (Clusters of two: 6144 10.5,
    // 12288 13.8 for 15.0, 64 tiles of K 2048 11.1 for 10.4.  Up to 64 rows shared: the code alone took one row of 6144 from 8.7 to 10.8, 16 rows of 2048 x 2048 from 9.5 to 11.8.)
    if (a.R <= kSplitRows && a.blocks >= 8 && tiles <= 32 && sms >= 32 * kSplit) {
      a.split = ctas = kSplit;
      a.wide_scales = 0;           // (parts begin anywhere)
    }
  }
  const int units = tiles < sms / ctas ? (int)tiles : sms / ctas;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(units * ctas));
  cfg.blockDim = dim3((unsigned)kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<const Args&>(a));
}

template <bool kSwiglu>
int product(const void* codes, const float* scales, const void* w_codes, const float* w_scales, const int32_t* offsets, int n_rows, int n_experts, int n,
            int K, int dtype, void* out, float* out_scales, void* stream) {
  if (n_rows < 0 || n_rows >= 1 << kRowSlotShift || n_experts < 1 || n_experts > kMaxExperts || n < 1 || n > 1 << 30 || K < 16 || K > 1 << 30 || K % 16)
    return MOE_EINVAL;
  if (!kSwiglu && dtype != MOE_DTYPE_BF16 && dtype != MOE_DTYPE_FP16 && dtype != MOE_DTYPE_FP32) return MOE_EINVAL;
  if (n_rows == 0) return MOE_OK;
  if (!codes || !scales || !w_codes || !w_scales || !out || (kSwiglu && !out_scales) || (!offsets && n_experts != 1)) return MOE_EINVAL;
  const int el = kSwiglu ? 16 : dtype == MOE_DTYPE_FP32 ? 4 : 2;
  const auto address = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if (((address(codes) | address(w_codes)) & 15) || ((address(scales) | address(w_scales) | address(offsets) | address(out_scales)) & 3) ||
      (address(out) & (el - 1)))
    return MOE_EINVAL;
  Args a;
  a.x_scales = scales;
  a.w_scales = w_scales;
  a.offsets = offsets;
  a.out = out;
  a.out_scales = out_scales;
  a.R = n_rows; a.E = n_experts; a.N = n; a.I = n / 2;
  a.blocks = (K + kBlock - 1) / kBlock;
  a.row_blocks = (n + kBlock - 1) / kBlock;
  a.dtype = dtype;
  a.wide = (long long)n * el % 16 == 0 && (address(out) & 15) == 0;
  a.wide_scales = a.blocks % 4 == 0 && ((address(scales) | address(w_scales)) & 15) == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  // The form goes by the rows that an expert gets on average; the host does not know more.  us, by rows an expert (gate/up; down), weights that are not in L2:
  //                                   16        32        48        64        96        128       192       256       320       384       512       1024
  //   uneven (Zipf 0.8), 64 experts, 2048 x 768
  //     few                           40; 24    45; 28    50; 32    53; 38    77; 49    92; 64    127; 89   154; 111  187; 139  207; 161  285; 213  523; 405
  //     128 rows                      43; 25    44; 26    46; 26    47; 27    58; 33    60; 39    74; 46    100; 60   114; 71   137; 81   168; 98   301; 179
  //     256 rows, pairs               65; 37    69; 43    71; 42    75; 45    78; 46    79; 47    94; 52    106; 66   119; 70   139; 80   166; 100  293; 172
  //   even, 32 experts, 4096 x 1792
  //     few                           87; 45    90; 47    96; 50    101; 56   161; 90   161; 91   226; 140  287; 177  347; 224            525; 347  1069; 647
  //     128 rows                                          105; 52   107; 53   110; 55   113; 57   179; 90   178; 90   249; 130            316; 180  614; 318
  //     256 rows, pairs               137; 68   142; 73   146; 73   157; 77   156; 77   160; 80   163; 83   159; 81   290; 151            284; 161  552; 288
  const long long per = n_rows / n_experts;
  // Where tiles of 256 columns would be few, those of 64 are four times as many.  us, one matrix 4096 x 4096, by rows, 64 / 256 columns / few: 16 11.5 / 18.7 / 13.5, 64 12.7 / 19.8 / 20.1,
  // 256 13.1 / 19.7 / 20.6, 300 22.1 / 19.7 / 21.3; 8 experts, 1024 x 2048, 64 rows 7.9 / 11.6 / 9.0; 200 rows of 9472 x 1024 8.3 / 8.1 / 10.1.  Gate/up, four CTAs a block of outputs:
  // 4096 x 4096, 16 rows 12.3 / 19.9 / 14.1, 64 13.5 / 20.1 / 19.7, 512 of 2048 13.8 / 20.5 / 19.9; 8 experts, 1024 x 2048, 64 rows 8.9 / 12.6 / 9.5.
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e != cudaSuccess) return MOE_ECUDA;
  if (n_rows > kSplitRows && (kSwiglu ? most_tiles(a, 128, n / 2, 128) <= 32 && sms >= 32 * kSplit : 4 * most_tiles(a, 128, n, 256) <= sms))
    return product_launch<kNarrow, kSwiglu>(a, codes, w_codes, K, sms, st) == cudaSuccess ? MOE_OK : MOE_ECUDA;
  e = per <= 32    ? product_launch<kFew, kSwiglu>(a, codes, w_codes, K, sms, st)
      : per <= 384 ? product_launch<kTile, kSwiglu>(a, codes, w_codes, K, sms, st)
                   : product_launch<kTilePair, kSwiglu>(a, codes, w_codes, K, sms, st);
  return e == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // namespace
}  // namespace moe

extern "C" {

int moe_scaled_product(const void* codes, const float* scales, const void* w_codes, const float* w_scales, const int32_t* offsets, int32_t n_rows,
                       int32_t n_experts, int32_t n_cols, int32_t k_cols, int32_t dtype, void* out, void* stream) {
  return moe::product<false>(codes, scales, w_codes, w_scales, offsets, n_rows, n_experts, n_cols, k_cols, dtype, out, nullptr, stream);
}

int moe_scaled_swiglu(const void* codes, const float* scales, const void* w_codes, const float* w_scales, const int32_t* offsets, int32_t n_rows,
                      int32_t n_experts, int32_t inter, int32_t k_cols, void* out_codes, float* out_scales, void* stream) {
  if (inter < moe::kScaledBlock || inter % moe::kScaledBlock || inter > 1 << 29) return MOE_EINVAL;
  return moe::product<true>(codes, scales, w_codes, w_scales, offsets, n_rows, n_experts, 2 * inter, k_cols, 0, out_codes, out_scales, stream);
}

}  // extern "C"
