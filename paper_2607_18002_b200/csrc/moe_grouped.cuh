// What the products of sorted rows with experts' matrices share: the tiles that a block's segments of rows make, bounded waits, TMA boxes.
#pragma once
#include <cuda_bf16.h>

#include "moe_dev.cuh"
#include "moe_ptx.cuh"

namespace moe {

constexpr unsigned long long kWaitNs = 2000000000ull;

// false: gave up, or somebody of this block has.  kTry: mbar_try; where threads of the other CTA of a pair hand over what they wrote or read,
// mbar_try_cluster (an accumulator), or mbar_try_relaxed and a fence (the scales of a stage)
template <bool (*kTry)(void*, unsigned) = mbar_try>
__device__ __forceinline__ bool wait(unsigned long long* bar, unsigned parity, volatile int* dead) {
  if (kTry(bar, parity)) return true;
  const unsigned long long start = gtime_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 64; ++i)
      if (kTry(bar, parity)) return true;
    if (*dead) return false;
    if (gtime_ns() - start > kWaitNs) {
      *dead = 1;
      return false;
    }
  }
}

// bar: shared::cluster address of the barrier (of a pair: the leader's)
template <bool kPair>
__device__ __forceinline__ void tma_2d(unsigned dst, const CUtensorMap* m, int x, int y, unsigned bar) {
  if (kPair)
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(bar)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                 "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
template <bool kPair>
__device__ __forceinline__ void tma_3d(unsigned dst, const CUtensorMap* m, int x, int y, int z, unsigned bar, unsigned long long policy) {
  if (kPair)
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
                 ::"r"(dst), "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3, %4}], [%5], %6;"
                 ::"r"(dst), "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(z), "r"(bar), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void expect_tx(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tc_ld16(unsigned taddr, unsigned (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// In shared memory: the experts' segments of rows and the tiles that they make
struct Segments {
  int first_tile[kMaxExperts + 1];   // tiles before expert e
  int first_row[kMaxExperts + 1];    // segments: the offsets, held inside [0, R] and in ascending order
  __device__ __forceinline__ int rows(int e) const { return first_row[e + 1] - first_row[e]; }
};

// inclusive sum and maximum over the lanes
__device__ __forceinline__ int scan_sum(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int left = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += left;
  }
  return v;
}
__device__ __forceinline__ int scan_max(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int left = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v = max(v, left);
  }
  return v;
}
// Offsets -> ascending first rows, and the tiles before every expert; by one warp.  One expert a lane, or neighbouring ones: the maximum and the sum of
// theirs are scanned, then they are gone through once more (256 experts: 1.3 us less than 32 at a time, 8 experts 0.3 us more than that).
template <int kRows>
__device__ __forceinline__ void list_tiles(Segments& s, int E, int n_blocks, int lane) {
  const int first = s.first_row[0];
  if (E <= 32) {
    const int to = max(scan_max(lane < E ? s.first_row[lane + 1] : 0, lane), first), left = __shfl_up_sync(0xffffffffu, to, 1);
    const int mine = lane < E ? (to - (lane ? left : first) + kRows - 1) / kRows * n_blocks : 0, sum = scan_sum(mine, lane);
    if (lane < E) {
      s.first_row[lane + 1] = to;
      s.first_tile[lane] = sum - mine;
    }
    if (lane == 31) s.first_tile[E] = sum;
    return;
  }
  const int per = (E + 31) / 32, e0 = min(lane * per, E), e1 = min(e0 + per, E);
  int top = first;
#pragma unroll 1
  for (int e = e0; e < e1; ++e) top = max(top, s.first_row[e + 1]);
  top = scan_max(top, lane);
  int row = __shfl_up_sync(0xffffffffu, top, 1), tiles = 0;
  if (lane == 0) row = first;
#pragma unroll 1
  for (int e = e0; e < e1; ++e) {
    const int to = max(row, s.first_row[e + 1]);
    s.first_row[e + 1] = to;
    s.first_tile[e] = tiles;
    tiles += (to - row + kRows - 1) / kRows * n_blocks;
    row = to;
  }
  const int sum = scan_sum(tiles, lane);
#pragma unroll 1
  for (int e = e0; e < e1; ++e) s.first_tile[e] += sum - tiles;
  if (lane == 31) s.first_tile[E] = sum;
}

struct Tile {
  int expert, row0, rows, n0;    // n0: first weight row (swiglu: first gate row)
  bool alone;                    // the expert's only tile of these weights
};
template <int kRows>
__device__ __forceinline__ Tile tile_at(const Segments& s, int E, int t, int n_step) {
  int lo = 0, hi = E;            // first_tile[lo] <= t < first_tile[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.first_tile[mid] <= t) lo = mid; else hi = mid;
  }
  const int rows = s.rows(lo), m_tiles = (rows + kRows - 1) / kRows, local = t - s.first_tile[lo];
  const int n = local / m_tiles, m = local - n * m_tiles;
  return Tile{lo, s.first_row[lo] + m * kRows, min(kRows, rows - m * kRows), n * n_step, m_tiles == 1};
}

// Lane 0's value, which the compiler then knows to be the same in all lanes (without it gate/up took 2-5 % longer).
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ Tile uniform(const Tile& t) { return Tile{uniform(t.expert), uniform(t.row0), uniform(t.rows), uniform(t.n0), t.alone}; }

// silu(g) u in fp32: exp(-g) = 2^(-g log2 e) to 2 + 1.2 |g| steps, the reciprocal to one.  Powers below 2^-126 and reciprocals of those above 2^126 count
// as 0: nothing next to the 1 that is added, silu of less than -87.  (Gate/up with the forms that keep them 547 us, so 509.)
__device__ __forceinline__ float silu_times(float g, float u) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
  return g * r * u;
}
__device__ __forceinline__ unsigned pack_bf16(unsigned lo, unsigned hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const unsigned*>(&v);
}
typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// looked up once a process: the address of a driver function
inline EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(p) : nullptr;
  }();
  return fn;
}

}  // namespace moe
