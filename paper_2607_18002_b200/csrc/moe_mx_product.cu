// moe_mx_product / moe_mx_swiglu: sorted 4-bit rows times the experts' 4-bit matrices (format: moe_mx.cuh), with the 5th-generation tensor
// cores' block-scaled multiply: tcgen05.mma.kind::mxf4.block_scale takes e2m1 codes from shared memory and the scale bytes of 32-column blocks
// from TMEM, and accumulates in fp32.
//
//   product   out[p, n] = sum_k a[p, k] w[e, n, k]                      (e: the expert whose segment of rows holds p; rounded to bf16 once)
//   swiglu    g, u = products with rows n and I + n of w[e];  a' = g / (1 + exp(-g)) u in fp32, quantised per 32 columns to codes and scales
//
// The weight rows are the M of the instruction (128 TMEM lanes), the tile's rows its N in steps of 16, so an expert with a few rows costs a few
// columns.  A tile is 256 weight rows -- two accumulators; for swiglu 128 gate rows and the 128 up rows that go with them, so that a thread has
// both factors of an output -- and up to kRows rows of one expert.  A thread of the epilogue has one weight row (one output column): a warp writes 32
// neighbouring columns of a row at a time, and for swiglu those 32 are one block of the result, its largest magnitude one warp-wide maximum.
//
// One persistent CTA per SM walks the tiles (rows of an expert innermost: neighbours share a weight tile in L2).  Roles: one thread issues TMA
// (a stage is 256 columns of K: 128-byte rows, swizzled), two warps bring the stage's scale bytes through registers into the 512-byte
// form that tcgen05.cp copies to TMEM (128 rows x 4 blocks), one thread copies them and issues the MMAs, eight warps are the epilogue.
// Every wait is bounded; where one runs out the launch ends and what it has not computed is NaN.
#include "moe_dev.cuh"
#include "moe_mx.cuh"
#include "moe_ptx.cuh"

namespace moe {
namespace {

// Warps 0-7 epilogue, 8 TMA, 9 MMA, 10 and 11 scales.  Three warps a quarter of the SM leave a thread 168 registers, four would leave 128.
constexpr int kMxThreads = 384;
constexpr int kTmaWarp = 8, kMmaWarp = 9, kScaleWarp = 10, kScaleWarps = 2;
constexpr int kStageK = 256;                    // columns of K in a stage
constexpr int kGroupK = 128;                    // ... in one 512-byte block of scales (4 a row)
constexpr int kHalfRows = 128;                  // weight rows of an accumulator
constexpr int kScaleBlock = 512;
constexpr int kBoxRows = 32;                    // rows of a TMA box of activations
constexpr unsigned long long kWaitNs = 2000000000ull;

struct MxShared {
  unsigned long long full[8], landed[8], empty[8], acc_full[2], acc_empty[2], drained;
  unsigned tmem;
  volatile int dead;             // a wait ran out
  int first_tile[kMaxExperts + 1];   // tiles before expert e
  int first_row[kMaxExperts + 1];    // segments, held inside [0, R)
  __device__ __forceinline__ int rows(int e) const { return max(first_row[e + 1] - first_row[e], 0); }
};

// What depends on the rows of a tile.  Shared memory: stages of 32 KB weights, kRows * 128 bytes of rows and the scale blocks of both; TMEM: the
// accumulators (two buffers of them where they fit) from column 0, the stages' scales behind.
template <int kRows_>
struct Shape {
  static constexpr int kRows = kRows_;
  static constexpr int kRowBlocks = (kRows + 127) / 128;                      // 128-row blocks of row scales
  static constexpr int kScaleBytes = 2 * (2 + kRowBlocks) * kScaleBlock;
  static constexpr int kWBytes = 2 * kHalfRows * 128, kXBytes = kRows * 128;
  static constexpr int kStageBytes = kWBytes + kXBytes + kScaleBytes;
  static constexpr int kScaleCols = 2 * (2 + kRowBlocks) * 4;                 // TMEM columns of a stage's scales
  static constexpr int kLate = kRows / 16 < 6 ? kRows / 16 : 6;               // groups of 16 columns that the epilogue takes to registers
  static constexpr int kAccBufs = kRows <= 96 ? 2 : 1;
  static constexpr int kScaleCol0 = kAccBufs * 2 * kRows;
  static constexpr int kFitSmem = (227 * 1024 - 1024 - (int)sizeof(MxShared)) / kStageBytes, kFitTmem = (512 - kScaleCol0) / kScaleCols;
  static constexpr int kStages = kFitSmem < kFitTmem ? kFitSmem : kFitTmem;
  static_assert(kStages >= 2, "stages");
  static_assert(kStages <= 8, "barriers");
  static_assert(kScaleCol0 + kStages * kScaleCols <= 512, "TMEM");
};

struct MxArgs {
  CUtensorMap tm_w, tm_x;        // weights [E][N][K/2] bytes, boxes of 128 rows; rows [R][K/2], boxes of 32
  const unsigned char* x_scales; // [R, K/32]
  const unsigned char* w_scales; // [E, N, K/32]
  const int* offsets;            // [E + 1]
  void* out;                     // bf16 [R, N]; swiglu: codes [R, I/2]
  unsigned char* out_scales;     // swiglu: [R, I/32]
  int R, E, N, K, I;             // I: N / 2 for swiglu
  int wide;                      // rows of out are 16-byte aligned
};

// false: gave up, or somebody has
__device__ __noinline__ bool wait_slow(unsigned long long* bar, unsigned parity, volatile int* dead) {
  const unsigned long long start = gtime_ns();
  for (;;) {
    for (int i = 0; i < 64; ++i)
      if (mbar_try(bar, parity)) return true;
    if (*dead) return false;
    if (gtime_ns() - start > kWaitNs) {
      *dead = 1;
      return false;
    }
  }
}
__device__ __forceinline__ bool wait(unsigned long long* bar, unsigned parity, volatile int* dead) {
  return mbar_try(bar, parity) || wait_slow(bar, parity, dead);
}

// shared-memory descriptor of a scale block: 32 rows of 16 bytes, unswizzled, 8-row groups 128 bytes apart
__device__ __forceinline__ unsigned long long scale_desc(unsigned saddr) {
  return (unsigned long long)((saddr & 0x3ffffu) >> 4) | 8ull << 16 | 8ull << 32 | 1ull << 46;
}
__device__ __forceinline__ void copy_scales(unsigned tmem, unsigned saddr) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scale_desc(saddr)) : "memory");
}
__device__ __forceinline__ void mma_mxf4(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sfa, unsigned sfb,
                                         unsigned accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
      : "memory");
}
// e2m1 operands, both K-major, power-of-two scales, M = 128, N columns; half: which two of a block's four scales a row (K = 64 takes two)
__device__ __forceinline__ unsigned mx_idesc(unsigned n, unsigned half) {
  return 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 | (128u >> 4) << 24 | (2u * half) << 4 | (2u * half) << 29;
}
__device__ __forceinline__ void tma_2d(unsigned dst, const CUtensorMap* m, int x, int y, void* bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void tma_3d(unsigned dst, const CUtensorMap* m, int x, int y, int z, void* bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(reinterpret_cast<unsigned long long>(m)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void expect_tx(void* bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void tc_ld16(unsigned taddr, unsigned (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// 16 bytes of a row's scales, `left` of which are there (the others are not used), by loads of vec bytes
__device__ __forceinline__ uint4 load_scales(const unsigned char* p, int left, int vec) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (vec == 16) return __ldg(reinterpret_cast<const uint4*>(p));
  if (vec == 8) {
    const uint2 lo = __ldg(reinterpret_cast<const uint2*>(p));
    v.x = lo.x;
    v.y = lo.y;
    if (left > 8) {
      const uint2 hi = __ldg(reinterpret_cast<const uint2*>(p) + 1);
      v.z = hi.x;
      v.w = hi.y;
    }
    return v;
  }
  const unsigned* w = reinterpret_cast<const unsigned*>(p);
  v.x = __ldg(w);
  if (left > 4) v.y = __ldg(w + 1);
  if (left > 8) v.z = __ldg(w + 2);
  if (left > 12) v.w = __ldg(w + 3);
  return v;
}
__device__ __forceinline__ void st_word(unsigned saddr, unsigned v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(saddr), "r"(v) : "memory"); }

struct Tile {
  int expert, row0, rows, n0;    // n0: first weight row (swiglu: first gate row)
};
template <int kRows>
__device__ __forceinline__ Tile tile_at(const MxShared& s, int E, int t, int n_step) {
  int lo = 0, hi = E;            // first_tile[lo] <= t < first_tile[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s.first_tile[mid] <= t) lo = mid; else hi = mid;
  }
  const int rows = s.rows(lo), m_tiles = (rows + kRows - 1) / kRows, local = t - s.first_tile[lo];
  const int n = local / m_tiles, m = local - n * m_tiles;
  return Tile{lo, s.first_row[lo] + m * kRows, min(kRows, rows - m * kRows), n * n_step};
}

__device__ __forceinline__ float rcp_approx(float v) {      // to one step
  float r;
  asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// 8 x 8 four-bit values over eight neighbouring lanes: lane i gives value j of word i, gets value i of word j
__device__ __forceinline__ unsigned transpose_nibbles(unsigned v, int lane) {
#pragma unroll
  for (int s = 4; s >= 1; s >>= 1) {
    const unsigned low = s == 4 ? 0x0000ffffu : s == 2 ? 0x00ff00ffu : 0x0f0f0f0fu;
    const unsigned other = __shfl_xor_sync(0xffffffffu, v, s);
    v = lane & s ? (v & ~low) | ((other & ~low) >> (4 * s)) : (v & low) | ((other & low) << (4 * s));
  }
  return v;
}

__device__ __forceinline__ unsigned pack_bf16(unsigned lo, unsigned hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(__uint_as_float(lo), __uint_as_float(hi));
  return *reinterpret_cast<const unsigned*>(&v);
}
// 8 x 8 fp32 values over eight neighbouring lanes, lane i with value j of column i: lane j gets row j as eight bf16.  Lane bit 0 changes places with
// row bit 0 inside the packed pairs, then bits 1 and 2 with whole words.
__device__ __forceinline__ uint4 transpose_bf16(const unsigned* v, int lane) {
  unsigned q[4], lo[2], hi[2];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned own = pack_bf16(v[2 * i], v[2 * i + 1]), other = __shfl_xor_sync(0xffffffffu, own, 1);
    q[i] = __byte_perm(own, other, lane & 1 ? 0x3276u : 0x5410u);
  }
#pragma unroll
  for (int m = 0; m < 2; ++m) {
    const unsigned own = lane & 2 ? q[2 * m + 1] : q[2 * m];
    const unsigned other = __shfl_xor_sync(0xffffffffu, lane & 2 ? q[2 * m] : q[2 * m + 1], 2);
    lo[m] = lane & 2 ? other : own;
    hi[m] = lane & 2 ? own : other;
  }
  const unsigned own0 = lane & 4 ? lo[1] : lo[0], own1 = lane & 4 ? hi[1] : hi[0];
  const unsigned other0 = __shfl_xor_sync(0xffffffffu, lane & 4 ? lo[0] : lo[1], 4), other1 = __shfl_xor_sync(0xffffffffu, lane & 4 ? hi[0] : hi[1], 4);
  return lane & 4 ? make_uint4(other0, other1, own0, own1) : make_uint4(own0, own1, other0, other1);
}

template <int kRows_, bool kSwiglu>
__global__ void __launch_bounds__(kMxThreads, 1) mx_product_kernel(const __grid_constant__ MxArgs a) {
  using S = Shape<kRows_>;
  extern __shared__ unsigned char raw[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  MxShared& s = *reinterpret_cast<MxShared*>(stages + S::kStages * S::kStageBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr int kStep = kSwiglu ? kHalfRows : 2 * kHalfRows;       // output columns of a tile
  const int n_blocks = ((kSwiglu ? a.I : a.N) + kStep - 1) / kStep;

  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.landed[i], kScaleWarps);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 8);
    }
    mbar_init(&s.drained, 1);
    s.dead = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    fence_async_proxy_smem();
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dep_wait();
  for (int e = tid; e <= a.E; e += kMxThreads) s.first_row[e] = min(max(a.offsets[e], 0), a.R);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) {
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += 32) {
      const int e = e0 + lane, mine = e < a.E ? (s.rows(e) + S::kRows - 1) / S::kRows * n_blocks : 0;
      int sum = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += v;
      }
      if (e < a.E) s.first_tile[e] = before + sum - mine;
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) s.first_tile[a.E] = before;
  }
  __syncthreads();
  const unsigned tmem = s.tmem;
  const int n_tiles = s.first_tile[a.E];
  const int n_stages = (a.K + kStageK - 1) / kStageK;

  if (warp == kTmaWarp) {
    if (elect_one()) {
      unsigned n = 0;            // stages so far
      for (int t = blockIdx.x; t < n_tiles && !s.dead; t += gridDim.x) {
        const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
        const int boxes = (at.rows + kBoxRows - 1) / kBoxRows;
        for (int i = 0; i < n_stages; ++i, ++n) {
          const unsigned slot = n % S::kStages, round = n / S::kStages;
          if (round && !wait(&s.empty[slot], (round - 1) & 1, &s.dead)) break;
          const unsigned to = smem_u32(stages + slot * S::kStageBytes);
          expect_tx(&s.full[slot], S::kWBytes + boxes * kBoxRows * 128);
          tma_3d(to, &a.tm_w, i * 128, at.n0, at.expert, &s.full[slot]);
          tma_3d(to + kHalfRows * 128, &a.tm_w, i * 128, (kSwiglu ? a.I : kHalfRows) + at.n0, at.expert, &s.full[slot]);
          for (int b = 0; b < boxes; ++b) tma_2d(to + S::kWBytes + b * kBoxRows * 128, &a.tm_x, i * 128, at.row0 + b * kBoxRows, &s.full[slot]);
        }
      }
      // copies that nobody has waited for (after a wait that ran out): the block's shared memory is theirs until they have landed
      for (unsigned m = n > S::kStages ? n - S::kStages : 0; s.dead && m < n; ++m) {
        const unsigned long long start = gtime_ns();
        while (!mbar_try(&s.full[m % S::kStages], (m / S::kStages) & 1) && gtime_ns() - start < kWaitNs) {}
      }
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    if (elect_one()) {
      unsigned n = 0, k = 0;     // stages, tiles so far
      bool ok = true;
      for (int t = blockIdx.x; t < n_tiles && ok; t += gridDim.x, ++k) {
        const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
        const unsigned buf = k % S::kAccBufs, use = k / S::kAccBufs;
        if (use) ok = wait(&s.acc_empty[buf], (use - 1) & 1, &s.dead);
        if (!ok) break;
        tc_fence_after();
        const unsigned cols = (unsigned)(at.rows + 15) & ~15u;
        const unsigned acc = tmem + buf * 2 * S::kRows;
        for (int i = 0; i < n_stages; ++i, ++n) {
          const unsigned slot = n % S::kStages, round = n / S::kStages;
          ok = wait(&s.full[slot], round & 1, &s.dead) && wait(&s.landed[slot], round & 1, &s.dead);
          if (!ok) break;
          tc_fence_after();
          const unsigned st = smem_u32(stages + slot * S::kStageBytes);
          const unsigned sc = st + S::kWBytes + S::kXBytes, tsc = tmem + S::kScaleCol0 + slot * S::kScaleCols;
          const int groups = min(2, (a.K - i * kStageK) / kGroupK);
          for (int g = 0; g < groups; ++g) {
            const unsigned from = sc + g * (2 + S::kRowBlocks) * kScaleBlock, to = tsc + g * (2 + S::kRowBlocks) * 4;
#pragma unroll
            for (int b = 0; b < 2 + S::kRowBlocks; ++b) copy_scales(to + 4 * b, from + b * kScaleBlock);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const unsigned step = (2 * g + h) * 32;       // 64 columns, 32 bytes
              const unsigned long long xd = umma_desc(st + S::kWBytes + step, 128);
              const unsigned idesc = mx_idesc(cols, h), first = (i | g | h) != 0;
              mma_mxf4(acc, umma_desc(st + step, 128), xd, idesc, to, to + 8, first);
              mma_mxf4(acc + S::kRows, umma_desc(st + kHalfRows * 128 + step, 128), xd, idesc, to + 4, to + 8, first);
            }
          }
          tc_commit(&s.empty[slot]);
        }
        if (ok) tc_commit(&s.acc_full[buf]);
      }
      tc_commit(&s.drained);     // nothing of this block's is left in the tensor core when it frees its TMEM
      const unsigned long long start = gtime_ns();
      while (!mbar_try(&s.drained, 0) && gtime_ns() - start < kWaitNs) {}
    }
    __syncwarp();
  } else if (warp >= kScaleWarp) {
    // A thread has two rows of every 128-row block, in the order that spreads a warp's stores over all banks: their four bytes of a group of
    // 128 columns go to 16 (r % 32) + 4 (r / 32) of the group's block.  16 bytes of a row are two stages; those of the next two are on their
    // way to registers meanwhile, whether or not their stages are free.
    const int r0 = 32 * (lane & 3) + 8 * (warp - kScaleWarp) + (lane >> 2);      // and r0 + 16
    const unsigned spot = (unsigned)(r0 & 31) * 16 + (unsigned)(r0 >> 5) * 4;
    const int per_row = a.K / kMxBlock, n_pairs = (n_stages + 1) / 2;
    const int vec = per_row % 16 == 0 ? 16 : per_row % 8 == 0 ? 8 : 4;
    const bool vec_w = ((size_t)a.w_scales & (vec - 1)) == 0, vec_x = ((size_t)a.x_scales & (vec - 1)) == 0;
    constexpr int kBlocks = 2 + S::kRowBlocks;
    struct Pair {
      uint4 b[kBlocks][2];
      int stages;                // 1 or 2; 0: there is no more
    };
    int t = blockIdx.x, pair = 0;
    const unsigned char* from[kBlocks][2];
    unsigned n = 0;
    const auto fetch = [&](Pair& p) {
      p.stages = 0;
      if (t >= n_tiles) return;
      if (pair == 0) {
        const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int r = r0 + 16 * q;
#pragma unroll
          for (int b = 0; b < 2; ++b) {    // a weight row behind the last one: any other's scales (its products are not stored)
            const int row = kSwiglu ? min(at.n0 + r, a.I - 1) + b * a.I : min(at.n0 + b * kHalfRows + r, a.N - 1);
            from[b][q] = a.w_scales + ((size_t)at.expert * a.N + row) * per_row;
          }
#pragma unroll
          for (int b = 0; b < S::kRowBlocks; ++b) from[2 + b][q] = a.x_scales + (size_t)(at.row0 + min(b * 128 + r, at.rows - 1)) * per_row;
        }
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int q = 0; q < 2; ++q) p.b[b][q] = load_scales(from[b][q] + pair * 16, per_row - pair * 16, (b < 2 ? vec_w : vec_x) ? vec : 4);
      p.stages = min(2, n_stages - 2 * pair);
      if (++pair == n_pairs) {
        pair = 0;
        t += gridDim.x;
      }
    };
    const auto put = [&](const Pair& p) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h >= p.stages) break;
        const unsigned slot = n % S::kStages, round = n / S::kStages;
        if (round && !__all_sync(0xffffffffu, wait(&s.empty[slot], (round - 1) & 1, &s.dead))) return false;
        const unsigned to = smem_u32(stages + slot * S::kStageBytes) + S::kWBytes + S::kXBytes + spot;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint4& v = p.b[b][q];
            st_word(to + b * kScaleBlock + 256 * q, h ? v.z : v.x);
            st_word(to + (kBlocks + b) * kScaleBlock + 256 * q, h ? v.w : v.y);
          }
        fence_async_proxy_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.landed[slot]);
        ++n;
      }
      return true;
    };
    Pair even, odd;
    fetch(even);
    while (even.stages) {
      fetch(odd);
      if (!put(even) || !odd.stages) break;
      fetch(even);
      if (!put(odd)) break;
    }
  } else {
    const int quad = warp & 3, half = warp >> 2;
    unsigned k = 0;
    bool ok = true;
    for (int t = blockIdx.x; t < n_tiles; t += gridDim.x, ++k) {
      const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
      const unsigned buf = k % S::kAccBufs, use = k / S::kAccBufs;
      if (ok) ok = __all_sync(0xffffffffu, wait(&s.acc_full[buf], use & 1, &s.dead));
      tc_fence_after();
      const unsigned acc = tmem + buf * 2 * S::kRows + ((unsigned)quad << 21);      // this warp's 32 lanes
      // The last columns of the accumulator go to registers all at once and are worked off after it has been handed back, while the next
      // tile's MMAs run.
      const auto hand_back = [&] {
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&s.acc_empty[buf]);
      };
      const int groups = (at.rows + 15) / 16;
      if (!kSwiglu) {            // warps 0-3 have the first accumulator, 4-7 the second
        const unsigned mine = acc + half * S::kRows;
        const int col = at.n0 + half * kHalfRows + quad * 32 + lane;
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (size_t)at.row0 * a.N + col;
        const auto store = [&](unsigned (&v)[16], int c) {
          if (!ok) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = 0x7fffffffu;
          }
          if (a.wide) {          // eight neighbouring columns of a row a lane, 16 bytes: stores of 2 bytes took the down product 1.4 times as long
#pragma unroll
            for (int j0 = 0; j0 < 16; j0 += 8) {
              const uint4 w = transpose_bf16(v + j0, lane);
              const int row = c + j0 + (lane & 7), col8 = col - lane + (lane >> 3) * 8;
              if (row < at.rows && col8 < a.N)
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.out) + (size_t)(at.row0 + row) * a.N + col8) = w;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c + j < at.rows && col < a.N) out[(size_t)(c + j) * a.N] = __float2bfloat16_rn(__uint_as_float(v[j]));
          }
        };
        const int direct = max(groups - S::kLate, 0);
        for (int g = 0; g < direct; ++g) {
          unsigned v[16];
          tc_ld16(mine + 16 * g, v);
          tc_wait_ld();
          store(v, 16 * g);
        }
        unsigned v[S::kLate][16];
#pragma unroll
        for (int i = 0; i < S::kLate; ++i)
          if (direct + i < groups) tc_ld16(mine + 16 * (direct + i), v[i]);
        hand_back();
#pragma unroll
        for (int i = 0; i < S::kLate; ++i)
          if (direct + i < groups) store(v[i], 16 * (direct + i));
      } else {                   // warps 0-3 and 4-7 take turns at groups of 16 rows
        const int col = at.n0 + quad * 32, per_row = a.I / kMxBlock;
        const auto store = [&](const unsigned (&gate)[16], const unsigned (&up)[16], int c) {
#pragma unroll
          for (int j0 = 0; j0 < 16; j0 += 8) {
            unsigned word = 0u, mine = 0u;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
              float q[2];
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float gv = __uint_as_float(gate[j0 + j + i]), uv = __uint_as_float(up[j0 + j + i]);
                const float v = gv * rcp_approx(1.f + __expf(-gv)) * uv;
                const unsigned top = __reduce_max_sync(0xffffffffu, __float_as_uint(v) & 0x7f800000u);
                if ((lane & 7) == j + i) mine = top;
                q[i] = v * __uint_as_float(min(0x80000000u - top, 0x7f000000u));     // 2^(127 - scale byte)
              }
              word |= mx_codes2(q[0], q[1]) << (4 * j);
            }
            word = transpose_nibbles(word, lane);            // lane 8 i + j: columns 8 i .. 8 i + 7 of row j
            const int row = c + j0 + (lane & 7);
            if (row < at.rows && col < a.I) {
              const size_t p = (size_t)(at.row0 + row);
              *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(a.out) + p * (a.I / 2) + col / 2 + (lane >> 3) * 4) = word;
              if (lane < 8) a.out_scales[p * per_row + col / kMxBlock] = (unsigned char)(ok ? mx_scale_byte(mine) : 255u);
            }
          }
        };
        constexpr int kLate = (S::kLate + 1) / 2;
        const int my_groups = (groups - half + 1) / 2, direct = max(my_groups - kLate, 0);
        for (int g = 0; g < direct; ++g) {
          unsigned gate[16], up[16];
          tc_ld16(acc + 16 * (half + 2 * g), gate);
          tc_ld16(acc + S::kRows + 16 * (half + 2 * g), up);
          tc_wait_ld();
          store(gate, up, 16 * (half + 2 * g));
        }
        unsigned gate[kLate][16], up[kLate][16];
#pragma unroll
        for (int i = 0; i < kLate; ++i)
          if (direct + i < my_groups) {
            tc_ld16(acc + 16 * (half + 2 * (direct + i)), gate[i]);
            tc_ld16(acc + S::kRows + 16 * (half + 2 * (direct + i)), up[i]);
          }
        hand_back();
#pragma unroll
        for (int i = 0; i < kLate; ++i)
          if (direct + i < my_groups) store(gate[i], up[i], 16 * (half + 2 * (direct + i)));
      }
    }
    // rows that belong to no expert: zeros, by the epilogue warps of the whole grid
    const size_t width = kSwiglu ? (size_t)a.I / 32 * 17 : (size_t)a.N;
    const int lo = s.first_row[0], hi = max(s.first_row[a.E], lo), none = lo + (a.R - hi);
    for (int i = blockIdx.x; i < none; i += gridDim.x) {
      const size_t p = (size_t)(i < lo ? i : hi + (i - lo));
      for (size_t c = tid; c < width; c += 256) {
        if (!kSwiglu) static_cast<__nv_bfloat16*>(a.out)[p * a.N + c] = __float2bfloat16_rn(0.f);
        else if (c < (size_t)a.I / 2) static_cast<unsigned char*>(a.out)[p * (a.I / 2) + c] = 0;
        else a.out_scales[p * (a.I / 32) + (c - a.I / 2)] = 0;
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

typedef CUresult (*EncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                             const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// looked up once a process: the address of a driver function
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found);
    return e == cudaSuccess && found == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeFn>(p) : nullptr;
  }();
  return fn;
}

// codes as bytes [planes][rows][bytes], boxes of 128 bytes x box_rows rows
bool encode_codes(CUtensorMap* out, const void* base, int bytes, int rows, int planes, int box_rows) {
  const EncodeFn fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)bytes, (cuuint64_t)rows, (cuuint64_t)planes};
  const cuuint64_t strides[2] = {(cuuint64_t)bytes, (cuuint64_t)bytes * rows};
  const cuuint32_t box[3] = {128u, (cuuint32_t)box_rows, 1u}, one[3] = {1u, 1u, 1u};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, planes ? 3 : 2, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int kRows, bool kSwiglu>
cudaError_t product_launch(const MxArgs& a, cudaStream_t stream) {
  using S = Shape<kRows>;
  constexpr size_t smem = 1024 + (size_t)S::kStages * S::kStageBytes + sizeof(MxShared);
  static_assert(smem <= 227 * 1024, "shared memory");
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_product_kernel<kRows, kSwiglu>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // most tiles that the rows can make
  const int step = kSwiglu ? kHalfRows : 2 * kHalfRows;
  const long long m_tiles = a.R / kRows + (a.R < a.E ? a.R : a.E), tiles = m_tiles * (((kSwiglu ? a.I : a.N) + step - 1) / step);
  if (tiles > 0x3fffffffll) return cudaErrorInvalidValue;
  return launch_after(mx_product_kernel<kRows, kSwiglu>, tiles < sms ? (int)tiles : sms, kMxThreads, smem, stream, a);
}

template <bool kSwiglu>
int product(const void* codes, const void* scales, const void* w_codes, const void* w_scales, const int32_t* offsets, int n_rows, int n_experts,
            int n, int K, void* out, void* out_scales, void* stream) {
  if (n_rows < 0 || n_rows >= 1 << kRowSlotShift || n_experts < 1 || n_experts > kMaxExperts || n < 1 || K < kGroupK || K % kGroupK) return MOE_EINVAL;
  if (n_rows == 0) return MOE_OK;
  if (!codes || !scales || !w_codes || !w_scales || !offsets || !out || (kSwiglu && !out_scales)) return MOE_EINVAL;
  const uintptr_t wide = reinterpret_cast<uintptr_t>(codes) | reinterpret_cast<uintptr_t>(w_codes);
  const uintptr_t words = reinterpret_cast<uintptr_t>(scales) | reinterpret_cast<uintptr_t>(w_scales) | reinterpret_cast<uintptr_t>(offsets);
  if ((wide & 15) || (words & 3) || (reinterpret_cast<uintptr_t>(out) & (kSwiglu ? 3 : 1))) return MOE_EINVAL;
  MxArgs a;
  if (!encode_codes(&a.tm_w, w_codes, K / 2, n, n_experts, kHalfRows) || !encode_codes(&a.tm_x, codes, K / 2, n_rows, 0, kBoxRows)) return MOE_ECUDA;
  a.x_scales = static_cast<const unsigned char*>(scales);
  a.w_scales = static_cast<const unsigned char*>(w_scales);
  a.offsets = offsets;
  a.out = out;
  a.out_scales = static_cast<unsigned char*>(out_scales);
  a.R = n_rows; a.E = n_experts; a.N = n; a.K = K; a.I = n / 2;
  a.wide = n % 8 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int rows = n_rows <= 24ll * n_experts ? 32 : n_rows <= 64ll * n_experts ? 64 : 192;
  const cudaError_t e = rows == 32 ? product_launch<32, kSwiglu>(a, st) : rows == 64 ? product_launch<64, kSwiglu>(a, st)
                                                                                     : product_launch<192, kSwiglu>(a, st);
  return e == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // namespace
}  // namespace moe

extern "C" {

int moe_mx_product(const void* codes, const void* scales, const void* w_codes, const void* w_scales, const int32_t* offsets, int32_t n_rows,
                   int32_t n_experts, int32_t n_cols, int32_t k_cols, void* out, void* stream) {
  return moe::product<false>(codes, scales, w_codes, w_scales, offsets, n_rows, n_experts, n_cols, k_cols, out, nullptr, stream);
}

int moe_mx_swiglu(const void* codes, const void* scales, const void* w_codes, const void* w_scales, const int32_t* offsets, int32_t n_rows,
                  int32_t n_experts, int32_t inter, int32_t k_cols, void* out_codes, void* out_scales, void* stream) {
  if (inter < moe::kMxBlock || inter % moe::kMxBlock || inter > 1 << 29) return MOE_EINVAL;
  return moe::product<true>(codes, scales, w_codes, w_scales, offsets, n_rows, n_experts, 2 * inter, k_cols, out_codes, out_scales, stream);
}

}  // extern "C"
