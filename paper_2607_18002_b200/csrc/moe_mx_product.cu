// moe_mx_product / moe_mx_swiglu: sorted 4-bit rows times the experts' 4-bit matrices (format: moe_mx.cuh), with the 5th-generation tensor
// cores' block-scaled multiply: tcgen05.mma.kind::mxf4.block_scale takes e2m1 codes from shared memory and the scale bytes of 32-column blocks
// from TMEM, and accumulates in fp32.
//
//   product   out[p, n] = sum_k a[p, k] w[e, n, k]                      (e: the expert whose segment of rows holds p; rounded to bf16 once)
//   swiglu    g, u = products with rows n and I + n of w[e];  a' = g / (1 + exp(-g)) u in fp32, quantised per 32 columns to codes and scales
//
// The weight rows are the M of the instruction (128 TMEM lanes), the tile's rows its N in steps of 16, so an expert with a few rows costs a few
// columns.  A tile is 256 weight rows -- two accumulators; for swiglu 128 gate rows and the 128 up rows that go with them, so that a thread has
// both factors of an output -- and up to kRows rows of one expert.  A pair of CTAs (cta_group::2) has twice the weight rows, M = 256, and each of the
// two holds its own weight rows and half of the tile's rows in shared memory: swiglu with many rows an expert.
//
// One persistent CTA (or pair) per SM walks the tiles (rows of an expert innermost: neighbours share a weight tile in L2).  Roles: one thread issues
// TMA (a stage is 256 columns of K: 128-byte rows, swizzled), four warps bring the stage's scale bytes through registers into the 512-byte
// form that tcgen05.cp copies to TMEM (128 rows x 4 blocks), one thread copies them and issues the MMAs, eight warps are the epilogue: for the plain
// product through stmatrix and shared memory, for swiglu a warp's 32 lanes have one 32-column block of the result.
// What bounds them: few rows, the weight stream; many, energy and the accumulators' way out between two tiles' MMAs (65 536 rows of 64 experts, K 4096, inter
// 1792, boxes differ: gate/up 430-490 us, 3.9-4.4 PFLOP/s at 1 000 W; down 275-320 us, 3.0-3.5 PFLOP/s and 537 MB of outputs).
// Outputs are rounded to bf16, like the expert outputs of moe_run: half of the bytes that the down product writes and the merge reads.  A layer is then
// off by 2.4e-3 (2-norm, against 64 bits) where fp32 rows would give 1.7e-3, the rounding of the layer's own outputs.
// Code size counts: after another kernel, or a long stream through L2, the first tile waits for instructions from DRAM, and within a launch five
// roles share the instruction caches.  So the roles' loops are not unrolled and exist once, values that are alike in a warp are made known as such, and
// the block maxima go over pairs (gate/up and down in turn 10-20 % faster at 64-1 024 rows an expert, 15 % at one).  Executing the epilogue once without effects before the first tile, or one kernel for both products, then gained nothing.
// Weights that one tile alone reads leave L2 first.  With other weights in every launch that makes no difference (800 rows of 128 experts, 1.5 GB, the
// weight stream: gate/up 162 us, down 82, 6.1 TB/s); weights of about L2's size that come again gain 5-15 %.
// Every wait is bounded (2 s); where one runs out the launch ends, after another such limit for its copies in flight, and what it has not computed is NaN.
#include "moe_dev.cuh"
#include "moe_grouped.cuh"
#include "moe_mx.cuh"
#include "moe_ptx.cuh"

namespace moe {
namespace {

// Warps 0-7 epilogue, 8 TMA, 9 MMA, 12-15 scales (10 and 11 fill up a warpgroup).  A thread is launched with 128 registers; where tiles have many rows
// the epilogue's two warpgroups take 168, that of TMA and MMA keeps 72, the scales' 104 (2 x 168 + 72 + 104 = 4 x 128).
constexpr int kMxThreads = 512;
constexpr int kTmaWarp = 8, kMmaWarp = 9, kScaleWarp = 12, kScaleWarps = 4;
constexpr int kStageK = 256;                    // columns of K in a stage
constexpr int kGroupK = 128;                    // ... in one 512-byte block of scales (4 a row)
constexpr int kHalfRows = 128;                  // weight rows of an accumulator
constexpr int kScaleBlock = 512;
constexpr int kBoxRows = 32;                    // rows of a TMA box of activations
constexpr int kStorePitch = 2 * kHalfRows + 16;  // a row of 128 bf16 outputs on its way out; the 16 bytes spread eight rows over all banks
constexpr int kStoreBuf = 16 * kStorePitch;

struct MxShared : Segments {
  unsigned long long full[8], landed[8], empty[8], acc_full[2], acc_empty[2], drained;
  unsigned tmem;
  volatile int dead;             // a wait ran out
};

// What depends on the rows of a tile.  Shared memory: stages of 32 KB weights, kRows * 128 bytes of rows and the scale blocks of both; TMEM: the
// accumulators (two buffers of them where they fit) from column 0, the stages' scales behind.
template <int kRows_, bool kSwiglu, bool kPair>
struct Shape {
  static constexpr int kRows = kRows_;
  static constexpr int kRowBlocks = (kRows + 127) / 128;                      // 128-row blocks of row scales
  static constexpr int kScaleBytes = 2 * (2 + kRowBlocks) * kScaleBlock;
  static constexpr int kWBytes = 2 * kHalfRows * 128, kXBytes = (kPair ? kRows / 2 : kRows) * 128;
  static constexpr int kStageBytes = kWBytes + kXBytes + kScaleBytes;
  static constexpr int kScaleCols = 2 * (2 + kRowBlocks) * 4;                 // TMEM columns of a stage's scales
  static constexpr int kGroups = kRows / 16;                                  // groups of 16 columns, as the epilogue takes them
  static constexpr int kAccBufs = kRows <= 96 ? 2 : 1;
  static constexpr int kScaleCol0 = kAccBufs * 2 * kRows;
  static constexpr int kStoreBytes = kSwiglu ? 0 : 4 * kStoreBuf;
  static constexpr int kFitSmem = (227 * 1024 - 1024 - (int)sizeof(MxShared) - kStoreBytes) / kStageBytes, kFitTmem = (512 - kScaleCol0) / kScaleCols;
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

// shared-memory descriptor of a scale block: 32 rows of 16 bytes, unswizzled, 8-row groups 128 bytes apart
__device__ __forceinline__ unsigned long long scale_desc(unsigned saddr) {
  return (unsigned long long)((saddr & 0x3ffffu) >> 4) | 8ull << 16 | 8ull << 32 | 1ull << 46;
}
// (of a pair: in both CTAs, each from its own shared memory into its own TMEM)
template <bool kPair>
__device__ __forceinline__ void copy_scales(unsigned tmem, unsigned saddr) {
  if (kPair) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scale_desc(saddr)) : "memory");
  else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(scale_desc(saddr)) : "memory");
}
template <bool kPair>
__device__ __forceinline__ void mma_mxf4(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned sfa, unsigned sfb,
                                         unsigned accumulate) {
  if (kPair)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accumulate)
        : "memory");
}
// e2m1 operands, both K-major, power-of-two scales, M rows, N columns; half: which two of a block's four scales a row (K = 64 takes two)
__device__ __forceinline__ unsigned mx_idesc(unsigned m, unsigned n, unsigned half) {
  return 1u << 7 | 1u << 10 | (n >> 3) << 17 | 1u << 23 | (m >> 4) << 24 | (2u * half) << 4 | (2u * half) << 29;
}
// 16 bytes of a row's scales, `left` of which are there (the others are not used), by loads of vec bytes
__device__ __forceinline__ uint4 load_scales(const unsigned char* p, int left, int vec) {
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (vec == 16) {
    if (left > 0) v = __ldg(reinterpret_cast<const uint4*>(p));
  } else if (vec == 8) {
    const uint2* q = reinterpret_cast<const uint2*>(p);
    uint2 a = make_uint2(0u, 0u), b = a;
    if (left > 0) a = __ldg(q);
    if (left > 8) b = __ldg(q + 1);
    v = make_uint4(a.x, a.y, b.x, b.y);
  } else {
    const unsigned* q = reinterpret_cast<const unsigned*>(p);
    if (left > 0) v.x = __ldg(q);
    if (left > 4) v.y = __ldg(q + 1);
    if (left > 8) v.z = __ldg(q + 2);
    if (left > 12) v.w = __ldg(q + 3);
  }
  return v;
}
__device__ __forceinline__ void st_word(unsigned saddr, unsigned v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(saddr), "r"(v) : "memory"); }

// eight codes, the first in the lowest bits
__device__ __forceinline__ unsigned mx_codes8(const float* q) {
  unsigned r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r)
      : "f"(q[0]), "f"(q[1]), "f"(q[2]), "f"(q[3]), "f"(q[4]), "f"(q[5]), "f"(q[6]), "f"(q[7]));
  return r;
}
__device__ __forceinline__ unsigned max_u16x2(unsigned a, unsigned b) {
  unsigned r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ unsigned min_u16x2(unsigned a, unsigned b) {
  unsigned r;
  asm("min.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Exponent fields (bits 7 to 14) of the largest of the 32 lanes' v[r], in the low half, and of their v[r + 8], in the high half, for r = lane % 8.  The
// upper halves of floats as pairs of 16 bits; three steps halve the pairs that a lane follows, two more join the lanes of equal r.  (With
// sixteen reductions over the warp, and more rows handed on as they are, both products in turn took 851 us for 65 536 rows, 830 so.)
__device__ __forceinline__ unsigned block_exponents(const float (&v)[16], int lane) {
  unsigned p[8];
#pragma unroll
  for (int r = 0; r < 8; ++r) p[r] = __byte_perm(__float_as_uint(v[r]), __float_as_uint(v[r + 8]), 0x7632) & 0x7f807f80u;
#pragma unroll
  for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
    for (int r = 0; r < s; ++r) {
      const bool upper = lane & s;
      const unsigned other = __shfl_xor_sync(0xffffffffu, upper ? p[r] : p[r + s], s);
      p[r] = max_u16x2(upper ? p[r + s] : p[r], other);
    }
  p[0] = max_u16x2(p[0], __shfl_xor_sync(0xffffffffu, p[0], 8));
  return max_u16x2(p[0], __shfl_xor_sync(0xffffffffu, p[0], 16));
}
// 8 x 8 four-bit values over eight neighbouring lanes: lane i gives value j of word i, gets value i of word j
__device__ __forceinline__ unsigned transpose_nibbles(unsigned v, int lane) {
  v = __byte_perm(v, __shfl_xor_sync(0xffffffffu, v, 4), lane & 4 ? 0x3276 : 0x5410);
  v = __byte_perm(v, __shfl_xor_sync(0xffffffffu, v, 2), lane & 2 ? 0x3715 : 0x6240);
  const unsigned other = __shfl_xor_sync(0xffffffffu, v, 1), theirs = lane & 1 ? 0x0f0f0f0fu : 0xf0f0f0f0u;
  return (v & ~theirs) | (__funnelshift_l(other, other, lane & 1 ? 28 : 4) & theirs);
}

// 16 TMEM lanes x 16 columns as fragments: for column group j (8 columns) thread i holds row i / 4, columns 8 j + 2 (i % 4) and + 1 in r[4 j],
// r[4 j + 1], and the same columns of row i / 4 + 8 in r[4 j + 2], r[4 j + 3]
__device__ __forceinline__ void tc_ld_frag16(unsigned taddr, unsigned (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ unsigned short ld_shared2(unsigned saddr) {
  unsigned short v;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(saddr) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_shared16(unsigned saddr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(saddr) : "memory");
  return v;
}

template <int kRows_, bool kSwiglu, bool kPair>
__global__ void __launch_bounds__(kMxThreads, 1) mx_product_kernel(const __grid_constant__ MxArgs a) {
  using S = Shape<kRows_, kSwiglu, kPair>;
  extern __shared__ unsigned char raw[];
  unsigned char* stages = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
  unsigned char* store_bufs = stages + S::kStages * S::kStageBytes;
  MxShared& s = *reinterpret_cast<MxShared*>(store_bufs + S::kStoreBytes);
  const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31;
  constexpr int kCtas = kPair ? 2 : 1;
  constexpr int kStep = (kSwiglu ? 1 : 2) * kHalfRows * kCtas;     // output columns of a tile
  const unsigned rank = kPair ? cluster_ctarank() : 0u;            // weight rows of an accumulator: this CTA has the rank-th 128
  const int unit = (int)blockIdx.x / kCtas, n_units = (int)gridDim.x / kCtas;
  const int n_blocks = ((kSwiglu ? a.I : a.N) + kStep - 1) / kStep;

  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(&s.full[i], kCtas);
      mbar_init(&s.landed[i], kScaleWarps * kCtas);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 8 * kCtas);
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
  for (int e = tid; e <= a.E; e += kMxThreads) s.first_row[e] = min(max(a.offsets[e], 0), a.R);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0) list_tiles<S::kRows>(s, a.E, n_blocks, lane);
  __syncthreads();
  if (kPair) cluster_sync_all();          // the other CTA's barriers exist before anything arrives on them
  const unsigned tmem = s.tmem;
  const int n_tiles = uniform(s.first_tile[a.E]);
  const int n_stages = (a.K + kStageK - 1) / kStageK;

  if (warp < kTmaWarp) {
    if (S::kRows > 96) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    const int quad = warp & 3, half = warp >> 2;
    unsigned k = 0, stored = 0;  // tiles, groups of outputs so far
    bool ok = true;
    for (int t = unit; t < n_tiles; t += n_units, ++k) {
      const Tile at = uniform(tile_at<S::kRows>(s, a.E, t, kStep));
      const unsigned buf = k % S::kAccBufs, use = k / S::kAccBufs;
      if (ok) ok = __all_sync(0xffffffffu, wait(&s.acc_full[buf], use & 1, &s.dead));
      tc_fence_after();
      const unsigned acc = tmem + buf * 2 * S::kRows + ((unsigned)quad << 21);      // this warp's 32 lanes
      // Everything that is in the accumulator goes to registers first -- as bf16 for the plain product, for swiglu the last rows as they
      // are and the others as silu(gate) up -- and the accumulator is handed back: rounding, quantising and storing run beside the next tile's MMAs.
      const auto hand_back = [&] {
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0 && ok) {   // (what was waited for in vain others may still read)
          if (kPair) mbar_arrive_cluster(map_to_cta(&s.acc_empty[buf], 0));
          else mbar_arrive(&s.acc_empty[buf]);
        }
      };
      const int groups = uniform((at.rows + 15) / 16);
      if (!kSwiglu) {            // warps 0-3 have the first accumulator, 4-7 the second
        const unsigned mine = acc + half * S::kRows;
        const int col0 = at.n0 + (half * kCtas + (int)rank) * kHalfRows;      // of these four warps' 128 output columns
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (size_t)at.row0 * a.N + col0;
        unsigned v[S::kGroups][8];   // a group as eight 8 x 8 fragments: [4 j + m] rows 8 j .. of the group, columns 8 m ..
#pragma unroll
        for (int g = 0; g < S::kGroups; ++g) {
          if (g >= groups) break;
          unsigned lo[8], hi[8];
          tc_ld_frag16(mine + 16 * g, lo);
          tc_ld_frag16(mine + 16 * g + (16u << 16), hi);
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
              v[g][4 * j + m] = ok ? pack_bf16(lo[4 * j + 2 * m], lo[4 * j + 2 * m + 1]) : 0x7fff7fffu;
              v[g][4 * j + 2 + m] = ok ? pack_bf16(hi[4 * j + 2 * m], hi[4 * j + 2 * m + 1]) : 0x7fff7fffu;
            }
        }
        hand_back();
        // Transposed into shared memory, 16 rows of 256 bytes at a time, and out by 16 bytes a lane.  (65 536 rows of 4096 x 1792: 319 us; bulk copies of
        // a row each 343, the copy engine's rate of them bounds the launch; 32 rows at a time 320; each warp its own 64 bytes of the rows, with no barrier, 345.)
        const int cols = min(kHalfRows, a.N - col0);
        const auto stage = [&](int g) {
          const unsigned buf_at = smem_u32(store_bufs) + (2 * half + (stored++ & 1)) * kStoreBuf;
          const unsigned to = buf_at + (lane & 7) * kStorePitch + quad * 64 + (lane >> 3) * 16;
#pragma unroll
          for (int j = 0; j < 2; ++j) st_matrix4_trans(to + 8 * j * kStorePitch, v[g][4 * j], v[g][4 * j + 1], v[g][4 * j + 2], v[g][4 * j + 3]);
          asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");     // the other buffer, which the next group goes to, has been read too
          return buf_at;
        };
        if (a.wide) {
#pragma unroll
          for (int g = 0; g < S::kGroups; ++g) {
            if (g >= groups) break;
            const unsigned from = stage(g);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int row = 4 * quad + 2 * h + (lane >> 4), c = 8 * (lane & 15);
              const uint4 x = ld_shared16(from + row * kStorePitch + 2 * c);
              if (16 * g + row < at.rows && c < cols) *reinterpret_cast<uint4*>(out + (size_t)(16 * g + row) * a.N + c) = x;
            }
          }
        } else {                 // (kept short: what is never executed costs too where it parts what is)
#pragma unroll
          for (int g = 0; g < S::kGroups; ++g) {
            if (g >= groups) break;
            const unsigned from = stage(g);
#pragma unroll 1
            for (int row = 4 * quad; row < min(4 * quad + 4, at.rows - 16 * g); ++row) {
              unsigned short x[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = ld_shared2(from + row * kStorePitch + 64 * i + 2 * lane);
              unsigned short* to = reinterpret_cast<unsigned short*>(out) + (size_t)(16 * g + row) * a.N + lane;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (32 * i + lane < cols) to[32 * i] = x[i];
            }
          }
        }
      } else {                   // warps 0-3 and 4-7 take turns at groups of 16 rows
        const int col = at.n0 + (int)rank * kHalfRows + quad * 32, per_row = a.I / kMxBlock;
        const auto store = [&](const float (&v)[16], int c) {
          const unsigned top = block_exponents(v, lane), inverse = min_u16x2(0x80008000u - top, 0x7f007f00u);     // of 2^(127 - scale byte)
          float q[16];
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const unsigned both = __shfl_sync(0xffffffffu, inverse, r);
            q[r] = v[r] * __uint_as_float(both << 16);
            q[r + 8] = v[r + 8] * __uint_as_float(both & 0xffff0000u);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const unsigned word = transpose_nibbles(mx_codes8(q + 8 * h), lane);         // lane 8 i + j: columns 8 i .. 8 i + 7 of row j
            const int row = c + 8 * h + (lane & 7);
            if (row < at.rows && col < a.I) {
              const size_t p = (size_t)(at.row0 + row);
              *reinterpret_cast<unsigned*>(static_cast<unsigned char*>(a.out) + p * (a.I / 2) + col / 2 + (lane >> 3) * 4) = word;
              if (lane < 8) a.out_scales[p * per_row + col / kMxBlock] = (unsigned char)(ok ? mx_scale_byte((h ? top : top << 16) & 0x7f800000u) : 255u);
            }
          }
        };
        constexpr int kFirst = (S::kGroups + 1) / 2 - 1;
        const int my_groups = (groups - half + 1) / 2;
        float v[kFirst][16];
        unsigned gate[16], up[16];
        const auto load = [&](unsigned (&g)[16], unsigned (&u)[16], int i) {
          tc_ld16(acc + 16 * (half + 2 * i), g);
          tc_ld16(acc + S::kRows + 16 * (half + 2 * i), u);
        };
        const auto activate = [&](const unsigned (&g)[16], const unsigned (&u)[16], float (&to)[16]) {
#pragma unroll
          for (int j = 0; j < 16; ++j) to[j] = silu_times(__uint_as_float(g[j]), __uint_as_float(u[j]));
        };
#pragma unroll
        for (int i = 0; i < kFirst; ++i)
          if (i < my_groups) {
            unsigned g[16], u[16];
            load(g, u, i);
            tc_wait_ld();
            activate(g, u, v[i]);
          }
        if (kFirst < my_groups) load(gate, up, kFirst);
        hand_back();
#pragma unroll
        for (int i = 0; i < kFirst; ++i)
          if (i < my_groups) store(v[i], 16 * (half + 2 * i));
        if (kFirst < my_groups) {
          float w[16];
          activate(gate, up, w);
          store(w, 16 * (half + 2 * kFirst));
        }
      }
    }
    // rows that belong to no expert: zeros, by the epilogue warps of the whole grid
    const size_t width = kSwiglu ? (size_t)a.I / 32 * 17 : (size_t)a.N;
    const int lo = s.first_row[0], hi = s.first_row[a.E], none = lo + (a.R - hi);
    for (int i = blockIdx.x; i < none; i += gridDim.x) {
      const size_t p = (size_t)(i < lo ? i : hi + (i - lo));
#pragma unroll 1
      for (size_t c = tid; c < width; c += 256) {
        if (!kSwiglu) static_cast<__nv_bfloat16*>(a.out)[p * a.N + c] = __float2bfloat16_rn(0.f);
        else if (c < (size_t)a.I / 2) static_cast<unsigned char*>(a.out)[p * (a.I / 2) + c] = 0;
        else a.out_scales[p * (a.I / 32) + (c - a.I / 2)] = 0;
      }
    }
  } else if (warp < kScaleWarp) {
    if (S::kRows > 96) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == kTmaWarp) {
      if (elect_one()) {
        unsigned n = 0;            // stages so far
        for (int t = unit; t < n_tiles && !s.dead; t += n_units) {
          const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
          // of a pair each CTA has half of the rows
          const int mine = kPair ? (at.rows + 31) / 32 * 16 : at.rows, row0 = at.row0 + (int)rank * mine, boxes = (mine + kBoxRows - 1) / kBoxRows;
          const bool second = kSwiglu || at.n0 + kHalfRows * kCtas < a.N;
          const unsigned long long policy = at.alone ? l2_evict_first() : l2_evict_normal();
          const int n0 = at.n0 + (int)rank * kHalfRows;
#pragma unroll 1
          for (int i = 0; i < n_stages; ++i, ++n) {
            const unsigned slot = n % S::kStages, round = n / S::kStages;
            if (round && !wait(&s.empty[slot], (round - 1) & 1, &s.dead)) break;
            const unsigned to = smem_u32(stages + slot * S::kStageBytes);
            const unsigned bar = kPair ? map_to_cta(&s.full[slot], 0) : smem_u32(&s.full[slot]);
            expect_tx(bar, (second ? S::kWBytes : S::kWBytes / 2) + boxes * kBoxRows * 128);
            tma_3d<kPair>(to, &a.tm_w, i * 128, n0, at.expert, bar, policy);
            if (second) tma_3d<kPair>(to + kHalfRows * 128, &a.tm_w, i * 128, n0 + (kSwiglu ? a.I : kHalfRows * kCtas), at.expert, bar, policy);
#pragma unroll 1
            for (int b = 0; b < boxes; ++b) tma_2d<kPair>(to + S::kWBytes + b * kBoxRows * 128, &a.tm_x, i * 128, row0 + b * kBoxRows, bar);
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
        unsigned n = 0, k = 0;     // stages, tiles so far
        bool ok = true;
        for (int t = unit; t < n_tiles && ok; t += n_units, ++k) {
          const Tile at = tile_at<S::kRows>(s, a.E, t, kStep);
          const unsigned buf = k % S::kAccBufs, use = k / S::kAccBufs;
          if (use) ok = wait<kPair ? mbar_try_cluster : mbar_try>(&s.acc_empty[buf], (use - 1) & 1, &s.dead);
          if (!ok) break;
          tc_fence_after();
          const unsigned cols = kPair ? (unsigned)(at.rows + 31) & ~31u : (unsigned)(at.rows + 15) & ~15u;
          const bool second = kSwiglu || at.n0 + kHalfRows * kCtas < a.N;
          const unsigned acc = tmem + buf * 2 * S::kRows;
#pragma unroll 1
          for (int i = 0; i < n_stages; ++i, ++n) {
            const unsigned slot = n % S::kStages, round = n / S::kStages;
            ok = wait(&s.full[slot], round & 1, &s.dead) && wait<kPair ? mbar_try_relaxed : mbar_try>(&s.landed[slot], round & 1, &s.dead);
            if (!ok) break;
            if (kPair) fence_acquire_pair_smem();
            tc_fence_after();
            const unsigned st = smem_u32(stages + slot * S::kStageBytes);
            const unsigned sc = st + S::kWBytes + S::kXBytes, tsc = tmem + S::kScaleCol0 + slot * S::kScaleCols;
            const int groups = min(2, (a.K - i * kStageK) / kGroupK);
#pragma unroll 1
            for (int g = 0; g < groups; ++g) {
              const unsigned from = sc + g * (2 + S::kRowBlocks) * kScaleBlock, to = tsc + g * (2 + S::kRowBlocks) * 4;
#pragma unroll
              for (int b = 0; b < 2 + S::kRowBlocks; ++b) copy_scales<kPair>(to + 4 * b, from + b * kScaleBlock);
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const unsigned step = (2 * g + h) * 32;       // 64 columns, 32 bytes
                const unsigned long long xd = umma_desc(st + S::kWBytes + step, 128);
                const unsigned idesc = mx_idesc(kHalfRows * kCtas, cols, h), first = (i | g | h) != 0;
                mma_mxf4<kPair>(acc, umma_desc(st + step, 128), xd, idesc, to, to + 8, first);
                if (second) mma_mxf4<kPair>(acc + S::kRows, umma_desc(st + kHalfRows * 128 + step, 128), xd, idesc, to + 4, to + 8, first);
              }
            }
            commit(&s.empty[slot]);
          }
          if (ok) commit(&s.acc_full[buf]);
        }
        commit(&s.drained);     // nothing of this block's is left in the tensor core when it frees its TMEM
        const unsigned long long start = gtime_ns();
        while (!mbar_try(&s.drained, 0) && gtime_ns() - start < kWaitNs) {}
      }
      __syncwarp();
    }
  } else {
    if (S::kRows > 96) asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    // Two neighbouring lanes have a row: together they load a sector of 32 bytes, four stages, two each; the next sector is on its way to registers
    // meanwhile, whether or not its stages are free.  A thread has two rows of every 128-row block, in the order that spreads a warp's stores over
    // the banks: the four bytes of a group of 128 columns of row r go to 16 (r % 32) + 4 (r / 32) of the group's block.
    const int pair = lane & 1, r0 = 32 * (lane >> 1 & 3) + 4 * (warp - kScaleWarp) + (lane >> 3);      // and r0 + 16
    const unsigned spot = (unsigned)(r0 & 31) * 16 + (unsigned)(r0 >> 5) * 4;
    const int per_row = a.K / kMxBlock, n_quads = (n_stages + 3) / 4;
    const int places = per_row | (int)(size_t)a.w_scales | (int)(size_t)a.x_scales;
    const int vec = places % 16 == 0 ? 16 : places % 8 == 0 ? 8 : 4;
    constexpr int kBlocks = 2 + S::kRowBlocks;
    struct Quad {
      uint4 b[kBlocks][2];
      int stages;                // 1 to 4; 0: there is no more
    };
    int t = unit, quad = 0;
    Tile at{};
    unsigned n = 0;
    const auto fetch = [&](Quad& p) {
      p.stages = 0;
      if (t >= n_tiles) return;
      if (quad == 0) at = tile_at<S::kRows>(s, a.E, t, kStep);
      const int from = quad * 32 + pair * 16, left = per_row - from;
      const unsigned char* w = a.w_scales + (size_t)at.expert * a.N * per_row + from;
      const unsigned char* x = a.x_scales + (size_t)at.row0 * per_row + from;
      const auto rows = [&](const int bytes) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int r = r0 + 16 * q;
#pragma unroll
          for (int b = 0; b < 2; ++b) {    // a weight row behind the last one: any other's scales (its products are not stored)
            const int row = kSwiglu ? min(at.n0 + (int)rank * kHalfRows + r, a.I - 1) + b * a.I
                                    : min(at.n0 + (b * kCtas + (int)rank) * kHalfRows + r, a.N - 1);
            p.b[b][q] = load_scales(w + (size_t)row * per_row, left, bytes);
          }
#pragma unroll
          for (int b = 0; b < S::kRowBlocks; ++b) p.b[2 + b][q] = load_scales(x + (size_t)min(b * 128 + r, at.rows - 1) * per_row, left, bytes);
        }
      };
      if (vec == 16) rows(16);
      else if (vec == 8) rows(8);
      else rows(4);
      p.stages = min(4, n_stages - 4 * quad);
      if (++quad == n_quads) {
        quad = 0;
        t += n_units;
      }
    };
    const auto put = [&](const Quad& p) {    // false: gave up
#pragma unroll 1
      for (int h = 0; h < p.stages; ++h) {
        const unsigned slot = n % S::kStages, round = n / S::kStages;
        if (round && !__all_sync(0xffffffffu, wait(&s.empty[slot], (round - 1) & 1, &s.dead))) return false;
        if (pair == h / 2) {
          const unsigned to = smem_u32(stages + slot * S::kStageBytes) + S::kWBytes + S::kXBytes + spot;
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const uint4& v = p.b[b][q];
              st_word(to + b * kScaleBlock + 256 * q, h & 1 ? v.z : v.x);
              st_word(to + (kBlocks + b) * kScaleBlock + 256 * q, h & 1 ? v.w : v.y);
            }
          fence_async_proxy_smem();
        }
        __syncwarp();
        if (lane == 0) {
          if (kPair) {           // the leader's MMAs read this CTA's scales too: fences of shared memory alone (65 536 rows 434 us; an arrival and a wait that order all memory 707)
            fence_release_own_smem();
            mbar_arrive_relaxed(map_to_cta(&s.landed[slot], 0));
          } else {
            mbar_arrive(&s.landed[slot]);
          }
        }
        ++n;
      }
      return true;
    };
    Quad now, next;
    now.stages = 0;
#pragma unroll 1
    do {
      fetch(next);
      if (!put(now)) break;
      now = next;
    } while (now.stages);
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

template <int kRows, bool kSwiglu, bool kPair>
cudaError_t product_launch(const MxArgs& a, cudaStream_t stream) {
  using S = Shape<kRows, kSwiglu, kPair>;
  constexpr size_t smem = 1024 + (size_t)S::kStages * S::kStageBytes + S::kStoreBytes + sizeof(MxShared);
  static_assert(smem <= 227 * 1024, "shared memory");
  constexpr int kCtas = kPair ? 2 : 1;
  auto* kernel = mx_product_kernel<kRows, kSwiglu, kPair>;
  int dev = 0, sms = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  // most tiles that the rows can make
  const int step = (kSwiglu ? 1 : 2) * kHalfRows * kCtas;
  const long long m_tiles = a.R / kRows + (a.R < a.E ? a.R : a.E), tiles = m_tiles * (((kSwiglu ? a.I : a.N) + step - 1) / step);
  if (tiles > 0x3fffffffll) return cudaErrorInvalidValue;
  const int units = tiles < sms / kCtas ? (int)tiles : sms / kCtas;
  if (!kPair) return launch_after(kernel, units, kMxThreads, smem, stream, a);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)units * 2);
  cfg.blockDim = dim3((unsigned)kMxThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <bool kSwiglu>
int product(const void* codes, const void* scales, const void* w_codes, const void* w_scales, const int32_t* offsets, int n_rows, int n_experts,
            int n, int K, void* out, void* out_scales, void* stream) {
  if (n_rows < 0 || n_rows >= 1 << kRowSlotShift || n_experts < 1 || n_experts > kMaxExperts || n < 1 || n > 1 << 30 || K < kGroupK ||
      K > 1 << 30 || K % kGroupK)
    return MOE_EINVAL;
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
  // The tile's height goes by the rows that an expert gets on average (the host does not know more); the line lies where high tiles stop losing on uneven
  // loads, which costs even ones 9, 3 and 3 % of both products in turn at 128, 192 and 256 rows an expert.  Two buffers of 96 columns let the epilogue of a tile
  // run beside the next one's MMAs; 192 columns take the weights from L2 half as often, and for gate/up a pair of CTAs takes half of the rows each.
  // us (gate/up; down; both in turn), weights that are not in L2:
  //   rows an expert            64              128             192             256             320             384             512             1024
  //   even, 32 experts, 4096 x 1792
  //     96 rows                 50; 24; 81      73; 38; 112     87; 49; 136     106; 58; 163    132; 73; 205    150; 84; 234    197; 109; 306   356; 199; 556
  //     192 rows                54; 25; 88      60; 31; 103     75; 50; 132     96; 57; 159     99; 59; 166     113; 71; 189    139; 86; 231    248; 159; 415
  //   uneven (Zipf 0.8), 64 experts, 2048 x 768
  //     96 rows                 27; 16; 44      31; 22; 53      40; 28; 68      51; 34; 85      57; 41; 98      68; 47; 115     87; 58; 145     162; 108; 269
  //     192 rows                28; 18; 52      36; 23; 68      37; 27; 75      45; 32; 87      53; 39; 102     61; 44; 115     77; 54; 140     131; 94; 237
  // Gate/up without pairs takes 3-10 % longer (1024 rows: 128 for 122, 266 for 242), the down product on pairs 1-14 % (161 for 159, 107 for 94).  Tiles of
  // 64 and 32 rows are left out: 0-7 % faster below 32 rows an expert, up to 25 % slower at 64.
  const bool many = n_rows > 256ll * n_experts;
  const cudaError_t e = many ? product_launch<192, kSwiglu, kSwiglu>(a, st) : product_launch<96, kSwiglu, false>(a, st);
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
