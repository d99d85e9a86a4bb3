// moe_sort_rows / moe_merge_rows and their gradients: the rows of a batch laid out by expert and put together again, on the
// permutation that a plan left (flat_to_sorted and its inverse sorted_to_flat, R = T*k entries each).
//
//   sort        xs[f2s[t*k+j], :] = x[t, :]                  merge        y[t, :] = sum_j w[t,j] rows[f2s[t*k+j], :]
//   sort grad   dx[t, :] = sum_j dxs[f2s[t*k+j], :]          merge grad   drows[f2s[t*k+j], :] = w[t,j] dy[t, :]
//                                                                         dw[t,j] = <dy[t, :], rows[f2s[t*k+j], :]>
//
// All four are bound by memory: the R rows cross HBM once, and so do the T rows, because every kernel walks tokens: a token's row is
// read once and written (or added up) for all of its k slots.  Walking sorted rows instead reads a token's row k times, far apart
// in time, and a prefill chunk does not stay in L2 that long.  Sums are fp32 in slot order, rounded once; there are no
// atomics, so results do not depend on the schedule.  Addresses are 64 bits wide.  An entry of f2s outside [0, R) names no row: nothing is read
// or written for it; a row whose entry of s2f is outside [0, R) belongs to no token and is set to zero where rows are the output.
//
// Device time, bf16, and the rate of the bytes that have to move (a plain copy runs at 6.5 TB/s): 8 192 tokens x 8 slots x 4 096 columns sort 98 us
// (6.2 TB/s), its gradient 89 us (6.8); 4 096 x 8 x 6 144 merge 68 us (6.6), its gradient 134 us (6.4); 16 384 x 2 x 4 096 63 and 102 us; one token
// 2.2-2.5 us, launch included (gradient of merge 5.1).  8 192 x 8 rows of odd width (3 001) move at 2.6-4.4 TB/s: accesses of two bytes.
#include <cuda_fp16.h>

#include "moe_dev.cuh"

namespace moe {
namespace {

constexpr int kRowThreads = 256;

// kBytes of memory at a time: the widest that the row length, the strides and the addresses divide into
template <int kBytes> struct Unit;
template <> struct Unit<16> { using type = uint4; static __device__ uint4 zero() { return make_uint4(0u, 0u, 0u, 0u); } };
template <> struct Unit<8> { using type = uint2; static __device__ uint2 zero() { return make_uint2(0u, 0u); } };
template <> struct Unit<4> { using type = unsigned; static __device__ unsigned zero() { return 0u; } };
template <> struct Unit<2> { using type = unsigned short; static __device__ unsigned short zero() { return 0; } };
template <> struct Unit<1> { using type = unsigned char; static __device__ unsigned char zero() { return 0; } };

// Columns of one token's row for a thread: `tpt` threads share a token (a power of two), a block holds kRowThreads / tpt tokens and one of
// `slices` parts of their columns.
struct Walk {
  int tpt_log2, slices;
};
Walk walk_of(long long units, int per_thread) {
  Walk w{3, 1};
  while ((1 << w.tpt_log2) < kRowThreads && (long long)per_thread << w.tpt_log2 < units) ++w.tpt_log2;
  w.slices = (int)((units + ((long long)per_thread << w.tpt_log2) - 1) / ((long long)per_thread << w.tpt_log2));
  return w;
}
long long blocks_of(const Walk& w, int T) {
  const int tokens = kRowThreads >> w.tpt_log2;
  return ((long long)T + tokens - 1) / tokens * w.slices;
}
__device__ __forceinline__ int my_token(const Walk& w) {
  return (int)(blockIdx.x / (unsigned)w.slices) * (kRowThreads >> w.tpt_log2) + (int)(threadIdx.x >> w.tpt_log2);
}
__device__ __forceinline__ int my_column(const Walk& w, int per_thread) {
  return (int)(blockIdx.x % (unsigned)w.slices) * (per_thread << w.tpt_log2) + (int)(threadIdx.x & ((1u << w.tpt_log2) - 1));
}

// ------------------------------------------------------------------ sort
template <int kBytes, int kPer>
__global__ void __launch_bounds__(kRowThreads)
sort_rows_kernel(const typename Unit<kBytes>::type* __restrict__ x, long long x_stride, typename Unit<kBytes>::type* __restrict__ xs,
                 const int* __restrict__ s2f, const int* __restrict__ f2s, int T, int k, int units, Walk walk) {
  grid_dep_wait();
  const int t = my_token(walk), c0 = my_column(walk, kPer), step = 1 << walk.tpt_log2;
  if (t >= T) return;
  const unsigned R = (unsigned)T * (unsigned)k;
  typename Unit<kBytes>::type v[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (c0 + i * step < units) v[i] = x[t * x_stride + c0 + i * step];
  const int* mine = f2s + (size_t)t * k;
  const int* rows = s2f + (size_t)t * k;      // every row of the result is some token's to look after
#pragma unroll 4
  for (int j = 0; j < k; ++j) {
    const unsigned p = (unsigned)mine[j];
    if (p < R) {
      typename Unit<kBytes>::type* to = xs + (size_t)p * units + c0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (c0 + i * step < units) to[i * step] = v[i];
    }
    if ((unsigned)rows[j] >= R) {
      typename Unit<kBytes>::type* to = xs + ((size_t)t * k + j) * units + c0;
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (c0 + i * step < units) to[i * step] = Unit<kBytes>::zero();
    }
  }
}

// ------------------------------------------------------------------ elements
// kV neighbouring elements of a row: one 16-byte access, or a single element where rows are not 16-byte aligned.  Registers hold them as they
// lie in memory until they are used: as arrays of 16-bit elements they took a register each, and two blocks an SM instead of four (merge of
// 4 096 x 8 x 6 144 107 us instead of 68).
template <class E, int kV> struct Vec;
template <> struct Vec<float, 4> {
  using Raw = float4;
  static __device__ __forceinline__ Raw zero() { return make_float4(0.f, 0.f, 0.f, 0.f); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
  static __device__ __forceinline__ Raw pack(const float (&v)[4]) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<__half, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
  static __device__ __forceinline__ void two(unsigned w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x;
    b = f.y;
  }
  static __device__ __forceinline__ unsigned one(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[8]) { two(r.x, v[0], v[1]); two(r.y, v[2], v[3]); two(r.z, v[4], v[5]); two(r.w, v[6], v[7]); }
  static __device__ __forceinline__ Raw pack(const float (&v)[8]) { return make_uint4(one(v[0], v[1]), one(v[2], v[3]), one(v[4], v[5]), one(v[6], v[7])); }
};
template <> struct Vec<__nv_bfloat16, 8> {
  using Raw = uint4;
  static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
  static __device__ __forceinline__ void two(unsigned w, float& a, float& b) {
    a = __uint_as_float(w << 16);
    b = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ unsigned one(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const unsigned*>(&h);
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[8]) { two(r.x, v[0], v[1]); two(r.y, v[2], v[3]); two(r.z, v[4], v[5]); two(r.w, v[6], v[7]); }
  static __device__ __forceinline__ Raw pack(const float (&v)[8]) { return make_uint4(one(v[0], v[1]), one(v[2], v[3]), one(v[4], v[5]), one(v[6], v[7])); }
};
// two elements: rows that are aligned to two only
template <> struct Vec<float, 2> {
  using Raw = float2;
  static __device__ __forceinline__ Raw zero() { return make_float2(0.f, 0.f); }
  static __device__ __forceinline__ void unpack(const Raw& r, float (&v)[2]) { v[0] = r.x; v[1] = r.y; }
  static __device__ __forceinline__ Raw pack(const float (&v)[2]) { return make_float2(v[0], v[1]); }
};
template <> struct Vec<__half, 2> {
  using Raw = unsigned;
  static __device__ __forceinline__ Raw zero() { return 0u; }
  static __device__ __forceinline__ void unpack(Raw r, float (&v)[2]) { Vec<__half, 8>::two(r, v[0], v[1]); }
  static __device__ __forceinline__ Raw pack(const float (&v)[2]) { return Vec<__half, 8>::one(v[0], v[1]); }
};
template <> struct Vec<__nv_bfloat16, 2> {
  using Raw = unsigned;
  static __device__ __forceinline__ Raw zero() { return 0u; }
  static __device__ __forceinline__ void unpack(Raw r, float (&v)[2]) { Vec<__nv_bfloat16, 8>::two(r, v[0], v[1]); }
  static __device__ __forceinline__ Raw pack(const float (&v)[2]) { return Vec<__nv_bfloat16, 8>::one(v[0], v[1]); }
};
template <> struct Vec<float, 1> {
  using Raw = float;
  static __device__ __forceinline__ Raw zero() { return 0.f; }
  static __device__ __forceinline__ void unpack(Raw r, float (&v)[1]) { v[0] = r; }
  static __device__ __forceinline__ Raw pack(const float (&v)[1]) { return v[0]; }
};
template <> struct Vec<__half, 1> {
  using Raw = __half;
  static __device__ __forceinline__ Raw zero() { return __float2half_rn(0.f); }
  static __device__ __forceinline__ void unpack(Raw r, float (&v)[1]) { v[0] = __half2float(r); }
  static __device__ __forceinline__ Raw pack(const float (&v)[1]) { return __float2half_rn(v[0]); }
};
template <> struct Vec<__nv_bfloat16, 1> {
  using Raw = __nv_bfloat16;
  static __device__ __forceinline__ Raw zero() { return __float2bfloat16_rn(0.f); }
  static __device__ __forceinline__ void unpack(Raw r, float (&v)[1]) { v[0] = __bfloat162float(r); }
  static __device__ __forceinline__ Raw pack(const float (&v)[1]) { return __float2bfloat16_rn(v[0]); }
};

// ------------------------------------------------------------------ merge, and the gradient of sort (kWeights = false)
// A thread owns kPer times kV columns of a token and has kSlots of its rows in flight at a time; a slot without a row adds 0.
template <class E, int kV, int kSlots, int kPer, bool kWeights>
__global__ void __launch_bounds__(kRowThreads, kPer > 1 && kV > 1 ? 3 : 4)
merge_rows_kernel(const E* __restrict__ rows, long long stride, const float* __restrict__ w, const int* __restrict__ f2s,
                  E* __restrict__ y, int T, int k, int H, Walk walk) {
  grid_dep_wait();
  using V = Vec<E, kV>;
  const int t = my_token(walk), c = my_column(walk, kPer) * kV, step = kV << walk.tpt_log2;
  if (t >= T || c >= H) return;
  const unsigned R = (unsigned)T * (unsigned)k;
  const E* from = rows + c;
  float acc[kPer][kV];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int n = 0; n < kV; ++n) acc[i][n] = 0.f;
  for (int j0 = 0; j0 < k; j0 += kSlots) {
    typename V::Raw d[kSlots][kPer];
    unsigned p[kSlots];
    float wj[kSlots];
#pragma unroll
    for (int b = 0; b < kSlots; ++b) p[b] = j0 + b < k ? (unsigned)f2s[(size_t)t * k + j0 + b] : R;
#pragma unroll
    for (int b = 0; b < kSlots; ++b) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        d[b][i] = V::zero();
        if (p[b] < R && c + i * step < H) d[b][i] = *reinterpret_cast<const typename V::Raw*>(from + p[b] * stride + i * step);
      }
      wj[b] = 0.f;
      if (kWeights && p[b] < R) wj[b] = w[(size_t)t * k + j0 + b];
    }
#pragma unroll
    for (int b = 0; b < kSlots; ++b)
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        float v[kV];
        V::unpack(d[b][i], v);
#pragma unroll
        for (int n = 0; n < kV; ++n) acc[i][n] = kWeights ? fmaf(wj[b], v[n], acc[i][n]) : acc[i][n] + v[n];
      }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    if (c + i * step < H) *reinterpret_cast<typename V::Raw*>(y + (size_t)t * H + c + i * step) = V::pack(acc[i]);
}

// ------------------------------------------------------------------ gradient of merge
// A group of 32 to 256 threads owns a token: its threads share the columns, every one of them keeps the partial dot products of kSlots slots,
// and the group adds them up in a fixed order.  Each row of `rows` is read once and each row of drows written once; dy is read once for kSlots
// slots (from L1 again for the next ones).
template <class E, int kV, int kSlots, int kPer>
__global__ void __launch_bounds__(kRowThreads, 4)
merge_grad_kernel(const E* __restrict__ dy, long long dy_stride, const E* __restrict__ rows, long long stride, const float* __restrict__ w,
                  const int* __restrict__ s2f, const int* __restrict__ f2s, E* __restrict__ drows, float* __restrict__ dw, int T, int k, int H,
                  int group) {
  grid_dep_wait();
  using V = Vec<E, kV>;
  using Raw = typename V::Raw;
  __shared__ float part[kRowThreads / 32][kSlots];
  const int groups = kRowThreads / group, tid = threadIdx.x & (group - 1), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x * groups + (int)threadIdx.x / group, step = group * kV;
  const bool on = t < T;                               // (a group without a token takes part in the barriers)
  const unsigned R = (unsigned)T * (unsigned)k;
  const E* g_row = dy + t * dy_stride;
  // lane j has slot j, and row t k + j of the result to look after
  const size_t mine = (size_t)t * k + lane;
  const unsigned my_row = on && lane < k ? (unsigned)f2s[mine] : R;
  const float my_w = my_row < R ? w[mine] : 0.f;
  unsigned lost = __ballot_sync(0xffffffffu, on && lane < k && (unsigned)s2f[mine] >= R);
  for (int j0 = 0; j0 < k; j0 += kSlots) {
    unsigned p[kSlots];
    float wj[kSlots], dot[kSlots];
#pragma unroll
    for (int b = 0; b < kSlots; ++b) {
      p[b] = __shfl_sync(0xffffffffu, my_row, j0 + b);          // (lanes from k on have none; j0 + b < 32)
      wj[b] = __shfl_sync(0xffffffffu, my_w, j0 + b);
      dot[b] = 0.f;
    }
    for (int c = tid * kV; on && c < H; c += kPer * step) {
      Raw graw[kPer], d[kSlots][kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (c + i * step < H) graw[i] = *reinterpret_cast<const Raw*>(g_row + c + i * step);
#pragma unroll
      for (int b = 0; b < kSlots; ++b)
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (p[b] < R && c + i * step < H) d[b][i] = *reinterpret_cast<const Raw*>(rows + p[b] * stride + c + i * step);
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (c + i * step < H) {
          float g[kV];
          V::unpack(graw[i], g);
#pragma unroll
          for (int b = 0; b < kSlots; ++b)
            if (p[b] < R) {
              float v[kV], out[kV];
              V::unpack(d[b][i], v);
#pragma unroll
              for (int n = 0; n < kV; ++n) {
                dot[b] = fmaf(g[n], v[n], dot[b]);
                out[n] = wj[b] * g[n];
              }
              *reinterpret_cast<Raw*>(drows + (size_t)p[b] * H + c + i * step) = V::pack(out);
            }
        }
    }
    // kSlots sums over 32 lanes: lanes halve the set of slots that they keep while they add
    int b = 16;
#pragma unroll
    for (int s = kSlots / 2; s >= 1; s >>= 1, b >>= 1) {
      const bool high = lane & b;
#pragma unroll
      for (int i = 0; i < s; ++i) {
        const float give = high ? dot[i] : dot[i + s], keep = high ? dot[i + s] : dot[i];
        dot[i] = keep + __shfl_xor_sync(0xffffffffu, give, b);
      }
    }
    constexpr int kSame = 32 / kSlots;                // neighbouring lanes that now have the same slot
#pragma unroll
    for (int m = kSame / 2; m >= 1; m >>= 1) dot[0] += __shfl_xor_sync(0xffffffffu, dot[0], m);
    const bool first = (lane & (kSame - 1)) == 0;     // lane kSame * b has the sum of slot b
    if (group == 32) {
      if (on && first && j0 + lane / kSame < k) dw[(size_t)t * k + j0 + lane / kSame] = dot[0];      // 0 for a slot that names no row
      continue;
    }
    if (j0) __syncthreads();                          // the sums of the slots before have been read
    if (first) part[warp][lane / kSame] = dot[0];
    __syncthreads();
    if (on && tid < kSlots && j0 + tid < k) {
      float sum = 0.f;
      for (int i = 0; i < group / 32; ++i) sum += part[warp + i][tid];    // (tid < 32: the group's first warp)
      dw[(size_t)t * k + j0 + tid] = sum;
    }
  }
  for (; lost; lost &= lost - 1)                      // rows that belong to no token
    for (int c = tid * kV; c < H; c += step) *reinterpret_cast<Raw*>(drows + ((size_t)t * k + (__ffs(lost) - 1)) * H + c) = V::zero();
}

// ------------------------------------------------------------------ host
int element_bytes(int dtype) {
  return dtype == MOE_DTYPE_FP32 ? 4 : dtype == MOE_DTYPE_BF16 || dtype == MOE_DTYPE_FP16 ? 2 : dtype == MOE_DTYPE_FP8_E4M3 ? 1 : 0;
}
// sizes shared by the four calls; MOE_OK with *empty set where there is nothing to do
int check_sizes(int T, int k, int H, int dtype, bool bytes_ok, bool* empty) {
  if (T < 0 || k < 1 || k > 32 || H < 1 || H > 1 << 30) return MOE_EINVAL;
  if (!element_bytes(dtype) || (dtype == MOE_DTYPE_FP8_E4M3 && !bytes_ok)) return MOE_EINVAL;
  if ((long long)T * k >= (1ll << kRowSlotShift)) return MOE_EINVAL;        // as in a context
  *empty = T == 0;
  return MOE_OK;
}
bool element_aligned(int) { return true; }
template <class... More>
bool element_aligned(int el, const void* p, More... more) {
  return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(el - 1)) == 0 && element_aligned(el, more...);
}
// widest access (16, 8, 4, 2 or 1 bytes) that divides all of these
int widest(unsigned long long all) {
  int b = 16;
  while (all & (unsigned long long)(b - 1)) b >>= 1;
  return b;
}
unsigned long long bits(const void* p) { return reinterpret_cast<uintptr_t>(p); }

constexpr long long kFillThreads = 148ll * 2048 * 4;     // accesses that keep every thread of the GPU busy with four

template <int kBytes>
cudaError_t sort_launch(const void* x, long long x_stride_bytes, void* xs, const int* s2f, const int* f2s, int T, int k, long long row_bytes,
                        cudaStream_t stream) {
  using U = typename Unit<kBytes>::type;
  const long long units = row_bytes / kBytes;
  // Four accesses a thread where there are rows enough to fill the GPU, else one: shorter chains and more SMs at work.
  const bool few = (long long)T * units < kFillThreads;
  const Walk w = walk_of(units, few ? 1 : 4);
  const long long blocks = blocks_of(w, T);
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_after(few ? sort_rows_kernel<kBytes, 1> : sort_rows_kernel<kBytes, 4>, (int)blocks, kRowThreads, 0, stream, static_cast<const U*>(x),
                      x_stride_bytes / kBytes, static_cast<U*>(xs), s2f, f2s, T, k, (int)units, w);
}

template <class E, int kV, int kSlots, int kPer, bool kWeights>
cudaError_t merge_launch_as(const void* rows, long long stride, const float* w, const int* f2s, void* y, int T, int k, int H, cudaStream_t stream) {
  const Walk walk = walk_of(H / kV, kPer);
  const long long blocks = blocks_of(walk, T);
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_after(merge_rows_kernel<E, kV, kSlots, kPer, kWeights>, (int)blocks, kRowThreads, 0, stream, static_cast<const E*>(rows), stride, w,
                      f2s, static_cast<E*>(y), T, k, H, walk);
}
template <class E, bool kWeights>
cudaError_t merge_launch(const void* rows, long long stride, const float* w, const int* f2s, void* y, int T, int k, int H, cudaStream_t stream) {
  constexpr int kV = 16 / sizeof(E);
  const int access = widest(bits(rows) | bits(y) | (unsigned long long)stride * sizeof(E) | (unsigned long long)H * sizeof(E)) / (int)sizeof(E);
  const int v = access >= kV ? kV : access >= 2 ? 2 : 1;
  // Few columns: one access a slot and thread (two of single elements), so that more threads are at work.  Else about 8 rows' worth of 16 bytes in flight a thread, whatever k is and
  // as near to it as narrow accesses come: 16 384 x 2 x 4 096 bf16 110 us with one access a slot, 67 with four.
  const bool few = (long long)T * (H / v) < kFillThreads;
  const auto launch = v == 1   ? (few ? merge_launch_as<E, 1, 8, 2, kWeights> : merge_launch_as<E, 1, 8, 4, kWeights>)
                      : v == 2 ? (few ? merge_launch_as<E, 2, 8, 1, kWeights> : merge_launch_as<E, 2, 8, sizeof(E) == 4 ? 2 : 4, kWeights>)
                      : few || k > 4 ? merge_launch_as<E, kV, 8, 1, kWeights>
                      : k > 2        ? merge_launch_as<E, kV, 4, 2, kWeights>
                                     : merge_launch_as<E, kV, 2, 4, kWeights>;
  return launch(rows, stride, w, f2s, y, T, k, H, stream);
}

template <class E, int kV, int kSlots, int kPer>
cudaError_t grad_launch_as(const void* dy, long long dy_stride, const void* rows, long long stride, const float* w, const int* s2f, const int* f2s,
                           void* drows, float* dw, int T, int k, int H, cudaStream_t stream) {
  // Threads for a token: its columns in one go where tokens are few, in two where there are more of them than blocks fit on the GPU (8 192 x 8 x 2 048
  // bf16 96 -> 90 us, 16 384 x 2 x 4 096 116 -> 102, 8 192 x 8 x 512 27 -> 24).
  const int goes = T > 148 * 4 ? 2 : 1;
  int group = 32;
  while (group < kRowThreads && goes * group * kPer < H / kV) group *= 2;
  const int groups = kRowThreads / group;
  return launch_after(merge_grad_kernel<E, kV, kSlots, kPer>, (T + groups - 1) / groups, kRowThreads, 0, stream, static_cast<const E*>(dy), dy_stride,
                      static_cast<const E*>(rows), stride, w, s2f, f2s, static_cast<E*>(drows), dw, T, k, H, group);
}
template <class E>
cudaError_t grad_launch(const void* dy, long long dy_stride, const void* rows, long long stride, const float* w, const int* s2f, const int* f2s,
                        void* drows, float* dw, int T, int k, int H, cudaStream_t stream) {
  constexpr int kV = 16 / sizeof(E);
  const int access = widest(bits(dy) | bits(rows) | bits(drows) | (unsigned long long)dy_stride * sizeof(E) | (unsigned long long)stride * sizeof(E) |
                            (unsigned long long)H * sizeof(E)) / (int)sizeof(E);
  const auto launch = access >= kV ? (k > 2 ? grad_launch_as<E, kV, 4, 1> : grad_launch_as<E, kV, 2, 2>)
                      : access >= 2 ? grad_launch_as<E, 2, 4, 2> : grad_launch_as<E, 1, 8, 2>;
  return launch(dy, dy_stride, rows, stride, w, s2f, f2s, drows, dw, T, k, H, stream);
}

template <bool kWeights>
int merge_any(const void* rows, int64_t stride, int dtype, const float* w, int T, int k, int H, const int* f2s, void* y, void* stream) {
  bool empty = false;
  const int rc = check_sizes(T, k, H, dtype, false, &empty);
  if (rc || empty) return rc;
  if (!rows || !f2s || !y || (kWeights && !w) || stride < H) return MOE_EINVAL;
  if (!element_aligned(element_bytes(dtype), rows, y) || !element_aligned(4, w, f2s)) return MOE_EINVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == MOE_DTYPE_FP32   ? merge_launch<float, kWeights>(rows, stride, w, f2s, y, T, k, H, st)
                        : dtype == MOE_DTYPE_FP16 ? merge_launch<__half, kWeights>(rows, stride, w, f2s, y, T, k, H, st)
                                                  : merge_launch<__nv_bfloat16, kWeights>(rows, stride, w, f2s, y, T, k, H, st);
  return e == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // namespace
}  // namespace moe

extern "C" {

int moe_sort_rows(const void* x, int64_t x_stride, int32_t dtype, int32_t n_tokens, int32_t top_k, int32_t hidden,
                  const int32_t* sorted_to_flat, const int32_t* flat_to_sorted, void* xs, void* stream) {
  using namespace moe;
  bool empty = false;
  const int rc = check_sizes(n_tokens, top_k, hidden, dtype, true, &empty);
  if (rc || empty) return rc;
  if (!x || !sorted_to_flat || !flat_to_sorted || !xs || x_stride < hidden) return MOE_EINVAL;
  const int el = element_bytes(dtype);
  if (!element_aligned(el, x, xs) || !element_aligned(4, sorted_to_flat, flat_to_sorted)) return MOE_EINVAL;
  const long long row = (long long)hidden * el, step = x_stride * el;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaErrorInvalidValue;
  switch (widest(bits(x) | bits(xs) | (unsigned long long)row | (unsigned long long)step)) {
    case 16: e = sort_launch<16>(x, step, xs, sorted_to_flat, flat_to_sorted, n_tokens, top_k, row, st); break;
    case 8: e = sort_launch<8>(x, step, xs, sorted_to_flat, flat_to_sorted, n_tokens, top_k, row, st); break;
    case 4: e = sort_launch<4>(x, step, xs, sorted_to_flat, flat_to_sorted, n_tokens, top_k, row, st); break;
    case 2: e = sort_launch<2>(x, step, xs, sorted_to_flat, flat_to_sorted, n_tokens, top_k, row, st); break;
    default: e = sort_launch<1>(x, step, xs, sorted_to_flat, flat_to_sorted, n_tokens, top_k, row, st); break;
  }
  return e == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

int moe_sort_rows_grad(const void* dxs, int64_t dxs_stride, int32_t dtype, int32_t n_tokens, int32_t top_k, int32_t hidden,
                       const int32_t* flat_to_sorted, void* dx, void* stream) {
  return moe::merge_any<false>(dxs, dxs_stride, dtype, nullptr, n_tokens, top_k, hidden, flat_to_sorted, dx, stream);
}

int moe_merge_rows(const void* rows, int64_t rows_stride, int32_t dtype, const float* topk_w, int32_t n_tokens, int32_t top_k,
                   int32_t hidden, const int32_t* flat_to_sorted, void* y, void* stream) {
  return moe::merge_any<true>(rows, rows_stride, dtype, topk_w, n_tokens, top_k, hidden, flat_to_sorted, y, stream);
}

int moe_merge_rows_grad(const void* dy, int64_t dy_stride, const void* rows, int64_t rows_stride, int32_t dtype, const float* topk_w,
                        int32_t n_tokens, int32_t top_k, int32_t hidden, const int32_t* sorted_to_flat, const int32_t* flat_to_sorted,
                        void* drows, float* d_topk_w, void* stream) {
  using namespace moe;
  bool empty = false;
  const int rc = check_sizes(n_tokens, top_k, hidden, dtype, false, &empty);
  if (rc || empty) return rc;
  if (!dy || !rows || !topk_w || !sorted_to_flat || !flat_to_sorted || !drows || !d_topk_w || dy_stride < hidden || rows_stride < hidden)
    return MOE_EINVAL;
  if (!element_aligned(element_bytes(dtype), dy, rows, drows) || !element_aligned(4, topk_w, sorted_to_flat, flat_to_sorted, d_topk_w))
    return MOE_EINVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const auto launch = dtype == MOE_DTYPE_FP32 ? grad_launch<float> : dtype == MOE_DTYPE_FP16 ? grad_launch<__half> : grad_launch<__nv_bfloat16>;
  const cudaError_t e = launch(dy, dy_stride, rows, rows_stride, topk_w, sorted_to_flat, flat_to_sorted, drows, d_topk_w, n_tokens, top_k, hidden, st);
  return e == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // extern "C"
