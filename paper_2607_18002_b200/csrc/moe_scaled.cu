// moe_scaled_quantize / moe_scaled_quantize_weights / moe_scaled_dequantize: values to e4m3 codes with an fp32 scale per block, and back (moe_scaled.cuh).
//
// Bound by memory and, of 16-bit values, by the integer instructions of the exact rounding: a value is read once and a byte written, k times where rows are sorted on the
// way.  A thread has 16 neighbouring columns at a time: two or four 16-byte loads, one 16-byte store of codes.  As in moe_rows.cu the kernel walks tokens.  A block of weights is 128 such rows, read once: a CTA holds it in registers while its maximum is found.
#include <cuda_fp16.h>

#include "moe_dev.cuh"
#include "moe_scaled.cuh"

namespace moe {
namespace {

constexpr int kThreads = 256;
constexpr int kCols = 16;                          // of a thread
constexpr int kLanes = kScaledBlock / kCols;       // of a row's block

template <class E> struct Raw { static constexpr int kQuads = kCols * (int)sizeof(E) / 16; uint4 q[kQuads]; };
template <class E> __device__ __forceinline__ void unpack(const uint4& r, float (&v)[16 / sizeof(E)]);
template <> __device__ __forceinline__ void unpack<float>(const uint4& r, float (&v)[4]) {
  v[0] = __uint_as_float(r.x); v[1] = __uint_as_float(r.y); v[2] = __uint_as_float(r.z); v[3] = __uint_as_float(r.w);
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(const uint4& r, float (&v)[8]) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <> __device__ __forceinline__ void unpack<__half>(const uint4& r, float (&v)[8]) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    v[2 * i] = f.x;
    v[2 * i + 1] = f.y;
  }
}

// 16 values; without kWide one element at a time (rows that are not 16-byte aligned)
template <class E, bool kWide>
__device__ __forceinline__ Raw<E> load(const E* from) {
  Raw<E> r;
  if (kWide) {
#pragma unroll
    for (int i = 0; i < Raw<E>::kQuads; ++i) r.q[i] = reinterpret_cast<const uint4*>(from)[i];
  } else {
    E* e = reinterpret_cast<E*>(&r);
#pragma unroll
    for (int i = 0; i < kCols; ++i) e[i] = from[i];
  }
  return r;
}
// largest magnitude, as bits of the element's type (two 16-bit elements at a time)
template <class E>
__device__ __forceinline__ unsigned top_bits(const Raw<E>& r) {
  unsigned top = 0u;
#pragma unroll
  for (int q = 0; q < Raw<E>::kQuads; ++q) {
    const unsigned w[4] = {r.q[q].x, r.q[q].y, r.q[q].z, r.q[q].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (sizeof(E) == 4) top = max(top, w[i] & 0x7fffffffu);
      else asm("max.u16x2 %0, %0, %1;" : "+r"(top) : "r"(w[i] & 0x7fff7fffu));
    }
  }
  return sizeof(E) == 4 ? top : max(top >> 16, top & 0xffffu);
}
// ... as those of fp32
template <class E> __device__ __forceinline__ unsigned wide_bits(unsigned b);
template <> __device__ __forceinline__ unsigned wide_bits<float>(unsigned b) { return b; }
template <> __device__ __forceinline__ unsigned wide_bits<__nv_bfloat16>(unsigned b) { return b << 16; }
template <> __device__ __forceinline__ unsigned wide_bits<__half>(unsigned b) { return __float_as_uint(__half2float(__ushort_as_half((unsigned short)b))); }

// Values over their block's scale, such that rounding the result to e4m3 gives what rounding the exact quotient gives.  A product with the reciprocal, corrected once by
// its residue, is the nearest fp32 number (Markstein 1990); it becomes the quotient rounded to odd -- cut off, the last bit set where something was cut off --, which by
// what its own residue says takes five integer operations and no branch, and which is never a midpoint of two codes unless the quotient is one.  (A branch where the
// nearest number may be a midpoint: 98 304 x 2 048 bf16 147 us.)  kUp: scales below 2^-60 are taken 2^64 times, with the values, so that no residue falls below
// the normal numbers.
template <class E, bool kUp>
__device__ __forceinline__ uint4 codes_with(const Raw<E>& r, float scale) {
  constexpr int kIn = 16 / (int)sizeof(E);
  if (kUp) scale *= 0x1p64f;
  const float inv = 1.f / scale;
  unsigned w[4];
#pragma unroll
  for (int k = 0; k < Raw<E>::kQuads; ++k) {
    float v[kIn];
    unpack<E>(r.q[k], v);
#pragma unroll
    for (int n = 0; n < kIn; ++n) {
      const float x = kUp ? v[n] * 0x1p64f : v[n];
      float q = x * inv;
      q = fmaf(fmaf(-q, scale, x), inv, q);
      const float left = fmaf(-q, scale, x);
      const int bits = __float_as_int(q), below = (bits ^ __float_as_int(left)) >> 31;      // -1 where q is larger than the quotient
      v[n] = left != 0.f ? __int_as_float((bits + below) | 1) : q;
    }
#pragma unroll
    for (int n = 0; n < kIn; n += 4) w[(k * kIn + n) / 4] = e4m3_codes4(v + n);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <class E>
__device__ __forceinline__ uint4 codes_of(const Raw<E>& r, float scale) {
  return scale < 0x1p-60f ? codes_with<E, true>(r, scale) : codes_with<E, false>(r, scale);
}

// Four threads a block, twice 16 columns each, 64 apart: thread i % 4 of block i / 4, block b % blocks of token b / blocks.  (Eight threads and 16 columns each, with as much work
// on scales and addresses a thread: 98 304 x 2 048 bf16 135 us.)
constexpr int kRowLanes = kLanes / 2;
template <class E, bool kWide>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const E* __restrict__ x, long long stride, int T, int k, int cols, unsigned blocks, unsigned all, const int* __restrict__ s2f,
                const int* __restrict__ f2s, unsigned char* __restrict__ codes, float* __restrict__ scales) {
  grid_dep_wait();
  const unsigned b = blockIdx.x * (kThreads / kRowLanes) + threadIdx.x / kRowLanes, lane = threadIdx.x % kRowLanes;
  const unsigned t = b / blocks, c = b - t * blocks;
  const int col = (int)c * kScaledBlock + (int)lane * kCols;
  bool on[2];                                      // (whole warps meet in the exchange)
  Raw<E> r[2];
  unsigned top = 0u;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    on[h] = b < all && col + 64 * h < cols;
#pragma unroll
    for (int i = 0; i < Raw<E>::kQuads; ++i) r[h].q[i] = make_uint4(0u, 0u, 0u, 0u);
    if (on[h]) r[h] = load<E, kWide>(x + t * stride + col + 64 * h);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) top = max(top, top_bits<E>(r[h]));
#pragma unroll
  for (int s = kRowLanes / 2; s >= 1; s >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
  if (!on[0]) return;
  const float scale = scaled_scale(wide_bits<E>(top));
  uint4 out[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) out[h] = codes_of<E>(r[h], scale);
  const auto store = [&](size_t p, const uint4& first, const uint4& second, float s) {
    uint4* to = reinterpret_cast<uint4*>(codes + p * cols + col);
    to[0] = first;
    if (on[1]) to[4] = second;
    if (lane == 0) scales[p * blocks + c] = s;
  };
  if (!f2s) {
    store(t, out[0], out[1], scale);
    return;
  }
  const unsigned R = (unsigned)T * (unsigned)k;
#pragma unroll 4
  for (int j = 0; j < k; ++j) {
    const size_t i = (size_t)t * k + j;
    const unsigned p = (unsigned)f2s[i];
    if (p < R) store(p, out[0], out[1], scale);
    if ((unsigned)s2f[i] >= R) store(i, make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u), 1.f);      // a row that belongs to no token
  }
}

// A CTA a block of 128 x 128: thread i has the columns of lane i % 8 in rows i / 8 + 32 m.
constexpr int kRowsAtOnce = kThreads / kLanes, kPer = kScaledBlock / kRowsAtOnce;
template <class E>
__global__ void __launch_bounds__(kThreads)
quantize_weights_kernel(const E* __restrict__ w, int n, int cols, unsigned row_blocks, unsigned blocks, unsigned char* __restrict__ codes,
                        float* __restrict__ scales) {
  __shared__ unsigned tops[kThreads / 32];
  grid_dep_wait();
  const unsigned c = blockIdx.x % blocks, above = blockIdx.x / blocks, rb = above % row_blocks, e = above / row_blocks;
  const int col = (int)c * kScaledBlock + (int)(threadIdx.x % kLanes) * kCols;
  const int row0 = (int)rb * kScaledBlock + (int)threadIdx.x / kLanes;
  const size_t at = ((size_t)e * n + row0) * cols + col;
  Raw<E> r[kPer];
  unsigned top = 0u;
#pragma unroll
  for (int m = 0; m < kPer; ++m) {
#pragma unroll
    for (int i = 0; i < Raw<E>::kQuads; ++i) r[m].q[i] = make_uint4(0u, 0u, 0u, 0u);
    if (col < cols && row0 + m * kRowsAtOnce < n) r[m] = load<E, true>(w + at + (size_t)m * kRowsAtOnce * cols);
  }
#pragma unroll
  for (int m = 0; m < kPer; ++m) top = max(top, top_bits<E>(r[m]));
  top = __reduce_max_sync(0xffffffffu, top);
  if (threadIdx.x % 32 == 0) tops[threadIdx.x / 32] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 32; ++i) top = max(top, tops[i]);
  const float scale = scaled_scale(wide_bits<E>(top));
#pragma unroll
  for (int m = 0; m < kPer; ++m)
    if (col < cols && row0 + m * kRowsAtOnce < n) *reinterpret_cast<uint4*>(codes + at + (size_t)m * kRowsAtOnce * cols) = codes_of<E>(r[m], scale);
  if (threadIdx.x == 0) scales[blockIdx.x] = scale;
}

template <class E> __device__ __forceinline__ E rounded(float v);
template <> __device__ __forceinline__ float rounded(float v) { return v; }
template <> __device__ __forceinline__ __half rounded(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rounded(float v) { return __float2bfloat16_rn(v); }

// A thread writes 16 bytes of values at a time, four times: its loads are in flight together, and a warp writes 512 bytes in a row.  Where the second to fourth lie follows from the
// first by additions (kThreads values further on: `rows` rows and `left` places of a row of per_row); divisions for each took 102 us for 98 304 x 2 048 bf16, 92 so (6.5 TB/s).
constexpr int kAtOnce = 4;
struct Steps {
  unsigned per_row, rows, left;
};
template <class E>
__global__ void __launch_bounds__(kThreads)
dequantize_kernel(const unsigned char* __restrict__ codes, const float* __restrict__ scales, long long all, unsigned n, unsigned blocks, Steps step, int shift,
                  uint4* __restrict__ out) {
  constexpr int kN = 16 / (int)sizeof(E);
  grid_dep_wait();
  const unsigned row_blocks = (n + (1u << shift) - 1) >> shift;
  const long long i0 = (long long)blockIdx.x * (kThreads * kAtOnce) + threadIdx.x;
  unsigned long long row = i0 >> 32 ? i0 / step.per_row : (unsigned)i0 / step.per_row;
  unsigned c = (unsigned)(i0 - row * step.per_row);
  // the row of scales: that of the row itself, or of its 128 in matrix e (row `in` of it)
  unsigned long long e = 0;
  unsigned in = 0;
  if (shift) {
    e = row >> 32 ? row / n : (unsigned)row / n;
    in = (unsigned)(row - e * n);
  }
  uint2 word[kAtOnce];
  float scale[kAtOnce];
#pragma unroll
  for (int m = 0; m < kAtOnce; ++m) {
    const long long i = i0 + m * kThreads;
    if (i < all) {
      if (kN == 8) word[m] = reinterpret_cast<const uint2*>(codes)[i];
      else word[m].x = reinterpret_cast<const unsigned*>(codes)[i];
      scale[m] = scales[(shift ? e * row_blocks + (in >> shift) : row) * blocks + c * kN / kScaledBlock];
    }
    if (m + 1 < kAtOnce) {
      const bool over = c + step.left >= step.per_row;
      c += step.left - (over ? step.per_row : 0u);
      const unsigned down = step.rows + over;
      row += down;
      in += down;
      if (shift && in >= n) {
        e += in / n;
        in %= n;
      }
    }
  }
#pragma unroll
  for (int m = 0; m < kAtOnce; ++m) {
    const long long i = i0 + m * kThreads;
    if (i >= all) return;
    uint4 raw;
    E* v = reinterpret_cast<E*>(&raw);
#pragma unroll
    for (int q = 0; q < kN; q += 2) {
      const unsigned short two = (unsigned short)((q < 4 ? word[m].x : word[m].y) >> (8 * (q & 3)));
      unsigned h;                                  // e4m3 values are exact in fp16
      asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(two));
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      v[q] = rounded<E>(f.x * scale[m]);           // (fp32 first: 28 bits of a code and a scale; 16-bit types are rounded from that)
      v[q + 1] = rounded<E>(f.y * scale[m]);
    }
    out[i] = raw;
  }
}

bool value_type(int dtype) { return dtype == MOE_DTYPE_BF16 || dtype == MOE_DTYPE_FP16 || dtype == MOE_DTYPE_FP32; }
bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
bool bad_cols(int cols) { return cols < kCols || cols > 1 << 30 || cols % kCols; }
int blocks_of(int n) { return (n + kScaledBlock - 1) / kScaledBlock; }
int status(cudaError_t e) { return e == cudaSuccess ? MOE_OK : MOE_ECUDA; }

// f with a value of the type
template <class F>
cudaError_t of_type(int dtype, F f) {
  return dtype == MOE_DTYPE_FP32 ? f(float{}) : dtype == MOE_DTYPE_FP16 ? f(__half{}) : f(__nv_bfloat16{});
}

}  // namespace
}  // namespace moe

extern "C" {

int moe_scaled_quantize(const void* x, int64_t x_stride, int32_t dtype, int32_t n_tokens, int32_t top_k, int32_t cols,
                        const int32_t* sorted_to_flat, const int32_t* flat_to_sorted, void* codes, float* scales, void* stream) {
  using namespace moe;
  if (n_tokens < 0 || top_k < 1 || top_k > 32 || bad_cols(cols) || !value_type(dtype)) return MOE_EINVAL;
  if (n_tokens == 0) return MOE_OK;           // (a permutation of no rows may have no address)
  if (!sorted_to_flat != !flat_to_sorted || (!flat_to_sorted && top_k != 1)) return MOE_EINVAL;
  if (flat_to_sorted && (long long)n_tokens * top_k >= (1ll << kRowSlotShift)) return MOE_EINVAL;
  const long long all = (long long)n_tokens * blocks_of(cols);
  if (all > (1ll << 32) - kThreads || !x || !codes || !scales || x_stride < cols) return MOE_EINVAL;
  if (misaligned(x, dtype == MOE_DTYPE_FP32 ? 4 : 2) || misaligned(codes, 16) || misaligned(scales, 4) || misaligned(sorted_to_flat, 4) ||
      misaligned(flat_to_sorted, 4))
    return MOE_EINVAL;
  const int grid = (int)((all + kThreads / kRowLanes - 1) / (kThreads / kRowLanes));
  return status(of_type(dtype, [&](auto type) {
    using E = decltype(type);
    const bool wide = ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(x_stride * (long long)sizeof(E))) & 15) == 0;
    return launch_after(wide ? quantize_kernel<E, true> : quantize_kernel<E, false>, grid, kThreads, 0, static_cast<cudaStream_t>(stream),
                        static_cast<const E*>(x), (long long)x_stride, n_tokens, top_k, cols, (unsigned)blocks_of(cols), (unsigned)all, sorted_to_flat,
                        flat_to_sorted, static_cast<unsigned char*>(codes), scales);
  }));
}

int moe_scaled_quantize_weights(const void* w, int32_t dtype, int32_t n_experts, int32_t n_rows, int32_t cols, void* codes, float* scales,
                                void* stream) {
  using namespace moe;
  if (n_experts < 0 || n_rows < 1 || n_rows > 1 << 30 || bad_cols(cols) || !value_type(dtype)) return MOE_EINVAL;
  if (n_experts == 0) return MOE_OK;
  const __int128 grid = (__int128)n_experts * blocks_of(n_rows) * blocks_of(cols);
  if (grid > 0x7fffffff || (__int128)n_experts * n_rows * cols > ((__int128)1 << 40) || !w || !codes || !scales || misaligned(w, 16) || misaligned(codes, 16) || misaligned(scales, 4)) return MOE_EINVAL;
  return status(of_type(dtype, [&](auto type) {
    using E = decltype(type);
    return launch_after(quantize_weights_kernel<E>, (int)grid, kThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const E*>(w), n_rows, cols,
                        (unsigned)blocks_of(n_rows), (unsigned)blocks_of(cols), static_cast<unsigned char*>(codes), scales);
  }));
}

int moe_scaled_dequantize(const void* codes, const float* scales, int32_t n_experts, int32_t n_rows, int32_t cols, int32_t scale_rows, int32_t dtype,
                          void* values, void* stream) {
  using namespace moe;
  if (n_experts < 0 || n_rows < 0 || bad_cols(cols) || (scale_rows != 1 && scale_rows != kScaledBlock) || !value_type(dtype)) return MOE_EINVAL;
  if (n_experts == 0 || n_rows == 0) return MOE_OK;
  const __int128 count = (__int128)n_experts * n_rows * cols;
  if (count > ((__int128)1 << 40) || !codes || !scales || !values || misaligned(codes, 16) || misaligned(scales, 4) || misaligned(values, 16)) return MOE_EINVAL;
  return status(of_type(dtype, [&](auto type) {
    using E = decltype(type);
    const long long all = (long long)count / (16 / (int)sizeof(E)), grid = (all + kThreads * kAtOnce - 1) / (kThreads * kAtOnce);
    const unsigned per_row = (unsigned)(cols / (16 / (int)sizeof(E)));
    return launch_after(dequantize_kernel<E>, (int)grid, kThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const unsigned char*>(codes), scales,
                        all, (unsigned)n_rows, (unsigned)blocks_of(cols), Steps{per_row, kThreads / per_row, kThreads % per_row}, scale_rows == 1 ? 0 : 7,
                        static_cast<uint4*>(values));
  }));
}

}  // extern "C"
