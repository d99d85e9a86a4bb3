// moe_mx_quantize / moe_mx_dequantize: rows to 4-bit codes with a scale byte per 32 columns, and back (see moe_mx.cuh for the format).
//
// Bound by memory: a 16-bit value is read once and 17/32 byte written, k times where rows are sorted on the way.  As in moe_rows.cu the kernel walks
// tokens: a token is read and quantised once, whatever the number of rows that it becomes.  A thread quantises 8 columns (one 16-byte load of 16-bit
// values, a 4-byte store), four neighbouring lanes a block: two shuffles for the largest magnitude.
#include <cuda_fp16.h>

#include "moe_dev.cuh"
#include "moe_mx.cuh"

namespace moe {
namespace {

constexpr int kMxThreads = 256;
constexpr int kMxCols = 8;              // columns of a thread

template <class E> __device__ __forceinline__ float as_float(E v);
template <> __device__ __forceinline__ float as_float(float v) { return v; }
template <> __device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }

template <class E, bool kWide>
__device__ __forceinline__ void load8(const E* from, float (&v)[8]) {
  constexpr int kV = 16 / sizeof(E);
  if (kWide) {
#pragma unroll
    for (int i = 0; i < 8; i += kV) {
      const uint4 raw = *reinterpret_cast<const uint4*>(from + i);
      const E* e = reinterpret_cast<const E*>(&raw);
#pragma unroll
      for (int n = 0; n < kV; ++n) v[i + n] = as_float<E>(e[n]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = as_float<E>(from[i]);
  }
}

// Thread i of the launch has 8 columns of token i / (K / 8); blocks of 32 columns never straddle a warp's quads of lanes.
template <class E, bool kWide>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const E* __restrict__ x, long long stride, int T, int k, unsigned per_row, const int* __restrict__ s2f,
                   const int* __restrict__ f2s, unsigned* __restrict__ codes, unsigned char* __restrict__ scales) {
  grid_dep_wait();
  const long long i = (long long)blockIdx.x * kMxThreads + threadIdx.x;
  const long long all = (long long)T * per_row;
  const bool on = i < all;                              // per_row is a multiple of 4: lanes of a quad are on together
  const int t = on ? (int)(i / per_row) : 0;
  const unsigned c = on ? (unsigned)(i - (long long)t * per_row) : 0u;
  float v[8];
  load8<E, kWide>(x + t * stride + c * kMxCols, v);
  unsigned top = 0u;
#pragma unroll
  for (int n = 0; n < 8; ++n) top = max(top, __float_as_uint(v[n]) & 0x7fffffffu);
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
  top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
  if (!on) return;
  const unsigned byte = mx_scale_byte(top);
  const float inv = mx_inverse(byte);
  unsigned word = 0u;
#pragma unroll
  for (int n = 0; n < 8; n += 2) word |= mx_codes2(v[n] * inv, v[n + 1] * inv) << (4 * n);
  if (!f2s) {
    codes[(size_t)t * per_row + c] = word;
    if ((c & 3u) == 0u) scales[((size_t)t * per_row + c) >> 2] = (unsigned char)byte;
    return;
  }
  const unsigned R = (unsigned)T * (unsigned)k;
#pragma unroll 4
  for (int j = 0; j < k; ++j) {
    const unsigned p = (unsigned)f2s[(size_t)t * k + j];
    if (p < R) {
      codes[(size_t)p * per_row + c] = word;
      if ((c & 3u) == 0u) scales[((size_t)p * per_row + c) >> 2] = (unsigned char)byte;
    }
    if ((unsigned)s2f[(size_t)t * k + j] >= R) {       // a row that belongs to no token: zeros
      const size_t at = ((size_t)t * k + j) * per_row + c;
      codes[at] = 0u;
      if ((c & 3u) == 0u) scales[at >> 2] = 0;
    }
  }
}

// A thread writes 16 bytes of values: kN = 8 columns of 16 bits or 4 of 32.
template <class E> struct Codes;
template <> struct Codes<float> { using type = unsigned short; };
template <> struct Codes<__half> { using type = unsigned; };
template <> struct Codes<__nv_bfloat16> { using type = unsigned; };
template <class E> __device__ __forceinline__ E rounded(float v);
template <> __device__ __forceinline__ float rounded(float v) { return v; }
template <> __device__ __forceinline__ __half rounded(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rounded(float v) { return __float2bfloat16_rn(v); }

template <class E>
__global__ void __launch_bounds__(kMxThreads)
mx_dequantize_kernel(const typename Codes<E>::type* __restrict__ codes, const unsigned char* __restrict__ scales, long long all, uint4* __restrict__ out) {
  constexpr int kN = 16 / sizeof(E);
  grid_dep_wait();
  const long long i = (long long)blockIdx.x * kMxThreads + threadIdx.x;
  if (i >= all) return;
  const unsigned word = codes[i];
  const float scale = mx_scale(scales[i / (kMxBlock / kN)]);
  uint4 raw;
  E* e = reinterpret_cast<E*>(&raw);
#pragma unroll
  for (int n = 0; n < kN; ++n) {
    const unsigned code = word >> (4 * n);
    // e2m1 has fp32's form with a bias of 1 for 127: its bits in place, times 2^126, are its value, subnormal ones included
    const float v = __uint_as_float((code & 7u) << 22 | (code & 8u) << 28) * __uint_as_float(253u << 23);
    e[n] = rounded<E>(v * scale);
  }
  out[i] = raw;
}

template <class E>
cudaError_t quantize_launch(const void* x, long long stride, int T, int k, int K, const int* s2f, const int* f2s, void* codes, void* scales,
                            cudaStream_t stream) {
  const long long threads = (long long)T * (K / kMxCols), blocks = (threads + kMxThreads - 1) / kMxThreads;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(stride * (long long)sizeof(E))) & 15) == 0;
  return launch_after(wide ? mx_quantize_kernel<E, true> : mx_quantize_kernel<E, false>, (int)blocks, kMxThreads, 0, stream,
                      static_cast<const E*>(x), stride, T, k, (unsigned)(K / kMxCols), s2f, f2s, static_cast<unsigned*>(codes),
                      static_cast<unsigned char*>(scales));
}

template <class E>
cudaError_t dequantize_launch(const void* codes, const void* scales, long long values, void* out, cudaStream_t stream) {
  const long long all = values / (16 / (int)sizeof(E)), blocks = (all + kMxThreads - 1) / kMxThreads;
  if (blocks > 0x7fffffffll) return cudaErrorInvalidValue;
  return launch_after(mx_dequantize_kernel<E>, (int)blocks, kMxThreads, 0, stream, static_cast<const typename Codes<E>::type*>(codes),
                      static_cast<const unsigned char*>(scales), all, static_cast<uint4*>(out));
}

bool value_type(int dtype) { return dtype == MOE_DTYPE_BF16 || dtype == MOE_DTYPE_FP16 || dtype == MOE_DTYPE_FP32; }
bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

}  // namespace
}  // namespace moe

extern "C" {

int moe_mx_quantize(const void* x, int64_t x_stride, int32_t dtype, int32_t n_tokens, int32_t top_k, int32_t cols,
                    const int32_t* sorted_to_flat, const int32_t* flat_to_sorted, void* codes, void* scales, void* stream) {
  using namespace moe;
  if (n_tokens < 0 || top_k < 1 || top_k > 32 || cols < kMxBlock || cols % kMxBlock || !value_type(dtype)) return MOE_EINVAL;
  if (!sorted_to_flat != !flat_to_sorted || (!flat_to_sorted && top_k != 1)) return MOE_EINVAL;
  if (flat_to_sorted && (long long)n_tokens * top_k >= (1ll << kRowSlotShift)) return MOE_EINVAL;
  if (n_tokens == 0) return MOE_OK;
  if (!x || !codes || !scales || x_stride < cols) return MOE_EINVAL;
  if (misaligned(x, dtype == MOE_DTYPE_FP32 ? 4 : 2) || misaligned(codes, 4) || misaligned(sorted_to_flat, 4) || misaligned(flat_to_sorted, 4))
    return MOE_EINVAL;
  const auto launch = dtype == MOE_DTYPE_FP32 ? quantize_launch<float> : dtype == MOE_DTYPE_FP16 ? quantize_launch<__half> : quantize_launch<__nv_bfloat16>;
  return launch(x, x_stride, n_tokens, top_k, cols, sorted_to_flat, flat_to_sorted, codes, scales, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? MOE_OK : MOE_ECUDA;
}

int moe_mx_dequantize(const void* codes, const void* scales, int64_t n_rows, int32_t cols, int32_t dtype, void* values, void* stream) {
  using namespace moe;
  if (n_rows < 0 || cols < kMxBlock || cols % kMxBlock || !value_type(dtype) || n_rows > (1ll << 40) / cols) return MOE_EINVAL;
  if (n_rows == 0) return MOE_OK;
  if (!codes || !scales || !values || misaligned(codes, 4) || misaligned(values, 16)) return MOE_EINVAL;
  const auto launch = dtype == MOE_DTYPE_FP32 ? dequantize_launch<float> : dtype == MOE_DTYPE_FP16 ? dequantize_launch<__half> : dequantize_launch<__nv_bfloat16>;
  return launch(codes, scales, n_rows * cols, values, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // extern "C"
