// moe_mx_quantize / moe_mx_dequantize: rows to 4-bit codes with a scale byte per 32 columns, and back (see moe_mx.cuh for the format).
//
// Bound by memory: a 16-bit value is read once and 17/32 byte written, k times where rows are sorted on the way.  As in moe_rows.cu the kernel walks
// tokens: a token is read and quantised once, whatever the number of rows that it becomes.  A thread quantises a whole block of 32 columns: it has 64
// bytes of 16-bit values in flight, stores 16 bytes of codes, and the scale bytes of a warp's blocks are one sector.  (With 8 columns a thread and
// four lanes a block, 16 bytes in flight and scale bytes eight at a time, 98 304 x 2 048 bf16 took 145 us for 76, the 65 536
// sorted rows of 8 192 x 4 096 59 for 35: 6.7 and 6.0 TB/s now.)  Back to values: 80 us, 6.4 TB/s.
#include <cuda_fp16.h>

#include "moe_dev.cuh"
#include "moe_mx.cuh"

namespace moe {
namespace {

constexpr int kMxThreads = 256;

// the values of a block, four (fp32) or eight to a 16-byte register quad, as they lie in memory
template <class E>
struct Block {
  static constexpr int kQuads = kMxBlock * (int)sizeof(E) / 16, kIn = 16 / (int)sizeof(E);
  uint4 raw[kQuads];
};
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
// one element at a time where rows are not 16-byte aligned
template <class E>
__device__ __forceinline__ unsigned bits_of(E v);
template <> __device__ __forceinline__ unsigned bits_of(float v) { return __float_as_uint(v); }
template <> __device__ __forceinline__ unsigned bits_of(__half v) { return __half_as_ushort(v); }
template <> __device__ __forceinline__ unsigned bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }

template <class E, bool kWide>
__device__ __forceinline__ Block<E> load_block(const E* from) {
  Block<E> b;
  if (kWide) {
#pragma unroll
    for (int i = 0; i < Block<E>::kQuads; ++i) b.raw[i] = reinterpret_cast<const uint4*>(from)[i];
  } else {
    unsigned w[4 * Block<E>::kQuads];
    constexpr int kIn = 4 / (int)sizeof(E);
#pragma unroll
    for (int i = 0; i < 4 * Block<E>::kQuads; ++i) {
      w[i] = bits_of(from[kIn * i]);
      if (kIn == 2) w[i] |= bits_of(from[kIn * i + 1 % kIn]) << 16;
    }
#pragma unroll
    for (int i = 0; i < Block<E>::kQuads; ++i) b.raw[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
  return b;
}

// Thread i of the launch has block i % per_row of token i / per_row.
template <class E, bool kWide>
__global__ void __launch_bounds__(kMxThreads)
mx_quantize_kernel(const E* __restrict__ x, long long stride, int T, int k, unsigned per_row, unsigned all, const int* __restrict__ s2f,
                   const int* __restrict__ f2s, uint4* __restrict__ codes, unsigned char* __restrict__ scales) {
  grid_dep_wait();
  const unsigned i = blockIdx.x * kMxThreads + threadIdx.x;
  if (i >= all) return;
  const unsigned t = i / per_row, c = i - t * per_row;
  const Block<E> block = load_block<E, kWide>(x + t * stride + c * kMxBlock);
  constexpr int kIn = Block<E>::kIn;
  unsigned top = 0u;
#pragma unroll
  for (int q = 0; q < Block<E>::kQuads; ++q) {
    float v[kIn];
    unpack<E>(block.raw[q], v);
#pragma unroll
    for (int n = 0; n < kIn; ++n) top = max(top, __float_as_uint(v[n]) & 0x7fffffffu);
  }
  const unsigned byte = mx_scale_byte(top);
  const float inv = mx_inverse(byte);
  unsigned word[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int q = 0; q < Block<E>::kQuads; ++q) {
    float v[kIn];
    unpack<E>(block.raw[q], v);
#pragma unroll
    for (int n = 0; n < kIn; n += 2) {
      const int at = q * kIn + n;
      word[at / 8] |= mx_codes2(v[n] * inv, v[n + 1] * inv) << (4 * (at % 8));
    }
  }
  const uint4 out = make_uint4(word[0], word[1], word[2], word[3]);
  if (!f2s) {
    codes[i] = out;
    scales[i] = (unsigned char)byte;
    return;
  }
  const unsigned R = (unsigned)T * (unsigned)k;
#pragma unroll 4
  for (int j = 0; j < k; ++j) {
    const unsigned p = (unsigned)f2s[(size_t)t * k + j];
    if (p < R) {
      codes[(size_t)p * per_row + c] = out;
      scales[(size_t)p * per_row + c] = (unsigned char)byte;
    }
    if ((unsigned)s2f[(size_t)t * k + j] >= R) {       // a row that belongs to no token: zeros
      const size_t at = ((size_t)t * k + j) * per_row + c;
      codes[at] = make_uint4(0u, 0u, 0u, 0u);
      scales[at] = 0;
    }
  }
}

// A thread writes 16 bytes of values at a time, kN = 8 columns of 16 bits or 4 of 32, four times: its loads are in flight together, and a warp
// writes 512 bytes in a row.
constexpr int kMxPer = 4;
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
  const long long i0 = (long long)blockIdx.x * (kMxThreads * kMxPer) + threadIdx.x;
  unsigned word[kMxPer], byte[kMxPer];
#pragma unroll
  for (int m = 0; m < kMxPer; ++m) {
    const long long i = i0 + m * kMxThreads;
    if (i < all) {
      word[m] = codes[i];
      byte[m] = scales[i / (kMxBlock / kN)];
    }
  }
#pragma unroll
  for (int m = 0; m < kMxPer; ++m) {
    const long long i = i0 + m * kMxThreads;
    if (i >= all) return;
    const float scale = mx_scale(byte[m]);
    uint4 raw;
    E* e = reinterpret_cast<E*>(&raw);
#pragma unroll
    for (int n = 0; n < kN; ++n) {
      const unsigned code = word[m] >> (4 * n);
      // e2m1 has fp32's form with a bias of 1 for 127: its bits in place, times 2^126, are its value, subnormal ones included
      const float v = __uint_as_float((code & 7u) << 22 | (code & 8u) << 28) * __uint_as_float(253u << 23);
      e[n] = rounded<E>(v * scale);
    }
    out[i] = raw;
  }
}

template <class E>
cudaError_t quantize_launch(const void* x, long long stride, int T, int k, int K, const int* s2f, const int* f2s, void* codes, void* scales,
                            cudaStream_t stream) {
  const long long threads = (long long)T * (K / kMxBlock), blocks = (threads + kMxThreads - 1) / kMxThreads;
  const bool wide = ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(stride * (long long)sizeof(E))) & 15) == 0;
  return launch_after(wide ? mx_quantize_kernel<E, true> : mx_quantize_kernel<E, false>, (int)blocks, kMxThreads, 0, stream,
                      static_cast<const E*>(x), stride, T, k, (unsigned)(K / kMxBlock), (unsigned)threads, s2f, f2s, static_cast<uint4*>(codes),
                      static_cast<unsigned char*>(scales));
}

template <class E>
cudaError_t dequantize_launch(const void* codes, const void* scales, long long values, void* out, cudaStream_t stream) {
  const long long all = values / (16 / (int)sizeof(E)), blocks = (all + kMxThreads * kMxPer - 1) / (kMxThreads * kMxPer);
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
  if (n_tokens < 0 || top_k < 1 || top_k > 32 || cols < kMxBlock || cols > 1 << 30 || cols % kMxBlock || !value_type(dtype)) return MOE_EINVAL;
  if (n_tokens == 0) return MOE_OK;           // (a permutation of no rows may have no address)
  if (!sorted_to_flat != !flat_to_sorted || (!flat_to_sorted && top_k != 1)) return MOE_EINVAL;
  if (flat_to_sorted && (long long)n_tokens * top_k >= (1ll << kRowSlotShift)) return MOE_EINVAL;
  if ((long long)n_tokens * (cols / kMxBlock) >= (1ll << 32)) return MOE_EINVAL;
  if (!x || !codes || !scales || x_stride < cols) return MOE_EINVAL;
  if (misaligned(x, dtype == MOE_DTYPE_FP32 ? 4 : 2) || misaligned(codes, 16) || misaligned(sorted_to_flat, 4) || misaligned(flat_to_sorted, 4))
    return MOE_EINVAL;
  const auto launch = dtype == MOE_DTYPE_FP32 ? quantize_launch<float> : dtype == MOE_DTYPE_FP16 ? quantize_launch<__half> : quantize_launch<__nv_bfloat16>;
  return launch(x, x_stride, n_tokens, top_k, cols, sorted_to_flat, flat_to_sorted, codes, scales, static_cast<cudaStream_t>(stream)) == cudaSuccess
             ? MOE_OK : MOE_ECUDA;
}

int moe_mx_dequantize(const void* codes, const void* scales, int64_t n_rows, int32_t cols, int32_t dtype, void* values, void* stream) {
  using namespace moe;
  if (n_rows < 0 || cols < kMxBlock || cols > 1 << 30 || cols % kMxBlock || !value_type(dtype) || n_rows > (1ll << 40) / cols) return MOE_EINVAL;
  if (n_rows == 0) return MOE_OK;
  if (!codes || !scales || !values || misaligned(codes, 4) || misaligned(values, 16)) return MOE_EINVAL;
  const auto launch = dtype == MOE_DTYPE_FP32 ? dequantize_launch<float> : dtype == MOE_DTYPE_FP16 ? dequantize_launch<__half> : dequantize_launch<__nv_bfloat16>;
  return launch(codes, scales, n_rows * cols, values, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // extern "C"
