// moe_choose_experts / moe_choose_experts_grad: the routers that moe_route does not know -- scores by softmax or sigmoid, a bias that counts for
// the choice alone, groups of experts of which the best are kept -- and the gradient of their weights.
//
//   s_e = softmax(z)_e  or  1 / (1 + exp(-z_e));   c_e = s_e + bias_e;   value of a group: the sum of its one or two largest c
//   the top_groups groups of largest value are kept; the k largest c of their experts are chosen;   w_j = scale s_j  (/ sum_i s_i)
//
// Who is chosen is decided as in 64 bits.  c is computed in fp32 with a bound on its error, and where two candidates whose order matters lie closer
// than that (and are not equal by their inputs) the warp does the token again in fp64: one token of some hundreds.  Without a bias the order is
// that of the logits, which needs no bound.  (All of it in fp64 would be 480 double operations a lane and token: 14 us for 16 384 tokens of 256 experts.)
//
// One warp per token, its logits over the lanes' registers as order-preserving keys.  Equal values go to the lower index, as everywhere.
#include <cuda_fp16.h>

#include "moe_dev.cuh"

namespace moe {
namespace {

constexpr int kMaxE = 1024, kMaxK = 32, kMaxGroups = 32;
constexpr int kWarps = 8;
constexpr unsigned kAll = 0xffffffffu;

struct ChooseArgs {
  const void* logits;
  const float* bias;
  long long stride;
  int T, E, k, groups, top_groups, group_sum, sigmoid, renormalize;
  float scale;
  int* ids;
  float* w;
};

// unsigned order = float order (-0 counts as +0), NaN above every number; 0 is below everything: "no candidate"
__device__ __forceinline__ unsigned key_of(float v) {
  if (v != v) return kAll;
  const unsigned u = __float_as_uint(v + 0.0f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float of_key(unsigned key) { return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key); }
__device__ __forceinline__ unsigned long long key_of(double v) {
  if (v != v) return ~0ull;
  const unsigned long long u = __double_as_longlong(v + 0.0);
  return (u >> 63) ? ~u : (u | 1ull << 63);
}

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class L> __device__ __forceinline__ L as_logit(float v);
template <> __device__ __forceinline__ float as_logit(float v) { return v; }
template <> __device__ __forceinline__ __half as_logit(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 as_logit(float v) { return __float2bfloat16_rn(v); }

// four neighbouring elements, aligned to four
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
  const float4 r = *reinterpret_cast<const float4*>(p);
  v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w;
}
template <class L>
__device__ __forceinline__ void load4(const L* p, float (&v)[4]) {
  const uint2 r = *reinterpret_cast<const uint2*>(p);
  const L* e = reinterpret_cast<const L*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = as_float(e[i]);
}
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
template <class L>
__device__ __forceinline__ void store4(L* p, const float (&v)[4]) {
  uint2 r;
  L* e = reinterpret_cast<L*>(&r);
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = as_logit<L>(v[i]);
  *reinterpret_cast<uint2*>(p) = r;
}

// The expert of a lane's i-th element.  kVec: rows are aligned to four elements, a lane has four neighbours at a time.
template <bool kVec>
__device__ __forceinline__ int expert_of(int i, int lane) { return kVec ? 128 * (i / 4) + 4 * lane + i % 4 : lane + 32 * i; }
// the row's logits; -inf behind the last expert
template <class L, int kPer, bool kVec>
__device__ __forceinline__ void load_row(const L* z, int E, int lane, float (&v)[kPer]) {
  if (kVec) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      float q[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
      if (expert_of<true>(i, lane) < E) load4(z + expert_of<true>(i, lane), q);
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i + j] = q[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = expert_of<false>(i, lane) < E ? as_float(z[expert_of<false>(i, lane)]) : -INFINITY;
  }
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int b = 16; b >= 1; b >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, b));
  return v;
}
template <class F>
__device__ __forceinline__ F warp_sum(F v) {
#pragma unroll
  for (int b = 16; b >= 1; b >>= 1) v += __shfl_xor_sync(kAll, v, b);
  return v;
}

// Of a softmax: the largest logit (0 where there is none above -inf, so that exp gives 0), and 1 over the sum (0 for such a row, NaN for one with NaN or
// +inf)
struct Norm {
  float top, inv;
};
template <int kPer>
__device__ __forceinline__ Norm norm_of(const float (&z)[kPer]) {
  float m = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) m = fmaxf(m, z[i]);
  m = warp_max(m);
  if (m == -INFINITY) m = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += expf(z[i] - m);
  sum = warp_sum(sum);
  return Norm{m, sum == 0.f ? 0.f : 1.f / sum};
}
__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }
__device__ __forceinline__ double sigmoid(double z) { return 1.0 / (1.0 + exp(-z)); }

// Bounds on the error of a score and its sum with a bias, in units of 2^-23: exp is off by two steps of 2^-23 at most, the quotient and each addition by half
// of one, a softmax's sum by 13 additions and its terms by the rounding of z - top besides: s |z - top| / 2 <= 0.2 s_top; what sigmoid loses below
// 2^-126 is less than 2^-120.  6 and 25 times the score are about twice that.
__device__ __forceinline__ float error_of(float s, float c, float z, float top, bool is_sigmoid) {
  return ldexpf(s * (is_sigmoid ? 6.f : 24.f + fabsf(z - top)) + fabsf(c), -23) + 0x1p-120f;
}
__device__ __forceinline__ float error_of_any(float c, bool is_sigmoid) { return ldexpf((is_sigmoid ? 6.f : 25.f) + fabsf(c), -23); }

// The same in fp64, by the whole warp: rare.  Lane j < k gets the j-th expert.
template <class L, int kPer, bool kVec>
__device__ __noinline__ int choose_slowly(const ChooseArgs& a, const L* row, int lane) {
  double c[kPer];
  double m = -INFINITY, sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = expert_of<kVec>(i, lane);
    c[i] = e < a.E ? (double)as_float(row[e]) : -INFINITY;
    m = fmax(m, c[i]);
  }
  if (!a.sigmoid) {
#pragma unroll
    for (int b = 16; b >= 1; b >>= 1) m = fmax(m, __shfl_xor_sync(kAll, m, b));
    if (m == -INFINITY) m = 0.0;
#pragma unroll 1
    for (int i = 0; i < kPer; ++i) sum += exp(c[i] - m);
    sum = warp_sum(sum);
  }
  unsigned long long key[kPer];
  double value = -INFINITY;            // lane g: of group g
  const int size = a.E / a.groups;
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = expert_of<kVec>(i, lane);
    const double s = a.sigmoid ? sigmoid(c[i]) : sum == 0.0 ? 0.0 : exp(c[i] - m) / sum;
    c[i] = e < a.E ? s + (a.bias ? (double)a.bias[e] : 0.0) : -INFINITY;
  }
#pragma unroll 1
  for (int g = 0; g < a.groups && a.top_groups < a.groups; ++g) {
    double one = -INFINITY, two = -INFINITY;
#pragma unroll 1
    for (int i = 0; i < kPer; ++i) {
      const int e = expert_of<kVec>(i, lane);
      if (e >= a.E || e / size != g) continue;
      if (key_of(c[i]) > key_of(one)) {
        two = one;
        one = c[i];
      } else if (key_of(c[i]) > key_of(two)) {
        two = c[i];
      }
    }
#pragma unroll
    for (int b = 16; b >= 1; b >>= 1) {
      const double o1 = __shfl_xor_sync(kAll, one, b), o2 = __shfl_xor_sync(kAll, two, b);
      const bool mine = key_of(one) >= key_of(o1);
      const double less = mine ? o1 : one, next = mine ? two : o2;
      one = mine ? one : o1;
      two = key_of(less) > key_of(next) ? less : next;
    }
    if (lane == g) value = a.group_sum > 1 && size > 1 ? one + two : one;
  }
  bool kept = true;
  if (a.top_groups < a.groups) {
    int before = 0;
    for (int g = 0; g < a.groups; ++g) {
      const unsigned long long other = key_of(__shfl_sync(kAll, value, g));
      before += other > key_of(value) || (other == key_of(value) && g < lane);
    }
    kept = lane < a.groups && before < a.top_groups;
  }
  const unsigned groups = __ballot_sync(kAll, kept);
  // without a bias the order is that of the logits
#pragma unroll 1
  for (int i = 0; i < kPer; ++i) {
    const int e = expert_of<kVec>(i, lane);
    const bool on = e < a.E && (groups >> (a.top_groups < a.groups ? e / size : 0) & 1);
    key[i] = !on ? 0ull : a.bias ? key_of(c[i]) : key_of((double)as_float(row[e]));
  }
  int mine = 0;
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    unsigned long long best = 0;
    int id = kMaxE;
#pragma unroll 1
    for (int i = 0; i < kPer; ++i) {
      const int e = expert_of<kVec>(i, lane);
      if (key[i] > best || (key[i] == best && e < id)) {
        best = key[i];
        id = e;
      }
    }
#pragma unroll
    for (int b = 16; b >= 1; b >>= 1) {
      const unsigned long long other = __shfl_xor_sync(kAll, best, b);
      const int oid = __shfl_xor_sync(kAll, id, b);
      if (other > best || (other == best && oid < id)) {
        best = other;
        id = oid;
      }
    }
#pragma unroll 1
    for (int i = 0; i < kPer; ++i)
      if (expert_of<kVec>(i, lane) == id) key[i] = 0ull;
    if (lane == j) mine = id;
  }
  return mine;
}

// Which groups are kept, as a bit mask; close: whether fp32 cannot tell.  c: the warp's values by expert, in shared memory.
// Several neighbouring lanes have a group: each goes over a part of it, then the two largest are joined.
__device__ __forceinline__ unsigned keep_groups(const ChooseArgs& a, const float* c, int lane, bool& close) {
  const int size = a.E / a.groups;
  int per = 1;                          // lanes a group: a power of two
  while (2 * per * a.groups <= 32 && 2 * per <= size) per *= 2;
  const int g = lane / per, q = lane % per;
  float one = -INFINITY, two = -INFINITY;
  if (g < a.groups) {
    const int n = (size - q + per - 1) / per;
    int at = g % n;                     // (groups start at different places: other banks)
    for (int i = 0; i < n; ++i) {
      const float v = c[g * size + q + per * at];
      if (++at == n) at = 0;
      if (key_of(v) > key_of(one)) {
        two = one;
        one = v;
      } else if (key_of(v) > key_of(two)) {
        two = v;
      }
    }
  }
  for (int b = per / 2; b >= 1; b >>= 1) {
    const float o1 = __shfl_xor_sync(kAll, one, b), o2 = __shfl_xor_sync(kAll, two, b);
    const bool mine = key_of(one) >= key_of(o1);
    const float less = mine ? o1 : one, next = mine ? two : o2;
    one = mine ? one : o1;
    two = key_of(less) > key_of(next) ? less : next;
  }
  const float value = a.group_sum > 1 && size > 1 ? one + two : one;
  const bool mine = g < a.groups && q == 0;
  int before = 0;
  for (int o = 0; o < a.groups; ++o) {
    const unsigned other = key_of(__shfl_sync(kAll, value, o * per));
    before += other > key_of(value) || (other == key_of(value) && o < g);
  }
  unsigned kept = 0;
  const unsigned last = __ballot_sync(kAll, mine && before == a.top_groups - 1), next = __ballot_sync(kAll, mine && before == a.top_groups);
  const float in = __shfl_sync(kAll, value, __ffs(last) - 1), out = __shfl_sync(kAll, value, __ffs(next) - 1);
  // (a group of one expert, or one that holds -inf, has no second value that counts)
  const float err = !mine ? 0.f : error_of_any(one, a.sigmoid) + (two == -INFINITY ? 0.f : error_of_any(two, a.sigmoid) + ldexpf(fabsf(value), -23));
  close = !(in - out > 2.f * warp_max(err));
  const unsigned firsts = __ballot_sync(kAll, mine && before < a.top_groups);
  for (int o = 0; o < a.groups; ++o) kept |= (firsts >> (o * per) & 1u) << o;
  return kept;
}

template <class L, int kPer, bool kVec>
__global__ void __launch_bounds__(kWarps * 32) choose_kernel(const __grid_constant__ ChooseArgs a) {
  __shared__ float by_expert[kWarps][kPer * 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x * kWarps + warp;
  grid_dep_wait();
  if (t >= a.T) return;
  const L* row = static_cast<const L*>(a.logits) + (size_t)t * a.stride;
  const bool grouped = a.top_groups < a.groups;
  Norm norm{0.f, 0.f};
  unsigned key[kPer];
  bool close = false;
  {
    float z[kPer];
    load_row<L, kPer, kVec>(row, a.E, lane, z);
    if (!a.sigmoid && (a.bias || grouped || !a.renormalize)) norm = norm_of<kPer>(z);
    if (a.bias || grouped) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int e = expert_of<kVec>(i, lane);
        float c = -INFINITY;
        if (e < a.E) {
          c = a.sigmoid ? sigmoid(z[i]) : expf(z[i] - norm.top) * norm.inv;
          if (a.bias) c += a.bias[e];
        }
        if (grouped && e < a.E) by_expert[warp][e] = c;
        key[i] = e < a.E ? key_of(a.bias ? c : z[i]) : 0u;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) key[i] = expert_of<kVec>(i, lane) < a.E ? key_of(z[i]) : 0u;
    }
  }
  if (grouped) {
    __syncwarp();
    const unsigned kept = keep_groups(a, by_expert[warp], lane, close);
    const unsigned size = a.E / a.groups, inverse = ((1u << 20) + size - 1) / size;      // e / size = e inverse >> 20 for e < 2^10
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (!(kept >> (((unsigned)expert_of<kVec>(i, lane) * inverse >> 20) & 31) & 1)) key[i] = 0u;
  }
  // lane j keeps the j-th pick; with a bias one more is looked at, whether it is far enough from the last
  unsigned my_key = 0;
  int my_id = 0;
  unsigned kth = 0;
  int picked = 0;                       // with a bias: up to the first that is smaller than the k-th
  for (int j = 0; j < a.k || a.bias; ++j) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) m = max(m, key[i]);
    m = __reduce_max_sync(kAll, m);
    if (m == 0) break;                  // (k are always there)
    if (j == kMaxK) {                   // no lane for one more: let fp64 decide
      close = true;
      break;
    }
    unsigned id = kAll;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i)
      if (key[i] == m) id = (unsigned)expert_of<kVec>(i, lane);
    id = __reduce_min_sync(kAll, id);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if ((unsigned)expert_of<kVec>(i, lane) == id) key[i] = 0u;
    if (lane == j) { my_key = m; my_id = (int)id; }
    picked = j + 1;
    if (j == a.k - 1) kth = m;
    if (j >= a.k && m < kth) break;
  }
  float z = my_key ? as_float(row[my_id]) : 0.f;
  if (a.bias) {
    const float b = my_key ? a.bias[my_id] : 0.f, c = of_key(my_key), s = a.sigmoid ? sigmoid(z) : expf(z - norm.top) * norm.inv;
    const float err = error_of(s, c, z, norm.top, a.sigmoid);
    const unsigned next_key = __shfl_down_sync(kAll, my_key, 1);
    const float nc = of_key(next_key), nerr = __shfl_down_sync(kAll, err, 1), nz = __shfl_down_sync(kAll, z, 1), nb = __shfl_down_sync(kAll, b, 1);
    // neighbours in the order, unless equal by their inputs; and the first that is smaller than the k-th, which stands for all behind it
    bool near = lane < picked - 1 && !(z == nz && b == nb) && !(c - nc > err + nerr);
    if (lane == picked - 1 && lane >= a.k) near = !(of_key(kth) - c > error_of_any(c, a.sigmoid) + error_of_any(of_key(kth), a.sigmoid));
    close = __any_sync(kAll, close || near);
  }
  if (close) {
    my_id = choose_slowly<L, kPer, kVec>(a, row, lane);
    z = lane < a.k ? as_float(row[my_id]) : 0.f;
  }
  const bool mine = lane < a.k;
  float v;
  if (a.renormalize) {
    // relative to the largest of the chosen, so that scores that are tiny alike have weights.  sigmoid(z) = exp(z) / (1 + exp(z))
    const float top = warp_max(mine ? z : -INFINITY), shift = a.sigmoid ? fminf(top, 0.f) : top;
    v = !mine || z == -INFINITY ? 0.f : a.sigmoid && z > 0.f ? sigmoid(z) : expf(z - shift) / (a.sigmoid ? 1.f + expf(z) : 1.f);
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j) sum += __shfl_sync(kAll, v, j);
    v = sum == 0.f ? 0.f : v / sum;
    if (norm.inv != norm.inv) v = norm.inv;       // a NaN in the row (one that nobody looked for above is among the chosen)
  } else {
    v = a.sigmoid ? sigmoid(z) : expf(z - norm.top) * norm.inv;
  }
  if (mine) {
    a.ids[(size_t)t * a.k + lane] = my_id;
    a.w[(size_t)t * a.k + lane] = v * a.scale;
  }
}

struct GradArgs {
  const void* logits;
  long long stride;
  const int* ids;
  const float* dw;
  int T, E, k, sigmoid, renormalize;
  float scale;
  void* dz;
};

// The gradient of the weights, one warp per token; lane j has slot j.  With n = s / sum of the chosen s (renormalised) and d = scale dw:
//   sigmoid  renormalised  dz_e = sum_{j: id = e} n_j (1 - s_j) (d_j - sum_i n_i d_i)      else  s_j (1 - s_j) d_j
//   softmax  renormalised  dz_e = sum_{j: id = e} n_j (d_j - sum_i n_i d_i)                 else  p_e ([e chosen] d_e - sum_i p_i d_i) for every e
// The row is put together in shared memory and written once.  Bound by the T E elements that it writes (and, in the last form, reads).
template <class L, int kPer, bool kVec>
__global__ void __launch_bounds__(kWarps * 32) choose_grad_kernel(const __grid_constant__ GradArgs a) {
  __shared__ float4 rows[kWarps][kPer * 8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x * kWarps + warp;
  grid_dep_wait();
  if (t >= a.T) return;
  const L* z_row = static_cast<const L*>(a.logits) + (size_t)t * a.stride;
  float* sum_at = reinterpret_cast<float*>(rows[warp]);
  const int id = lane < a.k ? a.ids[(size_t)t * a.k + lane] : -1;
  const bool on = (unsigned)id < (unsigned)a.E;
  const float z = on ? as_float(z_row[id]) : -INFINITY, d = on ? a.dw[(size_t)t * a.k + lane] * a.scale : 0.f;
  const bool dense = !a.sigmoid && !a.renormalize;
  float p[kPer];
  Norm norm{0.f, 0.f};
  if (dense) {
    load_row<L, kPer, kVec>(z_row, a.E, lane, p);
    norm = norm_of<kPer>(p);
#pragma unroll
    for (int i = 0; i < kPer; ++i) p[i] = expf(p[i] - norm.top) * norm.inv;
  }
#pragma unroll
  for (int i = 0; i < kPer / 4; ++i) rows[warp][lane + 32 * i] = make_float4(0.f, 0.f, 0.f, 0.f);
  float v, mean = 0.f;
  if (a.renormalize) {
    const float top = warp_max(z), shift = a.sigmoid ? fminf(top, 0.f) : top;
    float n = !on || z == -INFINITY ? 0.f : a.sigmoid && z > 0.f ? sigmoid(z) : expf(z - shift) / (a.sigmoid ? 1.f + expf(z) : 1.f);
    const float total = warp_sum(n);
    n = total == 0.f ? 0.f : n / total;
    mean = warp_sum(n * d);
    v = n * (d - mean);
    if (a.sigmoid) v *= 1.f / (1.f + expf(z));
  } else if (a.sigmoid) {
    v = on ? sigmoid(z) * (1.f / (1.f + expf(z))) * d : 0.f;
  } else {
    v = d;
    mean = warp_sum(on ? expf(z - norm.top) * norm.inv * d : 0.f);
  }
  // an expert that the token names more than once: its first slot adds the others up, in order
  const unsigned same = __match_any_sync(kAll, on ? id : -1 - lane);
  const bool first = (same & ((1u << lane) - 1u)) == 0;
  if (__any_sync(kAll, !first)) {
    float sum = 0.f;
    for (int j = 0; j < a.k; ++j) {
      const float other = __shfl_sync(kAll, v, j);
      if (same >> j & 1) sum += other;
    }
    v = sum;
  }
  __syncwarp();
  if (on && first) sum_at[id] = v;
  __syncwarp();
  L* out = static_cast<L*>(a.dz) + (size_t)t * a.E;
  if (kVec) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      const int e = expert_of<true>(i, lane);
      if (e >= a.E) break;
      const float4 r = rows[warp][e / 4];
      float o[4] = {r.x, r.y, r.z, r.w};
      if (dense) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = p[i + j] * (o[j] - mean);
      }
      store4(out + e, o);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = expert_of<false>(i, lane);
      if (e < a.E) out[e] = as_logit<L>(dense ? p[i] * (sum_at[e] - mean) : sum_at[e]);
    }
  }
}

int bytes_of(int dtype) { return dtype == MOE_DTYPE_FP32 ? 4 : dtype == MOE_DTYPE_BF16 || dtype == MOE_DTYPE_FP16 ? 2 : 0; }
bool misaligned(const void* p, unsigned to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Keys a lane: 8 up to 256 experts, 32 beyond.
template <template <class, int, bool> class Kernel, class Args>
cudaError_t launch(const Args& a, int dtype, bool vec, cudaStream_t stream) {
  const int blocks = (a.T + kWarps - 1) / kWarps;
  const auto go = [&](auto* kernel) { return launch_after(kernel, blocks, kWarps * 32, 0, stream, a); };
  const auto of = [&](auto type) {
    using L = decltype(type);
    if (a.E <= 256) return vec ? go(Kernel<L, 8, true>::fn) : go(Kernel<L, 8, false>::fn);
    return vec ? go(Kernel<L, 32, true>::fn) : go(Kernel<L, 32, false>::fn);
  };
  return dtype == MOE_DTYPE_FP32 ? of(float{}) : dtype == MOE_DTYPE_FP16 ? of(__half{}) : of(__nv_bfloat16{});
}
template <class L, int kPer, bool kVec>
struct Choose {
  static constexpr auto* fn = choose_kernel<L, kPer, kVec>;
};
template <class L, int kPer, bool kVec>
struct Grad {
  static constexpr auto* fn = choose_grad_kernel<L, kPer, kVec>;
};

}  // namespace
}  // namespace moe

extern "C" {

int moe_choose_experts(const void* logits, int64_t logits_stride, int32_t dtype, const float* bias, int32_t n_tokens, int32_t n_experts,
                       int32_t top_k, int32_t n_groups, int32_t top_groups, int32_t group_sum, int32_t scores, int32_t renormalize, float scale,
                       int32_t* topk_ids, float* topk_w, void* stream) {
  using namespace moe;
  const int el = bytes_of(dtype);
  if (n_tokens < 0 || n_experts < 1 || n_experts > kMaxE || top_k < 1 || top_k > kMaxK || top_k > n_experts || !el) return MOE_EINVAL;
  if (n_groups < 1 || n_groups > kMaxGroups || n_experts % n_groups || top_groups < 1 || top_groups > n_groups || (group_sum != 1 && group_sum != 2) ||
      top_k > top_groups * (n_experts / n_groups))
    return MOE_EINVAL;
  if (scores != MOE_SCORES_SOFTMAX && scores != MOE_SCORES_SIGMOID) return MOE_EINVAL;
  if (n_tokens == 0) return MOE_OK;
  if (!logits || !topk_ids || !topk_w || logits_stride < n_experts) return MOE_EINVAL;
  if (misaligned(logits, el) || misaligned(bias, 4) || misaligned(topk_ids, 4) || misaligned(topk_w, 4)) return MOE_EINVAL;
  const ChooseArgs a{logits, bias, logits_stride, n_tokens, n_experts, top_k, n_groups, top_groups, group_sum, scores == MOE_SCORES_SIGMOID,
                     renormalize != 0, scale, topk_ids, topk_w};
  const bool vec = n_experts % 4 == 0 && logits_stride % 4 == 0 && !misaligned(logits, 4 * el);
  return launch<Choose>(a, dtype, vec, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

int moe_choose_experts_grad(const void* logits, int64_t logits_stride, int32_t dtype, const int32_t* topk_ids, const float* d_topk_w, int32_t n_tokens,
                            int32_t n_experts, int32_t top_k, int32_t scores, int32_t renormalize, float scale, void* d_logits, void* stream) {
  using namespace moe;
  const int el = bytes_of(dtype);
  if (n_tokens < 0 || n_experts < 1 || n_experts > kMaxE || top_k < 1 || top_k > kMaxK || top_k > n_experts || !el) return MOE_EINVAL;
  if (scores != MOE_SCORES_SOFTMAX && scores != MOE_SCORES_SIGMOID) return MOE_EINVAL;
  if (n_tokens == 0) return MOE_OK;
  if (!logits || !topk_ids || !d_topk_w || !d_logits || logits_stride < n_experts) return MOE_EINVAL;
  if (misaligned(logits, el) || misaligned(topk_ids, 4) || misaligned(d_topk_w, 4) || misaligned(d_logits, el)) return MOE_EINVAL;
  const GradArgs a{logits, logits_stride, topk_ids, d_topk_w, n_tokens, n_experts, top_k, scores == MOE_SCORES_SIGMOID, renormalize != 0, scale, d_logits};
  const bool vec = n_experts % 4 == 0 && logits_stride % 4 == 0 && !misaligned(logits, 4 * el) && !misaligned(d_logits, 4 * el);
  return launch<Grad>(a, dtype, vec, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MOE_OK : MOE_ECUDA;
}

}  // extern "C"
