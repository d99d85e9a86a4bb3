// moe_choose_experts / moe_choose_experts_grad: the routers that moe_route does not know -- scores by softmax or sigmoid, a bias that counts for
// the choice alone, groups of experts of which the best are kept -- and the gradient of their weights.
//
//   s_e = softmax(z)_e  or  1 / (1 + exp(-z_e));   c_e = s_e + bias_e;   value of a group: the sum of its one or two largest c
//   the top_groups groups of largest value are kept; the k largest c of their experts are chosen;   w_j = scale s_j  (/ sum_i s_i)
//
// Who is chosen is decided as in 64 bits.  c is computed in fp32 with a bound on its error, and where two candidates whose order matters lie closer than that
// (and are not equal by their inputs) those few are put in order by their values in fp64: one token of some hundreds.  (All of it in fp64 would be 480 double
// operations a lane and token: 14 us for 16 384 tokens of 256 experts.)
//
// One warp per token.  A lane sorts its own values once, as integers of the same order whose last bits say which of its experts it is (what they displace counts as
// an error of c like the others); then a pick is one maximum over the warp, one minimum over the ids that have it, and the winner's list moves up.
// Bound by instruction issue (0.75 a clock; 565 instructions a token of 256 experts, 110 more for scores and a bias, 320 for groups): 16 384 tokens of 256 experts, the best eight of
// all 13.5 us, of four of eight groups 19.9; their 16.8 MB take 2.6.  (Every pick a maximum over all keys of a lane, groups by loops: 37 and 67 us.  A warp that goes on to
// another token, with its loads ahead: 17 and 25; more blocks a multiprocessor: the same.)
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

// unsigned order = double order (-0 counts as +0), NaN above every number; 0 is below everything: "no candidate"
__device__ __forceinline__ unsigned long long key_of(double v) {
  if (v != v) return ~0ull;
  const unsigned long long u = __double_as_longlong(v + 0.0);
  return (u >> 63) ? ~u : (u | 1ull << 63);
}
// signed order = float order (not of NaN); kNone is below everything
constexpr int kNone = (int)0x80000000;
__device__ __forceinline__ int key_of(float v) {
  const int u = __float_as_int(v + 0.0f);
  return u ^ ((u >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float of_key(int key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }

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

// The expert of a lane's i-th element.  kVec: rows, and the bias, are aligned to four elements, a lane has four neighbours at a time.
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

__device__ __forceinline__ float sigmoid(float z) { return __fdividef(1.f, 1.f + expf(-z)); }
// of the weights: a score relative to that of a logit `shift` (softmax: the largest of the chosen; sigmoid(z) = exp(z) / (1 + exp(z)): the same where it is
// negative, else 0), so that scores that are tiny alike have weights
__device__ __forceinline__ float relative_score(float z, float shift, bool is_sigmoid) {
  if (z == -INFINITY) return 0.f;
  return is_sigmoid ? __fdividef(expf(fminf(z, 0.f) - shift), 1.f + expf(-fabsf(z))) : expf(z - shift);
}
__device__ __forceinline__ double sigmoid(double z) { return 1.0 / (1.0 + exp(-z)); }

// The same to some steps of fp32, for the comparison of experts: exp through 2^x (its argument rounded: |x| halves of a step of 2^-23, the power two), the
// reciprocal one.
__device__ __forceinline__ float quick_exp(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
  return r;
}
__device__ __forceinline__ float quick_sigmoid(float z) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + quick_exp(-z)));
  return r;
}
// Of a softmax: the largest logit (0 where there is none above -inf, so that exp gives 0), and 1 over the sum (0 for such a row, NaN for one with NaN or
// +inf)
struct Norm {
  float top, inv;
};
template <int kPer>
__device__ __forceinline__ Norm norm_of(const float (&z)[kPer]) {
  float m = -INFINITY, part[4] = {};         // (the longest chain of additions: kPer / 4 + 6)
#pragma unroll
  for (int i = 0; i < kPer; ++i) m = fmaxf(m, z[i]);
  m = warp_max(m);
  if (m == -INFINITY) m = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) part[i % 4] += quick_exp(z[i] - m);
  const float sum = warp_sum((part[0] + part[1]) + (part[2] + part[3]));
  return Norm{m, sum == 0.f ? 0.f : 1.f / sum};
}
// Bounds on the error of a quick score and of its sum with a bias, in steps of 2^-23.  exp(x): 2 + 0.8 |x| (softmax: 1.3 |x|, x itself is rounded); sigmoid: 1.5 for the
// addition and the reciprocal.  Softmax, at 1024 experts: half a step for each of the 14 additions that a term goes through, 7; its terms' errors, 2 and 1.3 times their mean |x| by
// shares, 8 (that mean is largest where n = E - 1 are alike below the top: a, with a = n exp(-1 - a), 4.5); quotient and product, 1; with the 2 of the score's own exp 18 of 25.  Of any
// score, where s |x| counts less than 1.  What is lost below 2^-126 is less than 2^-120.
__device__ __forceinline__ float error_of(float s, float c, float far, bool is_sigmoid) {
  return (s * (is_sigmoid ? 6.f + far : 25.f + 2.f * far) + fabsf(c)) * 0x1p-23f + 0x1p-120f;
}
__device__ __forceinline__ float error_of_any(float c) { return (26.f + fabsf(c)) * 0x1p-23f; }

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

__device__ __forceinline__ int warp_max_key(float v) { return __reduce_max_sync(kAll, key_of(v)); }

// The two largest of a group, on their way over its values
template <class V>
struct Two {
  V one = -INFINITY, two = -INFINITY;
  __device__ __forceinline__ void join(V o1, V o2) {
    two = fmax(fmin(one, o1), fmax(two, o2));
    one = fmax(one, o1);
  }
  __device__ __forceinline__ V value(const ChooseArgs& a, int size) const { return a.group_sum > 1 && size > 1 ? one + two : one; }
  // (a group of one expert, or one that holds -inf, has no second value that counts)
  __device__ __forceinline__ float error(V v) const {
    return one == -INFINITY ? 0.f : error_of_any(one) + (two == -INFINITY ? 0.f : error_of_any(two) + (fabsf(v)) * 0x1p-23f);
  }
};
// whether fp32 cannot tell which groups are kept: the least of those inside, the largest of those outside, the largest error
__device__ __forceinline__ bool groups_close(bool any, bool inside, float in, bool outside, float out, float err) {
  const float low = -of_key(warp_max_key(any && inside ? -in : -INFINITY)), high = of_key(warp_max_key(any && outside ? out : -INFINITY));
  return !(low - high > 2.f * of_key(warp_max_key(any ? err : 0.f)));
}

// Which groups are kept, as a bit mask; c(e): an expert's value; for groups of any size.  Several neighbouring lanes have a group: each goes over a part of it, then the two
// largest are joined.
template <class V, class F>
__device__ __forceinline__ unsigned keep_groups(const ChooseArgs& a, F c, int lane, bool& close) {
  const int size = a.E / a.groups;
  int per = 1;                          // lanes a group: a power of two
  while (2 * per * a.groups <= 32 && 2 * per <= size) per *= 2;
  const int g = lane / per, q = lane % per;
  Two<V> best;
  if (g < a.groups) {
#pragma unroll 1
    for (int i = q; i < size; i += per) best.join(c(g * size + i), -INFINITY);
  }
  for (int b = per / 2; b >= 1; b >>= 1) {
    const V o1 = __shfl_xor_sync(kAll, best.one, b), o2 = __shfl_xor_sync(kAll, best.two, b);
    best.join(o1, o2);
  }
  const V value = best.value(a, size);
  const bool mine = g < a.groups && q == 0;
  int before = 0;
#pragma unroll 1
  for (int o = 0; o < a.groups; ++o) {
    const V other = __shfl_sync(kAll, value, o * per);
    before += other > value || (other == value && o < g);
  }
  close = sizeof(V) == 4 && groups_close(mine, before < a.top_groups, value, before >= a.top_groups, value, best.error(value));
  const unsigned firsts = __ballot_sync(kAll, mine && before < a.top_groups);
  unsigned kept = 0;
  for (int o = 0; o < a.groups; ++o) kept |= (firsts >> (o * per) & 1u) << o;
  return kept;
}
// ... by their values in fp64
template <class L>
__device__ __noinline__ unsigned keep_groups_exactly(const ChooseArgs& a, const L* row, double top, int lane) {
  double sum = 0.0;
  if (!a.sigmoid) {
#pragma unroll 1
    for (int e = lane; e < a.E; e += 32) sum += exp((double)as_float(row[e]) - top);
    sum = warp_sum(sum);
  }
  bool close;
  return keep_groups<double>(a, [&](int e) {
    const double z = as_float(row[e]);
    return (a.sigmoid ? sigmoid(z) : sum == 0.0 ? 0.0 : exp(z - top) / sum) + (a.bias ? (double)a.bias[e] : 0.0);
  }, lane, close);
}
// The same where a lane's four neighbours are of one group and a group's lanes are a power of two.  Values become keys with the group in their last five bits, one a lane;
// the last of top_groups maxima over the warp says who is kept.
template <int kPer>
__device__ __forceinline__ unsigned keep_groups(const ChooseArgs& a, const float (&c)[kPer], int lane, bool& close) {
  const int size = a.E / a.groups, lanes = size / 4, shift = 31 - __clz(lanes);          // lanes of a group; 32 >> shift groups in 128 experts
  float value = -INFINITY, err = 0.f;
#pragma unroll
  for (int q = 0; q < kPer / 4; ++q) {
    const float h1 = fmaxf(c[4 * q], c[4 * q + 1]), l1 = fminf(c[4 * q], c[4 * q + 1]), h2 = fmaxf(c[4 * q + 2], c[4 * q + 3]), l2 = fminf(c[4 * q + 2], c[4 * q + 3]);
    Two<float> best;
    best.one = h1;
    best.two = l1;
    best.join(h2, l2);
    for (int b = 1; b < lanes; b <<= 1) {
      const float o1 = __shfl_xor_sync(kAll, best.one, b), o2 = __shfl_xor_sync(kAll, best.two, b);
      best.join(o1, o2);
    }
    const float mine = best.value(a, size);
    err = fmaxf(err, best.error(mine));
    const float v = __shfl_sync(kAll, mine, lane << shift & 31);
    if (lane >> (5 - shift) == q) value = v;
  }
  int key = lane < a.groups ? (key_of(value) & ~31) | (31 - lane) : kNone, last = 0;
  bool kept = false;
  for (int j = 0; j < a.top_groups; ++j) {
    last = __reduce_max_sync(kAll, key);
    if (key == last) {
      kept = true;
      key = kNone;
    }
  }
  const int next = __reduce_max_sync(kAll, key);
  const float in = of_key(last & ~31), out = of_key(next | 31);
  close = !(in - out > 2.f * __int_as_float(__reduce_max_sync(kAll, __float_as_int(err))));
  return __ballot_sync(kAll, kept);
}

// Whether all experts of a row are equal by their inputs (a padded token, say): the first ones are chosen then.
template <class L>
__device__ __noinline__ bool all_equal(const ChooseArgs& a, const L* row, int lane) {
  bool same = true;
#pragma unroll 1
  for (int e = lane; e < a.E; e += 32) same &= as_float(row[e]) == as_float(row[0]) && (!a.bias || a.bias[e] == a.bias[0]);
  return __all_sync(kAll, same);
}

// descending, by compare-exchanges of the largest first
template <int kN>
__device__ __forceinline__ void sort_down(int (&v)[kN]) {
  const auto order = [&](int i, int j) {
    const int hi = max(v[i], v[j]), lo = min(v[i], v[j]);
    v[i] = hi;
    v[j] = lo;
  };
  if (kN == 4) {
    order(0, 1); order(2, 3); order(0, 2); order(1, 3); order(1, 2);
  } else {                              // Batcher's merge exchange for eight
    order(0, 4); order(1, 5); order(2, 6); order(3, 7);
    order(0, 2); order(1, 3); order(4, 6); order(5, 7);
    order(2, 4); order(3, 5); order(0, 1); order(2, 3); order(4, 5); order(6, 7);
    order(1, 4); order(3, 6);
    order(1, 2); order(3, 4); order(5, 6);
  }
}

template <class L, int kPer, bool kVec>
__global__ void __launch_bounds__(kWarps * 32) choose_kernel(const __grid_constant__ ChooseArgs a) {
  constexpr int kList = kPer < 8 ? kPer : 8, kLists = kPer / kList, kWhich = kPer - 1;
  __shared__ union {
    float by_expert[kPer * 32];
    int4 sorted[kLists][32][kList / 4];
  } space[kWarps];
  __shared__ int2 picks[kWarps][kMaxK];            // key and lane
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = blockIdx.x * kWarps + warp;
  grid_dep_wait();
  if (t >= a.T) return;
  const L* row = static_cast<const L*>(a.logits) + (size_t)t * a.stride;
  const bool grouped = a.top_groups < a.groups, scored = a.bias || grouped;
  constexpr int kInf = 0x7f800000;                 // the key of infinity: those of NaN, which key_of makes positive, are above it
  Norm norm{0.f, 0.f};
  int key[kLists][kList];
  bool slow = false, flat = false;
  {
    float z[kPer], c[kPer];
    load_row<L, kPer, kVec>(row, a.E, lane, z);
    if (!a.sigmoid && (scored || !a.renormalize)) {
      norm = norm_of<kPer>(z);
      slow = norm.inv != norm.inv;
    }
    if (scored) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        c[i] = expert_of<kVec>(i, lane) < a.E ? a.sigmoid ? quick_sigmoid(z[i]) : quick_exp(z[i] - norm.top) * norm.inv : -INFINITY;
      if (a.bias) {
        load_row<float, kPer, kVec>(a.bias, a.E, lane, z);
#pragma unroll
        for (int i = 0; i < kPer; ++i) z[i] = c[i] += z[i];
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i / kList][i % kList] = expert_of<kVec>(i, lane) < a.E ? (key_of(z[i]) & ~kWhich) | (kWhich - i) : kNone;
    if (grouped) {
      int top = kNone;
#pragma unroll
      for (int i = 0; i < kPer; ++i) top = max(top, key[i / kList][i % kList]);
      slow |= __any_sync(kAll, top > (kInf | kWhich));
      const int size = a.E / a.groups;
      bool close;
      unsigned groups;
      if (kVec && size % 4 == 0 && size <= 128 && (size & (size - 1)) == 0) {
        groups = keep_groups<kPer>(a, c, lane, close);
      } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (expert_of<kVec>(i, lane) < a.E) space[warp].by_expert[expert_of<kVec>(i, lane)] = c[i];
        __syncwarp();
        groups = keep_groups<float>(a, [&](int e) { return space[warp].by_expert[e]; }, lane, close);
        __syncwarp();
      }
      if (close && !slow) {
        flat = all_equal(a, row, lane);
        if (!flat) groups = keep_groups_exactly(a, row, (double)norm.top, lane);
      }
      const unsigned inverse = ((1u << 20) + size - 1) / size;      // e / size = e inverse >> 20 for e < 2^10
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (kVec && i % 4 && size % 4 == 0) continue;      // (four neighbours at once)
        if (!(groups >> (((unsigned)expert_of<kVec>(i, lane) * inverse >> 20) & 31) & 1)) {
          key[i / kList][i % kList] = kNone;
          if (kVec && size % 4 == 0) key[i / kList][i % kList + 1] = key[i / kList][i % kList + 2] = key[i / kList][i % kList + 3] = kNone;
        }
      }
    }
  }
  int my_id = 0, pos = lane;            // the expert of this lane's slot, and which slot it is
  if (!slow && !flat) {
    int head[kLists], at[kLists];
#pragma unroll
    for (int l = 0; l < kLists; ++l) {
      sort_down<kList>(key[l]);
#pragma unroll
      for (int i = 0; i < kList; i += 4) space[warp].sorted[l][lane][i / 4] = make_int4(key[l][i], key[l][i + 1], key[l][i + 2], key[l][i + 3]);
      head[l] = key[l][0];
      at[l] = 0;
    }
    const auto best = [&] {
      int b = head[0];
#pragma unroll
      for (int l = 1; l < kLists; ++l) b = max(b, head[l]);
      return b;
    };
    const auto take = [&](int j, int mine, int m) {        // of the lanes that have the maximum the one whose expert is first
      bool won = (mine | kWhich) == m;
      const unsigned same = __ballot_sync(kAll, won);
      if (same & (same - 1)) {
        const unsigned id = won ? (unsigned)expert_of<kVec>(kWhich - (mine & kWhich), lane) : kAll;
        won = __reduce_min_sync(kAll, id) == id && won;
      }
      if (won) {
        picks[warp][j] = make_int2(mine, lane);
#pragma unroll
        for (int l = 0; l < kLists; ++l)
          if (kLists == 1 || head[l] == mine) head[l] = ++at[l] < kList ? reinterpret_cast<const int*>(space[warp].sorted[l][lane])[at[l]] : kNone;
      }
    };
    int m = 0, top = 0;
    for (int j = 0; j < a.k; ++j) {
      const int mine = best();
      m = __reduce_max_sync(kAll, mine | kWhich);
      if (j == 0) {
        top = m;
        slow = m > (kInf | kWhich);
      }
      take(j, mine, m);
    }
    // behind the k-th there follow those that may still be larger, until one is not (or none is left)
    float least = of_key(m & ~kWhich);
    if (a.bias) least -= error_of_any(least);
    int picked = a.k;
    for (;;) {
      const int mine = best();
      m = __reduce_max_sync(kAll, mine | kWhich);
      const float above = of_key(m);                      // nothing that is left is larger
      if (slow || m == (kNone | kWhich) || (a.bias ? above + error_of_any(above) < least || (above == -INFINITY && least > above) : above < least)) break;
      if (picked == a.k && m == top && all_equal(a, row, lane)) {
        flat = true;
        break;
      }
      if (picked == kMaxK) {            // no lane for one more
        slow = true;
        break;
      }
      take(picked++, mine, m);
    }
    __syncwarp();
    const int2 pick = lane < picked ? picks[warp][lane] : make_int2(0, 0);
    my_id = expert_of<kVec>(kWhich - (pick.x & kWhich), pick.y);
    // neighbours in the order: surely so, ...
    const float low = of_key(pick.x & ~kWhich), next = __shfl_down_sync(kAll, of_key(pick.x | kWhich), 1);
    if (!slow && !flat && __any_sync(kAll, lane < picked - 1 && !(low - next > (a.bias ? error_of_any(low) + error_of_any(next) : 0.f)))) {
      // ... by their own bounds, or because their inputs are equal?
      const float z = lane < picked ? as_float(row[my_id]) : 0.f, b = a.bias && lane < picked ? a.bias[my_id] : 0.f;
      float c = z, err = 0.f;
      if (a.bias) {
        const float s = a.sigmoid ? quick_sigmoid(z) : quick_exp(z - norm.top) * norm.inv;
        c = s + b;
        err = error_of(s, c, fabsf(z - norm.top), a.sigmoid);       // (sigmoid: norm.top is 0)
      }
      const float nc = __shfl_down_sync(kAll, c, 1), nerr = __shfl_down_sync(kAll, err, 1), nz = __shfl_down_sync(kAll, z, 1), nb = __shfl_down_sync(kAll, b, 1);
      if (__any_sync(kAll, lane < picked - 1 && !(z == nz && b == nb) && !(c - nc > err + nerr))) {      // by their values in fp64
        double exact = z;
        if (a.bias && a.sigmoid) exact = sigmoid((double)z) + (double)b;
        if (a.bias && !a.sigmoid) {
          double sum = 0.0;
#pragma unroll 1
          for (int e = lane; e < a.E; e += 32) sum += exp((double)as_float(row[e]) - (double)norm.top);
          sum = warp_sum(sum);
          exact = (sum == 0.0 ? 0.0 : exp((double)z - (double)norm.top) / sum) + (double)b;
        }
        pos = 0;
        for (int j = 0; j < picked; ++j) {
          const double other = __shfl_sync(kAll, exact, j);
          const int oid = __shfl_sync(kAll, my_id, j);
          pos += other > exact || (other == exact && oid < my_id);
        }
      }
    }
    if (lane >= picked) pos = kMaxK;
  }
  if (flat) my_id = pos = lane;
  if (slow) {                           // NaN, or more that are close than a warp has lanes
    my_id = choose_slowly<L, kPer, kVec>(a, row, lane);
    pos = lane;
  }
  const bool mine = pos < a.k;
  const float z = mine ? as_float(row[my_id]) : -INFINITY;
  float v;
  if (a.renormalize) {
    const float top = of_key(warp_max_key(z));
    v = relative_score(z, a.sigmoid ? fminf(top, 0.f) : top, a.sigmoid);
    const float sum = warp_sum(v);
    v = sum == 0.f ? 0.f : __fdividef(v, sum);
    if (norm.inv != norm.inv) v = norm.inv;       // a NaN in the row (one that nobody looked for above is among the chosen)
  } else {
    v = a.sigmoid ? sigmoid(z) : expf(z - norm.top) * norm.inv;
  }
  if (mine) {
    a.ids[(size_t)t * a.k + pos] = my_id;
    a.w[(size_t)t * a.k + pos] = v * a.scale;
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
    const float top = of_key(warp_max_key(z));
    float n = relative_score(z, a.sigmoid ? fminf(top, 0.f) : top, a.sigmoid);
    const float total = warp_sum(n);
    n = total == 0.f ? 0.f : __fdividef(n, total);
    mean = warp_sum(n * d);
    v = n * (d - mean);
    if (a.sigmoid) v *= sigmoid(-z);
  } else if (a.sigmoid) {
    v = on ? sigmoid(z) * sigmoid(-z) * d : 0.f;
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

// Experts a lane: 4 up to 128 experts, 8 up to 256, 16 up to 512, 32 beyond.  (us, 16 384 tokens of 384 experts, 16 / 32 a lane: the best eight of all 17 / 30, with scores and a
// bias 23 / 41, of four of eight groups 37 / 60, the gradient 10 / 13; one token 2.6 / 3.3.)
template <template <class, int, bool> class Kernel, class Args>
cudaError_t launch(const Args& a, int dtype, bool vec, cudaStream_t stream) {
  const int blocks = (a.T - 1) / kWarps + 1;
  const auto go = [&](auto* kernel) { return launch_after(kernel, blocks, kWarps * 32, 0, stream, a); };
  const auto of = [&](auto type) {
    using L = decltype(type);
    if (a.E <= 128) return vec ? go(Kernel<L, 4, true>::fn) : go(Kernel<L, 4, false>::fn);
    if (a.E <= 256) return vec ? go(Kernel<L, 8, true>::fn) : go(Kernel<L, 8, false>::fn);
    if (a.E <= 512) return vec ? go(Kernel<L, 16, true>::fn) : go(Kernel<L, 16, false>::fn);
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
  const bool vec = n_experts % 4 == 0 && logits_stride % 4 == 0 && !misaligned(logits, 4 * el) && !misaligned(bias, 16);
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
