// scored.hip - routing by scores (arXiv 2609.28053, Eq. 1 with the choice made on the scores
// themselves): the experts of the largest score plus bias within the best groups, their
// weights, and the gradient with respect to the logits.
#include "eqb_internal.hpp"

namespace eqb {
namespace {

constexpr int kPer = 8;                 // experts of a lane
constexpr int kScoredThreads = 256, kScoredWaves = kScoredThreads / 64;

template <int kDtype>
struct Logit;
template <>
struct Logit<EQB_DTYPE_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float to_f(raw x) { return __uint_as_float((uint32_t)x << 16); }
};
template <>
struct Logit<EQB_DTYPE_F16> {
  typedef _Float16 raw;
  static __device__ __forceinline__ float to_f(raw x) { return (float)x; }
};
template <>
struct Logit<EQB_DTYPE_F32> {
  typedef float raw;
  static __device__ __forceinline__ float to_f(raw x) { return x; }
};

// A masked logit (-inf or NaN) becomes -inf, +inf the largest finite number.
constexpr float kLargest = 3.402823466e38f;
__device__ __forceinline__ float clean(float z) {
  const float lowest = -__builtin_inff();
  return z > lowest ? fminf(z, kLargest) : lowest;
}

// exp(-a), a >= 0 (infinity gives 0): 2^(-p) (1 - l ln 2) with p + l = a log2 e in two parts,
// within 2^-22; without subnormal results.
__device__ __forceinline__ float exp_neg(float a) {
  const float kLog2e = 1.44269502162933349609375f, kLow = 1.92596303e-8f, kLn2 = 0.693147182f;
  a = fminf(a, 200.0f);
  const float p = a * kLog2e;
  const float l = __builtin_fmaf(a, kLow, __builtin_fmaf(a, kLog2e, -p));
  const float e = __builtin_amdgcn_exp2f(-p);
  return __builtin_fmaf(-e * kLn2, l, e);
}
__device__ __forceinline__ double exp_neg(double a) { return exp(-a); }

// sigmoid(z) and 1 - sigmoid(z); of -inf 0 and 1
__device__ __forceinline__ void sigmoid_pair(float z, float& s, float& rest) {
  const float e = exp_neg(fabsf(z)), r = newton_rcp(1.0f + e), q = e * r;
  s = z >= 0.0f ? r : q;
  rest = z >= 0.0f ? q : r;
}
__device__ __forceinline__ float sigmoid_of(float z) {
  float s, rest;
  sigmoid_pair(z, s, rest);
  return s;
}
__device__ __forceinline__ double sigmoid_of(double z) { return 1.0 / (1.0 + exp(-z)); }

// Normalized weights are ratios of scores.  Where the chosen ones of a row sum to less than this, as after a
// bias has chosen logits far below the largest, some may have few bits or none in binary32: they are formed
// again over a power of e, that of the largest chosen logit.  Left is what lies below 2^-106 of the weights' sum.
constexpr float kLowSum = 0x1p-20f;
__device__ __forceinline__ float raised_score(float z, float most, bool softmax) {
  float s, rest = 1.0f;
  if (!softmax) sigmoid_pair(z, s, rest);           // s = e^z (1 - s)
  return exp_neg(most - z) * rest;
}

template <class F>
__device__ __forceinline__ F lowest_of() { return -(F)__builtin_inf(); }

// Folds over the L lanes of a row.
template <int L>
__device__ __forceinline__ float row_max(float x) { return group_max<L>(x); }
template <int L>
__device__ __forceinline__ double row_max(double x) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) x = fmax(x, __shfl_xor(x, d));
  return x;
}
template <int L>
__device__ __forceinline__ float row_sum(float x) { return group_sum<L>(x); }
template <int L>
__device__ __forceinline__ double row_sum(double x) {
#pragma unroll
  for (int d = 1; d < L; d <<= 1) x += __shfl_xor(x, d);
  return x;
}
template <int L>
__device__ __forceinline__ int row_min(int x) {
  return group_fold<L>(x, [](int a, int b) { return a < b ? a : b; });
}

// The scores of a row's kPer experts of this lane in F, and what decides (-inf: masked).
template <int L, class F>
__device__ __forceinline__ void scores_of(const float (&z)[kPer], const float (&b)[kPer], bool softmax, F (&q)[kPer]) {
  if (softmax) {
    float top = z[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) top = fmaxf(top, z[i]);
    top = row_max<L>(top);
    if (top == -__builtin_inff()) top = 0.0f;
    F sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      q[i] = exp_neg((F)top - (F)z[i]);
      sum += q[i];
    }
    sum = row_sum<L>(sum);
#pragma unroll
    for (int i = 0; i < kPer; ++i) q[i] = q[i] / sum;
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) q[i] = sigmoid_of((F)z[i]);
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const F v = q[i] + (F)b[i];
    q[i] = z[i] > -__builtin_inff() && v == v ? v : lowest_of<F>();
  }
}

// (a1, a2): the largest and the next of two such pairs
template <class F>
__device__ __forceinline__ void merge2(F& a1, F& a2, F b1, F b2) {
  const F lo = fmin(a1, b1);
  a1 = fmax(a1, b1);
  a2 = fmax(lo, fmax(a2, b2));
}

// A group's score of its two best.  In binary32 a sum that it does not hold counts as its largest or lowest number, so that
// groups of such sums are no masked ones (-inf) and meet, which near() sends to binary64.
__device__ __forceinline__ float sum_of_two(float a, float b) { return fminf(fmaxf(a + b, -kLargest), kLargest); }
__device__ __forceinline__ double sum_of_two(double a, double b) { return a + b; }

// Every expert's group score.
template <int L, class F>
__device__ __forceinline__ void group_scores(const F (&q)[kPer], int each, int group_top, F (&g)[kPer]) {
  F t1[kPer], t2[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    t1[i] = q[i];
    t2[i] = lowest_of<F>();
  }
#pragma unroll
  for (int d = 1; d < kPer; d <<= 1) {
    if (each > d) {
      F o1[kPer], o2[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        o1[i] = t1[i ^ d];
        o2[i] = t2[i ^ d];
      }
#pragma unroll
      for (int i = 0; i < kPer; ++i) merge2(t1[i], t2[i], o1[i], o2[i]);
    }
  }
  if (each > kPer) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) {
      if (each > d * kPer) {
        const F o1 = __shfl_xor(t1[0], d), o2 = __shfl_xor(t2[0], d);
        merge2(t1[0], t2[0], o1, o2);
      }
    }
#pragma unroll
    for (int i = 1; i < kPer; ++i) {
      t1[i] = t1[0];
      t2[i] = t2[0];
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) g[i] = group_top == 2 && t2[i] > lowest_of<F>() ? sum_of_two(t1[i], t2[i]) : t1[i];
}

// The largest of a row's values and the lowest place that has it (kNone: all -inf).
constexpr int kNone = 1 << 20;
template <int L, class F>
__device__ __forceinline__ int largest(const F (&q)[kPer], int l, F& top) {
  F m = q[0];
#pragma unroll
  for (int i = 1; i < kPer; ++i) m = fmax(m, q[i]);
  top = row_max<L>(m);
  int at = kNone;
#pragma unroll
  for (int i = kPer - 1; i >= 0; --i) at = q[i] == top ? l * kPer + i : at;
  at = row_min<L>(at);
  return top > lowest_of<F>() ? at : kNone;
}

// Two sums q of a score and its bias in binary32 nearer than this may be the other way round. s is at most
// |q| and the largest bias, and q is rounded once (2^-24 |q|).
//   A sigmoid is off by (1 - s) |z| 2^-23.4 of itself from its exponential's argument and by 2^-21.7 from the
//   exponential, the sum and the reciprocal. Of each 0.75 2^-20 (|q| + bias) covers all but
//   s max(0, |z| - 3.8) 2^-23.4 < 2^-30.3 (the maximum of e^-z (z - 3.8), at z = 4.8): 2^-28 covers that for two pairs.
//   A softmax's exponential is off by d 2^-22.7 of itself, d the distance to the largest logit (2^-17.4 up to
//   d = 39, less than 2^-56 behind that), and its sum of 256, a tree of 32 and 3 levels or of 8 and 5, by 35
//   2^-24, the same way for a row: 2^-16 (|q| + bias) + 2^-54.
__device__ __forceinline__ bool near(float a, float b, float most_bias, bool softmax) {
  // two infinities are near
  return !(a - b > (softmax ? 0x1p-16f : 0x1.8p-20f) * (fabsf(a) + most_bias) + (softmax ? 0x1p-54f : 0x1p-28f));
}
__device__ __forceinline__ bool near(double, double, float, bool) { return false; }

// Chooses a row's K experts by rank into `chosen` (kNone where there are none left); whether an
// order that matters was too near to call.  In binary32 the (K + 1)st is looked at as well.
template <int L, class F>
__device__ __forceinline__ bool choose(const ScoredArgs& a, const float (&z)[kPer], const float (&b)[kPer],
                                       float most_bias, int l, int16_t* chosen) {
  constexpr bool kQuick = sizeof(F) == 4;
  F q[kPer];
  scores_of<L>(z, b, a.softmax, q);
  bool doubt = false;
  if (a.top_groups < a.groups) {
    const int each = a.E / a.groups;
    F g[kPer];
    group_scores<L>(q, each, a.group_top, g);
    bool in[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      in[i] = false;
      if ((l * kPer + i) & (each - 1)) g[i] = lowest_of<F>();     // the first of a group stands for it
    }
    F last = 0;
    for (int k = 0; k < a.top_groups + (kQuick ? 1 : 0); ++k) {
      F top;
      const int at = largest<L>(g, l, top);
      if (k == a.top_groups) {
        doubt = doubt || (at != kNone && near(last, top, 2 * most_bias, a.softmax));
      } else {
        last = top;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int e = l * kPer + i;
          in[i] = in[i] || (e & -each) == at;
          if (e == at) g[i] = lowest_of<F>();
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (!in[i]) q[i] = lowest_of<F>();
  }
  // without a bias the scores are in the logits' order, which is exact
  const bool by_logits = a.bias == nullptr;
  if (by_logits) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) q[i] = q[i] > lowest_of<F>() ? (F)z[i] : lowest_of<F>();
  }
  F last = 0;
  for (int k = 0; k < a.K + (kQuick && !by_logits ? 1 : 0); ++k) {
    F top;
    const int at = largest<L>(q, l, top);
    if (kQuick && !by_logits && k > 0) doubt = doubt || (at != kNone && near(last, top, most_bias, a.softmax));
    last = top;
    if (k < a.K && l == 0) chosen[k] = (int16_t)(at == kNone ? -1 : at);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (l * kPer + i == at) q[i] = lowest_of<F>();
  }
  return doubt;
}

template <int E, int kDtype>
__device__ __forceinline__ void load_row(const void* z, int64_t t, int l, float (&v)[kPer]) {
  typedef typename Logit<kDtype>::raw raw;
  typedef raw vec __attribute__((ext_vector_type(kPer), aligned(16)));       // what a caller promises
  const vec x = *reinterpret_cast<const vec*>(static_cast<const raw*>(z) + t * E + l * kPer);
#pragma unroll
  for (int i = 0; i < kPer; ++i) v[i] = clean(Logit<kDtype>::to_f(x[i]));
}

template <int E, int kDtype>
__global__ __launch_bounds__(kScoredThreads) void route_scored_kernel(const ScoredArgs a) {
  constexpr int L = E / kPer, kRows = 64 / L;           // rows of a wave
  __shared__ int16_t sh_chosen[kScoredWaves * kRows][E];
  typedef typename Logit<kDtype>::raw raw;
  const int lane = threadIdx.x & 63, l = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int16_t* const chosen = sh_chosen[wave * kRows + lane / L];
  float b[kPer];
  float most_bias = 0.0f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    b[i] = a.bias ? a.bias[l * kPer + i] : 0.0f;
    const float m = fabsf(b[i]);
    most_bias = fmaxf(most_bias, m < __builtin_inff() ? m : 0.0f);
  }
  most_bias = row_max<L>(most_bias);
  const int64_t step = (int64_t)gridDim.x * kScoredWaves * kRows;
  for (int64_t t0 = ((int64_t)blockIdx.x * kScoredWaves + wave) * kRows; t0 < a.T; t0 += step) {
    const bool live = t0 + lane / L < a.T;
    const int64_t t = live ? t0 + lane / L : a.T - 1;
    float z[kPer];
    load_row<E, kDtype>(a.z, t, l, z);
    const bool doubt = choose<L, float>(a, z, b, most_bias, l, chosen);
    if (__ballot(doubt)) {
      // all rows of the wave once more (the shuffles need all lanes): the same where they were right
      choose<L, double>(a, z, b, most_bias, l, chosen);
    }
    lds_wave_sync();
    // the weights, a chosen expert a lane
    float top = 0.0f, total = 1.0f;
    if (a.softmax) {
      top = z[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) top = fmaxf(top, z[i]);
      top = row_max<L>(top);
      if (top == -__builtin_inff()) top = 0.0f;
      total = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) total += exp_neg(top - z[i]);
      total = row_sum<L>(total);
    }
    const raw* row = static_cast<const raw*>(a.z) + t * E;
    auto score = [&](int e) {
      const float x = clean(Logit<kDtype>::to_f(row[e]));
      return a.softmax ? exp_neg(top - x) / total : sigmoid_of(x);
    };
    float sum = 0.0f;
    if (a.normalize) {
      for (int k = l; k < a.K; k += L) sum += chosen[k] >= 0 ? score(chosen[k]) : 0.0f;
      sum = row_sum<L>(sum);
    }
    const bool low = a.normalize && sum < kLowSum;
    float most = -__builtin_inff();
    auto raised = [&](int e) { return raised_score(clean(Logit<kDtype>::to_f(row[e])), most, a.softmax); };
    if (__ballot(low && chosen[0] >= 0)) {
      float again = 0.0f;
      for (int k = l; k < a.K; k += L) most = fmaxf(most, chosen[k] >= 0 ? clean(Logit<kDtype>::to_f(row[chosen[k]])) : most);
      most = row_max<L>(most);
      for (int k = l; k < a.K; k += L) again += chosen[k] >= 0 ? raised(chosen[k]) : 0.0f;
      again = row_sum<L>(again);
      sum = low ? again : sum;
    }
    if (live) {
      for (int k = l; k < a.K; k += L) {
        const int e = chosen[k];
        float w = e < 0 ? 0.0f : low ? raised(e) : score(e);
        if (a.normalize) w = sum > 0.0f ? w / sum : 0.0f;
        a.idx[t * a.K + k] = e;
        a.weight[t * a.K + k] = a.scale * w;
      }
    }
    lds_wave_sync();
  }
}

// What the routing kernels share behind the choice: the weights of a row's experts `chosen`, a
// lane's k at a time.  z: this lane's logits of the row, L lanes together all of them.
template <int L, int kDtype, int V>
__device__ __forceinline__ void softmax_of(const float (&z)[V], float& top, float& total) {
  top = z[0];
#pragma unroll
  for (int i = 1; i < V; ++i) top = fmaxf(top, z[i]);
  top = row_max<L>(top);
  if (top == -__builtin_inff()) top = 0.0f;
  total = 0.0f;
#pragma unroll
  for (int i = 0; i < V; ++i) total += exp_neg(top - z[i]);
  total = row_sum<L>(total);
}

// ---------------------------------------------------- up to sixteen experts --
// Keys are binary64: a binary32 score with its expert's place in the low bits, so that one maximum
// and one minimum order two of them, ties to the lower expert.  A row lies in L lanes of V experts
// each; a lane sorts its keys in lists of N (8, or 16 for K above 8), merges those to its best N, and
// the lanes' lists are merged in pairs.  It is bound by the issue of instructions and of the waves that
// wait for their rows: 147,456 tokens of 256 experts, 8 groups, K = 6, bf16 logits, at four waves on a
// SIMD: 55 us (1.4 TB/s; the bytes alone take 15), K = 8 60, without groups 47, without a bias as well 35,
// a softmax 77; K = 12 77 and K = 16 82 at three waves, 80 and 84 at four, 89 and 94 at two.  Where a wider
// bound of doubt sent more rows to binary64: K = 6 at four waves 68, five 70, six 79, two waves with all
// 32 keys of a lane in registers 151.  All of that is with biases of which no two are equal: two experts of equal
// logits and biases are in doubt as well, and with a bias of zeros, or of steps of 0.001, K = 6 takes 212 and 74 us,
// K = 8 288 and 87, without groups 224 and 74; the bound grows with the largest bias, and one of -1e9 sends every row
// to binary64 (485 us).  With K rounds of a maximum over 32 lanes, as above, K = 6 215, K = 12 280.
__device__ __forceinline__ double key_max(double a, double b) {
  double r;
  asm("v_max_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
__device__ __forceinline__ double key_min(double a, double b) {
  double r;
  asm("v_min_f64 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
  return r;
}
// Below every score, whatever the low bits.
constexpr uint32_t kMaskedHigh = 0xFFE00000u;
constexpr double kMasked = -0x1p1023;
__device__ __forceinline__ double key_with(double q, uint32_t low) {
  const uint64_t u = __builtin_bit_cast(uint64_t, key_max(q, kMasked));    // an infinity with low bits would be no number
  return __builtin_bit_cast(double, (u & 0xFFFFFFFF00000000ull) | ((uint32_t)u + low));
}
// Of a logit: ties go to the lower expert.
__device__ __forceinline__ double key_of_logit(float z, int e) {
  z += 0.0f;                            // -0 is 0
  return key_with(z, z < 0.0f ? (uint32_t)e : 255u - e);      // a larger significand is less there
}
// Of a score, e = first + i: the order of equal scores does not matter, they are too near to call.
__device__ __forceinline__ double key_of_score(float q, uint32_t last, int i) { return key_with(q, last + (uint32_t)(31 - i)); }
__device__ __forceinline__ bool key_masked(double k) { return k < -1e300; }
__device__ __forceinline__ int key_expert(double k, bool of_logit) {
  const int low = (int)(__builtin_bit_cast(uint64_t, k) & 255u);
  return of_logit && k < 0.0 ? low : 255 - low;
}
__device__ __forceinline__ void order(double& a, double& b) {
  const double hi = key_max(a, b);
  b = key_min(a, b);
  a = hi;
}
__device__ __forceinline__ void sort8(double* k) {
  constexpr int pairs[19][2] = {{0, 1}, {2, 3}, {4, 5}, {6, 7}, {0, 2}, {1, 3}, {4, 6}, {5, 7}, {1, 2}, {5, 6},
                                {0, 4}, {1, 5}, {2, 6}, {3, 7}, {2, 4}, {3, 5}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
  for (int i = 0; i < 19; ++i) order(k[pairs[i][0]], k[pairs[i][1]]);
}
// What is sorted but for a turn in its middle, sorted.
template <int N>
__device__ __forceinline__ void straighten(double* k) {
#pragma unroll
  for (int d = N / 2; d > 0; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((i & d) == 0) order(k[i], k[i + d]);
}
// Sixteen keys; eight (half), the others masked.
__device__ __forceinline__ void sort16(double* k, bool half) {
  sort8(k);
  if (half) return;
  sort8(k + 8);
#pragma unroll
  for (int i = 0; i < 8; ++i) order(k[i], k[15 - i]);
  straighten<8>(k);
  straighten<8>(k + 8);
}
// The best N of two sorted N, sorted, in a; lost: the largest of those that are not among
// them (more: N are to be chosen, and how near the next one is matters).
template <int N>
__device__ __forceinline__ void merge(double* a, const double* b, double& lost, bool more) {
  if (more) {
#pragma unroll
    for (int i = 0; i < N; ++i) lost = key_max(lost, key_min(a[i], b[N - 1 - i]));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) a[i] = key_max(a[i], b[N - 1 - i]);
  straighten<N>(a);
}
template <int kCtrl, class T>
__device__ __forceinline__ T moved(T x) {
  if constexpr (sizeof(T) == 8) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, kCtrl, 0xF, 0xF, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), kCtrl, 0xF, 0xF, false);
    return __builtin_bit_cast(T, (uint64_t)hi << 32 | lo);
  } else {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), kCtrl, 0xF, 0xF, false));
  }
}
// From the lane whose number within the row's eight differs by x
template <int x, class T>
__device__ __forceinline__ T from_lane(T v) {
  static_assert(x >= 1 && x <= 7, "eight lanes");
  if constexpr (x == 1) return moved<0xB1>(v);
  else if constexpr (x == 2) return moved<0x4E>(v);
  else if constexpr (x == 3) return moved<0x1B>(v);
  else if constexpr (x == 7) return moved<0x141>(v);
  else return from_lane<7 - x>(moved<0x141>(v));
}

// The sums of a group's two best in this lane and, over the lanes that share the group, theirs;
// whether the lane's group is among the best, and whether that was too near to call.
template <int L>
__device__ __forceinline__ bool group_kept(const ScoredArgs& a, float t1, float t2, int V, int l, float most_bias, bool& doubt) {
  const int share = a.E / a.groups / V;         // lanes of a group
  auto join = [&](float o1, float o2) { merge2(t1, t2, o1, o2); };
  if constexpr (L >= 2) {
    if (share >= 2) join(from_lane<1>(t1), from_lane<1>(t2));
  }
  if constexpr (L >= 4) {
    if (share >= 4) join(from_lane<2>(t1), from_lane<2>(t2));
  }
  const float none = -__builtin_inff();
  const float g = a.group_top == 2 && t2 > none ? sum_of_two(t1, t2) : t1;
  const int mine = l / share;
  int better = 0;
  auto look = [&](auto x) {
    constexpr int d = decltype(x)::value;
    if constexpr (d < L) {
      const float o = from_lane<d>(g);
      better += o > g || (o == g && (l ^ d) / share < mine) ? 1 : 0;
    }
  };
  look(std::integral_constant<int, 1>{});
  look(std::integral_constant<int, 2>{});
  look(std::integral_constant<int, 3>{});
  look(std::integral_constant<int, 4>{});
  look(std::integral_constant<int, 5>{});
  look(std::integral_constant<int, 6>{});
  look(std::integral_constant<int, 7>{});
  const bool kept = better < a.top_groups * share;
  const float least = -row_max<L>(kept ? -g : none), most = row_max<L>(kept ? none : g);
  doubt = doubt || (most > none && near(least, most, 2.0f * most_bias, a.softmax));
  return kept;
}

template <int E, int kDtype, bool kSoftmax, int N>
__global__ __launch_bounds__(kScoredThreads, N == 8 ? 4 : 3) void route_scored_best_kernel(const ScoredArgs a) {
  constexpr int V = E / 8 > kPer ? E / 8 : kPer, L = E / V, kRows = 64 / L, kPieces = V / 8;
  constexpr int kLists = V > N ? V / N : 1, kListPieces = kPieces / kLists;       // a lane's lists of N
  constexpr int kSlow = E / kPer;               // lanes of a row that is looked at once more
  typedef typename Logit<kDtype>::raw raw;
  typedef raw vec __attribute__((ext_vector_type(kPer), aligned(16)));       // what a caller promises
  __shared__ __attribute__((aligned(16))) float sh_bias[E];
  __shared__ int16_t sh_chosen[kScoredWaves][N];
  const int lane = threadIdx.x & 63, l = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float none = -__builtin_inff();
  float most_bias = 0.0f;
  if (a.bias) {
    for (int e = threadIdx.x; e < E; e += kScoredThreads) {
      const float v = a.bias[e];
      sh_bias[e] = v == v ? fminf(v, kLargest) : none;
    }
    __syncthreads();
    for (int i = 0; i < V; ++i) {
      const float m = fabsf(sh_bias[l * V + i]);
      most_bias = fmaxf(most_bias, m < kLargest ? m : 0.0f);
    }
    most_bias = row_max<L>(most_bias);
  }
  const bool by_groups = a.top_groups < a.groups, by_logits = a.bias == nullptr, more = a.K == N;
  const int64_t step = (int64_t)gridDim.x * kScoredWaves * kRows;
  for (int64_t t0 = ((int64_t)blockIdx.x * kScoredWaves + wave) * kRows; t0 < a.T; t0 += step) {
    const bool live = t0 + lane / L < a.T;
    const int64_t t = live ? t0 + lane / L : a.T - 1;
    const raw* row = static_cast<const raw*>(a.z) + t * E;
    auto piece = [&](int i, float (&z)[kPer]) {
      const vec x = *reinterpret_cast<const vec*>(row + l * V + i * kPer);
#pragma unroll
      for (int j = 0; j < kPer; ++j) z[j] = clean(Logit<kDtype>::to_f(x[j]));
    };
    float top = 0.0f, total = 1.0f;
    if (kSoftmax) {
      top = none;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        float z[kPer];
        piece(i, z);
#pragma unroll
        for (int j = 0; j < kPer; ++j) top = fmaxf(top, z[j]);
      }
      top = row_max<L>(top);
      if (top == none) top = 0.0f;
      if (!a.normalize || !by_logits || by_groups) {        // else the sum is not needed
        total = 0.0f;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          float z[kPer];
          piece(i, z);
#pragma unroll
          for (int j = 0; j < kPer; ++j) total += exp_neg(top - z[j]);
          __builtin_amdgcn_sched_barrier(0);
        }
        total = row_sum<L>(total);
      }
    }
    // scores for the choice only, as near() says
    const float rcp_total = __builtin_amdgcn_rcpf(total);
    auto quick = [&](float x) {
      const float kLog2e = 1.44269502162933349609375f;
      if constexpr (kSoftmax) return __builtin_amdgcn_exp2f((x - top) * kLog2e) * rcp_total;
      else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -kLog2e));
    };
    bool doubt = false;
    const double masked = __builtin_bit_cast(double, (uint64_t)kMaskedHigh << 32);
    double key[N], lost = masked;
    // N at a time, so that few registers are in use and many waves run
    auto lists = [&](auto logits) {
#pragma unroll
      for (int n = 0; n < kLists; ++n) {
        double other[N], (&list)[N] = n == 0 ? key : other;
#pragma unroll
        for (int h = 0; h < kListPieces; ++h) {
          const int i = n * kListPieces + h;
          const vec x = *reinterpret_cast<const vec*>(row + l * V + i * kPer);
          double* const to = list + h * kPer;
          if constexpr (decltype(logits)::value) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) to[j] = key_of_logit(clean(Logit<kDtype>::to_f(x[j])), l * V + i * kPer + j);
          } else {
#pragma unroll
            for (int j = 0; j < kPer; j += 4) {
              const float4 b = *reinterpret_cast<const float4*>(&sh_bias[l * V + i * kPer + j]);
              const float bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
              for (int m = 0; m < 4; ++m) {
                // +inf gives a sigmoid of 1 as it is
                const float z = kSoftmax ? clean(Logit<kDtype>::to_f(x[j + m])) : Logit<kDtype>::to_f(x[j + m]);
                const float q = quick(z) + bs[m];
                to[j + m] = key_of_score(z > none ? q : none, 224u - (uint32_t)(l * V), i * kPer + j + m);
              }
            }
          }
        }
        if constexpr (N == 8) sort8(list);
        else {
#pragma unroll
          for (int i = kListPieces * kPer; i < N; ++i) list[i] = masked;
          sort16(list, kListPieces == 1);
        }
        if (n > 0) merge<N>(key, other, lost, more);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    if (by_logits) lists(std::integral_constant<bool, true>{});
    else lists(std::integral_constant<bool, false>{});
    bool kept = true;
    if (by_groups) {
      auto score = [&](double k) { return key_masked(k) ? none : by_logits ? quick((float)k) : (float)k; };
      kept = group_kept<L>(a, score(key[0]), score(key[1]), V, l, most_bias, doubt);
    }
    auto drop = [&](double k) {
      const uint64_t u = __builtin_bit_cast(uint64_t, k);
      return __builtin_bit_cast(double, (uint64_t)(kept ? (uint32_t)(u >> 32) : kMaskedHigh) << 32 | (uint32_t)u);
    };
    if (by_groups) {
#pragma unroll
      for (int i = 0; i < N; ++i) key[i] = drop(key[i]);
      lost = drop(lost);
    }
    auto meet = [&](auto x) {
      constexpr int d = decltype(x)::value;
      double other[N];
#pragma unroll
      for (int i = 0; i < N; ++i) other[i] = from_lane<d>(key[i]);
      if (more) lost = key_max(lost, from_lane<d>(lost));
      merge<N>(key, other, lost, more);
    };
    if constexpr (L >= 2) meet(std::integral_constant<int, 1>{});
    if constexpr (L >= 4) meet(std::integral_constant<int, 2>{});
    if constexpr (L >= 8) meet(std::integral_constant<int, 7>{});    // the four lanes of a half have the same
    // the k-th best to lane k (and k + L, ...)
    constexpr int kEach = N / L > 1 ? N / L : 1;
    int e[kEach];
    float s[kEach], sum = 0.0f;
#pragma unroll
    for (int h = 0; h < kEach; ++h) {
      const int k = l + h * L;
      double mine = key[0], next = key[1];
#pragma unroll
      for (int i = 1; i < N; ++i) {
        mine = k == i ? key[i] : mine;
        next = k == i ? (i + 1 < N ? key[i + 1 < N ? i + 1 : 0] : lost) : next;
      }
      const bool on = k < a.K && !key_masked(mine);
      e[h] = on ? key_expert(mine, by_logits) : -1;
      if (!by_logits) doubt = doubt || (on && !key_masked(next) && near((float)mine, (float)next, most_bias, kSoftmax));
      s[h] = 0.0f;
      if (on) {
        const float x = clean(Logit<kDtype>::to_f(row[e[h]]));
        s[h] = kSoftmax ? exp_neg(top - x) : sigmoid_of(x);
      }
      sum += s[h];
    }
    float by = a.normalize ? row_sum<L>(sum) : total;
    const bool low = a.normalize && by < kLowSum;
    if (__ballot(low && e[0] >= 0)) {
      float x[kEach], most = none;
#pragma unroll
      for (int h = 0; h < kEach; ++h) {
        x[h] = e[h] >= 0 ? clean(Logit<kDtype>::to_f(row[e[h]])) : none;
        most = fmaxf(most, x[h]);
      }
      most = row_max<L>(most);
      sum = 0.0f;
#pragma unroll
      for (int h = 0; h < kEach; ++h) {
        const float again = e[h] >= 0 ? raised_score(x[h], most, kSoftmax) : 0.0f;
        s[h] = low ? again : s[h];
        sum += s[h];
      }
      sum = row_sum<L>(sum);
      by = low ? sum : by;
    }
    const uint64_t doubts = __ballot(doubt && live);
    const bool again = (doubts >> (lane / L * L) & (L == 64 ? ~0ull : (1ull << (L & 63)) - 1)) != 0;
    if (live && !again) {
#pragma unroll
      for (int h = 0; h < kEach; ++h) {
        const int k = l + h * L;
        if (k < a.K) {
          a.idx[t * a.K + k] = e[h];
          a.weight[t * a.K + k] = by > 0.0f ? a.scale * (s[h] / by) : 0.0f;
        }
      }
    }
    // rows with scores too near to call, one at a time in binary64, by all lanes
    for (uint64_t left = __ballot(again && l == 0); left != 0; left &= left - 1) {
      const int64_t tr = t0 + __builtin_ctzll(left) / L;
      const int ls = lane % kSlow;
      float zs[kPer], bs[kPer];
      load_row<E, kDtype>(a.z, tr, ls, zs);
#pragma unroll
      for (int i = 0; i < kPer; ++i) bs[i] = a.bias ? a.bias[ls * kPer + i] : 0.0f;
      choose<kSlow, double>(a, zs, bs, most_bias, ls, sh_chosen[wave]);
      lds_wave_sync();
      float top_s = 0.0f, total_s = 1.0f;
      if (kSoftmax) softmax_of<kSlow, kDtype>(zs, top_s, total_s);
      const raw* at = static_cast<const raw*>(a.z) + tr * E;
      const int es = lane < a.K ? sh_chosen[wave][lane & (N - 1)] : -1;
      float ss = 0.0f, x = none;
      if (es >= 0) {
        x = clean(Logit<kDtype>::to_f(at[es]));
        ss = kSoftmax ? exp_neg(top_s - x) : sigmoid_of(x);
      }
      float by_s = a.normalize ? row_sum<N>(ss) : total_s;      // lanes 0 .. N - 1 hold them
      if (__ballot(a.normalize && es >= 0 && by_s < kLowSum)) {
        const float most = row_max<N>(x);
        ss = es >= 0 ? raised_score(x, most, kSoftmax) : 0.0f;
        by_s = row_sum<N>(ss);
      }
      if (lane < a.K) {
        a.idx[tr * a.K + lane] = es;
        a.weight[tr * a.K + lane] = by_s > 0.0f ? a.scale * (ss / by_s) : 0.0f;
      }
      lds_wave_sync();
    }
  }
}

// The gradient of a row by the lanes that hold it, in LDS, since a row may name an expert twice.  Of the
// logits only the chosen ones are read (all of them for a softmax of weights that are not normalized).  Bound by memory, 4 E bytes of stores a
// row, which pass the caches by: 147,456 rows of 256 experts, K = 6, bf16 logits, 35 us; through the caches
// 43, and with the forward before it on inputs that change 109 where both take 87.  A softmax 39, not
// normalized 48.
typedef float floats4 __attribute__((ext_vector_type(4)));
template <int E, int kDtype>
__global__ __launch_bounds__(kScoredThreads) void route_scored_backward_kernel(const ScoredArgs a) {
  constexpr int L = E / kPer, kRows = 64 / L;
  __shared__ __attribute__((aligned(16))) float sh_grad[kScoredWaves * kRows][E];
  typedef typename Logit<kDtype>::raw raw;
  const int lane = threadIdx.x & 63, l = lane % L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* const grad = sh_grad[wave * kRows + lane / L];
  const int64_t step = (int64_t)gridDim.x * kScoredWaves * kRows;
  for (int64_t t0 = ((int64_t)blockIdx.x * kScoredWaves + wave) * kRows; t0 < a.T; t0 += step) {
    const bool live = t0 + lane / L < a.T;
    const int64_t t = live ? t0 + lane / L : a.T - 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) grad[l * kPer + i] = 0.0f;
    float z[kPer], top = 0.0f, total = 1.0f;
    if (a.softmax && !a.normalize) {
      load_row<E, kDtype>(a.z, t, l, z);
      top = z[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) top = fmaxf(top, z[i]);
      top = row_max<L>(top);
      if (top == -__builtin_inff()) top = 0.0f;
      total = 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        z[i] = exp_neg(top - z[i]);
        total += z[i];
      }
      total = row_sum<L>(total);
    }
    const raw* row = static_cast<const raw*>(a.z) + t * E;
    const int32_t* idx = a.idx + t * a.K;
    const float* gw = a.grad_weight + t * a.K;
    if (a.softmax && a.normalize) {      // the chosen scores' ratios are enough
      top = -__builtin_inff();
      for (int k = l; k < a.K; k += L) {
        const int e = idx[k];
        if (e >= 0 && e < E) top = fmaxf(top, clean(Logit<kDtype>::to_f(row[e])));
      }
      top = row_max<L>(top);
      if (top == -__builtin_inff()) top = 0.0f;
    }
    float most = 0.0f;
    bool low = false;                     // a sigmoid's scores are over e^most
    auto score = [&](int e, float& s, float& rest) {
      const float x = clean(Logit<kDtype>::to_f(row[e]));
      if (low) {
        sigmoid_pair(x, s, rest);
        s = exp_neg(most - x) * rest;
      } else if (a.softmax) {
        s = total > 0.0f ? exp_neg(top - x) / total : 0.0f;
        rest = 1.0f;
      } else {
        sigmoid_pair(x, s, rest);
      }
    };
    // S = sum of the chosen scores and the sum of g s
    float S, gs;
    auto sums = [&]() {
      S = gs = 0.0f;
      for (int k = l; k < a.K; k += L) {
        const int e = idx[k];
        if (e < 0 || e >= E) continue;
        float s, rest;
        score(e, s, rest);
        S += s;
        gs += gw[k] * s;
      }
      S = row_sum<L>(S);
      gs = row_sum<L>(gs);
    };
    sums();
    if (a.normalize && !a.softmax && __ballot(S < kLowSum)) {
      most = -__builtin_inff();
      for (int k = l; k < a.K; k += L) {
        const int e = idx[k];
        if (e >= 0 && e < E) most = fmaxf(most, clean(Logit<kDtype>::to_f(row[e])));
      }
      most = row_max<L>(most);
      low = S < kLowSum && most > -__builtin_inff();
      sums();
    }
    const float inv = a.normalize ? (S > 0.0f ? 1.0f / S : 0.0f) : 1.0f, mean = a.normalize ? gs * inv : 0.0f;
    lds_wave_sync();
    // entry by entry, so that an expert that a row names twice gets both in their order
    for (int k0 = 0; k0 < a.K; k0 += L) {
      const int k = k0 + l;
      int e = -1;
      float v = 0.0f;
      if (k < a.K) {
        e = idx[k];
        if (e >= 0 && e < E) {
          float s, rest;
          score(e, s, rest);
          v = a.scale * ((gw[k] - mean) * inv) * s * rest;
        }
      }
      for (int j = 0; j < L && k0 + j < a.K; ++j) {
        if (l == j && e >= 0 && e < E) grad[e] += v;
        lds_wave_sync();
      }
    }
    // every expert lowers the others
    if (a.softmax && !a.normalize) {
      const float back = total > 0.0f ? a.scale * gs / total : 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) grad[l * kPer + i] -= back * z[i];
      lds_wave_sync();
    }
    if (live) {
      floats4* const to = reinterpret_cast<floats4*>(a.grad_z + t * E);
#pragma unroll
      for (int i = 0; i < kPer / 4; ++i) __builtin_nontemporal_store(reinterpret_cast<const floats4*>(grad)[i * L + l], to + i * L + l);
    }
    lds_wave_sync();
  }
}

template <int E, int kDtype, int N>
void launch_best(const ScoredArgs& a, hipStream_t s) {
  constexpr int V = E / 8 > kPer ? E / 8 : kPer, kRows = 64 / (E / V) * kScoredWaves;
  int64_t blocks = (a.T + kRows - 1) / kRows, most = (int64_t)num_cus() * 8;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < most) most = cap;
  if (blocks > most) blocks = most;
  if (a.softmax) route_scored_best_kernel<E, kDtype, true, N><<<(uint32_t)blocks, kScoredThreads, 0, s>>>(a);
  else route_scored_best_kernel<E, kDtype, false, N><<<(uint32_t)blocks, kScoredThreads, 0, s>>>(a);
}

template <int E, int kDtype>
eqb_status launch_scored_e(const ScoredArgs& a, bool backward, hipStream_t s) {
  constexpr int kRows = 64 / (E / kPer) * kScoredWaves;
  int64_t blocks = (a.T + kRows - 1) / kRows, most = (int64_t)num_cus() * 8;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < most) most = cap;
  if (blocks > most) blocks = most;
  // sorted lists: up to 16 experts, of groups that fill lanes
  constexpr int V = E / 8 > kPer ? E / 8 : kPer;
  const bool lanes = a.top_groups == a.groups || a.E / a.groups >= V;
  constexpr int kMost = E > 8 ? 16 : 8;
  if (backward) route_scored_backward_kernel<E, kDtype><<<(uint32_t)blocks, kScoredThreads, 0, s>>>(a);
  else if (lanes && a.K <= 8) launch_best<E, kDtype, 8>(a, s);
  else if (lanes && a.K <= kMost) launch_best<E, kDtype, kMost>(a, s);
  else route_scored_kernel<E, kDtype><<<(uint32_t)blocks, kScoredThreads, 0, s>>>(a);
  return launch_status();
}

template <int kDtype>
eqb_status launch_scored_d(const ScoredArgs& a, bool backward, hipStream_t s) {
  switch (a.E) {
    case 8: return launch_scored_e<8, kDtype>(a, backward, s);
    case 16: return launch_scored_e<16, kDtype>(a, backward, s);
    case 32: return launch_scored_e<32, kDtype>(a, backward, s);
    case 64: return launch_scored_e<64, kDtype>(a, backward, s);
    case 128: return launch_scored_e<128, kDtype>(a, backward, s);
    case 256: return launch_scored_e<256, kDtype>(a, backward, s);
    default: return EQB_ERR_UNSUPPORTED;
  }
}

eqb_status launch_scored(const ScoredArgs& a, bool backward, hipStream_t s) {
  if (a.dtype == EQB_DTYPE_BF16) return launch_scored_d<EQB_DTYPE_BF16>(a, backward, s);
  if (a.dtype == EQB_DTYPE_F16) return launch_scored_d<EQB_DTYPE_F16>(a, backward, s);
  return launch_scored_d<EQB_DTYPE_F32>(a, backward, s);
}

}  // namespace

eqb_status launch_route_scored(const ScoredArgs& a, hipStream_t s) { return launch_scored(a, false, s); }
eqb_status launch_route_scored_backward(const ScoredArgs& a, hipStream_t s) { return launch_scored(a, true, s); }

}  // namespace eqb
