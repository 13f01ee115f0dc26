// adamw.hip - one AdamW step over a list of tensors, with binary32 or 8-bit states.
#include "eqb_internal.hpp"

namespace eqb {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
// the same at the alignment of one element: tensors may start anywhere in a flat buffer
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));

constexpr int kAdamwThreads = 256, kAdamwWaves = kAdamwThreads / 64;

// Tensors of one launch, passed by value (kernel arguments hold 4 KiB): as many as fit.
struct AdamwScales {
  float* exp_avg;
  float* exp_avg_sq;
  uint32_t key;           // of the random bits; with a counter the tensor's place
};
struct AdamwCopy {
  uint16_t* copy;
};
template <int> struct AdamwNone {};
template <bool k8, bool kCopy>
struct AdamwSlot : std::conditional_t<k8, AdamwScales, AdamwNone<0>>, std::conditional_t<kCopy, AdamwCopy, AdamwNone<1>> {
  float* param;
  const void* grad;
  void* m;
  void* v;
  int64_t numel;
  float keep;             // 1 - lr * weight_decay
  uint32_t first_block;
};
template <bool k8, bool kCopy>
struct AdamwBatch {
  static constexpr int kMost = (4096 - 64) / sizeof(AdamwSlot<k8, kCopy>);
  int n;                  // tensors
  AdamwScalars c;
  AdamwSlot<k8, kCopy> t[kMost];
};
static_assert(sizeof(AdamwBatch<true, true>) <= 4096 && sizeof(AdamwBatch<false, false>) <= 4096, "kernel arguments");

// The E4M3 code of y (0 <= y <= 448), rounded up where the random 16 bits exceed what y
// lacks to the next code; the code with its bit 6 flipped is in bits 20 to 26.  From 2^-6
// on a code is the binary32 pattern without its last 20 bits, less 960; y + 2^-6 has the
// subnormal codes' spacing, and its pattern counts 8 more.  Below 2^-6 the second is the
// greater (or they agree), from there on the first.  rnd20: the random bits times 16.
__device__ __forceinline__ uint32_t encode_e4m3(float y, uint32_t rnd20) {
  const uint32_t a = __float_as_uint(y) + rnd20, b = __float_as_uint(y + 0x1p-6f) + rnd20 - (8u << 20);
  return a > b ? a : b;
}

// Bits 20 to 26 of four words as the low 7 bits of a word's bytes, bit 6 flipped; byte i
// gets the sign of s[i] as its bit 7.
template <bool kSigned>
__device__ __forceinline__ uint32_t pack_e4m3x4(const uint32_t (&w)[4], f32x4 s) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    b[i] = kSigned ? (w[i] << 4 & 0x7FFFFFFFu) | (__float_as_uint(s[i]) & 0x80000000u) : w[i] << 4;
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0703u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x07030C0Cu);
  return ((kSigned ? lo | hi : (lo | hi) & 0x7F7F7F7Fu)) ^ 0x40404040u;
}

__device__ __forceinline__ f32x4 decode_e4m3x4(uint32_t w) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// 32 bits mixed by shifts and odd multipliers, those that C. Wellons published in 2018 as the
// least biased of a search (every input bit turns every output bit half of the time).
__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

// The key of a tensor's random bits at a step: seed, step and place mixed to 32 bits.  Steps
// and places count in multiples that spread evenly over 2^64 (2^64 by the golden ratio, and by
// the root of x^4 = x + 1, its like for three dimensions), the mixer's multipliers are D.
// Stafford's (published with Steele, Lea and Flood's splittable generators, 2014).
__host__ __device__ inline uint64_t adamw_base(uint64_t seed, int64_t step) {
  return seed + (uint64_t)step * 0x9E3779B97F4A7C15ull;
}
__host__ __device__ inline uint32_t adamw_key(uint64_t base, uint32_t i) {
  uint64_t k = base + (uint64_t)i * 0xD1B54A32D192ED03ull;
  k = (k ^ (k >> 32)) * 0xBF58476D1CE4E5B9ull;
  k = (k ^ (k >> 29)) * 0x94D049BB133111EBull;
  return (uint32_t)(k ^ (k >> 32));
}

// Blocks of one launch: times 256 threads they stay below 2^32.
constexpr int64_t kAdamwMostBlocks = 1 << 23;

// Maximum of values from 0 on over the wave (their patterns order like them).
__device__ __forceinline__ float wave_max(float x) {
  return __uint_as_float(group_fold<64>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
}

// One more step, unless found_inf skips it, and what it takes from its number.  The blocks of
// the step itself run behind this and only read it.
__global__ void adamw_count_kernel(AdamwCounter* c, const float* __restrict__ found_inf, double lr, double beta1,
                                   double beta2, uint64_t seed) {
  if (threadIdx.x != 0 || (found_inf && *found_inf != 0.0f)) return;
  const int64_t step = c->steps + 1;
  c->steps = step;
  c->base = adamw_base(seed, step);
  c->inv_root = (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step)));
  c->rate = (float)(lr / (1.0 - pow(beta1, (double)step)));
}

template <bool kStream, class T>
__device__ __forceinline__ std::remove_const_t<T> get(T* p) {
  return kStream ? __builtin_nontemporal_load(p) : *p;
}
template <bool kStream, class T, class V>
__device__ __forceinline__ void put(T* p, V v) {
  if (kStream) __builtin_nontemporal_store((T)v, p);
  else *p = (T)v;
}

// A block of 256 elements is a wave's: 4 elements a lane, at the alignment of one.
template <bool k8, bool kGradBf16, bool kCopy, bool kStream>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(const AdamwBatch<k8, kCopy> batch) {
  typedef std::conditional_t<kGradBf16, uint16_t, float> grad_e;
  typedef std::conditional_t<kGradBf16, u16x4, f32x4> grad_t;
  typedef std::conditional_t<kGradBf16, u16x4_any, f32x4_any> grad_any;
  typedef std::conditional_t<k8, uint8_t, float> state_e;
  typedef std::conditional_t<k8, uint32_t, f32x4> state_t;
  typedef std::conditional_t<k8, u32_any, f32x4_any> state_any;
  const AdamwScalars& c = batch.c;
  if (c.found_inf && *c.found_inf != 0.0f) return;
  // the tensor of this block: the last whose first block is not past it
  int lo = 0, hi = batch.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (batch.t[mid].first_block <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwSlot<k8, kCopy>& t = batch.t[lo];
  const float scale = c.grad_scale ? *c.grad_scale : 1.0f;
  const float inv_root = c.counter ? c.counter->inv_root : c.inv_root, rate = c.counter ? c.counter->rate : c.rate;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // at most 2^33 elements: block numbers have 25 bits
  const int qb = (int)(blockIdx.x - t.first_block) * kAdamwWaves + wave;
  const int whole = (int)(t.numel / EQB_ADAMW_BLOCK), rest = (int)(t.numel % EQB_ADAMW_BLOCK);
  const int blocks = whole + (rest > 0);

  if (qb >= blocks) return;
  const bool all = qb < whole;          // 256 elements, or the rest of the tensor
  const int left = all ? 4 : rest - 4 * lane;
  const int64_t base = (int64_t)qb * EQB_ADAMW_BLOCK;
  float* pw = t.param + base;
  const grad_e* pg = static_cast<const grad_e*>(t.grad) + base;
  state_e* pm = static_cast<state_e*>(t.m) + base;
  state_e* pv = static_cast<state_e*>(t.v) + base;

  f32x4 w = {0, 0, 0, 0}, g = w, m = w, v = w, r;
  state_t cm = {}, cv = {};
  float sm = 1.0f, sv = 1.0f;
  if constexpr (k8) {
    sm = static_cast<const AdamwScales&>(t).exp_avg[qb];
    sv = static_cast<const AdamwScales&>(t).exp_avg_sq[qb];
  }
  grad_t gr = {};
  if (all) {
    w = get<kStream>(&at<const f32x4_any>(pw, 16u * lane));
    gr = get<kStream>(&at<const grad_any>(pg, 4u * sizeof(grad_e) * lane));
    cm = get<kStream>(&at<const state_any>(pm, 4u * sizeof(state_e) * lane));
    cv = get<kStream>(&at<const state_any>(pv, 4u * sizeof(state_e) * lane));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i < left) {
        w[i] = pw[4 * lane + i];
        gr[i] = pg[4 * lane + i];
        if constexpr (k8) {
          cm |= (uint32_t)pm[4 * lane + i] << (8 * i);
          cv |= (uint32_t)pv[4 * lane + i] << (8 * i);
        } else {
          cm[i] = pm[4 * lane + i];
          cv[i] = pv[4 * lane + i];
        }
      }
    }
  }
  if constexpr (k8) {
    m = decode_e4m3x4(cm);
    v = decode_e4m3x4(cv);
  } else {
    m = cm;
    v = cv;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kGradBf16) g[i] = __uint_as_float((uint32_t)gr[i] << 16);
    else g[i] = gr[i];
    if constexpr (k8) {
      m[i] = m[i] * sm;
      const float x = v[i] * sv;
      v[i] = x * x;
    }
    const float gi = g[i] * scale;
    m[i] = m[i] * c.beta1 + gi * c.rest1;
    v[i] = v[i] * c.beta2 + (gi * c.rest2) * gi;
    r[i] = sqrtf(v[i]);
    const float d = r[i] * inv_root + c.eps;
    w[i] = w[i] * t.keep - (m[i] / d) * rate;
  }
  if constexpr (k8) {
    // lanes past the tensor's end hold zeros
    const AdamwScales& q = t;
    const float tm = wave_max(max3_abs(max3_abs(0.0f, m[0], m[1]), m[2], m[3]));
    const float tv = wave_max(max3_abs(max3_abs(0.0f, r[0], r[1]), r[2], r[3]));
    const float nm = tm < 0x1p-100f ? 0.0f : tm * (float)(1.0 / 448.0);
    const float nv = tv < 0x1p-100f ? 0.0f : tv * (float)(1.0 / 448.0);
    const float im = nm > 0.0f ? 1.0f / nm : 0.0f, iv = nv > 0.0f ? 1.0f / nv : 0.0f;
    // a block of 256 elements does not cross a multiple of 2^32
    const uint32_t key = c.counter ? adamw_key(c.counter->base, q.key) : q.key;
    const uint32_t high = (uint32_t)((uint64_t)base >> 32) * 0x9E3779B1u, low = (uint32_t)(uint64_t)base + key;
    uint32_t bm[4], bv[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t h = mix32((low + 4 * lane + i) ^ high);
      bm[i] = encode_e4m3(fminf(fabsf(m[i]) * im, 448.0f), h << 4 & 0xFFFF0u);
      // a second moment above 0 keeps a code above 0: 2^-9 is that of 1
      const float y = __builtin_amdgcn_fmed3f(r[i] * iv, 0x1p-9f, 448.0f);
      bv[i] = encode_e4m3(r[i] > 0.0f ? y : 0.0f, h >> 12 & 0xFFFF0u);
    }
    cm = pack_e4m3x4<true>(bm, m);
    cv = pack_e4m3x4<false>(bv, r);
    if (iv == 0.0f) cv = 0;
    // a value that is no number (or none after the scaling) keeps being none
    if (__any(!(fabsf(w[0]) + fabsf(w[1]) + (fabsf(w[2]) + fabsf(w[3])) < INFINITY)) || !(tv < INFINITY) || !(tm < INFINITY)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ym = m[i] * im, yv = r[i] * iv;
        if (ym != ym) cm |= 0x7Fu << (8 * i);
        if (yv != yv) cv |= 0x7Fu << (8 * i);
      }
    }
    if (lane == 0) {
      q.exp_avg[qb] = nm;
      q.exp_avg_sq[qb] = nv;
    }
  } else {
    cm = m;
    cv = v;
  }
  if (all) {
    put<kStream>(&at<f32x4_any>(pw, 16u * lane), w);
    if constexpr (kCopy) {
      const uint32_t c0 = bf16x2_bits(w[0], w[1]), c1 = bf16x2_bits(w[2], w[3]);
      const u16x4 o = {(uint16_t)c0, (uint16_t)(c0 >> 16), (uint16_t)c1, (uint16_t)(c1 >> 16)};
      put<kStream>(&at<u16x4_any>(t.copy + base, 8u * lane), o);
    }
    put<kStream>(&at<state_any>(pm, 4u * sizeof(state_e) * lane), cm);
    put<kStream>(&at<state_any>(pv, 4u * sizeof(state_e) * lane), cv);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < left) {
      pw[4 * lane + i] = w[i];
      if constexpr (kCopy) t.copy[base + 4 * lane + i] = (uint16_t)bf16x2_bits(w[i], 0.0f);
      if constexpr (k8) {
        pm[4 * lane + i] = (uint8_t)(cm >> (8 * i));
        pv[4 * lane + i] = (uint8_t)(cv >> (8 * i));
      } else {
        pm[4 * lane + i] = cm[i];
        pv[4 * lane + i] = cv[i];
      }
    }
  }
}

// Steps over more bytes than the memory-side cache holds stream them past it: 268 M elements
// with 8-bit states 838 -> 812 us, 100 M with binary32 ones 524 -> 480; 4 M, 120 MB, 19.9 -> 22.9.
constexpr int64_t kAdamwStreamBytes = (int64_t)256 << 20;

template <bool k8, bool kGradBf16, bool kCopy>
static eqb_status launch_adamw_as(const eqb_adamw_tensor* tensors, int n, const AdamwScalars& c, double lr, uint64_t seed,
                                  int64_t step, hipStream_t s) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += tensors[i].numel;
  const bool stream = total * (8 + (kGradBf16 ? 2 : 4) + (kCopy ? 2 : 0) + (k8 ? 4 : 16)) > kAdamwStreamBytes;
  AdamwBatch<k8, kCopy> b;
  b.n = 0;
  b.c = c;
  const int64_t per_block = (int64_t)kAdamwWaves * EQB_ADAMW_BLOCK;
  int64_t blocks = 0;
  auto launch = [&]() {
    if (b.n == 0) return EQB_OK;
    if (stream) adamw_kernel<k8, kGradBf16, kCopy, true><<<(uint32_t)blocks, kAdamwThreads, 0, s>>>(b);
    else adamw_kernel<k8, kGradBf16, kCopy, false><<<(uint32_t)blocks, kAdamwThreads, 0, s>>>(b);
    b.n = 0;
    blocks = 0;
    return launch_status();
  };
  for (int i = 0; i < n; ++i) {
    const eqb_adamw_tensor& t = tensors[i];
    if (t.numel == 0) continue;
    const int64_t more = (t.numel + per_block - 1) / per_block;
    if (b.n == AdamwBatch<k8, kCopy>::kMost || (b.n > 0 && blocks + more > kAdamwMostBlocks)) {
      const eqb_status st = launch();
      if (st != EQB_OK) return st;
    }
    AdamwSlot<k8, kCopy>& o = b.t[b.n++];
    o.param = t.param;
    o.grad = t.grad;
    o.m = t.exp_avg;
    o.v = t.exp_avg_sq;
    o.numel = t.numel;
    o.keep = (float)(1.0 - lr * t.weight_decay);
    o.first_block = (uint32_t)blocks;
    if constexpr (k8) {
      AdamwScales& q = o;
      q.exp_avg = t.exp_avg_scale;
      q.exp_avg_sq = t.exp_avg_sq_scale;
      q.key = c.counter ? (uint32_t)i : adamw_key(adamw_base(seed, step), (uint32_t)i);
    }
    if constexpr (kCopy) o.copy = t.copy;
    blocks += more;
  }
  return launch();
}

eqb_status launch_adamw(const eqb_adamw_tensor* tensors, int n, const AdamwScalars& c, double lr, double beta1,
                        double beta2, uint64_t seed, int64_t step, AdamwCounter* counter, bool eight, bool grad_bf16,
                        bool copies, hipStream_t s) {
  if (counter) {
    adamw_count_kernel<<<1, 64, 0, s>>>(counter, c.found_inf, lr, beta1, beta2, seed);
    const eqb_status st = launch_status();
    if (st != EQB_OK) return st;
  }
  const auto launch = eight ? grad_bf16 ? copies ? launch_adamw_as<true, true, true> : launch_adamw_as<true, true, false>
                                        : copies ? launch_adamw_as<true, false, true> : launch_adamw_as<true, false, false>
                            : grad_bf16 ? copies ? launch_adamw_as<false, true, true> : launch_adamw_as<false, true, false>
                                        : copies ? launch_adamw_as<false, false, true> : launch_adamw_as<false, false, false>;
  return launch(tensors, n, c, lr, seed, step, s);
}

}  // namespace eqb
