// codes.hip - rows, columns and weights as E4M3 codes with a power of two for each block
// of 128, and the gated activation between an expert's two products (what FFN_e of Eq. 1,
// arXiv 2609.28053, works on).
//
// A block's scale is the least power of two under which no finite value exceeds 448, so
// that scaling is exact and a code's rounding is the only one.  All of it is bound by
// memory.
#include "eqb_internal.hpp"

namespace eqb {
namespace {

// Eight neighbouring elements of a row, and what they are in memory.
template <int kDtype>
struct Elem;
template <>
struct Elem<EQB_DTYPE_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ float to_f(raw x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ raw from_f(float x) { return (raw)bf16x2_bits(x, x); }
};
template <>
struct Elem<EQB_DTYPE_F16> {
  typedef _Float16 raw;
  static __device__ __forceinline__ float to_f(raw x) { return (float)x; }
  static __device__ __forceinline__ raw from_f(float x) { return (raw)x; }
};
template <>
struct Elem<EQB_DTYPE_F32> {
  typedef float raw;
  static __device__ __forceinline__ float to_f(raw x) { return x; }
  static __device__ __forceinline__ raw from_f(float x) { return x; }
};

constexpr int kPer = 8;                  // elements of a lane
template <int kDtype>
struct Eight {
  typedef typename Elem<kDtype>::raw raw;
  typedef raw vec __attribute__((ext_vector_type(kPer)));
  // gfx950's global loads and stores take any address
  typedef vec any __attribute__((aligned(alignof(raw))));
};

// Calls that read or write more than the memory-side cache holds pass it by (kStream), where rows are whole
// lines of 128 bytes: the others' lines are shared by neighbouring rows.  884,736 rows of 1,024 bf16 to their
// experts 261 -> 241 us, 64 weights of 2,048 x 2,048 208 -> 191, 98,304 rows of 2,048 by columns 125
// -> 119, gates and their gradients 496 -> 483; but 20,012 rows of 1,001 by columns 20.3 -> 23.8.
constexpr int64_t kStreamBytes = (int64_t)256 << 20;
template <bool kStream, class V>
__device__ __forceinline__ void store_at(V* at, V v) {
  if constexpr (kStream) __builtin_nontemporal_store(v, at);
  else *at = v;
}

// Elements c .. c + 7 of a row of H, zeros behind its end.
template <int kDtype, bool kStream>
__device__ __forceinline__ void load8(const typename Elem<kDtype>::raw* row, int c, int H, float (&v)[kPer]) {
  typedef Elem<kDtype> D;
  if (c + kPer <= H) {
    // not through a template over the type, which would drop its alignment
    const auto* const at = reinterpret_cast<const typename Eight<kDtype>::any*>(row + c);
    const typename Eight<kDtype>::vec x = kStream ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = D::to_f(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) v[i] = c + i < H ? D::to_f(row[c + i]) : 0.0f;
  }
}

template <int kDtype, bool kStream>
__device__ __forceinline__ void store8(typename Elem<kDtype>::raw* row, int c, int H, const float (&v)[kPer]) {
  typedef Elem<kDtype> D;
  typename Eight<kDtype>::vec x;
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = D::from_f(v[i]);
  if (c + kPer <= H) {
    auto* const at = reinterpret_cast<typename Eight<kDtype>::any*>(row + c);
    if constexpr (kStream) __builtin_nontemporal_store(x, at);
    else *at = x;
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (c + i < H) row[c + i] = x[i];
  }
}

// |v| where it is finite, else 0
__device__ __forceinline__ float finite_abs(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;
}
// The scale's byte for a largest magnitude: its exponent less 8, one more where its
// significand exceeds 1.75.
__device__ __forceinline__ int scale_byte(float top) {
  const int b = (int)((__float_as_uint(top) + 0x1FFFFFu) >> 23) - 8;
  return b > 1 ? b : 1;
}
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

// Codes of four values, rounded to nearest even by the conversion itself.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// sigmoid(x) and 1 - sigmoid(x) of any x: exp(-|x|) = 2^(-p) (1 - l ln 2) with p + l = |x| log2 e
// in two parts (the hardware's 2^p is off by one ulp), then a reciprocal with one Newton step.
__device__ __forceinline__ void sigmoid_both(float x, float& s, float& rest) {
  const float kLog2e = 1.44269502162933349609375f, kLow = 1.92596303e-8f, kLn2 = 0.693147182f;
  const float a = fminf(fabsf(x), 200.0f);
  const float p = a * kLog2e;
  const float l = __builtin_fmaf(a, kLow, __builtin_fmaf(a, kLog2e, -p));
  const float e0 = __builtin_amdgcn_exp2f(-p);
  const float e = __builtin_fmaf(-e0 * kLn2, l, e0);
  const float r = newton_rcp(1.0f + e), q = e * r;
  s = x >= 0.0f ? r : q;
  rest = x >= 0.0f ? q : r;
}

// ------------------------------------------------------------- the rows --
constexpr int kCodeThreads = 256, kCodeWaves = kCodeThreads / 64;
constexpr int kWaveCols = 64 * kPer;          // a wave's part of a row: four blocks, one word of scales

template <int kDtype>
struct PlainRow {
  typedef typename Elem<kDtype>::raw raw;
  static constexpr bool kOpen = false;
  template <bool kExact, bool kStream>
  static __device__ __forceinline__ float load(const CodeArgs& a, int64_t t, int c, float (&v)[kPer]) {
    load8<kDtype, kStream>(static_cast<const raw*>(a.x) + t * a.H, c, a.H, v);
    return 0.0f;
  }
};
// A gated value that is to become a code is computed in binary32, within 11 2^-24 for gates above -80 (a
// sigmoid 8, three roundings).  Where that leaves open which of two codes it is, some six in a hundred
// thousand, and for lower gates, it is computed once more to some 50 bits and rounded to the odd neighbour in
// binary32, so that the code's rounding is as if it were the only one.  The exponential is then its series to
// y^12 for |y| <= ln 2 / 2 (off by 2e-16), e^-a of a from 1,200 on 0.  98,304 rows of 2,048: bf16 249 us
// (4.0 TB/s), f16 269.
__device__ __forceinline__ double sigmoid_wide(double x) {
  const double a = fmin(fabs(x), 1200.0), n = __builtin_rint(a * 1.4426950408889634);
  const double y = __builtin_fma(n, 2.3190468138462996e-17, __builtin_fma(n, 0.6931471805599453, -a));      // n ln 2 in two parts
  double e = 1.0 / 479001600;
  constexpr double c[12] = {1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720,
                            1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5, 1.0, 1.0};
#pragma unroll
  for (int i = 0; i < 12; ++i) e = __builtin_fma(e, y, c[i]);
  e = __builtin_amdgcn_ldexp(e, -(int)n);
  const double d = 1.0 + e, r0 = __builtin_amdgcn_rcp(d);      // within 2^-23, squared by each step
  const double r1 = __builtin_fma(__builtin_fma(-d, r0, 1.0), r0, r0), r = __builtin_fma(__builtin_fma(-d, r1, 1.0), r1, r1);
  return x >= 0.0 ? r : e * r;
}
// g sigmoid(g) u.  Of a small gate it is p (1 + g / 2), p = g u / 2 (the next term is below 2^-64 of p): p has at most 48
// bits and may be the middle between two codes, so that the side on which the rest lies is kept however small it is.
__device__ __forceinline__ double gated_wide(double g, double u) {
  if (fabs(g) >= 0x1p-30) return g * sigmoid_wide(g) * u;
  const double p = 0.5 * g * u, h = __builtin_fma(p, 0.5 * g, p);
  if (p == 0.0) return p;                     // with its sign
  if (h != p) return h;
  return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, p) + (g > 0.0 ? 1 : -1));
}
__device__ __forceinline__ float round_odd(double h) {
  const float r = (float)h;
  const double back = r;
  if (back == h || !(fabsf(r) < __builtin_inff())) return r;
  return __uint_as_float((__float_as_uint(r) - (fabs(back) > fabs(h) ? 1u : 0u)) | 1u);
}

template <int kDtype>
struct GatedRow {
  typedef typename Elem<kDtype>::raw raw;
  static constexpr bool kOpen = true;        // its values are not exact
  // Infinity if a gate is so low that its sigmoid has fewer than 24 bits in binary32; else what multiplies the
  // 2^-150 that g sigmoid(g) is off by where it is subnormal, the largest |u| (F16's gates begin at 2^-24).
  template <bool kExact, bool kStream>
  static __device__ __forceinline__ float load(const CodeArgs& a, int64_t t, int c, float (&v)[kPer]) {
    const raw* row = static_cast<const raw*>(a.x) + t * 2 * a.H;
    float g[kPer], u[kPer];
    load8<kDtype, kStream>(row, c, a.H, g);
    load8<kDtype, kStream>(row + a.H, c, a.H, u);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if constexpr (kExact) {
        v[i] = round_odd(gated_wide(g[i], u[i]));
      } else {
        float s, rest;
        sigmoid_both(g[i], s, rest);
        v[i] = g[i] * s * u[i];
      }
    }
    float least = g[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) least = fminf(least, g[i]);
    if (least < -80.0f) return __builtin_inff();
    float most = 0.0f;
    if constexpr (kDtype != EQB_DTYPE_F16) {
#pragma unroll
      for (int i = 0; i < kPer; ++i) most = fmaxf(most, fabsf(u[i]));
    }
    return most;
  }
};

// The gated value as eqb_gated stores it, in binary32 where the type does not hold it (F16 ends at 65,504).  98,304
// rows of 2,048 bf16 of 64 experts by columns: 217 us (4.6 TB/s), stored and read again 335.
template <int kDtype>
struct StoredGate {
  typedef typename Elem<kDtype>::raw raw;
  template <bool kExact, bool kStream>
  static __device__ __forceinline__ void load(const CodeArgs& a, int64_t t, int c, float (&v)[kPer]) {
    const raw* row = static_cast<const raw*>(a.x) + t * 2 * a.H;
    float g[kPer], u[kPer];
    load8<kDtype, kStream>(row, c, a.H, g);
    load8<kDtype, kStream>(row + a.H, c, a.H, u);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      float s, rest;
      sigmoid_both(g[i], s, rest);
      const float h = g[i] * s * u[i], stored = Elem<kDtype>::to_f(Elem<kDtype>::from_f(h));
      v[i] = fabsf(stored) < __builtin_inff() ? stored : h;
    }
  }
};

__device__ __forceinline__ int64_t rows_in_use(const CodeArgs& a) {
  if (!a.count) return a.T;
  const int64_t n = *a.count;
  return n < a.T ? n : a.T;
}

// Sixteen lanes hold a block; a wave holds four, of as many rows where rows are of one or two blocks
// (kBlocks; 355,390 rows of 47 to their experts: 35 -> 15 us, 600,000 gated ones of 36
// 375 -> 120).  With slots, a token's codes go to all
// of its rows.
template <class Row, bool kStream, int kBlocks>
__global__ __launch_bounds__(kCodeThreads) void quantize_rows_kernel(const CodeArgs a, int segments) {
  constexpr int kLanes = 16 * kBlocks, kRows = 4 / kBlocks;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = rows_in_use(a), width = code_width(a.H), scales = scale_width(a.H);
  for (int64_t seg = blockIdx.x; seg < segments; seg += gridDim.x) {
    const int c = (int)seg * kWaveCols + lane % kLanes * kPer;
    for (int64_t t0 = ((int64_t)blockIdx.y * kCodeWaves + wave) * kRows; t0 < rows; t0 += (int64_t)gridDim.y * kCodeWaves * kRows) {
      const bool live = kRows == 1 || t0 + lane / kLanes < rows;
      const int64_t t = kRows == 1 ? t0 : live ? t0 + lane / kLanes : rows - 1;
      float v[kPer], top;
      int byte;
      uint2 code;
      auto codes = [&](float by) {
        return make_uint2(codes4(v[0] * by, v[1] * by, v[2] * by, v[3] * by), codes4(v[4] * by, v[5] * by, v[6] * by, v[7] * by));
      };
      auto encode = [&]() {
        top = 0.0f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) top = fmaxf(top, finite_abs(v[i]));
        top = group_max<16>(top);
        byte = scale_byte(top);
        code = codes(scale_inverse(byte));
      };
      const float reach = Row::template load<false, kStream>(a, t, c, v);
      encode();
      if constexpr (Row::kOpen) {
        constexpr float kLess = 1.0f - 0x1p-19f, kMore = 1.0f + 0x1p-19f;
        const uint2 less = codes(scale_inverse(byte) * kLess), more = codes(scale_inverse(byte) * kMore);
        // the least middle between two codes is 2^(byte - 137), and 2^-20 of it is left beside the other roundings
        const float most = __uint_as_float((uint32_t)(byte < 134 ? byte + 120 : 254) << 23);
        const bool open = reach > most || less.x != more.x || less.y != more.y || scale_byte(top * kLess) != scale_byte(top * kMore);
        if (__ballot(open)) {
          Row::template load<true, kStream>(a, t, c, v);
          encode();
        }
      }
      const int mine = c < width ? byte : 0;
      uint32_t word = (uint32_t)mine;
      if constexpr (kBlocks == 2) word |= (uint32_t)__shfl_down(mine, 16) << 8;
      if constexpr (kBlocks == 4)
        word = (uint32_t)__builtin_amdgcn_readlane(mine, 0) | (uint32_t)__builtin_amdgcn_readlane(mine, 16) << 8 |
               (uint32_t)__builtin_amdgcn_readlane(mine, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane(mine, 48) << 24;
      if (!live) continue;
      for (int k = 0; k < a.K; ++k) {
        const int64_t r = a.slot ? a.slot[t * a.K + k] : t;
        if (r < 0 || r >= a.rows) continue;
        if (c < width) store_at<kStream>(reinterpret_cast<uint64_t*>(a.codes + r * width + c), __builtin_bit_cast(uint64_t, code));
        if (lane % kLanes == 0) *reinterpret_cast<uint32_t*>(a.scales + r * scales + seg * 4) = word;
      }
    }
  }
}

// ---------------------------------------------------------- the gate --
// kLanes of a row: 64, or as many as its elements need (16 or 32).
template <int kDtype, bool kBackward, bool kStream, int kLanes>
__global__ __launch_bounds__(kCodeThreads) void gated_kernel(const CodeArgs a, int segments) {
  typedef typename Elem<kDtype>::raw raw;
  constexpr int kRows = 64 / kLanes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rows = rows_in_use(a);
  for (int64_t seg = blockIdx.x; seg < segments; seg += gridDim.x) {
    const int c = (int)seg * kWaveCols + lane % kLanes * kPer;
    if (c >= a.H) continue;
    for (int64_t t = ((int64_t)blockIdx.y * kCodeWaves + wave) * kRows + lane / kLanes; t < rows; t += (int64_t)gridDim.y * kCodeWaves * kRows) {
      const raw* row = static_cast<const raw*>(a.x) + t * 2 * a.H;
      if constexpr (!kBackward) {
        float g[kPer], u[kPer];
        load8<kDtype, kStream>(row, c, a.H, g);
        load8<kDtype, kStream>(row + a.H, c, a.H, u);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          float s, rest;
          sigmoid_both(g[i], s, rest);
          g[i] = g[i] * s * u[i];
        }
        store8<kDtype, kStream>(static_cast<raw*>(a.out) + t * a.H, c, a.H, g);
      } else {
        raw* to = static_cast<raw*>(a.out) + t * 2 * a.H;
        float g[kPer], u[kPer], h[kPer];
        load8<kDtype, kStream>(row, c, a.H, g);
        load8<kDtype, kStream>(row + a.H, c, a.H, u);
        load8<kDtype, kStream>(static_cast<const raw*>(a.grad) + t * a.H, c, a.H, h);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          float s, rest;
          sigmoid_both(g[i], s, rest);
          const float hs = h[i] * s;
          const float gu = hs * g[i];
          g[i] = hs * u[i] * __builtin_fmaf(g[i], rest, 1.0f);
          u[i] = gu;
        }
        store8<kDtype, kStream>(to, c, a.H, g);
        store8<kDtype, kStream>(to + a.H, c, a.H, u);
      }
    }
  }
}

// ------------------------------------------------- columns and weights --
// A tile of 128 rows and kCols columns: a thread holds kRows neighbouring rows of 8 neighbouring columns,
// and the transposed codes go through LDS.  kWeights: one scale for the tile (of 128 x 128), and the
// codes in the rows' order too.
typedef uint32_t word4 __attribute__((ext_vector_type(4)));
constexpr int kTileStride = kCodeBlock + 4;        // bytes of a column in LDS: 33 words, so that columns 8 apart differ by 8 banks

// The expert whose blocks of columns hold block b, the last one whose first block is at most b, and its rows
// (e = -1: none).  By a whole wave, with one wait for the offsets.
__device__ __forceinline__ void expert_of_block(const int32_t* offsets, int E, int64_t rows, int64_t b, int lane, int& e,
                                                int64_t& begin, int64_t& end) {
  e = -1;
  begin = end = 0;
  for (int e0 = 0; e0 < E; e0 += 64) {
    const int i = e0 + lane;
    const int from = i < E ? offsets[i] : 0, to = i < E ? offsets[i + 1] : 0;
    const int64_t off = from < 0 ? 0 : from > rows ? rows : from;
    const uint64_t up_to = __ballot(i < E && off / kCodeBlock + i <= b);
    if (up_to == 0) break;
    const int last = 63 - __builtin_clzll(up_to);
    e = e0 + last;
    begin = __builtin_amdgcn_readlane(from, last);
    end = __builtin_amdgcn_readlane(to, last);
  }
  begin = begin < 0 ? 0 : begin > rows ? rows : begin;
  end = end > rows ? rows : end;
}

template <class Row, bool kWeights, bool kStream, int kRows, int kCols>
__global__ __launch_bounds__(kCodeThreads) void quantize_tiles_kernel(const CodeArgs a) {
  constexpr int kGroups = kCols / kPer;         // of columns
  static_assert(kCodeBlock / kRows * kGroups == kCodeThreads && (!kWeights || kCols == kCodeBlock), "a thread for each");
  __shared__ __attribute__((aligned(16))) uint8_t sh_code[kCols * kTileStride];
  __shared__ float sh_top[kCodeWaves][kCols];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cg = tid % kGroups, rg = tid / kGroups;
  // this tile's place among the tiles of columns, and of (an expert's) rows
  const uint32_t across = (uint32_t)((a.H + kCols - 1) / kCols);
  const uint32_t bx = blockIdx.x % across, down = (uint32_t)(code_width(a.N) / kCodeBlock);
  const uint32_t by = kWeights ? blockIdx.x / across % down : blockIdx.x / across;
  int e, first;                 // the expert, and the first of its rows here
  int64_t base;                 // the row before those
  int nr;                       // rows of the tile
  if (kWeights) {
    e = blockIdx.x / across / down;
    first = by * kCodeBlock;
    base = (int64_t)e * a.N;
    nr = a.N - first;
  } else {
    int64_t begin, end;
    expert_of_block(a.offsets, a.E, a.rows, by, lane, e, begin, end);
    if (e < 0) return;
    const int64_t local = ((int64_t)by - (begin / kCodeBlock + e)) * kCodeBlock;
    if (local < 0 || local >= end - begin) return;
    first = (int)local;
    base = begin;
    nr = (int)(end - begin - local);
  }
  if (nr > kCodeBlock) nr = kCodeBlock;
  const int c0 = bx * kCols, c = c0 + cg * kPer;
  float v[kRows][kPer];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = rg * kRows + i;
    if (r < nr && c < a.H) {
      Row::template load<false, kStream>(a, base + first + r, c, v[i]);
    } else {
#pragma unroll
      for (int j = 0; j < kPer; ++j) v[i][j] = 0.0f;
    }
  }
  float top[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    top[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) top[j] = fmaxf(top[j], finite_abs(v[i][j]));
#pragma unroll
    for (int d = kGroups; d < 64; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor(top[j], d));
  }
  if (kWeights) {
#pragma unroll
    for (int j = 1; j < kPer; ++j) top[0] = fmaxf(top[0], top[j]);
    top[0] = group_max<kGroups>(top[0]);
    if (lane == 0) sh_top[wave][0] = top[0];
  } else if (lane < kGroups) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) sh_top[wave][cg * kPer + j] = top[j];
  }
  __syncthreads();
  int byte[kPer];
  float inv[kPer];
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int at = kWeights ? 0 : cg * kPer + j;
    byte[j] = scale_byte(fmaxf(fmaxf(sh_top[0][at], sh_top[1][at]), fmaxf(sh_top[2][at], sh_top[3][at])));
    inv[j] = scale_inverse(byte[j]);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i)
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[i][j] *= inv[j];
  if (kWeights && a.codes) {
    const int64_t width = code_width(a.H);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int r = rg * kRows + i;
      if (r >= nr) continue;
      uint2 code;
      code.x = codes4(v[i][0], v[i][1], v[i][2], v[i][3]);
      code.y = codes4(v[i][4], v[i][5], v[i][6], v[i][7]);
      store_at<kStream>(reinterpret_cast<uint64_t*>(a.codes + (base + first + r) * width + c), __builtin_bit_cast(uint64_t, code));
    }
    // with the last block of a row, the zeros behind its scales
    const int64_t scales = scale_width(a.H);
    const int more = (int)(bx + 1 == across ? scales - bx : 1);
    if (tid < more)
      a.scales[((int64_t)e * down + by) * scales + bx + tid] = tid == 0 ? (uint8_t)byte[0] : 0;
  }
  uint8_t* const to = kWeights ? a.codes_t : a.codes;
  if (!to) return;
#pragma unroll
  for (int j = 0; j < kPer; ++j)
#pragma unroll
    for (int i = 0; i < kRows; i += 4)
      *reinterpret_cast<uint32_t*>(sh_code + (cg * kPer + j) * kTileStride + rg * kRows + i) = codes4(v[i][j], v[i + 1][j], v[i + 2][j], v[i + 3][j]);
  __syncthreads();
  const int64_t width = kWeights ? code_width(a.N) : column_width(a.rows, a.E);
  const int64_t lead = kWeights ? (int64_t)e * a.H : 0;
#pragma unroll
  for (int i = 0; i < kCols * 8 / kCodeThreads; ++i) {
    const int at = tid + i * kCodeThreads, col = at >> 3, piece = at & 7;
    const uint32_t* from = reinterpret_cast<const uint32_t*>(sh_code + col * kTileStride + piece * 16);
    if (c0 + col < a.H)
      store_at<kStream>(reinterpret_cast<word4*>(to + (lead + c0 + col) * width + (int64_t)by * kCodeBlock + piece * 16), word4{from[0], from[1], from[2], from[3]});
  }
  const int64_t scales = scale_width(width);
  if (kWeights) {
    const int more = (int)(by + 1 == down ? scales - by : 1);
    if (tid < more)
      a.scales_t[((int64_t)e * across + bx) * scales + by + tid] = tid == 0 ? (uint8_t)byte[0] : 0;
  } else if (rg == 0) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
      if (c + j < a.H) a.scales[(int64_t)(c + j) * scales + by] = (uint8_t)byte[j];
  }
}

// rows: of a wave at a time
dim3 row_grid(const CodeArgs& a, int64_t width, int rows, int* segments) {
  *segments = (int)((width + kWaveCols - 1) / kWaveCols);
  int64_t y = (a.T + kCodeWaves * rows - 1) / (kCodeWaves * rows), most = 65535;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < most) most = cap;
  if (y > most) y = most;
  return dim3((uint32_t)(*segments < 1024 ? *segments : 1024), (uint32_t)y);
}

int64_t bytes_of(int32_t dtype) { return dtype == EQB_DTYPE_F32 ? 4 : 2; }

template <class Row, int kBlocks>
void launch_rows_in(const CodeArgs& a, bool stream, hipStream_t s) {
  int segments;
  const dim3 grid = row_grid(a, code_width(a.H), 4 / kBlocks, &segments);
  if (stream) quantize_rows_kernel<Row, true, kBlocks><<<grid, kCodeThreads, 0, s>>>(a, segments);
  else quantize_rows_kernel<Row, false, kBlocks><<<grid, kCodeThreads, 0, s>>>(a, segments);
}
template <class Row>
void launch_rows_by(const CodeArgs& a, bool stream, hipStream_t s) {
  const int64_t width = code_width(a.H);
  if (width <= kCodeBlock) launch_rows_in<Row, 1>(a, stream, s);
  else if (width <= 2 * kCodeBlock) launch_rows_in<Row, 2>(a, stream, s);
  else launch_rows_in<Row, 4>(a, stream, s);
}
template <template <int> class Row>
eqb_status launch_rows_of(const CodeArgs& a, int per_value, hipStream_t s) {
  const int64_t row = a.H * per_value * bytes_of(a.dtype), codes = a.T * a.K * code_width(a.H);
  const bool stream = row % 128 == 0 && (a.T * row >= kStreamBytes || codes >= kStreamBytes);
  if (a.dtype == EQB_DTYPE_BF16) launch_rows_by<Row<EQB_DTYPE_BF16>>(a, stream, s);
  else if (a.dtype == EQB_DTYPE_F16) launch_rows_by<Row<EQB_DTYPE_F16>>(a, stream, s);
  else launch_rows_by<Row<EQB_DTYPE_F32>>(a, stream, s);
  return launch_status();
}

template <int kDtype, bool kBackward, int kLanes>
void launch_gate_lanes(const CodeArgs& a, bool stream, hipStream_t s) {
  int segments;
  const dim3 grid = row_grid(a, a.H, 64 / kLanes, &segments);
  if (stream) gated_kernel<kDtype, kBackward, true, kLanes><<<grid, kCodeThreads, 0, s>>>(a, segments);
  else gated_kernel<kDtype, kBackward, false, kLanes><<<grid, kCodeThreads, 0, s>>>(a, segments);
}
template <int kDtype, bool kBackward>
void launch_gate_in(const CodeArgs& a, bool stream, hipStream_t s) {
  if (a.H <= 16 * kPer) launch_gate_lanes<kDtype, kBackward, 16>(a, stream, s);
  else if (a.H <= 32 * kPer) launch_gate_lanes<kDtype, kBackward, 32>(a, stream, s);
  else launch_gate_lanes<kDtype, kBackward, 64>(a, stream, s);
}
template <bool kBackward>
eqb_status launch_gate(const CodeArgs& a, hipStream_t s) {
  const int64_t row = a.H * bytes_of(a.dtype);
  const bool stream = row % 128 == 0 && a.T * row * 2 >= kStreamBytes;
  if (a.dtype == EQB_DTYPE_BF16) launch_gate_in<EQB_DTYPE_BF16, kBackward>(a, stream, s);
  else if (a.dtype == EQB_DTYPE_F16) launch_gate_in<EQB_DTYPE_F16, kBackward>(a, stream, s);
  else launch_gate_in<EQB_DTYPE_F32, kBackward>(a, stream, s);
  return launch_status();
}

// Columns: 19,000 rows of 1,024 bf16 over 32 experts 16.9 us with 64 columns a tile, 17.7 with 128; 88,000 of
// 2,048 90 and 98 (4.2 TB/s).  Weights, 64 of 2,048 x 2,048 bf16, both ways: 191 us (5.6 TB/s).
constexpr int kColumnRows = 4, kColumnCols = 64;
template <template <int> class Row, bool kWeights, bool kStream>
eqb_status launch_tiles(const CodeArgs& a, int64_t tiles, hipStream_t s) {
  if (tiles > INT32_MAX) return EQB_ERR_UNSUPPORTED;
  const uint32_t grid = (uint32_t)tiles;
  constexpr int R = kWeights ? 8 : kColumnRows, C = kWeights ? kCodeBlock : kColumnCols;
  if (a.dtype == EQB_DTYPE_BF16) quantize_tiles_kernel<Row<EQB_DTYPE_BF16>, kWeights, kStream, R, C><<<grid, kCodeThreads, 0, s>>>(a);
  else if (a.dtype == EQB_DTYPE_F16) quantize_tiles_kernel<Row<EQB_DTYPE_F16>, kWeights, kStream, R, C><<<grid, kCodeThreads, 0, s>>>(a);
  else quantize_tiles_kernel<Row<EQB_DTYPE_F32>, kWeights, kStream, R, C><<<grid, kCodeThreads, 0, s>>>(a);
  return launch_status();
}

}  // namespace

eqb_status launch_quantize_rows(const CodeArgs& a, hipStream_t s) { return launch_rows_of<PlainRow>(a, 1, s); }
eqb_status launch_dispatch_quantized(const CodeArgs& a, hipStream_t s) { return launch_rows_of<PlainRow>(a, 1, s); }
eqb_status launch_gated_quantize(const CodeArgs& a, hipStream_t s) { return launch_rows_of<GatedRow>(a, 2, s); }
eqb_status launch_gated(const CodeArgs& a, hipStream_t s) { return launch_gate<false>(a, s); }
eqb_status launch_gated_backward(const CodeArgs& a, hipStream_t s) { return launch_gate<true>(a, s); }

template <template <int> class Row>
static eqb_status launch_columns_of(const CodeArgs& a, int per_value, hipStream_t s) {
  const int64_t tiles = ((int64_t)a.H + kColumnCols - 1) / kColumnCols * (column_width(a.rows, a.E) / kCodeBlock);
  const int64_t row = a.H * bytes_of(a.dtype);
  if (row % 128 == 0 && a.rows * row * per_value >= kStreamBytes) return launch_tiles<Row, false, true>(a, tiles, s);
  return launch_tiles<Row, false, false>(a, tiles, s);
}
eqb_status launch_quantize_columns(const CodeArgs& a, hipStream_t s) { return launch_columns_of<PlainRow>(a, 1, s); }
eqb_status launch_gated_quantize_columns(const CodeArgs& a, hipStream_t s) { return launch_columns_of<StoredGate>(a, 2, s); }
eqb_status launch_quantize_weights(const CodeArgs& a, hipStream_t s) {
  const int64_t tiles = code_width(a.H) / kCodeBlock * (code_width(a.N) / kCodeBlock) * a.E, row = a.H * bytes_of(a.dtype);
  if (row % 128 == 0 && (int64_t)a.E * a.N * row >= kStreamBytes) return launch_tiles<PlainRow, true, true>(a, tiles, s);
  return launch_tiles<PlainRow, true, false>(a, tiles, s);
}

}  // namespace eqb
