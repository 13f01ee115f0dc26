// products.hip - the experts' products of E4M3 codes with a power of two for each block of
// 128 (what FFN_e of Eq. 1, arXiv 2609.28053, is made of): the rows with the weights, and
// the gradient of the weights.
//
// Both are out[p, q] = sum over k of P[p, k] Q[q, k] with k contiguous in P and Q: P is an
// expert's rows and Q its weights, or P the gradient's columns and Q the rows' columns,
// contracted over an expert's rows.  One matrix instruction contracts over a whole block
// of 128 and takes both scales, which are powers of two, so that a block costs no
// operation beside it.  But it adds a block's 128 products with what lies some 16 bits
// below the largest of them cut off: on codes of 11 binades a sum is off by 5e-5 of itself,
// a quarter of what rounding to f16 costs.  That serves results of 16 bits; for results in
// binary32 the codes become BF16 with their scale (exact down to 2^-133) on the way from LDS,
// and the instruction for those sums in full (6e-8), at half the rate.
#include "eqb_internal.hpp"

namespace eqb {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) uint32_t lds_word;
typedef const __attribute__((address_space(1))) uint32_t global_word;

template <int kDtype>
struct OutType;
template <>
struct OutType<EQB_DTYPE_F32> {
  typedef float raw;
  static __device__ __forceinline__ raw from_f(float x) { return x; }
};
template <>
struct OutType<EQB_DTYPE_BF16> {
  typedef uint16_t raw;
  static __device__ __forceinline__ raw from_f(float x) { return (raw)bf16x2_bits(x, x); }
};
template <>
struct OutType<EQB_DTYPE_F16> {
  typedef _Float16 raw;
  static __device__ __forceinline__ raw from_f(float x) { return (raw)x; }
};

// Tiles of an expert's rows, found from the offsets alone: lane l of every wave holds the
// experts 4l .. 4l + 3 and how many tiles come before them.
struct Experts {
  int begin[4], count[4], tiles[4], before;
  int total;
  __device__ __forceinline__ Experts(const int32_t* offsets, int E, int64_t rows, int BP) {
    const int lane = threadIdx.x & 63;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane * 4 + i;
      int64_t a = e < E ? offsets[e] : 0, b = e < E ? offsets[e + 1] : 0;
      a = a < 0 ? 0 : a > rows ? rows : a;
      b = b > rows ? rows : b;
      begin[i] = (int)a;
      count[i] = b > a ? (int)(b - a) : 0;
      tiles[i] = (count[i] + BP - 1) / BP;
      sum += tiles[i];
    }
    int incl = sum;
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    before = incl - sum;
    total = __builtin_amdgcn_readlane(incl, 63);
  }
  // Expert and first row of row tile t < total; n: the expert's rows from there on.
  __device__ __forceinline__ void find(int t, int BP, int& e, int64_t& first, int& n) const {
    const int l = __popcll(__ballot(before <= t)) - 1;
    int left = t - __builtin_amdgcn_readlane(before, l);
    e = l * 4;
    int b = 0, c = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int m = __builtin_amdgcn_readlane(tiles[i], l);
      const int bi = __builtin_amdgcn_readlane(begin[i], l), ci = __builtin_amdgcn_readlane(count[i], l);
      if (!found && left < m) {
        found = true;
        e = l * 4 + i;
        b = bi;
        c = ci;
      } else if (!found) {
        left -= m;
      }
    }
    first = (int64_t)b + (int64_t)left * BP;
    n = c - left * BP;
  }
};

constexpr int kStep = kCodeBlock;       // bytes of a row per step

// Eight codes (words 2j and 2j + 1) times their scale.
__device__ __forceinline__ bf16x8_t widen(const int8v& code, int j, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j], scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j], scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j + 1], scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j + 1], scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// BP x BQ of out per block of WP x WQ waves.
template <int BP, int BQ, int WP, int WQ, bool kGrad, int kDtype>
__global__ __launch_bounds__(64 * WP * WQ) void product_kernel(const ProductArgs a) {
  constexpr int kWaves = WP * WQ, TP = BP / WP / 16, TQ = BQ / WQ / 16;
  constexpr int kLoads = (BP + BQ) / 8 / kWaves;      // a wave's loads of 8 rows per step
  typedef OutType<kDtype> O;
  __shared__ __attribute__((aligned(16))) uint8_t sh[2][(BP + BQ) * kStep];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = wave / WQ, wq = wave % WQ;
  const int lrow = lane & 15, quarter = lane >> 4;
  const int64_t W = kGrad ? column_width(a.rows, a.E) : code_width(a.H);
  const int64_t SW = scale_width(W);
  const int q_tiles = ((kGrad ? a.H : a.N) + BQ - 1) / BQ;
  const int p_tiles = kGrad ? (a.N + BP - 1) / BP : 0;
  const Experts experts(a.offsets, a.E, a.rows, kGrad ? 1 : BP);
  const int64_t tiles = kGrad ? (int64_t)a.E * p_tiles * q_tiles : (int64_t)experts.total * q_tiles;

  for (int64_t id = blockIdx.x; id < tiles; id += gridDim.x) {
    const int qt = (int)(id % q_tiles);
    const int64_t pt = id / q_tiles;
    int64_t p0;              // row of out
    int np, nq, steps, e;
    const uint8_t *p, *q, *ps, *qs;
    const int q0 = qt * BQ;
    if (kGrad) {
      e = (int)(pt / p_tiles);
      p0 = pt % p_tiles * BP;
      np = a.N - (int)p0;
      nq = a.H - q0;
      const int l = e >> 2;
      int begin = 0, count = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = __builtin_amdgcn_readlane(experts.begin[i], l), c = __builtin_amdgcn_readlane(experts.count[i], l);
        if ((e & 3) == i) {
          begin = b;
          count = c;
        }
      }
      const int64_t block = begin / kCodeBlock + e;
      steps = (count + kCodeBlock - 1) / kCodeBlock;
      p = a.x + p0 * W + block * kStep;
      ps = a.x_scales + p0 * SW + block;
      q = a.w + (int64_t)q0 * W + block * kStep;
      qs = a.w_scales + (int64_t)q0 * SW + block;
    } else {
      experts.find((int)pt, BP, e, p0, np);
      nq = a.N - q0;
      steps = (int)(W / kStep);
      p = a.x + p0 * W;
      ps = a.x_scales + p0 * SW;
      q = a.w + ((int64_t)e * a.N + q0) * W;
      qs = a.w_scales + ((int64_t)e * ((a.N + kCodeBlock - 1) / kCodeBlock) + q0 / kCodeBlock) * SW;
    }
    np = np < BP ? np : BP;
    nq = nq < BQ ? nq : BQ;

    // this lane's place in each of the wave's loads: row, and the 16 bytes that its place in
    // LDS is for (the pieces of a row are permuted by the row's number, so that lanes that
    // read the same piece of neighbouring rows use different banks)
    const uint8_t* from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      int r = (wave * kLoads + i) * 8 + (lane >> 3);
      const int piece = (lane & 7) ^ (r & 7);
      const bool is_p = r < BP;
      r = is_p ? r : r - BP;
      const int most = (is_p ? np : nq) - 1;
      r = r < most ? r : most;
      from[i] = (is_p ? p : q) + r * W + piece * 16;
    }
    auto load = [&](int step) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        __builtin_amdgcn_global_load_lds((global_word*)(from[i] + (int64_t)step * kStep),
                                         (lds_word*)(&sh[step & 1][(wave * kLoads + i) * 8 * kStep]), 16, 0, 0);
      }
    };
    // the scales of this lane's rows
    const uint8_t *p_scale[TP], *q_scale[TQ];
#pragma unroll
    for (int i = 0; i < TP; ++i) {
      int r = (wp * TP + i) * 16 + lrow;
      r = r < np ? r : np - 1;
      p_scale[i] = ps + r * SW;
    }
#pragma unroll
    for (int i = 0; i < TQ; ++i) {
      int r = (wq * TQ + i) * 16 + lrow;
      r = r < nq ? r : nq - 1;
      q_scale[i] = kGrad ? qs + r * SW : qs + r / kCodeBlock * SW;
    }

    float4v acc[TP][TQ];
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
      for (int j = 0; j < TQ; ++j) acc[i][j] = float4v{0, 0, 0, 0};

    __syncthreads();       // the last tile's reads of LDS are done
    if (steps > 0) load(0);
    for (int step = 0; step < steps; ++step) {
      int sp[TP], sq[TQ];
#pragma unroll
      for (int i = 0; i < TP; ++i) sp[i] = p_scale[i][step];
#pragma unroll
      for (int j = 0; j < TQ; ++j) sq[j] = q_scale[j][step];
      __syncthreads();     // this step's codes are there, and the other buffer is free
      if (step + 1 < steps) load(step + 1);
      const uint8_t* at = sh[step & 1];
      int8v fp[TP], fq[TQ];
      auto piece = [&](int r, int k) {
        return *reinterpret_cast<const int4v*>(at + r * kStep + ((k ^ (r & 7)) * 16));
      };
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        const int r = (wp * TP + i) * 16 + lrow;
        fp[i] = __builtin_shufflevector(piece(r, quarter * 2), piece(r, quarter * 2 + 1), 0, 1, 2, 3, 4, 5, 6, 7);
      }
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        const int r = BP + (wq * TQ + j) * 16 + lrow;
        fq[j] = __builtin_shufflevector(piece(r, quarter * 2), piece(r, quarter * 2 + 1), 0, 1, 2, 3, 4, 5, 6, 7);
      }
      if constexpr (kDtype == EQB_DTYPE_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          bf16x8_t wide[TQ];
#pragma unroll
          for (int j = 0; j < TQ; ++j) wide[j] = widen(fq[j], k, __uint_as_float((uint32_t)sq[j] << 23));
#pragma unroll
          for (int i = 0; i < TP; ++i) {
            const bf16x8_t x = widen(fp[i], k, __uint_as_float((uint32_t)sp[i] << 23));
#pragma unroll
            for (int j = 0; j < TQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[j], x, acc[i][j], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < TP; ++i)
#pragma unroll
          for (int j = 0; j < TQ; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fq[j], fp[i], acc[i][j], 0, 0, 0, sq[j], 0, sp[i]);
      }
    }

    // a lane holds four neighbouring q of one p
    typename O::raw* const out = static_cast<typename O::raw*>(a.out);
    const int64_t width = kGrad ? a.H : a.N;
    const int64_t row0 = kGrad ? (int64_t)e * a.N + p0 : p0;
#pragma unroll
    for (int i = 0; i < TP; ++i) {
      const int r = (wp * TP + i) * 16 + lrow;
      if (r >= np) continue;
#pragma unroll
      for (int j = 0; j < TQ; ++j) {
        const int c = (wq * TQ + j) * 16 + quarter * 4;
        typename O::raw* to = out + (row0 + r) * width + q0 + c;
        typedef typename O::raw vec __attribute__((ext_vector_type(4)));
        typedef vec any __attribute__((aligned(alignof(typename O::raw))));
        const vec v = {O::from_f(acc[i][j][0]), O::from_f(acc[i][j][1]), O::from_f(acc[i][j][2]), O::from_f(acc[i][j][3])};
        if (c + 4 <= nq) {
          *reinterpret_cast<any*>(to) = v;
        } else {
#pragma unroll
          for (int k = 0; k < 3; ++k)
            if (c + k < nq) to[k] = v[k];
        }
      }
    }
  }
}

template <bool kGrad>
eqb_status launch_product(const ProductArgs& a, hipStream_t s) {
  constexpr int BP = 128, BQ = 128;
  const int64_t q_tiles = ((kGrad ? a.H : a.N) + BQ - 1) / BQ;
  const int64_t p_tiles = kGrad ? (int64_t)a.E * ((a.N + BP - 1) / BP) : a.rows / BP + (a.rows < a.E ? a.rows : a.E);
  int64_t grid = (int64_t)num_cus() * 2;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < grid) grid = cap;
  if (p_tiles * q_tiles < grid) grid = p_tiles * q_tiles;
  const uint32_t blocks = (uint32_t)grid;
  if (a.dtype == EQB_DTYPE_BF16) product_kernel<BP, BQ, 2, 2, kGrad, EQB_DTYPE_BF16><<<blocks, 256, 0, s>>>(a);
  else if (a.dtype == EQB_DTYPE_F16) product_kernel<BP, BQ, 2, 2, kGrad, EQB_DTYPE_F16><<<blocks, 256, 0, s>>>(a);
  else product_kernel<BP, BQ, 2, 2, kGrad, EQB_DTYPE_F32><<<blocks, 256, 0, s>>>(a);
  return launch_status();
}

}  // namespace

eqb_status launch_experts_product(const ProductArgs& a, hipStream_t s) { return launch_product<false>(a, s); }
eqb_status launch_experts_grad_weight(const ProductArgs& a, hipStream_t s) { return launch_product<true>(a, s); }

}  // namespace eqb
