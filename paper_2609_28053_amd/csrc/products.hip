// products.hip - the experts' products of E4M3 codes with a power of two for each block of
// 128 (what FFN_e of Eq. 1, arXiv 2609.28053, is made of): the rows with the weights, and
// the gradient of the weights.
//
// Both are out[p, q] = sum over k of P[p, k] Q[q, k] with k contiguous in P and Q: P is an
// expert's rows and Q its weights, or P the gradient's columns and Q the rows' columns,
// contracted over an expert's rows.  One matrix instruction contracts over a whole block
// of 128 and takes both scales, which are powers of two, so that a block costs no
// operation beside it.  But it adds a block's 128 products with what lies some 16 bits
// below the largest of them cut off: at most 2^-9 of the largest, however small the sum is; on
// random codes of 11 binades 5e-5 of the sum, a quarter of what rounding to f16 costs.  That
// serves results of 16 bits, which are rounded by up to 2^-8 (bf16) or 2^-11 of themselves; for
// results in binary32 the codes become BF16 with their scale (exact down to 2^-133) on the way
// from LDS, and the instruction for those sums in full (6e-8), at half the rate.
#include "eqb_internal.hpp"

namespace eqb {
namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

typedef __attribute__((address_space(3))) uint32_t lds_word;

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

// The experts' rows in LDS, and how many tiles of rows come before every fourth expert.
struct Experts {
  int2 rows[kMostExperts];        // first row, and how many
  int before[kMostExperts / 4], total;
  uint8_t largest[kMostExperts];  // the experts by their rows, most first

  // By every wave of the block; lane l takes the experts 4l .. 4l + 3.
  __device__ __forceinline__ void fill(const int32_t* offsets, int E, int64_t most, int BP) {
    const int lane = threadIdx.x & 63;
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane * 4 + i;
      int64_t a = e < E ? offsets[e] : 0, b = e < E ? offsets[e + 1] : 0;
      a = a < 0 ? 0 : a > most ? most : a;
      b = b > most ? most : b;
      const int n = b > a ? (int)(b - a) : 0;
      rows[e] = make_int2((int)a, n);
      sum += (n + BP - 1) / BP;
    }
    int incl = sum;
    for (int d = 1; d < 64; d <<= 1) {
      const int y = __shfl_up(incl, d);
      if (lane >= d) incl += y;
    }
    before[lane] = incl - sum;
    if (lane == 63) total = incl;
  }
  // By all threads, behind a barrier.
  __device__ __forceinline__ void sort(int E) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
      const int n = rows[e].y;
      int rank = 0;
      for (int i = 0; i < E; ++i) rank += rows[i].y > n || (rows[i].y == n && i < e) ? 1 : 0;
      largest[rank] = (uint8_t)e;
    }
  }
  __device__ __forceinline__ int2 of(int e) const {
    const int2 r = rows[e];
    return make_int2(__builtin_amdgcn_readfirstlane(r.x), __builtin_amdgcn_readfirstlane(r.y));
  }
  // Expert and first row of row tile t < total; n: the expert's rows from there on.
  __device__ __forceinline__ void find(int t, int BP, int& e, int64_t& first, int& n) const {
    const int l = __popcll(__ballot(before[threadIdx.x & 63] <= t)) - 1;
    int left = t - __builtin_amdgcn_readfirstlane(before[l]);
    e = l * 4;
    int2 r = of(e);
    for (int i = 0; i < 3; ++i) {
      const int m = (r.y + BP - 1) / BP;
      if (left < m) break;
      left -= m;
      r = of(++e);
    }
    first = (int64_t)r.x + (int64_t)left * BP;
    n = r.y - left * BP;
  }
};

constexpr int kStep = kCodeBlock;       // bytes of a row per step
constexpr int64_t kMemorySideCache = (int64_t)256 << 20;

// Eight codes (words 2j and 2j + 1) times their scale.
__device__ __forceinline__ bf16x8_t widen(const int4v& code, int j, float scale) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j], scale, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j], scale, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j + 1], scale, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[2 * j + 1], scale, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Waits for this wave's loads, stores and LDS reads, then for the block's other waves.
__device__ __forceinline__ void step_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Memory to LDS: 16 (4) bytes a lane from base + off to to + 16 (4) lane.  Written out, since
// the compiler would wait for all of them before any LDS read: step_barrier waits for them.
// They change m0, which the compiler reserves: it says that it will not keep what was there, and need not.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void copy16(uint8_t* to, const uint8_t* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"((uint32_t)(uintptr_t)(lds_word*)to), "v"(off), "s"(base)
               : "m0", "memory");
}
__device__ __forceinline__ void copy4(uint32_t* to, const uint8_t* base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"((uint32_t)(uintptr_t)(lds_word*)to), "v"(off), "s"(base)
               : "m0", "memory");
}
#pragma clang diagnostic pop

// What a tile of out is computed from.
struct Tile {
  int64_t row;             // first row of out
  int col, np, nq;         // first column, rows and columns that exist
  int block, end;          // the blocks of codes to contract over
  const uint8_t *p, *q, *ps, *qs;      // the first row's first code and scale (of block 0)
};

// BP x BQ of out per block of WP x WQ waves.  Blocks are as many as run at once and go from
// tile to tile, and the steps of all their tiles (128 of k each) are one sequence: codes and
// scales go from memory to LDS directly, two steps ahead.  A wave reads a step's fragments in
// this order: first the columns and the first rows, while the matrix instructions of the last
// kTail rows of the step before run; then the other rows, each ahead of its instructions.  When
// it has the last of them its buffer is free for the step after the next: that is the barrier.
//   By BF16 a step is two halves, each of its columns, widened once, and then its rows one by
// one, so that a tile of 256 x 256 fits the registers (93,389 rows of 2,048 to 2,048, gradients in
// binary32, before the tiles' order: 1,057 -> 891 us; 156 of them are stores, 50 the widening; without
// stores and loads the matrix pipes are busy two thirds of the time, at a clock of 1.6 GHz).
template <int BP, int BQ, int WP, int WQ, bool kGrad, int kDtype>
__global__ __launch_bounds__(64 * WP * WQ, 1) void product_kernel(const ProductArgs a) {
  typedef OutType<kDtype> O;
  typedef typename O::raw raw;
  constexpr bool kWide = kDtype == EQB_DTYPE_F32;     // by BF16
  constexpr int kWaves = WP * WQ, TP = BP / WP / 16, TQ = BQ / WQ / 16;
  constexpr int kTail = TP >= 4 ? 2 : 1;
  constexpr int kAhead = TP >= 8 ? 2 : 1;      // rows whose fragments are read before they are needed
  constexpr bool kOneScale = !kGrad;     // a wave's columns lie in one block of the weights
  static_assert(kGrad || kCodeBlock % (TQ * 16) == 0, "they do");
  constexpr int kLoadsP = BP / 8 / kWaves, kLoadsQ = BQ / 8 / kWaves;      // a wave's loads of 8 rows per step
  // A lane gets four neighbouring columns of out from a matrix instruction.  With results of 16
  // bits, two instructions' columns are interleaved in fours, so that it has eight: 16 bytes.
  constexpr int kPair = sizeof(raw) == 2 ? 2 : 1;
  static_assert(TQ % kPair == 0 && kLoadsP > 0 && kLoadsQ > 0 && TP >= kTail, "whole loads and stores");
  __shared__ __attribute__((aligned(16))) uint8_t sh[2][(BP + BQ) * kStep];
  __shared__ __attribute__((aligned(16))) uint32_t sh_scale[2][BP + BQ];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = wave / WQ, wq = wave % WQ, lrow = lane & 15, quarter = lane >> 4;
  const int64_t W = kGrad ? column_width(a.rows, a.E) : code_width(a.H);
  const int SW = (int)scale_width(W);
  const int q_tiles = ((kGrad ? a.H : a.N) + BQ - 1) / BQ;
  const int p_tiles = kGrad ? (a.N + BP - 1) / BP : 0;
  __shared__ __attribute__((aligned(16))) Experts experts;
  experts.fill(a.offsets, a.E, a.rows, BP);
  __syncthreads();
  if (kGrad) {
    experts.sort(a.E);
    __syncthreads();
  }
  const uint32_t tiles = (uint32_t)((kGrad ? a.E * p_tiles : __builtin_amdgcn_readfirstlane(experts.total)) * q_tiles);

  auto tile_of = [&](uint32_t id) {
    Tile t;
    const uint32_t pt = id / (uint32_t)q_tiles;
    t.col = (int)(id - pt * q_tiles) * BQ;
    if (kGrad) {
      const int n = (int)(pt / (uint32_t)p_tiles), p0 = ((int)pt - n * p_tiles) * BP;
      const int e = __builtin_amdgcn_readfirstlane(experts.largest[n]);
      t.row = (int64_t)e * a.N + p0;
      t.np = a.N - p0;
      t.nq = a.H - t.col;
      const int2 r = experts.of(e);
      t.block = r.x / kCodeBlock + e;
      t.end = t.block + (r.y + kCodeBlock - 1) / kCodeBlock;
      t.p = a.x + p0 * W;
      t.ps = a.x_scales + (int64_t)p0 * SW;
      t.q = a.w + t.col * W;
      t.qs = a.w_scales + (int64_t)t.col * SW;
    } else {
      int e;
      experts.find((int)pt, BP, e, t.row, t.np);
      t.nq = a.N - t.col;
      t.block = 0;
      t.end = (int)(W / kStep);
      t.p = a.x + t.row * W;
      t.ps = a.x_scales + t.row * SW;
      t.q = a.w + ((int64_t)e * a.N + t.col) * W;
      t.qs = a.w_scales + ((int64_t)e * ((a.N + kCodeBlock - 1) / kCodeBlock) + t.col / kCodeBlock) * SW;
    }
    t.np = t.np < BP ? t.np : BP;
    t.nq = t.nq < BQ ? t.nq : BQ;
    return t;
  };

  // Column of row r of Q in LDS, within its tile: row 16 j + m of a pair's 32 is column
  // 8 (m / 4) + 4 j + m % 4.
  auto column_of = [](int r) { return kPair == 2 ? (r & ~31) + (r >> 2 & 3) * 8 + (r >> 4 & 1) * 4 + (r & 3) : r; };

  // ---- the loads: a sequence of steps over this block's tiles
  const uint32_t eighth = gridDim.x / 8;
  const uint32_t first_id = blockIdx.x < eighth * 8 ? (blockIdx.x % 8) * eighth + blockIdx.x / 8 : blockIdx.x;
  // The gradients' tiles are as long as their experts are large: the largest come first, and the blocks
  // take every other round of tiles in the other direction (64 gradients of 521 x 1,023 over 100,362 rows,
  // the largest expert of 4.7 times the mean: 271 -> 183 us; 128 of 128 x 140, all in one round, 111 -> 117).
  auto id_after = [&](uint32_t id) {
    return kGrad ? 2 * gridDim.x * (id / gridDim.x + 1) - 1 - id : id + gridDim.x;
  };
  // A load takes 8 rows (64 of scales).  A lane's place in each load is found once a tile, as an
  // offset from the tile's first row: its row, and the 16 bytes that its place in LDS is for.  The
  // pieces of a row are permuted by half the row's number, so that lanes that read the same piece
  // of neighbouring rows use different banks.  Rows behind the last are the last once more.
  constexpr int kLoads = kLoadsP + kLoadsQ, kScaleLoads = ((BP + BQ) / 64 + kWaves - 1) / kWaves;
  static_assert(BP % 64 == 0 && BQ % 64 == 0, "whole loads of scales");
  uint32_t load_id = first_id, off[kLoads], scale_off[kScaleLoads];
  const uint8_t *from_p = nullptr, *from_q = nullptr, *from_ps = nullptr, *from_qs = nullptr;
  int from_block = 0, from_end = 0, from_word = 0;
  int buffer = 0;                     // where the next step's codes and scales go
  // Goes on to the next step; behind the last one it stays, and what is loaded again is not used.
  auto aim = [&]() {
    while (from_block == from_end && load_id < tiles) {
      const Tile t = tile_of(load_id);
      load_id = id_after(load_id);
      from_block = t.block;
      from_end = t.end;
      if (t.block == t.end) continue;
      from_p = t.p + (int64_t)t.block * kStep - kStep;
      from_q = t.q + (int64_t)t.block * kStep - kStep;
      from_ps = t.ps;
      from_qs = t.qs;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const bool is_p = i < kLoadsP;
        const int group = is_p ? wave * kLoadsP + i : wave * kLoadsQ + i - kLoadsP, most = (is_p ? t.np : t.nq) - 1;
        const int to = group * 8 + (lane >> 3);
        const int r = is_p ? to : column_of(to);
        off[i] = (uint32_t)(r < most ? r : most) * (uint32_t)W + (((lane & 7) ^ (to >> 1 & 7)) * 16);
      }
#pragma unroll
      for (int k = 0; k < kScaleLoads; ++k) {
        const int i = k * kWaves + wave;
        const bool is_p = i * 64 < BP;
        const int r = (is_p ? i * 64 : i * 64 - BP) + lane, most = (is_p ? t.np : t.nq) - 1;
        const int at = r < most ? r : most;
        scale_off[k] = (uint32_t)(kGrad || is_p ? at : at / kCodeBlock) * (uint32_t)SW;
      }
    }
    if (from_block < from_end) {
      from_p += kStep;
      from_q += kStep;
      from_word = from_block & ~3;
      ++from_block;
    }
  };
  // the words with the step's scales (and those of its neighbours)
  auto load_scales = [&]() {
#pragma unroll
    for (int k = 0; k < kScaleLoads; ++k) {
      const int i = k * kWaves + wave;
      if ((BP + BQ) / 64 % kWaves != 0 && i >= (BP + BQ) / 64) break;
      copy4(&sh_scale[buffer][i * 64], (i * 64 < BP ? from_ps : from_qs) + from_word, scale_off[k]);
    }
  };
  // the i-th of a wave's loads of codes
  auto load_codes = [&](int i) {
    const bool is_p = i < kLoadsP;
    const int group = is_p ? wave * kLoadsP + i : BP / 8 + wave * kLoadsQ + i - kLoadsP;
    copy16(sh[buffer] + group * 8 * kStep, is_p ? from_p : from_q, off[i]);
  };

  // ---- the fragments
  const uint8_t* codes = sh[0];            // of the step that they are read from
  const uint8_t* scales = nullptr;
  int8v fp[TP], fq[TQ];
  int sp[TP], sq[kOneScale ? 1 : TQ];
  // rows 16 i + lrow: the permutation of the pieces is the same for all i
  const int piece0 = lrow * kStep + ((quarter * 2) ^ (lrow >> 1)) * 16, piece1 = lrow * kStep + ((quarter * 2 + 1) ^ (lrow >> 1)) * 16;
  auto fragment = [&](int base, int i) {
    const uint8_t* at = codes + base * kStep + i * 16 * kStep;
    return __builtin_shufflevector(*reinterpret_cast<const int4v*>(at + piece0), *reinterpret_cast<const int4v*>(at + piece1),
                                   0, 1, 2, 3, 4, 5, 6, 7);
  };
  auto read_p = [&](int i) {
    fp[i] = fragment(wp * TP * 16, i);
    sp[i] = scales[(wp * TP * 16 + lrow) * 4 + i * 64];
  };
  auto read_q = [&](int j) {
    fq[j] = fragment(BP + wq * TQ * 16, j);
    if (!kOneScale || j == TQ - 1) sq[kOneScale ? 0 : j] = scales[(BP + wq * TQ * 16 + column_of(lrow)) * 4 + column_of(j * 16) * 4];
  };
  // the wide form's: half of a lane's 32 codes at a time
  int4v hp[TP], hq[TQ];
  auto half = [&](int base, int i, int h) {
    return *reinterpret_cast<const int4v*>(codes + base * kStep + i * 16 * kStep + (h ? piece1 : piece0));
  };
  auto read_half_p = [&](int i, int h) {
    hp[i] = half(wp * TP * 16, i, h);
    sp[i] = scales[(wp * TP * 16 + lrow) * 4 + i * 64];
  };
  auto read_half_q = [&](int j, int h) {
    hq[j] = half(BP + wq * TQ * 16, j, h);
    if (h == 0 && (!kOneScale || j == TQ - 1)) sq[kOneScale ? 0 : j] = scales[(BP + wq * TQ * 16 + column_of(lrow)) * 4 + column_of(j * 16) * 4];
  };
  auto power = [](int byte) { return __uint_as_float((uint32_t)byte << 23); };
  auto read_first = [&]() {
#pragma unroll
    for (int j = 0; j < TQ; ++j) {
      if constexpr (kWide) read_half_q(j, 0);
      else read_q(j);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if constexpr (kWide) read_half_p(i, 0);
      else read_p(i);
    }
  };
  float4v acc[TP][TQ];
  auto multiply = [&](int i, int j) {
    acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fq[j], fp[i], acc[i][j], 0, 0, 0, sq[kOneScale ? 0 : j], 0, sp[i]);
  };

  if (first_id >= tiles) return;
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    aim();
    if (from_p == nullptr) break;        // no tile has steps
    load_scales();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) load_codes(i);
    buffer ^= 1;
  }
  step_barrier();
  int read_buffer = 0;     // of the next step to be read
  auto next_step = [&](int block) {
    codes = sh[read_buffer];
    scales = reinterpret_cast<const uint8_t*>(sh_scale[read_buffer]) + (block & 3);
    read_buffer ^= 1;
  };

  uint32_t id = first_id;
  Tile t = tile_of(id);
  bool ready = false;      // whether the tile's first fragments are read (or being read)
  while (true) {
#pragma unroll
    for (int i = 0; i < TP; ++i)
#pragma unroll
      for (int j = 0; j < TQ; ++j) acc[i][j] = float4v{0, 0, 0, 0};
    const uint32_t next_id = id_after(id);
    if (t.block < t.end && !ready) {
      next_step(t.block);
      read_first();
    }
    Tile next = t;
    for (int block = t.block; block < t.end; ++block) {
      const bool last = block + 1 == t.end;
      aim();
      bool on = !last;         // whether another step follows that is known here
      if (last && next_id < tiles) {
        next = tile_of(next_id);
        on = next.block < next.end;
      }
      if constexpr (kWide) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          bf16x8_t wide[2][TQ];
#pragma unroll
          for (int j = 0; j < TQ; ++j) {
            wide[0][j] = widen(hq[j], 0, power(sq[kOneScale ? 0 : j]));
            wide[1][j] = widen(hq[j], 1, power(sq[kOneScale ? 0 : j]));
          }
          __builtin_amdgcn_sched_barrier(0);
          if (h == 0) {
#pragma unroll
            for (int j = 0; j < TQ; ++j) read_half_q(j, 1);
          }
#pragma unroll
          for (int i = 0; i < TP; ++i) {
            constexpr int kFree = TP - kAhead;       // from this row on of the second half all is read
            if (h == 1 && i == kFree) {
              step_barrier();
              if (on) next_step(last ? next.block : block + 1);
              load_scales();
#pragma unroll
              for (int j = 0; j < TQ; ++j) read_half_q(j, 0);
            }
            const int n = (h * TP + i + kAhead) % (2 * TP);
            read_half_p(n % TP, n / TP);
            if (h == 1 && i >= kFree) {
#pragma unroll
              for (int k = i - kFree; k < kLoads; k += kAhead) load_codes(k);
            }
            const float scale = power(sp[i]);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const bf16x8_t x = widen(hp[i], k, scale);
#pragma unroll
              for (int j = 0; j < TQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wide[k][j], x, acc[i][j], 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < TP; ++i) {
          if (i + kAhead < TP) read_p(i + kAhead);
          if (i >= TP - kTail) continue;
#pragma unroll
          for (int j = 0; j < TQ; ++j) multiply(i, j);
          __builtin_amdgcn_sched_barrier(0);      // or all rows are read at once, into registers that there are not
        }
        __builtin_amdgcn_sched_barrier(0);
        step_barrier();
        if (on) next_step(last ? next.block : block + 1);
        load_scales();
        __builtin_amdgcn_sched_barrier(0);
        // the last rows, column by column, and the next step's fragments in the place of those
        // that are not needed any more (with no next step they are not used)
        static_assert(kTail + kAhead <= TP, "row 0 is read while the last rows are multiplied");
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_p(i);
#pragma unroll
        for (int j = 0; j < TQ; ++j) {
#pragma unroll
          for (int i = TP - kTail; i < TP; ++i) multiply(i, j);
          read_q(j);
#pragma unroll
          for (int i = j; i < kLoads; i += TQ) load_codes(i);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      buffer ^= 1;
      if (last) ready = on;
    }

    // the places in out are computed here, not kept in registers through the loops above
    int64_t width = kGrad ? a.H : a.N;
    int row = wp * TP * 16 + lrow, col = wq * TQ * 16 + quarter * 4 * kPair;
    asm volatile("" : "+s"(width), "+v"(row), "+v"(col));
    typedef raw vec __attribute__((ext_vector_type(4 * kPair)));
    typedef vec any __attribute__((aligned(alignof(raw))));
    raw* to = static_cast<raw*>(a.out) + (t.row + row) * width + t.col + col;
    auto values = [&](int i, int j) {
      vec v;
#pragma unroll
      for (int h = 0; h < kPair; ++h)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[h * 4 + k] = O::from_f(acc[i][j + h][k]);
      return v;
    };
    // a result that the memory-side cache does not hold passes the caches by (884,736 rows of
    // 1,024 by 1,024: 1,171 -> 1,118 us)
    const bool past = (kGrad ? (int64_t)a.E * a.N : a.rows) * width * (int64_t)sizeof(raw) > kMemorySideCache;
    if (t.np == BP && t.nq == BQ) {
#pragma unroll
      for (int i = 0; i < TP; ++i) {
#pragma unroll
        for (int j = 0; j < TQ; j += kPair) {
          if constexpr (TQ % (2 * kPair) == 0) {
            if (j % (2 * kPair) != 0) continue;
            // a store of 8 whole lines of 128 bytes instead of 16 halves: lanes of rows 8 apart
            // exchange halves (884,736 rows of 1,024 by 1,024: 1,179 -> 1,168 us before they passed
            // the caches by; binary32, 20,012 rows of 1,001 by 777, 69 -> 65)
            const int4v x = __builtin_bit_cast(int4v, values(i, j)), y = __builtin_bit_cast(int4v, values(i, j + kPair));
            int4v up, down;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              up[k] = __builtin_amdgcn_update_dpp(x[k], y[k], 0x128, 0xF, 0xC, false);
              down[k] = __builtin_amdgcn_update_dpp(y[k], x[k], 0x128, 0xF, 0x3, false);
            }
            raw* const at = to + j * 16 + ((lane & 8) ? 16 * kPair - 8 * width : 0);
            if (BP == 256 && past) {
              asm volatile("" ::: "memory");      // or the compiler makes one of both branches, without the hint
              __builtin_nontemporal_store(__builtin_bit_cast(vec, up), reinterpret_cast<any*>(at));
              __builtin_nontemporal_store(__builtin_bit_cast(vec, down), reinterpret_cast<any*>(at + 8 * width));
              asm volatile("" ::: "memory");
            } else {
              *reinterpret_cast<any*>(at) = __builtin_bit_cast(vec, up);
              *reinterpret_cast<any*>(at + 8 * width) = __builtin_bit_cast(vec, down);
            }
          } else {
            *reinterpret_cast<any*>(to + j * 16) = values(i, j);
          }
        }
        to += 16 * width;
      }
    } else {
      const int left = t.nq - col;
#pragma unroll
      for (int i = 0; i < TP; ++i) {
        if (row + i * 16 < t.np) {
#pragma unroll
          for (int j = 0; j < TQ; j += kPair) {
            const vec v = values(i, j);
            if (left >= j * 16 + 4 * kPair) {
              *reinterpret_cast<any*>(to + j * 16) = v;
            } else {
#pragma unroll
              for (int k = 0; k < 4 * kPair - 1; ++k)
                if (left > j * 16 + k) to[j * 16 + k] = v[k];
            }
          }
        }
        to += 16 * width;
      }
    }
    if (next_id >= tiles) {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the last loads to LDS, before it is another block's
      return;
    }
    if (t.block == t.end) {
      next = tile_of(next_id);
      ready = false;
    }
    id = next_id;
    t = next;
  }
}

template <int BP, int BQ, int WP, int WQ, bool kGrad, bool kWide>
eqb_status launch_form(const ProductArgs& a, int per_cu, hipStream_t s) {
  const int64_t q_tiles = ((kGrad ? a.H : a.N) + BQ - 1) / BQ;
  const int64_t p_tiles = kGrad ? (int64_t)a.E * ((a.N + BP - 1) / BP) : a.rows / BP + (a.rows < a.E ? a.rows : a.E);
  int64_t grid = (int64_t)num_cus() * per_cu;
  if (p_tiles * q_tiles > INT32_MAX - grid) return EQB_ERR_UNSUPPORTED;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < grid) grid = cap;
  if (p_tiles * q_tiles < grid) grid = p_tiles * q_tiles;
  const uint32_t blocks = (uint32_t)grid, threads = 64 * WP * WQ;
  if constexpr (kWide) product_kernel<BP, BQ, WP, WQ, kGrad, EQB_DTYPE_F32><<<blocks, threads, 0, s>>>(a);
  else if (a.dtype == EQB_DTYPE_BF16) product_kernel<BP, BQ, WP, WQ, kGrad, EQB_DTYPE_BF16><<<blocks, threads, 0, s>>>(a);
  else product_kernel<BP, BQ, WP, WQ, kGrad, EQB_DTYPE_F16><<<blocks, threads, 0, s>>>(a);
  return launch_status();
}

// Tiles of 64 x 64 (four blocks on a compute unit), 128 x 128 (two) and 256 x 256 (one), all times in us, results bf16 where nothing is said:
//   few rows an expert, up to 64 on average: 64 rows of 2,048 to 2,048 columns, E = 256, 38.5 with 64,
//   39.6 with 128, 54 with 256; one row 9.9, 13.0, 25; 4,096 rows of 1,024, E = 64, 21.7, 24.1, 23.8;
//   but 4,096 rows of 1,024, E = 8, 16.7, 14.7, 20.8.
//   weight gradients of up to two tiles of 128 a compute unit: 16 of 512 x 256, 15.2, 18.4, 40; and the more
//   where experts are uneven, since a large one's tiles are as many more steps: with the largest of 6 times the
//   mean 128 of 128 x 140 over 256,879 rows 77, 124, 262 (binary32), with 4.7 times 64 of 256 x 512 over 100,362
//   84, 104, 170; but 8 even ones of 1,024 x 1,024 20.2, 17.0, 23.4, 16 with 2.3 times 212, 168, 240.
//   256 once two of its tiles come on a compute unit and what they reach over the edges costs no more
//   than an eighth: 98,304 rows of 2,048 to 2,048, E = 64, 454 against 561 with 128; 196,608 of 1,024
//   to 1,024, E = 256, 304, 352; 24,576 rows of 2,048 160 both; but 80,000 of 500 to 300, E = 32,
//   37.6, 30.8; gradients 64 of 2,048 x 2,048 over 98,304 rows 583, 794; 32 of 777 x 1,001 59, 55.
//   binary32: 93,389 rows of 2,048 to 2,048, E = 64, 814, 907; the gradients 937, 1,131; over 23,347 rows
//   319, 460; but 32 of 777 x 1,001 74, 62.
template <bool kGrad>
eqb_status launch_product(const ProductArgs& a, hipStream_t s) {
  const int64_t cus = num_cus(), E = a.E, most = a.rows < E ? a.rows : E;
  const int64_t p = kGrad ? a.N : a.rows, q = kGrad ? a.H : a.N;
  auto up = [](int64_t n, int64_t to) { return (n + to - 1) / to; };
  // an expert's rows end in the middle of a tile
  auto tiles = [&](int64_t side) { return (kGrad ? E * up(p, side) : p / side + most / 2) * up(q, side); };
  const bool small = kGrad ? tiles(128) <= 2 * cus : a.rows <= 64 * E;
  const bool large = tiles(256) >= 2 * cus && 4 * tiles(256) * 8 <= tiles(128) * 9;
  if (a.dtype == EQB_DTYPE_F32) {
    if (small) return launch_form<64, 64, 2, 2, kGrad, true>(a, 4, s);
    if (large) return launch_form<256, 256, 2, 4, kGrad, true>(a, 1, s);
    return launch_form<128, 128, 2, 2, kGrad, true>(a, 2, s);
  }
  if (small) return launch_form<64, 64, 2, 2, kGrad, false>(a, 4, s);
  if (large) return launch_form<256, 256, 2, 4, kGrad, false>(a, 1, s);
  return launch_form<128, 128, 2, 2, kGrad, false>(a, 2, s);
}

}  // namespace

eqb_status launch_experts_product(const ProductArgs& a, hipStream_t s) { return launch_product<false>(a, s); }
eqb_status launch_experts_grad_weight(const ProductArgs& a, hipStream_t s) { return launch_product<true>(a, s); }

}  // namespace eqb
