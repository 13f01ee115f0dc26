// experts.hip - rows between the tokens' order and the experts' (arXiv 2609.28053,
// Sec. 2, Eq. 1: y_t = sum over e in I_t of s_{t,e} FFN_e(x_t)): the sorted order of
// the routed pairs, the gather of the tokens' rows, the weighted sum of the experts'
// rows, and the gradients of both.
#include "eqb_internal.hpp"

namespace eqb {

// ------------------------------------------------------------ the order --
// A counting sort by expert that keeps the pairs' order.  Every block owns a
// contiguous range of pairs.  dispatch_count_kernel stores its counts per expert;
// dispatch_rank_kernel sums the counts of the blocks before it and of all blocks
// (which gives the experts' offsets), counts its waves' shares, and then every wave
// walks its share 64 pairs at a time: a lane's place is its expert's running count
// plus the number of lower lanes with the same expert, found with one ballot per bit
// of the expert's index.
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

__global__ __launch_bounds__(kPlanThreads) void dispatch_count_kernel(const int32_t* __restrict__ idx, uint32_t N,
                                                                      int E, uint32_t per_block,
                                                                      int32_t* __restrict__ counts) {
  __shared__ int32_t sh[kNBins];
  if (threadIdx.x < kNBins) sh[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t begin = blockIdx.x * per_block, end = begin + per_block < N ? begin + per_block : N;
  for (uint32_t i = begin + threadIdx.x; i < end; i += kPlanThreads) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicAdd(&sh[e], 1);
  }
  __syncthreads();
  if ((int)threadIdx.x < E) counts[blockIdx.x * E + threadIdx.x] = sh[threadIdx.x];
}

// lanes of the wave with the same expert (valid lanes only)
__device__ __forceinline__ uint64_t same_expert(int e, bool valid, int bits) {
  uint64_t same = __ballot(valid);
  for (int b = 0; b < bits; ++b) {
    const bool on = (e >> b) & 1;
    const uint64_t m = __ballot(on);
    same &= on ? m : ~m;
  }
  return same;
}

__global__ __launch_bounds__(kPlanThreads) void dispatch_rank_kernel(const int32_t* __restrict__ idx, uint32_t N,
                                                                     int E, int bits, uint32_t per_block,
                                                                     const int32_t* __restrict__ counts,
                                                                     int32_t* __restrict__ offsets,
                                                                     int32_t* __restrict__ slot) {
  __shared__ int32_t sh_cnt[kPlanWaves][kNBins];
  __shared__ int32_t sh_before[kNBins], sh_total[kNBins];
  __shared__ int32_t sh_scan[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int i = tid; i < kPlanWaves * kNBins; i += kPlanThreads) (&sh_cnt[0][0])[i] = 0;
  if (tid < kNBins) sh_before[tid] = sh_total[tid] = 0;
  __syncthreads();
  const uint32_t begin = blockIdx.x * per_block, end = begin + per_block < N ? begin + per_block : N;
  // the waves' shares, in whole groups of 64 pairs
  const uint32_t groups = (end - begin + 63) / 64, share = (groups + kPlanWaves - 1) / kPlanWaves * 64;
  const uint32_t w0 = begin + wave * share, w1 = w0 + share < end ? w0 + share : end;
  for (uint32_t i = w0 + lane; i < w1; i += 64) {
    const int e = idx[i];
    if (e >= 0 && e < E) atomicAdd(&sh_cnt[wave][e], 1);
  }
  if (counts) {
    // a row of counts by E/4 threads, 16 bytes each and four rows in flight: with one
    // count a load their latency was most of the kernel's time
    const int q = tid % (E / 4), step = 4 * kPlanThreads / E;
    int before[4] = {}, total[4] = {};
    for (int b0 = tid / (E / 4); b0 < (int)gridDim.x; b0 += 4 * step) {
      int4 c[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int b = b0 + j * step;
        c[j] = b < (int)gridDim.x ? *reinterpret_cast<const int4*>(counts + b * E + 4 * q) : make_int4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int in = b0 + j * step < (int)blockIdx.x ? -1 : 0;
        const int v[4] = {c[j].x, c[j].y, c[j].z, c[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          total[i] += v[i];
          before[i] += v[i] & in;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (before[i]) atomicAdd(&sh_before[4 * q + i], before[i]);
      if (total[i]) atomicAdd(&sh_total[4 * q + i], total[i]);
    }
  }
  __syncthreads();
  if (!counts && tid < E) {       // one block: its own counts are all
    int total = 0;
    for (int w = 0; w < kPlanWaves; ++w) total += sh_cnt[w][tid];
    sh_total[tid] = total;
  }
  __syncthreads();
  // exclusive scan of the totals: within each of the four first waves, then over them
  int incl = tid < E ? sh_total[tid] : 0;
  const int own = incl;
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(incl, d);
    if (lane >= d) incl += y;
  }
  if (lane == 63 && wave < 4) sh_scan[wave] = incl;
  __syncthreads();
  if (tid < E) {
    for (int w = 0; w < wave; ++w) incl += sh_scan[w];
    int at = incl - own;
    if (blockIdx.x == 0) offsets[tid] = at;
    if (blockIdx.x == 0 && tid == E - 1) offsets[E] = incl;
    at += sh_before[tid];
    for (int w = 0; w < kPlanWaves; ++w) {
      const int c = sh_cnt[w][tid];
      sh_cnt[w][tid] = at;
      at += c;
    }
  }
  __syncthreads();
  for (uint32_t i0 = w0; i0 < w1; i0 += 64) {
    const uint32_t i = i0 + lane;
    const int e = i < w1 ? idx[i] : -1;
    const bool valid = e >= 0 && e < E;
    const uint64_t same = same_expert(e, valid, bits);
    const int lower = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
    int at = -1;
    if (valid) at = sh_cnt[wave][e] + lower;
    lds_wave_sync();
    if (valid && lower == 0) sh_cnt[wave][e] = at + __popcll(same);
    lds_wave_sync();
    if (i < w1) slot[i] = at;
  }
}

__global__ void zero_offsets_kernel(int32_t* __restrict__ offsets, int n) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) offsets[i] = 0;
}

uint32_t dispatch_plan_blocks(int64_t N) {
  const int64_t want = (N + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  return (uint32_t)(want < 1 ? 1 : want < kPlanMaxBlocks ? want : kPlanMaxBlocks);
}

eqb_status launch_dispatch_plan(const int32_t* idx, int64_t N, int E, int32_t* offsets, int32_t* slot, int32_t* counts,
                                hipStream_t s) {
  if (N == 0) {
    zero_offsets_kernel<<<2, 256, 0, s>>>(offsets, E + 1);
    return launch_status();
  }
  const uint32_t want = dispatch_plan_blocks(N);
  const uint32_t per_block = (uint32_t)((N + want - 1) / want);
  const uint32_t blocks = (uint32_t)((N + per_block - 1) / per_block);
  if (blocks > 1) dispatch_count_kernel<<<blocks, kPlanThreads, 0, s>>>(idx, (uint32_t)N, E, per_block, counts);
  dispatch_rank_kernel<<<blocks, kPlanThreads, 0, s>>>(idx, (uint32_t)N, E, __builtin_ctz(E), per_block,
                                                       blocks > 1 ? counts : nullptr, offsets, slot);
  return launch_status();
}

// ------------------------------------------------------------- the rows --
// Rows move in pieces of 16 bytes at the alignment of one element (gfx950's global
// loads and stores take any address).  All of it is bound by memory.
template <class T>
struct Piece {
  static constexpr int n = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef vec any __attribute__((aligned(alignof(T))));
};

struct Bf16 {
  typedef uint16_t raw;
  static __device__ __forceinline__ float to_f(raw x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ void put(Piece<raw>::vec* v, int i, float a, float b) {
    const uint32_t w = bf16x2_bits(a, b);
    (*v)[i] = (raw)w;
    (*v)[i + 1] = (raw)(w >> 16);
  }
};
struct F16 {
  typedef _Float16 raw;
  static __device__ __forceinline__ float to_f(raw x) { return (float)x; }
  static __device__ __forceinline__ void put(Piece<raw>::vec* v, int i, float a, float b) {
    (*v)[i] = (raw)a;
    (*v)[i + 1] = (raw)b;
  }
};
struct F32 {
  typedef float raw;
  static __device__ __forceinline__ float to_f(raw x) { return x; }
  static __device__ __forceinline__ void put(Piece<raw>::vec* v, int i, float a, float b) {
    (*v)[i] = a;
    (*v)[i + 1] = b;
  }
};

// L lanes work on a token, with NP pieces of its row each in registers: a row of up to
// L * NP pieces in one go, longer ones by segments.  The K rows on the experts' side are
// taken kBatch at a time, so that kBatch * NP loads are in flight before the first is used.
constexpr int kRowThreads = 256;

template <class D, int L, int NP, bool kStream>
struct RowPart {
  typedef typename D::raw raw;
  typedef typename Piece<raw>::vec vec;
  typedef typename Piece<raw>::any any;
  static constexpr int V = Piece<raw>::n;
  int64_t c[NP];      // first element of each piece
  int skip[NP];       // its leading elements that other pieces hold too
  // A row's last piece ends with the row, over part of the one before it, and lanes past
  // the row hold its last piece once more (all with the same values, so that stores may
  // overlap): a row of 333 f16 elements took 347 us to combine (100,000 tokens, K = 8) with
  // its last elements one by one, and takes 169.  Only rows shorter than a piece go by
  // elements, in the first lane.
  __device__ __forceinline__ RowPart(int64_t seg, int H) {
    const int l = threadIdx.x % L;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      c[i] = ((seg * NP + i) * L + l) * V;
      const int64_t over = c[i] + V - H;
      skip[i] = over <= 0 || H < V ? (c[i] < H ? 0 : V) : over < V ? (int)over : V;
      if (over > 0 && H >= V) c[i] = H - V;
    }
  }
  template <bool kNt>
  __device__ __forceinline__ void load(const raw* row, int H, vec (&v)[NP]) const {
    if (H >= V) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const any* at = reinterpret_cast<const any*>(row + c[i]);
        v[i] = kNt && kStream ? __builtin_nontemporal_load(at) : *at;
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        v[i] = vec{};
        if (skip[i] < V) {
#pragma unroll
          for (int j = 0; j < V - 1; ++j)
            if (j < H) v[i][j] = row[j];
        }
      }
    }
  }
  __device__ __forceinline__ void store(raw* row, int H, const vec (&v)[NP]) const {
    if (H >= V) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        any* at = reinterpret_cast<any*>(row + c[i]);
        if (kStream) __builtin_nontemporal_store((any)v[i], at);
        else *at = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (skip[i] < V) {
#pragma unroll
          for (int j = 0; j < V - 1; ++j)
            if (j < H) row[j] = v[i][j];
        }
      }
    }
  }
};

// Tokens: t, t + stride, ...  A whole wave's token is known to be the same in its lanes, so
// that its slots and weights are scalar loads.  near: blocks b, b + 8, ... run on one XCD
// and get neighbouring tokens, whose short rows share lines of its L2.
template <int L>
__device__ __forceinline__ int64_t first_token(bool near) {
  const int group = L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : (int)threadIdx.x / L;
  const uint32_t per = gridDim.y / 8;
  uint32_t y = blockIdx.y;
  if (near && y < per * 8) y = (y % 8) * per + y / 8;
  return (int64_t)y * (kRowThreads / L) + group;
}
template <int L>
__device__ __forceinline__ int64_t token_stride() { return (int64_t)gridDim.y * (kRowThreads / L); }

template <class D, int L, int NP, bool kStream>
__global__ __launch_bounds__(kRowThreads) void dispatch_kernel(const RowArgs a, int segments) {
  typedef typename D::raw raw;
  const raw* x = static_cast<const raw*>(a.tokens);
  raw* out = static_cast<raw*>(a.out);
  for (int64_t seg = blockIdx.x; seg < segments; seg += gridDim.x) {
    const RowPart<D, L, NP, kStream> part(seg, a.H);
    for (int64_t t = first_token<L>(a.near); t < a.T; t += token_stride<L>()) {
      typename RowPart<D, L, NP, kStream>::vec v[NP];
      part.template load<false>(x + t * a.H, a.H, v);
      for (int k = 0; k < a.K; ++k) {
        const int64_t r = a.slot[t * a.K + k];
        if (r >= 0 && r < a.rows) part.store(out + r * a.H, a.H, v);
      }
    }
  }
}

template <class D, int L, int NP, bool kStream>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(const RowArgs a, int segments) {
  typedef typename D::raw raw;
  constexpr int V = Piece<raw>::n, kBatch = NP == 2 ? 8 : 4;
  const raw* in = static_cast<const raw*>(a.experts);
  raw* y = static_cast<raw*>(a.out);
  for (int64_t seg = blockIdx.x; seg < segments; seg += gridDim.x) {
    const RowPart<D, L, NP, kStream> part(seg, a.H);
    for (int64_t t = first_token<L>(a.near); t < a.T; t += token_stride<L>()) {
      float acc[NP][V] = {};
      for (int k0 = 0; k0 < a.K; k0 += kBatch) {
        int64_t r[kBatch];
        float w[kBatch];
        typename RowPart<D, L, NP, kStream>::vec v[kBatch][NP];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
          const int64_t at = t * a.K + k0 + j;
          r[j] = k0 + j < a.K ? a.slot[at] : -1;
          w[j] = k0 + j < a.K && a.weight ? a.weight[at] : 1.0f;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (r[j] >= 0 && r[j] < a.rows) part.template load<true>(in + r[j] * a.H, a.H, v[j]);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (r[j] >= 0 && r[j] < a.rows) {
#pragma unroll
            for (int i = 0; i < NP; ++i)
#pragma unroll
              for (int e = 0; e < V; ++e) acc[i][e] += w[j] * D::to_f(v[j][i][e]);
          }
      }
      typename RowPart<D, L, NP, kStream>::vec o[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i)
#pragma unroll
        for (int e = 0; e < V; e += 2) D::put(&o[i], e, acc[i][e], acc[i][e + 1]);
      part.store(y + t * a.H, a.H, o);
    }
  }
}

// A token's L lanes go over all its segments: the products of grad_y's row with each of
// its experts' rows are theirs alone.  With one segment grad_y's row stays in registers.
template <class D, int L, int NP, bool kStream>
__global__ __launch_bounds__(kRowThreads) void combine_backward_kernel(const RowArgs a, int segments) {
  typedef typename D::raw raw;
  typedef RowPart<D, L, NP, kStream> Part;
  constexpr int V = Piece<raw>::n, kBatch = 4;
  __shared__ float sh_dot[kBatch][4];
  const raw* gy = static_cast<const raw*>(a.tokens);
  const raw* in = static_cast<const raw*>(a.experts);
  raw* gin = static_cast<raw*>(a.out);
  const bool whole = a.H % (L * NP * V) == 0;
  for (int64_t t = first_token<L>(a.near); t < a.T; t += token_stride<L>()) {
    typename Part::vec g[NP];
    if (segments == 1) Part(0, a.H).template load<false>(gy + t * a.H, a.H, g);
    for (int k0 = 0; k0 < a.K; k0 += kBatch) {
      int64_t r[kBatch];
      float w[kBatch], dot[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int64_t at = t * a.K + k0 + j;
        r[j] = k0 + j < a.K ? a.slot[at] : -1;
        w[j] = k0 + j < a.K ? a.weight[at] : 0.0f;
        dot[j] = 0.0f;
      }
      for (int seg = 0; seg < segments; ++seg) {
        const Part part(seg, a.H);
        typename Part::vec v[kBatch][NP];
        if (segments > 1) part.template load<false>(gy + t * a.H, a.H, g);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (r[j] >= 0 && r[j] < a.rows) part.template load<true>(in + r[j] * a.H, a.H, v[j]);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (r[j] >= 0 && r[j] < a.rows) {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              float y[V];
#pragma unroll
              for (int e = 0; e < V; e += 2) {
                const float x0 = D::to_f(g[i][e]), x1 = D::to_f(g[i][e + 1]);
                y[e] = x0 * D::to_f(v[j][i][e]);
                y[e + 1] = x1 * D::to_f(v[j][i][e + 1]);
                D::put(&v[j][i], e, w[j] * x0, w[j] * x1);
              }
              if (!whole) {
                int skip = part.skip[i];      // compared here, not in V * NP masks kept from before the loops
                asm volatile("" : "+v"(skip));
#pragma unroll
                for (int e = 0; e < V; ++e) y[e] = e >= skip ? y[e] : 0.0f;
              }
              // a piece's products in pairs: V times fewer roundings of the running sum
#pragma unroll
              for (int n = V / 2; n > 0; n /= 2)
#pragma unroll
                for (int e = 0; e < n; ++e) y[e] += y[e + n];
              dot[j] += y[0];
            }
            part.store(gin + r[j] * a.H, a.H, v[j]);
          }
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) dot[j] = group_sum<(L < 64 ? L : 64)>(dot[j]);
      if (L > 64) {       // over the block's waves, in their order
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
          if (threadIdx.x % 64 == 0) sh_dot[j][threadIdx.x / 64] = dot[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kBatch; ++j) dot[j] = (sh_dot[j][0] + sh_dot[j][1]) + (sh_dot[j][2] + sh_dot[j][3]);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (k0 + j < a.K && threadIdx.x % L == 0) a.grad_weight[t * a.K + k0 + j] = dot[j];
    }
  }
}

// What differs between the calls when they choose their form: whether a row's segments go
// to waves of their own, and whether the call writes the experts' rows.
#define EQB_ROW_CALL(name, splits, writes)                                              \
  struct name##_call {                                                                  \
    static constexpr bool split = splits, writes_rows = writes;                         \
    template <class D, int L, int NP, bool kStream>                                     \
    static void launch(dim3 grid, const RowArgs& a, int segments, hipStream_t s) {      \
      name##_kernel<D, L, NP, kStream><<<grid, kRowThreads, 0, s>>>(a, segments);       \
    }                                                                                   \
  };
EQB_ROW_CALL(dispatch, true, true)
EQB_ROW_CALL(combine, true, false)
EQB_ROW_CALL(combine_backward, false, true)
#undef EQB_ROW_CALL

template <class Call, class D, int L, int NP, bool kStream>
static void launch_form(const RowArgs& a, hipStream_t s) {
  const int64_t per = (int64_t)L * NP * Piece<typename D::raw>::n;
  const int64_t segments = (a.H + per - 1) / per;
  int64_t y = (a.T + kRowThreads / L - 1) / (kRowThreads / L), most = 65535;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < most) most = cap;
  if (y > most) y = most;
  const int64_t x = Call::split ? (segments < 1024 ? segments : 1024) : 1;
  Call::template launch<D, L, NP, kStream>(dim3((uint32_t)x, (uint32_t)y), a, (int)segments, s);
}

// Lanes and pieces for a row, by the number of its pieces: the fewest lanes that hold a row
// of up to 64 pieces, whole waves with 2 or 4 pieces each beyond.  Few tokens: split over
// more waves.  8 to 512 tokens of 2,048 bf16, K = 8: combine 5.2 to 6.1 us whole, 5.1 to 5.5
// split, dispatch 4.2 to 7.1 and 4.2 to 6.3; of 7,168, 8 to 128 tokens: 5.8 to 6.2 and 5.1 to
// 5.5, 5.0 to 7.2 and 4.3 to 6.0.  Past 4,096 waves of 64 pieces it costs: 1,000 tokens of
// 4,096, combine 13.3 -> 17.3, 8,000 of 1,024 25.9 -> 34.0; dispatch within 3% either way.
// In the backward pass over a block's waves: one token of 8,192 bf16, K = 8, 42 us in a wave,
// 12.9 in a block; 64 to 1,000 tokens of 1,024 to 7,168, K = 2 and 8, a wave takes 0.85 (1,000
// of 1,024) to 1.9 times as long as a block (64 of 7,168), 2,000 tokens 0.78 to 1.05.
// Calls on experts' rows of kStreamBytes (the memory-side cache) and more pass by it: loads
// of the experts' rows and all stores are non-temporal, in calls that write experts' rows
// only where those are whole lines of 128 bytes; dispatch then splits rows over waves by the
// piece.  16,384 tokens of 2,048 bf16, K = 6: combine 95.9 -> 80 us, dispatch 91.7 -> 78,
// backward 183 -> 159; but 147,456 rows of 100 bf16: dispatch 40 -> 104, and 5,003 rows of
// 1,001 f32 (in the cache): combine 16.5 -> 21.6.
// Rows under kNearBytes: neighbouring tokens on one XCD.  147,456 tokens, K = 6, rows of 32
// bytes: combine 17.6 -> 11.7 us, of 200: 47.4 -> 38.2; of 4,096: 92 -> 96 (not taken).
// At 147,456 tokens of 1,024 bf16, K = 6: dispatch 402 us (5.3 TB/s), combine 351 (6.0),
// backward 755 (5.2).
constexpr int64_t kStreamBytes = (int64_t)256 << 20;
constexpr int64_t kNearBytes = 512;
constexpr int64_t kRowWaves = 4096;
constexpr int64_t kBlockTokens = 1024;

template <class Call, class D>
static void launch_rows(RowArgs a, hipStream_t s) {
  const int64_t pieces = ((int64_t)a.H + Piece<typename D::raw>::n - 1) / Piece<typename D::raw>::n;
  const int64_t bytes = (int64_t)a.H * sizeof(typename D::raw);
  const bool stream = a.T * a.K * bytes >= kStreamBytes && (!Call::writes_rows || bytes % 128 == 0);
  const bool few = a.T * pieces <= 64 * kRowWaves;
  a.near = bytes < kNearBytes;
  if (pieces <= 4) return launch_form<Call, D, 4, 1, false>(a, s);
  if (pieces <= 8) return launch_form<Call, D, 8, 1, false>(a, s);
  if (pieces <= 16) return launch_form<Call, D, 16, 1, false>(a, s);
  if (pieces <= 32) return launch_form<Call, D, 32, 1, false>(a, s);
  if (pieces <= 64) return launch_form<Call, D, 64, 1, false>(a, s);
  if constexpr (Call::split) {
    if (few) return launch_form<Call, D, 64, 1, false>(a, s);
    if constexpr (Call::writes_rows) {
      if (stream) return launch_form<Call, D, 64, 1, true>(a, s);
    }
  } else {
    if (few || a.T <= kBlockTokens) return launch_form<Call, D, 256, 1, false>(a, s);
  }
  if constexpr (!(Call::split && Call::writes_rows)) {
    if (stream) {
      if (pieces <= 128) return launch_form<Call, D, 64, 2, true>(a, s);
      return launch_form<Call, D, 64, 4, true>(a, s);
    }
  }
  if (pieces <= 128) return launch_form<Call, D, 64, 2, false>(a, s);
  return launch_form<Call, D, 64, 4, false>(a, s);
}

template <class Call>
static eqb_status launch_call(const RowArgs& a, hipStream_t s) {
  if (a.dtype == EQB_DTYPE_BF16) launch_rows<Call, Bf16>(a, s);
  else if (a.dtype == EQB_DTYPE_F16) launch_rows<Call, F16>(a, s);
  else launch_rows<Call, F32>(a, s);
  return launch_status();
}

eqb_status launch_dispatch(const RowArgs& a, hipStream_t s) { return launch_call<dispatch_call>(a, s); }
eqb_status launch_combine(const RowArgs& a, hipStream_t s) { return launch_call<combine_call>(a, s); }
eqb_status launch_combine_backward(const RowArgs& a, hipStream_t s) { return launch_call<combine_backward_call>(a, s); }

}  // namespace eqb
