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
    // eight loads in flight: one at a time their latency was 15 of the kernel's 20 us at
    // 885,000 pairs
    int before = 0, total = 0;
    const int e = tid % E, step = kPlanThreads / E;
    for (int b0 = tid / E; b0 < (int)gridDim.x; b0 += 8 * step) {
      int c[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int b = b0 + j * step;
        c[j] = b < (int)gridDim.x ? counts[b * E + e] : 0;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        total += c[j];
        before += b0 + j * step < (int)blockIdx.x ? c[j] : 0;
      }
    }
    atomicAdd(&sh_before[e], before);
    atomicAdd(&sh_total[e], total);
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
// loads and stores take any address), a row's last elements one at a time.
template <class T>
struct Piece {
  static constexpr int n = 16 / sizeof(T);
  typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
  typedef vec any __attribute__((aligned(alignof(T))));
};

struct Bf16 {
  typedef uint16_t raw;
  static __device__ __forceinline__ float to_f(raw x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ raw of_f(float x) { return (raw)bf16x2_bits(x, 0.0f); }
};
struct F16 {
  typedef _Float16 raw;
  static __device__ __forceinline__ float to_f(raw x) { return (float)x; }
  static __device__ __forceinline__ raw of_f(float x) { return (raw)x; }
};
struct F32 {
  typedef float raw;
  static __device__ __forceinline__ float to_f(raw x) { return x; }
  static __device__ __forceinline__ raw of_f(float x) { return x; }
};

constexpr int kRowThreads = 256;

// A wave's work: one token and a piece of its row of 64 * 16 bytes.
struct RowItem {
  int64_t t;
  int64_t c;      // first element of this lane's piece
  int n;          // its elements, 0 .. Piece::n
};
template <class D>
__device__ __forceinline__ RowItem row_item(int64_t item, int H, int segments) {
  constexpr int V = Piece<typename D::raw>::n;
  RowItem it;
  it.t = item / segments;
  it.c = ((item - it.t * segments) * 64 + (threadIdx.x & 63)) * V;
  const int64_t left = H - it.c;
  it.n = left <= 0 ? 0 : left < V ? (int)left : V;
  return it;
}
// the wave's number and the number of waves: item, item + stride, ...
__device__ __forceinline__ int64_t first_item() { return (int64_t)blockIdx.x * (kRowThreads / 64) + (threadIdx.x >> 6); }
__device__ __forceinline__ int64_t item_stride() { return (int64_t)gridDim.x * (kRowThreads / 64); }
template <class D>
__device__ __forceinline__ typename Piece<typename D::raw>::vec load_piece(const typename D::raw* p, int n) {
  typename Piece<typename D::raw>::vec v = {};
  if (n == Piece<typename D::raw>::n) return *reinterpret_cast<const typename Piece<typename D::raw>::any*>(p);
#pragma unroll
  for (int i = 0; i < Piece<typename D::raw>::n; ++i)
    if (i < n) v[i] = p[i];
  return v;
}
template <class D>
__device__ __forceinline__ void store_piece(typename D::raw* p, typename Piece<typename D::raw>::vec v, int n) {
  if (n == Piece<typename D::raw>::n) {
    *reinterpret_cast<typename Piece<typename D::raw>::any*>(p) = v;
    return;
  }
#pragma unroll
  for (int i = 0; i < Piece<typename D::raw>::n; ++i)
    if (i < n) p[i] = v[i];
}

template <class D>
__global__ __launch_bounds__(kRowThreads) void dispatch_kernel(const typename D::raw* __restrict__ x,
                                                               const int32_t* __restrict__ slot, int64_t T, int K,
                                                               int64_t rows, int H, int segments,
                                                               typename D::raw* __restrict__ out) {
  for (int64_t item = first_item(); item < T * segments; item += item_stride()) {
    const RowItem it = row_item<D>(item, H, segments);
    const auto v = load_piece<D>(x + it.t * H + it.c, it.n);
    for (int k = 0; k < K; ++k) {
      const int64_t r = slot[it.t * K + k];
      if (r >= 0 && r < rows) store_piece<D>(out + r * H + it.c, v, it.n);
    }
  }
}

template <class D>
__global__ __launch_bounds__(kRowThreads) void combine_kernel(const typename D::raw* __restrict__ in,
                                                              const int32_t* __restrict__ slot,
                                                              const float* __restrict__ weight, int64_t T, int K,
                                                              int64_t rows, int H, int segments,
                                                              typename D::raw* __restrict__ y) {
  constexpr int V = Piece<typename D::raw>::n;
  for (int64_t item = first_item(); item < T * segments; item += item_stride()) {
    const RowItem it = row_item<D>(item, H, segments);
    float acc[V] = {};
    for (int k = 0; k < K; ++k) {
      const int64_t r = slot[it.t * K + k];
      if (r < 0 || r >= rows) continue;
      const float w = weight ? weight[it.t * K + k] : 1.0f;
      const auto v = load_piece<D>(in + r * H + it.c, it.n);
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += w * D::to_f(v[i]);
    }
    typename Piece<typename D::raw>::vec o;
#pragma unroll
    for (int i = 0; i < V; ++i) o[i] = D::of_f(acc[i]);
    store_piece<D>(y + it.t * H + it.c, o, it.n);
  }
}

// One wave per token: grad_y's row against each of its experts' rows.
template <class D>
__global__ __launch_bounds__(kRowThreads) void combine_backward_kernel(
    const typename D::raw* __restrict__ gy, const typename D::raw* __restrict__ in, const int32_t* __restrict__ slot,
    const float* __restrict__ weight, int64_t T, int K, int64_t rows, int H, typename D::raw* __restrict__ gin,
    float* __restrict__ gw) {
  constexpr int V = Piece<typename D::raw>::n;
  const int lane = threadIdx.x & 63;
  for (int64_t t = first_item(); t < T; t += item_stride()) {
    for (int k = 0; k < K; ++k) {
      const int64_t r = slot[t * K + k];
      float dot = 0.0f;
      if (r >= 0 && r < rows) {
        const float w = weight[t * K + k];
        for (int64_t c = lane * V; c < H; c += 64 * V) {
          const int n = H - c < V ? (int)(H - c) : V;
          const auto a = load_piece<D>(gy + t * H + c, n);
          const auto b = load_piece<D>(in + r * H + c, n);
          typename Piece<typename D::raw>::vec o;
#pragma unroll
          for (int i = 0; i < V; ++i) {
            dot += D::to_f(a[i]) * D::to_f(b[i]);
            o[i] = D::of_f(w * D::to_f(a[i]));
          }
          store_piece<D>(gin + r * H + c, o, n);
        }
      }
      for (int off = 32; off > 0; off >>= 1) dot += __shfl_xor(dot, off);
      if (lane == 0) gw[t * K + k] = dot;
    }
  }
}

// Blocks for that many waves' items; past 2^20 blocks they walk on by the grid.
static uint32_t row_blocks(int64_t items) {
  const int64_t want = (items + kRowThreads / 64 - 1) / (kRowThreads / 64);
  int64_t most = 1 << 20;
  const int cap = max_blocks_cap();
  if (cap > 0 && cap < most) most = cap;
  return (uint32_t)(want < most ? want : most);
}
template <class D>
static int row_segments(int H) {
  constexpr int per = 64 * Piece<typename D::raw>::n;
  return (int)(((int64_t)H + per - 1) / per);
}

template <class D>
static void launch_dispatch_as(const RowArgs& a, hipStream_t s) {
  typedef typename D::raw R;
  const int seg = row_segments<D>(a.H);
  dispatch_kernel<D><<<row_blocks(a.T * seg), kRowThreads, 0, s>>>(static_cast<const R*>(a.tokens), a.slot, a.T, a.K,
                                                                  a.rows, a.H, seg, static_cast<R*>(a.out));
}
template <class D>
static void launch_combine_as(const RowArgs& a, hipStream_t s) {
  typedef typename D::raw R;
  const int seg = row_segments<D>(a.H);
  combine_kernel<D><<<row_blocks(a.T * seg), kRowThreads, 0, s>>>(static_cast<const R*>(a.experts), a.slot, a.weight,
                                                                 a.T, a.K, a.rows, a.H, seg, static_cast<R*>(a.out));
}
template <class D>
static void launch_combine_backward_as(const RowArgs& a, hipStream_t s) {
  typedef typename D::raw R;
  combine_backward_kernel<D><<<row_blocks(a.T), kRowThreads, 0, s>>>(
      static_cast<const R*>(a.tokens), static_cast<const R*>(a.experts), a.slot, a.weight, a.T, a.K, a.rows, a.H,
      static_cast<R*>(a.out), a.grad_weight);
}

#define EQB_ROW_LAUNCH(name)                                      \
  eqb_status launch_##name(const RowArgs& a, hipStream_t s) {     \
    if (a.dtype == EQB_DTYPE_BF16) launch_##name##_as<Bf16>(a, s); \
    else if (a.dtype == EQB_DTYPE_F16) launch_##name##_as<F16>(a, s); \
    else launch_##name##_as<F32>(a, s);                           \
    return launch_status();                                       \
  }
EQB_ROW_LAUNCH(dispatch)
EQB_ROW_LAUNCH(combine)
EQB_ROW_LAUNCH(combine_backward)
#undef EQB_ROW_LAUNCH

}  // namespace eqb
