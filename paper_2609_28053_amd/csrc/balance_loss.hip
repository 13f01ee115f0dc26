// balance_loss.hip - the auxiliary balance loss (arXiv 2609.28053, Sec. 2, "GShard";
// App. D) with the experts' counts, and its gradient fused with the router backward
// (Sec. 2, Eq. 1) and the load-error injection (Sec. 4).
#include "eqb_internal.hpp"

namespace eqb {

// Sum (maximum) over aligned groups of G lanes, the same in every lane of the group.
template <int G>
__device__ __forceinline__ float group_sum(float x) {
#pragma unroll
  for (int off = 1; off < G; off <<= 1) x += __shfl_xor(x, off);
  return x;
}
template <int G>
__device__ __forceinline__ float group_max(float x) {
#pragma unroll
  for (int off = 1; off < G; off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

constexpr float kLog2e = 1.4426950408889634f;
// Below this sum the sigmoids of a row equal their exponentials to binary32, and may have
// lost digits to underflow: the row's probabilities are then those of a softmax.
constexpr float kTinySum = 0x1p-100f;

// A row's exponentials exp(x - max) over the group's lanes, whole rows of -inf giving 0;
// returns their sum.
template <int G, int N>
__device__ __forceinline__ float softmax_terms(const float (&x)[N], float (&w)[N]) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
  m = group_max<G>(m);
  m = fmaxf(m, -3.0e38f);
  float d = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    w[i] = __builtin_amdgcn_exp2f((x[i] - m) * kLog2e);
    d += w[i];
  }
  return group_sum<G>(d);
}

// ------------------------------------------------------------- the loss --
// G = E/8 lanes hold a row, 8 experts each.  A lane sums the probabilities of its
// experts over its rows in binary32; at the end of a block's piece of a group the block
// adds its lanes' sums, and stores them with its counts.  The block that completes a
// group (by the group's ticket) adds the pieces in their order in binary64, writes the
// group's results and sets the ticket back to 0.  Blocks sit on XCDs with an L2 each:
// pieces pass between them in agent-scope stores and loads, complete (vmcnt) before the
// ticket is drawn.
constexpr int kLossThreads = 1024, kLossWaves = kLossThreads / 64;
constexpr int kLossU = 4;          // rows per lane and step

__device__ __forceinline__ uint64_t pack_piece(float prob, int count) {
  return (uint64_t)__float_as_uint(prob) | ((uint64_t)(uint32_t)count << 32);
}

template <int E, bool kSoftmax>
__global__ __launch_bounds__(kLossThreads) void balance_loss_kernel(
    const uint16_t* __restrict__ z, const int32_t* __restrict__ idx, const uint8_t* __restrict__ valid, int64_t T,
    int K, const PartTable pt, int64_t rows_per_block, double alpha, const BalanceWorkspace ws, int32_t* load,
    int32_t* __restrict__ tokens, float* __restrict__ prob, float* __restrict__ loss) {
  constexpr int G = E / 8, R = 64 / G, ROWS = kLossWaves * R * kLossU;
  __shared__ float sh_sum[kLossWaves][E];
  __shared__ int32_t sh_cnt[E];
  __shared__ int32_t sh_tokens, sh_ticket;
  __shared__ double sh_d[kLossThreads];
  __shared__ int64_t sh_c[kLossThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane % G, rr = lane / G;
  if (blockIdx.x == 0) {           // groups without tokens
    for (int p = 0; p < pt.P; ++p) {
      if (pt.off[p + 1] > pt.off[p]) continue;
      if (tid < E) {
        prob[p * E + tid] = 0.0f;
        if (idx || T == 0) load[p * E + tid] = 0;
      }
      if (tid == 0) {
        tokens[p] = 0;
        loss[p] = 0.0f;
      }
    }
  }
  if (tid < E) sh_cnt[tid] = 0;
  if (tid == 0) sh_tokens = 0;
  int64_t r0, r1;
  block_rows(T, rows_per_block, &r0, &r1);
  int p = 0;
  for (int64_t s0 = r0; s0 < r1;) {
    while (p < pt.P - 1 && pt.off[p + 1] <= s0) ++p;
    const int64_t s1 = pt.off[p + 1] < r1 ? pt.off[p + 1] : r1;
    __syncthreads();
    if (idx) {
      for (int64_t i = s0 * K + tid; i < s1 * K; i += kLossThreads) {
        const int e = idx[i];
        if (e >= 0 && e < E && (!valid || valid[i / K])) atomicAdd(&sh_cnt[e], 1);
      }
    }
    float acc[8] = {};
    int n = 0;
    for (int64_t base = s0; base < s1; base += ROWS) {
      uint4 zw[kLossU];
      bool on[kLossU];
#pragma unroll
      for (int u = 0; u < kLossU; ++u) {
        const int64_t t = base + (u * kLossWaves + wave) * R + rr;
        on[u] = t < s1 && (!valid || valid[t]);
        zw[u] = make_uint4(0, 0, 0, 0);
        if (on[u]) zw[u] = *reinterpret_cast<const uint4*>(z + t * E + 8 * g);
      }
#pragma unroll
      for (int u = 0; u < kLossU; ++u) {
        const float x[8] = {bf16_lo(zw[u].x), bf16_hi(zw[u].x), bf16_lo(zw[u].y), bf16_hi(zw[u].y),
                            bf16_lo(zw[u].z), bf16_hi(zw[u].z), bf16_lo(zw[u].w), bf16_hi(zw[u].w)};
        float w[8], d = 0.0f;
        if (kSoftmax) {
          d = softmax_terms<G>(x, w);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            w[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * -kLog2e));
            d += w[i];
          }
          d = group_sum<G>(d);
          const bool tiny = on[u] && d < kTinySum;
          if (__any(tiny)) {
            float ws_[8];
            const float ds = softmax_terms<G>(x, ws_);
            d = tiny ? ds : d;
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = tiny ? ws_[i] : w[i];
          }
        }
        const float inv = on[u] && d != 0.0f ? 1.0f / d : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(w[i], inv, acc[i]);
        n += on[u] && g == 0;
      }
    }
    // the block's sums: over the rows of a wave, then over the waves
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int off = G; off < 64; off <<= 1) acc[i] += __shfl_xor(acc[i], off);
      if (lane < G) sh_sum[wave][8 * g + i] = acc[i];
    }
    for (int off = 32; off > 0; off >>= 1) n += __shfl_xor(n, off);
    if (lane == 0 && n) atomicAdd(&sh_tokens, n);
    __syncthreads();
    const int64_t piece = (int64_t)blockIdx.x + p;
    if (tid < E) {
      double s = 0.0;
      for (int w = 0; w < kLossWaves; ++w) s += (double)sh_sum[w][tid];
      __hip_atomic_store(ws.pieces + piece * E + tid, pack_piece((float)s, sh_cnt[tid]), __ATOMIC_RELAXED,
                         __HIP_MEMORY_SCOPE_AGENT);
      sh_cnt[tid] = 0;
    }
    if (tid == 0) {
      __hip_atomic_store(ws.tokens + piece, sh_tokens, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sh_tokens = 0;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int first = (int)(pt.off[p] / rows_per_block), last = (int)((pt.off[p + 1] - 1) / rows_per_block);
    if (tid == 0) sh_ticket = __hip_atomic_fetch_add(ws.tickets + p, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (sh_ticket == last - first) {
      // every piece of the group is there
      constexpr int J = kLossThreads / E;
      const int e = tid % E, j = tid / E;
      double s = 0.0;
      int64_t c = 0;
      for (int b = first + j; b <= last; b += J) {
        const uint64_t v = __hip_atomic_load(ws.pieces + (int64_t)(b + p) * E + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s += (double)__uint_as_float((uint32_t)v);
        c += (int)(v >> 32);
      }
      sh_d[tid] = s;
      sh_c[tid] = c;
      int64_t nv = 0;
      if (valid) {
        for (int b = first + lane; b <= last; b += 64)
          nv += __hip_atomic_load(ws.tokens + b + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int off = 32; off > 0; off >>= 1) nv += (int64_t)__shfl_xor((unsigned long long)nv, off);
      } else {
        nv = pt.off[p + 1] - pt.off[p];
      }
      __syncthreads();
      double part = 0.0;
      if (tid < E) {
        for (int q = 1; q < J; ++q) {
          s += sh_d[q * E + tid];
          c += sh_c[q * E + tid];
        }
        if (!idx) c = load[(int64_t)p * E + tid];
        const double mean = nv > 0 ? s / (double)nv : 0.0;
        prob[(int64_t)p * E + tid] = (float)mean;
        if (idx) load[(int64_t)p * E + tid] = (int32_t)c;
        part = nv > 0 ? (double)c * E / ((double)K * (double)nv) * mean : 0.0;
      }
      __syncthreads();
      sh_d[tid] = part;
      __syncthreads();
      if (tid < 64) {
        for (int q = tid + 64; q < E; q += 64) part += sh_d[q];
        for (int off = 32; off > 0; off >>= 1) part += __shfl_xor(part, off);
        if (tid == 0) {
          loss[p] = (float)(alpha * part);
          tokens[p] = (int32_t)nv;
          __hip_atomic_store(ws.tickets + p, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
      }
    }
    s0 = s1;
  }
}

template <int E>
static void launch_loss_e(const BalanceArgs& a, const BalanceWorkspace& ws, hipStream_t s) {
  int blocks;
  int64_t rpb;
  grid_for(a.T, kLossWaves * (512 / E) * kLossU, 1, &blocks, &rpb);
  if (blocks > kBalanceBlocks) {
    rpb = (a.T + kBalanceBlocks - 1) / kBalanceBlocks;
    blocks = (int)((a.T + rpb - 1) / rpb);
  }
  if (a.softmax)
    balance_loss_kernel<E, true><<<blocks, kLossThreads, 0, s>>>(a.z, a.idx, a.valid, a.T, a.K, a.pt, rpb, a.alpha, ws,
                                                                a.load, a.tokens, a.prob, a.loss);
  else
    balance_loss_kernel<E, false><<<blocks, kLossThreads, 0, s>>>(a.z, a.idx, a.valid, a.T, a.K, a.pt, rpb, a.alpha,
                                                                 ws, a.load, a.tokens, a.prob, a.loss);
}

eqb_status launch_balance_loss(const BalanceArgs& a, const BalanceWorkspace& ws, hipStream_t s) {
  switch (a.E) {
    case 8: launch_loss_e<8>(a, ws, s); break;
    case 16: launch_loss_e<16>(a, ws, s); break;
    case 32: launch_loss_e<32>(a, ws, s); break;
    case 64: launch_loss_e<64>(a, ws, s); break;
    case 128: launch_loss_e<128>(a, ws, s); break;
    case 256: launch_loss_e<256>(a, ws, s); break;
    default: return EQB_ERR_UNSUPPORTED;
  }
  return launch_status();
}

// --------------------------------------------------------- the gradient --
// G = E/4 lanes hold a row, 4 experts each.  With C_e = alpha gl_p F_e / n_p a row's
// gradient is p q (C - sum p C) + (g + inj) sigmoid'.  The K mixture gradients of a row
// are scattered into a per-wave LDS row of zeros, read back 4 at a time, and their
// places zeroed again.
constexpr int kGradThreads = 512, kGradWaves = kGradThreads / 64;

template <int E, bool kSoftmax, bool kRouter>
__global__ __launch_bounds__(kGradThreads) void balance_backward_kernel(
    const uint16_t* __restrict__ z, const int32_t* __restrict__ load, const int32_t* __restrict__ tokens,
    const float* __restrict__ grad_loss, const int32_t* __restrict__ idx, const float* __restrict__ gs,
    const float* __restrict__ inj, const uint8_t* __restrict__ valid, int64_t T, int K, const PartTable pt,
    int64_t rows_per_block, double alpha, float* __restrict__ grad_z) {
  constexpr int G = E / 4, R = 64 / G, ROWS = kGradWaves * R;
  __shared__ __align__(16) float sh_g[kGradWaves][R][E];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane % G, rr = lane / G;
  float* my = &sh_g[wave][rr][0];
  if (kRouter && idx) {
#pragma unroll
    for (int i = 0; i < 4; ++i) my[4 * g + i] = 0.0f;
    lds_wave_sync();
  }
  int64_t r0, r1;
  block_rows(T, rows_per_block, &r0, &r1);
  for_each_segment(r0, r1, pt, [&](int p, int64_t s0, int64_t s1) {
    const int nv = tokens[p];
    const double c0 = nv > 0 ? alpha * (double)grad_loss[p] * E / ((double)K * (double)nv * (double)nv) : 0.0;
    float C[4], d0[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      C[i] = (float)(c0 * (double)load[(int64_t)p * E + 4 * g + i]);
      d0[i] = kRouter && inj ? inj[(int64_t)p * E + 4 * g + i] : 0.0f;
    }
    for (int64_t base = s0; base < s1; base += ROWS) {
      const int64_t t = base + wave * R + rr;
      const bool in = t < s1, on = in && (!valid || valid[t]);
      uint2 zw = make_uint2(0, 0);
      if (on) zw = *reinterpret_cast<const uint2*>(z + t * E + 4 * g);
      const float x[4] = {bf16_lo(zw.x), bf16_hi(zw.x), bf16_lo(zw.y), bf16_hi(zw.y)};
      if (kRouter && idx) {
        if (on)
          for (int k = g; k < K; k += G) {
            const int e = idx[t * K + k];
            if (e >= 0 && e < E) my[e] = gs[t * K + k];
          }
        lds_wave_sync();
      }
      float w[4], q[4], sd[4], d;
      if (!kSoftmax || kRouter) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e = __builtin_amdgcn_exp2f(fabsf(x[i]) * -kLog2e);
          const float r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
          w[i] = x[i] >= 0.0f ? r : er;
          q[i] = x[i] >= 0.0f ? er : r;
          sd[i] = er * r;
        }
      }
      if (kSoftmax) {
        d = softmax_terms<G>(x, w);
      } else {
        d = group_sum<G>(w[0] + w[1] + (w[2] + w[3]));
        const bool tiny = on && d < kTinySum;
        if (__any(tiny)) {
          float v[4];
          const float dv = softmax_terms<G>(x, v);
          d = tiny ? dv : d;
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = tiny ? v[i] : w[i];
        }
      }
      const float inv = d != 0.0f ? 1.0f / d : 0.0f;
      float c = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] *= inv;
        c = __builtin_fmaf(w[i], C[i], c);
      }
      c = group_sum<G>(c);
      float4 o;
      float* po = &o.x;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a = w[i] * (C[i] - c);
        if (!kSoftmax) a *= q[i];
        if (kRouter) a = __builtin_fmaf((idx ? my[4 * g + i] : 0.0f) + d0[i], sd[i], a);
        po[i] = on ? a : 0.0f;
      }
      if (in) *reinterpret_cast<float4*>(grad_z + t * E + 4 * g) = o;
      if (kRouter && idx) {
        lds_wave_sync();
#pragma unroll
        for (int i = 0; i < 4; ++i) my[4 * g + i] = 0.0f;
        lds_wave_sync();
      }
    }
  });
}

template <int E, bool kSoftmax>
static void launch_backward_es(const BalanceArgs& a, hipStream_t s) {
  int blocks;
  int64_t rpb;
  grid_for(a.T, kGradWaves * (256 / E), 4, &blocks, &rpb);
  if (a.idx || a.inj)
    balance_backward_kernel<E, kSoftmax, true><<<blocks, kGradThreads, 0, s>>>(
        a.z, a.load, a.tokens, a.grad_loss, a.idx, a.grad_score, a.inj, a.valid, a.T, a.K, a.pt, rpb, a.alpha, a.grad_z);
  else
    balance_backward_kernel<E, kSoftmax, false><<<blocks, kGradThreads, 0, s>>>(
        a.z, a.load, a.tokens, a.grad_loss, a.idx, a.grad_score, a.inj, a.valid, a.T, a.K, a.pt, rpb, a.alpha, a.grad_z);
}
template <int E>
static void launch_backward_e(const BalanceArgs& a, hipStream_t s) {
  if (a.softmax) launch_backward_es<E, true>(a, s);
  else launch_backward_es<E, false>(a, s);
}

eqb_status launch_balance_backward(const BalanceArgs& a, hipStream_t s) {
  switch (a.E) {
    case 8: launch_backward_e<8>(a, s); break;
    case 16: launch_backward_e<16>(a, s); break;
    case 32: launch_backward_e<32>(a, s); break;
    case 64: launch_backward_e<64>(a, s); break;
    case 128: launch_backward_e<128>(a, s); break;
    case 256: launch_backward_e<256>(a, s); break;
    default: return EQB_ERR_UNSUPPORTED;
  }
  return launch_status();
}

}  // namespace eqb
