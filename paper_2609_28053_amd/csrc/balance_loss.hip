// balance_loss.hip - the auxiliary balance loss (arXiv 2609.28053, Sec. 2, "GShard";
// App. D) with the experts' counts, and its gradient fused with the router backward
// (Sec. 2, Eq. 1) and the load-error injection (Sec. 4).
#include "eqb_internal.hpp"

namespace eqb {

// The partition that holds row t.
__device__ __forceinline__ int partition_of(const PartTable& pt, int64_t t) {
  int lo = 0, hi = pt.P - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (pt.off[mid + 1] <= t) lo = mid + 1;
    else hi = mid;
  }
  return lo;
}

constexpr float kLog2e = 1.4426950408889634f;
// Below this sum the sigmoids of a row equal their exponentials to binary32, and they or
// their products may have lost digits to underflow: the row's probabilities are then those of
// a softmax.
constexpr float kTinySum = 0x1p-60f;

// A row's exponentials exp(x - max) over the group's lanes, whole rows of -inf giving 0, and
// their sum; where a row does not take part its terms w and sum d stay as they are.
template <int G, int N>
__device__ __forceinline__ float softmax_where(bool part, const float (&x)[N], float (&w)[N], float d) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < N; ++i) m = fmaxf(m, x[i]);
  m = fmaxf(group_max<G>(m), -3.402823466e38f);     // BF16's lowest value is above it
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float v = __builtin_amdgcn_exp2f((x[i] - m) * kLog2e);
    w[i] = part ? v : w[i];
    sum += v;
  }
  sum = group_sum<G>(sum);
  return part ? sum : d;
}
template <int G, int N>
__device__ __forceinline__ float softmax_terms(const float (&x)[N], float (&w)[N]) {
  return softmax_where<G>(true, x, w, 0.0f);
}

// ------------------------------------------------------------- the loss --
// Every group is cut into pieces of a block's rows.  Where blocks went on from one group's
// last rows to the next one's first, these were the last to finish: 99,991 rows of E = 128
// in three groups 19.0 us, in pieces 17.5; 20,000 of E = 256 in 64 groups 13.8 and 9.8.
// G = E/8 lanes hold a row, 8 experts each.  A lane sums the probabilities of its
// experts over its rows in binary32, 128 rows at most: then its wave's sums are added to
// binary64 ones in LDS (one sum over 80,000 equal rows was off by 1.2e-3, so by 1.9e-6; a
// step costs nothing measurable more).  At the end of a piece the block adds its lanes' sums,
// the waves' in binary64.  The pieces of a group are handed over (in binary32) through the
// workspace: the last of a bunch of neighbours to come, by a ticket, adds theirs, and the
// last of those adds the sums, each in a fixed order in binary64, and writes the group's
// results.  Who completes a count sets its ticket back to 0.  Blocks sit on XCDs with an L2
// each: pieces pass between them in agent-scope stores and loads, complete (vmcnt) before
// the ticket is drawn.
constexpr int kLossThreads = 768, kLossWaves = kLossThreads / 64;
constexpr int kLossU = 2;          // rows per lane and step
constexpr uint32_t kLossSteps = 64;     // steps of a lane's sum in binary32

// The pieces: `rows` rows each, but for a group's last; group p's are first[p] to
// first[p + 1] - 1, and first is above them all past first[P].
constexpr int kPieceChunk = 16;
struct Pieces {
  int32_t first[EQB_MAX_PARTITIONS + kPieceChunk];
  int32_t rows;
};

// The group of a piece, by a count of kPieceChunk groups at a time: a search would wait for
// each of its loads, and the arguments are far away (20,000 rows in 64 groups: 9.8 us in
// chunks of 16, 15.0 of 4).
__device__ __forceinline__ int group_of(const Pieces& pieces, int P, int piece) {
  int p = -1;
  for (int q = 0; q < P; q += kPieceChunk) {
#pragma unroll
    for (int i = 0; i < kPieceChunk; ++i) p += pieces.first[q + i] <= piece ? 1 : 0;
  }
  return p;
}

__device__ __forceinline__ uint64_t pack_piece(float prob, int count) {
  return (uint64_t)__float_as_uint(prob) | ((uint64_t)(uint32_t)count << 32);
}

template <int E, bool kSoftmax, bool kMask>
__global__ __launch_bounds__(kLossThreads, 6) void balance_loss_kernel(
    const uint16_t* __restrict__ z, const int32_t* __restrict__ idx, const uint8_t* __restrict__ valid, int64_t T,
    int K, const PartTable pt, const Pieces pieces, int bunch_bits, double alpha, const BalanceWorkspace ws, int32_t* load,
    int32_t* __restrict__ tokens, float* __restrict__ prob, float* __restrict__ loss) {
  constexpr int G = E / 8, R = 64 / G;
  constexpr uint32_t ROWS = kLossWaves * R * kLossU;
  __shared__ float sh_sum[kLossWaves][E];
  __shared__ double sh_long[kLossWaves][E];      // sums of the wave's earlier steps
  // counts in 256/E copies, a lane adding to copy lane % copies: with one, the 64 lanes of
  // a wave queue on the few counters of a small E
  __shared__ int32_t sh_cnt[kNBins / E][E];
  __shared__ int32_t sh_tokens, sh_ticket;
  __shared__ double sh_d[kLossThreads];
  __shared__ int64_t sh_c[kLossThreads];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane % G, rr = lane / G;
  if (blockIdx.x == 0) {           // groups without tokens
    for (int q = tid >> 6; q < pt.P; q += kLossWaves) {
      if (pt.off[q + 1] > pt.off[q]) continue;
      for (int e = lane; e < E; e += 64) {
        prob[q * E + e] = 0.0f;
        if (idx || T == 0) load[q * E + e] = 0;
      }
      if (lane == 0) {
        tokens[q] = 0;
        loss[q] = 0.0f;
      }
    }
  }
  if (tid < kNBins) (&sh_cnt[0][0])[tid] = 0;
  if (tid == 0) sh_tokens = 0;
  const int all = pieces.first[pt.P];
  for (int piece = blockIdx.x; piece < all; piece += gridDim.x) {
    const int p = group_of(pieces, pt.P, piece);
    const int first = pieces.first[p], last = pieces.first[p + 1] - 1;
    const int64_t s0 = pt.off[p] + (int64_t)(piece - first) * pieces.rows;
    const int64_t s1 = pt.off[p + 1] < s0 + pieces.rows ? pt.off[p + 1] : s0 + pieces.rows;
    __syncthreads();
    float acc[8] = {};
    int n = 0;
    uint32_t steps = 0;
    // pieces of at most kSegMax rows: 32-bit offsets from their bases
    for (int64_t c0 = s0; c0 < s1; c0 += kSegMax) {
      const int64_t cu = wave_uniform(c0);
      const uint16_t* zc = z + cu * E;
      const uint8_t* vc = kMask ? valid + cu : nullptr;
      const uint32_t rows = (uint32_t)(s1 - c0 < kSegMax ? s1 - c0 : kSegMax);
      // rows past the last one read the last one, and count as 0
      auto row_of = [&](uint32_t base, int u) { return base + (uint32_t)((u * kLossWaves + wave) * R + rr); };
      auto fetch = [&](uint32_t base, uint4 (&zw)[kLossU], uint32_t (&vb)[kLossU]) {
#pragma unroll
        for (int u = 0; u < kLossU; ++u) {
          const uint32_t t = row_of(base, u), tc = t < rows ? t : rows - 1;
          zw[u] = at<const uint4>(zc, (tc * E + 8 * g) * 2u);
          vb[u] = kMask ? at<const uint8_t>(vc, tc) : 1u;
        }
      };
      uint4 zn[kLossU];
      uint32_t next[kLossU];         // the mask's bytes: to compare them here would wait for them
      fetch(0, zn, next);
      if (idx) {
        const int32_t* ic = idx + cu * K;
        const uint32_t pairs = rows * (uint32_t)K, inv_K = 0xFFFFFFFFu / (uint32_t)K + 1, one = K == 1 ? ~0u : 0u;
        for (uint32_t i = tid; i < pairs; i += 4 * kLossThreads) {
          // all loads first, of places in range, and no branches among them
          int e[4], ok[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t k = i + j * kLossThreads, kc = k < pairs ? k : pairs - 1;
            e[j] = at<const int32_t>(ic, 4u * kc);
            // kc / K: exact below 2^24 for K < 256 by the rounded-up reciprocal (0 for K = 1)
            ok[j] = kMask ? at<const uint8_t>(vc, __umulhi(kc, inv_K) + (kc & one)) : 1;
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool in = (i + j * kLossThreads < pairs) & (ok[j] != 0) & ((uint32_t)e[j] < (uint32_t)E);
            if (in) atomicAdd(&sh_cnt[lane % (kNBins / E)][e[j]], 1);
          }
        }
      }
      for (uint32_t base = 0; base < rows; base += ROWS) {
        if (__builtin_expect(++steps > kLossSteps && steps % kLossSteps == 1, 0)) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            double& to = sh_long[wave][8 * g + i];
            const float v = column_sum<G>(acc[i]);
            if (lane < G) to = steps > 2 * kLossSteps ? to + (double)v : (double)v;
            acc[i] = 0.0f;
          }
        }
        uint4 zw[kLossU];
        bool on[kLossU];
#pragma unroll
        for (int u = 0; u < kLossU; ++u) {
          zw[u] = zn[u];
          on[u] = row_of(base, u) < rows && next[u] != 0;
        }
        fetch(base + ROWS, zn, next);
#pragma unroll
        for (int u = 0; u < kLossU; ++u) {
          if (kMask && !on[u]) zw[u] = make_uint4(0, 0, 0, 0);      // whatever a masked token holds
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
            const bool tiny = d < kTinySum;
            if (__any(tiny)) {
              // the logits unpacked again, rather than kept for this in registers
              asm volatile("" : "+v"(zw[u].x), "+v"(zw[u].y), "+v"(zw[u].z), "+v"(zw[u].w));
              const float y[8] = {bf16_lo(zw[u].x), bf16_hi(zw[u].x), bf16_lo(zw[u].y), bf16_hi(zw[u].y),
                                  bf16_lo(zw[u].z), bf16_hi(zw[u].z), bf16_lo(zw[u].w), bf16_hi(zw[u].w)};
              d = softmax_where<G>(tiny, y, w, d);
            }
          }
          const float inv = on[u] && d != 0.0f ? __builtin_amdgcn_rcpf(d) : 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[i] = __builtin_fmaf(w[i], inv, acc[i]);
          if (kMask) n += on[u] && g == 0;
        }
      }
    }
    // the block's sums: over the rows of a wave, then over the waves
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      acc[i] = column_sum<G>(acc[i]);
      if (lane < G) sh_sum[wave][8 * g + i] = acc[i];
    }
    if (kMask) {
      n = group_fold<64>(n, [](int a, int b) { return a + b; });
      if (lane == 0 && n) atomicAdd(&sh_tokens, n);
    }
    __syncthreads();
    double sum = 0.0;
    int64_t count = 0, nv = pt.off[p + 1] - pt.off[p];
    if (tid < E) {
      for (int w = 0; w < kLossWaves; ++w) sum += (double)sh_sum[w][tid];
      if (steps > kLossSteps)
        for (int w = 0; w < kLossWaves; ++w) sum += sh_long[w][tid];
      for (int c = 0; c < kNBins / E; ++c) {
        count += sh_cnt[c][tid];
        sh_cnt[c][tid] = 0;
      }
    }
    if (kMask) nv = sh_tokens;
    bool whole = true;             // sum, count and nv are the group's
    if (first < last) {
      // Pieces of a bunch of neighbours are summed by the last of these to come, and the
      // bunches' sums by the last to bring one.  A bunch of a group has place bunch + p: both
      // only grow from piece to piece.
      const int bunch = piece >> bunch_bits, bunch0 = first >> bunch_bits, bunch1 = last >> bunch_bits;
      const int i0 = bunch == bunch0 ? first : bunch << bunch_bits;
      const int i1 = bunch == bunch1 ? last : ((bunch + 1) << bunch_bits) - 1;
      auto hand_over = [&](uint64_t* to, int32_t* to_tokens, int at, int32_t* ticket, int others) {
        if (tid < E)
          __hip_atomic_store(to + (int64_t)at * E + tid, pack_piece((float)sum, (int)count), __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
        if (kMask && tid == 0)
          __hip_atomic_store(to_tokens + at, (int)nv, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) {
          const int before = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (before == others) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          sh_ticket = before;
        }
        __syncthreads();
        return sh_ticket == others;
      };
      auto collect = [&](const uint64_t* from, const int32_t* from_tokens, int lo, int hi) {
        constexpr int J = kLossThreads / E, kAhead = 8;
        const int e = tid % E, j = tid / E;
        sum = 0.0;
        count = 0;
        for (int b0 = lo + j; b0 <= hi; b0 += kAhead * J) {
          uint64_t v[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
            v[i] = b0 + i * J <= hi ? __hip_atomic_load(from + (int64_t)(b0 + i * J) * E + e, __ATOMIC_RELAXED,
                                                        __HIP_MEMORY_SCOPE_AGENT) : 0;
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            sum += (double)__uint_as_float((uint32_t)v[i]);
            count += (int)(v[i] >> 32);
          }
        }
        sh_d[tid] = sum;
        sh_c[tid] = count;
        if (kMask) {
          nv = 0;
          for (int b = lo + lane; b <= hi; b += 64)
            nv += __hip_atomic_load(from_tokens + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          for (int off = 32; off > 0; off >>= 1) nv += (int64_t)__shfl_xor((unsigned long long)nv, off);
        }
        __syncthreads();
        if (tid < E) {
#pragma unroll 2
          for (int q = 1; q < J; ++q) {
            sum += sh_d[q * E + tid];
            count += sh_c[q * E + tid];
          }
        }
        __syncthreads();
      };
      whole = hand_over(ws.pieces, ws.tokens, piece, ws.bunch_tickets + bunch + p, i1 - i0);
      if (whole) {
        collect(ws.pieces, ws.tokens, i0, i1);
        if (bunch0 < bunch1) {
          whole = hand_over(ws.bunches, ws.bunch_tokens, bunch + p, ws.tickets + p, bunch1 - bunch0);
          if (whole) collect(ws.bunches, ws.bunch_tokens, bunch0 + p, bunch1 + p);
        }
      }
    }
    if (whole) {
      double part = 0.0;
      if (tid < E) {
        if (!idx) count = load[(int64_t)p * E + tid];
        else load[(int64_t)p * E + tid] = (int32_t)count;
        const double mean = nv > 0 ? sum / (double)nv : 0.0;
        prob[(int64_t)p * E + tid] = (float)mean;
        part = nv > 0 ? (double)count * E / ((double)K * (double)nv) * mean : 0.0;
        sh_d[tid] = part;
      }
      __syncthreads();
      if (tid < 64) {
        part = lane < E ? part : 0.0;
        for (int q = lane + 64; q < E; q += 64) part += sh_d[q];
        part = wave_sum(part);
        if (lane == 0) {
          loss[p] = (float)(alpha * part);
          tokens[p] = (int32_t)nv;
          sh_tokens = 0;
        }
      }
    } else if (tid == 0) {
      sh_tokens = 0;
    }
  }
}

// Pieces of the same number of rows as far as they go: no more than `most` of them where that
// leaves the groups several each, or else up to one more for each group.  Returns the blocks
// to launch for them.
static int cut_groups(const PartTable& pt, int64_t T, int64_t most, Pieces* c) {
  int64_t rows = 1;
  auto cut = [&](int64_t n) {
    int64_t all = 0;
    rows = 1;
    for (int p = 0; p < pt.P; ++p) {
      const int64_t own = pt.off[p + 1] - pt.off[p], parts = (own + n - 1) / n;
      c->first[p] = (int32_t)all;
      all += parts;
      if (parts > 0 && (own + parts - 1) / parts > rows) rows = (own + parts - 1) / parts;
    }
    return all;
  };
  int64_t all = cut(T > most ? (T + most - 1) / most : 1);
  if (all > most && most >= 4 * pt.P) all = cut((T + most - pt.P - 1) / (most - pt.P));
  all = cut(rows);          // evened out: every group has as many parts as before or fewer
  c->first[pt.P] = (int32_t)all;
  for (int p = pt.P + 1; p < EQB_MAX_PARTITIONS + kPieceChunk; ++p) c->first[p] = INT32_MAX;
  c->rows = (int32_t)rows;
  const int cap = max_blocks_cap();
  return all < 1 ? 1 : cap > 0 && cap < all ? cap : (int)all;
}

template <int E, bool kSoftmax, bool kMask>
static void launch_loss_as(const BalanceArgs& a, const BalanceWorkspace& ws, hipStream_t s) {
  int most;
  int64_t rows;
  // One block for 32,768 logits, blocks of at least 16,384 beyond: 4,096 rows of E = 8 take
  // 8.8 us in one block and 12.4 in two, 16,384 rows of E = 64 8.7 in 64 and 9.4 in 32.
  // One block per compute unit for up to 2^26 logits (99,991 rows of E = 128 19.0 us, with
  // two 22.4; 147,456 of E = 256 24 either way), two beyond, where they hide more latency.
  const int64_t logits = a.T * E;
  grid_for(a.T, logits <= 32768 ? 32768 / E : 16384 / E, logits <= 1 << 26 ? 1 : 2, &most, &rows);
  most = most < kBalanceBlocks ? most : kBalanceBlocks;
  Pieces pieces;
  const int blocks = cut_groups(a.pt, a.T, most, &pieces), all = pieces.first[a.pt.P];
  // Bunches pay where one block would read more than 256 KiB of pieces.  One group, without and
  // with them: 16,384 rows of E = 256 17.7 and 12.4 us, 147,456 28.2 and 22.8, 1,000,003 of E =
  // 128 61.2 and 55.8; of E = 64 34.2 and 34.6, of E = 16 19.0 and 22.3, of E = 8 18.8 and 24.0;
  // at the line, 99,991 of E = 128 (254 KiB) 17.8 and 16.2, in three groups 15.1 and 15.5.  (10
  // bits: all blocks are one bunch.)
  const int bunch_bits = (int64_t)all * E * (int64_t)sizeof(uint64_t) > (256 << 10) ? kBunchBits : 10;
  static_assert(kBalanceBlocks + EQB_MAX_PARTITIONS <= 1 << 10, "one bunch");
  balance_loss_kernel<E, kSoftmax, kMask><<<blocks, kLossThreads, 0, s>>>(
      a.z, a.idx, a.valid, a.T, a.K, a.pt, pieces, bunch_bits, a.alpha, ws, a.load, a.tokens, a.prob, a.loss);
}
template <int E>
static void launch_loss_e(const BalanceArgs& a, const BalanceWorkspace& ws, hipStream_t s) {
  if (a.softmax) {
    if (a.valid) launch_loss_as<E, true, true>(a, ws, s);
    else launch_loss_as<E, true, false>(a, ws, s);
  } else {
    if (a.valid) launch_loss_as<E, false, true>(a, ws, s);
    else launch_loss_as<E, false, false>(a, ws, s);
  }
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
// sigmoid' is computed as in the router backward alone, so that with C = 0 the results are
// the same bits, and p q of a sigmoid row is sigmoid' / d.  Against the bare exponential and
// reciprocal, which lose digits of large logits and all beyond 87, that costs up to 2% (the
// gradient of 1,000,003 rows of E = 128, K = 8: 160.5 -> 163.6 us, of 131,072 of E = 256 36.0
// and 36.2; with logits of -inf among them, which do not take the longer form, 36.1 and 36.5),
// of a softmax in the caches more (300,000 of E = 64 24.0 -> 26.0).
// Bound by memory: 2E + 8K bytes read and 4E written per row, all of it once.  The
// gradient's stores are non-temporal, and so are the logits' loads when these take more than
// a quarter of the memory-side cache (kStream); fewer are still there from the loss or the
// routing.  With the loss before it, 99,991 rows of E = 128 (26 MB) 35.8 us with non-temporal
// loads, 32.0 without; 131,072 of E = 256 (64 MiB) 56.0 and 55.2; 2,000,000 of E = 32 (128
// MB) 96 and 105; the gradient alone of 4,194,304 of E = 256 1,274 and 1,325.
// Two rows a lane and eight waves a SIMD: when this was chosen, over one set of buffers,
// 4,194,304 rows of E = 256, K = 8 took 1,276 us, with three rows and six waves 1,324, four
// and four 1,320, one and eight 1,306; 1,000,003 of E = 128 161, 175, 161, 164.  Over buffers
// that change they take 1,345 (5.0 TB/s) and 164.
constexpr int kGradThreads = 512, kGradWaves = kGradThreads / 64;
constexpr int kGradU = 2;          // rows per lane and step
constexpr int kGradWavesPerSimd = 8;
constexpr int kGradBlocksPerCu = kGradWavesPerSimd * 256 / kGradThreads;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Whether any of four BF16 values has a magnitude from 32 to 104.  2 |x| - 2 * 32 in 16-bit
// patterns, the sign shifted out: below 32 it wraps past all others.
__device__ __forceinline__ bool any_from_32_to_104(uint32_t w0, uint32_t w1) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  constexpr uint16_t k32 = 0x4200, k104 = 0x42D0;
  const u16x2 two = {2, 2}, low = {(uint16_t)(2 * k32), (uint16_t)(2 * k32)};
  const u16x2 a = __builtin_bit_cast(u16x2, w0) * two - low, b = __builtin_bit_cast(u16x2, w1) * two - low;
  const u16x2 m = __builtin_elementwise_min(a, b);
  return (m.x < m.y ? m.x : m.y) <= 2 * (k104 - k32);
}

// What goes with the loss's gradient: nothing, the router backward where a lane of a
// row's group holds at most one of its K pairs, or the router backward with any K (and
// the injection without pairs).
enum { kAlone, kOnePair, kAnyPairs };
constexpr int64_t kGradStreamBytes = (int64_t)64 << 20;

template <int E, bool kSoftmax, int kRouter, bool kStream>
__global__ __launch_bounds__(kGradThreads, kGradWavesPerSimd) void balance_backward_kernel(
    const uint16_t* __restrict__ z, const int32_t* __restrict__ load, const int32_t* __restrict__ tokens,
    const float* __restrict__ grad_loss, const int32_t* __restrict__ idx, const float* __restrict__ gs,
    const float* __restrict__ inj, const uint8_t* __restrict__ valid, int64_t T, int K, const PartTable pt,
    int64_t rows_per_block, double alpha, float* __restrict__ grad_z) {
  constexpr int G = E / 4, R = 64 / G;
  constexpr uint32_t ROWS = kGradWaves * R * kGradU;
  constexpr bool kSigmoid = !kSoftmax || kRouter != kAlone;
  __shared__ __align__(16) float sh_g[kRouter == kAlone ? 1 : kGradWaves][kGradU][R][E];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane % G, rr = lane / G;
  float* my = &sh_g[kRouter == kAlone ? 0 : wave][0][rr][0];      // row u of this lane: my + u * R * E
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  auto place = [&](int u) -> f32x4& { return *reinterpret_cast<f32x4*>(my + u * R * E + 4 * g); };
  if (kRouter != kAlone) {
#pragma unroll
    for (int u = 0; u < kGradU; ++u) place(u) = zero;
    lds_wave_sync();
  }
  int64_t r0, r1;
  block_rows(T, rows_per_block, &r0, &r1);
  for (int64_t s0 = r0, s1; s0 < r1; s0 = s1) {
    const int p = partition_of(pt, s0);
    s1 = pt.off[p + 1] < r1 ? pt.off[p + 1] : r1;
    if (s1 - s0 > kSegMax) s1 = s0 + kSegMax;
    // a segment holds at most kSegMax rows: 32-bit byte offsets from its bases
    const int64_t su = wave_uniform(s0);
    const uint16_t* seg_z = z + su * E;
    const int32_t* seg_idx = idx + su * K;
    const float* seg_gs = gs + su * K;
    const uint8_t* seg_valid = valid + su;
    float* seg_gz = grad_z + su * E;
    const uint32_t n = (uint32_t)(s1 - s0);
    const int nv = tokens[p];
    const double c0 = nv > 0 ? alpha * (double)grad_loss[p] * E / ((double)K * (double)nv * (double)nv) : 0.0;
    f32x4 C, d0 = zero;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      C[i] = (float)(c0 * (double)load[(int64_t)p * E + 4 * g + i]);
      if (kRouter != kAlone && inj) d0[i] = inj[(int64_t)p * E + 4 * g + i];
    }
    auto row_of = [&](uint32_t base, int u) -> uint32_t { return base + (uint32_t)((wave * kGradU + u) * R + rr); };
    // logits, mask and this lane's pair of its rows at step base
    auto fetch = [&](uint32_t base, u32x2 (&zw)[kGradU], uint32_t (&vb)[kGradU], int (&e)[kGradU], float (&gv)[kGradU]) {
#pragma unroll
      for (int u = 0; u < kGradU; ++u) {
        const uint32_t t = row_of(base, u);
        zw[u] = u32x2{0, 0};
        e[u] = -1;
        gv[u] = 0.0f;
        vb[u] = 0;
        if (t < n) {
          vb[u] = valid ? at<const uint8_t>(seg_valid, t) : 1;
          const u32x2& from = at<const u32x2>(seg_z, (t * E + 4 * g) * 2u);
          zw[u] = kStream ? __builtin_nontemporal_load(&from) : from;
          if (kRouter == kOnePair && g < K) {
            e[u] = at<const int32_t>(seg_idx, (t * K + g) * 4u);
            gv[u] = at<const float>(seg_gs, (t * K + g) * 4u);
          }
        }
      }
    };
    u32x2 zn[kGradU];
    uint32_t vn[kGradU];           // the mask's bytes: to compare them here would wait for them
    int en[kGradU];
    float gn[kGradU];
    fetch(0, zn, vn, en, gn);
    for (uint32_t base = 0; base < n; base += ROWS) {
      u32x2 zw[kGradU];
      bool on[kGradU];
      int ec[kGradU];
      float gc[kGradU];
#pragma unroll
      for (int u = 0; u < kGradU; ++u) {
        on[u] = vn[u] != 0;
        // whatever a masked token holds
        zw[u] = on[u] ? zn[u] : u32x2{0, 0};
        ec[u] = on[u] ? en[u] : -1;
        gc[u] = gn[u];
      }
      if (base + ROWS < n) fetch(base + ROWS, zn, vn, en, gn);
      // scatter the rows' mixture gradients
      if (kRouter != kAlone) {
#pragma unroll
        for (int u = 0; u < kGradU; ++u) {
          if (kRouter == kOnePair) {
            if (ec[u] >= 0 && ec[u] < E) my[u * R * E + ec[u]] = gc[u];
          } else if (idx && on[u]) {
            const uint32_t t = row_of(base, u);
            for (int k = g; k < K; k += G) {
              const int e = at<const int32_t>(seg_idx, (t * K + k) * 4u);
              if (e >= 0 && e < E) my[u * R * E + e] = at<const float>(seg_gs, (t * K + k) * 4u);
            }
          }
        }
        lds_wave_sync();
      }
#pragma unroll
      for (int u = 0; u < kGradU; ++u) {
        const uint32_t t = row_of(base, u);
        const float x[4] = {bf16_lo(zw[u].x), bf16_hi(zw[u].x), bf16_lo(zw[u].y), bf16_hi(zw[u].y)};
        // w: p without the division by d; pq: p q without it
        float w[4], sd[4], pq[4], d;
        if (kSigmoid) {
          // exp(-|x|) as in the router backward alone: logits from 32 to 104 take a longer form,
          // chosen per wave and row.  Beyond (masked experts) both forms give 0.  Without the router
          // nothing is a multiple of sigmoid': what the short form loses, 1e-7 of a probability at 90,
          // does not matter.
          float ex[4];
          if (kRouter != kAlone && __builtin_expect(__any(any_from_32_to_104(zw[u].x, zw[u].y)), 0)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) ex[i] = exp_neg_bf16_wide(fabsf(x[i]));
            asm volatile("; large logits");
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) ex[i] = exp_neg_bf16<true>(fabsf(x[i]));
          }
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float r = newton_rcp(1.0f + ex[i]), er = ex[i] * r;     // sigmoid(|x|), sigmoid(-|x|)
            w[i] = x[i] >= 0.0f ? r : er;
            pq[i] = sd[i] = __builtin_fmaf(-er, er, er);
          }
        }
        if (kSoftmax) {
          d = softmax_terms<G>(x, w);
#pragma unroll
          for (int i = 0; i < 4; ++i) pq[i] = w[i];
        } else {
          d = group_sum<G>(w[0] + w[1] + (w[2] + w[3]));
          const bool tiny = d < kTinySum;
          if (__any(tiny)) {
            // the logits unpacked again, rather than kept for this in registers
            uint32_t w0 = zw[u].x, w1 = zw[u].y;
            asm volatile("" : "+v"(w0), "+v"(w1));
            const float y[4] = {bf16_lo(w0), bf16_hi(w0), bf16_lo(w1), bf16_hi(w1)};
            d = softmax_where<G>(tiny, y, w, d);
#pragma unroll
            for (int i = 0; i < 4; ++i) pq[i] = tiny ? w[i] : pq[i];      // q is 1 there
          }
        }
        const float inv = d != 0.0f ? newton_rcp(d) : 0.0f;
        float c = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_fmaf(w[i], C[i], c);
        c = group_sum<G>(c) * inv;
        const f32x4 gm = kRouter != kAlone ? place(u) + d0 : zero;
        f32x4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = (C[i] - c) * inv;
          const float a = kRouter != kAlone ? __builtin_fmaf(pq[i], s, gm[i] * sd[i]) : pq[i] * s;
          o[i] = on[u] ? a : 0.0f;
        }
        if (t < n) __builtin_nontemporal_store(o, &at<f32x4>(seg_gz, (t * E + 4 * g) * 4u));
      }
      if (kRouter != kAlone) {
        lds_wave_sync();          // every place has been read
#pragma unroll
        for (int u = 0; u < kGradU; ++u) {
          if (kRouter == kAnyPairs) place(u) = zero;
          else if (ec[u] >= 0 && ec[u] < E) my[u * R * E + ec[u]] = 0.0f;
        }
        lds_wave_sync();          // the next step scatters into zeros
      }
    }
  }
}

template <int E, bool kSoftmax, int kRouter>
static void launch_backward_as(const BalanceArgs& a, hipStream_t s) {
  int blocks;
  int64_t rpb;
  grid_for(a.T, kGradWaves * (256 / E) * kGradU, kGradBlocksPerCu, &blocks, &rpb);
  const bool stream = a.T * E * (int64_t)sizeof(uint16_t) > kGradStreamBytes;
  const auto kernel = stream ? balance_backward_kernel<E, kSoftmax, kRouter, true>
                             : balance_backward_kernel<E, kSoftmax, kRouter, false>;
  kernel<<<blocks, kGradThreads, 0, s>>>(
      a.z, a.load, a.tokens, a.grad_loss, a.idx, a.grad_score, a.inj, a.valid, a.T, a.K, a.pt, rpb, a.alpha, a.grad_z);
}
template <int E, bool kSoftmax>
static void launch_backward_es(const BalanceArgs& a, hipStream_t s) {
  if (!a.idx && !a.inj) launch_backward_as<E, kSoftmax, kAlone>(a, s);
  else if (a.idx && a.K <= E / 4) launch_backward_as<E, kSoftmax, kOnePair>(a, s);
  else launch_backward_as<E, kSoftmax, kAnyPairs>(a, s);
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
