// adamw.hip - one AdamW step over a list of tensors, with binary32 or 8-bit states.
#include "eqb_internal.hpp"

namespace eqb {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
// the same at the alignment of one element: tensors may start anywhere in a flat buffer
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u16x4 u16x4_any __attribute__((aligned(2)));
typedef uint32_t u32_any __attribute__((aligned(1)));

constexpr int kAdamwThreads = 256;
constexpr int kAdamwBlocks = 4;                                     // blocks of EQB_ADAMW_BLOCK elements per wave
constexpr int64_t kAdamwChunk = kAdamwThreads / 64 * kAdamwBlocks * EQB_ADAMW_BLOCK;

// E4M3 codes of y (0 <= y <= 448) rounded up where the random 16 bits exceed what y
// lacks to the next code.  From 2^-6 on a code is the top of the binary32 pattern with
// 20 bits dropped; below, y + 2^-6 has the subnormal codes' spacing.
__device__ __forceinline__ uint32_t encode_e4m3(float y, uint32_t rnd16) {
  const bool small = y < 0x1p-6f;
  const float t = small ? y + 0x1p-6f : y;
  return ((__float_as_uint(t) + (rnd16 << 4)) >> 20) - (small ? 968u : 960u);
}

__device__ __forceinline__ f32x4 decode_e4m3x4(uint32_t w) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

// Maximum over the wave, the same in every lane.
__device__ __forceinline__ float wave_max(float x) {
  for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off));
  return x;
}

template <bool k8, bool kGradBf16, bool kCopy>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(const AdamwBatch batch) {
  if (batch.found_inf && *batch.found_inf != 0.0f) return;
  // the tensor of this block: the last whose first block is not past it
  int lo = 0, hi = batch.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (batch.t[mid].first_block <= blockIdx.x) lo = mid;
    else hi = mid - 1;
  }
  const AdamwSlot& t = batch.t[lo];
  const float scale = batch.grad_scale ? *batch.grad_scale : 1.0f;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t begin = (int64_t)(blockIdx.x - t.first_block) * kAdamwChunk;
  for (int u = 0; u < kAdamwBlocks; ++u) {
    const int64_t base = begin + (int64_t)(u * (kAdamwThreads / 64) + wave) * EQB_ADAMW_BLOCK;
    if (base >= t.numel) return;
    const int64_t j = base + 4 * lane;
    const int left = (int)(t.numel - base < EQB_ADAMW_BLOCK ? t.numel - base : EQB_ADAMW_BLOCK) - 4 * lane;
    f32x4 w = {0, 0, 0, 0}, g = w, m = w, v = w;
    if (left >= 4) {
      w = *reinterpret_cast<const f32x4_any*>(t.param + j);
      if (kGradBf16) {
        const u16x4 b = *reinterpret_cast<const u16x4_any*>(static_cast<const uint16_t*>(t.grad) + j);
        for (int i = 0; i < 4; ++i) g[i] = __uint_as_float((uint32_t)b[i] << 16);
      } else {
        g = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(t.grad) + j);
      }
      if (k8) {
        m = decode_e4m3x4(*reinterpret_cast<const u32_any*>(static_cast<const uint8_t*>(t.exp_avg) + j));
        v = decode_e4m3x4(*reinterpret_cast<const u32_any*>(static_cast<const uint8_t*>(t.exp_avg_sq) + j));
      } else {
        m = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(t.exp_avg) + j);
        v = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(t.exp_avg_sq) + j);
      }
    } else {
      uint32_t cm = 0, cv = 0;
      for (int i = 0; i < left; ++i) {
        w[i] = t.param[j + i];
        g[i] = kGradBf16 ? __uint_as_float((uint32_t) static_cast<const uint16_t*>(t.grad)[j + i] << 16)
                         : static_cast<const float*>(t.grad)[j + i];
        if (k8) {
          cm |= (uint32_t) static_cast<const uint8_t*>(t.exp_avg)[j + i] << (8 * i);
          cv |= (uint32_t) static_cast<const uint8_t*>(t.exp_avg_sq)[j + i] << (8 * i);
        } else {
          m[i] = static_cast<const float*>(t.exp_avg)[j + i];
          v[i] = static_cast<const float*>(t.exp_avg_sq)[j + i];
        }
      }
      if (k8) {
        m = decode_e4m3x4(cm);
        v = decode_e4m3x4(cv);
      }
    }
    const int64_t qb = base / EQB_ADAMW_BLOCK;
    if (k8) {
      const float sm = t.exp_avg_scale[qb], sv = t.exp_avg_sq_scale[qb];
      for (int i = 0; i < 4; ++i) {
        m[i] = m[i] * sm;
        const float r = v[i] * sv;
        v[i] = r * r;
      }
    }
    f32x4 r;
    for (int i = 0; i < 4; ++i) {
      const float gi = g[i] * scale;
      m[i] = m[i] * batch.beta1 + gi * batch.rest1;
      v[i] = v[i] * batch.beta2 + (gi * batch.rest2) * gi;
      r[i] = sqrtf(v[i]);
      const float d = r[i] * batch.inv_root + batch.eps;
      w[i] = w[i] * t.keep - (m[i] / d) * batch.rate;
    }
    uint32_t cm = 0, cv = 0;
    if (k8) {
      float tm = 0.0f, tv = 0.0f;
      for (int i = 0; i < 4; ++i) {
        if (i < left) {
          tm = fmaxf(tm, fabsf(m[i]));
          tv = fmaxf(tv, r[i]);
        }
      }
      tm = wave_max(tm);
      tv = wave_max(tv);
      const float sm = tm < 0x1p-100f ? 0.0f : tm * (float)(1.0 / 448.0);
      const float sv = tv < 0x1p-100f ? 0.0f : tv * (float)(1.0 / 448.0);
      const float im = sm > 0.0f ? 1.0f / sm : 0.0f, iv = sv > 0.0f ? 1.0f / sv : 0.0f;
      for (int i = 0; i < 4; ++i) {
        const uint64_t e = (uint64_t)(j + i);
        const uint32_t h = mix32(((uint32_t)e + t.key) ^ ((uint32_t)(e >> 32) * 0x9E3779B1u));
        const float ym = fabsf(m[i]) * im, yv = r[i] * iv;
        uint32_t a = encode_e4m3(fminf(ym, 448.0f), h & 0xFFFFu);
        uint32_t b = encode_e4m3(fminf(yv, 448.0f), h >> 16);
        if (b == 0 && yv > 0.0f) b = 1;
        if (ym != ym) a = 0x7F;            // not a number stays one
        if (yv != yv) b = 0x7F;
        cm |= (a | (__float_as_uint(m[i]) >> 31 << 7)) << (8 * i);
        cv |= b << (8 * i);
      }
      if (lane == 0) {
        t.exp_avg_scale[qb] = sm;
        t.exp_avg_sq_scale[qb] = sv;
      }
    }
    if (left >= 4) {
      *reinterpret_cast<f32x4_any*>(t.param + j) = w;
      if (kCopy) {
        const uint32_t c0 = bf16x2_bits(w[0], w[1]), c1 = bf16x2_bits(w[2], w[3]);
        *reinterpret_cast<u16x4_any*>(t.copy + j) =
            u16x4{(uint16_t)c0, (uint16_t)(c0 >> 16), (uint16_t)c1, (uint16_t)(c1 >> 16)};
      }
      if (k8) {
        *reinterpret_cast<u32_any*>(static_cast<uint8_t*>(t.exp_avg) + j) = cm;
        *reinterpret_cast<u32_any*>(static_cast<uint8_t*>(t.exp_avg_sq) + j) = cv;
      } else {
        *reinterpret_cast<f32x4_any*>(static_cast<float*>(t.exp_avg) + j) = m;
        *reinterpret_cast<f32x4_any*>(static_cast<float*>(t.exp_avg_sq) + j) = v;
      }
    } else {
      for (int i = 0; i < left; ++i) {
        t.param[j + i] = w[i];
        if (kCopy) t.copy[j + i] = (uint16_t)bf16x2_bits(w[i], 0.0f);
        if (k8) {
          static_cast<uint8_t*>(t.exp_avg)[j + i] = (uint8_t)(cm >> (8 * i));
          static_cast<uint8_t*>(t.exp_avg_sq)[j + i] = (uint8_t)(cv >> (8 * i));
        } else {
          static_cast<float*>(t.exp_avg)[j + i] = m[i];
          static_cast<float*>(t.exp_avg_sq)[j + i] = v[i];
        }
      }
    }
  }
}

uint32_t adamw_blocks(int64_t numel) { return (uint32_t)((numel + kAdamwChunk - 1) / kAdamwChunk); }

template <bool k8, bool kGradBf16>
static void launch_adamw_as(const AdamwBatch& b, uint32_t blocks, hipStream_t s) {
  if (b.t[0].copy) adamw_kernel<k8, kGradBf16, true><<<blocks, kAdamwThreads, 0, s>>>(b);
  else adamw_kernel<k8, kGradBf16, false><<<blocks, kAdamwThreads, 0, s>>>(b);
}

eqb_status launch_adamw(const AdamwBatch& b, uint32_t blocks, bool eight, bool grad_bf16, hipStream_t s) {
  if (eight) {
    if (grad_bf16) launch_adamw_as<true, true>(b, blocks, s);
    else launch_adamw_as<true, false>(b, blocks, s);
  } else {
    if (grad_bf16) launch_adamw_as<false, true>(b, blocks, s);
    else launch_adamw_as<false, false>(b, blocks, s);
  }
  return launch_status();
}

}  // namespace eqb
