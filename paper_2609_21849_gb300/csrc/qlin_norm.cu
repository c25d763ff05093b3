// Residual addition and root-mean-square norm, written as the 16-bit, FP8 or NVFP4
// input of the next linear:
//   s = x + residual,  n = s * (1 / sqrt(mean(s^2) + eps)) * weight.
// A unit is 16 elements of a row: one NVFP4 block, 16 bytes of FP8 codes.
#include "qlin_internal.h"

namespace qlin {

namespace {

constexpr int kThreads = 256;

enum class NormOut { k16, kFp8Rows, kFp8, kNvfp4 };

struct NormParams {
  const uint8_t* x;
  const uint8_t* residual;
  uint8_t* sum;
  const uint8_t* weight;
  int64_t x_row, residual_row, sum_row;   // bytes
  int64_t K;
  float eps;
  int fp16;
  const float* static_scale;
  float* scale;        // FP8 / NVFP4: receives the static scale, or a scale per row
  uint8_t* y;          // 16-bit values or codes
  uint8_t* block_scales;
};

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// Loads that stay after the grid dependency wait (volatile, as that is).
__device__ __forceinline__ uint4 ldg128(const void* p) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

__device__ __forceinline__ void unpack2(uint32_t w, bool fp16, float& lo, float& hi) {
  if (fp16) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
  } else {
    lo = bf16_lo(w);
    hi = bf16_hi(w);
  }
}

__device__ __forceinline__ void load16(const uint8_t* p, bool fp16, float (&f)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint4 v = ldg128(p + 16 * h);
    unpack2(v.x, fp16, f[8 * h], f[8 * h + 1]);
    unpack2(v.y, fp16, f[8 * h + 2], f[8 * h + 3]);
    unpack2(v.z, fp16, f[8 * h + 4], f[8 * h + 5]);
    unpack2(v.w, fp16, f[8 * h + 6], f[8 * h + 7]);
  }
}

__device__ __forceinline__ void store16(uint8_t* p, bool fp16, const float (&f)[16]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float lo = f[8 * h + 2 * i], hi = f[8 * h + 2 * i + 1];
      w[i] = fp16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
    }
    *reinterpret_cast<uint4*>(p + 16 * h) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

__device__ __forceinline__ float block_reduce(float v, bool maximum, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xFFFFFFFFu, v, o);
    v = maximum ? max_nan(v, u) : v + u;
  }
  __syncthreads();   // red's last readers are done
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) v = maximum ? max_nan(v, red[w]) : v + red[w];
  return v;
}

// 1 / sqrt(ss / K + eps); a row whose squares overflowed takes them of s * 2^-80
// instead (2^-80 times the largest sum of two 16-bit values squares to 2^98).
constexpr float kDown = 0x1p-80f;
__device__ __forceinline__ float inverse_rms(float ss, float K, float eps) {
  return __frsqrt_rn(__fadd_rn(__fdiv_rn(ss, K), eps));
}

// The 16 codes of one unit.
template <NormOut kOut>
__device__ __forceinline__ void write_unit(const NormParams& p, int64_t row, int u,
                                           const float (&n)[16], float s_enc) {
  if constexpr (kOut == NormOut::k16) {
    store16(p.y + (row * p.K + 16 * u) * 2, p.fp16 != 0, n);
  } else if constexpr (kOut == NormOut::kNvfp4) {
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) amax = max_nan(amax, fabsf(n[i]));
    const uint32_t sb = e4m3_code_div6(__fmul_rn(amax, s_enc));
    const float r_b = sb == 0u ? 0.0f : __fdiv_rn(s_enc, e4m3_value(sb));
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __fmul_rn(n[8 * h + i], r_b);
      w[h] = e2m1x8(f);
    }
    *reinterpret_cast<uint2*>(p.y + row * (p.K / 2) + 8 * u) = make_uint2(w[0], w[1]);
    p.block_scales[scale_offset(row, u, p.K)] = (uint8_t)sb;
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = e4m3x4(__fmul_rn(n[4 * i], s_enc), __fmul_rn(n[4 * i + 1], s_enc),
                    __fmul_rn(n[4 * i + 2], s_enc), __fmul_rn(n[4 * i + 3], s_enc));
    *reinterpret_cast<uint4*>(p.y + row * p.K + 16 * u) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// One CTA per row, which it reads once per pass (sum of squares; FP8 rows: the
// maximum; output).  sum is written in the last pass, by the thread that reads the
// same elements, so that it may be x or residual.
template <NormOut kOut>
__global__ void __launch_bounds__(kThreads) rmsnorm_kernel(const NormParams p) {
  __shared__ float red[kThreads / 32];
  const int64_t row = blockIdx.x;
  const bool fp16 = p.fp16 != 0;
  const int units = (int)(p.K / 16);
  const uint8_t* const x = p.x + row * p.x_row;
  const uint8_t* const r = p.residual == nullptr ? nullptr : p.residual + row * p.residual_row;
  grid_dep_wait();
  grid_dep_launch();
  auto load_s = [&](int u, float (&s)[16]) {
    load16(x + 32 * (int64_t)u, fp16, s);
    if (r != nullptr) {
      float f[16];
      load16(r + 32 * (int64_t)u, fp16, f);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __fadd_rn(s[i], f[i]);
    }
  };
  auto load_n = [&](const float (&s)[16], int u, float inv, float (&n)[16]) {
    float w[16];
    if (p.weight != nullptr) load16(p.weight + 32 * (int64_t)u, fp16, w);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      n[i] = __fmul_rn(s[i], inv);
      if (p.weight != nullptr) n[i] = __fmul_rn(n[i], w[i]);
    }
  };
  auto squares = [&](float pre) {
    float ss = 0.0f, s[16];
    for (int u = threadIdx.x; u < units; u += kThreads) {
      load_s(u, s);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float v = s[i] * pre;
        ss = __fmaf_rn(v, v, ss);
      }
    }
    return block_reduce(ss, false, red);
  };
  float ss = squares(1.0f), inv;
  if (ss <= FLT_MAX)
    inv = inverse_rms(ss, (float)p.K, p.eps);
  else
    inv = inverse_rms(squares(kDown), (float)p.K, 0.0f) * kDown;
  float s_enc = 0.0f;
  if constexpr (kOut == NormOut::kFp8Rows) {
    float amax = 0.0f, s[16], n[16];
    for (int u = threadIdx.x; u < units; u += kThreads) {
      load_s(u, s);
      load_n(s, u, inv, n);
#pragma unroll
      for (int i = 0; i < 16; ++i) amax = max_nan(amax, fabsf(n[i]));
    }
    amax = block_reduce(amax, true, red);
    const float s_dec = amax == 0.0f ? 1.0f : __fdiv_rn(amax, 448.0f);
    if (threadIdx.x == 0) p.scale[row] = s_dec;
    s_enc = encode_scale(s_dec);
  } else if constexpr (kOut != NormOut::k16) {
    const float s_dec = *p.static_scale;
    if (row == 0 && threadIdx.x == 0 && p.scale != p.static_scale) *p.scale = s_dec;
    s_enc = encode_scale(s_dec);
  }
  for (int u = threadIdx.x; u < units; u += kThreads) {
    float s[16], n[16];
    load_s(u, s);
    load_n(s, u, inv, n);
    if (p.sum != nullptr) store16(p.sum + row * p.sum_row + 32 * (int64_t)u, fp16, s);
    write_unit<kOut>(p, row, u, n, s_enc);
  }
}

}  // namespace

cudaError_t launch_rmsnorm(const qlin_rmsnorm_t& a, void* y16, const float* static_scale,
                           const qlin_fp8_t* fp8, const qlin_nvfp4_t* nvfp4, cudaStream_t s) {
  NormParams p{};
  p.x = static_cast<const uint8_t*>(a.x);
  p.residual = static_cast<const uint8_t*>(a.residual);
  p.sum = static_cast<uint8_t*>(a.sum);
  p.weight = static_cast<const uint8_t*>(a.weight);
  p.x_row = a.x_stride * 2;
  p.residual_row = a.residual_stride * 2;
  p.sum_row = a.sum_stride * 2;
  p.K = a.K;
  p.eps = a.eps;
  p.fp16 = a.dtype == QLIN_FP16 ? 1 : 0;
  p.static_scale = static_scale;
  p.y = static_cast<uint8_t*>(y16);
  auto kern = rmsnorm_kernel<NormOut::k16>;
  if (fp8 != nullptr) {
    p.y = fp8->codes;
    p.scale = fp8->scale;
    kern = fp8->per_channel ? rmsnorm_kernel<NormOut::kFp8Rows> : rmsnorm_kernel<NormOut::kFp8>;
  } else if (nvfp4 != nullptr) {
    p.y = nvfp4->codes;
    p.scale = nvfp4->tensor_scale;
    p.block_scales = nvfp4->scales;
    kern = rmsnorm_kernel<NormOut::kNvfp4>;
  }
  return launch_pdl(kern, (unsigned)a.M, kThreads, 0, s, p);
}

}  // namespace qlin
