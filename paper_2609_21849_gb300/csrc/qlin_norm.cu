// Residual addition and root-mean-square norm, written as the 16-bit, FP8 or NVFP4
// input of the next linear:
//   s = x + residual,  n = s * (1 / sqrt(mean(s^2) + eps)) * weight.
// A row is an array of 16-byte chunks (8 elements); neighbouring threads take
// neighbouring chunks.  Two of them hold one NVFP4 block (K % 64 == 0: both inside).
//
// Bound by HBM: 2 bytes read (4 with a residual, 2 more for the sum) and 0.5625 to 2
// written per element.  A row stays in registers between its reduction and its output,
// so everything is read once: 4608 x 3072 bf16 with residual to FP8 rows 16.5 us, 99 MB
// at 90% of the measured copy rate; the same kernel with three reads per row took 28.
// Below that it is instructions: at 18432 x 3072 fp16 a run-time choice of the 16-bit
// type, bounds tests and tests for weight and residual in every chunk cost as many as
// the arithmetic (42 us; the type and the residual as template parameters, ones for a
// missing weight and a path without bounds tests: 29.5).  Copies ahead through shared
// memory (cp.async, three rows in flight per CTA) measured slower, 42.
#include "qlin_internal.h"

namespace qlin {

namespace {

enum class NormOut { k16, kFp8Rows, kFp8, kNvfp4 };

struct NormParams {
  const uint8_t* x;
  const uint8_t* residual;
  uint8_t* sum;
  const uint8_t* weight;
  int64_t x_row, residual_row, sum_row;   // bytes
  int64_t M, K;
  float one_over_K, eps;
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
// (x and residual are read once)
__device__ __forceinline__ uint4 ldg128_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// kF16: fp16 data, else bf16 (as a run-time choice both conversions were computed and
// one selected: a third of all instructions).
template <bool kF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (kF16)
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else
    return make_float2(bf16_lo(w), bf16_hi(w));
}

template <bool kF16>
__device__ __forceinline__ void unpack8(uint4 v, float2 (&f)[4]) {
  f[0] = unpack2<kF16>(v.x);
  f[1] = unpack2<kF16>(v.y);
  f[2] = unpack2<kF16>(v.z);
  f[3] = unpack2<kF16>(v.w);
}

template <bool kF16>
__device__ __forceinline__ uint4 pack8(const float2 (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = kF16 ? pack_f16x2(f[i].x, f[i].y) : pack_bf16x2(f[i].x, f[i].y);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float abs_max8(float m, const float2 (&f)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max_nan(m, max_nan(fabsf(f[i].x), fabsf(f[i].y)));
  return m;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(v));
  return r;
}

// The sum of a and the maximum of m over the threads of a row (a warp, or the CTA;
// red: an entry per warp, not written again before another barrier).
template <bool kWarpRow, bool kMax>
__device__ __forceinline__ float2 row_reduce(float a, float m, float2* red) {
  a = warp_sum(a);
  if (kMax) m = warp_max(m);
  if constexpr (!kWarpRow) {
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, m);
    __syncthreads();
    const int warps = (int)(blockDim.x >> 5);
    a = red[0].x;
    m = red[0].y;
    for (int w = 1; w < warps; ++w) {
      const float2 v = red[w];
      a += v.x;
      if (kMax) m = max_nan(m, v.y);
    }
  }
  return make_float2(a, m);
}

// 1 / sqrt(ss / K + eps); a row whose squares overflow takes them of s * 2^-80 instead
// (squares below 2^96, K < 2^31 of them).  With an infinity among s the result is 0: n is
// NaN there and 0 elsewhere.
constexpr float kDown = 0x1p-80f;
__device__ __forceinline__ float inverse_rms(float ss, float one_over_K, float eps) {
  return __frsqrt_rn(__fmaf_rn(ss, one_over_K, eps));
}

// The output of a chunk: 16-bit values, FP8 codes of n * s_enc, or half an NVFP4 block
// (the neighbouring lane has the other half; whole warps call).  y: the chunk's place in
// the output, c its number in the row.
template <NormOut kOut, bool kF16>
__device__ __forceinline__ void write_chunk(const NormParams& p, uint8_t* y, int64_t row, int c, bool own,
                                            float2 (&n)[4], float s_enc) {
  if constexpr (kOut == NormOut::k16) {
    if (own) *reinterpret_cast<uint4*>(y) = pack8<kF16>(n);
  } else if constexpr (kOut == NormOut::kNvfp4) {
    float amax = abs_max8(0.0f, n);
    amax = max_nan(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
    const uint32_t sb = e4m3_code_div6(__fmul_rn(amax, s_enc));
    const float r_b = sb == 0u ? 0.0f : __fdiv_rn(s_enc, e4m3_value(sb));
    float f[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 q = mul2(n[i], make_float2(r_b, r_b));
      f[2 * i] = q.x;
      f[2 * i + 1] = q.y;
    }
    if (own) *reinterpret_cast<uint32_t*>(y) = e2m1x8(f);
    if (own && (c & 1) == 0) p.block_scales[scale_offset(row, c / 2, p.K)] = (uint8_t)sb;
  } else {
    if (own)
      *reinterpret_cast<uint2*>(y) =
          make_uint2(e4m3x4(n[0].x, n[0].y, n[1].x, n[1].y), e4m3x4(n[2].x, n[2].y, n[3].x, n[3].y));
  }
}
// Bytes of a chunk's output.
template <NormOut kOut>
constexpr int kOutChunk = kOut == NormOut::k16 ? 16 : kOut == NormOut::kNvfp4 ? 4 : 8;

// s of one chunk from x and the residual, its squares added to ss.
template <bool kF16, bool kResidual>
__device__ __forceinline__ void add_chunk(uint4 x, uint4 r, float2 (&s)[4], float2& ss) {
  unpack8<kF16>(x, s);
  if (kResidual) {
    float2 f[4];
    unpack8<kF16>(r, f);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = add2(s[i], f[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) ss = fma2(s[i], s[i], ss);
}

// s * pre * weight of one chunk.
template <bool kF16>
__device__ __forceinline__ void weigh(float2 (&s)[4], float pre, const uint4& w) {
  float2 f[4];
  unpack8<kF16>(w, f);
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = mul2(mul2(s[i], make_float2(pre, pre)), f[i]);
}

// A weight of ones (without one).
template <bool kF16>
__device__ __forceinline__ uint4 ones() {
  const uint32_t w = kF16 ? 0x3C003C00u : 0x3F803F80u;
  return make_uint4(w, w, w, w);
}

// The factor of s in FP8 codes, (s * pre) * weight: 448 / max |s * weight| for a scale per
// row (tot: the row's sum of squares and that maximum, found in one reduction, since
// max |n| is the maximum / rms), inv * f for a static one.  False where a factor or a
// product with it could overflow (|s * inv| <= sqrt(K)); codes are then n * f, n = (s *
// inv) * weight, with f of max |n|.
template <NormOut kOut>
__device__ __forceinline__ bool fp8_factor(float2 tot, float inv, float f, float& pre, float& s_dec) {
  if constexpr (kOut == NormOut::kFp8Rows) {
    if (!(tot.x <= FLT_MAX && tot.y >= 0x1p-50f && tot.y <= FLT_MAX)) return false;
    pre = __fdiv_rn(448.0f, tot.y);   // (exact ties stay ties, and any finite maximum)
    s_dec = __fmul_rn(__fmul_rn(tot.y, inv), 1.0f / 448.0f);
  } else {
    if (!(f >= 0x1p-64f && f <= 0x1p64f && inv >= 0x1p-60f)) return false;
    pre = __fmul_rn(inv, f);
  }
  return true;
}

// A row from registers: chunks tid, tid + T, ... of thread tid of the row's T.  kFull:
// every thread has kChunks of them.
template <NormOut kOut, bool kF16, bool kResidual, int kChunks, bool kWarpRow, bool kFull>
__device__ __forceinline__ void held_row(const NormParams& p, int64_t row, int tid, int T, int chunks,
                                         float2* red) {
  auto in = [&](int i) { return kFull || tid + i * T < chunks; };
  uint4 vx[kChunks], vr[kChunks], vw[kChunks];
  {
    const uint8_t* const x = p.x + row * p.x_row + 16 * tid;
    const uint8_t* const r = kResidual ? p.residual + row * p.residual_row + 16 * tid : nullptr;
    const uint8_t* const w = p.weight + 16 * tid;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (!in(i)) continue;
      vx[i] = ldg128_once(x + 16 * i * T);
      if (kResidual) vr[i] = ldg128_once(r + 16 * i * T);
    }
    if (p.weight != nullptr) {
#pragma unroll
      for (int i = 0; i < kChunks; ++i)
        if (in(i)) vw[i] = ldg128(w + 16 * i * T);
    } else {
#pragma unroll
      for (int i = 0; i < kChunks; ++i) vw[i] = ones<kF16>();
    }
  }
  float s_dec = 1.0f, f = 1.0f;
  if constexpr (kOut == NormOut::kFp8 || kOut == NormOut::kNvfp4) {
    s_dec = *p.static_scale;
    if (row == 0 && tid == 0 && p.scale != p.static_scale) *p.scale = s_dec;
    f = encode_scale(s_dec);
  }
  float2 s[kChunks][4], ss = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < kChunks; ++i) {
    if (in(i)) {
      add_chunk<kF16, kResidual>(vx[i], vr[i], s[i], ss);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) s[i][k] = make_float2(0.0f, 0.0f);
      vw[i] = ones<kF16>();
    }
  }
  if (kResidual && p.sum != nullptr) {
    uint8_t* const sum = p.sum + row * p.sum_row + 16 * tid;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      if (in(i)) *reinterpret_cast<uint4*>(sum + 16 * i * T) = pack8<kF16>(s[i]);
  }
  // max |s * pre * weight|
  auto peak = [&](float pre) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      float2 t[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) t[k] = s[i][k];
      weigh<kF16>(t, pre, vw[i]);
      m = abs_max8(m, t);
    }
    return m;
  };
  float m = 0.0f;
  if (kOut == NormOut::kFp8Rows) m = peak(1.0f);
  const float2 tot = row_reduce<kWarpRow, kOut == NormOut::kFp8Rows>(ss.x + ss.y, m, red);
  float inv;
  if (tot.x <= FLT_MAX) {
    inv = inverse_rms(tot.x, p.one_over_K, p.eps);
  } else {               // squares overflowed, or an infinity or a NaN
    float2 s2 = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 v = mul2(s[i][k], make_float2(kDown, kDown));
        s2 = fma2(v, v, s2);
      }
    inv = inverse_rms(row_reduce<kWarpRow, false>(s2.x + s2.y, 0.0f, red + 32).x, p.one_over_K, 0.0f) * kDown;
  }
  float pre = inv;
  bool one = true;
  if constexpr (kOut == NormOut::kFp8Rows || kOut == NormOut::kFp8) {
    one = fp8_factor<kOut>(tot, inv, f, pre, s_dec);
    if (kOut == NormOut::kFp8Rows) {
      if (!one) {
        m = row_reduce<kWarpRow, true>(0.0f, peak(inv), red + 64).y;
        s_dec = m == 0.0f ? 1.0f : __fdiv_rn(m, 448.0f);
        f = encode_scale(s_dec);
      }
      if (tid == 0) p.scale[row] = s_dec;
    }
  }
#pragma unroll
  for (int i = 0; i < kChunks; ++i) weigh<kF16>(s[i], pre, vw[i]);
  if (!one) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[i][k] = mul2(s[i][k], make_float2(f, f));
  }
  uint8_t* const y = p.y + (row * (p.K / 8) + tid) * kOutChunk<kOut>;
#pragma unroll
  for (int i = 0; i < kChunks; ++i)
    write_chunk<kOut, kF16>(p, y + i * T * kOutChunk<kOut>, row, tid + i * T, in(i), s[i], f);
}

// A row per CTA, or per warp, held in registers in fp32 between its reduction and its
// output: x and the residual are read once.  (Four chunks: 80 registers, so that two
// CTAs of a 12288-element row fit an SM; 2048 such rows 37.0 us with 82, now 28.3.)
template <NormOut kOut, bool kF16, bool kResidual, int kChunks, bool kWarpRow>
__global__ void __launch_bounds__(kWarpRow ? 256 : kChunks == 2 ? 1024 : 768)
    rmsnorm_held_kernel(const NormParams p) {
  __shared__ float2 red[kWarpRow ? 1 : 3 * 32];
  const int tid = kWarpRow ? threadIdx.x & 31 : threadIdx.x;
  const int T = kWarpRow ? 32 : (int)blockDim.x;
  const int64_t row = kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5) : blockIdx.x;
  const int chunks = (int)(p.K / 8);
  grid_dep_wait();
  grid_dep_launch();
  if (row >= p.M) return;   // (whole warps)
  if (chunks == kChunks * T)
    held_row<kOut, kF16, kResidual, kChunks, kWarpRow, true>(p, row, tid, T, chunks, red);
  else
    held_row<kOut, kF16, kResidual, kChunks, kWarpRow, false>(p, row, tid, T, chunks, red);
}

// Rows beyond the registers of a CTA: one CTA per row, which it reads once per pass
// (squares and maximum; output), by the same formulas.  The sum is written in the last
// pass, by the thread that reads the same elements, so that it may be x or residual.
constexpr int kLongThreads = 512;

template <NormOut kOut, bool kF16, bool kResidual>
__global__ void __launch_bounds__(kLongThreads) rmsnorm_long_kernel(const NormParams p) {
  __shared__ float2 red[3 * 32];
  const int64_t row = blockIdx.x;
  const int chunks = (int)(p.K / 8);
  const uint8_t* const x = p.x + row * p.x_row;
  const uint8_t* const r = p.residual + row * p.residual_row;
  grid_dep_wait();
  grid_dep_launch();
  auto load = [&](int c, float2 (&s)[4], float2& ss) {
    const uint4 a = ldg128(x + 16 * (int64_t)c);
    add_chunk<kF16, kResidual>(a, kResidual ? ldg128(r + 16 * (int64_t)c) : a, s, ss);
  };
  auto load_w = [&](int c) { return p.weight != nullptr ? ldg128(p.weight + 16 * (int64_t)c) : ones<kF16>(); };
  float2 s[4], ss = make_float2(0.0f, 0.0f), unused = ss;
  // max |s * pre * weight| of chunk c's s
  auto peak = [&](float m, int c, float pre) {
    weigh<kF16>(s, pre, load_w(c));
    return abs_max8(m, s);
  };
  float m = 0.0f;
  for (int c = threadIdx.x; c < chunks; c += kLongThreads) {
    load(c, s, ss);
    if (kOut == NormOut::kFp8Rows) m = peak(m, c, 1.0f);
  }
  const float2 tot = row_reduce<false, kOut == NormOut::kFp8Rows>(ss.x + ss.y, m, red);
  float inv;
  if (tot.x <= FLT_MAX) {
    inv = inverse_rms(tot.x, p.one_over_K, p.eps);
  } else {
    ss = make_float2(0.0f, 0.0f);
    for (int c = threadIdx.x; c < chunks; c += kLongThreads) {
      load(c, s, unused);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 v = mul2(s[k], make_float2(kDown, kDown));
        ss = fma2(v, v, ss);
      }
    }
    inv = inverse_rms(row_reduce<false, false>(ss.x + ss.y, 0.0f, red + 32).x, p.one_over_K, 0.0f) * kDown;
  }
  float f = 1.0f, s_dec = 1.0f, pre = inv;
  if constexpr (kOut == NormOut::kFp8 || kOut == NormOut::kNvfp4) {
    s_dec = *p.static_scale;
    if (row == 0 && threadIdx.x == 0 && p.scale != p.static_scale) *p.scale = s_dec;
    f = encode_scale(s_dec);
  }
  bool one = true;
  if constexpr (kOut == NormOut::kFp8Rows || kOut == NormOut::kFp8) {
    one = fp8_factor<kOut>(tot, inv, f, pre, s_dec);
    if (kOut == NormOut::kFp8Rows) {
      if (!one) {
        m = 0.0f;
        for (int c = threadIdx.x; c < chunks; c += kLongThreads) {
          load(c, s, unused);
          m = peak(m, c, inv);
        }
        m = row_reduce<false, true>(0.0f, m, red + 64).y;
        s_dec = m == 0.0f ? 1.0f : __fdiv_rn(m, 448.0f);
        f = encode_scale(s_dec);
      }
      if (threadIdx.x == 0) p.scale[row] = s_dec;
    }
  }
  for (int c0 = 0; c0 < chunks; c0 += kLongThreads) {
    const int c = c0 + (int)threadIdx.x;
    const bool own = c < chunks;
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = make_float2(0.0f, 0.0f);
    if (own) {
      load(c, s, unused);
      if (kResidual && p.sum != nullptr)
        *reinterpret_cast<uint4*>(p.sum + row * p.sum_row + 16 * (int64_t)c) = pack8<kF16>(s);
      weigh<kF16>(s, pre, load_w(c));
      if (!one) {
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = mul2(s[k], make_float2(f, f));
      }
    }
    write_chunk<kOut, kF16>(p, p.y + (row * (p.K / 8) + c) * kOutChunk<kOut>, row, c, own, s, f);
  }
}

template <NormOut kOut, bool kF16, bool kResidual>
cudaError_t launch_out(const NormParams& p, int num_sms, cudaStream_t s) {
  const int64_t chunks = p.K / 8;
  if (chunks <= 128) {
    const unsigned grid = (unsigned)((p.M + 7) / 8);
    return chunks <= 32   ? launch_pdl(rmsnorm_held_kernel<kOut, kF16, kResidual, 1, true>, grid, 256, 0, s, p)
           : chunks <= 64 ? launch_pdl(rmsnorm_held_kernel<kOut, kF16, kResidual, 2, true>, grid, 256, 0, s, p)
                          : launch_pdl(rmsnorm_held_kernel<kOut, kF16, kResidual, 4, true>, grid, 256, 0, s, p);
  }
  // Four chunks per thread halve a row's share of the reduction (18432 x 3072 fp16 to
  // static FP8 31.0 us, with two 36.2; 2255 x 6208 to FP8 rows 18.2 and 20.8); two leave
  // fewer threads idle in short rows that four do not divide (5468 x 2560 to static FP8
  // 10.8 against 11.4) and have the shorter chain where rows are few (300 x 6208 4.1
  // against 4.5), up to where their CTAs fill an SM (300 x 9216 6.3 against 4.9).
  if (chunks > 2048)
    return launch_pdl(rmsnorm_long_kernel<kOut, kF16, kResidual>, (unsigned)p.M, kLongThreads, 0, s, p);
  if (chunks > 1024 || (p.M >= 4 * num_sms && (chunks % 128 == 0 || chunks >= 384)))
    return launch_pdl(rmsnorm_held_kernel<kOut, kF16, kResidual, 4, false>, (unsigned)p.M,
                      (int)((chunks + 127) / 128) * 32, 0, s, p);
  const int threads = (int)((chunks + 63) / 64) * 32;
  return launch_pdl(rmsnorm_held_kernel<kOut, kF16, kResidual, 2, false>, (unsigned)p.M, threads, 0, s, p);
}

template <NormOut kOut>
cudaError_t launch_types(const NormParams& p, int dtype, int num_sms, cudaStream_t s) {
  if (dtype == QLIN_FP16)
    return p.residual != nullptr ? launch_out<kOut, true, true>(p, num_sms, s)
                                 : launch_out<kOut, true, false>(p, num_sms, s);
  return p.residual != nullptr ? launch_out<kOut, false, true>(p, num_sms, s)
                               : launch_out<kOut, false, false>(p, num_sms, s);
}

}  // namespace

cudaError_t launch_rmsnorm(const qlin_rmsnorm_t& a, void* y16, const float* static_scale,
                           const qlin_fp8_t* fp8, const qlin_nvfp4_t* nvfp4, cudaStream_t s, Device dev) {
  NormParams p{};
  p.x = static_cast<const uint8_t*>(a.x);
  p.residual = static_cast<const uint8_t*>(a.residual);
  p.sum = static_cast<uint8_t*>(a.sum);
  p.weight = static_cast<const uint8_t*>(a.weight);
  p.x_row = a.x_stride * 2;
  p.residual_row = a.residual_stride * 2;
  p.sum_row = a.sum_stride * 2;
  p.M = a.M;
  p.K = a.K;
  p.one_over_K = 1.0f / (float)a.K;
  p.eps = a.eps;
  p.static_scale = static_scale;
  p.y = static_cast<uint8_t*>(y16);
  if (fp8 != nullptr) {
    p.y = fp8->codes;
    p.scale = fp8->scale;
    return fp8->per_channel ? launch_types<NormOut::kFp8Rows>(p, a.dtype, dev.num_sms, s) : launch_types<NormOut::kFp8>(p, a.dtype, dev.num_sms, s);
  }
  if (nvfp4 != nullptr) {
    p.y = nvfp4->codes;
    p.scale = nvfp4->tensor_scale;
    p.block_scales = nvfp4->scales;
    return launch_types<NormOut::kNvfp4>(p, a.dtype, dev.num_sms, s);
  }
  return launch_types<NormOut::k16>(p, a.dtype, dev.num_sms, s);
}

}  // namespace qlin
