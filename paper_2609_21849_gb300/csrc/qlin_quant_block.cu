// The block-scaled FP8 quantizer: one scale for each 128 elements of a row (activations)
// or for each 128 x 128 (weights), so that an outlier spoils the codes of its block alone.
//   S = max |x over the block| / 448 (1 for a block of zeros), code = E4M3(x / S as x * (1 / S)).
// Bound by HBM: 2 bytes in and 1 out per element (and a scale per block), one read of x that
// stays in registers between a block's maximum and its codes.
//   rows:  eight lanes hold a block of 128, 16 elements each, so that its maximum is three shuffles;
//          a warp's four blocks are four rows of one block of K where there are rows enough (their
//          scales adjacent), else four blocks of a row.
//   tiles: a CTA of 512 threads holds 128 x 128 values, 32 each, and joins the maxima in shared memory.
// Measured: 4608 x 12288 27.4 us, 94% of the copy rate; 12288 x 3072 in tiles 20.0, 84% (the codes of
// a tile wait for its last value); one row of 3072 1.4, a launch.
#include "qlin_internal.h"

namespace qlin {

namespace {

constexpr int kRowThreads = 256;   // row blocks: eight lanes to a block
constexpr int kTileThreads = 512;  // 128 x 128 blocks: one CTA each

struct BlockParams {
  const uint16_t* x;
  int64_t x_stride;   // elements
  uint8_t* codes;
  float* scales;
  int64_t rows, K;
  int64_t scale_rows;
  int kblocks;
  int rows4;          // row blocks: a warp takes four rows of one block of K (else four blocks of a row)
};

// max(|a|, |b|) of two pairs of 16-bit floats, as bits: a NaN is above every number.
__device__ __forceinline__ uint32_t absmax2(uint32_t m, uint32_t w) {
  return __vmaxu2(m, w & 0x7FFF7FFFu);
}

template <bool kF16>
__device__ __forceinline__ float2 unpack(uint32_t w) {
  if constexpr (kF16)
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else
    return make_float2(bf16_lo(w), bf16_hi(w));
}

template <bool kF16>
__device__ __forceinline__ float value16(uint32_t bits) {
  return unpack<kF16>(bits).x;
}

__device__ __forceinline__ float block_scale(float amax) {
  return amax == 0.0f ? 1.0f : __fdiv_rn(amax, 448.0f);
}

// Eight elements' codes.
template <bool kF16>
__device__ __forceinline__ uint2 codes8(uint4 w, float s_enc) {
  float2 a = unpack<kF16>(w.x), b = unpack<kF16>(w.y), c = unpack<kF16>(w.z), d = unpack<kF16>(w.w);
  mul2_rn(a.x, a.y, s_enc);
  mul2_rn(b.x, b.y, s_enc);
  mul2_rn(c.x, c.y, s_enc);
  mul2_rn(d.x, d.y, s_enc);
  return make_uint2(e4m3x4(a.x, a.y, b.x, b.y), e4m3x4(c.x, c.y, d.x, d.y));
}

__device__ __forceinline__ uint4 ld16(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// Row blocks.  Lane l of eight holds elements 16 l .. 16 l + 15 of a block.
template <bool kF16>
__global__ void __launch_bounds__(kRowThreads) quant_rows128_kernel(const BlockParams p) {
  grid_dep_wait();
  grid_dep_launch();
  const int64_t group = ((int64_t)blockIdx.x * kRowThreads + threadIdx.x) >> 3;
  const int sub = threadIdx.x & 7;
  int64_t row, kb;
  if (p.rows4) {
    const int64_t unit = group >> 2;   // (four rows, block of K), blocks of K fastest
    row = unit / p.kblocks * 4 + (group & 3);
    kb = unit % p.kblocks;
  } else {
    row = group / p.kblocks;
    kb = group % p.kblocks;
  }
  const int64_t k = kb * 128 + sub * 16;
  const bool in = row < p.rows && k < p.K;   // (K ends after 64 elements of a block, at most)
  uint4 v[2] = {make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  if (in) {
    const uint16_t* const src = p.x + row * p.x_stride + k;
    v[0] = ld16(src);
    v[1] = ld16(src + 8);
  }
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < 2; ++i) m = absmax2(absmax2(absmax2(absmax2(m, v[i].x), v[i].y), v[i].z), v[i].w);
  m = max(m & 0xFFFFu, m >> 16);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const float s = block_scale(value16<kF16>(m)), s_enc = encode_scale(s);
  if (!in) return;
  const uint2 a = codes8<kF16>(v[0], s_enc), b = codes8<kF16>(v[1], s_enc);
  *reinterpret_cast<uint4*>(p.codes + row * p.K + k) = make_uint4(a.x, a.y, b.x, b.y);
  if (sub == 0) p.scales[kb * p.scale_rows + row] = s;
}

// 128 x 128 blocks: a thread holds 16 bytes of four rows.
template <bool kF16>
__global__ void __launch_bounds__(kTileThreads) quant_tiles128_kernel(const BlockParams p) {
  constexpr int kPer = 128 * 16 / kTileThreads;
  __shared__ uint32_t warp_max[kTileThreads / 32];
  grid_dep_wait();
  grid_dep_launch();
  const int64_t rb = blockIdx.x / (unsigned)p.kblocks, kb = blockIdx.x % (unsigned)p.kblocks;
  const int64_t k = kb * 128 + (threadIdx.x & 15) * 8;
  const int64_t row0 = rb * 128 + (threadIdx.x >> 4);
  uint4 v[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t row = row0 + i * (kTileThreads / 16);
    v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (row < p.rows && k < p.K) v[i] = ld16(p.x + row * p.x_stride + k);
  }
  uint32_t m = 0u;
#pragma unroll
  for (int i = 0; i < kPer; ++i) m = absmax2(absmax2(absmax2(absmax2(m, v[i].x), v[i].y), v[i].z), v[i].w);
  m = __reduce_max_sync(0xFFFFFFFFu, max(m & 0xFFFFu, m >> 16));
  if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kTileThreads / 32; ++i) m = max(m, warp_max[i]);
  const float s = block_scale(value16<kF16>(m)), s_enc = encode_scale(s);
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int64_t row = row0 + i * (kTileThreads / 16);
    if (row < p.rows && k < p.K) *reinterpret_cast<uint2*>(p.codes + row * p.K + k) = codes8<kF16>(v[i], s_enc);
  }
  if (threadIdx.x == 0) p.scales[kb * p.scale_rows + rb] = s;
}

}  // namespace

cudaError_t launch_quant_fp8_block(const void* x, int64_t x_stride, bool fp16, const qlin_fp8_block_t& out,
                                   cudaStream_t s) {
  BlockParams p{};
  p.x = static_cast<const uint16_t*>(x);
  p.x_stride = x_stride;
  p.codes = out.codes;
  p.scales = out.scales;
  p.rows = out.rows;
  p.K = out.K;
  p.scale_rows = (out.rows + out.block_rows - 1) / out.block_rows;
  p.kblocks = (int)((out.K + 127) / 128);
  if (out.block_rows == 128) {
    const dim3 grid((unsigned)(p.scale_rows * p.kblocks));
    return fp16 ? launch_pdl(quant_tiles128_kernel<true>, grid, kTileThreads, 0, s, p)
                : launch_pdl(quant_tiles128_kernel<false>, grid, kTileThreads, 0, s, p);
  }
  p.rows4 = out.rows >= 4 ? 1 : 0;
  const int64_t groups = p.rows4 ? (out.rows + 3) / 4 * 4 * p.kblocks : out.rows * p.kblocks;
  const dim3 grid((unsigned)((groups * 8 + kRowThreads - 1) / kRowThreads));
  return fp16 ? launch_pdl(quant_rows128_kernel<true>, grid, kRowThreads, 0, s, p)
              : launch_pdl(quant_rows128_kernel<false>, grid, kRowThreads, 0, s, p);
}

}  // namespace qlin
