// Rotary positions.  The angle of a pair is position * f, held as turns: a pair's
// turns per position are a 64-bit fraction (units of 2^-64 turn), so that position *
// turns modulo 2^64 is the angle without whole turns, exact for every position; its
// top 32 bits give the angle to 2^-32 turn.  (In fp32 the product alone is off by
// 0.03 radians at position 10^6.)
#include "qlin_internal.h"

namespace qlin {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 512;   // head_dim <= 1024

struct RopeParams {
  const uint16_t* x;
  uint16_t* y;
  int64_t x_token, x_head, y_token, y_head;   // elements
  const void* positions;
  int64_t pos_token, pos_axis;
  const uint64_t* turns;
  float magnitude;
  int heads, head_dim, pairs;
  int pos64;
  int axis_end[3];   // first pairs of the second, third and fourth axis
  int half, inverse, fp16;
};

__device__ __forceinline__ float load16(const uint16_t* p, bool fp16) {
  const uint16_t w = *p;
  return fp16 ? __half2float(__ushort_as_half(w)) : __uint_as_float((uint32_t)w << 16);
}

__device__ __forceinline__ uint16_t pack16(float v, bool fp16) {
  return (uint16_t)(fp16 ? pack_f16x2(v, 0.0f) : pack_bf16x2(v, 0.0f));
}

// (cos, sin) of pair i at the token's positions, times the magnitude.
__device__ __forceinline__ float2 rotation(const RopeParams& p, int64_t token, int i) {
  const int axis = (i >= p.axis_end[0]) + (i >= p.axis_end[1]) + (i >= p.axis_end[2]);
  const int64_t at = token * p.pos_token + axis * p.pos_axis;
  const int64_t pos = p.pos64 ? static_cast<const int64_t*>(p.positions)[at]
                              : (int64_t)static_cast<const int32_t*>(p.positions)[at];
  const uint64_t t = (uint64_t)pos * p.turns[i];
  // a signed 32-bit fraction of a turn is twice as many half turns
  float s, c;
  sincospif((float)(int32_t)(uint32_t)(t >> 32) * 0x1p-31f, &s, &c);
  if (p.inverse) s = -s;
  return make_float2(c * p.magnitude, s * p.magnitude);
}

// One CTA per token: the rotations of its pairs once, then the heads.
__global__ void __launch_bounds__(kThreads) rope_kernel(const RopeParams p) {
  __shared__ float2 rot[kMaxPairs];
  const int64_t token = blockIdx.x;
  const bool fp16 = p.fp16 != 0;
  grid_dep_wait();
  grid_dep_launch();
  for (int i = threadIdx.x; i < p.pairs; i += kThreads) rot[i] = rotation(p, token, i);
  __syncthreads();
  const int rest = p.head_dim - 2 * p.pairs;
  const int per_head = p.pairs + rest;
  for (int j = threadIdx.x; j < p.heads * per_head; j += kThreads) {
    const int head = j / per_head, i = j % per_head;
    const uint16_t* const x = p.x + token * p.x_token + head * p.x_head;
    uint16_t* const y = p.y + token * p.y_token + head * p.y_head;
    if (i >= p.pairs) {
      const int d = i + p.pairs;
      y[d] = x[d];
      continue;
    }
    const int da = p.half ? i : 2 * i, db = p.half ? i + p.pairs : 2 * i + 1;
    const float a = load16(x + da, fp16), b = load16(x + db, fp16);
    const float2 r = rot[i];
    y[da] = pack16(__fsub_rn(__fmul_rn(a, r.x), __fmul_rn(b, r.y)), fp16);
    y[db] = pack16(__fadd_rn(__fmul_rn(a, r.y), __fmul_rn(b, r.x)), fp16);
  }
}

// ---- 16-byte accesses ----
// An item is eight pairs of one head (16 elements: two chunks of 8, eight pairs
// apart in the half layout, adjacent in the interleaved one), or a chunk past
// rot_dim.  A CTA takes whole tokens; each thread issues the loads of its first items
// before the rotations are computed, which overlap them.
constexpr int kItems = 2;

__device__ __forceinline__ uint4 ldg128(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

template <bool kF16>
__device__ __forceinline__ void unpack8(const uint4 v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kF16) {
      const float2 h = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = h.x;
      f[2 * i + 1] = h.y;
    } else {
      f[2 * i] = bf16_lo(w[i]);
      f[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}

template <bool kF16>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = kF16 ? pack_f16x2(f[2 * i], f[2 * i + 1]) : pack_bf16x2(f[2 * i], f[2 * i + 1]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// (a, b) of a pair turned by r = (cos, sin).
__device__ __forceinline__ void turn(float& a, float& b, float c, float s) {
  const float x = a;
  a = __fsub_rn(__fmul_rn(x, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(x, s), __fmul_rn(b, c));
}

// The threads of a CTA are a multiple of the items of a head, so that a thread keeps
// its place in the head and steps through heads.  kOneToken: a CTA has one token.
template <bool kF16, bool kHalf, bool kOneToken>
__global__ void __launch_bounds__(512) rope_vec_kernel(const RopeParams p, int tokens_per_cta,
                                                       int64_t tokens) {
  extern __shared__ float2 rot[];   // [tokens_per_cta][pairs]
  const int64_t token0 = (int64_t)blockIdx.x * tokens_per_cta;
  const int here = kOneToken ? 1 : (int)min((int64_t)tokens_per_cta, tokens - token0);
  const int eights = p.pairs / 8, per_head = eights + (p.head_dim - 2 * p.pairs) / 8;
  const int heads = here * p.heads;
  const int first = (int)threadIdx.x / per_head, at = (int)threadIdx.x - first * per_head;
  const int step = (int)blockDim.x / per_head;
  const bool turns = at < eights;
  const int off0 = turns ? (kHalf ? 8 : 16) * at : 8 * at + p.pairs;
  const int off1 = kHalf ? 8 * at + p.pairs : 16 * at + 8;
  grid_dep_wait();
  grid_dep_launch();
  bool have_rot = false;
  for (int h0 = first; h0 < heads || !have_rot; h0 += kItems * step) {
    uint4 v[kItems][2];
    int64_t yo[kItems];
    int tok[kItems];
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      const int q = h0 + k * step;
      if (q >= heads) continue;
      tok[k] = kOneToken ? 0 : q / p.heads;
      const int head = q - tok[k] * p.heads;
      const uint16_t* const xp = p.x + (token0 + tok[k]) * p.x_token + head * p.x_head;
      yo[k] = (token0 + tok[k]) * p.y_token + head * p.y_head;
      v[k][0] = ldg128(xp + off0);
      if (turns) v[k][1] = ldg128(xp + off1);
    }
    if (!have_rot) {
      for (int j = threadIdx.x; j < here * p.pairs; j += blockDim.x) {
        const int t = kOneToken ? 0 : j / p.pairs;
        rot[j] = rotation(p, token0 + t, j - t * p.pairs);
      }
      __syncthreads();
      have_rot = true;
    }
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (h0 + k * step >= heads) continue;
      uint16_t* const yp = p.y + yo[k];
      if (!turns) {
        *reinterpret_cast<uint4*>(yp + off0) = v[k][0];
        continue;
      }
      const float4* const r = reinterpret_cast<const float4*>(rot + tok[k] * p.pairs + 8 * at);
      float a[8], b[8];
      unpack8<kF16>(v[k][0], a);
      unpack8<kF16>(v[k][1], b);
#pragma unroll
      for (int j = 0; j < 4; ++j) {   // two pairs
        const float4 c = r[j];
        if (kHalf) {
          turn(a[2 * j], b[2 * j], c.x, c.y);
          turn(a[2 * j + 1], b[2 * j + 1], c.z, c.w);
        } else if (j < 2) {
          turn(a[4 * j], a[4 * j + 1], c.x, c.y);
          turn(a[4 * j + 2], a[4 * j + 3], c.z, c.w);
        } else {
          turn(b[4 * j - 8], b[4 * j - 7], c.x, c.y);
          turn(b[4 * j - 6], b[4 * j - 5], c.z, c.w);
        }
      }
      *reinterpret_cast<uint4*>(yp + off0) = pack8<kF16>(a);
      *reinterpret_cast<uint4*>(yp + off1) = pack8<kF16>(b);
    }
  }
}

}  // namespace

cudaError_t launch_rope(const qlin_rope_t& a, cudaStream_t s) {
  RopeParams p{};
  p.x = static_cast<const uint16_t*>(a.x);
  p.y = static_cast<uint16_t*>(a.y);
  p.x_token = a.x_token_stride;
  p.x_head = a.x_head_stride;
  p.y_token = a.y_token_stride;
  p.y_head = a.y_head_stride;
  p.positions = a.positions;
  p.pos_token = a.position_token_stride;
  p.pos_axis = a.position_axis_stride;
  p.turns = a.turns;
  p.magnitude = a.magnitude;
  p.heads = (int)a.heads;
  p.head_dim = a.head_dim;
  p.pairs = a.rot_dim / 2;
  p.pos64 = a.position_bits == 64 ? 1 : 0;
  int end = 0;
  for (int i = 0; i < 3; ++i) {
    end = i < a.axes ? end + a.axis_pairs[i] : end;
    p.axis_end[i] = i + 1 < a.axes ? end : p.pairs;   // no pair reaches the last ones
  }
  p.half = a.layout == QLIN_ROPE_HALF ? 1 : 0;
  p.inverse = a.inverse ? 1 : 0;
  p.fp16 = a.dtype == QLIN_FP16 ? 1 : 0;
  // 16-byte accesses: every row starts on a 16-byte boundary, and chunks of eight
  // elements divide the pairs, the halves and what follows them
  const bool vec = p.pairs % 8 == 0 && p.head_dim % 8 == 0 &&
                   ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y)) & 15u) == 0 &&
                   ((p.x_token | p.x_head | p.y_token | p.y_head) & 7) == 0;
  if (vec) {
    const int per_head = p.pairs / 8 + (p.head_dim - 2 * p.pairs) / 8;
    const int64_t per_token = (int64_t)p.heads * per_head;
    const int most = 8192 / (p.pairs * (int)sizeof(float2));
    const int per_cta = (int)std::max<int64_t>(1, std::min<int64_t>({(int64_t)most, 256 / per_token, a.tokens}));
    // threads: whole heads, kItems of them per thread and round, at most 512 threads
    const int64_t heads = per_cta * p.heads;
    const int64_t fit = 512 / per_head;   // per_head <= 128
    const int64_t rounds = (heads + fit * kItems - 1) / (fit * kItems);
    const int threads = (int)((heads + rounds * kItems - 1) / (rounds * kItems)) * per_head;
    const unsigned grid = (unsigned)((a.tokens + per_cta - 1) / per_cta);
    const int smem = per_cta * p.pairs * (int)sizeof(float2);
    using Kernel = void (*)(RopeParams, int, int64_t);
    static constexpr Kernel kKernels[2][2][2] = {
        {{rope_vec_kernel<false, false, false>, rope_vec_kernel<false, false, true>},
         {rope_vec_kernel<false, true, false>, rope_vec_kernel<false, true, true>}},
        {{rope_vec_kernel<true, false, false>, rope_vec_kernel<true, false, true>},
         {rope_vec_kernel<true, true, false>, rope_vec_kernel<true, true, true>}}};
    const Kernel kern = kKernels[p.fp16][p.half][per_cta == 1];
    return launch_pdl(kern, grid, threads, smem, s, p, per_cta, a.tokens);
  }
  return launch_pdl(rope_kernel, (unsigned)a.tokens, kThreads, 0, s, p);
}

}  // namespace qlin
