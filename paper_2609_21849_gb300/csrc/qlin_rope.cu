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
  return launch_pdl(rope_kernel, (unsigned)a.tokens, kThreads, 0, s, p);
}

}  // namespace qlin
