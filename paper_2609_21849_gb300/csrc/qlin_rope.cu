// Rotary positions.  The angle of a pair is position * f, held as turns: a pair's
// turns per position are a 64-bit fraction (units of 2^-64 turn), so that position *
// turns modulo 2^64 is the angle without whole turns, exact for every position; its
// top 32 bits give the angle to 2^-32 turn.  (In fp32 the product alone is off by
// 0.03 radians at position 10^6.)
#include <type_traits>

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
    // (rounded as turn2 below: a value's bits do not depend on where its row starts)
    y[da] = pack16(__fmaf_rn(a, r.x, __fmul_rn(b, -r.y)), fp16);
    y[db] = pack16(__fmaf_rn(a, r.y, __fmul_rn(b, r.x)), fp16);
  }
}

// ---- 16-byte accesses ----
// A lane takes 16 elements of a head in two chunks of 8: eight pairs (the chunks half a
// rotation apart in the half layout, adjacent in the interleaved one; the last lane of
// the pairs perhaps fewer), or elements past rot_dim (the last lane of a head perhaps one
// chunk of them; none in place).
// A warp works alone, on some heads of one token or, where heads are few, on several
// tokens: a lane keeps its place in the head, so its eight rotations stay in registers
// for all of its heads, and nothing waits for another warp.  The loads of its first
// heads are issued before the rotations are computed.
//
// Bound by HBM (2 bytes in, 2 out per element; positions and turns are small): 4608 x
// 48 x 128 with strided rows 20.0 us interleaved, 20.1 in halves, 84-85% of the measured
// copy rate; 9216 x 48 x 128 of which 64 turn 35.4 us, 96%.  A CTA per token with the
// rotations behind a barrier took 24.8 us, scalar accesses 57.  Where the lanes of a
// head do not divide a warp some idle (192 of 192: 24 of 32 lanes, 70%), and where the
// pairs do not fill their last lane; 9079 x 25 x 80 of which 40 turn 17.4 us interleaved,
// 19.3 in halves (element by element 57).  One token takes 1.8 us, a launch and one chain
// of loads.
// kItems heads of a lane are in flight at once (4, where work is plenty).
constexpr int kMostItems = 4;
constexpr int kVecWarps = 4;

// 32 bytes (32-byte aligned).
__device__ __forceinline__ void ldg256(const uint16_t* p, uint4 (&v)[2]) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(v[0].x), "=r"(v[0].y), "=r"(v[0].z), "=r"(v[0].w), "=r"(v[1].x), "=r"(v[1].y),
                 "=r"(v[1].z), "=r"(v[1].w)
               : "l"(p));
}
__device__ __forceinline__ void stg256(uint16_t* p, uint4 a, uint4 b) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x),
               "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
               : "memory");
}

__device__ __forceinline__ uint4 ldg128(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// Four or eight elements from an eight-byte boundary.
__device__ __forceinline__ void ldg_fours(const uint16_t* p, int n, uint4& v) {
  const uint2 a = *reinterpret_cast<const uint2*>(p);
  uint2 b = make_uint2(0u, 0u);
  if (n > 4) b = *reinterpret_cast<const uint2*>(p + 4);
  v = make_uint4(a.x, a.y, b.x, b.y);
}
__device__ __forceinline__ void stg_fours(uint16_t* p, int n, uint4 v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y);
  if (n > 4) *reinterpret_cast<uint2*>(p + 4) = make_uint2(v.z, v.w);
}

template <bool kF16>
__device__ __forceinline__ float2 unpack2(uint32_t w) {
  if constexpr (kF16)
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else
    return make_float2(bf16_lo(w), bf16_hi(w));
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
}

// The eight pairs (a[i], b[i]) of two chunks: element i of each (kHalf), or elements
// 2 i and 2 i + 1 of both in a row.
template <bool kF16, bool kHalf>
__device__ __forceinline__ void unpack_pairs(const uint4 (&v)[2], float (&a)[8], float (&b)[8]) {
  const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 f = unpack2<kF16>(w[i]);
    if (!kHalf) {
      a[i] = f.x;
      b[i] = f.y;
    } else {
      float* const d = i < 4 ? a : b;
      d[2 * (i & 3)] = f.x;
      d[2 * (i & 3) + 1] = f.y;
    }
  }
}
// The interleaved elements past `turned` (even) pairs stay as they came.
template <bool kF16, bool kHalf>
__device__ __forceinline__ void pack_pairs(const float (&a)[8], const float (&b)[8], int turned, uint4 (&v)[2]) {
  uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float* const d = i < 4 ? a : b;
    if (kHalf)
      w[i] = pack2<kF16>(d[2 * (i & 3)], d[2 * (i & 3) + 1]);
    else if ((i & ~1) < turned)
      w[i] = pack2<kF16>(a[i], b[i]);
  }
  v[0] = make_uint4(w[0], w[1], w[2], w[3]);
  v[1] = make_uint4(w[4], w[5], w[6], w[7]);
}

// Two pairs turned by packed arithmetic: (a, b) -> (a c - b s, b c + a s); ns = -s.
__device__ __forceinline__ void turn2(float (&a)[8], float (&b)[8], int i, float2 c, float2 s, float2 ns) {
  asm("{\n\t.reg .b64 a, b, c, s, n, x, y;\n\t"
      "mov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\tmov.b64 c, {%4, %5};\n\t"
      "mov.b64 s, {%6, %7};\n\tmov.b64 n, {%8, %9};\n\t"
      "mul.rn.f32x2 x, b, n;\n\tmul.rn.f32x2 y, b, c;\n\t"
      "fma.rn.f32x2 x, a, c, x;\n\tfma.rn.f32x2 y, a, s, y;\n\t"
      "mov.b64 {%0, %1}, x;\n\tmov.b64 {%2, %3}, y;\n\t}"
      : "+f"(a[i]), "+f"(a[i + 1]), "+f"(b[i]), "+f"(b[i + 1])
      : "f"(c.x), "f"(c.y), "f"(s.x), "f"(s.y), "f"(ns.x), "f"(ns.y));
}

// The split of the work: units (warps) of `tokens` tokens or of `heads` heads of one.
// The CTAs' y counts the groups of heads.
struct RopeUnits {
  int64_t count;
  int per_head, slots;    // lanes of a head; heads that a warp takes at a time
  int tokens, heads;
  // n / d of the small n here is n * ceil(2^20 / d) >> 20 (n d < 2^20)
  uint32_t by_per_head, by_heads, by_pairs;
  int wide;               // rows start on 32-byte boundaries: a lane's adjacent chunks in one access
};

// kFours: halves that are no multiple of eight take eight-byte accesses, the last lane one
// per half.  (An instance of its own: the branch cost the others 6%.)
template <bool kF16, bool kHalf, bool kFours, int kItems>
__global__ void __launch_bounds__(kVecWarps * 32) rope_vec_kernel(const RopeParams p, const RopeUnits u,
                                                                  int64_t tokens) {
  extern __shared__ float2 rot_all[];   // per warp [tokens][pairs]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t unit = (int64_t)blockIdx.x * kVecWarps + warp;
  grid_dep_wait();
  grid_dep_launch();
  if (unit >= u.count) return;   // (whole warps)
  const int group = (int)blockIdx.y;
  const int64_t token0 = unit * u.tokens;
  const int here = (int)min((int64_t)u.tokens, tokens - token0);
  const int eights = (kFours || !kHalf ? p.pairs + 7 : p.pairs) / 8;
  auto div20 = [](int n, uint32_t by) { return (int)(((uint32_t)n * by) >> 20); };
  const int slot = div20(lane, u.by_per_head), at = lane - slot * u.per_head;
  // the lane's token, and its heads: first, then every slots-th
  const int tok = u.tokens == 1 ? 0 : div20(slot, u.by_heads);
  int head = u.tokens == 1 ? group * u.heads + slot : slot - tok * p.heads;
  const int head_end = slot >= u.slots || tok >= here ? 0
                       : u.tokens == 1                ? min(p.heads, (group + 1) * u.heads)
                                                      : head + 1;
  constexpr bool kPart = kFours || !kHalf;
  const int turned = kPart ? min(8, p.pairs - 8 * at) : 8;   // pairs of a lane that turns
  const bool turns = kPart ? turned > 0 : at < eights;
  // (2 pairs precede the rest: 16 eights, or less)
  const int off0 = kHalf && turns ? 8 * at : kFours ? 2 * p.pairs + 16 * (at - eights) : 16 * at;
  const int off1 = kHalf && turns ? off0 + p.pairs : off0 + 8;
  const bool second = off1 < p.head_dim;
  const bool wide = u.wide && second && (!kHalf || !turns);
  const bool fours = kFours && turns;
  const uint16_t* x = p.x + (token0 + tok) * p.x_token + head * p.x_head;
  uint16_t* y = p.y + (token0 + tok) * p.y_token + head * p.y_head;
  const int64_t x_step = u.slots * p.x_head, y_step = u.slots * p.y_head;
  uint4 v[kItems][2];
  auto load = [&] {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (head + k * u.slots >= head_end) continue;
      if (wide) {
        ldg256(x + off0, v[k]);
      } else if (fours) {
        ldg_fours(x + off0, turned, v[k][0]);
        ldg_fours(x + off1, turned, v[k][1]);
      } else {
        v[k][0] = ldg128(x + off0);
        if (second) v[k][1] = ldg128(x + off1);
      }
      x += x_step;
    }
  };
  load();
  float2* const rot = rot_all + warp * u.tokens * p.pairs;
#pragma unroll 2
  for (int j = lane; j < here * p.pairs; j += 32) {
    const int t = u.tokens == 1 ? 0 : div20(j, u.by_pairs);
    rot[j] = rotation(p, token0 + t, j - t * p.pairs);
  }
  __syncwarp();
  float2 c[4], sn[4], ns[4];   // of pairs 2 j and 2 j + 1
  if (head < head_end && turns) {
    const float4* const src = reinterpret_cast<const float4*>(rot + tok * p.pairs + 8 * at);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float4 r = !kPart || 2 * j < turned ? src[j] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      c[j] = make_float2(r.x, r.z);
      sn[j] = make_float2(r.y, r.w);
      ns[j] = make_float2(-r.y, -r.w);
    }
  }
  while (head < head_end) {
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
      if (head + k * u.slots >= head_end) continue;
      if (turns) {
        float a[8], b[8];
        unpack_pairs<kF16, kHalf>(v[k], a, b);
#pragma unroll
        for (int j = 0; j < 4; ++j) turn2(a, b, 2 * j, c[j], sn[j], ns[j]);
        pack_pairs<kF16, kHalf>(a, b, turned, v[k]);
      }
      if (wide) {
        stg256(y + off0, v[k][0], v[k][1]);
      } else if (fours) {
        stg_fours(y + off0, turned, v[k][0]);
        stg_fours(y + off1, turned, v[k][1]);
      } else {
        *reinterpret_cast<uint4*>(y + off0) = v[k][0];
        if (second) *reinterpret_cast<uint4*>(y + off1) = v[k][1];
      }
      y += y_step;
    }
    head += kItems * u.slots;
    load();
  }
}

}  // namespace

cudaError_t launch_rope(const qlin_rope_t& a, int num_sms, cudaStream_t s) {
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
  // 16-byte accesses: every row starts on a 16-byte boundary, chunks of eight elements
  // divide the head, an access never divides a pair (in halves, eight bytes at least
  // where their length is no multiple of eight), a warp's lanes hold a head
  const int eights = (p.pairs + 7) / 8;
  const int past = p.head_dim - (p.half ? 2 * p.pairs : std::min(16 * eights, p.head_dim));
  const int per_head = eights + (p.x == p.y ? 0 : (past + 15) / 16);
  const bool vec = p.pairs % (p.half ? 4 : 2) == 0 && per_head <= 32 && p.head_dim % 8 == 0 &&
                   ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y)) & 15u) == 0 &&
                   ((p.x_token | p.x_head | p.y_token | p.y_head) & 7) == 0;
  if (vec) {
    RopeUnits u{};
    u.per_head = per_head;
    u.slots = 32 / u.per_head;
    u.tokens = std::max(1, u.slots / p.heads);
    const int steps = (p.heads + u.slots - 1) / u.slots;
    // Two of them per warp (T x H x D in halves, us with one and two: 1 x 64 x 128 2.1, 1.8;
    // 206 x 35 x 256 5.3, 3.9; with two and four: 2048 x 32 x 128 8.0, 9.1), four where
    // warps are plenty even so (4608 x 24 x 192 20.2, 18.3), three rather than two and
    // one (5674 x 9 x 128 8.8, 8.4).
    const int64_t fill = (a.tokens + u.tokens - 1) / u.tokens * steps / (16 * num_sms);
    const int most = fill >= 16 ? kMostItems : fill >= 4 && steps == 3 ? 3 : 2;
    const int groups = std::min((steps + most - 1) / most, 65535);
    const int per_warp = (steps + groups - 1) / groups;
    u.heads = per_warp * u.slots;
    u.count = (a.tokens + u.tokens - 1) / u.tokens;
    auto by = [](int d) { return (uint32_t)(((1 << 20) + d - 1) / d); };
    u.by_per_head = by(u.per_head);
    u.by_heads = u.tokens > 1 ? by(p.heads) : 0;
    u.by_pairs = by(p.pairs);
    u.wide = ((reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.y)) & 31u) == 0 &&
                     ((p.x_token | p.x_head | p.y_token | p.y_head) & 15) == 0 && (!p.half || p.pairs % 8 == 0)
                 ? 1
                 : 0;
    const unsigned grid = (unsigned)((u.count + kVecWarps - 1) / kVecWarps);
    const int smem = kVecWarps * u.tokens * p.pairs * (int)sizeof(float2);
    auto launch = [&](auto kern) {
      return launch_pdl(kern, dim3(grid, (unsigned)groups), kVecWarps * 32, smem, s, p, u, a.tokens);
    };
    using T = std::true_type;
    using F = std::false_type;
    auto with_items = [&](auto f16, auto half, auto fours) {
      constexpr bool kF16 = decltype(f16)::value, kHalf = decltype(half)::value, kFours = decltype(fours)::value;
      return per_warp == 1   ? launch(rope_vec_kernel<kF16, kHalf, kFours, 1>)
             : per_warp == 2 ? launch(rope_vec_kernel<kF16, kHalf, kFours, 2>)
                             : launch(rope_vec_kernel<kF16, kHalf, kFours, 4>);
    };
    auto with_layout = [&](auto f16) {
      return !p.half            ? with_items(f16, F{}, F{})
             : p.pairs % 8 != 0 ? with_items(f16, T{}, T{})
                                : with_items(f16, T{}, F{});
    };
    return p.fp16 ? with_layout(T{}) : with_layout(F{});
  }
  return launch_pdl(rope_kernel, (unsigned)a.tokens, kThreads, 0, s, p);
}

}  // namespace qlin
