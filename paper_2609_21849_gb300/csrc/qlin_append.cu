// New tokens' keys and values into a paged cache, with the rotary positions of q and k
// applied on the way and, for an FP8 cache, the codes taken from the fp32 result: each
// value is rounded once.
//   slot = cached[b] + (token - q_start[b]);  page = table[b][slot / page_size]
//   k_cache[page][slot % page_size][h] = round(turn(k, position));  v likewise, unturned
// Angles as in the rotary-position kernels: position * turns modulo 2^64, a fraction of a
// turn that needs no reduction.
#include <type_traits>

#include "qlin_cache.h"
#include "qlin_internal.h"

namespace qlin {

namespace {

constexpr int kWarps = 4;

struct Strided {
  const uint16_t* p;
  int64_t token, head;   // elements
};

struct AppendParams {
  Strided q, k, v;
  uint16_t* q_out;
  int64_t q_out_token, q_out_head;
  uint8_t *k_cache, *v_cache;
  int64_t kc_page, kc_slot, kc_head, vc_page, vc_slot, vc_head;   // elements
  const int32_t* table;
  int64_t table_stride;
  const int32_t* cached;
  const int32_t* q_start;
  const float *k_scale, *v_scale;
  int64_t tokens;
  int sequences, pages, page_size, table_width;
  int q_heads, heads, head_dim, pairs;
  const void* positions;   // null: a token's slot
  int64_t pos_token, pos_axis;
  int pos64, half;
  int axis_end[3];
  const uint64_t* turns;
  float magnitude;
  unsigned* err;
  // the split: a warp takes some steps of `slots` heads of one token, all of q, of k or of v
  int slots;
  int q_groups, kv_groups, q_steps, kv_steps;   // warps of a token for each, and steps of a warp
};

// Where a token's keys and values go, the same in all lanes of a warp.
struct Place {
  bool token_ok;    // the token belongs to a sequence
  bool ok;          // and its slot lies in a page
  int64_t at;       // its slot in the sequence
  int64_t page;
  int slot;
};

// The sequence of a token by a search of 32 starts at a time: loads that depend on one
// another are what a small call waits for.
__device__ __forceinline__ Place find_place(const AppendParams& p, int64_t token, int lane) {
  Place r{false, false, 0, 0, 0};
  int lo = 0, len = p.sequences + 1;
  for (;;) {
    const int step = (len + 31) / 32;
    const int i = lane * step;
    const bool below = i < len && p.q_start[lo + i] <= token;
    const unsigned hits = __ballot_sync(0xFFFFFFFFu, below);
    const int n = __popc(hits);
    if (n == 0) return r;   // before the first
    lo += (n - 1) * step;
    len = min(step, len - (n - 1) * step);
    if (step == 1) break;
  }
  if (lo >= p.sequences) return r;   // behind the last
  const CacheSeq s = cache_seq(p.q_start[lo], p.q_start[lo + 1], p.cached[lo], p.tokens, p.page_size, p.table_width);
  r.at = s.cached + (token - s.first);
  r.token_ok = !(s.bad && s.fresh == 0) && token - s.first < s.fresh;
  int index;
  if (r.token_ok && cache_place(r.at, p.page_size, p.table_width, &index, &r.slot)) {
    r.page = p.table[lo * p.table_stride + index];
    r.ok = r.page >= 0 && r.page < p.pages;
  }
  if (!r.ok && lane == 0) report_invalid(p.err);
  return r;
}

// (cos, sin) of pair i of the token, times the magnitude.
__device__ __forceinline__ float2 rotation(const AppendParams& p, int64_t token, int64_t at, int i) {
  int64_t pos = at;
  if (p.positions != nullptr) {
    const int axis = (i >= p.axis_end[0]) + (i >= p.axis_end[1]) + (i >= p.axis_end[2]);
    const int64_t o = token * p.pos_token + axis * p.pos_axis;
    pos = p.pos64 ? static_cast<const int64_t*>(p.positions)[o]
                  : (int64_t)static_cast<const int32_t*>(p.positions)[o];
  }
  const float2 r = turn_by(pos, p.turns[i]);
  return make_float2(r.x * p.magnitude, r.y * p.magnitude);
}

template <bool kF16>
__device__ __forceinline__ float2 unpack(uint32_t w) {
  if constexpr (kF16)
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
  else
    return make_float2(bf16_lo(w), bf16_hi(w));
}
template <bool kF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  return kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
}

// Which of the three a head of the list q, k, v is, and its place.
enum { kQ, kK, kV };
__device__ __forceinline__ int head_of(const AppendParams& p, int h, int* head) {
  if (h < p.q_heads) {
    *head = h;
    return kQ;
  }
  h -= p.q_heads;
  *head = h < p.heads ? h : h - p.heads;
  return h < p.heads ? kK : kV;
}

// Eight elements per lane and head: four pairs (the halves' four elements each, or adjacent
// pairs), or eight elements that do not turn.  A lane keeps its place in the head, so its
// rotations stay in registers for all heads of its warp, and addresses advance by a stride.
// Bound by HBM: 2 bytes in and the cache's 1 or 2 (q: 2) out per element.  4608 tokens of 24 heads
// of 128 in q, k and v 29.0 us, 88% of the measured copy rate; with heads of all three in one warp,
// each picking its own addresses, 42.7; with four steps a warp 32.1, twelve 28.9 (FP8 29.1, six 28.7).
// 64 tokens of 32 + 2 x 8 heads 3.1 us, a launch and the loads that wait for one another.
template <bool kF16, bool kFp8, int kItems>
__global__ void __launch_bounds__(kWarps * 32) append_kernel(const AppendParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t token = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  int group = (int)blockIdx.y;
  const int which = group < p.q_groups ? kQ : group < p.q_groups + p.kv_groups ? kK : kV;
  group -= which == kQ ? 0 : which == kK ? p.q_groups : p.q_groups + p.kv_groups;
  const Strided& in = which == kQ ? p.q : which == kK ? p.k : p.v;
  const int per = (which == kQ ? p.q_steps : p.kv_steps) * p.slots;
  grid_dep_wait();
  grid_dep_launch();
  if (token >= p.tokens) return;   // (whole warps)
  const int per_head = p.head_dim / 8;
  const int slot = lane / per_head, at8 = lane - slot * per_head;
  const bool turns = which != kV && 8 * at8 < 2 * p.pairs;
  const bool pieces = turns && p.half;   // two of four elements
  const int o0 = pieces ? 4 * at8 : 8 * at8, o1 = pieces ? p.pairs + 4 * at8 : 8 * at8 + 4;
  int head = group * per + slot;
  const int end = slot < p.slots ? min(which == kQ ? p.q_heads : p.heads, (group + 1) * per) : 0;
  const uint16_t* x = in.p + token * in.token + head * in.head;
  const int64_t x_step = p.slots * in.head;

  uint4 v[kItems];
  auto load = [&] {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (head + i * p.slots >= end) continue;
      if (pieces) {
        const uint2 a = *reinterpret_cast<const uint2*>(x + o0);
        const uint2 b = *reinterpret_cast<const uint2*>(x + o1);
        v[i] = make_uint4(a.x, a.y, b.x, b.y);
      } else {
        v[i] = *reinterpret_cast<const uint4*>(x + o0);
      }
      x += x_step;
    }
  };
  load();
  const Place place = find_place(p, token, lane);
  if (!place.token_ok || (which != kQ && !place.ok)) return;
  float2 rot[4];
  if (turns) {
#pragma unroll
    for (int j = 0; j < 4; ++j) rot[j] = rotation(p, token, place.at, 4 * at8 + j);
  }
  // elements of the output: 16-bit ones, or an FP8 cache's codes
  const bool codes = kFp8 && which != kQ;
  const int64_t base = which == kQ   ? token * p.q_out_token
                       : which == kK ? place.page * p.kc_page + place.slot * p.kc_slot
                                     : place.page * p.vc_page + place.slot * p.vc_slot;
  const int64_t y_head = which == kQ ? p.q_out_head : which == kK ? p.kc_head : p.vc_head;
  uint8_t* const out = which == kQ ? reinterpret_cast<uint8_t*>(p.q_out) : which == kK ? p.k_cache : p.v_cache;
  uint8_t* y = out + (base + head * y_head) * (codes ? 1 : 2);
  const int64_t y_step = p.slots * y_head * (codes ? 1 : 2);
  const float enc = codes ? encode_scale(which == kK ? *p.k_scale : *p.v_scale) : 1.0f;
  while (head < end) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (head + i * p.slots >= end) continue;
      float2 f[4] = {unpack<kF16>(v[i].x), unpack<kF16>(v[i].y), unpack<kF16>(v[i].z), unpack<kF16>(v[i].w)};
      if (turns) {
        if (p.half) {   // a in f[0], f[1], b in f[2], f[3]
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float2 a = f[j], b = f[j + 2], r0 = rot[2 * j], r1 = rot[2 * j + 1];
            f[j] = make_float2(__fmaf_rn(a.x, r0.x, __fmul_rn(b.x, -r0.y)), __fmaf_rn(a.y, r1.x, __fmul_rn(b.y, -r1.y)));
            f[j + 2] = make_float2(__fmaf_rn(a.x, r0.y, __fmul_rn(b.x, r0.x)), __fmaf_rn(a.y, r1.y, __fmul_rn(b.y, r1.x)));
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 a = f[j];
            f[j] = make_float2(__fmaf_rn(a.x, rot[j].x, __fmul_rn(a.y, -rot[j].y)),
                               __fmaf_rn(a.x, rot[j].y, __fmul_rn(a.y, rot[j].x)));
          }
        }
        if (!codes)
          v[i] = make_uint4(pack<kF16>(f[0].x, f[0].y), pack<kF16>(f[1].x, f[1].y), pack<kF16>(f[2].x, f[2].y),
                            pack<kF16>(f[3].x, f[3].y));
      }
      if (codes) {
#pragma unroll
        for (int j = 0; j < 4; ++j) mul2_rn(f[j].x, f[j].y, enc);
        const uint32_t w0 = e4m3x4(f[0].x, f[0].y, f[1].x, f[1].y), w1 = e4m3x4(f[2].x, f[2].y, f[3].x, f[3].y);
        if (pieces) {
          *reinterpret_cast<uint32_t*>(y + o0) = w0;
          *reinterpret_cast<uint32_t*>(y + o1) = w1;
        } else {
          *reinterpret_cast<uint2*>(y + o0) = make_uint2(w0, w1);
        }
      } else if (pieces) {
        *reinterpret_cast<uint2*>(y + 2 * o0) = make_uint2(v[i].x, v[i].y);
        *reinterpret_cast<uint2*>(y + 2 * o1) = make_uint2(v[i].z, v[i].w);
      } else {
        *reinterpret_cast<uint4*>(y + 2 * o0) = v[i];
      }
      y += y_step;
    }
    head += kItems * p.slots;
    if (head < end) load();
  }
}

// The same element by element, for rows that start off those boundaries or pairs that do
// not come in fours: a warp per token, a lane's pairs for all heads.
__device__ __forceinline__ float load16(const uint16_t* p, bool fp16) {
  const uint16_t w = *p;
  return fp16 ? __half2float(__ushort_as_half(w)) : __uint_as_float((uint32_t)w << 16);
}

template <bool kF16, bool kFp8>
__global__ void __launch_bounds__(kWarps * 32) append_scalar_kernel(const AppendParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t token = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  grid_dep_wait();
  grid_dep_launch();
  if (token >= p.tokens) return;
  const Place place = find_place(p, token, lane);
  if (!place.token_ok) return;
  float k_enc = 1.0f, v_enc = 1.0f;
  if (kFp8) {
    k_enc = encode_scale(*p.k_scale);
    v_enc = encode_scale(*p.v_scale);
  }
  auto store = [&](int which, int head, int d, float f) {
    if (which == kQ) {
      p.q_out[token * p.q_out_token + head * p.q_out_head + d] = (uint16_t)pack<kF16>(f, 0.0f);
      return;
    }
    if (!place.ok) return;
    const int64_t o = which == kK ? place.page * p.kc_page + place.slot * p.kc_slot + head * p.kc_head + d
                                  : place.page * p.vc_page + place.slot * p.vc_slot + head * p.vc_head + d;
    uint8_t* const c = which == kK ? p.k_cache : p.v_cache;
    if (kFp8)
      c[o] = (uint8_t)e4m3_code(__fmul_rn(f, which == kK ? k_enc : v_enc));
    else
      reinterpret_cast<uint16_t*>(c)[o] = (uint16_t)pack<kF16>(f, 0.0f);
  };
  const int all = p.q_heads + 2 * p.heads, rest = p.head_dim - 2 * p.pairs;
  for (int i = lane; i < p.pairs + rest; i += 32) {
    const bool turns = i < p.pairs;
    const float2 r = turns ? rotation(p, token, place.at, i) : make_float2(1.0f, 0.0f);
    const int da = !turns ? i + p.pairs : p.half ? i : 2 * i, db = p.half ? i + p.pairs : 2 * i + 1;
    for (int h = 0; h < all; ++h) {
      int head;
      const int which = head_of(p, h, &head);
      const Strided& s = which == kQ ? p.q : which == kK ? p.k : p.v;
      const uint16_t* const x = s.p + token * s.token + head * s.head;
      const float a = load16(x + da, kF16);
      if (!turns) {
        store(which, head, da, a);
        continue;
      }
      const float b = load16(x + db, kF16);
      if (which == kV) {
        store(which, head, da, a);
        store(which, head, db, b);
      } else {
        store(which, head, da, __fmaf_rn(a, r.x, __fmul_rn(b, -r.y)));
        store(which, head, db, __fmaf_rn(a, r.y, __fmul_rn(b, r.x)));
      }
    }
  }
}

}  // namespace

cudaError_t launch_cache_append(const qlin_cache_t& c, const qlin_cache_append_t& a, cudaStream_t s, Device dev,
                                unsigned* err) {
  AppendParams p{};
  p.q = {static_cast<const uint16_t*>(a.q), a.q_token_stride, a.q_head_stride};
  p.k = {static_cast<const uint16_t*>(a.k), a.k_token_stride, a.k_head_stride};
  p.v = {static_cast<const uint16_t*>(a.v), a.v_token_stride, a.v_head_stride};
  p.q_out = static_cast<uint16_t*>(a.q_out);
  p.q_out_token = a.q_out_token_stride;
  p.q_out_head = a.q_out_head_stride;
  p.k_cache = static_cast<uint8_t*>(c.k);
  p.v_cache = static_cast<uint8_t*>(c.v);
  p.kc_page = c.k_page_stride;
  p.kc_slot = c.k_slot_stride;
  p.kc_head = c.k_head_stride;
  p.vc_page = c.v_page_stride;
  p.vc_slot = c.v_slot_stride;
  p.vc_head = c.v_head_stride;
  p.table = c.page_table;
  p.table_stride = c.table_stride;
  p.cached = c.cached;
  p.q_start = c.q_start;
  p.k_scale = c.k_scale;
  p.v_scale = c.v_scale;
  p.tokens = a.tokens;
  p.sequences = c.sequences;
  p.pages = c.pages;
  p.page_size = c.page_size;
  p.table_width = c.table_width;
  p.q_heads = a.q != nullptr ? a.q_heads : 0;
  p.heads = c.heads;
  p.head_dim = c.head_dim;
  p.pairs = a.turns != nullptr ? a.rot_dim / 2 : 0;
  p.positions = a.positions;
  p.pos_token = a.position_token_stride;
  p.pos_axis = a.position_axis_stride;
  p.pos64 = a.position_bits == 64 ? 1 : 0;
  p.half = a.layout == QLIN_ROPE_HALF ? 1 : 0;
  int end = 0;
  for (int i = 0; i < 3; ++i) {
    end = i < a.axes ? end + a.axis_pairs[i] : end;
    p.axis_end[i] = i + 1 < a.axes ? end : p.pairs;   // no pair reaches the last ones
  }
  p.turns = a.turns;
  p.magnitude = a.magnitude;
  p.err = err;
  const bool fp16 = a.dtype == QLIN_FP16, fp8 = c.format == QLIN_CACHE_E4M3;
  // 16-byte rows (a cache of codes: 8), pairs in fours
  auto bits = [](const void* q) { return reinterpret_cast<uintptr_t>(q); };
  const uintptr_t at = bits(a.k) | bits(a.v) | (p.q_heads ? bits(a.q) | bits(a.q_out) : 0u);
  const int64_t strides = a.k_token_stride | a.k_head_stride | a.v_token_stride | a.v_head_stride |
                          (p.q_heads ? a.q_token_stride | a.q_head_stride | a.q_out_token_stride | a.q_out_head_stride
                                     : 0);
  const int64_t cstrides = c.k_page_stride | c.k_slot_stride | c.k_head_stride | c.v_page_stride | c.v_slot_stride |
                           c.v_head_stride;
  const bool vec = p.pairs % 4 == 0 && c.head_dim % 8 == 0 && (at & 15u) == 0 && (strides & 7) == 0 &&
                   (cstrides & 7) == 0 && ((bits(c.k) | bits(c.v)) & (fp8 ? 7u : 15u)) == 0;
  using T = std::true_type;
  using F = std::false_type;
  if (!vec) {
    const dim3 grid((unsigned)((p.tokens + kWarps - 1) / kWarps));
    auto launch = [&](auto f16, auto codes) {
      return launch_pdl(append_scalar_kernel<decltype(f16)::value, decltype(codes)::value>, grid, kWarps * 32, 0, s, p);
    };
    return fp16 ? (fp8 ? launch(T{}, T{}) : launch(T{}, F{})) : (fp8 ? launch(F{}, T{}) : launch(F{}, F{}));
  }
  p.slots = 32 / (c.head_dim / 8);
  const int q_all = (p.q_heads + p.slots - 1) / p.slots, kv_all = (p.heads + p.slots - 1) / p.slots;
  // steps of a warp: one while warps are few, up to six where they are plenty (the rotations
  // and the search are a warp's fixed cost)
  const int64_t fill = p.tokens * (q_all + 2 * kv_all) / (16 * dev.num_sms);
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>(6, fill));
  p.q_groups = (q_all + most - 1) / most;
  p.kv_groups = (kv_all + most - 1) / most;
  const int limit = 20000;   // (of groups, three kinds of them in a grid's y)
  p.q_groups = std::min(p.q_groups, limit);
  p.kv_groups = std::min(p.kv_groups, limit);
  p.q_steps = p.q_groups > 0 ? (q_all + p.q_groups - 1) / p.q_groups : 0;
  p.kv_steps = (kv_all + p.kv_groups - 1) / p.kv_groups;
  const int steps = std::max(p.q_steps, p.kv_steps);
  const dim3 grid((unsigned)((p.tokens + kWarps - 1) / kWarps), (unsigned)(p.q_groups + 2 * p.kv_groups));
  auto launch = [&](auto f16, auto codes) {
    constexpr bool kF16 = decltype(f16)::value, kFp8 = decltype(codes)::value;
    return steps == 1  ? launch_pdl(append_kernel<kF16, kFp8, 1>, grid, kWarps * 32, 0, s, p)
           : steps < 5 ? launch_pdl(append_kernel<kF16, kFp8, 4>, grid, kWarps * 32, 0, s, p)
                       : launch_pdl(append_kernel<kF16, kFp8, 6>, grid, kWarps * 32, 0, s, p);
  };
  return fp16 ? (fp8 ? launch(T{}, T{}) : launch(T{}, F{})) : (fp8 ? launch(F{}, T{}) : launch(F{}, F{}));
}

}  // namespace qlin
