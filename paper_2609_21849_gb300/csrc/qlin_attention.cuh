// Attention of new tokens over a paged cache: out = softmax(scale q k^T, masked) v in one
// pass over the keys with the running maximum and sum of each row.
//
// The rows of a KV head's group (its query heads times the sequence's new tokens) share its
// keys, so that these are read once for up to 16 or 32 rows; few rows leave HBM as the bound.
// Work is counted in tiles of keys of one (sequence, KV head, rows) item, and the CTAs get
// equal runs of tiles whatever the sequences' lengths.  A run that ends inside an item
// leaves its sums in the workspace, and the last CTA of the item to arrive joins them in the
// order of the keys: the same bits whichever CTA that is.
//
// A CTA has four warps that work alone: each takes a quarter of a tile's keys through a ring
// of its own of cp.async copies, a page's rows wherever the table says.  Scores by mma.sync
// with the rows as M: Q's fragments stay in registers, K's come as 16-byte pieces in K order
// 8 t (an MMA sums in any order as long as both operands agree), V's through transposing
// ldmatrix.  The warps' sums meet once an item.
//   E4M3: codes become fp16, exactly.  Q is brought into fp16 by a power of two per row
// (bf16 exponents exceed fp16's; elements 2^-14 below the row's largest lose bits that are
// below 2^-25 of it), and P is fp16.
//   P is rounded to the values' 16-bit type for the second product, the row's sum is taken
// before that rounding: errors of half a step of P, independent from key to key, average out.
// fp16 has few exponents below 1: there the kept maximum is 2^15 below the row's, and P up to
// 2^15, so that weights down to 2^-40 of the largest one count (bf16 has those of fp32).
//   Measured: 64 tokens over 64 caches of 2048-8192 keys in E4M3, 8 KV heads of 128, 8 query heads
// each, 142 us, 72% of the copy rate (half of an MMA's rows are empty, and the conversion of codes
// takes more issue slots than the products); one token over 1000 keys 9.8: a launch, six tiles' worth
// of latency and the join.
#include <type_traits>

#include "qlin_attention_work.cuh"

namespace qlin {

namespace {

constexpr int kWarps = kFewWarps;
constexpr float kRaise = 15.0f;   // powers of two above 1 of an fp16 P's maximum

__device__ __forceinline__ void ldmatrix_trans(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a));
}

// c += A B, 16 x 8 x 16; a0, a2 of row g, a1, a3 of row g + 8.
template <bool kF16>
__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
  if constexpr (kF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, "
        "%2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, "
        "%2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Two E4M3 codes as two halves, exactly.
__device__ __forceinline__ uint32_t e4m3x2_half2(uint32_t codes) {
  uint32_t h;
  const uint16_t c = (uint16_t)codes;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return h;
}

template <CacheKind kKind, int kD, int kM>
struct AttnCfg {
  static constexpr int kEs = kKind == CacheKind::kE4m3 ? 1 : 2;
  static constexpr int kRows = 16 * kM;
  static constexpr int kKeys = few_warp_keys(kEs, kRows);   // of a warp and tile
  static constexpr int kTile = kWarps * kKeys;
  static constexpr int kRow = kD * kEs;                    // bytes
  static constexpr int kPieces = kRow / 16;
  // rows of whole 128-byte lines: 16-byte pieces permuted by the row; else a stride that
  // spreads the rows over the banks (64 modulo 128 for K's reads, 16 for ldmatrix)
  static constexpr bool kSwizzle = kRow % 128 == 0;
  static constexpr int kKStride = kRow;
  static constexpr int kVStride = kSwizzle ? kRow : kRow + 16;
  static constexpr int kKBytes = kKeys * kKStride, kVBytes = kKeys * kVStride;
  static constexpr int kSlot = kKBytes + kVBytes;          // one warp's part of a stage
  static constexpr int kStageBytes = kWarps * kSlot;
  static constexpr int kMergeBytes = kRows * kD * 4;       // one warp's sums
  static constexpr bool kOwnMerge = kMergeBytes > kSlot;   // else in the stage just used
  static constexpr int kExtra = kOwnMerge ? kWarps * kMergeBytes : 0;
  static constexpr int kStagesTwo = (112 * 1024 - kExtra) / kStageBytes, kStagesOne = (224 * 1024 - kExtra) / kStageBytes;
  static constexpr int kStages = kStagesTwo >= 3 ? (kStagesTwo > 4 ? 4 : kStagesTwo) : kStagesOne > 4 ? 4 : kStagesOne;
  static constexpr int kSmem = kStages * kStageBytes + kExtra;
  static constexpr int kCtas = 2 * (kSmem + 2048) <= 227 * 1024 ? 2 : 1;   // of an SM
  static_assert(kStages >= 2, "shared memory");
  static_assert(kRow % 64 == 0, "K is read in 64-byte chunks");
};

// An item that other CTAs share: its rows, and the first and last of its CTAs.
struct Unfinished {
  int64_t token0;
  int row0, head0, rows, first, last;
};

// The rows of an item (few), whose parts the CTAs from, from + step, ... to left in the workspace
// (first: the item's first CTA), joined in the order of the keys: to the output, or to from's part
// in place.  What it costs is waiting for L2: a thread has four elements of 16 parts and their
// maxima and sums on their way at a time, and meets no other.  stat: kRows of them in shared memory.
constexpr int kJoin = 16;
template <int kRows, int kD>
__device__ __forceinline__ void join_few(const AttnParams& p, const Unfinished& u, int from, int to, int step,
                                         bool output, float v_scale, float2* stat) {
  constexpr int kThreads = kWarps * 32;
  const int d4s = p.head_dim / 4, items = u.rows * d4s, parts = (to - from) / step + 1;
  for (int i = threadIdx.x; i < items; i += kThreads) {
    const int row = i / d4s, d = i - row * d4s << 2;
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int q0 = 0; q0 < parts; q0 += kJoin) {
      float4 v[kJoin];
      float2 ml[kJoin];
      // (past the last part its own again, with a maximum of minus infinity: no branch between the loads)
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const int64_t at = part_row<kRows>(from + min(q0 + k, parts - 1) * step, u.first, row);
        ml[k] = __ldcg(&p.part_ml[at]);
        v[k] = __ldcg(reinterpret_cast<const float4*>(p.part + at * kD + d));
      }
      float now = m;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        if (q0 + k >= parts) ml[k].x = -INFINITY;
        now = fmaxf(now, ml[k].x);
      }
      const float base = now == -INFINITY ? 0.0f : now, keep = exp2_fast(m - base);
      l *= keep;
      o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const float w = exp2_fast(ml[k].x - base);
        // (whatever its weight: a part of NaN scores has a weight of 0 and a NaN sum)
        if (known_here(q0 + k < parts)) {
          l = fmaf(ml[k].y, w, l);
          o = make_float4(fmaf(v[k].x, w, o.x), fmaf(v[k].y, w, o.y), fmaf(v[k].z, w, o.z), fmaf(v[k].w, w, o.w));
        }
      }
      m = now;
    }
    if (output) {
      const int r = u.row0 + row;
      const int64_t token = u.token0 + r / p.group;
      const int head = u.head0 + r % p.group;
      const float inv = l == 0.0f ? 0.0f : v_scale / l;
      store_out4(p, token, head, d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (p.lse != nullptr && d == 0) p.lse[token * p.lse_token + head] = log_sum(m, l);
    } else {
      *reinterpret_cast<float4*>(p.part + part_row<kRows>(from, u.first, row) * kD + d) = o;
      if (d == 0) stat[row] = make_float2(m, l);
    }
  }
  if (!output) {
    __syncthreads();   // the maxima and sums have been read
    if ((int)threadIdx.x < u.rows) p.part_ml[part_row<kRows>(from, u.first, threadIdx.x)] = stat[threadIdx.x];
  }
}

template <CacheKind kKind, int kD, int kM>
__global__ void __launch_bounds__(kWarps * 32, (AttnCfg<kKind, kD, kM>::kCtas)) attn_kernel(const __grid_constant__ AttnParams p) {
  using C = AttnCfg<kKind, kD, kM>;
  constexpr bool kFp8 = kKind == CacheKind::kE4m3, kF16 = kKind != CacheKind::kBf16;
  constexpr int kKeys = C::kKeys, kNT = kKeys / 8, kDT = kD / 8, kRows = C::kRows;
  constexpr int kThreads = kWarps * 32;
  constexpr int kQWords = kD / 8;          // 32-bit words of a lane's share of a row
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ unsigned ok_bits[kWarps][C::kStages];
  __shared__ float2 warp_ml[kWarps][kRows];
  __shared__ bool last_flag[2];
  __shared__ Unfinished unfinished[2];   // the run's first item and its last
  __shared__ RunScratch scratch;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;

  grid_dep_wait();
  grid_dep_launch();
  Cursor cur;
  const Run run = find_run<kRows, C::kTile, kThreads>(p, cur, (int)blockIdx.x, (int)gridDim.x, scratch);
  if (run.begin >= run.end) return;
  float k_scale = 1.0f, v_scale = 1.0f;
  if (kFp8) {
    k_scale = *p.k_scale;
    v_scale = *p.v_scale;
  }

  // ---- loads: lane r < kKeys finds the page of the warp's key r, one tile ahead ----
  Cursor ahead = cur;
  int64_t to_fetch = run.begin;   // a unit
  struct Place {
    bool in;
    int page, slot, h;
  };
  auto fetch = [&] {
    Place f{false, -1, 0, 0};
    if (to_fetch >= run.end) return f;
    const int64_t key = (int64_t)ahead.tile * C::kTile + warp * kKeys + lane;
    int index;
    f.h = ahead.h;
    if (lane < kKeys && key < ahead.s.keys && cache_place(key, p.page_size, p.table_width, &index, &f.slot)) {
      f.page = p.table[ahead.b * p.table_stride + index];
      f.in = true;
    }
    to_fetch += 1 + (ahead.tile + 1 == ahead.tiles ? p.item_cost : 0);
    if (to_fetch < run.end) {
      advance<kRows, C::kTile>(p, ahead);
      if (ahead.tile == 0 && warp == 0) {   // a new item: its rows of Q towards L2
        const int64_t row = (int64_t)ahead.rt * kRows + lane;
        if (lane < kRows && row < (int64_t)ahead.s.fresh * p.group) {
          const uint16_t* const q =
              p.q + (ahead.s.first + row / p.group) * p.q_token + (ahead.h * p.group + row % p.group) * p.q_head;
          for (int at = 0; at < p.head_dim; at += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + at));
        }
      }
    }
    return f;
  };
  auto issue = [&](int stage, const Place& f) {
    const bool ok = f.in && f.page >= 0 && f.page < p.pages;
    if (f.in && !ok) report_invalid(p.err);   // the keys of a bad page are not seen
    const unsigned bits = __ballot_sync(0xFFFFFFFFu, ok);
    if (lane == 0) ok_bits[warp][stage] = bits;
    if (bits != 0u) {
      const int64_t ko = ok ? f.page * p.k_page + f.slot * p.k_slot + f.h * p.k_head : 0;
      const int64_t vo = ok ? f.page * p.v_page + f.slot * p.v_slot + f.h * p.v_head : 0;
      const uint32_t kbase = smem_u32(smem + stage * C::kStageBytes + warp * C::kSlot), vbase = kbase + C::kKBytes;
#pragma unroll
      for (int i = 0; i < kKeys * C::kPieces / 32; ++i) {
        const int at = i * 32 + lane, row = at / C::kPieces, piece = at % C::kPieces;
        const int64_t kr = __shfl_sync(0xFFFFFFFFu, ko, row), vr = __shfl_sync(0xFFFFFFFFu, vo, row);
        const bool in = ((bits >> row) & 1u) != 0u && piece * 16 < p.head_dim * C::kEs;
        const int kp = C::kSwizzle ? piece ^ ((row & 1) * 4) : piece, vp = C::kSwizzle ? piece ^ (row & 7) : piece;
        const int o = in ? piece * 16 : 0;
        cp_async16(kbase + row * C::kKStride + kp * 16, p.k + kr + o, in);
        cp_async16(vbase + row * C::kVStride + vp * 16, p.v + vr + o, in);
      }
    }
    cp_async_commit();
  };

  int num_unfinished = 0;
  // ---- one item's state ----
  uint32_t qf[kM][2][kQWords];
  float o[kM][kDT][4], m[kM][2], l[kM][2], mult[kM][2];
  auto begin_item = [&] {
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int64_t row = (int64_t)cur.rt * kRows + i * 16 + r * 8 + g;
        const bool in = row < (int64_t)cur.s.fresh * p.group;
        const uint16_t* const q = p.q + (in ? (cur.s.first + row / p.group) * p.q_token +
                                                  (cur.h * p.group + row % p.group) * p.q_head
                                            : 0);
        m[i][r] = -INFINITY;
        l[i][r] = 0.0f;
        mult[i][r] = p.scale_log2;
        constexpr int kLane = kFp8 ? 16 : 8;   // adjacent elements of a lane
#pragma unroll
        for (int c = 0; c < kD / (4 * kLane); ++c)
#pragma unroll
          for (int h = 0; h < kLane / 8; ++h) {
            const int d = c * 4 * kLane + t * kLane + h * 8;
            uint4 w = make_uint4(0u, 0u, 0u, 0u);
            if (in && d < p.head_dim) w = *reinterpret_cast<const uint4*>(q + d);
            uint32_t* const f = &qf[i][r][(c * (kLane / 8) + h) * 4];
            f[0] = w.x;
            f[1] = w.y;
            f[2] = w.z;
            f[3] = w.w;
          }
        if constexpr (kFp8) {
          // the row's power of two: its largest |q| into [1, 2) (a zero, infinite or NaN row as it is)
          uint32_t top = 0u;
#pragma unroll
          for (int k = 0; k < kQWords; ++k) top = __vmaxu2(top, qf[i][r][k] & 0x7FFF7FFFu);
          top = max(top & 0xFFFFu, top >> 16);
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
          top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
          const float big = p.fp16 ? __half2float(__ushort_as_half((unsigned short)top))
                                   : __uint_as_float(top << 16);
          int e = (int)(__float_as_uint(big) >> 23);   // biased
          e = e == 0 || e == 255 ? 127 : min(e, 252);
          const float down = signed_factor(__uint_as_float((uint32_t)(254 - e) << 23), k_scale);
          mult[i][r] =
              fminf(fmaxf(p.scale_log2 * __uint_as_float((uint32_t)e << 23) * fabsf(k_scale), FLT_MIN), FLT_MAX);
#pragma unroll
          for (int k = 0; k < kQWords; ++k) {
            const uint32_t w = qf[i][r][k];
            const float2 v = p.fp16 ? __half22float2(*reinterpret_cast<const __half2*>(&w))
                                    : make_float2(bf16_lo(w), bf16_hi(w));
            qf[i][r][k] = pack_f16x2(v.x * down, v.y * down);
          }
        }
#pragma unroll
        for (int j = 0; j < kDT; ++j) o[i][j][2 * r] = o[i][j][2 * r + 1] = 0.0f;
      }
  };

  // Element d of the output that word k (0, 1) of accumulator tile j holds in this lane.
  auto column = [&](int j, int k) {
    return kFp8 ? (j >> 1) * 16 + 4 * t + 2 * k + (j & 1) : j * 8 + 2 * t + k;
  };

  auto compute = [&](int stage) {
    const unsigned bits = ok_bits[warp][stage];
    if (bits == 0u) return;
    const uint32_t kbase = smem_u32(smem + stage * C::kStageBytes + warp * C::kSlot), vbase = kbase + C::kKBytes;
    float s[kM][kNT][4];
#pragma unroll
    for (int j = 0; j < kNT; ++j) {
#pragma unroll
      for (int i = 0; i < kM; ++i) s[i][j][0] = s[i][j][1] = s[i][j][2] = s[i][j][3] = 0.0f;
      const int row = 8 * j + g;
#pragma unroll
      for (int c = 0; c < C::kRow / 64; ++c) {
        const int piece = 4 * c + t;
        const uint4 w = lds128(kbase + row * C::kKStride + (C::kSwizzle ? piece ^ ((row & 1) * 4) : piece) * 16);
        if constexpr (kFp8) {
          const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const uint32_t b0 = e4m3x2_half2(words[q]), b1 = e4m3x2_half2(words[q] >> 16);
#pragma unroll
            for (int i = 0; i < kM; ++i)
              mma16<true>(s[i][j], qf[i][0][8 * c + 2 * q], qf[i][1][8 * c + 2 * q], qf[i][0][8 * c + 2 * q + 1],
                          qf[i][1][8 * c + 2 * q + 1], b0, b1);
          }
        } else {
#pragma unroll
          for (int i = 0; i < kM; ++i) {
            const uint32_t *q0 = &qf[i][0][4 * c], *q1 = &qf[i][1][4 * c];
            mma16<kF16>(s[i][j], q0[0], q1[0], q0[1], q1[1], w.x, w.y);
            mma16<kF16>(s[i][j], q0[2], q1[2], q0[3], q1[3], w.z, w.w);
          }
        }
      }
    }
    const int64_t key0 = (int64_t)cur.tile * C::kTile + warp * kKeys;
    const bool tail = key0 + kKeys > cur.s.cached;   // new tokens among the keys
    if (tail || bits != (kKeys == 32 ? 0xFFFFFFFFu : (1u << kKeys) - 1u)) {
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int64_t row = (int64_t)cur.rt * kRows + i * 16 + r * 8 + g;
          const bool in = row < (int64_t)cur.s.fresh * p.group;
          const int tok = in ? (int)(row / p.group) : 0;
#pragma unroll
          for (int j = 0; j < kNT; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int key = 8 * j + 2 * t + k;
              const int64_t i_new = key0 + key - cur.s.cached;
              const bool seen = ((bits >> key) & 1u) != 0u && (i_new < 0 || sees(p, cur.s.first + tok, tok, i_new));
              if (!seen) s[i][j][2 * r + k] = -INFINITY;
            }
        }
    }
    bool moved = false;
    float keep[kM][2];
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float mx = fmaxf(s[i][0][2 * r], s[i][0][2 * r + 1]);
#pragma unroll
        for (int j = 1; j < kNT; ++j) mx = fmaxf(mx, fmaxf(s[i][j][2 * r], s[i][j][2 * r + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
        // (fp16: rounded up, so that no P passes 2^15)
        const float top = kF16 ? __fadd_ru(__fmul_ru(mx, mult[i][r]), -kRaise) : mx * mult[i][r];
        const float now = fmaxf(m[i][r], top);
        const float base = now == -INFINITY ? 0.0f : now;   // (nothing seen yet)
        keep[i][r] = exp2_fast(m[i][r] - base);
        moved |= now != m[i][r];
        m[i][r] = now;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < kNT; ++j)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float e = exp2_fast(fmaf(s[i][j][2 * r + k], mult[i][r], -base));
            s[i][j][2 * r + k] = e;
            sum += e;
          }
        l[i][r] = fmaf(l[i][r], keep[i][r], sum);
      }
    if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int j = 0; j < kDT; ++j) {
          o[i][j][0] *= keep[i][0];
          o[i][j][1] *= keep[i][0];
          o[i][j][2] *= keep[i][1];
          o[i][j][3] *= keep[i][1];
        }
    }
    // A value that is not finite must not reach rows that do not see its key, and in a
    // product 0 times it would: such a tile (of new tokens; all others are seen by every
    // row) is added up key by key.
    if (tail) {
      bool odd = false;
      for (int at = lane; at < kKeys * C::kPieces; at += 32) {
        const uint4 w = lds128(vbase + at / C::kPieces * C::kVStride + at % C::kPieces * 16);
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (kFp8)
            odd |= __vcmpeq4(words[q] & 0x7F7F7F7Fu, 0x7F7F7F7Fu) != 0u;
          else
            odd |= __vcmpgeu2(words[q] & 0x7FFF7FFFu, kF16 ? 0x7C007C00u : 0x7F807F80u) != 0u;
        }
      }
      if (__builtin_expect(__any_sync(0xFFFFFFFFu, odd), 0)) {
        // in K's place, or where that is too small in the warp's place for its sums
        constexpr bool kFits = kRows * 4 <= C::kRow;
        static_assert(kFits || C::kOwnMerge, "room for the probabilities");
        float* const probs = reinterpret_cast<float*>(
            kFits ? smem + stage * C::kStageBytes + warp * C::kSlot
                  : smem + C::kStages * C::kStageBytes + warp * C::kMergeBytes);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kM; ++i)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int64_t row = (int64_t)cur.rt * kRows + i * 16 + r * 8 + g;
            const int tok = row < (int64_t)cur.s.fresh * p.group ? (int)(row / p.group) : 0;
#pragma unroll
            for (int j = 0; j < kNT; ++j)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                // (a key that the row does not see is -1: one that it sees may have a weight of 0 too)
                const int key = 8 * j + 2 * t + k;
                const int64_t i_new = key0 + key - cur.s.cached;
                const bool seen = ((bits >> key) & 1u) != 0u && (i_new < 0 || sees(p, cur.s.first + tok, tok, i_new));
                probs[(i * 16 + r * 8 + g) * kKeys + key] = seen ? s[i][j][2 * r + k] : -1.0f;
              }
          }
        __syncwarp();
        const uint8_t* const vs = smem + stage * C::kStageBytes + warp * C::kSlot + C::kKBytes;
        for (int key = 0; key < kKeys; ++key) {
#pragma unroll
          for (int j = 0; j < kDT; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int at = column(j, k) * C::kEs, piece = at / 16;
              const uint8_t* const a = vs + key * C::kVStride + (C::kSwizzle ? piece ^ (key & 7) : piece) * 16 + at % 16;
              float v;
              if (kFp8)
                v = e4m3_value(*a);
              else if (kF16)
                v = __half2float(*reinterpret_cast<const __half*>(a));
              else
                v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(a) << 16);
#pragma unroll
              for (int i = 0; i < kM; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                  const float pr = probs[(i * 16 + r * 8 + g) * kKeys + key];
                  if (!(pr <= 0.0f))
                    o[i][j][2 * r + k] = fmaf(pr, v, o[i][j][2 * r + k]);
                  else if (pr == 0.0f && !(fabsf(v) < INFINITY))
                    o[i][j][2 * r + k] += v;
                }
            }
        }
        __syncwarp();
        return;
      }
    }
#pragma unroll
    for (int c = 0; c < kKeys / 16; ++c) {
      uint32_t a[kM][4];
#pragma unroll
      for (int i = 0; i < kM; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float lo = s[i][2 * c + (k >> 1)][2 * (k & 1)], hi = s[i][2 * c + (k >> 1)][2 * (k & 1) + 1];
          a[i][k] = kF16 ? pack_f16x2(lo, hi) : pack_bf16x2(lo, hi);
        }
      // lane -> row of one of four 8 x 16-byte matrices: keys 0-7, 8-15 of one piece, then of the next
      const int key = c * 16 + ((lane >> 3) & 1) * 8 + (lane & 7);
#pragma unroll
      for (int j = 0; j < C::kPieces / 2; ++j) {
        const int piece = 2 * j + (lane >> 4);
        uint32_t r[4];
        ldmatrix_trans(vbase + key * C::kVStride + (C::kSwizzle ? piece ^ (key & 7) : piece) * 16, r);
        if constexpr (kFp8) {
          // a 16-bit unit is two adjacent elements of one key: even and odd ones apart
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const uint32_t w0 = __byte_perm(r[2 * q], 0u, 0x3120), w1 = __byte_perm(r[2 * q + 1], 0u, 0x3120);
            const uint32_t e0 = e4m3x2_half2(w0), e1 = e4m3x2_half2(w1);
            const uint32_t d0 = e4m3x2_half2(w0 >> 16), d1 = e4m3x2_half2(w1 >> 16);
#pragma unroll
            for (int i = 0; i < kM; ++i) {
              mma16<true>(o[i][4 * j + 2 * q], a[i][0], a[i][1], a[i][2], a[i][3], e0, e1);
              mma16<true>(o[i][4 * j + 2 * q + 1], a[i][0], a[i][1], a[i][2], a[i][3], d0, d1);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < kM; ++i) {
            mma16<kF16>(o[i][2 * j], a[i][0], a[i][1], a[i][2], a[i][3], r[0], r[1]);
            mma16<kF16>(o[i][2 * j + 1], a[i][0], a[i][1], a[i][2], a[i][3], r[2], r[3]);
          }
        }
      }
    }
  };

  // The end of an item, or of the CTA's run inside one: the warps' sums meet in shared
  // memory (the stage just used is free until the next tile's turn).
  auto end_item = [&](int stage, int64_t unit) {
    float* const own = reinterpret_cast<float*>(
        C::kOwnMerge ? smem + C::kStages * C::kStageBytes + warp * C::kMergeBytes
                     : smem + stage * C::kStageBytes + warp * C::kSlot);
    const int rows = (int)min((int64_t)kRows, (int64_t)cur.s.fresh * p.group - (int64_t)cur.rt * kRows);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kM; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        float sum = l[i][r];
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 1);
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, 2);
        const int row = i * 16 + r * 8 + g;
        if (t == 0) warp_ml[warp][row] = make_float2(m[i][r], sum);
        // adjacent elements in one store, the rows' columns permuted over the banks
        if (row < rows) {
#pragma unroll
          for (int j = 0; j < kDT; j += 2) {
            const float* const x = &o[i][j][2 * r];
            const float* const y = &o[i][j + 1][2 * r];
            if constexpr (kFp8) {
              *reinterpret_cast<float4*>(own + row * kD + (column(j, 0) ^ ((row & 7) * 4))) =
                  make_float4(x[0], y[0], x[1], y[1]);
            } else {
              *reinterpret_cast<float2*>(own + row * kD + (column(j, 0) ^ ((row & 7) * 4))) = make_float2(x[0], x[1]);
              *reinterpret_cast<float2*>(own + row * kD + (column(j + 1, 0) ^ ((row & 7) * 4))) = make_float2(y[0], y[1]);
            }
          }
        }
      }
    __syncthreads();
    const int64_t item0 = unit - cur.tile, item1 = item0 + cur.tiles - 1;   // the item's first and last unit
    const bool whole = item0 >= run.begin && item1 < run.end;
    const int64_t part_row = (int64_t)(2 * blockIdx.x + (item0 < run.begin ? 0 : 1)) * kRows;
    const uint8_t* const sums = C::kOwnMerge ? smem + C::kStages * C::kStageBytes : smem + stage * C::kStageBytes;
    constexpr int kStep = C::kOwnMerge ? C::kMergeBytes : C::kSlot;
    for (int i = threadIdx.x; i < rows * (p.head_dim / 4); i += kThreads) {
      const int row = i / (p.head_dim / 4), d = i % (p.head_dim / 4) * 4;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, warp_ml[w][row].x);
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2 ml = warp_ml[w][row];
        const float f = exp2_fast(ml.x - base);
        const float4 x = *reinterpret_cast<const float4*>(sums + w * kStep + (row * kD + (d ^ ((row & 7) * 4))) * 4);
        sum = fmaf(ml.y, f, sum);
        v = make_float4(fmaf(x.x, f, v.x), fmaf(x.y, f, v.y), fmaf(x.z, f, v.z), fmaf(x.w, f, v.w));
      }
      if (whole) {
        const int64_t r = (int64_t)cur.rt * kRows + row;
        const int64_t token = cur.s.first + r / p.group;
        const int head = cur.h * p.group + (int)(r % p.group);
        const float inv = sum == 0.0f ? 0.0f : v_scale / sum;
        store_out4(p, token, head, d, make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
        if (p.lse != nullptr && d == 0) p.lse[token * p.lse_token + head] = log_sum(top, sum);
      } else {
        if (d == 0) p.part_ml[part_row + row] = make_float2(top, sum);
        *reinterpret_cast<float4*>(p.part + (part_row + row) * kD + d) = v;
      }
    }
    if (!whole) {
      if (threadIdx.x == 0) {
        Unfinished& u = unfinished[num_unfinished];
        u = {cur.s.first, cur.rt * kRows, cur.h * p.group, rows, (int)split_owner(run.split, item0),
             (int)split_owner(run.split, item1)};
      }
      ++num_unfinished;
    }
    __syncthreads();
  };

  Place next;
  {
    Place early[C::kStages - 1];   // (their table entries are on their way together)
#pragma unroll
    for (int s = 0; s < C::kStages - 1; ++s) early[s] = fetch();
#pragma unroll
    for (int s = 0; s < C::kStages - 1; ++s) issue(s, early[s]);
    next = fetch();
  }
  bool fresh_item = true;
  int stage = 0;
  for (int64_t unit = run.begin, after; unit < run.end; unit = after) {
    if (fresh_item) begin_item();
    cp_async_wait<C::kStages - 2>();
    __syncwarp();
    issue(stage == 0 ? C::kStages - 1 : stage - 1, next);
    next = fetch();
    compute(stage);
    const bool done = cur.tile + 1 == cur.tiles;
    if (done || unit + 1 == run.end) end_item(stage, unit);
    fresh_item = done;
    after = unit + 1 + (done ? p.item_cost : 0);
    if (after < run.end) advance<kRows, C::kTile>(p, cur);
    if (++stage == C::kStages) stage = 0;
    __syncwarp();
  }
  cp_async_wait<0>();
  // The unfinished items, now that the registers are free: the last CTA of a group to arrive joins
  // the group's parts, the last group's the groups'.
  auto arrive = [&](unsigned* count, int parties) {   // whether the last
    // (alone it takes no count: an item's last group, of this CTA alone, has the number that the item
    // which begins here counts with)
    if (parties == 1) return true;
    // (releases the CTA's stores, which the barrier orders before, and acquires the other CTAs'; a
    // relaxed one between two __threadfence() took 0.35 of 10.1 us longer)
    unsigned before;
    asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(before) : "l"(count) : "memory");
    const bool all = before == (unsigned)(parties - 1);
    if (all) *count = 0u;   // as it was before the call
    return all;
  };
  auto group_of = [&](const Unfinished& u) { return few_join_group(u.rows, p.head_dim); };
  __syncthreads();
  if ((int)threadIdx.x < num_unfinished) {   // (both at a time)
    const Unfinished u = unfinished[threadIdx.x];
    const int group = group_of(u), from = u.first + ((int)blockIdx.x - u.first) / group * group;
    last_flag[threadIdx.x] = arrive(&p.counts[from], min(u.last, from + group - 1) - from + 1);
  }
  __syncthreads();
  for (int i = 0; i < num_unfinished; ++i) {
    if (!last_flag[i]) continue;
    const Unfinished u = unfinished[i];
    const int group = group_of(u), groups = (u.last - u.first) / group + 1;
    const int from = u.first + ((int)blockIdx.x - u.first) / group * group;
    join_few<kRows, kD>(p, u, from, min(u.last, from + group - 1), 1, groups == 1, v_scale, warp_ml[0]);
    __syncthreads();
    if (groups == 1) continue;
    if (threadIdx.x == 0) last_flag[i] = arrive(&p.counts[kMostCtas + u.first], groups);
    __syncthreads();
    if (last_flag[i]) join_few<kRows, kD>(p, u, u.first, u.last, group, true, v_scale, warp_ml[0]);
    __syncthreads();
  }
}


template <CacheKind kKind, int kD, int kM>
cudaError_t launch_attn(AttnParams p, cudaStream_t s, Device dev) {
  using C = AttnCfg<kKind, kD, kM>;
  struct Setup {
    cudaError_t err;
    int ctas;
  };
  static PerDevice<Setup> per_device;
  const Setup& setup = per_device.get(dev.index, [&] {
    Setup t{cudaFuncSetAttribute(attn_kernel<kKind, kD, kM>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem), 0};
    if (t.err == cudaSuccess)
      t.err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&t.ctas, attn_kernel<kKind, kD, kM>, kWarps * 32, C::kSmem);
    if (t.err == cudaSuccess && t.ctas < 1) t.err = cudaErrorInvalidConfiguration;
    return t;
  });
  if (setup.err != cudaSuccess) return setup.err;
  // two unfinished items per CTA in the workspace, behind the counts
  constexpr int64_t kPart = 2 * C::kRows * ((int64_t)kD * 4 + 8);
  const int64_t most = std::min<int64_t>(kMostCtas, (kWorkspaceBytes - kCountBytes) / kPart);
  const int ctas = (int)std::min<int64_t>((int64_t)setup.ctas * dev.num_sms, most);
  p.part_ml = reinterpret_cast<float2*>(reinterpret_cast<uint8_t*>(p.counts) + kCountBytes);
  p.part = reinterpret_cast<float*>(p.part_ml + (int64_t)2 * C::kRows * ctas);
  p.least = few_least(C::kTile);
  p.item_cost = kFewItemCost;
  return launch_pdl(attn_kernel<kKind, kD, kM>, dim3((unsigned)ctas), kWarps * 32, C::kSmem, s, p);
}

// Rows past 16 come here where pages do not fit the tiles.  Heads of up to 64 then take 32 rows to a
// read of the keys (16 sequences of 4096-8192 keys, 20 rows: 61 us, twice 16 rows 112); longer heads'
// fragments for 32 rows do not fit the registers (heads of 128: 181 us, twice 16 rows 157).
template <CacheKind kKind>
cudaError_t launch_attn_kind(const AttnParams& p, cudaStream_t s, Device dev) {
  if (p.head_dim <= 64)
    return p.tokens * p.group > (int64_t)16 * p.sequences ? launch_attn<kKind, 64, 2>(p, s, dev)
                                                          : launch_attn<kKind, 64, 1>(p, s, dev);
  if constexpr (kKind != CacheKind::kE4m3)
    if (p.head_dim <= 96) return launch_attn<kKind, 96, 1>(p, s, dev);
  if (p.head_dim <= 128) return launch_attn<kKind, 128, 1>(p, s, dev);
  if (p.head_dim <= 192) return launch_attn<kKind, 192, 1>(p, s, dev);
  return launch_attn<kKind, 256, 1>(p, s, dev);
}

}  // namespace

}  // namespace qlin
