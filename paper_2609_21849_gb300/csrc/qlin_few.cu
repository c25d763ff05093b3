// Linears of a few tokens (few_tokens says which).  The weights are read once per 16
// tokens and everything else is small, so the bound is HBM: a row's elements meet at most
// 16 tokens at a time.  A tcgen05 tile of 128 x 64 spends its 128 rows on them and has
// N / 64 CTAs to pull W with; here a CTA takes 16 or 32 rows of W, its warps (or a
// cluster's) split K among them, and W goes straight from global memory into mma.sync
// fragments.
//
// Measured with bias and SiLU, operands of several calls in turn: bf16 1 x 12288 x 3072
// 12.6 us, 90% of the measured copy rate, 8 x 3072 x 12288 13.7, 83%; FP8 1 x 12288 x 3072
// 7.6 us, 75%, 8 x 3072 x 12288 8.9, 64%, 1 x 3072 x 3072 4.4.  What is left is a launch,
// the first loads and the joined sums, about three microseconds.  NVFP4 1 x 12288 x 3072
// takes 7.9 us, 40%: codes become fp16 and meet their block scales in registers, sixteen
// instructions per 16 bytes.
//
// Fragments without shared memory: an MMA sums over K in any order, as long as both
// operands agree.  Lane (g, t) = (lane / 4, lane % 4) loads the 16 bytes at 16 t of a
// 64-byte chunk of W's rows g and g + 8 and of token g, and hands the four words to
// two MMAs of 32 bytes of K as they come: words 0 and 1 are the lane's two K slots of
// the first, 2 and 3 of the second.
#include "qlin_internal.h"

namespace qlin {

namespace {

enum class Kind { kNvfp4, kFp8, kBf16, kFp16 };

constexpr int kBlock = 16;        // rows of W per MMA, and of an NVFP4 block of y
constexpr int kChunk = 64;        // bytes of a row per warp and step
constexpr int kMinWarps = 4, kMaxWarps = 8, kMaxSplit = 8;   // (a thread has kTiles outputs at most)

struct FewParams {
  const uint8_t* a;
  int64_t a_row;            // bytes
  const uint8_t* w;
  const uint8_t* sfa;       // NVFP4 block scales
  const uint8_t* sfb;
  const float* sdec_a;
  const float* sdec_w;
  int a_per_row, w_per_channel;
  const uint16_t* bias;
  const uint16_t* residual;
  int64_t residual_stride;
  int act;
  uint16_t* y;
  int M;
  int64_t N, K;
  const float* next_scale;
  uint8_t* rq_codes;
  uint8_t* rq_scales;
  float* rq_tensor_scale;
  int64_t rq_col0, rq_cols;
  int split;                // CTAs of a cluster
};

__device__ __forceinline__ uint4 ld_stream(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

__device__ __forceinline__ uint4 ld_keep(const uint8_t* p) {
  uint4 v;
  asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// c += A B of 16 x 8: A's rows of W (a0, a2 of row g, a1, a3 of row g + 8), B's tokens.
template <Kind kKind>
__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                    uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (kKind == Kind::kBf16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32"
        " {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32"
        " {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// NVFP4: eight e2m1 codes times their block scale as fp16, exactly (two bits times
// four bits of significand; 2^-10 to 2688).
__device__ __forceinline__ void e2m1x8_scaled(uint32_t w, __half2 s, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(w));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 v = __hmul2(*reinterpret_cast<__half2*>(&h[i]), s);
    h[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}

// FP8: four E4M3 codes as fp16, exactly.  (sm_103a has no E4M3 mma.sync of its own: the
// instruction becomes these conversions, repeated for every product.)
__device__ __forceinline__ void e4m3x4_half(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\t"
      "cvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
      : "=r"(lo), "=r"(hi)
      : "r"(w));
}

// Two adjacent E4M3 scales as two pairs of equal halves.
__device__ __forceinline__ void scale_pairs(uint16_t s2, __half2 (&s)[2]) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(s2));
  const __half2 v = *reinterpret_cast<const __half2*>(&h);
  s[0] = __low2half2(v);
  s[1] = __high2half2(v);
}

__device__ __forceinline__ float load16f(const uint16_t* p, bool fp16) {
  const uint16_t w = *p;
  return fp16 ? __half2float(__ushort_as_half(w)) : __uint_as_float((uint32_t)w << 16);
}

__device__ __forceinline__ void st_cluster(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// Chunks in flight per warp.
template <Kind kKind, int kTiles, int kRowTiles>
constexpr int kUnrollOf = kRowTiles == 2 ? 2 : kKind == Kind::kNvfp4 ? 2 : 4;

// kTiles: groups of eight tokens; kRowTiles: of sixteen rows of W.  A cluster of CTAs shares the rows of W, all of
// its warps taking chunks of K in turn; the CTAs' sums meet in distributed shared memory.
template <Kind kKind, int kTiles, int kRowTiles>
__global__ void __launch_bounds__(kMaxWarps * 32) few_kernel(const FewParams p) {
  constexpr bool kFp4 = kKind == Kind::kNvfp4;
  constexpr int kRows = kBlock * kRowTiles, kOuts = kTiles * kRowTiles;
  constexpr int kUnroll = kUnrollOf<kKind, kTiles, kRowTiles>;
  __shared__ float red[kMaxWarps][kTiles * 8][kRows + 1];
  __shared__ float part[kMaxSplit][kTiles * 8][kRows];   // the cluster's sums of this CTA's tokens
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int warps = blockDim.x >> 5;
  const int m0 = (int)blockIdx.y * kTiles * 8;   // the CTA's first token
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
  const int64_t n0 = (int64_t)(blockIdx.x / (unsigned)p.split) * kRows;
  const int64_t w_row = kFp4 ? p.K / 2 : kKind == Kind::kFp8 ? p.K : p.K * 2;
  const int chunks = (int)((w_row + kChunk - 1) / kChunk);
  const int stride = warps * p.split;   // warps that share the rows
  // every CTA of the cluster runs before one writes into another's shared memory
  if (p.split > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  // the warp's first chunks of W into L2 while the previous kernel still runs (a hint
  // that returns no data, so that it may be issued before the wait)
  for (int u = 0; u < kUnroll; ++u) {
    const int c = rank * warps + warp + u * stride;
    if (t < 2 * kRowTiles && c < chunks)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(p.w + (n0 + g + 8 * t) * w_row + (int64_t)c * kChunk));
  }
  grid_dep_wait();
  grid_dep_launch();
  // what this thread's outputs need beside the sums: loaded now, used after them
  // (loaded there, they cost a chain of two loads at the end)
  constexpr bool kF16 = kKind == Kind::kFp16;
  const bool requant = kKind != Kind::kBf16 && !kF16 && p.next_scale != nullptr;
  float o_scale[kOuts], o_bias[kOuts], o_res[kOuts];
  bool o_own[kOuts];   // (the same for the sixteen threads of a token)
#pragma unroll
  for (int k = 0; k < kOuts; ++k) {
    const int i = threadIdx.x + k * blockDim.x, m = m0 + i / kRows;
    const int64_t n = n0 + i % kRows;
    // of a cluster's CTAs each takes every split-th token
    const bool own = i < kTiles * 8 * kRows && m < p.M && (p.split == 1 || (m - m0) % p.split == rank);
    o_own[k] = own;
    o_scale[k] = 1.0f;
    o_bias[k] = o_res[k] = 0.0f;
    if (!own) continue;
    if constexpr (kFp4)
      o_scale[k] = __fmul_rn(*p.sdec_a, *p.sdec_w);
    else if constexpr (kKind == Kind::kFp8)
      o_scale[k] = __fmul_rn(p.sdec_a[p.a_per_row ? m : 0], p.sdec_w[p.w_per_channel ? n : 0]);
    if (p.bias != nullptr) o_bias[k] = load16f(p.bias + n, kF16);
    if (p.residual != nullptr) o_res[k] = load16f(p.residual + m * p.residual_stride + n, kF16);
  }
  const float s_next = requant ? *p.next_scale : 1.0f;

  // Chunks through a ring of registers: each is loaded kUnroll chunks ahead of its use.
  // The pointers run along the warp's chunks; a token past M reads the CTA's first one's row
  // (its column of the sums is not used).
  float acc[kRowTiles][kTiles][4] = {};
  uint4 va[kUnroll][kRowTiles][2], vb[kUnroll][kTiles];
  uint16_t sa[kUnroll][kRowTiles][2], sb[kUnroll][kTiles];
  const int first = rank * warps + warp;
  int left = (chunks - first + stride - 1) / stride;   // chunks to load
  int tail = kFp4 ? (int)(w_row - (int64_t)first * kChunk) - 16 * t : 0;   // bytes of the row from here
  const uint8_t* w = p.w + (n0 + g) * w_row + 16 * t + (int64_t)first * kChunk;
  const uint8_t *a[kTiles], *fa[kTiles], *fw[kRowTiles][2];
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    const int64_t m = m0 + j * 8 + g < p.M ? m0 + j * 8 + g : m0;
    a[j] = p.a + m * p.a_row + 16 * t + (int64_t)first * kChunk;
    // the scales of blocks 8 c + 2 t and the next: 1024 bytes per chunk of 128 elements
    fa[j] = kFp4 ? p.sfa + scale_offset(m, 8 * (int64_t)first + 2 * t, p.K) : nullptr;
  }
#pragma unroll
  for (int h = 0; h < 2 * kRowTiles; ++h)
    fw[h / 2][h % 2] = kFp4 ? p.sfb + scale_offset(n0 + g + 8 * h, 8 * (int64_t)first + 2 * t, p.K) : nullptr;
  const int step = stride * kChunk, fstep = stride * 1024;
  auto load = [&](int u) {
    // NVFP4 rows are multiples of 32 bytes: the last chunk may be half a chunk
    const bool in = left > 0 && (!kFp4 || tail > 0);
#pragma unroll
    for (int h = 0; h < 2 * kRowTiles; ++h) {
      va[u][h / 2][h % 2] = make_uint4(0u, 0u, 0u, 0u);
      if (in) va[u][h / 2][h % 2] = ld_stream(w + 8 * h * w_row);
      if (kFp4) {
        sa[u][h / 2][h % 2] = 0;
        if (in) sa[u][h / 2][h % 2] = *reinterpret_cast<const uint16_t*>(fw[h / 2][h % 2]);
        fw[h / 2][h % 2] += fstep;
      }
    }
#pragma unroll
    for (int j = 0; j < kTiles; ++j) {
      vb[u][j] = make_uint4(0u, 0u, 0u, 0u);
      if (in) vb[u][j] = ld_keep(a[j]);
      a[j] += step;
      if (kFp4) {
        sb[u][j] = 0;
        if (in) sb[u][j] = *reinterpret_cast<const uint16_t*>(fa[j]);
        fa[j] += fstep;
      }
    }
    w += step;
    tail -= step;
    --left;
  };
  auto multiply = [&](int u) {
    if constexpr (kFp4) {
      __half2 sw[kRowTiles][2][2], st[kTiles][2];
#pragma unroll
      for (int h = 0; h < 2 * kRowTiles; ++h) scale_pairs(sa[u][h / 2][h % 2], sw[h / 2][h % 2]);
#pragma unroll
      for (int j = 0; j < kTiles; ++j) scale_pairs(sb[u][j], st[j]);
#pragma unroll
      for (int q = 0; q < 4; ++q) {   // eight elements of K per lane
        auto word = [&](const uint4& v) { return q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w; };
        uint32_t hb[kTiles][4];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) e2m1x8_scaled(word(vb[u][j]), st[j][q >> 1], hb[j]);
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
          uint32_t h0[4], h1[4];
          e2m1x8_scaled(word(va[u][i][0]), sw[i][0][q >> 1], h0);
          e2m1x8_scaled(word(va[u][i][1]), sw[i][1][q >> 1], h1);
#pragma unroll
          for (int j = 0; j < kTiles; ++j) {
            mma<kKind>(acc[i][j], h0[0], h1[0], h0[1], h1[1], hb[j][0], hb[j][1]);
            mma<kKind>(acc[i][j], h0[2], h1[2], h0[3], h1[3], hb[j][2], hb[j][3]);
          }
        }
      }
    } else if constexpr (kKind == Kind::kFp8) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {   // four elements of K per lane
        auto word = [&](const uint4& v) { return q == 0 ? v.x : q == 1 ? v.y : q == 2 ? v.z : v.w; };
        uint32_t hb[kTiles][2];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) e4m3x4_half(word(vb[u][j]), hb[j][0], hb[j][1]);
#pragma unroll
        for (int i = 0; i < kRowTiles; ++i) {
          uint32_t h0[2], h1[2];
          e4m3x4_half(word(va[u][i][0]), h0[0], h0[1]);
          e4m3x4_half(word(va[u][i][1]), h1[0], h1[1]);
#pragma unroll
          for (int j = 0; j < kTiles; ++j) mma<kKind>(acc[i][j], h0[0], h1[0], h0[1], h1[1], hb[j][0], hb[j][1]);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          const uint4 &x = va[u][i][0], &y = va[u][i][1], &b = vb[u][j];
          mma<kKind>(acc[i][j], x.x, y.x, x.y, y.y, b.x, b.y);
          mma<kKind>(acc[i][j], x.z, y.z, x.w, y.w, b.z, b.w);
        }
    }
  };
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) load(u);
  for (int done = left + kUnroll; done > 0; done -= kUnroll) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      multiply(u);   // (zeros past the last chunk)
      load(u);
    }
  }
  // the warps' sums, in order
#pragma unroll
  for (int i = 0; i < kRowTiles; ++i)
#pragma unroll
    for (int j = 0; j < kTiles; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) red[warp][j * 8 + 2 * t + (k & 1)][i * kBlock + g + 8 * (k >> 1)] = acc[i][j][k];
  __syncthreads();
  auto cta_sum = [&](int m, int r) {
    float v = 0.0f;
    for (int w = 0; w < warps; ++w) v = __fadd_rn(v, red[w][m][r]);
    return v;
  };
  if (p.split > 1) {
    // each CTA's sums go to the CTA that finishes the token, which adds them in order
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    for (int i = threadIdx.x; i < kTiles * 8 * kRows; i += blockDim.x) {
      const int m = i / kRows, r = i % kRows;
      st_cluster(mapa_shared(&part[rank][m][r], (uint32_t)(m % p.split)), cta_sum(m, r));
    }
    cluster_sync();
  }
  // sixteen neighbouring threads finish a token's sixteen outputs
  const float s_enc = encode_scale(s_next);
  if (requant && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && p.rq_tensor_scale != p.next_scale)
    *p.rq_tensor_scale = s_next;
#pragma unroll
  for (int k = 0; k < kOuts; ++k) {
    const int i = threadIdx.x + k * blockDim.x;
    if (i >= kTiles * 8 * kRows) break;   // (whole warps)
    const int i_m = i / kRows, r = i % kRows;
    const bool own = o_own[k];
    const int64_t n = n0 + r, m = m0 + i_m;
    float v = 0.0f;
    if (own) {
      if (p.split == 1) {
        v = cta_sum(i_m, r);
      } else {
        for (int q = 0; q < p.split; ++q) v = __fadd_rn(v, part[q][i_m][r]);
      }
      v = __fadd_rn(__fmul_rn(v, o_scale[k]), o_bias[k]);
      float2 one[1] = {make_float2(v, v)};
      activate(one, p.act);
      v = __fadd_rn(one[0].x, o_res[k]);
    }
    const uint32_t bits = (kF16 ? pack_f16x2(v, 0.0f) : pack_bf16x2(v, 0.0f)) & 0xFFFFu;
    if (own && p.y != nullptr) p.y[m * p.N + n] = (uint16_t)bits;
    if (!requant) continue;
    const int64_t col = n - p.rq_col0;
    const int64_t b0 = n - r % kBlock;   // of the sixteen
    const bool inside = own && b0 >= p.rq_col0 && b0 + kBlock <= p.rq_col0 + p.rq_cols;
    const float y16 = __uint_as_float(bits << 16);
    if constexpr (kKind == Kind::kFp8) {
      if (inside) p.rq_codes[m * p.rq_cols + col] = (uint8_t)e4m3_code(__fmul_rn(y16, s_enc));
    } else if constexpr (kFp4) {
      uint32_t mx = bits & 0x7FFFu;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = max(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, o));
      const uint32_t code = e4m3_code_div6(__fmul_rn(__uint_as_float(mx << 16), s_enc));
      const float r_b = code == 0u ? 0.0f : __fdiv_rn(s_enc, e4m3_value(code));
      const float q = __fmul_rn(y16, r_b), q1 = __shfl_down_sync(0xFFFFFFFFu, q, 1);
      const float f[8] = {q, q1, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      if (inside && (r & 1) == 0) p.rq_codes[m * (p.rq_cols / 2) + col / 2] = (uint8_t)e2m1x8(f);
      if (inside && r % kBlock == 0) p.rq_scales[scale_offset(m, col / 16, p.rq_cols)] = (uint8_t)code;
    }
  }
}

// How a launch splits its work: row tiles per CTA, warps per CTA, CTAs per cluster.
struct Split {
  int row_tiles, warps, ctas;
};

// One wave: CTAs have a fixed cost (16 x 12288 x 3072 NVFP4 with 768 CTAs on 760 places
// 12.0 us, with 384 of twice the rows 10.0), so the warps that share rows are as many as
// stay resident together (`resident` warps per SM of each row tiling), at most one per
// four chunks of K, or two while that leaves the machine near empty (NVFP4 48 x 512 x 2048
// 3.5 -> 3.1 us).  A cluster pays where it gives sixteen warps or more and either few of
// them share an SM (fp16 2 x 1024 x 2560 4.1 -> 3.2 us; bf16 48 x 512 x 2048, ten per SM,
// 3.9 -> 4.6) or K is long (FP8 8 x 3072 x 12288 10.3 -> 8.9 us with two CTAs; bf16 1 x 3072
// x 3072 6.0 -> 8.6), never over short rows (bf16 10 x 320 x 1280 2.9 -> 3.3 us, 4 x 1024 x
// 1984 3.7 -> 3.1; an NVFP4 chunk takes longer: 10 x 320 x 4352 4.3 -> 4.4, x 5120 4.5 -> 3.8).
Split choose_split(Kind kind, int64_t N, int64_t token_groups, int64_t K, int64_t chunks,
                   const int (&resident)[2], int num_sms) {
  const int64_t least = kind == Kind::kNvfp4 ? 40 : 60;
  Split best{1, kMinWarps, 1};
  for (int rt = 1; rt <= 2; ++rt) {
    const int64_t units = N / (kBlock * rt) * token_groups;
    bool fits = false;
    for (int ctas = 1; ctas <= kMaxSplit; ++ctas)
      for (int w = kMinWarps; w <= kMaxWarps; ++w) {
        const int64_t warps = w * ctas, all = units * warps;
        const int64_t per = all <= 6 * num_sms ? 2 : 4;
        if (units * ctas > (int64_t)num_sms * (resident[rt - 1] / w)) continue;
        if (warps > std::max<int64_t>(kMinWarps, (chunks + per - 1) / per)) continue;
        if (ctas > 1 && (warps < 16 || chunks < least || (all > 9 * num_sms && (K < 8192 || ctas > 2)))) continue;
        if (!fits || warps > best.warps * best.ctas) best = {rt, w, ctas};
        fits = true;
      }
    if (fits) return best;
  }
  return {2, kMinWarps, 1};
}

template <Kind kKind, int kTiles>
cudaError_t launch_tiles(FewParams p, cudaStream_t s, Device dev) {
  static constexpr void (*kKernels[2])(FewParams) = {few_kernel<kKind, kTiles, 1>, few_kernel<kKind, kTiles, 2>};
  struct Setup {
    cudaError_t err;
    int resident[2];
  };
  static PerDevice<Setup> per_device;
  const Setup& setup = per_device.get(dev.index, [&] {
    Setup t{cudaSuccess, {0, 0}};
    for (int i = 0; i < 2 && t.err == cudaSuccess; ++i) {
      int blocks = 0;
      t.err = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&blocks, kKernels[i], kMinWarps * 32, 0);
      t.resident[i] = blocks * kMinWarps;
    }
    return t;
  });
  if (setup.err != cudaSuccess) return setup.err;
  const int64_t row = kKind == Kind::kNvfp4 ? p.K / 2 : kKind == Kind::kFp8 ? p.K : p.K * 2;
  const Split split = choose_split(kKind, p.N, (p.M + kTiles * 8 - 1) / (kTiles * 8), p.K, (row + kChunk - 1) / kChunk,
                                   setup.resident, dev.num_sms);
  p.split = split.ctas;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)p.split;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(p.N / (kBlock * split.row_tiles) * p.split),
                     (unsigned)((p.M + kTiles * 8 - 1) / (kTiles * 8)), 1);
  cfg.blockDim = dim3((unsigned)split.warps * 32, 1, 1);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kKernels[split.row_tiles - 1], p);
}

template <Kind kKind>
cudaError_t launch_kind(const FewParams& p, cudaStream_t s, Device dev) {
  return p.M <= 8 ? launch_tiles<kKind, 1>(p, s, dev) : launch_tiles<kKind, 2>(p, s, dev);
}

}  // namespace

cudaError_t launch_few(const GemmArgs& a, cudaStream_t s, Device dev) {
  FewParams p{};
  p.a = static_cast<const uint8_t*>(a.a_codes);
  p.a_row = a.bf16 ? a.a_row_bytes : a.fp4 ? a.K / 2 : a.K;
  p.w = static_cast<const uint8_t*>(a.w_codes);
  p.sfa = a.sfa;
  p.sfb = a.sfb;
  p.sdec_a = a.sdec_a;
  p.sdec_w = a.sdec_w;
  p.a_per_row = a.a_per_row ? 1 : 0;
  p.w_per_channel = a.w_per_channel;
  p.bias = static_cast<const uint16_t*>(a.bias);
  p.residual = static_cast<const uint16_t*>(a.residual);
  p.residual_stride = a.residual_stride;
  p.act = a.act;
  p.y = static_cast<uint16_t*>(a.y);
  p.M = (int)a.M;
  p.N = a.N;
  p.K = a.K;
  p.next_scale = a.next_scale;
  p.rq_codes = a.rq_codes;
  p.rq_scales = a.rq_scales;
  p.rq_tensor_scale = a.rq_tensor_scale;
  p.rq_col0 = a.rq_col0;
  p.rq_cols = a.rq_cols;
  return a.bf16 ? (a.fp16 ? launch_kind<Kind::kFp16>(p, s, dev) : launch_kind<Kind::kBf16>(p, s, dev))
         : a.fp4 ? launch_kind<Kind::kNvfp4>(p, s, dev)
                 : launch_kind<Kind::kFp8>(p, s, dev);
}

}  // namespace qlin
