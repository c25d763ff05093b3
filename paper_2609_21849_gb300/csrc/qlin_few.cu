// Linears of a few tokens (qlin_linear_* up to kFewTokens rows).  The weights are
// read once and everything else is small, so the bound is HBM: each of a row's
// elements meets at most 16 tokens.  A tcgen05 tile of 128 x 64 spends its 128 rows
// on one token and has N / 64 CTAs to pull W with; here a CTA takes 16 rows of W
// (N / 16 CTAs, several to an SM), its warps split K among them, and W goes straight
// from global memory into mma.sync fragments.
//
// Fragments without shared memory: an MMA sums over K in any order, as long as both
// operands agree.  Lane (g, t) = (lane / 4, lane % 4) loads the 16 bytes at 16 t of a
// 64-byte chunk of W's rows g and g + 8 and of token g, and hands the four words to
// two MMAs of 32 bytes of K as they come: words 0 and 1 are the lane's two K slots of
// the first, 2 and 3 of the second.
#include "qlin_internal.h"

namespace qlin {

namespace {

#ifndef FW
#define FW 32
#endif
enum class Kind { kNvfp4, kFp8, kBf16, kFp16 };

constexpr int kRows = 16;         // rows of W per CTA: one MMA's M, one NVFP4 block of y
constexpr int kChunk = 64;        // bytes of a row per warp and step
constexpr int kMaxWarps = 8, kMaxSplit = 8;

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
  if constexpr (kKind == Kind::kFp8)
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32"
        " {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else if constexpr (kKind == Kind::kBf16)
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

__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// kTiles: groups of eight tokens.  A cluster of CTAs shares 16 rows of W, all of its
// warps taking chunks of K in turn; the CTAs' sums meet in distributed shared memory.
template <Kind kKind, int kTiles>
__global__ void __launch_bounds__(kMaxWarps * 32) few_kernel(const FewParams p) {
  constexpr bool kFp4 = kKind == Kind::kNvfp4;
  constexpr int kUnroll = kFp4 ? 2 : 4;
  __shared__ float red[kMaxWarps][kTiles * 8][kRows + 1];
  __shared__ float part[kTiles * 8][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int warps = blockDim.x >> 5;
  const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
  const int64_t n0 = (int64_t)(blockIdx.x / (unsigned)p.split) * kRows;
  const int64_t w_row = kFp4 ? p.K / 2 : kKind == Kind::kFp8 ? p.K : p.K * 2;
  const int chunks = (int)((w_row + kChunk - 1) / kChunk);
  const uint8_t* const w0 = p.w + (n0 + g) * w_row + 16 * t;
  const uint8_t* const w1 = w0 + 8 * w_row;
  const int stride = warps * p.split;   // warps that share the rows
  grid_dep_wait();
  grid_dep_launch();
  float acc[kTiles][4] = {};
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  for (int c0 = rank * warps + warp; c0 < chunks; c0 += stride * kUnroll) {
    uint4 va[kUnroll][2], vb[kUnroll][kTiles];
    uint16_t sa[kUnroll][2], sb[kUnroll][kTiles];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int c = c0 + u * stride;
      const int64_t at = (int64_t)c * kChunk;
      // NVFP4 rows are multiples of 32 bytes: the last chunk may be half a chunk
      const bool in = c < chunks && (!kFp4 || at + 16 * t < w_row);
      va[u][0] = in ? ld_stream(w0 + at) : zero;
      va[u][1] = in ? ld_stream(w1 + at) : zero;
      const int64_t blk = (int64_t)c * 8 + 2 * t;   // NVFP4: first block of the 16 bytes
      if (kFp4) {
        sa[u][0] = in ? *reinterpret_cast<const uint16_t*>(p.sfb + scale_offset(n0 + g, blk, p.K)) : 0;
        sa[u][1] = in ? *reinterpret_cast<const uint16_t*>(p.sfb + scale_offset(n0 + g + 8, blk, p.K)) : 0;
      }
#pragma unroll
      for (int j = 0; j < kTiles; ++j) {
        const int m = j * 8 + g;
        const bool tok = in && m < p.M;
        vb[u][j] = tok ? ld_keep(p.a + m * p.a_row + at + 16 * t) : zero;
        if (kFp4)
          sb[u][j] = tok ? *reinterpret_cast<const uint16_t*>(p.sfa + scale_offset(m, blk, p.K)) : 0;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if constexpr (kFp4) {
        __half2 s0[2], s1[2], st[kTiles][2];
        scale_pairs(sa[u][0], s0);
        scale_pairs(sa[u][1], s1);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) scale_pairs(sb[u][j], st[j]);
        const uint32_t a0[4] = {va[u][0].x, va[u][0].y, va[u][0].z, va[u][0].w};
        const uint32_t a1[4] = {va[u][1].x, va[u][1].y, va[u][1].z, va[u][1].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {   // eight elements of K per lane
          uint32_t h0[4], h1[4];
          e2m1x8_scaled(a0[q], s0[q >> 1], h0);
          e2m1x8_scaled(a1[q], s1[q >> 1], h1);
#pragma unroll
          for (int j = 0; j < kTiles; ++j) {
            const uint32_t b[4] = {vb[u][j].x, vb[u][j].y, vb[u][j].z, vb[u][j].w};
            uint32_t hb[4];
            e2m1x8_scaled(b[q], st[j][q >> 1], hb);
            mma<kKind>(acc[j], h0[0], h1[0], h0[1], h1[1], hb[0], hb[1]);
            mma<kKind>(acc[j], h0[2], h1[2], h0[3], h1[3], hb[2], hb[3]);
          }
        }
      } else {
#pragma unroll
        for (int j = 0; j < kTiles; ++j) {
          mma<kKind>(acc[j], va[u][0].x, va[u][1].x, va[u][0].y, va[u][1].y, vb[u][j].x, vb[u][j].y);
          mma<kKind>(acc[j], va[u][0].z, va[u][1].z, va[u][0].w, va[u][1].w, vb[u][j].z, vb[u][j].w);
        }
      }
    }
  }
  // the warps' sums, in order
#pragma unroll
  for (int j = 0; j < kTiles; ++j) {
    red[warp][j * 8 + 2 * t][g] = acc[j][0];
    red[warp][j * 8 + 2 * t + 1][g] = acc[j][1];
    red[warp][j * 8 + 2 * t][g + 8] = acc[j][2];
    red[warp][j * 8 + 2 * t + 1][g + 8] = acc[j][3];
  }
  __syncthreads();
  auto cta_sum = [&](int m, int r) {
    float v = 0.0f;
    for (int w = 0; w < warps; ++w) v = __fadd_rn(v, red[w][m][r]);
    return v;
  };
  if (p.split > 1) {
    for (int i = threadIdx.x; i < kTiles * 8 * kRows; i += blockDim.x)
      part[i / kRows][i % kRows] = cta_sum(i / kRows, i % kRows);
    cluster_sync();
  }
  // sixteen neighbouring threads finish a token's sixteen outputs; of a cluster's CTAs
  // each takes every split-th token
  constexpr bool kF16 = kKind == Kind::kFp16;
  const bool requant = p.next_scale != nullptr;
  const float s_next = requant ? *p.next_scale : 1.0f;
  const float s_enc = encode_scale(s_next);
  if (requant && blockIdx.x == 0 && threadIdx.x == 0 && p.rq_tensor_scale != p.next_scale)
    *p.rq_tensor_scale = s_next;
  for (int i = threadIdx.x; i < kTiles * 8 * kRows; i += blockDim.x) {
    const int m = i / kRows, r = i % kRows;
    const bool own = m < p.M && (p.split == 1 || m % p.split == rank);   // for all sixteen
    const int64_t n = n0 + r;
    float v = 0.0f;
    if (own) {
      if (p.split == 1) {
        v = cta_sum(m, r);
      } else {
        for (int q = 0; q < p.split; ++q) v = __fadd_rn(v, ld_cluster(mapa_shared(&part[m][r], q)));
      }
      if constexpr (kFp4)
        v = __fmul_rn(v, __fmul_rn(*p.sdec_a, *p.sdec_w));
      else if constexpr (kKind == Kind::kFp8)
        v = __fmul_rn(v, __fmul_rn(p.sdec_a[p.a_per_row ? m : 0], p.sdec_w[p.w_per_channel ? n : 0]));
      if (p.bias != nullptr) v = __fadd_rn(v, load16f(p.bias + n, kF16));
      float2 one[1] = {make_float2(v, v)};
      activate(one, p.act);
      v = one[0].x;
      if (p.residual != nullptr) v = __fadd_rn(v, load16f(p.residual + m * p.residual_stride + n, kF16));
    }
    const uint32_t bits = (kF16 ? pack_f16x2(v, 0.0f) : pack_bf16x2(v, 0.0f)) & 0xFFFFu;
    if (own && p.y != nullptr) p.y[m * p.N + n] = (uint16_t)bits;
    if (kF16 || kKind == Kind::kBf16 || !requant) continue;
    const int64_t col = n - p.rq_col0;
    const bool inside = own && n0 >= p.rq_col0 && n0 + kRows <= p.rq_col0 + p.rq_cols;
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
      if (inside && r == 0) p.rq_scales[scale_offset(m, col / 16, p.rq_cols)] = (uint8_t)code;
    }
  }
  if (p.split > 1) cluster_sync();   // no CTA leaves while another reads its sums
}

template <Kind kKind>
cudaError_t launch_kind(FewParams p, cudaStream_t s, int num_sms) {
  // Warps that share 16 rows of W: as many as fill the machine once (32 per SM), at most
  // one per two chunks of K; beyond a CTA's eight they spread over a cluster.
  const int64_t groups = p.N / kRows;
  const int64_t chunks = ((kKind == Kind::kNvfp4 ? p.K / 2 : kKind == Kind::kFp8 ? p.K : p.K * 2) + kChunk - 1) / kChunk;
  const int64_t want = std::max<int64_t>(1, std::min<int64_t>({(int64_t)num_sms * FW / groups, (chunks + 1) / 2,
                                                              (int64_t)kMaxWarps * kMaxSplit}));
  p.split = (int)((want + kMaxWarps - 1) / kMaxWarps);
  const int warps = (int)std::max<int64_t>(2, want / p.split);
  auto kern = p.M <= 8 ? few_kernel<kKind, 1> : few_kernel<kKind, 2>;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)p.split;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(groups * p.split), 1, 1);
  cfg.blockDim = dim3((unsigned)warps * 32, 1, 1);
  cfg.stream = s;
  cfg.attrs = at;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

}  // namespace

cudaError_t launch_few(const GemmArgs& a, cudaStream_t s, int num_sms) {
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
  return a.bf16 ? (a.fp16 ? launch_kind<Kind::kFp16>(p, s, num_sms) : launch_kind<Kind::kBf16>(p, s, num_sms))
         : a.fp4 ? launch_kind<Kind::kNvfp4>(p, s, num_sms)
                 : launch_kind<Kind::kFp8>(p, s, num_sms);
}

}  // namespace qlin
