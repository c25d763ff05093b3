// The FP8 linear with a scale for each 128 elements of K: A's per row, W's per 128 rows.
//   y = act( sum_b (S_A[m, b] S_W[n / 128, b]) sum_{k in b} a w + bias ) + residual
// The scales are any fp32 values, so the tensor cores' own block scales (powers of two) do
// not serve: a block's products leave tensor memory before the next one's are added, scaled
// on the way into fp32 registers.  A block is a pipeline stage (128 bytes of K): the MMA
// issuer writes its four products' sum into one of the tensor-memory buffers in turn, and
// the epilogue's two warpgroups, which hold the tile's accumulators, take it from there.
//   pair   256 x 256 tiles on a CTA pair (cta_group::2): a block is 512 cycles of MMAs, in
//          which a CTA's 128 x 256 sums leave tensor memory (256 cycles of its bandwidth)
//          and pass 32768 FMAs (256 cycles, two per instruction); 128 accumulators a thread.
//   single 128 x 128 tiles on one CTA, for fewer rows.
// Roles: warp 0 loads (TMA), warp 1 issues the MMAs, warps 4-11 hold the accumulators.
#include "qlin_internal.h"
#include "qlin_tiles.h"

namespace qlin {

namespace {

constexpr int kBM = kTileM;
constexpr int kRowBytes = kStageRowBytes;   // a block of K
constexpr int kSteps = 4;                   // MMAs of 32 elements of a block
constexpr int kRoleWarps = 4, kEpiWarps = 8;
constexpr int kThreads = (kRoleWarps + kEpiWarps) * 32;
constexpr int kRoleRegs = 56, kHoldRegs = 224, kLaunchRegs = 168;
static_assert(kRoleWarps * 32 * kRoleRegs + kEpiWarps * 32 * kHoldRegs <= kThreads * kLaunchRegs, "registers");

template <int kBN, bool kPair>
struct BlockCfg {
  static constexpr int kCM = kPair ? 2 : 1;
  static constexpr int kSplit = kPair ? 4 : 2;   // row boxes per operand tile, whose copies overlap
  static constexpr int kABytes = kBM * kRowBytes;
  static constexpr int kBBytes = kBN / kCM * kRowBytes;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kCols = kBN / 2;          // of an epilogue thread: one 128-row block of W at most
  static constexpr int kBiasBytes = kEpiWarps * kCols * 4;
  static constexpr int kStagesRaw = (232448 - 1024 - 512 - kBiasBytes) / kStageBytes;
  static constexpr int kStages = kStagesRaw > 8 ? 8 : kStagesRaw;
  static constexpr int kBuffers = 512 / kBN;     // of block sums in tensor memory
  static constexpr int kSmem = 1024 + kStages * kStageBytes + kBiasBytes + 512;
  static_assert(kStages >= 3 && kSmem <= 232448, "shared memory");
};

struct BlockParams {
  const float* sa;    // [K blocks, M]
  const float* sw;    // [K blocks, N blocks]
  uint16_t* y;
  int64_t M, N, K;
  const uint16_t* bias;
  const uint16_t* residual;
  int64_t residual_stride;
  int act;
  int y_v8, r_v8;     // rows start on 32-byte boundaries
  unsigned* err;
  uint64_t timeout_ns;
};

// Bounded wait that ignores the abort flag: for copies and MMAs in flight at the end.
__device__ __forceinline__ void drain(uint64_t* bar, uint32_t parity, const BlockParams& p) {
  const uint32_t a = smem_u32(bar);
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(a, parity)) {
    if (global_timer_ns() - t0 > p.timeout_ns) {
      atomicExch(p.err, kErrTimeout);
      return;
    }
  }
}

template <bool kWide>
__device__ __forceinline__ void load32(const uint16_t* p, uint32_t (&r)[8]) {
  if (kWide) {
    asm volatile("ld.global.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p));
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(r[4 * k]), "=r"(r[4 * k + 1]), "=r"(r[4 * k + 2]), "=r"(r[4 * k + 3])
                   : "l"(p + 8 * k));
  }
}

__device__ __forceinline__ void store32(uint16_t* p, const uint32_t* v, bool wide) {
  if (wide) {
    asm volatile("st.global.L1::no_allocate.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]),
                 "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(p + 8 * k), "r"(v[4 * k]), "r"(v[4 * k + 1]),
                   "r"(v[4 * k + 2]), "r"(v[4 * k + 3])
                   : "memory");
  }
}

template <int kBN, bool kPair>
__global__ void __launch_bounds__(kThreads, 1)
    gemm_block_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                      const BlockParams p) {
  using C = BlockCfg<kBN, kPair>;
  constexpr int kCM = C::kCM;
  constexpr uint16_t kMask = (uint16_t)((1u << kCM) - 1u);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* const bias_copies = reinterpret_cast<float*>(smem + C::kStages * C::kStageBytes);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kStages * C::kStageBytes + C::kBiasBytes);
  uint64_t* empty = full + C::kStages;
  uint64_t* tmem_full = empty + C::kStages;
  uint64_t* tmem_empty = tmem_full + C::kBuffers;
  uint64_t* mma_done = tmem_empty + C::kBuffers;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;
  const int rank = kPair ? __shfl_sync(0xFFFFFFFFu, (int)cluster_ctarank(), 0) : 0;
  const bool leader = rank == 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < C::kBuffers; ++a) {
      mbar_init(&tmem_full[a], 1);
      mbar_init(&tmem_empty[a], kCM * kEpiWarps);
    }
    mbar_init(mma_done, 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane < 2) prefetch_tmap(lane == 0 ? &tmap_a : &tmap_b);
  if (warp == 1) {
    if (kPair)
      tmem_alloc_pair(tmem_slot, 512);
    else
      tmem_alloc(tmem_slot, 512);
  }
  tc_fence_before();
  if (kPair)
    cluster_sync();
  else
    __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
  const WaitCtl ctl{abort_flag, p.err, p.timeout_ns};
  const int tiles_m = (int)((p.M + kBM - 1) / kBM), tiles_n = (int)((p.N + kBN - 1) / kBN);
  const int groups_m = (tiles_m + kCM - 1) / kCM;
  const int num_ctiles = groups_m * tiles_n;
  const int cid = (int)blockIdx.x / kCM, ncl = (int)gridDim.x / kCM;
  const int num_kb = (int)((p.K + kRowBytes - 1) / kRowBytes);
  grid_dep_wait();

  if (warp < kRoleWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRoleRegs));
    if (warp == 0) {
      // ---- TMA producer ----
      constexpr int kSplit = C::kSplit, kARows = kBM / kSplit, kWRows = kBN / kCM / kSplit;
      const uint32_t bar0 = kPair ? __shfl_sync(0xFFFFFFFFu, mapa_shared(full, 0), 0) : smem_u32(full);
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int ct = cid; ct < num_ctiles && ok; ct += ncl) {
        const int a_row = (ct % groups_m * kCM + rank) * kBM;
        const int w_row = ct / groups_m * kBN + rank * (kBN / kCM);
        if (ct + ncl >= num_ctiles) grid_dep_launch();
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait_warp(&empty[stage], phase ^ 1u, ctl)) {
            ok = false;
            break;
          }
          uint8_t* const sA = smem + stage * C::kStageBytes;
          const uint32_t bar = bar0 + (uint32_t)(stage * 8);
          if (elect_one()) {
            if (leader) mbar_arrive_expect_tx(&full[stage], kCM * C::kStageBytes);
#pragma unroll
            for (int b = 0; b < kSplit; ++b) {
              if (kPair) {
                tma_load_4d_pair(sA + b * kARows * kRowBytes, &tmap_a, bar, kb * kRowBytes, a_row + b * kARows, 0, 0);
                tma_load_4d_pair(sA + C::kABytes + b * kWRows * kRowBytes, &tmap_b, bar, kb * kRowBytes,
                                 w_row + b * kWRows, 0, 0);
              } else {
                tma_load_4d(sA + b * kARows * kRowBytes, &tmap_a, bar, kb * kRowBytes, a_row + b * kARows, 0, 0);
                tma_load_4d(sA + C::kABytes + b * kWRows * kRowBytes, &tmap_b, bar, kb * kRowBytes,
                            w_row + b * kWRows, 0, 0);
              }
            }
          }
          ++issued;
          if (++stage == C::kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (leader && lane == 0) {   // the last copies land before the CTA exits
        const int n_drain = min(issued, C::kStages);
        for (int i = 0; i < n_drain; ++i) {
          if (--stage < 0) {
            stage = C::kStages - 1;
            phase ^= 1u;
          }
          drain(&full[stage], phase, p);
        }
      }
    } else if (warp == 1 && leader) {
      // ---- MMA issuer: a block of K into each tensor-memory buffer in turn ----
      constexpr uint32_t idesc = idesc_fp8(kBN, kPair ? 256 : 128);
      const int k_steps = (int)(p.K / 32);
      int stage = 0, buf = 0;
      uint32_t phase = 0, buf_phase = 0;
      bool ok = true;
      for (int ct = cid; ct < num_ctiles && ok; ct += ncl) {
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait_warp(&tmem_empty[buf], buf_phase ^ 1u, ctl) || !mbar_wait_warp(&full[stage], phase, ctl)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sA = smem_u32(smem + stage * C::kStageBytes);
          const uint64_t adesc = sdesc_k128(sA), bdesc = sdesc_k128(sA + C::kABytes);
          const uint32_t d = tmem_base + (uint32_t)(buf * kBN);
          const int steps = min(kSteps, k_steps - kb * kSteps);
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
              if (j < steps) {   // (32 bytes further per step)
                if (kPair)
                  mma_fp8_pair(d, adesc + 2 * j, bdesc + 2 * j, idesc, j > 0 ? 1u : 0u);
                else
                  mma_fp8(d, adesc + 2 * j, bdesc + 2 * j, idesc, j > 0 ? 1u : 0u);
              }
            }
            if (kPair) {
              tc_commit_pair_mc(&empty[stage], kMask);
              tc_commit_pair_mc(&tmem_full[buf], kMask);
            } else {
              tc_commit(&empty[stage]);
              tc_commit(&tmem_full[buf]);
            }
          }
          if (++stage == C::kStages) {
            stage = 0;
            phase ^= 1u;
          }
          if (++buf == C::kBuffers) {
            buf = 0;
            buf_phase ^= 1u;
          }
        }
      }
      // The epilogues' last arrivals have landed here (the barrier at the end orders nothing).
      if (ok) {
        for (int i = 0; i < C::kBuffers; ++i) {
          (void)mbar_wait_warp(&tmem_empty[buf], buf_phase ^ 1u, ctl);
          if (++buf == C::kBuffers) {
            buf = 0;
            buf_phase ^= 1u;
          }
        }
      }
      // Every MMA issued must finish before the tensor memory is released.
      if (elect_one()) {
        if (kPair)
          tc_commit_pair_mc(mma_done, 1);
        else
          tc_commit(mma_done);
        drain(mma_done, 0, p);
      }
    }
  } else {
    // ---- accumulators ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kHoldRegs));
    constexpr int kCols = C::kCols, kChunks = kCols / 32;
    const int e = warp - kRoleWarps, quarter = warp & 3, half = e >> 2;
    float* const bias_s = bias_copies + e * kCols;
    const int64_t w_blocks = (p.N + 127) / 128;
    int buf = 0;
    uint32_t buf_phase = 0;
    bool ok = true;
    for (int ct = cid; ct < num_ctiles && ok; ct += ncl) {
      const int64_t row = (int64_t)(ct % groups_m * kCM + rank) * kBM + quarter * 32 + lane;
      const int64_t col0 = (int64_t)(ct / groups_m) * kBN + half * kCols;
      const bool row_in = row < p.M;
      __syncwarp();   // the tile before has read its biases
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int64_t n = col0 + c * 32 + lane;
        bias_s[c * 32 + lane] = p.bias != nullptr && n < p.N ? bf16_lo(__ldg(p.bias + n)) : 0.0f;
      }
      __syncwarp();
      const float* const sa = p.sa + (row_in ? row : 0);
      const float* const sw = p.sw + min(col0 >> 7, w_blocks - 1);
      float2 acc[kChunks][16];
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] = make_float2(0.0f, 0.0f);
      // scales three blocks ahead of their use
      constexpr int kAhead = 4;
      float ra[kAhead], rw[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead - 1; ++i) {
        const int kb = min(i, num_kb - 1);
        ra[i] = __ldg(sa + kb * p.M);
        rw[i] = __ldg(sw + kb * w_blocks);
      }
      for (int kb0 = 0; kb0 < num_kb && ok; kb0 += kAhead) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
          if (kb0 + u < num_kb && ok) {
            const int next = min(kb0 + u + kAhead - 1, num_kb - 1);
            ra[(u + kAhead - 1) % kAhead] = __ldg(sa + next * p.M);
            rw[(u + kAhead - 1) % kAhead] = __ldg(sw + next * w_blocks);
            if (!mbar_wait_warp(&tmem_full[buf], buf_phase, ctl)) {
              ok = false;
            } else {
              tc_fence_after();
              const float2 s = splat(__fmul_rn(ra[u], rw[u]));
              const uint32_t t = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kBN + half * kCols);
              uint32_t v[2][32];
              tmem_ld32(t, v[0]);
              tmem_ld_wait();
#pragma unroll
              for (int c = 0; c < kChunks; ++c) {
                if (c + 1 < kChunks) tmem_ld32(t + 32 * (c + 1), v[(c + 1) & 1]);
                if (c + 1 == kChunks) {   // the buffer goes back to the MMAs
                  tc_fence_before();
                  __syncwarp();
                  if (lane == 0) {
                    if (kPair && rank == 1)
                      mbar_arrive_cluster(mapa_shared(&tmem_empty[buf], 0));
                    else
                      mbar_arrive(&tmem_empty[buf]);
                  }
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                  acc[c][i] = fma2(make_float2(__uint_as_float(v[c & 1][2 * i]), __uint_as_float(v[c & 1][2 * i + 1])), s,
                                   acc[c][i]);
                if (c + 1 < kChunks) tmem_ld_wait();
              }
              if (++buf == C::kBuffers) {
                buf = 0;
                buf_phase ^= 1u;
              }
            }
          }
        }
      }
      if (!ok) break;
      // ---- the tile's end: N % 64 == 0, so 32 columns are wholly inside or outside ----
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int64_t n = col0 + c * 32;
        if (n >= p.N) break;
        uint32_t res[2][8];
        if (p.residual != nullptr && row_in) {
          const uint16_t* const r = p.residual + row * p.residual_stride + n;
          if (p.r_v8) {
            load32<true>(r, res[0]);
            load32<true>(r + 16, res[1]);
          } else {
            load32<false>(r, res[0]);
            load32<false>(r + 16, res[1]);
          }
        }
        if (p.bias != nullptr) {
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            const float4 b = *reinterpret_cast<const float4*>(bias_s + c * 32 + 2 * i);
            acc[c][i] = add2(acc[c][i], make_float2(b.x, b.y));
            acc[c][i + 1] = add2(acc[c][i + 1], make_float2(b.z, b.w));
          }
        }
        activate(acc[c], p.act);
        if (!row_in) continue;
        if (p.residual != nullptr) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t w = res[i / 8][i % 8];
            acc[c][i] = add2(acc[c][i], make_float2(bf16_lo(w), bf16_hi(w)));
          }
        }
        uint32_t out[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) out[i] = pack_bf16x2(acc[c][i].x, acc[c][i].y);
        uint16_t* const y = p.y + row * p.N + n;
        store32(y, out, p.y_v8 != 0);
        store32(y + 16, out + 8, p.y_v8 != 0);
      }
    }
  }

  // No CTA of a pair may exit while the peer can still arrive on its barriers.
  __syncwarp();
  tc_fence_before();
  if (kPair)
    cluster_sync_relaxed();
  else
    __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if (kPair)
      tmem_dealloc_pair(tmem_base, 512);
    else
      tmem_dealloc(tmem_base, 512);
  }
}

template <int kBN, bool kPair>
cudaError_t launch_cfg(const GemmArgs& a, cudaStream_t s, Device dev, unsigned* err, uint64_t timeout_ns) {
  using C = BlockCfg<kBN, kPair>;
  constexpr int kCM = C::kCM;
  CUtensorMap ta, tb;
  if (encode_tensor_map_codes(&ta, a.a_codes, (uint64_t)a.K, (uint64_t)a.M, kBM / C::kSplit) != CUDA_SUCCESS ||
      encode_tensor_map_codes(&tb, a.w_codes, (uint64_t)a.K, (uint64_t)a.N, kBN / kCM / C::kSplit) != CUDA_SUCCESS)
    return cudaErrorInvalidValue;
  BlockParams p{};
  p.sa = a.sdec_a;
  p.sw = a.sdec_w;
  p.y = static_cast<uint16_t*>(a.y);
  p.M = a.M;
  p.N = a.N;
  p.K = a.K;
  p.bias = static_cast<const uint16_t*>(a.bias);
  p.residual = static_cast<const uint16_t*>(a.residual);
  p.residual_stride = a.residual_stride;
  p.act = a.act;
  p.y_v8 = (reinterpret_cast<uintptr_t>(a.y) & 31u) == 0 ? 1 : 0;
  p.r_v8 = ((reinterpret_cast<uintptr_t>(a.residual) | (uintptr_t)(a.residual_stride * 2)) & 31u) == 0 ? 1 : 0;
  p.err = err;
  p.timeout_ns = timeout_ns;
  auto kern = gemm_block_kernel<kBN, kPair>;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCM;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  struct Setup {
    cudaError_t err;
    int max_clusters;
  };
  static PerDevice<Setup> per_device;
  const Setup& setup = per_device.get(dev.index, [&] {
    Setup t{cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem), 0};
    if (t.err != cudaSuccess) return t;
    cfg.gridDim = dim3((unsigned)(dev.num_sms / kCM * kCM), 1, 1);
    t.err = cudaOccupancyMaxActiveClusters(&t.max_clusters, kern, &cfg);
    if (t.err == cudaSuccess && t.max_clusters < 1) t.err = cudaErrorInvalidConfiguration;
    return t;
  });
  if (setup.err != cudaSuccess) return setup.err;
  const int64_t tiles_m = (a.M + kBM - 1) / kBM;
  const int64_t ctiles = ((tiles_m + kCM - 1) / kCM) * ((a.N + kBN - 1) / kBN);
  if (ctiles > INT32_MAX / 2) return cudaErrorInvalidValue;
  const int clusters = (int)std::min<int64_t>(ctiles, std::min(setup.max_clusters, dev.num_sms / kCM));
  cfg.gridDim = dim3((unsigned)(clusters * kCM), 1, 1);
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, ta, tb, p);
}

}  // namespace

cudaError_t launch_gemm_block(const GemmArgs& a, cudaStream_t s, Device dev, unsigned* err, uint64_t timeout_ns) {
  const int64_t tiles_m = (a.M + kBM - 1) / kBM;
  if (tiles_m * ((a.N + 255) / 256) >= dev.num_sms) return launch_cfg<256, true>(a, s, dev, err, timeout_ns);
  return launch_cfg<128, false>(a, s, dev, err, timeout_ns);
}

}  // namespace qlin
