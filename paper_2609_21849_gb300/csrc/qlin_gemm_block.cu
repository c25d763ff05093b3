// The FP8 linear with a scale for each 128 elements of K: A's per row, W's per 128 rows.
//   y = act( sum_b (S_A[m, b] S_W[n / 128, b]) sum_{k in b} a w + bias ) + residual
// The scales are any fp32 values, so the tensor cores' own block scales (powers of two) do
// not serve: a block's products leave tensor memory before the next one's are added, scaled
// on the way into fp32 registers.  A block is a pipeline stage (128 bytes of K): the MMA
// issuer writes its four products' sum into one of the tensor-memory buffers in turn, and the
// epilogue's warpgroups (one per 64 columns), which hold the tile's accumulators, take it from there.
//   wide   128 x 256 tiles.  A block is 512 cycles of MMAs, in which 128 x 256 sums leave tensor memory
//          and pass 32768 FMAs (256 cycles, two per instruction); 48 KB reach the SM for it, 750 cycles
//          at 64 bytes each.  It takes 0.43-0.45 us, about 830, a tile's begin and end 6 us: 4608 x 12288
//          x 3072 160 us.  (With W's half sent by each CTA of two to both it took 160.4: what a copy sent
//          to two CTAs saves is reads of L2, not what comes into an SM.  As a CTA pair with cta_group::2,
//          every buffer's way to the epilogue and back crossed the pair: 950 cycles a block.)
//   single 128 x 128 tiles, for fewer rows, also with K shared by a cluster.
// Roles: warp 0 loads (TMA), warp 1 issues the MMAs, warp 2 multiplies the scales of a block's rows
// and columns into shared memory (loads of them by the epilogue's own warps cost 20 to 40 of 180
// us), the warps from 4 on hold the accumulators, 64 columns of a row each.
#include "qlin_internal.h"
#include "qlin_tiles.h"

namespace qlin {

namespace {

constexpr int kBM = kTileM;
constexpr int kRowBytes = kStageRowBytes;   // a block of K
constexpr int kSteps = 4;                   // MMAs of 32 elements of a block
constexpr int kRawSlots = 8;   // blocks whose scales are loaded ahead
constexpr int kRoleWarps = 4, kCols = 64;   // columns of an epilogue thread: inside one 128-row block of W

template <int kBN>
struct BlockCfg {
  static constexpr int kEpiWarps = kBN / kCols * 4;
  static constexpr int kThreads = (kRoleWarps + kEpiWarps) * 32;
  static constexpr int kSplit = 2;               // row boxes per load of 128 rows, whose copies overlap
  static constexpr int kABytes = kBM * kRowBytes;
  static constexpr int kBBytes = kBN * kRowBytes;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kBiasBytes = kEpiWarps * kCols * 2;    // 16-bit, a copy per warp
  static constexpr int kBuffers = 512 / kBN;     // of block sums in tensor memory
  static constexpr int kWBlocks = kBN / 128;
  // scales: of each buffer's block, [W's block][row]; on their way, S_A of the rows and S_W
  static constexpr int kScaleBytes = kBuffers * kWBlocks * kBM * 4, kRawSlot = kBM + 4;
  static constexpr int kRawBytes = kRawSlots * kRawSlot * 4;
  static constexpr int kStagesRaw = (232448 - 1024 - 512 - kBiasBytes - kScaleBytes - kRawBytes) / kStageBytes;
  static constexpr int kStages = kStagesRaw > 8 ? 8 : kStagesRaw;
  static constexpr int kSmem = 1024 + kStages * kStageBytes + kBiasBytes + kScaleBytes + kRawBytes + 512;
  // registers: the roles' warpgroup and those with accumulators
  static constexpr int kRoleRegs = kThreads == 640 ? 64 : 80, kHoldRegs = kThreads == 640 ? 104 : 128;
  static constexpr int kLaunchRegs = kThreads == 640 ? 96 : 112;
  static_assert(kRoleWarps * 32 * kRoleRegs + kEpiWarps * 32 * kHoldRegs <= kThreads * kLaunchRegs, "registers");
  static_assert(kThreads == 640 || kThreads == 384, "whole warpgroups");
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
  int split;          // kSplitK: CTAs of a cluster (2, 4 or 8)
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

__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
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

template <int kBN, bool kSplitK>
__global__ void __launch_bounds__(BlockCfg<kBN>::kThreads, 1)
    gemm_block_kernel(const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_b,
                      const BlockParams p) {
  using C = BlockCfg<kBN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* const bias_copies = smem + C::kStages * C::kStageBytes;
  float* const scales = reinterpret_cast<float*>(bias_copies + C::kBiasBytes);
  uint64_t* full = reinterpret_cast<uint64_t*>(bias_copies + C::kBiasBytes + C::kScaleBytes + C::kRawBytes);
  uint64_t* empty = full + C::kStages;
  uint64_t* tmem_full = empty + C::kStages;
  uint64_t* tmem_empty = tmem_full + C::kBuffers;
  uint64_t* mma_done = tmem_empty + C::kBuffers;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(mma_done + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = __shfl_sync(0xFFFFFFFFu, (int)(threadIdx.x >> 5), 0);
  const int lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < C::kBuffers; ++a) {
      mbar_init(&tmem_full[a], 2);   // the block's products, and its scales
      mbar_init(&tmem_empty[a], C::kEpiWarps);
    }
    mbar_init(mma_done, 1);
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 0 && lane < 2) prefetch_tmap(lane == 0 ? &tmap_a : &tmap_b);
  if (warp == 1) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  if (kSplitK)
    cluster_sync();
  else
    __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xFFFFFFFFu, *tmem_slot, 0);
  const WaitCtl ctl{abort_flag, p.err, p.timeout_ns};
  const int tiles_m = (int)((p.M + kBM - 1) / kBM), tiles_n = (int)((p.N + kBN - 1) / kBN);
  const int num_tiles = tiles_m * tiles_n;
  // kSplitK: the CTAs of a cluster take a tile's blocks of K in equal runs (split <= blocks)
  const int splits = kSplitK ? p.split : 1;
  const int krank = kSplitK ? __shfl_sync(0xFFFFFFFFu, (int)cluster_ctarank(), 0) : 0;
  const int cid = (int)blockIdx.x / splits, ncl = (int)gridDim.x / splits;
  const int all_kb = (int)((p.K + kRowBytes - 1) / kRowBytes);
  const int kb0 = krank * all_kb / splits, num_kb = (krank + 1) * all_kb / splits - kb0;
  grid_dep_wait();

  if (warp < kRoleWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRoleRegs));
    if (warp == 0) {
      // ---- TMA producer ----
      constexpr int kARows = kBM / C::kSplit, kWRows = kBN / C::kSplit;
      int stage = 0, issued = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int ct = cid; ct < num_tiles && ok; ct += ncl) {
        const int a_row = ct % tiles_m * kBM, w_row = ct / tiles_m * kBN;
        if (ct + ncl >= num_tiles) grid_dep_launch();
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait_warp(&empty[stage], phase ^ 1u, ctl)) {
            ok = false;
            break;
          }
          uint8_t* const sA = smem + stage * C::kStageBytes;
          uint8_t* const sW = sA + C::kABytes;
          const uint32_t bar = smem_u32(&full[stage]);
          if (elect_one()) {
            mbar_arrive_expect_tx(&full[stage], C::kStageBytes);
#pragma unroll
            for (int b = 0; b < C::kSplit; ++b) {
              tma_load_4d(sA + b * kARows * kRowBytes, &tmap_a, bar, (kb0 + kb) * kRowBytes, a_row + b * kARows, 0, 0);
              tma_load_4d(sW + b * kWRows * kRowBytes, &tmap_b, bar, (kb0 + kb) * kRowBytes, w_row + b * kWRows, 0, 0);
            }
          }
          ++issued;
          if (++stage == C::kStages) {
            stage = 0;
            phase ^= 1u;
          }
        }
      }
      if (lane == 0) {   // the last copies land before the CTA exits
        const int n_drain = min(issued, C::kStages);
        for (int i = 0; i < n_drain; ++i) {
          if (--stage < 0) {
            stage = C::kStages - 1;
            phase ^= 1u;
          }
          drain(&full[stage], phase, p);
        }
      }
    } else if (warp == 1) {
      // ---- MMA issuer: a block of K into each tensor-memory buffer in turn ----
      constexpr uint32_t idesc = idesc_fp8(kBN, 128);
      const int k_steps = (int)(p.K / 32);
      int stage = 0, buf = 0;
      uint32_t phase = 0, buf_phase = 0;
      bool ok = true;
      for (int ct = cid; ct < num_tiles && ok; ct += ncl) {
        for (int kb = 0; kb < num_kb; ++kb) {
          if (!mbar_wait_warp(&tmem_empty[buf], buf_phase ^ 1u, ctl) || !mbar_wait_warp(&full[stage], phase, ctl)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sA = smem_u32(smem + stage * C::kStageBytes);
          const uint64_t adesc = sdesc_k128(sA), bdesc = sdesc_k128(sA + C::kABytes);
          const uint32_t d = tmem_base + (uint32_t)(buf * kBN);
          const int steps = min(kSteps, k_steps - (kb0 + kb) * kSteps);
          if (elect_one()) {
#pragma unroll
            for (int j = 0; j < kSteps; ++j) {
              // (32 bytes further per step)
              if (j < steps) mma_fp8(d, adesc + 2 * j, bdesc + 2 * j, idesc, j > 0 ? 1u : 0u);
            }
            tc_commit(&empty[stage]);
            tc_commit(&tmem_full[buf]);
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
        tc_commit(mma_done);
        drain(mma_done, 0, p);
      }
    } else if (warp == 2) {
      // ---- scales: S_A S_W of a block for the tile's rows ----
      // Loaded by cp.async seven blocks ahead, across the tiles.  (Into registers, the loop waited for
      // the loads it had just issued: 740 cycles a block, and the MMAs with it.)
      const int64_t w_blocks = (p.N + 127) / 128;
      const uint32_t raw = smem_u32(scales) + (uint32_t)(C::kScaleBytes + lane * 4);
      int next_ct = cid, next_kb = 0, next_slot = 0;
      const float *next_a[4], *next_w = nullptr;
      auto fetch = [&] {
        if (next_ct < num_tiles) {
          if (next_kb == 0) {
            const int64_t row0 = (int64_t)(next_ct % tiles_m) * kBM + lane;
#pragma unroll
            for (int i = 0; i < 4; ++i) next_a[i] = p.sa + kb0 * p.M + min(row0 + 32 * i, p.M - 1);
            next_w = p.sw + kb0 * w_blocks + min((int64_t)(next_ct / tiles_m) * C::kWBlocks + min(lane, C::kWBlocks - 1), w_blocks - 1);
          }
          const uint32_t dst = raw + (uint32_t)(next_slot * C::kRawSlot * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            cp_async4(dst + 128 * i, next_a[i]);
            next_a[i] += p.M;
          }
          if (lane < C::kWBlocks) cp_async4(dst + 4 * kBM, next_w);
          next_w += w_blocks;
          if (++next_kb == num_kb) {
            next_kb = 0;
            next_ct += ncl;
          }
          if (++next_slot == kRawSlots) next_slot = 0;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      };
      for (int i = 0; i < kRawSlots - 1; ++i) fetch();
      int buf = 0, slot = 0;
      uint32_t buf_phase = 0;
      bool ok = true;
      for (int ct = cid; ct < num_tiles && ok; ct += ncl) {
        for (int kb = 0; kb < num_kb; ++kb) {
          asm volatile("cp.async.wait_group %0;" ::"n"(kRawSlots - 2) : "memory");
          __syncwarp();   // (the others' loads too; and all are done with the slot that the next fills)
          const float* const from = scales + C::kScaleBytes / 4 + slot * C::kRawSlot;
          float a[4], w[C::kWBlocks];
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = from[lane + 32 * i];
#pragma unroll
          for (int i = 0; i < C::kWBlocks; ++i) w[i] = from[kBM + i];
          if (++slot == kRawSlots) slot = 0;
          if (!mbar_wait_warp(&tmem_empty[buf], buf_phase ^ 1u, ctl)) {
            ok = false;
            break;
          }
          float* const to = scales + buf * C::kWBlocks * kBM + lane;
#pragma unroll
          for (int k = 0; k < C::kWBlocks; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) to[k * kBM + 32 * i] = __fmul_rn(a[i], w[k]);
          __syncwarp();
          if (lane == 0) mbar_arrive(&tmem_full[buf]);
          fetch();
          if (++buf == C::kBuffers) {
            buf = 0;
            buf_phase ^= 1u;
          }
        }
      }
      asm volatile("cp.async.wait_group 0;" ::: "memory");
    }
  } else {
    // ---- accumulators ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kHoldRegs));
    constexpr int kChunks = kCols / 32;
    const int e = warp - kRoleWarps, quarter = warp & 3, part = e >> 2;   // lanes, columns
    const uint32_t bias_s = smem_u32(bias_copies) + (uint32_t)(e * kCols * 2);
    // kSplitK: every CTA sends its sums of a column to the CTA that finishes that column, through
    // shared memory that the stages have left; they are added in the order of K.
    auto split_end = [&](float2 (&acc)[kChunks][16], int ct) {
      cluster_sync();   // no MMA reads a stage of any of the CTAs, no copy is on its way
      const int width = kBN / splits, pitch = (width + 4) * 4;   // columns of a CTA; bytes of a row of them
      const int my_row = quarter * 32 + lane;
#pragma unroll
      for (int c = 0; c < 4; ++c) {   // 16 columns
        const int col = part * kCols + 16 * c, owner = col / width;
        const uint32_t to = mapa_shared(smem + (krank * kBM + my_row) * pitch + (col - owner * width) * 4, (uint32_t)owner);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = acc[c >> 1][8 * (c & 1) + 2 * i], b = acc[c >> 1][8 * (c & 1) + 2 * i + 1];
          asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + 16 * i), "f"(a.x), "f"(a.y),
                       "f"(b.x), "f"(b.y)
                       : "memory");
        }
      }
      cluster_sync();
      for (int i = threadIdx.x - kRoleWarps * 32; i < kBM * width / 16; i += C::kEpiWarps * 32) {
        const int r = i % kBM, group = i / kBM;
        const int64_t row = (int64_t)(ct % tiles_m) * kBM + r;
        const int64_t n = (int64_t)(ct / tiles_m) * kBN + krank * width + 16 * group;
        if (row >= p.M || n >= p.N) continue;
        float2 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = make_float2(0.0f, 0.0f);
        for (int q = 0; q < splits; ++q) {
          const float4* const from = reinterpret_cast<const float4*>(smem + (q * kBM + r) * pitch + 64 * group);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float4 x = from[k];
            v[2 * k] = add2(v[2 * k], make_float2(x.x, x.y));
            v[2 * k + 1] = add2(v[2 * k + 1], make_float2(x.z, x.w));
          }
        }
        uint32_t w[8];
        if (p.bias != nullptr) {
          load32<false>(p.bias + n, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = add2(v[k], make_float2(bf16_lo(w[k]), bf16_hi(w[k])));
        }
        activate(v, p.act);
        if (p.residual != nullptr) {
          load32<false>(p.residual + row * p.residual_stride + n, w);
#pragma unroll
          for (int k = 0; k < 8; ++k) v[k] = add2(v[k], make_float2(bf16_lo(w[k]), bf16_hi(w[k])));
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = pack_bf16x2(v[k].x, v[k].y);
        store32(p.y + row * p.N + n, w, p.y_v8 != 0);
      }
    };
    int buf = 0;
    uint32_t buf_phase = 0;
    bool ok = true;
    for (int ct = cid; ct < num_tiles && ok; ct += ncl) {
      const int64_t row = (int64_t)(ct % tiles_m) * kBM + quarter * 32 + lane;
      const int64_t col0 = (int64_t)(ct / tiles_m) * kBN + part * kCols;
      const bool row_in = row < p.M;
      if (p.bias != nullptr) {   // read at the tile's end
        __syncwarp();            // (the tile before has read its own)
        if (8 * lane < kCols && col0 + 8 * lane < p.N) cp_async16(bias_s + 16 * lane, p.bias + col0 + 8 * lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      float2 acc[kChunks][16];
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[c][i] = make_float2(0.0f, 0.0f);
      for (int kb = 0; kb < num_kb; ++kb) {
        if (!mbar_wait_warp(&tmem_full[buf], buf_phase, ctl)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const uint32_t t = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kBN + part * kCols);
        uint32_t v[32];
        tmem_ld32(t, v);
        float scale;
        asm volatile("ld.shared.f32 %0, [%1];"
                     : "=f"(scale)
                     : "r"(smem_u32(scales + (buf * C::kWBlocks + part * kCols / 128) * kBM + quarter * 32 + lane)));
        const float2 s = splat(scale);
        tmem_ld_wait();
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
#pragma unroll
          for (int i = 0; i < 16; ++i)
            acc[c][i] = fma2(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), s, acc[c][i]);
          if (c + 1 < kChunks) {
            tmem_ld32(t + 32 * (c + 1), v);
            tmem_ld_wait();
          }
          if (c + 2 == kChunks) {   // the buffer goes back to the MMAs
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&tmem_empty[buf]);
          }
        }
        if (++buf == C::kBuffers) {
          buf = 0;
          buf_phase ^= 1u;
        }
      }
      if constexpr (kSplitK) {   // (one tile)
        split_end(acc, ct);
        break;
      }
      if (!ok) break;
      // ---- the tile's end: N % 64 == 0, so 32 columns are wholly inside or outside ----
      if (p.bias != nullptr) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
      }
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
          for (int i = 0; i < 16; i += 4) {
            uint32_t w[4];
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                         : "r"(bias_s + c * 64 + 4 * i));
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[c][i + k] = add2(acc[c][i + k], make_float2(bf16_lo(w[k]), bf16_hi(w[k])));
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

  if constexpr (kSplitK) {
    if (warp < kRoleWarps) {   // the epilogue's two cluster barriers
      __syncwarp();
      cluster_sync();
      cluster_sync();
    }
  }
  __syncwarp();
  tc_fence_before();
  if (kSplitK)
    cluster_sync_relaxed();
  else
    __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

template <int kBN, bool kSplitK = false>
cudaError_t launch_cfg(const GemmArgs& a, cudaStream_t s, Device dev, unsigned* err, uint64_t timeout_ns) {
  using C = BlockCfg<kBN>;
  CUtensorMap ta, tb;
  if (encode_tensor_map_codes(&ta, a.a_codes, (uint64_t)a.K, (uint64_t)a.M, kBM / C::kSplit) != CUDA_SUCCESS ||
      encode_tensor_map_codes(&tb, a.w_codes, (uint64_t)a.K, (uint64_t)a.N, kBN / C::kSplit) != CUDA_SUCCESS)
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
  p.split = a.split;
  p.err = err;
  p.timeout_ns = timeout_ns;
  auto kern = gemm_block_kernel<kBN, kSplitK>;
  static PerDevice<cudaError_t> per_device;
  const cudaError_t e = per_device.get(
      dev.index, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem); });
  if (e != cudaSuccess) return e;
  const int64_t tiles = ((a.M + kBM - 1) / kBM) * ((a.N + kBN - 1) / kBN);
  if (tiles > INT32_MAX / 2) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;   // kSplitK: a cluster per tile
  attr[1].val.clusterDim.x = kSplitK ? (unsigned)a.split : 1u;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(kSplitK ? tiles * a.split : std::min<int64_t>(tiles, dev.num_sms)), 1, 1);
  cfg.blockDim = dim3(C::kThreads, 1, 1);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = kSplitK ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, ta, tb, p);
}

}  // namespace

cudaError_t launch_gemm_block(const GemmArgs& a, cudaStream_t s, Device dev, unsigned* err, uint64_t timeout_ns) {
  switch (choose_block_tile(a.M, a.N, a.K, dev.num_sms)) {
    case BlockTile::kWide:
      return launch_cfg<256>(a, s, dev, err, timeout_ns);
    case BlockTile::kSingle:
      return launch_cfg<128>(a, s, dev, err, timeout_ns);
    default: {
      GemmArgs b = a;
      b.split = choose_block_split(a.M, a.N, a.K, dev.num_sms);
      return launch_cfg<128, true>(b, s, dev, err, timeout_ns);
    }
  }
}

}  // namespace qlin
