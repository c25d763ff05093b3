// The GEMM's choice of a tile configuration: host code without CUDA, so that a
// CPU test can run it.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace qlin {

constexpr int kTileM = 128;         // rows of a CTA's tile (a pair tile: 256)
constexpr int kStageRowBytes = 128; // bytes of K per pipeline stage and row

// The staging box (of a warp's two) that its next TMA store of y takes.  The warp waits
// until at most one of its stores still reads shared memory, so a store may never take
// the box of the store before it: the boxes alternate over the stores that are issued,
// across tiles.  (Not over a tile's chunks of columns: with an odd number of them, or some
// past N, a tile began in the box that the last one had ended in.)
struct StagingBoxes {
  int next = 0;
#ifdef __CUDACC__
  __host__ __device__
#endif
  int take() {
    const int box = next;
    next ^= 1;
    return box;
  }
};

enum class Tile { kPair, kSingle, kNarrow, kWide };   // 256 x 256, 128 x 128, x 64, x 192
enum class GemmKind { kNvfp4, kFp8, k16 };     // k16: bf16 / fp16 operands

// What the epilogue does beside writing y (kLinear: bias, activation and residual).
enum class Epilogue { kPlain, kRequant, kAmax, kLinear, kLinearRequant };

inline int64_t k_row_bytes(GemmKind kind, int64_t K) {
  return kind == GemmKind::kNvfp4 ? K / 2 : kind == GemmKind::k16 ? K * 2 : K;
}

// Time of a launch in a tile configuration, in microseconds: a launch, then
// waves of tiles that each cost a start and end and their K stages.  Fitted
// to graph-replayed launches over M 16-4608, N 256-6144, K 256-3072 (operands
// in L2; rms error 5-9%).
struct TileCost {
  double launch, wave, stage;
  double us(int64_t tiles, int64_t slots, int64_t stages, double wave_extra,
            double wave_least = 0.0) const {
    return launch + (double)((tiles + slots - 1) / slots) *
                        std::max(wave + wave_extra + (double)stages * stage, wave_least);
  }
};

// Pair tiles when there are enough of them to fill the machine, else 128 x 128
// single-CTA tiles, or 128 x 64 when those would leave at least half the SMs
// idle -- unless the fitted times say that another configuration is at least 10%
// faster: mostly a last wave that is nearly empty (NVFP4 1000 x 3072 x 3072: 192
// single tiles on 152 SMs 10.4 us, 48 pair tiles 8.0) or a K too short for the
// pair tiles' start and end (NVFP4 4608 x 2560 x 256: pairs 7.8 us, single tiles
// 6.8).  The margin covers the fit's error.  Each configuration timed at 5934
// calls over M 16-18432, N 64-12288 and K 64-12288, far beyond the fit: the fit
// overrides the count in 795 of them, which take 0.81 of the time on average; ten
// are more than 5% slower for it, all with one or two waves or K = 64 (worst NVFP4
// 18432 x 1024 x 64: 10.4 -> 12.8 us).
inline Tile choose_tile(GemmKind kind, Epilogue epi, int64_t M, int64_t N, int64_t K,
                        int num_sms) {
  static const TileCost kCosts[3][3] = {
      {{2.5, 1.65, 0.24}, {2.7, 0.5, 0.29}, {2.7, 0.3, 0.26}},     // NVFP4
      {{3.3, 2.2, 0.265}, {2.7, 1.1, 0.205}, {2.8, 0.5, 0.175}},   // FP8
      {{3.0, 1.1, 0.275}, {2.6, 0.6, 0.18}, {2.6, 0.6, 0.18}}};    // bf16 / fp16
  const bool fp4 = kind == GemmKind::kNvfp4;
  // the fused re-quantization's 64-column groups need 128-column tiles, and no
  // 16-bit kernel has narrow ones
  const bool linear = epi == Epilogue::kLinear || epi == Epilogue::kLinearRequant;
  const bool narrow_ok =
      epi != Epilogue::kRequant && epi != Epilogue::kLinearRequant && kind != GemmKind::k16;
  const TileCost* cost = kCosts[(int)kind];
  const int64_t stages = (k_row_bytes(kind, K) + kStageRowBytes - 1) / kStageRowBytes;
  const int64_t tiles_m = (M + kTileM - 1) / kTileM;
  const int64_t n128 = (N + 127) / 128, n256 = (N + 255) / 256;
  // An output amax costs single-CTA tiles more per wave (its reductions, and y
  // through the staging) and a pair tile more at its end: without these terms
  // short K chains took single tiles where pairs are faster (NVFP4 9216 x 3072 x 64:
  // 33.0 us, single tiles 37.6).
  const double wave_extra = epi == Epilogue::kAmax ? 0.2 : 0.0;
  // With bias, activation and residual a wave takes at least its epilogue, and a pair
  // tile, with twice the columns per thread, ends later: bf16 1500 x 6144 x 512 with GELU
  // 15.7 us in pairs, 13.1 in single tiles; FP8 2048 x 2048 x 2048 11.9 and 10.8; NVFP4
  // 2048 x 2048 x 2048 8.6 and 9.2.
  // 128 x 192 tiles for the 16-bit linears, where they need a wave less (with GELU and
  // residual, W from HBM: 1333 x 2112 x 1088 12.8 -> 11.6 us, x 256 8.9 -> 7.5; 2000 x 5120
  // x 1088 26.4, in pairs 28.3, -> 24.2).
  static const TileCost kWide{2.6, 0.8, 0.275};
  const bool wide_ok = epi == Epilogue::kLinear && kind == GemmKind::k16;
  double us[4] = {cost[0].us((tiles_m + 1) / 2 * n256, num_sms / 2, stages, 0.0, linear ? 4.0 : 0.0),
                  cost[1].us(tiles_m * n128, num_sms, stages, wave_extra, linear ? 2.1 : 0.0),
                  cost[2].us(tiles_m * ((N + 63) / 64), num_sms, stages, wave_extra, linear ? 1.2 : 0.0),
                  kWide.us(tiles_m * ((N + 191) / 192), num_sms, stages, wave_extra, 3.1)};
  if (linear) us[0] += fp4 ? 1.0 : 1.5;
  // a pair tile's re-quantizing epilogue ends about this much later
  if (epi == Epilogue::kRequant) us[0] += fp4 ? 1.0 : 0.6;
  if (epi == Epilogue::kAmax) us[0] += 1.0;
  int pick = tiles_m * n256 >= num_sms ? 0 : narrow_ok && 2 * tiles_m * n128 <= num_sms ? 2 : 1;
  int best = pick;
  for (int t = 0; t < 4; ++t)
    if (us[t] < us[best] && (t < 2 || (t == 2 ? narrow_ok : wide_ok))) best = t;
  if (us[best] < 0.9 * us[pick]) pick = best;
  return static_cast<Tile>(pick);
}

// CTAs of a cluster that share a tile's K, for 128 x 128 tiles too few to fill the machine.
// Sending the sums and joining them costs 1.5-3 us, so K has to be long, longer where there
// is room for two CTAs only or, with two more barriers' worth of skew, for eight.  (M x N x K
// in us with one, two and four CTAs: NVFP4 552 x 832 x 2048 6.5, 7.3, 7.5; x 3072 8.2, 8.2,
// 8.0; x 12288 20.8, 14.7, 11.6; FP8 x 3072 8.1, 8.5, 8.2; x 12288 20.2, 15.1, 12.1; bf16 x
// 1024 7.9, 7.5, 7.7; x 12288 43.2, 23.9, 17.0.  With four and eight: 352 x 320 x 12288 NVFP4
// 10.4, 8.9; FP8 10.5, 9.3; bf16 352 x 640 x 2048 7.7, 8.0.  All with W from HBM; from L2 a
// single CTA gains more, NVFP4 555 x 832 x 4096 7.6 against 8.2.)  A cluster of eight needs eight
// SMs of one GPC: fifteen run at once on 152 SMs, with sixteen tiles some wait (bf16 500 x
// 512 x 2048 14.3 us, with four CTAs 7.8).
inline int choose_split_k(GemmKind kind, int64_t M, int64_t N, int64_t K, int num_sms) {
  static const int kLeast[3][3] = {{20, 16, 24}, {48, 32, 48}, {24, 20, 44}};   // stages; 2, 4, 8 CTAs
  const int64_t stages = (k_row_bytes(kind, K) + kStageRowBytes - 1) / kStageRowBytes;
  const int64_t tiles_m = (M + kTileM - 1) / kTileM, tiles_n = (N + 127) / 128;
  if (tiles_m > num_sms || tiles_n > num_sms) return 1;
  const int64_t tiles = tiles_m * tiles_n;
  const int* least = kLeast[(int)kind];
  if (10 * 8 * tiles <= 8 * (int64_t)num_sms && stages >= least[2]) return 8;
  if (4 * tiles <= num_sms && stages >= least[1]) return 4;
  return 2 * tiles <= num_sms && stages >= least[0] ? 2 : 1;
}

// Whether a linear takes the few-token kernel, which reads W once per 16 tokens, rather
// than the tiles above: always up to 16 tokens, beyond that as long as its units, 16 rows
// of W and 16 tokens, are at most 5.2 per SM with 16-bit operands, 2.6 with others (1.9
// over rows of W shorter than 2048 bytes, from 33 tokens).  Few / tiles, timed over N
// 64-12288, K 512-12288 and M 16-1600, in us: bf16 128 x 768 x 12288 16.6 / 45.4 (4.9
// units per SM), 552 x 64 x 12288 10.9 / 42.8 (0.9), 1600 x 128 x 768 6.1 / 6.2 (5.3), 352
// x 768 x 6144 42 / 24 (6.9); FP8 960 x 64 x 6144 8.4 / 12.1 (1.6), 32 x 3072 x 3072 7.9 /
// 7.9 (2.5), 48 x 2048 x 768 4.7 / 4.1 (2.5), 352 x 320 x 12288 18.2 / 19.8 (2.9); NVFP4
// 552 x 128 x 768 3.3 / 3.9 (1.8), 32 x 3072 x 3072 6.9 / 8.1 (2.5), 1600 x 64 x 2560 6.6 /
// 5.7 and x 12288 18.0 / 21.1 (2.6); at 16 tokens NVFP4 N = 12288 9.9 / 10.2.
inline bool few_tokens(bool float16, int64_t M, int64_t N, int64_t row_bytes, int num_sms) {
  if (M <= 16) return true;
  const int limit = float16 ? 52 : M <= 32 || row_bytes >= 2048 ? 26 : 19;
  // (M < 2^31 and N / 16 < 2^59: beyond a limit that large grids exceed anyway)
  return N / 16 <= limit * (int64_t)num_sms && 10 * (N / 16) * ((M + 15) / 16) <= limit * (int64_t)num_sms;
}

// Whether tiles with a split K take a linear that few_tokens would give to the few-token
// kernel: from 65 tokens, once the few-token kernel's units have much of W to read (units
// per SM times kilobytes of a row).  Few / split, in us: bf16 552 x 64 x 4096 7.2 / 8.1 (7),
// 176 x 768 x 2560 9.2 / 8.1 (18), 176 x 320 x 12288 16.7 / 11.2 (35), 48 x 768 x 12288 10.9
// / 11.9; FP8 960 x 64 x 4096 6.9 / 7.5 (6.5), 128 x 768 x 4096 8.8 / 7.1 (10); NVFP4 552 x
// 128 x 4096 5.7 / 6.4 (3.7), 352 x 128 x 12288 11.7 / 8.1 (7).
inline bool split_over_few(GemmKind kind, int64_t M, int64_t N, int64_t K, int num_sms) {
  const double units = (double)(N / 16) * (double)((M + 15) / 16) / num_sms;
  const double least = kind == GemmKind::kNvfp4 ? 4.5 : kind == GemmKind::kFp8 ? 8.0 : 12.0;
  return M > 64 && units * ((double)k_row_bytes(kind, K) / 1024) >= least &&
         choose_split_k(kind, M, N, K, num_sms) > 1;
}

}  // namespace qlin
