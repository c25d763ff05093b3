// Parameters of the attention kernels over a paged cache.
#pragma once

#include "qlin_cache.h"
#include "qlin_internal.h"

namespace qlin {

enum class CacheKind { kBf16, kFp16, kE4m3 };

// An item of the tiles' kernel that begins in a CTA and ends in another (rows 0: none does).
struct JoinItem {
  int64_t token0;
  int row0, head0, rows, last;   // last: the CTA that it ends in
};

struct AttnParams {
  const uint16_t* q;
  int64_t q_token, q_head;        // elements
  uint16_t* out;
  int64_t out_token, out_head;
  float* lse;                     // or null
  int64_t lse_token;
  const uint64_t* mask;           // or null: a token sees those before it
  int64_t mask_token;             // words
  int mask_words;
  const uint8_t *k, *v;
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;   // bytes
  const int32_t* table;
  int64_t table_stride;
  const int32_t* cached;
  const int32_t* q_start;
  const float *k_scale, *v_scale;   // E4M3
  int64_t tokens;
  int sequences, pages, page_size, table_width;
  int heads, group, head_dim;       // group: query heads of a KV head
  float scale_log2;                 // scale * log2(e)
  int fp16;                         // q and out are fp16, not bf16
  // workspace: counts (zero between calls), (maximum, sum) and sums of unfinished rows
  unsigned* counts;
  JoinItem* join;            // of the tiles' kernel
  float2* part_ml;
  float* part;
  int least;                        // tiles that a CTA should have
  int item_cost;                    // tiles that an item's begin and end take as long as
  unsigned* err;
};

// Workspace: two counts per CTA (mma.sync) and an item to join (tiles), then two unfinished items per CTA.
constexpr int kMostCtas = 1024;
constexpr int64_t kCountBytes = 2 * kMostCtas * 4;
constexpr int64_t kJoinBytes = kMostCtas * sizeof(JoinItem);
constexpr int64_t kWorkspaceBytes = (int64_t)64 << 20;

// Many rows on tcgen05 (qlin_attention_tiles.cu): whether it takes these pages and heads.
bool attention_tiles_fit(const AttnParams& p);
cudaError_t launch_attention_tiles(const AttnParams& p, CacheKind kind, uint64_t timeout_ns, cudaStream_t s, Device dev);
cudaError_t launch_attention_bf16(const AttnParams& p, cudaStream_t s, Device dev);
cudaError_t launch_attention_fp16(const AttnParams& p, cudaStream_t s, Device dev);
cudaError_t launch_attention_e4m3(const AttnParams& p, cudaStream_t s, Device dev);

}  // namespace qlin
