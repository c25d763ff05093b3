// Attention over a paged cache: the call's parameters, and which kernel takes it.
#include "qlin_attention.h"

namespace qlin {

cudaError_t launch_cache_attention(const qlin_cache_t& c, const qlin_cache_attention_t& a, void* workspace,
                                   cudaStream_t s, Device dev, unsigned* err, uint64_t timeout_ns) {
  const int es = c.format == QLIN_CACHE_E4M3 ? 1 : 2;
  AttnParams p{};
  p.q = static_cast<const uint16_t*>(a.q);
  p.q_token = a.q_token_stride;
  p.q_head = a.q_head_stride;
  p.out = static_cast<uint16_t*>(a.out);
  p.out_token = a.out_token_stride;
  p.out_head = a.out_head_stride;
  p.lse = a.lse;
  p.lse_token = a.q_heads;
  p.mask = a.mask;
  p.mask_token = a.mask_stride;
  p.mask_words = a.mask_words;
  p.k = static_cast<const uint8_t*>(c.k);
  p.v = static_cast<const uint8_t*>(c.v);
  p.k_page = c.k_page_stride * es;
  p.k_slot = c.k_slot_stride * es;
  p.k_head = c.k_head_stride * es;
  p.v_page = c.v_page_stride * es;
  p.v_slot = c.v_slot_stride * es;
  p.v_head = c.v_head_stride * es;
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
  p.heads = c.heads;
  p.group = a.q_heads / c.heads;
  p.head_dim = c.head_dim;
  p.scale_log2 = a.scale * 1.442695041f;
  p.fp16 = a.dtype == QLIN_FP16 ? 1 : 0;
  p.counts = static_cast<unsigned*>(workspace);
  p.err = err;
  // more rows per sequence and KV head, on average, than the mma.sync kernel shares a read among
  const CacheKind kind = c.format == QLIN_CACHE_E4M3   ? CacheKind::kE4m3
                         : c.format == QLIN_CACHE_FP16 ? CacheKind::kFp16
                                                       : CacheKind::kBf16;
  if (p.tokens * p.group > (int64_t)32 * p.sequences && attention_tiles_fit(p))
    return launch_attention_tiles(p, kind, timeout_ns, s, dev);
  return c.format == QLIN_CACHE_E4M3   ? launch_attention_e4m3(p, s, dev)
         : c.format == QLIN_CACHE_FP16 ? launch_attention_fp16(p, s, dev)
                                       : launch_attention_bf16(p, s, dev);
}

}  // namespace qlin
