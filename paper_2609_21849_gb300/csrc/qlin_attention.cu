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
  p.k_scale = c.format == QLIN_CACHE_E4M3 ? c.k_scale : nullptr;   // (16-bit values have none, whatever is set)
  p.v_scale = c.format == QLIN_CACHE_E4M3 ? c.v_scale : nullptr;
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
  const CacheKind kind = c.format == QLIN_CACHE_E4M3   ? CacheKind::kE4m3
                         : c.format == QLIN_CACHE_FP16 ? CacheKind::kFp16
                                                       : CacheKind::kBf16;
  // The tiles from 17 rows per sequence and KV head on (on average), where the mma.sync kernel would
  // read the keys again for every 16: in us, 16 sequences of 4096-8192 keys, 8 heads of 128, tiles and
  // mma.sync, 16 rows 86, 86 (E4M3 97, 62), 20 rows 86, 181 (97, 173), 64 rows 90, 344 (102, 328).  And
  // for 16-bit heads past 192, whose fragments leave mma.sync one CTA of four warps per SM, over a
  // table with room for 128 MB of keys and values (one token, heads of 256, 4096 keys: 86, 126; one
  // sequence of 500 16, 14).
  const bool many = p.tokens * p.group > (int64_t)16 * p.sequences;
  const bool wide = kind != CacheKind::kE4m3 && p.head_dim > 192 &&
                    (int64_t)p.sequences * p.table_width * p.page_size >= ((int64_t)128 << 20) / (4 * p.heads * p.head_dim);
  if ((many || wide) && attention_tiles_fit(p)) return launch_attention_tiles(p, kind, timeout_ns, s, dev);
  return c.format == QLIN_CACHE_E4M3   ? launch_attention_e4m3(p, s, dev)
         : c.format == QLIN_CACHE_FP16 ? launch_attention_fp16(p, s, dev)
                                       : launch_attention_bf16(p, s, dev);
}

}  // namespace qlin
