// Attention over a paged cache of e4m3 keys and values (a translation unit per type, so that
// they compile side by side).
#include "qlin_attention.cuh"

namespace qlin {

cudaError_t launch_attention_e4m3(const AttnParams& p, cudaStream_t s, Device dev) {
  return launch_attn_kind<CacheKind::kE4m3>(p, s, dev);
}

}  // namespace qlin
