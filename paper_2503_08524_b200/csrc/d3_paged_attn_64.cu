// Paged attention for head dimension 64 (see d3_paged_attn.cuh).
#include "d3_paged_attn.cuh"

namespace d3 {

int launch_paged_attention_64(const TMap &k, const TMap &v, PagedAttnArgs a, int cache, int x, cudaStream_t st) {
  return paged_attn::launch_types<64>(k, v, a, cache, x, st);
}

}  // namespace d3
