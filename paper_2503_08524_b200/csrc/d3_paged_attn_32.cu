// Paged attention for head dimension 32 (see d3_paged_attn.cuh).
#include "d3_paged_attn.cuh"

namespace d3 {

int launch_paged_attention_32(const TMap &k, const TMap &v, PagedAttnArgs a, int cache, int x, cudaStream_t st) {
  return paged_attn::launch_types<32>(k, v, a, cache, x, st);
}

}  // namespace d3
