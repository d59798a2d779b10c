// Paged attention for head dimension 128 (see d3_paged_attn.cuh).
#include "d3_paged_attn.cuh"

namespace d3 {

int launch_paged_attention_128(const TMap &k, const TMap &v, PagedAttnArgs a, int cache, int x, cudaStream_t st) {
  return paged_attn::launch_types<128>(k, v, a, cache, x, st);
}

}  // namespace d3
