// Paged attention for head dimension 64 (see d3_paged_attn.cuh).
#include "d3_paged_attn.cuh"

namespace d3 {

int launch_paged_attention_64(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st) {
  return paged_attn::launch_types<64>(m, a, x, st);
}

}  // namespace d3
