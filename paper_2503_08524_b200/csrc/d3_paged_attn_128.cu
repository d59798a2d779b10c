// Paged attention for head dimension 128 (see d3_paged_attn.cuh).
#include "d3_paged_attn.cuh"

namespace d3 {

int launch_paged_attention_128(const PoolMaps &m, const PagedAttnArgs &a, int x, cudaStream_t st) {
  return paged_attn::launch_types<128>(m, a, x, st);
}

}  // namespace d3
