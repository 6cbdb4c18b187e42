// Attention of a chunk over a cache in 8 bits (chunk_attn.cuh).
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_q8(const ChunkCall& c) {
  return few_fits(c.T, c.B, c.Hq / c.Hkv) ? launch_few_attn_q8(c) : launch_chunk<kQ8>(c);
}

}  // namespace libraspec
