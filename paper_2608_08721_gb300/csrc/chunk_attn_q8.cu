// Attention of a chunk over a cache in 8 bits (chunk_attn.cuh), heads of 128; few rows go to few_attn_q8.cu.
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_q8(const ChunkCall& c) {
  if (few_fits(c.T, c.B, c.Hq / c.Hkv)) return launch_few_attn_q8(c);
  return c.D == 128 ? launch_chunk<kQ8, 128>(c) : launch_chunk_attn_q8_64(c);
}

}  // namespace libraspec
