// Attention of a chunk over a cache in 8 bits (chunk_attn.cuh), heads of 128; few rows go to few_attn_q8.cu.
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_q8(const ChunkCall& c) {
  const int g = c.Hq / c.Hkv;
  ChunkCall rest = c;
  if (few_fits(c.T, c.B, g)) {
    const cudaError_t e = launch_few_attn_q8(c);
    if (e != cudaSuccess || few_alone(c.T, g)) return e;
    rest.least_new = few_rows(c.T, c.B, g) / g + 1;
  }
  return c.D == 128 ? launch_chunk<kQ8, 128>(rest) : launch_chunk_attn_q8_64(rest);
}

}  // namespace libraspec
