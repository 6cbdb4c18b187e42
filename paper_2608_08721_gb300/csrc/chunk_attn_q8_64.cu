// Attention of a chunk over a cache in 8 bits (chunk_attn.cuh), heads of 64.
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_q8_64(const ChunkCall& c) { return launch_chunk<kQ8, 64>(c); }

}  // namespace libraspec
