// Attention of a chunk over a cache in 8 bits (chunk_attn.cuh).
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_q8(const ChunkCall& c) { return launch_chunk<kQ8>(c); }

}  // namespace libraspec
