// Attention of a chunk over a cache of bf16 (chunk_attn.cuh), heads of 64.
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_chunk_attn_64(const ChunkCall& c) { return launch_chunk<0, 64>(c); }

}  // namespace libraspec
