// Attention of a chunk over a cache of bf16 in a window whose first tokens stay visible (chunk_attn.cuh).
#include "chunk_attn.cuh"

namespace libraspec {

cudaError_t launch_sink_attn(const ChunkCall& c) {
  return c.D == 128 ? launch_chunk<kSink, 128>(c) : launch_chunk<kSink, 64>(c);
}

}  // namespace libraspec
