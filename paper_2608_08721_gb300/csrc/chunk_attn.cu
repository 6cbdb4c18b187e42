// Attention of a chunk over a cache of bf16 (chunk_attn.cuh), heads of 128.
#include "chunk_attn.cuh"

namespace libraspec {

size_t chunk_workspace_bytes(long long T, int B, int Hq, int Hkv, int d, bool q8) {
  const ChunkWs w = chunk_ws(T, B, Hq, Hkv, d);
  return q8 ? w.total : w.q_parts;
}

cudaError_t launch_chunk_attn(const ChunkCall& c) {
  return c.D == 128 ? launch_chunk<0, 128>(c) : launch_chunk_attn_64(c);
}

}  // namespace libraspec
