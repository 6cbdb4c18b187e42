// One call of the chunk attention, from the C ABI to the kernels' launches.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace libraspec {

constexpr int kChunkMaxSinks = 1 << 20;  // LIBRASPEC_MAX_SINKS

// One call. block_table == nullptr: dense caches [B, Hkv, S_cap, D]. page_size: a multiple of 16.
struct ChunkCall {
  const uint16_t* Q;
  const void *K, *V;           // bf16, or e4m3 codes with
  const uint8_t *Ks, *Vs;      // their exponents for every `block` tokens
  int block;
  const int32_t* block_table;
  int max_pages, page_size, n_pages;
  const int32_t *cu_new, *kv_len;
  int T, B, Hq, Hkv, D, S_cap;
  float scale, softcap;
  const float* slopes;
  int window, sinks;
  const int32_t *first_key, *prefix_len;
  uint16_t* O;
  float* lse;
  char* ws;
  cudaStream_t stream;
  int least_new;  // sequences with fewer new tokens are left out
};

size_t chunk_workspace_bytes(long long T, int B, int Hq, int Hkv, int d, bool q8);
cudaError_t launch_chunk_attn(const ChunkCall& c);
cudaError_t launch_sink_attn(const ChunkCall& c);     // without first keys
cudaError_t launch_chunk_attn_q8(const ChunkCall& c);
// what these pass on: heads of 64, and calls that few_fits
cudaError_t launch_chunk_attn_64(const ChunkCall& c);
cudaError_t launch_chunk_attn_q8_64(const ChunkCall& c);
cudaError_t launch_few_attn_q8(const ChunkCall& c);

}  // namespace libraspec
