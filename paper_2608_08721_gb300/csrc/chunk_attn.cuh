// Attention of a ragged chunk of new tokens over the KV cache, dense or paged
// (a prompt, a part of one, or the one token of a decode step), one layer.
//
// Row (b, j, h): query head h of the j-th new token of sequence b, at position
// p = kv_len_b + j; the keys of the new tokens are in the cache already, so
// the sequence has N_b = kv_len_b + n_b keys. The row sees keys [lo, hi):
//   lo = max(0, p - window + 1 if a window is given, first_key of the token)
//   hi = min(N_b, max(p + 1, prefix_len_b))
// and with s = scale q.k (then cap tanh(s / cap), then - slope_h |p - k|):
//   O = sum exp(s - m) V / sum exp(s - m),  lse = m + log sum exp(s - m);
// a row that sees nothing has O = 0 and lse = -inf.
//
// Work. The rows of a (sequence, kv head), g = Hq / Hkv per token, are cut into
// blocks of two row tiles of R = g floor(128 / g) rows (whole tokens, one
// tcgen05 M = 128 tile each), the keys that a block sees into 128-key tiles.
// All (block, kv head, key tile) triples form one sequence, cut over the
// persistent grid (one CTA per SM) by cost: each block weighs its tiles plus C
// tile-equivalents (its queries' load and its epilogue), and CTA c takes the
// tiles of the c-th share of the weight, so that CTAs finish together whatever
// the lengths. The blocks and their key tiles follow from the device-resident
// lengths: a plan kernel lists them, and a launch dependent on it does the
// work; up to 64 blocks each CTA's producer lists for itself.
//
// Two streams per CTA, each a softmax warpgroup with its own P and O
// accumulator in tensor memory, so that one stream's MMAs run beside the
// other's softmax. A block of two row tiles gives each stream one of them, both
// reading the same K and V tiles in shared memory (loaded once for 256 rows:
// at 128 rows per load, L2 would bound a prompt's attention). A block of one
// row tile (decode, short chunks) gives the streams alternate key tiles of the
// same rows; the epilogue combines them.
//
// Roles in a CTA (384 threads): two softmax warpgroups; a producer warp whose
// lanes each load their own piece of a K or V tile by TMA (a piece lies within
// one page) into a ring of chunks; an MMA warp, converged, whose elected lane
// issues. Thread i of a warpgroup owns row i of its tile: it takes the tile's
// 128 scores into registers, masks them only where the tile reaches beyond
// what its warp's rows all see, and writes P as bf16 (16 bits are what the
// tensor cores take; sums are of the unrounded values, in 32 bits). With the
// scores in registers their place is free for the next S, which runs beside
// this tile's softmax: at D = 64 the stream's own next, at D = 128, where O
// and P leave room for the scores of one tile only, the other stream's. (With
// P over its scores, S waited for the PV before it: 1039 us where it now takes
// 960, at D = 64 931 where it takes 816.) The reference maximum of a row is
// raised only when a score exceeds it by more than 8 (a factor of 2^8), so O
// is rarely rescaled; p <= 2^8 keeps P and O in range.
//
// What bounds it, with 128-wide heads: prompts, shared memory, from which S =
// Q K^T alone reads 128 bytes a cycle, and the tensor pipe beside it: 16384
// tokens of 8 heads over as many keys run at 1.72 PFLOP/s, where a matrix
// product reaches 1.92; an item's start and end cost as much as three tiles or
// four, which is why short prompts stay further off. Capped or biased scores,
// the softmax warps' arithmetic (a capped score takes two exponentials and a
// reciprocal). Decode steps, the cache's bytes: 64 sequences over 512 to 32768
// keys run at the copy rate. One sequence over 512 keys: 11 us of first
// instruction fetches and of round trips (plan, K, S, softmax, V, merge),
// hardly of bytes.
//
// Keys that no row of a block sees take no part: K and V pieces that hold none
// of them are not read (their pages need not exist), and V rows beyond the
// block's range are cleared in shared memory before the MMA, so that what an
// unwritten cache row holds (NaN, say) does not meet the zeros of P; so are the
// rows within it of tokens that no row sees (padding), which first keys allow.
//
// A cache in 8 bits (kQ8): codes c of e4m3, values c 2^e with an exponent for every 16 to 64 keys of a kv head. Keys meet
// the queries as e4m3, as they lie in memory, the queries in two e4m3 parts (split_q_kernel), one behind the other along
// the contraction, which costs the tensor pipe what one product of 16-bit operands does. The rows' and keys' scales enter
// the softmax, which multiplies scores by them anyway. Values are converted to f16 by a fourth warpgroup, code by code
// (exactly), and P is f16, times its value's scale: P' = 2^(s - m + e), O = sum P' V8, l = sum P' 2^-e. The exponent e of
// each 16 keys enters behind the mask, so neither the reference m nor P' of a row depends on a key that it does not see.
// (With a tile's values brought to its largest exponent instead, a hidden key's scale took the bits of what the row sees;
// it was no faster either: a prompt of 8192 tokens 484 us, 466 so.) One more warp brings the exponents, two tiles'
// look-ups ahead; a tile's count with its scores on one barrier. What bounds it: the softmax warps' steps, beside which
// the converters issue (25 of the 466 us go when the conversion is left out, 25 are the queries' parts; bf16 takes 385).
// Measured and not kept, when the prompt took 518: K converted as well (647), the queries' parts in the kernel (615).
//
// Sinks (kSink): keys below `sinks` stay visible to every row behind them. A block's tiles are then the first ones of the
// sequence that hold sinks, and those of its window; what lies between is not read.
//
// A block cut over CTAs c0..c1 leaves one fp32 partial (O, m, l) per CTA; the
// CTA that delivers the last of them merges all, in CTA order (results do not
// depend on timing). No CTA waits for another.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include <cudaTypedefs.h>

#include "chunk_call.h"
#include "common.cuh"
#include "tc.cuh"

namespace libraspec {

int num_sms_current();

constexpr int kCStreams = 2;
constexpr int kCSoftmaxWarps = 4 * kCStreams;
constexpr int kCProducerWarp = kCSoftmaxWarps;
constexpr int kCMmaWarp = kCSoftmaxWarps + 1;
constexpr int kCThreads = (kCSoftmaxWarps + 4) * 32;  // (the last two warps only make up a warpgroup)
constexpr int kCRows = 128;                 // rows of a tile (tensor-memory lanes)
constexpr int kCBlockRows = 2 * kCRows;     // rows of a block, at most
constexpr int kCKeys = 128;                 // keys of a tile
constexpr int kCMaxCtas = 192;
constexpr int kCMaxCounts = 2048;           // counters: the few-row kernel has two per CTA, up to three CTAs on an SM
constexpr int kCTmemCols = 512;
constexpr float kCRescaleLog2 = 8.f;
// A cache in 8 bits has P in f16, whose least step is 2^-24: the reference lies 2^7 below the maximum (P <= 2^15 then,
// f16 ends at 2^16), so that terms down to 2^-31 of the largest take part.
constexpr float kHeadroomLog2 = 7.f;
constexpr uint32_t kBf16Operands = 1u << 7 | 1u << 10;  // of an instruction descriptor; without: f16
constexpr int kPlanThreads = 1024;
constexpr int kCSharedBytes = 64 << 20;     // K and V beyond half of L2: see the plan's waves
constexpr int kNoPage = -2;                 // (of a block table: -1 and below are invalid alike)
constexpr int kCMaxKeys = 0x7fffffff - 2 * kCKeys;  // of a sequence: its last tile's end is an int

// ---------------------------------------------------------------------------
// Workspace: status, plan header, merge counters, block table of the plan,
// partials.
// ---------------------------------------------------------------------------
struct PlanBlock {       // the rows of one block and the key tiles that they see
  long long tiles_before;  // key tiles of the blocks before it (per kv head)
  int pairs_before;        // blocks of two row tiles before it
  int b, tok0, n_tok;      // sequence; first packed row and tokens
  int pos0;                // position of the first token
  int klo, khi;            // keys that some row sees lie in [klo, khi)
  // 128-key tiles: the first `sink` of the sequence, which hold the sinks, then tile0 + i for the others (i >= sink)
  int tile0, n_tiles;
  int gaps;                // keys within [klo, khi) may be seen by no row
  int sink, pad;
};
static_assert(sizeof(PlanBlock) == 56, "");

struct PlanHead {
  long long tiles;  // of all blocks (per kv head)
  int blocks, pairs;
  int waves;        // whole items (a block for a kv head) that each CTA takes before the rest is cut by cost
  int pad;
};

struct ChunkWs {
  size_t status, head, count, blocks, seen, part_o, part_ml, q_parts, q_exp, total;
};

// Tokens of a block and the most blocks that T tokens of B sequences have.
inline int block_tokens(int g) { return 2 * (kCRows / g); }
inline long long max_blocks(long long T, int B, int g) {
  const long long a = T / block_tokens(g) + B;
  return a < T ? a : T;
}

// The few-row kernel (few_attn_q8.cu) has blocks of 8 rows, or of 16. It takes part where the sequences have 16 rows per kv
// head on average at most. Up to 1024 rows are all its own; of more it takes the sequences whose tokens fit a block and the
// other kernel the rest, whose keys would be read for 16 rows at a time: 255 tokens decoded over 2000 keys each beside a
// chunk of 512 over 8000 (g = 4) take 312 us so and 640 by itself, 127 beside 300 over 2000 keys 172 and 210; a chunk of
// 4096 over 2000 keys among 4095 sequences without new tokens 97 and 556. The launches for the rest cost 5 to 16 us, though,
// also where there is none, in a decode step of many sequences (one token each of 300 over 512 keys, g = 4: 89 us, 81
// without them; of 1024 over 1024 keys 377 and 365); with fewer rows that is more than it gives (63 beside 100 over 500 keys
// 73 and 52, four tokens each of 8 sequences 25 and 19; but 63 over 500 keys beside 100 over 16000 110 and 189). The host
// knows T and B, not how the tokens are spread: T <= B alone does not make a decode step.
constexpr int kFewRows = 16, kFewAlone = 1024;
inline bool few_alone(long long T, int g) { return T * g <= kFewAlone; }
inline bool few_fits(long long T, int B, int g) { return g <= kFewRows && T * g <= (long long)kFewRows * B; }
inline int few_rows(long long T, int B, int g) { return g <= 8 && T * g <= 8ll * B ? 8 : 16; }
inline long long few_blocks(long long T, int B, int tokens) { return std::min(T, T / tokens + B); }

static ChunkWs chunk_ws(long long T, int B, int Hq, int Hkv, int d) {
  ChunkWs w{};
  const int g = Hq / Hkv;
  long long blocks = max_blocks(T, B, g);
  // (also of calls with fewer tokens)
  if (g <= kFewRows) blocks = std::max(blocks, few_blocks(std::min(T, (long long)kFewRows * B / g), B, std::max(1, 8 / g)));
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = align256(off + bytes); return o; };
  w.status = take(256);
  w.head = take(sizeof(PlanHead));
  w.count = take(kCMaxCounts * sizeof(uint32_t));
  w.blocks = take((size_t)blocks * sizeof(PlanBlock));
  w.seen = take((size_t)blocks * (kCBlockRows / 8));  // a bit for each token of a block
  // two slots per CTA: its first item, and its last where that goes on in the next CTA
  w.part_o = take(size_t(2 * kCMaxCtas) * kCBlockRows * d * sizeof(float));
  w.part_ml = take(size_t(2 * kCMaxCtas) * kCBlockRows * 2 * sizeof(float));
  // (a cache in 8 bits alone: the other calls' workspaces end here) the queries as e4m3 parts, and their exponents
  w.q_parts = take((size_t)T * Hq * d * 2);
  w.q_exp = take((size_t)T * Hq);
  w.total = off;
  return w;
}

// bits [0, n) set, n clamped to [0, 32]
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

// What a row sees.
struct MaskArgs {
  const int32_t* first_key;   // [T] or NULL
  const int32_t* prefix_len;  // [B] or NULL
  int window;                 // 0: none
  int sinks;                  // first keys that the window does not hide (0 with first keys)
};

__device__ __forceinline__ void row_range(int pos, int n_keys, int prefix, int first, int window, int& lo, int& hi) {
  lo = max(0, first);
  if (window > 0 && pos >= window) lo = max(lo, pos - window + 1);
  hi = min(n_keys, max(pos + 1, prefix));
  if (hi < lo) hi = lo;
}

// ---------------------------------------------------------------------------
// The plan: blocks in sequence order.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ T block_scan(T v, T* warp_sums, T& total) {  // inclusive, kPlanThreads threads
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const T a = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v += a;
  }
  __syncthreads();  // (the sums of the scan before have been read)
  if (lane == 31) warp_sums[warp] = v;
  __syncthreads();
  T w = warp_sums[lane];
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const T a = __shfl_up_sync(0xffffffffu, w, off);
    if (lane >= off) w += a;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const T before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  return warp > 0 ? v + before : v;
}

struct PlanArgs {
  const int32_t* cu_new;
  const int32_t* kv_len;
  MaskArgs mask;
  int T, B, TB;      // TB: tokens of a block
  int S_cap, Hkv, grid;
  int shared_tiles;  // key tiles (of all kv heads) beyond which L2 does not hold them
  int least, most;   // sequences with fewer or more new tokens are another kernel's
  int* status;
};

// New tokens of sequence b, 0 where its offsets or length are out of range (reported if asked to).
__device__ __forceinline__ int new_tokens(const PlanArgs& a, int b, bool report, int& c0, int& kv) {
  c0 = a.cu_new[b];
  kv = a.kv_len[b];
  const int hi = a.cu_new[b + 1];
  if (c0 < 0 || hi < c0 || hi > a.T) {
    if (report) raise_status(a.status, LIBRASPEC_ST_BAD_LENGTH);
    return 0;
  }
  if (kv < 0 || (long long)kv + (hi - c0) > a.S_cap) {
    if (report) raise_status(a.status, LIBRASPEC_ST_KV_OVERFLOW);
    return 0;
  }
  return hi - c0 < a.least || hi - c0 > a.most ? 0 : hi - c0;
}

// The most blocks that T tokens of B sequences have: offsets that run backwards could ask for more.
__device__ __forceinline__ int block_room(const PlanArgs& a) {
  return (int)min((long long)a.T, (long long)a.T / a.TB + a.B);
}

// Keys that some row of tokens [j0, j1) of a sequence sees lie in [klo, khi). Its n tokens start at row c0 and position
// kv. Rows that see their own key leave no gap between them. A row whose document starts behind it does not, and then
// its key may be one that no row of the block sees. No other key of the range can be: one before the block is seen by
// the row whose range starts there; one behind it is in the range only through the prefix, with which the rows' ranges
// end. `gaps`: there are such rows; bits of the tokens whose keys some row sees then lie in a table.
struct KeyRange {
  int lo, hi, gaps;
};
constexpr int kSeenWords = kCBlockRows / 32;  // of a block
// without first keys: ranges move forward with the position
__device__ __forceinline__ KeyRange key_range(const PlanArgs& a, int b, int n, int kv, int j0) {
  const int j1 = min(n, j0 + a.TB), N = kv + n, prefix = a.mask.prefix_len ? a.mask.prefix_len[b] : 0;
  KeyRange k;
  int l, h;
  row_range(kv + j0, N, prefix, 0, a.mask.window, k.lo, h);
  row_range(kv + j1 - 1, N, prefix, 0, a.mask.window, l, k.hi);
  k.gaps = 0;
  return k;
}
// with them, by a warp (a thread for each block, one key after the other, took 17 us longer for 5721 tokens)
__device__ __forceinline__ KeyRange key_range_docs(const PlanArgs& a, int b, int c0, int n, int kv, int j0,
                                                   uint32_t* seen) {
  const int j1 = min(n, j0 + a.TB), N = kv + n, prefix = a.mask.prefix_len ? a.mask.prefix_len[b] : 0;
  int klo = 0x7fffffff, khi = 0;
  bool gaps = false;
  for (int j = j0 + (threadIdx.x & 31); j < j1; j += 32) {
    int l, h;
    row_range(kv + j, N, prefix, a.mask.first_key[c0 + j], a.mask.window, l, h);
    gaps |= l > kv + j;
    if (l < h) {
      klo = min(klo, l);
      khi = max(khi, h);
    }
  }
  klo = __reduce_min_sync(0xffffffffu, klo);
  khi = __reduce_max_sync(0xffffffffu, khi);
  if (klo >= khi) klo = khi = (N - 1) / kCKeys * kCKeys;  // no row sees a key: one tile, no piece of it read
  gaps = __any_sync(0xffffffffu, gaps);
  if (gaps) {
    uint32_t bits[kSeenWords] = {};
    for (int j = j0 + (threadIdx.x & 31); j < j1; j += 32) {
      int l, h;
      row_range(kv + j, N, prefix, a.mask.first_key[c0 + j], a.mask.window, l, h);
      l = max(l - (kv + j0), 0);
      h = min(h - (kv + j0), j1 - j0);
#pragma unroll
      for (int w = 0; w < kSeenWords; ++w)
        if (l < h) bits[w] |= bits_below(h - 32 * w) & ~bits_below(l - 32 * w);
    }
#pragma unroll
    for (int w = 0; w < kSeenWords; ++w) {
      const uint32_t all = __reduce_or_sync(0xffffffffu, bits[w]);
      if ((threadIdx.x & 31) == 0) seen[w] = all;
    }
  }
  return KeyRange{klo, khi, gaps};
}

// Block of tokens [j0, j0 + TB) of sequence b.
__device__ __forceinline__ PlanBlock make_block(const PlanArgs& a, int b, int c0, int n, int kv, int j0, KeyRange k) {
  PlanBlock p{};
  p.b = b;
  p.tok0 = c0 + j0;
  p.n_tok = min(n - j0, a.TB);
  p.pos0 = kv + j0;
  p.klo = k.lo;
  p.khi = k.hi;
  const int tile0 = k.lo / kCKeys;
  p.sink = min((min(a.mask.sinks, k.hi) + kCKeys - 1) / kCKeys, tile0);
  p.tile0 = tile0 - p.sink;
  p.n_tiles = p.sink + max(1, (k.hi + kCKeys - 1) / kCKeys - tile0);
  p.gaps = k.gaps;
  return p;
}

// Blocks of a sequence that start together and walk its keys in step read each K and V tile from HBM once and from L2
// after that; cut by cost their CTAs are all at different keys, which matters where the keys do not fit L2 (1024 tokens
// over 131072 keys: 2.96 ms instead of 3.17).
__device__ __forceinline__ int whole_waves(const PlanArgs& a, int n_blocks, int n_seqs, long long kv_tiles, int t_min,
                                           int t_max) {
  const bool together = n_blocks >= 2 * n_seqs && kv_tiles * a.Hkv > a.shared_tiles && t_max - t_min <= t_max / 8;
  return together ? (int)min((long long)n_blocks * a.Hkv / a.grid, 1ll << 20) : 0;
}

// (Two scans of up to a thousand entries each, all else by shared atomics: with four scans a prompt of 8192 tokens took
// 374 us, with two 368.)
static __global__ void __launch_bounds__(kPlanThreads) chunk_plan_kernel(const PlanArgs a, PlanBlock* __restrict__ blocks,
                                                                  PlanHead* __restrict__ head,
                                                                  uint32_t* __restrict__ seen) {
  __shared__ int first_block[LIBRASPEC_MAX_B + 1];  // of each sequence
  __shared__ long long warp_sums[32];
  __shared__ KeyRange ranges[kPlanThreads];  // (first keys)
  __shared__ unsigned long long kv_tiles;    // of the sequences that have new tokens
  __shared__ int n_seqs, t_min, t_max;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31;
  if (tid == 0) {
    kv_tiles = 0;
    n_seqs = t_max = 0;
    t_min = 0x7fffffff;
  }
  long long carry = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    int nb = 0;
    unsigned nt = 0;
    if (b < a.B) {
      int c0, kv;
      const int n = new_tokens(a, b, true, c0, kv);
      nb = (n + a.TB - 1) / a.TB;
      if (nb) nt = ((unsigned)kv + (unsigned)n + kCKeys - 1) / kCKeys;
    }
    long long total;
    const long long inc = block_scan((long long)nb, warp_sums, total);
    if (b < a.B) first_block[b] = (int)min(carry + inc - nb, (long long)0x7fffffff);
    carry += total;
    const unsigned seqs = __popc(__ballot_sync(0xffffffffu, nb > 0));
    nt = __reduce_add_sync(0xffffffffu, nt);  // (32 of at most 2^24)
    if (lane == 0 && seqs) {
      atomicAdd(&kv_tiles, (unsigned long long)nt);
      atomicAdd(&n_seqs, (int)seqs);
    }
  }
  const int room = block_room(a), n_blocks = (int)min(carry, (long long)room);
  if (tid == 0) {
    first_block[a.B] = n_blocks;
    if (carry > room) raise_status(a.status, LIBRASPEC_ST_BAD_LENGTH);
  }
  __syncthreads();
  auto seq_of = [&](int e) {  // the last b with first_block[b] <= e (it has blocks: e < first_block[b + 1])
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first_block[mid] <= e) lo = mid;
      else hi = mid;
    }
    return lo;
  };
  long long tiles = 0;
  int pairs = 0;
  for (int e0 = 0; e0 < n_blocks; e0 += kPlanThreads) {
    const int e = e0 + tid;
    PlanBlock p{};
    if (a.mask.first_key) {
      for (int i = tid >> 5; i < kPlanThreads && e0 + i < n_blocks; i += kPlanThreads / 32) {
        int c0, kv;
        const int b = seq_of(e0 + i), n = new_tokens(a, b, false, c0, kv);
        const KeyRange k = key_range_docs(a, b, c0, n, kv, (e0 + i - first_block[b]) * a.TB,
                                          seen + (size_t)(e0 + i) * kSeenWords);
        if (lane == 0) ranges[i] = k;
      }
      __syncthreads();
    }
    if (e < n_blocks) {
      int c0, kv;
      const int b = seq_of(e), n = new_tokens(a, b, false, c0, kv), j0 = (e - first_block[b]) * a.TB;
      p = make_block(a, b, c0, n, kv, j0, a.mask.first_key ? ranges[tid] : key_range(a, b, n, kv, j0));
    }
    // tiles and pairs in one sum (of a thousand blocks: at most 2^34 tiles, 2^10 pairs)
    const long long v = ((long long)p.n_tiles << 12) | (p.n_tok > a.TB / 2);
    long long total;
    const long long before = block_scan(v, warp_sums, total) - v;
    const int lo = __reduce_min_sync(0xffffffffu, e < n_blocks ? p.n_tiles : 0x7fffffff);
    const int hi = __reduce_max_sync(0xffffffffu, p.n_tiles);
    if (lane == 0 && hi) {
      atomicMin(&t_min, lo);
      atomicMax(&t_max, hi);
    }
    if (e < n_blocks) {
      p.tiles_before = tiles + (before >> 12);
      p.pairs_before = pairs + (int)(before & 4095);
      blocks[e] = p;
    }
    tiles += total >> 12;
    pairs += (int)(total & 4095);
  }
  __syncthreads();
  if (tid == 0) {
    head->tiles = tiles;
    head->blocks = n_blocks;
    head->pairs = pairs;
    head->waves = whole_waves(a, n_blocks, n_seqs, (long long)kv_tiles, t_min, t_max);
  }
}

// The same for up to kWarpBlocks blocks by one warp, in its registers: lane l has blocks l and l + 32. Every CTA's
// producer then plans for itself, and the call is one launch (a decode step of one sequence over 512 keys: 12.8 us with
// the plan's launch, 10.9 without).
constexpr int kWarpBlocks = 64;
constexpr int kWarpSeqs = 512;

__device__ __forceinline__ int warp_scan(int v) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, v, off);
    if (lane >= off) v += x;
  }
  return v;
}

static __device__ PlanHead warp_plan(const PlanArgs& a, PlanBlock (&mine)[2]) {
  const int lane = threadIdx.x & 31, room = block_room(a);
  mine[0] = mine[1] = PlanBlock{};
  int carry = 0, n_seqs = 0;
  long long kv_tiles = 0;
  for (int b0 = 0; b0 < a.B; b0 += 32) {
    int c0 = 0, kv = 0, n = 0;
    if (b0 + lane < a.B) n = new_tokens(a, b0 + lane, blockIdx.x == 0, c0, kv);
    const int nb = (n + a.TB - 1) / a.TB, inc = warp_scan(nb), total = __shfl_sync(0xffffffffu, inc, 31);
    n_seqs += __popc(__ballot_sync(0xffffffffu, nb > 0));
    kv_tiles += nb ? ((long long)kv + n + kCKeys - 1) / kCKeys : 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e = lane + 32 * k - carry;  // among these sequences' blocks
      int s = 0;                            // its sequence: the first whose inclusive count is above e
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
        if (__shfl_sync(0xffffffffu, inc, s + off - 1) <= e) s += off;
      s = min(s, 31);
      const int sc = __shfl_sync(0xffffffffu, c0, s), sn = __shfl_sync(0xffffffffu, n, s);
      const int skv = __shfl_sync(0xffffffffu, kv, s), before = __shfl_sync(0xffffffffu, inc - nb, s);
      if (e >= 0 && e < total && lane + 32 * k < room) {
        const int j0 = (e - before) * a.TB;
        mine[k] = make_block(a, b0 + s, sc, sn, skv, j0, key_range(a, b0 + s, sn, skv, j0));
      }
    }
    carry += total;
  }
  if (carry > room && blockIdx.x == 0 && lane == 0) raise_status(a.status, LIBRASPEC_ST_BAD_LENGTH);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) kv_tiles += __shfl_xor_sync(0xffffffffu, kv_tiles, off);
  PlanHead h{};
  h.blocks = min(carry, room);
  int t_min = 0x7fffffff, t_max = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    // (at most 64 blocks of 2^24 tiles: an int)
    const int nt = mine[k].n_tiles, pair = mine[k].n_tok > a.TB / 2, inc = warp_scan(nt), inc_p = warp_scan(pair);
    mine[k].tiles_before = h.tiles + inc - nt;
    mine[k].pairs_before = h.pairs + inc_p - pair;
    h.tiles += __shfl_sync(0xffffffffu, inc, 31);
    h.pairs += __shfl_sync(0xffffffffu, inc_p, 31);
    if (nt) {
      t_min = min(t_min, nt);
      t_max = max(t_max, nt);
    }
  }
  t_min = __reduce_min_sync(0xffffffffu, t_min);
  t_max = __reduce_max_sync(0xffffffffu, t_max);
  h.waves = whole_waves(a, h.blocks, n_seqs, kv_tiles, t_min, t_max);
  return h;
}

// ---------------------------------------------------------------------------
// The attention kernel.
// ---------------------------------------------------------------------------
// What a block weighs beside its tiles, in tiles: `one` for every block, `pair` more for two row tiles. (A prompt
// of 8192 tokens of 32 heads: 445 us at 1 + 1, 380 at 2 + 1, 372 at 2 + 2, 376 at 2 + 3 and at 3 + 2;
// decoding is best at 2.)
struct FixedCost {
  int one, pair;
};

// Of a cap and the scores' scale, from the host.
struct CapArgs {
  float log2;           // the cap in units of log 2
  float twice_inverse;  // 2 scale / cap in units of log 2 (finite: under the smallest caps a score of zero stays zero)
  float inverse;        // scale / cap
};

struct ChunkArgs {
  CUtensorMap K, V, Q;
  __nv_bfloat16* O;
  float* lse;
  const int32_t* cu_new;
  const int32_t* kv_len;
  const int32_t* block_table;
  const float* slopes;  // [Hq] or NULL
  MaskArgs mask;
  PlanArgs plan;
  const PlanBlock* blocks;  // NULL: each producer plans for itself
  const PlanHead* head;
  const uint32_t* seen;     // [blocks][kSeenWords], of blocks with gaps
  float* part_o;
  float* part_ml;
  uint32_t* count;
  int* status;
  float scale;
  CapArgs cap;
  int Hq, Hkv, max_pages, page_size, n_pages, piece;  // piece: keys of one TMA box
  FixedCost fixed;
  int o_wide;  // O is aligned to 32 bytes
  // cache in 8 bits: exponents of the scales [planes, Hkv, rows / 2^block_log2] (rows: of a page, or S_cap)
  const uint8_t *Ks, *Vs;
  int block_log2, rows;
  const uint8_t* q_exp;  // [T, Hq]: exponent + 127 of what the queries were multiplied by
};

// One item: a run of key tiles of one block for one kv head.
struct ChunkItem {
  int b, kvh, tok0, pos0;
  int rows;            // of the block
  int pair;            // two row tiles (a stream each), else one (alternate key tiles)
  int tile0, n_tiles;
  int klo, khi;
  int partial, slot;   // write a partial to this slot, else O
  int c0, np;          // first CTA of the block and how many share it
  int last;            // the CTA's last item; 2: it has none
  // the sink tiles among its own: 2^16 times the block's, and how many of them (the last) it has
  int sink;
  int gaps;            // (first keys) the block, if it has gaps, else -1
  int pad[3];
};
static_assert(sizeof(ChunkItem) == 80, "items lie in 80-byte slots");
static_assert(kChunkMaxSinks / kCKeys < 1 << 15, "");

// The sequence's tile that is the item's j-th.
template <bool SINK>
__device__ __forceinline__ int item_tile(const ChunkItem& it, int j) {
  if (SINK) {
    const int left = it.sink & 0xffff;
    if (j < left) return (it.sink >> 16) - left + j;
  }
  return it.tile0 + j;
}

// What scores are beside a scaled product: bit 0 capped, bit 1 biased by distance, bit 2 capped far above the scores;
// bit 3: rows have first keys; bit 4: the cache is in 8 bits; bit 5: sinks. (Instantiations: the code of each in the
// plain kernel costs it instruction fetches, also beside its loop.)
constexpr int kCap = 1, kBias = 2, kWideCap = 4, kDocs = 8, kQ8 = 16, kSink = 32;

// (8 bits) What the softmax takes of a tile's scales, for every 16 keys: K's scale, and the exponent of V's.
struct TileScales {
  float k[8];
  __half v_log2[8];
};
static_assert(sizeof(TileScales) == 48, "");

// A cache in 8 bits: tiles of K in a ring that the MMAs read as it is; raw tiles of V in another, converted to f16 by a
// warpgroup into the ring of chunks.
template <int D, bool Q8>
struct ChunkSmem {
  static constexpr int kBoxes = D / 64;
  static constexpr int kTile = kBoxes * 16384;           // 128 rows of Q, K or V: per 64 columns 128 rows of 128 bytes
  static constexpr int kChunks = Q8 ? (D == 128 ? 3 : 4) : (D == 128 ? 5 : 10);
  static constexpr int kRawTile = 128 * D;
  static constexpr int kKs = D == 128 ? 2 : 6, kRaws = D == 128 ? 2 : 6;
  static constexpr int kQ = 0;                           // two row tiles
  static constexpr int kRing = 2 * kTile;
  static constexpr int kKRing = kRing + kChunks * kTile;
  static constexpr int kRaw = kKRing + (Q8 ? kKs * kRawTile : 0);
  static constexpr int kBar = kRaw + (Q8 ? kRaws * kRawTile : 0);
  // full[chunks], empty[chunks], ifull[2], iempty[2], sfull[2], got[2][2], pvdone[2], ofree[2], qfull,
  // qempty, drain, gap; 8 bits: kfull[ks], kempty[ks], rfull[raws], rempty[raws], cempty[2]
  static constexpr int kNumBars = 2 * kChunks + 14 + 4 + (Q8 ? 2 * kKs + 2 * kRaws + 2 : 0);
  static constexpr int kInfo = kBar + (8 * kNumBars + 15) / 16 * 16;
  static constexpr int kMisc = kInfo + 2 * 80;           // [0] misaligned, [1] this CTA merges, [2] tensor memory
  static constexpr int kStat = kMisc + 16;               // (m, l) of streams to be combined: of each, or of one at a time
  static constexpr int kScales = kStat + (Q8 ? 1 : kCStreams) * kCRows * 8;  // [stream]: struct TileScales
  static constexpr int kBytes = kScales + (Q8 ? kCStreams * 48 : 0);
  // tensor memory: scores, of each stream (D = 64) or of the step at hand (128: no room for two), P and O of each
  static constexpr int kScores = D == 128 ? 1 : 2;
  static constexpr int kColS = 0, kColP = kScores * 128, kColO = kColP + kCStreams * 64;
  static_assert(kColO + kCStreams * D == kCTmemCols, "");
  static_assert(kScales % 16 == 0 && kBytes <= 227 * 1024, "shared memory per CTA");
};

// Registers by role: 384 threads start with 168 each (64512 in all); the softmax warpgroups take 208, the third
// warpgroup keeps 88 (256 x 208 + 128 x 88 = 64512).
constexpr int kCSoftmaxRegs = 208, kCOtherRegs = 88;
static_assert(kCSoftmaxWarps * 32 * kCSoftmaxRegs + 128 * kCOtherRegs <= kCThreads * 168, "");
// A cache in 8 bits takes a warpgroup more: 512 threads start with 128 each (65536 in all), of which the softmax keeps
// 200, the third warpgroup 80 and the converters 32 (256 x 200 + 128 x 80 + 128 x 32 = 65536), which suffices for two
// units of a tile at a time. (With 72 and 40, and four units, the producer spills: a prompt of 8192 tokens 461 us, 466 so,
// but 38 sequences of 41 to 82 tokens over up to 336 keys 48.4 and 44.1, chunks with sinks 67.5 and 65.5.)
constexpr int kCThreadsQ8 = kCThreads + 128;
constexpr int kScaleWarp = kCMmaWarp + 1, kConvertWarp = kCMmaWarp + 3, kConverters = 4;
constexpr int kQ8SoftmaxRegs = 200, kQ8OtherRegs = 80, kQ8ConvertRegs = 32;
static_assert(kCSoftmaxWarps * 32 * kQ8SoftmaxRegs + 128 * kQ8OtherRegs + 128 * kQ8ConvertRegs <= kCThreadsQ8 * 128, "");
template <int N>
__device__ __forceinline__ void regs_take() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_leave() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ void bar_sync_n(int bar, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(threads) : "memory");
}
constexpr int kCAllBar = 1;

// A wait that the first ask did not end.
static __device__ __noinline__ bool slow_wait(uint32_t bar, uint32_t parity) { return warp_wait(bar, parity); }

// (d0, d1) = (a0, a1) * b + (c0, c1)
__device__ __forceinline__ void fma2v(float& d0, float& d1, float a0, float a1, float b, float c0, float c1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %6};\n\t"
      "fma.rn.f32x2 a, a, b, c;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "=f"(d0), "=f"(d1)
      : "f"(a0), "f"(a1), "f"(b), "f"(c0), "f"(c1));
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// cap tanh(s / cap) in units of log 2, of a score s = scale x: by the series s (1 - t^2 / 3 + 2 t^4 / 15 -
// 17 t^6 / 315 + 62 t^8 / 2835), t = s / cap, whose next term is below 2^-26 of s for |t| <= 1 / 4; beyond that with
// r = 1 / (exp(2 t) + 1).
constexpr float kSeriesTop = 0.25f;
__device__ __forceinline__ float cap_series(float x, float scale_log2, float inverse) {
  const float t = x * inverse, t2 = t * t, s = x * scale_log2;
  const float p = fmaf(fmaf(fmaf(62.f / 2835.f, t2, -17.f / 315.f), t2, 2.f / 15.f), t2, -1.f / 3.f);
  return fmaf(s, t2 * p, s);
}
__device__ __forceinline__ float wide_cap(float x, float r, float scale_log2, const CapArgs& cap) {
  return fabsf(x * cap.inverse) <= kSeriesTop ? cap_series(x, scale_log2, cap.inverse)
                                              : cap.log2 * fmaf(-2.f, r, 1.f);
}
// 32 bytes at once
__device__ __forceinline__ void store32(void* p, const uint32_t (&r)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
               "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ uint32_t c_pack(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// two values as e4m3, to the nearest, ties to even, saturating
__device__ __forceinline__ uint32_t e4m3_of(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// two e4m3 codes as f16, exactly
__device__ __forceinline__ uint32_t f16_of_e4m3(uint16_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return h;
}
__device__ __forceinline__ float power_of_two_biased(uint32_t e) { return __uint_as_float(e << 23); }  // 2^(e - 127)

// (8 bits) The queries as two e4m3 parts: a row (a token's head) times the power of two that brings its largest into
// [2^7, 2^8) becomes the nearest e4m3 and the rest, together all eight bits of what lies within 2^-9 of the largest, else
// off by 2^-17 of it at most. Per 64 elements the first parts, then the second, in the bytes that the elements took. A
// launch of its own (25 us for a prompt of 8192 tokens of 32 heads, as long beside the plan as behind it): in the
// attention, where each CTA did it for its items, the prompt took 92 us longer, and 104 in place by the converters (what a
// warp reads of shared memory beside the MMAs takes 150 to 400 cycles, a shuffle too).
// e4m3 has no infinity: of a row that holds some, they become 1 with their sign, finite elements 0 beside them, NaN stays,
// and the row's factor is infinite (kInfiniteRow in the place of its exponent). Scores are then infinite or NaN as the
// formula's are.
constexpr int kSplitThreads = 256, kInfiniteRow = 255;
template <int D>
static __global__ void __launch_bounds__(kSplitThreads) split_q_kernel(const uint16_t* __restrict__ Q, long long rows,
                                                                       uint8_t* __restrict__ parts,
                                                                       uint8_t* __restrict__ exps) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr int kLanes = D / 16;  // of a row
  const long long i = (long long)blockIdx.x * kSplitThreads + threadIdx.x, row = i / kLanes;
  const int j = (int)(i % kLanes);
  uint4 v[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (row < rows) {
    const uint4* src = reinterpret_cast<const uint4*>(Q + row * D) + 2 * j;
    v[0] = src[0];
    v[1] = src[1];
  }
  const uint32_t w[8] = {v[0].x, v[0].y, v[0].z, v[0].w, v[1].x, v[1].y, v[1].z, v[1].w};
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) top = __vmaxu2(top, w[k] & 0x7fff7fffu);
  top = max(top & 0xffffu, top >> 16);
#pragma unroll
  for (int off = 1; off < kLanes; off <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
  // (rows below 2^-119 are not brought up that far: the factor and its inverse are normal numbers)
  const bool infinite = top >= 0x7f80u;
  const int fe = infinite ? kInfiniteRow : min(261 - (int)(top >> 7), 253);
  const float f = infinite ? 1.f : power_of_two_biased(fe);
  auto part_of = [&](float x) { return !infinite ? x * f : fabsf(x) == INFINITY ? copysignf(1.f, x) : x == x ? 0.f : x; };
  uint32_t first[4], rest[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float x0 = part_of(bf16_lo(w[2 * k])), x1 = part_of(bf16_hi(w[2 * k]));
    const float x2 = part_of(bf16_lo(w[2 * k + 1])), x3 = part_of(bf16_hi(w[2 * k + 1]));
    const uint32_t lo = e4m3_of(x0, x1), hi = e4m3_of(x2, x3);
    const uint32_t hl = f16_of_e4m3((uint16_t)lo), hh = f16_of_e4m3((uint16_t)hi);
    const float2 yl = __half22float2(*reinterpret_cast<const __half2*>(&hl));
    const float2 yh = __half22float2(*reinterpret_cast<const __half2*>(&hh));
    first[k] = lo | hi << 16;
    rest[k] = e4m3_of(x0 - yl.x, x1 - yl.y) | e4m3_of(x2 - yh.x, x3 - yh.y) << 16;
  }
  if (row >= rows) return;
  uint4* dst = reinterpret_cast<uint4*>(parts + row * D * 2 + j / 4 * 128 + j % 4 * 16);
  dst[0] = make_uint4(first[0], first[1], first[2], first[3]);
  dst[4] = make_uint4(rest[0], rest[1], rest[2], rest[3]);
  if (j == 0) exps[row] = (uint8_t)fe;
}

// a / b for a >= 0, b > 0, in 32 bits where both fit (a 64-bit division is a long sequence, and a call of one token has
// several of them between its launch and its first copy)
__device__ __forceinline__ long long quotient(long long a, long long b) {
  if ((((unsigned long long)a | (unsigned long long)b) >> 32) == 0) return (long long)((uint32_t)a / (uint32_t)b);
  return a / b;
}

// The CTA whose share of the weight W holds position y: the largest c with floor(c W / G) <= y.
__device__ __forceinline__ int share_of(long long y, long long W, int G) {
  return (int)quotient((y + 1) * (long long)G - 1, W);
}

// Weight of the blocks before block e (per kv head), and of block e.
__device__ __forceinline__ long long weight_before(const PlanBlock& p, int e, FixedCost f) {
  return p.tiles_before + (long long)f.one * e + (long long)f.pair * p.pairs_before;
}
__device__ __forceinline__ int fixed_of(const PlanBlock& p, int g, FixedCost f) {
  return f.one + (p.n_tok > kCRows / g ? f.pair : 0);
}

// Where weighted position x lies.
struct Place {
  int e, kvh, tile;     // block, kv head, tile within the block
  long long before;     // tiles before it in the tile sequence
};

// The plan's blocks, by the warp: from the table, or from the lanes' registers.
struct Blocks {
  const PlanBlock* __restrict__ table;  // NULL: registers
  const PlanBlock (&mine)[2];
  int n;
  // block e, the same for all lanes
  __device__ __forceinline__ PlanBlock at(int e) const {
    if (table) return table[e];
    const PlanBlock& m = e < 32 ? mine[0] : mine[1];
    PlanBlock p;
    p.tiles_before = __shfl_sync(0xffffffffu, m.tiles_before, e);
    p.pairs_before = __shfl_sync(0xffffffffu, m.pairs_before, e);
    p.b = __shfl_sync(0xffffffffu, m.b, e);
    p.tok0 = __shfl_sync(0xffffffffu, m.tok0, e);
    p.n_tok = __shfl_sync(0xffffffffu, m.n_tok, e);
    p.pos0 = __shfl_sync(0xffffffffu, m.pos0, e);
    p.klo = __shfl_sync(0xffffffffu, m.klo, e);
    p.khi = __shfl_sync(0xffffffffu, m.khi, e);
    p.tile0 = __shfl_sync(0xffffffffu, m.tile0, e);
    p.n_tiles = __shfl_sync(0xffffffffu, m.n_tiles, e);
    p.gaps = 0;  // (without first keys)
    p.sink = __shfl_sync(0xffffffffu, m.sink, e);
    return p;
  }
};

// Whether a row of a block with gaps sees a key of [key0, key1), which lies in the block's range. seen: as in KeyRange.
__device__ __forceinline__ bool some_row_sees(const uint32_t* seen, int pos0, int n_tok, int key0, int key1) {
  const int j0 = key0 - pos0, j1 = key1 - pos0;
  if (j0 < 0 || j1 > n_tok) return true;
  for (int w = j0 / 32; w <= (j1 - 1) / 32; ++w)
    if (seen[w] & bits_below(j1 - 32 * w) & ~bits_below(j0 - 32 * w)) return true;
  return false;
}

// Block e's Hkv copies start at Hkv times the weight before it, each with its fixed cost first; x < the total.
static __device__ Place find_place(long long x, const Blocks& blocks, int Hkv, int g, FixedCost f) {
  const int lane = threadIdx.x & 31;
  int lo = 0;  // the last block that starts at or before x
  if (blocks.table) {
    for (int n = blocks.n; n > 1;) {  // it is in [lo, lo + n)
      const int step = (n + 31) / 32, i = lo + lane * step;
      const bool at = lane * step < n && (long long)Hkv * weight_before(blocks.table[i], i, f) <= x;
      const int k = 31 - __clz(__ballot_sync(0xffffffffu, at));  // (lane 0 always holds)
      n = min(step, n - k * step);
      lo += k * step;
    }
  } else {
    for (int k = 0; k < 2; ++k) {
      const int e = lane + 32 * k;
      const bool at = e < blocks.n && (long long)Hkv * weight_before(k ? blocks.mine[1] : blocks.mine[0], e, f) <= x;
      lo += __popc(__ballot_sync(0xffffffffu, at));
    }
    --lo;
  }
  Place p;
  p.e = lo;
  const PlanBlock b = blocks.at(lo);
  const long long o = x - (long long)Hkv * weight_before(b, lo, f);
  const int c = fixed_of(b, g, f), w = b.n_tiles + c;
  p.kvh = (int)quotient(o, w);
  const int r = (int)(o - (long long)p.kvh * w);
  p.tile = r > c ? r - c : 0;
  p.before = (long long)Hkv * b.tiles_before + (long long)p.kvh * b.n_tiles + p.tile;
  return p;
}

// Merges the np partials of an item's rows: O = sum_p w_p O_p / sum_p w_p l_p with w_p = 2^(m_p - M), M = max m_p. A
// thread of the softmax warpgroups takes a row and eight columns at a time, U of them with P parts' loads in flight
// (one by four columns a merge of two parts of 256 rows took 20 us, a round trip for each of 32 steps); neighbouring
// threads take neighbouring rows, which lie side by side in the partials.
template <int D, int U, int P>
__device__ __forceinline__ void merge_parts(const ChunkArgs& A, const ChunkItem& it, int g) {
  const int np = it.np, c0 = it.c0, rows = it.rows, units = rows * (D / 8);
  const int step = kCSoftmaxWarps * 32;
  for (int k0 = threadIdx.x; k0 < units; k0 += U * step) {
    float M[U], L[U];
    float acc[U][8];
    int r[U], c[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + u * step, units - 1);  // (a unit past the end repeats the last)
      c[u] = k / rows;
      r[u] = k - c[u] * rows;
      M[u] = -INFINITY;
      L[u] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[u][e] = 0.f;
    }
    for (int p0 = 0; p0 < np; p0 += P) {
      float2 ml[U][P];
      float4 v[U][P][2];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < P; ++q) {
          const int p = p0 + q;
          ml[u][q] = make_float2(-INFINITY, 0.f);
          v[u][q][0] = v[u][q][1] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (p < np) {
            const size_t slot = p == 0 ? 2 * c0 + 1 : 2 * (c0 + p);
            ml[u][q] = __ldcg(reinterpret_cast<const float2*>(A.part_ml) + slot * kCBlockRows + r[u]);
            const float4* o =
                reinterpret_cast<const float4*>(A.part_o) + (slot * (D / 4) + 2 * c[u]) * kCBlockRows + r[u];
            v[u][q][0] = __ldcg(o);
            v[u][q][1] = __ldcg(o + kCBlockRows);
          }
        }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float Mn = M[u];
#pragma unroll
        for (int q = 0; q < P; ++q) Mn = fmaxf(Mn, ml[u][q].x);
        const bool none = Mn == -INFINITY;  // nothing seen so far, or NaN alone
        const float f = none ? 1.f : ex2_approx(M[u] - Mn);  // 0 while M is -inf
        M[u] = Mn;
        L[u] *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[u][e] *= f;
#pragma unroll
        for (int q = 0; q < P; ++q) {
          const float w = none ? 1.f : ex2_approx(ml[u][q].x - Mn);
          L[u] += w * ml[u][q].y;
          const float x[8] = {v[u][q][0].x, v[u][q][0].y, v[u][q][0].z, v[u][q][0].w,
                              v[u][q][1].x, v[u][q][1].y, v[u][q][1].z, v[u][q][1].w};
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[u][e] += w * x[e];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * step >= units) continue;
      const float inv = L[u] > 0.f ? 1.f / L[u] : L[u] == 0.f ? 0.f : L[u];  // (NaN stays)
      const size_t row = (size_t)(it.tok0 + r[u] / g) * A.Hq + it.kvh * g + r[u] % g;
      reinterpret_cast<uint4*>(A.O + row * D)[c[u]] =
          make_uint4(c_pack(acc[u][0] * inv, acc[u][1] * inv), c_pack(acc[u][2] * inv, acc[u][3] * inv),
                     c_pack(acc[u][4] * inv, acc[u][5] * inv), c_pack(acc[u][6] * inv, acc[u][7] * inv));
      if (A.lse && c[u] == 0) A.lse[row] = (M[u] + __log2f(L[u])) * kLn2;
    }
  }
}

// Largest cap that kCap alone takes. Its cap (1 - 2 / (e + 1)) is off by up to 2^-23 of the cap (of 256: 3e-5, an
// eighth of what a sum of products may be off); above it scores below a quarter of the cap take the odd series of the
// tangent (4000 tokens in windows of 1024 keys: 222 us, 175 under a cap that kCap takes).
constexpr float kNarrowCap = 256.f;
constexpr float kFloatMax = 3.402823466e38f, kFloatMin = 1.175494351e-38f;

// The tile that step t of n takes. With a bias by distance from the last one back: the keys nearest to the rows come
// first and set the reference, which each tile towards the rows would raise (16384 tokens of 8 heads over as many keys:
// 1457 us from the front, 1105 from the back; at a head dim of 64, 1374 and 1165).
template <int SHAPE>
__device__ __forceinline__ int tile_of(int t, int n) { return SHAPE & kBias ? n - 1 - t : t; }

template <int D, int SHAPE>
__global__ void __launch_bounds__(SHAPE & kQ8 ? kCThreadsQ8 : kCThreads, 1)
    chunk_attn_kernel(const __grid_constant__ ChunkArgs A) {
  constexpr bool Q8 = SHAPE & kQ8, SINK = SHAPE & kSink;
  using SM = ChunkSmem<D, Q8>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sQ = smem_u32(smem + SM::kQ);
  const uint32_t sRing = smem_u32(smem + SM::kRing);
  const uint32_t sK = smem_u32(smem + SM::kKRing), sRaw = smem_u32(smem + SM::kRaw);
  const uint32_t bFull = smem_u32(smem + SM::kBar);
  const uint32_t bEmpty = bFull + 8 * SM::kChunks;
  const uint32_t bIFull = bEmpty + 8 * SM::kChunks;
  const uint32_t bIEmpty = bIFull + 16;
  const uint32_t bSFull = bIEmpty + 16;   // [stream]
  const uint32_t bGot = bSFull + 16;      // [stream][word & 1]
  const uint32_t bPVDone = bGot + 32;     // [stream]
  const uint32_t bOFree = bPVDone + 16;   // [stream]
  const uint32_t bQFull = bOFree + 16;
  const uint32_t bQEmpty = bQFull + 8;
  const uint32_t bDrain = bQEmpty + 8;
  const uint32_t bGap = bDrain + 8;       // V tiles of which the producer clears rows
  const uint32_t bKFull = bGap + 8;       // 8 bits: tiles of K, raw ones of V, the tiles' scales
  const uint32_t bKEmpty = bKFull + 8 * SM::kKs;
  const uint32_t bRFull = bKEmpty + 8 * SM::kKs;
  const uint32_t bREmpty = bRFull + 8 * SM::kRaws;
  const uint32_t bCEmpty = bREmpty + 8 * SM::kRaws;  // [stream]
  ChunkItem* info = reinterpret_cast<ChunkItem*>(smem + SM::kInfo);
  volatile int* misc = reinterpret_cast<int*>(smem + SM::kMisc);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = A.Hq / A.Hkv;
  const int Rt = kCRows / g, R = g * Rt;  // tokens and rows of a row tile

  if (warp == kCProducerWarp && lane < 3)
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane == 0   ? &A.Q
                                                                             : lane == 1 ? &A.K
                                                                                         : &A.V))
                 : "memory");
  if (tid == 0) {
    for (int s = 0; s < SM::kChunks; ++s) {
      mbar_init(bFull + 8 * s, Q8 ? kConverters : 1);
      mbar_init(bEmpty + 8 * s, 1);  // the MMA warp's commit after the chunk's last use
    }
    for (int q = 0; q < 2; ++q) {
      mbar_init(bIFull + 8 * q, 1);
      mbar_init(bIEmpty + 8 * q, 1 + kCSoftmaxWarps + (Q8 ? 1 + kConverters : 0));
      mbar_init(bSFull + 8 * q, Q8 ? 2 : 1);  // (8 bits: the tile's scales count as well)
      mbar_init(bGot + 16 * q, 4);
      mbar_init(bGot + 16 * q + 8, 4);
      mbar_init(bPVDone + 8 * q, 1);
      mbar_init(bOFree + 8 * q, 4);
    }
    mbar_init(bQFull, 1);
    mbar_init(bQEmpty, 1);
    mbar_init(bDrain, 1);
    mbar_init(bGap, 1);
    if constexpr (Q8) {
      for (int s = 0; s < SM::kKs; ++s) {
        mbar_init(bKFull + 8 * s, 1);
        mbar_init(bKEmpty + 8 * s, 1);
      }
      for (int s = 0; s < SM::kRaws; ++s) {
        mbar_init(bRFull + 8 * s, 1);
        mbar_init(bREmpty + 8 * s, kConverters);
      }
      for (int s = 0; s < 2; ++s) mbar_init(bCEmpty + 8 * s, 4);
    }
    misc[0] = (sQ & 1023) != 0;  // (the swizzled tiles need the alignment that the declaration asks for)
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kCMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     smem_u32(const_cast<int*>(misc + 2))),
                 "n"(kCTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = (uint32_t)misc[2];
  const bool misaligned = misc[0] != 0;

  if (misaligned) {
    if (tid == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
  } else if (Q8 && warp >= kConvertWarp) {
    // ======================= converters: raw tiles of V to f16 =======================
    regs_leave<kQ8ConvertRegs>();
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int ct = tid - kConvertWarp * 32;
    constexpr int kUnits = D / 16, kRowStep = 128 / kUnits;  // 16-byte units of a row; rows between a thread's units
    // (a row's second box lies on the first's banks: its threads take the row beside it, whose swizzle differs)
    const int cj = ct % kUnits, crow = ct / kUnits ^ (D == 128 ? cj >> 2 : 0);
    const int to0 = (D == 128 ? cj / 4 * 16384 : 0) + crow * 128 + ((2 * cj ^ crow) & 7) * 16;
    const int to1 = to0 ^ 16;
    uint32_t item_ctr = 0, raw_ctr = 0;
    bool ok = true;
    for (int last = 0; !last && ok; ++item_ctr) {
      ok = warp_wait(bIFull + 8 * (item_ctr & 1), (item_ctr >> 1) & 1);
      if (!ok) break;
      const ChunkItem& src = info[item_ctr & 1];
      ChunkItem it;
      it.n_tiles = src.n_tiles;
      it.tile0 = src.tile0;
      it.sink = src.sink;
      it.klo = src.klo;
      it.khi = src.khi;
      it.gaps = src.gaps;
      it.pos0 = src.pos0;
      it.rows = src.rows;
      last = src.last;
      if (last == 2) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bIEmpty + 8 * (item_ctr & 1));
      const int n = it.n_tiles, n_tok = it.rows / g;
      const int sinks = SINK ? min(A.mask.sinks, it.khi) : 0;
      const uint32_t* seen = A.seen + (size_t)max(it.gaps, 0) * kSeenWords;
      for (int t = 0; t < n; ++t, ++raw_ctr) {
        const uint32_t rc = raw_ctr % SM::kRaws, ch = raw_ctr % SM::kChunks;
        ok = warp_wait(bRFull + 8 * rc, (raw_ctr / SM::kRaws) & 1) &&
             warp_wait(bEmpty + 8 * ch, ((raw_ctr / SM::kChunks) & 1) ^ 1);
        if (!ok) break;
        const int kt0 = item_tile<SINK>(it, tile_of<SHAPE>(t, n)) * kCKeys;
        // rows that no row of the block sees become zeros (what they hold, NaN say, does not meet the zeros of P)
        const bool gap = (SHAPE & kDocs) && it.gaps >= 0 && kt0 + kCKeys > it.pos0 && kt0 < it.pos0 + n_tok;
        const bool edge = kt0 < it.klo || kt0 + kCKeys > it.khi || gap;
        const uint8_t* raw = smem + SM::kRaw + rc * SM::kRawTile + crow * D + cj * 16;
        uint8_t* dst = smem + SM::kRing + ch * SM::kTile;
#pragma unroll 1
        for (int i0 = 0; i0 < kUnits; i0 += 2) {
          uint4 v[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const uint4*>(raw + (i0 + i) * 2048);
          if (edge) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int key = kt0 + crow + (i0 + i) * kRowStep;
              bool some = key < it.khi && (key >= it.klo || key < sinks);
              if (some && gap) some = some_row_sees(seen, it.pos0, n_tok, key, key + 1);
              if (!some) v[i] = make_uint4(0, 0, 0, 0);
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            auto to_f16 = [&](uint32_t codes) { return f16_of_e4m3((uint16_t)codes); };
            const uint4 lo = make_uint4(to_f16(v[i].x), to_f16(v[i].x >> 16), to_f16(v[i].y), to_f16(v[i].y >> 16));
            const uint4 hi = make_uint4(to_f16(v[i].z), to_f16(v[i].z >> 16), to_f16(v[i].w), to_f16(v[i].w >> 16));
            uint8_t* r = dst + (i0 + i) * kRowStep * 128;  // (a multiple of eight rows on: the same swizzle)
            *reinterpret_cast<uint4*>(r + to0) = lo;
            *reinterpret_cast<uint4*>(r + to1) = hi;
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bFull + 8 * ch);
          mbar_arrive(bREmpty + 8 * rc);
        }
      }
    }
    if (!ok && lane == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
  } else if (warp >= kCSoftmaxWarps) {
    regs_leave<Q8 ? kQ8OtherRegs : kCOtherRegs>();
    if (warp == kCProducerWarp) {
      // ======================= producer =======================
      asm volatile("griddepcontrol.wait;" ::: "memory");
      PlanBlock mine[2];
      const PlanHead head = A.blocks ? *A.head : warp_plan(A.plan, mine);
      const Blocks blocks{A.blocks, mine, head.blocks};
      const int c = blockIdx.x;
      // the whole items first, in step; the items from n_whole on are cut by cost
      const long long all = (long long)A.Hkv * head.tiles;
      const int n_whole = head.waves * (int)gridDim.x;
      FixedCost fixed = A.fixed;
      auto place_of_item = [&](int id) {
        Place p;
        p.e = id / A.Hkv;
        p.kvh = id - p.e * A.Hkv;
        p.tile = 0;
        p.before = all;
        if (p.e < head.blocks) {
          const PlanBlock b = blocks.at(p.e);
          p.before = (long long)A.Hkv * b.tiles_before + (long long)p.kvh * b.n_tiles;
        }
        return p;
      };
      Place first_cut{};
      if (n_whole) first_cut = place_of_item(n_whole);
      const long long tiles = all - first_cut.before;  // to be cut
      int G = (int)gridDim.x;
      if (tiles < G) G = (int)tiles;
      if (tiles > 0) {  // (a CTA with few tiles would get none if a block's fixed cost were several)
        const int most = (int)min(1ll << 20, quotient(tiles, 4 * (long long)G));
        fixed.one = min(fixed.one, most);
        fixed.pair = min(fixed.pair, most - fixed.one);
      }
      const long long x_all = (long long)A.Hkv * (head.tiles + (long long)fixed.one * head.blocks +
                                                  (long long)fixed.pair * head.pairs);
      long long x_cut = 0;
      if (n_whole && first_cut.e < head.blocks) {
        const PlanBlock p = blocks.at(first_cut.e);
        x_cut = (long long)A.Hkv * weight_before(p, first_cut.e, fixed) +
                (long long)first_cut.kvh * (p.n_tiles + fixed_of(p, g, fixed));
      }
      const long long W = tiles > 0 ? x_all - x_cut : 0;
      Place at{};
      long long left = 0;  // the CTA's tiles of the cut part
      if (c < G) {
        // where its share ends, then where it starts (one copy of the code: each line of it is a first fetch)
        long long end = all;
#pragma unroll 1
        for (int k = 1; k >= 0; --k) {
          const long long x = x_cut + quotient((c + k) * W, G);
          if (x < x_all) at = find_place(x, blocks, A.Hkv, g, fixed);
          if (k && x < x_all) end = at.before;
        }
        left = end - at.before;
      }
      int whole = head.waves;  // whole items still to do
      if (whole == 0 && left <= 0 && lane == 0) {
        info[0].last = 2;
        mbar_arrive(bIFull);
      }
      // a lane's piece of a K or V tile: keys [row, row + piece) of the tile, columns [64 hb, 64 hb + 64)
      const int per_tile = kCKeys / A.piece;
      const int my_row = (lane % per_tile) * A.piece, my_hb = lane / per_tile;
      const bool has_piece = my_hb < (Q8 ? 1 : SM::kBoxes);  // (in 8 bits a box holds whole rows)
      uint32_t item_ctr = 0, chunk_ctr = 0, gap_ctr = 0;
      uint32_t n_k = 0;
      const uint64_t once = evict_first_policy(), again = evict_normal_policy();
      bool ok = true;
      while ((whole > 0 || left > 0) && ok) {
        const bool cut = whole == 0;
        const Place pl = cut ? at : place_of_item((head.waves - whole) * (int)gridDim.x + c);
        const PlanBlock p = blocks.at(pl.e);
        ChunkItem it{};
        it.b = p.b;
        it.kvh = pl.kvh;
        it.tok0 = p.tok0;
        it.pos0 = p.pos0;
        it.rows = p.n_tok * g;
        it.pair = p.n_tok > Rt;
        it.tile0 = p.tile0 + pl.tile;
        it.sink = SINK ? p.sink << 16 | max(p.sink - pl.tile, 0) : 0;
        it.gaps = p.gaps ? pl.e : -1;
        it.n_tiles = cut ? (int)min((long long)(p.n_tiles - pl.tile), left) : p.n_tiles;
        it.klo = p.klo;
        it.khi = p.khi;
        it.partial = it.n_tiles != p.n_tiles;
        it.slot = pl.tile == 0 ? 2 * c + 1 : 2 * c;
        it.c0 = c;
        it.np = 1;
        if (it.partial) {
          const int fc = fixed_of(p, g, fixed);
          // of the block's first tile, from the cut part's start
          const long long y = (long long)A.Hkv * weight_before(p, pl.e, fixed) +
                              (long long)pl.kvh * (p.n_tiles + fc) + fc - x_cut;
          it.c0 = share_of(y, W, G);
          it.np = share_of(y + p.n_tiles - 1, W, G) - it.c0 + 1;
        }
        if (cut) left -= it.n_tiles;
        else --whole;
        it.last = whole == 0 && left <= 0;
        const int n = it.n_tiles, lag = it.pair ? 2 : 3;
        // keys of a sequence that has one block are read once per kv head
        const int n_new = A.cu_new[p.b + 1] - A.cu_new[p.b];
        const uint64_t policy = n_new <= 2 * Rt ? once : again;
        const bool gaps = (SHAPE & kDocs) && p.gaps;
        const uint32_t* seen = A.seen + (size_t)pl.e * kSeenWords;  // (if it has gaps)
        // pages of the item's tiles, four tiles at a time: lane 8 k + i holds that of piece i of the k-th (kNoPage: no
        // row of a block with gaps sees the piece)
        const int sinks = SINK ? min(A.mask.sinks, p.khi) : 0;
        auto load_pages = [&](int group) {
          if (!A.block_table && !gaps) return p.b;
          const int tile = 4 * group + lane / 8, i = lane % 8;
          const int key = item_tile<SINK>(it, tile_of<SHAPE>(tile, n)) * kCKeys + i * A.piece;
          if (tile >= n || i >= per_tile || key >= p.khi || (key + A.piece <= p.klo && key >= sinks)) return 0;
          if (gaps) {
            if (!some_row_sees(seen, p.pos0, p.n_tok, max(key, p.klo), min(key + A.piece, p.khi))) return kNoPage;
            if (!A.block_table) return p.b;
            return max(-1, __ldg(A.block_table + (size_t)p.b * A.max_pages + key / A.page_size));
          }
          return __ldg(A.block_table + (size_t)p.b * A.max_pages + key / A.page_size);
        };
        int pages_before = 0, pages = load_pages(0), pages_next = load_pages(1);
        // the item's queries, once the item before has issued its last S
        ok = warp_wait(bIEmpty + 8 * (item_ctr & 1), ((item_ctr >> 1) & 1) ^ 1) &&
             warp_wait(bQEmpty, (item_ctr & 1) ^ 1);
        if (!ok) break;
        if (lane == 0) {
          info[item_ctr & 1] = it;
          mbar_arrive(bIFull + 8 * (item_ctr & 1));
          mbar_expect_tx(bQFull, (it.pair ? 2 : 1) * R * D * 2);
          for (int s = 0; s <= it.pair; ++s)
            for (int hb = 0; hb < SM::kBoxes; ++hb)
              tma_load_3d(sQ + s * SM::kTile + hb * 16384, &A.Q, bQFull, hb * 64, it.kvh * g, it.tok0 + s * Rt);
        }
        __syncwarp();
        // chunks in the order in which the MMA warp uses them: K of tile t, then V of tile t - lag + 1
        for (int kt = 0, vt = 0; vt < n && ok;) {
          const bool is_k = kt < n && kt < vt + lag;
          const int t = is_k ? kt++ : vt++;
          // (in 8 bits K and V have rings of their own; n_k: the tiles of K loaded so far)
          const uint32_t nth = !Q8 ? chunk_ctr : is_k ? n_k++ : chunk_ctr - n_k;
          const uint32_t size = !Q8 ? SM::kChunks : is_k ? SM::kKs : SM::kRaws;
          const uint32_t ch = nth % size;
          ok = warp_wait((!Q8 ? bEmpty : is_k ? bKEmpty : bREmpty) + 8 * ch, ((nth / size) & 1) ^ 1);
          if (!ok) break;
          if (is_k && t > 0 && (t & 3) == 0) {
            pages_before = pages;
            pages = pages_next;
            pages_next = load_pages((t >> 2) + 1);
          }
          const int from = t >> 2 == (kt - 1) >> 2 ? pages : pages_before;  // kt - 1: the last K tile
          int page = __shfl_sync(0xffffffffu, from, (t & 3) * 8 + lane % per_tile);
          const int key = item_tile<SINK>(it, tile_of<SHAPE>(t, n)) * kCKeys + my_row;
          const bool load = has_piece && key < p.khi && (key + A.piece > p.klo || key < sinks) && !(gaps && page == kNoPage);
          if (A.block_table && load && (page < 0 || page >= A.n_pages)) {
            raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
            page = 0;  // a valid page; the sequence's output is then meaningless
          }
          // Rows of V within the block's range that no row sees are cleared before the chunk counts as filled. (Here
          // and not by the softmax warps, who clear those outside the range: with this in their loop, and in kernels
          // for calls without first keys, a prompt of 64-wide heads took 871 us instead of 812.)
          const int kt0 = key - my_row;
          const bool gap = !Q8 && gaps && !is_k && kt0 + kCKeys > p.pos0 && kt0 < p.pos0 + p.n_tok;
          const uint32_t bar = gap ? bGap : (!Q8 ? bFull : is_k ? bKFull : bRFull) + 8 * ch;
          const int pieces = __popc(__ballot_sync(0xffffffffu, load));
          if (lane == 0) mbar_expect_tx(bar, pieces * A.piece * (Q8 ? D : 128));
          __syncwarp();
          if (load) {
            const int z = page * A.Hkv + it.kvh, y = A.block_table ? key % A.page_size : key;
            const uint32_t to = Q8 ? (is_k ? sK : sRaw) + ch * SM::kRawTile + my_row * D
                                   : sRing + ch * SM::kTile + my_hb * 16384 + my_row * 128;
            tma_load_3d_hint(to, is_k ? &A.K : &A.V, bar, my_hb * 64, y, z, policy);
          }
          if (gap) {
            ok = warp_wait(bGap, gap_ctr++ & 1);
            for (int r = lane; r < kCKeys && ok; r += 32) {
              const int k = kt0 + r;
              if (k < p.klo || k >= p.khi || some_row_sees(seen, p.pos0, p.n_tok, k, k + 1)) continue;
              for (int u = 0; u < SM::kBoxes * 8; ++u)
                reinterpret_cast<uint4*>(smem + SM::kRing + ch * SM::kTile + u / 8 * 16384 + r * 128)[u % 8] =
                    make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bFull + 8 * ch);
          }
          ++chunk_ctr;
        }
        ++item_ctr;
        if (cut) {  // the next item: the next kv head, or the next block
          at.tile = 0;
          if (++at.kvh == A.Hkv) {
            at.kvh = 0;
            ++at.e;
          }
        }
      }
      if (!ok && lane == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
      // before leaving, wait (bounded) for the copies still in flight
      if (lane == 0) {
        auto drain = [&](uint32_t bars, uint32_t size, uint32_t count) {
          for (uint32_t k = 0; k < size && k < count; ++k) mbar_wait(bars + 8 * ((count - 1 - k) % size), ((count - 1 - k) / size) & 1);
        };
        if constexpr (Q8) {
          drain(bKFull, SM::kKs, n_k);
          drain(bRFull, SM::kRaws, chunk_ctr - n_k);
        } else {
          drain(bFull, SM::kChunks, chunk_ctr);
        }
        if (item_ctr > 0) mbar_wait(bQFull, (item_ctr - 1) & 1);
      }
      __syncwarp();
    } else if (warp == kCMmaWarp) {
      // ======================= MMA issue =======================
      // The whole warp walks the steps, one elected lane issues.
      uint32_t item_ctr = 0;
      uint32_t ch = 0, ch_par = 0;             // the next chunk and its parity
      uint32_t g0 = 0, g1 = 0;                 // words heard from the streams
      uint32_t o0 = 1, o1 = 1;                 // parities: their accumulators are free
      bool ok = true;
      // (a wait that gives up is noticed at the next tile; what is issued until then stays within the CTA's memory)
      auto need = [&](uint32_t bar, uint32_t parity) {
        if (!__all_sync(0xffffffffu, mbar_try_wait(bar, parity)))
          ok = __all_sync(0xffffffffu, ok && slow_wait(bar, parity));
      };
      auto next_of = [&](uint32_t bars, uint32_t& at, uint32_t& par, uint32_t size) {
        const uint32_t c = at;
        need(bars + 8 * c, par);
        if (++at == size) {
          at = 0;
          par ^= 1;
        }
        return c;
      };
      uint32_t kch = 0, kch_par = 0;  // (8 bits) the next tile of K
      // the next chunk of V, or of K, once it is filled
      auto take = [&]() { return next_of(bFull, ch, ch_par, SM::kChunks); };
      auto take_k = [&]() {
        if constexpr (Q8) return next_of(bKFull, kch, kch_par, SM::kKs);
        else return take();
      };
      auto free_k = [&](uint32_t c) { mma_commit_warp((Q8 ? bKEmpty : bEmpty) + 8 * c); };
      auto word = [&](int s, uint32_t& w) {
        need(bGot + 16 * s + 8 * (w & 1), (w >> 1) & 1);
        ++w;
      };
      const uint32_t k_desc = desc_lo(sRing, 16), v_desc = desc_lo(sRing, 16384), q_desc = desc_lo(sQ, 16);
      auto issue_s = [&](int s, int qs, uint32_t c) {  // S = Q K^T
        constexpr uint32_t idesc = mma_idesc(128, kCKeys, 0) & ~(Q8 ? kBf16Operands : 0u);
        const uint32_t ts = tmem + SM::kColS + (SM::kScores == 2 ? s * 128 : 0);
        tc_fence_after();
        const uint32_t qa = q_desc + qs * (SM::kTile / 16);
        if constexpr (Q8) {  // both parts of Q's 64 columns at a time
          const uint32_t ka = desc_lo(sK, 16) + c * (SM::kRawTile / 16);
#pragma unroll
          for (int hb = 0; hb < SM::kBoxes; ++hb)
            mma_f8_ss4_warp<D == 64>(ts, qa + hb * 1024, ka + hb * 4, idesc, hb != 0 ? 1u : 0u);
        } else {
          const uint32_t ka = k_desc + c * (SM::kTile / 16);
#pragma unroll
          for (int hb = 0; hb < SM::kBoxes; ++hb)
            mma_ss4_warp<32, 32>(ts, qa + hb * 1024, ka + hb * 1024, idesc, hb != 0 ? 1u : 0u);
        }
        mma_commit_warp(bSFull + 8 * s);
      };
      auto issue_pv = [&](int s, uint32_t c, uint32_t acc) {  // O += P V
        constexpr uint32_t idesc = mma_idesc(128, D, 1) & ~(Q8 ? kBf16Operands : 0u);
        const uint32_t va = v_desc + c * (SM::kTile / 16);
        const uint32_t d = tmem + SM::kColO + s * D, tp = tmem + SM::kColP + s * 64;
        tc_fence_after();
        mma_ts4_warp<2048>(d, tp, va, idesc, acc);
        mma_ts4_warp<2048>(d, tp + 32, va + 512, idesc, 1u);
        mma_commit_warp(bPVDone + 8 * s);
      };
      for (int last = 0; !last && ok; ++item_ctr) {
        need(bIFull + 8 * (item_ctr & 1), (item_ctr >> 1) & 1);
        if (!ok) break;
        const int n_tiles = __shfl_sync(0xffffffffu, info[item_ctr & 1].n_tiles, 0);
        const bool pair = __shfl_sync(0xffffffffu, info[item_ctr & 1].pair, 0);
        last = __shfl_sync(0xffffffffu, info[item_ctr & 1].last, 0);
        if (last == 2) break;
        if (lane == 0) mbar_arrive(bIEmpty + 8 * (item_ctr & 1));
        __syncwarp();
        need(bQFull, item_ctr & 1);
        // One word from a stream for each of its tiles, and one more: the tile's scores are in registers, and P of the
        // tile before is written. Behind it go the next S into the place that it left (D = 64: the stream's own next
        // tile; D = 128: the other stream's) and that PV. Chunks are asked for before the word. (Words lie on two
        // barriers in turn: the last two of an item may be there before the first of them is heard, and a warp may be
        // at the second while another has yet to say the first.)
        // (A warp by itself takes 5 cycles for an instruction that depends on another, and 150 to 400 for an ask of a
        // barrier beside MMAs that read shared memory at its full rate: every one of them counts here.)
        constexpr bool kOwn = SM::kScores == 2;
        uint32_t kc = take_k(), vc = 0;
        if (pair) {
          issue_s(0, 0, kc);
          if (kOwn) {
            issue_s(1, 1, kc);
            free_k(kc);
            if (n_tiles == 1) mma_commit_warp(bQEmpty);
          }
          for (int t = 0; t <= n_tiles && ok; ++t) {
            if (t > 0) vc = take();
            if (t == 1) {
              need(bOFree, o0);
              need(bOFree + 8, o1);
              o0 ^= 1;
              o1 ^= 1;
            }
            if (kOwn && t + 1 < n_tiles) kc = take_k();
            word(0, g0);
            if (kOwn) {
              if (t + 1 < n_tiles) issue_s(0, 0, kc);
            } else if (t < n_tiles) {
              issue_s(1, 1, kc);
              free_k(kc);
              if (t == n_tiles - 1) mma_commit_warp(bQEmpty);
            }
            if (t > 0) issue_pv(0, vc, t > 1);
            if (!kOwn && t + 1 < n_tiles) kc = take_k();
            word(1, g1);
            if (t + 1 < n_tiles) {
              if (kOwn) {
                issue_s(1, 1, kc);
                free_k(kc);
                if (t == n_tiles - 2) mma_commit_warp(bQEmpty);
              } else {
                issue_s(0, 0, kc);
              }
            }
            if (t > 0) {
              issue_pv(1, vc, t > 1);
              mma_commit_warp(bEmpty + 8 * vc);
            }
          }
        } else {
          auto next_s = [&](int n) {
            issue_s(n & 1, 0, kc);
            free_k(kc);
            if (n == n_tiles - 1) mma_commit_warp(bQEmpty);
          };
          next_s(0);
          for (int n = 0; n < n_tiles + 2 && ok; ++n) {  // stream n & 1 has tile n
            const int s = n & 1;
            if (n >= 2) vc = take();
            if (n == 2 || n == 3) {
              need(bOFree + 8 * s, s ? o1 : o0);
              if (s) o1 ^= 1;
              else o0 ^= 1;
            }
            if (n < n_tiles || n >= 2) {
              if (s) word(1, g1);
              else word(0, g0);
            }
            if (n >= 2) {
              issue_pv(s, vc, n >= 4);
              mma_commit_warp(bEmpty + 8 * vc);
            }
            if (n + 1 < n_tiles) {  // (asked for behind the PV, which gives its chunk back while K is on its way)
              kc = take_k();
              next_s(n + 1);
            }
          }
        }
      }
      if (!ok && lane == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
      // every MMA issued has completed before the tensor memory is released
      mma_commit_warp(bDrain);
      warp_wait(bDrain, 0);
    } else if (Q8 && warp == kScaleWarp) {
      // ======================= scales of the tiles =======================
      // Lane 8 k + i has those of the i-th 16 keys of the k-th of four tiles; the next four are on their way meanwhile.
      asm volatile("griddepcontrol.wait;" ::: "memory");
      const int i = lane & 7;
      uint32_t item_ctr = 0, ctr[2] = {0, 0};
      bool ok = true;
      for (int last = 0; !last && ok; ++item_ctr) {
        ok = warp_wait(bIFull + 8 * (item_ctr & 1), (item_ctr >> 1) & 1);
        if (!ok) break;
        const ChunkItem it = info[item_ctr & 1];
        last = it.last;
        if (last == 2) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(bIEmpty + 8 * (item_ctr & 1));
        const int n = it.n_tiles, sinks = SINK ? min(A.mask.sinks, it.khi) : 0, per = A.rows >> A.block_log2;
        auto load = [&](int t0) {  // exponents of K (low byte) and V
          const int t = t0 + lane / 8;
          const uint32_t none = 127u | 127u << 8;
          if (t >= n) return none;
          const int key = item_tile<SINK>(it, tile_of<SHAPE>(t, n)) * kCKeys + 16 * i;
          if (key >= it.khi || (key + 16 <= it.klo && key >= sinks)) return none;
          // (within, first keys may hide the 16 from all rows: whatever lies there then, any scale will do)
          int plane = it.b, row = key;
          if (A.block_table) {
            plane = __ldg(A.block_table + (size_t)it.b * A.max_pages + key / A.page_size);
            if (plane < 0 || plane >= A.n_pages) plane = 0;  // (the producer reports it if the page is read)
            row = key % A.page_size;
          }
          const size_t at = ((size_t)plane * A.Hkv + it.kvh) * per + (row >> A.block_log2);
          const uint32_t ek = min(max((int)__ldg(A.Ks + at), 67), 187), ev = min(max((int)__ldg(A.Vs + at), 67), 187);
          return ek | ev << 8;
        };
        uint32_t now = load(0);
        for (int t0 = 0; t0 < n && ok; t0 += 4) {
          const uint32_t next = load(t0 + 4);
          for (int k = 0; k < 4 && t0 + k < n && ok; ++k) {
            for (int s = 0; s < 2 && ok; ++s) {
              if (!it.pair && s != ((t0 + k) & 1)) continue;
              // once the stream has read those of its tile before (two arrivals could else make one phase of bSFull)
              const uint32_t c = s ? ctr[1]++ : ctr[0]++;
              ok = warp_wait(bCEmpty + 8 * s, (c & 1) ^ 1);
              if (!ok) break;
              if (lane / 8 == k) {
                TileScales* to = reinterpret_cast<TileScales*>(smem + SM::kScales) + s;
                to->k[i] = power_of_two_biased(now & 0xffu);
                to->v_log2[i] = __int2half_rn((int)(now >> 8) - 127);
              }
              __syncwarp();
              if (lane == 0) mbar_arrive(bSFull + 8 * s);
            }
          }
          now = next;
        }
      }
      if (!ok && lane == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
    }
  } else {
    regs_take<Q8 ? kQ8SoftmaxRegs : kCSoftmaxRegs>();
    // ======================= softmax warpgroups =======================
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int st = warp >> 2, wq = warp & 3;
    const int row = wq * 32 + lane;  // tensor-memory lane
    const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
    const uint32_t ts = tmem + lane_off + SM::kColS + (SM::kScores == 2 ? st * 128 : 0);
    const uint32_t tp = tmem + lane_off + SM::kColP + st * 64;
    const uint32_t to = tmem + lane_off + SM::kColO;
    float2* stat = reinterpret_cast<float2*>(smem + SM::kStat);  // [stream][128]
    const float scale_log2 = A.scale * kLog2e;
    // The quarter of a tile's keys whose probabilities are the first to be written, with those before them: by then the
    // PV that reads the tile before's should be done. (At D = 128 it comes behind an S of the other stream: 16384
    // tokens of 8 heads over as many keys 960 us at 3, 969 at 2, 1004 at 1; at D = 64, 816 at 1, 827 at 0, 934 at 3.)
    constexpr int kFirstP = D == 64 ? 1 : 3;
    uint32_t item_ctr = 0, chunk_base = 0;
    uint32_t words = 0;             // of this stream in the items before this one
    uint32_t done0 = 0, done1 = 0;  // steps of streams 0 and 1 in the items before this one
    bool ok = true;
    // A wait that fails leaves `ok` false; the item is then finished without further waits, so that every thread
    // still reaches every named barrier.
    auto wait = [&](uint32_t bar, uint32_t parity) { ok = ok && warp_wait(bar, parity); };
    for (int last = 0; !last;) {
      wait(bIFull + 8 * (item_ctr & 1), (item_ctr >> 1) & 1);
      if (bar_any<kCAllBar, kCSoftmaxWarps * 32>(!ok)) {
        ok = false;
        break;
      }
      const ChunkItem& it = info[item_ctr & 1];
      last = it.last;
      if (last == 2) break;
      const bool pair = it.pair;
      const int n_tiles = it.n_tiles;
      const int steps0 = pair ? n_tiles : (n_tiles + 1) >> 1, steps1 = pair ? n_tiles : n_tiles >> 1;
      const int my_steps = st ? steps1 : steps0;
      const int rr = (pair ? st * R : 0) + row;  // row of the block
      const bool valid = row < R && rr < it.rows;
      const bool warp_live = wq * 32 < R && (pair ? st * R : 0) + wq * 32 < it.rows;
      const int tok = it.tok0 + rr / g, hq = it.kvh * g + rr % g, pos = it.pos0 + rr / g;
      int lo = 0, hi = 0;
      float slope = 0.f;
      if (valid) {
        const int n_keys = A.kv_len[it.b] + A.cu_new[it.b + 1] - A.cu_new[it.b];
        row_range(pos, n_keys, A.mask.prefix_len ? A.mask.prefix_len[it.b] : 0,
                  A.mask.first_key ? A.mask.first_key[tok] : 0, A.mask.window, lo, hi);
        if (SHAPE & kBias) slope = A.slopes[hq] * kLog2e;
      }
      float unscale = 1.f;  // of the row's Q
      if constexpr (Q8) {
        if (valid) {
          const uint32_t e = __ldcg(A.q_exp + (size_t)tok * A.Hq + hq);
          unscale = e == kInfiniteRow ? INFINITY : power_of_two_biased(254u - e);
        }
      }
      const float sc = SHAPE & (kCap | kBias) ? 1.f : scale_log2 * unscale;
      const int sinks = SINK ? min(A.mask.sinks, hi) : 0;  // (the row's)
      const float cap2 = A.cap.log2, u2 = A.cap.twice_inverse;
      float m_run = -INFINITY, l_run = 0.f;
      for (int i = 0; i < my_steps; ++i) {
        const int j = pair ? i : 2 * i + st;  // the item's tile
        const int kt0 = item_tile<SINK>(it, tile_of<SHAPE>(j, n_tiles)) * kCKeys;
        const uint32_t n = (st ? done1 : done0) + i;
        wait(bSFull + 8 * st, n & 1);
        float k_scale[8] = {};
        uint32_t v_exps[4] = {};
        if constexpr (Q8) {
          const float4* from = reinterpret_cast<const float4*>(smem + SM::kScales + st * 48);
          const float4 a = from[0], b = from[1], c = from[2];
          k_scale[0] = a.x, k_scale[1] = a.y, k_scale[2] = a.z, k_scale[3] = a.w;
          k_scale[4] = b.x, k_scale[5] = b.y, k_scale[6] = b.z, k_scale[7] = b.w;
          v_exps[0] = __float_as_uint(c.x), v_exps[1] = __float_as_uint(c.y);
          v_exps[2] = __float_as_uint(c.z), v_exps[3] = __float_as_uint(c.w);
          __syncwarp();
          if (lane == 0) mbar_arrive(bCEmpty + 8 * st);
        }
        if (!Q8 && (kt0 < it.klo || kt0 + kCKeys > it.khi)) {
          // V rows that no row of the block sees: cleared once they have landed. (Asked after S: a wait on a parity
          // may be one phase ahead of the barrier, not two, and the MMA warp has by now taken every chunk that lay
          // in this place of the ring before.)
          const uint32_t ci = chunk_base + j + min(j + (pair ? 2 : 3), n_tiles);
          const uint32_t ch = ci % SM::kChunks;
          wait(bFull + 8 * ch, (ci / SM::kChunks) & 1);
          const int key = kt0 + row;
          if (ok && (key >= it.khi || (key < it.klo && !(SINK && key < A.mask.sinks)))) {
#pragma unroll
            for (int hb = 0; hb < SM::kBoxes; ++hb) {
              uint4* v = reinterpret_cast<uint4*>(smem + SM::kRing + ch * SM::kTile + hb * 16384 + row * 128);
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] = make_uint4(0, 0, 0, 0);
            }
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        if (!warp_live) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bGot + 16 * st + 8 * ((words + i) & 1));
          continue;
        }
        tc_fence_after();
        uint32_t x[4][32];
#pragma unroll
        for (int q = 0; q < 4; ++q) tmem_ld32(ts + 32 * q, x[q]);
        tmem_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bGot + 16 * st + 8 * ((words + i) & 1));
        if constexpr (Q8 && (SHAPE & (kCap | kBias))) {
#pragma unroll
          for (int gr = 0; gr < 8; ++gr) {
            const float f = k_scale[gr] * unscale;
#pragma unroll
            for (int c = 0; c < 16; ++c)
              x[gr / 2][gr % 2 * 16 + c] = __float_as_uint(__uint_as_float(x[gr / 2][gr % 2 * 16 + c]) * f);
          }
        }
        if constexpr (SHAPE & kCap) {  // the scores in units of log 2
          bool series = false;  // all of the warp's scores are small beside the cap
          if constexpr (SHAPE & kWideCap) {
            float top = 0.f;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int c = 0; c < 32; ++c) top = fmaxf(top, fabsf(__uint_as_float(x[q][c])));
            series = !__any_sync(0xffffffffu, valid && top * A.cap.inverse > kSeriesTop);
            if (series) {
#pragma unroll
              for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int c = 0; c < 32; ++c)
                  x[q][c] = __float_as_uint(cap_series(__uint_as_float(x[q][c]), scale_log2, A.cap.inverse));
            }
          }
          // cap tanh(s / cap) = cap (1 - 2 / (e + 1)), e = exp(2 s / cap)
          if (!series) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int c = 0; c < 32; c += 2) {
                float a, b;
                fma2(a, b, __uint_as_float(x[q][c]), __uint_as_float(x[q][c + 1]), u2, 0.f);
                a = ex2_approx(a);
                b = ex2_approx(b);
                add2(a, b, 1.f, 1.f);
                a = rcp_approx(a);
                b = rcp_approx(b);
                if constexpr (SHAPE & kWideCap) {
                  a = wide_cap(__uint_as_float(x[q][c]), a, scale_log2, A.cap);
                  b = wide_cap(__uint_as_float(x[q][c + 1]), b, scale_log2, A.cap);
                } else {
                  fma2(a, b, a, b, -2.f * cap2, cap2);
                }
                x[q][c] = __float_as_uint(a);
                x[q][c + 1] = __float_as_uint(b);
              }
          }
        }
        if constexpr (SHAPE & kBias) {
          const float to_log2 = SHAPE & kCap ? 1.f : scale_log2, d0 = (float)(kt0 - pos);
          if (__any_sync(0xffffffffu, valid && kt0 + kCKeys - 1 > pos)) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int c = 0; c < 32; ++c)
                x[q][c] = __float_as_uint(
                    fmaf(__uint_as_float(x[q][c]), to_log2, -slope * fabsf(d0 + (float)(32 * q + c))));
          } else {  // no key lies ahead: |p - k| = p - k
            const float b0 = slope * d0;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
              for (int c = 0; c < 32; c += 2) {
                float y0, y1;
                fma2v(y0, y1, __uint_as_float(x[q][c]), __uint_as_float(x[q][c + 1]), to_log2,
                      fmaf(slope, (float)(32 * q + c), b0), fmaf(slope, (float)(32 * q + c + 1), b0));
                x[q][c] = __float_as_uint(y0);
                x[q][c + 1] = __float_as_uint(y1);
              }
          }
        }
        if (__any_sync(0xffffffffu, valid && (kt0 < lo || kt0 + kCKeys > hi))) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            uint32_t seen = bits_below(hi - kt0 - 32 * q) & ~bits_below(lo - kt0 - 32 * q);
            if (SINK) seen |= bits_below(sinks - kt0 - 32 * q);
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (!((seen >> c) & 1u)) x[q][c] = __float_as_uint(-INFINITY);
          }
        }
        float cmax;
        // (not zero: a masked score stays minus infinity)
        auto group_scale = [&](int gr) { return SHAPE & (kCap | kBias) ? 1.f : fmaxf(sc * k_scale[gr], kFloatMin); };
        auto v_log2 = [&](int gr) {
          const __half2 two = *reinterpret_cast<const __half2*>(&v_exps[gr / 2]);
          return gr % 2 ? __high2float(two) : __low2float(two);
        };
        if constexpr (Q8) {
          // the largest term of O's sum: P times its value's scale. (Behind the mask: what a row does not see has no
          // part in its reference.)
          cmax = -INFINITY;
#pragma unroll
          for (int gr = 0; gr < 8; ++gr) {
            const uint32_t* y = x[gr / 2] + gr % 2 * 16;
            float m = __uint_as_float(y[0]);
#pragma unroll
            for (int c = 1; c < 15; c += 2) m = fmaxf(fmaxf(m, __uint_as_float(y[c])), __uint_as_float(y[c + 1]));
            m = fmaxf(m, __uint_as_float(y[15]));
            cmax = fmaxf(cmax, fmaf(m, group_scale(gr), v_log2(gr)));
          }
          cmax = valid ? cmax : 0.f;
        } else {
          float mx[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            mx[q] = __uint_as_float(x[q][0]);
#pragma unroll
            for (int c = 1; c < 31; c += 2)
              mx[q] = fmaxf(fmaxf(mx[q], __uint_as_float(x[q][c])), __uint_as_float(x[q][c + 1]));
            mx[q] = fmaxf(mx[q], __uint_as_float(x[q][31]));
          }
          // (a lane past the block's rows holds scores of whatever its Q row is: it asks for no raise)
          cmax = valid ? fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sc : 0.f;
        }
        if (cmax != cmax) cmax = 0.f;  // nothing but NaN: the row's sum is NaN whatever the reference
        if (Q8) cmax -= kHeadroomLog2;
        if (i == 0) {
          m_run = cmax;
        } else if (__any_sync(0xffffffffu, cmax > m_run + kCRescaleLog2)) {
          // O and l against the new reference
          const bool raise = cmax > m_run + kCRescaleLog2;
          const float f = !raise ? 1.f : m_run == -INFINITY ? 0.f : ex2_approx(m_run - cmax);
          m_run = raise ? cmax : m_run;
          l_run *= f;
          wait(bPVDone + 8 * st, (n - 1) & 1);
          tc_fence_after();
#pragma unroll 1
          for (int c0 = 0; c0 < D; c0 += 16) {
            uint32_t o[16];
            tmem_ld16(to + st * D + c0, o);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tmem_st16(to + st * D + c0, o);
          }
          tmem_wait_st();
        }
        const float neg_m = m_run == -INFINITY ? 0.f : -m_run;
        float la[2] = {0.f, 0.f}, lb[2] = {0.f, 0.f};
        uint32_t pk[4][16];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if constexpr (Q8) {
#pragma unroll
            for (int gr = 2 * q; gr < 2 * q + 2; ++gr) {
              const float f = group_scale(gr), v = v_log2(gr), to = neg_m + v;
              // 2^-v: 1.5 2^23 - v has -v in its lowest bits
              const float inv = __uint_as_float((__float_as_uint(12582912.f - v) << 23) + 0x3f800000u);
              float ga[2], gb[2];  // sums of P times V's scale
#pragma unroll
              for (int c = gr % 2 * 16; c < gr % 2 * 16 + 16; c += 4) {
                float y0, y1, y2, y3;
                fma2(y0, y1, __uint_as_float(x[q][c]), __uint_as_float(x[q][c + 1]), f, to);
                fma2(y2, y3, __uint_as_float(x[q][c + 2]), __uint_as_float(x[q][c + 3]), f, to);
                y0 = ex2_approx(y0);
                y1 = ex2_approx(y1);
                y2 = ex2_approx(y2);
                y3 = ex2_approx(y3);
                if (c % 16 == 0) {
                  ga[0] = y0, ga[1] = y1, gb[0] = y2, gb[1] = y3;
                } else {
                  add2(ga[0], ga[1], y0, y1);
                  add2(gb[0], gb[1], y2, y3);
                }
                pk[q][c >> 1] = pack_f16(y0, y1);
                pk[q][(c >> 1) + 1] = pack_f16(y2, y3);
              }
              add2(ga[0], ga[1], gb[0], gb[1]);
              fma2v(la[0], la[1], ga[0], ga[1], inv, la[0], la[1]);
            }
          } else {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              float y0, y1, y2, y3;
              fma2(y0, y1, __uint_as_float(x[q][c]), __uint_as_float(x[q][c + 1]), sc, neg_m);
              fma2(y2, y3, __uint_as_float(x[q][c + 2]), __uint_as_float(x[q][c + 3]), sc, neg_m);
              y0 = ex2_approx(y0);
              y1 = ex2_approx(y1);
              y2 = ex2_approx(y2);
              y3 = ex2_approx(y3);
              add2(la[0], la[1], y0, y1);
              add2(lb[0], lb[1], y2, y3);
              pk[q][c >> 1] = c_pack(y0, y1);
              pk[q][(c >> 1) + 1] = c_pack(y2, y3);
            }
          }
          if (q == kFirstP) {
            if (i > 0) {  // the PV before has read P
              wait(bPVDone + 8 * st, (n - 1) & 1);
              tc_fence_after();
            }
#pragma unroll
            for (int k = 0; k <= q; ++k) tmem_st16(tp + 16 * k, pk[k]);
          } else if (q > kFirstP) {
            tmem_st16(tp + 16 * q, pk[q]);
          }
        }
        tmem_wait_st();
        l_run += (la[0] + la[1]) + (lb[0] + lb[1]);
      }
      if (my_steps > 0) {  // the last P
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bGot + 16 * st + 8 * ((words + my_steps) & 1));
        words += my_steps + 1;
      }
      // ---- epilogue ----
      float f0 = 1.f, f1 = 0.f;  // factors of the streams' O
      const bool both = !pair && steps1 > 0;  // the streams hold keys of the same rows
      if (both) {
        float2 a, b;  // of streams 0 and 1
        if constexpr (Q8) {  // (through one place for each row, in turns)
          a = b = make_float2(m_run, l_run);
          if (warp_live && st == 1) stat[row] = b;
          bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
          if (warp_live && st == 0) {
            b = stat[row];
            stat[row] = a;
          }
          bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
          if (warp_live && st == 1) a = stat[row];
        } else {
          if (warp_live) stat[st * kCRows + row] = make_float2(m_run, l_run);
          bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
          if (warp_live) {
            a = stat[row];
            b = stat[kCRows + row];
          }
        }
        if (warp_live) {
          const float M = fmaxf(a.x, b.x);
          f0 = M == -INFINITY ? 0.f : ex2_approx(a.x - M);
          f1 = M == -INFINITY ? 0.f : ex2_approx(b.x - M);
          m_run = M;
          l_run = f0 * a.y + f1 * b.y;
        }
      }
      if (pair) {
        wait(bPVDone + 8 * st, ((st ? done1 : done0) + my_steps - 1) & 1);
      } else {
        wait(bPVDone, (done0 + steps0 - 1) & 1);
        if (both) wait(bPVDone + 8, (done1 + steps1 - 1) & 1);
      }
      tc_fence_after();
      // of rows in two streams each warpgroup writes half of the columns; a single step leaves all to the first
      if (warp_live && (pair || both || st == 0)) {
        const bool partial = it.partial;
        const size_t prow = (size_t)it.slot * kCBlockRows + rr;
        if (!partial) {
          const float inv = l_run > 0.f ? 1.f / l_run : l_run == 0.f ? 0.f : l_run;  // (NaN stays)
          f0 *= inv;
          f1 *= inv;
        }
        const uint32_t oa = to + (pair ? st * D : 0);
        const int cb = both ? st * (D / 2) : 0, ce = both ? cb + D / 2 : D;
        __nv_bfloat16* orow = A.O + ((size_t)tok * A.Hq + hq) * D;
#pragma unroll 1
        for (int c0 = cb; c0 < ce; c0 += 32) {
          uint32_t o[32];
          tmem_ld32(oa + c0, o);
          if (both) {
            uint32_t o1[32];
            tmem_ld32(oa + D + c0, o1);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c)
              o[c] = __float_as_uint(fmaf(__uint_as_float(o1[c]), f1, __uint_as_float(o[c]) * f0));
          } else {
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f0);
          }
          if (!valid) continue;
          if (!partial) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              uint32_t r[8];
#pragma unroll
              for (int e = 0; e < 8; ++e)
                r[e] = c_pack(__uint_as_float(o[16 * k + 2 * e]), __uint_as_float(o[16 * k + 2 * e + 1]));
              if (A.o_wide) {
                store32(orow + c0 + 16 * k, r);
              } else {
                reinterpret_cast<uint4*>(orow + c0)[2 * k] = make_uint4(r[0], r[1], r[2], r[3]);
                reinterpret_cast<uint4*>(orow + c0)[2 * k + 1] = make_uint4(r[4], r[5], r[6], r[7]);
              }
            }
          } else {
            uint4* dst = reinterpret_cast<uint4*>(A.part_o) + ((size_t)it.slot * (D / 4) + c0 / 4) * kCBlockRows + rr;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              dst[k * kCBlockRows] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
          }
        }
        if (valid && (pair || st == 0)) {
          if (partial) *reinterpret_cast<float2*>(A.part_ml + prow * 2) = make_float2(m_run, l_run);
          else if (A.lse) A.lse[(size_t)tok * A.Hq + hq] = (m_run + __log2f(l_run)) * kLn2;
        }
      }
      tc_fence_before();
      __syncwarp();
      // a stream's accumulator is free once all that read it have: its own rows' warps, or (combined) both streams'
      if (both) bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
      if (lane == 0 && my_steps > 0) mbar_arrive(bOFree + 8 * st);
      if (it.partial) {
        // counted in once every thread's part is written; the CTA that counts the last merges
        // (the barrier orders the others' stores before this thread's release, and its acquire before their loads)
        bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
        if (tid == 0) {
          uint32_t old;
          asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(old) : "l"(A.count + it.c0) : "memory");
          misc[1] = old == (uint32_t)it.np - 1;
          if (misc[1]) A.count[it.c0] = 0u;
        }
        bar_sync_n(kCAllBar, kCSoftmaxWarps * 32);
        if (misc[1]) {
          if (it.np <= 2) merge_parts<D, 4, 2>(A, it, g);
          else merge_parts<D, 1, 8>(A, it, g);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bIEmpty + 8 * (item_ctr & 1));  // `it` has been read
      done0 += steps0;
      done1 += steps1;
      chunk_base += 2 * n_tiles;
      ++item_ctr;
    }
    if (!ok && lane == 0) raise_status(A.status, LIBRASPEC_ST_TIMEOUT);
  }
  // every role is done with the tensor memory
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == kCMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kCTmemCols) : "memory");
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// A [planes, rows, D] tensor of bf16 in boxes of 64 columns x `box_rows` rows x `box_planes` planes (of dimension 1
// for the queries [T, Hq, D]: box_rows heads of box_planes tokens), 128-byte swizzle.
static bool make_map(CUtensorMap* map, const void* base, int D, long long rows, long long planes, int box_rows,
                     int box_planes, CUtensorMapL2promotion promote) {
  auto enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)rows * D * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_planes};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, promote,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline CapArgs cap_args(float scale, float softcap) {
  return CapArgs{std::min(softcap * kLog2e, kFloatMax), std::min(2.f * (scale * kLog2e) / softcap, kFloatMax),
                 scale / softcap};
}

// Codes of a cache in 8 bits [planes, rows, D] in boxes of whole rows; swizzled for the MMA, or as they are.
static bool make_map8(CUtensorMap* map, const void* base, int D, long long rows, long long planes, int box_rows,
                      bool swizzled) {
  auto enc = get_encode();
  if (!enc) return false;
  cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)D, (cuuint64_t)rows * D};
  cuuint32_t box[3] = {(cuuint32_t)D, (cuuint32_t)box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE,
             !swizzled ? CU_TENSOR_MAP_SWIZZLE_NONE : D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int SHAPE>
static cudaError_t launch_attn_t(const ChunkArgs& a, int grid, cudaStream_t stream) {
  using SM = ChunkSmem<D, (SHAPE & kQ8) != 0>;
  static std::atomic<uint64_t> devices{0};
  const cudaError_t e = allow_shared(chunk_attn_kernel<D, SHAPE>, SM::kBytes, devices);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(SHAPE & kQ8 ? kCThreadsQ8 : kCThreads);
  cfg.dynamicSmemBytes = SM::kBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, chunk_attn_kernel<D, SHAPE>, a);
}

// KIND: kQ8, kSink or none. (A cache in 8 bits knows sinks in every kernel without first keys, which exclude them.)
template <int D, int KIND>
static cudaError_t launch_shape(int shape, const ChunkArgs& a, int grid, cudaStream_t stream) {
  switch (shape) {
#define LAUNCH_SHAPE(S)                                                                   \
  case S: return launch_attn_t<D, (S) | KIND | (KIND ? kSink : 0)>(a, grid, stream);      \
  case (S) | kDocs:                                                                       \
    if constexpr (KIND != kSink) return launch_attn_t<D, (S) | kDocs | KIND>(a, grid, stream); \
    break
    LAUNCH_SHAPE(0);
    LAUNCH_SHAPE(kBias);
    LAUNCH_SHAPE(kCap);
    LAUNCH_SHAPE(kCap | kBias);
    LAUNCH_SHAPE(kCap | kWideCap);
    LAUNCH_SHAPE(kCap | kWideCap | kBias);
#undef LAUNCH_SHAPE
  }
  return cudaErrorInvalidValue;
}

// (D: c.D. A translation unit for each: they take a minute and more)
template <int KIND, int D>
static cudaError_t launch_chunk(const ChunkCall& c) {
  constexpr bool Q8 = KIND == kQ8;
  if (c.T == 0 || c.B == 0) return cudaSuccess;
  const ChunkWs lay = chunk_ws(c.T, c.B, c.Hq, c.Hkv, D);
  const int g = c.Hq / c.Hkv;
  char* ws = c.ws;
  ChunkArgs a;
  a.O = reinterpret_cast<__nv_bfloat16*>(c.O);
  a.lse = c.lse;
  a.cu_new = c.cu_new;
  a.kv_len = c.kv_len;
  a.block_table = c.block_table;
  a.slopes = c.slopes;
  a.mask = MaskArgs{c.first_key, c.prefix_len, c.window, c.window > 0 ? c.sinks : 0};
  a.blocks = reinterpret_cast<const PlanBlock*>(ws + lay.blocks);
  a.head = reinterpret_cast<const PlanHead*>(ws + lay.head);
  a.seen = reinterpret_cast<const uint32_t*>(ws + lay.seen);
  a.part_o = reinterpret_cast<float*>(ws + lay.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + lay.part_ml);
  a.count = reinterpret_cast<uint32_t*>(ws + lay.count);
  a.status = reinterpret_cast<int*>(ws + lay.status);
  a.scale = c.scale;
  a.cap = c.softcap > 0.f ? cap_args(c.scale, c.softcap) : CapArgs{};
  a.Hq = c.Hq;
  a.Hkv = c.Hkv;
  a.max_pages = c.max_pages;
  a.page_size = c.page_size;
  a.n_pages = c.n_pages;
  // a box lies within one page: the largest power of two up to 64 that divides the page size
  a.piece = 64;
  if (c.block_table)
    while (c.page_size % a.piece) a.piece /= 2;
  a.fixed = FixedCost{2, 2};
  a.o_wide = reinterpret_cast<uintptr_t>(c.O) % 32 == 0;
  const long long rows = c.block_table ? c.page_size : c.S_cap, planes = (long long)(c.block_table ? c.n_pages : c.B) * c.Hkv;
  a.Ks = c.Ks;
  a.Vs = c.Vs;
  a.rows = (int)rows;
  a.block_log2 = 0;
  while ((1 << a.block_log2) < c.block) ++a.block_log2;
  auto cache_map = [&](CUtensorMap* m, const void* base, bool keys) {
    return Q8 ? make_map8(m, base, D, rows, planes, a.piece, keys)
              : make_map(m, base, D, rows, planes, a.piece, 1, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
  };
  if (!cache_map(&a.K, c.K, true) || !cache_map(&a.V, c.V, false) ||
      !make_map(&a.Q, Q8 ? reinterpret_cast<const uint16_t*>(ws + lay.q_parts) : c.Q, D, c.Hq, c.T, g, kCRows / g,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B))
    return cudaErrorInvalidValue;
  const int grid = std::min(num_sms_current(), kCMaxCtas);
  a.plan = PlanArgs{c.cu_new, c.kv_len, a.mask, c.T, c.B, block_tokens(g), std::min(c.S_cap, kCMaxKeys), c.Hkv, grid,
                    kCSharedBytes / (2 * kCKeys * D * (Q8 ? 1 : 2)), c.least_new, 0x7fffffff, a.status};
  // (a lane would go through a block's first keys one by one)
  if (max_blocks(c.T, c.B, g) <= kWarpBlocks && c.B <= kWarpSeqs && !c.first_key) {
    a.blocks = nullptr;
  } else {
    chunk_plan_kernel<<<1, kPlanThreads, 0, c.stream>>>(a.plan, reinterpret_cast<PlanBlock*>(ws + lay.blocks),
                                                        reinterpret_cast<PlanHead*>(ws + lay.head),
                                                        reinterpret_cast<uint32_t*>(ws + lay.seen));
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  if constexpr (Q8) {
    uint8_t *parts = reinterpret_cast<uint8_t*>(ws + lay.q_parts), *exps = reinterpret_cast<uint8_t*>(ws + lay.q_exp);
    a.q_exp = exps;
    const long long heads = (long long)c.T * c.Hq, grid_q = (heads * (D / 16) + kSplitThreads - 1) / kSplitThreads;
    if (grid_q > 0x7fffffffll) return cudaErrorInvalidValue;
    split_q_kernel<D><<<(int)grid_q, kSplitThreads, 0, c.stream>>>(c.Q, heads, parts, exps);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  const int shape = (c.softcap > kNarrowCap ? kCap | kWideCap : c.softcap > 0.f ? kCap : 0) | (c.slopes ? kBias : 0) |
                    (c.first_key ? kDocs : 0);
  return launch_shape<D, KIND>(shape, a, grid, c.stream);
}

}  // namespace libraspec
