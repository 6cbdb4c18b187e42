// Rotary positions, and the append of a ragged chunk of new tokens to the KV
// cache with the rotation on the way.
//
// Pair i of a head turns by the angle pos * f_i: (x0, x1) -> m (x0 cos - x1
// sin, x0 sin + x1 cos). The frequencies come as turns per position, f / 2pi
// = hi + lo in two floats, so that the part of the angle that counts, its
// fraction of a turn, is exact to 2^-24 turns at any position: p = pos hi has
// the exact error e = fma(pos, hi, -p), p - rint(p) is exact, and sincospi
// needs no further reduction. (A binary32 angle of 131072 radians is off by
// 0.004.)
//
// Bound by HBM: every element is read once and written once. One CTA works on
// one token or two: its threads form the tokens' cosines and sines in shared
// memory (once for all heads) while their first loads are on their way, then
// they share out the tokens' heads in units of 16 bytes. 8192 tokens of 64
// heads of 128 in fp32 take 80 us, 98% of the copy rate; the append of 8587
// tokens of 28 + 2 x 4 heads (158 MB) 30 us, 78% of it, 64 decoding tokens 3.1.
#include <cmath>

#include "rope.cuh"

namespace libraspec {

int num_sms_current();

constexpr int kRopeThreads = 512;   // of a CTA, at most

// Rows h of a token: h < Hq queries, then (append) Hkv keys and Hkv values.
struct RopeArgs {
  const void *Q, *K, *V;
  long long q_stride, k_stride, v_stride, o_stride;  // elements between tokens
  const int32_t* pos;     // [T], or NULL (append): kv_len of the token's sequence + its index there
  const float2* turns;    // [rot / 2]
  float magnitude;
  int inverse;
  int T, Hq, Hkv, d, half;
  void* Qo;
  // append
  const int32_t *cu_new, *kv_len, *block_table;
  int B, max_pages, page_size, n_pages, S_cap;
  uint16_t *Kc, *Vc;
  int* status;
};

template <typename Tin, typename Tout, int N, bool INTER, bool APPEND, int TOKENS>
__global__ void __launch_bounds__(kRopeThreads, 3) rope_kernel(const RopeArgs A) {
  __shared__ alignas(16) float2 cs[TOKENS][kRopeMaxPairs];
  __shared__ int s_pos[TOKENS];
  // (append) a token's sequence, whether that has no room for it, and its key's index there, from bits 33, 32 and 0
  __shared__ unsigned long long s_owner[TOKENS];
  __shared__ long long s_row[TOKENS];  // the token's row of the cache (of kv head 0); -1: no room; -2: of no sequence
  const int t0 = blockIdx.x * TOKENS, tid = threadIdx.x;
  const int n_tok = min(TOKENS, A.T - t0);
  const int per_head = A.d / (2 * N), heads = APPEND ? A.Hq + 2 * A.Hkv : A.Hq;
  long long head_step = 0;  // between the rows of neighbouring kv heads in the cache
  if constexpr (APPEND) head_step = (long long)(A.block_table ? A.page_size : A.S_cap) * A.d;
  // A thread has one unit of a head, in every step-th head of all the CTA's tokens: what it adds up for an address it
  // adds up once for two tokens, whose loads are in flight together.
  const int step = blockDim.x / per_head, u = tid % per_head;
  int h = tid / per_head;
  if (h >= step) h = heads;  // (a thread past the last whole head has none)
  RopeUnit<Tin, Tout, N, INTER> unit[TOKENS];
  auto load = [&](int h, RopeUnit<Tin, Tout, N, INTER>(&to)[TOKENS]) {
    const Tin* src = static_cast<const Tin*>(A.Q) + (long long)t0 * A.q_stride + h * A.d;
    long long stride = A.q_stride;
    if (APPEND && h >= A.Hq) {
      const bool key = h < A.Hq + A.Hkv;
      stride = key ? A.k_stride : A.v_stride;
      src = static_cast<const Tin*>(key ? A.K : A.V) + t0 * stride + (h - A.Hq - (key ? 0 : A.Hkv)) * A.d;
    }
#pragma unroll
    for (int j = 0; j < TOKENS; ++j)
      if (TOKENS == 1 || j < n_tok) to[j].load(src + j * stride, u, A.half);
  };

  if constexpr (APPEND) {
    if (tid < TOKENS) s_owner[tid] = kRopeNone;
    __syncthreads();
    // The tokens' sequences: every thread looks at its share of the offsets. (Ranges overlap only beside offsets that
    // run backwards: the token is the first sequence's then.)
    for (int b = tid; b < A.B; b += blockDim.x) {
      const int lo = A.cu_new[b], hi = A.cu_new[b + 1], kv = A.kv_len[b];
      if (lo < 0 || hi < lo || hi > A.T) {  // skipped; of the others t - lo lies in [0, T)
        if (blockIdx.x == 0) raise_status(A.status, LIBRASPEC_ST_BAD_LENGTH);
        continue;
      }
#pragma unroll
      for (int j = 0; j < TOKENS; ++j) {
        const int t = t0 + j;
        if (j >= n_tok || t < lo || t >= hi) continue;
        const long long s = (long long)kv + (t - lo);
        const bool room = kv >= 0 && s < A.S_cap;
        atomicMin(&s_owner[j], (unsigned long long)b << 33 | (unsigned long long)!room << 32 | (uint32_t)s);
      }
    }
    __syncthreads();
  } else if (TOKENS > 1) {
    if (tid < n_tok) s_pos[tid] = A.pos[t0 + tid];
    __syncthreads();
  }
  if (APPEND && tid >= (int)blockDim.x - TOKENS) {  // the rows, by the CTA's last threads
    const int j = blockDim.x - 1 - tid;
    const unsigned long long owner = s_owner[j];
    const uint32_t b = (uint32_t)(owner >> 33), s = (uint32_t)owner;
    long long at = -2;
    if (owner != kRopeNone) {
      at = -1;
      if (owner >> 32 & 1) {
        raise_status(A.status, LIBRASPEC_ST_KV_OVERFLOW);
      } else if (A.block_table) {
        const uint32_t nth = s / (uint32_t)A.page_size;  // (s < S_cap, an int)
        const int page = A.block_table[(size_t)b * A.max_pages + nth];
        if (page < 0 || page >= A.n_pages) raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
        else at = ((long long)page * A.Hkv * A.page_size + (s - nth * A.page_size)) * A.d;
      } else {
        at = ((long long)b * A.Hkv * A.S_cap + s) * A.d;
      }
    }
    s_row[j] = at;
  }
  // The first units, in flight while the cosines are formed. (Ahead of the page's look-up, which then queues behind
  // them: 30.3 us for 8587 bf16 tokens of 36 heads; so, 29.8.)
  if (h < heads) load(h, unit);
  for (int i = tid; i < n_tok * A.half; i += blockDim.x) {
    const int j = TOKENS == 1 ? 0 : i / A.half, k = i - j * A.half;
    if (APPEND && s_owner[j] == kRopeNone) continue;
    const int pos = APPEND ? (A.pos ? A.pos[t0 + j] : (int)(uint32_t)s_owner[j]) : TOKENS > 1 ? s_pos[j] : A.pos[t0];
    float2 c = rope_turn(pos, A.turns[k], A.magnitude);
    if (A.inverse) c.y = -c.y;
    cs[j][RopeUnit<Tin, Tout, N, INTER>::slot(k, A.half)] = c;
  }
  __syncthreads();
  for (; h < heads; h += step) {
    RopeUnit<Tin, Tout, N, INTER> ahead[TOKENS];
    if (TOKENS == 1 && h + step < heads) load(h + step, ahead);
    const bool query = !APPEND || h < A.Hq, turns = !APPEND || h < A.Hq + A.Hkv;
    Tout* dst = static_cast<Tout*>(A.Qo) + t0 * A.o_stride + h * A.d;
    if (!query)
      dst = reinterpret_cast<Tout*>(turns ? A.Kc : A.Vc) + (h - A.Hq - (turns ? 0 : A.Hkv)) * head_step;
#pragma unroll
    for (int j = 0; j < TOKENS; ++j) {
      if (TOKENS > 1 && j >= n_tok) break;
      // (the query of a token without room is rotated all the same)
      if (APPEND && s_row[j] < (query ? -1 : 0)) continue;
      unit[j].store(dst + (query ? j * A.o_stride : s_row[j]), turns, u, A.half, cs[j]);
    }
    if (TOKENS == 1) unit[0] = ahead[0];
    else if (h + step < heads) load(h + step, unit);
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Turns per position of each pair as (hi, lo) floats; scaling as in the header. False if one of them is beyond what the
// kernels multiply with a position in binary32.
bool rope_frequencies(int rot, double theta, int scaling, double factor, double low, double high, double original_len,
                      float* turns) {
  const double two_pi = 6.283185307179586476925;
  if (scaling == LIBRASPEC_ROPE_NTK) theta *= std::pow(factor, rot / (rot - 2.0));
  for (int i = 0; i < rot / 2; ++i) {
    double f = std::pow(theta, -2.0 * i / rot);
    if (scaling == LIBRASPEC_ROPE_LINEAR) f /= factor;
    if (scaling == LIBRASPEC_ROPE_BY_PARTS) {
      const double r = original_len * f / two_pi;  // turns over the original context
      const double keep = std::min(1.0, std::max(0.0, (r - low) / (high - low)));
      f = (1.0 - keep) * f / factor + keep * f;
    }
    const double t = f / two_pi;
    if (!(t <= 1e29)) return false;  // (times 2^31: finite)
    turns[2 * i] = (float)t;
    turns[2 * i + 1] = (float)(t - (double)turns[2 * i]);
  }
  return true;
}

template <typename Tin, typename Tout, int N, bool APPEND, int TOKENS>
static cudaError_t launch_tokens(const RopeArgs& a, int interleaved, int threads, cudaStream_t stream) {
  const int grid = (a.T + TOKENS - 1) / TOKENS;
  if (interleaved) rope_kernel<Tin, Tout, N, true, APPEND, TOKENS><<<grid, threads, 0, stream>>>(a);
  else rope_kernel<Tin, Tout, N, false, APPEND, TOKENS><<<grid, threads, 0, stream>>>(a);
  return cudaGetLastError();
}

// Two tokens a CTA, with a thread for each of a token's units, where a CTA has room for them and every SM gets a few
// CTAs; else one token in passes of up to 256 threads over its heads. (8587 bf16 tokens of 36 heads: 29.8 us at two
// tokens, 37 at one, 39 at four; in passes of 256 threads, which leave 7 of 8 warps idle in the second, slower still.
// 8192 fp32 tokens of 64 heads: 80 us in passes of 256 threads, 82 in passes of 512.)
template <typename Tin, typename Tout, int N, bool APPEND>
static cudaError_t launch_n(const RopeArgs& a, int interleaved, cudaStream_t stream) {
  const int per_head = a.d / (2 * N), heads = APPEND ? a.Hq + 2 * a.Hkv : a.Hq;
  auto threads_for = [&](int step) { return std::max(64, (step * per_head + 31) / 32 * 32); };
  if (heads <= kRopeThreads / per_head) {
    return a.T >= 8 * num_sms_current()
               ? launch_tokens<Tin, Tout, N, APPEND, 2>(a, interleaved, threads_for(heads), stream)
               : launch_tokens<Tin, Tout, N, APPEND, 1>(a, interleaved, threads_for(heads), stream);
  }
  const int most = 256 / per_head, passes = (heads + most - 1) / most;
  return launch_tokens<Tin, Tout, N, APPEND, 1>(a, interleaved, threads_for((heads + passes - 1) / passes), stream);
}

// Units of N elements where every access they make is aligned to its size: the rotated half and the head in whole
// units, and all rows starting on a multiple of N elements. Else pair by pair.
template <typename Tin, typename Tout, bool APPEND>
static cudaError_t launch_rope_t(const RopeArgs& a, int interleaved, cudaStream_t stream) {
  constexpr int N = 16 / (int)sizeof(Tin);
  auto fits = [&](const void* p, long long stride, size_t size) {
    return reinterpret_cast<uintptr_t>(p) % (N * size) == 0 && stride % N == 0;
  };
  bool vec = a.half % N == 0 && a.d % (2 * N) == 0;
  if (a.Hq > 0) vec = vec && fits(a.Q, a.q_stride, sizeof(Tin)) && fits(a.Qo, a.o_stride, sizeof(Tout));
  if (APPEND) vec = vec && fits(a.K, a.k_stride, sizeof(Tin)) && fits(a.V, a.v_stride, sizeof(Tin));
  return vec ? launch_n<Tin, Tout, N, APPEND>(a, interleaved, stream)
             : launch_n<Tin, Tout, 1, APPEND>(a, interleaved, stream);
}

template <typename T>
cudaError_t launch_rope(const T* X, long long x_stride, const int32_t* pos, const float* turns, float magnitude,
                        int n_tokens, int H, int d, int rot, int interleaved, int inverse, T* Y, long long y_stride,
                        cudaStream_t stream) {
  if (n_tokens == 0) return cudaSuccess;
  RopeArgs a{};
  a.Q = X;
  a.q_stride = x_stride;
  a.o_stride = y_stride;
  a.pos = pos;
  a.turns = reinterpret_cast<const float2*>(turns);
  a.magnitude = magnitude;
  a.inverse = inverse;
  a.T = n_tokens;
  a.Hq = H;
  a.d = d;
  a.half = rot / 2;
  a.Qo = Y;
  return launch_rope_t<T, T, false>(a, interleaved, stream);
}
template cudaError_t launch_rope<float>(const float*, long long, const int32_t*, const float*, float, int, int, int,
                                        int, int, int, float*, long long, cudaStream_t);
template cudaError_t launch_rope<uint16_t>(const uint16_t*, long long, const int32_t*, const float*, float, int, int,
                                           int, int, int, int, uint16_t*, long long, cudaStream_t);

template <typename T>
cudaError_t launch_rope_append(const T* Q, long long q_stride, const T* K, long long k_stride, const T* V,
                               long long v_stride, const int32_t* cu_new, const int32_t* kv_len, const int32_t* pos,
                               const float* turns, float magnitude, const int32_t* block_table, int max_pages,
                               int page_size, int n_pages, int n_tokens, int B, int Hq, int Hkv, int d, int rot,
                               int interleaved, uint16_t* Qo, uint16_t* Kc, uint16_t* Vc, int S_cap, int* status,
                               cudaStream_t stream) {
  if (n_tokens == 0 || B == 0) return cudaSuccess;
  RopeArgs a{};
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.o_stride = (long long)Hq * d;
  a.pos = pos;
  a.turns = reinterpret_cast<const float2*>(turns);
  a.magnitude = magnitude;
  a.T = n_tokens;
  a.Hq = Q ? Hq : 0;
  a.Hkv = Hkv;
  a.d = d;
  a.half = rot / 2;
  a.Qo = Qo;
  a.cu_new = cu_new;
  a.kv_len = kv_len;
  a.block_table = block_table;
  a.B = B;
  a.max_pages = max_pages;
  a.page_size = page_size;
  a.n_pages = n_pages;
  a.S_cap = S_cap;
  a.Kc = Kc;
  a.Vc = Vc;
  a.status = status;
  return launch_rope_t<T, uint16_t, true>(a, interleaved, stream);
}
template cudaError_t launch_rope_append<float>(const float*, long long, const float*, long long, const float*,
                                               long long, const int32_t*, const int32_t*, const int32_t*, const float*,
                                               float, const int32_t*, int, int, int, int, int, int, int, int, int, int,
                                               uint16_t*, uint16_t*, uint16_t*, int, int*, cudaStream_t);
template cudaError_t launch_rope_append<uint16_t>(const uint16_t*, long long, const uint16_t*, long long,
                                                  const uint16_t*, long long, const int32_t*, const int32_t*,
                                                  const int32_t*, const float*, float, const int32_t*, int, int, int,
                                                  int, int, int, int, int, int, int, uint16_t*, uint16_t*, uint16_t*,
                                                  int, int*, cudaStream_t);

}  // namespace libraspec
