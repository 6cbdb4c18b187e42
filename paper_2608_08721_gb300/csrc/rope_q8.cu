// Query and key heads normed and rotated in one pass; and the KV cache in 8
// bits: its append with that norm and rotation on the way, and its read-back.
//
// Norm: x -> x r w with r = 1 / sqrt(mean x^2 + eps) over the head, w its
// weights; then the rotation of rope.cu. A group of lanes holds the head in
// registers, so that it is read once.
//
// The cache in 8 bits holds e4m3 codes c (three bits behind the leading one)
// and, for every block of 16, 32 or 64 tokens of a kv head, the exponent e of
// a power of two: the values are c 2^e. With amax the largest finite magnitude
// of the block's new values,
//   e = floor(log2 amax) - 7, within [-60, 60],
// so the codes of the largest lie in [128, 256] (448 is e4m3's largest).
// Powers of two, because a change of scale then moves codes without a second
// rounding (those that stay above 2^-6 of the scale: 2^-14 of amax), so what a
// cache holds hardly depends on the steps in which it was filled; and because
// values are exact in bf16. A block that had tokens keeps its e, or takes the
// larger one that the new tokens ask for, and then the codes that it had are
// rounded to it (to the nearest, ties to even, as the new ones).
//
// A CTA takes one block of a (sequence, kv head), keys or values: its threads
// hold the new rows in registers between the maximum and the codes. Other CTAs
// of the launch rotate the queries, a token each.
#include <cuda_fp16.h>

#include "rope.cuh"

namespace libraspec {

int num_sms_current();

constexpr int kQThreads = 256;
constexpr int kQMaxBlock = 64;          // tokens of a block
constexpr int kQMinExp = -60, kQMaxExp = 60;

struct NormArgs {
  const float *q, *k;  // [d], or NULL: no norm
  float eps;
};

// A lane's U units of a head that G lanes share: unit l + k G is the k-th of lane l. N elements and their partners a unit.
template <typename Tin, int N, bool INTER, int U>
struct HeadPart {
  using Unit = RopeUnit<Tin, Tin, N, INTER>;
  Pack<Tin, N> a[U], b[U];
  float x[U][N], y[U][N];

  __device__ __forceinline__ void load(const Tin* src, int l, int G, int per_head, int half) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u < per_head) {
        a[k] = *reinterpret_cast<const Pack<Tin, N>*>(src + Unit::at(u, half));
        b[k] = *reinterpret_cast<const Pack<Tin, N>*>(src + Unit::partner(u, half));
      }
    }
  }
  __device__ __forceinline__ void widen_all(int l, int G, int per_head) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (l + k * G < per_head) {
        widen(a[k], x[k]);
        widen(b[k], y[k]);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[k][i] = y[k][i] = 0.f;
      }
    }
  }
  // x r w; all lanes of the warp take part, groups of G lanes (a power of two) have a head each
  __device__ __forceinline__ void norm(const float* w, float eps, int d, int l, int G, int per_head, int half) {
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(x[k][i], x[k][i], fmaf(y[k][i], y[k][i], ss));
    for (int off = G >> 1; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
    const float r = rsqrtf(ss / (float)d + eps);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u >= per_head) continue;
      const float *wa = w + Unit::at(u, half), *wb = w + Unit::partner(u, half);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[k][i] = x[k][i] * r * wa[i];
        y[k][i] = y[k][i] * r * wb[i];
      }
    }
  }
  // The rotation, with the token's cosines and sines `cs` in the order of RopeUnit::slot; turn(i): the pair's.
  template <typename F>
  __device__ __forceinline__ void rotate(int l, int G, int half, F&& turn_of) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u * N >= half) continue;
      float v[N], z[N];
      if constexpr (INTER && N > 1) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          Unit::turn(x[k][i], x[k][i + 1], turn_of(u * N + i / 2), v[i], v[i + 1]);
          Unit::turn(y[k][i], y[k][i + 1], turn_of(u * N + N / 2 + i / 2), z[i], z[i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) Unit::turn(x[k][i], y[k][i], turn_of(u * N + i), v[i], z[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[k][i] = v[i];
        y[k][i] = z[i];
      }
    }
  }
  template <typename Tout>
  __device__ __forceinline__ void store(Tout* dst, int l, int G, int per_head, int half) const {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u >= per_head) continue;
      Pack<Tout, N> p, q;
      narrow(x[k], p);
      narrow(y[k], q);
      *reinterpret_cast<Pack<Tout, N>*>(dst + Unit::at(u, half)) = p;
      *reinterpret_cast<Pack<Tout, N>*>(dst + Unit::partner(u, half)) = q;
    }
  }
};

// Lanes that share a head of `units` units: a power of two, at most a warp.
__host__ __device__ constexpr int head_lanes(int units) {
  int g = 1;
  while (g < units && g < 32) g *= 2;
  return g;
}

// Heads [0, H) of one token: normed (if w_q is given; heads from Hq on take w_k), rotated by cs, written.
template <typename Tin, typename Tout, int N, bool INTER, int U>
__device__ __forceinline__ void turn_heads(const Tin* src, Tout* dst, int H, int Hq, int d, int half, const NormArgs& nm,
                                           const float2* cs) {
  const int per_head = d / (2 * N), G = head_lanes(per_head), l = threadIdx.x % G;
  const int step = blockDim.x / G;
  for (int h0 = 0; h0 < H; h0 += step) {  // (all lanes of a warp go round together)
    const int h = h0 + threadIdx.x / G;
    const bool has = h < H;
    HeadPart<Tin, N, INTER, U> p;
    p.load(src + (size_t)(has ? h : 0) * d, l, G, per_head, half);
    p.widen_all(l, G, per_head);
    if (nm.q || nm.k) p.norm(has && h >= Hq ? nm.k : nm.q, nm.eps, d, l, G, per_head, half);
    p.rotate(l, G, half, [&](int i) { return cs[i]; });
    if (has) p.store(dst + (size_t)h * d, l, G, per_head, half);
  }
}

struct NormRopeArgs {
  const void* X;
  long long x_stride, y_stride;
  const int32_t* pos;
  const float2* turns;
  float magnitude;
  NormArgs norm;
  int T, H, Hq, d, half;
  void* Y;
};

template <typename T, int N, bool INTER, int U>
__global__ void __launch_bounds__(kQThreads) norm_rope_kernel(const NormRopeArgs A) {
  __shared__ alignas(16) float2 cs[kRopeMaxPairs];
  const int t = blockIdx.x, pos = A.pos[t];
  for (int i = threadIdx.x; i < A.half; i += blockDim.x) cs[i] = rope_turn(pos, A.turns[i], A.magnitude);
  __syncthreads();
  turn_heads<T, T, N, INTER, U>(static_cast<const T*>(A.X) + t * A.x_stride, static_cast<T*>(A.Y) + t * A.y_stride, A.H,
                                A.Hq, A.d, A.half, A.norm, cs);
}

// ---------------------------------------------------------------------------
// Append.
// ---------------------------------------------------------------------------
struct AppendQ8Args {
  const void *Q, *K, *V;
  long long q_stride, k_stride, v_stride;
  const int32_t *cu_new, *kv_len, *pos, *block_table;
  const float2* turns;
  float magnitude;
  NormArgs norm;
  int T, B, Hq, Hkv, half;
  int max_pages, page_size, n_pages, S_cap, block;
  int n_blocks;  // blocks that the launch has CTAs for
  uint16_t* Qo;
  uint8_t *K8, *V8, *Ks, *Vs;
  int* status;
};

// The n-th block that the chunk writes to: its sequence, first token and the rows of it that are new.
struct BlockOf {
  int b, key0;      // sequence, key of the block's first row
  int r0, r1;       // rows [r0, r1) are new
  int t0;           // packed row of row r0
};

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {  // saturating, to the nearest, ties to even
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 of_e4m3x2(uint16_t c) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(c));
  return __half22float2(*reinterpret_cast<__half2*>(&h));
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }
__device__ __forceinline__ int clamp_exp(int e) { return min(max(e, kQMinExp), kQMaxExp); }

template <int N>
struct alignas(N) Codes {
  uint8_t v[N];
};
template <int N>
__device__ __forceinline__ Codes<N> encode(const float (&x)[N], float inv) {
  Codes<N> c;
  if constexpr (N == 1) {
    c.v[0] = (uint8_t)e4m3x2(x[0] * inv, 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) *reinterpret_cast<uint16_t*>(c.v + i) = (uint16_t)e4m3x2(x[i] * inv, x[i + 1] * inv);
  }
  return c;
}

// New tokens of sequence b (0 where its offsets are out of range), and the blocks that they touch.
__device__ __forceinline__ int new_blocks(const AppendQ8Args& A, int b, bool report, int& lo, int& kv, int& n) {
  lo = A.cu_new[b];
  kv = A.kv_len[b];
  const int hi = A.cu_new[b + 1];
  n = 0;
  if (lo < 0 || hi < lo || hi > A.T) {
    if (report) raise_status(A.status, LIBRASPEC_ST_BAD_LENGTH);
    return 0;
  }
  n = hi - lo;
  if (n == 0) return 0;
  if (kv < 0 || (long long)kv + n > A.S_cap) {  // rows that have no room are skipped
    if (report) raise_status(A.status, LIBRASPEC_ST_KV_OVERFLOW);
    n = kv < 0 || kv >= A.S_cap ? 0 : A.S_cap - kv;
    if (n == 0) return 0;
  }
  return (kv + n - 1) / A.block - kv / A.block + 1;
}

// Block `i` of the chunk, by all threads of the CTA; false: there is none.
__device__ bool find_block(const AppendQ8Args& A, int i, bool report, BlockOf& out) {
  __shared__ long long warp_sum[kQThreads / 32];
  __shared__ BlockOf found;
  __shared__ int is_found;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) is_found = 0;
  long long before = 0;
  for (int b0 = 0; b0 < A.B; b0 += kQThreads) {
    int lo = 0, kv = 0, n = 0, nb = 0;
    if (b0 + tid < A.B) nb = new_blocks(A, b0 + tid, report, lo, kv, n);
    const long long mine = nb;
    long long inc = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, inc, off);
      if (lane >= off) inc += x;
    }
    __syncthreads();
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long base = before, total = 0;
#pragma unroll
    for (int w = 0; w < kQThreads / 32; ++w) {
      if (w < warp) base += warp_sum[w];
      total += warp_sum[w];
    }
    const long long first = base + inc - mine;
    if (i >= first && i < first + mine) {
      const int k = (int)(i - first), kb = kv / A.block + k;
      BlockOf f;
      f.b = b0 + tid;
      f.key0 = kb * A.block;
      f.r0 = k == 0 ? kv - f.key0 : 0;
      f.r1 = min(A.block, kv + n - f.key0);
      f.t0 = lo + f.key0 + f.r0 - kv;
      found = f;
      is_found = 1;
    }
    before += total;
    if (before > i && !report) break;  // (the same for all threads)
  }
  __syncthreads();
  out = found;
  return is_found != 0;
}

template <typename Tin, int N, bool INTER, int D>
__global__ void __launch_bounds__(kQThreads) append_q8_kernel(const AppendQ8Args A) {
  constexpr int kPer = D / (2 * N), kG = kPer < 32 ? kPer : 32, kU = kPer / kG;
  constexpr int kRows = kQThreads / kG, kPasses = (kQMaxBlock + kRows - 1) / kRows;
  const int tid = threadIdx.x, half = A.half;
  const int n_kv = A.n_blocks * A.Hkv * 2;
  if ((int)blockIdx.x < n_kv) {
    const int i = blockIdx.x / (2 * A.Hkv), hk = blockIdx.x % (2 * A.Hkv);
    const bool key = hk < A.Hkv;
    const int h = key ? hk : hk - A.Hkv;
    __shared__ uint32_t s_amax;
    __shared__ int s_exp[2];  // the block's exponent now and before
    if (tid == 0) s_amax = 0;
    BlockOf o;
    if (!find_block(A, i, blockIdx.x == 0, o)) return;
    size_t row0, sc;  // the block's first row, and its scale
    if (A.block_table) {
      int page = A.block_table[(size_t)o.b * A.max_pages + o.key0 / A.page_size];
      if (page < 0 || page >= A.n_pages) {
        if (tid == 0) raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
        return;
      }
      const size_t plane = (size_t)page * A.Hkv + h;
      row0 = plane * A.page_size + o.key0 % A.page_size;
      sc = plane * (A.page_size / A.block) + o.key0 % A.page_size / A.block;
    } else {
      const size_t plane = (size_t)o.b * A.Hkv + h;
      row0 = plane * A.S_cap + o.key0;
      sc = plane * (A.S_cap / A.block) + o.key0 / A.block;
    }
    const Tin* src = static_cast<const Tin*>(key ? A.K : A.V) + h * D;
    const long long stride = key ? A.k_stride : A.v_stride;
    uint8_t* codes = (key ? A.K8 : A.V8) + row0 * D;
    uint8_t* scales = key ? A.Ks : A.Vs;
    const int l = tid % kG, rr = tid / kG;
    HeadPart<Tin, N, INTER, kU> part[kPasses];
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = rr + p * kRows;
      if (r >= o.r0 && r < o.r1) part[p].load(src + (o.t0 + r - o.r0) * stride, l, kG, kPer, half);
    }
    uint32_t amax = 0;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = rr + p * kRows;
      const bool has = r >= o.r0 && r < o.r1;
      if (has) part[p].widen_all(l, kG, kPer);
      if (key) {
        if (A.norm.k) part[p].norm(A.norm.k, A.norm.eps, D, l, kG, kPer, half);
        if (has) {
          const int pos = A.pos ? A.pos[o.t0 + r - o.r0] : o.key0 + r;
          part[p].rotate(l, kG, half, [&](int j) { return rope_turn(pos, A.turns[j], A.magnitude); });
        }
      }
      if (!has) continue;
#pragma unroll
      for (int k = 0; k < kU; ++k)
#pragma unroll
        for (int e = 0; e < N; ++e) {
          const uint32_t a = __float_as_uint(part[p].x[k][e]) & 0x7fffffffu, b = __float_as_uint(part[p].y[k][e]) & 0x7fffffffu;
          if (a < 0x7f800000u) amax = max(amax, a);  // (of finite values; magnitudes are ordered as their bits)
          if (b < 0x7f800000u) amax = max(amax, b);
        }
    }
    amax = __reduce_max_sync(0xffffffffu, amax);
    if (tid % 32 == 0) atomicMax(&s_amax, amax);
    __syncthreads();
    if (tid == 0) {
      int e = clamp_exp((int)(s_amax >> 23) - 127 - 7), before = e;
      if (o.r0 > 0) {
        before = clamp_exp((int)scales[sc] - 127);
        e = max(e, before);
      }
      s_exp[0] = e;
      s_exp[1] = before;
      scales[sc] = (uint8_t)(e + 127);
    }
    __syncthreads();
    const int e = s_exp[0], before = s_exp[1];
    if (e != before) {  // the rows that the block had, to the new scale
      const float f = power_of_two(before - e);
      for (int u = tid; u < o.r0 * (D / 16); u += kQThreads) {
        uint4* at = reinterpret_cast<uint4*>(codes) + u;
        uint4 c = *at;
        uint32_t* w = &c.x;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float2 a = of_e4m3x2((uint16_t)w[k]), b = of_e4m3x2((uint16_t)(w[k] >> 16));
          w[k] = e4m3x2(a.x * f, a.y * f) | e4m3x2(b.x * f, b.y * f) << 16;
        }
        *at = c;
      }
    }
    const float inv = power_of_two(-e);
    using Unit = RopeUnit<Tin, Tin, N, INTER>;
#pragma unroll
    for (int p = 0; p < kPasses; ++p) {
      const int r = rr + p * kRows;
      if (r < o.r0 || r >= o.r1) continue;
#pragma unroll
      for (int k = 0; k < kU; ++k) {
        const int u = l + k * kG;
        *reinterpret_cast<Codes<N>*>(codes + r * D + Unit::at(u, half)) = encode(part[p].x[k], inv);
        *reinterpret_cast<Codes<N>*>(codes + r * D + Unit::partner(u, half)) = encode(part[p].y[k], inv);
      }
    }
    return;
  }
  // queries, a token a CTA
  __shared__ alignas(16) float2 cs[D / 2];
  __shared__ unsigned long long s_owner;  // the token's first sequence and its position there
  const int t = blockIdx.x - n_kv;
  if (tid == 0) s_owner = kRopeNone;
  __syncthreads();
  for (int b = tid; b < A.B; b += kQThreads) {
    const int lo = A.cu_new[b], hi = A.cu_new[b + 1];
    if (lo < 0 || hi < lo || hi > A.T || t < lo || t >= hi) continue;
    atomicMin(&s_owner, (unsigned long long)b << 32 | (uint32_t)((unsigned)A.kv_len[b] + (unsigned)(t - lo)));
  }
  __syncthreads();
  if (s_owner == kRopeNone) return;
  const int pos = A.pos ? A.pos[t] : (int)(uint32_t)s_owner;
  for (int i = tid; i < half; i += kQThreads) cs[i] = rope_turn(pos, A.turns[i], A.magnitude);
  __syncthreads();
  turn_heads<Tin, uint16_t, N, INTER, kU>(static_cast<const Tin*>(A.Q) + t * A.q_stride, A.Qo + (size_t)t * A.Hq * D, A.Hq,
                                          A.Hq, D, half, A.norm, cs);
}

// ---------------------------------------------------------------------------
// Read-back: packed row cu[b] + j is key start[b] + j of sequence b.
// ---------------------------------------------------------------------------
struct ReadQ8Args {
  const uint8_t *K8, *V8, *Ks, *Vs;
  const int32_t *cu, *start, *block_table;
  int T, B, Hkv, max_pages, page_size, n_pages, S_cap, block;
  uint16_t *K, *V;
  int* status;
};
constexpr int kReadTokens = 8;  // of a CTA

template <int D>
__global__ void __launch_bounds__(kQThreads) read_q8_kernel(const ReadQ8Args A) {
  __shared__ unsigned long long s_owner[kReadTokens];  // sequence and key
  __shared__ long long s_row[kReadTokens], s_scale[kReadTokens];  // of kv head 0; -1: none
  const int tid = threadIdx.x, t0 = blockIdx.x * kReadTokens, n_tok = min(kReadTokens, A.T - t0);
  if (tid < kReadTokens) s_owner[tid] = kRopeNone;
  __syncthreads();
  for (int b = tid; b < A.B; b += kQThreads) {
    const int lo = A.cu[b], hi = A.cu[b + 1];
    if (lo < 0 || hi < lo || hi > A.T) {
      if (blockIdx.x == 0) raise_status(A.status, LIBRASPEC_ST_BAD_LENGTH);
      continue;
    }
    if (lo >= t0 + n_tok || hi <= t0) continue;
    const int first = A.start[b];
    for (int j = max(0, lo - t0); j < min(n_tok, hi - t0); ++j) {
      const long long key = (long long)first + (t0 + j - lo);
      const bool room = first >= 0 && key < A.S_cap;
      atomicMin(&s_owner[j], (unsigned long long)b << 33 | (unsigned long long)!room << 32 | (uint32_t)key);
    }
  }
  __syncthreads();
  if (tid < n_tok) {
    const unsigned long long owner = s_owner[tid];
    const uint32_t b = (uint32_t)(owner >> 33), key = (uint32_t)owner;
    long long row = -1, scale = 0;
    if (owner != kRopeNone) {
      if (owner >> 32 & 1) {
        raise_status(A.status, LIBRASPEC_ST_KV_OVERFLOW);
      } else if (A.block_table) {
        const uint32_t nth = key / (uint32_t)A.page_size, in = key - nth * A.page_size;
        const int page = A.block_table[(size_t)b * A.max_pages + nth];
        if (page < 0 || page >= A.n_pages) {
          raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
        } else {
          row = (long long)page * A.Hkv * A.page_size + in;
          scale = (long long)page * A.Hkv * (A.page_size / A.block) + in / A.block;
        }
      } else {
        row = (long long)b * A.Hkv * A.S_cap + key;
        scale = (long long)b * A.Hkv * (A.S_cap / A.block) + key / A.block;
      }
    }
    s_row[tid] = row;
    s_scale[tid] = scale;
  }
  __syncthreads();
  const int rows = A.block_table ? A.page_size : A.S_cap, scales = rows / A.block;
  constexpr int kUnits = D / 16;
  const int per_token = A.Hkv * kUnits;
  for (int u = tid; u < n_tok * per_token * 2; u += kQThreads) {
    const int j = u / (2 * per_token), x = u - j * 2 * per_token;
    const bool key = x < per_token;
    const int h = (key ? x : x - per_token) / kUnits, c = x % kUnits;
    if (s_row[j] < 0) continue;
    const uint4 v = __ldg(reinterpret_cast<const uint4*>((key ? A.K8 : A.V8) + (s_row[j] + (long long)h * rows) * D) + c);
    const float f = power_of_two(clamp_exp((int)(key ? A.Ks : A.Vs)[s_scale[j] + (long long)h * scales] - 127));
    const uint32_t* w = &v.x;
    float y[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 a = of_e4m3x2((uint16_t)w[k]), b = of_e4m3x2((uint16_t)(w[k] >> 16));
      y[4 * k] = a.x * f;
      y[4 * k + 1] = a.y * f;
      y[4 * k + 2] = b.x * f;
      y[4 * k + 3] = b.y * f;
    }
    Pack<uint16_t, 16> p;
    narrow(y, p);
    uint4* dst = reinterpret_cast<uint4*>((key ? A.K : A.V) + ((size_t)(t0 + j) * A.Hkv + h) * D) + 2 * c;
    dst[0] = reinterpret_cast<const uint4*>(p.v)[0];
    dst[1] = reinterpret_cast<const uint4*>(p.v)[1];
  }
}

// ---------------------------------------------------------------------------
// Host side. Units of N elements where every access that they make is aligned to its size, else pair by pair (rope.cu).
// ---------------------------------------------------------------------------
template <typename T>
cudaError_t launch_norm_rope(const T* X, long long x_stride, const int32_t* pos, const float* turns, float magnitude,
                             const float* q_weight, const float* k_weight, float eps, int n_tokens, int Hq, int Hk, int d,
                             int rot, int interleaved, T* Y, long long y_stride, cudaStream_t stream) {
  if (n_tokens == 0 || Hq + Hk == 0) return cudaSuccess;
  constexpr int N = 16 / (int)sizeof(T);
  const NormRopeArgs a{X, x_stride, y_stride, pos, reinterpret_cast<const float2*>(turns), magnitude,
                       NormArgs{q_weight, k_weight, eps}, n_tokens, Hq + Hk, Hq, d, rot / 2, Y};
  auto fits = [&](const void* p, long long stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % N == 0;
  };
  const bool vec = a.half % N == 0 && d % (2 * N) == 0 && fits(X, x_stride) && fits(Y, y_stride);
  constexpr int kWideU = 256 / N / 32 ? 256 / N / 32 : 1;  // units of a lane: heads of 512
  if (vec) {
    if (interleaved) norm_rope_kernel<T, N, true, kWideU><<<n_tokens, kQThreads, 0, stream>>>(a);
    else norm_rope_kernel<T, N, false, kWideU><<<n_tokens, kQThreads, 0, stream>>>(a);
  } else {
    if (interleaved) norm_rope_kernel<T, 1, true, 8><<<n_tokens, kQThreads, 0, stream>>>(a);
    else norm_rope_kernel<T, 1, false, 8><<<n_tokens, kQThreads, 0, stream>>>(a);
  }
  return cudaGetLastError();
}
template cudaError_t launch_norm_rope<float>(const float*, long long, const int32_t*, const float*, float, const float*,
                                             const float*, float, int, int, int, int, int, int, float*, long long,
                                             cudaStream_t);
template cudaError_t launch_norm_rope<uint16_t>(const uint16_t*, long long, const int32_t*, const float*, float,
                                                const float*, const float*, float, int, int, int, int, int, int,
                                                uint16_t*, long long, cudaStream_t);

template <typename T, int N, int D>
static cudaError_t launch_append_n(const AppendQ8Args& a, int interleaved, cudaStream_t stream) {
  const long long grid = (long long)a.n_blocks * a.Hkv * 2 + (a.Qo ? a.T : 0);
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  if (interleaved) append_q8_kernel<T, N, true, D><<<(int)grid, kQThreads, 0, stream>>>(a);
  else append_q8_kernel<T, N, false, D><<<(int)grid, kQThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_rope_append_q8(const T* Q, long long q_stride, const T* K, long long k_stride, const T* V,
                                  long long v_stride, const int32_t* cu_new, const int32_t* kv_len, const int32_t* pos,
                                  const float* turns, float magnitude, const float* q_weight, const float* k_weight,
                                  float eps, const int32_t* block_table, int max_pages, int page_size, int n_pages,
                                  int n_tokens, int B, int Hq, int Hkv, int d, int rot, int interleaved, uint16_t* Qo,
                                  uint8_t* K8, uint8_t* V8, uint8_t* Ks, uint8_t* Vs, int S_cap, int block, int* status,
                                  cudaStream_t stream) {
  if (n_tokens == 0 || B == 0) return cudaSuccess;
  AppendQ8Args a{Q, K, V, q_stride, k_stride, v_stride, cu_new, kv_len, pos, block_table,
                 reinterpret_cast<const float2*>(turns), magnitude, NormArgs{q_weight, k_weight, eps}, n_tokens, B,
                 Q ? Hq : 0, Hkv, rot / 2, max_pages, page_size, n_pages, S_cap, block, 0, Qo, K8, V8, Ks, Vs, status};
  // a sequence's tokens lie in at most n / block + 2 blocks, and in at most n
  a.n_blocks = (int)std::min((long long)n_tokens, (long long)n_tokens / block + 2ll * B);
  constexpr int N = 16 / (int)sizeof(T);
  auto fits = [&](const void* p, long long stride) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && stride % N == 0;
  };
  const bool vec = a.half % N == 0 && fits(K, k_stride) && fits(V, v_stride) && (!Q || fits(Q, q_stride));
  if (d == 128)
    return vec ? launch_append_n<T, N, 128>(a, interleaved, stream) : launch_append_n<T, 1, 128>(a, interleaved, stream);
  return vec ? launch_append_n<T, N, 64>(a, interleaved, stream) : launch_append_n<T, 1, 64>(a, interleaved, stream);
}
#define INSTANCE(T)                                                                                                       \
  template cudaError_t launch_rope_append_q8<T>(                                                                          \
      const T*, long long, const T*, long long, const T*, long long, const int32_t*, const int32_t*, const int32_t*,      \
      const float*, float, const float*, const float*, float, const int32_t*, int, int, int, int, int, int, int, int, int, \
      int, uint16_t*, uint8_t*, uint8_t*, uint8_t*, uint8_t*, int, int, int*, cudaStream_t)
INSTANCE(float);
INSTANCE(uint16_t);
#undef INSTANCE

cudaError_t launch_kv_read_q8(const uint8_t* K8, const uint8_t* V8, const uint8_t* Ks, const uint8_t* Vs,
                              const int32_t* block_table, int max_pages, int page_size, int n_pages, const int32_t* cu,
                              const int32_t* start, int n_tokens, int B, int Hkv, int d, int S_cap, int block, uint16_t* K,
                              uint16_t* V, int* status, cudaStream_t stream) {
  if (n_tokens == 0 || B == 0) return cudaSuccess;
  const ReadQ8Args a{K8, V8, Ks, Vs, cu, start, block_table, n_tokens, B, Hkv, max_pages, page_size, n_pages, S_cap, block,
                     K, V, status};
  const int grid = (n_tokens + kReadTokens - 1) / kReadTokens;
  if (d == 128) read_q8_kernel<128><<<grid, kQThreads, 0, stream>>>(a);
  else read_q8_kernel<64><<<grid, kQThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace libraspec
