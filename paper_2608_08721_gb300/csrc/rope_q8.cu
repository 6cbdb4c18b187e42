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
// A CTA (or, with few new tokens, a warp) takes one block of a (sequence, kv
// head), keys or values, at a time: its threads hold the new rows in registers
// between the maximum and the codes.
//
// What bounds them: the norm of 8192 x 72 fp32 heads takes 91 us, 98% of the
// copy rate; the read-back of 16 caches (740 MB) 118 us, 93%; the append of 8587
// tokens of 28 + 2 x 4 heads 34 us, 64%: the instructions of turns, conversions
// and maxima take as long as the bytes; 64 single tokens of 32 + 8 heads 5.1 us,
// a chain of look-ups (sequence, page, scale).
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

// rope_turn with what its sums round off of the angle (up to 2^-24 of a turn) put in by the angle's derivative: the turn is
// then as exact as sincospi. (Codes are rounded from what it turns: the further off that is, the more of them are those of
// the neighbouring step.)
__device__ __forceinline__ float sum_exactly(float a, float b, float& rest) {  // a + b = sum + rest
  const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
  rest = __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t));
  return s;
}
__device__ __forceinline__ float2 fine_turn(int pos, float2 f, float magnitude) {
  const float hi = (float)(pos & ~255), lo = (float)(pos & 255);
  const float p = __fmul_rn(hi, f.x), q = __fmul_rn(lo, f.x);
  const float e = __fmaf_rn(hi, f.x, -p) + __fmaf_rn(lo, f.x, -q) + __fmaf_rn(hi, f.y, lo * f.y);
  float r0, r1, sn, cs;
  const float s = sum_exactly(sum_exactly(p - rintf(p), q - rintf(q), r0), e, r1);
  sincospif(2.f * (s - rintf(s)), &sn, &cs);
  const float d = 6.283185307179586f * (r0 + r1);
  return make_float2(fmaf(-d, sn, cs) * magnitude, fmaf(d, cs, sn) * magnitude);
}

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
  __device__ __forceinline__ void norm(const float* w, float eps, float inv_d, int l, int G, int per_head, int half) {
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < U; ++k)
#pragma unroll
      for (int i = 0; i < N; ++i) ss = fmaf(x[k][i], x[k][i], fmaf(y[k][i], y[k][i], ss));
    for (int off = G >> 1; off > 0; off >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
    const float r = __frsqrt_rn(fmaf(ss, inv_d, eps));
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u >= per_head) continue;
      const Pack<float, N> wa = *reinterpret_cast<const Pack<float, N>*>(w + Unit::at(u, half));
      const Pack<float, N> wb = *reinterpret_cast<const Pack<float, N>*>(w + Unit::partner(u, half));
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[k][i] = x[k][i] * r * wa.v[i];
        y[k][i] = y[k][i] * r * wb.v[i];
      }
    }
  }
  // The rotation; turns(u, t): the cosines and sines of unit u's pairs.
  template <typename F>
  __device__ __forceinline__ void rotate(int l, int G, int half, F&& turns) {
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const int u = l + k * G;
      if (u * N >= half) continue;
      float v[N], z[N];
      float2 c[N];
      turns(u, c);
      if constexpr (INTER && N > 1) {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          Unit::turn(x[k][i], x[k][i + 1], c[i / 2], v[i], v[i + 1]);
          Unit::turn(y[k][i], y[k][i + 1], c[N / 2 + i / 2], z[i], z[i + 1]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i) Unit::turn(x[k][i], y[k][i], c[i], v[i], z[i]);
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[k][i] = v[i];
        y[k][i] = z[i];
      }
    }
  }
  // ... from the table `cs` of a token, in the order of RopeUnit::slot
  __device__ __forceinline__ void rotate_by(const float2* cs, int l, int G, int half) {
    rotate(l, G, half, [&](int u, float2(&c)[N]) {
      if constexpr (N == 1) {
        c[0] = cs[u];
      } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) {
          const float4 two = *reinterpret_cast<const float4*>(cs + Unit::slot(u * N + i, half));
          c[i] = make_float2(two.x, two.y);
          c[i + 1] = make_float2(two.z, two.w);
        }
      }
    });
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

// Heads [0, H) of one token: normed (w: the weights in shared memory, those of heads from Hq on behind the others', or
// NULL), rotated by the table cs, written. The heads of the next pass are on their way meanwhile.
template <typename Tin, typename Tout, int N, bool INTER, int U>
__device__ __forceinline__ void turn_heads(const Tin* src, Tout* dst, int H, int Hq, int d, int half, const float* w,
                                           float eps, const float2* cs) {
  const int per_head = d / (2 * N), G = head_lanes(per_head), l = threadIdx.x % G;
  const int step = blockDim.x / G;
  const float inv_d = 1.f / (float)d;
  HeadPart<Tin, N, INTER, U> now, next;
  int h = threadIdx.x / G;
  if (h < H) now.load(src + (size_t)h * d, l, G, per_head, half);
  for (int h0 = 0; h0 < H; h0 += step, h += step) {  // (all lanes of a warp go round together)
    if (h + step < H) next.load(src + (size_t)(h + step) * d, l, G, per_head, half);
    if (h0 == 0) __syncthreads();  // the tables are written
    now.widen_all(l, G, per_head);
    if (w) now.norm(h >= Hq ? w + d : w, eps, inv_d, l, G, per_head, half);
    now.rotate_by(cs, l, G, half);
    if (h < H) now.store(dst + (size_t)h * d, l, G, per_head, half);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      now.a[k] = next.a[k];
      now.b[k] = next.b[k];
    }
  }
}

// A token's table of turns, and the weights, into shared memory.
template <typename Unit>
__device__ __forceinline__ void fill_tables(float2* cs, float* w, int pos, const float2* turns, float magnitude, int half,
                                            const NormArgs& nm, int d) {
  for (int i = threadIdx.x; i < half; i += blockDim.x) cs[Unit::slot(i, half)] = fine_turn(pos, turns[i], magnitude);
  if (nm.q)
    for (int i = threadIdx.x; i < 2 * d; i += blockDim.x) w[i] = i < d ? nm.q[i] : nm.k[i - d];
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
  __shared__ alignas(32) float w[2 * LIBRASPEC_ROPE_MAX_DIM];
  const int t = blockIdx.x;
  fill_tables<RopeUnit<T, T, N, INTER>>(cs, w, A.pos[t], A.turns, A.magnitude, A.half, A.norm, A.d);
  turn_heads<T, T, N, INTER, U>(static_cast<const T*>(A.X) + t * A.x_stride, static_cast<T*>(A.Y) + t * A.y_stride, A.H,
                                A.Hq, A.d, A.half, w, A.norm.eps, cs);
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
  int n_blocks;    // blocks that the launch has CTAs for
  int per;         // of each
  int block_ctas;  // all of them; the queries' follow
  int heads;       // kv heads that one of them takes one after the other
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

// New tokens of sequence b that have room (0 where its offsets are out of range), and the blocks that they touch.
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
  if (kv < 0 || (long long)kv + n > A.S_cap) {
    if (report) raise_status(A.status, LIBRASPEC_ST_KV_OVERFLOW);
    n = kv < 0 || kv >= A.S_cap ? 0 : A.S_cap - kv;
    if (n == 0) return 0;
  }
  return (kv + n - 1) / A.block - kv / A.block + 1;
}

// Block `i` of the chunk, by all threads of the CTA; false: there is none.
static __device__ bool find_block(const AppendQ8Args& A, int i, bool report, BlockOf& out) {
  __shared__ long long warp_sum[kQThreads / 32];
  __shared__ BlockOf found;
  __shared__ int is_found;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) is_found = 0;
  long long before = 0;
  for (int b0 = 0; b0 < A.B; b0 += kQThreads) {
    int lo = 0, kv = 0, n = 0;
    long long mine = 0;
    if (b0 + tid < A.B) mine = new_blocks(A, b0 + tid, report, lo, kv, n);
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

// Where block `o` lies for kv head 0: its first row and its scale, with the steps from head to head.
struct BlockPlace {
  size_t row, scale;
  int row_step, scale_step;
};
// (false: its page does not exist)
__device__ __forceinline__ bool place_block(const AppendQ8Args& A, const BlockOf& o, BlockPlace& p) {
  const int rows = A.block_table ? A.page_size : A.S_cap;
  size_t plane = o.b;
  int key = o.key0;
  if (A.block_table) {
    const int page = A.block_table[(size_t)o.b * A.max_pages + key / A.page_size];
    if (page < 0 || page >= A.n_pages) {
      if (threadIdx.x == 0) raise_status(A.status, LIBRASPEC_ST_BAD_PAGE);
      return false;
    }
    plane = page;
    key %= A.page_size;
  }
  p.row_step = rows;
  p.scale_step = rows / A.block;
  p.row = plane * A.Hkv * p.row_step + key;
  p.scale = plane * A.Hkv * p.scale_step + key / A.block;
  return true;
}

template <typename Tin, int N, bool INTER, int U>
__device__ __forceinline__ uint32_t largest_of(const HeadPart<Tin, N, INTER, U>& p, uint32_t amax) {
#pragma unroll
  for (int k = 0; k < U; ++k)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const uint32_t a = __float_as_uint(p.x[k][e]) & 0x7fffffffu, b = __float_as_uint(p.y[k][e]) & 0x7fffffffu;
      if (a < 0x7f800000u) amax = max(amax, a);  // (of finite values; magnitudes are ordered as their bits)
      if (b < 0x7f800000u) amax = max(amax, b);
    }
  return amax;
}
__device__ __forceinline__ int exponent_of(uint32_t amax) { return clamp_exp((int)(amax >> 23) - 127 - 7); }

// 16 codes to another scale, f = 2^(old - new)
__device__ __forceinline__ void recode(uint4* at, float f) {
  uint4 c = *at;
  uint32_t* w = &c.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 a = of_e4m3x2((uint16_t)w[k]), b = of_e4m3x2((uint16_t)(w[k] >> 16));
    w[k] = e4m3x2(a.x * f, a.y * f) | e4m3x2(b.x * f, b.y * f) << 16;
  }
  *at = c;
}

template <typename Tin, int N, bool INTER, int U>
__device__ __forceinline__ void write_codes(const HeadPart<Tin, N, INTER, U>& p, uint8_t* row, float inv, int l, int G,
                                            int half) {
  using Unit = RopeUnit<Tin, Tin, N, INTER>;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const int u = l + k * G;
    *reinterpret_cast<Codes<N>*>(row + Unit::at(u, half)) = encode(p.x[k], inv);
    *reinterpret_cast<Codes<N>*>(row + Unit::partner(u, half)) = encode(p.y[k], inv);
  }
}

// CTAs of the launch: first those of the blocks, `per` each, then those of the queries (kTokens tokens each). With FEW, a
// CTA has 8 of a block's (kv head, K or V), a warp each; else it goes through `heads` kv heads of the block's keys or
// values one after the other, the rows of the next on their way, all from one table of cosines.
template <typename Tin, int N, bool INTER, int D, bool FEW>
__global__ void __launch_bounds__(kQThreads, 4) append_q8_kernel(const AppendQ8Args A) {
  constexpr int kTokens = FEW ? 1 : 2;
  constexpr int kPer = D / (2 * N), kG = kPer < 32 ? kPer : 32, kU = kPer / kG;
  using Part = HeadPart<Tin, N, INTER, kU>;
  using Unit = RopeUnit<Tin, Tin, N, INTER>;
  __shared__ alignas(32) float w[2 * D];
  // cosines and sines: of the block's rows, or of the token
  __shared__ alignas(16) float2 cs[FEW ? 1 : kQMaxBlock][D / 2];
  const int tid = threadIdx.x, half = A.half, l = tid % kG;
  if ((int)blockIdx.x < A.block_ctas) {
    const int per = A.per, i = blockIdx.x / per, sub = blockIdx.x % per;
    BlockOf o;
    BlockPlace at;
    if (!find_block(A, i, blockIdx.x == 0, o)) return;
    if (!place_block(A, o, at)) return;
    if constexpr (FEW) {
      if (A.norm.k)
        for (int j = tid; j < D; j += kQThreads) w[j] = A.norm.k[j];
      __syncthreads();
      const int hk = sub * (kQThreads / 32) + tid / 32, lane = tid % 32;
      if (hk >= 2 * A.Hkv) return;
      const bool key = hk < A.Hkv;
      const int h = key ? hk : hk - A.Hkv;
      const Tin* src = static_cast<const Tin*>(key ? A.K : A.V) + h * D;
      const long long stride = key ? A.k_stride : A.v_stride;
      uint8_t* codes = (key ? A.K8 : A.V8) + (at.row + (size_t)h * at.row_step) * D;
      uint8_t* scale = (key ? A.Ks : A.Vs) + at.scale + (size_t)h * at.scale_step;
      const int before = o.r0 > 0 ? clamp_exp((int)*scale - 127) : kQMinExp;
      constexpr int kRows = 32 / kG;  // at a time
      Part part;
      auto form = [&](int r) {
        const bool has = r < o.r1;
        const int t = o.t0 + r - o.r0;
        if (has) part.load(src + t * stride, l, kG, kPer, half);
        part.widen_all(l, kG, has ? kPer : 0);
        if (key) {
          if (A.norm.k) part.norm(w, A.norm.eps, 1.f / D, l, kG, kPer, half);
          if (has) {
            const int pos = A.pos ? A.pos[t] : o.key0 + r;
            part.rotate(l, kG, half, [&](int u, float2(&c)[N]) {
#pragma unroll
              for (int j = 0; j < N; ++j) c[j] = fine_turn(pos, A.turns[u * N + j], A.magnitude);
            });
          }
        }
      };
      uint32_t amax = 0;
      for (int r = o.r0; r < o.r1; r += kRows) {
        form(r + lane / kG);
        amax = largest_of(part, amax);
      }
      const int e = max(exponent_of(__reduce_max_sync(0xffffffffu, amax)), before);
      if (o.r0 > 0 && e != before)  // the rows that the block had, to the new scale
        for (int u = lane; u < o.r0 * (D / 16); u += 32) recode(reinterpret_cast<uint4*>(codes) + u, power_of_two(before - e));
      const float inv = power_of_two(-e);
      for (int r = o.r0; r < o.r1; r += kRows) {
        if (o.r1 - o.r0 > kRows) form(r + lane / kG);  // (a single pass is still in registers)
        if (r + lane / kG < o.r1) write_codes(part, codes + (r + lane / kG) * D, inv, l, kG, half);
      }
      __syncwarp();  // (all lanes have read the scale)
      if (lane == 0) *scale = (uint8_t)(e + 127);
    } else {
      constexpr int kRows = kQThreads / kG, kPasses = (kQMaxBlock + kRows - 1) / kRows;
      __shared__ uint32_t s_amax[2];
      const int groups = per / 2;
      const bool key = sub < groups;
      const int h0 = (key ? sub : sub - groups) * A.heads, h1 = min(h0 + A.heads, A.Hkv);
      const long long stride = key ? A.k_stride : A.v_stride;
      const Tin* src = static_cast<const Tin*>(key ? A.K : A.V) + o.t0 * stride;
      const int rr = tid / kG;
      Part part[kPasses];
      auto load = [&](int h) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int r = rr + p * kRows;
          if (r >= o.r0 && r < o.r1) part[p].load(src + (r - o.r0) * stride + h * D, l, kG, kPer, half);
        }
      };
      load(h0);
      if (tid < 2) s_amax[tid] = 0;
      if (key) {
        for (int j = tid; j < (o.r1 - o.r0) * half; j += kQThreads) {
          const int r = o.r0 + j / half, k = j % half;
          cs[r][Unit::slot(k, half)] = fine_turn(A.pos ? A.pos[o.t0 + r - o.r0] : o.key0 + r, A.turns[k], A.magnitude);
        }
        if (A.norm.k)
          for (int j = tid; j < D; j += kQThreads) w[j] = A.norm.k[j];
      }
      __syncthreads();
      for (int h = h0; h < h1; ++h) {
        uint8_t* codes = (key ? A.K8 : A.V8) + (at.row + (size_t)h * at.row_step) * D;
        uint8_t* scale = (key ? A.Ks : A.Vs) + at.scale + (size_t)h * at.scale_step;
        const int before = o.r0 > 0 ? clamp_exp((int)*scale - 127) : kQMinExp;
        uint32_t amax = 0;
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int r = rr + p * kRows;
          const bool has = r >= o.r0 && r < o.r1;
          part[p].widen_all(l, kG, has ? kPer : 0);
          if (key && A.norm.k) part[p].norm(w, A.norm.eps, 1.f / D, l, kG, kPer, half);
          if (key && has) part[p].rotate_by(cs[r], l, kG, half);
          amax = largest_of(part[p], amax);
        }
        if (h + 1 < h1) load(h + 1);  // (the raw values have been widened)
        amax = __reduce_max_sync(0xffffffffu, amax);
        if (tid % 32 == 0) atomicMax(&s_amax[h & 1], amax);
        __syncthreads();
        const int e = max(exponent_of(s_amax[h & 1]), before);
        if (tid == 0) s_amax[(h + 1) & 1] = 0;  // (read by all before the second barrier of the head before)
        if (o.r0 > 0 && e != before)
          for (int u = tid; u < o.r0 * (D / 16); u += kQThreads)
            recode(reinterpret_cast<uint4*>(codes) + u, power_of_two(before - e));
        const float inv = power_of_two(-e);
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const int r = rr + p * kRows;
          if (r >= o.r0 && r < o.r1) write_codes(part[p], codes + r * D, inv, l, kG, half);
        }
        __syncthreads();  // all have read the scale, and the largest is cleared
        if (tid == 0) *scale = (uint8_t)(e + 127);
      }
    }
    return;
  }
  // queries: the first heads are on their way while the tokens' sequences are looked up
  __shared__ unsigned long long s_owner[kTokens];  // the token's first sequence and its position there
  const int t0 = (blockIdx.x - A.block_ctas) * kTokens, n_tok = min(kTokens, A.T - t0), step = kQThreads / kG;
  const Tin* src = static_cast<const Tin*>(A.Q) + t0 * A.q_stride;
  Part part[kTokens];
  auto load = [&](int h) {
#pragma unroll
    for (int j = 0; j < kTokens; ++j)
      if (j < n_tok && h < A.Hq) part[j].load(src + j * A.q_stride + (long long)h * D, l, kG, kPer, half);
  };
  load(tid / kG);
  if (tid < kTokens) s_owner[tid] = kRopeNone;
  if (A.norm.q)
    for (int j = tid; j < D; j += kQThreads) w[j] = A.norm.q[j];
  __syncthreads();
  for (int b = tid; b < A.B; b += kQThreads) {
    const int lo = A.cu_new[b], hi = A.cu_new[b + 1];
    if (lo < 0 || hi < lo || hi > A.T) continue;
#pragma unroll
    for (int j = 0; j < kTokens; ++j)
      if (j < n_tok && t0 + j >= lo && t0 + j < hi)
        atomicMin(&s_owner[j], (unsigned long long)b << 32 | (uint32_t)((unsigned)A.kv_len[b] + (unsigned)(t0 + j - lo)));
  }
  __syncthreads();
  for (int i = tid; i < kTokens * half; i += kQThreads) {
    const int j = kTokens == 1 ? 0 : i / half, k = i - j * half;
    if (j >= n_tok || s_owner[j] == kRopeNone) continue;
    cs[j][Unit::slot(k, half)] = fine_turn(A.pos ? A.pos[t0 + j] : (int)(uint32_t)s_owner[j], A.turns[k], A.magnitude);
  }
  __syncthreads();
  for (int h0 = 0; h0 < A.Hq; h0 += step) {  // (all lanes of a warp go round together)
    const int h = h0 + tid / kG;
#pragma unroll
    for (int j = 0; j < kTokens; ++j) {
      if (j >= n_tok) continue;
      part[j].widen_all(l, kG, h < A.Hq ? kPer : 0);
      if (A.norm.q) part[j].norm(w, A.norm.eps, 1.f / D, l, kG, kPer, half);
      if (s_owner[j] == kRopeNone || h >= A.Hq) continue;
      part[j].rotate_by(cs[j], l, kG, half);
      part[j].store(A.Qo + ((size_t)(t0 + j) * A.Hq + h) * D, l, kG, kPer, half);
    }
    load(h + step);
  }
}

// ---------------------------------------------------------------------------
// Read-back: packed row cu[b] + j is key start[b] + j of sequence b.
// ---------------------------------------------------------------------------
struct ReadQ8Args {
  const uint8_t *K8, *V8, *Ks, *Vs;
  const int32_t *cu, *start, *block_table;
  int T, B, Hkv, max_pages, page_size, n_pages, S_cap, block;
  uint16_t *K, *V;
  int wide;  // both aligned to 32 bytes
  int* status;
};
constexpr int kReadTokens = kQThreads / 32;  // of a CTA

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
  constexpr int kUnits = D / 16, kStep = 32 / kUnits;  // 16-byte units of a row; heads that a warp takes at a time
  const int c = tid % kUnits, j = tid / 32;            // (a warp a token: what it writes is one piece)
  if (j >= n_tok || s_row[j] < 0) return;
  const long long row = s_row[j], scale = s_scale[j];
  // heads of K, then of V. (One load in flight for each thread, and 32-byte stores: 160 MB of codes in 117 us, 93% of the
  // copy rate; 16-byte stores 123; two loads 138, four 165: rows of different heads lie far apart.)
  const int heads = 2 * A.Hkv;
  for (int hk = tid % 32 / kUnits; hk < heads; hk += kStep) {
    const int h = hk < A.Hkv ? hk : hk - A.Hkv;
    const uint4 v = __ldg(reinterpret_cast<const uint4*>((hk < A.Hkv ? A.K8 : A.V8) + (row + (long long)h * rows) * D) + c);
    const float f = power_of_two(clamp_exp((int)__ldg((hk < A.Hkv ? A.Ks : A.Vs) + scale + (long long)h * scales) - 127));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float y[16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 a = of_e4m3x2((uint16_t)w[i]), b = of_e4m3x2((uint16_t)(w[i] >> 16));
      y[4 * i] = a.x * f;
      y[4 * i + 1] = a.y * f;
      y[4 * i + 2] = b.x * f;
      y[4 * i + 3] = b.y * f;
    }
    Pack<uint16_t, 16> p;
    narrow(y, p);
    uint4* dst = reinterpret_cast<uint4*>((hk < A.Hkv ? A.K : A.V) + ((size_t)(t0 + j) * A.Hkv + h) * D) + 2 * c;
    const uint4 *lo = reinterpret_cast<const uint4*>(p.v), *hi = lo + 1;
    if (A.wide) {
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(lo->x), "r"(lo->y), "r"(lo->z),
                   "r"(lo->w), "r"(hi->x), "r"(hi->y), "r"(hi->z), "r"(hi->w)
                   : "memory");
    } else {
      dst[0] = *lo;
      dst[1] = *hi;
    }
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
  // passes of equal size over the heads, of up to 256 threads
  const int G = head_lanes(d / (2 * (vec ? N : 1))), H = Hq + Hk, most = kQThreads / G, passes = (H + most - 1) / most;
  const int threads = std::max(64, ((H + passes - 1) / passes * G + 31) / 32 * 32);
  auto launch = [&](auto kernel) { kernel<<<n_tokens, threads, 0, stream>>>(a); };
  constexpr int kWideU = 256 / N / 32 > 1 ? 256 / N / 32 : 1;  // units of a lane: heads of 512
  if (!vec) launch(interleaved ? norm_rope_kernel<T, 1, true, 8> : norm_rope_kernel<T, 1, false, 8>);
  else if (d <= 64 * N) launch(interleaved ? norm_rope_kernel<T, N, true, 1> : norm_rope_kernel<T, N, false, 1>);
  else launch(interleaved ? norm_rope_kernel<T, N, true, kWideU> : norm_rope_kernel<T, N, false, kWideU>);
  return cudaGetLastError();
}
template cudaError_t launch_norm_rope<float>(const float*, long long, const int32_t*, const float*, float, const float*,
                                             const float*, float, int, int, int, int, int, int, float*, long long,
                                             cudaStream_t);
template cudaError_t launch_norm_rope<uint16_t>(const uint16_t*, long long, const int32_t*, const float*, float,
                                                const float*, const float*, float, int, int, int, int, int, int,
                                                uint16_t*, long long, cudaStream_t);

// Few new tokens (four of a sequence on average, at most): a warp for each (block, kv head, K or V). Else CTAs that go
// through a block's heads with one table of cosines, as many heads each as leave every SM four of them. (8587 tokens of 28
// + 2 x 4 heads, with their read-back: 41 us, 48 with a head each. CTAs that go through keys, values and queries of a block:
// 45; the blocks' CTAs spread among the queries': 42.)
template <typename T, int N, int D>
static cudaError_t launch_append_n(AppendQ8Args a, int interleaved, cudaStream_t stream) {
  const bool few = a.T <= 4ll * a.B;
  const long long units = 2ll * a.Hkv * a.n_blocks;
  a.heads = (int)std::max(1ll, std::min((long long)a.Hkv, units / (4 * num_sms_current())));
  a.per = few ? (2 * a.Hkv + kQThreads / 32 - 1) / (kQThreads / 32) : 2 * ((a.Hkv + a.heads - 1) / a.heads);
  const long long tokens = few ? 1 : 2, ctas = (long long)a.per * a.n_blocks;
  const long long grid = ctas + (a.Qo ? (a.T + tokens - 1) / tokens : 0);
  if (grid > 0x7fffffffll) return cudaErrorInvalidValue;
  a.block_ctas = (int)ctas;
  auto launch = [&](auto kernel) { kernel<<<(int)grid, kQThreads, 0, stream>>>(a); };
  if (few) launch(interleaved ? append_q8_kernel<T, N, true, D, true> : append_q8_kernel<T, N, false, D, true>);
  else launch(interleaved ? append_q8_kernel<T, N, true, D, false> : append_q8_kernel<T, N, false, D, false>);
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
                 Q ? Hq : 0, Hkv, rot / 2, max_pages, page_size, n_pages, S_cap, block, 0, 0, 0, 0, Qo, K8, V8, Ks, Vs, status};
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
                     K, V, (reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) % 32 == 0, status};
  const int grid = (n_tokens + kReadTokens - 1) / kReadTokens;
  if (d == 128) read_q8_kernel<128><<<grid, kQThreads, 0, stream>>>(a);
  else read_q8_kernel<64><<<grid, kQThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace libraspec
