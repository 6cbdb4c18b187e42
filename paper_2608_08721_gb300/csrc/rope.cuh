// Rotation of a head's pairs, shared by the kernels that rotate: the angle of a position, accesses of N elements, and
// a head in units of them. (What a rotation computes, and why so, is written in rope.cu.)
#pragma once
#include <type_traits>

#include "common.cuh"

namespace libraspec {

constexpr int kRopeMaxPairs = LIBRASPEC_ROPE_MAX_DIM / 2;
constexpr unsigned long long kRopeNone = ~0ull;

// cos and sin of a pair at position pos, times the magnitude. The position in two parts that are binary32 numbers each.
__device__ __forceinline__ float2 rope_turn(int pos, float2 f, float magnitude) {
  const float hi = (float)(pos & ~255), lo = (float)(pos & 255);
  const float p = __fmul_rn(hi, f.x), q = __fmul_rn(lo, f.x);
  const float e = __fmaf_rn(hi, f.x, -p) + __fmaf_rn(lo, f.x, -q);
  const float r = ((p - rintf(p)) + (q - rintf(q))) + (e + __fmaf_rn(hi, f.y, lo * f.y));
  float s, c;
  sincospif(2.f * r, &s, &c);
  return make_float2(c * magnitude, s * magnitude);
}

// N consecutive elements as one access of N * sizeof(T) bytes
template <typename T, int N>
struct alignas(sizeof(T) * N) Pack {
  T v[N];
};

template <int N>
__device__ __forceinline__ void widen(const Pack<float, N>& a, float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = a.v[i];
}
template <int N>
__device__ __forceinline__ void widen(const Pack<uint16_t, N>& a, float (&x)[N]) {
  if constexpr (N == 1) {
    x[0] = __uint_as_float((uint32_t)a.v[0] << 16);
  } else {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(a.v);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      x[2 * i] = bf16_lo(w[i]);
      x[2 * i + 1] = bf16_hi(w[i]);
    }
  }
}
template <int N>
__device__ __forceinline__ void narrow(const float (&x)[N], Pack<float, N>& a) {
#pragma unroll
  for (int i = 0; i < N; ++i) a.v[i] = x[i];
}
template <int N>
__device__ __forceinline__ void narrow(const float (&x)[N], Pack<uint16_t, N>& a) {
  if constexpr (N == 1) {
    a.v[0] = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
  } else {
    __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(a.v);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
  }
}
template <typename Tin, typename Tout, int N>
__device__ __forceinline__ Pack<Tout, N> convert(const Pack<Tin, N>& a) {
  if constexpr (std::is_same<Tin, Tout>::value) {
    return a;
  } else {
    float x[N];
    widen(a, x);
    Pack<Tout, N> r;
    narrow(x, r);
    return r;
  }
}

// A head as units: N elements of the first half of the rotated part with the N they pair with (half layout), or 2N
// consecutive ones (interleaved), then 2N at a time of the part that is only copied.
template <typename Tin, typename Tout, int N, bool INTER>
struct RopeUnit {
  Pack<Tin, N> a, b;
  __device__ __forceinline__ void load(const Tin* src, int u, int half) {
    a = *reinterpret_cast<const Pack<Tin, N>*>(src + at(u, half));
    b = *reinterpret_cast<const Pack<Tin, N>*>(src + partner(u, half));
  }
  // cs: cosine and sine of the token's pairs; turns: the head is a query's or a key's
  __device__ __forceinline__ void store(Tout* dst, bool turns, int u, int half, const float2* cs) const {
    Pack<Tout, N> p, q;
    if (u * N >= half || !turns) {
      p = convert<Tin, Tout, N>(a);
      q = convert<Tin, Tout, N>(b);
    } else {
      float x[N], y[N], v[N], w[N];
      widen(a, x);
      widen(b, y);
      float2 t[N];
      if constexpr (N == 1) {
        t[0] = cs[u];
      } else {
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          const float4 two = *reinterpret_cast<const float4*>(cs + slot(u * N + k, half));
          t[k] = make_float2(two.x, two.y);
          t[k + 1] = make_float2(two.z, two.w);
        }
      }
      if constexpr (INTER && N > 1) {  // pairs (x0, x1), (x2, x3) ..., then those of y
#pragma unroll
        for (int k = 0; k < N; k += 2) {
          turn(x[k], x[k + 1], t[k / 2], v[k], v[k + 1]);
          turn(y[k], y[k + 1], t[N / 2 + k / 2], w[k], w[k + 1]);
        }
      } else {  // pairs (x0, y0), (x1, y1) ...
#pragma unroll
        for (int k = 0; k < N; ++k) turn(x[k], y[k], t[k], v[k], w[k]);
      }
      narrow(v, p);
      narrow(w, q);
    }
    *reinterpret_cast<Pack<Tout, N>*>(dst + at(u, half)) = p;
    *reinterpret_cast<Pack<Tout, N>*>(dst + partner(u, half)) = q;
  }
  // Where pair i's cosine and sine lie: two pairs of a unit side by side, then the same two of its neighbours, so that
  // neighbouring threads read neighbouring 16 bytes of shared memory. (In the pairs' own order, 8 N bytes apart, they
  // meet in the same banks: 34.7 us for 8587 bf16 tokens of 36 heads, 29.8 so. Units of four fp32 elements gain
  // nothing: 27.1 and 28.1 for 8192 tokens of 48 heads of 64.)
  __device__ static __forceinline__ int slot(int i, int half) {
    if (N == 1) return i;
    const int e = i % N;
    return ((e / 2) * (half / N) + i / N) * 2 + (e & 1);
  }
  // (past the rotated part both layouts take 2N consecutive elements)
  __device__ static __forceinline__ int at(int u, int half) { return INTER || u * N >= half ? 2 * u * N : u * N; }
  __device__ static __forceinline__ int partner(int u, int half) {
    return INTER || u * N >= half ? (2 * u + 1) * N : half + u * N;
  }
  __device__ static __forceinline__ void turn(float x0, float x1, float2 t, float& y0, float& y1) {
    y0 = fmaf(x0, t.x, -x1 * t.y);
    y1 = fmaf(x0, t.y, x1 * t.x);
  }
};

}  // namespace libraspec
