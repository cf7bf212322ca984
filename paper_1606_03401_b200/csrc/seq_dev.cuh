// Device helpers of the operators over sequences (convolution, scan, loss over a vocabulary): eight elements of a row at a
// time in either storage type, and the elementwise functions in 32 bits.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstring>

namespace mebptt {
namespace seq {

using bf16 = __nv_bfloat16;

template <class T>
__device__ __forceinline__ float to_f(T v);
template <>
__device__ __forceinline__ float to_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f<bf16>(bf16 v) { return __bfloat162float(v); }

template <class T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16(v); }   // to nearest: half a step of the type

// N consecutive elements (4 to 32 bytes of them) as they lie in memory.
template <class T, int N>
struct Raw {
  static constexpr int W = N * (int)sizeof(T) / 4;   // 32-bit words
  uint32_t w[W];
};

// `n` of N elements at p, zeros in place of the rest.  whole: all are there and p is aligned to their size (to 16 bytes at most).
template <int N, class T>
__device__ __forceinline__ Raw<T, N> load_raw(const T* p, int n, bool whole) {
  Raw<T, N> r;
  if (whole) {
    if constexpr (sizeof r == 4) {
      r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (sizeof r == 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      r.w[0] = v.x; r.w[1] = v.y;
    } else {
#pragma unroll
      for (int q = 0; q < (int)sizeof r / 16; ++q) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[q];
        r.w[4 * q] = v.x; r.w[4 * q + 1] = v.y; r.w[4 * q + 2] = v.z; r.w[4 * q + 3] = v.w;
      }
    }
  } else {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = i < n ? p[i] : from_f<T>(0.f);
    memcpy(&r, e, sizeof r);
  }
  return r;
}
template <class T, int N>
__device__ __forceinline__ Raw<T, N> raw_zeros() {
  Raw<T, N> r;
#pragma unroll
  for (int q = 0; q < Raw<T, N>::W; ++q) r.w[q] = 0;
  return r;
}
template <int N>
__device__ __forceinline__ void unpack(const Raw<bf16, N>& r, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    f[2 * i] = __uint_as_float(r.w[i] << 16);
    f[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
  }
}
template <int N>
__device__ __forceinline__ void unpack(const Raw<float, N>& r, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = __uint_as_float(r.w[i]);
}
template <int N, class T>
__device__ __forceinline__ void store_n(T* p, const float (&f)[N], int n, bool whole) {
  if (whole) {
    T e[N];
#pragma unroll
    for (int i = 0; i < N; ++i) e[i] = from_f<T>(f[i]);
    Raw<T, N> r;
    memcpy(&r, e, sizeof r);
    if constexpr (sizeof r == 4) {
      *reinterpret_cast<uint32_t*>(p) = r.w[0];
    } else if constexpr (sizeof r == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
    } else {
#pragma unroll
      for (int q = 0; q < (int)sizeof r / 16; ++q)
        reinterpret_cast<uint4*>(p)[q] = make_uint4(r.w[4 * q], r.w[4 * q + 1], r.w[4 * q + 2], r.w[4 * q + 3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = from_f<T>(f[i]);
  }
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float sigmoid(float x) { return rcp(1.f + ex2(-kLog2e * x)); }

// log(1 + e^x) = max(x, 0) + log1p(e^{-|x|}), and log1p(e) = 2 atanh(e / (2 + e)) by its series: the argument is at most 1/3, so
// eight terms leave 2e-9 of the value, and a small e keeps its relative precision.
__device__ __forceinline__ float softplus(float x) {
  const float e = ex2(-kLog2e * fabsf(x));
  const float t = e * rcp(2.f + e), q = t * t;
  float p = 1.f / 15.f;
  p = fmaf(p, q, 1.f / 13.f);
  p = fmaf(p, q, 1.f / 11.f);
  p = fmaf(p, q, 1.f / 9.f);
  p = fmaf(p, q, 1.f / 7.f);
  p = fmaf(p, q, 1.f / 5.f);
  p = fmaf(p, q, 1.f / 3.f);
  p = fmaf(p, q, 1.f);
  return fmaf(2.f * t, p, fmaxf(x, 0.f));   // a NaN comes through t
}

// Two floats in a register pair: one instruction works on both.
using pair = unsigned long long;
__device__ __forceinline__ pair pack2(float lo, float hi) {
  pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ float2 unpack2(pair v) {
  float2 f;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(v));
  return f;
}
__device__ __forceinline__ pair mul2(pair a, pair b) {
  pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ pair add2(pair a, pair b) {
  pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ pair fma2(pair a, pair b, pair c) {
  pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ pair both(float v) { return pack2(v, v); }
__device__ __forceinline__ float sum2(pair v) {
  const float2 f = unpack2(v);
  return f.x + f.y;
}
__device__ __forceinline__ pair sigmoid2(pair x) {
  const float2 e = unpack2(mul2(x, both(-kLog2e)));
  const float2 d = unpack2(add2(pack2(ex2(e.x), ex2(e.y)), both(1.f)));
  return pack2(rcp(d.x), rcp(d.y));
}
__device__ __forceinline__ pair softplus2(pair x) {
  const float2 f = unpack2(x);
  const float2 y = unpack2(mul2(pack2(fabsf(f.x), fabsf(f.y)), both(-kLog2e)));
  const pair e = pack2(ex2(y.x), ex2(y.y));
  const float2 w = unpack2(add2(e, both(2.f)));
  const pair t = mul2(e, pack2(rcp(w.x), rcp(w.y))), q = mul2(t, t);
  pair p = both(1.f / 15.f);
  p = fma2(p, q, both(1.f / 13.f));
  p = fma2(p, q, both(1.f / 11.f));
  p = fma2(p, q, both(1.f / 9.f));
  p = fma2(p, q, both(1.f / 7.f));
  p = fma2(p, q, both(1.f / 5.f));
  p = fma2(p, q, both(1.f / 3.f));
  p = fma2(p, q, both(1.f));
  return fma2(add2(t, t), p, pack2(fmaxf(f.x, 0.f), fmaxf(f.y, 0.f)));
}
// pairs of N elements as they lie in memory
template <int N>
__device__ __forceinline__ void unpack_pairs(const Raw<bf16, N>& r, pair (&f)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) f[i] = pack2(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xffff0000u));
}
template <int N>
__device__ __forceinline__ void unpack_pairs(const Raw<float, N>& r, pair (&f)[N / 2]) {
#pragma unroll
  for (int i = 0; i < N / 2; ++i) f[i] = pack2(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
}
template <int N, class T>
__device__ __forceinline__ void store_pairs(T* p, const pair (&f)[N / 2], int n, bool whole) {
  float g[N];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float2 v = unpack2(f[i]);
    g[2 * i] = v.x; g[2 * i + 1] = v.y;
  }
  store_n<N>(p, g, n, whole);
}

__device__ __forceinline__ int row_steps(const int32_t* lengths, int b, int64_t t) {
  if (!lengths) return (int)t;
  const int n = lengths[b];
  return n < 0 ? 0 : n > (int)t ? (int)t : n;
}

}  // namespace seq
}  // namespace mebptt
