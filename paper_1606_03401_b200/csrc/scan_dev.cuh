// Device parts that the scan's kernels share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "scan.hpp"
#include "seq_dev.cuh"

namespace mebptt {
namespace seq {

// exp(dt A) of two states, A in units of log 2.  The instruction's results are 2e-8 too small on average (measured between -0.5
// and -0.002, where a state lasts for hundreds of steps and the error of its decay is raised to their power); the constant takes
// that back, and leaves exp(0) = 1.
constexpr float kDecayUp = 2.2e-8f;
__device__ __forceinline__ pair decay2(pair dt, pair A) {
  const float2 x = unpack2(fma2(dt, A, both(kDecayUp)));
  return pack2(ex2(x.x), ex2(x.y));
}

constexpr int PER_LANE = 8;     // states of a lane, as four pairs
constexpr int FOLD = 4;         // segments whose ends are loaded together

// Pair i of a lane's states lies here, from the first of them on.  `turn` exchanges pairs: bit 1 the halves of four states, bit 0 the
// pairs of a half (lanes with other channels hold their states in another order, see sum_channels).
__device__ __forceinline__ int pair_at(int i, int turn) { return 2 * (i ^ turn); }

__device__ __forceinline__ pair load_pair(const float* row, int n0, int states, bool vec) {
  if (vec && n0 + 2 <= states) return *reinterpret_cast<const pair*>(row + n0);
  return pack2(n0 < states ? row[n0] : 0.f, n0 + 1 < states ? row[n0 + 1] : 0.f);
}
__device__ __forceinline__ void store_pair(float* row, int n0, int states, bool vec, pair v) {
  if (vec && n0 + 2 <= states) {
    *reinterpret_cast<pair*>(row + n0) = v;
    return;
  }
  const float2 f = unpack2(v);
  if (n0 < states) row[n0] = f.x;
  if (n0 + 1 < states) row[n0 + 1] = f.y;
}
// A lane's states out of a row of `states` values (zeros past the last), and back.
__device__ __forceinline__ void load_states(const float* row, int l, int states, bool vec, pair (&s)[4]) {
  if (vec && PER_LANE * (l + 1) <= states) {
    const ulonglong2* const p = reinterpret_cast<const ulonglong2*>(row + PER_LANE * l);
    const ulonglong2 a = p[0], b = p[1];
    s[0] = a.x; s[1] = a.y; s[2] = b.x; s[3] = b.y;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = load_pair(row, PER_LANE * l + 2 * i, states, vec);
}
__device__ __forceinline__ void store_states(float* row, int l, int states, bool vec, const pair (&s)[4]) {
  if (vec && PER_LANE * (l + 1) <= states) {
    ulonglong2* const p = reinterpret_cast<ulonglong2*>(row + PER_LANE * l);
    p[0] = make_ulonglong2(s[0], s[1]);
    p[1] = make_ulonglong2(s[2], s[3]);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) store_pair(row, PER_LANE * l + 2 * i, states, vec, s[i]);
}

// Where (channel, step) of a tile lies in shared memory: steps of a channel together, so that a lane loads four at once, and groups of
// eight channels shifted against one another, so that neither the walk along steps nor that along channels meets a bank twice.
template <int STEPS, int CH>
struct Tile {
  static constexpr int SKEW = 256 / CH < 4 ? 4 : 256 / CH;
  static constexpr int FLOATS = CH * (STEPS + 4) + CH / 8 * SKEW;
  static __device__ __forceinline__ int at(int c, int step) { return c * (STEPS + 4) + (c >> 3) * SKEW + step; }
  static __device__ __forceinline__ void four(const float* tile, int c, int step, float (&v)[4]) {
    const float4 f = *reinterpret_cast<const float4*>(tile + at(c, step));
    v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
  }
};

// Sums of v[0..3] (four steps) over the LANES lanes of a channel.  With four lanes or more, lane l gets step l % 4 in v[0]; with two,
// lane l gets steps 2 l and 2 l + 1; with one, all four.
template <int LANES>
__device__ __forceinline__ void sum_lanes(float (&v)[4], int l) {
  if constexpr (LANES == 2) {
    const bool hi = l & 1;
    const float s0 = hi ? v[0] : v[2], s1 = hi ? v[1] : v[3];
    v[0] = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, s0, 1);
    v[1] = (hi ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, s1, 1);
  } else if constexpr (LANES >= 4) {
    const bool hi = l & 2, odd = l & 1;
    const float s0 = hi ? v[0] : v[2], s1 = hi ? v[1] : v[3];
    v[0] = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, s0, 2);
    v[1] = (hi ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, s1, 2);
    const float s = odd ? v[0] : v[1];
    v[0] = (odd ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, s, 1);
#pragma unroll
    for (int m = 4; m < LANES; m *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
  }
}
template <int LANES>
constexpr int steps_of_lane = LANES >= 4 ? 1 : 4 / LANES;
template <int LANES>
__device__ __forceinline__ int first_step(int l) { return LANES >= 4 ? (l & 3) : l * steps_of_lane<LANES>; }
// what sum_lanes left to a lane, to the places of its steps
template <int LANES>
__device__ __forceinline__ void put_steps(float* at, int l, const float (&v)[4]) {
  float* const p = at + first_step<LANES>(l);
  if constexpr (LANES == 1) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else if constexpr (LANES == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
  else *p = v[0];
}

__device__ __forceinline__ float step_size(float pre, int soft) { return soft ? softplus(pre) : pre; }

__device__ __forceinline__ void async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void async8(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
// N elements into shared memory, asked for where they load as one, else loaded.
template <int N, class T>
__device__ __forceinline__ void fetch_n(uint8_t* to, const T* from, int n, bool whole) {
  if (whole) {
    if constexpr (N * sizeof(T) == 8) {
      async8(to, from);
    } else {
#pragma unroll
      for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) async16(to + 16 * i, reinterpret_cast<const uint8_t*>(from) + 16 * i);
    }
  } else {
    const Raw<T, N> r = load_raw<N>(from, n, false);
    memcpy(to, &r, sizeof r);
  }
}
template <class T, int N>
__device__ __forceinline__ Raw<T, N> fetched(const uint8_t* from) {
  return load_raw<N>(reinterpret_cast<const T*>(from), N, true);
}

// Decay over a whole segment applied to a carried value, as its root twice, since the factor may lie past the type's range where the
// product does not (a state that has all but faded and then grows, or the other way round; step by step it never leaves the range).
// A zero stays one whatever the factor.
__device__ __forceinline__ pair carry2(pair A, float dts, pair v, pair end) {
  const float2 h = unpack2(fma2(both(0.5f * dts), A, both(kDecayUp)));
  const pair root = pack2(ex2(h.x), ex2(h.y));
  const float2 x = unpack2(v), r = unpack2(fma2(root, mul2(root, v), end)), e = unpack2(end);
  return pack2(x.x == 0.f ? e.x : r.x, x.y == 0.f ? e.y : r.y);
}
// sum over a lane's states of x y
__device__ __forceinline__ float dot(const pair (&x)[4], const pair (&y)[4]) {
  return sum2(add2(fma2(x[0], y[0], mul2(x[1], y[1])), fma2(x[2], y[2], mul2(x[3], y[3]))));
}
// a lane's eight values of a row in shared memory
__device__ __forceinline__ void lds8(const float* p, pair (&v)[4]) {
  const ulonglong2 a = *reinterpret_cast<const ulonglong2*>(p), b = *reinterpret_cast<const ulonglong2*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
}

}  // namespace seq
}  // namespace mebptt
