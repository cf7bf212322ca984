// Device parts that the scan's kernels share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "scan.hpp"
#include "seq_dev.cuh"

namespace mebptt {
namespace seq {

// exp(dt A) of two states, A in units of log 2
__device__ __forceinline__ pair decay2(pair dt, pair A) {
  const float2 x = unpack2(mul2(dt, A));
  return pack2(ex2(x.x), ex2(x.y));
}

// Four states of a lane.
struct Four {
  pair a, b;
};
__device__ __forceinline__ Four lds4(const float* p) {
  const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(p);
  return Four{v.x, v.y};
}
__device__ __forceinline__ void st4(float* p, const Four& f) {
  *reinterpret_cast<ulonglong2*>(p) = make_ulonglong2(f.a, f.b);
}
// Four of `states` values of a row (channel) from n0 on, zeros past the last.
__device__ __forceinline__ Four load_states(const float* row, int n0, int states, bool vec) {
  if (vec && n0 + 4 <= states) return lds4(row + n0);
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = n0 + i < states ? row[n0 + i] : 0.f;
  return Four{pack2(f[0], f[1]), pack2(f[2], f[3])};
}
__device__ __forceinline__ void store_states(float* row, int n0, int states, bool vec, const Four& v) {
  if (vec && n0 + 4 <= states) {
    st4(row + n0, v);
    return;
  }
  const float2 x = unpack2(v.a), y = unpack2(v.b);
  const float f[4] = {x.x, x.y, y.x, y.y};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (n0 + i < states) row[n0 + i] = f[i];
}

// Where (channel, step) of a tile lies in shared memory: steps of a channel together, so that a lane loads four at once; groups of
// four steps are exchanged by channel group, so that neither the walk along steps nor that along channels meets a bank twice.
template <int STEPS>
__device__ __forceinline__ int at(int c, int step) {
  return c * (STEPS + 4) + ((((step >> 2) ^ (2 * (c >> 3))) & (STEPS / 4 - 1)) << 2 | (step & 3));
}
template <int STEPS>
__device__ __forceinline__ float4 four_steps(const float* tile, int c, int step) {
  return *reinterpret_cast<const float4*>(tile + at<STEPS>(c, step));
}

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

__device__ __forceinline__ float step_size(float pre, int soft) { return soft ? softplus(pre) : pre; }

// decay over a whole segment applied to a carried value; a zero stays one whatever the factor
__device__ __forceinline__ pair carry2(pair A, float dts, pair v, pair end) {
  const float2 p = unpack2(decay2(both(dts), A)), x = unpack2(v), e = unpack2(end);
  return pack2(x.x == 0.f ? e.x : fmaf(p.x, x.x, e.x), x.y == 0.f ? e.y : fmaf(p.y, x.y, e.y));
}

}  // namespace seq
}  // namespace mebptt
