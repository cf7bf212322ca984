// Selective state space scan, backward.
//
// A block owns 128 / LANES channels of one row and walks a segment's tiles of 32 steps from the last to the first; LANES lanes share
// a channel, eight states each, two to an instruction.  States are not kept but every `spacing` steps: eight steps at a time are
// run forwards from the state before them, with the decays and the states of the eight steps in registers, and then backwards.
// Where states are kept further apart, a tile first runs forwards once more to have the state before each of its eights (one
// exponential more for each state and step).
//
// Sums go three ways.  Over the states of a channel (v, g B, A a s g): the lanes of a channel, four steps at a time, each lane ending
// with steps of its own.  Over channels (dB, dC): halving exchanges among the lanes of a warp with the same states, then the
// block's warps through shared memory, then the blocks of a group in a second kernel.  Over time (dA, dskip, ddelta_bias): a sum per
// tile added to a sum of tiles, then rows and segments in the second kernel.  The order is fixed.
//
// An exchange sends the half of the values that the other lane keeps, which takes a selection for each value and side, unless lanes
// that keep the upper half hold it where the others hold the lower one.  So lanes hold their states in one of four orders
// (`turn`), B and C lie in shared memory in all four, and the first two exchanges need no selections.
//
// Bound by instruction issue: two exponentials and some 24 other instructions for eight states of a step, and two shuffles.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.hpp"
#include "scan.hpp"
#include "scan_dev.cuh"
#include "scan_kernels.hpp"

namespace mebptt {
namespace seq {

namespace {

constexpr int EIGHT = 8, NT = 128;

template <int LANES>
struct Shape {
  static constexpr int CH = NT / LANES, NP = PER_LANE * LANES, WARPS = NT / 32;
  static constexpr int CHUNKS = TILE * CH / 8 / NT > 0 ? TILE * CH / 8 / NT : 1;    // groups of eight channels a thread, in the elementwise part
  using At = Tile<TILE, CH>;
  static constexpr int ORDERS = 4;                                                  // of B and C
  static constexpr int ROW = ORDERS * NP;                                           // of B or C, of a step
  static constexpr int RED = WARPS * EIGHT * 2 * NP;                                // sums of one eight, by warp
  // planes of the tile, B and C, sums, and the channels' bias and skip; states before the eights of a tile if they are not kept
  static constexpr int FLOATS = 4 * At::FLOATS + TILE * 2 * ROW + 2 * RED + 2 * CH + NT * PER_LANE;
  static constexpr int STARTS = 3 * NT * PER_LANE;
};

// Sums of dB and dC (eight values each) over the 32 / LANES lanes with the same states.  Lanes halve the values among them as long as
// there are any to halve.  The lane with bits 16 and 8 of its number set in `turn` ends with the first pair of its own order;
// of that, lanes with four or fewer to a channel keep dB or dC (bit 4), with two or fewer one element (bit 2).
template <int LANES>
__device__ __forceinline__ void sum_channels(pair (&b)[4], pair (&c)[4], int lane) {
  auto other = [](pair v, int m) {
    const float2 f = unpack2(v);
    return pack2(__shfl_xor_sync(0xffffffffu, f.x, m), __shfl_xor_sync(0xffffffffu, f.y, m));
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    b[i] = add2(b[i], other(b[i + 2], 16));
    c[i] = add2(c[i], other(c[i + 2], 16));
  }
  b[0] = add2(b[0], other(b[1], 8));
  c[0] = add2(c[0], other(c[1], 8));
  if constexpr (LANES <= 4) {
    const bool hi = lane & 4;
    b[0] = add2(hi ? c[0] : b[0], other(hi ? b[0] : c[0], 4));
  }
  if constexpr (LANES <= 2) {
    const float2 f = unpack2(b[0]);
    const bool hi = lane & 2;
    float v = (hi ? f.y : f.x) + __shfl_xor_sync(0xffffffffu, hi ? f.x : f.y, 2);
    if constexpr (LANES == 1) v += __shfl_xor_sync(0xffffffffu, v, 1);
    b[0] = pack2(v, 0.f);
  }
}
// where they go: [dB, dC][NP]
template <int LANES>
__device__ __forceinline__ void put_channels(float* at, const pair (&b)[4], const pair (&c)[4], int lane, int l, int turn) {
  constexpr int NP = PER_LANE * LANES;
  float* const p = at + PER_LANE * l + 2 * turn;
  if constexpr (LANES == 8) {
    *reinterpret_cast<pair*>(p) = b[0];
    *reinterpret_cast<pair*>(p + NP) = c[0];
  } else if constexpr (LANES == 4) {
    *reinterpret_cast<pair*>(p + (lane & 4 ? NP : 0)) = b[0];
  } else {
    p[(lane & 4 ? NP : 0) + (lane & 2 ? 1 : 0)] = unpack2(b[0]).x;     // (with one lane a channel two lanes store the same)
  }
}

__device__ __forceinline__ void load_turned(const float* row, int l, int turn, int states, bool vec, pair (&s)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = load_pair(row, PER_LANE * l + pair_at(i, turn), states, vec);
}

template <class T, int LANES, bool GATE>
__global__ void __launch_bounds__(NT, 3) scan_bwd(const ScanArgs a) {
  using S = Shape<LANES>;
  using At = typename S::At;
  constexpr int CH = S::CH, NP = S::NP, WARPS = S::WARPS, CHUNKS = S::CHUNKS;
  extern __shared__ __align__(16) float sm[];
  float* const s_dt = sm;                         // dt
  float* const s_x = s_dt + At::FLOATS;           // dt u, then the sums over states of g B, then dv u
  float* const s_dv = s_x + At::FLOATS;           // dv, then of A a s g, then ddelta
  float* const s_v = s_dv + At::FLOATS;           // of C s
  float* const s_bc = s_v + At::FLOATS;           // [TILE][B, C][two halves of a lane's states][orders][LANES][4]
  float* const s_red = s_bc + TILE * 2 * S::ROW;  // [2][WARPS][EIGHT][2 NP]
  float* const s_dA = s_red + 2 * S::RED;         // [NT][8]: sums of the tiles so far
  float* const s_bias = s_dA + NT * PER_LANE;     // [CH]
  float* const s_skip = s_bias + CH;              // [CH]
  float* const s_start = s_skip + CH;             // [3][NT][8]: states before the eights of a tile but the first

  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, b = blockIdx.y, seg = blockIdx.z;
  const int g = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks, base = block * CH;
  const int d0 = g * a.gchannels + base;
  const int live = min(CH, a.gchannels - base);
  const int n = row_steps(a.lengths, b, a.t);
  const int first = seg * a.segment, last = min(first + a.segment, a.t);

  const T* const Bm = (const T*)a.B + (int64_t)b * a.pb.row + g * a.states;
  const T* const Cm = (const T*)a.C + (int64_t)b * a.pc.row + g * a.states;

  const int c = tid / LANES, l = tid % LANES;
  const int turn = (lane & 16 ? 2 : 0) | (lane & 8 ? 1 : 0);
  const float* const my_bc = s_bc + (turn * LANES + l) * 4;    // this lane's first half of a row; the second one 16 LANES floats on
  const bool mine = c < live;
  const int d = d0 + c;
  pair A[4] = {}, carry[4] = {};                  // A in units of log 2; carry: what later steps hand down, a_{k+1} g_{k+1}
  const int64_t place = ((int64_t)b * a.channels + d) * NP, row = ((int64_t)b * a.channels + d) * a.states;
  const int64_t layer = (int64_t)a.batch * a.channels * NP;
  if (mine) {
    load_turned(a.A + (int64_t)d * a.states, l, turn, a.states, a.vec_s, A);
#pragma unroll
    for (int i = 0; i < 4; ++i) A[i] = mul2(A[i], both(kLog2e));
    if (a.ds_out) load_turned(a.ds_out + row, l, turn, a.states, a.vec_s, carry);
    for (int j = a.segments - 1; j > seg; --j) {
      pair e[4];
      load_turned(a.ends + (j + 1) * layer + place, l, turn, NP, true, e);
      const float dts = a.dts[((int64_t)j * a.batch + b) * a.channels + d];
#pragma unroll
      for (int i = 0; i < 4; ++i) carry[i] = carry2(A[i], dts, carry[i], e[i]);
    }
  }
  for (int i = 0; i < PER_LANE; ++i) s_dA[tid * PER_LANE + i] = 0.f;
  for (int i = tid; i < CH; i += NT) {
    s_bias[i] = a.bias && i < live ? a.bias[d0 + i] : 0.f;
    s_skip[i] = a.skip && i < live ? a.skip[d0 + i] : 0.f;
  }
  float dskip = 0.f, dbias = 0.f;

  // eight channels of a step, in the elementwise parts
  struct Chunk {
    int ec, es, en;
    bool in, whole;
  };
  auto chunk = [&](int p, int k0) {
    const int q = tid + p * NT;
    Chunk h;
    h.ec = (q % (CH / 8)) * 8;
    h.es = q / (CH / 8);
    h.en = min(8, live - h.ec);
    h.in = h.es < TILE && h.en > 0 && k0 + h.es < min(n, last);
    h.whole = a.vec_d && h.en == 8;
    return h;
  };
  auto read = [&](const void* x, const Places& p, const Chunk& h, int k0) {
    return h.in ? load_raw<8>((const T*)x + (int64_t)(k0 + h.es) * p.step + (int64_t)b * p.row + d0 + h.ec, h.en, h.whole) : raw_zeros<T, 8>();
  };
  auto write = [&](void* x, const Places& p, const Chunk& h, int k0, const float (&f)[8]) {
    store_n<8>((T*)x + (int64_t)(k0 + h.es) * p.step + (int64_t)b * p.row + d0 + h.ec, f, h.en, h.whole);
  };
  // state s over step k of the tile: returns its decays
  auto advance = [&](pair (&s)[4], float dt, float x, int k, pair (&e)[4]) {
    pair B[4];
    const float* const p = my_bc + k * 2 * S::ROW;
    const ulonglong2 v0 = *reinterpret_cast<const ulonglong2*>(p), v1 = *reinterpret_cast<const ulonglong2*>(p + 16 * LANES);
    B[0] = v0.x; B[1] = v0.y; B[2] = v1.x; B[3] = v1.y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e[i] = decay2(both(dt), A[i]);
      s[i] = fma2(e[i], s[i], mul2(both(x), B[i]));
    }
  };

  const int tiles = (last - first + TILE - 1) / TILE;
  const int busy = n <= first ? 0 : min(tiles, (n - first + TILE - 1) / TILE);
  for (int i = tiles - 1; i >= 0; --i) {
    const int k0 = first + i * TILE, steps = min(TILE, min(n, last) - k0);
    if (i >= busy) {
      // behind the row's last step: zeros (dB and dC of these steps are the second kernel's)
      const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < CHUNKS; ++p) {
        const Chunk h = chunk(p, k0);
        if (h.es >= TILE || h.en <= 0 || k0 + h.es >= last) continue;
        write(a.du, a.pu, h, k0, zero);
        write(a.ddelta, a.pd, h, k0, zero);
        if (GATE) write(a.dz, a.pz, h, k0, zero);
      }
      continue;
    }
    __syncthreads();                              // the tile before has been read
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const Chunk h = chunk(p, k0);
      if (h.es >= TILE) continue;
      float fu[8], pre[8], dv[8], z[8];
      unpack<8>(read(a.u, a.pu, h, k0), fu);
      unpack<8>(read(a.delta, a.pd, h, k0), pre);
      unpack<8>(read(a.dy, a.py, h, k0), dv);
      if (GATE) unpack<8>(read(a.z, a.pz, h, k0), z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int w = At::at(h.ec + j, h.es);
        const float dt = h.in ? step_size(pre[j] + s_bias[h.ec + j], a.softplus) : 0.f;
        s_dt[w] = dt;
        s_x[w] = h.in ? dt * fu[j] : 0.f;
        s_dv[w] = !h.in ? 0.f : GATE ? dv[j] * z[j] * sigmoid(z[j]) : dv[j];
      }
    }
    for (int q = tid; q < TILE * NP / 2; q += NT) {
      const int n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, step = q / (NP / 2), k = k0 + step;
      float f[4] = {0, 0, 0, 0};
      if (k < n && k < last && n4 < a.states)
        unpack<4>(load_raw<4>((which ? Cm + (int64_t)k * a.pc.step : Bm + (int64_t)k * a.pb.step) + n4, a.states - n4, a.vec_s && n4 + 4 <= a.states), f);
      const int half = (n4 / 4) & 1, at_lane = n4 / PER_LANE;
#pragma unroll
      for (int o = 0; o < S::ORDERS; ++o) {
        // order o exchanges the halves (bit 1) and the pairs of a half (bit 0)
        float* const to = s_bc + (step * 2 + which) * S::ROW + (((half ^ (o >> 1)) * S::ORDERS + o) * LANES + at_lane) * 4;
        *reinterpret_cast<float4*>(to) = o & 1 ? make_float4(f[2], f[3], f[0], f[1]) : make_float4(f[0], f[1], f[2], f[3]);
      }
    }
    // the state before the tile; with states kept further apart than eight steps, those before its other eights
    pair s0[4] = {};
    if (mine) load_turned(a.kept + (int64_t)(k0 / a.spacing) * layer + place, l, turn, NP, true, s0);
    __syncthreads();
    if (a.spacing > EIGHT) {
      pair s[4] = {s0[0], s0[1], s0[2], s0[3]};
      for (int e = 0; (e + 1) * EIGHT < steps; ++e) {
        if (((e + 1) * EIGHT & (a.spacing - 1)) == 0) {
          if (mine) load_turned(a.kept + (int64_t)((k0 + (e + 1) * EIGHT) / a.spacing) * layer + place, l, turn, NP, true, s);
        } else {
#pragma unroll
          for (int j0 = 0; j0 < EIGHT; j0 += 4) {
            float dt[4], x[4];
            At::four(s_dt, c, e * EIGHT + j0, dt);
            At::four(s_x, c, e * EIGHT + j0, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              pair decay[4];
              advance(s, dt[j], x[j], e * EIGHT + j0 + j, decay);
            }
          }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<pair*>(s_start + (e * NT + tid) * PER_LANE + 2 * q) = s[q];
      }
    }
    pair tA[4] = {};
    const int eights = (steps + EIGHT - 1) / EIGHT;
    for (int e = eights - 1; e >= 0; --e) {
      pair decay[EIGHT][4], state[EIGHT + 1][4];  // of a step; before it
#pragma unroll
      for (int q = 0; q < 4; ++q) state[0][q] = s0[q];
      if (e > 0) {
        if (a.spacing > EIGHT) {
#pragma unroll
          for (int q = 0; q < 4; ++q) state[0][q] = *reinterpret_cast<const pair*>(s_start + ((e - 1) * NT + tid) * PER_LANE + 2 * q);
        } else if (mine) {
          load_turned(a.kept + (int64_t)(k0 / EIGHT + e) * layer + place, l, turn, NP, true, state[0]);
        }
      }
      float* const red = s_red + (e & 1) * S::RED + warp * EIGHT * 2 * NP;
#pragma unroll
      for (int j0 = 0; j0 < EIGHT; j0 += 4) {
        float dt[4], x[4];
        At::four(s_dt, c, e * EIGHT + j0, dt);
        At::four(s_x, c, e * EIGHT + j0, x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
          for (int q = 0; q < 4; ++q) state[j0 + j + 1][q] = state[j0 + j][q];
          advance(state[j0 + j + 1], dt[j], x[j], e * EIGHT + j0 + j, decay[j0 + j]);
        }
      }
#pragma unroll
      for (int j0 = EIGHT - 4; j0 >= 0; j0 -= 4) {
        const int k = e * EIGHT + j0;
        float dt[4], x[4], dv[4], sv[4], sB[4], sA[4];
        At::four(s_dt, c, k, dt);
        At::four(s_x, c, k, x);
        At::four(s_dv, c, k, dv);
#pragma unroll
        for (int j = 3; j >= 0; --j) {
          const float* const p = my_bc + (k + j) * 2 * S::ROW;
          const ulonglong2 b0 = *reinterpret_cast<const ulonglong2*>(p), b1 = *reinterpret_cast<const ulonglong2*>(p + 16 * LANES);
          const ulonglong2 c0 = *reinterpret_cast<const ulonglong2*>(p + S::ROW), c1 = *reinterpret_cast<const ulonglong2*>(p + S::ROW + 16 * LANES);
          const pair B[4] = {b0.x, b0.y, b1.x, b1.y}, C[4] = {c0.x, c0.y, c1.x, c1.y};
          const pair (&after)[4] = state[j0 + j + 1];
          const pair (&before)[4] = state[j0 + j];
          const pair x2 = both(x[j]), v2 = both(dv[j]), dt2 = both(dt[j]);
          if (GATE) sv[j] = dot(C, after);
          pair G[4], dB[4], dC[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            G[q] = fma2(v2, C[q], carry[q]);
            dB[q] = mul2(x2, G[q]);
            dC[q] = mul2(v2, after[q]);
          }
          sB[j] = dot(G, B);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            carry[q] = mul2(decay[j0 + j][q], G[q]);
            G[q] = mul2(carry[q], before[q]);      // g a s_{k-1}
            tA[q] = fma2(dt2, G[q], tA[q]);
          }
          sA[j] = dot(G, A);
          sum_channels<LANES>(dB, dC, lane);
          put_channels<LANES>(red + (j0 + j) * 2 * NP, dB, dC, lane, l, turn);
        }
        if (GATE) sum_lanes<LANES>(sv, l);
        sum_lanes<LANES>(sB, l);
        sum_lanes<LANES>(sA, l);
        const int w = At::at(c, k);
        if (GATE) put_steps<LANES>(s_v + w, l, sv);
        put_steps<LANES>(s_x + w, l, sB);
        put_steps<LANES>(s_dv + w, l, sA);
      }
      __syncthreads();
      // this eight's sums over the block's channels
      for (int q = tid; q < EIGHT * 2 * NP; q += NT) {
        const int j = q / (2 * NP), k = k0 + e * EIGHT + j;
        if (k >= n || k >= last) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += s_red[(e & 1) * S::RED + w * EIGHT * 2 * NP + q];
        a.part_bc[((((int64_t)block * a.t + k) * a.batch + b) * a.groups + g) * 2 * NP + q % (2 * NP)] = v;
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      pair* const sum = reinterpret_cast<pair*>(s_dA + tid * PER_LANE + 2 * q);
      *sum = add2(*sum, tA[q]);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const Chunk h = chunk(p, k0);
      if (h.es >= TILE) continue;
      float fu[8], pre[8], dy[8], z[8], du[8], dd[8], dz[8];
      unpack<8>(read(a.u, a.pu, h, k0), fu);
      unpack<8>(read(a.delta, a.pd, h, k0), pre);
      unpack<8>(read(a.dy, a.py, h, k0), dy);
      if (GATE) unpack<8>(read(a.z, a.pz, h, k0), z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int w = At::at(h.ec + j, h.es);
        const float skip = s_skip[h.ec + j];
        float dv = dy[j];
        if (GATE) {
          const float sig = sigmoid(z[j]);
          dv = dy[j] * z[j] * sig;
          dz[j] = h.in ? dy[j] * fmaf(skip, fu[j], s_v[w]) * dsilu(z[j], sig) : 0.f;
        }
        const float gB = s_x[w];
        du[j] = h.in ? fmaf(skip, dv, s_dt[w] * gB) : 0.f;
        dd[j] = h.in ? fmaf(fu[j], gB, s_dv[w] * (1.f / kLog2e)) * (a.softplus ? sigmoid(pre[j] + s_bias[h.ec + j]) : 1.f) : 0.f;   // A is in units of log 2
        s_x[w] = h.in ? dv * fu[j] : 0.f;
        s_dv[w] = dd[j];
      }
      if (h.en > 0 && k0 + h.es < last) {
        write(a.du, a.pu, h, k0, du);
        write(a.ddelta, a.pd, h, k0, dd);
        if (GATE) write(a.dz, a.pz, h, k0, dz);
      }
    }
    __syncthreads();
    {
      float v = 0.f, w = 0.f;
#pragma unroll
      for (int q = 0; q < TILE / 4 / LANES; ++q) {
        float x[4], y[4];
        At::four(s_x, c, (q * LANES + l) * 4, x);
        At::four(s_dv, c, (q * LANES + l) * 4, y);
        v += (x[0] + x[1]) + (x[2] + x[3]);
        w += (y[0] + y[1]) + (y[2] + y[3]);
      }
      dskip += v;
      dbias += w;
    }
  }
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) {
    dskip += __shfl_xor_sync(0xffffffffu, dskip, m);
    dbias += __shfl_xor_sync(0xffffffffu, dbias, m);
  }
  if (!mine) return;
  const int64_t at_part = ((int64_t)seg * a.batch + b) * a.channels + d;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int at = PER_LANE * l + pair_at(q, turn);
    *reinterpret_cast<pair*>(a.part_a + at_part * NP + at) = *reinterpret_cast<const pair*>(s_dA + tid * PER_LANE + 2 * q);
    if (seg == 0 && a.ds_in) store_pair(a.ds_in + row, at, a.states, a.vec_s, carry[q]);
  }
  if (l == 0) {
    a.part_d[at_part] = dskip;
    a.part_b[at_part] = dbias;
  }
}

// Sums over blocks (dB, dC: the first `rows` blocks of the grid, a thread each value) and over rows and segments (dA, dskip,
// ddelta_bias: 32 values a block, eight threads each).
struct Sums {
  const float* part_bc; const float* part_a; const float* part_d; const float* part_b;
  const int32_t* lengths;
  void* dB; void* dC; float* dA; float* dskip; float* dbias;
  Places pb, pc;
  int t, batch, channels, states, groups, blocks, np, parts;
  unsigned bc_blocks;
};
template <class T>
__global__ void __launch_bounds__(256) scan_sums(const Sums a) {
  __shared__ float red[8][32];
  const int tid = threadIdx.x;
  const int width = a.groups * 2 * a.np;
  if (blockIdx.x < a.bc_blocks) {
    const int64_t i = (int64_t)blockIdx.x * 256 + tid, all = (int64_t)a.t * a.batch * width;
    if (i >= all) return;
    const int64_t row = i / width;
    const int k = (int)(row / a.batch), b = (int)(row % a.batch), w = (int)(i % width);
    const int g = w / (2 * a.np), which = w / a.np & 1, q = w % a.np;
    if (q >= a.states) return;
    float v = 0.f;
    if (k < row_steps(a.lengths, b, a.t))
      for (int p = 0; p < a.blocks; ++p) v += a.part_bc[p * all + i];
    T* const out = which ? (T*)a.dC + (int64_t)k * a.pc.step + (int64_t)b * a.pc.row : (T*)a.dB + (int64_t)k * a.pb.step + (int64_t)b * a.pb.row;
    out[g * a.states + q] = from_f<T>(v);
    return;
  }
  // a value of [D][states + 2]
  const int64_t i = (int64_t)(blockIdx.x - a.bc_blocks) * 32 + tid % 32, all = (int64_t)a.channels * (a.states + 2);
  const int64_t d = i / (a.states + 2);
  const int q = (int)(i % (a.states + 2));
  float v = 0.f;
  if (i < all)
    for (int p = tid / 32; p < a.parts; p += 8) {
      const int64_t at_part = (int64_t)p * a.channels + d;
      v += q < a.states ? a.part_a[at_part * a.np + q] : q == a.states ? a.part_d[at_part] : a.part_b[at_part];
    }
  red[tid / 32][tid % 32] = v;
  __syncthreads();
  if (tid >= 32 || i >= all) return;
  for (int p = 1; p < 8; ++p) v += red[p][tid];
  if (q < a.states) a.dA[d * a.states + q] = v;
  else if (q == a.states) { if (a.dskip) a.dskip[d] = v; }
  else if (a.dbias) a.dbias[d] = v;
}

template <class T, int LANES, bool GATE>
bool launch_gate(const ScanArgs& a, cudaStream_t s) {
  const int bytes = (Shape<LANES>::FLOATS + (a.spacing > EIGHT ? Shape<LANES>::STARTS : 0)) * 4;
  // per call: function attributes belong to the current device
  if (cudaFuncSetAttribute(scan_bwd<T, LANES, GATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  const dim3 grid((unsigned)(a.groups * a.blocks), (unsigned)a.batch, (unsigned)a.segments);
  scan_bwd<T, LANES, GATE><<<grid, NT, bytes, counted(s)>>>(a);
  return true;
}
template <class T, int LANES>
bool launch(const ScanArgs& a, cudaStream_t s) {
  return a.z ? launch_gate<T, LANES, true>(a, s) : launch_gate<T, LANES, false>(a, s);
}
template <class T>
bool launch_lanes(const ScanArgs& a, cudaStream_t s) {
  switch (scan_lanes(a.states)) {
    case 1: return launch<T, 1>(a, s);
    case 2: return launch<T, 2>(a, s);
    case 4: return launch<T, 4>(a, s);
    default: return launch<T, 8>(a, s);
  }
}

}  // namespace

int scan_bwd_channels(int lanes) { return NT / lanes; }

bool scan_backward(const ScanArgs& a, bool half, float* dA, void* dB, void* dC, float* dskip, float* dbias, cudaStream_t s) {
  if (!(half ? launch_lanes<bf16>(a, s) : launch_lanes<float>(a, s))) return false;
  const int np = PER_LANE * scan_lanes(a.states);
  Sums r = {a.part_bc, a.part_a, a.part_d, a.part_b, a.lengths, dB, dC, dA, dskip, dbias, a.pb, a.pc,
            a.t, a.batch, a.channels, a.states, a.groups, a.blocks, np, a.batch * a.segments, 0};
  const int64_t bc = (int64_t)a.t * a.batch * a.groups * 2 * np, rest = (int64_t)a.channels * (a.states + 2);
  r.bc_blocks = (unsigned)((bc + 255) / 256);
  const unsigned grid = r.bc_blocks + (unsigned)((rest + 31) / 32);
  if (half) scan_sums<bf16><<<grid, 256, 0, counted(s)>>>(r);
  else scan_sums<float><<<grid, 256, 0, counted(s)>>>(r);
  return true;
}

}  // namespace seq
}  // namespace mebptt
