// Selective state space scan, backward.
//
// A block owns 128 / LANES channels of one row and walks a segment's tiles of 8 steps from the last to the first; LANES lanes share
// a channel, eight states each, two to an instruction.  A tile runs forwards from the state before it, with the states of its
// steps in registers, and then backwards.  States are not kept but every `spacing` steps: where that is more than a tile, the tiles
// from one kept state to the next are first visited in ascending order to find those between.  Every thread fetches the
// next tile's inputs and kept state while a tile is worked on.
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
// Measured at 1000 steps x 64 rows x 1024 channels x 16 states in bfloat16, states kept every 8 steps: 1350 us; issue slots 56 %,
// shared-memory pipe 64 %, special functions 43 %: bound by the chains of a step (exponential, product, shuffles) at 16 warps an SM.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.hpp"
#include "scan.hpp"
#include "scan_dev.cuh"
#include "scan_kernels.hpp"
#include "sm100.cuh"

namespace mebptt {
namespace seq {

namespace {

constexpr int NT = 128, STEPS = 8, GW = 4;         // threads; steps of a tile; channels of a group in the elementwise parts

template <class T, int LANES>
struct Shape {
  static constexpr int CH = NT / LANES, NP = PER_LANE * LANES, WARPS = NT / 32;
  static constexpr int GROUPS = STEPS * CH / GW;
  static constexpr int QG = GROUPS > NT ? GROUPS / NT : 1;                          // groups of a thread
  static constexpr int QUARTERS = STEPS * NP / 2;                                   // of B and C: four states each
  static constexpr int QB = QUARTERS > NT ? QUARTERS / NT : 1;                      // of a thread
  using At = Tile<STEPS, CH>;
  static constexpr int ORDERS = 4;                                                  // of B and C
  static constexpr int ROW = ORDERS * NP;                                           // of B or C, of a step
  static constexpr int RED = WARPS * STEPS * 2 * NP;                                // sums over channels, by warp
  // What threads fetch for a tile, in bytes: u, delta, dy, z (twice); B and C; a state.  Each thread reads what it fetched itself.
  static constexpr int ARRAY = QG * NT * GW * (int)sizeof(T), BC = QB * NT * 4 * (int)sizeof(T), STATE = NT * PER_LANE * 4;
  static constexpr int RAW = 2 * 4 * ARRAY + BC + STATE;
  // those, planes of the tile, B and C, sums over channels, of tiles, the channels' bias and skip
  static constexpr int BYTES = RAW + 4 * (4 * At::FLOATS + STEPS * 2 * ROW + RED + NT * PER_LANE + 2 * CH);
  static constexpr int STARTS = (TILE / STEPS - 1) * STATE;                         // states before the tiles between those that are kept
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

// VISITS: states are kept further apart than a tile is long.  (Without them the loop keeps its shape all the same: as straight code the
// compiler would move so much of the backward half into the forward one that it spilt 276 bytes a thread, 1795 us instead of 1374.)
template <class T, int LANES, bool GATE, bool VISITS>
__global__ void __launch_bounds__(NT, 4) scan_bwd(const ScanArgs a) {
  using S = Shape<T, LANES>;
  using At = typename S::At;
  constexpr int CH = S::CH, NP = S::NP, WARPS = S::WARPS, QG = S::QG, QB = S::QB, E4 = 4 * (int)sizeof(T);
  sm100::grid_dep_wait();                         // for the kernel of the adjoints
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* const s_arrays = smem;                                         // [2][u, delta, dy, z][groups][4]
  uint8_t* const s_rows = s_arrays + 8 * S::ARRAY;                        // [STEPS][B, C][NP], as in memory
  float* const s_state = reinterpret_cast<float*>(s_rows + S::BC);        // [NT][8]: the state before the next tile, in two halves
  float* const s_dt = s_state + NT * PER_LANE;    // dt
  float* const s_x = s_dt + At::FLOATS;           // dt u, then the sums over states of g B, then dv u
  float* const s_dv = s_x + At::FLOATS;           // dv, then of A a s g, then ddelta
  float* const s_v = s_dv + At::FLOATS;           // of C s
  float* const s_bc = s_v + At::FLOATS;           // [STEPS][B, C][two halves of a lane's states][orders][LANES][4]
  float* const s_red = s_bc + STEPS * 2 * S::ROW; // [WARPS][STEPS][2 NP]
  float* const s_dA = s_red + S::RED;             // [NT][8]: sums of the tiles so far
  float* const s_bias = s_dA + NT * PER_LANE;     // [CH]
  float* const s_skip = s_bias + CH;              // [CH]
  float* const s_start = s_skip + CH;             // [3][NT][8]: states before the tiles between those that are kept

  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, b = blockIdx.y, seg = blockIdx.z;
  const int g = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks, base = block * CH;
  const int d0 = g * a.gchannels + base;
  const int live = min(CH, a.gchannels - base);
  const int n = row_steps(a.lengths, b, a.t);
  const int first = seg * a.segment, last = min(first + a.segment, a.t), stop = min(n, last);

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
    for (int j0 = a.segments - 1; j0 > seg; j0 -= FOLD) {
      pair e[FOLD][4];
      float dts[FOLD];
#pragma unroll
      for (int j = 0; j < FOLD; ++j)
        if (j0 - j > seg) {
          load_turned(a.ends + (j0 - j + 1) * layer + place, l, turn, NP, true, e[j]);
          dts[j] = a.dts[((int64_t)(j0 - j) * a.batch + b) * a.channels + d];
        }
#pragma unroll
      for (int j = 0; j < FOLD; ++j)
        if (j0 - j > seg)
#pragma unroll
          for (int i = 0; i < 4; ++i) carry[i] = carry2(A[i], dts[j], carry[i], e[j][i]);
    }
  }
  for (int i = 0; i < PER_LANE; ++i) s_dA[tid * PER_LANE + i] = 0.f;
  for (int i = tid; i < CH; i += NT) {
    s_bias[i] = a.bias && i < live ? a.bias[d0 + i] : 0.f;
    s_skip[i] = a.skip && i < live ? a.skip[d0 + i] : 0.f;
  }
  float dskip = 0.f, dbias = 0.f;

  // four channels of a step, in the elementwise parts
  struct Group {
    int c, step, n;
    bool there, whole;
  };
  auto group = [&](int p) {
    const int q = tid + p * NT;
    Group h;
    h.c = (q % (CH / GW)) * GW;
    h.step = q / (CH / GW);
    h.n = min(GW, live - h.c);
    h.there = h.step < STEPS && h.n > 0;
    h.whole = a.vec_d && h.n == GW;
    return h;
  };
  // Asks for the tile at k0, arrays into half `to`: for all of it, or for what a visit takes.  kept: and for the state before it.
  auto fetch = [&](int k0, int to, bool kept, bool all) {
#pragma unroll
    for (int q = 0; q < QG; ++q) {
      const Group h = group(q);
      if (!h.there || k0 + h.step >= stop) continue;
      uint8_t* const at = s_arrays + to * 4 * S::ARRAY + (tid + q * NT) * E4;
      const int arrays = all ? GATE ? 4 : 3 : 2;
      const void* const x[4] = {a.u, a.delta, a.dy, a.z};
      const Places* const p[4] = {&a.pu, &a.pd, &a.py, &a.pz};
      auto from = [&](int w) { return (const T*)x[w] + (int64_t)(k0 + h.step) * p[w]->step + (int64_t)b * p[w]->row + d0 + h.c; };
      if (h.whole) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (w < arrays) fetch_n<4>(at + w * S::ARRAY, from(w), GW, true);
      } else {
        Raw<T, 4> r[4];
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (w < arrays) r[w] = load_raw<4>(from(w), h.n, false);
#pragma unroll
        for (int w = 0; w < 4; ++w)
          if (w < arrays) memcpy(at + w * S::ARRAY, &r[w], sizeof r[w]);
      }
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, k = k0 + q / (NP / 2);
      if (q >= S::QUARTERS || k >= stop || n4 >= a.states || (which && !all)) continue;
      fetch_n<4>(s_rows + q * E4, (which ? Cm + (int64_t)k * a.pc.step : Bm + (int64_t)k * a.pb.step) + n4, a.states - n4, a.vec_s && n4 + 4 <= a.states);
    }
    if (mine && kept) {
      const float* const from = a.kept + (int64_t)(k0 / a.spacing) * layer + place + PER_LANE * l;
      async16(s_state + tid * 4, from);
      async16(s_state + (NT + tid) * 4, from + 4);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto array = [&](int half, int which, int q) { return fetched<T, 4>(s_arrays + (half * 4 + which) * S::ARRAY + (tid + q * NT) * E4); };
  auto kept_state = [&](pair (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = i ^ turn;
      s[i] = mine ? *reinterpret_cast<const pair*>(s_state + ((at >> 1) * NT + tid) * 4 + (at & 1) * 2) : 0;
    }
  };
  auto start = [&](int j) { return reinterpret_cast<pair*>(s_start + ((j - 1) * NT + tid) * PER_LANE); };   // before tile j of those between kept states
  auto write = [&](void* x, const Places& p, const Group& h, int k0, const pair (&f)[2]) {
    store_pairs<4>((T*)x + (int64_t)(k0 + h.step) * p.step + (int64_t)b * p.row + d0 + h.c, f, h.n, h.whole);
  };
  // four values of a plane at one step
  auto plane = [&](const float* s, const Group& h, pair (&f)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) f[j] = pack2(s[At::at(h.c + 2 * j, h.step)], s[At::at(h.c + 2 * j + 1, h.step)]);
  };
  auto to_plane = [&](float* s, const Group& h, const pair (&f)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float2 v = unpack2(f[j]);
      s[At::at(h.c + 2 * j, h.step)] = v.x;
      s[At::at(h.c + 2 * j + 1, h.step)] = v.y;
    }
  };
  auto channel_values = [&](const float* s, const Group& h, pair (&f)[2]) {
    const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(s + h.c);
    f[0] = v.x; f[1] = v.y;
  };
  // the tile's planes and its B and C out of what was fetched
  auto stage = [&](int k0, int half, bool all) {
#pragma unroll
    for (int p = 0; p < QG; ++p) {
      const Group h = group(p);
      if (h.step >= STEPS) continue;
      pair dt[2] = {}, x[2] = {}, dv[2] = {};
      if (h.there && k0 + h.step < stop) {
        pair bias[2];
        unpack_pairs<4>(array(half, 1, p), dt);
        unpack_pairs<4>(array(half, 0, p), x);
        if (all) unpack_pairs<4>(array(half, 2, p), dv);
        channel_values(s_bias, h, bias);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          dt[j] = add2(dt[j], bias[j]);
          if (a.softplus) dt[j] = softplus2(dt[j]);
          x[j] = mul2(x[j], dt[j]);
        }
        if (GATE && all) {
          pair z[2];
          unpack_pairs<4>(array(half, 3, p), z);
#pragma unroll
          for (int j = 0; j < 2; ++j) dv[j] = mul2(dv[j], mul2(z[j], sigmoid2(z[j])));
        }
      }
      to_plane(s_dt, h, dt);
      to_plane(s_x, h, x);
      if (all) to_plane(s_dv, h, dv);
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, step = q / (NP / 2);
      if (q >= S::QUARTERS || (which && !all)) continue;
      float f[4] = {0, 0, 0, 0};
      if (k0 + step < stop && n4 < a.states) unpack<4>(fetched<T, 4>(s_rows + q * E4), f);
      const int upper = (n4 / 4) & 1, at_lane = n4 / PER_LANE;
#pragma unroll
      for (int o = 0; o < S::ORDERS; ++o) {
        // order o exchanges the halves (bit 1) and the pairs of a half (bit 0)
        float* const to = s_bc + (step * 2 + which) * S::ROW + (((upper ^ (o >> 1)) * S::ORDERS + o) * LANES + at_lane) * 4;
        *reinterpret_cast<float4*>(to) = o & 1 ? make_float4(f[2], f[3], f[0], f[1]) : make_float4(f[0], f[1], f[2], f[3]);
      }
    }
  };
  auto lane_row = [&](const float* p, pair (&v)[4]) {
    const ulonglong2 v0 = *reinterpret_cast<const ulonglong2*>(p), v1 = *reinterpret_cast<const ulonglong2*>(p + 16 * LANES);
    v[0] = v0.x; v[1] = v0.y; v[2] = v1.x; v[3] = v1.y;
  };

  const int tiles = (last - first + STEPS - 1) / STEPS;
  const int busy = n <= first ? 0 : min(tiles, (n - first + STEPS - 1) / STEPS);
  // behind the row's last step: zeros (dB and dC of these steps are the second kernel's)
  for (int i = busy; i < tiles; ++i) {
    const pair zero[2] = {};
#pragma unroll
    for (int p = 0; p < QG; ++p) {
      const Group h = group(p);
      const int k0 = first + i * STEPS;
      if (!h.there || k0 + h.step >= last) continue;
      write(a.du, a.pu, h, k0, zero);
      write(a.ddelta, a.pd, h, k0, zero);
      if (GATE) write(a.dz, a.pz, h, k0, zero);
    }
  }
  // Tiles from the last to the first, those between two kept states together: with `per` of them, the states before all but the first
  // are found by visits to the tiles before them, in ascending order.  (Segments begin where states are kept.)
  const int per = a.spacing / STEPS;
  int i = busy - 1, half = 0;                     // the tile to be worked on
  int visit = i >= 0 && i % per ? i - i % per : -1;   // the tile to be visited first, -1: none
  if (i >= 0) fetch(first + (visit >= 0 ? visit : i) * STEPS, half, true, !VISITS || visit < 0);
  while (i >= 0) {
    const bool visiting = visit >= 0;
    const int tile = visiting ? visit : i, k0 = first + tile * STEPS, steps = min(STEPS, stop - k0);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                              // the tile before has been read
    pair state[STEPS + 1][4];                     // before a step
    if (tile % per == 0) {
      kept_state(state[0]);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) state[0][q] = start(tile % per)[q];
    }
    stage(k0, half, !VISITS || !visiting);
    int next = i, next_visit = -1;
    if (!visiting) {
      --next;
      if (next >= 0 && next % per == per - 1 && per > 1) next_visit = next - (per - 1);
    } else if (visit + 1 < i) {
      next_visit = visit + 1;
    }
    const int next_tile = next_visit >= 0 ? next_visit : next;
    if (next_tile >= 0) fetch(first + next_tile * STEPS, half ^ 1, next_tile % per == 0, !VISITS || next_visit < 0);
    __syncthreads();
    // forwards
#pragma unroll
    for (int j0 = 0; j0 < STEPS; j0 += 4) {
      float dt[4], x[4];
      At::four(s_dt, c, j0, dt);
      At::four(s_x, c, j0, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pair B[4];
        lane_row(my_bc + (j0 + j) * 2 * S::ROW, B);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          state[j0 + j + 1][q] = fma2(decay2(both(dt[j]), A[q]), state[j0 + j][q], mul2(both(x[j]), B[q]));
      }
    }
    half ^= 1;
    if (visiting) {
#pragma unroll
      for (int q = 0; q < 4; ++q) start(tile % per + 1)[q] = state[STEPS][q];
      visit = next_visit;
      continue;
    }
    // Backwards.  The decays are computed once more: to hold them too would leave an SM 12 warps instead of 16.  (The compiler,
    // which would rather hold them, is told that A may be another now; and between groups of steps, that memory may be.)
    asm volatile("" : "+l"(A[0]), "+l"(A[1]), "+l"(A[2]), "+l"(A[3])::"memory");
    pair tA[4] = {};
    float* const red = s_red + warp * STEPS * 2 * NP;
#pragma unroll
    for (int j0 = STEPS - 4; j0 >= 0; j0 -= 4) {
      float dt[4], x[4], dv[4], sv[4], sB[4], sA[4];
      asm volatile("" ::: "memory");
      At::four(s_dt, c, j0, dt);
      At::four(s_x, c, j0, x);
      At::four(s_dv, c, j0, dv);
#pragma unroll
      for (int j = 3; j >= 0; --j) {
        const float* const p = my_bc + (j0 + j) * 2 * S::ROW;
        pair B[4], C[4], G[4], dB[4], dC[4];
        lane_row(p, B);
        lane_row(p + S::ROW, C);
        const pair (&after)[4] = state[j0 + j + 1];
        const pair x2 = both(x[j]), v2 = both(dv[j]), dt2 = both(dt[j]);
        if (GATE) sv[j] = dot(C, after);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          G[q] = fma2(v2, C[q], carry[q]);
          dB[q] = mul2(x2, G[q]);
          dC[q] = mul2(v2, after[q]);
        }
        sB[j] = dot(G, B);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          carry[q] = mul2(decay2(dt2, A[q]), G[q]);
          G[q] = mul2(carry[q], state[j0 + j][q]);   // g a s_{k-1}
          tA[q] = fma2(dt2, G[q], tA[q]);
        }
        sA[j] = dot(G, A);
        sum_channels<LANES>(dB, dC, lane);
        put_channels<LANES>(red + (j0 + j) * 2 * NP, dB, dC, lane, l, turn);
      }
      if (GATE) sum_lanes<LANES>(sv, l);
      sum_lanes<LANES>(sB, l);
      sum_lanes<LANES>(sA, l);
      const int w = At::at(c, j0);
      if (GATE) put_steps<LANES>(s_v + w, l, sv);
      put_steps<LANES>(s_x + w, l, sB);
      put_steps<LANES>(s_dv + w, l, sA);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      pair* const sum = reinterpret_cast<pair*>(s_dA + tid * PER_LANE + 2 * q);
      *sum = add2(*sum, tA[q]);
    }
    __syncthreads();
    // this tile's sums over the block's channels
    {
      float* const out = a.part_bc + ((((int64_t)block * a.t + k0) * a.batch + b) * a.groups + g) * 2 * NP;
      const int64_t step = (int64_t)a.batch * a.groups * 2 * NP;
      for (int q = tid; q < steps * 2 * NP; q += NT) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += s_red[w * STEPS * 2 * NP + q];
        out[q / (2 * NP) * step + q % (2 * NP)] = v;
      }
    }
    const int was = half ^ 1;
#pragma unroll
    for (int p = 0; p < QG; ++p) {
      const Group h = group(p);
      if (h.step >= STEPS) continue;
      pair du[2] = {}, dd[2] = {}, dz[2] = {}, vu[2] = {};
      if (h.there && k0 + h.step < stop) {
        pair skip[2], bias[2], u[2], dv[2], gB[2], gA[2], dt[2];
        channel_values(s_skip, h, skip);
        channel_values(s_bias, h, bias);
        unpack_pairs<4>(array(was, 0, p), u);
        unpack_pairs<4>(array(was, 1, p), dd);
        unpack_pairs<4>(array(was, 2, p), dv);
        if (GATE) {
          pair z[2], v[2];
          unpack_pairs<4>(array(was, 3, p), z);
          plane(s_v, h, v);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const pair sig = sigmoid2(z[j]), zs = mul2(z[j], sig);
            // silu' = s + z s (1 - s)
            const pair f = fma2(zs, fma2(sig, both(-1.f), both(1.f)), sig);
            dz[j] = mul2(mul2(dv[j], fma2(skip[j], u[j], v[j])), f);
            dv[j] = mul2(dv[j], zs);
          }
        }
        plane(s_x, h, gB);
        plane(s_dv, h, gA);
        plane(s_dt, h, dt);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          du[j] = fma2(skip[j], dv[j], mul2(dt[j], gB[j]));
          const pair ddt = fma2(u[j], gB[j], mul2(gA[j], both(1.f / kLog2e)));        // A is in units of log 2
          dd[j] = a.softplus ? mul2(ddt, sigmoid2(add2(dd[j], bias[j]))) : ddt;
          vu[j] = mul2(dv[j], u[j]);
        }
      }
      to_plane(s_x, h, vu);
      to_plane(s_dv, h, dd);
      if (h.there && k0 + h.step < last) {
        write(a.du, a.pu, h, k0, du);
        write(a.ddelta, a.pd, h, k0, dd);
        if (GATE) write(a.dz, a.pz, h, k0, dz);
      }
    }
    __syncthreads();
    {
      float v = 0.f, w = 0.f;
      if constexpr (LANES <= 2) {
#pragma unroll
        for (int q = 0; q < STEPS / 4 / LANES; ++q) {
          float x[4], y[4];
          At::four(s_x, c, (q * LANES + l) * 4, x);
          At::four(s_dv, c, (q * LANES + l) * 4, y);
          v += (x[0] + x[1]) + (x[2] + x[3]);
          w += (y[0] + y[1]) + (y[2] + y[3]);
        }
      } else {
#pragma unroll
        for (int q = 0; q < STEPS / LANES; ++q) {
          v += s_x[At::at(c, q * LANES + l)];
          w += s_dv[At::at(c, q * LANES + l)];
        }
      }
      dskip += v;
      dbias += w;
    }
    i = next;
    visit = next_visit;
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
  sm100::grid_dep_wait();
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

template <class T, int LANES, bool GATE, bool VISITS>
bool launch_kernel(const ScanArgs& a, cudaStream_t s) {
  constexpr int bytes = Shape<T, LANES>::BYTES + (VISITS ? Shape<T, LANES>::STARTS : 0);
  // per call: function attributes belong to the current device
  if (bytes > 48 * 1024 && cudaFuncSetAttribute(scan_bwd<T, LANES, GATE, VISITS>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  const dim3 grid((unsigned)(a.groups * a.blocks), (unsigned)a.batch, (unsigned)a.segments);
  return launch_on(a.segments > 1, scan_bwd<T, LANES, GATE, VISITS>, grid, dim3(NT), bytes, s, a) == cudaSuccess;
}
template <class T, int LANES>
bool launch(const ScanArgs& a, cudaStream_t s) {
  if (a.spacing > STEPS) return a.z ? launch_kernel<T, LANES, true, true>(a, s) : launch_kernel<T, LANES, false, true>(a, s);
  return a.z ? launch_kernel<T, LANES, true, false>(a, s) : launch_kernel<T, LANES, false, false>(a, s);
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

template <class T>
static int blocks_of_sm(int lanes, int spacing) {
  auto room = [&](int bytes, int starts) {
    const int n = 227 * 1024 / (bytes + (spacing > STEPS ? starts : 0) + 1024);
    return n < 4 ? n : 4;
  };
  switch (lanes) {
    case 1: return room(Shape<T, 1>::BYTES, Shape<T, 1>::STARTS);
    case 2: return room(Shape<T, 2>::BYTES, Shape<T, 2>::STARTS);
    case 4: return room(Shape<T, 4>::BYTES, Shape<T, 4>::STARTS);
    default: return room(Shape<T, 8>::BYTES, Shape<T, 8>::STARTS);
  }
}
int scan_bwd_blocks(int lanes, bool half, int spacing) { return half ? blocks_of_sm<bf16>(lanes, spacing) : blocks_of_sm<float>(lanes, spacing); }

bool scan_backward(const ScanArgs& a, bool half, float* dA, void* dB, void* dC, float* dskip, float* dbias, cudaStream_t s) {
  if (!(half ? launch_lanes<bf16>(a, s) : launch_lanes<float>(a, s))) return false;
  const int np = PER_LANE * scan_lanes(a.states);
  Sums r = {a.part_bc, a.part_a, a.part_d, a.part_b, a.lengths, dB, dC, dA, dskip, dbias, a.pb, a.pc,
            a.t, a.batch, a.channels, a.states, a.groups, a.blocks, np, a.batch * a.segments, 0};
  const int64_t bc = (int64_t)a.t * a.batch * a.groups * 2 * np, rest = (int64_t)a.channels * (a.states + 2);
  r.bc_blocks = (unsigned)((bc + 255) / 256);
  const unsigned grid = r.bc_blocks + (unsigned)((rest + 31) / 32);
  return (half ? launch_pdl(scan_sums<bf16>, dim3(grid), dim3(256), 0, s, r) : launch_pdl(scan_sums<float>, dim3(grid), dim3(256), 0, s, r)) == cudaSuccess;
}

}  // namespace seq
}  // namespace mebptt
