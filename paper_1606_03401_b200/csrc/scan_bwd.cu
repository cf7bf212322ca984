// Selective state space scan, backward.
//
// A block owns 128 / LANES channels of one row and walks a segment's tiles of 16 steps from the last to the first; LANES lanes share
// a channel, eight states each, two to an instruction.  States are not kept but every `spacing` steps: eight steps at a time are
// run forwards from the state before them, with the decays and the states of the eight steps in registers, and then backwards.
// Where states are kept further apart, those between are found by running forwards once more.  Every thread fetches the next
// tile's inputs and states while a tile is worked on (12 warps an SM would not hide them).
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

constexpr int EIGHT = 8, NT = 128, STEPS = 16;     // steps of a tile

template <class T, int LANES>
struct Shape {
  static constexpr int CH = NT / LANES, NP = PER_LANE * LANES, WARPS = NT / 32;
  static constexpr int CHUNKS = STEPS * CH / 8 > NT ? STEPS * CH / 8 / NT : 1;      // groups of eight channels a thread, in the elementwise part
  static constexpr int QUARTERS = STEPS * NP / 2;                                   // of B and C: four states each
  static constexpr int QB = QUARTERS > NT ? QUARTERS / NT : 1;                      // of a thread
  using At = Tile<STEPS, CH>;
  static constexpr int ORDERS = 4;                                                  // of B and C
  static constexpr int ROW = ORDERS * NP;                                           // of B or C, of a step
  static constexpr int RED = WARPS * EIGHT * 2 * NP;                                // sums of one eight, by warp
  // What a thread fetches for a tile, in 16-byte pieces: u, delta, dy, z; B and C; two states.  Each thread reads what it fetched itself.
  static constexpr int ARRAY = CHUNKS * (int)sizeof(T) / 2, BC = QB * (int)sizeof(T) / 4 > 0 ? QB * (int)sizeof(T) / 4 : 1;
  static constexpr int PIECES = 4 * ARRAY + BC + 4;
  // planes of the tile, B and C, sums of an eight and of tiles, the channels' bias and skip, what is fetched (twice)
  static constexpr int FLOATS = 4 * At::FLOATS + STEPS * 2 * ROW + RED + NT * PER_LANE + 2 * CH + 2 * PIECES * NT * 4;
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

__device__ __forceinline__ void async16(void* dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void async8(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

template <class T, int LANES, bool GATE>
__global__ void __launch_bounds__(NT, 3) scan_bwd(const ScanArgs a) {
  using S = Shape<T, LANES>;
  using At = typename S::At;
  constexpr int CH = S::CH, NP = S::NP, WARPS = S::WARPS, CHUNKS = S::CHUNKS, QB = S::QB;
  extern __shared__ __align__(16) float sm[];
  uint4* const s_raw = reinterpret_cast<uint4*>(sm);                                // [2][PIECES][NT]
  float* const s_dt = sm + 2 * S::PIECES * NT * 4;   // dt
  float* const s_x = s_dt + At::FLOATS;           // dt u, then the sums over states of g B, then dv u
  float* const s_dv = s_x + At::FLOATS;           // dv, then of A a s g, then ddelta
  float* const s_v = s_dv + At::FLOATS;           // of C s
  float* const s_bc = s_v + At::FLOATS;           // [STEPS][B, C][two halves of a lane's states][orders][LANES][4]
  float* const s_red = s_bc + STEPS * 2 * S::ROW; // [WARPS][EIGHT][2 NP]
  float* const s_dA = s_red + S::RED;             // [NT][8]: sums of the tiles so far
  float* const s_bias = s_dA + NT * PER_LANE;     // [CH]
  float* const s_skip = s_bias + CH;              // [CH]

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
    bool here, whole;
  };
  auto chunk = [&](int p) {
    const int q = tid + p * NT;
    Chunk h;
    h.ec = (q % (CH / 8)) * 8;
    h.es = q / (CH / 8);
    h.en = min(8, live - h.ec);
    h.here = h.es < STEPS && h.en > 0;
    h.whole = a.vec_d && h.en == 8;
    return h;
  };
  // Asks for the tile at k0: into the thread's own pieces of stage st.  Where groups do not load as one they come by plain loads.
  auto fetch = [&](int k0, int st) {
    uint4* const raw = s_raw + st * S::PIECES * NT + tid;
    auto array = [&](const void* x, const Places& p, int which) {
#pragma unroll
      for (int q = 0; q < CHUNKS; ++q) {
        const Chunk h = chunk(q);
        if (!h.here || k0 + h.es >= stop) continue;
        const T* const from = (const T*)x + (int64_t)(k0 + h.es) * p.step + (int64_t)b * p.row + d0 + h.ec;
        uint4* const to = raw + (which * S::ARRAY + q * (int)sizeof(T) / 2) * NT;
        if (h.whole) {
#pragma unroll
          for (int i = 0; i < (int)sizeof(T) / 2; ++i) async16(to + i * NT, reinterpret_cast<const uint4*>(from) + i);
        } else {
          const Raw<T, 8> r = load_raw<8>(from, h.en, false);
#pragma unroll
          for (int i = 0; i < (int)sizeof(T) / 2; ++i) to[i * NT] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
        }
      }
    };
    array(a.u, a.pu, 0);
    array(a.delta, a.pd, 1);
    array(a.dy, a.py, 2);
    if (GATE) array(a.z, a.pz, 3);
    uint8_t* const bc = reinterpret_cast<uint8_t*>(raw - tid + 4 * S::ARRAY * NT);
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, k = k0 + q / (NP / 2);
      if (q >= S::QUARTERS || k >= stop || n4 >= a.states) continue;
      const T* const from = (which ? Cm + (int64_t)k * a.pc.step : Bm + (int64_t)k * a.pb.step) + n4;
      void* const to = bc + (size_t)q * 4 * sizeof(T);
      if (a.vec_s && n4 + 4 <= a.states) {
        if constexpr (sizeof(T) == 2) async8(to, from);
        else async16(to, from);
      } else {
        const Raw<T, 4> r = load_raw<4>(from, a.states - n4, false);
        memcpy(to, &r, sizeof r);
      }
    }
    if (mine) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int k = k0 + e * EIGHT;
        if (k >= stop || (k & (a.spacing - 1))) continue;
        const uint4* const from = reinterpret_cast<const uint4*>(a.kept + (int64_t)(k / a.spacing) * layer + place + PER_LANE * l);
#pragma unroll
        for (int i = 0; i < 2; ++i) async16(raw + (4 * S::ARRAY + S::BC + 2 * e + i) * NT, from + i);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto raw_chunk = [&](int st, int which, int q) {
    const uint4* const p = s_raw + st * S::PIECES * NT + tid + (which * S::ARRAY + q * (int)sizeof(T) / 2) * NT;
    Raw<T, 8> r;
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      const uint4 v = p[i * NT];
      r.w[4 * i] = v.x; r.w[4 * i + 1] = v.y; r.w[4 * i + 2] = v.z; r.w[4 * i + 3] = v.w;
    }
    return r;
  };
  auto kept_state = [&](int st, int e, pair (&s)[4]) {       // pairs 2 i and 2 i + 1 lie in piece i
    const pair* const p = reinterpret_cast<const pair*>(s_raw + st * S::PIECES * NT + tid + (4 * S::ARRAY + S::BC + 2 * e) * NT);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = i ^ turn;
      s[i] = mine ? p[(at >> 1) * 2 * NT + (at & 1)] : 0;
    }
  };
  auto write = [&](void* x, const Places& p, const Chunk& h, int k0, const pair (&f)[4]) {
    store_pairs<8>((T*)x + (int64_t)(k0 + h.es) * p.step + (int64_t)b * p.row + d0 + h.ec, f, h.en, h.whole);
  };
  // eight values of a plane at one step
  auto plane = [&](const float* s, const Chunk& h, pair (&f)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = pack2(s[At::at(h.ec + 2 * j, h.es)], s[At::at(h.ec + 2 * j + 1, h.es)]);
  };
  auto to_plane = [&](float* s, const Chunk& h, const pair (&f)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 v = unpack2(f[j]);
      s[At::at(h.ec + 2 * j, h.es)] = v.x;
      s[At::at(h.ec + 2 * j + 1, h.es)] = v.y;
    }
  };
  auto channel_values = [&](const float* s, const Chunk& h, pair (&f)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const pair*>(s + h.ec + 2 * j);
  };
  // the tile's planes and its B and C out of what was fetched
  auto stage = [&](int k0, int st) {
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const Chunk h = chunk(p);
      if (h.es >= STEPS) continue;
      pair dt[4] = {}, x[4] = {}, dv[4] = {};
      if (h.here && k0 + h.es < stop) {
        pair bias[4];
        unpack_pairs<8>(raw_chunk(st, 1, p), dt);
        unpack_pairs<8>(raw_chunk(st, 0, p), x);
        unpack_pairs<8>(raw_chunk(st, 2, p), dv);
        channel_values(s_bias, h, bias);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dt[j] = add2(dt[j], bias[j]);
          if (a.softplus) dt[j] = softplus2(dt[j]);
          x[j] = mul2(x[j], dt[j]);
        }
        if (GATE) {
          pair z[4];
          unpack_pairs<8>(raw_chunk(st, 3, p), z);
#pragma unroll
          for (int j = 0; j < 4; ++j) dv[j] = mul2(dv[j], mul2(z[j], sigmoid2(z[j])));
        }
      }
      to_plane(s_dt, h, dt);
      to_plane(s_x, h, x);
      to_plane(s_dv, h, dv);
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, step = q / (NP / 2);
      if (q >= S::QUARTERS) continue;
      float f[4] = {0, 0, 0, 0};
      if (k0 + step < stop && n4 < a.states) {
        Raw<T, 4> r;
        memcpy(&r, reinterpret_cast<const uint8_t*>(s_raw + (st * S::PIECES + 4 * S::ARRAY) * NT) + (size_t)q * 4 * sizeof(T), sizeof r);
        unpack<4>(r, f);
      }
      const int half = (n4 / 4) & 1, at_lane = n4 / PER_LANE;
#pragma unroll
      for (int o = 0; o < S::ORDERS; ++o) {
        // order o exchanges the halves (bit 1) and the pairs of a half (bit 0)
        float* const to = s_bc + (step * 2 + which) * S::ROW + (((half ^ (o >> 1)) * S::ORDERS + o) * LANES + at_lane) * 4;
        *reinterpret_cast<float4*>(to) = o & 1 ? make_float4(f[2], f[3], f[0], f[1]) : make_float4(f[0], f[1], f[2], f[3]);
      }
    }
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
  auto forwards = [&](pair (&s)[4], int from, int to) {
    for (int k = from; k < to; k += 4) {
      float dt[4], x[4];
      At::four(s_dt, c, k, dt);
      At::four(s_x, c, k, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        pair e[4];
        advance(s, dt[j], x[j], k + j, e);
      }
    }
  };
  // The state before a tile that a visit to the tile before it has found: in the place of a kept state that this spacing never has.
  auto found = [&](bool put, pair (&s)[4]) {
    pair* const p = reinterpret_cast<pair*>(s_raw + tid + (4 * S::ARRAY + S::BC + 2) * NT);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (put) p[(i >> 1) * 2 * NT + (i & 1)] = s[i];
      else s[i] = p[(i >> 1) * 2 * NT + (i & 1)];
    }
  };

  const int tiles = (last - first + STEPS - 1) / STEPS;
  const int busy = n <= first ? 0 : min(tiles, (n - first + STEPS - 1) / STEPS);
  // behind the row's last step: zeros (dB and dC of these steps are the second kernel's)
  for (int i = busy; i < tiles; ++i) {
    const pair zero[4] = {};
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const Chunk h = chunk(p);
      const int k0 = first + i * STEPS;
      if (!h.here || k0 + h.es >= last) continue;
      write(a.du, a.pu, h, k0, zero);
      write(a.ddelta, a.pd, h, k0, zero);
      if (GATE) write(a.dz, a.pz, h, k0, zero);
    }
  }
  // Tiles from the last to the first.  With states kept every 32 steps an odd tile's first state is found by a visit to the even
  // tile before it.  (Segments begin at multiples of 32.)
  auto needs_visit = [&](int i) { return a.spacing > STEPS && (i & 1); };
  int i = busy - 1, st = 0;
  bool visit = i >= 0 && needs_visit(i);
  if (i >= 0) fetch(first + (visit ? i - 1 : i) * STEPS, st);
  while (i >= 0) {
    const int k0 = first + (visit ? i - 1 : i) * STEPS, steps = min(STEPS, stop - k0);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                              // the tile before has been read
    stage(k0, st);
    const int next = visit ? i : i - 1;
    const bool next_visit = !visit && next >= 0 && needs_visit(next);
    if (next >= 0) fetch(first + (next_visit ? next - 1 : next) * STEPS, st ^ 1);
    else asm volatile("cp.async.commit_group;" ::: "memory");
    __syncthreads();
    if (visit) {
      pair s[4];
      kept_state(st, 0, s);
      forwards(s, 0, STEPS);
      found(true, s);
      visit = false;
      st ^= 1;
      continue;
    }
    auto before = [&](int e, pair (&s)[4]) {      // the state before an eight
      if (((k0 + e * EIGHT) & (a.spacing - 1)) == 0) return kept_state(st, e, s);
      if ((k0 & (a.spacing - 1)) == 0) kept_state(st, 0, s);
      else found(false, s);
      if (e > 0) forwards(s, 0, EIGHT);
    };
    pair tA[4] = {};
    for (int e = steps > EIGHT ? 1 : 0; e >= 0; --e) {
      pair decay[EIGHT][4], state[EIGHT + 1][4];  // of a step; before it
      before(e, state[0]);
      float* const red = s_red + warp * EIGHT * 2 * NP;
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
          const pair (&at_start)[4] = state[j0 + j];
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
            G[q] = mul2(carry[q], at_start[q]);    // g a s_{k-1}
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
        if (k >= stop) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) v += s_red[w * EIGHT * 2 * NP + q];
        a.part_bc[((((int64_t)block * a.t + k) * a.batch + b) * a.groups + g) * 2 * NP + q % (2 * NP)] = v;
      }
      if (e > 0) __syncthreads();                 // they have been read
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      pair* const sum = reinterpret_cast<pair*>(s_dA + tid * PER_LANE + 2 * q);
      *sum = add2(*sum, tA[q]);
    }
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const Chunk h = chunk(p);
      if (h.es >= STEPS) continue;
      pair du[4] = {}, dd[4] = {}, dz[4] = {}, vu[4] = {};
      if (h.here && k0 + h.es < stop) {
        pair skip[4], bias[4], u[4], dv[4];
        channel_values(s_skip, h, skip);
        channel_values(s_bias, h, bias);
        unpack_pairs<8>(raw_chunk(st, 0, p), u);
        unpack_pairs<8>(raw_chunk(st, 1, p), dd);
        unpack_pairs<8>(raw_chunk(st, 2, p), dv);
        if (GATE) {
          pair z[4], v[4];
          unpack_pairs<8>(raw_chunk(st, 3, p), z);
          plane(s_v, h, v);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const pair sig = sigmoid2(z[j]), zs = mul2(z[j], sig);
            // silu' = s + z s (1 - s)
            const pair f = fma2(zs, fma2(sig, both(-1.f), both(1.f)), sig);
            dz[j] = mul2(mul2(dv[j], fma2(skip[j], u[j], v[j])), f);
            dv[j] = mul2(dv[j], zs);
          }
        }
        pair gB[4], gA[4], dt[4];
        plane(s_x, h, gB);
        plane(s_dv, h, gA);
        plane(s_dt, h, dt);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          du[j] = fma2(skip[j], dv[j], mul2(dt[j], gB[j]));
          const pair ddt = fma2(u[j], gB[j], mul2(gA[j], both(1.f / kLog2e)));        // A is in units of log 2
          dd[j] = a.softplus ? mul2(ddt, sigmoid2(add2(dd[j], bias[j]))) : ddt;
          vu[j] = mul2(dv[j], u[j]);
        }
      }
      to_plane(s_x, h, vu);
      to_plane(s_dv, h, dd);
      if (h.here && k0 + h.es < last) {
        write(a.du, a.pu, h, k0, du);
        write(a.ddelta, a.pd, h, k0, dd);
        if (GATE) write(a.dz, a.pz, h, k0, dz);
      }
    }
    __syncthreads();
    {
      float v = 0.f, w = 0.f;
      if constexpr (LANES <= 4) {
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
    st ^= 1;
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
  constexpr int bytes = Shape<T, LANES>::FLOATS * 4;
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
