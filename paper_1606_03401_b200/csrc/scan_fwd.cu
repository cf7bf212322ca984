// Selective state space scan, forward: whole sequences, and one token of every row.
//
// Every state decays by a factor of its own, so there is no matrix product in it: a step of a channel takes N exponentials and some
// 4 N multiply-adds on 8 bytes, and the special function unit (16 results a clock and SM) bounds it, at three times what
// the memory would allow for N = 16.  A block owns 128 / LANES channels of one row and walks its steps in tiles; LANES lanes
// share a channel, eight states each in registers, two to an instruction.  Per tile: the elementwise part (dt, dt u), eight channels
// of a step to a thread; the scan out of shared memory; the gate, again elementwise.  Every thread fetches its part of the
// next tile meanwhile, into shared memory, so that 72 registers are enough and an SM keeps seven blocks.
// Measured at 1000 steps x 64 rows x 1024 channels x 16 states in bfloat16, states kept every 8 steps: 471 us; special functions
// 61 % busy, shared-memory pipe 56 %, issue slots 57 %; 2.2 TB/s.
//
// Few rows and channels leave SMs without work, so long sequences are then cut into segments: a first kernel finds the state
// that each segment ends in when it begins with zeros, and the sum of its dt, and the second one starts from those of the
// segments before (s <- exp(A sum dt) s + end, one after the other).  4000 steps of one row of 2048 channels: 628 us without, 44 + 68
// with 32 segments.
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

constexpr int NT = 128;

// What a pass of the kernel computes: outputs; the states that segments end in; the adjoints that they begin with (backward in time).
enum Pass { OUTPUTS, ENDS, ADJOINTS };

template <class T, int LANES>
struct Shape {
  static constexpr int CH = NT / LANES;                                                      // channels of a block
  static constexpr int STEPS = LANES == 1 ? 8 : LANES == 2 ? 16 : 32;                        // of a tile: no more than a group of channels a thread
  static constexpr int NP = PER_LANE * LANES;                                                // states, with those that pad
  static constexpr int QUARTERS = STEPS * 2 * NP / 4;                                        // of the rows of B and C, four states each
  static constexpr int QB = QUARTERS > NT ? QUARTERS / NT : 1;                               // of a thread
  using At = Tile<STEPS, CH>;
  // What threads fetch for a tile, in bytes: three arrays, B and C.  Each thread reads what it fetched itself.
  static constexpr int ARRAY = NT * 8 * (int)sizeof(T), ROWS = QB * NT * 4 * (int)sizeof(T), RAW = 3 * ARRAY + ROWS;
  static constexpr int BYTES = 2 * RAW + 4 * (2 * At::FLOATS + STEPS * 2 * NP + 2 * CH);
};

template <class T, int LANES, int PASS>
__global__ void __launch_bounds__(NT, 7) scan_fwd(const ScanArgs a) {
  using S = Shape<T, LANES>;
  using At = typename S::At;
  constexpr int CH = S::CH, STEPS = S::STEPS, NP = S::NP, QB = S::QB, E8 = 8 * (int)sizeof(T), E4 = 4 * (int)sizeof(T);
  if (PASS == OUTPUTS) sm100::grid_dep_wait();         // for the kernel of the segments' ends
  extern __shared__ __align__(16) uint8_t smem[];
  float* const s_dt = reinterpret_cast<float*>(smem + 2 * S::RAW);    // dt, later the sums over states
  float* const s_x = s_dt + At::FLOATS;                // dt u; ADJOINTS: dy times the gate
  float* const s_bc = s_x + At::FLOATS;                // [STEPS][B, C][NP]
  float* const s_bias = s_bc + STEPS * 2 * NP;         // [CH]
  float* const s_skip = s_bias + CH;                   // [CH]

  const int tid = threadIdx.x, b = blockIdx.y, seg = blockIdx.z + (PASS == ADJOINTS);   // segment 0 hands its adjoint to none
  const int g = blockIdx.x / a.blocks, base = (blockIdx.x % a.blocks) * CH;     // first channel, within the group
  const int d0 = g * a.gchannels + base;
  const int live = min(CH, a.gchannels - base);
  const int n = row_steps(a.lengths, b, a.t);
  const int first = seg * a.segment, last = min(first + a.segment, a.t), stop = min(n, last);

  // scan: a channel and eight of its states
  const int c = tid / LANES, l = tid % LANES;
  const bool mine = c < live;
  const int d = d0 + c;
  pair A[4] = {}, s[4] = {};
  if (mine) {
    load_states(a.A + (int64_t)d * a.states, l, a.states, a.vec_s, A);
#pragma unroll
    for (int i = 0; i < 4; ++i) A[i] = mul2(A[i], both(kLog2e));
  }
  const int64_t place = ((int64_t)b * a.channels + d) * NP;                     // of this channel's states in a layer of `ends`
  const int64_t layer = (int64_t)a.batch * a.channels * NP;
  const int64_t row = ((int64_t)b * a.channels + d) * a.states;
  if (PASS == OUTPUTS && a.segments > 1) {
    if (mine) {
      load_states(a.ends + place, l, NP, true, s);
      // FOLD segments' loads at a time: one after the other they would cost a trip to the L2 each
      for (int j0 = 0; j0 < seg; j0 += FOLD) {
        pair e[FOLD][4];
        float dts[FOLD];
#pragma unroll
        for (int j = 0; j < FOLD; ++j)
          if (j0 + j < seg) {
            load_states(a.ends + (j0 + j + 1) * layer + place, l, NP, true, e[j]);
            dts[j] = a.dts[((int64_t)(j0 + j) * a.batch + b) * a.channels + d];
          }
#pragma unroll
        for (int j = 0; j < FOLD; ++j)
          if (j0 + j < seg)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = carry2(A[i], dts[j], s[i], e[j][i]);
      }
    }
  } else if (PASS == OUTPUTS || (PASS == ENDS && seg == 0)) {
    if (mine && a.s_in) load_states(a.s_in + row, l, a.states, a.vec_s, s);
    if (PASS == ENDS) {
      // the second kernel has the first states from here, as s_out may be where s_in lies
      if (mine) store_states(a.ends + place, l, NP, true, s);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = 0;
    }
  }
  for (int i = tid; i < CH; i += NT) {
    s_bias[i] = a.bias && i < live ? a.bias[d0 + i] : 0.f;
    s_skip[i] = PASS == OUTPUTS && a.skip && i < live ? a.skip[d0 + i] : 0.f;
  }

  // elementwise part: eight channels of a step
  const int ec = (tid % (CH / 8)) * 8, es = tid / (CH / 8), en = min(8, live - ec);
  const bool worker = es < STEPS && en > 0, whole = a.vec_d && en == 8;
  // asks for the tile at k0, into one half of the room
  auto fetch = [&](int k0, int half) {
    uint8_t* const raw = smem + half * S::RAW;
    if (worker && k0 + es < stop) {
      const bool gate = PASS != ENDS && a.z;
      const void* const x[3] = {a.delta, PASS == ADJOINTS ? a.dy : a.u, a.z};
      const Places* const p[3] = {&a.pd, PASS == ADJOINTS ? &a.py : &a.pu, &a.pz};
      auto from = [&](int w) { return (const T*)x[w] + (int64_t)(k0 + es) * p[w]->step + (int64_t)b * p[w]->row + d0 + ec; };
      uint8_t* const to = raw + tid * E8;
      if (whole) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
          if (w < 2 || gate) fetch_n<8>(to + w * S::ARRAY, from(w), 8, true);
      } else {
        Raw<T, 8> r[3];
#pragma unroll
        for (int w = 0; w < 3; ++w)
          if (w < 2 || gate) r[w] = load_raw<8>(from(w), en, false);
#pragma unroll
        for (int w = 0; w < 3; ++w)
          if (w < 2 || gate) memcpy(to + w * S::ARRAY, &r[w], sizeof r[w]);
      }
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1, k = k0 + q / (NP / 2);
      if (q >= S::QUARTERS || k >= stop || n4 >= a.states || (PASS != OUTPUTS && which != (PASS == ADJOINTS))) continue;
      const T* const from = which ? (const T*)a.C + (int64_t)k * a.pc.step + (int64_t)b * a.pc.row : (const T*)a.B + (int64_t)k * a.pb.step + (int64_t)b * a.pb.row;
      fetch_n<4>(raw + 3 * S::ARRAY + q * E4, from + g * a.states + n4, a.states - n4, a.vec_s && n4 + 4 <= a.states);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // the tile's planes and its B and C out of what was fetched
  auto stage = [&](int k0, int half) {
    const uint8_t* const raw = smem + half * S::RAW;
    if (es < STEPS) {
      pair dt[4] = {}, x[4] = {};
      if (worker && k0 + es < stop) {
        unpack_pairs<8>(fetched<T, 8>(raw + tid * E8), dt);
        unpack_pairs<8>(fetched<T, 8>(raw + S::ARRAY + tid * E8), x);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          dt[j] = add2(dt[j], *reinterpret_cast<const pair*>(s_bias + ec + 2 * j));
          if (a.softplus) dt[j] = softplus2(dt[j]);
          if (PASS != ADJOINTS) x[j] = mul2(x[j], dt[j]);
        }
        if (PASS == ADJOINTS && a.z) {
          pair z[4];
          unpack_pairs<8>(fetched<T, 8>(raw + 2 * S::ARRAY + tid * E8), z);
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] = mul2(x[j], mul2(z[j], sigmoid2(z[j])));
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = unpack2(dt[j]), w = unpack2(x[j]);
        s_dt[At::at(ec + 2 * j, es)] = v.x;
        s_dt[At::at(ec + 2 * j + 1, es)] = v.y;
        s_x[At::at(ec + 2 * j, es)] = w.x;
        s_x[At::at(ec + 2 * j + 1, es)] = w.y;
      }
    }
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const int q = tid + i * NT, n4 = (q % (NP / 4)) * 4, which = (q / (NP / 4)) & 1;
      if (q >= S::QUARTERS || (PASS != OUTPUTS && which != (PASS == ADJOINTS))) continue;
      float f[4] = {0, 0, 0, 0};
      if (k0 + q / (NP / 2) < stop && n4 < a.states) unpack<4>(fetched<T, 4>(raw + 3 * S::ARRAY + q * E4), f);
      *reinterpret_cast<float4*>(s_bc + q * 4) = make_float4(f[0], f[1], f[2], f[3]);
    }
  };

  const int tiles = (last - first + STEPS - 1) / STEPS;
  const int busy = n <= first ? 0 : min(tiles, (n - first + STEPS - 1) / STEPS);     // tiles with a step of the row
  float dts = 0.f;
  if (busy > 0) fetch(first + (PASS == ADJOINTS ? busy - 1 : 0) * STEPS, 0);
  __syncthreads();                                     // bias and skip are there
  for (int i = 0, half = 0; i < busy; ++i, half ^= 1) {
    const int k0 = first + (PASS == ADJOINTS ? busy - 1 - i : i) * STEPS, steps = min(STEPS, stop - k0);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    stage(k0, half);
    if (i + 1 < busy) fetch(PASS == ADJOINTS ? k0 - STEPS : k0 + STEPS, half ^ 1);
    __syncthreads();
    for (int jj = 0; jj < steps; jj += 4) {
      const int j0 = PASS == ADJOINTS ? (steps - 1) / 4 * 4 - jj : jj;
      float dt[4], x[4], part[4];
      At::four(s_dt, c, j0, dt);
      At::four(s_x, c, j0, x);
      if (PASS == OUTPUTS && a.kept && ((k0 + j0) & (a.spacing - 1)) == 0 && mine)
        store_states(a.kept + (int64_t)((k0 + j0) / a.spacing) * layer + place, l, NP, true, s);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int j = PASS == ADJOINTS ? 3 - q : q;
        const pair dt2 = both(dt[j]), x2 = both(x[j]);
        const float* const bc = s_bc + (j0 + j) * 2 * NP + PER_LANE * l;
        pair in[4], C[4];
        lds8(bc + (PASS == ADJOINTS ? NP : 0), in);
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const pair e = decay2(dt2, A[i4]);
          s[i4] = PASS == ADJOINTS ? mul2(e, fma2(x2, in[i4], s[i4])) : fma2(e, s[i4], mul2(x2, in[i4]));
        }
        if (PASS != OUTPUTS) dts += dt[j];
        if (PASS == OUTPUTS) {
          lds8(bc + NP, C);
          part[j] = dot(C, s);
        }
      }
      if (PASS == OUTPUTS) {
        sum_lanes<LANES>(part, l);
        put_steps<LANES>(s_dt + At::at(c, j0), l, part);
      }
    }
    __syncthreads();
    if (PASS == OUTPUTS && worker && k0 + es < last) {
      pair out[4] = {};
      if (k0 + es < n) {
        const uint8_t* const raw = smem + half * S::RAW;
        pair u[4], z[4];
        unpack_pairs<8>(fetched<T, 8>(raw + S::ARRAY + tid * E8), u);
        if (a.z) unpack_pairs<8>(fetched<T, 8>(raw + 2 * S::ARRAY + tid * E8), z);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const pair v = pack2(s_dt[At::at(ec + 2 * j, es)], s_dt[At::at(ec + 2 * j + 1, es)]);
          out[j] = fma2(*reinterpret_cast<const pair*>(s_skip + ec + 2 * j), u[j], v);
          if (a.z) out[j] = mul2(mul2(out[j], z[j]), sigmoid2(z[j]));
        }
      }
      store_pairs<8>((T*)a.y + (int64_t)(k0 + es) * a.py.step + (int64_t)b * a.py.row + d0 + ec, out, en, whole);
    }
  }
  if (PASS == OUTPUTS) {
    // what lies behind the row's last step: zeros
    const pair zero[4] = {};
    if (worker)
      for (int k = first + busy * STEPS + es; k < last; k += STEPS)
        store_pairs<8>((T*)a.y + (int64_t)k * a.py.step + (int64_t)b * a.py.row + d0 + ec, zero, en, whole);
    if (mine && a.s_out && seg == a.segments - 1) store_states(a.s_out + row, l, a.states, a.vec_s, s);
  } else if (mine) {
    store_states(a.ends + (int64_t)(seg + 1) * layer + place, l, NP, true, s);
    if (l == 0) a.dts[((int64_t)seg * a.batch + b) * a.channels + d] = dts;
  }
}

// One step of every row: the states are read and written once, and nothing is staged.
constexpr int NT1 = 256;
template <class T, int LANES>
__global__ void __launch_bounds__(NT1) scan_token(const ScanArgs a) {
  constexpr int CH = NT1 / LANES, NP = PER_LANE * LANES;
  const int b = blockIdx.y, c = threadIdx.x / LANES, l = threadIdx.x % LANES;
  const int64_t d = (int64_t)blockIdx.x * CH + c;
  const bool mine = d < a.channels;
  const int n = row_steps(a.lengths, b, 1);
  pair A[4] = {}, s[4] = {}, B[4] = {}, C[4] = {};
  float u = 0.f, pre = 0.f, z = 0.f, skip = 0.f;
  const int64_t row = ((int64_t)b * a.channels + d) * a.states;
  if (mine) {
    if (a.s_in) load_states(a.s_in + row, l, a.states, a.vec_s, s);
    if (n > 0) {
      load_states(a.A + d * a.states, l, a.states, a.vec_s, A);
      const int g = (int)(d / a.gchannels);
      auto load = [&](const void* base, const Places& p, pair (&v)[4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n4 = PER_LANE * l + 4 * h;
          if (n4 >= a.states) continue;
          pair f[2];
          unpack_pairs<4>(load_raw<4>((const T*)base + (int64_t)b * p.row + g * a.states + n4, a.states - n4, a.vec_s && n4 + 4 <= a.states), f);
          v[2 * h] = f[0];
          v[2 * h + 1] = f[1];
        }
      };
      load(a.B, a.pb, B);
      load(a.C, a.pc, C);
      u = to_f<T>(((const T*)a.u)[(int64_t)b * a.pu.row + d]);
      pre = to_f<T>(((const T*)a.delta)[(int64_t)b * a.pd.row + d]) + (a.bias ? a.bias[d] : 0.f);
      if (a.z) z = to_f<T>(((const T*)a.z)[(int64_t)b * a.pz.row + d]);
      if (a.skip) skip = a.skip[d];
    }
    if (a.kept) store_states(a.kept + ((int64_t)b * a.channels + d) * NP, l, NP, true, s);
  }
  float v = 0.f;
  if (n > 0) {
    const float dt = step_size(pre, a.softplus);
    const pair dt2 = both(dt), x2 = both(dt * u);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fma2(decay2(dt2, mul2(A[i], both(kLog2e))), s[i], mul2(x2, B[i]));
    v = dot(C, s);
  }
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  if (!mine) return;
  if (a.s_out) store_states(a.s_out + row, l, a.states, a.vec_s, s);
  if (l == 0) {
    v = fmaf(skip, u, v);
    ((T*)a.y)[(int64_t)b * a.py.row + d] = from_f<T>(n > 0 ? (a.z ? v * z * sigmoid(z) : v) : 0.f);
  }
}

template <class T, int LANES, int PASS>
bool launch_pass(const ScanArgs& a, int segments, cudaStream_t s) {
  constexpr int bytes = Shape<T, LANES>::BYTES;
  // per call: function attributes belong to the current device
  if (bytes > 48 * 1024 && cudaFuncSetAttribute(scan_fwd<T, LANES, PASS>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  const dim3 grid((unsigned)(a.groups * a.blocks), (unsigned)a.batch, (unsigned)segments);
  return launch_on(PASS == OUTPUTS && a.segments > 1, scan_fwd<T, LANES, PASS>, grid, dim3(NT), bytes, s, a) == cudaSuccess;
}
template <class T, int LANES>
bool launch(const ScanArgs& a, cudaStream_t s) {
  if (a.t == 1) {
    const dim3 grid((unsigned)((a.channels + NT1 / LANES - 1) / (NT1 / LANES)), (unsigned)a.batch);
    scan_token<T, LANES><<<grid, NT1, 0, counted(s)>>>(a);
    return true;
  }
  if (a.segments > 1 && !launch_pass<T, LANES, ENDS>(a, a.segments - 1, s)) return false;    // nothing begins where the last one ends
  return launch_pass<T, LANES, OUTPUTS>(a, a.segments, s);
}
template <class T, int LANES>
bool launch_adj(const ScanArgs& a, cudaStream_t s) {
  return launch_pass<T, LANES, ADJOINTS>(a, a.segments - 1, s);
}

}  // namespace

int scan_fwd_channels(int lanes) { return NT / lanes; }

template <class T>
static int blocks_of_sm(int lanes) {
  const int bytes = lanes == 1 ? Shape<T, 1>::BYTES : lanes == 2 ? Shape<T, 2>::BYTES : lanes == 4 ? Shape<T, 4>::BYTES : Shape<T, 8>::BYTES;
  const int n = 227 * 1024 / (bytes + 1024);
  return n < 7 ? n : 7;
}
int scan_fwd_blocks(int lanes, bool half) { return half ? blocks_of_sm<bf16>(lanes) : blocks_of_sm<float>(lanes); }

#define BY_LANES(F, T)                          \
  switch (scan_lanes(a.states)) {               \
    case 1: return F<T, 1>(a, s);               \
    case 2: return F<T, 2>(a, s);               \
    case 4: return F<T, 4>(a, s);               \
    default: return F<T, 8>(a, s);              \
  }
bool scan_forward(const ScanArgs& a, bool half, cudaStream_t s) {
  if (half) { BY_LANES(launch, bf16) }
  BY_LANES(launch, float)
}
bool scan_adjoints(const ScanArgs& a, bool half, cudaStream_t s) {
  if (half) { BY_LANES(launch_adj, bf16) }
  BY_LANES(launch_adj, float)
}
#undef BY_LANES

}  // namespace seq
}  // namespace mebptt
