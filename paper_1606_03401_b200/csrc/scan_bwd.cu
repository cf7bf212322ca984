// Selective state space scan, backward.
//
// A block owns NT / LANES channels of one row and walks a segment's tiles of 32 steps from the last to the first; LANES lanes share
// a channel, four states each.  States are not kept but every `spacing` steps: eight steps at a time are run forwards from the
// state before them, with the decays a and a s_{k-1} of the eight steps in registers, and then backwards.  Where states are kept
// further apart, a tile first runs forwards once more to have the state before each of its eights (one exponential more for
// each state and step).
//
// Sums go three ways.  Over the states of a channel (v, g B, A a s g): the lanes of a channel, four steps at a time, so that lane l
// ends with the sums of step l.  Over channels (dB, dC): halving exchanges among the lanes of a warp with the same states, then
// the block's warps through shared memory, then the blocks of a group in a second kernel.  Over time (dA, dskip, ddelta_bias): in
// registers, a sum per tile added to a sum of tiles, then rows and segments in the second kernel.  The order is fixed.
//
// Bound by instruction issue: some 14 multiply-adds (two states an instruction), one exponential and two shuffles for each
// state and step.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.hpp"
#include "scan.hpp"
#include "scan_dev.cuh"
#include "scan_kernels.hpp"

namespace mebptt {
namespace seq {

namespace {

constexpr int EIGHT = 8;

template <int LANES>
struct Shape {
  static constexpr int NT = LANES <= 2 ? 128 : 256;
  static constexpr int CH = NT / LANES, NP = 4 * LANES, WARPS = NT / 32;
  static constexpr int CHUNKS = TILE * CH / 8 / NT > 0 ? TILE * CH / 8 / NT : 1;    // groups of eight channels a thread, in the elementwise part
  static constexpr int PLANE = CH * (TILE + 4);
  static constexpr int RED = WARPS * EIGHT * 2 * NP;                                // sums of one eight, by warp
  static constexpr int FLOATS = 3 * PLANE + TILE * 2 * NP + 2 * RED + 3 * NT * 4;
};

// Sums of the eight values v (dB and dC of a lane's four states) over the 32 / LANES lanes with the same states.  Lanes halve the
// values among them as long as there are any to halve; what a lane ends with begins at index `first` and is 8 / min(8, 32 / LANES)
// values long, in v[0..].
template <int LANES>
__device__ __forceinline__ int sum_channels(float (&v)[8], int lane) {
  int first = 0;
#pragma unroll
  for (int m = 16, left = 8; m >= LANES; m /= 2) {
    if (left > 1) {
      const bool hi = lane & m;
      left /= 2;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i < left) {
          const float send = hi ? v[i] : v[i + left];
          v[i] = (hi ? v[i + left] : v[i]) + __shfl_xor_sync(0xffffffffu, send, m);
        }
      }
      if (hi) first += left;
    } else {
      v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
    }
  }
  return first;
}

template <class T, int LANES, bool GATE>
__global__ void __launch_bounds__(Shape<LANES>::NT, 512 / Shape<LANES>::NT) scan_bwd(const ScanArgs a) {
  using S = Shape<LANES>;
  constexpr int NT = S::NT, CH = S::CH, NP = S::NP, WARPS = S::WARPS, CHUNKS = S::CHUNKS;
  extern __shared__ __align__(16) float sm[];
  float* const s_dt = sm;                         // dt, then the sums over states of C s
  float* const s_x = s_dt + S::PLANE;             // dt u, then of g B, then dv u
  float* const s_dv = s_x + S::PLANE;             // dv, then of A a s g, then ddelta
  float* const s_bc = s_dv + S::PLANE;            // [TILE][B, C][NP]
  float* const s_red = s_bc + TILE * 2 * NP;      // [2][WARPS][EIGHT][2 NP]
  float* const s_start = s_red + 2 * S::RED;      // [3][NT][4]: states before the eights of a tile but the first

  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, b = blockIdx.y, seg = blockIdx.z;
  const int g = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks, base = block * CH;
  const int d0 = g * a.gchannels + base;
  const int live = min(CH, a.gchannels - base);
  const int n = row_steps(a.lengths, b, a.t);
  const int first = seg * a.segment, last = min(first + a.segment, a.t);

  const T* const Bm = (const T*)a.B + (int64_t)b * a.pb.row + g * a.states;
  const T* const Cm = (const T*)a.C + (int64_t)b * a.pc.row + g * a.states;

  const int c = tid / LANES, l = tid % LANES;
  const bool mine = c < live;
  const int d = d0 + c;
  Four A = {0, 0};                                // in units of log 2
  if (mine) {
    A = load_states(a.A + (int64_t)d * a.states, 4 * l, a.states, a.vec_s);
    const pair k = both(kLog2e);
    A.a = mul2(A.a, k); A.b = mul2(A.b, k);
  }
  const int64_t place = ((int64_t)b * a.channels + d) * NP + 4 * l;
  const int64_t layer = (int64_t)a.batch * a.channels * NP;
  // what later steps hand down: a_{k+1} g_{k+1}
  Four carry = {0, 0};
  if (mine) {
    if (a.ds_out) carry = load_states(a.ds_out + ((int64_t)b * a.channels + d) * a.states, 4 * l, a.states, a.vec_s);
    for (int j = a.segments - 1; j > seg; --j) {
      const Four e = lds4(a.ends + (j + 1) * layer + place);
      const float dts = a.dts[((int64_t)j * a.batch + b) * a.channels + d];
      carry.a = carry2(A.a, dts, carry.a, e.a);
      carry.b = carry2(A.b, dts, carry.b, e.b);
    }
  }
  Four dA = {0, 0};
  float dskip = 0.f, dbias = 0.f;

  const int tiles = (last - first + TILE - 1) / TILE;
  const int busy = n <= first ? 0 : min(tiles, (n - first + TILE - 1) / TILE);
  for (int i = tiles - 1; i >= 0; --i) {
    const int k0 = first + i * TILE, steps = min(TILE, min(n, last) - k0);
    if (i >= busy) {
      // behind the row's last step: zeros (dB and dC of these steps are the second kernel's)
      const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      for (int q = tid; q < TILE * (CH / 8); q += NT) {
        const int ec = (q % (CH / 8)) * 8, k = k0 + q / (CH / 8), en = min(8, live - ec);
        if (en <= 0 || k >= last) continue;
        const bool whole = a.vec_d && en == 8;
        store_n<8>((T*)a.du + (int64_t)k * a.pu.step + (int64_t)b * a.pu.row + d0 + ec, zero, en, whole);
        store_n<8>((T*)a.ddelta + (int64_t)k * a.pd.step + (int64_t)b * a.pd.row + d0 + ec, zero, en, whole);
        if (GATE) store_n<8>((T*)a.dz + (int64_t)k * a.pz.step + (int64_t)b * a.pz.row + d0 + ec, zero, en, whole);
      }
      continue;
    }
    __syncthreads();                              // the tile before has been read
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const int q = tid + p * NT, ec = (q % (CH / 8)) * 8, es = q / (CH / 8), k = k0 + es, en = min(8, live - ec);
      if (es >= TILE) continue;
      const bool in = en > 0 && k < n && k < last, whole = a.vec_d && en == 8;
      float fu[8], pre[8], dv[8], z[8];
      unpack<8>(in ? load_raw<8>((const T*)a.u + (int64_t)k * a.pu.step + (int64_t)b * a.pu.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), fu);
      unpack<8>(in ? load_raw<8>((const T*)a.delta + (int64_t)k * a.pd.step + (int64_t)b * a.pd.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), pre);
      unpack<8>(in ? load_raw<8>((const T*)a.dy + (int64_t)k * a.py.step + (int64_t)b * a.py.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), dv);
      if (GATE) unpack<8>(in ? load_raw<8>((const T*)a.z + (int64_t)k * a.pz.step + (int64_t)b * a.pz.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float dt = in ? step_size(pre[j] + (a.bias && j < en ? a.bias[d0 + ec + j] : 0.f), a.softplus) : 0.f;
        s_dt[at<TILE>(ec + j, es)] = dt;
        s_x[at<TILE>(ec + j, es)] = in ? dt * fu[j] : 0.f;
        s_dv[at<TILE>(ec + j, es)] = !in ? 0.f : GATE ? dv[j] * z[j] * sigmoid(z[j]) : dv[j];
      }
    }
    for (int q = tid; q < TILE * 2 * LANES; q += NT) {
      const int n4 = (q % LANES) * 4, which = (q / LANES) & 1, k = k0 + q / (2 * LANES);
      float f[4] = {0, 0, 0, 0};
      if (k < n && k < last && n4 < a.states)
        unpack<4>(load_raw<4>((which ? Cm + (int64_t)k * a.pc.step : Bm + (int64_t)k * a.pb.step) + n4, a.states - n4, a.vec_s && n4 + 4 <= a.states), f);
      *reinterpret_cast<float4*>(s_bc + q * 4) = make_float4(f[0], f[1], f[2], f[3]);
    }
    // the state before the tile; with states kept further apart than eight steps, those before its other eights
    Four s0 = {0, 0};
    if (mine) s0 = lds4(a.kept + (int64_t)(k0 / a.spacing) * layer + place);
    __syncthreads();
    if (a.spacing > EIGHT) {
      Four s = s0;
      for (int e = 0; (e + 1) * EIGHT < steps; ++e) {
#pragma unroll
        for (int j0 = 0; j0 < EIGHT; j0 += 4) {
          const float4 dt4 = four_steps<TILE>(s_dt, c, e * EIGHT + j0), x4 = four_steps<TILE>(s_x, c, e * EIGHT + j0);
          const float dt[4] = {dt4.x, dt4.y, dt4.z, dt4.w}, x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const Four B = lds4(s_bc + (e * EIGHT + j0 + j) * 2 * NP + 4 * l);
            s.a = fma2(decay2(both(dt[j]), A.a), s.a, mul2(both(x[j]), B.a));
            s.b = fma2(decay2(both(dt[j]), A.b), s.b, mul2(both(x[j]), B.b));
          }
        }
        st4(s_start + (e * NT + tid) * 4, s);
      }
    }
    Four tA = {0, 0};
    const int eights = (steps + EIGHT - 1) / EIGHT;
    for (int e = eights - 1; e >= 0; --e) {
      Four s = s0;
      if (e > 0) {
        if (a.spacing > EIGHT) s = lds4(s_start + ((e - 1) * NT + tid) * 4);
        else if (mine) s = lds4(a.kept + (int64_t)(k0 / EIGHT + e) * layer + place);
      }
      float* const red = s_red + (e & 1) * S::RED + warp * EIGHT * 2 * NP;
      pair da[EIGHT][2], h[EIGHT][2];             // decay of a step; decayed state that it begins with
#pragma unroll
      for (int j0 = 0; j0 < EIGHT; j0 += 4) {
        const float4 dt4 = four_steps<TILE>(s_dt, c, e * EIGHT + j0), x4 = four_steps<TILE>(s_x, c, e * EIGHT + j0);
        const float dt[4] = {dt4.x, dt4.y, dt4.z, dt4.w}, x[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const Four B = lds4(s_bc + (e * EIGHT + j0 + j) * 2 * NP + 4 * l);
          da[j0 + j][0] = decay2(both(dt[j]), A.a);
          da[j0 + j][1] = decay2(both(dt[j]), A.b);
          h[j0 + j][0] = mul2(da[j0 + j][0], s.a);
          h[j0 + j][1] = mul2(da[j0 + j][1], s.b);
          s.a = fma2(both(x[j]), B.a, h[j0 + j][0]);
          s.b = fma2(both(x[j]), B.b, h[j0 + j][1]);
        }
      }
#pragma unroll
      for (int j0 = EIGHT - 4; j0 >= 0; j0 -= 4) {
        const int k = e * EIGHT + j0;
        const float4 dt4 = four_steps<TILE>(s_dt, c, k), x4 = four_steps<TILE>(s_x, c, k), v4 = four_steps<TILE>(s_dv, c, k);
        const float dt[4] = {dt4.x, dt4.y, dt4.z, dt4.w}, x[4] = {x4.x, x4.y, x4.z, x4.w}, dv[4] = {v4.x, v4.y, v4.z, v4.w};
        float sv[4], sB[4], sA[4];
#pragma unroll
        for (int j = 3; j >= 0; --j) {
          const Four B = lds4(s_bc + (k + j) * 2 * NP + 4 * l), C = lds4(s_bc + ((k + j) * 2 + 1) * NP + 4 * l);
          const pair x2 = both(x[j]), v2 = both(dv[j]);
          const pair sa = fma2(x2, B.a, h[j0 + j][0]), sb = fma2(x2, B.b, h[j0 + j][1]);
          if (GATE) sv[j] = sum2(fma2(C.a, sa, mul2(C.b, sb)));
          const pair ga = fma2(v2, C.a, carry.a), gb = fma2(v2, C.b, carry.b);
          sB[j] = sum2(fma2(ga, B.a, mul2(gb, B.b)));
          const pair gha = mul2(ga, h[j0 + j][0]), ghb = mul2(gb, h[j0 + j][1]);
          sA[j] = sum2(fma2(A.a, gha, mul2(A.b, ghb)));
          tA.a = fma2(both(dt[j]), gha, tA.a);
          tA.b = fma2(both(dt[j]), ghb, tA.b);
          carry.a = mul2(da[j0 + j][0], ga);
          carry.b = mul2(da[j0 + j][1], gb);
          const float2 b0 = unpack2(mul2(x2, ga)), b1 = unpack2(mul2(x2, gb)), c0 = unpack2(mul2(v2, sa)), c1 = unpack2(mul2(v2, sb));
          float r[8] = {b0.x, b0.y, b1.x, b1.y, c0.x, c0.y, c1.x, c1.y};
          const int r0 = sum_channels<LANES>(r, lane);
          // (with fewer than four lanes a channel, several lanes have the same sums and store the same values)
#pragma unroll
          for (int q = 0; q < (LANES >= 4 ? LANES / 4 : 1); ++q)
            red[(j0 + j) * 2 * NP + ((r0 + q) >> 2) * NP + 4 * l + ((r0 + q) & 3)] = r[q];
        }
        if (GATE) sum_lanes<LANES>(sv, l);
        sum_lanes<LANES>(sB, l);
        sum_lanes<LANES>(sA, l);
#pragma unroll
        for (int q = 0; q < steps_of_lane<LANES>; ++q) {
          const int w = at<TILE>(c, k + first_step<LANES>(l) + q);
          if (GATE) s_dt[w] = sv[q];
          s_x[w] = sB[q];
          s_dv[w] = sA[q];
        }
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
    __syncthreads();
#pragma unroll
    for (int p = 0; p < CHUNKS; ++p) {
      const int q = tid + p * NT, ec = (q % (CH / 8)) * 8, es = q / (CH / 8), k = k0 + es, en = min(8, live - ec);
      if (es >= TILE) continue;
      const bool in = en > 0 && k < n && k < last, whole = a.vec_d && en == 8;
      float fu[8], pre[8], dy[8], z[8], du[8], dd[8], dz[8];
      unpack<8>(in ? load_raw<8>((const T*)a.u + (int64_t)k * a.pu.step + (int64_t)b * a.pu.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), fu);
      unpack<8>(in ? load_raw<8>((const T*)a.delta + (int64_t)k * a.pd.step + (int64_t)b * a.pd.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), pre);
      unpack<8>(in ? load_raw<8>((const T*)a.dy + (int64_t)k * a.py.step + (int64_t)b * a.py.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), dy);
      if (GATE) unpack<8>(in ? load_raw<8>((const T*)a.z + (int64_t)k * a.pz.step + (int64_t)b * a.pz.row + d0 + ec, en, whole) : raw_zeros<T, 8>(), z);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int w = at<TILE>(ec + j, es);
        const float skip = a.skip && j < en ? a.skip[d0 + ec + j] : 0.f;
        const float p1 = pre[j] + (a.bias && j < en ? a.bias[d0 + ec + j] : 0.f);
        float dv = dy[j];
        if (GATE) {
          const float sig = sigmoid(z[j]);
          dv = dy[j] * z[j] * sig;
          dz[j] = in ? dy[j] * fmaf(skip, fu[j], s_dt[w]) * dsilu(z[j], sig) : 0.f;
        }
        const float gB = s_x[w];
        du[j] = in ? fmaf(skip, dv, step_size(p1, a.softplus) * gB) : 0.f;
        dd[j] = in ? fmaf(fu[j], gB, s_dv[w] * (1.f / kLog2e)) * (a.softplus ? sigmoid(p1) : 1.f) : 0.f;   // A is in units of log 2
        s_x[w] = in ? dv * fu[j] : 0.f;
        s_dv[w] = dd[j];
      }
      if (en > 0 && k < last) {
        store_n<8>((T*)a.du + (int64_t)k * a.pu.step + (int64_t)b * a.pu.row + d0 + ec, du, en, whole);
        store_n<8>((T*)a.ddelta + (int64_t)k * a.pd.step + (int64_t)b * a.pd.row + d0 + ec, dd, en, whole);
        if (GATE) store_n<8>((T*)a.dz + (int64_t)k * a.pz.step + (int64_t)b * a.pz.row + d0 + ec, dz, en, whole);
      }
    }
    __syncthreads();
    {
      float v = 0.f, w = 0.f;
      if constexpr (LANES <= 8) {
#pragma unroll
        for (int q = 0; q < TILE / 4 / LANES; ++q) {
          const int k = (q * LANES + l) * 4;
          const float4 v4 = four_steps<TILE>(s_x, c, k), w4 = four_steps<TILE>(s_dv, c, k);
          v += (v4.x + v4.y) + (v4.z + v4.w);
          w += (w4.x + w4.y) + (w4.z + w4.w);
        }
      } else {
#pragma unroll
        for (int q = 0; q < TILE / LANES; ++q) {
          v += s_x[at<TILE>(c, q * LANES + l)];
          w += s_dv[at<TILE>(c, q * LANES + l)];
        }
      }
      dskip += v;
      dbias += w;
      dA.a = add2(dA.a, tA.a);
      dA.b = add2(dA.b, tA.b);
    }
  }
#pragma unroll
  for (int m = 1; m < LANES; m *= 2) {
    dskip += __shfl_xor_sync(0xffffffffu, dskip, m);
    dbias += __shfl_xor_sync(0xffffffffu, dbias, m);
  }
  if (!mine) return;
  const int64_t at_part = ((int64_t)seg * a.batch + b) * a.channels + d;
  st4(a.part_a + at_part * NP + 4 * l, dA);
  if (l == 0) {
    a.part_d[at_part] = dskip;
    a.part_b[at_part] = dbias;
  }
  if (seg == 0 && a.ds_in) store_states(a.ds_in + ((int64_t)b * a.channels + d) * a.states, 4 * l, a.states, a.vec_s, carry);
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
  constexpr int bytes = Shape<LANES>::FLOATS * 4;
  // per call: function attributes belong to the current device
  if (cudaFuncSetAttribute(scan_bwd<T, LANES, GATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return false;
  const dim3 grid((unsigned)(a.groups * a.blocks), (unsigned)a.batch, (unsigned)a.segments);
  scan_bwd<T, LANES, GATE><<<grid, Shape<LANES>::NT, bytes, counted(s)>>>(a);
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
    case 8: return launch<T, 8>(a, s);
    default: return launch<T, 16>(a, s);
  }
}

}  // namespace

int scan_bwd_channels(int lanes) { return (lanes <= 2 ? 128 : 256) / lanes; }

bool scan_backward(const ScanArgs& a, bool half, float* dA, void* dB, void* dC, float* dskip, float* dbias, cudaStream_t s) {
  if (!(half ? launch_lanes<bf16>(a, s) : launch_lanes<float>(a, s))) return false;
  const int np = 4 * scan_lanes(a.states);
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
