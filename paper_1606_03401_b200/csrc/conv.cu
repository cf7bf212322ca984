// Short causal convolution, channel by channel, with a state for token-by-token use; forward and backward.
//
// A thread has `C` neighbouring channels of one row and walks a run of time steps with the last width - 1 inputs in registers, so that
// every input is loaded once (and width - 1 of them a second time where a run begins).  Loads of U steps are issued together,
// while the U steps before them are computed; two channels share an instruction.
// Bound by memory (2 accesses an element forward, 3 backward), with the gate's exponential and reciprocal close behind: 1000 steps
// x 64 rows x 1024 channels, width 4, bfloat16: forward 56 us (4.7 TB/s, special functions 55 %), backward 100 us (3.9 TB/s, issue 51 %).
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "launch.hpp"
#include "mebptt.h"
#include "seq.hpp"
#include "seq_dev.cuh"
#include "sm100.cuh"

namespace mebptt {
namespace seq {

namespace {

constexpr int FWD = 4;        // channels of a thread: taps, inputs, and backward also gradients and sums, are held for each
constexpr int bwd_channels(int bytes, int width) { return bytes == 2 && width <= 4 ? 4 : 2; }
// Blocks an SM keeps: as many registers as that leaves a thread hold its channels without spilling.  (1000 x 64 x 1024 bfloat16, width 4:
// 4 channels and 4 blocks 110 us, 2 channels and 5 blocks 135; float32, 32 rows: 2 and 5 83 us, 4 and 2 110.)
constexpr int bwd_blocks(int bytes, int width) { return width > 4 ? 3 : bytes == 2 ? 4 : 5; }
constexpr int U = 4;          // steps whose loads are issued together
constexpr int ROWS = 4;       // runs of a block that share their channels
constexpr int COLS = 32;      // groups of channels of a block

struct ConvArgs {
  const void* x; const void* w; const float* bias; const void* s_in; const int32_t* lengths;
  const void* dy; const void* ds_out;
  void* y; void* s_out;                  // forward
  void* dx; void* ds_in; float* part;    // backward
  Places px, py;
  int batch, channels, t, run, runs;     // steps of a run, runs of a row
  int groups;                            // of C channels
  int silu;
};

// `n` of the C channels at p, as pairs.  VEC: all of them, as one.
template <int C, bool VEC, class T>
__device__ __forceinline__ Raw<T, C> get(const T* p, int n) { return load_raw<C>(p, n, VEC); }
template <int C, bool VEC, class T>
__device__ __forceinline__ void put(T* p, const pair (&f)[C / 2], int n) { store_pairs<C>(p, f, n, VEC); }

// The last W - 1 inputs before step k0 of a row: inputs, or the state before step 0 (k0 = 0, or k0 >= W - 1).  Zeros at or past step n.
template <int C, int W, bool VEC, class T>
__device__ __forceinline__ void load_before(const ConvArgs& a, const T* x, int b, int k0, int n, int c0, int nc, pair (&f)[W > 1 ? W - 1 : 1][C / 2]) {
#pragma unroll
  for (int i = 0; i < W - 1; ++i) {
    const int k = k0 - (W - 1) + i;
    Raw<T, C> r = raw_zeros<T, C>();
    if (k0 == 0) {
      if (a.s_in) r = get<C, VEC>((const T*)a.s_in + ((int64_t)b * (W - 1) + i) * a.channels + c0, nc);
    } else if (k < n) {
      r = get<C, VEC>(x + (int64_t)k * a.px.step, nc);
    }
    unpack_pairs<C>(r, f[i]);
  }
}
template <int C, int W, class T>
__device__ __forceinline__ void load_taps(const ConvArgs& a, int c0, int nc, pair (&w)[W][C / 2], pair (&bias)[C / 2]) {
#pragma unroll
  for (int c = 0; c < C; c += 2) {
    const bool one = c < nc, two = c + 1 < nc;
    bias[c / 2] = pack2(a.bias && one ? a.bias[c0 + c] : 0.f, a.bias && two ? a.bias[c0 + c + 1] : 0.f);
    const T* t = (const T*)a.w + (int64_t)(c0 + c) * W;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][c / 2] = pack2(one ? to_f<T>(t[j]) : 0.f, two ? to_f<T>(t[W + j]) : 0.f);
  }
}

template <class T, int C, int W, bool VEC>
__global__ void __launch_bounds__(COLS* ROWS) conv_fwd(const ConvArgs a) {
  constexpr int P = C / 2, B = W > 1 ? W - 1 : 1;
  const int group = blockIdx.y * COLS + threadIdx.x;
  const int64_t item = (int64_t)blockIdx.x * ROWS + threadIdx.y;    // run of a row: rows of one run are neighbours
  if (group >= a.groups || item >= (int64_t)a.batch * a.runs) return;
  const int b = (int)(item % a.batch), r = (int)(item / a.batch);
  const int c0 = group * C, nc = min(C, a.channels - c0);
  const int n = row_steps(a.lengths, b, a.t);
  const int k0 = r * a.run, k1 = min(k0 + a.run, a.t), live = max(k0, min(k1, n));      // steps k0 .. live - 1 are the row's
  const T* x = (const T*)a.x + (int64_t)b * a.px.row + c0;
  T* y = (T*)a.y + (int64_t)b * a.py.row + c0 + (int64_t)k0 * a.py.step;

  pair win[B][P];
  load_before<C, W, VEC>(a, x, b, k0, n, c0, nc, win);
  if (W > 1 && r == 0 && a.s_out) {
    // the last W - 1 of state and inputs; this thread alone reads and writes this part of the state
    pair out[B][P];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      const int k = n - (W - 1) + i;
      if (k >= 0) {
        unpack_pairs<C>(get<C, VEC>(x + (int64_t)k * a.px.step, nc), out[i]);
      } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
          if (j == n + i) {
#pragma unroll
            for (int c = 0; c < P; ++c) out[i][c] = win[j][c];
          }
      }
    }
    T* const so = (T*)a.s_out + (int64_t)b * (W - 1) * a.channels + c0;
#pragma unroll
    for (int i = 0; i < W - 1; ++i) put<C, VEC>(so + (int64_t)i * a.channels, out[i], nc);
  }

  pair w[W][P], bias[P];
  load_taps<C, W, T>(a, c0, nc, w, bias);
  const T* next_x = x + (int64_t)k0 * a.px.step;
  Raw<T, C> raw[U], next[U];
  auto load = [&](int k) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      next[i] = k + i < live ? get<C, VEC>(next_x, nc) : raw_zeros<T, C>();
      next_x += a.px.step;
    }
  };
  load(k0);
  for (int k = k0; k < live; k += U) {
#pragma unroll
    for (int i = 0; i < U; ++i) raw[i] = next[i];
    load(k + U);
    const bool full = k + U <= live;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      pair v[P], p[P];
      unpack_pairs<C>(raw[i], v);
#pragma unroll
      for (int c = 0; c < P; ++c) {
        p[c] = fma2(w[W - 1][c], v[c], bias[c]);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) p[c] = fma2(w[j][c], win[j][c], p[c]);
        if (a.silu) p[c] = mul2(p[c], sigmoid2(p[c]));
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j][c] = win[j + 1][c];
        if (W > 1) win[B - 1][c] = v[c];
      }
      if (full || k + i < live) put<C, VEC>(y, p, nc);
      y += a.py.step;
    }
  }
  const pair zero[P] = {};
  y = (T*)a.y + (int64_t)b * a.py.row + c0;
  for (int k = live; k < k1; ++k) put<C, VEC>(y + (int64_t)k * a.py.step, zero, nc);
}

// dext_e = sum_j w[j] dp_{e - j} (+ ds_out where e >= n) over positions e = k + W - 1 of state and inputs together: the walk over k
// emits position k, the input of step k - W + 1 (or the state's, for k < W - 1 in a row's first run).
template <class T, int C, int W, bool VEC>
__global__ void __launch_bounds__(COLS* ROWS, bwd_blocks(sizeof(T), W)) conv_bwd(const ConvArgs a) {
  constexpr int P = C / 2, B = W > 1 ? W - 1 : 1;
  __shared__ float red[ROWS][COLS * C];
  const int group = blockIdx.y * COLS + threadIdx.x;
  const int64_t item = (int64_t)blockIdx.x * ROWS + threadIdx.y;
  pair dw[W + 1][P];             // the last one: bias
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int c = 0; c < P; ++c) dw[j][c] = 0;

  if (group < a.groups && item < (int64_t)a.batch * a.runs) {
    const int b = (int)(item % a.batch), r = (int)(item / a.batch);
    const int c0 = group * C, nc = min(C, a.channels - c0);
    const int n = row_steps(a.lengths, b, a.t);
    const int k0 = r * a.run, k1 = min(k0 + a.run, a.t);
    const T* const x = (const T*)a.x + (int64_t)b * a.px.row + c0;
    T* dx = (T*)a.dx + (int64_t)b * a.px.row + c0 + (int64_t)(k0 - (W - 1)) * a.px.step;     // of position k0
    pair w[W][P], bias[P], win[B][P], dp[W][P];    // dp[j]: that of step k - j
    load_taps<C, W, T>(a, c0, nc, w, bias);
    load_before<C, W, VEC>(a, x, b, k0, n, c0, nc, win);
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int c = 0; c < P; ++c) dp[j][c] = 0;

    const int end = k1 + W - 1, live = min(end, n); // steps k1 .. end - 1 are the next run's: only their dp is needed
    const int own = min(k1, n);                     // a step that the row does not have adds nothing, whatever lies before it
    const T* next_x = x + (int64_t)k0 * a.px.step;
    const T* next_dy = (const T*)a.dy + (int64_t)b * a.py.row + c0 + (int64_t)k0 * a.py.step;
    Raw<T, C> raw[U], rdy[U], next[U], ndy[U];
    auto load = [&](int k) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool in = k + i < live;
        next[i] = in ? get<C, VEC>(next_x, nc) : raw_zeros<T, C>();
        ndy[i] = in ? get<C, VEC>(next_dy, nc) : raw_zeros<T, C>();
        next_x += a.px.step;
        next_dy += a.py.step;
      }
    };
    load(k0);
    for (int k = k0; k < end; k += U) {
#pragma unroll
      for (int i = 0; i < U; ++i) { raw[i] = next[i]; rdy[i] = ndy[i]; }
      load(k + U);
      // inside: the steps are the row's and this run's own, and the inputs that they emit are too
      auto steps = [&](auto inside) {
        constexpr bool IN = decltype(inside)::value;
#pragma unroll
        for (int i = 0; i < U; ++i) {
          const int kk = k + i;
          pair v[P], g[P], out[P];
          unpack_pairs<C>(raw[i], v);
          unpack_pairs<C>(rdy[i], g);
#pragma unroll
          for (int c = 0; c < P; ++c) {
            if (a.silu) {
              pair p = fma2(w[W - 1][c], v[c], bias[c]);
#pragma unroll
              for (int j = 0; j < W - 1; ++j) p = fma2(w[j][c], win[j][c], p);
              // silu' = s (1 + p (1 - s))
              const pair s = sigmoid2(p), rest = fma2(s, both(-1.f), both(1.f));
              g[c] = mul2(g[c], mul2(s, fma2(p, rest, both(1.f))));
            }
            if (!IN && kk >= live) g[c] = 0;
            if (IN || kk < own) {
              dw[W][c] = add2(dw[W][c], g[c]);
              dw[W - 1][c] = fma2(g[c], v[c], dw[W - 1][c]);
#pragma unroll
              for (int j = 0; j < W - 1; ++j) dw[j][c] = fma2(g[c], win[j][c], dw[j][c]);
            }
#pragma unroll
            for (int j = W - 1; j > 0; --j) dp[j][c] = dp[j - 1][c];
            dp[0][c] = g[c];
            out[c] = mul2(w[0][c], dp[0][c]);
#pragma unroll
            for (int j = 1; j < W; ++j) out[c] = fma2(w[j][c], dp[j][c], out[c]);
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) win[j][c] = win[j + 1][c];
            if (W > 1) win[B - 1][c] = v[c];
          }
          if constexpr (IN) {
            put<C, VEC>(dx, out, nc);
          } else if (kk < end) {
            const int at = kk - (W - 1);             // the input that position kk belongs to; negative: the state's
            if (W > 1 && a.ds_out && kk >= n && kk - n < W - 1) {
              pair d[P];
              unpack_pairs<C>(get<C, VEC>((const T*)a.ds_out + ((int64_t)b * (W - 1) + (kk - n)) * a.channels + c0, nc), d);
#pragma unroll
              for (int c = 0; c < P; ++c) out[c] = add2(out[c], d[c]);
            }
            if (at >= k0) {
              if (at >= n)
#pragma unroll
                for (int c = 0; c < P; ++c) out[c] = 0;
              put<C, VEC>(dx, out, nc);
            } else if (W > 1 && at < 0 && a.ds_in) {
              put<C, VEC>((T*)a.ds_in + ((int64_t)b * (W - 1) + kk) * a.channels + c0, out, nc);
            }
          }
          dx += a.px.step;
        }
      };
      if (k >= k0 + W - 1 && k + U <= min(k1, live)) steps(std::true_type{});
      else steps(std::false_type{});
    }
  }
  // sums over the block's runs, one parameter after the other
  const int tid = threadIdx.y * COLS + threadIdx.x;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < P; ++c) *reinterpret_cast<float2*>(&red[threadIdx.y][threadIdx.x * C + 2 * c]) = unpack2(dw[j][c]);
    __syncthreads();
    for (int i = tid; i < COLS * C; i += COLS * ROWS) {
      const int d = blockIdx.y * COLS * C + i;
      if (d >= a.channels) continue;
      float s = 0.f;
#pragma unroll
      for (int q = 0; q < ROWS; ++q) s += red[q][i];
      a.part[((int64_t)blockIdx.x * (W + 1) + j) * a.channels + d] = s;
    }
  }
}

// part [parts][width + 1][D] -> dw [D][width], dbias [D]; 8 threads share a column's sum.
__global__ void __launch_bounds__(256) conv_sums(const float* part, int parts, int width, int D, float* dw, float* dbias) {
  sm100::grid_dep_wait();
  __shared__ float red[8][32];
  const int64_t i = (int64_t)blockIdx.x * 32 + threadIdx.x, n = (int64_t)(width + 1) * D;
  float s = 0.f;
  if (i < n) {
#pragma unroll 8
    for (int q = threadIdx.y; q < parts; q += 8) s += part[q * n + i];
  }
  red[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || i >= n) return;
  for (int q = 1; q < 8; ++q) s += red[q][threadIdx.x];
  const int j = (int)(i / D), d = (int)(i % D);
  if (j < width) dw[(int64_t)d * width + j] = s;
  else if (dbias) dbias[d] = s;
}

struct ConvPlan {
  int C, groups, run, runs;
  int64_t items;
  unsigned blocks, cols;   // of runs, of channels
};

// Steps of a run: as many as leave every SM a thousand threads, 8 at least (a run begins with width - 1 inputs that its
// neighbour also loads) and 32 at most, backward 64 (blocks of several waves even the SMs out).
bool conv_plan(const mebptt_conv_desc* d, bool back, ConvPlan& p) {
  const int C = p.C = back ? bwd_channels((int)elem_size(d->dtype), d->width) : FWD;
  p.groups = (d->channels + C - 1) / C;
  const int64_t threads = (int64_t)148 * 1024;
  int64_t run = (int64_t)p.groups * d->batch * d->t / threads;
  const int64_t most = back ? 64 : 32;
  run = run < 8 ? 8 : run > most ? most : run / 4 * 4;
  p.runs = (int)((d->t + run - 1) / run);
  p.run = (int)run;
  p.items = (int64_t)d->batch * p.runs;
  const int64_t blocks = (p.items + ROWS - 1) / ROWS;
  const int64_t cols = (p.groups + COLS - 1) / COLS;
  p.blocks = (unsigned)blocks;
  p.cols = (unsigned)cols;
  return cols <= 65535 && blocks < ((int64_t)1 << 31);
}

bool conv_check(const mebptt_conv_desc* d, Places& px, Places& py) {
  if (!d || d->batch < 1 || d->channels < 1 || d->width < 1 || d->width > 8 || d->t < 1 || d->t > (1 << 30)) return false;
  if (d->batch > (1 << 24) || d->channels > (1 << 24) || !valid_dtype(d->dtype) || (d->flags & ~MEBPTT_CONV_SILU) || d->reserved) return false;
  return places(d->x_step, d->x_row, d->t, d->batch, d->channels, px) && places(d->y_step, d->y_row, d->t, d->batch, d->channels, py);
}

template <class T, int W>
void conv_launch(bool back, bool vec, const ConvPlan& p, const ConvArgs& a, cudaStream_t s) {
  const dim3 grid(p.blocks, p.cols), block(COLS, ROWS);
  (void)counted(s);
  constexpr int CB = bwd_channels(sizeof(T), W);
  if (back) vec ? conv_bwd<T, CB, W, true><<<grid, block, 0, s>>>(a) : conv_bwd<T, CB, W, false><<<grid, block, 0, s>>>(a);
  else vec ? conv_fwd<T, FWD, W, true><<<grid, block, 0, s>>>(a) : conv_fwd<T, FWD, W, false><<<grid, block, 0, s>>>(a);
}
template <class T>
void conv_launch(int width, bool back, bool vec, const ConvPlan& p, const ConvArgs& a, cudaStream_t s) {
  switch (width) {
    case 1: return conv_launch<T, 1>(back, vec, p, a, s);
    case 2: return conv_launch<T, 2>(back, vec, p, a, s);
    case 3: return conv_launch<T, 3>(back, vec, p, a, s);
    case 4: return conv_launch<T, 4>(back, vec, p, a, s);
    case 5: return conv_launch<T, 5>(back, vec, p, a, s);
    case 6: return conv_launch<T, 6>(back, vec, p, a, s);
    case 7: return conv_launch<T, 7>(back, vec, p, a, s);
    default: return conv_launch<T, 8>(back, vec, p, a, s);
  }
}

int conv_run(const mebptt_conv_desc* d, const ConvPlan& p, const Places& px, const Places& py, ConvArgs& a, bool back, cudaStream_t s) {
  const size_t e = elem_size(d->dtype);
  const void* const typed[] = {a.x, a.w, a.s_in, a.dy, a.ds_out, a.y, a.s_out, a.dx, a.ds_in};
  for (const void* q : typed)
    if (!natural(q, e)) return MEBPTT_ERR_ARG;
  if (!natural(a.bias, 4) || !natural(a.lengths, 4)) return MEBPTT_ERR_ARG;
  const Places state{0, (int64_t)d->channels};
  a.px = px; a.py = py;
  a.batch = d->batch; a.channels = d->channels; a.t = (int)d->t; a.run = p.run; a.runs = p.runs; a.groups = p.groups;
  a.silu = d->flags & MEBPTT_CONV_SILU;
  if (d->width == 1) { a.s_in = a.ds_out = nullptr; a.s_out = a.ds_in = nullptr; }
  // whole groups of channels, on their own size's boundaries: loaded and stored as one
  const void* const xs[] = {a.x, a.dx};
  const void* const ys[] = {a.y, a.dy};
  const void* const ss[] = {a.s_in, a.s_out, a.ds_in, a.ds_out};
  bool vec = d->channels % p.C == 0;
  for (const void* q : xs) vec = vec && aligned(q, px, p.C, e);
  for (const void* q : ys) vec = vec && aligned(q, py, p.C, e);
  for (const void* q : ss) vec = vec && aligned(q, state, p.C, e);
  if (d->dtype == MEBPTT_BF16) conv_launch<bf16>(d->width, back, vec, p, a, s);
  else conv_launch<float>(d->width, back, vec, p, a, s);
  return cudaGetLastError() == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

}  // namespace
}  // namespace seq
}  // namespace mebptt

using namespace mebptt;
using namespace mebptt::seq;

extern "C" {

int mebptt_conv_forward(const mebptt_conv_desc* desc, const void* x, const void* w, const float* bias, const void* s_in,
                        const int32_t* lengths, void* stream, void* y, void* s_out) {
  Places px, py;
  ConvPlan p;
  if (!conv_check(desc, px, py) || !x || !w || !y) return MEBPTT_ERR_ARG;
  if (!conv_plan(desc, false, p)) return MEBPTT_ERR_UNSUPPORTED;
  ConvArgs a = {};
  a.x = x; a.w = w; a.bias = bias; a.s_in = s_in; a.lengths = lengths; a.y = y; a.s_out = s_out;
  return conv_run(desc, p, px, py, a, false, (cudaStream_t)stream);
}

size_t mebptt_conv_workspace_bytes(const mebptt_conv_desc* desc) {
  Places px, py;
  ConvPlan p;
  if (!conv_check(desc, px, py) || !conv_plan(desc, true, p)) return 0;
  return (size_t)p.blocks * (desc->width + 1) * desc->channels * sizeof(float);
}

int mebptt_conv_backward(const mebptt_conv_desc* desc, const void* x, const void* w, const float* bias, const void* s_in,
                         const int32_t* lengths, const void* dy, const void* ds_out, void* workspace, size_t workspace_bytes,
                         void* stream, void* dx, float* dw, float* dbias, void* ds_in) {
  Places px, py;
  ConvPlan p;
  if (!conv_check(desc, px, py) || !x || !w || !dy || !dx || !dw || !natural(dw, 4) || !natural(dbias, 4)) return MEBPTT_ERR_ARG;
  if (!conv_plan(desc, true, p)) return MEBPTT_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < mebptt_conv_workspace_bytes(desc))
    return MEBPTT_ERR_WORKSPACE;
  ConvArgs a = {};
  a.x = x; a.w = w; a.bias = bias; a.s_in = s_in; a.lengths = lengths; a.dy = dy; a.ds_out = ds_out;
  a.dx = dx; a.ds_in = ds_in; a.part = (float*)workspace;
  const int st = conv_run(desc, p, px, py, a, true, (cudaStream_t)stream);
  if (st != MEBPTT_OK) return st;
  const int64_t n = (int64_t)(desc->width + 1) * desc->channels;
  const cudaError_t e = launch_pdl(conv_sums, dim3((unsigned)((n + 31) / 32)), dim3(32, 8), 0, (cudaStream_t)stream, a.part, (int)p.blocks, desc->width,
                                   desc->channels, dw, dbias);
  return e == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

}  // extern "C"
