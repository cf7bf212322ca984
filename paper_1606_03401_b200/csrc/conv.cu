// Short causal convolution, channel by channel, with a state for token-by-token use; forward and backward.
//
// A thread has `C` neighbouring channels of one row and walks a run of time steps with the last
// width - 1 inputs in registers, so that every input is loaded once (and width - 1 of them a second time where a run begins).
// Loads of U steps are issued together, while the U steps before them are computed.  Bound by memory: 2 accesses an element forward, 3 backward.
#include <cuda_runtime.h>

#include <cstdint>

#include "launch.hpp"
#include "mebptt.h"
#include "seq.hpp"
#include "seq_dev.cuh"

namespace mebptt {
namespace seq {

namespace {

constexpr int C = 4;          // channels of a thread: taps, inputs, and backward also gradients and sums, are held for each
constexpr int U = 4;          // steps whose loads are issued together
constexpr int ROWS = 8;       // runs of a block that share their channels
constexpr int COLS = 32;      // groups of channels of a block

struct ConvArgs {
  const void* x; const void* w; const float* bias; const void* s_in; const int32_t* lengths;
  const void* dy; const void* ds_out;
  void* y; void* s_out;                  // forward
  void* dx; void* ds_in; float* part;    // backward
  Places px, py;
  int batch, channels, t, run, runs;     // steps of a run, runs of a row
  int groups;                            // of C channels
  int aligned_x, aligned_y, aligned_s;   // groups that are whole can be loaded as one
  int silu;
};

// The state of row b as float [W - 1][C]; zeros without one.
template <int W, class T>
__device__ __forceinline__ void load_state(const T* s, int b, int D, int c0, int n, bool whole, float (&f)[W > 1 ? W - 1 : 1][C]) {
#pragma unroll
  for (int i = 0; i < W - 1; ++i) {
    if (s) {
      unpack<C>(load_raw<C>(s + ((int64_t)b * (W - 1) + i) * D + c0, n, whole), f[i]);
    } else {
#pragma unroll
      for (int c = 0; c < C; ++c) f[i][c] = 0.f;
    }
  }
}

// What precedes step k0 of a row: inputs, or the state before step 0 (k0 = 0 or k0 >= W - 1).  Steps at or past n are zeros.
template <int W, class T>
__device__ __forceinline__ void load_before(const ConvArgs& a, const T* x, int b, int k0, int n, int c0, int nc, float (&f)[W > 1 ? W - 1 : 1][C]) {
  if (k0 == 0) {
    load_state<W, T>((const T*)a.s_in, b, a.channels, c0, nc, nc == C && a.aligned_s, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < W - 1; ++i) {
    const int k = k0 - (W - 1) + i;
    unpack<C>(k < n ? load_raw<C>(x + (int64_t)k * a.px.step, nc, nc == C && a.aligned_x) : raw_zeros<T, C>(), f[i]);
  }
}

template <class T, int W>
__global__ void __launch_bounds__(COLS* ROWS) conv_fwd(const ConvArgs a) {
  const int group = blockIdx.y * COLS + threadIdx.x;
  const int64_t item = (int64_t)blockIdx.x * ROWS + threadIdx.y;    // run of a row: rows of one run are neighbours
  if (group >= a.groups || item >= (int64_t)a.batch * a.runs) return;
  const int b = (int)(item % a.batch), r = (int)(item / a.batch);
  const int c0 = group * C, nc = min(C, a.channels - c0);
  const int n = row_steps(a.lengths, b, a.t);
  const int k0 = r * a.run, k1 = min(k0 + a.run, a.t);
  const T* x = (const T*)a.x + (int64_t)b * a.px.row + c0;
  T* y = (T*)a.y + (int64_t)b * a.py.row + c0;
  const bool wx = nc == C && a.aligned_x, wy = nc == C && a.aligned_y;

  float win[W > 1 ? W - 1 : 1][C];
  load_before<W, T>(a, x, b, k0, n, c0, nc, win);
  if (W > 1 && r == 0 && a.s_out) {
    // the last W - 1 of state and inputs; this thread alone reads and writes this part of the state
    T* so = (T*)a.s_out + (int64_t)b * (W - 1) * a.channels + c0;
    const bool ws = nc == C && a.aligned_s;
    float out[W > 1 ? W - 1 : 1][C];
#pragma unroll
    for (int i = 0; i < W - 1; ++i) {
      const int k = n - (W - 1) + i;
      if (k >= 0) {
        unpack<C>(load_raw<C>(x + (int64_t)k * a.px.step, nc, wx), out[i]);
      } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
          if (j == n + i) {
#pragma unroll
            for (int c = 0; c < C; ++c) out[i][c] = win[j][c];
          }
      }
    }
#pragma unroll
    for (int i = 0; i < W - 1; ++i) store_n<C>(so + (int64_t)i * a.channels, out[i], nc, ws);
  }

  float w[W][C], bias[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    bias[c] = a.bias && c < nc ? a.bias[c0 + c] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][c] = c < nc ? to_f<T>(((const T*)a.w)[(int64_t)(c0 + c) * W + j]) : 0.f;
  }
  Raw<T, C> raw[U], next[U];
  auto load = [&](Raw<T, C>(&to)[U], int k) {
#pragma unroll
    for (int i = 0; i < U; ++i) to[i] = k + i < n && k + i < k1 ? load_raw<C>(x + (int64_t)(k + i) * a.px.step, nc, wx) : raw_zeros<T, C>();
  };
  load(next, k0);
  for (int k = k0; k < k1; k += U) {
#pragma unroll
    for (int i = 0; i < U; ++i) raw[i] = next[i];
    load(next, k + U);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float v[C], p[C];
      unpack<C>(raw[i], v);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        p[c] = fmaf(w[W - 1][c], v[c], bias[c]);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) p[c] = fmaf(w[j][c], win[j][c], p[c]);
        if (a.silu) p[c] *= sigmoid(p[c]);
        if (k + i >= n) p[c] = 0.f;
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j][c] = win[j + 1][c];
        if (W > 1) win[W - 2 < 0 ? 0 : W - 2][c] = v[c];
      }
      if (k + i < k1) store_n<C>(y + (int64_t)(k + i) * a.py.step, p, nc, wy);
    }
  }
}

// dext_e = sum_j w[j] dp_{e - j} (+ ds_out where e >= n) over positions e = k + W - 1 of state and inputs together: the walk over k
// emits position k, the input of step k - W + 1 (or the state's, for k < W - 1 in a row's first run).
template <class T, int W>
__global__ void __launch_bounds__(COLS* ROWS) conv_bwd(const ConvArgs a) {
  __shared__ float red[ROWS][COLS * C];
  const int group = blockIdx.y * COLS + threadIdx.x;
  const int64_t item = (int64_t)blockIdx.x * ROWS + threadIdx.y;
  float dw[W + 1][C];            // the last one: bias
#pragma unroll
  for (int j = 0; j <= W; ++j)
#pragma unroll
    for (int c = 0; c < C; ++c) dw[j][c] = 0.f;

  if (group < a.groups && item < (int64_t)a.batch * a.runs) {
    const int b = (int)(item % a.batch), r = (int)(item / a.batch);
    const int c0 = group * C, nc = min(C, a.channels - c0);
    const int n = row_steps(a.lengths, b, a.t);
    const int k0 = r * a.run, k1 = min(k0 + a.run, a.t);
    const T* x = (const T*)a.x + (int64_t)b * a.px.row + c0;
    const T* dy = (const T*)a.dy + (int64_t)b * a.py.row + c0;
    T* dx = (T*)a.dx + (int64_t)b * a.px.row + c0;
    const bool wx = nc == C && a.aligned_x, wy = nc == C && a.aligned_y, ws = nc == C && a.aligned_s;
    float w[W][C], bias[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
      bias[c] = a.bias && c < nc ? a.bias[c0 + c] : 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][c] = c < nc ? to_f<T>(((const T*)a.w)[(int64_t)(c0 + c) * W + j]) : 0.f;
    }
    float win[W > 1 ? W - 1 : 1][C], dp[W][C];     // dp[j]: that of step k - j
    load_before<W, T>(a, x, b, k0, n, c0, nc, win);
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int c = 0; c < C; ++c) dp[j][c] = 0.f;

    const int end = k1 + W - 1;                    // steps k1 .. end - 1 are the next run's: only their dp is needed
    Raw<T, C> raw[U], rdy[U], next[U], ndy[U];
    auto load = [&](int k) {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool in = k + i < n && k + i < end;
        next[i] = in ? load_raw<C>(x + (int64_t)(k + i) * a.px.step, nc, wx) : raw_zeros<T, C>();
        ndy[i] = in ? load_raw<C>(dy + (int64_t)(k + i) * a.py.step, nc, wy) : raw_zeros<T, C>();
      }
    };
    load(k0);
    for (int k = k0; k < end; k += U) {
#pragma unroll
      for (int i = 0; i < U; ++i) { raw[i] = next[i]; rdy[i] = ndy[i]; }
      load(k + U);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int kk = k + i;
        float v[C], g[C], out[C];
        unpack<C>(raw[i], v);
        unpack<C>(rdy[i], g);
#pragma unroll
        for (int c = 0; c < C; ++c) {
          if (a.silu) {
            float p = fmaf(w[W - 1][c], v[c], bias[c]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p = fmaf(w[j][c], win[j][c], p);
            g[c] *= dsilu(p, sigmoid(p));
          }
          if (kk >= n || kk >= end) g[c] = 0.f;
          if (kk < k1) {
            dw[W][c] += g[c];
            dw[W - 1][c] = fmaf(g[c], v[c], dw[W - 1][c]);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) dw[j][c] = fmaf(g[c], win[j][c], dw[j][c]);
          }
#pragma unroll
          for (int j = W - 1; j > 0; --j) dp[j][c] = dp[j - 1][c];
          dp[0][c] = g[c];
          out[c] = w[0][c] * dp[0][c];
#pragma unroll
          for (int j = 1; j < W; ++j) out[c] = fmaf(w[j][c], dp[j][c], out[c]);
#pragma unroll
          for (int j = 0; j + 1 < W - 1; ++j) win[j][c] = win[j + 1][c];
          if (W > 1) win[W - 2 < 0 ? 0 : W - 2][c] = v[c];
        }
        if (kk >= end) continue;
        const int i_out = kk - (W - 1);            // the input that position kk belongs to; negative: the state's
        if (i_out < k0 && !(r == 0 && a.ds_in)) continue;
        if (W > 1 && a.ds_out && kk >= n && kk - n < W - 1) {
          float d[C];
          unpack<C>(load_raw<C>((const T*)a.ds_out + ((int64_t)b * (W - 1) + (kk - n)) * a.channels + c0, nc, ws), d);
#pragma unroll
          for (int c = 0; c < C; ++c) out[c] += d[c];
        }
        if (i_out >= 0) {
#pragma unroll
          for (int c = 0; c < C; ++c)
            if (i_out >= n) out[c] = 0.f;
          store_n<C>(dx + (int64_t)i_out * a.px.step, out, nc, wx);
        } else {
          store_n<C>((T*)a.ds_in + ((int64_t)b * (W - 1) + kk) * a.channels + c0, out, nc, ws);
        }
      }
    }
  }
  // sums over the block's runs, one parameter after the other
  const int tid = threadIdx.y * COLS + threadIdx.x;
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    __syncthreads();
#pragma unroll
    for (int c = 0; c < C; ++c) red[threadIdx.y][threadIdx.x * C + c] = dw[j][c];
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
  __shared__ float red[8][32];
  const int64_t i = (int64_t)blockIdx.x * 32 + threadIdx.x, n = (int64_t)(width + 1) * D;
  float s = 0.f;
  if (i < n)
    for (int q = threadIdx.y; q < parts; q += 8) s += part[q * n + i];
  red[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y != 0 || i >= n) return;
  for (int q = 1; q < 8; ++q) s += red[q][threadIdx.x];
  const int j = (int)(i / D), d = (int)(i % D);
  if (j < width) dw[(int64_t)d * width + j] = s;
  else if (dbias) dbias[d] = s;
}

struct ConvPlan {
  int groups, run, runs;
  int64_t items;
  unsigned blocks, cols;   // of runs, of channels
};

// Steps of a run: as many as leave every SM a thousand threads, 8 at least (a run begins with width - 1 inputs that its
// neighbour also loads) and 32 at most (blocks of several waves even the SMs out).
bool conv_plan(const mebptt_conv_desc* d, ConvPlan& p) {
  p.groups = (d->channels + C - 1) / C;
  const int64_t threads = (int64_t)148 * 1024;
  int64_t run = (int64_t)p.groups * d->batch * d->t / threads;
  run = run < 8 ? 8 : run > 32 ? 32 : run / 4 * 4;
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
void conv_launch(bool back, const ConvPlan& p, const ConvArgs& a, cudaStream_t s) {
  const dim3 grid(p.blocks, p.cols), block(COLS, ROWS);
  if (back) conv_bwd<T, W><<<grid, block, 0, counted(s)>>>(a);
  else conv_fwd<T, W><<<grid, block, 0, counted(s)>>>(a);
}
template <class T>
void conv_launch(int width, bool back, const ConvPlan& p, const ConvArgs& a, cudaStream_t s) {
  switch (width) {
    case 1: return conv_launch<T, 1>(back, p, a, s);
    case 2: return conv_launch<T, 2>(back, p, a, s);
    case 3: return conv_launch<T, 3>(back, p, a, s);
    case 4: return conv_launch<T, 4>(back, p, a, s);
    case 5: return conv_launch<T, 5>(back, p, a, s);
    case 6: return conv_launch<T, 6>(back, p, a, s);
    case 7: return conv_launch<T, 7>(back, p, a, s);
    default: return conv_launch<T, 8>(back, p, a, s);
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
  a.aligned_x = aligned(a.x, px, C, e) && aligned(a.dx, px, C, e);
  a.aligned_y = aligned(back ? a.dy : a.y, py, C, e);
  a.aligned_s = aligned(a.s_in, state, C, e) && aligned(a.s_out, state, C, e) && aligned(a.ds_in, state, C, e) && aligned(a.ds_out, state, C, e);
  if (d->dtype == MEBPTT_BF16) conv_launch<bf16>(d->width, back, p, a, s);
  else conv_launch<float>(d->width, back, p, a, s);
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
  if (!conv_plan(desc, p)) return MEBPTT_ERR_UNSUPPORTED;
  ConvArgs a = {};
  a.x = x; a.w = w; a.bias = bias; a.s_in = s_in; a.lengths = lengths; a.y = y; a.s_out = s_out;
  return conv_run(desc, p, px, py, a, false, (cudaStream_t)stream);
}

size_t mebptt_conv_workspace_bytes(const mebptt_conv_desc* desc) {
  Places px, py;
  ConvPlan p;
  if (!conv_check(desc, px, py) || !conv_plan(desc, p)) return 0;
  return (size_t)p.blocks * (desc->width + 1) * desc->channels * sizeof(float);
}

int mebptt_conv_backward(const mebptt_conv_desc* desc, const void* x, const void* w, const float* bias, const void* s_in,
                         const int32_t* lengths, const void* dy, const void* ds_out, void* workspace, size_t workspace_bytes,
                         void* stream, void* dx, float* dw, float* dbias, void* ds_in) {
  Places px, py;
  ConvPlan p;
  if (!conv_check(desc, px, py) || !x || !w || !dy || !dx || !dw || !natural(dw, 4) || !natural(dbias, 4)) return MEBPTT_ERR_ARG;
  if (!conv_plan(desc, p)) return MEBPTT_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < mebptt_conv_workspace_bytes(desc))
    return MEBPTT_ERR_WORKSPACE;
  ConvArgs a = {};
  a.x = x; a.w = w; a.bias = bias; a.s_in = s_in; a.lengths = lengths; a.dy = dy; a.ds_out = ds_out;
  a.dx = dx; a.ds_in = ds_in; a.part = (float*)workspace;
  const int st = conv_run(desc, p, px, py, a, true, (cudaStream_t)stream);
  if (st != MEBPTT_OK) return st;
  const int64_t n = (int64_t)(desc->width + 1) * desc->channels;
  conv_sums<<<(unsigned)((n + 31) / 32), dim3(32, 8), 0, counted((cudaStream_t)stream)>>>(a.part, (int)p.blocks, desc->width, desc->channels, dw, dbias);
  return cudaGetLastError() == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

}  // extern "C"
