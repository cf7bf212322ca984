// Distillation from a teacher's top logits: entry points, and the kernel for what the rings (distill_ring.cu) do not take -- gradients that
// lie otherwise within 16 bytes than the logits, and rows longer than a cluster's shared memory.
//
// A row is held in the registers of a block of 32 to 512 threads, or of a cluster of up to eight blocks (up to 131072 logits): each
// thread loads all its 16-byte pieces at once, takes their maximum m, turns them into exp((x - m) / T), and what remains once
// the row's maximum and sum are known is one factor a thread.  Longer rows are read a second time for the gradient.  Clusters are
// also taken where there are few rows, to spread them over the SMs.  Bound by the latency of that chain (760 us where the
// ring takes 102: 4096 rows of 32000 bfloat16 logits).
//
// The gradient is first written as that of the student's distribution alone; then, behind a barrier, the elements that the teacher
// lists are written over, each by the thread of its first entry, which adds up the entries that name the same token, in their
// order.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include <cfloat>
#include <cstdint>

#include "distill.hpp"
#include "launch.hpp"
#include "mebptt.h"
#include "seq.hpp"
#include "seq_dev.cuh"
#include "sm100.cuh"

namespace cg = cooperative_groups;

namespace mebptt {
namespace seq {

namespace {

constexpr int PER_THREAD = 32;          // logits of a thread
constexpr int MAX_THREADS = 512, MAX_CLUSTER = 8, MAX_ENTRIES = 1024;

// Reductions over the block; `red` holds 32 floats for each of the values.
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int m = 16; m > 0; m /= 2) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, m));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
template <bool SUM>
__device__ __forceinline__ float2 block_reduce(float x, float y, float2* red) {
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
  x = SUM ? warp_sum(x) : warp_max(x);
  y = SUM ? warp_sum(y) : warp_max(y);
  if (warps == 1) return make_float2(x, y);
  __syncthreads();                      // the last reduction's values have been read
  if (lane == 0) red[warp] = make_float2(x, y);
  __syncthreads();
  const float2 v = lane < warps ? red[lane] : SUM ? make_float2(0.f, 0.f) : make_float2(-INFINITY, -INFINITY);
  return make_float2(SUM ? warp_sum(v.x) : warp_max(v.x), SUM ? warp_sum(v.y) : warp_max(v.y));
}

// exp((x - m) / T): a difference first, so that neither a large common value nor the type's lowest one loses or overflows anything.
__device__ __forceinline__ float exp_over(float x, float m, float k) { return ex2((x - m) * k); }

// WHOLE: a row fits the registers of its blocks.
template <class T, bool WHOLE, bool CLUSTER>
__global__ void __launch_bounds__(MAX_THREADS) distill_kernel(const DistillArgs a) {
  constexpr int VE = 16 / (int)sizeof(T), PIECES = PER_THREAD / VE;
  extern __shared__ __align__(16) float sm[];
  __shared__ float2 red[32], mine;
  int32_t* const s_idx = reinterpret_cast<int32_t*>(sm);     // [entries]: token, or -1
  float* const s_q = sm + a.entries;                         // value, then exp((value - largest) / T)
  float* const s_z = s_q + a.entries;                        // the student's logit there

  const int tid = threadIdx.x, NT = blockDim.x;
  unsigned rank = 0, blocks = 1;
  int64_t r = blockIdx.x;
  if constexpr (CLUSTER) {
    rank = cg::this_cluster().block_rank();
    blocks = cg::this_cluster().num_blocks();
    r = blockIdx.x / blocks;
  }
  const int V = a.vocabulary;
  const T* const x = (const T*)a.logits + r * a.row;
  T* const dx = (T*)a.dlogits + r * a.drow;
  // pieces of VE elements on 16-byte boundaries; the row begins at element `phase` of the first one
  const int phase = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % VE);
  const int pieces = (phase + V + VE - 1) / VE, share = (pieces + (int)blocks - 1) / (int)blocks;
  const int p0 = (int)rank * share, p1 = min(p0 + share, pieces);
  const float weight = a.weights ? a.weights[r] : 1.f;
  const float k = kLog2e / a.T;

  auto load_piece = [&](int p, float (&f)[VE]) {
    const int i = p * VE - phase;
    if (i >= 0 && i + VE <= V) {
      unpack<VE>(load_raw<VE>(x + i, VE, true), f);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) f[j] = i + j >= 0 && i + j < V ? to_f<T>(x[i + j]) : -INFINITY;
    }
  };
  auto store_piece = [&](int p, const float (&f)[VE]) {
    const int i = p * VE - phase;
    if (a.same_phase && i >= 0 && i + VE <= V) {
      store_n<VE>(dx + i, f, VE, true);
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j)
        if (i + j >= 0 && i + j < V) dx[i + j] = from_f<T>(f[j]);
    }
  };

  // a row that counts nothing: no branch below depends on more than the block's row, so all of it leaves here
  bool counts = weight != 0.f;
  float e[PIECES][VE], m = -INFINITY;
  if (counts) {
    if (WHOLE) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = p0 + tid + i * NT;
        if (p < p1) {
          load_piece(p, e[i]);
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) e[i][j] = -INFINITY;
        }
      }
    }
    // the teacher's entries
    float top = -INFINITY;
    int any = 0;
    for (int j = tid; j < a.entries; j += NT) {
      const int idx = a.indices[r * a.entries + j];
      const float v = idx >= 0 && idx < V ? a.values[r * a.entries + j] : -INFINITY;
      const bool there = v != -INFINITY;
      s_idx[j] = there ? idx : -1;
      s_q[j] = v;
      s_z[j] = there ? to_f<T>(x[idx]) : 0.f;
      top = fmaxf(top, v);
      any |= there;
    }
    // a thread's largest logit, and the sum over it
    float s = 0.f;
    if (WHOLE) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) m = fmaxf(m, e[i][j]);
      const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          e[i][j] = exp_over(e[i][j], from, k);
          s += e[i][j];
        }
    } else if (!a.stats_in) {
      for (int p = p0 + tid; p < p1; p += NT) {
        float f[VE], top_f = -INFINITY;
        load_piece(p, f);
#pragma unroll
        for (int j = 0; j < VE; ++j) top_f = fmaxf(top_f, f[j]);
        if (top_f > m) {
          s = m == -INFINITY ? s : s * exp_over(m, top_f, k);     // (s is 0, or not a number, before the first finite logit)
          m = top_f;
        }
        const float from = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int j = 0; j < VE; ++j) s += exp_over(f[j], from, k);
      }
    }
    counts = __syncthreads_or(any);
    if (counts) {
      float2 tops = block_reduce<false>(m, top, red);      // largest logit of the block, largest value
      float factor = m == -INFINITY ? 0.f : exp_over(m, tops.x, k);
      float q = 0.f;
      for (int j = tid; j < a.entries; j += NT) {
        const float v = s_q[j];
        s_q[j] = s_idx[j] < 0 ? 0.f : exp_over(v, tops.y, k);
        q += s_q[j];
      }
      float2 sums = block_reduce<true>(s * factor, q, red);
      float M = tops.x, S = sums.x;
      const float Q = sums.y;
      if (a.stats_in) {
        M = a.stats_in[2 * r];
        S = a.stats_in[2 * r + 1];
        factor = m == -INFINITY ? 0.f : exp_over(m, M, k);
      } else if constexpr (CLUSTER) {
        cg::cluster_group cl = cg::this_cluster();
        if (tid == 0) mine = make_float2(M, S);
        cl.sync();
        float top_all = -INFINITY, sum_all = 0.f;
        for (unsigned c = 0; c < blocks; ++c) top_all = fmaxf(top_all, cl.map_shared_rank(&mine, c)->x);
        for (unsigned c = 0; c < blocks; ++c) {
          const float2 o = *cl.map_shared_rank(&mine, c);
          sum_all += o.x == -INFINITY ? o.y : o.y * exp_over(o.x, top_all, k);
        }
        M = top_all;
        S = sum_all;
        factor = m == -INFINITY ? 0.f : exp_over(m, M, k);
      }
      const float rS = 1.f / S, rQ = 1.f / Q;
      if (a.row_loss && rank == 0) {
        // sum_j q_j (log q_j - log p_j)
        const float logS = logf(S) - logf(Q), rT = 1.f / a.T;
        float loss = 0.f;
        for (int j = tid; j < a.entries; j += NT) {
          const float w = s_q[j] * rQ;
          if (s_idx[j] >= 0 && w != 0.f) {
            // log q = (v - largest) / T - log Q; s_q holds the exponential, its value is read again
            const float v = a.values[r * a.entries + j];
            loss += w * (((v - tops.y) - (s_z[j] - M)) * rT + logS);
          }
        }
        loss = block_reduce<true>(loss, 0.f, red).x;
        if (tid == 0) {
          a.row_loss[r] = weight * a.T * a.T * loss;
          if (a.row_stats) {
            a.row_stats[2 * r] = M;
            a.row_stats[2 * r + 1] = S;
          }
        }
      }
      if (a.gradient) {
        const float coef = (a.dloss ? *a.dloss : 1.f) * a.scale * weight * a.T;
        if (WHOLE) {
          const float by = coef * factor * rS;
#pragma unroll
          for (int i = 0; i < PIECES; ++i) {
            const int p = p0 + tid + i * NT;
            if (p < p1) {
#pragma unroll
              for (int j = 0; j < VE; ++j) e[i][j] *= by;
              store_piece(p, e[i]);
            }
          }
        } else {
          for (int p = p0 + tid; p < p1; p += NT) {
            float f[VE];
            load_piece(p, f);
#pragma unroll
            for (int j = 0; j < VE; ++j) f[j] = coef * (exp_over(f[j], M, k) * rS);
            store_piece(p, f);
          }
        }
        __syncthreads();
        // the listed tokens of this block's share
        const int64_t lo = (int64_t)p0 * VE - phase, hi = (int64_t)p1 * VE - phase;
        for (int j = tid; j < a.entries; j += NT) {
          const int idx = s_idx[j];
          if (idx < lo || idx >= hi || idx < 0) continue;
          float q = 0.f;
          bool first = true;
          for (int i = 0; i < a.entries; ++i)
            if (s_idx[i] == idx) {
              if (i < j) { first = false; break; }
              q += s_q[i];
            }
          if (first) dx[idx] = from_f<T>(coef * (exp_over(s_z[j], M, k) * rS - q * rQ));
        }
      }
    }
  }
  if (!counts) {
    if (tid == 0 && rank == 0 && a.row_loss) {
      a.row_loss[r] = 0.f;
      if (a.row_stats) {
        a.row_stats[2 * r] = 0.f;
        a.row_stats[2 * r + 1] = 1.f;
      }
    }
    if (a.gradient) {
      float zero[VE] = {};
      for (int p = p0 + tid; p < p1; p += NT) store_piece(p, zero);
    }
  }
  if constexpr (CLUSTER) cg::this_cluster().sync();        // no block leaves while another reads its sums
}

// loss = scale sum of the rows' losses, one block, in a fixed order and in 64 bits
__global__ void __launch_bounds__(1024) distill_total(const float* row_loss, int64_t rows, float scale, float* loss) {
  sm100::grid_dep_wait();
  __shared__ double red[32];
  double s = 0.;
  for (int64_t i = threadIdx.x; i < rows; i += 1024) s += (double)row_loss[i];
#pragma unroll
  for (int m = 16; m > 0; m /= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = s;
  __syncthreads();
  if (threadIdx.x >= 32) return;
  s = red[threadIdx.x];
#pragma unroll
  for (int m = 16; m > 0; m /= 2) s += __shfl_xor_sync(0xffffffffu, s, m);
  if (threadIdx.x == 0) *loss = (float)(s * (double)scale);
}

template <class T, bool WHOLE>
cudaError_t launch(const DistillArgs& a, int64_t rows, int cluster, int threads, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)a.entries * 12;
  cfg.stream = counted(s);
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  if constexpr (WHOLE)
    if (cluster == 1) return cudaLaunchKernelEx(&cfg, distill_kernel<T, true, false>, a);
  return cudaLaunchKernelEx(&cfg, distill_kernel<T, WHOLE, true>, a);      // (rows that are read twice have passed a cluster of the largest size)
}

int finish(cudaError_t st, const DistillArgs& a, const mebptt_distill_desc* d, float* loss, cudaStream_t s) {
  if (st == cudaSuccess && loss) st = launch_pdl(distill_total, dim3(1), dim3(1024), 0, s, a.row_loss, d->rows, d->scale, loss);
  return st == cudaSuccess ? MEBPTT_OK : MEBPTT_ERR_CUDA;
}

int run(const mebptt_distill_desc* d, DistillArgs& a, float* loss, cudaStream_t s) {
  if (d->rows >= ((int64_t)1 << 31)) return MEBPTT_ERR_UNSUPPORTED;
  const size_t e = d->dtype == MEBPTT_BF16 ? 2 : 4;
  const int VE = (int)(16 / e);
  a.row = d->logits_row ? d->logits_row : d->vocabulary;
  a.drow = d->dlogits_row ? d->dlogits_row : d->vocabulary;
  a.rows = d->rows; a.vocabulary = d->vocabulary; a.entries = d->entries; a.T = d->temperature; a.scale = d->scale;
  a.same_phase = a.gradient && !((reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.dlogits)) & 15) && (d->rows == 1 || !((a.row - a.drow) * (int64_t)e & 15));
  // blocks of a row: so many that its logits fit their registers, and twice as many while a third of the SMs' places is not
  // taken and a block keeps 2048 logits
  cudaError_t st;
  if (distill_ring(a, d->dtype == MEBPTT_BF16, s, st)) return finish(st, a, d, loss, s);
  const int64_t pieces = ((int64_t)VE - 1 + d->vocabulary + VE - 1) / VE;
  const int64_t most = (int64_t)MAX_THREADS * PER_THREAD / VE;
  int cluster = 1;
  while (cluster < MAX_CLUSTER && (pieces > most * cluster || (d->rows * cluster < 296 && d->vocabulary / (2 * cluster) >= 2048))) cluster *= 2;
  const int64_t share = (pieces + cluster - 1) / cluster;
  const bool whole = share <= most;
  int64_t threads = (share + PER_THREAD / VE - 1) / (PER_THREAD / VE);
  threads = threads > MAX_THREADS ? MAX_THREADS : (threads + 31) / 32 * 32;
  if (d->rows * cluster >= ((int64_t)1 << 31)) return MEBPTT_ERR_UNSUPPORTED;
  if (d->dtype == MEBPTT_BF16) st = whole ? launch<bf16, true>(a, d->rows, cluster, (int)threads, s) : launch<bf16, false>(a, d->rows, cluster, (int)threads, s);
  else st = whole ? launch<float, true>(a, d->rows, cluster, (int)threads, s) : launch<float, false>(a, d->rows, cluster, (int)threads, s);
  return finish(st, a, d, loss, s);
}

bool check(const mebptt_distill_desc* d, const void* logits, const int32_t* indices, const float* values, const float* weights) {
  if (!d || d->rows < 1 || d->vocabulary < 1 || d->vocabulary > (1 << 30) || d->entries < 1 || d->entries > MAX_ENTRIES) return false;
  if (!valid_dtype(d->dtype) || d->reserved || !(d->scale - d->scale == 0.f)) return false;
  // the losses carry the square: one that is infinite, or below the type's normal numbers, would make them so too
  const float square = d->temperature * d->temperature;
  if (!(d->temperature > 0.f) || !(square >= FLT_MIN) || square > FLT_MAX) return false;
  const int64_t most = (int64_t)1 << 40;
  if (d->rows > most || d->logits_row > most || d->dlogits_row > most) return false;
  if ((d->logits_row && d->logits_row < d->vocabulary) || (d->dlogits_row && d->dlogits_row < d->vocabulary)) return false;
  return logits && indices && values && natural(logits, elem_size(d->dtype)) && natural(indices, 4) && natural(values, 4) && natural(weights, 4);
}

}  // namespace
}  // namespace seq
}  // namespace mebptt

using namespace mebptt::seq;

extern "C" {

int mebptt_distill_loss(const mebptt_distill_desc* desc, const void* logits, const int32_t* indices, const float* values,
                        const float* weights, void* stream, float* loss, float* row_loss, float* row_stats) {
  if (!check(desc, logits, indices, values, weights) || !row_loss || !row_stats || !natural(loss, 4) || !natural(row_loss, 4) || !natural(row_stats, 4))
    return MEBPTT_ERR_ARG;
  DistillArgs a = {};
  a.logits = logits; a.indices = indices; a.values = values; a.weights = weights; a.row_loss = row_loss; a.row_stats = row_stats;
  return run(desc, a, loss, (cudaStream_t)stream);
}

int mebptt_distill_grad(const mebptt_distill_desc* desc, const void* logits, const int32_t* indices, const float* values,
                        const float* weights, const float* row_stats, const float* dloss, void* stream, void* dlogits) {
  if (!check(desc, logits, indices, values, weights) || !row_stats || !dlogits || !natural(row_stats, 4) || !natural(dloss, 4) ||
      !natural(dlogits, elem_size(desc->dtype)))
    return MEBPTT_ERR_ARG;
  DistillArgs a = {};
  a.logits = logits; a.indices = indices; a.values = values; a.weights = weights; a.stats_in = row_stats; a.dloss = dloss;
  a.dlogits = dlogits; a.gradient = 1;
  return run(desc, a, nullptr, (cudaStream_t)stream);
}

int mebptt_distill_loss_grad(const mebptt_distill_desc* desc, const void* logits, const int32_t* indices, const float* values,
                             const float* weights, const float* dloss, void* stream, float* loss, float* row_loss, void* dlogits) {
  if (!check(desc, logits, indices, values, weights) || !row_loss || !dlogits || !natural(loss, 4) || !natural(row_loss, 4) ||
      !natural(dloss, 4) || !natural(dlogits, elem_size(desc->dtype)))
    return MEBPTT_ERR_ARG;
  DistillArgs a = {};
  a.logits = logits; a.indices = indices; a.values = values; a.weights = weights; a.dloss = dloss; a.row_loss = row_loss;
  a.dlogits = dlogits; a.gradient = 1;
  return run(desc, a, loss, (cudaStream_t)stream);
}

}  // extern "C"
