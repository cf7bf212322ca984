// Distillation loss over wide vocabularies: rows stream through shared memory.
//
// One resident block an SM (a few where rows are short), or a cluster of blocks that share a row, walks its rows through a ring of
// two to four stages: while one row is worked on, the next ones are on their way in and the last one's gradient on its way out, all
// by bulk copies, so that memory is busy all the time although a row's own path is a chain (maximum, sum, gradient).  Each thread
// keeps its logits as exponentials in registers, relative to its own largest one, and what is left once the row's maximum and
// sum are known is one factor a thread: one exponential a logit.  The gradient is written over the logits in the stage, the
// listed tokens are put right there, and the stage is copied out.
//
// A warp of its own moves data and prepares the next row's teacher (softmax of the listed values, tokens listed twice).
//
// Row begins and ends that are not on 16-byte boundaries go by plain loads and stores of that warp.
#include <cuda_runtime.h>

#include <cstdint>

#include "distill.hpp"
#include "launch.hpp"
#include "seq.hpp"
#include "seq_dev.cuh"
#include "sm100.cuh"

namespace mebptt {
namespace seq {

namespace {

using namespace sm100;

constexpr int PIECES = 8;               // 16-byte pieces of a thread: 64 bfloat16 or 32 float32 logits
constexpr int MAX_CONSUMERS = 512, MAX_STAGES = 4;
constexpr int SMEM = 227 * 1024;

__device__ __forceinline__ void bulk_in(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
__device__ __forceinline__ void bulk_out(void* dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
               ::"l"(reinterpret_cast<uint64_t>(dst)), "r"(smem_u32(src)), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void consumers_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
// a pair of floats into another block's shared memory
__device__ __forceinline__ void put_pair(float2* at, unsigned rank, float2 v) {
  uint32_t there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(at)), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(v.x), "f"(v.y) : "memory");
}
__device__ __forceinline__ float exp_over(float x, float m, float k) { return ex2((x - m) * k); }

struct RingArgs {
  DistillArgs a;
  int cluster, stages, consumers, share;          // share: pieces of a block at most
};

// Shared memory behind the stages.
struct Small {
  uint64_t full[MAX_STAGES];
  float2 red[MAX_CONSUMERS / 32];                 // largest logit and sum of a warp
  float2 all[2][8];                               // those of the cluster's blocks, by parity of the row
  float2 part[2][8];                              // their parts of the loss (x)
  float loss[2][MAX_CONSUMERS / 32];              // parts of the loss, by warp
  float weight[MAX_STAGES];
  int any[2];                                     // a row has entries
  int failed;                                     // a wait has run out
};

template <class T, bool CLUSTER>
__global__ void __launch_bounds__(MAX_CONSUMERS + 32, 1) distill_rows(const RingArgs g) {
  constexpr int VE = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) uint8_t sm[];
  const DistillArgs& a = g.a;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, NC = g.consumers, warps = NC / 32, NS = g.stages, K = a.entries, V = a.vocabulary;
  const uint32_t stage_bytes = (uint32_t)g.share * 16;
  Small& o = *reinterpret_cast<Small*>(sm + NS * stage_bytes);
  uint32_t* const seen = reinterpret_cast<uint32_t*>(&o + 1);                  // a bit for each logit of the share
  const int words = (g.share * VE + 31) / 32;
  int32_t* const t_at = reinterpret_cast<int32_t*>(seen + words);              // [2][K]: place in the share; -1: not there, -2: another block's
  float* const t_q = reinterpret_cast<float*>(t_at + 2 * K);                   // [2][K]: q
  float* const t_log = t_q + 2 * K;                                            // [2][K]: log q
  float* const t_sum = t_log + 2 * K;                                          // [2][K]: q of all entries with this token; -1: an earlier one has it
  float* const t_z = t_sum + 2 * K;                                            // [K]: the student's logit

  unsigned rank = 0;
  if constexpr (CLUSTER) asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const unsigned clusters = gridDim.x / g.cluster, mine = blockIdx.x / g.cluster;
  const int64_t rows = (a.rows - mine + clusters - 1) / clusters;              // of this cluster: mine, mine + clusters, ...
  const float k = kLog2e / a.T, rT = 1.f / a.T;

  // Where row r lies: pieces on 16-byte boundaries, the row beginning at element `phase` of the first; this block's are p0 .. p1 - 1.
  struct Row {
    const T* x; T* dx;
    int phase, p0, p1, in0, in1;                  // in0 .. in1 - 1: pieces that are whole
  };
  auto row_at = [&](int64_t it) {
    const int64_t r = (int64_t)mine + it * clusters;
    Row w;
    w.x = (const T*)a.logits + r * a.row;
    w.dx = (T*)a.dlogits + r * a.drow;
    w.phase = (int)(reinterpret_cast<uintptr_t>(w.x) / sizeof(T) % VE);
    const int pieces = (w.phase + V + VE - 1) / VE, share = (pieces + g.cluster - 1) / g.cluster;
    w.p0 = min((int)rank * share, pieces);
    w.p1 = min(w.p0 + share, pieces);
    w.in0 = w.p0 == 0 && w.phase ? min(1, w.p1) : w.p0;
    w.in1 = w.p1 == pieces && (w.phase + V) % VE ? max(w.in0, w.p1 - 1) : w.p1;
    return w;
  };
  auto stage = [&](int64_t it) { return sm + (uint32_t)(it % NS) * stage_bytes; };

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) mbar_init(&o.full[s], 2);
    mbar_fence_init();
    o.failed = 0;
  }
  for (int i = tid; i < words; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  if constexpr (CLUSTER) { cluster_arrive(); cluster_wait(); }                 // no block writes to another before it is there

  if (warp == warps) {
    // ---- the warp that moves data ----
    auto weight_of = [&](int64_t it) { return it < rows && a.weights ? a.weights[(int64_t)mine + it * clusters] : 1.f; };
    auto fetch = [&](int64_t it, float weight) {
      if (it >= rows) return;
      const int s = (int)(it % NS);
      if (lane == 0) o.weight[s] = weight;
      if (weight == 0.f) return;                  // not loaded, and not waited for
      const Row w = row_at(it);
      T* const buf = (T*)stage(it);
      if (lane == 0) {
        const uint32_t bytes = (uint32_t)(w.in1 - w.in0) * 16;
        mbar_arrive_expect_tx(&o.full[s], bytes);
        if (bytes) bulk_in(buf + (w.in0 - w.p0) * VE, w.x + ((int64_t)w.in0 * VE - w.phase), bytes, &o.full[s]);
      }
      // what is not whole: elements before in0 and from in1 on
      const int head = (w.in0 - w.p0) * VE, tail = (w.p1 - w.in1) * VE;
      if (lane < head + tail) {
        const int at = lane < head ? lane : (w.in1 - w.p0) * VE + lane - head, i = w.p0 * VE + at - w.phase;
        buf[at] = i >= 0 && i < V ? w.x[i] : from_f<T>(-INFINITY);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&o.full[s]);
    };
    // softmax of the listed values of row `it`
    auto teach = [&](int64_t it) {
      if (it >= rows) return;
      const int64_t r = (int64_t)mine + it * clusters;
      const Row w = row_at(it);
      const int slot = (int)(it & 1) * K, lo = w.p0 * VE - w.phase, n = (w.p1 - w.p0) * VE;
      float top = -INFINITY;
      bool any = false;
      for (int j = lane; j < K; j += 32) {
        const int idx = a.indices[r * K + j];
        const float v = idx >= 0 && idx < V ? a.values[r * K + j] : -INFINITY;
        const int at = idx - lo;
        t_at[slot + j] = v == -INFINITY ? -1 : at >= 0 && at < n ? at : -2;
        t_log[slot + j] = v;
        any |= v != -INFINITY;
        top = fmaxf(top, v);
      }
      any = __any_sync(0xffffffffu, any);
#pragma unroll
      for (int m = 16; m > 0; m /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, m));
      if (lane == 0) o.any[it & 1] = any;
      if (!any) return;
      float Q = 0.f;
      bool twice = false;
      for (int j = lane; j < K; j += 32) {
        const int at = t_at[slot + j];
        const float q = at == -1 ? 0.f : exp_over(t_log[slot + j], top, k);
        t_q[slot + j] = q;
        Q += q;
        if (at >= 0) twice |= (atomicOr(&seen[at >> 5], 1u << (at & 31)) >> (at & 31)) & 1;
      }
#pragma unroll
      for (int m = 16; m > 0; m /= 2) Q += __shfl_xor_sync(0xffffffffu, Q, m);
      twice = __any_sync(0xffffffffu, twice);
      const float rQ = 1.f / Q, logQ = logf(Q);
      for (int j = lane; j < K; j += 32) {
        const int at = t_at[slot + j];
        const float q = t_q[slot + j] * rQ;
        t_q[slot + j] = t_sum[slot + j] = q;
        t_log[slot + j] = (t_log[slot + j] - top) * rT - logQ;
        if (at >= 0) seen[at >> 5] = 0;
      }
      __syncwarp();
      if (twice)
        for (int j = lane; j < K; j += 32) {
          const int at = t_at[slot + j];
          if (at < 0) continue;
          float q = 0.f;
          for (int i = 0; i < K; ++i)
            if (t_at[slot + i] == at) {
              if (i < j) { q = -1.f; break; }
              q += t_q[slot + i];
            }
          t_sum[slot + j] = q;
        }
    };

    for (int64_t i = 0; i < NS - 1; ++i) fetch(i, weight_of(i));
    teach(0);
    float weight = weight_of(NS - 1);
    for (int64_t it = 0; it <= rows; ++it) {
      __syncthreads();                            // row it - 1 is done with, row it has its teacher
      // the row before: gradient out, loss
      const int64_t was = it - 1;
      if (was >= 0 && a.gradient) {
        const Row w = row_at(was);
        const T* const buf = (const T*)stage(was);
        if (lane == 0) {
          const uint32_t bytes = (uint32_t)(w.in1 - w.in0) * 16;
          if (bytes) bulk_out(w.dx + ((int64_t)w.in0 * VE - w.phase), buf + (w.in0 - w.p0) * VE, bytes);
          asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
        const int head = (w.in0 - w.p0) * VE, tail = (w.p1 - w.in1) * VE;
        if (lane < head + tail) {
          const int at = lane < head ? lane : (w.in1 - w.p0) * VE + lane - head, i = w.p0 * VE + at - w.phase;
          if (i >= 0 && i < V) w.dx[i] = buf[at];
        }
      }
      if (was >= 0 && a.row_loss) {
        float v = lane < warps ? o.loss[was & 1][lane] : 0.f;
#pragma unroll
        for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
        if (o.failed) v = NAN;
        if (lane == 0) {
          if constexpr (CLUSTER) put_pair(&o.part[was & 1][rank], 0, make_float2(v, 0.f));
          else a.row_loss[(int64_t)mine + was * clusters] = v;
        }
      }
      __syncwarp();
      if constexpr (CLUSTER) cluster_arrive();
      const float next = weight_of(it + NS);
      if (it < rows) {
        if (it >= 1) {
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
        }
        fetch(it - 1 + NS, weight);
        teach(it + 1);
      }
      weight = next;
      if constexpr (CLUSTER) {
        cluster_wait();
        if (was >= 0 && a.row_loss && rank == 0 && lane == 0) {
          float v = 0.f;
          for (int c = 0; c < g.cluster; ++c) v += o.part[was & 1][c].x;
          a.row_loss[(int64_t)mine + was * clusters] = v;
        }
      }
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    return;
  }

  // ---- the warps that compute ----
  uint32_t phases = 0;                            // of the stages' barriers: a stage that was not loaded keeps its own
  const float dscale = (a.gradient && a.dloss ? *a.dloss : 1.f) * a.scale * a.T;
  for (int64_t it = 0; it <= rows; ++it) {
    __syncthreads();
    if (it == rows) {
      if constexpr (CLUSTER) { cluster_arrive(); cluster_wait(); }
      break;
    }
    const int s = (int)(it % NS), slot = (int)(it & 1) * K;
    const int64_t r = (int64_t)mine + it * clusters;
    const float weight = o.weight[s];
    const bool live = weight != 0.f && o.any[it & 1];
    T* const buf = (T*)stage(it);
    const Row w = row_at(it);
    const int n = w.p1 - w.p0;
    if (weight != 0.f) {
      if (!mbar_wait(&o.full[s], (phases >> s) & 1)) o.failed = 1;      // bounded; a load of mapped memory always lands
      phases ^= 1u << s;
    }
    float e[PIECES][VE], m = -INFINITY, sum = 0.f;
    if (live) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * NC;
        if (p < n) {
          unpack<VE>(load_raw<VE>(buf + p * VE, VE, true), e[i]);
        } else {
#pragma unroll
          for (int j = 0; j < VE; ++j) e[i][j] = -INFINITY;
        }
      }
      for (int j = tid; j < K; j += NC) {
        const int at = t_at[slot + j];
        t_z[j] = at >= 0 ? to_f<T>(buf[at]) : 0.f;
      }
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
          sum += e[i][j];
        }
      float top = m;
#pragma unroll
      for (int q = 16; q > 0; q /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, q));
      float v = m == -INFINITY ? sum : sum * exp_over(m, top, k);
#pragma unroll
      for (int q = 16; q > 0; q /= 2) v += __shfl_xor_sync(0xffffffffu, v, q);
      if (lane == 0) o.red[warp] = make_float2(top, v);
    }
    consumers_sync(NC);
    float M = -INFINITY, S = 0.f;
    if (live) {
      float2 v = lane < warps ? o.red[lane] : make_float2(-INFINITY, 0.f);
      M = v.x;
#pragma unroll
      for (int q = 16; q > 0; q /= 2) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, q));
      S = v.x == -INFINITY ? v.y : v.y * exp_over(v.x, M, k);
#pragma unroll
      for (int q = 16; q > 0; q /= 2) S += __shfl_xor_sync(0xffffffffu, S, q);
      if constexpr (CLUSTER)
        if (tid < g.cluster) put_pair(&o.all[it & 1][rank], (unsigned)tid, make_float2(M, S));
    }
    if constexpr (CLUSTER) {
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      if (live) {
        M = -INFINITY;
        S = 0.f;
        for (int c = 0; c < g.cluster; ++c) M = fmaxf(M, o.all[it & 1][c].x);
        for (int c = 0; c < g.cluster; ++c) {
          const float2 v = o.all[it & 1][c];
          S += v.x == -INFINITY ? v.y : v.y * exp_over(v.x, M, k);
        }
      }
    }
    const float rS = 1.f / S, coef = dscale * weight;
    if (a.gradient) {
      const float by = live ? (m == -INFINITY ? 0.f : coef * exp_over(m, M, k) * rS) : 0.f;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * NC;
        if (p < n) {
          float f[VE];
#pragma unroll
          for (int j = 0; j < VE; ++j) f[j] = live ? e[i][j] * by : 0.f;
          store_n<VE>(buf + p * VE, f, VE, true);
        }
      }
      consumers_sync(NC);
    }
    float loss = 0.f;
    if (live) {
      const float logS = logf(S);
      for (int j = tid; j < K; j += NC) {
        const int at = t_at[slot + j];
        if (at < 0) continue;
        const float q = t_q[slot + j], z = t_z[j], all = t_sum[slot + j];
        if (q != 0.f) loss += q * (t_log[slot + j] - (z - M) * rT + logS);
        if (a.gradient && all >= 0.f) buf[at] = from_f<T>(coef * (exp_over(z, M, k) * rS - all));
      }
      loss *= weight * a.T * a.T;
      if (a.row_stats && tid == 0 && rank == 0) {
        a.row_stats[2 * r] = M;
        a.row_stats[2 * r + 1] = S;
      }
    } else if (a.row_stats && tid == 0 && rank == 0) {
      a.row_stats[2 * r] = 0.f;
      a.row_stats[2 * r + 1] = 1.f;
    }
#pragma unroll
    for (int q = 16; q > 0; q /= 2) loss += __shfl_xor_sync(0xffffffffu, loss, q);
    if (lane == 0) o.loss[it & 1][warp] = loss;
    if (a.gradient) fence_proxy_async_shared();
  }
}

size_t small_bytes(int share, int VE, int entries) {
  return sizeof(Small) + (size_t)((share * VE + 31) / 32) * 4 + (size_t)entries * 4 * 9;
}

template <class T>
cudaError_t launch(const RingArgs& g, int grid, size_t smem, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)g.consumers + 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)g.cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = g.cluster > 1 ? 1 : 0;
  void (*const kernel)(const RingArgs) = g.cluster > 1 ? distill_rows<T, true> : distill_rows<T, false>;
  // per call: function attributes belong to the current device
  cudaError_t st = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (st != cudaSuccess) return st;
  st = cudaLaunchKernelEx(&cfg, kernel, g);
  if (st == cudaSuccess) (void)counted(s);
  return st;
}

}  // namespace

bool distill_ring(const DistillArgs& a, bool half, cudaStream_t s, cudaError_t& st) {
  const int VE = half ? 8 : 4;
  if (a.stats_in || (a.gradient && !a.same_phase)) return false;
  const int64_t pieces = ((int64_t)VE - 1 + a.vocabulary + VE - 1) / VE;
  if (pieces < 2048 / VE) return false;           // a warp or two a row: the kernel that holds a row in registers only
  for (int cluster = 1; cluster <= 8; cluster *= 2) {
    const int64_t share = (pieces + cluster - 1) / cluster;
    if (share > MAX_CONSUMERS * PIECES) continue;
    RingArgs g = {};
    g.a = a;
    g.cluster = cluster;
    g.share = (int)share;
    g.consumers = (int)((share + PIECES - 1) / PIECES + 31) / 32 * 32;
    const int per_sm = cluster > 1 ? 1 : g.consumers <= 96 ? 4 : g.consumers <= 224 ? 2 : 1;
    const size_t small = small_bytes(g.share, VE, a.entries), stage = (size_t)share * 16, room = SMEM / per_sm - 1024 * (per_sm > 1);
    if (small + 2 * stage > room) continue;
    const int64_t stages = (int64_t)((room - small) / stage);
    g.stages = stages > MAX_STAGES ? MAX_STAGES : (int)stages;
    const int sms = sm_count();
    int64_t clusters = (int64_t)sms * per_sm / cluster;
    if (clusters > a.rows) clusters = a.rows;
    const size_t smem = small + (size_t)g.stages * stage;
    st = half ? launch<bf16>(g, (int)(clusters * cluster), smem, s) : launch<float>(g, (int)(clusters * cluster), smem, s);
    return true;
  }
  return false;
}

}  // namespace seq
}  // namespace mebptt
