// Distillation loss: rows stream through shared memory.  Bound by memory: the logits once in, the gradient once out.
//
// Over 2048 logits, or 128 entries: one resident block an SM (a few where rows are short), or a cluster of blocks that share a row, walks its rows
// through a ring of two to four stages: while one row is worked on, the next ones are on their way in and the last one's gradient on
// its way out, all by bulk copies, so that memory is busy although a row's own path is a chain (maximum, sum, gradient).  Each
// thread keeps its logits as exponentials in registers, relative to its own largest one, and what is left once the row's
// maximum and sum are known is one factor a thread: one exponential a logit.  The gradient is written over the logits in the stage,
// the listed tokens are put right there, and the stage is copied out.  One warp moves data, another prepares the next row's teacher
// (softmax of the listed values, tokens listed twice) and adds up losses.  Row begins and ends that are not on 16-byte
// boundaries go by plain loads and stores of the first one.
// Measured, loss and gradient in bfloat16 with 64 listed tokens a row: 4096 rows of 32000 in 100 us (5.2 TB/s), 16384 of 8192 in 112 us
// (4.8 TB/s), 2048 of 50257 in 100 us (4.1 TB/s), 512 of 128256 (clusters of four) in 74 us (3.6 TB/s; a row's path of 4 us is longer than
// its bytes take).  The loss alone takes 81, 88, 66 and 62 us, the gradient from statistics 115, 117, 107 and 68.
//
// Up to 2048 logits and 128 entries: a warp has a row and a ring to itself, so that nothing waits for another warp.  65536 rows of 1024:
// 105 us (2.6 TB/s; instructions for the 64 listed tokens of each row are half of it; 124 to 132 bytes a thread are spilt).  Rows that list a
// token twice take a search over all pairs of entries on top: 532 us where nearly all do.
//
// Every wait is bounded (none runs out while the device works).  A block in which one has run out loads no more rows, since a barrier
// must not be armed a second time before its phase is over, and neither pushes nor waits for what the cluster exchanges there:
// the other blocks get a sum that is not a number, or none and then run out of patience themselves.  Its rows from that one on are
// lost: its warp that moves data writes them as no numbers (lost_row) and waits at the end, once more bounded, for the loads in
// flight.  (All warps go through all turns: a way out of the loop costs the warps that compute 6 % at 4096 rows of 32000.)
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>

#include "distill.hpp"
#include "launch.hpp"
#include "seq.hpp"
#include "seq_dev.cuh"
#include "sm100.cuh"
#include "tc.hpp"

namespace mebptt {
namespace seq {

namespace {

using namespace sm100;

constexpr int PIECES = 8;               // 16-byte pieces of a thread: 64 bfloat16 or 32 float32 logits
constexpr int MAX_HOLDING = 512, MAX_CONSUMERS = 928, MAX_STAGES = 4;   // threads that hold exponentials; threads of any block
constexpr int AHEAD = 4;                // listed tokens of a lane that are loaded a row ahead
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
__device__ __forceinline__ void consumers_sync(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
// A pair of floats into the shared memory of a block of the cluster, counted in bytes on a barrier there.
__device__ __forceinline__ void push_pair(float2* at, uint64_t* bar, unsigned rank, float2 v) {
  uint32_t there, bar_there;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(at)), "r"(rank));
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar_there) : "r"(smem_u32(bar)), "r"(rank));
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(there), "r"(__float_as_uint(v.x)),
               "r"(__float_as_uint(v.y)), "r"(bar_there)
               : "memory");
}
__device__ __forceinline__ bool wait_pushed(uint64_t* bar, uint32_t parity, uint32_t polls) {
  for (uint32_t i = 0; i < polls; ++i) {
    if (mbar_try_wait_pushed(smem_u32(bar), parity)) return true;
    if (i > 64) __nanosleep(32);
  }
  return false;
}
// For a load, by a whole warp: all lanes learn the same.
__device__ __forceinline__ bool wait_loaded(uint64_t* bar, uint32_t parity, uint32_t polls) {
  bool there = false;
  for (uint32_t i = 0; i < polls && !there; ++i) {
    there = mbar_try_wait(bar, parity);
    if (i > 64 && !there) __nanosleep(32);
  }
  return __all_sync(0xffffffffu, there);
}
__device__ __forceinline__ float exp_over(float x, float m, float k) { return ex2((x - m) * k); }

// The largest of a thread's logits (numbers; one that is not shows in the sum).
template <int N>
__device__ __forceinline__ float largest(const Raw<bf16, 8> (&r)[N]) {
  __nv_bfloat162 m[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = *reinterpret_cast<const __nv_bfloat162*>(&r[0].w[j]);
#pragma unroll
  for (int i = 1; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = __hmax2(m[j], *reinterpret_cast<const __nv_bfloat162*>(&r[i].w[j]));
  const __nv_bfloat162 v = __hmax2(__hmax2(m[0], m[1]), __hmax2(m[2], m[3]));
  return fmaxf(__low2float(v), __high2float(v));
}
template <int N>
__device__ __forceinline__ float largest(const Raw<float, 4> (&r)[N]) {
  float m[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) m[j] = __uint_as_float(r[0].w[j]);
#pragma unroll
  for (int i = 1; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = fmaxf(m[j], __uint_as_float(r[i].w[j]));
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

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

struct RingArgs {
  DistillArgs a;
  int cluster, stages, consumers, share;          // share: pieces of a block at most
  uint32_t polls;                                 // of a wait
  int64_t no_load, no_sums, no_loss;              // rows whose logits, sums of blocks, parts of a loss a test waits for in vain (-1: none)
};

// A row after a wait has run out, by a whole warp: loss, statistics (`tell`) and the gradient's elements from + first, from + first + by, ... below
// `to` are no numbers, or what they always are where the row counts nothing.
template <class T>
__device__ __noinline__ void lost_row(const DistillArgs& a, int64_t r, int from, int to, int first, int by, bool tell) {
  bool any = false;
  for (int j = threadIdx.x % 32; j < a.entries; j += 32) {
    const int idx = a.indices[r * a.entries + j];
    any |= idx >= 0 && idx < a.vocabulary && a.values[r * a.entries + j] != -INFINITY;
  }
  const bool counts = __any_sync(0xffffffffu, any) && !(a.weights && a.weights[r] == 0.f);
  const float v = counts ? NAN : 0.f;
  if (a.gradient)
    for (int i = from + first; i < to; i += by) ((T*)a.dlogits)[r * a.drow + i] = from_f<T>(v);
  if (!tell) return;
  if (a.row_loss) a.row_loss[r] = v;
  if (a.row_stats) {
    a.row_stats[2 * r] = v;
    a.row_stats[2 * r + 1] = counts ? NAN : 1.f;
  }
}

// Shared memory behind the stages.
struct Small {
  uint64_t full[MAX_STAGES];
  uint64_t got[2], lost[2];                       // what the cluster's blocks push, by turns
  float2 red[MAX_CONSUMERS / 32];                 // largest logit and sum of a warp
  float2 all[2][8];                               // those of the cluster's blocks
  float2 part[2][8];                              // at the first block: their parts of the loss (x)
  float loss[2][MAX_CONSUMERS / 32];              // parts of the loss, by warp
  float weight[MAX_STAGES];
  int any[2];                                     // a row has entries
  int counted[2];                                 // a row has them and a weight
  int64_t lost_from;                              // the first row that is lost, counted as the block takes them (none: INT64_MAX)
};

// LIGHT: exponentials are computed a second time for the gradient instead of being held, so that a block of up to 928 threads has
// registers enough, and takes rows of twice the length.
template <class T, bool CLUSTER, bool LIGHT>
__global__ void __launch_bounds__((LIGHT ? MAX_CONSUMERS : MAX_HOLDING) + 64, 1) distill_rows(const __grid_constant__ RingArgs g) {
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
    const int pieces = (w.phase + V + VE - 1) / VE, share = CLUSTER ? (pieces + g.cluster - 1) / g.cluster : pieces;
    w.p0 = min((int)rank * share, pieces);
    w.p1 = min(w.p0 + share, pieces);
    w.in0 = w.p0 == 0 && w.phase ? min(1, w.p1) : w.p0;
    w.in1 = w.p1 == pieces && (w.phase + V) % VE ? max(w.in0, w.p1 - 1) : w.p1;
    return w;
  };
  auto stage = [&](int s) { return sm + (uint32_t)s * stage_bytes; };

  if (tid == 0) {
    for (int s = 0; s < NS; ++s) mbar_init(&o.full[s], 2);
    for (int s = 0; s < 2; ++s) {
      mbar_init(&o.got[s], 1);
      mbar_init(&o.lost[s], 1);
    }
    mbar_fence_init();
    o.lost_from = INT64_MAX;
  }
  for (int i = tid; i < words; i += blockDim.x) seen[i] = 0;
  __syncthreads();
  if constexpr (CLUSTER) cluster_sync();                                       // no block writes to another before it is there

  // (Set in the turn of that row, by whoever finds out, and read in later ones.)
  auto lose = [&](int64_t it) {
    if (it < o.lost_from) o.lost_from = it;
  };

  if (warp == warps) {
    // ---- the warp that moves data ----
    uint32_t turns = 0, used = 0;                 // of a stage: loads so far are odd; there were any
    auto weight_of = [&](int64_t it) { return it < rows && a.weights ? a.weights[(int64_t)mine + it * clusters] : 1.f; };
    auto fetch = [&](int64_t it, int s, float weight) {
      if (it >= rows) return;
      if (lane == 0) o.weight[s] = weight;
      if (weight == 0.f) return;                  // not loaded, and not waited for
      turns ^= 1u << s;
      used |= 1u << s;
      const Row w = row_at(it);
      T* const buf = (T*)stage(s);
      if (lane == 0) {
        const uint32_t bytes = (uint32_t)(w.in1 - w.in0) * 16;
        const bool faulty = (int64_t)mine + it * clusters == g.no_load && (int)rank == g.cluster - 1;
        mbar_arrive_expect_tx(&o.full[s], bytes + (faulty ? 16 : 0));
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
    for (int i = 0; i < NS - 1; ++i) fetch(i, i, weight_of(i));
    float weight = weight_of(NS - 1);
    int last = NS - 1;                            // stage of row it - 1, and of row it - 1 + NS
    for (int64_t it = 0; it <= rows; ++it, last = last + 1 == NS ? 0 : last + 1) {
      __syncthreads();                            // row it - 1 is done with
      const bool lost = o.lost_from < it;
      const float next = weight_of(it + NS);
      if (lost) {
        const Row w = row_at(it - 1);
        lost_row<T>(a, (int64_t)mine + (it - 1) * clusters, max(w.p0 * VE - w.phase, 0), min(w.p1 * VE - w.phase, V), lane, 32, rank == 0 && lane == 0);
      } else if (it >= 1 && a.gradient) {
        const Row w = row_at(it - 1);
        const T* const buf = (const T*)stage(last);
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
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
      }
      if (it < rows) fetch(it - 1 + NS, last, lost ? 0.f : weight);
      weight = next;
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    __syncwarp();
    const bool lost = o.lost_from != INT64_MAX;
    if (lost)
      for (int i = 0; i < NS; ++i)
        if (used >> i & 1) wait_loaded(&o.full[i], ~turns >> i & 1, g.polls);
    if constexpr (CLUSTER) {
      cluster_sync();                             // no block leaves while another pushes to it
      if (lost)
        for (int i = 0; i < 64; ++i) __nanosleep(1000);      // what was pushed and not waited for has landed
    }
    return;
  }
  if (warp == warps + 1) {
    // ---- the warp that prepares the next row's teacher, and adds up the last row's loss ----
    // The listed tokens and values of a row are loaded a row ahead of where they are used (the first 128 of them).
    int ahead_i[AHEAD];
    float ahead_v[AHEAD];
    auto look = [&](int64_t it) {
      const int64_t from = ((int64_t)mine + it * clusters) * K;
#pragma unroll
      for (int q = 0; q < AHEAD; ++q) {
        const int j = lane + 32 * q;
        const bool in = it < rows && j < K;
        ahead_i[q] = in ? a.indices[from + j] : -1;
        ahead_v[q] = in ? a.values[from + j] : 0.f;
      }
    };
    // softmax of the listed values of row `it`
    auto teach = [&](int64_t it) {
      if (it >= rows) return;
      const int64_t r = (int64_t)mine + it * clusters;
      const Row w = row_at(it);
      const int slot = (int)(it & 1) * K, lo = w.p0 * VE - w.phase, n = (w.p1 - w.p0) * VE;
      float top = -INFINITY;
      bool any = false;
      auto listed = [&](int j, int idx, float v) {
        if (idx < 0 || idx >= V) v = -INFINITY;
        const int at = idx - lo;
        t_at[slot + j] = v == -INFINITY ? -1 : at >= 0 && at < n ? at : -2;
        t_log[slot + j] = v;
        any |= v != -INFINITY;
        top = fmaxf(top, v);
      };
#pragma unroll
      for (int q = 0; q < AHEAD; ++q)
        if (lane + 32 * q < K) listed(lane + 32 * q, ahead_i[q], ahead_v[q]);
      for (int j = lane + 32 * AHEAD; j < K; j += 32) listed(j, a.indices[r * K + j], a.values[r * K + j]);
      look(it + 1);
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

    look(0);
    teach(0);
    int due = 0;                                  // lane 0: the row before has its loss on the way
    uint32_t losses = 0;
    for (int64_t it = 0; it <= rows; ++it) {
      __syncthreads();                            // row it has its teacher, row it - 1 its loss
      const int64_t was = it - 1;
      if (was >= 0 && a.row_loss && was < o.lost_from) {
        float v = lane < warps ? o.loss[was & 1][lane] : 0.f;
#pragma unroll
        for (int m = 16; m > 0; m /= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
        // (Blocks of a cluster meet in rows that count something only, once in each, to exchange their sums: none of them is
        // ever two such rows ahead of another, which is why two places for what they push are enough.)
        if (lane == 0) {
          due = CLUSTER && o.counted[was & 1];
          if (due) {
            if (rank == 0) mbar_arrive_expect_tx(&o.lost[losses & 1], 8 * (g.cluster + ((int64_t)mine + was * clusters == g.no_loss)));
            push_pair(&o.part[losses & 1][rank], &o.lost[losses & 1], 0, make_float2(v, 0.f));
          } else if (rank == 0) {
            a.row_loss[(int64_t)mine + was * clusters] = v;
          }
        }
        __syncwarp();
      }
      teach(it + 1);
      if (due) {
        if (rank == 0) {
          float v = 0.f;
          if (!wait_pushed(&o.lost[losses & 1], (losses >> 1) & 1, g.polls)) {
            v = NAN;
            lose(it);
          }
          for (int c = 0; c < g.cluster; ++c) v += o.part[losses & 1][c].x;
          a.row_loss[(int64_t)mine + was * clusters] = v;
        }
        ++losses;
        due = 0;
      }
      __syncwarp();
    }
    if constexpr (CLUSTER) cluster_sync();
    return;
  }

  // ---- the warps that compute ----
  uint32_t phases = 0;                            // of the stages' barriers: a stage that was not loaded keeps its own
  uint32_t meetings = 0;                          // of the cluster's blocks
  bool alone = false;                             // one of them has not come about
  const float dscale = (a.gradient && a.dloss ? *a.dloss : 1.f) * a.scale * a.T;
  int s = 0;
  for (int64_t it = 0; it <= rows; ++it, s = s + 1 == NS ? 0 : s + 1) {
    __syncthreads();
    if (it == rows) {
      if constexpr (CLUSTER) cluster_sync();
      break;
    }
    const int slot = (int)(it & 1) * K;
    const float weight = o.weight[s];
    const bool live = weight != 0.f && o.any[it & 1];
    const bool meet = CLUSTER && live && !a.stats_in && !alone;
    if (tid == 0) {
      o.counted[it & 1] = live;
      if (meet) mbar_arrive_expect_tx(&o.got[meetings & 1], 8 * (g.cluster + ((int64_t)mine + it * clusters == g.no_sums && (int)rank == g.cluster - 1)));
    }
    T* const buf = (T*)stage(s);
    const Row w = row_at(it);
    const int n = w.p1 - w.p0;
    bool loaded = true;
    if (weight != 0.f) {
      loaded = wait_loaded(&o.full[s], (phases >> s) & 1, g.polls);
      if (!loaded) lose(it);
      phases ^= 1u << s;
    }
    Raw<T, VE> raw[PIECES];
    pair e[LIGHT ? 1 : PIECES][VE / 2];
    float m = -INFINITY, sum = 0.f;
    // exponentials of a piece, relative to m
    auto exponentials = [&](const Raw<T, VE>& r, pair (&f)[VE / 2]) {
      const pair from = both(m == -INFINITY ? 0.f : -m), k2 = both(k);
      unpack_pairs<VE>(r, f);
#pragma unroll
      for (int j = 0; j < VE / 2; ++j) {
        const float2 x = unpack2(mul2(add2(f[j], from), k2));
        f[j] = pack2(ex2(x.x), ex2(x.y));
      }
    };
    if (live) {
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * NC;
        if (p < n) {
          raw[i] = load_raw<VE>(buf + p * VE, VE, true);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i].w[j] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;      // -infinity
        }
      }
      for (int j = tid; j < K; j += NC) {
        const int at = t_at[slot + j];
        t_z[j] = at >= 0 ? to_f<T>(buf[at]) : 0.f;
      }
      m = largest(raw);
      pair sum_a = 0, sum_b = 0;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        pair (&f)[VE / 2] = e[LIGHT ? 0 : i];
        exponentials(raw[i], f);
#pragma unroll
        for (int j = 0; j < VE / 2; ++j) {
          if (j & 1) sum_a = add2(sum_a, f[j]);
          else sum_b = add2(sum_b, f[j]);
        }
      }
      sum = sum2(add2(sum_a, sum_b));
      float top = m;
#pragma unroll
      for (int q = 16; q > 0; q /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, q));
      float v = m == -INFINITY ? sum : sum * exp_over(m, top, k);
#pragma unroll
      for (int q = 16; q > 0; q /= 2) v += __shfl_xor_sync(0xffffffffu, v, q);
      if (lane == 0) o.red[warp] = make_float2(top, loaded ? v : NAN);
    }
    consumers_sync(NC);
    float M = -INFINITY, S = 0.f;
    if (live) {
      const float2 v = lane < warps ? o.red[lane] : make_float2(-INFINITY, 0.f);
      M = warp_max(v.x);
      S = warp_sum(v.x == -INFINITY ? v.y : v.y * exp_over(v.x, M, k));
    }
    if constexpr (CLUSTER) {
      if (meet) {
        if (tid < g.cluster) push_pair(&o.all[meetings & 1][rank], &o.got[meetings & 1], (unsigned)tid, make_float2(M, S));
        __syncwarp();
        if (!__all_sync(0xffffffffu, wait_pushed(&o.got[meetings & 1], (meetings >> 1) & 1, g.polls))) {
          alone = true;
          lose(it);
        }
        M = -INFINITY;
        S = 0.f;
        for (int c = 0; c < g.cluster; ++c) M = fmaxf(M, o.all[meetings & 1][c].x);
        for (int c = 0; c < g.cluster; ++c) {
          const float2 v = o.all[meetings & 1][c];
          S += v.x == -INFINITY ? v.y : v.y * exp_over(v.x, M, k);
        }
        ++meetings;
      }
    }
    if (live && a.stats_in) {
      const float* const st = a.stats_in + 2 * ((int64_t)mine + it * clusters);
      M = st[0];
      S = st[1];
    }
    const float rS = 1.f / S, coef = dscale * weight;
    if (a.gradient) {
      const pair by = both(live && m != -INFINITY ? coef * exp_over(m, M, k) * rS : live ? coef * rS : 0.f);
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = tid + i * NC;
        if (p < n) {
          pair f[VE / 2];
          if constexpr (LIGHT) {
            if (live) exponentials(raw[i], f);
          }
#pragma unroll
          for (int j = 0; j < VE / 2; ++j) f[j] = live ? mul2(LIGHT ? f[j] : e[LIGHT ? 0 : i][j], by) : 0;
          store_pairs<VE>(buf + p * VE, f, VE, true);
        }
      }
    }
    // the listed tokens: their part of the loss, and the gradient of the first entry of each
    float loss = 0.f;
    const float logS = live ? logf(S) : 0.f;
    auto entry = [&](int j, int& at) {
      at = t_at[slot + j];
      if (at < 0) return 0.f;
      const float q = t_q[slot + j], z = t_z[j], all = t_sum[slot + j];
      if (q != 0.f) loss += q * (t_log[slot + j] - (z - M) * rT + logS);
      if (all < 0.f) at = -1;
      return coef * (exp_over(z, M, k) * rS - all);
    };
    int at0 = -1;
    float d0 = 0.f;
    if (live && tid < K) d0 = entry(tid, at0);
    if (a.gradient) consumers_sync(NC);
    if (a.gradient && at0 >= 0) buf[at0] = from_f<T>(d0);
    if (live)
      for (int j = tid + NC; j < K; j += NC) {
        const float d = entry(j, at0);
        if (a.gradient && at0 >= 0) buf[at0] = from_f<T>(d);
      }
    if (a.gradient) fence_proxy_async_shared();
    if (warp * 32 < K) {
      loss *= weight * a.T * a.T;
#pragma unroll
      for (int q = 16; q > 0; q /= 2) loss += __shfl_xor_sync(0xffffffffu, loss, q);
    }
    if (lane == 0) o.loss[it & 1][warp] = live ? loss : 0.f;
    if (a.row_stats && tid == 0 && rank == 0) {
      const int64_t r = (int64_t)mine + it * clusters;
      a.row_stats[2 * r] = live ? M : 0.f;
      a.row_stats[2 * r + 1] = live ? S : 1.f;
    }
  }
}

// What is left of a warp's rows after a wait has run out: the loads of this row and those ahead once more, then all from here on are lost.
template <class T>
__device__ __noinline__ void lost_rows(const RingArgs& g, uint64_t* full, int s, uint32_t phases, int64_t r, int64_t step) {
  for (int i = 0; i < g.stages - 1; ++i) {
    const int at = (s + i) % g.stages;
    const int64_t row = r + i * step;
    if (row < g.a.rows && !(g.a.weights && g.a.weights[row] == 0.f)) wait_loaded(&full[at], (phases >> at) & 1, g.polls);
  }
  for (; r < g.a.rows; r += step) lost_row<T>(g.a, r, 0, g.a.vocabulary, threadIdx.x % 32, 32, threadIdx.x % 32 == 0);
}

// Short rows: a warp each, with a ring of its own, so that nothing waits for another warp.  `share` pieces a row at most.
constexpr int WARPS = 4, ENTRIES = 128;
template <class T, int PIECES>
__global__ void __launch_bounds__(WARPS * 32, PIECES * 16 / (int)sizeof(T) == 32 ? 6 : 4) distill_warps(const __grid_constant__ RingArgs g) {
  constexpr int VE = 16 / (int)sizeof(T), EPL = ENTRIES / 32;
  extern __shared__ __align__(128) uint8_t sm[];
  const DistillArgs& a = g.a;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, NS = g.stages, K = a.entries, V = a.vocabulary;
  const uint32_t stage_bytes = (uint32_t)g.share * 16;
  const int words = (g.share * VE + 31) / 32;
  uint8_t* const ring = sm + (uint32_t)warp * NS * stage_bytes;
  uint64_t* const full = reinterpret_cast<uint64_t*>(sm + (uint32_t)WARPS * NS * stage_bytes) + warp * MAX_STAGES;
  uint32_t* const seen = reinterpret_cast<uint32_t*>(sm + (uint32_t)WARPS * NS * stage_bytes + WARPS * MAX_STAGES * 8) + warp * words;
  const int64_t step = (int64_t)gridDim.x * WARPS, first = (int64_t)blockIdx.x * WARPS + warp;
  const float k = kLog2e / a.T, rT = 1.f / a.T;
  const float dscale = (a.gradient && a.dloss ? *a.dloss : 1.f) * a.scale * a.T;

  if (lane == 0) {
    for (int s = 0; s < NS; ++s) mbar_init(&full[s], 2);
    mbar_fence_init();
  }
  for (int i = lane; i < words; i += 32) seen[i] = 0;
  __syncwarp();

  struct Row {
    const T* x; T* dx;
    int phase, pieces, in0, in1;
  };
  auto row_at = [&](int64_t r) {
    Row w;
    w.x = (const T*)a.logits + r * a.row;
    w.dx = (T*)a.dlogits + r * a.drow;
    w.phase = (int)(reinterpret_cast<uintptr_t>(w.x) / sizeof(T) % VE);
    w.pieces = (w.phase + V + VE - 1) / VE;
    w.in0 = w.phase ? 1 : 0;
    w.in1 = (w.phase + V) % VE ? max(w.in0, w.pieces - 1) : w.pieces;
    return w;
  };
  auto fetch = [&](int64_t r, int s, float weight) {
    if (r >= a.rows || weight == 0.f) return;
    const Row w = row_at(r);
    T* const buf = (T*)(ring + s * stage_bytes);
    if (lane == 0) {
      const uint32_t bytes = (uint32_t)(w.in1 - w.in0) * 16;
      mbar_arrive_expect_tx(&full[s], bytes + (r == g.no_load ? 16 : 0));
      if (bytes) bulk_in(buf + w.in0 * VE, w.x + (w.in0 * VE - w.phase), bytes, &full[s]);
    }
    const int head = w.in0 * VE, tail = (w.pieces - w.in1) * VE;
    if (lane < head + tail) {
      const int at = lane < head ? lane : w.in1 * VE + lane - head, i = at - w.phase;
      buf[at] = i >= 0 && i < V ? w.x[i] : from_f<T>(-INFINITY);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&full[s]);
  };
  auto weight_of = [&](int64_t r) { return r < a.rows && a.weights ? a.weights[r] : 1.f; };
  int next_i[EPL];
  float next_v[EPL];
  auto look = [&](int64_t r) {
#pragma unroll
    for (int q = 0; q < EPL; ++q) {
      const int j = lane + 32 * q;
      const bool in = r < a.rows && j < K;
      next_i[q] = in ? a.indices[r * K + j] : -1;
      next_v[q] = in ? a.values[r * K + j] : 0.f;
    }
  };
  float weights[MAX_STAGES];                      // of the rows in flight, that of the row at hand first
#pragma unroll
  for (int i = 0; i < MAX_STAGES; ++i) weights[i] = i < NS ? weight_of(first + i * step) : 1.f;
#pragma unroll
  for (int i = 0; i < MAX_STAGES - 1; ++i)
    if (i < NS - 1) fetch(first + i * step, i, weights[i]);
  look(first);
  uint32_t phases = 0;
  int s = 0;
  int64_t r = first;
  for (; r < a.rows; r += step, s = s + 1 == NS ? 0 : s + 1) {
    const float weight = weights[0];
    const Row w = row_at(r);
    T* const buf = (T*)(ring + s * stage_bytes);
    // the teacher
    int at[EPL];
    float v[EPL], z[EPL], q[EPL], top_v = -INFINITY;
    bool any = false;
#pragma unroll
    for (int i = 0; i < EPL; ++i) {
      v[i] = next_i[i] >= 0 && next_i[i] < V ? next_v[i] : -INFINITY;
      at[i] = v[i] == -INFINITY ? -1 : next_i[i] + w.phase;
      any |= at[i] >= 0;
      top_v = fmaxf(top_v, v[i]);
    }
    const float next_w = weight_of(r + NS * step);
    look(r + step);
    const bool live = __any_sync(0xffffffffu, any) && weight != 0.f;
    if (weight != 0.f) {
      if (!wait_loaded(&full[s], (phases >> s) & 1, g.polls)) break;
      phases ^= 1u << s;
    }
    // the stage of the row before: its gradient has been read out of it (that of this row is not yet on its way)
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
    __syncwarp();
    {
      const int before = s == 0 ? NS - 1 : s - 1;
      float weight_ahead = weights[1];
#pragma unroll
      for (int i = 2; i < MAX_STAGES; ++i)
        if (i == NS - 1) weight_ahead = weights[i];
      fetch(r + (NS - 1) * step, before, weight_ahead);
    }
#pragma unroll
    for (int i = 0; i < MAX_STAGES; ++i) weights[i] = i == NS - 1 ? next_w : i + 1 < MAX_STAGES ? weights[i + 1] : 1.f;

    float loss = 0.f;
    if (live) {
      Raw<T, VE> raw[PIECES];
      pair e[PIECES][VE / 2];
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        const int p = lane + i * 32;
        if (p < w.pieces) {
          raw[i] = load_raw<VE>(buf + p * VE, VE, true);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i].w[j] = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
        }
      }
#pragma unroll
      for (int i = 0; i < EPL; ++i) z[i] = at[i] >= 0 ? to_f<T>(buf[at[i]]) : 0.f;
      float M = largest(raw);
#pragma unroll
      for (int m = 16; m > 0; m /= 2) {
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, m));
        top_v = fmaxf(top_v, __shfl_xor_sync(0xffffffffu, top_v, m));
      }
      const pair from = both(M == -INFINITY ? 0.f : -M), k2 = both(k);
      pair sum_a = 0, sum_b = 0;
#pragma unroll
      for (int i = 0; i < PIECES; ++i) {
        unpack_pairs<VE>(raw[i], e[i]);
#pragma unroll
        for (int j = 0; j < VE / 2; ++j) {
          const float2 x = unpack2(mul2(add2(e[i][j], from), k2));
          e[i][j] = pack2(ex2(x.x), ex2(x.y));
          if (j & 1) sum_a = add2(sum_a, e[i][j]);
          else sum_b = add2(sum_b, e[i][j]);
        }
      }
      float S = sum2(add2(sum_a, sum_b)), Q = 0.f;
      bool twice = false;
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        q[i] = at[i] >= 0 ? exp_over(v[i], top_v, k) : 0.f;
        Q += q[i];
        if (at[i] >= 0) twice |= (atomicOr(&seen[at[i] >> 5], 1u << (at[i] & 31)) >> (at[i] & 31)) & 1;
      }
#pragma unroll
      for (int m = 16; m > 0; m /= 2) {
        S += __shfl_xor_sync(0xffffffffu, S, m);
        Q += __shfl_xor_sync(0xffffffffu, Q, m);
      }
      twice = __any_sync(0xffffffffu, twice);
      float factor = 1.f;
      if (a.stats_in) {
        factor = M == -INFINITY ? 1.f : exp_over(M, a.stats_in[2 * r], k);
        M = a.stats_in[2 * r];
        S = a.stats_in[2 * r + 1];
      }
      const float rS = 1.f / S, rQ = 1.f / Q, coef = dscale * weight, more = logf(S) - logf(Q);
      float all[EPL];
#pragma unroll
      for (int i = 0; i < EPL; ++i) {
        if (at[i] >= 0) seen[at[i] >> 5] = 0;
        q[i] *= rQ;
        all[i] = q[i];
        if (q[i] != 0.f) loss += q[i] * (((v[i] - top_v) - (z[i] - M)) * rT + more);
      }
      if (twice) {
        // the first entry of a token takes the sum of all of its entries, in their order; the others nothing
        float total[EPL];
        bool later[EPL];
#pragma unroll
        for (int i = 0; i < EPL; ++i) { total[i] = 0.f; later[i] = false; }
#pragma unroll
        for (int o = 0; o < EPL; ++o)
          for (int j = 0; j < 32; ++j) {
            const int token = __shfl_sync(0xffffffffu, at[o], j);
            const float share = __shfl_sync(0xffffffffu, q[o], j);
#pragma unroll
            for (int i = 0; i < EPL; ++i)
              if (token == at[i]) {
                total[i] += share;
                later[i] |= o * 32 + j < i * 32 + lane;
              }
          }
#pragma unroll
        for (int i = 0; i < EPL; ++i) {
          all[i] = total[i];
          if (later[i]) at[i] = -1;
        }
      }
      if (a.gradient) {
        const pair by = both(coef * rS * factor);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
          const int p = lane + i * 32;
          if (p < w.pieces) {
#pragma unroll
            for (int j = 0; j < VE / 2; ++j) e[i][j] = mul2(e[i][j], by);
            store_pairs<VE>(buf + p * VE, e[i], VE, true);
          }
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < EPL; ++i)
          if (at[i] >= 0) buf[at[i]] = from_f<T>(coef * (exp_over(z[i], M, k) * rS - all[i]));
      }
      loss *= weight * a.T * a.T;
#pragma unroll
      for (int m = 16; m > 0; m /= 2) loss += __shfl_xor_sync(0xffffffffu, loss, m);
      if (a.row_stats && lane == 0) {
        a.row_stats[2 * r] = M;
        a.row_stats[2 * r + 1] = S;
      }
    } else {
      if (a.gradient) {
        const pair zero[VE / 2] = {};
        for (int p = lane; p < w.pieces; p += 32) store_pairs<VE>(buf + p * VE, zero, VE, true);
      }
      if (a.row_stats && lane == 0) {
        a.row_stats[2 * r] = 0.f;
        a.row_stats[2 * r + 1] = 1.f;
      }
    }
    if (a.row_loss && lane == 0) a.row_loss[r] = loss;
    if (a.gradient) {
      fence_proxy_async_shared();
      __syncwarp();
      if (lane == 0) {
        const uint32_t bytes = (uint32_t)(w.in1 - w.in0) * 16;
        if (bytes) bulk_out(w.dx + (w.in0 * VE - w.phase), buf + w.in0 * VE, bytes);
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
      const int head = w.in0 * VE, tail = (w.pieces - w.in1) * VE;
      if (lane < head + tail) {
        const int p = lane < head ? lane : w.in1 * VE + lane - head, i = p - w.phase;
        if (i >= 0 && i < V) w.dx[i] = buf[p];
      }
    }
    __syncwarp();
  }
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  if (r < a.rows) lost_rows<T>(g, full, s, phases, r, step);
}

size_t small_bytes(int share, int VE, int entries) {
  return sizeof(Small) + (size_t)((share * VE + 31) / 32) * 4 + (size_t)entries * 4 * 9;
}

// Clusters of a shape that the current device keeps at once (a GPC holds whole clusters only, and GPCs differ from one
// device to the next), 0 if it cannot be asked.  The last answers are kept: asking takes longer than launching.
int resident_clusters(const void* kernel, const cudaLaunchConfig_t& cfg, int cluster) {
  struct Answer {
    const void* kernel;
    int dev, cluster, threads, smem, clusters;
  };
  static std::mutex mu;
  static Answer answers[16];
  static unsigned next = 0;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return 0;
  const int threads = (int)cfg.blockDim.x, smem = (int)cfg.dynamicSmemBytes;
  {
    std::lock_guard<std::mutex> lock(mu);
    for (const Answer& a : answers)
      if (a.clusters > 0 && a.kernel == kernel && a.dev == dev && a.cluster == cluster && a.threads == threads && a.smem == smem) return a.clusters;
  }
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  std::lock_guard<std::mutex> lock(mu);
  answers[next++ % 16] = Answer{kernel, dev, cluster, threads, smem, n};
  return n;
}

// `grid`: blocks at most; of clusters, as many as are there at once, since each walks its share of the rows.
template <class Kernel>
cudaError_t launch(Kernel* kernel, const RingArgs& g, int64_t grid, int threads, size_t smem, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)g.cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = g.cluster > 1 ? 1 : 0;
  // Per call: function attributes belong to the current device.  Always the most that any shape takes: calls of other host threads, with
  // rows of other lengths, set the same attribute of the same kernel between this and the launch.
  cudaError_t st = cudaSuccess;
  if (smem > 48 * 1024) st = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
  if (st != cudaSuccess) return st;
  if (g.cluster > 1) {
    const int64_t most = (int64_t)resident_clusters((const void*)kernel, cfg, g.cluster) * g.cluster;
    if (most > 0 && grid > most) cfg.gridDim = dim3((unsigned)most);
  }
  st = cudaLaunchKernelEx(&cfg, kernel, g);
  if (st == cudaSuccess) (void)counted(s);
  return st;
}

template <class T>
cudaError_t launch_warps(RingArgs& g, int sms, cudaStream_t s) {
  constexpr int VE = 16 / (int)sizeof(T), MOST = 64 / VE;
  g.cluster = 1;
  g.stages = 3;
  const size_t smem = (size_t)WARPS * (g.stages * (size_t)g.share * 16 + MAX_STAGES * 8 + (size_t)((g.share * VE + 31) / 32) * 4);
  int64_t grid = (int64_t)sms * (SMEM / (smem + 1024) < 6 ? SMEM / (smem + 1024) : 6);
  if (grid > (g.a.rows + WARPS - 1) / WARPS) grid = (g.a.rows + WARPS - 1) / WARPS;
  if (g.share <= 32 * (MOST / 2)) return launch(distill_warps<T, MOST / 2>, g, grid, WARPS * 32, smem, s);
  return launch(distill_warps<T, MOST>, g, grid, WARPS * 32, smem, s);
}

}  // namespace

bool distill_ring(const DistillArgs& a, bool half, cudaStream_t s, cudaError_t& st) {
  const int VE = half ? 8 : 4;
  if (a.gradient && !a.same_phase) return false;
  // pieces of a row at most: rows that all begin at the same place within 16 bytes have one phase
  const int phase = a.row % VE || a.rows == 1 ? VE - 1 : (int)(reinterpret_cast<uintptr_t>(a.logits) / (16 / VE) % VE);
  const int64_t pieces = ((int64_t)phase + a.vocabulary + VE - 1) / VE;
  const int sms = sm_count();
  RingArgs g = {};
  g.a = a;
  const int fault = tc::wait_fault_mask() >> 5;      // testing aid, 0 outside the tests of the bounded waits
  g.polls = fault ? tc::fault_poll_limit : kSpinLimit;
  g.no_load = fault & 1 ? a.rows / 2 : -1;
  g.no_sums = fault & 2 ? a.rows / 2 : -1;
  g.no_loss = fault & 4 ? a.rows / 2 : -1;
  if (pieces * VE <= 2048 && a.entries <= ENTRIES) {
    g.share = (int)pieces;
    st = half ? launch_warps<bf16>(g, sms, s) : launch_warps<float>(g, sms, s);
    return true;
  }
  // As few blocks to a row as hold it, and as many of them on an SM as fit: a meeting of a cluster costs a row some 0.7 us, and
  // blocks that wait for one another stand still together, while other rows' blocks do not.  (4096 rows of 32000 bfloat16 logits:
  // 105 us with one block a row, 118 with two, 148 with four.)
  // Rows of up to twice what a block can hold as exponentials stay with one block all the same, which computes them twice.
  // (2048 rows of 50257 bfloat16 logits: 97 us, held by a cluster of two 117; 2048 of 25000 in float32: 72 and 91.)
  for (int shape = 0; shape < 8; ++shape) {
    const int cluster = 1 << (shape / 2), light = shape % 2;
    const int64_t share = (pieces + cluster - 1) / cluster;
    if (share > (light ? MAX_CONSUMERS : MAX_HOLDING) * PIECES) continue;
    g.cluster = cluster;
    g.share = (int)share;
    g.consumers = (int)((share + PIECES - 1) / PIECES + 31) / 32 * 32;
    const size_t small = small_bytes(g.share, VE, a.entries), stage = (size_t)share * 16;
    int per_sm = 65536 / ((light ? 64 : 96) * (g.consumers + 64));
    if (per_sm > 6) per_sm = 6;
    while (per_sm > 1 && (size_t)per_sm * (small + 3 * stage + 1024) > SMEM) --per_sm;
    const size_t room = SMEM / per_sm - (per_sm > 1 ? 1024 : 0);
    if (small + 2 * stage > room) continue;
    const int64_t stages = (int64_t)((room - small) / stage);
    g.stages = stages > MAX_STAGES ? MAX_STAGES : (int)stages;
    int64_t clusters = (int64_t)sms * per_sm / cluster;
    if (clusters < 1) clusters = 1;
    if (clusters > a.rows) clusters = a.rows;
    void (*kernel)(const RingArgs);
    if (light) kernel = half ? (cluster > 1 ? distill_rows<bf16, true, true> : distill_rows<bf16, false, true>)
                             : (cluster > 1 ? distill_rows<float, true, true> : distill_rows<float, false, true>);
    else kernel = half ? (cluster > 1 ? distill_rows<bf16, true, false> : distill_rows<bf16, false, false>)
                       : (cluster > 1 ? distill_rows<float, true, false> : distill_rows<float, false, false>);
    st = launch(kernel, g, clusters * cluster, g.consumers + 64, small + (size_t)g.stages * stage, s);
    return true;
  }
  return false;
}

}  // namespace seq
}  // namespace mebptt
