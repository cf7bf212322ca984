// Distillation loss: what its kernels share.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace mebptt {
namespace seq {

struct DistillArgs {
  const void* logits; const int32_t* indices; const float* values; const float* weights;
  const float* dloss; float* row_loss; float* row_stats; const float* stats_in;
  void* dlogits;
  int64_t rows, row, drow;              // rows, and elements between them
  int vocabulary, entries;
  float T, scale;
  int gradient;                         // dlogits is wanted
  int same_phase;                       // logits and dlogits begin at the same place within 16 bytes, in every row
};

// Rows through a ring in shared memory; false: none of its shapes fits.  `st` is what the launch returned.
bool distill_ring(const DistillArgs& a, bool half, cudaStream_t s, cudaError_t& st);

}  // namespace seq
}  // namespace mebptt
