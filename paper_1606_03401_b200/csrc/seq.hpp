// Host side of the operators over sequences: what their entry points check and derive alike.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "mebptt.h"

namespace mebptt {
namespace seq {

inline bool valid_dtype(int dtype) { return dtype == MEBPTT_FP32 || dtype == MEBPTT_TF32 || dtype == MEBPTT_BF16; }
inline size_t elem_size(int dtype) { return dtype == MEBPTT_BF16 ? 2 : 4; }

// Places of an array [t][B][width]: the element of step k, row b, column i is k * step + b * row + i.
struct Places {
  int64_t step, row;
};

// Strides as a descriptor has them -> places; false where two elements would share one, or an offset leaves 63 bits.
inline bool places(int64_t step, int64_t row, int64_t t, int64_t batch, int64_t width, Places& p) {
  if (step == 0 && row == 0) { step = batch * width; row = width; }
  if (step < 0 || row < 0 || step > ((int64_t)1 << 40) || row > ((int64_t)1 << 40)) return false;
  if (t > 1 && step < width) return false;
  if (batch > 1 && row < width) return false;
  if (t > 1 && batch > 1) {
    // one of the two walks over the other's whole extent
    const bool rows_inside = (row <= (INT64_MAX - width) / batch) && step >= (batch - 1) * row + width;
    const bool steps_inside = (step <= (INT64_MAX - width) / t) && row >= (t - 1) * step + width;
    if (!rows_inside && !steps_inside) return false;
  }
  const double reach = (double)(t - 1) * (double)step + (double)(batch - 1) * (double)row + (double)width;
  if (reach > 1e15) return false;
  p.step = step; p.row = row;
  return true;
}

// Whether groups of `n` elements from column 0 on can be loaded and stored as one: in `bytes` of an address and both strides.
inline bool aligned(const void* base, const Places& p, int64_t n, size_t esz) {
  const uint64_t unit = (uint64_t)n * esz < 16 ? (uint64_t)n * esz : 16;
  return !((reinterpret_cast<uintptr_t>(base) | (uint64_t)p.step * esz | (uint64_t)p.row * esz) & (unit - 1));
}
// Whether the type's elements lie on their own size.
inline bool natural(const void* p, size_t esz) { return !(reinterpret_cast<uintptr_t>(p) & (esz - 1)); }

inline int sm_count() {
  int dev = 0, sms = 148;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms;
}

}  // namespace seq
}  // namespace mebptt
