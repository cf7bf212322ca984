// Launchers of the scan's kernels.
#pragma once

#include <cuda_runtime.h>

#include "scan.hpp"

namespace mebptt {
namespace seq {

int scan_fwd_channels(int lanes);       // channels of a block
int scan_bwd_channels(int lanes);
int scan_fwd_blocks(int lanes, bool half);      // blocks that an SM keeps at once
int scan_bwd_blocks(int lanes, bool half, int spacing);
// Outputs and, with more than one segment, what they begin with.  False (here and below): a kernel's shared memory was refused.
bool scan_forward(const ScanArgs& a, bool half, cudaStream_t s);
// The adjoint that each segment hands to the one before it, for a gradient of zeros behind it (-> ends[segment + 1], dts).
bool scan_adjoints(const ScanArgs& a, bool half, cudaStream_t s);
// Gradients: the walk backwards and the sums over blocks, rows and segments.
bool scan_backward(const ScanArgs& a, bool half, float* dA, void* dB, void* dC, float* dskip, float* dbias, cudaStream_t s);

}  // namespace seq
}  // namespace mebptt
