// Selective state space scan: what the forward and the backward kernels share.
#pragma once

#include <cstddef>
#include <cstdint>

#include "mebptt.h"
#include "seq.hpp"

namespace mebptt {
namespace seq {

constexpr int TILE = 32;        // the widest spacing of kept states

struct ScanArgs {
  const void* u; const void* delta; const void* z; const void* B; const void* C; const void* dy;
  const float* A; const float* skip; const float* bias;
  const float* s_in; const float* ds_out; const int32_t* lengths;
  void* y; float* s_out; float* kept;
  void* du; void* ddelta; void* dz; float* ds_in;
  // workspace: states (adjoints) at the ends of segments, [segments + 1][batch][D][8 lanes], and the sums of dt within them;
  // backward: sums over a block's channels [blocks][t][batch][groups][2][8 lanes], and over the steps of a segment
  float* ends; float* dts;
  float* part_bc; float* part_a; float* part_d; float* part_b;
  Places pu, pd, pz, pb, pc, py;
  int batch, channels, states, groups, gchannels;    // gchannels: channels of a group
  int t, spacing, softplus;
  int segment, segments;                             // steps of one; how many
  int blocks;                                        // of channels, in a group
  int vec_d, vec_s;                                  // whole groups of 8 channels, of 4 states, load as one
};

// Lanes that share a channel, eight states each.
inline int scan_lanes(int states) { return states <= 8 ? 1 : states <= 16 ? 2 : states <= 32 ? 4 : 8; }

}  // namespace seq
}  // namespace mebptt
